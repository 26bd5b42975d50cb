"""Layer norm on the GPU against 64 bits (oracle/network_end.py), with bounds counted in roundings: u = 2^-24 for fp32
arithmetic, half a step of the type (bf16 2^-8, fp32 2^-24) for the one rounding on store.  A row's sums are chains of at most
72 elements a thread and 14 joins here, a column's of at most 64 rows a lane, 32 lanes and 64 ranges, so 192 u covers a sum and
the few operations behind it, relative to the sum of its terms' magnitudes."""
import numpy as np
import pytest
import torch

from oracle import network_end as ne

pytestmark = pytest.mark.gpu
U, CHAIN = 2.0 ** -24, 192


@pytest.fixture(scope="module")
def B():
    from paper_1606_04487_amd import binding
    assert torch.cuda.is_available()
    return binding


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def pitched(values, dtype, extra, pad=float("nan")):
    """values [rows][width] on the GPU as a slice of a matrix with `extra` more columns, filled with `pad`."""
    rows, width = values.shape
    full = torch.full((rows, width + extra), pad, dtype=dtype, device="cuda")
    full[:, :width] = torch.from_numpy(np.ascontiguousarray(values)).to(dtype)
    return full[:, :width]


def host(t):
    return t.detach().double().cpu().numpy()


def make(rows, width, dtype, seed=1, mean=0.5, sigma=1.5):
    g = np.random.default_rng(seed)
    x = torch.from_numpy(g.standard_normal((rows, width)) * sigma + mean).to(dtype)
    dy = torch.from_numpy(g.standard_normal((rows, width))).to(dtype)
    gamma, beta = (torch.from_numpy(g.standard_normal(width)).float() for _ in range(2))
    return x.double().numpy(), dy.double().numpy(), gamma, beta


SHAPES = [(1, 1, 0), (3, 2, 1), (2, 7, 0), (5, 8, 0), (4, 63, 5), (7, 64, 0), (3, 65, 0), (2, 513, 3), (6, 1001, 0), (3, 2048, 0), (2, 2049, 7),
          (2, 4097, 0), (3, 8200, 8), (2, 16391, 0), (1, 40001, 0), (2, 70000, 1), (700, 33, 0), (2100, 20, 4), (4099, 130, 1), (65, 9216, 0), (4100, 8200, 0)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("affine", [True, False])
@pytest.mark.parametrize("rows,width,extra", SHAPES)
def test_forward_and_backward(B, rows, width, extra, affine, dtype):
    x, dy, gamma, beta = make(rows, width, dtype)
    ga, be = (gamma.cuda(), beta.cuda()) if affine else (None, None)
    G, Bt = (np.abs(gamma.double().numpy()), np.abs(beta.double().numpy())) if affine else (np.ones(width), np.zeros(width))
    xg, dyg = pitched(x, dtype, extra), pitched(dy, dtype, extra)
    out, dxo = (pitched(np.zeros((rows, width)), dtype, extra, 7.0) for _ in range(2))
    y, mean, rstd = B.layer_norm_forward(xg, ga, be, 1e-5, out)
    ref, rm, rr = ne.layer_norm_forward(x, gamma.double().numpy() if affine else None, beta.double().numpy() if affine else None, 1e-5)
    # the mean's error moves every element; the spread's is relative, and takes the mean's squared
    em = CHAIN * U * np.abs(x).mean(1)
    er = CHAIN * U + (em * rr) ** 2
    assert np.all(np.abs(host(mean) - rm) <= em)
    assert np.all(np.abs(host(rstd) - rr) <= er * rr)
    xh = np.abs(x - rm[:, None]) * rr[:, None]
    tol = (xh * er[:, None] + 8 * U * xh + (em * rr)[:, None]) * G * 1.01 + 4 * U * Bt + half_step(dtype) * np.abs(ref) * 1.01
    assert np.all(np.abs(host(y) - ref) <= tol)
    only, none, _ = B.layer_norm_forward(xg, ga, be, 1e-5, want_stats=False)
    assert none is None and torch.equal(only, y)
    # the backward pass from statistics that fp32 holds exactly as given
    mean, rstd = torch.from_numpy(rm).float().cuda(), torch.from_numpy(rr).float().cuda()
    dx, dgamma, dbeta = B.layer_norm_backward(xg, dyg, mean, rstd, ga, dx=dxo)
    ms, rs = host(mean), host(rstd)
    rdx, rdg, rdb = ne.layer_norm_backward(x, dy, ms, rs, gamma.double().numpy() if affine else None)
    xh, g = np.abs(x - ms[:, None]) * rs[:, None], np.abs(dy) * G
    size = rs[:, None] * (g + g.mean(1, keepdims=True) + xh * (g * xh).mean(1, keepdims=True))
    assert np.all(np.abs(host(dx) - rdx) <= CHAIN * U * size + half_step(dtype) * np.abs(rdx) * 1.01)
    assert np.all(np.abs(host(dgamma) - rdg) <= CHAIN * U * (np.abs(dy) * xh).sum(0))
    assert np.all(np.abs(host(dbeta) - rdb) <= CHAIN * U * np.abs(dy).sum(0))
    if extra:
        for t in (out, dxo):
            assert bool((t.as_strided((rows, extra), (width + extra, 1), width) == 7.0).all()), "the pitch's columns were written"
    again = B.layer_norm_backward(xg, dyg, mean, rstd, ga)
    assert torch.equal(again[0], dx) and torch.equal(again[1], dgamma) and torch.equal(again[2], dbeta)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_each_gradient_alone_and_in_place(B, dtype):
    x, dy, gamma, _ = make(300, 257, dtype)
    xg, dyg, ga = pitched(x, dtype, 0), pitched(dy, dtype, 0), gamma.cuda()
    y, mean, rstd = B.layer_norm_forward(xg, ga)
    dx, dgamma, dbeta = B.layer_norm_backward(xg, dyg, mean, rstd, ga)
    assert torch.equal(B.layer_norm_backward(xg, dyg, mean, rstd, ga, want_dweights=False)[0], dx)
    only = B.layer_norm_backward(xg, dyg, mean, rstd, ga, want_dx=False)
    assert only[0] is None and torch.equal(only[1], dgamma) and torch.equal(only[2], dbeta)
    alone = torch.empty_like(dgamma)
    got = B.layer_norm_backward(xg, dyg, mean, rstd, ga, want_dx=False, want_dweights=False, dgamma=alone)
    assert got[2] is None and torch.equal(alone, dgamma)
    for over in ("x", "dy"):
        a, b = xg.clone(), dyg.clone()
        to = a if over == "x" else b
        got = B.layer_norm_backward(a, b, mean, rstd, ga, dx=to)
        assert torch.equal(to, dx) and torch.equal(got[1], dgamma) and torch.equal(got[2], dbeta)
    a = xg.clone()
    B.layer_norm_forward(a, ga, y=a)
    assert torch.equal(a, y)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("width", [40, 70000])
def test_values_out_of_the_ordinary(B, width, dtype):
    # a constant row: x - mu = 0 exactly (a mean of equal values is that value here: powers of two and their sums), so y = beta and
    # rstd = eps^-1/2; a NaN and an infinity make their own rows NaN and no other
    x = torch.randn(5, width, device="cuda").to(dtype)
    x[1] = 2.0
    x[2, width // 2] = float("nan")
    x[3, width - 1] = float("inf")
    gamma, beta = torch.randn(width, device="cuda"), torch.randn(width, device="cuda")
    y, mean, rstd = B.layer_norm_forward(x, gamma, beta, 2.0 ** -16)
    assert torch.equal(y[1], beta.to(dtype)) and float(rstd[1]) == 256.0 and float(mean[1]) == 2.0
    assert bool(y[2].isnan().all()) and bool(y[3].isnan().all())
    assert bool(y[0].isfinite().all()) and bool(y[4].isfinite().all())
    dx, _, _ = B.layer_norm_backward(x, torch.ones_like(x), mean, rstd, gamma)
    assert bool(dx[2].isnan().all()) and bool(dx[0].isfinite().all()) and bool(dx[1].isfinite().all())
    # far from zero: the squares are taken about the mean, so a mean of 4096 costs its own rounding and no more
    far = (torch.randint(-8, 9, (4, width), device="cuda") * 32.0 + 4096.0).to(dtype)
    y, mean, rstd = B.layer_norm_forward(far)
    ref, rm, rr = ne.layer_norm_forward(host(far))
    em = CHAIN * U * 4096.0 * rr[:, None]
    assert np.all(np.abs(host(y) - ref) <= em + np.abs(ref) * (CHAIN * U + em ** 2 + half_step(dtype)))


def test_no_rows_clear_the_weights_gradients(B):
    x, s = torch.empty((0, 50), device="cuda"), torch.empty((0,), device="cuda")
    dg, db = torch.ones(50, device="cuda"), torch.ones(50, device="cuda")
    dx, _, _ = B.layer_norm_backward(x, x, s, s, dgamma=dg, dbeta=db)
    assert dx.shape == (0, 50) and not bool(dg.any()) and not bool(db.any())
    assert B.layer_norm_forward(x)[0].shape == (0, 50)


def test_many_rows_and_far_offsets(B):
    # more rows than one grid dimension takes, and rows whose offsets pass 32 bits
    rows = (1 << 20) + 77
    x = torch.randn(rows, 3, device="cuda")
    y, mean, rstd = B.layer_norm_forward(x)
    dx, dg, db = B.layer_norm_backward(x, y, mean, rstd)
    sel = torch.tensor([0, 1, (1 << 20) - 1, 1 << 20, rows - 1], device="cuda")
    xs, ys = host(x[sel]), host(y[sel])
    ref, rm, rr = ne.layer_norm_forward(xs)
    slack = CHAIN * U * (1 + np.abs(rm) * rr)[:, None] * (1 + np.abs(ref))
    assert np.all(np.abs(ys - ref) <= slack)
    rdx, _, _ = ne.layer_norm_backward(xs, ys, host(mean[sel]), host(rstd[sel]))
    size = rr[:, None] * (np.abs(ys) + 2.0 + 3.0 * np.abs(ref) * (1 + np.abs(rm) * rr)[:, None])
    assert np.all(np.abs(host(dx[sel]) - rdx) <= CHAIN * U * size)
    ld = (1 << 30) + 8
    full = torch.empty(2 * ld + 100, dtype=torch.bfloat16, device="cuda")
    far = full.as_strided((3, 100), (ld, 1))
    near = torch.randn(3, 100, device="cuda").to(torch.bfloat16)
    far.copy_(near)
    want = B.layer_norm_forward(near)
    got = B.layer_norm_forward(far, y=far)
    assert torch.equal(far, want[0]) and torch.equal(got[1], want[1])
    far.copy_(near)
    b = B.layer_norm_backward(near, near, want[1], want[2])
    c = B.layer_norm_backward(far, far, want[1], want[2], dx=far)
    assert torch.equal(far, b[0]) and torch.equal(c[1], b[1]) and torch.equal(c[2], b[2])
    del full, far
    torch.cuda.empty_cache()


def test_other_stream_and_a_replayed_graph(B):
    x, dy = torch.randn(2000, 300, device="cuda"), torch.randn(2000, 300, device="cuda")
    gamma = torch.randn(300, device="cuda")
    out = {k: torch.empty_like(x) for k in ("y", "dx")}
    mean, rstd, dg, db = torch.empty(2000, device="cuda"), torch.empty(2000, device="cuda"), torch.empty(300, device="cuda"), torch.empty(300, device="cuda")
    ws = torch.empty(max(B.layer_norm_workspace_bytes(2000, 300), 16), dtype=torch.uint8, device="cuda")

    def step():
        B.layer_norm_forward(x, gamma, None, 1e-5, out["y"], mean, rstd)
        B.layer_norm_backward(x, dy, mean, rstd, gamma, out["dx"], dg, db, workspace=ws)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    side.synchronize()
    want = [t.clone() for t in (out["y"], out["dx"], dg, db)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(3):
        x.add_(0.25 * i)
        step()
        want = [t.clone() for t in (out["y"], out["dx"], dg, db)]
        for t in (out["y"], out["dx"], dg, db):
            t.fill_(-1.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, (out["y"], out["dx"], dg, db)))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_widest_row(B, dtype):
    # 2^28 columns, whose tiles are more than one grid dimension takes.  x = +-1 and eps = 0: xh = x exactly, dy = 0, 1, 2, 3, 0, ...:
    # mean dy = 3/2 and mean dy xh = -1/2, and every partial sum is a whole number a thread can hold, so nothing is rounded.
    n = 1 << 28
    x = torch.tensor([1.0, -1.0], device="cuda", dtype=dtype).repeat(n // 2).view(1, n)
    dy = torch.tensor([0.0, 1.0, 2.0, 3.0], device="cuda", dtype=dtype).repeat(n // 4).view(1, n)
    y, mean, rstd = B.layer_norm_forward(x, eps=0.0)
    assert torch.equal(y, x) and mean.item() == 0.0 and rstd.item() == 1.0
    dx, dg, db = B.layer_norm_backward(x, dy, mean, rstd)
    assert torch.equal(db, dy.view(-1).float())
    assert torch.equal(dg.view(-1, 4), torch.tensor([0.0, -1.0, 2.0, -3.0], device="cuda").expand(n // 4, 4))
    assert torch.equal(dx.view(-1, 4), torch.tensor([-1.0, -1.0, 1.0, 1.0], device="cuda", dtype=dtype).expand(n // 4, 4))
    del x, dy, y, dx, dg, db
    torch.cuda.empty_cache()


def test_rows_of_three_dimensions_and_what_is_refused(B):
    base = torch.randn(3, 8, 40, device="cuda")
    x = base[:, ::2, :33]  # 12 rows, 80 apart
    gamma = torch.randn(33, device="cuda")
    y, mean, rstd = B.layer_norm_forward(x, gamma)
    want = B.layer_norm_forward(x.contiguous().view(12, 33), gamma)
    assert y.shape == x.shape and mean.shape == x.shape[:-1] and torch.equal(y.view(12, 33), want[0]) and torch.equal(rstd.view(-1), want[2])
    got = B.layer_norm_backward(x, y, mean, rstd, gamma)
    wanted = B.layer_norm_backward(x.contiguous().view(12, 33), y.view(12, 33), want[1], want[2], gamma)
    assert got[0].shape == x.shape and all(torch.equal(a.reshape(b.shape), b) for a, b in zip(got, wanted))
    one = torch.randn(33, device="cuda")
    assert torch.equal(B.layer_norm_forward(one)[0], B.layer_norm_forward(one.view(1, 33))[0][0])
    for bad in (base[:, :5, :33],                       # rows that are not evenly spaced
                base.transpose(1, 2),                   # rows that are not contiguous
                torch.randn(1, 33, device="cuda").expand(4, 33),  # one row four times
                torch.randn(70, device="cuda").as_strided((3, 33), (10, 1)),
                torch.empty(4, 0, device="cuda"), torch.tensor(1.0, device="cuda"), torch.zeros(4, 33, device="cuda", dtype=torch.int32)):
        with pytest.raises((ValueError, TypeError, B.OmniError)):
            B.layer_norm_forward(bad)
    for kw in (dict(gamma=gamma[:32]), dict(gamma=gamma.double()), dict(gamma=gamma.cpu()), dict(y=torch.empty(11, 33, device="cuda")),
               dict(y=torch.empty(12, 33, device="cuda", dtype=torch.bfloat16)), dict(mean=torch.empty(11, device="cuda")), dict(eps=-1.0)):
        with pytest.raises((ValueError, B.OmniError)):
            B.layer_norm_forward(x, **kw)
    many = torch.zeros(4099, 130, device="cuda")
    rows = torch.zeros(4099, device="cuda")
    with pytest.raises((ValueError, B.OmniError)):
        B.layer_norm_backward(many, many, rows, rows, workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))


@pytest.mark.parametrize("dtype,rows,width", [(torch.bfloat16, 17000, 4096), (torch.float32, 8400, 4099), (torch.bfloat16, 4100, 16400)])
def test_large_gradients_are_those_of_their_rows(B, dtype, rows, width):
    # more than 2^27 bytes of dx, rows that begin anywhere
    x, dy = torch.randn(rows, width, device="cuda").to(dtype), torch.randn(rows, width, device="cuda").to(dtype)
    gamma = torch.randn(width, device="cuda")
    _, mean, rstd = B.layer_norm_forward(x, gamma)
    dx, _, _ = B.layer_norm_backward(x, dy, mean, rstd, gamma)
    half = rows // 4 * 2
    for s in (slice(0, half), slice(half, rows)):
        part, _, _ = B.layer_norm_backward(x[s].clone(), dy[s].clone(), mean[s].clone(), rstd[s].clone(), gamma)
        assert torch.equal(part, dx[s])


def whole_numbers(rows, width, dtype, seed=1):
    """x, dy of small whole numbers, mean 0 and rstd 1 given: xh = x, and every sum of dy and dy xh below 2^24 is exact in any order."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    x, dy = (torch.randint(-3, 4, (rows, width), generator=g, device="cuda").to(dtype) for _ in range(2))
    return x, dy, torch.zeros(rows, device="cuda"), torch.ones(rows, device="cuda")


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows", [2049, 4095, 4097, 4100, 10001, (1 << 20) + 77])
@pytest.mark.parametrize("width", [1, 2, 3, 5, 7])
def test_weights_gradients_of_many_narrow_rows(B, width, rows, dtype):
    # rows narrower than 16 bytes, in numbers that leave some of a workgroup's 16 teams, and whole workgroups, without a row
    x, dy, mean, rstd = whole_numbers(rows, width, dtype)
    _, dgamma, dbeta = B.layer_norm_backward(x, dy, mean, rstd)
    assert torch.equal(dbeta.double(), dy.double().sum(0)) and torch.equal(dgamma.double(), (dy.double() * x.double()).sum(0))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_wide_rows_of_nearly_equal_values(B, dtype):
    # 2^24 columns whose sums' roundings all go the same way: a thread adds 2^14 values.  In fp32 those are 4096 chunks of 4: a sum of
    # 4, 64 of those, 64 of those, then 6 + 15 joins, 153 roundings with those of the terms; in bf16 fewer.
    n = 1 << 24
    g = np.random.default_rng(3)
    x = torch.full((2, n), 0.1).to(dtype)
    x[1] = (0.1 + 1e-3 * torch.from_numpy(g.standard_normal(n))).to(dtype)
    dy = torch.full((2, n), 0.7).to(dtype)
    dy[1, ::2] = 0.3
    xg, dyg = x.cuda(), dy.cuda()
    x, dy = x.double().numpy(), dy.double().numpy()
    y, mean, rstd = B.layer_norm_forward(xg)
    ref, rm, rr = ne.layer_norm_forward(x)
    em = CHAIN * U * np.abs(x).mean(1)
    er = CHAIN * U + (em * rr) ** 2
    assert np.all(np.abs(host(mean) - rm) <= em)
    assert np.all(np.abs(host(rstd) - rr) <= er * rr)
    xh = np.abs(x - rm[:, None]) * rr[:, None]
    assert np.all(np.abs(host(y) - ref) <= (xh * er[:, None] + 8 * U * xh + (em * rr)[:, None]) * 1.01 + half_step(dtype) * np.abs(ref) * 1.01)
    mean, rstd = torch.from_numpy(rm).float().cuda(), torch.from_numpy(rr).float().cuda()
    dx, _, _ = B.layer_norm_backward(xg, dyg, mean, rstd)
    ms, rs = host(mean), host(rstd)
    rdx, _, _ = ne.layer_norm_backward(x, dy, ms, rs)
    xh, d = np.abs(x - ms[:, None]) * rs[:, None], np.abs(dy)
    size = rs[:, None] * (d + d.mean(1, keepdims=True) + xh * (d * xh).mean(1, keepdims=True))
    assert np.all(np.abs(host(dx) - rdx) <= CHAIN * U * size + half_step(dtype) * np.abs(rdx) * 1.01)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows", [2049, 4100])
@pytest.mark.parametrize("width", [8, 255, 256, 300, 512, 777, 1000, 1024, 2000, 2048, 4096, 4100, 8191, 8192])
def test_weights_gradients_of_every_team(B, width, rows, dtype):
    # 64 to 1024 threads a row, whole and cut rows; dx beside them, and over x and dy
    x, dy, mean, rstd = whole_numbers(rows, width, dtype)
    gamma = torch.randint(1, 4, (width,), device="cuda").float()
    dx, dgamma, dbeta = B.layer_norm_backward(x, dy, mean, rstd, gamma)
    assert torch.equal(dbeta.double(), dy.double().sum(0)) and torch.equal(dgamma.double(), (dy.double() * x.double()).sum(0))
    # the two means are exact sums divided once; a product and two differences behind them, and the rounding on store
    xd, g = x.double(), dy.double() * gamma.double()
    mg, mgx = g.mean(1, keepdim=True), (g * xd).mean(1, keepdim=True)
    ref = g - mg - xd * mgx
    bound = 6 * U * (g.abs() + mg.abs() + (xd * mgx).abs()) + half_step(dtype) * ref.abs() * 1.01
    assert bool(((dx.double() - ref).abs() <= bound).all())
    for over in ("x", "dy"):
        a, b = x.clone(), dy.clone()
        to = a if over == "x" else b
        got = B.layer_norm_backward(a, b, mean, rstd, gamma, dx=to)
        assert torch.equal(to, dx) and torch.equal(got[1], dgamma) and torch.equal(got[2], dbeta)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,width,extra", [(3, 8199, 0), (3, 70001, 3), (2, 140000, 0), (4100, 8200, 0)])
def test_long_rows_in_place(B, rows, width, extra, dtype):
    # what a row has beyond a workgroup's registers is read again while the row is written over
    x, dy, gamma, beta = make(rows, width, dtype, seed=8)
    x, dy, ga, be = pitched(x, dtype, extra), pitched(dy, dtype, extra), gamma.cuda(), beta.cuda()
    copy = lambda t: t.as_strided((rows, width + extra), (width + extra, 1)).clone()[:, :width]
    y, mean, rstd = B.layer_norm_forward(x, ga, be)
    a = copy(x)
    B.layer_norm_forward(a, ga, be, y=a)
    assert torch.equal(a, y)
    dx, dgamma, dbeta = B.layer_norm_backward(x, dy, mean, rstd, ga)
    for over in ("x", "dy"):
        a, b = copy(x), copy(dy)
        got = B.layer_norm_backward(a, b, mean, rstd, ga, dx=a if over == "x" else b)
        assert torch.equal(got[0], dx) and torch.equal(got[1], dgamma) and torch.equal(got[2], dbeta)
