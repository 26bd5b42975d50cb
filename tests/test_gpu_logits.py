"""Log probabilities and the distillation loss on the GPU against 64 bits (oracle/network_end.py).  Bounds are counted in
roundings of fp32 arithmetic (u = 2^-24): a row's sum is a chain of at most n / 64 terms a thread (n / 256 for n above 4096),
rescaled at most once a chunk, and 14 joins -- chain(n) below -- and an exponent z costs 4 u |z| relative to its power; what is
stored in bf16 is off by half a step (2^-8) more.  Indexes are equal."""
import numpy as np
import pytest
import torch

from oracle import network_end as ne

pytestmark = pytest.mark.gpu
U, TINY = 2.0 ** -24, 1e-37


@pytest.fixture(scope="module")
def B():
    from paper_1606_04487_amd import binding
    assert torch.cuda.is_available()
    return binding


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def host(t):
    return t.detach().double().cpu().numpy()


def chain(n):
    return 2.0 * (n / 64 if n <= 4096 else n / 256) + 64


def pitched(t, extra, pad=float("nan")):
    rows, width = t.shape
    full = torch.full((rows, width + extra), pad, dtype=t.dtype, device="cuda")
    full[:, :width] = t
    return full[:, :width]


def untouched(t, extra, pad):
    rows, width = t.shape
    return extra == 0 or bool((t.as_strided((rows, extra), (width + extra, 1), t.storage_offset() + width) == pad).all())


def near(got, ref, tol):
    """Within tol where the reference is finite; the same infinities and NaN elsewhere.  A reference past fp32's largest value,
    (2 - 2^-23) 2^127, is the infinity that it rounds to: a class of fp32's lowest value at temperature 1/4 has ln p = -1.4e39."""
    ref = np.where(np.abs(ref) > np.finfo(np.float32).max, np.copysign(np.inf, ref), ref)
    ok = np.isfinite(ref)
    assert np.array_equal(np.isnan(got), np.isnan(ref)) and np.array_equal(got[~ok & ~np.isnan(ref)], ref[~ok & ~np.isnan(ref)])
    assert np.all(np.abs(got[ok] - ref[ok]) <= np.broadcast_to(tol, ref.shape)[ok]), np.max((np.abs(got - ref) / np.broadcast_to(tol, ref.shape))[ok])


def logits(rows, n, dtype, seed=1, sigma=2.5, masked=0.0):
    g = torch.Generator().manual_seed(seed)
    x = (torch.randn(rows, n, generator=g) * sigma).to(dtype)
    if masked:
        x[torch.rand(rows, n, generator=g) < masked] = -float("inf")
    return x.cuda()


def log_probabilities(x, temperature):
    """(ln p, relative bound of p) of every element, in 64 bits."""
    lp = np.array([ne.log_softmax_row(v, temperature) for v in x])
    n = x.shape[1]
    with np.errstate(invalid="ignore"):
        return lp, U * (chain(n) + 8 * (np.where(np.isfinite(lp), np.abs(lp), 0.0) + np.log(n) + 1))


def check_logprob(B, x, targets, top, temperature, extra=0, dlp=None, dh=None, entropy_too=True):
    rows, n = x.shape
    xg = pitched(x, extra)
    lp, h, index, best, stats = B.logprob_forward(xg, targets, top, temperature)
    xh = host(x)
    tg = None if targets is None else targets.view(rows, -1).cpu().numpy()
    rlp, rh, rindex, rbest = ne.logprob_forward(xh, tg, top, temperature)
    full, rel = log_probabilities(xh, temperature)
    worst = U * (chain(n) + 8 * (np.log(n) + 1))
    if targets is not None:
        near(host(lp).reshape(rows, -1), rlp, worst + 8 * U * np.abs(np.nan_to_num(rlp, neginf=0.0)))
    near(host(h), rh, 2 * worst * (1 + np.log(n)))
    if top:
        assert np.array_equal(index.view(rows, top).cpu().numpy(), rindex)
        near(host(best).reshape(rows, top), rbest, worst + 8 * U * np.abs(np.nan_to_num(rbest, neginf=0.0)))
    if dlp is None and dh is None:
        return
    out = pitched(torch.zeros_like(x), extra, 7.0)
    d = B.logprob_backward(xg, stats, targets, dlp, dh, h if dh is not None else None, temperature, out)
    ref = ne.logprob_backward(xh, tg, None if dlp is None else host(dlp).reshape(rows, -1), None if dh is None else host(dh), temperature)
    p, l = np.exp(full), np.where(np.isfinite(full), np.abs(full), 0.0)
    factor = np.zeros_like(p) if dlp is None else np.abs(host(dlp).reshape(rows, -1)).sum(1)[:, None] + np.zeros_like(p)
    if dh is not None:
        factor = factor + np.abs(host(dh))[:, None] * (1 + l + rh[:, None])
    listed = np.zeros_like(p)
    if dlp is not None:
        for r in range(rows):
            for j, t in enumerate(tg[r]):
                if 0 <= t < n:
                    listed[r, t] += abs(float(host(dlp).reshape(rows, -1)[r, j]))
    # a power below 2^-126 is zero, and |ln p| = 87 there: with a factor of 100 that is 1e-36, above TINY
    tol = (2 * rel * factor * p + 2.0 ** -125 * factor + 1100 * U * listed) / temperature
    near(host(d), ref, tol + half_step(x.dtype) * np.abs(ref) * 1.01 + TINY)
    assert untouched(out, extra, 7.0)
    inplace = xg.clone() if extra == 0 else xg
    B.logprob_backward(inplace, stats, targets, dlp, dh, h if dh is not None else None, temperature, inplace)
    assert torch.equal(inplace.view(torch.int16 if x.dtype == torch.bfloat16 else torch.int32),
                       d.view(torch.int16 if x.dtype == torch.bfloat16 else torch.int32))


# lengths around the chunks' and workgroups' edges, to long ones
LENGTHS = [1, 2, 3, 7, 8, 9, 15, 17, 63, 65, 255, 257, 511, 1000, 1025, 2049, 4099, 5003, 8193, 16385, 33001, 70001, 131072]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n", LENGTHS)
def test_logprob_lengths(B, n, dtype):
    for rows, extra, temperature, top in ((3, 0, 1.0, 5), (2, 1, 0.7, 64)):
        x = logits(rows, n, dtype, seed=n)
        g = torch.Generator().manual_seed(n)
        targets = torch.randint(0, n, (rows,), generator=g).cuda()
        check_logprob(B, x, targets, top, temperature, extra, torch.randn(rows, generator=g).cuda(), torch.randn(rows, generator=g).cuda())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,n", [(1, 32769), (5, 65541), (2, 700001), (511, 33000), (512, 33000), (63, 33000), (64, 33000), (95, 33000), (96, 33000)])
def test_few_long_rows_in_parts(B, rows, n, dtype):
    # parts that end inside a chunk, more parts than a row may have, and both sides of the number of rows that are split; rows
    # whose largest elements lie in one part, in ties across all parts, and parts without any possible class
    x = logits(rows, n, dtype, seed=rows)
    x[0, 5000:15000] = 20.0
    x[-1, ::977] = 25.0
    if rows > 3:
        x[1, 9000:] = -float("inf")
        x[2] = -float("inf")
        x[2, n - 1] = 1.0
        x[3, n // 2] = float("nan")
    g = torch.Generator().manual_seed(5)
    targets = torch.randint(0, n, (rows, 2), generator=g).cuda()
    check_logprob(B, x, targets, 40, 0.8, 3, torch.randn(rows, 2, generator=g).cuda())
    check_logprob(B, x, targets, 0, 1.0)
    if rows > 3:
        x[3, n // 2] = 0.0
    for temperature, alpha in ((2.0, 0.5), (3.0, 0.5), (1.0, 1.0)):
        check_distill(B, x, *teacher(rows, n, 7, 2), temperature, alpha, 1 if temperature == 1.0 else 0)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,n,top", [(700, 40, 3), (520, 9001, 20), (1030, 2600, 0), (257, 1000, 5)])
def test_logprob_many_rows(B, rows, n, top, dtype):
    x = logits(rows, n, dtype, masked=0.1)
    g = torch.Generator().manual_seed(5)
    targets = torch.randint(0, n, (rows,), generator=g).cuda()
    check_logprob(B, x, targets, top, 1.3, 0, torch.randn(rows, generator=g).cuda())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n,given", [(5, 1024), (1000, 3), (9001, 17), (300, 256)])
def test_logprob_several_targets(B, n, given, dtype):
    rows, g = 4, torch.Generator().manual_seed(3)
    targets = torch.randint(-n // 4, n, (rows, given), generator=g)      # some left out, many named twice
    targets[1] = -1
    targets[2, :given // 2] = n - 1
    check_logprob(B, logits(rows, n, dtype), targets.cuda(), 0, 2.0, 3, torch.randn(rows, given, generator=g).cuda(), torch.randn(rows, generator=g).cuda())


def test_logprob_entropy_or_targets_alone(B):
    x = logits(9, 777, torch.float32)
    check_logprob(B, x, None, 0, 1.0, 0, None, torch.randn(9).cuda())
    t = torch.randint(0, 777, (9,)).cuda()
    a = B.logprob_forward(x, t, want_entropy=False, want_stats=False)
    b = B.logprob_forward(x, t, 7)
    assert a[1] is None and a[2] is None and a[4] is None and torch.equal(a[0], b[0])


def out_of_the_ordinary(n, dtype):
    lo = torch.finfo(dtype).min
    x = logits(12, n, dtype, seed=n)
    inf = float("inf")
    x[0] = -inf                                  # nothing possible
    x[1] = -inf
    x[1, n // 2] = 3.0                           # one class possible
    x[2] = lo                                    # the type's lowest value everywhere: uniform
    x[3, : n - n // 3] = lo                      # ... as a mask
    x[4] = 0.0                                   # all equal
    x[5, n // 3] = float("nan")
    x[6, n - 1] = inf
    x[7, 0] = float("nan")
    x[7, 1:] = -inf
    x[8] = torch.arange(n).to(dtype)             # ascending
    x[9] = torch.arange(n).flip(0).to(dtype)
    x[10, : n // 2] = 1e4                        # many equal largest
    x[11, ::2] = -0.0
    x[11, 1::2] = 0.0                            # signed zeros are equal
    return x


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n", [6, 100, 1001, 9001, 40000])
def test_logprob_out_of_the_ordinary(B, n, dtype):
    x = out_of_the_ordinary(n, dtype)
    for temperature in (1.0, 0.25):
        targets = torch.tensor([[0, n // 2, -1]] * 12).cuda()
        dlp, dh = torch.randn(12, 3).cuda(), torch.randn(12).cuda()
        check_logprob(B, x, targets, min(n, 20), temperature, 0, dlp, dh)
    x = logits(3, n, dtype)
    targets = torch.tensor([[0], [n], [2 ** 40]]).cuda()                 # past the classes: NaN, and no access there
    check_logprob(B, x, targets, 1, 1.0, 0, torch.ones(3, 1).cuda())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows", [2, 600])
def test_top_alternatives_oddly_placed(B, rows, dtype):
    # the largest values all in the chunks of one thread, for workgroups of 64, 256 and 1024 threads; more equal values than the
    # collection has room for, at the end and everywhere
    n = 40000
    for period in (64, 256, 1024):
        x = logits(rows, n, dtype, sigma=0.5)
        v = 16 // x.element_size()
        at = (torch.arange(n) // v) % period == 3
        x[:, at.cuda()] = 50.0 + torch.randint(0, 40, (int(at.sum()),)).to(dtype).cuda()
        check_logprob(B, x, None, 64, 1.0)
    x = logits(rows, n, dtype, sigma=0.5)
    x[0, 20000:] = 30.0
    x[1, 39000:] = 30.0
    x[1, 38990] = 31.0
    check_logprob(B, x, None, 33, 1.0)


def test_logprob_many_rows_and_far_offsets(B):
    rows = (1 << 20) + 5
    x = torch.randn(rows, 5, device="cuda")
    t = torch.randint(0, 5, (rows,), device="cuda")
    lp, h, index, best, stats = B.logprob_forward(x, t, 2)
    d = B.logprob_backward(x, stats, t, torch.ones(rows, device="cuda"))
    full = torch.log_softmax(x.double(), 1)
    assert float((lp - full.gather(1, t[:, None])[:, 0]).abs().max()) < 200 * U * 10
    assert torch.equal(index, x.topk(2, dim=1).indices)
    ref = -full.exp()
    ref.scatter_add_(1, t[:, None], torch.ones(rows, 1, dtype=torch.float64, device="cuda"))
    assert float((d - ref).abs().max()) < 200 * U * 10
    ld = (1 << 30) + 8
    whole = torch.empty(2 * ld + 5000, dtype=torch.bfloat16, device="cuda")
    far, close = whole.as_strided((3, 5000), (ld, 1)), logits(3, 5000, torch.bfloat16)
    far.copy_(close)
    t = torch.tensor([0, 4999, 7], device="cuda")
    a, b = B.logprob_forward(close, t, 9), B.logprob_forward(far, t, 9)
    assert all(torch.equal(p, q) for p, q in zip(a, b))
    one = torch.ones(3, device="cuda")
    want = B.logprob_backward(close, a[4], t, one)
    assert torch.equal(B.logprob_backward(far, a[4], t, one, dlogits=far), want)
    far.copy_(close)
    want = B.distill_forward_backward(close, labels=t, alpha=0.0)
    got = B.distill_forward_backward(far, labels=t, alpha=0.0, dlogits=far)
    assert torch.equal(got[0], want[0]) and torch.equal(far, want[1])
    del whole, far
    torch.cuda.empty_cache()


# ---------------------------------------------------------------- distillation
def teacher(rows, n, kept, seed, ragged=True):
    g = torch.Generator().manual_seed(seed)
    index = torch.stack([torch.randperm(n, generator=g)[:kept] if kept <= n else torch.randint(0, n, (kept,), generator=g) for _ in range(rows)])
    values = torch.randn(rows, kept, generator=g) * 3
    if ragged and rows > 2 and kept > 1:
        index[0, kept // 2:] = -1
        values[1, 0] = -float("inf")
        index[2] = -1                            # a row without entries
        index[rows - 1, kept - 1] = index[rows - 1, 0]                   # the same class twice
    labels = torch.randint(0, n, (rows,), generator=g)
    labels[rows // 2] = -1
    if rows > 1:
        labels[rows - 1] = index[rows - 1, 0]
    return index.cuda(), values.cuda(), labels.cuda(), torch.rand(rows, generator=g).cuda() + 0.5


def check_distill(B, x, index, values, labels, w, temperature, alpha, extra=0):
    rows, n = x.shape
    xg, out = pitched(x, extra), pitched(torch.zeros_like(x), extra, 7.0)
    args = (index, values, labels, temperature, alpha)
    loss, stats = B.distill_forward(xg, *args)
    d = B.distill_backward(xg, *args, stats=stats, dloss=w, scale=0.5, dlogits=out)
    xh, soft = host(x), index is not None and alpha > 0
    ih, vh = (index.cpu().numpy(), host(values)) if soft else (None, None)
    lh = None if labels is None else labels.cpu().numpy()
    rloss, rd = ne.distill(xh, ih, vh, lh, temperature, alpha, 0.5 * host(w))
    lp, rel = log_probabilities(xh, temperature)
    lp1, rel1 = log_probabilities(xh, 1.0)
    mag, tol = np.zeros(rows), TINY + np.zeros((rows, n))
    ws = 0.5 * host(w)
    for r in range(rows):
        if soft:
            there = (ih[r] >= 0) & (ih[r] < n) & np.isfinite(vh[r])
            at, t = ih[r][there], vh[r][there]
            if at.size:
                lnq = ne.log_softmax_row(t, temperature)
                q, l = np.exp(lnq), np.nan_to_num(np.abs(lp[r, at]), nan=0.0, posinf=0.0)
                mag[r] += alpha * temperature ** 2 * (q * (1 + np.abs(lnq) + l) * (chain(n) + 300 + 8 * (np.abs(lnq) + l + np.log(n) + 1))).sum()
                tol[r] += ws[r] * alpha * temperature * np.nan_to_num(np.exp(lp[r]) * rel[r], nan=0.0)
                np.add.at(tol[r], at, ws[r] * alpha * temperature * q * U * (600 + 8 * np.abs(lnq)))
        if lh is not None and alpha < 1 and 0 <= lh[r] < n:
            l = np.nan_to_num(abs(lp1[r, lh[r]]), nan=0.0, posinf=0.0)
            mag[r] += (1 - alpha) * (chain(n) + 8 * (l + np.log(n) + 1)) * 1.0
            tol[r] += ws[r] * (1 - alpha) * np.nan_to_num(np.exp(lp1[r]) * rel1[r], nan=0.0)
            tol[r, lh[r]] += ws[r] * (1 - alpha) * 8 * U
    near(host(loss), rloss, U * mag + 4 * U * np.abs(np.nan_to_num(rloss, posinf=0.0)))
    bound = 1.5 * tol + 8 * U * np.abs(np.nan_to_num(rd)) + half_step(x.dtype) * np.abs(np.nan_to_num(rd)) * 1.01
    near(host(d), rd, bound)
    assert untouched(out, extra, 7.0)
    both = pitched(torch.zeros_like(x), extra, 7.0)
    loss2, d2 = B.distill_forward_backward(xg, *args, dloss=w, scale=0.5, dlogits=both)
    near(host(loss2), rloss, U * mag + 4 * U * np.abs(np.nan_to_num(rloss, posinf=0.0)))
    near(host(d2), rd, bound)
    assert untouched(both, extra, 7.0)
    for again in range(2):                       # bit-identical, also over the logits themselves
        to = xg.clone() if extra == 0 else pitched(x, extra)
        loss3, _ = B.distill_forward_backward(to, *args, dloss=w, scale=0.5, dlogits=to)
        assert torch.equal(loss3.view(torch.int32), loss2.view(torch.int32)) and np.array_equal(host(to), host(d2), equal_nan=True)
    B.distill_backward(xg, *args, stats=stats, dloss=w, scale=0.5, dlogits=xg)
    assert np.array_equal(host(xg), host(d), equal_nan=True)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n", LENGTHS)
def test_distill_lengths(B, n, dtype):
    for rows, kept, temperature, alpha, extra in ((4, 5, 2.0, 0.6, 0), (3, 33, 1.0, 1.0, 1)):
        check_distill(B, logits(rows, n, dtype, seed=n), *teacher(rows, n, kept, n), temperature, alpha, extra)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,n,kept,temperature,alpha", [(600, 50, 256, 3.0, 0.5), (515, 9001, 8, 1.0, 0.4), (300, 1000, 10, 4.0, 0.7), (1100, 2500, 1, 0.5, 1.0)])
def test_distill_many_rows(B, rows, n, kept, temperature, alpha, dtype):
    check_distill(B, logits(rows, n, dtype), *teacher(rows, n, kept, 3), temperature, alpha)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_cross_entropy_alone_and_each_part_alone(B, dtype):
    x = logits(37, 1000, dtype)
    index, values, labels, w = teacher(37, 1000, 6, 1)
    check_distill(B, x, None, None, labels, w, 1.0, 0.0)
    check_distill(B, x, None, None, labels, w, 5.0, 0.0)
    check_distill(B, x, None, None, labels, w, 5.0, 0.3)
    check_distill(B, x, index, values, None, w, 2.0, 0.3)
    check_distill(B, x, index, values, labels, w, 2.0, 1.0)
    check_distill(B, x, index, values, labels, w, 2.0, 0.0)
    loss, d = B.distill_forward_backward(x, labels=labels, alpha=0.0)      # no weights: ones
    one, d1 = B.distill_forward_backward(x, labels=labels, alpha=0.0, dloss=torch.ones(37, device="cuda"))
    assert torch.equal(loss, one) and torch.equal(d, d1)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n", [6, 1001, 9001, 40000])
@pytest.mark.parametrize("temperature,alpha", [(2.0, 0.5), (0.25, 1.0), (1.0, 0.0)])
def test_distill_out_of_the_ordinary(B, n, temperature, alpha, dtype):
    x = out_of_the_ordinary(n, dtype)
    index = torch.tensor([[0, n // 2, n - 1, 1]] * 12)
    values = torch.tensor([[0.5, -1.0, 2.0, -float("inf")]] * 12)
    labels = torch.arange(12) % n
    labels[4] = -100
    check_distill(B, x, index.cuda(), values.cuda(), labels.cuda(), torch.ones(12).cuda(), temperature, alpha)
    # entries and labels past the classes, and entries that are no numbers: NaN, and no access there
    x = logits(5, n, dtype)
    index, values, labels = torch.zeros((5, 2), dtype=torch.int64), torch.zeros(5, 2), torch.zeros(5, dtype=torch.int64)
    index[0, 1], index[1, 0], values[2, 1], values[3, 0], labels[4] = n, 2 ** 40, float("nan"), float("inf"), n
    check_distill(B, x, index.cuda(), values.cuda(), labels.cuda(), torch.ones(5).cuda(), temperature, alpha)


def test_gradients_by_differences(B):
    # fp32 losses of a few rows against their gradients: central differences of width h = 2^-6 are off by h^2 / 6 times the third
    # derivative (of a log-sum-exp at most 0.1, of an entropy at most 8) plus the rounding of two losses of at most 10, over h
    rows, n, h = 3, 21, 2.0 ** -6
    x = logits(rows, n, torch.float32, sigma=1.0)
    index, values, labels, w = teacher(rows, n, 4, 9, ragged=False)
    _, d = B.distill_forward_backward(x, index, values, labels, 2.0, 0.5, dloss=w)
    lp0, h0, _, _, stats = B.logprob_forward(x, labels.clamp(min=0))
    e = B.logprob_backward(x, stats, labels.clamp(min=0), w, w, h0)
    for i in range(n):
        up, down = x.clone(), x.clone()
        up[:, i] += h
        down[:, i] -= h
        step = (up[:, i] - down[:, i]).double()
        fd = (B.distill_forward(up, index, values, labels, 2.0, 0.5)[0] - B.distill_forward(down, index, values, labels, 2.0, 0.5)[0]).double() * w / step
        assert float((fd - d[:, i]).abs().max()) < 1.5 * h * h + 64 * U * 10 * 1.5 / h
        a, b = B.logprob_forward(up, labels.clamp(min=0)), B.logprob_forward(down, labels.clamp(min=0))
        fd = ((a[0] - b[0]).double() + (a[1] - b[1]).double()) * w / step
        assert float((fd - e[:, i]).abs().max()) < 1.5 * 8 * h * h + 64 * U * 20 * 1.5 / h


def test_together_on_other_streams_and_in_a_replayed_graph(B):
    """The teacher's top alternatives are the student's entries: one after the other, on a side stream, and as one graph."""
    rows, n, k = 300, 5001, 12
    student, big = logits(rows, n, torch.bfloat16, seed=1), logits(rows, n, torch.bfloat16, seed=2)
    labels = torch.randint(0, n, (rows,)).cuda()
    w = torch.rand(rows).cuda()
    index, best = torch.empty((rows, k), dtype=torch.int64, device="cuda"), torch.empty((rows, k), device="cuda")
    loss, out = torch.empty(rows, device="cuda"), torch.empty_like(student)
    lp, h, st = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda"), torch.empty((rows, 2), device="cuda")

    def together():
        B.logprob_forward(big, labels, k, logprob=lp, entropy=h, top_index=index, top_logprob=best, stats=st)
        B.distill_forward_backward(student, index, best, labels, 2.0, 0.5, dloss=w, loss=loss, dlogits=out)
        B.logprob_backward(student, st, labels, w, dlogits=big)          # (with the teacher's sums: only its repetition is looked at)
    outs = (index, best, loss, out, lp, h, st, big)
    side = torch.cuda.Stream()
    keep = big.clone()
    together()
    want = [t.clone() for t in outs]
    rl, rd = ne.distill(host(student), index.cpu().numpy(), host(best), labels.cpu().numpy(), 2.0, 0.5, host(w))
    assert np.max(np.abs(host(loss) - rl)) <= U * 4 * (chain(n) + 400) * 25
    assert np.all(np.abs(host(out) - rd) <= half_step(torch.bfloat16) * np.abs(rd) * 1.01 + U * 2 * (chain(n) + 600 + 400))
    big.copy_(keep)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        together()
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, outs))
    graph = torch.cuda.CUDAGraph()
    big.copy_(keep)
    with torch.cuda.graph(graph):
        together()
    for i in range(3):
        keep.mul_(1.5)
        student.add_(0.125 * (i + 1))
        big.copy_(keep)
        together()
        want = [t.clone() for t in outs]
        big.copy_(keep)
        for t in (index, best, loss, out, lp, h, st):
            t.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, outs))


def test_widest_row(B):
    # 2^30 classes of 0 but for three.  A thread of the 64 parts adds 2^16 terms in two chains, so the sum is off by 2^15 + 64
    # roundings at most, relatively; a gradient by as much and the half step it is stored with.
    n = 1 << 30
    x = torch.zeros(1, n, dtype=torch.bfloat16, device="cuda")
    x[0, 5], x[0, n - 1], x[0, 1 << 29] = 1.0, 2.0, -float("inf")
    s = (n - 3) * np.exp(-2.0) + np.exp(-1.0) + 1.0
    slack = (2.0 ** 15 + 64) * U
    targets = torch.tensor([[n - 1, 5, 1 << 29, 7]], device="cuda")
    lp, entropy, index, best, stats = B.logprob_forward(x, targets, top=2)
    ref = np.array([0.0, -1.0, -np.inf, -2.0]) - np.log(s)
    near(host(lp)[0], ref, slack + 8 * U * np.log(s))
    assert index.tolist() == [[n - 1, 5]] and np.all(np.abs(host(best)[0] - ref[:2]) <= slack + 8 * U * np.log(s))
    h = -((n - 3) * np.exp(ref[3]) * ref[3] + np.exp(ref[1]) * ref[1] + np.exp(ref[0]) * ref[0])
    assert abs(entropy.item() - h) <= 3 * slack * (np.log(s) + 2.0)
    grad = B.logprob_backward(x, stats, targets[:, :1].contiguous(), torch.ones(1, device="cuda"))
    p = np.exp(ref)
    tol = 2 * slack + 2.0 ** -8
    got = host(grad[0, targets[0]])
    assert abs(got[0] - (1 - p[0])) <= tol and np.all(np.abs(got[1:] + p[1:]) <= tol * p[1:])
    grad[0, targets[0]] = grad[0, 8].item()
    assert bool((grad == grad[0, 8]).all()) and abs(grad[0, 8].item() + p[3]) <= tol * p[3]
    loss, both = B.distill_forward_backward(x, index, best, temperature=1.0, alpha=1.0, dlogits=grad)
    q = np.exp(ref[:2]) / np.exp(ref[:2]).sum()
    assert abs(loss.item() - (q * (np.log(q) - ref[:2])).sum()) <= slack + 16 * U * np.log(s)
    got = host(both[0, targets[0]])
    assert np.all(np.abs(got - (p - np.array([q[0], q[1], 0.0, 0.0]))) <= tol * np.array([1.0, 1.0, p[2], p[3]]))
    del x, grad, both
    torch.cuda.empty_cache()


@pytest.mark.parametrize("extra", [0, 7])
def test_large_gradients_are_those_of_their_rows(B, extra):
    # more than 2^27 bytes of results, rows that begin anywhere, and outputs whose rows are aligned otherwise
    rows, n, k = 2100, 33001, 4
    x = logits(rows, n, torch.bfloat16)
    index, labels = torch.randint(0, n, (rows, k)).cuda(), torch.randint(0, n, (rows,)).cuda()
    best, w, stats = torch.randn(rows, k).cuda(), torch.rand(rows).cuda(), None
    out = [pitched(torch.zeros_like(x), extra, 3.0) for _ in range(3)]
    loss, _ = B.distill_forward_backward(x, index, best, labels, 2.0, 0.5, dloss=w, dlogits=out[0])
    _, stats = B.distill_forward(x, index, best, labels, 2.0, 0.5)
    B.distill_backward(x, index, best, labels, 2.0, 0.5, stats=stats, dloss=w, dlogits=out[1])
    lp, h, _, _, st = B.logprob_forward(x, labels)
    B.logprob_backward(x, st, labels, w, w, h, dlogits=out[2])
    # A row's sums are taken in an order that depends on where it begins within 16 bytes, so the parts begin at whole multiples of 8
    # rows: there a row of the part begins where it does in the whole.
    for a in range(0, rows, 704):
        s = slice(a, a + 704)
        part = x[s].clone()
        l, d = B.distill_forward_backward(part, index[s].clone(), best[s].clone(), labels[s].clone(), 2.0, 0.5, dloss=w[s].clone())
        assert torch.equal(l, loss[s]) and torch.equal(d, out[0][s])
        d = B.distill_backward(part, index[s].clone(), best[s].clone(), labels[s].clone(), 2.0, 0.5, stats=stats[s].clone(), dloss=w[s].clone())
        assert torch.equal(d, out[1][s])
        d = B.logprob_backward(part, st[s].clone(), labels[s].clone(), w[s].clone(), w[s].clone(), h[s].clone())
        assert torch.equal(d, out[2][s])
    assert all(untouched(t, extra, 3.0) for t in out)


def test_shapes_and_what_the_binding_refuses(B):
    x = torch.randn(2, 3, 50, device="cuda")
    t = torch.randint(0, 50, (2, 3), device="cuda")
    lp, h, index, best, stats = B.logprob_forward(x, t, top=4)
    assert lp.shape == h.shape == (2, 3) and index.shape == best.shape == (2, 3, 4) and stats.shape == (2, 3, 2)
    flat = B.logprob_forward(x.view(6, 50), t.view(6), top=4)
    assert all(torch.equal(a.reshape(b.shape), b) for a, b in zip((lp, h, index, best, stats), flat))
    loss, grad = B.distill_forward_backward(x, index, best, t, 2.0, 0.5)
    assert loss.shape == (2, 3) and grad.shape == x.shape
    ones = torch.ones(2, 3, device="cuda")
    long = torch.randn(2, 131072, device="cuda")
    small = torch.empty(16, dtype=torch.uint8, device="cuda")
    for call in (lambda: B.logprob_forward(x, t.int()), lambda: B.logprob_forward(x, t.cpu()), lambda: B.logprob_forward(x, t.view(-1)[:4]),
                 lambda: B.logprob_forward(x[:, :1].expand(2, 3, 50), t), lambda: B.logprob_forward(x, t, top=65), lambda: B.logprob_forward(x, t, temperature=0.0),
                 lambda: B.logprob_forward(x.half(), t), lambda: B.logprob_forward(x.transpose(1, 2), None),
                 lambda: B.logprob_forward(long, None, top=5, workspace=small),
                 lambda: B.logprob_backward(x, stats, t, None), lambda: B.logprob_backward(x, stats.view(-1)[:6], t, ones),
                 lambda: B.logprob_backward(x, stats, t, ones, dentropy=ones), lambda: B.logprob_backward(x, stats, t, ones, dlogits=torch.empty(5, 50, device="cuda")),
                 lambda: B.distill_forward(x, index, best[..., :3].contiguous(), t, 2.0, 0.5), lambda: B.distill_forward(x, index, None, t, 2.0, 0.5),
                 lambda: B.distill_forward(x, None, None, t), lambda: B.distill_forward(x, index, best, t.int(), 2.0, 0.5),
                 lambda: B.distill_forward(x, index, best, t, 2.0, 1.5), lambda: B.distill_forward(long, None, None, t[:, 0].contiguous(), alpha=0.0, workspace=small),
                 lambda: B.distill_backward(x, index, best, t, 2.0, 0.5, stats=stats), lambda: B.distill_forward_backward(x, index, best, t, 2.0, 0.5, dloss=ones[:1])):
        with pytest.raises((ValueError, B.OmniError)):
            call()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,n", [(9, 6), (9, 100), (9, 1001), (9, 9001), (9, 40000), (99, 40000)])
def test_rows_without_a_loss_have_no_gradient(B, rows, n, dtype):
    # the rows that fill a batch up: no entries and no label, whatever their logits are (parts of a row, and whole rows)
    x = logits(rows, n, dtype, seed=n)
    inf, nan = float("inf"), float("nan")
    x[0, n // 2] = nan
    x[1, 0] = inf
    x[2] = nan
    x[3, n - 1], x[3, 1] = inf, nan
    x[4] = -inf
    x[5, n // 3] = nan                           # with entries: NaN
    x[7, n // 3] = nan                           # with a label: NaN where the labels count
    g = torch.Generator().manual_seed(n)
    index, values = torch.randint(0, n, (rows, 5), generator=g), torch.randn(rows, 5, generator=g)
    labels, w = torch.randint(0, n, (rows,), generator=g), torch.rand(rows, generator=g) + 0.5
    index[:5], index[7] = -1, -1
    index[1] = 2
    values[1] = -inf
    labels[:7] = -1
    for temperature, alpha, extra in ((2.0, 0.5, 0), (4.0, 0.5, 1), (3.0, 0.5, 0), (2.0, 1.0, 3), (1.0, 0.0, 0)):
        check_distill(B, x, index.cuda(), values.cuda(), labels.cuda(), w.cuda(), temperature, alpha, extra)


def test_ties_in_many_short_rows(B):
    # values of a set of four: nearly every row has equal ones among its largest, which rank by index
    rows, g = (1 << 20) + 5, torch.Generator(device="cuda").manual_seed(2)
    x = torch.randint(0, 4, (rows, 5), generator=g, device="cuda").float() * 0.5
    index, best = B.logprob_forward(x, top=3)[2:4]
    order = torch.arange(5, device="cuda") - 8 * (x * 2).long()          # descending, then ascending by index; no two are equal
    assert torch.equal(index, order.sort(dim=1).indices[:, :3])
    full = torch.log_softmax(x.double(), 1)
    assert float((best - full.gather(1, index)).abs().max()) < 200 * U * 10


def test_what_belongs_to_the_rows_is_in_their_order(B):
    """[S][B] beside logits of [B][S][classes] holds as many values and means others."""
    x = torch.randn(2, 3, 50).cuda()
    t, w = torch.randint(0, 50, (2, 3)).cuda(), torch.rand(2, 3).cuda()
    lp, h, index, best, stats = B.logprob_forward(x, t, top=4)
    turned = lambda v: v.transpose(0, 1).contiguous()
    for call in (lambda: B.logprob_forward(x, turned(t)), lambda: B.logprob_forward(x, t, logprob=turned(lp)), lambda: B.logprob_forward(x, entropy=turned(h)),
                 lambda: B.logprob_backward(x, turned(stats), t, w), lambda: B.logprob_backward(x, stats, turned(t), w), lambda: B.logprob_backward(x, stats, t, turned(w)),
                 lambda: B.logprob_backward(x, stats, t, w, turned(w), h), lambda: B.logprob_backward(x, stats, t, w, w, turned(h)),
                 lambda: B.distill_forward(x, turned(index), turned(best), t, 2.0, 0.5), lambda: B.distill_forward(x, index, best, turned(t), 2.0, 0.5),
                 lambda: B.distill_forward(x, index, best, t, 2.0, 0.5, loss=turned(w)), lambda: B.distill_forward_backward(x, index, best, t, dloss=turned(w)),
                 lambda: B.distill_forward_backward(x, index, best, turned(t), 2.0, 0.5), lambda: B.layer_norm_forward(x, mean=turned(w)),
                 lambda: B.layer_norm_backward(x, x, turned(w), w), lambda: B.layer_norm_backward(x, x, w, turned(w)),
                 lambda: B.layer_norm_forward(x, y=turned(x)), lambda: B.layer_norm_backward(x, turned(x), w, w), lambda: B.distill_forward_backward(x, index, best, dlogits=turned(x)),
                 lambda: B.distill_forward(x.view(6, 50), index.view(6, 4).t().contiguous(), best.view(6, 4).t().contiguous())):
        with pytest.raises(ValueError):
            call()
    # the same rows counted together, or with an axis of one or several targets a row more
    for same in (t.view(6), t.view(2, 3, 1), t.view(1, 2, 3), t.view(6, 1)):
        assert torch.equal(B.logprob_forward(x, same)[0].view(2, 3), lp)
    two = torch.stack([t, t], 2)
    assert torch.equal(B.logprob_forward(x, two)[0], torch.stack([lp, lp], 2)) and torch.equal(B.logprob_forward(x, two.view(6, 2))[0].view(2, 3, 2), torch.stack([lp, lp], 2))
    assert torch.equal(B.logprob_forward(x.view(6, 50), t)[0], lp)
    assert torch.equal(B.layer_norm_forward(x, y=torch.empty(6, 50, device="cuda"))[0], B.layer_norm_forward(x)[0].view(6, 50))


def test_small_inputs_that_begin_anywhere(B):
    """The next-token call: targets one token on, from the middle of their tensor; and inputs that are not contiguous."""
    rows, n = 33, 301
    x = logits(rows, n, torch.bfloat16)
    tokens, far = torch.randint(0, n, (rows + 1,)).cuda(), torch.rand(2 * rows + 3).cuda()
    odd = lambda t: torch.cat([t.new_zeros(1), t.reshape(-1)])[1:].view(t.shape)  # the same values, one element further on
    assert all(odd(t).data_ptr() % 16 for t in (tokens, far))
    t, w = tokens[1:], far[1:rows + 1]
    want = B.logprob_forward(x, t.clone(), 5)
    got = B.logprob_forward(x, t, 5)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    lp, h, index, best, stats = want
    want = B.logprob_backward(x, stats, t.clone(), w.clone(), w.clone(), h)
    assert torch.equal(B.logprob_backward(x, odd(stats), t, w, torch.stack([w, h], 1)[:, 0], odd(h)), want)
    wanted = B.distill_forward_backward(x, index, best, t.clone(), 2.0, 0.5, dloss=w.clone())
    wide, deep = torch.cat([index, index], 1), torch.cat([best, best], 1)
    loss, d = B.distill_forward_backward(x, wide[:, 5:], deep[:, :5], t, 2.0, 0.5, dloss=w)
    assert torch.equal(loss, wanted[0]) and torch.equal(d, wanted[1])
    loss, st = B.distill_forward(x, odd(index), odd(best), t, 2.0, 0.5)
    assert torch.equal(B.distill_backward(x, odd(index), odd(best), t, 2.0, 0.5, stats=odd(st), dloss=w),
                       B.distill_backward(x, index, best, t.clone(), 2.0, 0.5, stats=st, dloss=w.clone()))
    gamma, beta = torch.rand(n).cuda(), torch.rand(n).cuda()
    y, mean, rstd = B.layer_norm_forward(x, gamma, beta)
    assert torch.equal(B.layer_norm_forward(x, odd(gamma), odd(beta))[0], y)
    assert all(torch.equal(a, b) for a, b in zip(B.layer_norm_backward(x, y, odd(mean), odd(rstd), odd(gamma)), B.layer_norm_backward(x, y, mean, rstd, gamma)))
    # what is written has to lie where the library takes it
    with pytest.raises(B.OmniError):
        B.distill_forward(x, index, best, t, 2.0, 0.5, loss=far[1:rows + 1])


def test_small_inputs_that_begin_anywhere_in_a_replayed_graph(B):
    x, tokens = logits(40, 1000, torch.float32), torch.randint(0, 1000, (41,)).cuda()
    loss, out = torch.empty(40, device="cuda"), torch.empty_like(x)

    def step():
        B.distill_forward_backward(x, labels=tokens[1:], alpha=0.0, loss=loss, dlogits=out)
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(3):
        tokens.copy_(torch.randint(0, 1000, (41,)))
        want = B.distill_forward_backward(x, labels=tokens[1:].clone(), alpha=0.0)
        loss.zero_(), out.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(loss, want[0]) and torch.equal(out, want[1])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,n,extra", [(96, 70001, 0), (97, 140003, 1)])
def test_distill_long_rows_that_are_not_split(B, rows, n, extra, dtype):
    # workgroups of 1024 that keep a whole row, and rows longer than they keep
    check_distill(B, logits(rows, n, dtype), *teacher(rows, n, 9, 4), 2.0, 0.5, extra)
