"""Refusals of the entry points at the end of a network: argument checks are host code, made before anything is launched."""
import ctypes

import pytest
import torch

F = ctypes.c_float
P, ODD = ctypes.c_void_p(0x1000), ctypes.c_void_p(0x1008)
BIG = 1 << 40


@pytest.fixture(scope="module")
def B():
    from paper_1606_04487_amd import binding
    return binding


@pytest.fixture(scope="module")
def L(B):
    return B.raw()


def norm_forward(L, dtype=0, rows=4, width=8, x=P, ldx=8, gamma=P, beta=P, eps=1e-5, y=P, ldy=8, mean=P, rstd=P):
    return L.omni_layer_norm_forward(dtype, rows, width, x, ldx, gamma, beta, F(eps), y, ldy, mean, rstd, None)


def norm_backward(L, dtype=0, rows=4, width=8, x=P, ldx=8, dy=P, lddy=8, gamma=P, mean=P, rstd=P, dx=P, lddx=8, dgamma=P, dbeta=P, ws=P, nws=BIG):
    return L.omni_layer_norm_backward(dtype, rows, width, x, ldx, dy, lddy, gamma, mean, rstd, dx, lddx, dgamma, dbeta, ws, nws, None)


def logprob_forward(L, dtype=0, rows=4, classes=8, x=P, ld=8, t=1.0, targets=P, given=1, lp=P, entropy=P, top=2, index=P, best=P, stats=P, ws=P, nws=BIG):
    return L.omni_logprob_forward(dtype, rows, classes, x, ld, F(t), targets, given, lp, entropy, top, index, best, stats, ws, nws, None)


def logprob_backward(L, dtype=0, rows=4, classes=8, x=P, ld=8, t=1.0, stats=P, targets=P, given=1, dlp=P, dh=P, h=P, out=P, ldo=8):
    return L.omni_logprob_backward(dtype, rows, classes, x, ld, F(t), stats, targets, given, dlp, dh, h, out, ldo, None)


def distill_forward(L, dtype=0, rows=4, classes=8, x=P, ld=8, index=P, values=P, kept=3, labels=P, t=1.0, alpha=0.5, loss=P, stats=P, ws=P, nws=BIG):
    return L.omni_distill_forward(dtype, rows, classes, x, ld, index, values, kept, labels, F(t), F(alpha), loss, stats, ws, nws, None)


def distill_backward(L, dtype=0, rows=4, classes=8, x=P, ld=8, index=P, values=P, kept=3, labels=P, t=1.0, alpha=0.5, stats=P, dloss=P, scale=1.0, out=P, ldo=8):
    return L.omni_distill_backward(dtype, rows, classes, x, ld, index, values, kept, labels, F(t), F(alpha), stats, dloss, F(scale), out, ldo, None)


def distill_both(L, dtype=0, rows=4, classes=8, x=P, ld=8, index=P, values=P, kept=3, labels=P, t=1.0, alpha=0.5, dloss=P, scale=1.0, loss=P, out=P, ldo=8, ws=P,
                 nws=BIG):
    return L.omni_distill_forward_backward(dtype, rows, classes, x, ld, index, values, kept, labels, F(t), F(alpha), dloss, F(scale), loss, out, ldo, ws, nws, None)


NAN, INF = float("nan"), float("inf")
SHAPE = [(dict(dtype=2), -2), (dict(rows=-1), -1), (dict(rows=1 << 31), -2)]
CLASSES = SHAPE + [(dict(classes=0), -1), (dict(classes=(1 << 30) + 1, ld=1 << 31), -2), (dict(rows=1 << 20, classes=1 << 30, ld=1 << 30), -2), (dict(ld=7), -1),
                   (dict(x=None), -1), (dict(x=ODD), -4), (dict(t=0.0), -1), (dict(t=-1.0), -1), (dict(t=NAN), -1), (dict(t=INF), -1), (dict(t=1e-35), -1)]


LONG = [(dict(classes=131072, ld=131072, ws=None), -1), (dict(classes=131072, ld=131072, nws=0), -3)]  # rows that are worked on in parts


@pytest.mark.parametrize("change,status", SHAPE + [
    (dict(width=0), -1), (dict(width=(1 << 28) + 1, ldx=1 << 29, ldy=1 << 29), -2), (dict(ldx=7), -1), (dict(ldy=7), -1), (dict(x=None), -1), (dict(y=None), -1),
    (dict(eps=-1.0), -1), (dict(eps=NAN), -1), (dict(eps=INF), -1), (dict(y=P, ldy=9), -1)] + [(dict([(k, ODD)]), -4) for k in ("x", "gamma", "beta", "y", "mean", "rstd")])
def test_layer_norm_forward_refuses(L, change, status):
    assert norm_forward(L, **change) == status


@pytest.mark.parametrize("change,status", SHAPE + [
    (dict(width=0), -1), (dict(ldx=7), -1), (dict(lddy=7), -1), (dict(lddx=7), -1), (dict(dx=None, dgamma=None, dbeta=None), -1), (dict(lddx=9), -1),
    (dict(rows=100000, ws=None), -1), (dict(rows=100000, nws=0), -3)]
    + [(dict([(k, None)]), -1) for k in ("x", "dy", "mean", "rstd")]
    + [(dict([(k, ODD)]), -4) for k in ("x", "dy", "gamma", "mean", "rstd", "dx", "dgamma", "dbeta", "ws")])
def test_layer_norm_backward_refuses(L, change, status):
    assert norm_backward(L, **change) == status


@pytest.mark.parametrize("change,status", CLASSES + [
    (dict(given=-1), -1), (dict(top=-1), -1), (dict(given=1025), -2), (dict(top=65), -2), (dict(targets=None), -1), (dict(lp=None), -1), (dict(index=None), -1),
    (dict(best=None), -1)] + [(dict([(k, ODD)]), -4) for k in ("targets", "lp", "entropy", "index", "best", "stats", "ws")] + LONG)
def test_logprob_forward_refuses(L, change, status):
    assert logprob_forward(L, **change) == status


@pytest.mark.parametrize("change,status", CLASSES + [
    (dict(ldo=7), -1), (dict(ldo=9), -1), (dict(given=-1), -1), (dict(given=1025), -2), (dict(h=None), -1)]
    + [(dict([(k, None)]), -1) for k in ("stats", "targets", "dlp", "out")] + [(dict([(k, ODD)]), -4) for k in ("stats", "targets", "dlp", "dh", "h", "out")])
def test_logprob_backward_refuses(L, change, status):
    assert logprob_backward(L, **change) == status


PARTS = [(dict(kept=-1), -1), (dict(kept=257), -2), (dict(index=None), -1), (dict(values=None), -1), (dict(alpha=-0.1), -1), (dict(alpha=1.1), -1), (dict(alpha=NAN), -1),
         (dict(kept=0, labels=None), -1), (dict(alpha=0.0, labels=None), -1), (dict(alpha=1.0, kept=0), -1), (dict(t=1e-20), -1), (dict(t=1e20), -1)] \
    + [(dict([(k, ODD)]), -4) for k in ("index", "values", "labels")]


@pytest.mark.parametrize("change,status", CLASSES + PARTS + [(dict(loss=None), -1), (dict(loss=ODD), -4), (dict(stats=ODD), -4), (dict(ws=ODD), -4)] + LONG)
def test_distill_forward_refuses(L, change, status):
    assert distill_forward(L, **change) == status


@pytest.mark.parametrize("change,status", CLASSES + PARTS + [(dict(stats=None), -1), (dict(out=None), -1), (dict(ldo=7), -1), (dict(ldo=9), -1)]
                         + [(dict([(k, ODD)]), -4) for k in ("stats", "dloss", "out")])
def test_distill_backward_refuses(L, change, status):
    assert distill_backward(L, **change) == status


@pytest.mark.parametrize("change,status", CLASSES + PARTS + [(dict(loss=None), -1), (dict(out=None), -1), (dict(ldo=7), -1), (dict(ldo=9), -1)]
                         + [(dict([(k, ODD)]), -4) for k in ("loss", "dloss", "out", "ws")]
                         + [(dict(ldo=131072, **c), st) for c, st in LONG])
def test_distill_both_refuses(L, change, status):
    assert distill_both(L, **change) == status


def test_no_rows_need_no_buffers(L):
    nothing = dict(rows=0, x=None)
    assert norm_forward(L, y=None, mean=None, rstd=None, **nothing) == 0
    assert norm_backward(L, dy=None, mean=None, rstd=None, dgamma=None, dbeta=None, ws=None, nws=0, **nothing) == 0
    assert logprob_forward(L, targets=None, lp=None, index=None, best=None, ws=None, nws=0, **nothing) == 0
    assert logprob_backward(L, stats=None, targets=None, dlp=None, out=None, **nothing) == 0
    assert distill_forward(L, index=None, values=None, loss=None, ws=None, nws=0, **nothing) == 0
    assert distill_backward(L, index=None, values=None, stats=None, out=None, **nothing) == 0
    assert distill_both(L, index=None, values=None, loss=None, out=None, ws=None, nws=0, **nothing) == 0


def test_workspace_never_shrinks_with_more_rows(B, L):
    for dtype in (torch.float32, torch.bfloat16):
        for width in (1, 33, 1000, 4096, 131072):
            for size in (lambda r: B.layer_norm_workspace_bytes(r, width, dtype), lambda r: B.logprob_workspace_bytes(r, width, 64, dtype),
                         lambda r: B.distill_workspace_bytes(r, width, dtype)):
                sizes = [size(r) for r in (0, 1, 2, 3, 7, 16, 31, 63, 64, 65, 100, 255, 256, 500, 511, 512, 513, 1000, 1024, 5000, 70000)]
                assert sizes == sorted(sizes), (width, dtype)
    b = ctypes.c_size_t()
    assert L.omni_logprob_workspace_bytes(0, 4, 8, 65, ctypes.byref(b)) == -2 and L.omni_logprob_workspace_bytes(0, 4, 8, -1, ctypes.byref(b)) == -1
    assert L.omni_distill_workspace_bytes(0, 4, 0, ctypes.byref(b)) == -1 and L.omni_distill_workspace_bytes(0, 4, 8, None) == -1
    assert L.omni_layer_norm_workspace_bytes(0, 4, 8, None) == -1 and L.omni_layer_norm_workspace_bytes(3, 4, 8, ctypes.byref(b)) == -2


def test_binding_refuses_what_is_not_on_the_gpu(B):
    x = torch.zeros(4, 8)
    for call in (lambda: B.layer_norm_forward(x), lambda: B.layer_norm_backward(x, x, x[:, 0], x[:, 0]), lambda: B.logprob_forward(x),
                 lambda: B.logprob_backward(x, x), lambda: B.distill_forward(x), lambda: B.distill_backward(x), lambda: B.distill_forward_backward(x)):
        with pytest.raises(ValueError):
            call()


@pytest.mark.parametrize("lead,shape,ordered", [
    ((2, 3), (2, 3), True), ((2, 3), (6,), True), ((2, 3), (2, 3, 4), True), ((2, 3), (6, 4), True), ((2, 3), (1, 2, 1, 3), True), ((6,), (2, 3), True), ((6,), (3, 2), True),
    ((2, 3, 4), (6, 4), True), ((2, 3, 4), (2, 12, 5), True), ((6, 4), (2, 3, 4), True), ((1, 1), (5,), True), ((0, 3), (3, 0), True), ((2, 3), (2, 3, 0), True), ((3, 3), (3, 3), True),
    ((2, 3), (3, 2), False), ((2, 3), (3, 2, 4), False), ((6,), (4, 6), False), ((2, 3, 4), (2, 4, 3), False), ((2, 3, 4), (8, 3), False), ((6, 4), (8, 3), False)])
def test_what_belongs_to_rows_is_in_their_order(B, lead, shape, ordered):
    if ordered:
        B._check_order(torch.Size(lead), torch.Size(shape), "targets")
    else:
        with pytest.raises(ValueError):
            B._check_order(torch.Size(lead), torch.Size(shape), "targets")


@pytest.mark.parametrize("name,cls", [
    ("void omni::layer_norm_forward_kernel<float, 512, 2, (omni::Fit)0>(float const*, long)", "layer_norm"),
    ("void omni::layer_norm_backward_long_kernel<unsigned short>(omni::NormBackward<unsigned short>, int)", "layer_norm"),
    ("omni::layer_norm_join_kernel(float const*, int, int, float*, float*)", "layer_norm"),
    ("void omni::logprob_forward_kernel<float, 64, 4, true>(float const*, long)", "logprob"), ("void omni::logprob_join_kernel<float, true>(float const*, long)", "logprob"),
    ("void omni::logprob_backward_kernel<unsigned short, 256, true>(unsigned short const*, long)", "logprob"),
    ("void omni::row_parts_kernel<unsigned short, 4, 1, true>(unsigned short const*, long)", "row_parts"),
    ("void omni::distill_loss_kernel<float, 64, 0>(float const*, long)", "distill"), ("void omni::distill_join_kernel<float, 3>(float const*, long)", "distill"),
    ("void omni::distill_both_kernel<float, 64, 4, 4>(float const*, long)", "distill"), ("void omni::distill_backward_kernel<float, 256, 0>(float const*, long)", "distill"),
    ("void omni::lrn_forward_kernel<float>(float const*)", "lrn"), ("void at::native::vectorized_elementwise_kernel<4>(int)", None)])
def test_every_kernel_has_its_class_in_the_tables(name, cls):
    from paper_1606_04487_amd.rocprof_tables import kernel_class
    assert kernel_class(name) == cls
