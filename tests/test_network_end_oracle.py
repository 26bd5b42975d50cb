"""The 64-bit functions that the kernels at the end of a network are compared with, pinned on the CPU: by torch's routines and
their automatic gradients in 64 bits, by central differences, and by closed forms."""
import numpy as np
import pytest
import torch

from oracle import network_end as ne


def rng_rows(seed, *shape, sigma=2.0):
    return np.random.default_rng(seed).standard_normal(shape) * sigma


@pytest.mark.parametrize("rows,width", [(1, 1), (3, 2), (4, 7), (5, 64)])
@pytest.mark.parametrize("affine", [False, True])
def test_layer_norm_is_torchs_and_its_gradient(rows, width, affine):
    x, dy = rng_rows(1, rows, width) + 0.5, rng_rows(2, rows, width)
    gamma, beta = (rng_rows(3, width), rng_rows(4, width)) if affine else (None, None)
    xt = torch.tensor(x, requires_grad=True)
    gt, bt = (torch.tensor(v, requires_grad=True) if affine else None for v in (gamma, beta))
    yt = torch.nn.functional.layer_norm(xt, (width,), gt, bt, 1e-5)
    yt.backward(torch.tensor(dy))
    y, mean, rstd = ne.layer_norm_forward(x, gamma, beta, 1e-5)
    np.testing.assert_allclose(y, yt.detach().numpy(), rtol=1e-11, atol=1e-11)
    dx, dgamma, dbeta = ne.layer_norm_backward(x, dy, mean, rstd, gamma)
    np.testing.assert_allclose(dx, xt.grad.numpy(), rtol=1e-8, atol=1e-9)
    if affine:
        np.testing.assert_allclose(dgamma, gt.grad.numpy(), rtol=1e-10, atol=1e-10)
        np.testing.assert_allclose(dbeta, bt.grad.numpy(), rtol=1e-10, atol=1e-10)


def test_layer_norm_gradient_by_differences():
    x, dy, gamma = rng_rows(5, 3, 6), rng_rows(6, 3, 6), rng_rows(7, 6)
    _, mean, rstd = ne.layer_norm_forward(x, gamma)
    dx, _, _ = ne.layer_norm_backward(x, dy, mean, rstd, gamma)
    for i in np.ndindex(x.shape):
        up, down = x.copy(), x.copy()
        up[i] += 1e-5
        down[i] -= 1e-5
        fd = ((ne.layer_norm_forward(up, gamma)[0] - ne.layer_norm_forward(down, gamma)[0]) * dy).sum() / 2e-5
        assert abs(fd - dx[i]) < 1e-6


@pytest.mark.parametrize("temperature", [1.0, 0.5, 3.0])
def test_logprob_is_torchs_and_its_gradient(temperature):
    x = rng_rows(8, 6, 11)
    x[1, 3] = x[2, 0] = -np.inf
    targets = np.array([[0, 0, 5], [1, 2, 4], [-1, 10, 10], [-100, -1, -7], [3, 4, 5], [6, 6, 6]])
    dlp, dh = rng_rows(9, 6, 3), rng_rows(10, 6)
    xt = torch.tensor(x, requires_grad=True)
    lp = torch.log_softmax(xt / temperature, 1)
    picked = torch.where(torch.tensor(targets) >= 0, lp.gather(1, torch.tensor(targets).clamp(min=0)), 0.0)
    p = lp.exp()
    h = -(p * torch.where(p > 0, lp, 0.0)).sum(1)
    ((picked * torch.tensor(dlp)).sum() + (h * torch.tensor(dh)).sum()).backward()
    got, entropy, index, best = ne.logprob_forward(x, targets, 4, temperature)
    np.testing.assert_allclose(got, picked.detach().numpy(), rtol=1e-12, atol=1e-12)
    np.testing.assert_allclose(entropy, h.detach().numpy(), rtol=1e-12)
    tv, ti = lp.topk(4, dim=1)
    np.testing.assert_allclose(best, tv.detach().numpy(), rtol=1e-12)
    assert np.array_equal(index, ti.numpy())
    grad = ne.logprob_backward(x, targets, dlp, dh, temperature)
    ref = xt.grad.numpy()
    possible = np.isfinite(x)
    np.testing.assert_allclose(grad[possible], ref[possible], rtol=1e-9, atol=1e-12)


def test_logprob_out_of_the_ordinary():
    x = np.array([[-np.inf] * 4, [1.0, 1.0, 1.0, 1.0], [1.0, np.nan, 2.0, -np.inf], [0.0, np.inf, 2.0, 1.0], [2.0, -np.inf, 2.0, 5.0]])
    lp, h, index, best = ne.logprob_forward(x, np.array([[0, 9]] * 5), 3)
    assert lp[0, 0] == -np.inf and h[0] == 0 and (index[0] == -1).all() and (best[0] == -np.inf).all()
    assert abs(h[1] - np.log(4)) < 1e-15 and index[1].tolist() == [0, 1, 2]            # ties: the lowest index
    assert np.isnan(lp[2, 0]) and np.isnan(h[2]) and index[2].tolist() == [2, 0, -1]
    assert np.isnan(lp[3, 0]) and index[3].tolist() == [1, 2, 3]
    assert index[4].tolist() == [3, 0, 2] and np.isnan(lp[:, 1]).all()
    g = ne.logprob_backward(x, np.array([[0]] * 5), np.ones((5, 1)))
    assert (g[0] == 0).all() and np.isnan(g[2]).all()


@pytest.mark.parametrize("temperature,alpha", [(1.0, 1.0), (2.0, 0.6), (4.0, 0.0), (1.0, 0.5)])
def test_distill_is_torchs_and_its_gradient(temperature, alpha):
    x, t = rng_rows(11, 5, 9), rng_rows(12, 5, 3)
    index = np.array([[0, 4, 8], [1, -1, 2], [3, 3, 5], [-1, -1, -1], [7, 6, 5]])
    t[4, 1] = -np.inf
    labels, w = np.array([0, 8, -1, 4, -100]), np.array([1.0, 0.5, 2.0, 0.25, 3.0])
    xt = torch.tensor(x, requires_grad=True)
    total, rows = 0.0, []
    for r in range(5):
        there = [k for k in range(3) if index[r, k] >= 0 and t[r, k] > -np.inf]
        loss = torch.zeros((), dtype=torch.float64)
        if there:
            target = torch.zeros(9, dtype=torch.float64)
            q = torch.softmax(torch.tensor(t[r, there]) / temperature, 0)
            lnp = torch.log_softmax(xt[r] / temperature, 0)
            for k, qk in zip(there, q):
                loss = loss + alpha * temperature ** 2 * qk * (qk.log() - lnp[index[r, k]])
        if labels[r] >= 0:
            loss = loss + (1 - alpha) * torch.nn.functional.cross_entropy(xt[r:r + 1], torch.tensor(labels[r:r + 1]))
        rows.append(loss.item())
        total = total + w[r] * loss
    total.backward()
    loss, grad = ne.distill(x, index, t, labels, temperature, alpha, w)
    np.testing.assert_allclose(loss, rows, rtol=1e-11, atol=1e-13)
    np.testing.assert_allclose(grad, xt.grad.numpy(), rtol=1e-9, atol=1e-12)


def test_distill_gradient_by_differences():
    x, t, index, labels = rng_rows(13, 2, 5), rng_rows(14, 2, 2), np.array([[0, 3], [2, 2]]), np.array([1, 4])
    _, grad = ne.distill(x, index, t, labels, 3.0, 0.3)
    for i in np.ndindex(x.shape):
        up, down = x.copy(), x.copy()
        up[i] += 1e-5
        down[i] -= 1e-5
        fd = (ne.distill(up, index, t, labels, 3.0, 0.3)[0].sum() - ne.distill(down, index, t, labels, 3.0, 0.3)[0].sum()) / 2e-5
        assert abs(fd - grad[i]) < 1e-7


def test_distill_closed_forms():
    x = rng_rows(15, 4, 6)
    # a teacher that keeps every class with the student's own logits: no loss, no gradient
    loss, grad = ne.distill(x, np.tile(np.arange(6), (4, 1)), x, None, 2.0, 1.0)
    assert np.abs(loss).max() < 1e-13 and np.abs(grad).max() < 1e-14
    # log probabilities in place of logits: the same
    lp = np.array([ne.log_softmax_row(v) for v in x])
    a, b = ne.distill(x[::-1], np.tile(np.arange(6), (4, 1)), x, None, 2.0), ne.distill(x[::-1], np.tile(np.arange(6), (4, 1)), lp, None, 2.0)
    np.testing.assert_allclose(a[0], b[0], rtol=1e-12)
    # uniform logits: cross entropy ln n
    loss, _ = ne.distill(np.zeros((1, 6)), None, None, np.array([2]), 5.0, 0.0)
    assert abs(loss[0] - np.log(6)) < 1e-15
    loss, grad = ne.distill(np.full((1, 3), -np.inf), np.array([[1]]), np.zeros((1, 1)), None)
    assert loss[0] == np.inf and (grad == 0).all()
