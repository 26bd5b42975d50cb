"""A stack with layer norm, trained on the distillation loss and asked for its log probabilities, against torch's automatic
gradients in 64 bits on the CPU.  Products and sums here have at most 2000 terms: in fp32 a result is off by at most 2000 u = 1.2e-4
of the sum of its terms' magnitudes, which 1e-4 of the largest value covers where terms cancel no more than they do here (as the
other fp32 tests of whole passes have it); in bf16 every stored value is a rounding of 2^-8, a few of them one behind the other."""
import numpy as np
import pytest
import torch

from paper_1606_04487_amd import workloads as wl

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_1606_04487_amd import binding
    assert torch.cuda.is_available()
    return binding


N, CLASSES = 12, 37
LAYERS = [wl.ConvLayer("conv", N, 3, 9, 9, 16, 3, 1, 1, norm_after=True),
          wl.ConvLayer("fc", N, 16, 9, 9, 24, 9, 1, 0, norm_after=True),
          wl.ConvLayer("out", N, 24, 1, 1, CLASSES, 1, 1, 0, relu=False)]


def parameters(seed):
    g = np.random.default_rng(seed)
    return ([g.standard_normal((L.F, L.C, L.k, L.k)).astype(np.float32) * (2.0 / L.K) ** 0.5 for L in LAYERS],
            [g.standard_normal(L.F).astype(np.float32) * 0.1 for L in LAYERS])


def reference(X, Ws, bs, norms, index, values, labels, temperature, alpha):
    """(logits, loss per image, gradients of the mean loss) in 64 bits."""
    Ws, bs = ([torch.tensor(np.asarray(v), dtype=torch.float64, requires_grad=True) for v in vs] for vs in (Ws, bs))
    ga, be = ([torch.tensor(np.asarray(v), dtype=torch.float64, requires_grad=True) for v in vs] for vs in zip(*norms))
    cur = torch.tensor(X, dtype=torch.float64)
    for i, L in enumerate(LAYERS):
        cur = torch.nn.functional.conv2d(cur, Ws[i], bs[i], L.s, L.p)
        if L.relu:
            cur = torch.relu(cur)
        if L.norm_after:
            shape = cur.shape
            flat = cur.reshape(N, -1)
            cur = torch.nn.functional.layer_norm(flat, flat.shape[1:], ga[i], be[i], 1e-5).reshape(shape)
    logits = cur.reshape(N, -1)
    lp, lp1 = torch.log_softmax(logits / temperature, 1), torch.log_softmax(logits, 1)
    q = torch.softmax(torch.tensor(values, dtype=torch.float64) / temperature, 1)
    at, lab = torch.tensor(index), torch.tensor(labels)
    loss = alpha * temperature ** 2 * (q * (q.log() - lp.gather(1, at))).sum(1) + (1 - alpha) * -lp1.gather(1, lab[:, None])[:, 0]
    loss.mean().backward()
    grads = {"W": [w.grad.numpy() for w in Ws], "b": [b.grad.numpy() for b in bs], "gamma": [g.grad.numpy() for g in ga], "beta": [b.grad.numpy() for b in be]}
    return logits.detach().numpy(), loss.detach().numpy(), grads


def close(got, ref, limit, what):
    got = got.detach().double().cpu().numpy().reshape(ref.shape)
    assert np.max(np.abs(got - ref)) <= limit * max(np.max(np.abs(ref)), 1e-30), (what, np.max(np.abs(got - ref)) / np.max(np.abs(ref)))


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("temperature,alpha", [(2.0, 0.5), (1.0, 1.0)])
def test_distill_step_of_a_stack_with_layer_norm(B, temperature, alpha, dtype):
    from paper_1606_04487_amd.stack import ConvStack
    g = np.random.default_rng(7)
    net, teacher = (ConvStack(LAYERS, dtype=dtype, skip_first_dgrad=True) for _ in range(2))
    X = g.standard_normal((N, 3, 9, 9)).astype(np.float32)
    Ws, bs = parameters(1)
    if dtype == 1:
        X, Ws = wl.to_bf16_values(X), [wl.to_bf16_values(w) for w in Ws]
    net.set_parameters(Ws, bs)
    teacher.set_parameters(*parameters(2))
    for m in net.norms:
        if m is not None:
            m.gamma.copy_(torch.from_numpy(1 + 0.2 * g.standard_normal(m.gamma.numel())))
            m.beta.copy_(torch.from_numpy(0.2 * g.standard_normal(m.beta.numel())))
    norms = [(m.gamma.cpu().numpy(), m.beta.cpu().numpy()) for m in net.norms if m is not None]
    Xg = torch.from_numpy(X).cuda().to(B.torch_dtype(dtype))
    _, _, index, values = teacher.log_probs(Xg, top=6)
    labels = index[:, 0].clone()
    logits, loss, grads = reference(X, Ws, bs, norms, index.cpu().numpy(), values.cpu().numpy(), labels.cpu().numpy(), temperature, alpha)
    before = [w.clone() for w in net.W + net.b + [p for m in net.norms if m is not None for p in (m.gamma, m.beta)]]
    got = net.distill_step(Xg, index, values, labels, 0.25, 0.5, temperature=temperature, alpha=alpha)
    # bf16: 2^-8 for each of about eight roundings between the image and a gradient, some of them enlarged by the layers behind
    limit = 1e-4 if dtype == 0 else 0.06
    close(got, loss, limit, "loss")
    kept = [m for m in net.norms if m is not None]
    for i in range(3):
        close(net.dW[i], grads["W"][i], limit, ("dW", i))
        close(net.db[i], grads["b"][i], limit, ("db", i))
    for i, m in enumerate(kept):
        close(m.dgamma, grads["gamma"][i], limit, ("dgamma", i))
        close(m.dbeta, grads["beta"][i], limit, ("dbeta", i))
    # the update, V = -lr G and W += V, in fp32
    after = net.W + net.b + [p for m in kept for p in (m.gamma, m.beta)]
    for w0, w1, d in zip(before, after, net.dW + net.db + [d for m in kept for d in (m.dgamma, m.dbeta)]):
        assert torch.allclose(w1, w0 - 0.25 * d, rtol=1e-6, atol=1e-7)
    weights, biases = [w.float().cpu().numpy() for w in net.Wc], [b.cpu().numpy() for b in net.b]
    norms = [(m.gamma.cpu().numpy(), m.beta.cpu().numpy()) for m in kept]
    again = reference(X, weights, biases, norms, index.cpu().numpy(), values.cpu().numpy(), labels.cpu().numpy(), temperature, alpha)[0]
    close(net.logits(net.forward(Xg)), again, limit, "logits after the step")
    net.set_parameters(Ws, bs)
    assert all(bool((m.gamma == 1).all()) and not bool(m.beta.any()) and not bool(m.vgamma.any()) for m in kept)


def test_log_probs_leave_dropout_out(B):
    from dataclasses import replace
    from paper_1606_04487_amd.stack import ConvStack
    plain = ConvStack(LAYERS, dtype=0)
    dropped = ConvStack([replace(LAYERS[0], dropout_after=0.5)] + LAYERS[1:], dtype=0)
    Ws, bs = parameters(3)
    plain.set_parameters(Ws, bs)
    dropped.set_parameters(Ws, bs)
    X = torch.randn(N, 3, 9, 9, device="cuda")
    t = torch.randint(0, CLASSES, (N,), device="cuda")
    a, b = plain.log_probs(X, t, top=4, temperature=1.5), dropped.log_probs(X, t, top=4, temperature=1.5)
    assert all(torch.equal(p, q) for p, q in zip(a, b))
    assert not torch.equal(plain.forward(X), dropped.forward(X))
    full = torch.log_softmax(plain.logits(plain.forward(X)).double() / 1.5, 1)
    assert float((a[0] - full.gather(1, t[:, None])[:, 0]).abs().max()) < 1e-5
    assert torch.equal(a[2], full.topk(4, dim=1).indices)


def test_distill_step_captured_and_replayed(B):
    from paper_1606_04487_amd.stack import ConvStack
    Ws, bs = parameters(4)
    X = torch.randn(N, 3, 9, 9, device="cuda").bfloat16()
    labels = torch.randint(0, CLASSES, (N,), device="cuda")
    index = torch.randint(0, CLASSES, (N, 5), device="cuda")
    values = torch.randn(N, 5, device="cuda")
    nets = [ConvStack(LAYERS, dtype=1) for _ in range(2)]
    for net in nets:
        net.set_parameters(Ws, bs)
        net.distill_step(X, index, values, labels, 0.1, 0.9, temperature=2.0, alpha=0.5)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        nets[0].distill_step(X, index, values, labels, 0.1, 0.9, temperature=2.0, alpha=0.5)
    for i in range(3):
        X.add_(0.125)
        torch.cuda.synchronize()
        graph.replay()
        nets[1].distill_step(X, index, values, labels, 0.1, 0.9, temperature=2.0, alpha=0.5)
        torch.cuda.synchronize()
        for a, b in zip(nets[0].W + nets[0].b + [nets[0].loss] + [m.gamma for m in nets[0].norms if m is not None],
                        nets[1].W + nets[1].b + [nets[1].loss] + [m.gamma for m in nets[1].norms if m is not None]):
            assert torch.equal(a, b)


def test_backward_of_a_pass_without_dropout(B):
    """After forward(train=False) backward is the gradient of that pass: nothing was dropped."""
    from dataclasses import replace
    from paper_1606_04487_amd.stack import ConvStack
    plain, dropped = ConvStack(LAYERS, dtype=0), ConvStack([replace(LAYERS[0], dropout_after=0.5)] + LAYERS[1:], dtype=0)
    Ws, bs = parameters(5)
    X, d = torch.randn(N, 3, 9, 9).cuda(), torch.randn(N, CLASSES, 1, 1).cuda()
    for net in (plain, dropped):
        net.set_parameters(Ws, bs)
        net.forward(X, train=False)
        net.backward(d)
    assert all(torch.equal(a, b) for a, b in zip(plain.dW + plain.db, dropped.dW + dropped.db))
    dropped.forward(X)
    dropped.backward(d)
    assert not torch.equal(plain.dW[0], dropped.dW[0])


def test_answers_between_the_two_passes_of_a_step(B):
    """log_probs uses the buffers that backward reads: a backward pass behind it would be of the answered batch."""
    from paper_1606_04487_amd.stack import ConvStack
    net = ConvStack(LAYERS, dtype=0)
    net.set_parameters(*parameters(6))
    X, other, d = torch.randn(N, 3, 9, 9).cuda(), torch.randn(N, 3, 9, 9).cuda(), torch.randn(N, CLASSES, 1, 1).cuda()
    net.forward(X)
    net.backward(d)
    want = [w.clone() for w in net.dW + net.db]
    net.forward(X)
    net.log_probs(other)
    with pytest.raises(RuntimeError):
        net.backward(d)
    net.log_probs(other)
    net.forward(X)
    net.backward(d)
    assert all(torch.equal(a, b) for a, b in zip(net.dW + net.db, want))
    net.distill_step(X, None, None, torch.zeros(N, dtype=torch.int64, device="cuda"), 0.1, 0.9, alpha=0.0)
