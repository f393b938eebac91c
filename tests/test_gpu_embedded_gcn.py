"""Lookup, layer norm and clipping under autograd, and the training step that runs them with the aggregation: against the same model in 64 bits."""
import os
import sys

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def B():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_1906_03707_amd import binding
    binding.lib()
    return binding


def near(got, want, tol):
    return (got.double() - want.double()).norm().item() <= tol * want.double().norm().item()


def model64(rowptr, col, ids, params, labels, padding):
    """embedded_gcn2_loss with a dense matrix (A + I) / (degree + 1), in 64 bits."""
    table, w, b, w1, w2 = params
    n = rowptr.size - 1
    adj = np.eye(n)
    for v in range(n):
        adj[v, col[rowptr[v]:rowptr[v + 1]]] += 1
    adj = torch.from_numpy(adj / (np.diff(rowptr) + 1)[:, None]).cuda()
    x = table[ids.clamp(min=0)] * table.shape[1] ** 0.5
    x = torch.where((ids == padding)[:, None], 0.0, x)
    x = torch.nn.functional.layer_norm(x, (x.shape[1],), w, b, 1e-5)
    return torch.nn.functional.cross_entropy(adj @ (torch.relu(adj @ (x @ w1)) @ w2), labels)


def make(B, d=20, rows=37, seed=0):
    from paper_1906_03707_amd import synth
    rowptr, col = synth.sbm(6, 40, 0.3, 0.01, seed=11)
    n = rowptr.size - 1
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rnd = lambda *s: torch.randn(*s, device="cuda", generator=gen)   # noqa: E731
    params = [rnd(rows, d) * d ** -0.5, 1 + 0.1 * rnd(d), 0.1 * rnd(d), rnd(d, 16) * d ** -0.5, rnd(16, 8) * 0.25]
    ids = torch.randint(-1, rows, (n,), device="cuda", generator=gen)
    labels = torch.randint(0, 8, (n,), device="cuda", generator=gen)
    labels[::5] = -100
    return rowptr, col, B.hag_search(rowptr, col, n // 4).upload(), params, ids, labels


@pytest.mark.parametrize("d", [20, 64])
def test_loss_and_gradients(B, d):
    from paper_1906_03707_amd import layers
    rowptr, col, h, params, ids, labels = make(B, d)
    ours = [p.clone().requires_grad_() for p in params]
    ref = [p.double().requires_grad_() for p in params]
    loss, want = layers.embedded_gcn2_loss(h, ids, *ours, labels, padding=-1), model64(rowptr, col, ids, ref, labels, -1)
    assert abs(loss.item() - want.item()) <= 1e-5 * want.item()                    # the bars of the layer tests
    loss.backward()
    want.backward()
    for p, q in zip(ours, ref):
        assert near(p.grad, q.grad, 1e-4)
    assert not bool(ours[0].grad[~torch.isin(torch.arange(37, device="cuda"), ids)].any())


def test_step_clips_and_descends(B):
    from paper_1906_03707_amd import layers
    rowptr, col, h, params, ids, labels = make(B)
    ours = [p.clone().requires_grad_() for p in params]
    ref = [p.double().requires_grad_() for p in params]
    for _ in range(3):
        loss, norm = layers.embedded_gcn2_step(h, ids, ours, labels, lr=0.5, max_norm=0.05, padding=-1)
        want = model64(rowptr, col, ids, ref, labels, -1)
        grads = torch.autograd.grad(want, ref)
        size = torch.sqrt(sum(g.square().sum() for g in grads)).item()
        with torch.no_grad():
            for p, g in zip(ref, grads):
                p -= 0.5 * g * min(1.0, 0.05 / size)
        assert abs(loss.item() - want.item()) <= 1e-4 * want.item() and abs(norm.item() - size) <= 1e-3 * size
        clipped = torch.sqrt(sum(p.grad.double().square().sum() for p in ours)).item()
        assert size > 0.05 and abs(clipped - 0.05) <= 1e-6
    for p, q in zip(ours, ref):
        assert near(p.detach(), q.detach(), 1e-5)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_under_autograd(B, dtype):
    from paper_1906_03707_amd import layers
    gen = torch.Generator(device="cuda").manual_seed(1)
    table = torch.randn(30, 12, device="cuda", generator=gen).to(dtype)
    w, b = torch.randn(12, device="cuda", generator=gen), torch.randn(12, device="cuda", generator=gen)
    ids = torch.randint(0, 30, (4, 7), device="cuda", generator=gen)
    tol = 1e-5 if dtype == torch.float32 else 2e-2

    def run(lookup, norm, cast):
        t, ww, bb = (cast(p).requires_grad_() for p in (table, w, b))
        y = norm(lookup(t, ids), ww, bb)
        # the gradients that reach the norm are broadcast and transposed ones
        return y, torch.autograd.grad(y.sum() + (y.transpose(0, 2) * torch.arange(7, device="cuda")[:, None]).float().sum() + (y.float() ** 2).sum(), (t, ww, bb))

    y, grads = run(lambda t, i: layers.embedding(t, i, 2.0), layers.layer_norm, lambda p: p.clone())
    want, ref = run(lambda t, i: 2 * t[i], lambda x, ww, bb: torch.nn.functional.layer_norm(x, (12,), ww, bb), lambda p: p.double())
    assert y.shape == (4, 7, 12) and y.dtype == dtype and near(y.detach(), want.detach(), tol)
    for g, r in zip(grads, ref):
        assert near(g, r, 4 * tol)
    x = table.clone().requires_grad_()
    layers.layer_norm(x[:, :5]).sum().backward()           # a view, a broadcast gradient
    assert x.grad.shape == x.shape and not bool(x.grad[:, 5:].any())
    y = layers.layer_norm(x, w.requires_grad_(), None)
    y.float().sum().backward()
    assert w.grad.shape == (12,)
    with pytest.raises(RuntimeError):                                              # not twice
        g, = torch.autograd.grad(layers.layer_norm(x).float().square().sum(), x, create_graph=True)
        torch.autograd.grad(g.float().sum(), x)


def test_clipping_of_parameters(B):
    from paper_1906_03707_amd import layers
    params = [torch.ones(5, 4, device="cuda", requires_grad=True), torch.ones(3, device="cuda", requires_grad=True), torch.ones(2, device="cuda", requires_grad=True)]
    (3 * params[0].sum() + 4 * params[1].sum()).backward()
    norm = layers.clip_gradients(params, 1.0)
    assert params[2].grad is None and abs(norm.item() - (9 * 20 + 16 * 3) ** 0.5) <= 1e-5
    assert abs((params[0].grad.square().sum() + params[1].grad.square().sum()).item() - 1) <= 1e-6
    assert layers.clip_gradients([params[2]], 1.0).item() == 0


def test_example(B):
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    try:
        import embedded_gcn
    finally:
        sys.path.pop(0)
    loss, accuracy = embedded_gcn.main(["--blocks", "8", "--block", "48", "--steps", "60"])
    assert loss < 0.5 and accuracy > 0.8
