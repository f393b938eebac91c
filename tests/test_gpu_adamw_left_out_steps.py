"""layers.AdamW where a step is left out because its gradients' norm is no finite number: what follows is as if it had not been asked for, the count of steps among it."""
import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_1906_03707_amd import binding
    binding.lib()
    return binding


def start(gen):
    return [torch.randn(33, 20, device="cuda", generator=gen), torch.randn(7, device="cuda", generator=gen)]


def same(a, b):
    return all(torch.equal(p.detach(), q.detach()) for p, q in zip(a.params, b.params)) and all(
        torch.equal(s.view(torch.uint8), t.view(torch.uint8)) for k in a.states for s, t in zip(a.states[k], b.states[k]))


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("when", ["x.", "xx..x.", ".x.x", "..x", "x.n.x.n"])
def test_steps_after_one_that_was_left_out(B, when, bad, bits):
    """x: a step whose gradients are no numbers; n: one without clipping.  The other optimiser never hears of the x."""
    from paper_1906_03707_amd import layers
    gen = torch.Generator(device="cuda").manual_seed(len(when))
    first = start(gen)
    ours, plain = (layers.AdamW([p.clone().requires_grad_() for p in first], lr=0.01, weight_decay=0.1, bits=bits, seed=3) for _ in range(2))
    done = 0
    for kind in when:
        grads = [torch.randn(p.shape, device="cuda", generator=gen) for p in first]
        for opt in (ours, plain):
            for p, g in zip(opt.params, grads):
                p.grad = g.clone()
        if kind == "x":
            ours.params[1].grad[3] = bad
            assert not bool(ours.step(max_norm=1.0).isfinite())
        else:
            limit = 1.0 if kind == "." else None
            ours.step(max_norm=limit)
            plain.step(max_norm=limit)
            done += 1
        assert ours.steps == plain.steps == done and same(ours, plain)
    # saved and loaded in another, the count goes along
    other = layers.AdamW([p.detach().clone().requires_grad_() for p in ours.params], lr=0.01, weight_decay=0.1, bits=bits)
    other.load_state_dict(ours.state_dict())
    assert isinstance(ours.state_dict()["steps"], int) and other.steps == done
    for opt in (ours, other):
        for p, g in zip(opt.params, grads):
            p.grad = g.clone()
        opt.step(max_norm=0.5)
    assert same(ours, other) and ours.steps == other.steps == done + 1


def test_first_update_after_an_overflow(B):
    """Against the formulas: with betas of 0.9 and 0.999 the first step moves a parameter by lr, also after ten that were left out."""
    from paper_1906_03707_amd import layers
    p = torch.zeros(100, device="cuda", requires_grad=True)
    opt = layers.AdamW([p], lr=0.5, weight_decay=0.0)
    for _ in range(10):
        p.grad = torch.full((100,), math.inf, device="cuda")
        opt.step(max_norm=1.0)
    p.grad = torch.ones(100, device="cuda")
    opt.step(max_norm=1.0)
    # gradients of 0.1 after clipping: lr * 0.1 / (0.1 + 1e-8), with some twenty roundings
    assert bool(((p.detach().double() + 0.5 * 0.1 / (0.1 + 1e-8)).abs() <= 0.5 * 24 * 2.0 ** -24).all())


def test_count_may_be_set_and_a_failed_call_does_not_count(B):
    from paper_1906_03707_amd import layers
    p = torch.zeros(8, device="cuda", requires_grad=True)
    opt = layers.AdamW([p], lr=0.1)
    opt.steps = 4
    p.grad = torch.ones(8, device="cuda")
    opt.step(max_norm=1.0)
    assert opt.steps == 5
    opt.lr = math.nan
    with pytest.raises(B.HagError):
        opt.step(max_norm=1.0)
    with pytest.raises(B.HagError):
        opt.step()
    assert opt.steps == 5


def test_steps_on_two_streams(B):
    """Steps in turn on two streams, each waiting for the one before, while the other stream goes on with work of its own: the count's memory is not given to that."""
    from paper_1906_03707_amd import layers
    gen = torch.Generator(device="cuda").manual_seed(4)
    first = start(gen)
    ours, plain = (layers.AdamW([p.clone().requires_grad_() for p in first], lr=0.01, weight_decay=0.1) for _ in range(2))
    streams, places = [torch.cuda.current_stream(), torch.cuda.Stream()], set()
    grads = [[torch.randn(p.shape, device="cuda", generator=gen) for p in first] for _ in range(6)]
    busy = torch.ones(1 << 24, device="cuda")
    for k, gs in enumerate(grads):
        if k == 3:
            gs[0][0, 0] = math.inf
        for p, q, g in zip(ours.params, plain.params, gs):
            p.grad, q.grad = g.clone(), g.clone()
        here, other = streams[k % 2], streams[1 - k % 2]
        here.wait_stream(other)
        with torch.cuda.stream(here):
            for _ in range(10):
                busy.mul_(1.0)
            ours.step(max_norm=1.0)
            places.add(ours._count.data_ptr())
        with torch.cuda.stream(other):
            for _ in range(20):
                torch.full((), -7, dtype=torch.int64, device="cuda")
        torch.cuda.synchronize()
        if k != 3:
            plain.step(max_norm=1.0)
    assert same(ours, plain) and ours.steps == plain.steps == 5 and len(places) == 2
