"""hag_clip_gradients against 64-bit sums: one tensor to more than one launch holds, types and addresses mixed, in place and into other tensors, norms out of fp32's range."""
import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
EPS = 2.0 ** -24
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TINY = {torch.float32: 2.0 ** -150, torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25}
TYPES = [torch.float32, torch.bfloat16, torch.float16]


@pytest.fixture(scope="module")
def B():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_1906_03707_amd import binding
    binding.lib()
    return binding


def norm64(tensors):
    return math.sqrt(sum(t.double().square().sum().item() for t in tensors))


def check(norm, outs, tensors, max_norm):
    want = norm64(tensors)
    assert norm.dtype == torch.float32 and norm.shape == ()
    assert abs(norm.item() - want) <= 2 * EPS * want                               # 64-bit sums, rounded once
    scale = 1.0 if want <= max_norm else max_norm / want
    for o, t in zip(outs, tensors):
        exact = t.double() * scale
        # the factor and the product are rounded in fp32, the result to its type
        assert bool(((o.double() - exact).abs() <= (3 * EPS + HALF[t.dtype]) * exact.abs() * (1 + 1e-3) + TINY[t.dtype]).all())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("counts", [[1], [3], [5, 4, 0, 1], [63, 64, 65], [4095, 4096, 4097], [100000], [7, 1000003, 9], [2500000, 1, 2, 3, 12345], list(range(1, 40)), [17] * 700, [9000] * 300])
def test_clip(B, counts, dtype):
    gen = torch.Generator(device="cuda").manual_seed(len(counts))
    flat = torch.randn(sum(counts) + 1, device="cuda", generator=gen).to(dtype)
    for start in (0, 1):                                   # end to end in one buffer: pieces begin anywhere
        tensors = list(torch.split(flat[start:start + sum(counts)], counts))
        size = norm64(tensors)
        for max_norm in (0.3 * size, 1.7 * size, math.inf):
            into = [torch.full_like(t, 7.0) for t in tensors]
            norm = B.clip_gradients(tensors, max_norm, out=into)
            check(norm, into, tensors, max_norm)
            if max_norm > size:
                assert all(torch.equal(o, t) for o, t in zip(into, tensors))
            mine = torch.cat([flat.new_full((start,), 5.0), *tensors, flat.new_full((9,), 5.0)])
            again = B.clip_gradients(list(torch.split(mine[start:start + sum(counts)], counts)), max_norm)
            assert torch.equal(again, norm) and torch.equal(mine[start:-9], torch.cat(into))               # in place: the same bits
            assert bool((mine[:start] == 5).all()) and bool((mine[-9:] == 5).all())


def test_mixed_types_and_layouts(B):
    gen = torch.Generator(device="cuda").manual_seed(3)
    rnd = lambda *s: torch.randn(*s, device="cuda", generator=gen)   # noqa: E731
    tensors = [rnd(40, 30).bfloat16(), rnd(7, 9).t(), rnd(3, 5, 7).permute(2, 0, 1).half(), rnd(()), rnd(1, 6)[:, ::1], rnd(0, 4), rnd(50000).half()[1:], rnd(8, 1).expand(8, 1)]
    check(B.clip_gradients(tensors, 2.5, out=(into := [torch.empty_like(t) for t in tensors])), into, tensors, 2.5)
    copies = [t.clone() for t in tensors]
    B.clip_gradients(copies, 2.5)
    assert all(torch.equal(a, b) for a, b in zip(copies, into))
    assert torch.equal(B.clip_gradients(iter(tensors), math.inf), B.clip_gradients(tensors, 1e9, out=into))


def test_norms_out_of_range(B):
    for value, dtype in ((1e30, torch.float32), (1e-30, torch.float32), (3e38, torch.bfloat16), (6e4, torch.float16), (2.0 ** -140, torch.float32)):
        t = torch.full((3000,), value, device="cuda").to(dtype)
        want = t[0].double().item() * math.sqrt(3000)
        into = [torch.empty_like(t)]
        norm = B.clip_gradients([t], want / 4, out=into).item()
        assert norm == math.inf if want > 3.4028236e38 else abs(norm - want) <= 2 * EPS * want + 2.0 ** -150
        assert bool(((into[0].double() - t.double() / 4).abs() <= (HALF[dtype] + 3 * EPS) * t.double() / 4 + TINY[dtype]).all())
    zero = torch.zeros(10, device="cuda")
    assert B.clip_gradients([zero], 1.0).item() == 0 and not bool(zero.any())


def test_what_is_no_number(B):
    for bad in (float("nan"), float("inf"), float("-inf")):
        tensors = [torch.ones(5000, device="cuda"), torch.ones(9, device="cuda").bfloat16()]
        tensors[0][4321] = bad
        norm = B.clip_gradients(tensors, 1.0).item()
        if math.isnan(bad):
            assert math.isnan(norm) and all(bool(torch.isnan(t).all()) for t in tensors)
        else:
            assert norm == math.inf and math.isnan(tensors[0][4321].item()) and not bool(tensors[1].any())
            assert not bool(tensors[0][:4321].any()) and not bool(tensors[0][4322:].any())


def test_past_32_bits(B):
    t = torch.zeros(2 ** 31 + 5000, device="cuda", dtype=torch.bfloat16)
    t[-1], t[2 ** 31 + 1], t[0] = 3, 4, 12
    assert B.clip_gradients([t], 6.5).item() == 13
    assert (t[-1].item(), t[2 ** 31 + 1].item(), t[0].item()) == (1.5, 2, 6) and t.count_nonzero().item() == 3


def test_nothing(B):
    assert B.clip_gradients([], 1.0).item() == 0
    assert B.clip_gradients([torch.zeros(0, 3, device="cuda")], 1.0).item() == 0


def test_on_another_stream_and_captured(B):
    gen = torch.Generator(device="cuda").manual_seed(4)
    flat = torch.randn(300000, device="cuda", generator=gen)
    tensors = list(torch.split(flat, [7, 250000, 49993]))
    into = [torch.empty_like(t) for t in tensors]
    want, first = B.clip_gradients(tensors, 3.0, out=into), [t.clone() for t in into]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = B.clip_gradients(tensors, 3.0, out=into)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got, want) and all(torch.equal(a, b) for a, b in zip(first, into))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = B.clip_gradients(tensors, 3.0)
    for _ in range(4):
        flat.copy_(torch.randn(300000, device="cuda", generator=gen))
        want, before = B.clip_gradients(tensors, 3.0, out=into), norm64(tensors)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(got, want) and all(torch.equal(a, b) for a, b in zip(tensors, into)) and abs(got.item() - before) <= 2 * EPS * before
        torch.cuda.synchronize()


def test_refusals(B):
    t = torch.ones(6, 8, device="cuda")
    for call in (lambda: B.clip_gradients([t.cpu()], 1.0), lambda: B.clip_gradients([t.double()], 1.0), lambda: B.clip_gradients([t[:, :4]], 1.0), lambda: B.clip_gradients([t, t], 1.0),
                 lambda: B.clip_gradients([t], 1.0, out=[]), lambda: B.clip_gradients([t], 1.0, out=[t.half()]), lambda: B.clip_gradients([t], 1.0, out=[t[:5]]),
                 lambda: B.clip_gradients([t.t()], 1.0, out=[torch.ones(8, 6, device="cuda")]), lambda: B.clip_gradients([t[:1].expand(6, 8)], 1.0)):
        with pytest.raises(ValueError):
            call()
    for bad in (0.0, -1.0, float("nan")):
        with pytest.raises(B.HagError) as err:
            B.clip_gradients([t], bad)
        assert err.value.code == B.HAG_EINVAL
    assert bool((t == 1).all())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("count", [5, 3000, 4096, 70001])
def test_factors_below_fp32(B, count, dtype):
    gen = torch.Generator(device="cuda").manual_seed(count)
    z = torch.rand(count, device="cuda", generator=gen) + 0.25
    for large, max_norm in ((3e38, 1.0), (3e38, 1e-3), (3e38, 1e-12), (1e37, 1e-3), (2e38, 1e-30)):
        t = (large * (z - 0.5).clamp(-1, 1)).to(dtype)
        assert norm64([t]) / max_norm > 2.0 ** 126
        into = [torch.empty_like(t)]
        norm = B.clip_gradients([t], max_norm, out=into)
        want = t.double() * (max_norm / norm64([t]))
        assert bool(((into[0].double() - want).abs() <= (3 * EPS + HALF[dtype]) * want.abs() * (1 + 1e-3) + TINY[dtype]).all())     # as any other factor
        again = [t.clone()]
        assert torch.equal(B.clip_gradients(again, max_norm), norm) and torch.equal(again[0], into[0])
    for bad in (float("inf"), float("nan")):
        t[1] = bad
        norm = B.clip_gradients([t], 1.0, out=into).item()
        assert (math.isnan(norm) and bool(torch.isnan(into[0]).all())) if math.isnan(bad) else (norm == math.inf and math.isnan(into[0][1].item()) and int(into[0].count_nonzero()) == 1)
