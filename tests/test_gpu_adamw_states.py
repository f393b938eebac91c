"""hag_adamw's states in 8 bits, element by element, for every pair of types and for steps that are clipped: the formula's products and sums rounded one by one in fp32, the same bits."""
import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
PAIRS = [(F32, F32), (F32, BF16), (F32, F16), (BF16, BF16), (F16, F16)]
HYPER = dict(lr=2e-3, betas=(0.9, 0.99), eps=1e-8, weight_decay=0.05)


@pytest.fixture(scope="module")
def B():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_1906_03707_amd import binding
    binding.lib()
    return binding


def mixed(x):
    x = x & 0xFFFFFFFF
    x = (x ^ (x >> 15)) * 0x6A09E667 & 0xFFFFFFFF
    x = (x ^ (x >> 13)) * 0xBB67AE85 & 0xFFFFFFFF
    return x ^ (x >> 16)


def power(scales):
    return torch.exp2(scales.view(torch.uint8).double() - 127)


def rows(t):
    return torch.nn.functional.pad(t, (0, -t.numel() % 32)).view(-1, 32)


@pytest.mark.parametrize("pair", PAIRS)
@pytest.mark.parametrize("counts", [[1], [5, 31, 32, 33], [4096, 4097, 2047], [2500000, 3, 12345], [1000003] * 5, list(range(1, 60))])
def test_clipped_steps(B, counts, pair):
    gen = torch.Generator(device="cuda").manual_seed(len(counts))
    params = [torch.randn(c, device="cuda", generator=gen).to(pair[0]) for c in counts]
    states = B.adamw_states(params, bits=8)
    for step, limit in ((1, None), (2, 0.3), (3, 1e-3), (7, 5.0), (8, None)):
        grads = [(0.1 * torch.randn(c, device="cuda", generator=gen) * torch.exp(2 * torch.randn(c, device="cuda", generator=gen))).to(pair[1]) for c in counts]
        for g in grads:
            g[::5] = 0
        norm = torch.tensor(3.0, device="cuda")            # clips where the limit is below
        old = {k: [(c.double() * power(s).repeat_interleave(32)[:c.numel()]).float() for c, s in zip(states[k], states[k + "_scales"])] for k in "mv"}
        B.adamw(params, grads, **states, step=step, seed=9, norm=None if limit is None else norm, max_norm=limit, **HYPER)
        factor = 1.0 if limit is None else min(1.0, limit / 3.0)
        for i, g in enumerate(grads):
            count = g.numel()
            g = (g.double() * factor).float()              # (one rounding)
            m = 0.9 * old["m"][i] + (1 - 0.9) * g
            r = torch.sqrt(0.99 * (old["v"][i] * old["v"][i]) + (1 - 0.99) * (g * g))
            x = mixed(torch.arange(count, device="cuda") * 0x9E3779B1 + mixed(torch.tensor(9 + step * 0x9E3779B1, device="cuda")))
            for key, t, random in (("m", m, x & 0xFFFF), ("v", r, x >> 16)):
                s = power(states[key + "_scales"][i])
                most = rows(t.abs()).amax(1).double()
                assert bool(torch.where(most == 0, s == 1, ((448 * s >= most) & (224 * s < most)) | (s == 2.0 ** -127)).all())
                small = (t.abs().double() / s.repeat_interleave(32)[:count]).float() * 2.0 ** -120
                codes = (small.view(torch.int32) + (random * 16 + 8).int()) >> 20
                if key == "v":
                    codes = torch.where(t != 0, codes.clamp(min=1), codes)
                codes = codes | torch.signbit(t).int() << 7
                assert torch.equal(states[key][i].view(torch.uint8).int(), codes)


@pytest.mark.parametrize("limit", [None, 0.3, 1e-3])
def test_first_moments_of_many_elements(B, limit):
    """Against 64 bits, each element by itself: rounding up or down moves it by less than a step, and what fp32 loses is a part of its terms, which may cancel."""
    gen = torch.Generator(device="cuda").manual_seed(1)
    count = 1 << 20
    params, norm = [torch.zeros(count, device="cuda")], torch.tensor(3.0, device="cuda")
    states = B.adamw_states(params, bits=8)
    for step in range(1, 8):
        g = torch.randn(count, device="cuda", generator=gen)
        old = states["m"][0].double() * power(states["m_scales"][0]).repeat_interleave(32)
        B.adamw(params, [g], **states, step=step, norm=None if limit is None else norm, max_norm=limit, **HYPER)
        factor = 1.0 if limit is None else limit / 3.0
        want = 0.9 * old + 0.1 * factor * g.double()
        s = power(states["m_scales"][0]).repeat_interleave(32)
        got = states["m"][0].double() * s
        near = torch.maximum(want.abs(), 2.0 ** -6 * s)
        # a step is at most 2^-3 of the power of two below an amount, and of 2^-6 for the smallest; five roundings of the terms
        lost = 5 * 2.0 ** -24 * (0.9 * old.abs() + 0.1 * factor * g.double().abs())
        assert bool(((got - want).abs() <= near / 8 + lost).all())
        # and the mean is kept: half of a step's variance at most, six standard deviations of a million
        off = ((got - want) / near).mean().item()
        assert abs(off) <= 6 * (1 / 16) / math.sqrt(count)
