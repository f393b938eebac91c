"""hag_adamw against the formulas in 64 bits: one tensor to more than one launch holds, types and addresses mixed, clipping, copies, states in 8 bits by their thresholds, roots that stay above
zero, means that are kept over many steps, captured steps."""
import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
EPS = 2.0 ** -24
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TINY = {torch.float32: 2.0 ** -150, torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25}
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
PAIRS = [(F32, F32), (F32, BF16), (F32, F16), (BF16, BF16), (F16, F16)]
E4M3, E8M0 = torch.float8_e4m3fn, torch.float8_e8m0fnu
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


def thresholds(count, step, seed):
    x = mixed(torch.arange(count, device="cuda") * 0x9E3779B1 + mixed(torch.tensor(seed + step * 0x9E3779B1, device="cuda")))
    return x & 0xFFFF, x >> 16


def wide8(codes, scales):
    return codes.double().flatten() * scales.double().repeat_interleave(32)[:codes.numel()]


def step64(p, g, m, v, step, clip=1.0, lr=2e-3, betas=(0.9, 0.99), eps=1e-8, weight_decay=0.05):
    g = g.double().flatten() * clip
    m = betas[0] * m.double().flatten() + (1 - betas[0]) * g
    v = betas[1] * v.double().flatten() + (1 - betas[1]) * g * g
    update = m / (1 - betas[0] ** step) / ((v / (1 - betas[1] ** step)).sqrt() + eps)
    return p.double().flatten() * (1 - lr * weight_decay) - lr * update, m, v, g


def check_params(p, before, after64, m, g, b1=0.9, lr=2e-3, step=1, v=None, eps=1e-8, b2=0.99):
    """m carries three roundings of its terms (and the factors'), the root five, the quotient, the rate and the difference one or two each."""
    terms = b1 * (m - (1 - b1) * g).abs() / b1 + (1 - b1) * g.abs()
    update = lr / (1 - b1 ** step) * terms / ((v / (1 - b2 ** step)).sqrt() + eps)
    bound = 20 * EPS * update + 4 * EPS * before.double().flatten().abs()
    assert bool(((p.double().flatten() - after64).abs() <= bound + HALF[p.dtype] * (after64.abs() + bound) + TINY[p.dtype]).all())


def check_dithered(codes, scales, want, err, random, keep):
    """Every element is its amount's step below, or the next where the cut-off part and its threshold make one: either where the two are nearer than what fp32 loses (err, a part of the amount)."""
    count = want.numel()
    s, a = scales.double(), torch.nn.functional.pad(want.abs(), (0, -count % 32)).view(-1, 32)
    most = a.amax(1)
    assert bool((448 * s >= most * (1 - err)).all())
    assert bool(((448 * s / 2 < most * (1 + err)) | ((most == 0) & (s == 1)) | (s == 2.0 ** -127)).all())
    y = want.abs() / s.repeat_interleave(32)[:count]
    got = codes.double().flatten()
    assert bool(((got.abs() == 0) | (torch.signbit(got) == torch.signbit(want)) | (y < err)).all())
    step = torch.exp2(torch.floor(torch.log2(y.clamp(min=2.0 ** -6))) - 3)
    at, slack = y / step + (random + 0.5) / 65536, y / step * err + 2.0 ** -18
    low, high = torch.floor(at - slack) * step, torch.floor(at + slack) * step
    if keep:
        low, high = (torch.where(want != 0, t.clamp(min=2.0 ** -9), t) for t in (low, high))
    assert bool(((got.abs() >= low) & (got.abs() <= high)).all())
    # and nearly all are where the threshold says
    assert int((low != high).sum()) <= 3 + count * 1e-3


def make(counts, pair, gen, start=0, zeros=True):
    """Parameters and gradients end to end in one buffer each, from element `start` on."""
    total = sum(counts)
    p = torch.randn(total + start, device="cuda", generator=gen).to(pair[0])
    g = (0.1 * torch.randn(total + start, device="cuda", generator=gen) * torch.exp(2 * torch.randn(total + start, device="cuda", generator=gen))).to(pair[1])
    if zeros:
        g[::5] = 0
    return list(torch.split(p[start:], counts)), list(torch.split(g[start:], counts))


COUNTS = [[1], [3], [5, 4, 0, 1], [31, 32, 33], [63, 64, 65, 2], [4095, 4096, 4097], [100000], [7, 1000003, 9], [2500000, 1, 2, 3, 12345], list(range(1, 60)), [17] * 300]


@pytest.mark.parametrize("pair", PAIRS)
@pytest.mark.parametrize("counts", COUNTS)
def test_states_in_32_bits(B, counts, pair):
    gen = torch.Generator(device="cuda").manual_seed(len(counts))
    for start in (0, 1):
        params, grads = make(counts, pair, gen, start)
        states = B.adamw_states(params)
        assert all(not bool(t.any()) and t.dtype == F32 for k in "mv" for t in states[k])
        for step in (1, 2, 3):
            norm = torch.tensor(3.0, device="cuda") if step == 2 else None
            clip = 0.5 / 3.0 if step == 2 else 1.0
            before = [[t.clone() for t in x] for x in (params, states["m"], states["v"])]
            B.adamw(params, grads, **states, step=step, norm=norm, max_norm=0.5 if step == 2 else None, **HYPER)
            for i, (p, g) in enumerate(zip(params, grads)):
                p0, m0, v0 = (x[i] for x in before)
                want, m, v, gc = step64(p0, g, m0, v0, step, clip, **HYPER)
                m1, v1 = states["m"][i].double(), states["v"][i].double()
                assert bool(((m1 - m).abs() <= 4 * EPS * (0.9 * m0.double().abs() + 0.1 * gc.abs()) + TINY[F32]).all())
                assert bool(((v1 - v).abs() <= 6 * EPS * v + 2 * TINY[F32]).all())
                check_params(p, p0, want, m, gc, step=step, v=v)


@pytest.mark.parametrize("pair", PAIRS)
@pytest.mark.parametrize("counts", COUNTS)
def test_states_in_8_bits(B, counts, pair):
    gen = torch.Generator(device="cuda").manual_seed(len(counts) + 100)
    for start in (0, 1):
        params, grads = make(counts, pair, gen, start)
        states = B.adamw_states(params, bits=8)
        assert all(not bool(t.double().any()) and t.dtype == E4M3 for k in "mv" for t in states[k])
        for step in (1, 2, 7):
            norm = torch.tensor(3.0, device="cuda") if step == 2 else None
            clip = 0.5 / 3.0 if step == 2 else 1.0
            before = [[t.clone() for t in params]] + [[wide8(c, s) for c, s in zip(states[k], states[k + "_scales"])] for k in "mv"]
            B.adamw(params, grads, **states, step=step, norm=norm, max_norm=0.5 if step == 2 else None, seed=11, **HYPER)
            for i, (p, g) in enumerate(zip(params, grads)):
                if p.numel() == 0:
                    continue
                p0, m0, r0 = (x[i] for x in before)
                want, m, v, gc = step64(p0, g, m0, r0.square(), step, clip, **HYPER)
                check_params(p, p0, want, m, gc, step=step, v=v)
                random = thresholds(p.numel(), step, 11)
                # m: three roundings of its terms, which may cancel: elements where they do are left to the test of exact bits
                sound = (m.abs() >= 0.02 * (0.9 * m0.abs() + 0.1 * gc.abs())).all()
                if bool(sound):
                    check_dithered(states["m"][i], states["m_scales"][i], m, 200 * EPS, random[0], False)
                check_dithered(states["v"][i], states["v_scales"][i], v.sqrt(), 8 * EPS, random[1], True)


@pytest.mark.parametrize("pair", [(F32, F32), (F32, BF16)])
@pytest.mark.parametrize("counts", [[70], [4096, 33], [1000003]])
def test_8_bits_are_those_of_the_formula(B, counts, pair):
    """Products and sums rounded one by one in fp32, as separate operations are: the same bits everywhere."""
    gen = torch.Generator(device="cuda").manual_seed(3)
    params, grads = make(counts, pair, gen)
    states = B.adamw_states(params, bits=8)
    for step in range(1, 6):
        old = [[wide8(c, s).float() for c, s in zip(states[k], states[k + "_scales"])] for k in "mv"]
        B.adamw(params, grads, **states, step=step, seed=5, **HYPER)
        for i, g in enumerate(grads):
            g = g.float()
            m = 0.9 * old[0][i] + (1 - 0.9) * g
            r = torch.sqrt(0.99 * (old[1][i] * old[1][i]) + (1 - 0.99) * (g * g))
            for key, x, random in zip("mv", (m, r), thresholds(g.numel(), step, 5)):
                scales = states[key + "_scales"][i]
                small = (x.abs().double() / scales.double().repeat_interleave(32)[:x.numel()]).float() * 2.0 ** -120
                codes = (small.view(torch.int32) + (random * 16 + 8).int()) >> 20
                if key == "v":
                    codes = torch.where(x != 0, codes.clamp(min=1), codes)
                codes = codes | torch.signbit(x).int() << 7
                assert torch.equal(states[key][i].view(torch.uint8).int(), codes)


def test_8_bit_states_keep_their_means(B):
    """With one gradient throughout m becomes g and the root |g|.  Rounded to the nearest, the root would stay where the first step left it, at a tenth of |g| for b2 = 0.99.

    A step of an element is at most 1/8 of it; what rounding adds per step has a variance of at most change * step for the root, about 0.005 * 1/8 at its level, and decays by 0.01 a step,
    so that an element's standard deviation is below sqrt(0.005 / 8 / 0.02) = 0.18 and a mean's of n elements 0.18 / sqrt(n); for m it is below sqrt(1/4 / 64 / 0.19) = 0.15.  The
    root's mean square is what is kept, up to the variance of one step's rounding; levels are averaged over the last steps as well, which only helps."""
    n = 1 << 16
    g = torch.full((n,), 0.37, device="cuda")
    p = [torch.zeros(n, device="cuda")]
    states = B.adamw_states(p, bits=8)
    sums, steps = torch.zeros(2, dtype=torch.float64, device="cuda"), 0
    for step in range(1, 1501):
        B.adamw(p, [g], **states, step=step, **HYPER)
        if step > 1000 and step % 10 == 0:
            m, r = (wide8(states[k][0], states[k + "_scales"][0]) for k in "mv")
            sums += torch.stack([m.mean(), r.square().mean()])
            steps += 1
    m, square = (sums / steps).tolist()
    assert abs(m / 0.37 - 1) <= 6 * 0.15 / math.sqrt(n) + 1e-4
    # E[r_q^2] = E[r'^2] + the variance of one rounding, at most (1/8)^2 / 4 of it, every step: b2 E[r_q^2] + (1 - b2) g^2 + that
    assert 1 - 0.01 <= square / 0.37 ** 2 <= 1 + 0.2
    # a constant gradient moves every parameter by about lr a step (less the decay): the states may not slow or speed this by more than the root's spread
    assert abs(p[0].mean().item() / -(0.002 * (1 - (1 - 1e-4) ** 1500) / 1e-4) - 1) <= 0.1


def test_thresholds_are_even(B):
    """Elements halfway between two steps go up half of the time, at every step and over steps of one element; those of m and of the root independently."""
    n = 1 << 18
    p, g = [torch.zeros(n, device="cuda")], torch.full((n,), 17 / 16 * 1.0, device="cuda")   # between 1 and 9/8: halfway
    ups = []
    for step in range(1, 33):
        states = B.adamw_states(p, bits=8)
        g[::32] = 256.0                                    # the block's scale is 1 for m
        B.adamw(p, [g], **states, step=step, lr=0.0, betas=(0.0, 0.0), weight_decay=0.0)
        ups.append(torch.stack([(states[k][0].double() * states[k + "_scales"][0].double().repeat_interleave(32) > 17 / 16)[1::32] for k in "mv"]))
    ups = torch.stack(ups).double()                        # [steps, 2, elements]
    count = ups.shape[2]
    assert bool(((ups.mean(2) - 0.5).abs() <= 5.5 * 0.5 / math.sqrt(count)).all())
    total = ups.sum(0)                                     # of 32 steps each: variance 8
    assert bool((((total - 16).square().mean(1) / 8 - 1).abs() <= 6 * math.sqrt(2 / count)).all())
    both = (ups[:, 0] * ups[:, 1]).mean()
    assert abs(both.item() - 0.25) <= 6 * math.sqrt(3 / 16 / (32 * count))
    neighbours = (ups[:, 0, :-1] * ups[:, 0, 1:]).mean()
    assert abs(neighbours.item() - 0.25) <= 6 * math.sqrt(0.35 / (32 * count))


def test_roots_stay_above_zero(B):
    """An element far below its block's largest: its first moment lasts some steps, so may its root."""
    p = [torch.zeros(64, device="cuda")]
    g = torch.full((64,), 1e-12, device="cuda")
    g[0] = g[40] = 1e3
    states = B.adamw_states(p, bits=8)
    for step in range(1, 20):
        B.adamw(p, [g], **states, step=step, lr=1e-2, weight_decay=0.0)
        assert bool((states["v"][0].double() > 0).all())
        g = torch.zeros(64, device="cuda")
        g[0] = g[40] = 1e3
    assert bool((p[0].abs() < 1.0).all())                  # 19 steps of 0.01 with quotients of a few; without a root 1e-13 / 1e-8 is as harmless, 1e-3 / 1e-8 is not


@pytest.mark.parametrize("bits", [8, 32])
def test_clipping_and_norms_that_are_none(B, bits):
    gen = torch.Generator(device="cuda").manual_seed(8)
    params, grads = make([1000, 77], (F32, F32), gen)
    norm = B.clip_gradients(grads, math.inf)
    size = norm.item()

    def after(grads, **how):
        ps, states = [p.clone() for p in params], B.adamw_states(params, bits)
        B.adamw(ps, grads, **states, step=4, **how, **HYPER)
        return ps + [t.view(torch.uint8) for x in states.values() for t in x]

    plain = after(grads)
    assert all(torch.equal(a, b) for a, b in zip(plain, after(grads, norm=norm, max_norm=1.01 * size)))
    assert all(torch.equal(a, b) for a, b in zip(plain, after(grads, norm=norm, max_norm=math.inf)))
    factor = 0.25 * size / size
    scaled = [(g.double() * (0.25 * size / norm.double())).float() for g in grads]
    assert abs(factor - 0.25) < 1e-9
    assert all(torch.equal(a, b) for a, b in zip(after(scaled), after(grads, norm=norm, max_norm=0.25 * size)))
    untouched = [p.clone() for p in params] + [t.view(torch.uint8) for x in B.adamw_states(params, bits).values() for t in x]
    for none in (math.inf, math.nan):
        assert all(torch.equal(a, b) for a, b in zip(untouched, after(grads, norm=torch.tensor(none, device="cuda"), max_norm=1.0)))
    far = [(1e30 * g).clamp(-1e37, 1e37) for g in grads]   # a factor that is no ordinary fp32 number
    big = B.clip_gradients([t.clone() for t in far], math.inf)
    small = 1e-12
    small_grads = [(g.double() * (small / big.double())).float() for g in far]
    assert all(torch.equal(a, b) for a, b in zip(after(small_grads), after(far, norm=big, max_norm=small)))


@pytest.mark.parametrize("bits", [8, 32])
@pytest.mark.parametrize("copy", [BF16, F16, F32])
def test_copies_and_layouts(B, bits, copy):
    gen = torch.Generator(device="cuda").manual_seed(4)
    base = torch.randn(30, 40, device="cuda", generator=gen)
    params = [base.clone().t(), torch.randn(7, device="cuda", generator=gen), torch.randn(3, 5, 6, device="cuda", generator=gen).permute(2, 0, 1)]
    grads = [torch.randn(30, 40, device="cuda", generator=gen).t(), torch.randn(7, device="cuda", generator=gen), torch.randn(3, 5, 6, device="cuda", generator=gen).permute(2, 0, 1)]
    copies = [torch.empty_like(params[0], dtype=copy), None, torch.empty_like(params[2], dtype=copy)]
    flat = [p.clone(memory_format=torch.contiguous_format).contiguous() for p in (params[0].t(), params[1], params[2].permute(1, 2, 0))]
    fgrads = [g.contiguous() for g in (grads[0].t(), grads[1], grads[2].permute(1, 2, 0))]
    states, fstates = B.adamw_states(params, bits), B.adamw_states(flat, bits)
    for step in (1, 2):
        B.adamw(params, grads, **states, step=step, copies=copies, **HYPER)
        B.adamw(flat, fgrads, **fstates, step=step, **HYPER)
    assert torch.equal(params[0].t(), flat[0]) and torch.equal(params[1], flat[1]) and torch.equal(params[2].permute(1, 2, 0), flat[2])
    assert torch.equal(copies[0], params[0].to(copy)) and torch.equal(copies[2], params[2].to(copy))
    assert not torch.equal(base.t(), params[0])


@pytest.mark.parametrize("bits", [8, 32])
def test_what_lies_beside_is_left(B, bits):
    gen = torch.Generator(device="cuda").manual_seed(12)
    for count in (1, 30, 33, 4097):
        buffers = {k: torch.full((count + 64,), 7, dtype=torch.uint8, device="cuda") for k in ("m8", "v8", "ms", "vs")}
        p, m, v = (torch.full((count + 64,), 7.0, device="cuda") for _ in range(3))
        g = torch.randn(count, device="cuda", generator=gen)
        p[32:32 + count], m[32:32 + count], v[32:32 + count] = 1.0, 0.0, 0.0
        blocks = (count + 31) // 32
        if bits == 8:
            parts = [buffers[k][16:16 + count] for k in ("m8", "v8")] + [buffers[k][16:16 + blocks] for k in ("ms", "vs")]
            for t in parts[:2]:
                t.zero_()
            B.adamw([p[32:32 + count]], [g], [parts[0].view(E4M3)], [parts[1].view(E4M3)], 1, m_scales=[parts[2].view(E8M0)], v_scales=[parts[3].view(E8M0)])
            for k, used in (("m8", count), ("v8", count), ("ms", blocks), ("vs", blocks)):
                assert bool((buffers[k][:16] == 7).all()) and bool((buffers[k][16 + used:] == 7).all())
        else:
            B.adamw([p[32:32 + count]], [g], [m[32:32 + count]], [v[32:32 + count]], 1)
            assert bool((m[:32] == 7).all()) and bool((m[32 + count:] == 7).all()) and bool((v[:32] == 7).all()) and bool((v[32 + count:] == 7).all())
        assert bool((p[:32] == 7).all()) and bool((p[32 + count:] == 7).all()) and not bool((p[32:32 + count] == 1).any())


def test_elements_that_are_no_numbers(B):
    g = torch.ones(100, device="cuda")
    g[3], g[40] = float("nan"), float("inf")
    for bits in (8, 32):
        p = [torch.ones(100, device="cuda")]
        states = B.adamw_states(p, bits)
        B.adamw(p, [g], **states, step=1)
        clean = torch.ones(100, dtype=torch.bool, device="cuda")
        clean[3] = clean[40] = False
        assert bool(p[0][3].isnan()) and bool(p[0][40].isnan()) and bool((p[0][clean] == p[0][0]).all())
        m = states["m"][0].float()
        assert bool(m[3].isnan()) and not bool(m[clean].isnan().any())
        if bits == 8:
            assert bool(states["v"][0].float()[[3, 40]].isnan().all()) and bool(m[40].isnan())
            values = wide8(states["m"][0], states["m_scales"][0])
            assert bool(((values[clean] - 0.1).abs() <= 0.1 / 8).all())


def test_numbers_on_the_device_and_captured(B):
    gen = torch.Generator(device="cuda").manual_seed(21)
    params, grads = make([5000, 31, 260], (F32, BF16), gen)
    ref = [p.clone() for p in params]
    for bits in (8, 32):
        states, rstates = B.adamw_states(params, bits), B.adamw_states(ref, bits)
        step, lr = torch.zeros((), dtype=torch.int64, device="cuda"), torch.tensor(1e-3, device="cuda")
        norm = torch.tensor(2.0, device="cuda")

        def run():
            step.add_(1)
            B.adamw(params, grads, **states, step=step, lr=lr, norm=norm, max_norm=1.0)

        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            run()
        torch.cuda.current_stream().wait_stream(side)
        B.adamw(ref, grads, **rstates, step=1, lr=lr.item(), norm=norm, max_norm=1.0)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            run()
        for i in range(2, 7):
            lr.mul_(0.9)
            norm.mul_(1.1)
            for g in grads:
                g.copy_(torch.randn(g.shape, device="cuda", generator=gen))
            graph.replay()
            B.adamw(ref, grads, **rstates, step=i, lr=lr.item(), norm=norm, max_norm=1.0)
            assert all(torch.equal(a, b) for a, b in zip(params, ref))
            assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for k in states for a, b in zip(states[k], rstates[k]))
            torch.cuda.synchronize()


def test_late_steps_and_ends_of_the_numbers(B):
    gen = torch.Generator(device="cuda").manual_seed(2)
    for how in (dict(step=10 ** 6), dict(step=3, betas=(0.0, 0.999)), dict(step=3, betas=(0.9, 0.0)), dict(step=1, betas=(0.99999, 0.9999999)), dict(step=12, eps=1.0), dict(step=2 ** 40, lr=0.0),
                dict(step=5, weight_decay=0.0), dict(step=5, lr=0.5, weight_decay=1.9)):
        hyper = {**HYPER, **how}
        params, grads = make([777], (F32, F32), gen, zeros=False)
        states = B.adamw_states(params)
        states["m"][0].normal_(generator=gen)
        states["v"][0].uniform_(0.1, 1.0, generator=gen)
        before = [t.clone() for t in (params[0], states["m"][0], states["v"][0])]
        B.adamw(params, grads, **states, **hyper)
        want, m, v, g = step64(before[0], grads[0], before[1], before[2], hyper["step"], 1.0, hyper["lr"], hyper["betas"], hyper["eps"], hyper["weight_decay"])
        b1, b2 = hyper["betas"]
        terms = b1 * before[1].double().abs() + (1 - b1) * g.abs()
        update = hyper["lr"] / (1 - b1 ** hyper["step"]) * terms / ((v / (1 - b2 ** hyper["step"])).sqrt() + hyper["eps"])
        assert bool(((params[0].double() - want).abs() <= 20 * EPS * update + 4 * EPS * before[0].double().abs()).all())


def test_refusals(B):
    p, g = torch.ones(64, device="cuda"), torch.ones(64, device="cuda")
    s32, s8 = B.adamw_states([p]), B.adamw_states([p], 8)
    B.adamw([], [], [], [], 1)
    norm = torch.ones((), device="cuda")

    def call(params=(p,), grads=(g,), states=s32, step=1, **how):
        B.adamw(list(params), list(grads), **{**states, **{k: how.pop(k) for k in list(how) if k in ("m", "v", "m_scales", "v_scales")}}, step=step, **how)

    two = torch.ones(8, 8, device="cuda")
    for bad in (dict(grads=()), dict(params=(p, p), grads=(g, g)), dict(grads=(g.bfloat16().double(),)), dict(grads=(g[:32],)), dict(params=(p.bfloat16(),)), dict(params=(p.cpu(),), grads=(g.cpu(),)),
                dict(params=(p[::2],), grads=(g[::2],)), dict(params=(two,), grads=(two.clone().t(),)), dict(m=[s32["m"][0][:32]]), dict(m=[s32["m"][0].double()]), dict(states=s8, v_scales=None),
                dict(states=s8, m_scales=[s8["m_scales"][0][:1]]), dict(states=s8, m=s32["m"]), dict(v_scales=s8["v_scales"]), dict(m=s32["v"]), dict(norm=norm), dict(max_norm=1.0), dict(norm=norm.double(), max_norm=1.0),
                dict(step=torch.ones((), device="cuda")), dict(lr=torch.ones((), device="cuda").double()), dict(copies=[p[:3]]), dict(copies=[]), dict(copies=[p])):
        with pytest.raises(ValueError):
            call(**bad)
    for bad in (dict(step=0), dict(lr=math.nan), dict(betas=(1.0, 0.9)), dict(betas=(0.9, -0.1)), dict(eps=0.0), dict(eps=math.nan), dict(weight_decay=math.inf), dict(norm=norm, max_norm=0.0)):
        with pytest.raises(B.HagError):
            call(**bad)
    with pytest.raises(ValueError):
        B.adamw_states([p], 16)
    assert bool((p == 1).all())
