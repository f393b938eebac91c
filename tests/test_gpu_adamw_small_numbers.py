"""hag_adamw where squares of gradients are below fp32's ordinary numbers: roots have to be those of what is kept, which counts where eps is smaller still."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
EPS, LEAST = 2.0 ** -24, 2.0 ** -149
F32, E4M3, E8M0 = torch.float32, torch.float8_e4m3fn, torch.float8_e8m0fnu


@pytest.fixture(scope="module")
def B():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_1906_03707_amd import binding
    binding.lib()
    return binding


def gradients(count, low, high, ordinary=True):
    """Both signs, amounts 2^low to 2^high, zeros, and ordinary ones among them, so that one wavefront meets both (an 8-bit block's scale goes with those)."""
    gen = torch.Generator().manual_seed(count)
    g = torch.exp2(low + (high - low) * torch.rand(count, generator=gen, dtype=torch.float64)) * (torch.randint(0, 2, (count,), generator=gen) * 2 - 1)
    if ordinary:
        g[::7] = 0.25
    g[3::11] = 0.0
    return g.float()


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("eps", [1e-8, 1e-20, 1e-30, 2.0 ** -126])
@pytest.mark.parametrize("beta2", [0.999, 0.9])
@pytest.mark.parametrize("count", [5, 3000])
def test_first_step(B, count, beta2, eps, bits):
    """From states of zero every parameter moves by lr |g| / (|g| + eps), whatever the size of its gradient."""
    g = gradients(count, -63.0, -48.0)
    p = [torch.zeros(count, device="cuda")]
    states = B.adamw_states(p, bits)
    B.adamw(p, [g.cuda()], **states, step=1, lr=1.0, betas=(0.9, beta2), eps=eps, weight_decay=0.0)
    g64 = g.double()
    want = -g64 / (g64.abs() + eps)
    v = (1 - beta2) * g64.square()
    # the square, its part and the sum are rounded in fp32: EPS of them or half of the least number each; the root carries half of that part, the other roundings as ever
    part = (4 * EPS * v + 2 * LEAST) / torch.where(v > 0, v, 1.0)
    assert bool(((v == 0) | (part < 0.05)).all())
    off = (p[0].cpu().double() - want).abs()
    assert bool((off <= want.abs() * (part + 24 * EPS) + LEAST).all())


@pytest.mark.parametrize("beta2", [0.99, 0.5])
def test_8_bit_roots_are_those_of_the_formula(B, beta2):
    """The root of b2 r^2 + (1 - b2) g^2 in fp32, products and sums rounded one by one, rounded correctly (the CPU's is): the same bits, down to the least square."""
    for count, low, high in ((33, -60.0, -45.0), (5000, -74.0, -40.0), (64, -80.0, -70.0), (2000, -66.0, -63.0), (20000, -63.0, 3.0), (20001, -70.0, -62.0)):
        p, g = [torch.zeros(count, device="cuda")], gradients(count, low, high, count % 2 == 0 and low != -66.0)
        states = B.adamw_states(p, 8)
        x = torch.arange(count)

        def mixed(x):
            x = x & 0xFFFFFFFF
            x = (x ^ (x >> 15)) * 0x6A09E667 & 0xFFFFFFFF
            x = (x ^ (x >> 13)) * 0xBB67AE85 & 0xFFFFFFFF
            return x ^ (x >> 16)

        for step in (1, 2, 3):
            old = states["v"][0].cpu().double() * states["v_scales"][0].cpu().double().repeat_interleave(32)[:count]
            old = old.float()
            B.adamw(p, [g.cuda()], **states, step=step, lr=0.0, betas=(0.9, beta2), seed=5)
            # (on the CPU, which keeps numbers below 2^-126)
            r = torch.sqrt(torch.tensor(beta2, dtype=F32) * (old * old) + torch.tensor(1 - beta2, dtype=F32) * (g * g))
            random = mixed(x * 0x9E3779B1 + mixed(torch.tensor(5 + step * 0x9E3779B1))) >> 16
            scales = states["v_scales"][0].cpu().double().repeat_interleave(32)[:count]
            small = (r.double() / scales).float() * 2.0 ** -120
            codes = (small.view(torch.int32) + (random * 16 + 8).int()) >> 20
            codes = torch.where(r != 0, codes.clamp(min=1), codes)
            assert torch.equal(states["v"][0].cpu().view(torch.uint8).int(), codes)
            most = torch.nn.functional.pad(r, (0, -count % 32)).view(-1, 32).amax(1).double()
            s = states["v_scales"][0].cpu().double()
            assert bool(((448 * s >= most) & ((224 * s < most) | (s == 2.0 ** -127))).logical_or((most == 0) & (s == 1)).all())
            g = g.roll(1)
