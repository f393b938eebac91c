"""Sizes that one launch or 32 bits do not hold: RMS norm in both outputs and its gradient, products of 8-bit rows, AdamW.  Inputs are views of little memory (rows that begin a few elements
after each other); outputs are as large as they are."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
GB = 10 ** 9
E4M3, E8M0 = torch.float8_e4m3fn, torch.float8_e8m0fnu


@pytest.fixture(scope="module")
def B():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_1906_03707_amd import binding
    binding.lib()
    return binding


@pytest.fixture(autouse=True)
def memory():
    yield
    if torch.cuda.is_available():
        torch.cuda.empty_cache()


def need(nbytes):
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < nbytes:
        pytest.skip(f"{nbytes / GB:.0f} GB of free memory are needed")


def some_rows(n, step):
    """The first and the last rows, those where a launch may end, and some between."""
    seams = [s + k for s in range(0, n, step) for k in (-1, 0, 1) if 0 <= s + k < n][:400]
    return torch.tensor(sorted({0, 1, n // 3, n - 2, n - 1, *seams, *range(0, n, max(n // 200, 1))}), device="cuda")


@pytest.mark.parametrize("n,d", [(2 ** 27 + 9, 258), (2 ** 24 + 5, 1032), (2 ** 22 + 3, 4104), (2 ** 22 + 3, 8200)])
def test_rms_norm_of_many_rows(B, n, d):
    need(3 * n * d + 10 * GB)
    gen = torch.Generator(device="cuda").manual_seed(d)
    flat = torch.randn(n + d - 1, device="cuda", generator=gen).bfloat16()
    x = flat.as_strided((n, d), (1, 1))                    # each row one element after the one before
    w = 1 + 0.1 * torch.randn(d, device="cuda", generator=gen)
    some = some_rows(n, 2 ** 31 // 1024)
    x64, w64 = x[some].double(), w.double()
    r = (x64.square().mean(1, keepdim=True) + 1e-5).rsqrt()
    want = x64 * r * w64
    y, h, rstd = B.rms_norm(x, w)
    # 64 roundings on the way of a term
    assert h is x and bool(torch.isfinite(rstd).all()) and bool(((rstd[some].double()[:, None] - r).abs() <= 64 * 2.0 ** -24 * r).all())
    assert bool(((y[some].double() - want).abs() <= (2.0 ** -8 + 2.0 ** -16) * want.abs()).all())
    del y
    codes, scales, _ = B.rms_norm_fp8(x, w)
    s = scales[some].double().repeat_interleave(32, 1)[:, :d]
    assert bool(((codes[some].double() * s - want).abs() <= torch.maximum(want.abs() * (2.0 ** -4 + 2.0 ** -16), s * 2.0 ** -10)).all())
    assert bool((scales.float() > 0).all())
    del codes, scales
    gy = x[5:6].expand(n, d)
    gx, _ = B.rms_norm_grad(gy, x, rstd, w, params=False)
    u, xh = gy[:1].double() * w64, x64 * r
    want = r * (u - xh * (u * xh).mean(1, keepdim=True))
    assert bool(((gx[some].double() - want).abs() <= (2.0 ** -8 + 2.0 ** -16) * want.abs() + 2.0 ** -14).all())


@pytest.mark.parametrize("apart,w_apart", [(16, 40), (1, 40), (16, 48)])   # rows at any address, and both for tiles
def test_product_of_many_rows(B, apart, w_apart):
    n, d, k = 2 ** 28 + 77, 40, 20
    need(n * (apart + 2 * k + 8) + 10 * GB)
    gen = torch.Generator(device="cuda").manual_seed(apart)
    flat = torch.randint(0, 255, (n * apart + 64,), dtype=torch.uint8, device="cuda", generator=gen)
    flat[(flat & 0x7f) == 0x7f] = 0x40
    x = flat.view(E4M3).as_strided((n, d), (apart, 1))
    xs = (125 + torch.randint(0, 5, (n + 2,), device="cuda", generator=gen)).to(torch.uint8).view(E8M0).as_strided((n, 2), (1, 1))
    w = torch.randn(k, w_apart, device="cuda", generator=gen).to(E4M3)[:, :d]
    ws = torch.full((k, 2), 127, dtype=torch.uint8, device="cuda").view(E8M0)
    y = B.fp8_product(x, xs, w, ws, dtype=torch.bfloat16)
    some = some_rows(n, 2 ** 20 * 128 // 2)
    at = some[:, None] * apart + torch.arange(d, device="cuda")
    a = flat[at].view(E4M3).double() * xs.view(torch.uint8)[some].view(E8M0).double().repeat_interleave(32, 1)[:, :d]
    w64 = w.float().double().t().contiguous()
    want, size = a @ w64, a.abs() @ w64.abs()
    assert bool(((y[some].double() - want).abs() <= 2.0 ** -8 * want.abs() + (16 * 2.0 ** -14 + 64 * 2.0 ** -24) * size * (1 + 2.0 ** -8)).all())


@pytest.mark.parametrize("bits", [32, 8])
def test_step_of_more_elements_than_32_bits_number(B, bits):
    count = 2 ** 32 + 70001
    need(count * (2 + 2 + 2 * bits // 8) + 20 * GB)
    p, g = torch.zeros(count, dtype=torch.bfloat16, device="cuda"), torch.empty(count, dtype=torch.bfloat16, device="cuda")
    for part in range(0, count, 1 << 28):
        g[part:part + (1 << 28)].normal_()
    states = B.adamw_states([p], bits)
    B.adamw([p], [g], **states, step=1, weight_decay=0.0, lr=0.5, seed=7)

    def mixed(x):
        x = x & 0xFFFFFFFF
        x = (x ^ (x >> 15)) * 0x6A09E667 & 0xFFFFFFFF
        x = (x ^ (x >> 13)) * 0xBB67AE85 & 0xFFFFFFFF
        return x ^ (x >> 16)

    for begin in (0, 2 ** 31 - 512, 2 ** 32 - 4096, 2 ** 32, count // 32 * 32 - 4096):
        part = slice(begin, min(begin + 5000, count))
        some = g[part].float()
        # the first step moves every parameter by lr towards its gradient's sign
        want = -0.5 * some / (some.abs() + 1e-8)
        assert bool(((p[part].float() - want).abs() <= 2.0 ** -9 + 1e-5).all())
        m = 0.0 + (1 - 0.9) * some
        if bits == 32:
            assert torch.equal(states["m"][0][part], m)
            continue
        scales = states["m_scales"][0][begin // 32:(part.stop + 31) // 32].double().repeat_interleave(32)[:some.numel()]
        at = torch.arange(part.start, part.stop, device="cuda")
        random = mixed(at * 0x9E3779B1 + (at >> 32) * 0x85EBCA6B + mixed(torch.tensor(7 + 0x9E3779B1, device="cuda"))) & 0xFFFF
        small = (m.abs().double() / scales).float() * 2.0 ** -120
        codes = (small.view(torch.int32) + (random * 16 + 8).int()) >> 20
        assert torch.equal(states["m"][0][part].view(torch.uint8).int(), codes | torch.signbit(m).int() << 7)
