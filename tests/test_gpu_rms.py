"""hag_rms_norm, hag_rms_norm_fp8 and hag_rms_norm_grad against the formulas in 64 bits: widths from one column to more than a workgroup holds, odd ones, views, rows out of fp32's
range, elements that are no numbers, ties of 8 bits, gradients by differences, weight gradients that see a lost row."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
EPS = 2.0 ** -24
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TINY = {torch.float32: 2.0 ** -150, torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25}
TYPES = [torch.float32, torch.bfloat16, torch.float16]
WIDTHS = [1, 2, 3, 4, 7, 8, 16, 31, 32, 33, 64, 100, 127, 128, 130, 251, 256, 260, 500, 512, 513, 777, 1024, 1030, 2048, 2050, 4096, 4099, 8192, 8200, 16500]


@pytest.fixture(scope="module")
def B():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_1906_03707_amd import binding
    binding.lib()
    return binding


def forward64(h, w, eps):
    h = h.double()
    r = (h.square().mean(1, keepdim=True) + eps).rsqrt()
    return h * r * (1.0 if w is None else w.double()), r


def rounding(d):
    """Of y: the squares' sum (d additions and a product each, all of one sign) to half a part under the root, the root and two products."""
    return ((d + 4) / 2 + 6) * EPS


def check_sum(h, x, res):
    assert h is x if res is None else torch.equal(h, (x.float() + res.float()).to(x.dtype))


def check_forward(got, x, res, w, eps):
    y, h, rstd = got
    n, d = x.shape
    check_sum(h, x, res)
    want, r = forward64(h, w, eps)
    assert y.dtype == x.dtype and y.shape == x.shape and rstd.shape == (n,) and rstd.dtype == torch.float32
    assert bool(((rstd.double()[:, None] - r).abs() <= rounding(d) * r).all())
    dy = rounding(d) * want.abs()
    assert bool(((y.double() - want).abs() <= dy + HALF[y.dtype] * (want.abs() + dy) + TINY[y.dtype]).all())


def blocks(t, d):
    return torch.nn.functional.pad(t, (0, -d % 32)).unflatten(1, (-1, 32))


def check_fp8(got, x, res, w, eps):
    codes, scales, h = got
    n, d = x.shape
    check_sum(h, x, res)
    want, _ = forward64(h, w, eps)
    err = rounding(d)
    assert codes.dtype == torch.float8_e4m3fn and codes.shape == (n, d) and scales.dtype == torch.float8_e8m0fnu and scales.shape == (n, (d + 31) // 32)
    s, most = scales.double(), blocks(want.abs(), d).amax(2)
    assert bool((448 * s >= most * (1 - err)).all())                               # the largest fits,
    assert bool(((448 * s / 2 < most * (1 + err)) | ((most == 0) & (s == 1)) | (s == 2.0 ** -127)).all())          # and would not in a scale of half the size
    s = s.repeat_interleave(32, 1)[:, :d]
    # half a step of three mantissa bits, or of the steps near zero
    assert bool(((codes.double() * s - want).abs() <= torch.maximum(want.abs() * 2.0 ** -4, s * 2.0 ** -10) * (1 + 1e-6) + err * want.abs()).all())


def check_grad(got, gy, h, rstd, w, gh):
    gx, gw = got
    n, d = h.shape
    g, r = gy.double(), rstd.double()[:, None]
    xh = h.double() * r
    u = g if w is None else g * w.double()
    more = 0.0 if gh is None else gh.double()
    s = (u * xh).mean(1, keepdim=True)
    want = r * (u - xh * s) + more
    a = (u * xh).abs().mean(1, keepdim=True)
    # xh and u carry a rounding each, their sum d additions more; then five operations on terms of these sizes
    bound = r * (6 * EPS * u.abs() + xh.abs() * (d + 10) * EPS * a) + 2 * EPS * want.abs()
    bound = bound + HALF[gx.dtype] * (want.abs() + bound) + TINY[gx.dtype]
    assert gx.dtype == h.dtype and bool(((gx.double() - want).abs() <= bound).all())
    if gw is None:
        return
    terms = g * xh
    total, size = terms.sum(0), terms.abs().sum(0)
    bound = (n + 4) * EPS * size
    assert gw.dtype == (torch.float32 if w is None else w.dtype)
    assert bool(((gw.double() - total).abs() <= bound + HALF[gw.dtype] * (total.abs() + bound) + TINY[gw.dtype]).all())


def weights(d, dtype, gen):
    return (1 + 0.3 * torch.randn(d, device="cuda", generator=gen)).to(dtype)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d", WIDTHS)
def test_norm_and_gradient(B, d, dtype):
    gen = torch.Generator(device="cuda").manual_seed(d)
    rnd = lambda n: torch.randn(n, d, device="cuda", generator=gen)   # noqa: E731
    for n in (1, 2, 5, 67, 1030) if d < 600 else (1, 3, 130):
        x, gy = (2 * rnd(n)).to(dtype), rnd(n).to(dtype)
        for w, res in ((weights(d, torch.float32, gen), rnd(n).to(dtype)), (weights(d, dtype, gen), None), (None, rnd(n).to(dtype))):
            y, h, rstd = B.rms_norm(x, w, residual=res)
            check_forward((y, h, rstd), x, res, w, 1e-5)
            check_fp8(B.rms_norm_fp8(x, w, residual=res), x, res, w, 1e-5)
            gh = None if res is None else rnd(n).to(dtype)
            grads = B.rms_norm_grad(gy, h, rstd, w, g_h=gh)
            check_grad(grads, gy, h, rstd, w, gh)
    check_forward(B.rms_norm(x, w, eps=0.1), x, None, w, 0.1)
    again = B.rms_norm_grad(gy, h, rstd, w, g_h=gh)
    assert all(torch.equal(p, q) for p, q in zip(grads, again))
    gx, gw = B.rms_norm_grad(gy, h, rstd, w, g_h=gh, params=False)
    assert gw is None and torch.equal(gx, again[0])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d", [5, 64, 250, 1100, 9000])
def test_views(B, d, dtype):
    gen = torch.Generator(device="cuda").manual_seed(d)
    wide = torch.randn(41, 2 * d + 3, device="cuda", generator=gen).to(dtype)
    x, res, gy = wide[1::2, 1:d + 1], wide[:20, d + 2:2 * d + 2], wide[20:40, 2:d + 2]
    w = weights(2 * d, dtype, gen)[d:]
    got = B.rms_norm(x, w, residual=res)
    check_forward(got, x, res, w, 1e-5)
    codes, scales, _ = B.rms_norm_fp8(x, w, residual=res)
    check_fp8((codes, scales, got[1]), x, res, w, 1e-5)
    assert codes.stride(0) % 16 == 0
    check_grad(B.rms_norm_grad(gy, x, got[2], w, g_h=res), gy, x, got[2], w, res)
    row = wide[3, :d].expand(7, d)                         # one row throughout
    got = B.rms_norm(row, w, residual=row)
    check_forward(got, row, row, w, 1e-5)
    check_grad(B.rms_norm_grad(row, row, got[2], w, g_h=row), row, row, got[2], w, row)


@pytest.mark.parametrize("d", [1, 37, 64, 1000, 3000, 9000])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_rows_out_of_range(B, d, dtype):
    """Squares beyond fp32 or with lost bits, among ordinary rows; and eps that outweighs small ones."""
    gen = torch.Generator(device="cuda").manual_seed(d)
    x = torch.randn(19, d, device="cuda", generator=gen)
    x = (x * torch.tensor([1e30, 1.0, 1e-30, 1e19, 2e18, 1e-16, 1e-17, 1e37, 1e-35, 3.0, 1e-20, 1e20, 1, 1, 1, 1, 1e-25, 1e25, 2], device="cuda")[:, None]).to(dtype)
    w = weights(d, torch.float32, gen)
    for eps in (0.0, 1e-33, 1e-20, 1e-5):
        for res in (None, torch.zeros_like(x)):
            y, h, rstd = B.rms_norm(x, w, eps=eps, residual=res)
            check_forward((y, h, rstd), x, res, w, eps)
            check_fp8(B.rms_norm_fp8(x, w, eps=eps, residual=res), x, res, w, eps)
            gy = torch.randn(19, d, device="cuda", generator=gen).to(dtype)
            some = slice(9, 16)                            # (others' gradients may be beyond fp32)
            check_grad(B.rms_norm_grad(gy[some], h[some], rstd[some], w), gy[some], h[some], rstd[some], w, None)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d", [40, 300, 1200, 9000])
def test_elements_that_are_no_numbers(B, d, dtype):
    gen = torch.Generator(device="cuda").manual_seed(d)
    x = torch.randn(6, d, device="cuda", generator=gen).to(dtype)
    clean = x.clone()
    x[1, d // 2], x[3, 0], x[4] = float("nan"), float("inf"), 0.0
    y, h, rstd = B.rms_norm(x)
    assert bool(y[1].isnan().all()) and bool(y[3, 0].isnan()) and not bool(y[3, 1:].any()) and not bool(y[4].any())
    check_forward((y[::2], h[::2], rstd[::2]), h[::2], h[::2] * 0, None, 1e-5)
    codes, scales, _ = B.rms_norm_fp8(x)
    values = codes.float()
    assert bool(values[1].isnan().all()) and bool(values[3, 0].isnan()) and not bool(values[3, 1:].any()) and not bool(values[4].any())
    assert bool((scales[1].float() == 1).all()) and bool((scales[3:5].float() == 1).all())
    other = B.rms_norm_fp8(clean)
    for row in (0, 2, 5):
        assert torch.equal(codes[row].view(torch.uint8), other[0][row].view(torch.uint8)) and torch.equal(scales[row].view(torch.uint8), other[1][row].view(torch.uint8))
    # one element that is none leaves its block's scale to the others
    w = torch.ones(d, device="cuda")
    w[7] = float("inf")
    codes, scales, _ = B.rms_norm_fp8(clean, w)
    assert bool(codes[:, 7].float().isnan().all()) and not bool(codes[:, :7].float().isnan().any()) and not bool(codes[:, 8:].float().isnan().any())
    w[7] = 0.0
    assert torch.equal(scales.view(torch.uint8), B.rms_norm_fp8(clean, w)[1].view(torch.uint8))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d", [16, 32, 64, 256, 1024, 4096, 16384])
def test_8_bits_are_exact(B, d, dtype):
    """Rows of +-4 have a root of 4 without an eps: y is +-w, and its 8 bits the nearest ones, ties to even, in the smallest scale."""
    gen = torch.Generator(device="cuda").manual_seed(d)
    sign = torch.randint(0, 2, (9, d), device="cuda", generator=gen) * 2.0 - 1
    w = torch.randint(0, 512, (d,), device="cuda", generator=gen) / 16 * torch.exp2(torch.randint(-20, 20, ((d + 31) // 32,), device="cuda", generator=gen).float()).repeat_interleave(32)[:d]
    w[::7] = w[::7].round() + 0.5
    codes, scales, _ = B.rms_norm_fp8((4 * sign).to(dtype), w, eps=0.0)
    y = (sign * w).double()
    most = blocks(y.abs(), d).amax(2)
    want = torch.exp2(torch.ceil(torch.log2(most / 448)))
    assert torch.equal(scales.double(), torch.where(most == 0, 1.0, want))
    scaled = (y / scales.double().repeat_interleave(32, 1)[:, :d]).float()
    assert torch.equal(codes.float(), scaled.cpu().to(torch.float8_e4m3fn).float().cuda())
    edge = torch.tensor([448.0, 448.0 * (1 + 2.0 ** -23), 447.99], device="cuda")  # the largest at the border of two scales
    for v, s in zip(edge, (1.0, 2.0, 1.0)):
        w = torch.full((d,), v.item(), device="cuda")
        assert bool((B.rms_norm_fp8((4 * sign).to(dtype), w, eps=0.0)[1].float() == s).all())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,d", [(70001, 16), (40000, 64), (30000, 100), (9001, 250), (5000, 1000), (3001, 3000), (600, 9000)])
def test_weight_gradients_count_every_row_once(B, n, d, dtype):
    gen = torch.Generator(device="cuda").manual_seed(n)
    x, gy = (torch.randint(-3, 4, (n, d), device="cuda", generator=gen).to(dtype) for _ in range(2))
    one = torch.ones(n, device="cuda")
    _, gw = B.rms_norm_grad(gy, x, one)                    # with this rstd all terms are whole numbers, their sums exact in fp32
    assert torch.equal(gw.double(), (gy.double() * x.double()).sum(0))


@pytest.mark.parametrize("n,d", [(3, 5), (40, 64), (7, 333), (2, 5000)])
def test_gradient_by_differences(B, n, d):
    gen = torch.Generator(device="cuda").manual_seed(d)
    x, res, gy, gh = (torch.randn(n, d, device="cuda", generator=gen) for _ in range(4))
    w = weights(d, torch.float32, gen)
    _, h, rstd = B.rms_norm(x, w, residual=res)
    gx, gw = B.rms_norm_grad(gy, h, rstd, w, g_h=gh)
    for grad, where in ((gx, "x"), (gw, "w")):
        v = torch.randn(grad.shape, device="cuda", generator=gen, dtype=torch.float64)

        def loss(t):
            hh = x.double() + res.double() + (t * v if where == "x" else 0)
            return (forward64(hh, w.double() + (t * v if where == "w" else 0), 1e-5)[0] * gy.double()).sum() + (hh * gh.double()).sum()

        slope = ((loss(1e-5) - loss(-1e-5)) / 2e-5).item()
        # the differences' own error is about h^2 of the third derivative and 1e-16 / h of the sum; the gradient's elements have (d + 20) / 2 roundings, h one of its own
        size = (grad.double() * v).abs().sum().item()
        assert abs((grad.double() * v).sum().item() - slope) <= ((d + 20) * EPS + 1e-7) * size + 1e-8


def test_empty_and_refusals(B):
    x = torch.zeros(0, 8, device="cuda")
    y, h, rstd = B.rms_norm(x)
    assert y.shape == (0, 8) and rstd.shape == (0,) and h is x
    codes, scales, _ = B.rms_norm_fp8(x, residual=x)
    assert codes.shape == (0, 8) and scales.shape == (0, 1)
    gx, gw = B.rms_norm_grad(x, x, rstd)
    assert gx.shape == (0, 8) and not bool(gw.any())
    x = torch.ones(4, 8, device="cuda")
    r = torch.ones(4, device="cuda")
    for call in (lambda: B.rms_norm(x.double()), lambda: B.rms_norm(x[0]), lambda: B.rms_norm(x.cpu()), lambda: B.rms_norm(x.t()), lambda: B.rms_norm(x, r), lambda: B.rms_norm(x, residual=x[:3]),
                 lambda: B.rms_norm(x, residual=x.bfloat16()), lambda: B.rms_norm_fp8(x, torch.ones(8, device="cuda").half()), lambda: B.rms_norm_fp8(x.int()),
                 lambda: B.rms_norm_grad(x[:2], x, r), lambda: B.rms_norm_grad(x, x, r[:2]), lambda: B.rms_norm_grad(x, x, r, g_h=x.half()), lambda: B.rms_norm_grad(x, x, r.double()),
                 lambda: B.rms_norm_grad(x, x, r, g_h=x[:, :4])):
        with pytest.raises(ValueError):
            call()
    for eps in (-1.0, float("nan"), float("inf")):
        with pytest.raises(B.HagError):
            B.rms_norm(x, eps=eps)


def test_captured(B):
    gen = torch.Generator(device="cuda").manual_seed(5)
    x, res, gy = (torch.randn(777, 130, device="cuda", generator=gen) for _ in range(3))
    w = weights(130, torch.float32, gen)

    def run():
        y, h, rstd = B.rms_norm(x, w, residual=res)
        return (y, h, *B.rms_norm_fp8(x, w, residual=res)[:2], *B.rms_norm_grad(gy, h, rstd, w, g_h=res))

    run()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = run()
    for _ in range(4):
        x.copy_(torch.randn(777, 130, device="cuda", generator=gen))
        gy.mul_(1.5)
        graph.replay()
        for got, want in zip(outs, run()):
            assert torch.equal(got.view(torch.uint8) if got.element_size() == 1 else got, want.view(torch.uint8) if want.element_size() == 1 else want)
        torch.cuda.synchronize()


def test_on_another_stream(B):
    gen = torch.Generator(device="cuda").manual_seed(6)
    x = torch.randn(50000, 256, device="cuda", generator=gen)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(20):
            x = x * 1.01                                   # work on the stream that the norm has to follow
        got = B.rms_norm(x)
    side.synchronize()
    check_forward(got, x, None, None, 1e-5)
