"""hag_layer_norm and hag_layer_norm_grad against the formulas in 64 bits: widths from one column to more than a workgroup holds, odd ones, views, rows without spread,
gradients by differences, parameter gradients that see a lost row."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
EPS = 2.0 ** -24
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TINY = {torch.float32: 0.0, torch.bfloat16: 0.0, torch.float16: 2.0 ** -25}
TYPES = [torch.float32, torch.bfloat16, torch.float16]
WIDTHS = [1, 2, 3, 4, 7, 8, 16, 31, 36, 64, 100, 127, 128, 130, 251, 256, 260, 500, 512, 513, 777, 1024, 1030, 2048, 2050, 4096, 4099, 8192, 8200, 16500]


@pytest.fixture(scope="module")
def B():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_1906_03707_amd import binding
    binding.lib()
    return binding


def forward64(x, w, b, eps):
    x = x.double()
    m = x.mean(1, keepdim=True)
    r = ((x - m).square().mean(1, keepdim=True) + eps).rsqrt()
    xh = (x - m) * r
    return xh * (1.0 if w is None else w.double()) + (0.0 if b is None else b.double()), m, r, xh


def check_forward(got, x, w, b, eps):
    y, mean, rstd = got
    want, m, r, xh = forward64(x, w, b, eps)
    n, d = x.shape
    # mean: any order of d additions and a division; the deviations are from the mean as it came out
    dm = (d + 2) * EPS * x.double().abs().mean(1, keepdim=True)
    dr = r * ((d + 8) / 2 * EPS + 4 * EPS + (dm * r) ** 2 / 2)
    dxh = r * (dm + EPS * (x.double() - m).abs()) + xh.abs() * dr / r
    dy = dxh * (1.0 if w is None else w.double().abs()) + 3 * EPS * (xh.abs() * (1.0 if w is None else w.double().abs()) + (0.0 if b is None else b.double().abs()))
    dy = dy + HALF[y.dtype] * (want.abs() + dy) + TINY[y.dtype]
    assert y.dtype == x.dtype and mean.shape == rstd.shape == (n,)
    assert bool(((mean.double()[:, None] - m).abs() <= dm).all())
    assert bool(((rstd.double()[:, None] - r).abs() <= dr).all())
    assert bool(((y.double() - want).abs() <= dy).all())


def check_grad(got, gy, x, mean, rstd, w):
    gx, gw, gb = got
    n, d = x.shape
    g, r = gy.double(), rstd.double()[:, None]
    xh = (x.double() - mean.double()[:, None]) * r
    u = g if w is None else g * w.double()
    s1, s2 = u.mean(1, keepdim=True), (u * xh).mean(1, keepdim=True)
    want = r * (u - s1 - xh * s2)
    a1, a2 = u.abs().mean(1, keepdim=True), (u * xh).abs().mean(1, keepdim=True)
    # xh carries two roundings, u one, their sums d additions more; then four operations on terms of these sizes
    bound = r * (6 * EPS * u.abs() + (d + 6) * EPS * a1 + xh.abs() * ((d + 10) * EPS * a2 + 6 * EPS * s2.abs()) + 4 * EPS * s1.abs()) + 2 * EPS * want.abs()
    bound = bound + HALF[gx.dtype] * (want.abs() + bound) + TINY[gx.dtype]
    assert gx.dtype == x.dtype and bool(((gx.double() - want).abs() <= bound).all())
    if gw is None:
        return
    for got_p, terms, extra in ((gw, g * xh, 4), (gb, g, 1)):
        total, size = terms.sum(0), terms.abs().sum(0)
        bound = (n + extra) * EPS * size
        bound = bound + HALF[got_p.dtype] * (total.abs() + bound) + TINY[got_p.dtype]
        assert bool(((got_p.double() - total).abs() <= bound).all())


def params(d, dtype, gen):
    return ((1 + 0.3 * torch.randn(d, device="cuda", generator=gen)).to(dtype), (0.2 * torch.randn(d, device="cuda", generator=gen)).to(dtype))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d", WIDTHS)
def test_norm_and_gradient(B, d, dtype):
    gen = torch.Generator(device="cuda").manual_seed(d)
    for n in (1, 2, 5, 67, 1030) if d < 600 else (1, 3, 130):
        x = (2 * torch.randn(n, d, device="cuda", generator=gen) + torch.randn(n, 1, device="cuda", generator=gen)).to(dtype)
        gy = torch.randn(n, d, device="cuda", generator=gen).to(dtype)
        for w, b in (params(d, torch.float32, gen), params(d, dtype, gen), (None, None)):
            out = B.layer_norm(x, w, b)
            check_forward(out, x, w, b, 1e-5)
            check_grad(B.layer_norm_grad(gy, x, out[1], out[2], w), gy, x, out[1], out[2], w)
    w, b = params(d, torch.float32, gen)
    check_forward(B.layer_norm(x, w, None, eps=0.1), x, w, None, 0.1)
    check_forward(B.layer_norm(x, None, b, eps=0.1), x, None, b, 0.1)
    gx, gw, gb = B.layer_norm_grad(gy, x, out[1], out[2], w, params=False)
    assert gw is None and gb is None
    assert torch.equal(gx, B.layer_norm_grad(gy, x, out[1], out[2], w)[0])
    assert all(torch.equal(p, q) for p, q in zip(B.layer_norm_grad(gy, x, out[1], out[2], w), B.layer_norm_grad(gy, x, out[1], out[2], w)))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,d", [(70001, 16), (40000, 64), (30000, 100), (9001, 250), (5000, 1000), (3001, 3000), (600, 9000)])
def test_parameter_gradients_count_every_row_once(B, n, d, dtype):
    gen = torch.Generator(device="cuda").manual_seed(n)
    x, gy = (torch.randint(-3, 4, (n, d), device="cuda", generator=gen).to(dtype) for _ in range(2))
    zero, one = torch.zeros(n, device="cuda"), torch.ones(n, device="cuda")
    gx, gw, gb = B.layer_norm_grad(gy, x, zero, one)       # with these statistics all terms are whole numbers, their sums exact in fp32
    assert torch.equal(gw.double(), (gy.double() * x.double()).sum(0)) and torch.equal(gb.double(), gy.double().sum(0))
    check_grad((gx, None, None), gy, x, zero, one, None)


@pytest.mark.parametrize("n,d", [(3, 5), (40, 64), (7, 333), (2, 5000)])
def test_gradient_by_differences(B, n, d):
    gen = torch.Generator(device="cuda").manual_seed(d)
    x, gy = (torch.randn(n, d, device="cuda", generator=gen) for _ in range(2))
    w, b = params(d, torch.float32, gen)
    _, mean, rstd = B.layer_norm(x, w, b)
    grads = B.layer_norm_grad(gy, x, mean, rstd, w)
    for k, (grad, where) in enumerate(zip(grads, (x, w, b))):
        v = torch.randn(where.shape, device="cuda", generator=gen, dtype=torch.float64)
        h = 1e-5

        def loss(t):
            moved = [p.double() + t * v if k == j else p.double() for j, p in enumerate((x, w, b))]
            return (forward64(*moved, 1e-5)[0] * gy.double()).sum()

        slope = ((loss(h) - loss(-h)) / (2 * h)).item()
        # the differences' own error is about h^2 of the third derivative and 1e-16 / h of the sum; the gradient's elements have a few dozen roundings
        size = (grad.double().abs() * v.abs()).sum().item() + (gy.double().abs().sum() * 1e-6).item()
        assert abs((grad.double() * v).sum().item() - slope) <= (d + n + 40) * EPS * size + 1e-8 * gy.double().abs().sum().item()


def test_views(B):
    gen = torch.Generator(device="cuda").manual_seed(9)
    for dtype in TYPES:
        wide, other = (torch.randn(300, 75, device="cuda", generator=gen).to(dtype) for _ in range(2))
        for cut in (lambda t: t[:, 2:70], lambda t: t[::3, 1:9], lambda t: t[4:5].expand(300, 75), lambda t: t[:, 74:], lambda t: t[1:], lambda t: t[:, :64]):
            x, gy = cut(wide), cut(other)
            w, b = params(x.shape[1] + 1, torch.float32, gen)
            w, b = w[1:], b[1:]
            out = B.layer_norm(x, w, b)
            check_forward(out, x, w, b, 1e-5)
            check_grad(B.layer_norm_grad(gy, x, out[1], out[2], w), gy, x, out[1], out[2], w)


def test_rows_without_spread_and_of_what_is_no_number(B):
    for d in (1, 5, 64, 300, 5000):
        x = torch.full((4, d), 3.25, device="cuda")
        x[1] = 0
        x[2] = 1e30                                        # far beyond where squares are finite: of the deviations, which are 0
        w, b = torch.full((d,), 2.0, device="cuda"), torch.full((d,), -1.5, device="cuda")
        y, mean, rstd = B.layer_norm(x, w, b)
        assert torch.equal(y, torch.full_like(y, -1.5)) and torch.equal(mean, x[:, 0])
        assert bool(((rstd.double() - 1e-5 ** -0.5).abs() <= 8 * EPS * 1e-5 ** -0.5).all())
        x = torch.randn(6, d, device="cuda")
        clean = B.layer_norm(x, w, b)
        x[1, 0], x[3, d - 1], x[4, 0] = float("nan"), float("inf"), float("-inf")
        y, mean, rstd = B.layer_norm(x, w, b)
        for got, want in zip((y, mean, rstd), clean):
            assert torch.equal(got[[0, 2, 5]], want[[0, 2, 5]])                    # other rows do not see it
        assert bool(torch.isnan(y[[1, 3, 4]]).all())
        gy = torch.randn(6, d, device="cuda")
        gx = B.layer_norm_grad(gy, x, mean, rstd, w)[0]
        assert bool(torch.isfinite(gx[[0, 2, 5]]).all()) and bool(torch.isnan(gx[[1, 3, 4]]).all())
    # large offsets: the deviations are taken from the mean before they are squared
    x = 1000.0 + torch.randn(50, 256, device="cuda")
    check_forward(B.layer_norm(x), x, None, None, 1e-5)


def test_nothing(B):
    x = torch.zeros(0, 12, device="cuda")
    y, mean, rstd = B.layer_norm(x)
    assert y.shape == (0, 12) and mean.shape == (0,)
    gx, gw, gb = B.layer_norm_grad(x, x, mean, rstd)
    assert gx.shape == (0, 12) and not bool(gw.any()) and not bool(gb.any())


def test_past_32_bits(B):
    n, d = 1100000, 2000                                   # 2.2e9 elements
    x = torch.empty(n, d, device="cuda", dtype=torch.bfloat16)
    gen = torch.Generator(device="cuda").manual_seed(1)
    ends = [0, 1, n // 2, n - 2, n - 1]
    x.zero_()
    for i in ends:
        x[i] = torch.randn(d, device="cuda", generator=gen).bfloat16()
    y, mean, rstd = B.layer_norm(x)
    check_forward((y[ends], mean[ends], rstd[ends]), x[ends], None, None, 1e-5)
    del y
    gx, gw, gb = B.layer_norm_grad(x, x, mean, rstd)
    check_grad((gx[ends], None, None), x[ends], x[ends], mean[ends], rstd[ends], None)
    check_grad((gx[ends], gw, gb), x[ends], x[ends], mean[ends], rstd[ends], None)                       # all other rows are zero


def test_on_another_stream_and_captured(B):
    gen = torch.Generator(device="cuda").manual_seed(4)
    for n, d in ((7, 40), (5000, 64), (300, 5000)):
        x, gy = (torch.randn(n, d, device="cuda", generator=gen) for _ in range(2))
        w, b = params(d, torch.float32, gen)

        def both():
            out = B.layer_norm(x, w, b)
            return *out, *B.layer_norm_grad(gy, x, out[1], out[2], w)

        want = both()
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            got = both()
        torch.cuda.current_stream().wait_stream(side)
        assert all(torch.equal(p, q) for p, q in zip(got, want))
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            got = both()
        for _ in range(4):
            x.copy_(torch.randn(n, d, device="cuda", generator=gen))
            gy.copy_(torch.randn(n, d, device="cuda", generator=gen))
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(p, q) for p, q in zip(got, both()))
            torch.cuda.synchronize()


def test_refusals(B):
    x, w = torch.randn(6, 8, device="cuda"), torch.ones(8, device="cuda")
    y, mean, rstd = B.layer_norm(x, w)
    for call in (lambda: B.layer_norm(x.cpu()), lambda: B.layer_norm(x.double()), lambda: B.layer_norm(x.t()), lambda: B.layer_norm(x, w[:7]), lambda: B.layer_norm(x, w.half()),
                 lambda: B.layer_norm(x.half(), w.half(), w), lambda: B.layer_norm(x, w.cpu()), lambda: B.layer_norm(x[0]), lambda: B.layer_norm(x, torch.ones(16, device="cuda")[::2]),
                 lambda: B.layer_norm_grad(x[:5], x, mean, rstd), lambda: B.layer_norm_grad(x.half(), x, mean, rstd), lambda: B.layer_norm_grad(x, x, mean[:5], rstd),
                 lambda: B.layer_norm_grad(x, x, mean, rstd.double()), lambda: B.layer_norm_grad(x, x, mean, rstd, w[None])):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: B.layer_norm(x[:, :0]), lambda: B.layer_norm(x, eps=-1.0), lambda: B.layer_norm(x, eps=float("nan"))):
        with pytest.raises(B.HagError) as err:
            call()
        assert err.value.code == B.HAG_EINVAL


@pytest.mark.parametrize("d", [2, 16, 100, 251, 512, 1000, 1500, 4096, 8192, 16500])
def test_rows_that_are_not_around_their_first_element(B, d):
    gen = torch.Generator(device="cuda").manual_seed(d)
    # a sum's path to a lane's result, through the lanes and through the wavefronts has no more than 40 additions (of more than 8192 columns: and one for each 1024)
    depth = 40 + (d // 1024 if d > 8192 else 0)
    for dtype, large in ((torch.float32, 1e4), (torch.float32, -3e6), (torch.bfloat16, 1e4), (torch.float16, 6e4)):
        x = torch.randn(40, d, device="cuda", generator=gen).to(dtype)
        x[:30, 0] = large
        x[10:20, 1:] -= 50
        x64 = x.double()
        m = x64.mean(1)
        size = (x64 - m[:, None]).abs().mean(1)
        mean = B.layer_norm(x)[1].double()
        # the deviations' roundings, their sum's, the mean's own
        assert bool(((mean - m).abs() <= (depth + 3) * EPS * size + 2 * EPS * m.abs()).all())


@pytest.mark.parametrize("d", [2, 8, 64, 250, 1000, 4098, 9000])
def test_rows_whose_mean_is_no_fp32_number(B, d):
    for low, step in ((1e8, 8.0), (-1e8, 8.0), (2.0 ** 64, 2.0 ** 41), (2.0 ** 24, 2.0)):   # two neighbours in fp32
        x = torch.full((3, d), low, device="cuda")
        x[:, 1::2] += step
        x[2] = x[2].flip(0)
        y, mean, rstd = B.layer_norm(x, eps=0.0)
        want = torch.ones(3, d, device="cuda", dtype=torch.float64)
        want[:2, ::2] = -1
        want[2, 1::2] = -1
        # sums of steps and of their squares, exact; 1 / d, its products with them, the variance, its reciprocal root (half of them), the deviations and their product
        assert bool(((y.double() - want).abs() <= 12 * EPS).all()) and bool(((rstd.double() * step / 2 - 1).abs() <= 8 * EPS).all())
        assert bool(((mean.double() - (x.double()[:, 0] + x.double()[:, 1]) / 2).abs() <= step / 2).all())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("d", [2, 7, 16, 64, 130, 512, 777, 1024, 1500, 4100, 8192, 9001])
def test_rows_whose_squares_are_no_fp32_numbers(B, d, dtype):
    gen = torch.Generator(device="cuda").manual_seed(d)
    z = torch.randn(12, d, device="cuda", generator=gen)
    near = torch.cat([z[:3], 3 * z[3:6] + 1])              # ordinary rows beside them, which must not change
    x = torch.cat([near, 1e19 * z[:2], 1e25 * z[2:4], 1e30 + 1e29 * z[4:6], 6e37 * z[6:8].clamp(-5, 5), 3e38 * z[8:10].sign(), 1e36 * z[10:12].sign()]).to(dtype)
    x = torch.cat([x, torch.tensor([[float("inf")], [float("nan")], [3.3e38]], device="cuda").to(dtype).expand(3, d)])
    x[-3, 1:], x[-2, 0] = 1, 1
    w, b = params(d, torch.float32, gen)
    y, mean, rstd = B.layer_norm(x, w, b)
    assert all(torch.equal(p[:6], q) for p, q in zip((y, mean, rstd), B.layer_norm(x[:6], w, b)))
    assert bool(torch.isnan(y[-3:-1]).all()) and torch.equal(y[-1], b.to(dtype))
    x, y, mean, rstd = x[:-3], y[:-3], mean[:-3], rstd[:-3]
    x64 = x.double()
    want, m, r, xh = forward64(x, w, b, 1e-5)
    depth = 40 + (d // 1024 if d > 8192 else 0)            # additions on the way of a term into a row's sum
    size = (x64 - m).abs().mean(1, keepdim=True)
    dm = (depth + 3) * EPS * size + 2 * EPS * m.abs()
    assert bool(((mean.double()[:, None] - m).abs() <= dm).all())
    dr = (depth / 2 + 8) * EPS * r                         # squares and their sum, by half; the root; below 2^-126 the grid of small numbers
    assert bool(((rstd.double()[:, None] - r).abs() <= dr + 2.0 ** -150).all())
    # the deviations' mean is taken out of them, so their error is that of its sum
    dxh = r * (depth + 4) * EPS * (size + (x64 - m).abs()) + xh.abs() * dr / r
    dy = dxh * w.double().abs() + 3 * EPS * (xh.abs() * w.double().abs() + b.double().abs())
    assert bool(((y.double() - want).abs() <= dy + HALF[dtype] * (want.abs() + dy)).all())
    gy = torch.randn(x.shape, device="cuda", generator=gen).to(dtype)
    gx, gw, gb = B.layer_norm_grad(gy, x, mean, rstd, w)
    assert bool(torch.isfinite(gx).all()) and bool(torch.isfinite(gw).all())
    check_grad((gx[:8], None, None), gy[:8], x[:8], mean[:8], rstd[:8], w)
    xh = (x64 - mean.double()[:, None]) * rstd.double()[:, None]
    terms = gy.double() * xh
    assert bool(((gw.double() - terms.sum(0)).abs() <= (len(x) + 4) * EPS * terms.abs().sum(0)).all())
