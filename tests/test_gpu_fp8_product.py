"""hag_fp8_product against 64 bits: one row to many, odd sizes of every dimension, strides and addresses that suit a byte only, whole numbers that have to come out exactly, scales at their ends,
elements that are no numbers."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
EPS = 2.0 ** -24
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TINY = {torch.float32: 2.0 ** -150, torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25}
TYPES = [torch.float32, torch.bfloat16, torch.float16]
E4M3, E8M0 = torch.float8_e4m3fn, torch.float8_e8m0fnu


@pytest.fixture(scope="module")
def B():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_1906_03707_amd import binding
    binding.lib()
    return binding


def matrix(n, d, gen, low=-4, high=4):
    """Elements of all sizes, scales 2^low .. 2^(high - 1)."""
    codes = (40 * torch.randn(n, d, device="cuda", generator=gen) * torch.exp(torch.randn(n, d, device="cuda", generator=gen))).clamp(-448, 448).to(E4M3)
    scales = (torch.randint(low, high, (n, (d + 31) // 32), device="cuda", generator=gen) + 127).to(torch.uint8).view(E8M0)
    return codes, scales


def wide(codes, scales):
    return codes.double() * scales.double().repeat_interleave(32, 1)[:, :codes.shape[1]]


def check(y, x, xs, w, ws, dtype):
    a, b = wide(x, xs), wide(w, ws).t().contiguous()
    want, size = a @ b, a.abs() @ b.abs()
    # products are exact, any order of d additions; results of 16 bits: every product may have been cut off at 2^-14 of the largest of up to 16 neighbours, which is less than their sum of sizes
    bound = (x.shape[1] + 2) * EPS * size + (0.0 if dtype == torch.float32 else 16 * 2.0 ** -14 * size)
    assert y.dtype == dtype and y.shape == want.shape
    assert bool(((y.double() - want).abs() <= bound + HALF[dtype] * (want.abs() + bound) + TINY[dtype]).all())


SIZES = [(1, 1, 1), (1, 512, 512), (1, 33, 2000), (2, 7, 5), (3, 2048, 100), (15, 31, 17), (16, 32, 16), (17, 33, 15), (31, 64, 300), (33, 100, 47), (64, 128, 64), (65, 129, 65), (74, 64, 44), (100, 1000, 257),
         (127, 160, 128), (128, 256, 130), (129, 251, 74), (255, 96, 511), (257, 384, 256), (300, 512, 513), (1000, 777, 129), (1500, 128, 44), (2111, 1024, 640), (5000, 40, 16), (20000, 250, 60), (70000, 64, 9)]


@pytest.mark.parametrize("n,d,k", SIZES)
def test_product(B, n, d, k):
    gen = torch.Generator(device="cuda").manual_seed(n + d + k)
    (x, xs), (w, ws) = matrix(n, d, gen), matrix(k, d, gen)
    for dtype in TYPES:
        if dtype == torch.float16:                         # results within its range
            ws = (torch.randint(-16, -12, ws.shape, device="cuda", generator=gen) + 127).to(torch.uint8).view(E8M0)
        y = B.fp8_product(x, xs, w, ws, dtype=dtype)
        check(y, x, xs, w, ws, dtype)
        assert torch.equal(y, B.fp8_product(x, xs, w, ws, dtype=dtype))
    assert B.fp8_product(x, xs, w, ws).dtype == torch.float32


@pytest.mark.parametrize("n,d,k", SIZES)
def test_whole_numbers_are_exact(B, n, d, k):
    """Every column, row and scale has to be where it belongs: sums of products of small whole numbers are exact in fp32."""
    gen = torch.Generator(device="cuda").manual_seed(n * d + k)
    ints = lambda *s: torch.randint(-3, 4, s, device="cuda", generator=gen).float().to(E4M3)   # noqa: E731
    scale = lambda rows: (torch.randint(127, 130, (rows, (d + 31) // 32), device="cuda", generator=gen)).to(torch.uint8).view(E8M0)   # noqa: E731
    x, w, xs, ws = ints(n, d), ints(k, d), scale(n), scale(k)          # at most 9 * 16 * 2048 < 2^24, and no product is below 2^-8 of another
    want = wide(x, xs) @ wide(w, ws).t().contiguous()
    assert torch.equal(B.fp8_product(x, xs, w, ws).double(), want)
    assert torch.equal(B.fp8_product(x, xs, w, ws, dtype=torch.bfloat16), want.bfloat16())


@pytest.mark.parametrize("n,d,k", [(1, 300, 70), (5, 64, 40), (40, 128, 100), (150, 200, 90), (700, 512, 300), (900, 31, 5)])
@pytest.mark.parametrize("pad,start", [(0, 0), (1, 0), (16, 0), (16, 1), (48, 16), (5, 3)])
def test_strides_and_addresses(B, n, d, k, pad, start):
    """Rows anywhere in memory; what lies beside them is no number, and none of it may count."""
    gen = torch.Generator(device="cuda").manual_seed(d + pad)

    def placed(t, more, first):
        rows, cols = t.shape
        flat = torch.full((first + rows * (cols + more),), 0x7f if t.dtype == E4M3 else 0xff, dtype=torch.uint8, device="cuda")
        view = flat[first:].view(rows, cols + more)[:, :cols]
        view.copy_(t.view(torch.uint8))
        return view.view(t.dtype)

    (x, xs), (w, ws) = matrix(n, d, gen), matrix(k, d, gen)
    for dtype in (torch.float32, torch.bfloat16):
        y = B.fp8_product(placed(x, pad, start), placed(xs, pad % 7, start % 3), placed(w, pad, start), placed(ws, pad % 5, start), dtype=dtype)
        check(y, x, xs, w, ws, dtype)
        # (rows at multiples of 16 bytes and others may be added up in another order: either is within the bound, so nothing says that their last bits are the same)
        check(B.fp8_product(x, xs, w, ws, dtype=dtype), x, xs, w, ws, dtype)
    row = x[:1].expand(n, d), xs[:1].expand(n, xs.shape[1])           # one row throughout
    check(B.fp8_product(*row, w, ws), *row, w, ws, torch.float32)


def test_every_element_and_scale(B):
    """All 256 elements against 1; scales from one end to the other where the result is an fp32 number."""
    codes = torch.arange(256, device="cuda", dtype=torch.uint8)
    x = codes[:, None].view(E4M3)
    one, unit = torch.ones(1, 1, device="cuda").to(E4M3), torch.full((1, 1), 127, dtype=torch.uint8, device="cuda").view(E8M0)
    y = B.fp8_product(x, unit.expand(256, 1), one, unit)[:, 0]
    want = x[:, 0].float()
    assert torch.equal(y.isnan(), want.isnan()) and torch.equal(y[~want.isnan()], want[~want.isnan()]) and int(want.isnan().sum()) == 2
    scales = torch.arange(255, device="cuda", dtype=torch.uint8)[:, None]
    none = torch.full((1, 1), 255, dtype=torch.uint8, device="cuda").view(E8M0)
    for dtype in (torch.float32, torch.bfloat16):
        y = B.fp8_product(one.expand(255, 1), scales.view(E8M0), one.expand(255, 1), (254 - scales).view(E8M0), dtype=dtype).diagonal()
        assert bool((y[1:-1] == 1).all()) and all(v in (0.0, 1.0) for v in (y[0].item(), y[-1].item()))          # 2^-127 is below the ordinary numbers and may count as none
        y = B.fp8_product(one.expand(255, 1), scales.view(E8M0), one, unit, dtype=dtype)[:, 0]
        assert torch.equal(y[1:].double(), torch.exp2(torch.arange(1, 255, device="cuda").double() - 127)) and y[0].item() in (0.0, 2.0 ** -127)
        assert bool(B.fp8_product(one, none, one, unit, dtype=dtype).isnan().all()) and bool(B.fp8_product(one, unit, one, none, dtype=dtype).isnan().all())


@pytest.mark.parametrize("n,d,k", [(3, 200, 40), (200, 300, 130), (1100, 128, 70)])
def test_elements_that_are_no_numbers_stay_in_their_row(B, n, d, k):
    gen = torch.Generator(device="cuda").manual_seed(n)
    (x, xs), (w, ws) = matrix(n, d, gen), matrix(k, d, gen)
    types = (torch.float32, torch.bfloat16)
    clean = [B.fp8_product(x, xs, w, ws, dtype=t) for t in types]
    x.view(torch.uint8)[n // 2, d - 1] = 0x7f
    w.view(torch.uint8)[k // 3, 0] = 0xff
    hit = torch.zeros(n, k, dtype=torch.bool, device="cuda")
    hit[n // 2] = hit[:, k // 3] = True
    for t, before in zip(types, clean):
        y = B.fp8_product(x, xs, w, ws, dtype=t)
        assert torch.equal(y.isnan(), hit) and torch.equal(y[~hit], before[~hit])


def test_after_the_norm(B):
    """What the norm leaves in 8 bits, times weights: the whole way against 64 bits of the 8-bit values."""
    gen = torch.Generator(device="cuda").manual_seed(9)
    for d in (64, 251):
        x = torch.randn(3000, d, device="cuda", generator=gen).bfloat16()
        codes, scales, _ = B.rms_norm_fp8(x)
        w, ws = matrix(48, d, gen)
        check(B.fp8_product(codes, scales, w, ws), codes, scales, w, ws, torch.float32)


def test_empty_and_refusals(B):
    gen = torch.Generator(device="cuda").manual_seed(1)
    (x, xs), (w, ws) = matrix(4, 40, gen), matrix(3, 40, gen)
    assert B.fp8_product(x[:0], xs[:0], w, ws).shape == (0, 3) and B.fp8_product(x, xs, w[:0], ws[:0]).shape == (4, 0)
    for call in (lambda: B.fp8_product(x.float(), xs, w, ws), lambda: B.fp8_product(x, xs.float(), w, ws), lambda: B.fp8_product(x, xs[:, :1], w, ws), lambda: B.fp8_product(x, xs[:2], w, ws),
                 lambda: B.fp8_product(x, xs, w[:, :39], ws), lambda: B.fp8_product(x.t(), xs, w, ws), lambda: B.fp8_product(x, xs, w, ws, dtype=torch.float64), lambda: B.fp8_product(x, xs, w, ws, dtype=torch.int32),
                 lambda: B.fp8_product(x.cpu(), xs.cpu(), w, ws), lambda: B.fp8_product(x[0], xs[0], w, ws), lambda: B.fp8_product(x[:, ::2], xs[:, :1], w[:, :20], ws[:, :1])):
        with pytest.raises(ValueError):
            call()


def test_captured_and_on_another_stream(B):
    gen = torch.Generator(device="cuda").manual_seed(2)
    sizes = [(1, 700, 300), (50, 260, 90), (900, 128, 64)]
    data = [(*matrix(n, d, gen), *matrix(k, d, gen)) for n, d, k in sizes]
    run = lambda: [B.fp8_product(*t) for t in data]   # noqa: E731
    run()
    graph, second = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = run()
    with torch.cuda.graph(second):                         # two captured passes have workspaces of their own
        others = run()
    for _ in range(4):
        for x, _, w, _ in data:
            x.view(torch.uint8).copy_(x.view(torch.uint8).roll(1, 0))
        graph.replay()
        second.replay()
        for got, other, want in zip(outs, others, run()):
            assert torch.equal(got, want) and torch.equal(other, want)
        torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = run()
    here = run()                                           # two calls at once
    side.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(got, here))


@pytest.mark.parametrize("n,d,k", [(130, 1, 70), (200, 3, 1900), (40, 8, 40), (17, 33, 300), (300, 128, 300), (700, 300, 900)])
def test_small_elements_beside_large_ones(B, n, d, k):
    """Codes of all sizes, those without a leading bit among them: they count as 2^-6 of their scale where products of 16 bits' results are cut off, and are exact for fp32."""
    gen = torch.Generator(device="cuda").manual_seed(n)

    def codes(rows):
        c = torch.randint(0, 256, (rows, (d + 15) // 16 * 16), dtype=torch.uint8, device="cuda", generator=gen)
        c = torch.where(torch.rand(c.shape, device="cuda", generator=gen) < 0.3, c & 0x87, c)          # below 2^-6
        c = torch.where((c & 0x7f) == 0x7f, c - 7, c)
        return c.view(E4M3)[:, :d], torch.randint(118, 122, (rows, (d + 31) // 32), dtype=torch.uint8, device="cuda", generator=gen).view(E8M0)

    (x, xs), (w, ws) = codes(n), codes(k)
    check(B.fp8_product(x, xs, w, ws), x, xs, w, ws, torch.float32)
    a, b = wide(x, xs), wide(w, ws).t().contiguous()
    want = a @ b
    least = [2.0 ** -6 * s.double().repeat_interleave(32, 1)[:, :d] for s in (xs, ws)]
    size = torch.maximum(a.abs(), least[0]) @ torch.maximum(b.abs(), least[1].t()).contiguous()
    # each of up to 16 neighbours may lose 2^-13 of the largest of them, which is less than the sum of their sizes
    bound = ((d + 2) * EPS + 16 * 2.0 ** -13) * size
    for dtype in (torch.bfloat16, torch.float16):
        y = B.fp8_product(x, xs, w, ws, dtype=dtype).double()
        assert bool(((y - want).abs() <= bound + HALF[dtype] * (want.abs() + bound) + TINY[dtype])[want.abs() + bound < 60000].all())
