"""hag_fp8_product at sizes that go through LDS in tiles, one set of 128 columns to nine: rows at multiples of 16 bytes with no numbers behind their ends, remainders in every dimension, all
three types of results."""
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


def placed(t, more, first):
    """t's bytes as rows at multiples of 16 bytes (scales: bytes) of memory that holds no numbers elsewhere."""
    rows, cols = t.shape
    apart = (cols + 15) // 16 * 16 + 16 * more if t.dtype == E4M3 else cols + more
    flat = torch.full((first + rows * apart + 64,), 0x7f if t.dtype == E4M3 else 0xff, dtype=torch.uint8, device="cuda")
    view = flat[first:first + rows * apart].view(rows, apart)[:, :cols]
    view.copy_(t.view(torch.uint8))
    return view.view(t.dtype)


def matrix(n, d, gen, low=-4, high=4):
    """Elements of all sizes, those below 2^-6 among them, scales 2^low .. 2^(high - 1)."""
    codes = (40 * torch.randn(n, d, device="cuda", generator=gen) * torch.exp(torch.randn(n, d, device="cuda", generator=gen))).clamp(-448, 448).to(E4M3)
    return codes, (torch.randint(low, high, (n, (d + 31) // 32), device="cuda", generator=gen) + 127).to(torch.uint8).view(E8M0)


def wide(codes, scales):
    return codes.double() * scales.double().repeat_interleave(32, 1)[:, :codes.shape[1]]


def check(y, x, xs, w, ws, dtype):
    """Products are exact and d of them are added in some order; for 16 bits each may lose 2^-13 of the largest of up to 16 neighbours, elements below 2^-6 of their scale counting as that much."""
    a, b = wide(x, xs), wide(w, ws).t().contiguous()
    want, d = a @ b, x.shape[1]
    if dtype != torch.float32:
        least = [2.0 ** -6 * s.double().repeat_interleave(32, 1)[:, :d] for s in (xs, ws)]
        a, b = torch.maximum(a.abs(), least[0]), torch.maximum(b.abs(), least[1].t()).contiguous()
    size = a.abs() @ b.abs()
    bound = ((d + 2) * EPS + (0.0 if dtype == torch.float32 else 16 * 2.0 ** -13)) * size
    assert y.dtype == dtype and y.shape == want.shape
    assert bool(((y.double() - want).abs() <= bound + HALF[dtype] * (want.abs() + bound) + TINY[dtype]).all())


# up to 64 columns of y; up to 128 and more; and many results, which 16 bits take in larger tiles
SIZES = [(20000, 250, 60), (20000, 300, 33), (9000, 400, 64), (20000, 513, 7), (33000, 16, 64), (25000, 129, 3), (10000, 1100, 50), (15001, 385, 64),
         (9000, 251, 300), (9000, 300, 129), (4000, 1040, 500), (70000, 130, 100), (5003, 1, 200), (6001, 31, 333), (7000, 256, 128), (6144, 512, 384),
         (66000, 200, 260), (66000, 513, 257), (70001, 31, 250), (16400, 1024, 1030), (140000, 16, 129), (66000, 257, 512)]


@pytest.mark.parametrize("n,d,k", SIZES)
def test_product(B, n, d, k):
    gen = torch.Generator(device="cuda").manual_seed(n + d + k)
    (x, xs), (w, ws) = matrix(n, d, gen), matrix(k, d, gen)
    for i, dtype in enumerate(TYPES):
        if dtype == torch.float16:                         # results within its range
            ws = (torch.randint(-16, -12, ws.shape, device="cuda", generator=gen) + 127).to(torch.uint8).view(E8M0)
        args = placed(x, i, 16 * i), placed(xs, i, i), placed(w, 2 * i, 32 * i), placed(ws, 3 * i, 3 - i)
        y = B.fp8_product(*args, dtype=dtype)
        check(y, x, xs, w, ws, dtype)
        for _ in range(3):
            assert torch.equal(y, B.fp8_product(*args, dtype=dtype))


@pytest.mark.parametrize("n,d,k", SIZES)
def test_whole_numbers_are_exact(B, n, d, k):
    """Every column, row and scale has to be where it belongs: sums of products of small whole numbers are exact in fp32 (at most 9 * 16 * 1100 < 2^24, no product below 2^-8 of another)."""
    gen = torch.Generator(device="cuda").manual_seed(n * d + k)
    ints = lambda *s: torch.randint(-3, 4, s, device="cuda", generator=gen).float().to(E4M3)   # noqa: E731
    scale = lambda rows: (torch.randint(127, 130, (rows, (d + 31) // 32), device="cuda", generator=gen)).to(torch.uint8).view(E8M0)   # noqa: E731
    x, w, xs, ws = ints(n, d), ints(k, d), scale(n), scale(k)
    want = wide(x, xs) @ wide(w, ws).t().contiguous()
    args = placed(x, 0, 0), placed(xs, 0, 0), placed(w, 0, 0), placed(ws, 0, 0)
    assert torch.equal(B.fp8_product(*args).double(), want)
    for dtype in TYPES[1:]:
        assert torch.equal(B.fp8_product(*args, dtype=dtype), want.to(dtype))


@pytest.mark.parametrize("n,d,k", [(9000, 300, 60), (9000, 251, 300), (66000, 130, 260)])
def test_elements_that_are_no_numbers_stay_in_their_row(B, n, d, k):
    gen = torch.Generator(device="cuda").manual_seed(n)
    (x, xs), (w, ws) = matrix(n, d, gen, -8, -4), matrix(k, d, gen, -8, -4)
    x, w, xs, ws = placed(x, 0, 0), placed(w, 0, 0), placed(xs, 0, 0), placed(ws, 0, 0)
    clean = [B.fp8_product(x, xs, w, ws, dtype=t) for t in TYPES]
    assert not any(bool(y.isnan().any()) for y in clean)
    x.view(torch.uint8)[n // 2, d - 1] = 0x7f
    x.view(torch.uint8)[n - 1, 0] = 0xff
    w.view(torch.uint8)[k // 3, 0] = 0xff
    ws.view(torch.uint8)[k - 1, (d - 1) // 32] = 0xff
    hit = torch.zeros(n, k, dtype=torch.bool, device="cuda")
    hit[n // 2] = hit[n - 1] = hit[:, k // 3] = hit[:, k - 1] = True
    for t, before in zip(TYPES, clean):
        y = B.fp8_product(x, xs, w, ws, dtype=t)
        assert torch.equal(y.isnan(), hit) and torch.equal(y[~hit], before[~hit])


def test_rows_of_the_norm_and_of_weights(B):
    """As layers serve: rows that the norm leaves, matrices by quantize_fp8, into all three types."""
    from paper_1906_03707_amd import layers
    gen = torch.Generator(device="cuda").manual_seed(9)
    for n, d, k in ((9000, 251, 44), (9000, 300, 300), (66000, 251, 300)):
        codes, scales, _ = B.rms_norm_fp8(torch.randn(n, d, device="cuda", generator=gen).bfloat16())
        w, ws = layers.quantize_fp8(torch.randn(k, d, device="cuda", generator=gen) * d ** -0.5)
        for dtype in TYPES:
            check(B.fp8_product(codes, scales, w, ws, dtype=dtype), codes, scales, w, ws, dtype)


def test_captured_and_on_another_stream(B):
    gen = torch.Generator(device="cuda").manual_seed(2)
    data = []
    for n, d, k in ((9000, 300, 60), (9000, 400, 300), (66000, 160, 260)):
        (x, xs), (w, ws) = matrix(n, d, gen, -8, -4), matrix(k, d, gen, -8, -4)
        data += [(placed(x, 0, 0), xs, placed(w, 0, 0), ws, dtype) for dtype in TYPES]
    run = lambda: [B.fp8_product(*t) for t in data]   # noqa: E731
    run()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = run()
    for _ in range(4):
        for x, _, w, _, _ in data:
            x.view(torch.uint8).copy_(x.view(torch.uint8).roll(1, 0))
        graph.replay()
        assert all(torch.equal(got, want) for got, want in zip(outs, run()))
        torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = run()
    here = run()                                           # two calls at once
    side.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(got, here))
