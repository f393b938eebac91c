"""hag_embedding and hag_embedding_grad against 64-bit sums: widths and addresses of every alignment, ids that repeat from once to all the time, that are padding
or no row, lists of ids from none to more than one workgroup sorts."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
EPS = 2.0 ** -24                                           # half a unit in the last place, relative, of fp32 ...
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}   # ... and of each type
TINY = {torch.float32: 0.0, torch.bfloat16: 0.0, torch.float16: 2.0 ** -25}                # half the spacing of its subnormal numbers
TYPES = [torch.float32, torch.bfloat16, torch.float16]


@pytest.fixture(scope="module")
def B():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_1906_03707_amd import binding
    binding.lib()
    return binding


def make_ids(n, rows, kind, gen, dtype=torch.int64):
    u = torch.rand(n, device="cuda", generator=gen, dtype=torch.float64)
    if kind == "skew":                                     # the number of the row grows exponentially: a few rows are named most of the time
        ids = ((rows + 1.0) ** u - 1).long().clamp_(0, rows - 1)
    elif kind == "one":
        ids = torch.full((n,), rows // 2, device="cuda")
    else:
        ids = (u * rows).long().clamp_(0, rows - 1)
    return ids.to(dtype)


def reference_grad(gy, ids, rows, scale, padding):
    """(sum, sum of magnitudes, number of terms) in 64 bits, added up on the CPU."""
    kept = (ids >= 0) & (ids < rows)
    if padding is not None:
        kept &= ids != padding
    at, g = ids[kept].long().cpu(), gy[kept].cpu().double() * scale
    total, size = (torch.zeros(rows, gy.shape[1], dtype=torch.float64) for _ in range(2))
    return total.index_add_(0, at, g).cuda(), size.index_add_(0, at, g.abs()).cuda(), torch.bincount(at, minlength=rows)[:, None].cuda()


def check_grad(got, gy, ids, rows, scale, padding):
    want, size, terms = reference_grad(gy, ids, rows, scale, padding)
    # any order of fp32 additions, the scale (rounded, and its product), the result's rounding
    bound = (terms + 3) * EPS * size + HALF[got.dtype] * (want.abs() + (terms + 3) * EPS * size) + TINY[got.dtype]
    assert bool(((got.double() - want).abs() <= bound).all())
    assert not bool(got[terms[:, 0] == 0].any())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,rows,d", [(1, 1, 1), (1, 5, 16), (3, 2, 7), (74, 74, 64), (65, 300, 37), (1000, 41, 250), (5000, 100, 8), (77, 1000, 513), (9, 4, 2049), (4097, 70000, 100)])
def test_lookup(B, n, rows, d, dtype):
    gen = torch.Generator(device="cuda").manual_seed(n + d)
    table = torch.randn(rows, d, device="cuda", generator=gen).to(dtype)
    for id_dtype in (torch.int64, torch.int32):
        ids = make_ids(n, rows, "even", gen, id_dtype)
        ids[::3] = -1
        for scale, padding in ((1.0, -1), (0.37, -1), (-2.5, int(ids[-1]))):
            want = (table[ids.long().clamp(min=0)].float() * scale).to(dtype)
            want[(ids < 0)] = float("nan")                 # no row of the table, unless it is the padding
            want[ids == padding] = 0
            got = B.embedding(table, ids, scale, padding)
            assert got.dtype == dtype and torch.equal(torch.nan_to_num(got, 9e4), torch.nan_to_num(want, 9e4))   # one rounding each: the same bits


def test_lookup_of_strided_tables_and_shaped_ids(B):
    gen = torch.Generator(device="cuda").manual_seed(5)
    for dtype in TYPES:
        wide = torch.randn(50, 41, device="cuda", generator=gen).to(dtype)
        ids = torch.randint(0, 50, (6, 1, 7), device="cuda", generator=gen)
        for table in (wide[:, 3:20], wide[::2, 1:], wide[:1].expand(50, 41), wide[:, 40:]):
            want = table[(ids % table.shape[0])]
            assert torch.equal(B.embedding(table, ids % table.shape[0]), want)
    for bad in (2 ** 40, -2 ** 40, 2 ** 32 + 3, 50):
        assert bool(torch.isnan(B.embedding(wide, torch.full((2,), bad, device="cuda"))).all())
    table = torch.full((3, 5), float("inf"), device="cuda")
    assert not bool(B.embedding(table, torch.full((4,), 1, device="cuda"), padding=1).any())          # zeros, whatever the table holds there
    assert B.embedding(table, torch.zeros(0, device="cuda", dtype=torch.int64)).shape == (0, 5)
    assert bool(torch.isnan(B.embedding(table[:0], torch.zeros(2, device="cuda", dtype=torch.int64))).all())


def test_lookup_past_32_bits(B):
    rows, d = 70000, 33000                                 # 2.3e9 elements
    table = torch.empty(rows, d, device="cuda", dtype=torch.bfloat16)
    table[-3:] = torch.randn(3, d, device="cuda").bfloat16()
    table[0] = 1
    ids = torch.tensor([rows - 1, 0, rows - 3], device="cuda")
    assert torch.equal(B.embedding(table, ids), table[ids])
    del table
    gy = torch.randn(2, 4, device="cuda")
    far = torch.tensor([2 ** 31 - 3, 5], device="cuda")    # as many rows as there may be: sizes are checked, nothing of that size is made
    with pytest.raises((B.HagError, RuntimeError)):
        B.embedding_grad(gy, far, 2 ** 31)


@pytest.mark.parametrize("kind", ["even", "skew", "one"])
@pytest.mark.parametrize("n,rows,d", [(1, 1, 1), (1, 700, 5), (2, 3, 64), (63, 64, 3), (64, 10, 16), (65, 7, 37), (256, 1000, 64), (257, 74, 33), (1000, 5, 130), (1025, 4096, 20),
                                      (4096, 300, 64), (4097, 40, 96), (8191, 70000, 4), (8193, 1024, 65), (16385, 1025, 8), (50000, 74, 64), (70001, 12, 31), (33000, 1 << 20, 4),
                                      (20000, 3000001, 3), (300, 200, 1030), (5000, 100, 1025), (200001, 9000, 16), (2048, 33, 64), (2049, 33, 64), (8192, 3, 32), (8193, 5000, 16), (4100, 200000, 12),
                                      (16384, 900, 20), (16385, 900, 20), (600000, 2000, 4)])
def test_gradient(B, n, rows, d, kind):
    gen = torch.Generator(device="cuda").manual_seed(n + rows + d)
    ids = make_ids(n, rows, kind, gen)
    ids[3::7] = -1
    gy = torch.randn(n, d, device="cuda", generator=gen)
    got = B.embedding_grad(gy, ids, rows, 1.5, -1)
    assert got.shape == (rows, d) and got.dtype == torch.float32
    check_grad(got, gy, ids, rows, 1.5, -1)
    assert torch.equal(got, B.embedding_grad(gy, ids.int(), rows, 1.5, -1))        # the same bits, with ids of either type
    assert torch.equal(got, B.embedding_grad(gy, torch.where(ids == -1, rows + 11, ids), rows, 1.5))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("n,rows,d", [(1, 3, 1), (100, 50, 37), (3000, 700, 128), (30000, 74, 64), (30000, 20000, 9), (12345, 501, 257)])
def test_gradient_of_half_precision(B, n, rows, d, dtype):
    gen = torch.Generator(device="cuda").manual_seed(n)
    ids = make_ids(n, rows, "skew", gen)
    ids[::9] = rows - 1
    gy = torch.randn(n, d, device="cuda", generator=gen).to(dtype)
    for padding in (None, rows - 1, 0):
        for out in (None, torch.float32):
            got = B.embedding_grad(gy, ids, rows, 0.125, padding, dtype=out)
            assert got.dtype == (out or dtype)
            check_grad(got, gy, ids, rows, 0.125, padding)


@pytest.mark.parametrize("n,rows,d", [(200, 31, 12), (70000, 31, 12), (70000, 40000, 8), (6000, 31, 132)])
def test_gradient_counts_every_token_once(B, n, rows, d):
    gen = torch.Generator(device="cuda").manual_seed(1)
    ids = make_ids(n, rows, "skew", gen)
    gy = torch.randint(-3, 4, (n, d), device="cuda", generator=gen).float()
    want = torch.zeros(rows, d, device="cuda", dtype=torch.float64).index_add_(0, ids, gy.double())
    assert torch.equal(B.embedding_grad(gy, ids, rows).double(), want)             # whole numbers below 2^24: exact in any order


def test_gradient_past_32_bits(B):
    n, rows, d = 33000, 33000, 70000                       # 2.3e9 elements on both sides
    gy = torch.zeros(n, d, device="cuda", dtype=torch.bfloat16)
    ids = torch.arange(n, device="cuda")
    ids[:3], ids[-1] = rows - 1, 7
    for i in (0, 2, n - 2, n - 1):
        gy[i] = (torch.arange(d, device="cuda") % 50 + i % 7).bfloat16()
    got = B.embedding_grad(gy, ids, rows)
    assert torch.equal(got[rows - 1], gy[0] + gy[2]) and torch.equal(got[7], gy[n - 1]) and torch.equal(got[n - 2], gy[n - 2])
    assert int(got.count_nonzero()) == sum(int(got[i].count_nonzero()) for i in (7, n - 2, rows - 1))


def test_gradient_of_views(B):
    gen = torch.Generator(device="cuda").manual_seed(2)
    for dtype in TYPES:
        wide = torch.randn(1200, 45, device="cuda", generator=gen).to(dtype)
        for gy in (wide[:, 2:43], wide[::3, 1:8], wide[5:6].expand(1200, 45), wide[:, 44:], wide[1:]):
            ids = make_ids(gy.shape[0], 90, "skew", gen)
            check_grad(B.embedding_grad(gy, ids, 90, 2.0), gy, ids, 90, 2.0, None)


def test_gradient_of_nothing_and_of_what_is_no_number(B):
    none = torch.zeros(0, device="cuda", dtype=torch.int64)
    assert not bool(B.embedding_grad(torch.zeros(0, 6, device="cuda"), none, 9).any())
    assert B.embedding_grad(torch.ones(2, 6, device="cuda"), none.new_zeros(2), 0).shape == (0, 6)
    for n in (90, 9000):
        gen = torch.Generator(device="cuda").manual_seed(n)
        ids, gy = make_ids(n, 40, "even", gen), torch.randn(n, 20, device="cuda", generator=gen)
        assert not bool(B.embedding_grad(gy, torch.full_like(ids, 7), 40, padding=7).any())            # nothing but padding
        ids[5], ids[6] = 11, 12
        want = B.embedding_grad(gy, ids, 40, padding=3)
        gy[ids == 3] = float("nan")
        gy[5, 2], gy[6, 4] = float("nan"), float("inf")
        got = B.embedding_grad(gy, ids, 40, padding=3)
        assert bool(torch.isnan(got[11, 2])) and got[12, 4] == float("inf")
        got[11, 2], got[12, 4] = want[11, 2], want[12, 4]
        assert torch.equal(got, want)                      # and nothing else


def test_on_another_stream_and_captured(B):
    gen = torch.Generator(device="cuda").manual_seed(4)
    for n, rows in ((100, 30), (3000, 50), (60000, 5000)):
        table, gy = torch.randn(rows, 24, device="cuda", generator=gen), torch.randn(n, 24, device="cuda", generator=gen)
        ids = make_ids(n, rows, "skew", gen)
        want = B.embedding(table, ids, 2.0), B.embedding_grad(gy, ids, rows, 2.0)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            got = B.embedding(table, ids, 2.0), B.embedding_grad(gy, ids, rows, 2.0)
        torch.cuda.current_stream().wait_stream(side)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            got = B.embedding(table, ids, 2.0), B.embedding_grad(gy, ids, rows, 2.0)
        for _ in range(4):                                 # new inputs in the same memory, eager work between the replays
            ids.copy_(make_ids(n, rows, "skew", gen))
            gy.copy_(torch.randn(n, 24, device="cuda", generator=gen))
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(got[0], B.embedding(table, ids, 2.0)) and torch.equal(got[1], B.embedding_grad(gy, ids, rows, 2.0))
            torch.cuda.synchronize()


def test_refusals(B):
    table, gy, ids = torch.randn(9, 8, device="cuda"), torch.randn(5, 8, device="cuda"), torch.zeros(5, device="cuda", dtype=torch.int64)
    for call in (lambda: B.embedding(table.cpu(), ids), lambda: B.embedding(table, ids.cpu()), lambda: B.embedding(table, ids.float()), lambda: B.embedding(table.t(), ids),
                 lambda: B.embedding(table.double(), ids), lambda: B.embedding(table[0], ids), lambda: B.embedding(table, torch.zeros(5, 2, device="cuda").long()[:, 0]),
                 lambda: B.embedding_grad(gy[:4], ids, 9), lambda: B.embedding_grad(gy.t(), ids, 9), lambda: B.embedding_grad(gy, ids, -1),
                 lambda: B.embedding_grad(gy, ids, 9, dtype=torch.int32), lambda: B.embedding_grad(gy.int(), ids, 9), lambda: B.embedding_grad(gy, ids[None].cpu(), 9)):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: B.embedding(table[:, :0], ids), lambda: B.embedding_grad(gy[:, :0], ids, 9), lambda: B.embedding_grad(gy, ids, 9, dtype=torch.bfloat16)):
        with pytest.raises(B.HagError) as err:
            call()
        assert err.value.code == B.HAG_EINVAL


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d", [3, 4, 16, 70, 300])
def test_ids_of_the_lowest_number(B, d, dtype):
    low = torch.iinfo(torch.int64).min                     # what a NaN is as an int64 on many hosts, and the number that stands for no padding
    table = torch.randn(6, d, device="cuda").to(dtype)
    ids = torch.tensor([low, 2, low, -1, low + 1], device="cuda")
    none, some = B.embedding(table, ids), B.embedding(table, ids, padding=-1)
    assert torch.equal(none[1], table[2]) and bool(torch.isnan(none[[0, 2, 3, 4]]).all())
    assert torch.equal(some[1], table[2]) and bool(torch.isnan(some[[0, 2, 4]]).all()) and not bool(some[3].any())
    assert not bool(B.embedding(table, ids, padding=low + 1)[4].any())
    short = torch.tensor([torch.iinfo(torch.int32).min, 2], device="cuda", dtype=torch.int32)
    assert bool(torch.isnan(B.embedding(table, short)[0]).all()) and not bool(B.embedding(table, short, padding=int(short[0]))[0].any())
    for n in (5, 3000, 9000, 140000):
        many = ids.repeat(n // 5)
        gy = torch.ones(many.numel(), d, device="cuda", dtype=dtype)
        got = B.embedding_grad(gy, many, 6, dtype=torch.float32)
        assert bool((got[2] == n // 5).all()) and int(got.count_nonzero()) == d


def test_padding_that_no_id_can_be(B):
    table, gy = torch.randn(6, 8, device="cuda"), torch.randn(2, 8, device="cuda")
    ids = torch.tensor([3, 2 ** 63 - 1], device="cuda")
    for padding in (2 ** 64 + 3, 3 - 2 ** 64, -2 ** 63 - 1, 2 ** 63):              # their low 64 bits are one of the ids, or no padding
        got = B.embedding(table, ids, padding=padding)
        assert torch.equal(got[0], table[3]) and bool(torch.isnan(got[1]).all())
        assert torch.equal(B.embedding_grad(gy, ids, 6, padding=padding)[3], gy[0])
    assert not bool(B.embedding(table, ids, padding=2 ** 63 - 1)[1].any())
    for call in (lambda: B.embedding(table, ids, padding=-2 ** 63), lambda: B.embedding_grad(gy, ids, 6, padding=-2 ** 63)):
        with pytest.raises(ValueError):
            call()


@pytest.mark.parametrize("kind", ["even", "skew", "one"])
@pytest.mark.parametrize("n,rows,d", [(2000, 16, 1024), (2048, 33, 201), (2048, 33, 64), (2048, 33, 65), (700, 6000, 376), (700, 6000, 371), (64, 2, 2049), (65, 65, 5000), (5, 3, 40001), (2, 1, 70001),
                                      (1, 3, 262144), (1, 3, 262145)])
def test_gradient_of_few_wide_tokens(B, n, rows, d, kind):
    gen = torch.Generator(device="cuda").manual_seed(n + rows + d)
    ids = make_ids(n, rows, kind, gen)
    ids[3::7] = -1
    for dtype in TYPES:
        gy = torch.randn(n, d, device="cuda", generator=gen).to(dtype)
        got = B.embedding_grad(gy, ids, rows, 1.5, -1)
        check_grad(got, gy, ids, rows, 1.5, -1)
        assert torch.equal(got, B.embedding_grad(gy, ids.int(), rows, 1.5, -1))
    assert not bool(B.embedding_grad(gy, torch.full_like(ids, -1), rows, padding=-1).any())


def test_sizes_are_refused_before_anything_is_made(B):
    gy, ids = torch.randn(2, 4, device="cuda"), torch.tensor([2 ** 31 - 3, 5], device="cuda")
    torch.cuda.synchronize()
    before = torch.cuda.memory_allocated()
    torch.cuda.reset_peak_memory_stats()
    for rows in (2 ** 31, 2 ** 40, 2 ** 64 + 5):
        with pytest.raises(B.HagError) as err:
            B.embedding_grad(gy, ids, rows)
        assert err.value.code == B.HAG_EINVAL and torch.cuda.max_memory_allocated() == before
    for call in (lambda: B.embedding_grad(gy[:, :0], ids, 9), lambda: B.embedding_grad(gy[:0, :0], ids[:0], 9)):
        with pytest.raises(B.HagError) as err:
            call()
        assert err.value.code == B.HAG_EINVAL
    assert B.embedding_grad(gy, ids, 0).shape == (0, 4)
