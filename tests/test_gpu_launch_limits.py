"""Sizes that call for 2^32 threads and more, which one launch does not hold: lookups and their gradient, layer norm.  Inputs are views of little memory (a row throughout, or rows
that begin one element after the other); outputs are as large as they are."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
GB = 10 ** 9


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


def sliding(n, d, gen):
    """[n, d] rows of a bfloat16 buffer, each one element after the one before; the sums of all rows in 64 bits."""
    flat = torch.randn(n + d - 1, device="cuda", generator=gen).bfloat16()
    upto = torch.cat([torch.zeros(1, device="cuda", dtype=torch.float64), flat.double().cumsum(0)])
    return flat.as_strided((n, d), (1, 1)), upto[d:] - upto[:-d]


@pytest.mark.parametrize("n,rows", [(3, 2 ** 29 + 100), (0, 2 ** 29 + 100), (2000, 2 ** 30), (2000, 2 ** 31 - 2)])
def test_gradient_of_few_tokens_of_many_rows(B, n, rows):
    need(5 * GB)
    gen = torch.Generator(device="cuda").manual_seed(n)
    ids = torch.randint(0, rows, (n,), device="cuda", generator=gen)
    if n:
        ids[:3] = torch.tensor([rows - 1, 2 ** 28, 5], device="cuda")              # the last row, the first ones of launches
    gy = (torch.rand(n, 1, device="cuda", generator=gen) + 1).bfloat16()
    got = B.embedding_grad(gy, ids, rows)
    want, at = torch.unique(ids, return_inverse=True)
    total = torch.zeros(want.numel(), device="cuda", dtype=torch.float64).index_add_(0, at, gy[:, 0].double())
    assert torch.equal(got[want, 0], total.bfloat16()) and sum(int(p.count_nonzero()) for p in got.split(1 << 28)) == want.numel()


def test_lookup_of_many_ids(B):
    n, rows, d = 2 ** 28 + 77, 50, 257                     # a wavefront for a row: 138 GB
    need(145 * GB)
    table = torch.randn(rows, d, device="cuda").bfloat16()
    ids = torch.randint(-1, rows, (n,), device="cuda", dtype=torch.int32)
    y = B.embedding(table, ids, padding=-1)
    for begin in (0, n // 3, 2 ** 27 - 40, 2 ** 28 - 40, n - 100):                 # the seams of launches among them
        some = ids[begin:begin + 100].long()
        assert torch.equal(y[begin:begin + 100], torch.where(some[:, None] >= 0, table[some.clamp(min=0)], 0))
    assert torch.equal(y[::4099], torch.where(ids[::4099, None] >= 0, table[ids[::4099].long().clamp(min=0)], 0))


def test_gradient_of_as_many_tokens_as_there_may_be(B):
    n, rows, d = 2 ** 31 - 1, 1000, 132                    # 2^24 workgroups of the sums, and those of the rows
    need(80 * GB)
    ids = torch.arange(n, device="cuda", dtype=torch.int32)
    ids %= rows
    gy = torch.arange(1, d + 1, device="cuda").float()[None].remainder(5).expand(n, d)
    got = B.embedding_grad(gy, ids, rows)
    count = (n - 1 - torch.arange(rows, device="cuda")) // rows + 1
    assert torch.equal(got.double(), count.double()[:, None] * gy[:1].double())     # whole numbers below 2^24


@pytest.mark.parametrize("n,d", [(2 ** 27 + 9, 258), (2 ** 24 + 5, 1032), (2 ** 22 + 3, 4104), (2 ** 22 + 3, 8200)])
def test_layer_norm_of_many_rows(B, n, d):
    need(2 * n * d + 10 * GB)
    gen = torch.Generator(device="cuda").manual_seed(d)
    x, total = sliding(n, d, gen)
    w = 1 + 0.1 * torch.randn(d, device="cuda", generator=gen)
    y, mean, rstd = B.layer_norm(x, w)
    m = total / d
    # 64 roundings on the way of a term, and those of the sums of all that come before in 64 bits
    assert bool(((mean.double() - m).abs() <= 64 * 2.0 ** -24 + 2.0 ** -40).all()) and bool(torch.isfinite(rstd).all())
    seams = [s + k for s in range(0, n, 2 ** 31 // 1024) for k in (-1, 0, 1) if 0 <= s + k < n][:400]
    some = torch.tensor(sorted({0, 1, n // 3, n - 2, n - 1, *seams, *range(0, n, n // 200)}), device="cuda")
    x64, w64 = x[some].double(), w.double()
    dev = x64 - x64.mean(1, keepdim=True)
    r = (dev.square().mean(1, keepdim=True) + 1e-5).rsqrt()
    assert bool(((rstd[some].double()[:, None] - r).abs() <= 64 * 2.0 ** -24 * r).all())
    assert bool(((y[some].double() - dev * r * w64).abs() <= (2.0 ** -8 + 2.0 ** -16) * (dev * r * w64).abs() + 2.0 ** -16).all())
    del y
    if d < 8200:
        return
    gy = x[5:6].expand(n, d)                               # backward: rows of more than 8192 columns take a workgroup each
    gx, _, _ = B.layer_norm_grad(gy, x, mean, rstd, w, params=False)
    u, xh = gy[:1].double() * w64, dev * r
    want = r * (u - u.mean(1, keepdim=True) - xh * (u * xh).mean(1, keepdim=True))
    assert bool(((gx[some].double() - want).abs() <= (2.0 ** -8 + 2.0 ** -16) * want.abs() + 2.0 ** -14).all())


def test_gradient_of_as_many_rows_as_there_may_be(B):
    rows, n = 2 ** 31 - 1, 3000
    need(40 * GB)
    gen = torch.Generator(device="cuda").manual_seed(1)
    for many in (2, n):                                    # few tokens, and tokens put in order
        ids = torch.randint(0, rows, (many,), device="cuda", generator=gen)
        ids[0], ids[1] = rows - 1, rows                    # the last row, the first that is none
        got = B.embedding_grad(torch.ones(many, 1, device="cuda", dtype=torch.bfloat16), ids, rows)
        want, count = torch.unique(ids[ids < rows], return_counts=True)
        assert torch.equal(got[want, 0], count.bfloat16()) and sum(int(p.count_nonzero()) for p in got.split(1 << 28)) == want.numel()
