"""attend against its formula in 64 bits.

Bounds, element by element, with u = 2^-24: a score of D products in fp32, truncated by the tensor cores,
is off by (D + 8) 2 u of the sum of the products' magnitudes, and by 4 u of itself where it is scaled;
an exponential by what its argument's error makes of it and 2^-21; a probability that enters the second
product as two 16-bit values by 2^-17, as one fp16 value (bf16 queries over 8-bit values) by half of fp16's
step, 2^-11.  A warp adds the keys of its share one after another: shares are
the slots of 16 keys of all rows' tiles over 152 blocks of at least four warps, each slot 32 truncated
additions, and up to 160 joins follow.  The result is rounded once."""
import math

import pytest
import torch

import paper_2607_18957_gb300 as cfa

pytestmark = pytest.mark.gpu

BF16, F16, F32, F8 = torch.bfloat16, torch.float16, torch.float32, torch.float8_e4m3fn
HALF_ULP = {BF16: 2.0 ** -8, F16: 2.0 ** -11}
NEAR_ZERO = {BF16: 0.0, F16: 2.0 ** -25}
U = 2.0 ** -24


@pytest.fixture(scope="module", autouse=True)
def cuda_device():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    torch.cuda.set_device(0)


def normal(g, shape, dtype, scale=1.0):
    return (torch.randn(shape, generator=g, device="cuda") * scale).to(dtype)


class Setup:
    """A paged cache of random keys and values, the table's pages in random order, and queries.  What no
    sequence holds is NaN, in keys and values."""

    def __init__(self, lens, heads, kv, dim, dtype=BF16, cdtype=None, new=1, page=16, layout="tokens",
                 window=0, seed=0, spare=1, scale=1.0):
        g = torch.Generator(device="cuda").manual_seed(seed * 1009 + sum(lens) + dim)
        self.lens, self.heads, self.kv, self.dim, self.new = lens, heads, kv, dim, new
        self.dtype, self.page, self.window = dtype, page, window
        cdtype = cdtype or dtype
        self.ks, self.vs = (0.04, 0.03) if cdtype is F8 else (1.0, 1.0)
        held = [max(0, (n + page - 1) // page) for n in lens]
        per, pages = max(1, max(held)), sum(held) + spare
        order = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)
        self.pages = torch.full((len(lens), per), -7, dtype=torch.int32, device="cuda")
        shape = (pages, page, kv, dim) if layout != "heads" else (pages, kv, page, dim)
        if layout == "both":  # keys and values of a page side by side in one buffer
            both = torch.full((pages, 2, page, kv, dim), math.nan, device="cuda").to(cdtype)
            self.k, self.v = both[:, 0], both[:, 1]
        else:
            self.k, self.v = (torch.full(shape, math.nan, device="cuda").to(cdtype) for _ in range(2))
            if layout == "heads":
                self.k, self.v = self.k.transpose(1, 2), self.v.transpose(1, 2)
        at = 0
        for b, n in enumerate(lens):
            mine = order[at:at + held[b]]
            at += held[b]
            self.pages[b, :held[b]] = mine
            for i in range(held[b]):
                rows = min(page, n - i * page)
                for c, s in ((self.k, self.ks), (self.v, self.vs)):
                    c[mine[i].long(), :rows] = normal(g, (rows, kv, dim), F32, scale).div(s).to(cdtype)
        self.lengths = torch.tensor(lens, dtype=torch.int32, device="cuda")
        self.q = normal(g, (len(lens), new, heads, dim), dtype, scale)
        if new == 1:
            self.q = self.q[:, 0]

    def run(self, **kw):
        return cfa.attend(self.q, self.k, self.v, self.pages, self.lengths, window=self.window,
                          k_scale=self.ks, v_scale=self.vs, **kw)

    def keys(self, c, scale, b, n):
        pages = self.pages[b, :(n + self.page - 1) // self.page].long()
        ok = (pages >= 0) & (pages < c.shape[0])
        x = torch.where(ok[:, None, None, None], c[pages.clamp(0, c.shape[0] - 1)].double(), 0.0)
        return x.flatten(0, 1)[:n] * scale, ok.repeat_interleave(self.page)[:n]

    def check(self, scale=None, **kw):
        o, lse = self.run(lse=True, scale=scale, **kw)
        self.compare(o, lse, scale)
        return o, lse

    def compare(self, o, lse, scale=None):
        scale = self.dim ** -0.5 if scale is None else scale
        shape = (len(self.lens), self.new, self.heads, self.dim)
        assert o.shape == self.q.shape and o.dtype == self.dtype and lse.shape == o.shape[:-1]
        o, lse, q = o.double().view(shape), lse.double().view(shape[:-1]), self.q.double().view(shape)
        group, kv = self.heads // self.kv, self.kv
        rows = group * self.new
        tiles = kv * ((rows + 15) // 16 if rows > 8 else 1)
        slots = sum(max(1, n // 16 + 2) for n in self.lens) * tiles
        chain = 32 * (slots / (152 * 4) + 1) + 160
        for b, n in enumerate(self.lens):
            n = max(0, n)
            k, ok = self.keys(self.k, self.ks, b, n)
            v, _ = self.keys(self.v, self.vs, b, n)
            for i in range(self.new):
                end = n - self.new + i + 1
                begin = max(0, end - self.window) if self.window else 0
                see = torch.arange(n, device="cuda")
                see = (see < end) & (see >= begin) & ok
                got, got_lse = o[b, i].view(kv, group, -1), lse[b, i].view(kv, group)
                if not bool(see.any()):
                    assert not bool(got.any()) and bool((got_lse == -math.inf).all())
                    continue
                qi = q[b, i].view(kv, group, -1)
                z = torch.einsum("hgd,nhd->hgn", qi, k[see]) * scale
                size = torch.einsum("hgd,nhd->hgn", qi.abs(), k[see].abs()) * abs(scale)
                ez = ((self.dim + 8) * 2 * U * size + 8 * U * z.abs()).amax(2)
                p = torch.softmax(z, 2)
                ref = torch.einsum("hgn,nhd->hgd", p, v[see])
                mag = torch.einsum("hgn,nhd->hgd", p, v[see].abs())
                once = 2.0 ** -11 if self.dtype is BF16 and self.k.dtype is F8 else 0.0
                rel = (2 * ez + once + 2.0 ** -16 + 2 * (chain + 8) * 2 * U)[:, :, None]
                e = mag * rel * (1 + rel)
                e = e + HALF_ULP[self.dtype] * (ref.abs() + e) + NEAR_ZERO[self.dtype]
                assert bool(torch.isfinite(got).all())
                worst = ((got - ref).abs() - e).max().item()
                assert worst <= 0, f"sequence {b}, token {i}: off by {worst:g} more than the bound"
                ref = torch.logsumexp(z, 2)
                e = ez + (chain + 8) * 2 * U + 2.0 ** -20 + 4 * U * ref.abs()
                worst = ((got_lse - ref).abs() - e).max().item()
                assert worst <= 0, f"lse of {b}, {i}: off by {worst:g} more than the bound"


LENS = [[1], [2], [15], [16], [17], [31], [32], [33], [64], [65], [1000], [0, 1, 0, 16, 5], [100, 3, 257, 1, 64, 1023],
        [4097, 1, 300], list(range(1, 70))]


@pytest.mark.parametrize("lens", LENS, ids=lambda x: "-".join(map(str, x[:4])))
@pytest.mark.parametrize("dtype,cdtype", [(BF16, BF16), (F16, F16), (BF16, F8), (F16, F8)])
def test_lengths(lens, dtype, cdtype):
    Setup(lens, 8, 2, 128, dtype, cdtype).check()


@pytest.mark.parametrize("heads,kv", [(1, 1), (3, 3), (4, 1), (7, 1), (8, 8), (8, 1), (9, 1), (24, 2),
                                      (16, 1), (17, 1), (40, 1), (64, 8), (128, 1)])
@pytest.mark.parametrize("dim", [64, 96, 128, 256])
def test_heads(heads, kv, dim):
    for dtype, cdtype in ((BF16, BF16), (F16, F8)):
        Setup([200, 1, 49, 700], heads, kv, dim, dtype, cdtype).check()


@pytest.mark.parametrize("page", [1, 3, 16, 17, 24, 64, 100, 1000])
@pytest.mark.parametrize("layout", ["tokens", "heads", "both"])
def test_pages(page, layout):
    for cdtype, dim in ((BF16, 128), (F8, 64)):
        Setup([500, 16, 31, 1], 8, 2, dim, BF16, cdtype, page=page, layout=layout).check()


@pytest.mark.parametrize("new", [2, 3, 5, 8, 17, 40])
@pytest.mark.parametrize("heads,kv,dim", [(4, 4, 64), (8, 2, 128), (6, 2, 96), (16, 1, 256)])
@pytest.mark.parametrize("window", [0, 1, 20, 300])
def test_new_tokens(new, heads, kv, dim, window):
    """Sequences shorter than the new tokens too: their first rows see nothing."""
    for dtype, cdtype in ((BF16, BF16), (F16, F8)):
        Setup([500, 1, 40, 0, 16, new, 333], heads, kv, dim, dtype, cdtype, new=new,
              window=window).check()


@pytest.mark.parametrize("window", [1, 2, 15, 16, 17, 100, 1 << 30])
def test_windows(window):
    Setup([1, 16, 17, 100, 1000, 3000], 8, 2, 128, window=window).check()


@pytest.mark.parametrize("new", [1, 4])
def test_values_that_are_not_seen(new):
    """Infinities and NaN in keys and values that some rows do not see: behind a sequence's end, before
    its window, and those of later new tokens for the earlier ones."""
    s = Setup([100, 37, 16], 8, 2, 128, new=new, window=30)
    clean = s.run(lse=True)
    for b, n in enumerate(s.lens):
        gone = range(0, max(0, n - new + 1 - 30))
        for j in gone:
            s.k[s.pages[b, j // 16].long(), j % 16] = math.nan
            s.v[s.pages[b, j // 16].long(), j % 16] = math.inf
    o, lse = s.run(lse=True)
    assert torch.equal(o, clean[0]) and torch.equal(lse, clean[1])
    if new > 1:  # the last new token's own: it alone sees them
        for b, n in enumerate(s.lens):
            s.v[s.pages[b, (n - 1) // 16].long(), (n - 1) % 16] = math.inf
            s.k[s.pages[b, (n - 1) // 16].long(), (n - 1) % 16] = 0.0
        o, lse = s.run(lse=True)
        assert torch.equal(o[:, :-1], clean[0][:, :-1]) and torch.equal(lse[:, :-1], clean[1][:, :-1])
        assert bool((o[:, -1] == math.inf).all())


def test_nan_and_infinities_that_are_seen():
    s = Setup([50, 50, 50], 4, 2, 64)
    s.q[0, 1] = math.nan
    s.k[s.pages[1, 0].long(), 3, 0, 5] = math.nan
    s.v[s.pages[2, 1].long(), 2, 1, 7] = math.inf
    o, lse = s.run(lse=True)
    assert bool(o[0, 1].isnan().all()) and bool(o[0, [0, 2, 3]].isfinite().all())
    assert bool(o[1, :2].isnan().all()) and bool(o[1, 2:].isfinite().all()) and bool(lse[1, :2].isnan().all())
    assert bool((o[2, 2:, 7] == math.inf).all()) and bool(o[2, 2:, :7].isfinite().all())
    assert bool(o[2, :2].isfinite().all()) and bool(lse[2].isfinite().all())


def test_scores_that_all_are_minus_infinity():
    s = Setup([20], 2, 1, 64)
    s.q.fill_(0.0)
    s.q[0, 0, 0] = 1.0
    s.k[..., 0] = -math.inf
    o, lse = s.run(lse=True)
    assert not bool(o[0, 0].any()) and lse[0, 0].item() == -math.inf
    assert bool(o[0, 1].isnan().all())  # 0 times infinity


def test_pages_that_are_not_there():
    s = Setup([200, 90, 64, 10], 8, 2, 128, page=16)
    s.pages[0, 3], s.pages[0, 11] = -1, s.k.shape[0]
    s.pages[1, :] = -1
    s.pages[2, 0], s.pages[3, 0] = (1 << 31) - 1, -(1 << 31)
    s.check()


def test_lengths_that_leave_the_table():
    s = Setup([64, 64, 30], 8, 2, 128)
    o, lse = s.check()
    s.lengths[0], s.lengths[2] = 1 << 30, -5
    got, got_lse = s.run(lse=True)
    assert torch.equal(got[:2], o[:2]) and torch.equal(got_lse[:2], lse[:2])
    assert not bool(got[2].any()) and bool((got_lse[2] == -math.inf).all())


def test_large_scores():
    """Scores of hundreds, where one key takes all."""
    Setup([300, 2000], 8, 2, 128, F16, scale=6.0).check()
    Setup([300, 2000], 8, 2, 128, scale=3.0).check(scale=-0.3)


@pytest.mark.parametrize("cdtype", [F16, F8])
@pytest.mark.parametrize("scale", [0.0, 1e-42, -1e-42, -0.1])
def test_scales_around_zero(scale, cdtype):
    """Down to where scale and the keys' scale together leave fp32: all keys count alike."""
    Setup([100, 1, 33], 8, 2, 128, F16, cdtype).check(scale=scale)


@pytest.mark.parametrize("heads,kv,dim,cdtype", [(8, 1, 128, BF16), (64, 8, 128, BF16), (16, 2, 256, F8),
                                                 (4, 4, 64, BF16)])
def test_long_sequences_over_many_blocks(heads, kv, dim, cdtype):
    Setup([20000, 7], heads, kv, dim, BF16, cdtype, page=64).check()


@pytest.mark.parametrize("lens,heads,kv,dim,new", [
    ([200000], 16, 8, 128, 1), ([3, 90000, 120000, 1], 8, 8, 128, 1), ([150000, 30000], 16, 8, 128, 3),
    ([400000, 31], 8, 8, 64, 1), ([210000], 8, 4, 256, 1), ([90] * 20 + [180000], 9, 9, 128, 1)])
def test_very_long_sequences(lens, heads, kv, dim, new):
    """Megabytes to every block, and the same bits every time."""
    s = Setup(lens, heads, kv, dim, page=10000, new=new)
    o, lse = s.check()
    for _ in range(3):
        again = s.run(lse=True)
        assert torch.equal(o, again[0]) and torch.equal(lse, again[1])


def test_many_short_sequences():
    Setup([1 + i * 7 % 40 for i in range(700)], 8, 2, 64, page=8).check()


def test_more_sequences_than_threads():
    lens = [i % 5 for i in range(3000)]
    s = Setup(lens, 2, 1, 64, page=4)
    o, lse = s.run(lse=True)
    for b in list(range(0, 3000, 211)) + [2999]:
        part = Setup.__new__(Setup)
        part.__dict__.update(s.__dict__)
        part.lens, part.pages, part.q = lens[b:b + 1], s.pages[b:b + 1], s.q[b:b + 1]
        part.compare(o[b:b + 1], lse[b:b + 1])
    assert not bool(o[0].any()) and bool(o.isfinite().all())


def test_cache_behind_32_bits():
    """Pages 2^32 bytes and more into caches of 9 GiB."""
    kv, dim, page = 8, 128, 16
    pages = (9 << 30) // (page * kv * dim * 2)
    k = torch.empty(pages, page, kv, dim, dtype=BF16, device="cuda")
    v = torch.empty(pages, page, kv, dim, dtype=BF16, device="cuda")
    s = Setup([160], 32, kv, dim)
    want = s.run(lse=True)
    far = torch.arange(pages - 10, pages, device="cuda")
    k[far], v[far] = s.k[s.pages[0].long()], s.v[s.pages[0].long()]
    o, lse = cfa.attend(s.q, k, v, far.to(torch.int32)[None], s.lengths, lse=True)
    assert torch.equal(o, want[0]) and torch.equal(lse, want[1])


def test_strides_of_queries_results_and_tables():
    s = Setup([100, 17, 300], 8, 2, 128)
    want, want_lse = s.run(lse=True)
    qkv = torch.full((3, 12 * 128), math.nan, dtype=BF16, device="cuda")
    own = qkv[:, :8 * 128].unflatten(1, (8, 128))
    own.copy_(s.q)
    wide = torch.full((3, s.pages.shape[1] + 5), -1, dtype=torch.int32, device="cuda")
    wide[:, :-5] = s.pages
    room = torch.full((5, 9, 128), 7.0, dtype=BF16, device="cuda")
    out = room[1:4, :8]
    lse = torch.empty_like(want_lse)
    got = cfa.attend(own, s.k, s.v, wide[:, :-5], s.lengths, lse=True, out=(out, lse),
                     workspace=torch.empty(4 << 20, dtype=torch.uint8, device="cuda"))
    assert got[0] is out and torch.equal(out, want) and torch.equal(lse, want_lse)
    assert bool((room[0] == 7).all()) and bool((room[4] == 7).all()) and bool((room[:, 8] == 7).all())
    assert torch.equal(s.run(), want)


def test_same_bits_again():
    s = Setup([5000, 20, 333], 32, 8, 128)
    first = s.run(lse=True)
    for _ in range(5):
        again = s.run(lse=True)
        assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])


def test_no_sequences():
    s = Setup([20], 4, 2, 64)
    o = cfa.attend(s.q[:0], s.k, s.v, s.pages[:0], s.lengths[:0])
    assert o.shape == (0, 4, 64)
