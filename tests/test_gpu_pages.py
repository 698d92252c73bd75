"""The calls on a paged cache against their plain 64-bit versions (tests/pages_ref.py).

Bounds.  Writing, reading and selecting are exact: every stored value, bound and list is compared bit for bit.
Attention: a score is an f32 sum of D exact products (bf16 times bf16; three pieces of an f32 query leave 2^-24 of it), so with
S = the largest sum of |q_d k_d scale| of a row it is off by at most (D + 4) * 2^-24 * S, and its exponent, a product, a difference and one
exp2, by (|s| + |max|) * 2^-23 more; the weights are off by e = twice that (their sum takes the same terms).  The weights are rounded, for
bf16 queries to two bf16 pieces (2^-16), or to one (2^-8) where more than 32 rows share a KV head's keys, for f32 ones to three (2^-24).  Sums of n terms in steps of 32: (n / 32 + 64) * 2^-24.
Hence, with A = sum of weights times |v|:
    out   (e + pieces + (n / 32 + 64) * 2^-24) * A, and half a step of its type: 2^-8 (bf16) or 2^-23 (f32: two roundings) of |out|
    lse   e / 2 + (n / 32 + 64) * 2^-24 + 2^-23 |lse|
"""
from types import SimpleNamespace

import numpy as np
import pages_ref as ref
import pytest
import torch

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    from paper_2607_05722_amd import _lib as C
    from paper_2607_05722_amd import runtime as R

F32, BF16, E4M3 = torch.float32, torch.bfloat16, torch.float8_e4m3fn
DEV = "cuda:0"
NAN, INF = float("nan"), float("inf")


def gen(seed):
    return torch.Generator().manual_seed(seed)


def randn(shape, seed, dtype=BF16, scale=1.0):
    return (torch.randn(shape, generator=gen(seed)) * scale).to(dtype).to(DEV)


def starts_of(news):
    return [0] + np.cumsum(news).tolist()


def on_device(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


class Setup:
    """A cache of the library with a shuffled table, and the plain one beside it."""

    def __init__(self, pages, heads, dim, lens, news, seed=0, bounds=True, slack=64, garbage=None, spare=3, layers=1, layer=0):
        self.lens, self.news, self.H, self.D, self.layer = list(lens), list(news), heads, dim, layer
        B = len(lens)
        self.max_len = -(-(max(p + n for p, n in zip(lens, news)) + slack) // 64) * 64
        width = self.max_len // 64
        need = [-(-(p + n) // 64) for p, n in zip(lens, news)]
        n_pages = sum(need) + spare
        self.cache = R.PagedCache(heads, dim, B, self.max_len, n_layers=layers, n_pages=n_pages, dtype=pages, bounds=bounds, device=DEV)
        order = torch.randperm(n_pages, generator=gen(seed + 7)).to(torch.int32)
        table, at = torch.full((B, width), -1, dtype=torch.int32), 0
        for b, m in enumerate(need):
            table[b, :m] = order[at:at + m]
            at += m
        self.free = order[at:].tolist()
        self.cache.table.copy_(table)
        if garbage is not None:
            # everything that nothing writes holds what must not get into any result
            self.cache.k.view(torch.uint8).fill_(garbage)
            self.cache.v.view(torch.uint8).fill_(garbage)
            if self.cache.scale is not None:
                self.cache.scale.fill_(255)
        self.plain = ref.Cache(B, self.max_len, heads, dim, pages == E4M3, DEV)
        self.start = starts_of(news)
        self.row_start = on_device(self.start)
        self.rows, self.most = self.start[-1], max(news)

    def workspace(self, q_heads, max_rows=None, group=0):
        return R.PagesWorkspace(self.cache, q_heads, max_rows or max(self.most, 1), group)

    def fill(self, seed=1, dtype=BF16, k=None, v=None):
        """Writes the committed rows and then the new ones."""
        for lens, news, s in (([0] * len(self.lens), self.lens, seed), (self.lens, self.news, seed + 10)):
            st = starts_of(news)
            if st[-1] == 0:
                continue
            kk, vv = randn((st[-1], self.H, self.D), s, dtype), randn((st[-1], self.H, self.D), s + 1, dtype)
            self.write(lens, news, kk, vv)
        return self

    def write(self, lens, news, k, v):
        st = starts_of(news)
        ws = R.PagesWorkspace(self.cache, self.H, max(news))
        self.cache.lengths.copy_(on_device(lens))
        R.write_pages(self.cache, self.layer, k, v, ws, row_start=on_device(st), max_rows=max(news))
        self.plain.write(lens, st, k, v)
        self.cache.lengths.copy_(on_device(self.lens))
        assert R.read_device_status(ws) == 0

    def check(self, q, mode=0, bidir_from=0, scale=None, lists=None, group=1, **kw):
        ws = self.workspace(q.shape[1], group=group if lists is not None else 0)
        out, lse = R.attend_pages(self.cache, self.layer, q, ws, mode=mode, bidir_from=bidir_from, scale=scale, pages=lists, group=group,
                                  row_start=self.row_start, max_rows=self.most, want_lse=True, **kw)
        assert R.read_device_status(ws) == 0
        self.compare(out, lse, q, mode, bidir_from, scale, lists, group)
        return out, lse

    def compare(self, out, lse, q, mode=0, bidir_from=0, scale=None, lists=None, group=1):
        scale = self.D ** -0.5 if scale is None else scale
        o, l, a, s = ref.attend(self.plain, self.lens, self.start, q, scale, mode == 1, bidir_from, lists, group)
        n = self.max_len
        e = 2 * ((self.D + 4) * 2.0 ** -24 * s + 2 * s * 2.0 ** -23 + 2.0 ** -23)
        sums = (n / 32 + 64) * 2.0 ** -24
        many = min(group if lists is not None else self.most, self.most) * q.shape[1] // self.H > 32
        half, piece = (2.0 ** -8, 2.0 ** -8 if many else 2.0 ** -16) if out.dtype == BF16 else (2.0 ** -23, 2.0 ** -24)
        off = (out.double() - o).abs()
        most = half * o.abs() + (e[..., None] + piece + sums) * a
        assert bool((off <= most).all()), float((off - most).max())
        some = torch.isfinite(l)
        assert torch.equal(some, torch.isfinite(lse)) and bool((lse[~some] == -INF).all())
        off = (lse.double() - l)[some].abs()
        assert bool((off <= e[some] / 2 + sums + 2.0 ** -23 * l[some].abs()).all())


# ------------------------------------------------------------------------------------------ rows
LENS = [([0], [1]), ([63], [1]), ([64], [2]), ([5, 0, 130, 64], [70, 1, 0, 63]), ([127, 1, 60], [1, 200, 5])]


@pytest.mark.parametrize("pages", [BF16, E4M3])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("lens,news", LENS)
def test_rows_are_stored_and_read_back(pages, dim, lens, news):
    for dtype in (BF16, F32):
        s = Setup(pages, 3, dim, lens, news, layers=2, layer=1).fill(dtype=dtype)
        other = torch.equal(s.cache.k[0].view(torch.uint8), torch.zeros_like(s.cache.k[0].view(torch.uint8)))
        assert other and int(s.cache.bounds[0].abs().max()) == 0      # the other layer is not touched
        ws = s.workspace(3)
        total = [p + n for p, n in zip(lens, news)]
        st = on_device(starts_of(total))
        for to in (BF16, F32):
            k, v = R.read_pages(s.cache, 1, sum(total), ws, dtype=to, row_start=st, max_rows=max(total))
            for b, n in enumerate(total):
                at = starts_of(total)[b]
                assert torch.equal(k[at:at + n].double(), s.plain.k[b, :n]) and torch.equal(v[at:at + n].double(), s.plain.v[b, :n])
        # the new rows alone
        k, v = R.read_pages(s.cache, 1, s.rows, ws, first=s.cache.lengths, row_start=s.row_start, max_rows=s.most)
        for b, p in enumerate(lens):
            r0, r1 = s.start[b], s.start[b + 1]
            assert torch.equal(k[r0:r1].double(), s.plain.k[b, p:p + r1 - r0]) and torch.equal(v[r0:r1].double(), s.plain.v[b, p:p + r1 - r0])
        assert R.read_device_status(ws) == 0


@pytest.mark.parametrize("dim", [64, 128])
def test_values_in_8_bits(dim):
    """Ties, the largest and the least magnitudes, zeros, numbers that are not finite; each row by itself."""
    x = randn((64, 1, dim), 3, F32)
    x[1] = 0.0
    x[2, 0, :] = 448.0 * torch.linspace(-1, 1, dim, device=DEV)
    x[3, 0, :] = (torch.arange(dim, device=DEV) % 32 + 0.5) / 16.0          # halfway between codes
    x[4, 0, 0] = 449.0                                                       # the next power of two
    x[5] *= 1e-38
    x[6] = 1e-44
    x[7] *= 2.0 ** 100
    x[8, 0, :3] = torch.tensor([NAN, INF, -INF])
    x[9, 0, :] = NAN
    x[10, 0, :] = torch.tensor(3.3e38)
    x[11, 0, :] = -0.0
    x[12, 0, 1:] = 2.0 ** -17 * x[12, 0, 0]
    s = Setup(E4M3, 1, dim, [0], [64])
    s.write([0], [64], x, -x)
    k, v = R.read_pages(s.cache, 0, 64, s.workspace(1))
    for got, want in ((k, ref.stored(x, True)), (v, ref.stored(-x, True))):
        differ = (got.double() != want) & ~(torch.isnan(got) & torch.isnan(want))
        assert not bool(differ.any()), [(got[i].tolist()[0], want[i].tolist()[0]) for i in differ.flatten(1).any(1).nonzero()[:, 0].tolist()]


@pytest.mark.parametrize("pages", [BF16, E4M3])
def test_a_row_written_alone_is_the_row_of_a_chunk(pages):
    k, v = randn((150, 2, 128), 1), randn((150, 2, 128), 2)
    one, many = (Setup(pages, 2, 128, [30], [150], seed=4) for _ in range(2))
    many.write([30], [150], k, v)
    for i in range(150):
        one.write([30 + i], [1], k[i:i + 1], v[i:i + 1])
    for name in ("k", "v", "scale", "bounds", "bound_scale"):
        a, b = getattr(one.cache, name), getattr(many.cache, name)
        assert a is None or torch.equal(a.view(torch.uint8), b.view(torch.uint8)), name


@pytest.mark.parametrize("pages", [BF16, E4M3])
@pytest.mark.parametrize("dim", [64, 128])
def test_bounds(pages, dim):
    s = Setup(pages, 2, dim, [40, 0, 100], [1, 130, 64]).fill()
    for b, end in enumerate([41, 130, 164]):
        for page in range(-(-end // 64)):
            id_ = int(s.cache.table[b, page])
            for h in range(2):
                bd, bs = ref.bounds(s.plain.k[b, page * 64:page * 64 + 64, h], min(end - page * 64, 64))
                assert torch.equal(s.cache.bounds[0, id_, h], bd) and float(s.cache.bound_scale[0, id_, h]) == bs


def test_bounds_forget_rows_that_were_overwritten():
    """A rejected draft's row counts until the next write to its page."""
    s = Setup(BF16, 1, 64, [10], [8])
    big = torch.full((8, 1, 64), 100.0, dtype=BF16, device=DEV)
    s.write([0], [10], randn((10, 1, 64), 1), randn((10, 1, 64), 2))
    s.write([10], [8], big, big)
    assert float(s.cache.bound_scale.max()) > 0.7
    s.write([12], [1], randn((1, 1, 64), 5), randn((1, 1, 64), 6))
    bd, bs = ref.bounds(s.plain.k[0, :64, 0], 13)
    id_ = int(s.cache.table[0, 0])
    assert torch.equal(s.cache.bounds[0, id_, 0], bd) and float(s.cache.bound_scale[0, id_, 0]) == bs


@pytest.mark.parametrize("bad", [NAN, INF, -INF])
@pytest.mark.parametrize("pages", [BF16, E4M3])
def test_bounds_of_keys_that_are_not_finite(pages, bad):
    s = Setup(pages, 2, 64, [0], [70])
    k = randn((70, 2, 64), 1, F32)
    k[66, 1, 5] = bad
    s.write([0], [70], k, k)
    ids = s.cache.table[0, :2].long()
    assert float(s.cache.bound_scale[0, ids[1], 1]) == INF and int(s.cache.bounds[0, ids[1], 1].abs().max()) == 0
    assert bool(torch.isfinite(s.cache.bound_scale[0, ids[0]]).all()) and float(s.cache.bound_scale[0, ids[1], 0]) < INF


def strided(shape, dtype, row_pad, head_pad, lead, fill=NAN, heads_first=False):
    """A view with padded strides inside a buffer of `fill`."""
    n, h, d = shape
    hs = d + head_pad if not heads_first else n * (d + head_pad) + row_pad
    rs = h * (d + head_pad) + row_pad if not heads_first else d + head_pad
    buf = torch.full((lead + (n - 1) * rs + (h - 1) * hs + d + 8,), fill, dtype=dtype, device=DEV)
    return buf, buf.as_strided(shape, (rs, hs, 1), lead)


@pytest.mark.parametrize("pages", [BF16, E4M3])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("row_pad,head_pad,lead,heads_first", [(0, 0, 0, False), (8, 16, 8, False), (3, 1, 1, False), (8, 8, 0, True), (5, 3, 7, True)])
def test_strides_and_alignment(pages, dtype, row_pad, head_pad, lead, heads_first):
    s = Setup(pages, 2, 64, [70, 3], [5, 66])
    place = lambda x: strided(x.shape, dtype, row_pad, head_pad, lead, heads_first=heads_first)[1].copy_(x)
    old = [randn((73, 2, 64), i, dtype) for i in (1, 2)]
    s.write([0, 0], [70, 3], *map(place, old))
    s.write([70, 3], [5, 66], *(place(randn((71, 2, 64), i, dtype)) for i in (3, 4)))
    q = place(randn((71, 6, 64), 5, dtype))
    buf, out = strided(q.shape, dtype, row_pad, head_pad, lead, 77.0, heads_first)
    s.check(q, out=out)
    out.fill_(77.0)
    assert bool((buf == 77.0).all())        # nothing but the rows was written
    (kb, k), (vb, v) = (strided((71, 2, 64), dtype, row_pad, head_pad, lead, 77.0, heads_first) for _ in range(2))
    R.read_pages(s.cache, 0, 71, s.workspace(2), first=s.cache.lengths, row_start=s.row_start, max_rows=66, outs=(k, v))
    for x, plain, buf in ((k, s.plain.k, kb), (v, s.plain.v, vb)):
        assert torch.equal(x[:5].double(), plain[0, 70:75]) and torch.equal(x[5:].double(), plain[1, 3:69])
        x.fill_(77.0)
        assert bool((buf == 77.0).all())


@pytest.mark.parametrize("heads_apart", [False, True])
def test_arrays_that_share_a_buffer(heads_apart):
    """Queries and outputs, and keys and values read back, as the halves of every row, or of every head, of one tensor."""
    s = Setup(BF16, 2, 64, [70, 3], [5, 66]).fill()
    both = torch.full((71, 2, 4, 64), 7.0, dtype=BF16, device=DEV) if not heads_apart else torch.full((71, 4, 2, 64), 7.0, dtype=BF16, device=DEV).transpose(1, 2)
    q, out = both[:, 0], both[:, 1]
    q.copy_(randn((71, 4, 64), 5))
    s.check(q.contiguous())
    s.check(q, out=out)
    assert torch.equal(q, randn((71, 4, 64), 5))
    k, v = torch.zeros((71, 2, 2, 64), device=DEV).unbind(2 if heads_apart else 1)
    R.read_pages(s.cache, 0, 71, s.workspace(2), first=s.cache.lengths, row_start=s.row_start, max_rows=66, outs=(k, v))
    assert torch.equal(k[5:].double(), s.plain.k[1, 3:69]) and torch.equal(v[:5].double(), s.plain.v[0, 70:75])
    with pytest.raises(C.NLDError, match="overlaps"):
        R.read_pages(s.cache, 0, 71, s.workspace(2), row_start=s.row_start, outs=(k, k.as_strided(k.shape, k.stride(), k.storage_offset() + 32)))


def test_rows_outside_the_sequences_stay_as_they_are():
    s = Setup(BF16, 2, 64, [10, 20], [3, 2]).fill()
    start = on_device([2, 5, 7])     # rows 0, 1 and 7, 8 belong to nobody
    q = randn((9, 4, 64), 3)
    ws = s.workspace(4, 9)
    out, lse = torch.full_like(q, 5.0), torch.full((9, 4), 5.0, device=DEV)
    R.attend_pages(s.cache, 0, q, ws, row_start=start, max_rows=3, out=out, lse=lse)
    assert bool((out[[0, 1, 7, 8]] == 5.0).all()) and bool((lse[[0, 1, 7, 8]] == 5.0).all())
    s.compare(out[2:7], lse[2:7], q[2:7])
    k, v = torch.full((9, 2, 64), 5.0, device=DEV), torch.full((9, 2, 64), 5.0, device=DEV)
    R.read_pages(s.cache, 0, 9, ws, row_start=start, max_rows=3, outs=(k, v))
    assert bool((k[[0, 1, 7, 8]] == 5.0).all()) and torch.equal(v[5:7].double(), s.plain.v[1, :2])
    before = s.cache.k.clone()
    rows = randn((9, 2, 64), 8)
    R.write_pages(s.cache, 0, rows, rows, ws, row_start=on_device([9, 9, 9]), max_rows=3)
    assert torch.equal(s.cache.k, before) and R.read_device_status(ws) == 0


# ------------------------------------------------------------------------------------------ attention
HEADS = [(4, 2), (8, 8), (5, 1), (32, 8)]


@pytest.mark.parametrize("pages", [BF16, E4M3])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("lens,news", LENS)
def test_attention_over_lengths(pages, dim, dtype, lens, news):
    s = Setup(pages, 2, dim, lens, news, garbage=0xFF).fill()
    q = randn((s.rows, 4, dim), 5, dtype, 2.0)
    s.check(q)
    s.check(q, mode=1, bidir_from=1)


@pytest.mark.parametrize("q_heads,kv_heads", HEADS)
@pytest.mark.parametrize("n", [1, 2, 7, 16, 33])
def test_attention_over_heads_and_rows(q_heads, kv_heads, n):
    """1 to 264 rows of a KV head: one, two and four tiles of 32 and several blocks."""
    s = Setup(E4M3, kv_heads, 64, [100, 0, 67], [n, max(1, n - 1), n]).fill()
    for dtype in (BF16, F32):
        s.check(randn((s.rows, q_heads, 64), 5, dtype))


@pytest.mark.parametrize("bidir_from", [0, 1, 3, 16])
def test_draft_blocks(bidir_from):
    s = Setup(BF16, 2, 128, [200, 64, 0], [16, 16, 16]).fill()
    s.check(randn((48, 8, 128), 5), mode=1, bidir_from=bidir_from)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("pages", [BF16, E4M3])
def test_long_sequences_meet_from_many_workgroups(pages, dtype):
    s = Setup(pages, 2, 64, [5000, 12, 1300], [1, 1, 1]).fill()
    s.check(randn((3, 8, 64), 5, dtype, 2.0))


@pytest.mark.parametrize("cus", [1, 3])
@pytest.mark.parametrize("pages", [BF16, E4M3])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("n,q_heads,dim", [(1, 4, 64), (2, 8, 128), (7, 8, 64), (8, 8, 128), (20, 8, 64), (20, 8, 128), (70, 8, 64)])
def test_few_workgroups_with_long_shares(monkeypatch, cus, pages, dtype, n, q_heads, dim):
    """Shares of more pages than a window has, and of many units: tiles of 16 and of 32 rows, two of these, and eight."""
    monkeypatch.setenv("NLD_CUS", str(cus))
    s = Setup(pages, 2, dim, [64 * 150 + 5, 0, 700, 64 * 65], [n, n, 1, max(1, n // 2)], garbage=0xFF).fill()
    q = randn((s.rows, q_heads, dim), 5, dtype)
    s.check(q)
    s.check(q, mode=1, bidir_from=1)
    group = min(n, 3)
    width = s.max_len // 64
    lists = torch.stack([torch.randperm(width, generator=gen(i))[:90] for i in range(4 * -(-n // group) * 2)]).view(4, -1, 2, 90).to(torch.int32)
    lists[:, :, 1, 40:50] = -1
    s.check(q, lists=lists.to(DEV), group=group)


def test_many_sequences():
    """More blocks of rows than a workgroup has threads, some of them without rows."""
    lens = [(i * 37) % 150 for i in range(300)]
    news = [(i * 5) % 4 for i in range(300)]
    s = Setup(BF16, 1, 64, lens, news).fill()
    s.check(randn((s.rows, 2, 64), 5))


def test_many_sequences_of_many_rows():
    """More blocks than threads where several tiles share the pages: 520 sequences, half of them without rows."""
    lens = [(i * 37) % 150 for i in range(520)]
    news = [33 + i % 3 if i % 8 == 1 else i % 2 for i in range(520)]
    s = Setup(BF16, 1, 64, lens, news).fill()
    s.check(randn((s.rows, 1, 64), 5))


def test_one_number_of_rows_for_all_needs_no_row_start():
    s = Setup(BF16, 2, 64, [10, 70], [4, 4])
    rows = [randn((80, 2, 64), i) for i in (1, 2)]
    s.write([0, 0], [10, 70], *rows)
    k, v, q = (randn((8, h, 64), i) for h, i in ((2, 3), (2, 4), (4, 5)))
    ws = s.workspace(4)
    R.write_pages(s.cache, 0, k, v, ws)
    s.plain.write(s.lens, s.start, k, v)
    out, lse = R.attend_pages(s.cache, 0, q, ws, want_lse=True)
    s.compare(out, lse, q)
    got = R.read_pages(s.cache, 0, 8, ws, first=s.cache.lengths)
    assert torch.equal(got[0][4:].double(), s.plain.k[1, 70:74])


@pytest.mark.parametrize("scale", [0.0, -0.3, 8.0])
@pytest.mark.parametrize("pages", [BF16, E4M3])
def test_scales(pages, scale):
    s = Setup(pages, 2, 64, [150], [20]).fill()
    s.check(randn((20, 4, 64), 5, F32), scale=scale)


def test_sequences_share_pages():
    s = Setup(BF16, 2, 64, [128, 128], [3, 5]).fill()
    s.cache.table[1, :2] = s.cache.table[0, :2]
    s.plain.k[1, :128], s.plain.v[1, :128] = s.plain.k[0, :128], s.plain.v[0, :128]
    s.check(randn((8, 4, 64), 5))


@pytest.mark.parametrize("pages", [BF16, E4M3])
@pytest.mark.parametrize("bad", [NAN, INF, -INF])
@pytest.mark.parametrize("dim", [64, 128])
def test_what_a_row_does_not_see_does_not_reach_it(pages, bad, dim):
    """Keys and values of later rows that are not finite; the rows that see them are not finite either."""
    s = Setup(pages, 2, dim, [70], [30], garbage=0xFF).fill()
    k, v = randn((30, 2, dim), 3, F32), randn((30, 2, dim), 4, F32)
    k[20, 0] = NAN                     # position 90, KV head 0
    v[25, 1, 3] = bad                  # position 95, KV head 1, one dim
    s.write([70], [30], k, v)
    for dtype in (BF16, F32):
        q = randn((30, 4, dim), 5, dtype)
        ws = s.workspace(4)
        out, lse = R.attend_pages(s.cache, 0, q, ws, row_start=s.row_start, want_lse=True)
        clean = Setup(pages, 2, dim, [70], [30]).fill()
        clean.write([70], [30], torch.nan_to_num(k, 0.0, 0.0, 0.0), torch.nan_to_num(v, 0.0, 0.0, 0.0))
        o2, l2 = R.attend_pages(clean.cache, 0, q, ws, row_start=s.row_start, want_lse=True)
        fine = torch.ones_like(out, dtype=torch.bool)
        fine[20:, :2] = False
        fine[25:, 2:, 3] = False
        assert torch.equal(out[fine], o2[fine])
        assert bool(torch.isnan(out[20:, :2]).all()) and bool(torch.isnan(lse[20:, :2]).all())
        hit = out[25:, 2:, 3]
        # 8 bits have no infinity
        assert bool(torch.isnan(hit).all()) if pages == E4M3 or bad != bad else bool((hit == bad).all())
        assert torch.equal(lse[:20], l2[:20]) and torch.equal(lse[:, 2:], l2[:, 2:])


def test_values_not_finite_of_both_signs():
    s = Setup(BF16, 1, 64, [60], [10])
    rows = randn((60, 1, 64), 1)
    s.write([0], [60], rows, rows)
    v = randn((10, 1, 64), 2)
    v[3, 0, 5], v[6, 0, 5] = INF, -INF
    s.write([60], [10], randn((10, 1, 64), 3), v)
    out, _ = R.attend_pages(s.cache, 0, randn((10, 1, 64), 5), s.workspace(1), row_start=s.row_start)
    col = out[:, 0, 5]
    assert bool(torch.isfinite(col[:3]).all()) and bool((col[3:6] == INF).all()) and bool(torch.isnan(col[6:]).all())
    assert bool(torch.isfinite(out[:, 0, :5]).all())


TILES = [(1, 4, 1), (8, 8, 2), (40, 4, 2), (80, 8, 2)]     # rows, query heads, KV heads: a tile of 16, one of 32, several with two halves, eight


@pytest.mark.parametrize("n,q_heads,kv_heads", TILES)
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_infinite_values_wherever_they_stand(n, q_heads, kv_heads, dim, dtype):
    """Values among the first, middle and last committed rows and the new ones: each row that sees one has it in that dim, both signs
    make NaN, and all other numbers are those of the same call without them, bit for bit."""
    lens, news = [300, 1900], [n, n]
    k, v, kn, vn = (randn((m, kv_heads, dim), i, BF16) for i, m in ((1, 2200), (2, 2200), (3, 2 * n), (4, 2 * n)))
    q = randn((2 * n, q_heads, dim), 5, dtype)
    got = []
    at = [(0, INF, 3), (130, -INF, 4), (299, INF, 5), (17, INF, 6), (250, -INF, 6), (300, NAN, 8), (1500, INF, 9), (2199, -INF, 10)]   # row, value, dim
    G, H = q_heads // kv_heads, kv_heads - 1
    for odd in (True, False):
        v2, vn2 = v.clone(), vn.clone()
        if odd:
            for row, bad, d in at:
                v2[row, H, d] = bad
            vn2[0, H, 12] = INF
        s = Setup(BF16, kv_heads, dim, lens, news)
        s.write([0, 0], lens, k, v2)
        s.write(lens, news, kn, vn2)
        got.append(R.attend_pages(s.cache, 0, q, s.workspace(q_heads), row_start=s.row_start, max_rows=n, want_lse=True))
    (out, lse), (clean, lse2) = got
    want = clean.clone()
    hs = slice(H * G, (H + 1) * G)
    for d, bad in ((3, INF), (4, -INF), (5, INF), (6, NAN), (12, INF)):
        want[:n, hs, d] = bad
    for d, bad in ((8, NAN), (9, INF), (10, -INF)):
        want[n:, hs, d] = bad
    same = (out == want) | (torch.isnan(out) & torch.isnan(want))
    assert bool(same.all()), (~same).nonzero()[:5].tolist()
    assert torch.equal(lse, lse2)


@pytest.mark.parametrize("n,q_heads,kv_heads", TILES)
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_infinite_keys(n, q_heads, kv_heads, dim, dtype):
    """A score of -inf has weight 0: the row is that of a key of -1e30 there, bit for bit; one of +inf makes it NaN."""
    lens, news = [300, 1900], [n, n]
    k, v, kn, vn = (randn((m, kv_heads, dim), i, BF16) for i, m in ((1, 2200), (2, 2200), (3, 2 * n), (4, 2 * n)))
    q = randn((2 * n, q_heads, dim), 5, dtype)
    q[..., 7] += torch.where(q[..., 7] >= 0, 0.5, -0.5).to(dtype)
    G, got = q_heads // kv_heads, []
    for bad in (INF, 1e30):
        for row in (70, 900):
            k[row, :, 7] = -bad
        s = Setup(BF16, kv_heads, dim, lens, news)
        s.write([0, 0], lens, k, v)
        s.write(lens, news, kn, vn)
        got.append(R.attend_pages(s.cache, 0, q, s.workspace(q_heads), row_start=s.row_start, max_rows=n, want_lse=True))
    (out, lse), (clean, lse2) = got
    fine = q[..., 7] > 0
    assert bool(fine.any()) and bool((~fine).any())
    assert torch.equal(out[fine], clean[fine]) and torch.equal(lse[fine], lse2[fine])
    assert bool(torch.isnan(out[~fine]).all()) and bool(torch.isnan(lse[~fine]).all())


def test_large_scores_and_queries_not_finite():
    s = Setup(BF16, 1, 64, [100], [4])
    k = randn((100, 1, 64), 1, BF16, 100.0)
    s.write([0], [100], k, randn((100, 1, 64), 2))
    s.write([100], [4], k[:4], randn((4, 1, 64), 3))
    s.check(randn((4, 2, 64), 5, F32, 100.0))      # scores of thousands: one key has all of the weight
    q = randn((4, 2, 64), 6, F32)
    q[1, 0, 7], q[2, 1, 0] = NAN, INF
    out, lse = R.attend_pages(s.cache, 0, q, s.workspace(2), row_start=s.row_start, want_lse=True)
    odd = torch.zeros((4, 2), dtype=torch.bool, device=DEV)
    odd[1, 0] = odd[2, 1] = True
    assert torch.equal(torch.isnan(out).all(-1), odd) and torch.equal(torch.isnan(lse), odd)
    assert torch.equal(torch.isnan(out).any(-1), odd)


# ------------------------------------------------------------------------------------------ what only the device sees
def test_bad_pages_are_left_out():
    s = Setup(BF16, 2, 64, [130], [3]).fill()
    q = randn((3, 4, 64), 5)
    ws = R.PagesWorkspace(s.cache, 4, 133)
    for bad in (-1, s.cache.n_pages, 2 ** 31 - 1, -2 ** 31):
        s.cache.table[0, 1] = bad
        out, lse = R.attend_pages(s.cache, 0, q, ws, row_start=s.row_start, want_lse=True)
        assert R.read_device_status(ws) == C.NLD_DEV_BAD_PAGE
        lists = on_device([0, 2]).repeat(1, 1, 2, 1)
        s.compare(out, lse, q, lists=lists, group=3)
        k = torch.full((133, 2, 64), 5.0, device=DEV)
        v = k.clone()
        R.read_pages(s.cache, 0, 133, ws, outs=(k, v))
        assert R.read_device_status(ws) == C.NLD_DEV_BAD_PAGE and bool((k[64:128] == 5.0).all()) and torch.equal(v[128:].double(), s.plain.v[0, 128:133])
        s.cache.lengths.fill_(60)
        before = s.cache.k.clone()
        rows = randn((70, 2, 64), 9)
        R.write_pages(s.cache, 0, rows, rows, ws)
        assert R.read_device_status(ws) == C.NLD_DEV_BAD_PAGE
        same = (s.cache.k == before).flatten(2).all(-1)[0]
        assert int((~same).sum()) == 2       # pages 0 and 2
        s = Setup(BF16, 2, 64, [130], [3]).fill()


def test_rows_past_the_table_and_bad_lengths():
    s = Setup(BF16, 1, 64, [120], [8], slack=0).fill()     # 128 positions: the table is full
    ws = s.workspace(2, 20)
    rows = randn((20, 1, 64), 9)
    R.write_pages(s.cache, 0, rows, rows, ws)
    assert R.read_device_status(ws) == C.NLD_DEV_CAPACITY
    k, _ = R.read_pages(s.cache, 0, 8, ws, first=s.cache.lengths)
    assert torch.equal(k, rows[:8].float())
    q = randn((20, 2, 64), 3)
    out, _ = R.attend_pages(s.cache, 0, q, ws)
    assert R.read_device_status(ws) == C.NLD_DEV_CAPACITY and bool(torch.isfinite(out).all())
    for length, bit in ((-5, C.NLD_DEV_BAD_LENGTH), (-2 ** 31, C.NLD_DEV_BAD_LENGTH), (2 ** 31 - 1, C.NLD_DEV_CAPACITY), (129, C.NLD_DEV_CAPACITY)):
        s.cache.lengths.fill_(length)
        out, _ = R.attend_pages(s.cache, 0, q, ws)
        assert R.read_device_status(ws) == bit and bool(torch.isfinite(out).all())
        if length < 0:
            R.read_pages(s.cache, 0, 20, ws, first=s.cache.lengths)
            assert R.read_device_status(ws) == bit
        R.write_pages(s.cache, 0, rows, rows, ws)
        assert R.read_device_status(ws) == bit


def test_bad_row_starts():
    s = Setup(BF16, 1, 64, [20, 30], [4, 4]).fill()
    ws = s.workspace(2, 8)
    q = randn((8, 2, 64), 3)
    for start in ([0, 4, 9], [-1, 4, 8], [0, 2 ** 31 - 1, 8], [4, 0, 2], [0, 8, 8]):
        out = torch.full_like(q, 5.0)
        R.attend_pages(s.cache, 0, q, ws, row_start=on_device(start), max_rows=4, out=out)
        assert R.read_device_status(ws) == C.NLD_DEV_BAD_ROWS, start
        rows = randn((8, 1, 64), 9)
        R.write_pages(s.cache, 0, rows, rows, ws, row_start=on_device(start), max_rows=4)
        assert R.read_device_status(ws) == C.NLD_DEV_BAD_ROWS, start


def test_sequences_without_rows_report_nothing():
    """A padded batch: what stands in the places of a sequence that has no rows is not looked at."""
    s = Setup(BF16, 1, 64, [20, 30, 40], [4, 0, 4]).fill()
    ws = s.workspace(2, 8, 4)
    s.cache.table[1] = -7
    q, rows = randn((8, 2, 64), 3), randn((8, 1, 64), 4)
    for bad in (-1, -2 ** 31, 2 ** 31 - 1):
        s.cache.lengths[1] = bad
        first = on_device([20, bad, 40])
        R.write_pages(s.cache, 0, rows, rows, ws, row_start=s.row_start, max_rows=4)
        k, _ = R.read_pages(s.cache, 0, 8, ws, first=first, row_start=s.row_start, max_rows=4)
        assert torch.equal(k, rows.float())
        R.attend_pages(s.cache, 0, q, ws, row_start=s.row_start, max_rows=4)
        lists = R.select_pages(s.cache, 0, q, ws, 1, group=4, row_start=s.row_start, max_rows=4)
        assert bool((lists[1] == -1).all())
        R.attend_pages(s.cache, 0, q, ws, pages=lists, group=4, row_start=s.row_start, max_rows=4)
        assert R.read_device_status(ws) == 0, bad


@pytest.mark.parametrize("group", [1, 20])
def test_rows_past_the_table_with_a_list(group):
    s = Setup(BF16, 1, 64, [120], [8], slack=0).fill()     # 128 positions: the table is full
    ws = s.workspace(4, 20, 1)
    q = randn((20, 4, 64), 3)
    lists = on_device([0, 1]).repeat(1, 20 // group, 1, 1)
    R.attend_pages(s.cache, 0, q[:8], ws, pages=lists[:, :-(-8 // group)].contiguous(), group=group)
    assert R.read_device_status(ws) == 0
    out, lse = R.attend_pages(s.cache, 0, q, ws, pages=lists, group=group, want_lse=True)
    assert R.read_device_status(ws) == C.NLD_DEV_CAPACITY
    s.lens, s.start, s.news, s.most = [120], [0, 20], [20], 20
    s.compare(out, lse, q, lists=lists, group=group)       # rows past the table see all of it


STARTS = [([4, -2 ** 31, 8], [], [0, 1, 2, 3]), ([4, 3 - 2 ** 31, -2 ** 31], [], []), ([-2 ** 31, 4, -2 ** 31], [0, 1, 2, 3], []),
          ([0, 2 ** 31 - 1, -2 ** 31], [0, 1, 2, 3], []), ([-1, -1, 2 ** 31 - 1], [], [0, 1, 2, 3]), ([8, 8, -5], [], []), ([6, 9, 2], [6, 7], []),
          ([7, -2 ** 31 + 6, 3], [], [0, 1, 2])]


@pytest.mark.parametrize("pages", [BF16, E4M3])
@pytest.mark.parametrize("start,first,second", STARTS)
def test_bad_row_starts_reach_no_other_rows(pages, start, first, second):
    """8 rows, at most 4 each: the rows that either sequence has, and no others, are read and written, whatever the starts are.  The rows lie
    inside larger arrays."""
    s = Setup(pages, 1, 64, [20, 30], [4, 4]).fill()
    ws = s.workspace(2, 8, 4)
    has = torch.zeros(24, dtype=torch.bool, device=DEV)
    has[[8 + r for r in first + second]] = True
    inner = slice(8, 16)
    row_start = on_device(start)
    q, out, lse = randn((24, 2, 64), 3), torch.full((24, 2, 64), 5.0, dtype=BF16, device=DEV), torch.full((24, 2), 5.0, device=DEV)
    R.attend_pages(s.cache, 0, q[inner], ws, row_start=row_start, max_rows=4, out=out[inner], lse=lse[inner])
    assert R.read_device_status(ws) == C.NLD_DEV_BAD_ROWS
    assert torch.equal((out != 5.0).flatten(1).any(1), has) and torch.equal((lse != 5.0).any(1), has)
    k, v = (torch.full((24, 1, 64), 5.0, device=DEV) for _ in range(2))
    R.read_pages(s.cache, 0, 8, ws, row_start=row_start, max_rows=4, outs=(k[inner], v[inner]))
    assert R.read_device_status(ws) == C.NLD_DEV_BAD_ROWS
    for x, plain in ((k, s.plain.k), (v, s.plain.v)):
        for b, rows in enumerate((first, second)):
            for i, r in enumerate(rows):
                assert torch.equal(x[8 + r].double(), plain[b, i])
        assert bool((x[~has] == 5.0).all())
    lists = R.select_pages(s.cache, 0, q[inner], ws, 1, group=4, row_start=row_start, max_rows=4)
    assert R.read_device_status(ws) == C.NLD_DEV_BAD_ROWS
    assert [bool((lists[b] == -1).all()) for b in range(2)] == [not first, not second]
    rows = randn((24, 1, 64), 9)
    R.write_pages(s.cache, 0, rows[inner], rows[inner], ws, row_start=row_start, max_rows=4)
    assert R.read_device_status(ws) == C.NLD_DEV_BAD_ROWS
    for b, mine in enumerate((first, second)):
        new = ref.stored(rows[[8 + r for r in mine]], pages == E4M3)
        p = s.lens[b]
        s.plain.k[b, p:p + len(mine)] = s.plain.v[b, p:p + len(mine)] = new
    k, v = R.read_pages(s.cache, 0, 58, ws, row_start=on_device([0, 24, 58]), max_rows=34)
    assert torch.equal(k[:24].double(), s.plain.k[0, :24]) and torch.equal(k[24:].double(), s.plain.k[1, :34])
    assert torch.equal(v[:24].double(), s.plain.v[0, :24]) and torch.equal(v[24:].double(), s.plain.v[1, :34])


# ------------------------------------------------------------------------------------------ lists and selection
@pytest.mark.parametrize("group", [1, 3, 8])
def test_lists(group):
    s = Setup(E4M3, 2, 64, [500, 90], [8, 5]).fill()
    groups = -(-8 // group)
    lists = torch.full((2, groups, 2, 7), -1, dtype=torch.int32)
    for j in range(groups):
        lists[0, j, 0, :3] = torch.tensor([0, 3, 7])
        lists[0, j, 1, 2:7] = torch.tensor([7, 6, 1, 2, 8])      # any order, empty places in front; page 8 is past the last row
        lists[1, j, 0, 1] = 1
        # sequence 1, head 1: nothing at all
    s.check(randn((13, 4, 64), 5), lists=lists.to(DEV), group=group)
    s.check(randn((13, 4, 64), 5, F32), mode=1, lists=lists.to(DEV), group=group)


def test_a_page_listed_twice_counts_twice():
    s = Setup(BF16, 1, 64, [200], [1]).fill()
    s.check(randn((1, 2, 64), 5), lists=on_device([1, 1, 3]).view(1, 1, 1, 3))


def test_list_entries_out_of_range():
    s = Setup(BF16, 1, 64, [200], [1]).fill()
    ws = s.workspace(2, group=1)
    q = randn((1, 2, 64), 5)
    for bad in (-2, s.cache.max_len // 64, 2 ** 31 - 1, -2 ** 31):
        out, lse = R.attend_pages(s.cache, 0, q, ws, pages=on_device([0, bad, 3]).view(1, 1, 1, 3), row_start=s.row_start, want_lse=True)
        assert (R.read_device_status(ws) == C.NLD_DEV_BAD_PAGE) == (bad < 0)
        s.compare(out, lse, q, lists=on_device([0, 3]).view(1, 1, 1, 2))


SELECT = [([900], [1], 1, 4, 1, 0), ([64, 0, 700], [1, 1, 1], 1, 3, 0, 0), ([450, 127], [16, 9], 4, 2, 1, 0), ([130, 600], [70, 70], 16, 5, 2, 0),
          ([640], [16], 16, 6, 4, 1), ([300, 5], [33, 20], 8, 0, 1, 1), ([400], [3], 1, 100, 0, 0)]


@pytest.mark.parametrize("launches", ["one", "two"])
@pytest.mark.parametrize("pages", [BF16, E4M3])
@pytest.mark.parametrize("lens,news,group,n_top,n_first,mode", SELECT)
def test_selection(monkeypatch, launches, pages, lens, news, group, n_top, n_first, mode):
    monkeypatch.setenv("NLD_SELECT_ONE", "1" if launches == "one" else "0")
    for dim, dtype in ((64, F32), (128, BF16)):
        s = Setup(pages, 2, dim, lens, news).fill()
        q = randn((s.rows, 8, dim), 5, dtype)
        ws = s.workspace(8, group=group)
        got = R.select_pages(s.cache, 0, q, ws, n_top, group=group, n_first=n_first, mode=mode, bidir_from=min(2, s.most), row_start=s.row_start, max_rows=s.most)
        assert R.read_device_status(ws) == 0
        want = ref.select(s.plain, s.lens, s.start, q, n_top, n_first, group, got.shape[3], mode == 1, min(2, s.most))
        for b, n in enumerate(news):
            assert torch.equal(got[b, :-(-n // group)], want[b, :-(-n // group)])
            assert bool((got[b, -(-n // group):] == -1).all())
        s.check(q, mode=mode, bidir_from=min(2, s.most), lists=got, group=group)


@pytest.mark.parametrize("launches", ["one", "two"])
def test_selection_takes_the_lower_page_among_equal_scores(monkeypatch, launches):
    """Pages with one and the same keys, scores of zero of both signs, and more of them than the block of one count."""
    monkeypatch.setenv("NLD_SELECT_ONE", "1" if launches == "one" else "0")
    s = Setup(BF16, 1, 64, [64 * 40], [1])
    k = torch.zeros((64 * 40, 1, 64), dtype=BF16, device=DEV)
    k[64 * 5:64 * 6], k[64 * 31:64 * 32], k[64 * 33:64 * 35] = 1.0, 1.0, -1.0
    s.write([0], [64 * 40], k, k)
    s.write([64 * 40], [1], k[:1], k[:1])
    ws = s.workspace(1, group=1)
    q = torch.ones((1, 1, 64), device=DEV)
    assert R.select_pages(s.cache, 0, q, ws, 4, n_first=0)[0, 0, 0].tolist()[:5] == [0, 1, 5, 31, 40]
    assert R.select_pages(s.cache, 0, -q, ws, 4, n_first=0)[0, 0, 0].tolist()[:5] == [0, 1, 33, 34, 40]


@pytest.mark.parametrize("launches", ["one", "two"])
def test_selection_of_what_is_not_finite(monkeypatch, launches):
    monkeypatch.setenv("NLD_SELECT_ONE", "1" if launches == "one" else "0")
    s = Setup(BF16, 1, 64, [640], [2])
    k = randn((642, 1, 64), 1)
    k[64 * 7 + 3, 0, 9] = NAN
    s.write([0], [640], k[:640], k[:640])
    s.write([640], [2], k[640:], k[640:])
    ws = s.workspace(2, group=2)
    q = randn((2, 2, 64), 5)
    assert 7 in R.select_pages(s.cache, 0, q, ws, 1, n_first=0, group=2)[0, 0, 0].tolist()
    q[0, 0, 0], q[1, 1, 3] = NAN, INF          # the other two rows decide
    got = R.select_pages(s.cache, 0, q, ws, 3, n_first=0, group=2)
    assert torch.equal(got, ref.select(s.plain, [640], [0, 2], q, 3, 0, 2, got.shape[3]))
    q[:] = NAN
    assert R.select_pages(s.cache, 0, q, ws, 2, n_first=1, group=2)[0, 0, 0].tolist()[:4] == [0, 1, 7, 10]


@pytest.mark.parametrize("launches", ["one", "two"])
def test_selection_over_a_long_sequence(monkeypatch, launches):
    """More pages than one workgroup scores at a time, and than fit one round of the pick."""
    monkeypatch.setenv("NLD_SELECT_ONE", "1" if launches == "one" else "0")
    s = Setup(E4M3, 2, 64, [64 * 1100 + 7], [2]).fill()
    q = randn((2, 4, 64), 5)
    ws = s.workspace(4, group=2)
    got = R.select_pages(s.cache, 0, q, ws, 20, group=2)
    bd, bs = s.cache.bounds[0].double(), s.cache.bound_scale[0]
    ids = s.cache.table[0, :1101].long()
    qs = ref.over_127(q.float().abs().amax(-1))
    qi = torch.round(q.float() / qs[..., None]).double()
    for h in range(2):
        x, u = qi[:, 2 * h:2 * h + 2].reshape(4, 64), qs[:, 2 * h:2 * h + 2].reshape(4)
        acc = torch.maximum(x[:, None] * bd[ids, h, 0], x[:, None] * bd[ids, h, 1]).sum(-1).float()
        score = (acc * u[:, None]).amax(0) * bs[ids, h]
        score[0], score[1100] = -INF, -INF
        best = torch.sort(score, descending=True, stable=True)[1][:20].tolist()
        assert got[0, 0, h].tolist()[:22] == sorted(best + [0, 1100])
    s.check(q, lists=got, group=2)


@pytest.mark.parametrize("group", [1, 3])
def test_selection_over_more_pages_than_one_workgroup_keeps(group):
    """Over 4096 candidates: their scores stay in memory."""
    n, rows = 4200, 3
    s = Setup(E4M3, 1, 64, [64 * n + 7], [rows]).fill()
    q = randn((rows, 4, 64), 5)
    got = R.select_pages(s.cache, 0, q, s.workspace(4, group=group), 30, group=group)
    bd, bs = s.cache.bounds[0].double(), s.cache.bound_scale[0]
    ids = s.cache.table[0, :n].long()
    qs = ref.over_127(q.float().abs().amax(-1))
    qi = torch.round(q.float() / qs[..., None]).double()
    score = torch.cat([torch.clamp(qi, max=0.0), torch.clamp(qi, min=0.0)], -1) @ torch.cat([bd[ids, 0, 0], bd[ids, 0, 1]], -1).T     # whole numbers
    score = (score.float() * qs[..., None]).amax(1)
    for j in range(-(-rows // group)):
        best = torch.sort((score[j * group:(j + 1) * group].amax(0) * bs[ids, 0])[1:], descending=True, stable=True)[1][:30] + 1
        assert got[0, j, 0].tolist()[:32] == sorted(best.tolist() + [0, n])
    s.check(q, lists=got, group=group)


@pytest.mark.parametrize("launches", ["one", "two"])
@pytest.mark.parametrize("width", [300, 5000])
def test_selection_of_the_first_and_own_pages_alone(monkeypatch, launches, width):
    """n_top 0 needs no scores, and a workspace of 256 bytes will do: here the end of an allocation."""
    monkeypatch.setenv("NLD_SELECT_ONE", "1" if launches == "one" else "0")
    c = R.PagedCache(2, 64, 2, 64 * width, n_pages=1, bounds=True, device=DEV)
    c.table.zero_()                       # one page in every place: none is read
    c.lengths.copy_(on_device([64 * width - 66, 5]))
    buf = torch.zeros(1024, dtype=torch.uint8, device=DEV)[768:]
    ws = SimpleNamespace(buf=buf, ptr=buf.data_ptr(), nbytes=256)
    for group, n_first in ((1, 0), (4, 3)):
        got = R.select_pages(c, 0, randn((8, 4, 64), 5), ws, 0, group=group, n_first=n_first)
        assert R.read_device_status(ws) == 0
        for b, p in enumerate((64 * width - 66, 5)):
            for j in range(got.shape[1]):
                own = range((p + j * group) // 64, (p + min((j + 1) * group, 4) - 1) // 64 + 1)
                want = sorted(set(range(min(n_first, own[0]))) | set(own))
                assert got[b, j].tolist() == [want + [-1] * (got.shape[3] - len(want))] * 2


def test_a_workspace_serves_selections_in_one_launch_and_in_two():
    """300 units take one launch and room for 255 units' scores; 255, 254 and 100 of them take two, in the same workspace."""
    s = Setup(BF16, 1, 64, [64 * 300], [300]).fill()
    q = randn((300, 2, 64), 5)
    ws = s.workspace(2, 300, 1)
    ids = s.cache.table[0, :304].long()
    bd, bs = s.cache.bounds[0][ids, 0].double(), s.cache.bound_scale[0][ids, 0]
    qs = ref.over_127(q.float().abs().amax(-1))
    qi = torch.round(q.float() / qs[..., None]).double()
    score = torch.cat([torch.clamp(qi, max=0.0), torch.clamp(qi, min=0.0)], -1) @ torch.cat([bd[:, 0], bd[:, 1]], -1).T     # whole numbers
    score = (score.float() * qs[..., None]).amax(1) * bs
    for n in (300, 256, 255, 254, 100):
        got = R.select_pages(s.cache, 0, q[:n], ws, 6)[0, :, 0].tolist()
        assert R.read_device_status(ws) == 0
        for i in range(n):
            own = (64 * 300 + i) // 64
            best = torch.sort(score[i, 1:own], descending=True, stable=True)[1][:6] + 1
            assert got[i] == sorted(best.tolist() + [0, own]), (n, i)


# ------------------------------------------------------------------------------------------ together, as they are used
@pytest.mark.parametrize("pages", [BF16, E4M3])
def test_a_prompt_then_decoding_by_selected_pages(pages):
    """A prompt read in by chunks, then tokens one by one: write, select, attend, commit."""
    H, D, Hq = 2, 64, 8
    s = Setup(pages, H, D, [0, 0], [330, 290])
    ws = R.PagesWorkspace(s.cache, Hq, 128, 1)
    done = [0, 0]
    for step in range(4):
        news = [min(128, n - d) for n, d in zip((300, 260), done)]
        news = [max(n, 0) for n in news]
        if max(news) == 0:
            break
        st = starts_of(news)
        k, v, q = randn((st[-1], H, D), 10 + step), randn((st[-1], H, D), 20 + step), randn((st[-1], Hq, D), 30 + step)
        R.write_pages(s.cache, 0, k, v, ws, row_start=on_device(st), max_rows=max(news))
        out, lse = R.attend_pages(s.cache, 0, q, ws, row_start=on_device(st), max_rows=max(news), want_lse=True)
        s.plain.write(done, st, k, v)
        s.lens, s.start = list(done), st
        s.compare(out, lse, q)
        s.cache.lengths += on_device(news)
        done = [d + n for d, n in zip(done, news)]
    assert done == [300, 260]
    for step in range(24):
        k, v, q = randn((2, H, D), 50 + step), randn((2, H, D), 80 + step), randn((2, Hq, D), 110 + step)
        R.write_pages(s.cache, 0, k, v, ws)
        pages_ = R.select_pages(s.cache, 0, q, ws, 2)
        out, lse = R.attend_pages(s.cache, 0, q, ws, pages=pages_, want_lse=True)
        s.plain.write(done, [0, 1, 2], k, v)
        s.lens, s.start = list(done), [0, 1, 2]
        assert torch.equal(pages_, ref.select(s.plain, done, [0, 1, 2], q, 2, 1, 1, pages_.shape[3]))
        s.compare(out, lse, q, lists=pages_)
        s.cache.lengths += 1
        done = [d + 1 for d in done]
    assert R.read_device_status(ws) == 0


def test_captured_steps_follow_the_lengths():
    """write, select and attend in one graph; lengths, rows and table change between replays, eager work in between."""
    H, D, Hq = 2, 128, 8
    s = Setup(E4M3, H, D, [250, 100], [40, 40]).fill()
    ws = R.PagesWorkspace(s.cache, Hq, 1, 1)
    k, v, q = randn((2, H, D), 1), randn((2, H, D), 2), randn((2, Hq, D), 3)
    out, lse = torch.empty_like(q), torch.empty((2, Hq), device=DEV)
    pages_ = torch.empty((2, 1, H, R.C.load().nld_pages_list_len(1, 1, 2, 1, 0)), dtype=torch.int32, device=DEV)

    def step():
        R.write_pages(s.cache, 0, k, v, ws)
        R.select_pages(s.cache, 0, q, ws, 2, out=pages_)
        R.attend_pages(s.cache, 0, q, ws, pages=pages_, out=out, lse=lse)
        s.cache.lengths += 1

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    s.cache.lengths.copy_(on_device([250, 100]))
    done = [250, 100]
    for i in range(5):
        for x, seed in ((k, 200), (v, 300), (q, 400)):
            x.copy_(randn(x.shape, seed + i))
        graph.replay()
        s.plain.write(done, [0, 1, 2], k, v)
        s.lens, s.start = list(done), [0, 1, 2]
        s.compare(out, lse, q, lists=pages_)
        assert torch.equal(pages_, ref.select(s.plain, done, [0, 1, 2], q, 2, 1, 1, pages_.shape[3]))
        done = [d + 1 for d in done]
        assert s.cache.lengths.tolist() == done


def test_calls_on_another_stream_and_repeats_are_bit_identical():
    s = Setup(BF16, 4, 128, [3000, 700, 1500], [5, 16, 1]).fill()
    q = randn((s.rows, 16, 128), 5)
    ws = s.workspace(16)
    want = R.attend_pages(s.cache, 0, q, ws, row_start=s.row_start, max_rows=16, want_lse=True)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        for _ in range(5):
            got = R.attend_pages(s.cache, 0, q, ws, row_start=s.row_start, max_rows=16, want_lse=True)
    side.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_a_workspace_serves_smaller_calls():
    s = Setup(BF16, 2, 64, [300, 10], [60, 40]).fill()
    ws = R.PagesWorkspace(s.cache, 8, 60, 1)
    q = randn((100, 8, 64), 5)
    for group in (1, 4, 16):
        lists = R.select_pages(s.cache, 0, q, ws, 2, group=group, row_start=s.row_start, max_rows=60)
        out, lse = R.attend_pages(s.cache, 0, q, ws, pages=lists, group=group, row_start=s.row_start, max_rows=60, want_lse=True)
        s.compare(out, lse, q, lists=lists, group=group)
    with pytest.raises(C.NLDError, match="workspace"):
        R.attend_pages(s.cache, 0, randn((200, 8, 64), 1), R.PagesWorkspace(s.cache, 8, 1))


def test_outputs_given_count_as_changed():
    s = Setup(BF16, 1, 64, [10], [2]).fill()
    q = randn((2, 1, 64), 5)
    out = torch.zeros_like(q)
    versions = out._version, s.cache.k._version
    R.attend_pages(s.cache, 0, q, s.workspace(1), out=out)
    R.write_pages(s.cache, 0, q, q, s.workspace(1))
    assert out._version > versions[0] and s.cache.k._version > versions[1]
