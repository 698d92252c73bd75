"""Block-decode passes over a paged cache, in bf16 and in 8 bits, whole and over selected pages: against a 64-bit decoder over the same stored
rows (tests/pages_ref.py block_pass), and in bf16 against the passes over the other cache.

Bound: the normwise 2e-2 of every pass test.  Both sides hold keys and values in the pages' type; a projection's f32 sum next to a rounding
border may fall on the other side, one step of the type for that element."""
import ctypes

import numpy as np
import pages_ref as ref
import pytest
import torch
from gpu_common import rel_err

pytestmark = pytest.mark.gpu

from synth.workloads import SHAPE_TINY, LazyWeights, ModelShape, tokens  # noqa: E402

if torch.cuda.is_available():
    from paper_2607_05722_amd import _lib as C
    from paper_2607_05722_amd import runtime as R

BF16, E4M3 = torch.bfloat16, torch.float8_e4m3fn
TOL = 2e-2


@pytest.fixture(scope="module")
def tiny():
    src = LazyWeights(SHAPE_TINY, 0)
    return SHAPE_TINY, src, R.DeviceModel(SHAPE_TINY, src)


def ids(shape, name, batch, n):
    return torch.from_numpy(tokens(shape, 0, name, (batch, n)).astype(np.int32)).cuda()


class Both:
    """A paged cache with a shuffled table, and the plain caches of its layers."""

    def __init__(self, shape, pages, batch, max_len, bounds=False, seed=3):
        self.cache = R.PagedCache(shape.n_kv_heads, shape.head_dim, batch, max_len, n_layers=shape.n_layers, n_pages=batch * max_len // 64 + 2,
                                  dtype=pages, bounds=bounds)
        order = torch.randperm(self.cache.n_pages, generator=torch.Generator().manual_seed(seed))[:batch * max_len // 64]
        self.cache.table.copy_(order.to(torch.int32).view(batch, -1))
        self.plain = [ref.Cache(batch, max_len, shape.n_kv_heads, shape.head_dim, pages == E4M3, "cuda") for _ in range(shape.n_layers)]


def prefill(tiny, both, lens, name="prefix"):
    """Rows of random keys and values as committed prefixes, in every layer."""
    shape, _, _ = tiny
    both.cache.lengths.zero_()
    starts = [0] + np.cumsum(lens).tolist()
    ws = R.PagesWorkspace(both.cache, shape.n_q_heads, max(lens))
    for l in range(shape.n_layers):
        g = torch.Generator().manual_seed(100 + l)
        k, v = (torch.randn((starts[-1], shape.n_kv_heads, shape.head_dim), generator=g).cuda() for _ in range(2))
        R.write_pages(both.cache, l, k, v, ws, row_start=torch.tensor(starts, dtype=torch.int32, device="cuda"), max_rows=max(lens))
        both.plain[l].write([0] * len(lens), starts, k, v)
    both.cache.lengths.copy_(torch.tensor(lens, dtype=torch.int32))


@pytest.mark.parametrize("pages", [BF16, E4M3])
@pytest.mark.parametrize("lens,k", [([128], 8), ([100, 1, 190], 16), ([63, 64], 1), ([5], 64)])
def test_block_passes(tiny, pages, lens, k):
    shape, src, model = tiny
    both = Both(shape, pages, len(lens), 320)
    prefill(tiny, both, lens)
    ws = R.PagedPassWorkspace(model, both.cache, k)
    toks = ids(shape, "block", len(lens), k)
    for mode, bidir in ((R.VERIFY, 0), (R.DRAFT, 0), (R.DRAFT, min(3, k))):
        logits, argmax = R.block_forward(model, both.cache, ws, toks, mode, bidir)
        assert R.read_device_status(ws) == 0
        want = ref.block_pass(shape, src, both.plain, lens, toks, mode == R.DRAFT, bidir).cpu().numpy()
        got = logits.cpu().numpy()
        assert rel_err(got, want) <= TOL
        assert np.array_equal(argmax.cpu().numpy(), got.argmax(-1))
        assert both.cache.lengths.tolist() == lens


@pytest.mark.parametrize("pages", [BF16, E4M3])
@pytest.mark.parametrize("sparse", [(2, 1, 1), (1, 0, 4), (3, 1, 16)])
def test_block_passes_over_selected_pages(tiny, pages, sparse):
    shape, src, model = tiny
    lens, k = [700, 330], 16
    both = Both(shape, pages, 2, 768, bounds=True)
    prefill(tiny, both, lens)
    ws = R.PagedPassWorkspace(model, both.cache, k, sparse)
    toks = ids(shape, "block", 2, k)
    for mode in (R.VERIFY, R.DRAFT):
        logits, _ = R.block_forward(model, both.cache, ws, toks, mode, 0, sparse=sparse)
        assert R.read_device_status(ws) == 0
        want = ref.block_pass(shape, src, both.plain, lens, toks, mode == R.DRAFT, 0, sparse).cpu().numpy()
        err = np.abs(logits.cpu().numpy() - want).max(-1) / np.abs(want).max()
        # the second layer's queries differ by rounding, so a page next to the border may change for a row: few do
        assert (err <= TOL).mean() >= 0.9, err
    whole, _ = R.block_forward(model, both.cache, R.PagedPassWorkspace(model, both.cache, k), toks, R.VERIFY)
    every, _ = R.block_forward(model, both.cache, R.PagedPassWorkspace(model, both.cache, k, (12, 0, 16)), toks, R.VERIFY, sparse=(12, 0, 16))
    assert rel_err(every.cpu().numpy(), whole.cpu().numpy()) <= 1e-5     # all pages: the same sums in other parts


# head_dim 128: two query heads to a KV head, and five
WIDE = {g: ModelShape(n_layers=2, hidden=256, n_q_heads=2 * g, n_kv_heads=2, head_dim=128, ffn=344, vocab=512) for g in (2, 5)}


@pytest.fixture(scope="module")
def wide():
    src = {g: LazyWeights(shape, 1) for g, shape in WIDE.items()}
    return {g: (WIDE[g], src[g], R.DeviceModel(WIDE[g], src[g])) for g in WIDE}


def by_row(got, want):
    """Norm of the difference over the norm, of each row."""
    return np.linalg.norm(got - want, axis=-1) / np.linalg.norm(want, axis=-1)


@pytest.mark.parametrize("pages", [BF16, E4M3])
@pytest.mark.parametrize("heads,lens,k", [(2, [300], 1), (2, [100, 1, 190], 8), (2, [63, 400], 16), (2, [64, 250], 33), (5, [130, 700], 3), (5, [300, 9], 32),
                                          (5, [60], 51)])
def test_block_passes_of_128_dims(wide, pages, heads, lens, k):
    """2 to 255 rows of a KV head (256 are the most of a pass): one tile of 16, of 32, several, and eight."""
    shape, src, model = wide[heads]
    both = Both(shape, pages, len(lens), 768)
    prefill(wide[heads], both, lens)
    ws = R.PagedPassWorkspace(model, both.cache, k)
    toks = ids(shape, "block", len(lens), k)
    for mode, bidir in ((R.VERIFY, 0), (R.DRAFT, 0), (R.DRAFT, min(3, k))):
        logits, argmax = R.block_forward(model, both.cache, ws, toks, mode, bidir)
        assert R.read_device_status(ws) == 0
        want = ref.block_pass(shape, src, both.plain, lens, toks, mode == R.DRAFT, bidir).cpu().numpy()
        got = logits.cpu().numpy()
        assert float(by_row(got, want).max()) <= TOL
        assert np.array_equal(argmax.cpu().numpy(), got.argmax(-1))


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("k", [12, 24, 40])
def test_infinite_keys_in_a_pass(dim, k):
    """Rows whose queries score -inf against a committed key are those of a key of 1e8 there, bit for bit; the others are NaN."""
    shape = ModelShape(n_layers=1, hidden=256, n_q_heads=2, n_kv_heads=2, head_dim=dim, ffn=344, vocab=512)
    model = R.DeviceModel(shape, LazyWeights(shape, 2))
    cache = R.PagedCache(2, dim, 1, 256)
    g = torch.Generator().manual_seed(7)
    rows, values = (torch.randn((150, 2, dim), generator=g).cuda() for _ in range(2))
    toks, got = ids(shape, "block", 1, k), []
    for big in (float("inf"), 1e8):
        rows[30, 1, 9] = big
        cache.lengths.zero_()
        R.write_pages(cache, 0, rows, values, R.PagesWorkspace(cache, 2, 150))
        cache.lengths.fill_(150)
        ws = R.PagedPassWorkspace(model, cache, k)
        got.append(R.block_forward(model, cache, ws, toks, R.VERIFY)[0][0])
        assert R.read_device_status(ws) == 0
    odd = torch.isnan(got[0])
    lost = odd.any(-1)
    assert torch.equal(lost, odd.all(-1)) and 0 < int(lost.sum()) < k
    assert torch.equal(got[0][~lost], got[1][~lost]) and bool(torch.isfinite(got[1]).all())


@pytest.mark.parametrize("pages", [BF16, E4M3])
@pytest.mark.parametrize("heads,k,sparse", [(2, 16, (2, 1, 1)), (2, 16, (1, 0, 4)), (5, 16, (3, 1, 16)), (5, 1, (4, 0, 1))])
def test_passes_of_128_dims_over_selected_pages(wide, pages, heads, k, sparse):
    """Every page has the keys of the first, times a power of two of its own: the scores of two pages are apart by a factor of two, so
    both sides choose the same, and every row is compared."""
    shape, src, model = wide[heads]
    lens = [700, 330]
    both = Both(shape, pages, 2, 768, bounds=True)
    starts, rows = [0, 700, 1030], torch.cat([torch.arange(n) for n in lens])
    power = torch.cat([torch.randperm(-(-n // 64), generator=torch.Generator().manual_seed(n))[torch.arange(n) // 64] - 5 for n in lens])
    ws = R.PagesWorkspace(both.cache, shape.n_q_heads, 700)
    for l in range(shape.n_layers):
        g = torch.Generator().manual_seed(200 + l)
        page = torch.randn((64, shape.n_kv_heads, shape.head_dim), generator=g)
        k_rows = (page[rows % 64] * 2.0 ** power[:, None, None]).cuda()
        v_rows = torch.randn((1030, shape.n_kv_heads, shape.head_dim), generator=g).cuda()
        R.write_pages(both.cache, l, k_rows, v_rows, ws, row_start=torch.tensor(starts, dtype=torch.int32, device="cuda"), max_rows=700)
        both.plain[l].write([0, 0], starts, k_rows, v_rows)
    both.cache.lengths.copy_(torch.tensor(lens, dtype=torch.int32))
    ws = R.PagedPassWorkspace(model, both.cache, k, sparse)
    toks = ids(shape, "block", 2, k)
    for mode in (R.VERIFY, R.DRAFT):
        logits, _ = R.block_forward(model, both.cache, ws, toks, mode, 0, sparse=sparse)
        assert R.read_device_status(ws) == 0
        want = ref.block_pass(shape, src, both.plain, lens, toks, mode == R.DRAFT, 0, sparse).cpu().numpy()
        err = by_row(logits.cpu().numpy(), want)
        assert float(err.max()) <= TOL, err


@pytest.mark.parametrize("k,group", [(1, 4), (2, 16), (4, 64)])
def test_selected_pages_of_groups_larger_than_the_block(tiny, k, group):
    """One workspace for draft and verify passes of a batch large enough that a list's rounding to 256 bytes hides no entry."""
    shape, _, model = tiny
    batch, sparse = 64 // shape.n_kv_heads * 2, (3, 1, group)
    both = Both(shape, BF16, batch, 640, bounds=True)
    prefill(tiny, both, [(41 * i) % 560 + 1 for i in range(batch)])
    ws = R.PagedPassWorkspace(model, both.cache, k, sparse)
    toks = ids(shape, "block", batch, k)
    for mode in (R.VERIFY, R.DRAFT):
        logits, _ = R.block_forward(model, both.cache, ws, toks, mode, 0, sparse=sparse)
        same, _ = R.block_forward(model, both.cache, R.PagedPassWorkspace(model, both.cache, k, (3, 1, k)), toks, mode, 0, sparse=(3, 1, k))
        assert R.read_device_status(ws) == 0 and torch.equal(logits, same)
    if k == 1:
        R.verify_accept(model, both.cache, ws, toks[:, 0].contiguous(), None, 1, sparse=sparse)
        assert R.read_device_status(ws) == 0


def test_steps_in_bf16_pages_follow_the_other_cache(tiny):
    """Draft, verify, accept, commit: from the same prefix, over both caches."""
    shape, _, model = tiny
    k, batch = 8, 2
    flat = R.DeviceCache(shape, batch, 256)
    both = Both(shape, BF16, batch, 256)
    prefix = ids(shape, "p", batch, 64)
    wf, wp = R.Workspace(model, batch, 64, 256), R.PagedPassWorkspace(model, both.cache, 64)
    R.block_forward(model, flat, wf, prefix, R.VERIFY, want_logits=False)
    R.block_forward(model, both.cache, wp, prefix, R.VERIFY, want_logits=False)
    flat.lengths += 64
    both.cache.lengths += 64
    wf, wp = R.Workspace(model, batch, k, 256), R.PagedPassWorkspace(model, both.cache, k)
    anchor = ids(shape, "a", batch, 1)[:, 0].contiguous()
    for step in range(6):
        d, dl = R.draft(model, flat, wf, anchor, k, want_logits=True)
        d2, dl2 = R.draft(model, both.cache, wp, anchor, k, want_logits=True)
        assert rel_err(dl2.cpu().numpy(), dl.cpu().numpy()) <= TOL
        v = R.verify_accept(model, flat, wf, anchor, d, k, want_logits=True)
        v2 = R.verify_accept(model, both.cache, wp, anchor, d, k, want_logits=True)
        assert rel_err(v2["logits"].cpu().numpy(), v["logits"].cpu().numpy()) <= TOL
        # acceptance by the pass's own logits
        own = R.accept_from_logits(v2["logits"], d)
        for name in ("accept_len", "committed", "next_anchor"):
            assert torch.equal(v2[name], own[name])
        anchor = v["next_anchor"]
        both.cache.lengths.copy_(flat.lengths)
    assert R.read_device_status(wp) == 0


def test_self_speculation_in_8_bits_captured(tiny):
    """A loop of draft and verify in one graph, in place: every replay equals the eager steps of a second cache."""
    shape, _, model = tiny
    k, batch = 4, 2
    sets = [Both(shape, E4M3, batch, 512, bounds=True) for _ in range(2)]
    for s in sets:
        prefill(tiny, s, [200, 75])
    sparse = (2, 1, 4)
    state = []
    for s in sets:
        st = dict(anchor=ids(shape, "a", batch, 1)[:, 0].contiguous(), d=torch.empty((batch, k - 1), dtype=torch.int32, device="cuda"),
                  ws=R.PagedPassWorkspace(model, s.cache, k, sparse), cache=s.cache)
        st["outs"] = {"accept_len": torch.empty(batch, dtype=torch.int32, device="cuda"), "committed": torch.empty((batch, k), dtype=torch.int32, device="cuda"),
                      "next_anchor": st["anchor"]}
        state.append(st)

    def step(st):
        R.draft(model, st["cache"], st["ws"], st["anchor"], k, out=st["d"], sparse=sparse)
        R.verify_accept(model, st["cache"], st["ws"], st["anchor"], st["d"], k, outs=st["outs"], sparse=sparse)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(state[0])
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(state[0])
    step(state[1])
    for _ in range(5):
        graph.replay()
        step(state[1])
        torch.cuda.synchronize()
        a, b = state
        assert torch.equal(a["d"], b["d"]) and torch.equal(a["cache"].lengths, b["cache"].lengths)
        for name in a["outs"]:
            assert torch.equal(a["outs"][name], b["outs"][name])
    assert R.read_device_status(state[0]["ws"]) == 0 and state[0]["cache"].lengths.tolist()[0] >= 206


@pytest.mark.parametrize("sparse", [None, (2, 1, 4)])
def test_a_traced_pass_has_its_attention(tiny, sparse):
    """One instance of the attention class per layer, with the time of its kernels; a pass is the same with tracing on."""
    shape, _, model = tiny
    both = Both(shape, BF16, 2, 512, bounds=True)
    prefill(tiny, both, [400, 75])
    ws, toks = R.PagedPassWorkspace(model, both.cache, 4, sparse), ids(shape, "block", 2, 4)
    want, _ = R.block_forward(model, both.cache, ws, toks, R.VERIFY, sparse=sparse)
    lib, n = C.load(), len(C.TRACE_CLASSES)
    ms, counts = (ctypes.c_float * n)(), (ctypes.c_int32 * n)()
    torch.cuda.synchronize()
    lib.nld_trace_enable(1)
    try:
        got, _ = R.block_forward(model, both.cache, ws, toks, R.VERIFY, sparse=sparse)
        R.write_pages(both.cache, 0, *(torch.zeros((8, shape.n_kv_heads, shape.head_dim), device="cuda") for _ in range(2)),
                      R.PagesWorkspace(both.cache, shape.n_q_heads, 4))       # not a pass: not recorded
        torch.cuda.synchronize()
        C.check(lib.nld_trace_read(ms, counts, n))
    finally:
        lib.nld_trace_enable(0)
    by = {name: (counts[i], ms[i]) for i, name in enumerate(C.TRACE_CLASSES)}
    assert by["attention"][0] == shape.n_layers and by["attention"][1] > 0.0, by
    assert by["qkv"][0] == shape.n_layers and torch.equal(got, want)


def test_the_drafters_loss_over_pages(tiny):
    shape, _, model = tiny
    both = Both(shape, BF16, 1, 256)
    prefill(tiny, both, [100])
    anchor = ids(shape, "a", 1, 1)[:, 0].contiguous()
    out = R.drafter_loss(model, both.cache, R.PagedPassWorkspace(model, both.cache, 8), R.LogitsWorkspace(1, 7, shape.vocab, 32), anchor, 8, n_top=32)
    assert bool(torch.isfinite(out["loss"]).all()) and both.cache.lengths.item() == 101 + out["accept_len"].item()


def test_missing_pages_and_full_tables(tiny):
    shape, _, model = tiny
    both = Both(shape, BF16, 1, 128)
    prefill(tiny, both, [120])
    anchor = ids(shape, "a", 1, 1)[:, 0].contiguous()
    ws = R.PagedPassWorkspace(model, both.cache, 16)
    R.draft(model, both.cache, ws, anchor, 16)
    assert R.read_device_status(ws) & C.NLD_DEV_CAPACITY
    both.cache.table[0, 1] = -1
    R.draft(model, both.cache, ws, anchor, 4)
    assert R.read_device_status(ws) == C.NLD_DEV_BAD_PAGE


def test_refusals(tiny):
    shape, _, model = tiny
    good = R.PagedCache(shape.n_kv_heads, shape.head_dim, 2, 128, n_layers=shape.n_layers)
    anchor = torch.zeros(2, dtype=torch.int32, device="cuda")
    ws = R.PagedPassWorkspace(model, good, 8)
    for kw in (dict(kv_heads=1), dict(head_dim=128), dict(n_layers=1)):
        sizes = dict(kv_heads=shape.n_kv_heads, head_dim=shape.head_dim, n_layers=shape.n_layers)
        bad = R.PagedCache(batch=2, max_len=128, **{**sizes, **kw})
        with pytest.raises(C.NLDError, match="the model"):
            R.draft(model, bad, ws, anchor, 8)
        with pytest.raises(ValueError):
            R.PagedPassWorkspace(model, bad, 8)
    with pytest.raises(C.NLDError, match="bounds"):
        R.draft(model, good, ws, anchor, 8, sparse=(1, 1, 1))
    with pytest.raises(C.NLDError, match="workspace"):
        R.draft(model, good, ws, anchor, 64)
    with pytest.raises(C.NLDError):
        R.draft(model, good, ws, anchor, 1)
    with pytest.raises(ValueError):
        R.draft(model, good, ws, anchor[:1], 8)
    with pytest.raises(ValueError):
        R.draft(model, good, ws, anchor, 8, sparse=(1, 1, 0))
    with pytest.raises(ValueError):
        R.draft(model, R.DeviceCache(shape, 2, 128), R.Workspace(model, 2, 8, 128), anchor, 8, sparse=(1, 1, 1))
    with pytest.raises(ctypes.ArgumentError):
        R.decode_steps(model, good, ws, anchor, 4, 1)      # the calls that have no form over pages
