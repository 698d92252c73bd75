"""The calls on a paged cache: argument checks (nothing is enqueued), and the plain versions that the GPU tests compare with. No GPU needed."""
import ctypes
from types import SimpleNamespace

import pages_ref as ref
import pytest
import torch

from paper_2607_05722_amd import _lib as C
from paper_2607_05722_amd import runtime as R

P = 0x1000
WS = 1 << 40
NAN, INF = float("nan"), float("inf")


def pages(**kw):
    f = dict(k=P, v=P, scale=None, bounds=None, bound_scale=None, dtype=C.NLD_BF16, n_layers=2, n_pages=10, n_kv_heads=2, head_dim=64, table=P,
             lengths=P, batch=3, max_pages=4)
    f.update(kw)
    return C.Pages(**f)


def chunk(rows=6, max_rows=2, row_start=None):
    return C.Chunk(rows, max_rows, row_start)


def heads(data=P, dtype=C.NLD_BF16, row=512, head=64):
    return C.Heads(data, dtype, row, head)


def ref_of(x):
    return ctypes.byref(x) if x is not None else None


def write(p=None, layer=0, ch=None, k=None, v=None, ws=P, ws_bytes=WS):
    return C.load().nld_pages_write(ref_of(p or pages()), layer, ref_of(ch or chunk()), ref_of(k or heads()), ref_of(v or heads()), ws, ws_bytes, None)


def read(p=None, layer=0, ch=None, k=None, v=None, ws=P, ws_bytes=WS):
    return C.load().nld_pages_read(ref_of(p or pages()), layer, ref_of(ch or chunk()), None, ref_of(k or heads()), ref_of(v or heads(2 * P)), ws, ws_bytes, None)


def attend(p=None, layer=0, ch=None, q=None, n_q=4, scale=0.1, mode=0, bidir=0, lst=None, n_list=0, group=0, out=None, ws=P, ws_bytes=WS):
    return C.load().nld_pages_attend(ref_of(p or pages()), layer, ref_of(ch or chunk()), ref_of(q or heads()), n_q, scale, mode, bidir, lst, n_list, group,
                                     ref_of(out or heads(1 << 44)), None, ws, ws_bytes, None)


def select(p=None, layer=0, ch=None, q=None, n_q=4, n_top=2, n_first=1, group=1, mode=0, bidir=0, lst=P, n_list=50, ws=P, ws_bytes=WS):
    return C.load().nld_pages_select(ref_of(p or pages(bounds=P, bound_scale=P)), layer, ref_of(ch or chunk()), ref_of(q or heads()), n_q, n_top, n_first,
                                     group, mode, bidir, lst, n_list, ws, ws_bytes, None)


CALLS = {"write": write, "read": read, "attend": attend, "select": select}
INVALID, SHAPE, CAPACITY = C.NLD_ERR_INVALID_ARG, C.NLD_ERR_SHAPE, C.NLD_ERR_CAPACITY


def full(**kw):
    return pages(**{"bounds": P, "bound_scale": P, **kw})


@pytest.mark.parametrize("call", CALLS.values(), ids=CALLS)
@pytest.mark.parametrize("field,value,status,text", [
    ("k", None, INVALID, "NULL"), ("v", None, INVALID, "NULL"), ("table", None, INVALID, "NULL"), ("lengths", None, INVALID, "NULL"),
    ("dtype", C.NLD_F32, INVALID, "dtype"), ("dtype", C.NLD_E4M3, INVALID, "scales"), ("n_layers", 0, INVALID, "positive"),
    ("n_pages", 0, INVALID, "positive"), ("n_kv_heads", -1, INVALID, "positive"), ("batch", 0, INVALID, "positive"),
    ("max_pages", 0, INVALID, "positive"), ("head_dim", 96, SHAPE, "head_dim"), ("head_dim", 256, SHAPE, "head_dim"),
    ("max_pages", (1 << 24) + 1, SHAPE, "max_pages"), ("k", P + 8, INVALID, "aligned"), ("bounds", P + 4, INVALID, "aligned"),
    ("bound_scale", None, INVALID, "together"), ("bound_scale", P + 2, INVALID, "aligned"),
])
def test_pages_are_checked(call, field, value, status, text):
    assert call(p=full(**{field: value})) == status
    assert text in C.load().nld_last_error().decode()


@pytest.mark.parametrize("call", CALLS.values(), ids=CALLS)
@pytest.mark.parametrize("kw,status,text", [
    (dict(layer=-1), INVALID, "layer"), (dict(layer=2), INVALID, "layer"),
    (dict(ch=chunk(0, 1)), INVALID, "max_rows"), (dict(ch=chunk(6, 0)), INVALID, "max_rows"), (dict(ch=chunk(6, 7, P)), INVALID, "max_rows"),
    (dict(ch=chunk(7, 2)), INVALID, "batch"), (dict(ch=chunk((1 << 24) + 1, 4, P)), SHAPE, "rows"),
    (dict(ws=None), INVALID, "workspace"), (dict(ws_bytes=255), CAPACITY, "workspace"),
])
def test_chunks_and_workspaces_are_checked(call, kw, status, text):
    assert call(**kw) == status
    assert text in C.load().nld_last_error().decode()


@pytest.mark.parametrize("call,name", [(write, "k"), (write, "v"), (read, "k"), (read, "v"), (attend, "q"), (attend, "out"), (select, "q")])
def test_rows_are_checked(call, name):
    error = lambda: C.load().nld_last_error().decode()
    for x, text in ((heads(None), "NULL"), (heads(dtype=C.NLD_E4M3), "dtype"), (heads(row=-1), "strides"), (heads(head=1 << 38), "strides"),
                    (heads(P + 1), "aligned"), (heads(P + 2, C.NLD_F32), "aligned")):
        assert call(**{name: x}) == INVALID and text in error() and name in error()
    if (call, name) in ((read, "k"), (read, "v"), (attend, "out")):
        n = 4 if call is attend else 2
        for x in (heads(head=63), heads(row=64 * n - 1), heads(row=0), heads(row=63, head=6 * 64), heads(row=64, head=6 * 64 - 1)):
            assert call(**{name: x}) == INVALID and "overlap" in error()


def test_types_and_places_of_rows():
    assert write(v=heads(dtype=C.NLD_F32)) == INVALID
    assert read(v=heads(2 * P, C.NLD_F32)) == INVALID and read(v=heads(P)) == INVALID
    assert attend(out=heads(1 << 44, C.NLD_F32)) == INVALID
    # 6 rows of stride 512, 4 heads: 2816 elements
    assert attend(out=heads(P)) == INVALID and attend(out=heads(P + 2 * 2815)) == INVALID
    assert "overlaps" in C.load().nld_last_error().decode()


def test_rows_of_one_array():
    """6 rows of 4 heads of 64: 256 elements of a row of 512, or every second piece of 64.  What passes is refused for its workspace."""
    for apart, row, head, ok in ((256, 512, 64, True), (255, 512, 64, False), (257, 512, 64, False), (-256, 512, 64, True), (-255, 512, 64, False),
                                 (512 * 2 + 256, 512, 64, True), (512 * 2 + 255, 512, 64, False), (512 * 5, 512, 64, False), (512 * 6, 512, 64, True),
                                 (512 * 5 + 256, 512, 64, True), (64, 512, 128, True), (63, 512, 128, False), (65, 512, 128, False), (448, 512, 128, True),
                                 (-64, 512, 128, True), (64 + 512 * 3, 512, 128, True), (64, 128, 128 * 6, True), (64 + 128 * 6, 128, 128 * 6, True),
                                 (128 * 6, 128, 128 * 6, False)):
        got = attend(q=heads(1 << 20, row=row, head=head), out=heads((1 << 20) + 2 * apart, row=row, head=head), ws_bytes=0)
        assert got == (CAPACITY if ok else INVALID), (apart, row, head)
    assert attend(q=heads(P), out=heads(P + 2 * 256, row=1024), ws_bytes=0) == INVALID      # other strides
    assert attend(q=heads(P), out=heads(P + 513), ws_bytes=0) == INVALID                    # between two elements
    one = chunk(3, 1)                                                                       # strides of a single row or head count for nothing
    assert attend(p=pages(batch=1), ch=chunk(1, 1), q=heads(row=7), out=heads(P + 2 * 256, row=9), ws_bytes=0) == CAPACITY
    assert attend(p=pages(n_kv_heads=1), ch=one, n_q=1, q=heads(row=128, head=3), out=heads(P + 128, row=128, head=5), ws_bytes=0) == CAPACITY
    # (1 << 20) x 16 pages are too many for one launch: the check behind that of the rows
    many = dict(p=pages(batch=1 << 20, n_kv_heads=16), ch=chunk(1 << 20, 1), k=heads(row=2048))
    assert read(v=heads(P + 2 * 1024, row=2048), **many) == SHAPE and read(v=heads(P + 2 * 1023, row=2048), **many) == INVALID
    assert read(v=heads(P + 2 * 2048 * 77, row=2048), **many) == INVALID and "overlaps" in C.load().nld_last_error().decode()


@pytest.mark.parametrize("call", [attend, select])
def test_attention_arguments(call):
    for kw, status in ((dict(n_q=0), SHAPE), (dict(n_q=3), SHAPE), (dict(n_q=-2), SHAPE), (dict(mode=2), INVALID), (dict(mode=-1), INVALID),
                       (dict(bidir=-1), INVALID), (dict(bidir=3), INVALID)):
        assert call(**kw) == status, kw
    lst = dict(lst=P, n_list=4) if call is attend else {}
    assert call(group=0, **lst) == INVALID and call(group=-1, **lst) == INVALID and call(group=65, **lst) == SHAPE
    assert call(group=2 ** 31 - 1, **lst) == SHAPE


def test_attention_scale_and_list():
    for bad in (NAN, INF, -INF):
        assert attend(scale=bad) == INVALID
    assert attend(lst=P, n_list=0, group=1) == INVALID and attend(lst=P, n_list=(1 << 24) + 1, group=1) == INVALID
    big = pages(batch=1 << 20, n_kv_heads=16)
    assert attend(p=big, ch=chunk(1 << 20, 1), n_q=16, out=heads(1 << 44, row=1024)) == SHAPE and "too many" in C.load().nld_last_error().decode()
    assert write(p=big, ch=chunk(1 << 20, 1)) == SHAPE
    need = C.load().nld_pages_workspace_bytes(ctypes.byref(pages()), 4, 2, 0)
    assert need > 256 and attend(ws_bytes=need // 2) == CAPACITY


def test_attention_scales_that_pass_f32_in_base_2():
    for bad in (3e38, -3e38, 2.0 ** 127 * 1.0001):
        assert attend(scale=bad) == INVALID and "scale" in C.load().nld_last_error().decode()


@pytest.mark.parametrize("group", [0, 1])
def test_rows_of_a_kv_head_fit_an_int(group):
    n = 1 << 24
    kw = dict(p=pages(batch=1, n_kv_heads=1), ch=chunk(n, n, P), n_q=128, q=heads(row=128 * 64), out=heads(1 << 44, row=128 * 64), group=group, n_list=4)
    assert attend(lst=P if group else None, **kw) == SHAPE and "too many" in C.load().nld_last_error().decode()
    assert C.load().nld_pages_workspace_bytes(ctypes.byref(kw["p"]), 128, n, group) == 0


def test_selection_arguments():
    assert select(p=pages()) == INVALID and "bounds" in C.load().nld_last_error().decode()
    for kw, status in ((dict(lst=None), INVALID), (dict(n_top=-1), INVALID), (dict(n_first=-1), INVALID), (dict(n_top=(1 << 24) + 1), SHAPE),
                       (dict(n_top=48, n_first=2), INVALID), (dict(ws_bytes=256 + 4 * 3 * 2 * 2 * 4 - 1), CAPACITY)):
        assert select(**kw) == status, kw


def test_list_len():
    f = C.load().nld_pages_list_len
    # a token alone has one page of its own; 2 adjacent ones may lie on two; 65 on two, 66 on three
    assert [f(1, 1, 0, 0, 0), f(500, 1, 3, 2, 0), f(2, 2, 0, 0, 0), f(65, 65, 0, 0, 0), f(66, 66, 0, 0, 0), f(66, 1, 0, 0, 1)] == [1, 6, 2, 2, 3, 3]
    for bad in ((0, 1, 1, 1, 0), (1, 0, 1, 1, 0), (1, 1, -1, 0, 0), (1, 1, 0, -1, 0), (1, 1, 1, 1, 2), (2 ** 31 - 1, 1, 1, 1, 0),
                (1, 2 ** 31 - 1, 1, 1, 0), (1, 1, 2 ** 31 - 1, 1, 0)):
        assert f(*bad) == 0


def test_list_len_of_groups_larger_than_the_chunk():
    """A group has no more tokens than the chunk, and a draft's list is never the shorter one."""
    f = C.load().nld_pages_list_len
    assert [f(1, 4, 0, 0, 0), f(1, 1 << 24, 2, 1, 0), f(2, 128, 0, 0, 0), f(65, 128, 0, 0, 0), f(66, 128, 0, 0, 0)] == [1, 4, 2, 2, 3]
    for rows in (1, 2, 3, 16, 63, 64, 65, 66, 200):
        for group in (1, 2, 4, 16, 64, 128):
            assert f(rows, group, 5, 1, 0) <= f(rows, group, 5, 1, 1)


def test_workspace_bytes():
    f = lambda p, *a: C.load().nld_pages_workspace_bytes(ref_of(p), *a)
    assert f(None, 4, 2, 0) == 0 and f(pages(head_dim=80), 4, 2, 0) == 0 and f(pages(), 3, 2, 0) == 0
    assert f(pages(), 4, 0, 0) == 0 and f(pages(), 4, 2, -1) == 0 and f(pages(), 4, 2, 65) == 0 and f(pages(), 4, (1 << 24) + 1, 0) == 0
    # fewer rows and larger groups need no more
    assert f(pages(), 4, 1, 1) <= f(pages(), 4, 40, 1) and f(pages(), 4, 40, 16) <= f(pages(), 4, 40, 1)
    assert f(pages(), 4, 100, 0) <= f(pages(), 4, 100, 1)


def test_workspace_bytes_says_what_it_refuses():
    f, error = lambda p, *a: C.load().nld_pages_workspace_bytes(ref_of(p), *a), lambda: C.load().nld_last_error().decode()
    big = pages(batch=1 << 20, n_kv_heads=16)
    for args, text in (((pages(), 4, 0, 0), "max_rows"), ((pages(), 4, 2, -1), "group"), ((pages(), 4, (1 << 24) + 1, 0), "max_rows"), ((big, 16, 1, 0), "too many"),
                       ((pages(), 4, 2, 65), "group"), ((pages(), 3, 2, 0), "n_q_heads"), ((pages(head_dim=80), 4, 2, 0), "head_dim")):
        assert write(p=pages(n_layers=0)) == INVALID and f(*args) == 0 and text in error(), (args[1:], error())


def test_scores_of_a_selection_in_one_launch(monkeypatch):
    """Where there are 256 units and more of up to 4096 pages the scores need no workspace, and the launch has a workgroup per unit."""
    monkeypatch.delenv("NLD_SELECT_ONE", raising=False)
    f = lambda p, *a: C.load().nld_pages_workspace_bytes(ref_of(p), *a)
    p = full(batch=64, n_kv_heads=8, max_pages=1024)
    units = 64 * 2048 * 8
    assert f(p, 32, 2048, 1) <= f(p, 32, 2048, 0) + 255 * 1024 * 4 + 8 * units + 512
    assert f(p, 32, 1, 1) >= 255 * 1024 * 4 and f(full(batch=64, n_kv_heads=8, max_pages=4097), 32, 2048, 1) >= units * 4097 * 4
    n = 1 << 14
    many = dict(ch=chunk(64 * n, n), n_q=8, q=heads(row=512), ws_bytes=0)
    assert select(p=p, **many) == CAPACITY
    assert select(p=full(batch=64, n_kv_heads=8, max_pages=4097), **many) == SHAPE
    monkeypatch.setenv("NLD_SELECT_ONE", "0")
    assert select(p=p, **many) == SHAPE and f(p, 32, 2048, 1) >= units * 1024 * 4


# ------------------------------------------------------------------------------------------ the binding
def cpu_cache(**kw):
    return R.PagedCache(2, 64, 2, 128, device="cpu", **kw)


def test_cache_sizes_and_types():
    c = cpu_cache(n_layers=3, dtype=torch.float8_e4m3fn, bounds=True)
    assert c.k.shape == (3, 4, 2, 4096) and c.k.dtype == torch.float8_e4m3fn and c.scale.shape == (3, 4, 2, 2, 64)
    assert c.bounds.shape == (3, 4, 2, 2, 64) and c.table.tolist() == [[0, 1], [2, 3]] and c.lengths.tolist() == [0, 0]
    assert cpu_cache(n_pages=7).table.tolist() == [[-1, -1], [-1, -1]] and cpu_cache().scale is None
    for kw in (dict(dtype=torch.float16), dict(n_pages=0), dict(n_layers=0), dict(n_pages=2 ** 31)):
        with pytest.raises(ValueError):
            cpu_cache(**kw)
    for max_len in (0, 100):
        with pytest.raises(ValueError):
            R.PagedCache(2, 64, 1, max_len, device="cpu")


def test_binding_refuses():
    c = cpu_cache()
    x = torch.zeros(4, 2, 64, dtype=torch.bfloat16)
    start = torch.tensor([0, 2, 4], dtype=torch.int32)
    bad_rows = [x.half(), x[0], torch.zeros(4, 3, 64), torch.zeros(4, 2, 32), torch.zeros(4, 64, 2).transpose(1, 2)]
    for y in bad_rows:
        with pytest.raises(ValueError):
            R.write_pages(c, 0, y, x, None, row_start=start)
        with pytest.raises(ValueError):
            R.write_pages(c, 0, x, y, None, row_start=start)
    for kw in (dict(row_start=start.long()), dict(row_start=start[:2]), dict(row_start=start, max_rows=0), dict(row_start=start, max_rows=5),
               dict(max_rows=1)):
        with pytest.raises(ValueError):
            R.write_pages(c, 0, x, x, None, **kw)
        with pytest.raises(ValueError):
            R.read_pages(c, 0, 4, None, **kw)
        with pytest.raises(ValueError):
            R.attend_pages(c, 0, x, None, **kw)
    with pytest.raises(ValueError):
        R.write_pages(c, 0, x[:3], x[:3], None)
    with pytest.raises(ValueError):
        R.read_pages(c, 0, 4, None, first=start)
    with pytest.raises(ValueError):
        R.attend_pages(c, 0, x, None, pages=torch.zeros(2, 2, 2, 3), group=1)
    with pytest.raises(ValueError):
        R.attend_pages(c, 0, x, None, pages=torch.zeros(2, 2, 2, 3, dtype=torch.int32), group=2)
    with pytest.raises(ValueError):
        R.attend_pages(c, 0, x, None, out=x.float()[:2])
    for kw in (dict(n_top=-1), dict(n_top=1, group=0), dict(n_top=1, n_first=-1)):
        with pytest.raises(ValueError):
            R.select_pages(c, 0, x, None, **kw)


@pytest.mark.parametrize("by", [2 ** 32, -2 ** 32, 2 ** 31])
def test_binding_refuses_numbers_past_int32(by):
    c, x = cpu_cache(), torch.zeros(2, 2, 64, dtype=torch.bfloat16)
    for call in (lambda: R.write_pages(c, by, x, x, None), lambda: R.read_pages(c, by, 2, None), lambda: R.attend_pages(c, by, x, None),
                 lambda: R.attend_pages(c, 0, x, None, mode=by), lambda: R.attend_pages(c, 0, x, None, bidir_from=by),
                 lambda: R.select_pages(c, by, x, None, 1), lambda: R.select_pages(c, 0, x, None, 1, mode=by),
                 lambda: R.select_pages(c, 0, x, None, 1, bidir_from=by), lambda: R.PagesWorkspace(c, 2 + by, 1), lambda: R.PagesWorkspace(c, 2, 1 + by),
                 lambda: R.PagesWorkspace(c, 2, 1, by)):
        with pytest.raises(ValueError, match="int32"):
            call()
    if by > 2 ** 31:
        with pytest.raises(ValueError):
            R.attend_pages(c, 0, torch.zeros(64, dtype=torch.bfloat16).as_strided((2, by + 2, 64), (0, 0, 1)), None)


# ------------------------------------------------------------------------------------------ the plain versions
def test_plain_8_bit_values_are_the_types():
    """Against torch's own type at scale 1, over all of its finite values, halfway between them, and beside."""
    codes = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double()
    codes = torch.sort(codes[torch.isfinite(codes)])[0]
    x = torch.cat([codes, (codes[1:] + codes[:-1]) / 2, codes * 1.01])
    x = x[x.abs() <= 448].float()
    rows = torch.stack([x, torch.full_like(x, 448.0)], -1)
    assert torch.equal(ref.stored(rows, True)[:, 0], x.to(torch.float8_e4m3fn).double())
    assert ref.stored(torch.tensor([[449.0, 1.0]]), True).tolist() == [[448.0, 1.0]] and ref.stored(torch.tensor([[480.0, 1.0]]), True).tolist() == [[480.0, 1.0]]


def test_plain_attention_closed_forms():
    """Equal keys: the mean of the values seen; one key seen: its value; two with scores log 3 and 0."""
    c = ref.Cache(1, 128, 1, 64, False, "cpu")
    v = torch.randn(70, 1, 64).bfloat16()
    c.write([0], [0, 70], torch.zeros(70, 1, 64), v)
    o, lse, _, _ = ref.attend(c, [67], [0, 3], torch.randn(3, 2, 64), 1.0)
    for i in range(3):
        assert torch.allclose(o[i, 0], v[:68 + i, 0].double().mean(0)) and abs(float(lse[i, 1]) - torch.log(torch.tensor(68.0 + i)).item()) < 1e-6
    o, _, _, _ = ref.attend(c, [0], [0, 2], torch.randn(2, 1, 64), 1.0, draft=True, bidir_from=1)
    assert torch.equal(o[0, 0], v[0, 0].double()) and torch.allclose(o[1, 0], v[:2, 0].double().mean(0))
    q = torch.zeros(1, 1, 64)
    c.k[0, 0, 0, 0] = 1.0
    q[0, 0, 0] = torch.log(torch.tensor(3.0))
    o, _, _, _ = ref.attend(c, [1], [0, 1], q, 1.0)
    assert torch.allclose(o[0, 0], 0.75 * c.v[0, 0, 0] + 0.25 * c.v[0, 1, 0], atol=1e-7)


def test_plain_bounds_hold():
    """Up to the rounding of the scale and of a quotient to f32, 2^-24 each relative to the largest magnitude."""
    for seed in range(20):
        k = torch.randn(64, 128, generator=torch.Generator().manual_seed(seed)).bfloat16()
        bd, scale = ref.bounds(k, 50)
        near = 2.0 ** -22 * float(k[:50].abs().max())
        lo, hi = bd[0].double() * scale, bd[1].double() * scale
        assert bool((lo <= k[:50].double().amin(0) + near).all()) and bool((hi >= k[:50].double().amax(0) - near).all())
        assert int(bd.abs().max()) <= 127


@pytest.mark.parametrize("call", ["block_forward", "draft", "verify_accept"])
def test_passes_refuse_a_cache_on_another_device(call):
    cache = R.PagedCache(2, 64, 1, 64, device="cpu")
    model = SimpleNamespace(device=torch.device("cpu"), shape=SimpleNamespace(vocab=8), handle=None)
    ws = SimpleNamespace(buf=torch.empty(256, dtype=torch.uint8, device="meta"), ptr=0, nbytes=256)
    one = torch.zeros(1, dtype=torch.int32)
    args = {"block_forward": (one.view(1, 1), R.VERIFY), "draft": (one, 2), "verify_accept": (one, one.view(1, 1), 2)}[call]
    with pytest.raises(ValueError, match="workspace is on meta, the cache on cpu"):
        getattr(R, call)(model, cache, ws, *args)
