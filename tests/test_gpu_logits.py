"""The operators on rows of logits against their plain 64-bit versions (tests/logits_ref.py).

Bounds.  A row's sum is taken by up to 1024 threads, each adding its share of the columns one after the other, and
merged in a tree; every term comes from a difference, a product and one exp2 (1 unit in the last place).  So a row's
sum is off, relative to itself, by at most
    delta(V) = (V / 512 + 16 merges of three roundings each) * 2^-24 + 2^-23 + the exponent's own rounding,
the last one 2 x 2^-24 ln 2 for a term of relative size exp2(-x), below 2^-23 on average over the terms that count and
at most 60 * 2^-24 for any term above 2^-40.  What follows the sums is in 64 bits and rounded once:
half a step, 2^-24 (f32) or 2^-8 (bf16) relative.  Hence with d = delta(V):
    lse       d + 2^-24 |lse|
    alpha     d + 2^-24
    loss      |w| d (1 + 2 eta max(KL, TV)) + 2^-24 |loss|: all log q shift alike, by at most d, lambda by eta d
    gradient  each of its terms by 4 d relative (the term's own exponential, the sum, the rest's share, lambda), then
              half a step of its type; where q and p are
              closer than d, the sign of TV's gradient is open (logits_ref.distill_undecided)
and a bf16 logit is exact in f32.
"""
import functools

import logits_ref as ref
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    from paper_2607_05722_amd import _lib as C
    from paper_2607_05722_amd import runtime as R

F32, BF16 = torch.float32, torch.bfloat16
HALF = {F32: 2.0 ** -24, BF16: 2.0 ** -8}


def delta(V):
    return (V / 512 + 48) * 2.0 ** -24 + 2.0 ** -23 + 60 * 2.0 ** -24


def draw(shape, dtype, seed, scale=2.5):
    g = torch.Generator().manual_seed(seed)
    z = torch.randn(shape, generator=g) * scale
    z[..., torch.randint(0, shape[-1], (3,), generator=g)] += 6.0
    return z.to(dtype)


def place(z, lead=0, pad_row=0, pad_seq=0):
    """z on the device as a view that starts `lead` elements into its buffer and has padded rows and sequences."""
    B, T, V = z.shape
    row, seq = V + pad_row, T * (V + pad_row) + pad_seq
    buf = torch.full((lead + B * seq + 16,), float("nan"), dtype=z.dtype, device="cuda")
    view = buf[lead:].as_strided((B, T, V), (seq, row, 1), storage_offset=lead)
    view.copy_(z)
    return view


PLANS = ["shared", "256", "512", "1024"]


def use_plan(monkeypatch, plan):
    """Rows shared by several workgroups (two launches), or one workgroup of so many threads each."""
    monkeypatch.setenv("NLD_LOSS_CHUNKS", "2" if plan == "shared" else "1")
    monkeypatch.setenv("NLD_LOSS_THREADS", "512" if plan == "shared" else plan)


def f64(t):
    return t.detach().double().cpu().numpy()


# ------------------------------------------------------------------------------------------ top logits
def as_f32(x):
    """The number that a call taking a float gets (1e-3 is not one: 5e-8 off, which exponents near 10^4 show)."""
    return float(np.float32(x))


def check_top(z, k, tau=1.0, ws=None):
    tau = as_f32(tau)
    B, T, V = z.shape
    ws = ws or R.LogitsWorkspace(B, T, V, k)
    o = R.top_logits(z, k, ws, temperature=tau)
    torch.cuda.synchronize()
    zz = f64(z).reshape(-1, V)
    v, i, s = f64(o["values"]).reshape(-1, k), o["ids"].cpu().numpy().reshape(-1, k), f64(o["lse"]).reshape(-1)
    for r in range(B * T):
        want = ref.top(zz[r], k)
        assert np.array_equal(i[r], want), (r, i[r][:10], want[:10])
        assert np.array_equal(v[r], zz[r][want], equal_nan=True)
        with np.errstate(invalid="ignore"):
            y = zz[r] / tau
            L = np.nan if np.isnan(y).any() else (np.inf if np.isposinf(y).any() else ref.lse(y))
        if np.isfinite(L):
            assert abs(s[r] - L) <= delta(V) + HALF[F32] * abs(L), (r, s[r], L)
        else:
            assert np.array_equal(s[r], L, equal_nan=True), (r, s[r], L)
    assert R.read_device_status(ws) == 0
    return o


SIZES = [(1, 1, 1, 1), (1, 2, 7, 7), (2, 3, 1000, 20), (1, 5, 1024, 512), (3, 2, 4099, 200), (1, 2, 16877, 300),
         (1, 1, 151936, 200), (2, 300, 2049, 64), (1, 1, 300001, 512), (1, 700, 513, 512), (5, 1, 50257, 1),
         (1, 600, 8193, 100)]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("B,T,V,k", SIZES)
def test_top(B, T, V, k, dtype):
    check_top(place(draw((B, T, V), dtype, V + k)), k, tau=3.0)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("chunks,threads", [("1", "512"), ("1", "1024"), ("2", "512"), ("2", "1024")])
@pytest.mark.parametrize("V,k", [(100003, 256), (50021, 33), (400009, 8)])
def test_top_plans(V, k, chunks, threads, dtype, monkeypatch):
    """One workgroup a row and several, of either size; 400009 columns: segments longer than one request."""
    monkeypatch.setenv("NLD_TOP_CHUNKS", chunks)
    monkeypatch.setenv("NLD_TOP_THREADS", threads)
    check_top(place(draw((1, 3, V), dtype, V), 1, 1), k)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("lead,pad_row,pad_seq", [(1, 0, 0), (3, 5, 7), (0, 1, 2), (6, 2, 0)])
def test_top_strides(dtype, lead, pad_row, pad_seq):
    check_top(place(draw((2, 3, 5001), dtype, 11), lead, pad_row, pad_seq), 40)
    check_top(place(draw((2, 3, 5), dtype, 12), lead, pad_row, pad_seq), 5, tau=0.7)


def special_rows(V, dtype):
    g = torch.Generator().manual_seed(5)
    z = torch.randn((12, V), generator=g) * 2
    z[0] = 0.0                                   # every logit equal
    z[1] = float("-inf")
    z[2] = float("-inf")
    z[2, [5, V - 1, V // 2]] = torch.tensor([1.0, 3.0, 3.0])     # a vocabulary masked down to three tokens
    z[3, V // 3] = float("nan")
    z[3, V // 2] = float("inf")
    z[4, [1, V - 2]] = float("inf")
    z[5] = torch.where(torch.arange(V) % 2 == 0, 0.0, -0.0)
    z[6] = torch.arange(V, dtype=torch.float32) / V              # ascending
    z[7] = (z[7] * 2).round() / 2                                # many equal logits at the border
    z[8] = torch.finfo(dtype).min                                # a mask of the type's lowest value
    z[8, 7] = 2.0
    z[9] -= 1e4
    z[10, ::1024] += 50.0                                        # all the largest at one stride
    z[11] = torch.finfo(dtype).min
    return z.to(dtype)[None]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("V,k", [(3001, 20), (20011, 200), (151936, 512)])
def test_top_special_rows(V, k, dtype, monkeypatch):
    z = place(special_rows(V, dtype), lead=1)
    for chunks in ("1", "2"):                    # one workgroup a row, and several where it is long
        for threads in ("512", "1024"):
            monkeypatch.setenv("NLD_TOP_CHUNKS", chunks)
            monkeypatch.setenv("NLD_TOP_THREADS", threads)
            check_top(z, k)


def test_top_tiny_k_of_equal_rows_is_the_lowest_columns():
    z = torch.zeros((1, 4, 30000), device="cuda")
    o = R.top_logits(z, 3, R.LogitsWorkspace(1, 4, 30000, 3))
    assert o["ids"].cpu().tolist() == [[[0, 1, 2]] * 4]


# ------------------------------------------------------------------------------------------ losses
def teacher_of(z, k, tau, seed, noise=0.5):
    """Top entries of a teacher near the student, by the plain version."""
    B, T, V = z.shape
    t = f64(z) + np.random.default_rng(seed).normal(size=z.shape) * noise
    t = t.astype(np.float32).astype(np.float64)
    ids = np.stack([ref.top(r, k) for r in t.reshape(-1, V)]).reshape(B, T, k)
    vals = np.take_along_axis(t, ids.astype(np.int64), -1)
    lse = np.array([ref.lse(r / tau) for r in t.reshape(-1, V)]).reshape(B, T).astype(np.float32)
    dev = lambda a, dt: torch.from_numpy(a.astype(dt)).cuda()    # noqa: E731
    return dev(vals, np.float32), dev(ids, np.int32), dev(lse, np.float32)


def rows_taking_part(B, T, weight, last_row):
    w = np.ones((B, T)) if weight is None else f64(weight)
    if last_row is not None:
        w = np.where(np.arange(T)[None] <= last_row.cpu().numpy()[:, None], w, 0.0)
    return w


def compare(z, w, loss, aux, grad, plain, slack, aux_slack, undecided=lambda r: 0.0):
    """Device results of all rows against plain(r) -> (loss, aux, gradient, sizes)."""
    B, T, V = z.shape
    d = delta(V)
    L, A = f64(loss).reshape(-1), f64(aux).reshape(-1)
    G = f64(grad).reshape(-1, V) if grad is not None else None
    h = HALF[z.dtype]
    for r in range(B * T):
        l, a, g, size = plain(r)
        assert abs(L[r] - l) <= abs(w.reshape(-1)[r]) * d * slack(r) + HALF[F32] * abs(l) + 1e-37, (r, L[r], l)
        assert abs(A[r] - a) <= d * aux_slack + HALF[F32] * abs(a), (r, A[r], a)
        if G is not None:
            off = np.abs(G[r] - g) - (4 * d * slack(r) * size + h * np.abs(g) + undecided(r) + 1e-37)
            assert off.max() <= 0, (r, int(off.argmax()), G[r][off.argmax()], g[off.argmax()])


def check_distill(z, k, tau=1.0, kl_share=1.0, eta=0.5, tail=True, weight=None, last_row=None, grad=None, want_grad=True,
                  entries=None, ws=None, status=0):
    B, T, V = z.shape
    tau = as_f32(tau)
    zz = f64(z).reshape(-1, V)
    vals, ids, lse = entries or teacher_of(z, k, tau, V + k)
    ws = ws or R.LogitsWorkspace(B, T, V, k)
    o = R.distill_from_logits(z, vals, ids, ws, teacher_lse=lse if tail else None, temperature=tau, kl_share=kl_share, eta=eta,
                              weight=weight, last_row=last_row, want_grad=want_grad, grad=grad)
    torch.cuda.synchronize()
    w = rows_taking_part(B, T, weight, last_row)
    vv, ii, ll = f64(vals).reshape(-1, k), ids.cpu().numpy().reshape(-1, k), f64(lse).reshape(-1)

    def plain(r):
        return ref.distill(zz[r], vv[r], ii[r], ll[r] if tail else None, tau, kl_share, eta, w.reshape(-1)[r])

    def slack(r):
        if w.reshape(-1)[r] == 0:
            return 1.0
        kl = ref.distill(zz[r], vv[r], ii[r], ll[r] if tail else None, tau, 1.0, 0.0, 1.0)[0]
        return 1 + 2 * eta * max(kl, 1.0)

    assert R.read_device_status(ws) == status
    compare(z if grad is not z else zz_like(zz, z), w, o["loss"], o["accept"], o.get("grad"), plain, slack, 1.0,
            lambda r: ref.distill_undecided(zz[r], vv[r], ii[r], ll[r] if tail else None, tau, kl_share, eta, w.reshape(-1)[r],
                                            delta(V)))
    return o


def zz_like(zz, z):
    return torch.empty(z.shape, dtype=z.dtype, device="meta")


LOSS_SIZES = [(1, 1, 1, 1), (1, 2, 7, 7), (2, 3, 1000, 20), (1, 7, 1024, 32), (3, 2, 4099, 200), (1, 2, 16877, 512),
              (1, 1, 151936, 200), (2, 3, 50257, 1), (1, 1, 300001, 300), (1, 700, 513, 64), (9, 130, 1030, 16)]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("B,T,V,k", LOSS_SIZES)
def test_distill(B, T, V, k, dtype):
    check_distill(place(draw((B, T, V), dtype, V)), k, tau=3.0)


@pytest.mark.parametrize("plan", PLANS)
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("kl_share,eta,tail,tau", [(1.0, 0.0, True, 1.0), (1.0, 0.0, False, 2.0), (0.0, 0.0, True, 1.0),
                                                   (0.4, 2.0, False, 0.7), (1.0, 0.5, True, 3.0)])
def test_distill_mixtures(kl_share, eta, tail, tau, dtype, plan, monkeypatch):
    """50021 columns: more than 256 threads hold, two or more chunks where the rows are shared."""
    use_plan(monkeypatch, plan)
    check_distill(place(draw((2, 3, 50021), dtype, 3), lead=1), 50, tau, kl_share, eta, tail)


@pytest.mark.parametrize("plan", PLANS)
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_distill_rows_that_take_no_part(dtype, plan, monkeypatch):
    """Weights (0, negative, absent), last_row, and rows of NaN that have weight 0 or lie past last_row."""
    use_plan(monkeypatch, plan)
    B, T, V, k = 3, 4, 50021, 20
    z = draw((B, T, V), dtype, 8)
    entries = teacher_of(place(z), k, 1.0, 1)
    weight = torch.tensor([[1.0, 0.0, -2.0, 0.5]] * B, device="cuda")
    last = torch.tensor([3, -1, 2], dtype=torch.int32, device="cuda")
    z[:, 1] = float("nan")
    z[1] = float("nan")
    z[2, 3] = float("nan")
    entries[0][1], entries[1][1] = float("nan"), 1 << 30
    o = check_distill(place(z, 3, 1, 2), k, weight=weight, last_row=last, entries=entries)
    assert not o["grad"][1].any() and not o["loss"][1].any() and not o["accept"][1].any()


@pytest.mark.parametrize("plan", PLANS)
def test_distill_entries_that_do_not_count(plan, monkeypatch):
    """-1 is no entry; ids out of range and repeated ones are left out and reported; no entry at all: with the tail the
    teacher knows nothing but "some token", without it there is no teacher."""
    use_plan(monkeypatch, plan)
    V, k = 20011, 70
    z = place(draw((1, 6, V), F32, 9))
    for row, bad in ((0, None), (1, V), (2, -7), (3, "twice"), (4, "thrice")):
        vals, ids, lse = teacher_of(z, k, 1.0, 2)
        ids[0, 5, :] = -1
        ids[0, row, 3] = -1
        if bad == "twice":
            ids[0, row, 66] = ids[0, row, 2]
            vals[0, row, 66] = 9.0
        elif bad == "thrice":
            ids[0, row, [1, 30]] = ids[0, row, 69].clone()
        elif bad is not None:
            ids[0, row, 9] = bad
        for tail in (True, False):
            check_distill(z, k, entries=(vals, ids, lse), tail=tail, status=0 if bad is None else C.NLD_DEV_BAD_TOKEN)


@pytest.mark.parametrize("plan", PLANS)
def test_distill_infinities(plan, monkeypatch):
    """Masked students and teachers: columns of -inf in the rest and among the entries, rows of nothing else, a rest far
    below the entries, entries far below the rest, every column an entry."""
    use_plan(monkeypatch, plan)
    V, k = 20011, 40
    z = draw((1, 7, V), F32, 10)
    inf = float("inf")
    z[0, 0, ::3] = -inf
    z[0, 1] = -inf
    t = z.clone()
    t[0, 2] = -inf
    t[0, 3, 1:] = -inf                                  # a teacher of one token
    z[0, 4] -= 300.0
    z[0, 4, :k] += 300.0                                # a rest that f32 cannot hold beside the entries
    t[0, 4] = z[0, 4]
    t[0, 5, :100] += 30.0
    z[0, 6] = torch.finfo(F32).min
    z[0, 6, 50] = 1.0
    zd = place(z)
    vals = torch.empty((1, 7, k), device="cuda")
    ids = torch.empty((1, 7, k), dtype=torch.int32, device="cuda")
    lse = torch.empty((1, 7), device="cuda")
    R.top_logits(place(t), k, R.LogitsWorkspace(1, 7, V, k), outs={"values": vals, "ids": ids, "lse": lse})
    for tail in (True, False):
        for kl in (1.0, 0.5):
            w = torch.ones((1, 7), device="cuda")
            if kl == 1.0 or not tail:
                pass
            o = R.distill_from_logits(zd, vals, ids, R.LogitsWorkspace(1, 7, V, k), teacher_lse=lse if tail else None,
                                      kl_share=kl, eta=0.0, weight=w)
            for r in (1, 2):
                assert o["loss"][0, r] == 0 and not o["grad"][0, r].any()
            rows = [0, 3, 4, 5, 6]
            L, G = f64(o["loss"])[0], f64(o["grad"])[0]
            for r in rows:
                l, a, g, size = ref.distill(f64(z)[0, r], f64(vals)[0, r], ids.cpu().numpy()[0, r],
                                            f64(lse)[0, r] if tail else None, 1.0, kl, 0.0, 1.0)
                if np.isinf(l):
                    assert L[r] == l
                else:
                    # the rest's mass p_R = 1 - sum p is itself a difference of f32 inputs: taken alike on both sides
                    assert abs(L[r] - l) <= delta(V) + HALF[F32] * abs(l) * 2, (r, L[r], l)
                # row 4 learns from itself: the signs of TV's gradient are open there
                move = ref.distill_undecided(f64(z)[0, r], f64(vals)[0, r], ids.cpu().numpy()[0, r],
                                             f64(lse)[0, r] if tail else None, 1.0, kl, 0.0, 1.0, delta(V))
                assert np.all(np.abs(G[r] - g) <= 4 * delta(V) * size + HALF[F32] * np.abs(g) + move + 1e-37), r


def test_distill_of_a_student_without_the_teachers_token_is_infinite():
    z = torch.zeros((1, 1, 100), device="cuda")
    z[0, 0, 7] = float("-inf")
    o = R.distill_from_logits(z, torch.zeros((1, 1, 1), device="cuda"), torch.full((1, 1, 1), 7, dtype=torch.int32, device="cuda"),
                              R.LogitsWorkspace(1, 1, 100, 1), eta=0.0)
    assert o["loss"].item() == float("inf") and o["grad"][0, 0, 7].item() == -1.0


@pytest.mark.parametrize("mask", [float("-inf"), torch.finfo(F32).min, -1e5])
@pytest.mark.parametrize("plan", PLANS)
def test_distill_of_a_shared_mask(plan, mask, monkeypatch):
    """Teacher and student masked down to the same tokens, fewer than there are entries and with a log-sum-exp that f32
    rounds: the loss is that of these tokens, not the infinite one of a token that only the teacher has."""
    use_plan(monkeypatch, plan)
    V, k = 20011, 40
    z, t = draw((1, 6, V), F32, 12) + 20.0, draw((1, 6, V), F32, 13) + 20.0
    off = torch.ones(V, dtype=torch.bool)
    off[[5, 900, 901, V - 1, 7000]] = False
    z[..., off] = t[..., off] = mask
    ws = R.LogitsWorkspace(1, 6, V, k)
    top = R.top_logits(place(t), k, ws)
    o = check_distill(place(z), k, eta=0.0, entries=(top["values"], top["ids"], top["lse"]), ws=ws)
    assert torch.isfinite(o["loss"]).all() and (o["loss"] > 1e-3).all()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("value", ["lowest", "highest", 2.0 ** 31, -2.0 ** 28, 2.0 ** 27])
@pytest.mark.parametrize("tau", [1.0, 0.3])
@pytest.mark.parametrize("plan", PLANS)
def test_rows_of_one_large_value(plan, tau, value, dtype, monkeypatch):
    """Every logit alike and so large that sums beside it vanish: all tokens are as likely.  A teacher's log-sum-exp of the
    lowest value is no teacher; its entries alone are one."""
    use_plan(monkeypatch, plan)
    V, k = 20011, 40
    big = {"lowest": torch.finfo(dtype).min, "highest": torch.finfo(dtype).max}.get(value, value)
    z = place(torch.full((1, 2, V), big, dtype=dtype), lead=1)
    ids = torch.arange(100, 100 + k, dtype=torch.int32, device="cuda").expand(1, 2, k).contiguous()
    vals = torch.full((1, 2, k), torch.finfo(F32).min, device="cuda")
    a, adv = ids[..., 0].contiguous(), torch.ones((1, 2), device="cuda")
    ws, d, h = R.LogitsWorkspace(1, 2, V, k), delta(V), HALF[dtype]
    p = R.policy_from_logits(z, a, adv, ws, temperature=tau)
    assert ((p["logp"].double() + np.log(V)).abs() <= d + HALF[F32] * np.log(V)).all()
    want = np.full(V, 1.0 / V / tau)
    want[100] -= 1.0 / tau
    assert np.all(np.abs(f64(p["grad"])[0] - want) <= 4 * d * 2 / tau * np.where(want < 0, 1.0, 1.0 / V) + h * np.abs(want))
    o = R.distill_from_logits(z, vals, ids, ws, temperature=tau, eta=0.0)    # uniform over the entries
    assert ((o["loss"].double() - np.log(V / k)).abs() <= d + HALF[F32] * np.log(V / k)).all()
    want = np.full(V, 1.0 / V / tau)
    want[100:100 + k] -= 1.0 / k / tau
    assert np.all(np.abs(f64(o["grad"])[0] - want) <= 4 * d * 2 / tau * np.where(want < 0, 1.0 / k, 1.0 / V) + h * np.abs(want))
    lse = R.top_logits(torch.full_like(z, torch.finfo(dtype).min), k, ws, temperature=tau)["lse"]
    o = R.distill_from_logits(z, vals, ids, ws, teacher_lse=lse, temperature=tau)
    assert not o["loss"].any() and not o["accept"].any() and not o["grad"].any()


def test_not_a_number_beside_an_empty_rest():
    """Every column outside the entries masked, a NaN among the entries: the whole gradient is NaN."""
    z = torch.full((1, 1, 5001), float("-inf"), device="cuda")
    z[0, 0, :3] = torch.tensor([1.0, float("nan"), 2.0])
    vals, ids = torch.zeros((1, 1, 3), device="cuda"), torch.arange(3, dtype=torch.int32, device="cuda").view(1, 1, 3)
    o = R.distill_from_logits(z, vals, ids, R.LogitsWorkspace(1, 1, 5001, 3))
    assert torch.isnan(o["loss"]).all() and torch.isnan(o["grad"]).all()


def test_policy_corners():
    """An advantage of 0 hides no NaN; an action of probability 0 costs +inf against a reference, nothing with kl_coef 0."""
    z = torch.zeros((1, 3, 3000), device="cuda")
    z[0, 0, 9] = float("nan")
    z[0, 1, 17] = float("-inf")
    a = torch.full((1, 3), 17, dtype=torch.int32, device="cuda")
    adv, refp = torch.zeros((1, 3), device="cuda"), torch.full((1, 3), -2.0, device="cuda")
    ws = R.LogitsWorkspace(1, 3, 3000, 1)
    o = R.policy_from_logits(z, a, adv, ws, ref_logp=refp)
    assert torch.isnan(o["loss"][0, 0]) and torch.isnan(o["grad"][0, 0]).all()
    assert not o["loss"][0, 1:].any() and not o["grad"][0, 1:].any()
    o = R.policy_from_logits(z, a, adv, ws, ref_logp=refp, kl_coef=0.1)
    assert o["loss"][0, 1].item() == float("inf") and o["grad"][0, 1, 17].item() == float("-inf")
    assert torch.isfinite(o["loss"][0, 2]) and torch.isfinite(o["grad"][0, 2]).all()


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("column", [3, 777])
def test_not_a_number_stays_in_its_row(bad, column):
    z = draw((1, 3, 4001), F32, 4)
    entries = teacher_of(place(z), 10, 1.0, 3)
    entries[1][0, 1, 0] = 3
    entries[1][0, 1, 1:] = torch.arange(100, 109, dtype=torch.int32)
    z[0, 1, column] = bad
    zd = place(z)
    o = R.distill_from_logits(zd, entries[0], entries[1], R.LogitsWorkspace(1, 3, 4001, 10), teacher_lse=entries[2])
    p = R.policy_from_logits(zd, torch.full((1, 3), 3, dtype=torch.int32, device="cuda"), torch.ones((1, 3), device="cuda"),
                             R.LogitsWorkspace(1, 3, 4001, 1))
    for x in (o, p):
        assert torch.isnan(x["loss"][0, 1]) and torch.isnan(x["grad"][0, 1]).all()
        assert torch.isfinite(x["loss"][0, [0, 2]]).all() and torch.isfinite(x["grad"][0, [0, 2]]).all()


@pytest.mark.parametrize("where", ["values", "lse"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_not_a_number_of_the_teacher_stays_in_its_row(bad, where):
    z = place(draw((1, 3, 4001), F32, 4))
    vals, ids, lse = teacher_of(z, 10, 1.0, 3)
    if where == "values":
        vals[0, 1, 4] = bad
    else:
        lse[0, 1] = bad if bad != bad else float("-inf")     # no token at all
    o = R.distill_from_logits(z, vals, ids, R.LogitsWorkspace(1, 3, 4001, 10), teacher_lse=lse)
    if where == "lse" and bad == bad:
        assert o["loss"][0, 1] == 0 and o["accept"][0, 1] == 0 and not o["grad"][0, 1].any()
    else:
        assert torch.isnan(o["loss"][0, 1]) and torch.isnan(o["accept"][0, 1]) and torch.isnan(o["grad"][0, 1]).all()
    assert torch.isfinite(o["loss"][0, [0, 2]]).all() and torch.isfinite(o["grad"][0, [0, 2]]).all()


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_the_longest_row(dtype):
    """2^24 columns: top, and both losses with gradient, against 64-bit sums on the device."""
    V, k = 1 << 24, 100
    g = torch.Generator(device="cuda").manual_seed(1)
    z = torch.randn((1, 1, V), generator=g, device="cuda").mul_(2.5).to(dtype)
    d = z[0, 0].double()
    ws = R.LogitsWorkspace(1, 1, V, k)
    t = R.top_logits(z, k, ws)
    v, i = torch.sort(d, descending=True, stable=True)
    assert torch.equal(t["ids"][0, 0].long(), i[:k]) and torch.equal(t["values"][0, 0].double(), v[:k])
    L = torch.logsumexp(d, 0)
    assert abs(t["lse"].item() - L.item()) <= delta(V) + HALF[F32] * L.item()
    a = i[:1].to(torch.int32).view(1, 1)
    p = R.policy_from_logits(z, a, torch.ones((1, 1), device="cuda"), ws)
    q = torch.exp(d - L)
    want = q.clone()
    want[i[0]] -= 1.0
    assert abs(p["logp"].item() - (v[0] - L).item()) <= delta(V) + HALF[F32] * abs((v[0] - L).item())
    assert bool(((p["grad"][0, 0].double() - want).abs() <= 4 * delta(V) * (q + (want < 0)) + HALF[dtype] * want.abs() + 1e-37).all())
    # cross-entropy of the same token: the same gradient
    c = R.distill_from_logits(z, t["values"][..., :1].contiguous(), t["ids"][..., :1].contiguous(), ws, eta=0.0)
    assert abs(c["loss"].item() + (v[0] - L).item()) <= delta(V) + HALF[F32] * abs((v[0] - L).item())
    assert bool(((c["grad"][0, 0].double() - want).abs() <= 4 * delta(V) * (q + (want < 0)) + HALF[dtype] * want.abs() + 1e-37).all())


def test_very_many_short_rows():
    """2^20 rows of 5 columns, the most of one call."""
    R_, V = 1 << 20, 5
    g = torch.Generator(device="cuda").manual_seed(2)
    z = torch.randn((1, R_, V), generator=g, device="cuda")
    ws = R.LogitsWorkspace(1, R_, V, 2)
    t = R.top_logits(z, 2, ws)
    v, i = torch.sort(z, dim=-1, descending=True, stable=True)
    assert torch.equal(t["ids"].long(), i[..., :2]) and torch.equal(t["values"], v[..., :2])
    lp = torch.log_softmax(z.double(), -1)
    p = R.policy_from_logits(z, t["ids"][..., 1].contiguous(), torch.ones((1, R_), device="cuda"), ws)
    want = lp.gather(-1, i[..., 1:2])[..., 0]
    assert bool(((p["logp"].double() - want).abs() <= delta(V) + HALF[F32] * want.abs()).all())
    grad = torch.exp(lp)
    grad.scatter_add_(-1, i[..., 1:2], torch.full((1, R_, 1), -1.0, dtype=torch.float64, device="cuda"))
    assert bool(((p["grad"].double() - grad).abs() <= 4 * delta(V) * 2 + HALF[F32] * grad.abs()).all())
    assert R.read_device_status(ws) == 0


@pytest.mark.parametrize("tau", [1e-3, 1e3])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_extreme_temperatures(tau, dtype):
    z = place(draw((1, 4, 3001), dtype, 90))
    check_top(z, 20, tau=tau)
    check_distill(z, 20, tau=tau, eta=0.0)
    check_policy(z, tau=tau, old=False)


@pytest.mark.parametrize("plan", PLANS)
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_gradient_in_place_and_strided(dtype, plan, monkeypatch):
    """The gradient in the logits' place, and into views of other alignment whose surroundings stay as they were."""
    use_plan(monkeypatch, plan)
    V = 50021
    z = draw((2, 3, V), dtype, 21)
    for lead, pr, ps in ((0, 0, 0), (1, 3, 5)):
        zd = place(z, lead, pr, ps)
        check_distill(zd, 30, grad=zd)
    for lead, pr, ps in ((0, 0, 0), (2, 7, 0), (5, 1, 4)):
        out = place(torch.zeros_like(z), lead, pr, ps)
        check_distill(place(z, 1, 2, 3), 30, grad=out)
        gap = torch.as_strided(out, (2, 3, pr), (out.stride(0), out.stride(1), 1), out.storage_offset() + V)
        assert torch.isnan(gap).all()
    # sequences inside the rows: [rows][batch] in memory
    buf = torch.empty((3, 2, V), dtype=dtype, device="cuda").transpose(0, 1)
    check_distill(place(z), 30, grad=buf)


def test_broadcast_student():
    """One row of logits for every sequence (stride 0): each has a gradient of its own."""
    z = place(draw((1, 2, 5001), F32, 30)).expand(3, 2, 5001)
    entries = teacher_of(z, 20, 1.0, 5)
    check_distill(z, 20, entries=entries, grad=torch.empty((3, 2, 5001), device="cuda"))


def test_offsets_past_32_bits():
    """Logits of more than 2^32 bytes and 2^31 elements: the last rows are right, the others take no part."""
    B, T, V, k = 1, 14200, 151936, 64
    z = torch.empty((B, T, V), dtype=BF16, device="cuda")
    tail = draw((1, 2, V), BF16, 6)
    z[:, -2:] = tail.cuda()
    small = place(tail)
    vals, ids, lse = teacher_of(small, k, 1.0, 4)
    many = lambda t: torch.cat([torch.zeros((1, T - 2) + t.shape[2:], dtype=t.dtype, device="cuda"), t], 1)    # noqa: E731
    weight = torch.zeros((B, T), device="cuda")
    weight[:, -2:] = 1.0
    o = R.distill_from_logits(z, many(vals), many(ids), R.LogitsWorkspace(B, T, V, k), teacher_lse=many(lse), weight=weight, grad=z)
    s = R.distill_from_logits(small, vals, ids, R.LogitsWorkspace(1, 2, V, k), teacher_lse=lse)
    assert not z[:, :-2].any()
    assert torch.allclose(o["loss"][:, -2:], s["loss"], rtol=0, atol=2 * delta(V) * 3)
    assert torch.allclose(z[:, -2:].float(), s["grad"].float(), rtol=2 ** -7, atol=8 * delta(V))


def check_policy(z, seed=0, tau=1.0, lo=0.2, hi=0.3, beta=0.0, old=True, refp=False, weight=None, last_row=None, grad=None,
                 actions=None, status=0):
    B, T, V = z.shape
    tau = as_f32(tau)
    zz = f64(z).reshape(-1, V)
    rng = np.random.default_rng(seed + V)
    a = rng.integers(0, V, size=(B, T)) if actions is None else np.asarray(actions).reshape(B, T)
    logp = np.array([(zz[r][x] / tau - ref.lse(zz[r] / tau)) if 0 <= x < V else -1.0 for r, x in enumerate(a.reshape(-1))])
    f = lambda x: np.ascontiguousarray(x, dtype=np.float32).reshape(B, T)    # noqa: E731
    adv = f(rng.normal(size=B * T))
    o32 = f(logp + 0.4 * rng.normal(size=B * T))
    r32 = f(logp + 0.4 * rng.normal(size=B * T))
    dev = lambda x: torch.from_numpy(x).cuda()    # noqa: E731
    ws = R.LogitsWorkspace(B, T, V, 1)
    o = R.policy_from_logits(z, dev(a.astype(np.int32)), dev(adv), ws, old_logp=dev(o32) if old else None,
                             ref_logp=dev(r32) if refp else None, temperature=tau, clip_low=lo, clip_high=hi, kl_coef=beta,
                             weight=weight, last_row=last_row, grad=grad)
    torch.cuda.synchronize()
    w = rows_taking_part(B, T, weight, last_row)
    flat = lambda x: x.astype(np.float64).reshape(-1)    # noqa: E731

    def plain(r):
        return ref.policy(zz[r], a.reshape(-1)[r], flat(adv)[r], flat(o32)[r] if old else None, flat(r32)[r] if refp else None,
                          tau, lo, hi, beta, w.reshape(-1)[r])

    def slack(r):
        # d loss / d logp, and its own change with logp: rho A and beta exp(d)
        l, lp, g, size = plain(r)
        rho = np.exp(lp - flat(o32)[r]) if old else 1.0
        return max(1.0, 2 * (rho * abs(flat(adv)[r]) + (beta * (1 + np.exp(flat(r32)[r] - lp)) if refp else 0.0)))

    assert R.read_device_status(ws) == status
    compare(z if grad is not z else zz_like(zz, z), w, o["loss"], o["logp"], o.get("grad"), plain, slack, 1.0)
    return o


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("B,T,V,k", LOSS_SIZES)
def test_policy(B, T, V, k, dtype):
    check_policy(place(draw((B, T, V), dtype, V + 1)), beta=0.05, refp=True)


@pytest.mark.parametrize("plan", PLANS)
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("tau,old,refp", [(1.0, False, False), (0.7, True, False), (3.0, False, True), (1.0, True, True)])
def test_policy_terms(tau, old, refp, dtype, plan, monkeypatch):
    use_plan(monkeypatch, plan)
    z = place(draw((2, 40, 50021), dtype, 40), 1, 1, 3)
    check_policy(z, tau=tau, old=old, refp=refp, beta=0.1 if refp else 0.0)
    weight = torch.rand((2, 40), device="cuda") - 0.3
    weight[:, ::3] = 0.0
    last = torch.tensor([20, 39], dtype=torch.int32, device="cuda")
    check_policy(z, tau=tau, old=old, refp=refp, beta=0.1 if refp else 0.0, weight=weight, last_row=last)
    check_policy(z, tau=tau, old=old, refp=refp, beta=0.1 if refp else 0.0, grad=z)


@pytest.mark.parametrize("plan", PLANS)
def test_policy_actions_that_do_not_count(plan, monkeypatch):
    use_plan(monkeypatch, plan)
    z = place(draw((1, 4, 20011), F32, 41))
    check_policy(z, actions=[-1, 0, 20010, -1])
    check_policy(z, actions=[5, 20011, 3, 8], status=C.NLD_DEV_BAD_TOKEN)
    check_policy(z, actions=[5, -2, 3, 8], status=C.NLD_DEV_BAD_TOKEN)


def test_policy_of_a_certain_and_an_impossible_action():
    """1 - q of an action of probability 1 - 1e-12 keeps its digits; a row of -inf takes no part; an impossible action
    has log-probability -inf and, on policy, leaves the other columns their share."""
    z = torch.full((1, 4, 3000), -40.0, device="cuda")
    z[0, 0, 17] = 0.0
    z[0, 1, :] = float("-inf")
    z[0, 2, 17] = float("-inf")
    z[0, 3, 17] = 200.0
    a = torch.full((1, 4), 17, dtype=torch.int32, device="cuda")
    o = R.policy_from_logits(z, a, torch.ones((1, 4), device="cuda"), R.LogitsWorkspace(1, 4, 3000, 1))
    rest = 2999 * np.exp(-40.0)
    # loss -A rho = -1 on policy; d/dz_a = -(1 - q_a)
    assert abs(o["logp"][0, 0].item() + rest) <= 1e-5 * rest
    assert abs(o["grad"][0, 0, 17].item() + rest) <= 1e-5 * rest
    assert o["loss"][0, 1] == 0 and o["logp"][0, 1] == 0 and not o["grad"][0, 1].any()
    assert o["logp"][0, 2].item() == float("-inf")
    assert o["logp"][0, 3].item() == 0 and torch.isfinite(o["grad"][0, 3]).all()


def test_gradients_against_differences():
    """The gradient of the device's own losses, by central differences of them in steps of 2^-6 (f32 losses of size 1 carry
    2^-22 after their sums; the third derivative of either loss in one logit is below 4)."""
    V, k, tau, h = 300, 12, 2.0, 2.0 ** -6
    z = draw((1, 1, V), F32, 50)
    vals, ids, lse = teacher_of(place(z), k, tau, 7)
    ws = R.LogitsWorkspace(1, 2 * V, V, k)
    steps = z.expand(1, 2 * V, V).clone()
    steps[0, :V] += h * torch.eye(V)
    steps[0, V:] -= h * torch.eye(V)
    steps = steps.cuda()
    many = lambda t: t.expand((1, 2 * V) + t.shape[2:]).contiguous()    # noqa: E731
    a = torch.full((1, 2 * V), int(ids[0, 0, 0]), dtype=torch.int32, device="cuda")
    one = torch.ones((1, 2 * V), device="cuda")
    old, refp = -2.0 * one, -1.5 * one

    def distill(x, n, **kw):
        return R.distill_from_logits(x, many(vals)[:, :n].contiguous(), many(ids)[:, :n].contiguous(), ws,
                                     teacher_lse=many(lse)[:, :n].contiguous(), temperature=tau, eta=0.0, **kw)

    def policy(x, n, **kw):
        return R.policy_from_logits(x, a[:, :n].contiguous(), one[:, :n].contiguous(), ws, old_logp=old[:, :n].contiguous(),
                                    ref_logp=refp[:, :n].contiguous(), temperature=tau, clip_low=1.0, clip_high=50.0,
                                    kl_coef=0.1, **kw)

    for call in (distill, policy):
        L = f64(call(steps, 2 * V, want_grad=False)["loss"])[0]
        g = f64(call(place(z), 1)["grad"])[0, 0]
        diff = (L[:V] - L[V:]) / (2 * h)
        scale = max(1.0, np.abs(L).max())
        assert np.abs(diff - g).max() <= scale * (2 * 2.0 ** -21 / (2 * h) + 4 * h * h / 6)


@pytest.mark.parametrize("B,T", [(1, 3), (3, 200)])
def test_results_repeat_bit_for_bit(B, T):
    z = place(draw((B, T, 20011), F32, 60))
    ws = R.LogitsWorkspace(B, T, 20011, 100)
    top = R.top_logits(z, 100, ws)
    a = torch.zeros((B, T), dtype=torch.int32, device="cuda")
    calls = [lambda: R.top_logits(z, 100, ws), lambda: R.distill_from_logits(z, top["values"], top["ids"], ws, kl_share=0.5),
             lambda: R.policy_from_logits(z, a, torch.ones((B, T), device="cuda"), ws)]
    for call in calls:
        first = call()
        for _ in range(3):
            again = call()
            assert all(torch.equal(first[n].view(torch.uint8), again[n].view(torch.uint8)) for n in first)


@pytest.mark.parametrize("B,T", [(1, 3), (2, 400)])
def test_captured_run_of_all_three(B, T):
    """Teacher's entries, loss and gradient, policy loss and gradient as one graph, replayed over other inputs with eager
    calls on the same workspace in between: each replay equals the eager run."""
    V, k = 16877, 50
    student, teach = torch.empty((B, T, V), device="cuda"), torch.empty((B, T, V), device="cuda")
    a, adv = torch.zeros((B, T), dtype=torch.int32, device="cuda"), torch.ones((B, T), device="cuda")
    ws = R.LogitsWorkspace(B, T, V, k)

    def run(outs=None):
        t = R.top_logits(teach, k, ws, temperature=2.0, outs=outs and outs[0])
        d = R.distill_from_logits(student, t["values"], t["ids"], ws, teacher_lse=t["lse"], temperature=2.0,
                                  grad=outs and outs[1]["grad"], outs=outs and outs[1])
        p = R.policy_from_logits(student, a, adv, ws, old_logp=d["accept"], grad=outs and outs[2]["grad"], outs=outs and outs[2])
        return t, d, p

    def fill(seed):
        g = torch.Generator(device="cuda").manual_seed(seed)
        student.normal_(generator=g).mul_(2)
        teach.copy_(student).add_(torch.randn(teach.shape, generator=g, device="cuda"))
        a.random_(0, V, generator=g)

    fill(0)
    outs = run()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run(outs)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run(outs)
    for seed in (1, 2, 3):
        fill(seed)
        eager = run()
        for o in outs:
            for t in o.values():
                t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for o, e in zip(outs, eager):
            for n in e:
                assert torch.equal(o[n], e[n]), (seed, n)
    assert R.read_device_status(ws) == 0


def test_two_streams_with_workspaces_of_their_own():
    V, k = 50257, 64
    z = [place(draw((1, 5, V), F32, 70 + i)) for i in range(2)]
    want = [check_top(x, k) for x in z]
    streams = [torch.cuda.Stream() for _ in range(2)]
    spaces = [R.LogitsWorkspace(1, 5, V, k) for _ in range(2)]
    torch.cuda.synchronize()
    got = [None, None]
    for _ in range(5):
        for i in range(2):
            with torch.cuda.stream(streams[i]):
                got[i] = R.top_logits(z[i], k, spaces[i])
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(want[i][n], got[i][n]) for n in want[i])


def test_slices_of_longer_arrays():
    """Draft rows 1.. of [batch][k] logits, taught by rows ..k-1 of a longer teacher's arrays, without a copy."""
    z = place(draw((3, 6, 4099), F32, 80))
    vals, ids, lse = teacher_of(z, 30, 1.0, 9)
    o = R.distill_from_logits(z[:, 1:], vals[:, :5], ids[:, :5], R.LogitsWorkspace(3, 5, 4099, 30), teacher_lse=lse[:, :5])
    w = R.distill_from_logits(z[:, 1:].contiguous(), vals[:, :5].contiguous(), ids[:, :5].contiguous(),
                              R.LogitsWorkspace(3, 5, 4099, 30), teacher_lse=lse[:, :5].contiguous())
    # the rows lie on other 16-byte boundaries, so the sums run in another order: each side is off by delta at most (losses
    # below 4 and eta 0.5: times 5)
    d = delta(4099)
    assert torch.allclose(o["loss"], w["loss"], rtol=2 * HALF[F32], atol=2 * 5 * d)
    assert torch.allclose(o["accept"], w["accept"], rtol=2 * HALF[F32], atol=2 * d)
    assert torch.allclose(o["grad"], w["grad"], rtol=8 * 5 * d, atol=8 * 5 * d * float(w["grad"].abs().max()))


def test_binding_refusals():
    z = torch.zeros((2, 3, 64), device="cuda")
    ws = R.LogitsWorkspace(2, 3, 64, 4)
    v, i = torch.zeros((2, 3, 4), device="cuda"), torch.zeros((2, 3, 4), dtype=torch.int32, device="cuda")
    a, adv = torch.zeros((2, 3), dtype=torch.int32, device="cuda"), torch.zeros((2, 3), device="cuda")
    bad = [lambda: R.top_logits(z.half(), 4, ws), lambda: R.top_logits(z[0], 4, ws), lambda: R.top_logits(z.transpose(1, 2), 4, ws),
           lambda: R.top_logits(z.cpu(), 4, ws), lambda: R.distill_from_logits(z, v, i.long(), ws),
           lambda: R.distill_from_logits(z, v[:, :2], i[:, :2], ws), lambda: R.distill_from_logits(z, v, i[..., :3], ws),
           lambda: R.distill_from_logits(z, v, i, ws, teacher_lse=torch.zeros((3, 2), device="cuda").t()),
           lambda: R.distill_from_logits(z, v, i, ws, weight=adv.t().contiguous()),
           lambda: R.distill_from_logits(z, v, i, ws, last_row=a[:, 0]),
           lambda: R.policy_from_logits(z, a.float(), adv, ws), lambda: R.policy_from_logits(z, a, adv[:1], ws),
           lambda: R.policy_from_logits(z, None, adv, ws), lambda: R.LogitsWorkspace(1, 1, 100, 513)]
    for call in bad:
        with pytest.raises(ValueError):
            call()
    for call in (lambda: R.top_logits(z, 65, ws), lambda: R.distill_from_logits(z, v, i, ws, grad=z.bfloat16()),
                 lambda: R.policy_from_logits(z, a, adv, ws, grad=z[:, :2]), lambda: R.top_logits(z, 4, ws, temperature=0.0)):
        with pytest.raises(C.NLDError):
            call()


@pytest.mark.parametrize("batch,lora", [(1, False), (3, False), (2, True)])
def test_drafter_loss_on_the_tiny_model(batch, lora):
    """The whole run: draft pass (with the adapter of the LoRA-enhanced drafter, or without), verify pass and commit, the
    teacher's entries and the loss with its gradient, against the plain version on the two passes' own logits, and against the
    calls made one by one."""
    from synth.workloads import LazyWeights, ModelShape, WORKLOADS, lora_weights, prefix_kv, tokens
    wl = WORKLOADS["tiny"]
    shape, k, n_top = wl.shape, 8, 50
    model = R.DeviceModel(shape, LazyWeights(shape, wl.seed))
    if lora:
        lshape = ModelShape(**{**shape.__dict__, "lora_rank": 32, "lora_alpha": 128.0})
        model = model.with_lora(lshape, lambda l: lora_weights(lshape, wl.seed, l))
    caches = []
    for _ in range(2):
        c = R.DeviceCache(shape, batch, 256)
        for l in range(shape.n_layers):
            kb, vb = prefix_kv(shape, wl.seed, l, batch, 100)
            c.load_prefix(l, kb, vb)
        c.set_lengths([100 - 7 * b for b in range(batch)])
        caches.append(c)
    anchor = torch.from_numpy(tokens(shape, 3, "anchor", (batch,))).cuda()
    ws, lws = R.Workspace(model, batch, k, 256), R.LogitsWorkspace(batch, k, shape.vocab, n_top)
    o = R.drafter_loss(model, caches[0], ws, lws, anchor, k, n_top=n_top)
    d, dl = R.draft(model, caches[1], ws, anchor, k, want_logits=True)
    v = R.verify_accept(model, caches[1], ws, anchor, d, k, want_logits=True)
    torch.cuda.synchronize()
    assert torch.equal(o["drafts"], d) and torch.equal(o["draft_logits"], dl) and torch.equal(o["committed"], v["committed"])
    assert torch.equal(caches[0].lengths, caches[1].lengths)
    dz, vz, acc = f64(dl), f64(v["logits"]), v["accept_len"].cpu().numpy()
    eta, tau, dlt = 0.5, 3.0, delta(shape.vocab)
    for b in range(batch):
        for j in range(1, k):
            t = vz[b, j - 1]
            ids = ref.top(t, n_top)
            w = 1.0 if j - 1 <= acc[b] else 0.0
            l, a, g, size = ref.distill(dz[b, j], t[ids], ids, ref.lse(t / tau), tau, 1.0, eta, w)
            # the teacher's log-sum-exp is f32 here and off by delta itself, which moves every p by as much
            assert abs(f64(o["loss"])[b, j - 1] - l) <= 4 * dlt * (1 + 2 * eta) + HALF[F32] * abs(l)
            assert abs(f64(o["accept"])[b, j - 1] - a) <= 3 * dlt
            lse_off = (dlt + HALF[F32] * abs(ref.lse(t / tau)))
            assert np.all(np.abs(f64(o["grad"])[b, j - 1] - g) <= 4 * (dlt + lse_off) * (size + g_rest(size)) + 1e-12)
    assert R.read_device_status(ws) == 0 and R.read_device_status(lws) == 0


def g_rest(size):
    """A change of every p by e relative changes p_R by e (1 - p_R) / p_R of itself: the rest's terms by that much more."""
    return size * 4.0


@pytest.mark.parametrize("plan", PLANS)
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("V", [3, 5, 1003, 16877, 50257])
@pytest.mark.parametrize("from_end", [0, 1, None])
def test_entries_at_the_ends_of_a_row_in_place(from_end, V, dtype, plan, monkeypatch):
    """The action and the teacher's first entry in the last column, the last but one, or the first: eight adjacent rows of
    an odd length end at every place of the 16-byte grid, so in a vector that is partly another row's.  In the logits' place
    the gradient has the same bits as in a buffer of its own, where it is checked."""
    use_plan(monkeypatch, plan)
    col = 0 if from_end is None else V - 1 - from_end
    z = draw((1, 8, V), dtype, V + col)
    z[..., col] += 9.0
    actions, k = [col] * 8, 1 if V == 3 else 4
    entries = teacher_of(place(z), k, 1.0, 11)
    entries[1][..., 0] = torch.where((entries[1] == col).any(-1), entries[1][..., 0], col)
    for check in (lambda x, g: check_policy(x, actions=actions, beta=0.05, refp=True, grad=g),
                  lambda x, g: check_distill(x, k, entries=entries, grad=g)):
        apart = check(place(z), None)
        x = place(z)
        assert torch.equal(check(x, x)["grad"], apart["grad"])


# ------------------------------------------------------------------------------------------ without a gradient
@pytest.fixture
def forward_only(monkeypatch):
    """Both losses without their gradient, for the checks above."""
    for name in ("distill_from_logits", "policy_from_logits"):
        monkeypatch.setattr(R, name, functools.partial(getattr(R, name), want_grad=False))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("B,T,V,k", LOSS_SIZES)
def test_losses_without_gradient(B, T, V, k, dtype, forward_only):
    z = place(draw((B, T, V), dtype, V + 2), lead=1)
    assert check_distill(z, k, tau=3.0, want_grad=False)["grad"] is None
    assert check_policy(z, beta=0.05, refp=True)["grad"] is None


@pytest.mark.parametrize("plan", PLANS)
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("V", [1003, 50021, 151936])
def test_losses_without_gradient_by_plan(V, dtype, plan, monkeypatch, forward_only):
    """From less than one vector per thread to 149 of them, with rows that take no part, weights and strides."""
    use_plan(monkeypatch, plan)
    z = place(draw((2, 5, V), dtype, V + 3), 3, 1, 2)
    weight = torch.tensor([[1.0, 0.0, -2.0, 0.5, 3.0]] * 2, device="cuda")
    last = torch.tensor([4, 2], dtype=torch.int32, device="cuda")
    check_distill(z, 50, tau=2.0, kl_share=0.6, weight=weight, last_row=last, want_grad=False)
    check_distill(z, 300, tail=False, eta=0.0, want_grad=False)
    check_policy(z, weight=weight, last_row=last, actions=[V - 1, 0, V - 2, 1, V // 2] * 2)
    check_policy(z, tau=0.7, refp=True, beta=0.1, old=False)


@pytest.mark.parametrize("plan", PLANS)
@pytest.mark.parametrize("mask", [float("-inf"), torch.finfo(F32).min])
def test_masked_rows_without_gradient(mask, plan, monkeypatch, forward_only):
    """Teacher and student masked down to the same tokens; rows of nothing but the mask."""
    use_plan(monkeypatch, plan)
    V, k = 20011, 40
    z, t = draw((1, 4, V), F32, 14), draw((1, 4, V), F32, 15)
    off = torch.ones(V, dtype=torch.bool)
    off[[0, 900, 901, V - 1]] = False
    z[..., off] = t[..., off] = mask
    t[0, 2] = mask
    ws = R.LogitsWorkspace(1, 4, V, k)
    top = R.top_logits(place(t), k, ws)
    entries = (top["values"], top["ids"], top["lse"])
    rows = torch.tensor([[1.0, 1.0, 0.0, 1.0]], device="cuda")
    check_distill(place(z), k, eta=0.0, entries=entries, ws=ws, weight=rows, want_grad=False)
    o = R.distill_from_logits(place(z), *entries[:2], ws, teacher_lse=entries[2])
    assert o["loss"][0, 2] == 0 and o["accept"][0, 2] == 0
    check_policy(place(z), actions=[0, 900, 901, V - 1])


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_the_longest_row_without_gradient(dtype, forward_only):
    V, k = 1 << 24, 100
    g = torch.Generator(device="cuda").manual_seed(3)
    z = torch.randn((1, 1, V), generator=g, device="cuda").mul_(2.5).to(dtype)
    d, ws = z[0, 0].double(), R.LogitsWorkspace(1, 1, V, k)
    L = torch.logsumexp(d, 0).item()
    t = R.top_logits(z, k, ws)
    a = torch.full((1, 1), V - 1, dtype=torch.int32, device="cuda")
    p = R.policy_from_logits(z, a, torch.ones((1, 1), device="cuda"), ws)
    want = d[V - 1].item() - L
    assert abs(p["logp"].item() - want) <= delta(V) + HALF[F32] * abs(want)
    # a teacher that is the student, by its log-sum-exp alone: KL 0 and everything accepted, within what each side is off by
    o = R.distill_from_logits(z, t["values"], t["ids"], ws, teacher_lse=t["lse"], eta=0.0)
    assert abs(o["loss"].item()) <= 3 * delta(V) and abs(o["accept"].item() - 1.0) <= 3 * delta(V)


def test_gradients_of_rows_past_32_bits():
    """The last rows of more than 2^32 bytes, in place and apart, against the 64-bit gradient column by column; the rows
    before them hold other logits."""
    T, V, k = 14200, 151936, 64
    tail = draw((1, 2, V), BF16, 7)
    z = torch.empty((1, T, V), dtype=BF16, device="cuda")
    z[:, :-2] = tail[0, 0].roll(7).cuda()
    z[:, -2:] = tail.cuda()
    entries = teacher_of(tail, k, 1.0, 5)
    ws, d, h = R.LogitsWorkspace(1, T, V, k), delta(V), HALF[BF16]
    many = lambda t, fill: torch.cat([torch.full((1, T - 2) + t.shape[2:], fill, dtype=t.dtype, device="cuda"), t], 1)    # noqa: E731
    vals, ids, lse = (many(t, 0) for t in entries)
    weight = many(torch.ones((1, 2), device="cuda"), 0.0)
    top = R.top_logits(z, k, ws)
    actions = many(top["ids"][:, -2:, 5].contiguous(), -1)
    adv = torch.ones((1, T), device="cuda")
    zz = f64(tail)[0]
    plain = {"p": [ref.policy(zz[r], int(actions[0, T - 2 + r]), 1.0, None, None, 1.0, 0.2, 0.2, 0.0, 1.0) for r in range(2)],
             "d": [ref.distill(zz[r], f64(vals)[0, T - 2 + r], ids.cpu().numpy()[0, T - 2 + r], f64(lse)[0, T - 2 + r], 1.0, 1.0,
                               0.5, 1.0) for r in range(2)]}
    for r in range(2):
        assert np.array_equal(top["ids"][0, T - 2 + r].cpu().numpy(), ref.top(zz[r], k))
    grad = torch.empty_like(z)
    for name, call in (("p", lambda g: R.policy_from_logits(z, actions, adv, ws, grad=g)),
                       ("d", lambda g: R.distill_from_logits(z, vals, ids, ws, teacher_lse=lse, weight=weight, grad=g)),
                       ("d", lambda g: R.distill_from_logits(z, vals, ids, ws, teacher_lse=lse, weight=weight, grad=z))):
        o = call(grad)
        assert not o["grad"][:, :-2].any() and not o["loss"][:, :-2].any()
        G, L = f64(o["grad"][:, -2:])[0], f64(o["loss"])[0, -2:]
        for r, (l, a, g, size) in enumerate(plain[name]):
            slack = 1 + 2 * 0.5 * max(l, 1.0) if name == "d" else 2.0
            move = ref.distill_undecided(zz[r], f64(vals)[0, T - 2 + r], ids.cpu().numpy()[0, T - 2 + r], f64(lse)[0, T - 2 + r],
                                         1.0, 1.0, 0.5, 1.0, d) if name == "d" else 0.0
            assert abs(L[r] - l) <= d * slack + HALF[F32] * abs(l)
            assert np.all(np.abs(G[r] - g) <= 4 * d * slack * size + h * np.abs(g) + move + 1e-37)
    assert R.read_device_status(ws) == 0


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_top_of_logits_below_the_normal_range(dtype):
    z = (torch.arange(3001, dtype=torch.float32) - 1500.0).roll(700) * 2.0 ** -133
    check_top(place(z.to(dtype)[None, None].expand(1, 2, 3001).clone()), 40)


@pytest.mark.parametrize("plan", PLANS)
@pytest.mark.parametrize("tau", [1.0, 0.3])
def test_teacher_of_logits_whose_log_sum_exp_is_rounded_away(tau, plan, monkeypatch):
    """From 2^24 on an f32 log-sum-exp says nothing of the entries, which then are the teacher: row 0 has equal logits, row 1
    one token."""
    use_plan(monkeypatch, plan)
    V, k, tau = 20011, 40, as_f32(tau)
    t = torch.full((1, 2, V), 2.0 ** 27)
    t[0, 1] = 0.0
    t[0, 1, 5] = 2.0 ** 27
    ws, d, h = R.LogitsWorkspace(1, 2, V, k), delta(V), HALF[F32]
    top = R.top_logits(place(t), k, ws, temperature=tau)
    assert (top["lse"] >= 2.0 ** 24).all()
    for grad in (True, False):
        o = R.distill_from_logits(torch.zeros((1, 2, V), device="cuda"), top["values"], top["ids"], ws, teacher_lse=top["lse"],
                                  temperature=tau, eta=0.0, want_grad=grad)
        for r, n in ((0, k), (1, 1)):
            assert abs(o["loss"][0, r].item() - np.log(V / n)) <= d + h * np.log(V / n)
            assert abs(o["accept"][0, r].item() - n / V) <= d
            if grad:
                p = np.zeros(V)
                p[5 if n == 1 else slice(0, k)] = 1.0 / n
                want = (1.0 / V - p) / tau
                assert np.all(np.abs(f64(o["grad"])[0, r] - want) <= 4 * d * (1.0 / V + p) / tau + h * np.abs(want))


@pytest.mark.parametrize("plan", PLANS)
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("entries", [0, 10])
def test_a_log_sum_exp_that_is_no_number(entries, bad, plan, monkeypatch):
    """The teacher's own, with entries that are numbers or with none: NaN throughout the row and nowhere else."""
    use_plan(monkeypatch, plan)
    z = place(draw((1, 3, 20011), F32, 4))
    vals, ids, lse = teacher_of(z, 10, 1.0, 3)
    lse[0, 1] = bad
    ids[0, 1, entries:] = -1
    o = R.distill_from_logits(z, vals, ids, R.LogitsWorkspace(1, 3, 20011, 10), teacher_lse=lse)
    assert torch.isnan(o["loss"][0, 1]) and torch.isnan(o["accept"][0, 1]) and torch.isnan(o["grad"][0, 1]).all()
    assert torch.isfinite(o["loss"][0, [0, 2]]).all() and torch.isfinite(o["grad"][0, [0, 2]]).all()


def test_autograd_sees_what_a_call_writes():
    """A loss hangs on no graph; its gradient is handed on by logits.backward.  In the logits' place it is a change that
    autograd knows of, so that an operation which kept these logits for its own backward pass raises."""
    V, k = 1003, 8
    a, adv = torch.full((1, 2), 3, dtype=torch.int32, device="cuda"), torch.ones((1, 2), device="cuda")
    ws = R.LogitsWorkspace(1, 2, V, k)
    top = R.top_logits(torch.randn((1, 2, V), device="cuda"), k, ws)
    calls = (lambda z, **kw: R.distill_from_logits(z, top["values"], top["ids"], ws, teacher_lse=top["lse"], **kw),
             lambda z, **kw: R.policy_from_logits(z, a, adv, ws, **kw))
    for call in calls:
        x = torch.randn((1, 2, V), device="cuda", requires_grad=True)
        z = 2.0 * x
        o = call(z)
        assert not o["loss"].requires_grad and z._version == 0
        z.backward(o["grad"])
        assert torch.equal(x.grad, 2.0 * o["grad"])
        capped = torch.tanh(x)
        call(capped, grad=capped)
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            capped.sum().backward()
    outs = {n: torch.empty_like(t) for n, t in top.items()}
    R.top_logits(torch.randn((1, 2, V), device="cuda"), k, ws, outs=outs)
    loss = {n: torch.empty((1, 2), device="cuda") for n in ("loss", "accept", "logp")}
    for call in calls:
        call(torch.randn((1, 2, V), device="cuda"), outs=loss)
    assert all(t._version > 0 for t in list(outs.values()) + list(loss.values()))
    before = [t._version for t in loss.values()]
    with pytest.raises(C.NLDError):
        calls[0](torch.randn((1, 2, V), device="cuda"), outs=loss, temperature=0.0)
    assert before == [t._version for t in loss.values()]       # a refused call wrote nothing


@pytest.mark.parametrize("plan", PLANS)
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("column", [0, 9000, 20010])
def test_not_a_number_by_plan(column, bad, dtype, plan, monkeypatch):
    """In the first, a middle and the last column, which is an entry in one row and none in the other: NaN all over these
    rows, with a gradient and without one, and numbers in the rows beside them."""
    use_plan(monkeypatch, plan)
    V, k = 20011, 10
    z = draw((1, 5, V), dtype, 16)
    vals, ids, lse = teacher_of(z, k, 1.0, 17)
    ids[0, 1] = torch.arange(100, 100 + k, dtype=torch.int32)
    ids[0, 3] = ids[0, 1]
    ids[0, 3, 7] = column
    z[0, [1, 3], column] = bad
    zd = place(z, lead=1)
    a = torch.tensor([[5, 5, 5, column, 5]], dtype=torch.int32, device="cuda")
    ws = R.LogitsWorkspace(1, 5, V, k)
    for grad in (True, False):
        o = R.distill_from_logits(zd, vals, ids, ws, teacher_lse=lse, want_grad=grad)
        p = R.policy_from_logits(zd, a, torch.ones((1, 5), device="cuda"), ws, want_grad=grad)
        for x in [o["loss"], o["accept"], p["loss"], p["logp"]] + ([o["grad"], p["grad"]] if grad else []):
            assert torch.isnan(x[0, [1, 3]]).all() and torch.isfinite(x[0, [0, 2, 4]]).all()


@pytest.mark.parametrize("plan", PLANS)
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_rows_of_the_lowest_value_in_place(dtype, plan, monkeypatch):
    """Rows whose statistics take differences first: masked by the type's lowest value but for a few tokens, the last column among
    them, and throughout.  In the logits' place as in a buffer of its own."""
    use_plan(monkeypatch, plan)
    V = 20011
    z = draw((1, 8, V), dtype, 18)
    off = torch.ones(V, dtype=torch.bool)
    off[[0, 77, V - 4, V - 1]] = False
    z[0, ::2, off] = torch.finfo(dtype).min
    z[0, [2, 5]] = torch.finfo(dtype).min
    z[0, 7] = 2.0 ** 40
    k = 4
    ids = torch.tensor([0, V - 1, 77, 9], dtype=torch.int32, device="cuda").expand(1, 8, k).contiguous()
    vals, lse = torch.zeros((1, 8, k), device="cuda"), torch.full((1, 8), float(np.float32(np.log(5))), device="cuda")
    a, adv = torch.full((1, 8), V - 1, dtype=torch.int32, device="cuda"), torch.ones((1, 8), device="cuda")
    ws, one, d = R.LogitsWorkspace(1, 8, V, k), np.ones((1, 8)), delta(V)
    # less the row's largest, which is exact here and changes no softmax: beside 3e38 the logarithm of a sum is lost in 64 bits too
    zz = f64(z)[0]
    zz = zz - zz.max(-1, keepdims=True)
    t = float(lse[0, 0])
    for call, aux, plain, move in (
            (lambda x, g: R.policy_from_logits(x, a, adv, ws, grad=g), "logp",
             lambda r: ref.policy(zz[r], V - 1, 1.0, None, None, 1.0, 0.2, 0.2, 0.0, 1.0), lambda r: 0.0),
            (lambda x, g: R.distill_from_logits(x, vals, ids, ws, teacher_lse=lse, kl_share=0.0, eta=0.0, grad=g), "accept",
             lambda r: ref.distill(zz[r], np.zeros(k), ids[0, 0].cpu().numpy(), t, 1.0, 0.0, 0.0, 1.0),
             lambda r: ref.distill_undecided(zz[r], np.zeros(k), ids[0, 0].cpu().numpy(), t, 1.0, 0.0, 0.0, 1.0, d))):
        apart = call(place(z), None)
        compare(z, one, apart["loss"], apart[aux], apart["grad"], plain, lambda r: 2.0 if aux == "logp" else 1.0, 1.0, move)
        x = place(z)
        assert torch.equal(call(x, x)["grad"], apart["grad"])


def test_policy_on_what_a_verify_pass_commits():
    """committed, with its -1 behind the accepted drafts, is taken as actions as it is."""
    from synth.workloads import LazyWeights, WORKLOADS, prefix_kv, tokens
    wl = WORKLOADS["tiny"]
    shape, batch, k = wl.shape, 3, 8
    model = R.DeviceModel(shape, LazyWeights(shape, wl.seed))
    cache = R.DeviceCache(shape, batch, 256)
    for l in range(shape.n_layers):
        cache.load_prefix(l, *prefix_kv(shape, wl.seed, l, batch, 100))
    cache.set_lengths([100 - 7 * b for b in range(batch)])
    anchor = torch.from_numpy(tokens(shape, 3, "anchor", (batch,))).cuda()
    ws = R.Workspace(model, batch, k, 256)
    d, _ = R.draft(model, cache, ws, anchor, k)
    v = R.verify_accept(model, cache, ws, anchor, d, k, want_logits=True)
    adv, lws = torch.ones((batch, k), device="cuda"), R.LogitsWorkspace(batch, k, shape.vocab)
    o = R.policy_from_logits(v["logits"], v["committed"], adv, lws)
    a, zz = v["committed"].cpu().numpy().reshape(-1), f64(v["logits"]).reshape(-1, shape.vocab)
    compare(v["logits"], np.ones((batch, k)), o["loss"], o["logp"], o["grad"],
            lambda r: ref.policy(zz[r], int(a[r]), 1.0, None, None, 1.0, 0.2, 0.2, 0.0, 1.0), lambda r: 2.0, 1.0)
    behind = torch.arange(k, device="cuda")[None] > v["accept_len"][:, None]
    assert bool((v["committed"][behind] == -1).all()) and not o["grad"][behind].any()
    assert R.read_device_status(lws) == 0
