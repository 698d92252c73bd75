"""The operators on rows of logits: argument checks (nothing is enqueued), and the plain versions that the GPU tests
compare with, against differences and closed forms.  No GPU needed."""
import ctypes
from types import SimpleNamespace

import logits_ref as ref
import numpy as np
import pytest
import torch

from paper_2607_05722_amd import _lib as C
from paper_2607_05722_amd import runtime

P = 0x1000
WS = 1 << 40


def logits(data=P, dtype=C.NLD_F32, batch=2, rows=3, vocab=100, seq=300, row=100):
    return C.Logits(data, dtype, batch, rows, vocab, seq, row)


def top(z, n=5, tau=1.0, values=P, ids=P, ws=P, ws_bytes=WS):
    return C.load().nld_top_logits(ctypes.byref(z) if z is not None else None, n, tau, values, ids, None, ws, ws_bytes, None)


def distill(z=None, teacher=None, tau=1.0, kl=1.0, eta=0.5, loss=P, grad=None, ws=P, ws_bytes=WS):
    z = z or logits()
    teacher = teacher or C.Teacher(P, P, P, 5, 3)
    return C.load().nld_distill_from_logits(ctypes.byref(z), ctypes.byref(teacher), tau, kl, eta, None, None, loss, None,
                                            ctypes.byref(grad) if grad else None, ws, ws_bytes, None)


def policy(z=None, rollout=None, tau=1.0, lo=0.2, hi=0.2, beta=0.0, loss=P, grad=None, ws=P, ws_bytes=WS):
    z = z or logits()
    rollout = rollout or C.Rollout(P, P, None, None)
    return C.load().nld_policy_from_logits(ctypes.byref(z), ctypes.byref(rollout), tau, lo, hi, beta, None, None, loss, None,
                                           ctypes.byref(grad) if grad else None, ws, ws_bytes, None)


NAN, INF = float("nan"), float("inf")

BAD_LOGITS = [
    (dict(data=0), C.NLD_ERR_INVALID_ARG), (dict(dtype=2), C.NLD_ERR_INVALID_ARG), (dict(batch=0), C.NLD_ERR_INVALID_ARG),
    (dict(rows=-1), C.NLD_ERR_INVALID_ARG), (dict(vocab=0), C.NLD_ERR_INVALID_ARG), (dict(seq=-300), C.NLD_ERR_INVALID_ARG),
    (dict(row=1 << 40), C.NLD_ERR_INVALID_ARG), (dict(data=P + 2), C.NLD_ERR_INVALID_ARG),
    (dict(data=P + 1, dtype=C.NLD_BF16), C.NLD_ERR_INVALID_ARG), (dict(vocab=(1 << 24) + 1), C.NLD_ERR_SHAPE),
    (dict(batch=1 << 11, rows=1 << 10), C.NLD_ERR_SHAPE), (dict(rows=1 << 16, vocab=1 << 24), C.NLD_ERR_SHAPE)]


@pytest.mark.parametrize("over,status", BAD_LOGITS)
def test_every_call_refuses_bad_logits(over, status):
    z = logits(**over)
    assert top(z) == distill(z, C.Teacher(P, P, P, 5, 1 << 20)) == policy(z) == status


def test_top_refusals():
    z = logits()
    assert top(None) == C.NLD_ERR_INVALID_ARG
    for n, st in ((0, C.NLD_ERR_INVALID_ARG), (101, C.NLD_ERR_INVALID_ARG)):
        assert top(z, n=n) == st
    assert top(logits(vocab=1000, row=1000, seq=3000), n=513) == C.NLD_ERR_SHAPE
    for tau in (0.0, -1.0, 1e-4, 1e4, NAN, INF):
        assert top(z, tau=tau) == C.NLD_ERR_INVALID_ARG
    assert top(z, values=None) == top(z, ids=None) == top(z, ws=None) == C.NLD_ERR_INVALID_ARG
    need = C.load().nld_logits_workspace_bytes(2, 3, 100, 5)
    assert top(z, ws_bytes=need - 1) == C.NLD_ERR_CAPACITY


def test_distill_refusals():
    lib = C.load()
    bad = [distill(teacher=C.Teacher(None, P, P, 5, 3)), distill(teacher=C.Teacher(P, None, P, 5, 3)),
           distill(teacher=C.Teacher(P, P, P, 0, 3)), distill(teacher=C.Teacher(P, P, P, 5, 2)), distill(loss=None),
           distill(kl=-0.1), distill(kl=1.1), distill(kl=NAN), distill(eta=-1.0), distill(eta=NAN), distill(eta=INF),
           distill(tau=NAN), distill(ws=None)]
    assert bad == [C.NLD_ERR_INVALID_ARG] * len(bad)
    assert lib.nld_distill_from_logits(ctypes.byref(logits()), None, 1.0, 1.0, 0.5, None, None, P, None, None, P, WS, None) == \
        C.NLD_ERR_INVALID_ARG
    assert distill(ws_bytes=256) == C.NLD_ERR_CAPACITY


def test_policy_refusals():
    bad = [policy(rollout=C.Rollout(None, P, None, None)), policy(rollout=C.Rollout(P, None, None, None)), policy(loss=None),
           policy(lo=-0.1), policy(lo=1.5), policy(lo=NAN), policy(hi=-0.1), policy(hi=INF), policy(beta=-1.0),
           policy(beta=NAN), policy(tau=0.0), policy(ws=None)]
    assert bad == [C.NLD_ERR_INVALID_ARG] * len(bad)
    assert policy(ws_bytes=256) == C.NLD_ERR_CAPACITY


@pytest.mark.parametrize("call", [distill, policy])
def test_grad_refusals(call):
    """Other sizes, rows that overlap, a buffer that overlaps the logits without being them."""
    far = 0x100000
    bad = [dict(data=0), dict(data=far, dtype=C.NLD_BF16), dict(data=far, vocab=99), dict(data=far, rows=2),
           dict(data=far, row=99), dict(data=far, seq=299), dict(data=far, seq=0), dict(data=far, row=0),
           dict(data=far, row=100, seq=100), dict(data=P + 4), dict(data=P, row=101, seq=303), dict(data=P + 2396),
           dict(data=P - 2396)]
    for over in bad:
        assert call(grad=logits(**over)) == C.NLD_ERR_INVALID_ARG, over
    assert call(z=logits(seq=0), grad=logits(seq=0)) == C.NLD_ERR_INVALID_ARG    # broadcast rows in their own place


def test_workspace_serves_smaller_calls():
    lib = C.load()
    size = lib.nld_logits_workspace_bytes
    assert size(0, 1, 100, 1) == size(1, 1, 100, 101) == size(1, 1, 1000, 513) == size(1, 1, (1 << 24) + 1, 1) == 0
    for B, T, V, n in [(8, 512, 151936, 200), (1, 1, 151936, 200), (32, 32, 1 << 20, 512), (1, 40, 1 << 24, 512)]:
        big = size(B, T, V, n)
        assert big % 256 == 0
        for b in {1, B // 2 or 1, B}:
            for t in {1, 3, T // 2 or 1, T}:
                for v in {n, 5000, V // 2, V}:
                    for m in {1, n // 2 or 1, n}:
                        assert size(b, t, v, m) <= big, (b, t, v, m)


# ------------------------------------------------------------------------------------ the plain versions themselves
@pytest.mark.parametrize("tail,kl,eta,n", [(True, 1.0, 0.0, 5), (True, 1.0, 0.0, 12), (False, 0.3, 0.0, 5), (True, 0.0, 0.0, 1),
                                           (False, 1.0, 0.0, 1)])
def test_plain_distill_gradient_against_differences(tail, kl, eta, n):
    """eta = 0: lambda does not depend on the logits, so differences of the loss are the gradient."""
    rng = np.random.default_rng(1)
    V, tau, w, h = 12, 1.7, 0.6, 1e-6
    z, t = rng.normal(size=V) * 2, rng.normal(size=V) * 2
    ids = rng.permutation(V)[:n]
    c = ref.lse(t / tau) if tail else None
    f = lambda x: ref.distill(x, t[ids], ids, c, tau, kl, eta, w)[0]    # noqa: E731
    g = ref.distill(z, t[ids], ids, c, tau, kl, eta, w)[2]
    for j in range(V):
        e = np.zeros(V)
        e[j] = h
        assert abs((f(z + e) - f(z - e)) / (2 * h) - g[j]) < 1e-7
    assert abs(g.sum()) < 1e-14        # a shift of every logit changes nothing


def test_plain_distill_closed_forms():
    z = np.log(np.array([0.5, 0.25, 0.125, 0.125]))
    # the teacher equal to the student: nothing to learn, everything accepted
    loss, alpha, g, _ = ref.distill(z, z[:2], [0, 1], 0.0, 1.0, 1.0, 0.0, 1.0)
    assert abs(loss) < 1e-15 and abs(alpha - 1) < 1e-15 and np.max(np.abs(g)) < 1e-15
    # one entry alone: cross-entropy
    loss, alpha, g, _ = ref.distill(z, [3.0], [1], None, 1.0, 1.0, 0.0, 1.0)
    assert abs(loss - np.log(4)) < 1e-15 and np.allclose(g, [0.5, -0.75, 0.125, 0.125])
    # total variation of (0.75, 0.25 elsewhere) against (0.5, 0.5 elsewhere)
    assert abs(ref.distill(z, [np.log(0.75)], [0], 0.0, 1.0, 0.0, 0.0, 2.0)[0] - 2 * 0.25) < 1e-15


@pytest.mark.parametrize("adv,old,refp", [(1.0, -1.5, None), (-1.0, -1.5, -2.0), (0.7, None, -1.0), (1.0, -9.0, None),
                                          (-1.0, 2.0, None)])
def test_plain_policy_gradient_against_differences(adv, old, refp):
    rng = np.random.default_rng(2)
    V, tau, w, h, a = 9, 0.8, 1.3, 1e-6, 4
    z = rng.normal(size=V)
    logp = z[a] / tau - ref.lse(z / tau)
    f = lambda x: ref.policy(x, a, adv, old if old is not None else logp, refp, tau, 0.2, 0.3, 0.1, w)[0]    # noqa: E731
    g = ref.policy(z, a, adv, old, refp, tau, 0.2, 0.3, 0.1, w)[2]
    for j in range(V):
        e = np.zeros(V)
        e[j] = h
        assert abs((f(z + e) - f(z - e)) / (2 * h) - g[j]) < 1e-7


def test_plain_distill_of_a_shared_mask():
    """Teacher and student masked to the same three tokens: what rounding the teacher's log-sum-exp to f32 leaves of
    1 - sum p is no token that the student could lack; more than that is."""
    z = np.full(50, -np.inf)
    z[:3] = [1.0, 2.0, 3.0]
    c = float(np.float32(ref.lse(z + 20.0)))
    for off in (0.0, 1e-6):
        loss, alpha, g, _ = ref.distill(z, z[:3] + 20.0, [0, 1, 2], c + off, 1.0, 1.0, 0.0, 1.0)
        assert abs(loss) < 3e-6 and abs(alpha - 1) < 3e-6 and np.max(np.abs(g)) < 3e-6
    assert ref.distill(z, z[:3] + 20.0, [0, 1, 2], c + 1e-5, 1.0, 1.0, 0.0, 1.0)[0] == np.inf


BAD_DRAFTER_LOSS = [dict(k=1), dict(n_top=0), dict(n_top=513), dict(n_top=301), dict(temperature=0.0), dict(temperature=NAN),
                    dict(kl_share=1.5), dict(eta=-1.0), dict(eta=INF), dict(nbytes=0), dict(weight=(2, 8)), dict(device="meta")]


@pytest.mark.parametrize("bad", BAD_DRAFTER_LOSS, ids=lambda b: "-".join("%s_%s" % x for x in b.items()))
def test_drafter_loss_refuses_before_any_pass(bad):
    """The cache would have moved on otherwise: no model, cache or workspace is touched."""
    bad = dict(bad)
    model = SimpleNamespace(shape=SimpleNamespace(vocab=300))
    ws = SimpleNamespace(nbytes=bad.pop("nbytes", WS), buf=torch.empty(0, device=bad.pop("device", "cpu")))
    args = dict(k=8, n_top=50)
    args.update(bad)
    if "weight" in args:
        args["weight"] = torch.ones(args["weight"])
    with pytest.raises(ValueError):
        runtime.drafter_loss(model, None, None, ws, torch.zeros(2, dtype=torch.int32), **args)


def test_drafter_loss_refuses_an_eta_past_f32_before_any_pass():
    """1e39 is finite here and infinite in the call, which would refuse it after the verify pass."""
    ws = SimpleNamespace(nbytes=WS, buf=torch.empty(0))
    with pytest.raises(ValueError):
        runtime.drafter_loss(SimpleNamespace(shape=SimpleNamespace(vocab=300)), None, None, ws,
                             torch.zeros(2, dtype=torch.int32), k=8, n_top=50, eta=1e39)


def like_logits(shape, stride):
    """What the binding looks at of a device tensor."""
    return SimpleNamespace(dtype=torch.float32, shape=shape, is_cuda=True, device=torch.device("cuda", 0), dim=lambda: 3,
                           stride=lambda: stride, data_ptr=lambda: P)


@pytest.mark.parametrize("shape", [(1 << 32, 1, 5), (1, (1 << 32) + 3, 5), (1, 1, (1 << 32) + 5), (1 << 31, 1, 5)])
def test_binding_refuses_sizes_past_int32(shape):
    """The descriptor's fields would keep their lower halves: a call on the first few rows or columns, with no error."""
    with pytest.raises(ValueError):
        runtime._logits(like_logits(shape, (shape[1] * shape[2], shape[2], 1)), "logits")


def test_binding_refuses_entries_past_int32():
    meta = torch.device("meta")
    many = lambda B, T, n, seq, dt: torch.empty_strided((B, T, n), (seq, n, 1), dtype=dt, device=meta)    # noqa: E731
    for args in ((2, 3, 1, (1 << 32) + 3), (1, 1, (1 << 32) + 5, (1 << 32) + 5)):
        with pytest.raises(ValueError):
            runtime._entries(many(*args, torch.float32), many(*args, torch.int32), None, args[:2], meta)
    runtime._entries(many(2, 3, 4, 40, torch.float32), many(2, 3, 4, 40, torch.int32), None, (2, 3), meta)
    for n in ((1 << 32) + 5, -1):
        with pytest.raises(ValueError):
            runtime.top_logits(like_logits((1, 1, 100), (100, 100, 1)), n, None)
