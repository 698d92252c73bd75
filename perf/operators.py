"""Performance cases of the operators on rows of logits: the teacher's top logits, the distillation loss of
the drafter and the clipped policy loss, each loss with or without its gradient.

A case is one call on logits [batch][rows][vocab].  Logits are 2.5 x normal with eight likely tokens per row,
so that a row's probability sits on a few tokens and a long tail, as a language model's does; a teacher's are
the student's plus noise.  `share` is the share of rows that count (the others are padding, or drafts behind
the first rejected one): they have weight 0.

Case keys: op (top, distill, policy), dtype (f32: what the passes of this library return; bf16: a trainer's),
batch, rows, vocab, n_top (top, distill), tau (temperature), grad (the gradient too), share, tail (distill: the
teacher's log-sum-exp over the whole vocabulary is given), kl_share and eta (distill: the mixture), old and ref
(policy: log-probabilities of the behaviour and of the reference policy are given), kl_coef (policy).
"""
import math
import random

import torch

own = False

CLIP_LOW, CLIP_HIGH = 0.2, 0.28
_CHUNK = 1 << 25    # logits per slice where the inputs and the 64-bit results are made


def _case(name, op, dtype, batch, rows, vocab, n_top=1, tau=1.0, grad=False, share=1.0, tail=True, kl_share=1.0,
          eta=0.0, old=False, ref=False, kl_coef=0.0):
    c = {"op": op, "dtype": dtype, "batch": batch, "rows": rows, "vocab": vocab, "n_top": n_top, "tau": tau,
         "grad": grad, "share": share, "tail": tail, "kl_share": kl_share, "eta": eta, "old": old, "ref": ref,
         "kl_coef": kl_coef}
    return dict({"name": name}, **c) if name else c


def listed():
    return [
        # one token's best candidates out of a small vocabulary: latency is all there is
        _case("top_tiny", "top", "f32", 1, 1, 1024, n_top=20),
        # the verify rows of one block of the 8B shapes, as the drafter's teacher (top 200, temperature 3)
        _case("top_block_k16", "top", "f32", 1, 16, 151936, n_top=200, tau=3.0),
        # the verify rows of a batch of 32 blocks
        _case("top_b32_k16", "top", "f32", 32, 16, 151936, n_top=200, tau=3.0),
        # a teacher's logits of a training batch, stored as their top 64
        _case("top_train_bf16", "top", "bf16", 4, 512, 151936, n_top=64),
        # the drafter's loss over one tiny block
        _case("distill_tiny", "distill", "f32", 1, 7, 1024, n_top=32, tau=3.0, grad=True, eta=0.5),
        # the drafter's loss and gradient over eight blocks of 32, a part of them behind the first rejected draft
        _case("distill_b8_k32", "distill", "f32", 8, 31, 151936, n_top=200, tau=3.0, grad=True, share=0.4, eta=0.5),
        # the same loss as an evaluation of many blocks: no gradient
        _case("distill_eval", "distill", "f32", 32, 31, 151936, n_top=200, tau=3.0, eta=0.5),
        # a training step of distillation from stored top logits, the largest case
        _case("distill_train_bf16", "distill", "bf16", 8, 512, 151936, n_top=64, grad=True, share=0.9),
        # log-probability of one decoded token
        _case("policy_token", "policy", "f32", 1, 1, 151936),
        # rollouts of an odd vocabulary, scored and clipped without a gradient
        _case("policy_score_odd", "policy", "bf16", 5, 333, 50257, share=0.8, old=True),
        # a policy step over rollouts that are decoded with this library: f32 logits of verify passes
        _case("policy_blocks_f32", "policy", "f32", 32, 16, 151936, grad=True, old=True, ref=True, kl_coef=0.05),
        # a policy step of a trainer, ragged rollouts padded to 256 tokens
        _case("policy_train_bf16", "policy", "bf16", 16, 256, 151936, grad=True, share=0.7, old=True, ref=True,
              kl_coef=0.05),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng: random.Random):
    most = max(work(c)["bytes"] for c in listed())
    while True:
        op = rng.choice(["top", "distill", "policy"])
        dtype = rng.choice(["f32", "bf16"])
        batch = 1 if rng.random() < 0.3 else _log_int(rng, 2, 64)
        rows = _log_int(rng, 1, 1024)
        vocab = 151936 if rng.random() < 0.3 else _log_int(rng, 1000, 200000)
        n_top = min(vocab, _log_int(rng, 1, 256)) if op != "policy" else 1
        tau = rng.choice([1.0, 1.0, 0.7, 2.0, 3.0])
        grad = op != "top" and rng.random() < 0.7
        share = 1.0 if op == "top" or rng.random() < 0.4 else rng.uniform(0.2, 1.0)
        distill, policy = op == "distill", op == "policy"
        c = _case(None, op, dtype, batch, rows, vocab, n_top, tau, grad, share,
                  tail=rng.random() < 0.6 if distill else True,
                  kl_share=rng.choice([1.0, 1.0, 0.5]) if distill else 1.0,
                  eta=rng.choice([0.0, 0.5]) if distill else 0.0,
                  old=policy and rng.random() < 0.7, ref=policy and rng.random() < 0.5)
        c["kl_coef"] = 0.05 if c["ref"] else 0.0
        if work(c)["bytes"] <= most and batch * rows <= 16384:
            return c


def _active(case):
    return max(1, int(round(case["share"] * case["batch"] * case["rows"])))


def work(case):
    R, V, K = case["batch"] * case["rows"], case["vocab"], case["n_top"]
    es = 2 if case["dtype"] == "bf16" else 4
    n = _active(case)
    if case["op"] == "top":
        return {"bytes": R * V * es + R * (8 * K + 4), "flops": 4 * R * V}
    rows = 12 * R if case["op"] == "distill" else 20 * R     # weights, row inputs and row outputs
    entries = 8 * K * n if case["op"] == "distill" else 4 * n
    return {"bytes": n * V * es + entries + rows + (R * V * es if case["grad"] else 0),
            "flops": n * V * (7 if case["grad"] else 4)}


# ------------------------------------------------------------------------------------------ seeded inputs
def _gen(seed, tag):
    g = torch.Generator(device="cuda")
    g.manual_seed((seed * 1000003 + tag * 8191) & 0x7FFFFFFF)
    return g


def _logits(case, seed):
    R, V = case["batch"] * case["rows"], case["vocab"]
    dt = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
    g = _gen(seed, 1)
    z = torch.randn((R, V), generator=g, device="cuda", dtype=dt).mul_(2.5)
    likely = (torch.randint(0, V, (R, 1), generator=g, device="cuda") + torch.arange(8, device="cuda") * (V // 8)) % V
    lift = torch.rand((R, 8), generator=g, device="cuda").mul_(10.0).add_(4.0).to(dt)
    z.scatter_(1, likely, lift)
    return z


def _teacher(case, seed, z):
    """Top entries of a teacher near the student: values f32 (descending), ids int32, lse f32."""
    K, c = case["n_top"], 1.0 / case["tau"]
    g = _gen(seed, 2)
    vals, ids, lse = [], [], []
    n = max(1, _CHUNK // z.shape[1])
    for r in range(0, z.shape[0], n):
        t = z[r:r + n].float()
        t = t + torch.randn(t.shape, generator=g, device="cuda").mul_(0.5)
        v, i = torch.topk(t, K, dim=1)
        vals.append(v)
        ids.append(i.to(torch.int32))
        m = v[:, :1] * c
        lse.append((m[:, 0].double() + torch.log(torch.exp(t * c - m).sum(1, dtype=torch.float64))).float())
    return torch.cat(vals), torch.cat(ids), torch.cat(lse)


def prepare(case, seed):
    B, T, V = case["batch"], case["rows"], case["vocab"]
    R = B * T
    z = _logits(case, seed)
    st = {"case": case, "logits": z.view(B, T, V)}
    if case["op"] != "top":
        g = _gen(seed, 3)
        n = _active(case)
        w = torch.zeros(R, device="cuda")
        w[torch.randperm(R, generator=g, device="cuda")[:n]] = 1.0 / n
        st["weight"] = w.view(B, T)
    if case["op"] == "distill":
        v, i, s = _teacher(case, seed, z)
        st["values"], st["ids"] = v.view(B, T, -1), i.view(B, T, -1)
        st["lse"] = s.view(B, T) if case["tail"] else None
    if case["op"] == "policy":
        # tokens as the policy itself would decode them: the largest of logits / tau plus Gumbel noise
        a = torch.empty(R, dtype=torch.int64, device="cuda")
        logp = torch.empty(R, device="cuda")
        c = 1.0 / case["tau"]
        n = max(1, _CHUNK // V)
        for r in range(0, R, n):
            y = z[r:r + n].float() * c
            u = torch.rand(y.shape, generator=g, device="cuda").clamp_(1e-12, 1.0 - 1e-7)
            a[r:r + n] = torch.argmax(y - torch.log(-torch.log(u)), dim=1)
            logp[r:r + n] = y.gather(1, a[r:r + n, None])[:, 0] - torch.logsumexp(y, 1)
        st["actions"] = a.to(torch.int32).view(B, T)
        st["advantage"] = torch.randn((B, T), generator=g, device="cuda")
        noise = torch.randn((2, B, T), generator=g, device="cuda")
        st["old_logp"] = logp.view(B, T) + 0.2 * noise[0] if case["old"] else None
        st["ref_logp"] = logp.view(B, T) + 0.3 * noise[1] if case["ref"] else None
    if own:
        from paper_2607_05722_amd import runtime as rt
        st["ws"] = rt.LogitsWorkspace(B, T, V, case["n_top"])
    return st


# ------------------------------------------------------------------------------------------ one pass
def run(state):
    if own:
        return _run_own(state)
    return {"top": _plain_top, "distill": _plain_distill, "policy": _plain_policy}[state["case"]["op"]](state)


def _run_own(st):
    from paper_2607_05722_amd import runtime as rt
    c = st["case"]
    if c["op"] == "top":
        o = rt.top_logits(st["logits"], c["n_top"], st["ws"], temperature=c["tau"])
        return [o["values"], o["ids"], o["lse"]]
    if c["op"] == "distill":
        o = rt.distill_from_logits(st["logits"], st["values"], st["ids"], st["ws"], teacher_lse=st["lse"],
                                   temperature=c["tau"], kl_share=c["kl_share"], eta=c["eta"], weight=st["weight"],
                                   want_grad=c["grad"])
        return [o["loss"], o["accept"]] + ([o["grad"]] if c["grad"] else [])
    o = rt.policy_from_logits(st["logits"], st["actions"], st["advantage"], st["ws"], old_logp=st["old_logp"],
                              ref_logp=st["ref_logp"], temperature=c["tau"], clip_low=CLIP_LOW, clip_high=CLIP_HIGH,
                              kl_coef=c["kl_coef"], weight=st["weight"], want_grad=c["grad"])
    return [o["loss"], o["logp"]] + ([o["grad"]] if c["grad"] else [])


def _plain_top(st):
    """Keys that order by value and then by the lower index, so that equal logits tie as they have to."""
    c, z = st["case"], st["logits"].float()
    bits = (z + 0.0).view(torch.int32).long() & 0xFFFFFFFF
    order = torch.where(bits >= 1 << 31, (1 << 32) - 1 - bits, bits + (1 << 31)) - (1 << 31)
    key = order * (1 << 32) + ((1 << 32) - 1 - torch.arange(z.shape[-1], device=z.device))
    top = torch.topk(key, c["n_top"], dim=-1)[0]
    ids = ((1 << 32) - 1 - (top & 0xFFFFFFFF))
    y = z / c["tau"]
    m = y.amax(-1, keepdim=True)
    lse = m[..., 0] + torch.log(torch.exp(y - m).sum(-1))
    return [z.gather(-1, ids), ids.to(torch.int32), lse]


def _plain_distill(st):
    """The vocabulary's exponentials in 32 bits, their sums and everything per teacher entry in 64: the divergences
    are small differences of the entries' logarithms."""
    c, z = st["case"], st["logits"].float()
    w, ids = st["weight"], st["ids"].long()
    in_s = torch.zeros(z.shape, dtype=torch.bool, device=z.device).scatter_(-1, ids, True)
    m = z.amax(-1, keepdim=True)
    e = torch.exp((z - m) / c["tau"])
    y = (z.gather(-1, ids).double() - m.double()) / c["tau"]
    rest = torch.where(in_s, 0.0, e).sum(-1, dtype=torch.float64)
    total = rest + torch.exp(y).sum(-1)
    x = st["values"].double() / c["tau"]
    xm = x.amax(-1, keepdim=True)
    lse = st["lse"].double() if c["tail"] else xm[..., 0] + torch.log(torch.exp(x - xm).sum(-1))
    log_p, log_q = x - lse[..., None], y - torch.log(total)[..., None]
    p, q, q_r = torch.exp(log_p), torch.exp(log_q), rest / total
    p_r = torch.clamp(1.0 - p.sum(-1), min=0.0) if c["tail"] else torch.zeros_like(lse)
    kl = (p * (log_p - log_q)).sum(-1) + torch.where(p_r > 0, p_r * torch.log(p_r / q_r), 0.0)
    tv = 0.5 * ((p - q).abs().sum(-1) + (p_r - q_r).abs())
    accept = torch.minimum(p, q).sum(-1) + torch.minimum(p_r, q_r)
    lam = c["kl_share"] * torch.exp(-c["eta"] * accept)
    counts = w != 0
    out = [torch.where(counts, w * (lam * kl + (1.0 - lam) * tv), 0.0).float(), torch.where(counts, accept, 0.0).float()]
    if c["grad"]:
        s, s_r = torch.sign(q - p), torch.sign(q_r - p_r)
        mean = (s * q).sum(-1) + s_r * q_r
        mass = p.sum(-1) + p_r
        f = torch.where(counts, w / c["tau"], 0.0).double()
        half = 0.5 * (1.0 - lam)
        a_r = f * (lam * mass + half * (s_r - mean) - torch.where(p_r > 0, lam * p_r / q_r, 0.0))
        a_s = (lam * mass - half * mean)[..., None] + half[..., None] * s
        grad = (a_r / total).float()[..., None] * e
        grad.scatter_(-1, ids, (f[..., None] * (q * a_s - lam[..., None] * p)).float())
        out.append(grad.to(st["logits"].dtype))
    return out


def _plain_policy(st):
    c, dt = st["case"], st["logits"].dtype
    w, a, adv = st["weight"], st["actions"].long()[..., None], st["advantage"]
    y = st["logits"].float() / c["tau"]
    m = y.amax(-1, keepdim=True)
    e = torch.exp(y - m)
    total = e.sum(-1)
    logp = (y.gather(-1, a) - m)[..., 0] - torch.log(total)
    rho = torch.exp(logp - st["old_logp"]) if st["old_logp"] is not None else torch.ones_like(logp)
    free, held = rho * adv, torch.clamp(rho, 1.0 - CLIP_LOW, 1.0 + CLIP_HIGH) * adv
    loss = -torch.minimum(free, held)
    g = -torch.where(free <= held, free, 0.0)
    if st["ref_logp"] is not None:
        d = st["ref_logp"] - logp
        loss = loss + c["kl_coef"] * (torch.exp(d) - d - 1.0)
        g = g + c["kl_coef"] * (1.0 - torch.exp(d))
    counts = w != 0
    out = [torch.where(counts, w * loss, 0.0), torch.where(counts, logp, 0.0)]
    if c["grad"]:
        f = torch.where(counts, w * g / c["tau"], 0.0)[..., None]
        grad = e * (-f / total[..., None])
        # 1 - q of the action, from the others' sum
        others = total[..., None] - e.gather(-1, a)
        grad.scatter_(-1, a, f * others / total[..., None])
        out.append(grad.to(dt))
    return out


# ------------------------------------------------------------------------------------------ 64-bit results
def exact(case, seed):
    st = prepare(case, seed)
    z = st["logits"].reshape(-1, case["vocab"])
    n = max(1, (_CHUNK // 2) // case["vocab"])
    rows = {k: st[k].reshape(z.shape[0], *st[k].shape[2:]) for k in
            ("weight", "values", "ids", "lse", "actions", "advantage", "old_logp", "ref_logp") if st.get(k) is not None}
    fn = {"top": _exact_top, "distill": _exact_distill, "policy": _exact_policy}[case["op"]]
    parts = [fn(case, z[r:r + n], {k: v[r:r + n] for k, v in rows.items()}) for r in range(0, z.shape[0], n)]
    return [torch.cat(p).view(case["batch"], case["rows"], *p[0].shape[1:]) for p in zip(*parts)]


def _exact_top(case, z, rows):
    z = z.double()
    v, i = torch.sort(z, dim=-1, descending=True, stable=True)
    K = case["n_top"]
    return v[:, :K], i[:, :K].to(torch.int32), torch.logsumexp(z / case["tau"], -1)


def _finish(case, rows, loss, aux, z):
    """Row losses -> outputs; the gradient is taken by differentiation of the summed loss."""
    keep = rows["weight"] != 0
    loss = torch.where(keep, rows["weight"].double() * loss, 0.0)
    out = [loss.detach(), torch.where(keep, aux, 0.0).detach()]
    if case["grad"]:
        out.append(torch.autograd.grad(loss.sum(), z)[0])
    return out


def _exact_distill(case, z, rows):
    z = z.double().requires_grad_(case["grad"])
    ids = rows["ids"].long()
    logq = torch.log_softmax(z / case["tau"], -1)
    outside = torch.ones(z.shape, dtype=torch.bool, device=z.device).scatter_(-1, ids, False)
    lq = torch.cat([logq.gather(-1, ids), torch.logsumexp(logq.masked_fill(~outside, -torch.inf), -1, keepdim=True)], -1)
    x = rows["values"].double() / case["tau"]
    lp = x - (rows["lse"].double()[:, None] if case["tail"] else torch.logsumexp(x, -1, keepdim=True))
    p = torch.exp(lp)
    r = torch.clamp(1.0 - p.sum(-1, keepdim=True), min=0.0) if case["tail"] else torch.zeros_like(p[:, :1])
    p = torch.cat([p, r], -1)
    if ids.shape[1] == z.shape[1]:      # no token is left for the rest
        p, lq = p[:, :-1], lq[:, :-1]
    q = torch.exp(lq)
    alpha = torch.minimum(p, q).sum(-1).detach()
    lam = case["kl_share"] * torch.exp(-case["eta"] * alpha)
    kl = torch.where(p > 0, p * (torch.log(p) - torch.where(p > 0, lq, 0.0)), 0.0).sum(-1)
    tv = 0.5 * (p - q).abs().sum(-1)
    return _finish(case, rows, lam * kl + (1.0 - lam) * tv, alpha, z)


def _exact_policy(case, z, rows):
    z = z.double().requires_grad_(case["grad"])
    logp = torch.log_softmax(z / case["tau"], -1).gather(-1, rows["actions"].long()[:, None])[:, 0]
    adv = rows["advantage"].double()
    old = rows["old_logp"].double() if case["old"] else logp.detach()
    rho = torch.exp(logp - old)
    loss = -torch.minimum(rho * adv, torch.clamp(rho, 1.0 - CLIP_LOW, 1.0 + CLIP_HIGH) * adv)
    if case["ref"]:
        d = rows["ref_logp"].double() - logp
        loss = loss + case["kl_coef"] * (torch.exp(d) - d - 1.0)
    return _finish(case, rows, loss, logp.detach(), z)
