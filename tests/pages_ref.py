"""Plain 64-bit versions of the calls on a paged cache, from their formulas; torch on any device, no code of the library."""
import math

import torch

PAGE = 64
INF = float("inf")


def stored(x, e4m3):
    """What a page holds of rows [..., head_dim], in 64 bits."""
    if not e4m3:
        return x.to(torch.bfloat16).double()
    x = x.double()
    fin = torch.isfinite(x)
    top = torch.where(fin, x.abs(), 0.0).amax(-1, keepdim=True)
    m, e = torch.frexp(top)
    scale = torch.exp2(torch.where(top > 0, e - 9 + (m > 0.875), -100).clamp(min=-100).double())
    y = torch.where(fin, x, 0.0) / scale
    _, ey = torch.frexp(y)
    step = torch.exp2((ey - 1).clamp(min=-6).double() - 3.0)
    most = 1.875 * 2.0 ** 127        # the next one is not finite in 32 bits
    return torch.where(fin, (torch.round(y / step) * step * scale).clamp(-most, most), math.nan)


def over_127(x):
    """A division: by a plain number torch would multiply by its rounded reciprocal."""
    return x / torch.full_like(x, 127.0)


def bounds(keys, filled):
    """(int8 [2][dim], f32 scale) of a page's stored keys [64][dim], of which the first `filled` count; NaN scale of an inf one."""
    k = keys[:filled].float()
    if not bool(torch.isfinite(k).all()):
        return torch.zeros((2, k.shape[1]), dtype=torch.int8, device=k.device), INF
    lo, hi = k.amin(0), k.amax(0)
    scale = over_127(torch.maximum(lo.abs(), hi.abs()).amax())
    by = scale if float(scale) > 0 else torch.ones((), device=k.device)
    return torch.stack([torch.floor(lo / by), torch.ceil(hi / by)]).clamp(-127, 127).to(torch.int8), float(scale)


class Cache:
    """The stored rows of one layer: k, v [batch][max_len][heads][dim] f64."""

    def __init__(self, batch, max_len, heads, dim, e4m3, device):
        self.k = torch.zeros((batch, max_len, heads, dim), dtype=torch.float64, device=device)
        self.v = torch.zeros_like(self.k)
        self.e4m3, self.max_len = e4m3, max_len

    def write(self, lens, starts, k, v):
        for b, p in enumerate(lens):
            r0, r1 = starts[b], starts[b + 1]
            n = max(0, min(r1 - r0, self.max_len - p))
            self.k[b, p:p + n] = stored(k[r0:r0 + n], self.e4m3)
            self.v[b, p:p + n] = stored(v[r0:r0 + n], self.e4m3)


def sees(p, n, i, draft, bidir_from, cap):
    return min(p + (n if draft and i >= bidir_from else i + 1), cap)


def attend(cache, lens, starts, q, scale, draft=False, bidir_from=0, lists=None, group=1):
    """(out, lse, a, s): out [rows][heads][dim] and lse in 64 bits, a = sum of the weights times |v|, s = the largest sum of
    |q_d k_d| * |scale| that a row meets."""
    R, Hq, D = q.shape
    H = cache.k.shape[2]
    G = Hq // H
    out = torch.zeros((R, Hq, D), dtype=torch.float64, device=q.device)
    a = torch.zeros_like(out)
    lse = torch.full((R, Hq), -INF, dtype=torch.float64, device=q.device)
    s_most = torch.zeros((R, Hq), dtype=torch.float64, device=q.device)
    q = q.double()
    for b, p in enumerate(lens):
        n = starts[b + 1] - starts[b]
        for i in range(n):
            end = sees(p, n, i, draft, bidir_from, cache.max_len)
            r = starts[b] + i
            for h in range(H):
                if lists is None:
                    pos = torch.arange(end, device=q.device)
                else:
                    pages = lists[b, i // group, h]
                    pages = pages[pages >= 0].long()
                    pos = (pages[:, None] * PAGE + torch.arange(PAGE, device=q.device)).reshape(-1)
                    pos = pos[pos < end]
                if len(pos) == 0:
                    continue
                k, v, hs = cache.k[b, pos, h], cache.v[b, pos, h], slice(h * G, (h + 1) * G)
                s = q[r, hs] @ k.T * scale
                w = torch.softmax(s, -1)
                lse[r, hs] = torch.logsumexp(s, -1)
                out[r, hs] = w @ v
                a[r, hs] = w @ v.abs()
                s_most[r, hs] = (q[r, hs].abs() @ k.abs().T * abs(scale)).amax(-1)
    return out, lse, a, s_most


def select(cache, lens, starts, q, n_top, n_first, group, n_list, draft=False, bidir_from=0, filled=None):
    """Lists [batch][groups][heads][n_list]; scores in whole numbers and the f32 products that define them."""
    R, Hq, D = q.shape
    H = cache.k.shape[2]
    G = Hq // H
    most = max(starts[b + 1] - starts[b] for b in range(len(lens)))
    got = torch.full((len(lens), -(-most // group), H, n_list), -1, dtype=torch.int32, device=q.device)
    q = q.float()
    fin = torch.isfinite(q).all(-1)
    qs = over_127(torch.where(fin[..., None], q, 0.0).abs().amax(-1))
    qi = torch.round(torch.where(fin[..., None], q, 0.0) / torch.where(qs > 0, qs, 1.0)[..., None]).clamp(-127, 127).double()
    for b, p in enumerate(lens):
        n = starts[b + 1] - starts[b]
        written = min(p + n, cache.max_len)
        table = {}
        for g in range(-(-n // group)):
            t0, t1 = g * group, min((g + 1) * group, n)
            p0 = min((p + t0) // PAGE, cache.max_len // PAGE)
            end = -(-max(sees(p, n, i, draft, bidir_from, cache.max_len) for i in range(t0, t1)) // PAGE)
            for h in range(H):
                rows = [(starts[b] + i, j) for i in range(t0, t1) for j in range(h * G, (h + 1) * G) if fin[starts[b] + i, j]]
                best = []
                for page in range(n_first, p0):
                    if (page, h) not in table:
                        lo = page * PAGE
                        table[page, h] = bounds(cache.k[b, lo:lo + PAGE, h], min(written - lo, PAGE))
                    bd, bs = table[page, h]
                    score = INF if bs == INF else -INF
                    if rows and bs < INF:
                        x = torch.stack([qi[r, j] for r, j in rows])
                        acc = torch.maximum(x * bd[0].double(), x * bd[1].double()).sum(-1).float()
                        u = (acc * torch.stack([qs[r, j] for r, j in rows])).amax()
                        score = float(u * torch.tensor(bs, dtype=torch.float32, device=q.device))
                    best.append((-score, page))
                take = sorted(page for _, page in sorted(best)[:n_top])
                have = sorted(set(range(min(n_first, p0))) | set(take) | set(range(p0, end)))
                got[b, g, h, :len(have)] = torch.tensor(have, dtype=torch.int32, device=q.device)
    return got


def _bits(x, device):
    return torch.from_numpy(x.view("int16").copy()).to(device).view(torch.bfloat16).double()


def block_pass(shape, source, caches, lens, tokens, draft=False, bidir_from=0, sparse=None):
    """A block pass of the decoder in 64 bits over paged caches (one per layer, written here): pre-norm RMSNorm, rotate-half RoPE, GQA over
    the stored keys and values, SwiGLU, final norm, LM head.  tokens [batch][k].  Returns logits [batch][k][vocab]."""
    dev = caches[0].k.device
    B, k = tokens.shape
    H, Hq, D = shape.n_kv_heads, shape.n_q_heads, shape.head_dim
    starts = [b * k for b in range(B + 1)]
    x = _bits(source.embed, dev)[tokens.reshape(-1).long()]
    pos = (torch.tensor(lens, device=dev)[:, None] + torch.arange(k, device=dev)).reshape(-1).double()
    angle = pos[:, None] * shape.rope_base ** (-2.0 * torch.arange(D // 2, device=dev).double() / D)
    cos, sin = torch.cos(angle)[:, None], torch.sin(angle)[:, None]

    def norm(y, gain):
        return y / torch.sqrt((y * y).mean(-1, keepdim=True) + shape.rms_eps) * _bits(gain, dev)

    def rope(y):
        a, b = y[..., :D // 2], y[..., D // 2:]
        return torch.cat([a * cos - b * sin, b * cos + a * sin], -1)

    for l in range(shape.n_layers):
        w = {n: (v if "norm" in n else _bits(v, dev)) for n, v in source.layer(l).items()}
        y = norm(x, w["attn_norm"])
        q, kk, v = (y @ w[n].T for n in ("wq", "wk", "wv"))
        q, kk = rope(q.view(-1, Hq, D)), rope(kk.view(-1, H, D))
        caches[l].write(lens, starts, kk.float(), v.view(-1, H, D).float())
        lists, group = None, 1
        if sparse is not None:
            n_top, n_first, group = sparse
            n_list = n_first + n_top + ((k if draft else group) + 62) // PAGE + 1
            lists = select(caches[l], lens, starts, q.float(), n_top, n_first, group, n_list, draft, bidir_from)
        o = attend(caches[l], lens, starts, q, D ** -0.5, draft, bidir_from, lists, group)[0]
        x = x + o.reshape(B * k, -1) @ w["wo"].T
        y = norm(x, w["ffn_norm"])
        gate = y @ w["w_gate"].T
        x = x + (gate * torch.sigmoid(gate) * (y @ w["w_up"].T)) @ w["w_down"].T
    return (norm(x, source.final_norm) @ _bits(source.lm_head, dev).T).view(B, k, -1)
