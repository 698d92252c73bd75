"""Python binding of libnld: device buffers (PyTorch-ROCm) + C-ABI calls.

PyTorch only provides device memory and the stream; every step of the
block-decode path runs in libnld's HIP kernels.  Functions here marshal
arguments: they allocate outputs, pass raw pointers and check statuses.
"""
from __future__ import annotations

import ctypes

import numpy as np
import torch
from torch.autograd.graph import increment_version

from . import _lib as C

__all__ = ["DeviceModel", "DeviceCache", "Workspace", "block_forward", "draft", "verify_accept",
           "accept_from_logits", "verify_accept_noalloc", "denoise_step", "refresh_block", "commit_from_logits", "read_device_status",
           "stream_handle", "VERIFY", "DRAFT", "LogitsWorkspace", "top_logits", "distill_from_logits",
           "policy_from_logits", "drafter_loss"]

VERIFY = C.NLD_MODE_VERIFY
DRAFT = C.NLD_MODE_DRAFT


def stream_handle(stream=None) -> int:
    s = stream if stream is not None else torch.cuda.current_stream()
    return s.cuda_stream


# the current stream's handle by device index, without the stream object around it (2.7 us less per call)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda index: torch.cuda.current_stream(index).cuda_stream)


def _bits_to_device(bits: np.ndarray, device) -> torch.Tensor:
    """bf16 bit patterns (uint16, host) -> int16 tensor on the device (bitwise copy)."""
    return torch.from_numpy(np.ascontiguousarray(bits).view(np.int16)).to(device)


def _ptr(t) -> int:
    return 0 if t is None else t.data_ptr()


def make_config(shape) -> C.Config:
    rank = int(getattr(shape, "lora_rank", 0))
    scale = float(shape.lora_alpha) / rank if rank else 0.0
    return C.Config(shape.n_layers, shape.hidden, shape.n_q_heads, shape.n_kv_heads, shape.head_dim, shape.ffn,
                    shape.vocab, float(shape.rope_base), float(shape.rms_eps), int(shape.mask_token_id), rank, scale)


def _pack_lora(lib, shape, rank, device, w, packed, s):
    """Pack one layer's adapter: lora_a [rank][q_dim] and lora_b [hidden][rank] (row-major bits)."""
    qd, h = shape.q_dim, shape.hidden
    a, b = _bits_to_device(w["lora_a"], device), _bits_to_device(w["lora_b"], device)
    la, lb = packed(C.NLD_PACK_LINEAR, rank, qd), packed(C.NLD_PACK_LINEAR, h, rank)
    C.check(lib.nld_pack_linear(_ptr(a), rank, qd, _ptr(la), s))
    C.check(lib.nld_pack_linear(_ptr(b), h, rank, _ptr(lb), s))
    torch.cuda.current_stream().synchronize()
    return la, lb


class DeviceModel:
    """Uploads a model's row-major bf16 weights and packs them with the library's pack kernels.

    ``source`` provides ``layer(l)`` (dict of row-major [out][in] uint16 arrays
    named attn_norm, wq, wk, wv, wo, ffn_norm, w_gate, w_up, w_down),
    ``embed``, ``lm_head`` and ``final_norm``.
    """

    def __init__(self, shape, source, device="cuda"):
        self.lib = C.load()
        self.shape, self.device = shape, torch.device(device)
        self.cfg = make_config(shape)
        s = stream_handle()
        keep = []

        def packed(kind, out_dim, in_dim):
            n = self.lib.nld_packed_bytes(kind, ctypes.byref(self.cfg), out_dim, in_dim)
            assert n > 0
            t = torch.empty(n, dtype=torch.uint8, device=self.device)
            keep.append(t)
            return t

        h, qd, kvd, f = shape.hidden, shape.q_dim, shape.kv_dim, shape.ffn
        layers = (C.LayerWeights * shape.n_layers)()
        for l in range(shape.n_layers):
            w = source.layer(l)
            an, fn = _bits_to_device(w["attn_norm"], self.device), _bits_to_device(w["ffn_norm"], self.device)
            keep += [an, fn]
            wq, wk, wv = (_bits_to_device(w[n], self.device) for n in ("wq", "wk", "wv"))
            qkv = packed(C.NLD_PACK_QKV, qd + 2 * kvd, h)
            C.check(self.lib.nld_pack_qkv(ctypes.byref(self.cfg), _ptr(wq), _ptr(wk), _ptr(wv), _ptr(qkv), s))
            wo = _bits_to_device(w["wo"], self.device)
            o = packed(C.NLD_PACK_LINEAR, h, qd)
            C.check(self.lib.nld_pack_linear(_ptr(wo), h, qd, _ptr(o), s))
            wg, wu = _bits_to_device(w["w_gate"], self.device), _bits_to_device(w["w_up"], self.device)
            gu = packed(C.NLD_PACK_GATE_UP, f, h)
            C.check(self.lib.nld_pack_gate_up(ctypes.byref(self.cfg), _ptr(wg), _ptr(wu), _ptr(gu), s))
            wd = _bits_to_device(w["w_down"], self.device)
            dn = packed(C.NLD_PACK_LINEAR, h, f)
            C.check(self.lib.nld_pack_linear(_ptr(wd), h, f, _ptr(dn), s))
            la = lb = None
            if self.cfg.lora_rank:
                la, lb = self._pack_lora(w, packed, s)
            torch.cuda.current_stream().synchronize()     # row-major sources are freed below
            del wq, wk, wv, wo, wg, wu, wd
            layers[l] = C.LayerWeights(_ptr(an), _ptr(qkv), _ptr(o), _ptr(fn), _ptr(gu), _ptr(dn), _ptr(la), _ptr(lb))
        self.embed = _bits_to_device(source.embed, self.device)
        self.final_norm = _bits_to_device(source.final_norm, self.device)
        lm = _bits_to_device(source.lm_head, self.device)
        self.lm_head = packed(C.NLD_PACK_LINEAR, shape.vocab, h)
        C.check(self.lib.nld_pack_linear(_ptr(lm), shape.vocab, h, _ptr(self.lm_head), s))
        torch.cuda.current_stream().synchronize()
        del lm
        self._keep, self._layers = keep, layers
        self.weights = C.Weights(_ptr(self.embed), _ptr(self.final_norm), _ptr(self.lm_head), layers)
        handle = ctypes.c_void_p()
        C.check(self.lib.nld_model_create(ctypes.byref(self.cfg), ctypes.byref(self.weights), ctypes.byref(handle)))
        self.handle = handle

    def _pack_lora(self, w, packed, s):
        return _pack_lora(self.lib, self.shape, self.cfg.lora_rank, self.device, w, packed, s)

    def with_lora(self, lora_shape, lora_layer):
        """A second handle over these weights with a draft-pathway adapter attached.  lora_shape: this
        model's shape with lora_rank / lora_alpha set; lora_layer(l) -> dict with lora_a, lora_b bits."""
        view = ModelView(self, lora_shape)
        keep = []

        def packed(kind, out_dim, in_dim):
            n = self.lib.nld_packed_bytes(kind, ctypes.byref(view.cfg), out_dim, in_dim)
            t = torch.empty(n, dtype=torch.uint8, device=self.device)
            keep.append(t)
            return t

        s = stream_handle()
        layers = (C.LayerWeights * self.shape.n_layers)()
        for l in range(self.shape.n_layers):
            base = self._layers[l]
            la, lb = _pack_lora(self.lib, lora_shape, view.cfg.lora_rank, self.device, lora_layer(l), packed, s)
            layers[l] = C.LayerWeights(base.attn_norm, base.w_qkv, base.w_o, base.ffn_norm, base.w_gate_up,
                                       base.w_down, _ptr(la), _ptr(lb))
        view.finish(layers, keep)
        return view

    def close(self):
        if getattr(self, "handle", None):
            self.lib.nld_model_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class ModelView:
    """A model handle that borrows a DeviceModel's weights (see DeviceModel.with_lora)."""

    def __init__(self, base: DeviceModel, shape):
        self.base, self.shape, self.device, self.lib = base, shape, base.device, base.lib
        self.cfg = make_config(shape)
        self.handle = None

    def finish(self, layers, keep):
        self._layers, self._keep = layers, keep
        b = self.base
        self.weights = C.Weights(_ptr(b.embed), _ptr(b.final_norm), _ptr(b.lm_head), layers)
        handle = ctypes.c_void_p()
        C.check(self.lib.nld_model_create(ctypes.byref(self.cfg), ctypes.byref(self.weights), ctypes.byref(handle)))
        self.handle = handle

    def close(self):
        if getattr(self, "handle", None):
            self.lib.nld_model_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class DeviceCache:
    """KV cache in the library's layout (see nld_kv_cache in include/nld.h)."""

    def __init__(self, shape, batch: int, max_len: int, device="cuda"):
        assert max_len % 64 == 0
        self.shape, self.batch, self.max_len = shape, batch, max_len
        L, H, D = shape.n_layers, shape.n_kv_heads, shape.head_dim
        dev = torch.device(device)
        self.k = torch.zeros((L, batch, H, max_len, D), dtype=torch.int16, device=dev)
        self.v = torch.zeros((L, batch, H, max_len // 64, D, 64), dtype=torch.int16, device=dev)
        self.lengths = torch.zeros(batch, dtype=torch.int32, device=dev)
        self.struct = C.KVCache(_ptr(self.k), _ptr(self.v), _ptr(self.lengths), batch, max_len)

    def load_prefix(self, layer: int, k_bits: np.ndarray, v_bits: np.ndarray) -> None:
        """Write cached K/V given as [batch][kv_heads][P][head_dim] bf16 bits into positions [0, P)."""
        P = k_bits.shape[2]
        assert P <= self.max_len
        kd = _bits_to_device(k_bits, self.k.device)
        self.k[layer, :, :, :P] = kd
        vd = _bits_to_device(v_bits, self.v.device)
        P64 = (P + 63) // 64 * 64
        vpad = torch.zeros((self.batch, self.shape.n_kv_heads, P64, self.shape.head_dim), dtype=torch.int16,
                           device=self.v.device)
        vpad[:, :, :P] = vd
        tiles = vpad.view(self.batch, self.shape.n_kv_heads, P64 // 64, 64, self.shape.head_dim).transpose(-1, -2)
        self.v[layer, :, :, :P64 // 64] = tiles

    def set_lengths(self, lengths) -> None:
        self.lengths.copy_(torch.as_tensor(np.asarray(lengths, dtype=np.int32)))

    def read_kv(self, layer: int, start: int, stop: int):
        """Host copies of K/V rows [start, stop) as [batch][kv_heads][n][head_dim] bf16 bits (uint16)."""
        k = self.k[layer, :, :, start:stop].cpu().numpy().view(np.uint16)
        vt = self.v[layer].transpose(-1, -2).reshape(self.batch, self.shape.n_kv_heads, self.max_len,
                                                     self.shape.head_dim)
        v = vt[:, :, start:stop].contiguous().cpu().numpy().view(np.uint16)
        return k, v


class Workspace:
    def __init__(self, model: DeviceModel, batch: int, k: int, max_len: int):
        lib = C.load()
        self.nbytes = lib.nld_workspace_bytes(model.handle, batch, k, max_len)
        assert self.nbytes > 0
        self.buf = torch.empty(self.nbytes, dtype=torch.uint8, device=model.device)
        C.check(lib.nld_workspace_init(_ptr(self.buf), self.nbytes, stream_handle()))

    @property
    def ptr(self) -> int:
        return _ptr(self.buf)


class QuadWorkspace(Workspace):
    """Workspace of quadratic self-speculation steps with chain length k (k(k+1) block rows)."""

    def __init__(self, model: DeviceModel, batch: int, k: int, max_len: int):
        lib = C.load()
        self.nbytes = lib.nld_quad_workspace_bytes(model.handle, batch, k, max_len)
        assert self.nbytes > 0
        self.buf = torch.empty(self.nbytes, dtype=torch.uint8, device=model.device)
        C.check(lib.nld_workspace_init(_ptr(self.buf), self.nbytes, stream_handle()))


def block_forward(model, cache, ws, tokens: torch.Tensor, mode: int, bidir_from: int = 0, want_logits=True):
    """One block pass.  tokens: int32 [batch][k] on the device.  Returns (logits or None, argmax)."""
    batch, k = tokens.shape
    dev = model.device
    logits = torch.empty((batch, k, model.shape.vocab), dtype=torch.float32, device=dev) if want_logits else None
    argmax = torch.empty((batch, k), dtype=torch.int32, device=dev)
    C.check(C.load().nld_block_forward(model.handle, ctypes.byref(cache.struct), _ptr(tokens), batch, k, mode,
                                       bidir_from, _ptr(logits), _ptr(argmax), ws.ptr, ws.nbytes, stream_handle()))
    return logits, argmax


def draft(model, cache, ws, anchor: torch.Tensor, k: int, bidir_from: int = 0, want_logits=False, out=None):
    """Diffusion draft over [anchor, mask x (k-1)].  Returns (drafts int32 [batch][k-1], logits or None)."""
    batch = anchor.shape[0]
    dev = model.device
    d = out if out is not None else torch.empty((batch, k - 1), dtype=torch.int32, device=dev)
    logits = torch.empty((batch, k, model.shape.vocab), dtype=torch.float32, device=dev) if want_logits else None
    C.check(C.load().nld_draft(model.handle, ctypes.byref(cache.struct), _ptr(anchor), batch, k, bidir_from, _ptr(d),
                               _ptr(logits), ws.ptr, ws.nbytes, stream_handle()))
    return d, logits


def verify_accept(model, cache, ws, anchor: torch.Tensor, drafts, k: int, want_logits=False, outs=None):
    """AR verify + acceptance.  Returns dict of device tensors (accept_len, committed, next_anchor, logits)."""
    batch = anchor.shape[0]
    dev = model.device
    if outs is None:
        outs = {"accept_len": torch.empty(batch, dtype=torch.int32, device=dev),
                "committed": torch.empty((batch, k), dtype=torch.int32, device=dev),
                "next_anchor": torch.empty(batch, dtype=torch.int32, device=dev)}
    logits = torch.empty((batch, k, model.shape.vocab), dtype=torch.float32, device=dev) if want_logits else None
    C.check(C.load().nld_verify_accept(model.handle, ctypes.byref(cache.struct), _ptr(anchor), _ptr(drafts), batch, k,
                                       _ptr(outs["accept_len"]), _ptr(outs["committed"]), _ptr(outs["next_anchor"]),
                                       _ptr(logits), ws.ptr, ws.nbytes, stream_handle()))
    outs = dict(outs)
    outs["logits"] = logits
    return outs


def verify_accept_noalloc(model, cache, anchor: torch.Tensor, drafts, k: int, want_logits=False, outs=None,
                          device_status=None):
    """verify_accept without a workspace: the library's static per-device scratch array stands in for it.
    ``device_status`` (optional int32 device tensor of one element) receives the call's status bits."""
    batch = anchor.shape[0]
    dev = model.device
    if outs is None:
        outs = {"accept_len": torch.empty(batch, dtype=torch.int32, device=dev),
                "committed": torch.empty((batch, k), dtype=torch.int32, device=dev),
                "next_anchor": torch.empty(batch, dtype=torch.int32, device=dev)}
    logits = torch.empty((batch, k, model.shape.vocab), dtype=torch.float32, device=dev) if want_logits else None
    C.check(C.load().nld_verify_accept_noalloc(model.handle, ctypes.byref(cache.struct), _ptr(anchor), _ptr(drafts),
                                               batch, k, _ptr(outs["accept_len"]), _ptr(outs["committed"]),
                                               _ptr(outs["next_anchor"]), _ptr(logits), _ptr(device_status),
                                               stream_handle()))
    outs = dict(outs)
    outs["logits"] = logits
    return outs


def accept_from_logits(logits: torch.Tensor, drafts, device="cuda"):
    """Argmax + acceptance from given f32 logits [batch][k][vocab] and int32 drafts [batch][k-1]."""
    lib = C.load()
    batch, k, vocab = logits.shape
    n = lib.nld_accept_workspace_bytes(batch, k)
    ws = torch.zeros(n, dtype=torch.uint8, device=device)
    out = {"argmax": torch.empty((batch, k), dtype=torch.int32, device=device),
           "accept_len": torch.empty(batch, dtype=torch.int32, device=device),
           "committed": torch.empty((batch, k), dtype=torch.int32, device=device),
           "next_anchor": torch.empty(batch, dtype=torch.int32, device=device)}
    C.check(lib.nld_accept_from_logits(_ptr(logits), _ptr(drafts), batch, k, vocab, _ptr(out["argmax"]),
                                       _ptr(out["accept_len"]), _ptr(out["committed"]), _ptr(out["next_anchor"]),
                                       _ptr(ws), n, stream_handle()))
    return out


def denoise_step(model, cache, ws, block: torch.Tensor, threshold: float, bidir_from: int = 0, want_logits=False,
                 outs=None):
    """One Mode 2 denoising step; ``block`` (int32 [batch][k], device) is updated in place.
    Returns dict of device tensors: n_committed, n_masked, confidence [batch][k], logits (or None)."""
    batch, k = block.shape
    dev = model.device
    if outs is None:
        outs = {"n_committed": torch.empty(batch, dtype=torch.int32, device=dev),
                "n_masked": torch.empty(batch, dtype=torch.int32, device=dev),
                "confidence": torch.empty((batch, k), dtype=torch.float32, device=dev)}
    logits = torch.empty((batch, k, model.shape.vocab), dtype=torch.float32, device=dev) if want_logits else None
    C.check(C.load().nld_denoise_step(model.handle, ctypes.byref(cache.struct), _ptr(block), batch, k, bidir_from,
                                      float(threshold), _ptr(outs["n_committed"]), _ptr(outs["n_masked"]),
                                      _ptr(outs.get("confidence")), _ptr(logits), ws.ptr, ws.nbytes, stream_handle()))
    outs = dict(outs)
    outs["logits"] = logits
    return outs


def refresh_block(model, cache, ws, block: torch.Tensor, next_anchor=None):
    """Causal K/V refresh of completed blocks (commits k-1 rows).  Returns next_anchor (int32 [batch])."""
    batch, k = block.shape
    nxt = next_anchor if next_anchor is not None else torch.empty(batch, dtype=torch.int32, device=model.device)
    C.check(C.load().nld_refresh_block(model.handle, ctypes.byref(cache.struct), _ptr(block), batch, k, _ptr(nxt),
                                       ws.ptr, ws.nbytes, stream_handle()))
    return nxt


def commit_from_logits(logits: torch.Tensor, block: torch.Tensor, mask_token_id: int, threshold: float):
    """The denoising commit from given f32 logits [batch][k][vocab]; ``block`` is updated in place."""
    batch, k, vocab = logits.shape
    dev = logits.device
    out = {"argmax": torch.empty((batch, k), dtype=torch.int32, device=dev),
           "n_committed": torch.empty(batch, dtype=torch.int32, device=dev),
           "n_masked": torch.empty(batch, dtype=torch.int32, device=dev),
           "confidence": torch.empty((batch, k), dtype=torch.float32, device=dev)}
    C.check(C.load().nld_commit_from_logits(_ptr(logits), _ptr(block), batch, k, vocab, mask_token_id,
                                            float(threshold), _ptr(out["argmax"]), _ptr(out["n_committed"]),
                                            _ptr(out["n_masked"]), _ptr(out["confidence"]), stream_handle()))
    return out


def decode_steps(model, cache, ws, anchor: torch.Tensor, k: int, n_steps: int, bidir_from: int = 0, outs=None):
    """n_steps decoding steps on the device (self-speculation for k >= 2, AR for k = 1); ``anchor`` is
    updated in place.  Returns dict: accept_len [n_steps][batch], committed [n_steps][batch][k]."""
    batch = anchor.shape[0]
    dev = model.device
    if outs is None:
        outs = {"accept_len": torch.empty((n_steps, batch), dtype=torch.int32, device=dev),
                "committed": torch.empty((n_steps, batch, k), dtype=torch.int32, device=dev)}
    C.check(C.load().nld_decode_steps(model.handle, ctypes.byref(cache.struct), _ptr(anchor), batch, k, n_steps,
                                      bidir_from, _ptr(outs["accept_len"]), _ptr(outs["committed"]), ws.ptr,
                                      ws.nbytes, stream_handle()))
    return outs


def quad_step(model, cache, ws, anchor: torch.Tensor, spec: torch.Tensor, k: int, lam: float = 1.0,
              want_logits=False, outs=None):
    """One quadratic self-speculation step over [anchor, spec] and k groups of k masks.  Returns dict of
    device tensors: accept_len, committed [batch][k], next_anchor, next_spec [batch][k-1], logits or None
    ([batch][k(k+1)][vocab]).  ``outs`` may pass next_anchor=anchor and next_spec=spec to update in place."""
    batch = anchor.shape[0]
    dev = model.device
    o = dict(outs or {})
    o.setdefault("accept_len", torch.empty(batch, dtype=torch.int32, device=dev))
    o.setdefault("committed", torch.empty((batch, k), dtype=torch.int32, device=dev))
    o.setdefault("next_anchor", torch.empty(batch, dtype=torch.int32, device=dev))
    o.setdefault("next_spec", torch.empty((batch, k - 1), dtype=torch.int32, device=dev))
    logits = torch.empty((batch, k * (k + 1), model.shape.vocab), dtype=torch.float32, device=dev) \
        if want_logits else None
    C.check(C.load().nld_quad_step(model.handle, ctypes.byref(cache.struct), _ptr(anchor), _ptr(spec), batch, k,
                                   float(lam), _ptr(o["accept_len"]), _ptr(o["committed"]), _ptr(o["next_anchor"]),
                                   _ptr(o["next_spec"]), _ptr(logits), ws.ptr, ws.nbytes, stream_handle()))
    o["logits"] = logits
    return o


class LogitsWorkspace:
    """Workspace of the operators on rows of logits (top_logits, distill_from_logits, policy_from_logits) for up to
    batch x rows rows of vocab columns and n_top entries per row."""

    def __init__(self, batch: int, rows: int, vocab: int, n_top: int = 1, device="cuda"):
        lib = C.load()
        dev = torch.device(device)
        with torch.cuda.device(dev):
            self.nbytes = lib.nld_logits_workspace_bytes(batch, rows, vocab, n_top)
            if self.nbytes == 0:
                raise ValueError("no logits workspace for batch %d, rows %d, vocab %d, n_top %d" % (batch, rows, vocab, n_top))
            self.buf = torch.empty(self.nbytes, dtype=torch.uint8, device=dev)
            C.check(lib.nld_workspace_init(_ptr(self.buf), self.nbytes, stream_handle()))

        self.ptr = _ptr(self.buf)


_INT32_MAX = 2 ** 31 - 1   # a descriptor's field keeps the lower half of a larger number, without an error
_DTYPES = {torch.float32: C.NLD_F32, torch.bfloat16: C.NLD_BF16}


def _logits(t: torch.Tensor, name: str) -> C.Logits:
    """Descriptor of logits [batch][rows][vocab], f32 or bf16, columns adjacent, other strides free."""
    dtype = _DTYPES.get(t.dtype)
    if dtype is None or t.dim() != 3 or not t.is_cuda:
        raise ValueError("%s must be a float32 or bfloat16 device tensor [batch][rows][vocab]" % name)
    (batch, rows, vocab), (seq, row, col) = t.shape, t.stride()
    if col != 1 and vocab > 1:
        raise ValueError("%s: the columns of a row must be adjacent" % name)
    if (batch | rows | vocab) > _INT32_MAX:
        raise ValueError("%s: sizes must be int32" % name)
    return C.Logits(t.data_ptr(), dtype, batch, rows, vocab, seq, row)


def _rows_of(t, name: str, shape, dtype, device):
    """The address of a contiguous per-row argument on the logits' device (None: 0)."""
    if t is None:
        return 0
    if t.shape != shape or t.dtype != dtype or not t.is_contiguous() or t.device != device:
        raise ValueError("%s must be a contiguous %s tensor %s on %s" % (name, dtype, list(shape), device))
    return t.data_ptr()


def _out(outs, name: str, shape, dtype, device, like=None):
    """The caller's output tensor of this name, or a new one.  like: a tensor of this type on this device (0.4 us less than
    naming both)."""
    t = outs.get(name) if outs is not None else None
    if t is None:
        return torch.empty(shape, dtype=dtype, device=device) if like is None else like.new_empty(*shape)
    _rows_of(t, name, shape, dtype, device)
    return t


def _seq_rows(t, shape, width):
    """Rows from a sequence to the next, where the rows of one lie one behind the other; else None."""
    B, T = shape
    if t.is_contiguous():
        return T
    st = t.stride()
    ok = (width == 1 or t.dim() == 2 or st[2] == 1) and (T == 1 or st[1] == width)
    if B == 1:
        return T if ok else None
    return st[0] // width if ok and st[0] % width == 0 and st[0] >= T * width else None


def _entries(values, ids, lse, shape, device) -> C.Teacher:
    """Descriptor of a teacher's entries [batch][rows][n_top]; a leading slice [:, :rows] of longer arrays will do."""
    B, T = shape
    n = values.shape[-1]
    full = (B, T, n)
    if values.shape != full or ids.shape != full or (lse is not None and lse.shape != shape) or n < 1:
        raise ValueError("teacher: values and ids must be [batch][rows][n_top] and lse [batch][rows] for the logits' rows")
    if values.dtype != torch.float32 or ids.dtype != torch.int32 or values.device != device or ids.device != device or \
            (lse is not None and (lse.dtype != torch.float32 or lse.device != device)):
        raise ValueError("teacher: values must be float32, ids int32 and lse float32, on %s" % device)

    rows = T
    if not (values.is_contiguous() and ids.is_contiguous() and (lse is None or lse.is_contiguous())):
        rows = _seq_rows(values, shape, n)
        if rows is None or _seq_rows(ids, shape, n) != rows or (lse is not None and _seq_rows(lse, shape, 1) != rows):
            raise ValueError("teacher: values, ids and lse must be whole arrays or the same leading rows of such")
    if n > _INT32_MAX or rows > _INT32_MAX:
        raise ValueError("teacher: sizes must be int32")
    return C.Teacher(values.data_ptr(), ids.data_ptr(), 0 if lse is None else lse.data_ptr(), n, rows)


def _grad_for(logits, desc, want_grad, grad):
    """The gradient's tensor (the caller's, a new contiguous one, or None) and its descriptor."""
    if grad is None:
        if not want_grad:
            return None, None
        grad = logits.new_empty(desc.batch, desc.rows, desc.vocab)
        return grad, C.Logits(grad.data_ptr(), desc.dtype, desc.batch, desc.rows, desc.vocab, desc.rows * desc.vocab, desc.vocab)
    if grad.device != logits.device:
        raise ValueError("grad must be on %s" % logits.device)
    return grad, _logits(grad, "grad")


def _written(outs, names, grad=None):
    """Tells autograd that the caller's tensors were written, as torch's own operations in place do: what kept one of them
    for its backward pass raises there."""
    if outs is not None:
        increment_version([outs[n] for n in names if outs.get(n) is not None])
    if grad is not None:
        increment_version(grad)


def _call(fn, device, ws, *args):
    """fn(*args, workspace, its size, stream) on `device` and its current stream."""
    if ws.buf.device != device:
        raise ValueError("the workspace is on %s, the logits on %s" % (ws.buf.device, device))
    if device.index != torch.cuda.current_device():
        with torch.cuda.device(device):
            C.check(fn(*args, ws.ptr, ws.nbytes, stream_handle()))
        return
    status = fn(*args, ws.ptr, ws.nbytes, _raw_stream(device.index))
    if status != C.NLD_OK:
        C.check(status)


def top_logits(logits: torch.Tensor, n_top: int, ws: LogitsWorkspace, temperature: float = 1.0, outs=None):
    """The n_top largest logits of every row of logits [batch][rows][vocab] (f32 or bf16), largest first, the lower
    column first among equal ones.  Returns dict: values f32 and ids int32 [batch][rows][n_top], lse f32
    [batch][rows] (log-sum-exp of logits / temperature over the whole row).  No gradient flows through them."""
    desc = _logits(logits, "logits")
    if not 0 <= n_top <= _INT32_MAX:
        raise ValueError("n_top must be in [1, vocab] (got %d)" % n_top)
    dev, rows = logits.device, (desc.batch, desc.rows)
    values = _out(outs, "values", rows + (n_top,), torch.float32, dev)
    ids = _out(outs, "ids", rows + (n_top,), torch.int32, dev)
    lse = _out(outs, "lse", rows, torch.float32, dev, values)
    _call(C.load().nld_top_logits, dev, ws, desc, n_top, temperature, values.data_ptr(), ids.data_ptr(), lse.data_ptr())
    _written(outs, ("values", "ids", "lse"))
    return {"values": values, "ids": ids, "lse": lse}


def distill_from_logits(logits: torch.Tensor, values: torch.Tensor, ids: torch.Tensor, ws: LogitsWorkspace,
                        teacher_lse=None, temperature: float = 1.0, kl_share: float = 1.0, eta: float = 0.5, weight=None,
                        last_row=None, want_grad: bool = True, grad=None, outs=None):
    """Distillation loss of the student's logits [batch][rows][vocab] from a teacher's top logits (values, ids and,
    over the teacher's whole row, teacher_lse: what top_logits returns), with its gradient in the same call.  See
    nld_distill_from_logits in include/nld.h for the formula.  Returns dict: loss and accept f32 [batch][rows], grad
    (the gradient of loss.sum() by the logits, in their dtype; ``grad=logits`` puts it in their place; None without).
    The loss hangs on no autograd graph: a trainer goes on with ``logits.backward(grad)``.  ``grad=logits`` is a change in place
    of them, so an operation that kept them for its own backward pass (tanh, softmax) raises there; give such logits a
    gradient of its own."""
    desc = _logits(logits, "logits")
    dev, rows = logits.device, (desc.batch, desc.rows)
    teacher = _entries(values, ids, teacher_lse, rows, dev)
    w = _rows_of(weight, "weight", rows, torch.float32, dev)
    last = _rows_of(last_row, "last_row", rows[:1], torch.int32, dev)
    loss = _out(outs, "loss", rows, torch.float32, dev, values)
    accept = _out(outs, "accept", rows, torch.float32, dev, values)
    given = grad
    grad, grad_desc = _grad_for(logits, desc, want_grad, grad)
    _call(C.load().nld_distill_from_logits, dev, ws, desc, teacher, temperature, kl_share, eta, w, last, loss.data_ptr(),
          accept.data_ptr(), grad_desc)
    _written(outs, ("loss", "accept"), given)
    return {"loss": loss, "accept": accept, "grad": grad}


def policy_from_logits(logits: torch.Tensor, actions: torch.Tensor, advantage: torch.Tensor, ws: LogitsWorkspace,
                       old_logp=None, ref_logp=None, temperature: float = 1.0, clip_low: float = 0.2,
                       clip_high: float = 0.2, kl_coef: float = 0.0, weight=None, last_row=None, want_grad: bool = True,
                       grad=None, outs=None):
    """Clipped policy loss of the tokens ``actions`` (int32 [batch][rows], -1: none) under logits [batch][rows][vocab],
    with its gradient in the same call.  See nld_policy_from_logits in include/nld.h for the formula.  Returns dict:
    loss and logp f32 [batch][rows], grad (as distill_from_logits, also as to autograd)."""
    desc = _logits(logits, "logits")
    dev, rows, f32 = logits.device, (desc.batch, desc.rows), torch.float32
    if actions is None or advantage is None:
        raise ValueError("actions and advantage are needed")
    rollout = C.Rollout(_rows_of(actions, "actions", rows, torch.int32, dev), _rows_of(advantage, "advantage", rows, f32, dev),
                        _rows_of(old_logp, "old_logp", rows, f32, dev), _rows_of(ref_logp, "ref_logp", rows, f32, dev))
    w = _rows_of(weight, "weight", rows, f32, dev)
    last = _rows_of(last_row, "last_row", rows[:1], torch.int32, dev)
    loss = _out(outs, "loss", rows, f32, dev, advantage)
    logp = _out(outs, "logp", rows, f32, dev, advantage)
    given = grad
    grad, grad_desc = _grad_for(logits, desc, want_grad, grad)
    _call(C.load().nld_policy_from_logits, dev, ws, desc, rollout, temperature, clip_low, clip_high, kl_coef, w, last,
          loss.data_ptr(), logp.data_ptr(), grad_desc)
    _written(outs, ("loss", "logp"), given)
    return {"loss": loss, "logp": logp, "grad": grad}


def _check_drafter_loss(model, logits_ws, anchor, k, n_top, temperature, kl_share, eta, weight):
    """What the loss would refuse after the verify pass has committed."""
    batch, vocab, dev = anchor.shape[0], model.shape.vocab, anchor.device
    if k < 2:
        raise ValueError("k must be at least 2: row 0 is the anchor's")
    need = C.load().nld_logits_workspace_bytes(batch, k - 1, vocab, n_top)
    if need == 0:
        raise ValueError("no loss for batch %d, k %d, vocab %d, n_top %d" % (batch, k, vocab, n_top))
    if need > logits_ws.nbytes:
        raise ValueError("the logits workspace holds %d bytes, these sizes need %d" % (logits_ws.nbytes, need))
    if logits_ws.buf.device != dev:
        raise ValueError("the logits workspace is on %s, the anchors on %s" % (logits_ws.buf.device, dev))
    eta32 = ctypes.c_float(eta).value   # as the call gets it
    if not 1e-3 <= np.float32(temperature) <= np.float32(1e3) or not 0.0 <= kl_share <= 1.0 or not 0.0 <= eta32 < float("inf"):
        raise ValueError("temperature must be in [1e-3, 1e3], kl_share in [0, 1], eta >= 0 and finite")
    _rows_of(weight, "weight", (batch, k - 1), torch.float32, dev)


def drafter_loss(model, cache, ws, logits_ws: LogitsWorkspace, anchor: torch.Tensor, k: int, n_top: int = 200,
                 temperature: float = 3.0, kl_share: float = 1.0, eta: float = 0.5, bidir_from: int = 0, weight=None,
                 want_grad: bool = True):
    """A self-speculation step that also gives the drafter's training loss (Sec. 3.3): the draft pass, the verify pass
    with acceptance and commit, and the distillation of draft rows 1..k-1 from the verify rows that predict the same
    positions (verify row j-1 for draft row j), over the accepted drafts and the first rejected one.  ``weight``
    (optional, f32 [batch][k-1]) weighs the rows.  Returns the dict of verify_accept with loss and accept f32
    [batch][k-1], draft_logits [batch][k][vocab] and drafts added; with ``want_grad`` also grad [batch][k-1][vocab],
    the gradient of loss.sum() by draft_logits[:, 1:].  Arguments are checked before the passes: a call that raises
    ValueError has not moved the cache."""
    _check_drafter_loss(model, logits_ws, anchor, k, n_top, temperature, kl_share, eta, weight)
    drafts, draft_logits = draft(model, cache, ws, anchor, k, bidir_from, want_logits=True)
    out = verify_accept(model, cache, ws, anchor, drafts, k, want_logits=True)
    top = top_logits(out["logits"][:, :k - 1], n_top, logits_ws, temperature)
    o = distill_from_logits(draft_logits[:, 1:], top["values"], top["ids"], logits_ws, teacher_lse=top["lse"],
                            temperature=temperature, kl_share=kl_share, eta=eta, weight=weight,
                            last_row=out["accept_len"], want_grad=want_grad)
    out.update(o, drafts=drafts, draft_logits=draft_logits)
    return out


def choose_block(ar_step_ms: float, ss_step_ms: float, expected_committed: float, k_ss: int) -> int:
    return int(C.load().nld_choose_block(ar_step_ms, ss_step_ms, expected_committed, k_ss))


def read_device_status(ws) -> int:
    bits = ctypes.c_uint32(0)
    st = C.load().nld_read_device_status(ws.ptr, ctypes.byref(bits), stream_handle())
    if st not in (C.NLD_OK, C.NLD_ERR_DEVICE):
        C.check(st)
    return int(bits.value)
