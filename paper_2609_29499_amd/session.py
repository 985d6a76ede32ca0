"""Device-memory plumbing around the C ABI: PyTorch tensors own the INT8 store, the plan
workspace, activations and the KV cache; this module only builds the ABI structs from them and
forwards calls. No arithmetic of the decode path happens here.
"""
from __future__ import annotations

import ctypes as C
import struct
from typing import NamedTuple, Optional

import numpy as np
import torch

from . import binding as B  # noqa: F401  (re-exported for callers)

WEIGHT_NAMES = ("wq", "wk", "wv", "wo", "wg", "wu", "wd")


def model_desc(n_layers, d_model, n_q_heads, n_kv_heads, head_dim, d_ffn, vocab=0, max_batch=1,
               max_seq=4096, max_prefill=0, rms_eps=1e-5, rope_theta=500000.0):
    return B.tasp_model_desc(n_layers, d_model, n_q_heads, n_kv_heads, head_dim, d_ffn, vocab,
                             max_batch, max_seq, max_prefill, rms_eps, 0.0, rope_theta)


def desc_from_shape(sh, max_batch=1, max_seq=4096, max_prefill=0):
    """``sh`` is any object with the Shape fields (n_layers, d_model, ...)."""
    return model_desc(sh.n_layers, sh.d_model, sh.n_q_heads, sh.n_kv_heads, sh.head_dim, sh.d_ffn,
                      sh.vocab, max_batch, max_seq, max_prefill, sh.rms_eps, sh.rope_theta)


def current_stream():
    return C.c_void_p(torch.cuda.current_stream().cuda_stream)


def _dev(a, device):
    t = torch.from_numpy(np.ascontiguousarray(a))
    return t.to(device)


class DeviceStore:
    """The INT8 store on the device. ``layers`` is a list of dicts ``name: (int8 [out][in],
    float32 [out])`` plus ``attn_norm`` / ``ffn_norm`` BF16 bits (uint16 [d]); a layer may also be
    given directly as device tensors with the same keys."""

    def __init__(self, layers, final_norm=None, lm_head=None, device="cuda"):
        self.tensors = []
        arr = (B.tasp_layer * len(layers))()
        for i, lay in enumerate(layers):
            keep = {}
            for n in WEIGHT_NAMES:
                w, s = lay[n]
                w = w if torch.is_tensor(w) else _dev(w, device)
                s = s if torch.is_tensor(s) else _dev(s, device)
                keep[n] = (w, s)
                setattr(arr[i], n, B.tasp_qmat(w.data_ptr(), s.data_ptr()))
            for n in ("attn_norm", "ffn_norm"):
                g = lay[n] if torch.is_tensor(lay[n]) else _dev(lay[n], device)
                keep[n] = g
                setattr(arr[i], n, g.data_ptr())
            self.tensors.append(keep)
        self.final_norm = None if final_norm is None else (
            final_norm if torch.is_tensor(final_norm) else _dev(final_norm, device))
        self.lm_head = None if lm_head is None else (
            lm_head if torch.is_tensor(lm_head) else _dev(lm_head, device))
        self._layers = arr
        self.struct = B.tasp_store(arr, self.final_norm.data_ptr() if self.final_norm is not None else None,
                                   self.lm_head.data_ptr() if self.lm_head is not None else None)


class GroupStore:
    """The packed groupwise store on the device. ``layers`` is a list of dicts ``name: (int8
    [out][in], BF16 scale bits uint16 [out][in / 128])`` for wq, wk, wv, wo, wg, wu, wd plus the
    two gains; wq, wk and wv are stacked into the store's QKV matrix (layout only). A layer may
    also be given as device tensors with the same keys (scale bits as int16)."""

    def __init__(self, layers, final_norm=None, lm_head=None, device="cuda"):
        self.tensors = []
        arr = (B.tasp_glayer * len(layers))()
        for i, lay in enumerate(layers):
            keep = {}
            on_dev = torch.is_tensor(lay["wq"][0])
            cat = torch.cat if on_dev else np.concatenate
            qkv = (cat([lay["wq"][0], lay["wk"][0], lay["wv"][0]]),
                   cat([lay["wq"][1], lay["wk"][1], lay["wv"][1]]))
            for n, (w, sc) in (("wqkv", qkv), ("wo", lay["wo"]), ("wg", lay["wg"]),
                               ("wu", lay["wu"]), ("wd", lay["wd"])):
                if on_dev:
                    w, sc = w.contiguous(), sc.contiguous().view(torch.int16)
                else:
                    w, sc = _dev(w, device), _dev(np.ascontiguousarray(sc, np.uint16).view(np.int16), device)
                keep[n] = (w, sc)
                setattr(arr[i], n, B.tasp_gqmat(w.data_ptr(), sc.data_ptr()))
            for n in ("attn_norm", "ffn_norm"):
                g = lay[n] if torch.is_tensor(lay[n]) else _dev(lay[n], device)
                keep[n] = g
                setattr(arr[i], n, g.data_ptr())
            self.tensors.append(keep)
        self.final_norm = None if final_norm is None else (
            final_norm if torch.is_tensor(final_norm) else _dev(final_norm, device))
        self.lm_head = None if lm_head is None else (
            lm_head if torch.is_tensor(lm_head) else _dev(lm_head, device))
        self._layers = arr
        self.struct = B.tasp_gstore(arr, self.final_norm.data_ptr() if self.final_norm is not None else None,
                                    self.lm_head.data_ptr() if self.lm_head is not None else None)

    def nbytes(self):
        n = sum(t.numel() * t.element_size() for lay in self.tensors for v in lay.values()
                for t in (v if isinstance(v, tuple) else (v,)))
        for t in (self.final_norm, self.lm_head):
            if t is not None:
                n += t.numel() * t.element_size()
        return n


def mask_struct(mask):
    """(q_keep, kv_keep or None, ffn_keep) uint8 numpy arrays -> (tasp_mask, keepalive)."""
    if mask is None:
        return None, None
    q, kv, f = (None if a is None else np.ascontiguousarray(a, dtype=np.uint8) for a in mask)
    m = B.tasp_mask(q.ctypes.data, None if kv is None else kv.ctypes.data, f.ctypes.data)
    return C.pointer(m), (q, kv, f, m)


class KVCache:
    """BF16 K and V ``[L][B][Hkv][S][dh]`` owned by torch."""

    def __init__(self, desc, batch, max_seq, device="cuda", fill=0.0):
        shp = (desc.n_layers, batch, desc.n_kv_heads, max_seq, desc.head_dim)
        self.k = torch.full(shp, fill, dtype=torch.bfloat16, device=device)
        self.v = torch.full(shp, fill, dtype=torch.bfloat16, device=device)
        self.struct = B.tasp_kv_cache(self.k.data_ptr(), self.v.data_ptr(), batch, max_seq, 0)

    def load_layer(self, layer, k_bits, v_bits):
        """Copy BF16 bit patterns ``uint16 [B][Hkv][S][dh]`` into one layer."""
        self.k[layer].copy_(torch.from_numpy(np.ascontiguousarray(k_bits)).view(torch.bfloat16))
        self.v[layer].copy_(torch.from_numpy(np.ascontiguousarray(v_bits)).view(torch.bfloat16))

    def bits(self, which, layer):
        t = self.k if which == "k" else self.v
        return t[layer].view(torch.int16).cpu().numpy().view(np.uint16)


class SharedScratch:
    """Decode / prefill scratch arena that several shared-store plans of one desc may share
    (their calls must then run in order, e.g. on one stream)."""

    def __init__(self, desc, device="cuda"):
        self.bytes = B.tasp_shared_plan_workspace_bytes(desc)[1]
        self.buf = torch.empty(self.bytes + 256, dtype=torch.uint8, device=device)
        self.base = self.buf.data_ptr() + (-self.buf.data_ptr()) % 256


class Plan:
    """A compiled plan with its torch-owned workspace."""

    def __init__(self, desc, store, mask=None, stream=None, device="cuda"):
        self.desc = desc
        self.store = store
        mptr, self._mask_keep = mask_struct(mask)
        self.ws_bytes = B.tasp_plan_workspace_bytes(desc, mptr)
        self.ws = torch.empty(self.ws_bytes + 256, dtype=torch.uint8, device=device)
        off = (-self.ws.data_ptr()) % 256
        self.ws_base = self.ws.data_ptr() + off
        self.ws_off = off
        self.handle = B.tasp_compile_plan(desc, store.struct, mptr, self.ws_base, self.ws_bytes,
                                          stream if stream is not None else current_stream())

    def __del__(self):
        h = getattr(self, "handle", None)
        if h:
            try:
                B.tasp_plan_destroy(h)
            except Exception:
                pass
            self.handle = None

    @classmethod
    def shared(cls, desc, gstore, mask=None, stream=None, device="cuda", scratch=None):
        """A plan over the shared groupwise store (no weight copies). ``scratch``: a
        SharedScratch to share with other plans (else the plan gets its own)."""
        self = cls.__new__(cls)
        self.desc = desc
        self.store = gstore
        mptr, self._mask_keep = mask_struct(mask)
        self.ws_bytes = B.tasp_shared_plan_workspace_bytes(desc)[0]
        self.ws = torch.empty(self.ws_bytes + 256, dtype=torch.uint8, device=device)
        off = (-self.ws.data_ptr()) % 256
        self.ws_base = self.ws.data_ptr() + off
        self.ws_off = off
        self.scratch = scratch if scratch is not None else SharedScratch(desc, device)
        self.handle = B.tasp_compile_shared_plan(desc, gstore.struct, mptr, self.ws_base,
                                                 self.ws_bytes, self.scratch.base, self.scratch.bytes,
                                                 stream if stream is not None else current_stream())
        return self

    def counts(self, layer):
        return B.tasp_plan_counts(self.handle, layer)

    def indices(self, layer, which):
        return B.tasp_plan_indices(self.handle, layer, which)

    def ledger(self):
        ratio, wb, sb, sig = B.tasp_plan_ledger(self.handle)
        return {"active_flop_ratio": ratio, "weight_bytes": wb, "scale_bytes": sb, "signature": sig}

    def _view(self, ptr, nbytes, dtype):
        start = ptr - self.ws.data_ptr()
        return self.ws[start:start + nbytes].view(dtype)

    def panel(self, layer, which):
        """(int8 rows [rows][ld], float32 scales [rows]) as views into the workspace."""
        w, s, rows, cols, ld = B.tasp_plan_panel(self.handle, layer, which)
        if rows * ld == 0:
            return torch.empty((rows, ld), dtype=torch.int8), torch.empty(rows), cols
        wt = self._view(w, rows * ld, torch.int8).view(rows, ld)
        st = self._view(s, rows * 4, torch.float32)
        return wt, st, cols

    def bind(self, cache):
        B.tasp_kv_bind(self.handle, cache.struct)

    def decode(self, x, cache, pos, out, stream=None):
        B.tasp_decode_step(self.handle, x.data_ptr(), cache.struct, pos, out.data_ptr(),
                           stream if stream is not None else current_stream())

    def decode_timed(self, x, cache, pos, out, stream=None):
        return B.tasp_decode_step_timed(self.handle, x.data_ptr(), cache.struct, pos, out.data_ptr(),
                                        stream if stream is not None else current_stream())

    def prefill(self, x, T, cache, pos0, out, stream=None):
        B.tasp_prefill(self.handle, x.data_ptr(), T, cache.struct, pos0, out.data_ptr(),
                       stream if stream is not None else current_stream())

    def prefill_last(self, x, T, cache, pos0, out, stream=None):
        """The prefill with the last token's logits only: out is float32 [vocab]."""
        B.tasp_prefill_last(self.handle, x.data_ptr(), T, cache.struct, pos0, out.data_ptr(),
                            stream if stream is not None else current_stream())

    def generate(self, embed, embed_scale, prompt, n_new, cache, stream=None, scratch=None):
        """Prompt ids (device int32 [T]) -> n_new + 1 greedy ids (device int32). ``scratch`` may
        pass (x [T][d], logits [T][vocab]) float32 device tensors to reuse."""
        T = int(prompt.numel())
        dev = prompt.device
        if scratch is None:
            scratch = (torch.empty((T, self.desc.d_model), device=dev),
                       torch.empty((T, self.desc.vocab), device=dev))
        out = torch.empty(n_new + 1, dtype=torch.int32, device=dev)
        B.tasp_generate(self.handle, embed.data_ptr(), embed_scale.data_ptr(), prompt.data_ptr(), T,
                        n_new, cache.struct, out.data_ptr(), scratch[0].data_ptr(),
                        scratch[1].data_ptr(), stream if stream is not None else current_stream())
        return out

    def prefill_timed(self, x, T, cache, pos0, out, stream=None):
        return B.tasp_prefill_timed(self.handle, x.data_ptr(), T, cache.struct, pos0, out.data_ptr(),
                                    stream if stream is not None else current_stream())


    def seq_bind(self, cache):
        B.tasp_seq_bind(self.handle, cache.struct)

    def tree_workspace(self, cache, T, max_len=None, stream=None):
        """A workspace for tree_forward and tree_step calls of this shape."""
        n = B.tasp_tree_step_workspace_bytes(self.handle, cache.struct, T, cache.max_seq if max_len is None else max_len)
        return _workspace(n, cache.k.device, stream)

    def tree_forward(self, x, cache, parent=None, max_len=None, out=None, workspace=None, stream=None):
        """The plan over trees of nodes: x float32 [B][T][d] -> logits [B][T][V] (or residuals [B][T][d])."""
        dev = _device(cache.k, self.ws, x, parent, out)
        nb, T = x.shape[:2]
        width = self.desc.vocab or self.desc.d_model
        if out is None:
            out = _empty((nb, T, width), torch.float32, x.device, stream)
        ml = cache.max_seq if max_len is None else max_len
        ws = _on(dev, workspace) if workspace is not None else self.tree_workspace(cache, T, ml, stream)
        _launch(B.tasp_tree_forward, dev, stream, self.handle, _ptr(x, (cache.batch, T, self.desc.d_model), torch.float32, "x"),
                cache._parent(parent, T), T, cache.struct, ml, _ptr(out, (nb, T, width), torch.float32, "out"), ws[1], ws[2])
        return out

    def tree_step(self, embed, embed_scale, tokens, cache, u=None, parent=None, draft_logits=None, temperature=0.0,
                  max_len=None, out=None, scratch=None, workspace=None, stream=None):
        """One step over drafted tokens int32 [B][T] (node 0: the text's last token): returns (ids, path, n) as
        ``verify`` does, and the cache has grown by n rows (0 where it has none left for node 0). ``out``: those three;
        ``scratch``: (x [B][T][d], logits [B][T][V])."""
        dev = _device(cache.k, self.ws, embed, embed_scale, tokens, u, parent, draft_logits)
        nb, T = tokens.shape
        D, V = self.desc.d_model, self.desc.vocab
        if scratch is None:
            scratch = (_empty((nb, T, D), torch.float32, tokens.device, stream),
                       _empty((nb, T, max(V, 1)), torch.float32, tokens.device, stream))
        if out is None:
            ids, path = _empty((2, nb, T), torch.int32, tokens.device, stream)
            out = ids, path, _empty((nb,), torch.int32, tokens.device, stream)
        ml = cache.max_seq if max_len is None else max_len
        ws = _on(dev, workspace) if workspace is not None else self.tree_workspace(cache, T, ml, stream)
        _device(cache.k, *out, *scratch)
        _launch(B.tasp_tree_step, dev, stream, self.handle, _ptr(embed, (V, D), torch.int8, "embed"),
                _ptr(embed_scale, (V,), torch.float32, "embed_scale"), _ptr(tokens, (cache.batch, T), torch.int32, "tokens"),
                cache._parent(parent, T), _ptr(u, (nb, T), torch.float32, "u"),
                _ptr(draft_logits, (nb, T - 1, V), torch.float32, "draft_logits"), temperature, T, ml, cache.struct,
                _ptr(out[0], (nb, T), torch.int32, "ids"), _ptr(out[1], (nb, T), torch.int32, "path"),
                _ptr(out[2], (nb,), torch.int32, "n"), _ptr(scratch[0], (nb, T, D), torch.float32, "x"),
                _ptr(scratch[1], (nb, T, max(V, 1)), torch.float32, "logits"), ws[1], ws[2])
        return out


    def page_bind(self, cache):
        B.tasp_page_bind(self.handle, cache.struct)

    def page_workspace(self, cache, n_tokens, max_len=None, max_new=None, stream=None):
        """A workspace for page_forward calls of this shape (max_new None: with start and without)."""
        n = max(B.tasp_page_forward_workspace_bytes(self.handle, cache.struct, n_tokens, cache.max_seq if max_len is None else max_len, m)
                for m in _expected(n_tokens, max_new))
        return _workspace(n, cache.k.device, stream)

    def page_forward(self, x, cache, start=None, max_len=None, max_new=None, out=None, workspace=None, stream=None):
        """The plan over packed tokens x float32 [N][d] (start as page_append) -> logits [N][V] (or residuals [N][d]). The
        lengths stay: page_advance."""
        dev = _device(cache.k, self.ws, x, start, out)
        N = x.shape[0]
        width = self.desc.vocab or self.desc.d_model
        if out is None:
            out = _empty((N, width), torch.float32, x.device, stream)
        ml = cache.max_seq if max_len is None else max_len
        mn = max_new if max_new is not None else 1 if start is None else N
        ws = _on(dev, workspace) if workspace is not None else self.page_workspace(cache, N, ml, mn, stream)
        _launch(B.tasp_page_forward, dev, stream, self.handle, _ptr(x, (N, self.desc.d_model), torch.float32, "x"),
                cache._start(start), N, cache.struct, ml, mn, _ptr(out, (N, width), torch.float32, "out"), ws[1], ws[2])
        return out


def build_mask(desc, head_scores, chan_scores, granule, target, stream=None):
    """Greedy dependency-closed mask from device float32 scores ([L][Hq], [L][d_ffn/granule]).
    Returns (q_keep, kv_keep, ffn_keep) as device uint8 tensors and the FLOPs spent."""
    dev = head_scores.device
    n = B.tasp_mask_workspace_bytes(desc, granule)
    ws = torch.empty(n + 256, dtype=torch.uint8, device=dev)
    base = ws.data_ptr() + (-ws.data_ptr()) % 256
    q = torch.empty((desc.n_layers, desc.n_q_heads), dtype=torch.uint8, device=dev)
    kv = torch.empty((desc.n_layers, desc.n_kv_heads), dtype=torch.uint8, device=dev)
    f = torch.empty((desc.n_layers, desc.d_ffn), dtype=torch.uint8, device=dev)
    spent = B.tasp_build_mask(desc, head_scores.data_ptr(), chan_scores.data_ptr(), granule, target,
                              base, n, q.data_ptr(), kv.data_ptr(), f.data_ptr(),
                              stream if stream is not None else current_stream())
    return q, kv, f, spent


class Router:
    """Router weights on the device (float32 tensors keyed proj, w1, b1, w2, b2, w3, b3, row-major
    [out][in]) and the ABI struct over them."""

    def __init__(self, weights, temperature=1.0, tau=0.85, device="cuda"):
        self.t = {k: torch.as_tensor(np.ascontiguousarray(v, np.float32)).to(device)
                  for k, v in weights.items()}
        proj_dim, n_bins = self.t["proj"].shape
        self.struct = B.tasp_router(int(n_bins), int(proj_dim), int(self.t["w1"].shape[0]),
                                    int(self.t["w2"].shape[0]), int(self.t["w3"].shape[0]),
                                    float(temperature), float(tau),
                                    *[self.t[k].data_ptr() for k in ("proj", "w1", "b1", "w2",
                                                                      "b2", "w3", "b3")])
        self.feat_dim = int(proj_dim) + B.ROUTER_SCALARS
        self.n_tasks = int(self.t["w3"].shape[0])
        self._ws = {}

    def workspace(self, n, device):
        """A 256-byte aligned workspace for n prompts: (tensor, base pointer, bytes)."""
        if n not in self._ws:
            nb = B.tasp_router_workspace_bytes(self.struct, n)
            t = torch.empty(nb + 256, dtype=torch.uint8, device=device)
            self._ws[n] = (t, t.data_ptr() + (-t.data_ptr()) % 256, nb)
        return self._ws[n]

    def route(self, text, offsets, logprob, stream=None, features=True):
        """text: device uint8 [n_text]; offsets: device int32 [n + 1] (None: one prompt);
        logprob: device float32 [n]. Returns (features or None, probs, choice) device tensors."""
        n = int(logprob.numel())
        dev = logprob.device
        _, base, nb = self.workspace(n, dev)
        feats = torch.empty((n, self.feat_dim), device=dev) if features else None
        probs = torch.empty((n, self.n_tasks), device=dev)
        choice = torch.empty(n, dtype=torch.int32, device=dev)
        B.tasp_route(self.struct, text.data_ptr() if text.numel() else None, int(text.numel()),
                     offsets.data_ptr() if offsets is not None else None, n, logprob.data_ptr(),
                     base, nb, feats.data_ptr() if feats is not None else None, probs.data_ptr(),
                     choice.data_ptr(), stream if stream is not None else current_stream())
        return feats, probs, choice

    def serve_turn(self, task_plans, dense_plan, text, logprob, embed, embed_scale, prompt,
                   n_cached, n_new, cache, stream=None, scratch=None):
        """One routed turn. Returns (choice, reused, out ids device int32 [n_new + 1])."""
        T = int(prompt.numel())
        dev = prompt.device
        d = dense_plan.desc
        if scratch is None:
            scratch = (torch.empty((T, d.d_model), device=dev), torch.empty((T, d.vocab), device=dev))
        out = torch.empty(n_new + 1, dtype=torch.int32, device=dev)
        _, base, nb = self.workspace(1, dev)
        c, reused = B.tasp_serve_turn(
            self.struct, [p.handle for p in task_plans], dense_plan.handle,
            text.data_ptr() if text.numel() else None, int(text.numel()), logprob.data_ptr(),
            embed.data_ptr(), embed_scale.data_ptr(), prompt.data_ptr(), T, n_cached, n_new,
            cache.struct, out.data_ptr(), scratch[0].data_ptr(), scratch[1].data_ptr(), base, nb,
            stream if stream is not None else current_stream())
        return c, reused, out


# ------------------------------------------- sequences of their own lengths, drafted tokens

class _Types(dict):
    def __missing__(self, dtype):
        raise ValueError(f"{dtype} is none of {', '.join(map(str, self))}")


_SEQ_TYPES = _Types({torch.bfloat16: B.BF16, torch.float32: B.F32, torch.int8: B.INT8, torch.float8_e4m3fn: B.E4M3})

_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)   # (absent in builds without a GPU)
_current_device = getattr(torch._C, "_cuda_getDevice", None)
_pack_rows = struct.Struct("Pqqq").pack                              # a tasp_rows


def _launch(f, dev, stream, *args):
    """f(*args, stream) on device `dev`: on its current stream unless one is given."""
    if stream is None:
        stream = _raw_stream(dev)
    if dev == _current_device():
        f(*args, stream)
    else:
        with torch.cuda.device(dev):
            f(*args, stream)


def _device(t, *others):
    """The index of the GPU that holds every tensor given."""
    dev = t.get_device()
    for o in others:
        if o is not None and o.get_device() != dev:
            raise ValueError(f"tensors on {t.device} and {o.device}")
    if dev < 0:
        raise ValueError(f"tensors on {t.device}: a GPU is needed")
    return dev


def _ptr(t, shape, dtype, what):
    """Address of a contiguous tensor of the given shape and type; None for None."""
    if t is None:
        return None
    if t.shape != shape or t.dtype != dtype or not t.is_contiguous():
        raise ValueError(f"{what} must be a contiguous {dtype} tensor of {tuple(shape)}, not {t.dtype} {tuple(t.shape)}")
    return t.data_ptr()


def _rows(t, shape, dtype, what, token=1, head=2):
    """The tasp_rows (as bytes) of a tensor [B][..][..][dh]; token, head: the axes between."""
    st = t.stride()
    if t.shape != shape or t.dtype != dtype or st[3] != 1:
        raise ValueError(f"{what} must be a {dtype} tensor of {tuple(shape)} with contiguous heads, not {t.dtype} {tuple(t.shape)}")
    # (the stride of an axis of one is never used, and may be anything)
    return _pack_rows(t.data_ptr(), st[0] if shape[0] > 1 else 0, st[token] if shape[token] > 1 else 0,
                      st[head] if shape[head] > 1 else 0)


def _dense(t, seq, token, head):
    """The tasp_rows of a contiguous tensor made here, with its strides."""
    return _pack_rows(t.data_ptr(), seq, token, head)


def _empty(shape, dtype, device, stream):
    """A new tensor of the call's stream: the current one of the device, or the raw stream given."""
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    raw = stream.value if isinstance(stream, C.c_void_p) else stream
    with torch.cuda.stream(torch.cuda.ExternalStream(raw or 0, device)):
        return torch.empty(shape, dtype=dtype, device=device)


def _like(t, stream):
    """A new contiguous tensor of t's shape and type, as _empty (half a microsecond less where t is contiguous)."""
    if stream is None and t.is_contiguous():
        return torch.empty_like(t)
    return _empty(t.shape, t.dtype, t.device, stream)


def _workspace(nbytes, device, stream=None):
    t = _empty(nbytes + 256, torch.uint8, device, stream)
    return t, t.data_ptr() + (-t.data_ptr()) % 256, nbytes


def _on(dev, workspace):
    """A call's workspace, refused where its tensor lies on another device than the call's."""
    t = workspace[0]
    if t is not None and t.get_device() != dev:
        raise ValueError(f"the workspace lies on {t.device}, the call's tensors on cuda:{dev}")
    return workspace


class _Fixed:
    def __setattr__(self, name, value):
        if self.__dict__.get(name, value) is not value:  # (c.len += 1 sets the same tensor again)
            raise AttributeError(f"{name} of a cache stays what it is: copy into it, or make another cache")
        super().__setattr__(name, value)


class SeqCache(_Fixed):
    """A cache whose sequences have their own lengths: k, v ``[L][B][Hkv][S][dh]`` as bfloat16, int8 or
    float8_e4m3fn (8 bits with float32 scales ``[L][B][Hkv][S]``), len int32 ``[B]``, all owned by torch. They stay the
    tensors that the cache was made of, whose addresses ``struct`` holds: new values are copied into them."""

    def __init__(self, k, v, length, k_scale=None, v_scale=None):
        if k.dtype not in (torch.bfloat16, torch.int8, torch.float8_e4m3fn) or k.dim() != 5:
            raise ValueError(f"k must be a bfloat16, int8 or float8_e4m3fn tensor [L][B][Hkv][S][dh], not {k.dtype} {tuple(k.shape)}")
        self.dev = _device(k, v, length, k_scale, v_scale)
        self.k, self.v, self.len, self.k_scale, self.v_scale = k, v, length, k_scale, v_scale
        wide = k.dtype == torch.bfloat16
        if wide == (k_scale is not None) or wide == (v_scale is not None):
            raise ValueError("scales go with caches in 8 bits, and only with them")
        self.n_layers, self.batch, self.n_kv, self.max_seq, self.dh = k.shape
        self.struct = B.tasp_seq_cache(
            _ptr(k, k.shape, k.dtype, "k"), _ptr(v, k.shape, k.dtype, "v"),
            _ptr(k_scale, k.shape[:4], torch.float32, "k_scale"), _ptr(v_scale, k.shape[:4], torch.float32, "v_scale"),
            _ptr(length, (self.batch,), torch.int32, "len"), _SEQ_TYPES[k.dtype], *k.shape, 0)

    @classmethod
    def empty(cls, n_layers, batch, n_kv_heads, max_seq, head_dim, dtype=torch.int8, device="cuda"):
        """A cache of empty sequences."""
        shape = (n_layers, batch, n_kv_heads, max_seq, head_dim)
        k, v = (torch.zeros(shape, dtype=dtype, device=device) for _ in range(2))
        sc = [None, None] if dtype == torch.bfloat16 else [torch.zeros(shape[:4], device=device) for _ in range(2)]
        return cls(k, v, torch.zeros(batch, dtype=torch.int32, device=device), *sc)

    def _parent(self, parent, T):
        return None if parent is None else _ptr(parent, (self.batch, T), torch.int32, "parent")


class Rope:
    """Rotary positions (tasp_rope): layout "half" or "interleaved", scaling "none", "linear", "wavelength" or "index"."""

    def __init__(self, layout="half", rot_dim=128, theta=500000.0, scaling="none", factor=1.0, low=1.0, high=4.0,
                 orig_len=8192, mscale=1.0):
        self.struct = B.tasp_rope(B.ROPE_LAYOUTS[layout], rot_dim, B.ROPE_SCALINGS[scaling], orig_len, theta, factor,
                                  low, high, mscale)


def seq_append(cache, layer, q, k, v, rope=None, parent=None, q_out=None, stream=None):
    """Write k, v ``[B][T][Hkv][dh]`` behind the sequences (their lengths stay) and return q ``[B][T][Hq][dh]``
    rotated (None without queries). Any strides whose rows are 16-byte aligned; bfloat16 or float32."""
    dev = _device(cache.k, q, k, v, parent, q_out)
    T, dt = k.shape[1], k.dtype
    kv = (cache.batch, T, cache.n_kv, cache.dh)
    rq = ro = None
    n_q = 0
    if q is not None:
        n_q = q.shape[2]
        shape = (cache.batch, T, n_q, cache.dh)
        rq = _rows(q, shape, dt, "q")
        if q_out is None:
            q_out = _like(q, stream)
            ro = _dense(q_out, T * n_q * cache.dh, n_q * cache.dh, cache.dh)
        else:
            ro = _rows(q_out, shape, dt, "q_out")
    _launch(B.tasp_seq_append, dev, stream, cache.struct, layer, None if rope is None else rope.struct,
            cache._parent(parent, T), T, _SEQ_TYPES[dt], rq, _rows(k, kv, dt, "k"), _rows(v, kv, dt, "v"), n_q, ro)
    return q_out


def seq_read(cache, layer, n, first=None, dtype=torch.bfloat16, out=None, stream=None):
    """(k, v) ``[B][Hkv][n][dh]``: rows first .. first + n - 1 (device int32 [B]; None: 0) as values."""
    shape = (cache.batch, cache.n_kv, n, cache.dh)
    if out is not None:
        k, v = out
        dev, dt = _device(cache.k, first, k, v), k.dtype
        rk, rv = _rows(k, shape, dt, "k", 2, 1), _rows(v, shape, dt, "v", 2, 1)
    else:
        dev, dt = _device(cache.k, first), dtype
        k = _empty(shape, dt, cache.k.device, stream)
        v = _like(k, stream)
        strides = cache.n_kv * n * cache.dh, cache.dh, n * cache.dh
        rk, rv = _dense(k, *strides), _dense(v, *strides)
    _launch(B.tasp_seq_read, dev, stream, cache.struct, layer, _ptr(first, (cache.batch,), torch.int32, "first"), n,
            _SEQ_TYPES[dt], rk, rv)
    return k, v


def tree_attention_workspace(cache, n_q_heads, T, max_len=None, stream=None):
    """A workspace for tree_attention calls of this shape (any layer)."""
    n = B.tasp_tree_attention_workspace_bytes(cache.struct, n_q_heads, T, cache.max_seq if max_len is None else max_len)
    return _workspace(n, cache.k.device, stream)


def tree_attention(cache, layer, q, parent=None, scale=None, max_len=None, out=None, workspace=None, stream=None):
    """Attention of the appended nodes' queries ``[B][T][Hq][dh]`` over their sequences and ancestors. max_len: the
    largest length expected; workspace: of tree_attention_workspace with the same arguments (else one of the call's own)."""
    dev, dt = _device(cache.k, q, parent, out), q.dtype
    T, n_q = q.shape[1], q.shape[2]
    shape = (cache.batch, T, n_q, cache.dh)
    rq = _rows(q, shape, dt, "q")
    if out is None:
        out = _like(q, stream)
        ro = _dense(out, T * n_q * cache.dh, n_q * cache.dh, cache.dh)
    else:
        ro = _rows(out, shape, dt, "out")
    if max_len is None:
        max_len = cache.max_seq
    ws = _on(dev, workspace) if workspace is not None else tree_attention_workspace(cache, n_q, T, max_len, stream)
    _launch(B.tasp_tree_attention, dev, stream, cache.struct, layer, cache._parent(parent, T), T, _SEQ_TYPES[dt],
            rq, n_q, cache.dh ** -0.5 if scale is None else scale, max_len, ro, ws[1], ws[2])
    return out


def verify_workspace(batch, T, vocab, device="cuda", stream=None):
    """A workspace for verify calls of this shape."""
    return _workspace(B.tasp_verify_workspace_bytes(batch, T, vocab), device, stream)


def verify(logits, tokens, u, parent=None, draft_logits=None, temperature=1.0, workspace=None, stream=None):
    """Verify drafted tokens int32 ``[B][T]`` (node 0: the text's last token) against float32 logits ``[B][T][V]``
    with random numbers u ``[B][T]``. Returns (ids, path, n): the emitted tokens and the accepted nodes, -1 behind them."""
    dev = _device(logits, tokens, u, parent, draft_logits)
    nb, T, V = logits.shape
    ids, path = _like(tokens, stream), _like(tokens, stream)
    n = _empty((nb,), torch.int32, tokens.device, stream)
    ws = _on(dev, workspace) if workspace is not None else verify_workspace(nb, T, V, logits.device, stream)
    _launch(B.tasp_verify, dev, stream, _ptr(logits, (nb, T, V), torch.float32, "logits"),
            _ptr(tokens, (nb, T), torch.int32, "tokens"), _ptr(u, (nb, T), torch.float32, "u"),
            _ptr(parent, (nb, T), torch.int32, "parent"), _ptr(draft_logits, (nb, T - 1, V), torch.float32, "draft_logits"),
            nb, T, V, temperature, ids.data_ptr(), path.data_ptr(), n.data_ptr(), ws[1], ws[2])
    return ids, path, n


def seq_commit(cache, path, n, len_out=None, stream=None):
    """Move the accepted paths' rows together in every layer and return the new lengths (len_out None: in cache.len)."""
    if len_out is None:
        len_out = cache.len
    dev, nb, T = _device(cache.k, path, n, len_out), cache.batch, path.shape[1]
    _launch(B.tasp_seq_commit, dev, stream, cache.struct, _ptr(path, (nb, T), torch.int32, "path"),
            _ptr(n, (nb,), torch.int32, "n"), T, _ptr(len_out, (nb,), torch.int32, "len_out"))
    return len_out


# ------------------------------------------- caches in pages, scores of given tokens

class PageCache(_Fixed):
    """A cache in pages: k, v ``[L][pages][Hkv][rows][dh]`` as bfloat16, int8 or float8_e4m3fn (8 bits with float32 scales
    ``[L][pages][Hkv]``), table int32 ``[B][max_pages]``, len int32 ``[B]``, all owned by torch. They stay the tensors that the
    cache was made of, whose addresses ``struct`` holds: new values are copied into them."""

    def __init__(self, k, v, table, length, k_scale=None, v_scale=None):
        if k.dtype not in (torch.bfloat16, torch.int8, torch.float8_e4m3fn) or k.dim() != 5:
            raise ValueError(f"k must be a bfloat16, int8 or float8_e4m3fn tensor [L][pages][Hkv][rows][dh], not {k.dtype} {tuple(k.shape)}")
        if table.dim() != 2:
            raise ValueError(f"table must be [B][max_pages], not {tuple(table.shape)}")
        self.dev = _device(k, v, table, length, k_scale, v_scale)
        self.k, self.v, self.table, self.len, self.k_scale, self.v_scale = k, v, table, length, k_scale, v_scale
        wide = k.dtype == torch.bfloat16
        if wide == (k_scale is not None) or wide == (v_scale is not None):
            raise ValueError("scales go with caches in 8 bits, and only with them")
        self.n_layers, self.n_pages, self.n_kv, self.page_rows, self.dh = k.shape
        self.batch, self.max_pages = table.shape
        self.max_seq = self.max_pages * self.page_rows
        self.struct = B.tasp_page_cache(
            _ptr(k, k.shape, k.dtype, "k"), _ptr(v, k.shape, k.dtype, "v"),
            _ptr(k_scale, k.shape[:3], torch.float32, "k_scale"), _ptr(v_scale, k.shape[:3], torch.float32, "v_scale"),
            _ptr(table, table.shape, torch.int32, "table"), _ptr(length, (self.batch,), torch.int32, "len"), _SEQ_TYPES[k.dtype],
            *k.shape, self.batch, self.max_pages, 0)

    @classmethod
    def empty(cls, n_layers, n_pages, n_kv_heads, page_rows, head_dim, batch, max_pages, dtype=torch.int8, device="cuda"):
        """A pool of pages that no sequence has yet (table -1, lengths 0)."""
        shape = (n_layers, n_pages, n_kv_heads, page_rows, head_dim)
        k, v = (torch.zeros(shape, dtype=dtype, device=device) for _ in range(2))
        sc = [None, None] if dtype == torch.bfloat16 else [torch.zeros(shape[:3], device=device) for _ in range(2)]
        return cls(k, v, torch.full((batch, max_pages), -1, dtype=torch.int32, device=device),
                   torch.zeros(batch, dtype=torch.int32, device=device), *sc)

    def _start(self, start):
        return None if start is None else _ptr(start, (self.batch + 1,), torch.int32, "start")


def _packed(t, shape, dtype, what):
    """The tasp_rows (as bytes) of a tensor [N][heads][dh]."""
    st = t.stride()
    if t.shape != shape or t.dtype != dtype or st[2] != 1:
        raise ValueError(f"{what} must be a {dtype} tensor of {tuple(shape)} with contiguous heads, not {t.dtype} {tuple(t.shape)}")
    return _pack_rows(t.data_ptr(), 0, st[0] if shape[0] > 1 else 0, st[1] if shape[1] > 1 else 0)


def page_append(cache, layer, q, k, v, start=None, rope=None, q_out=None, stream=None):
    """Write packed k, v ``[N][Hkv][dh]`` into the pages of their sequences (lengths stay) and return q ``[N][Hq][dh]``
    rotated (None without queries). start int32 ``[B + 1]``: tokens start[b] .. start[b + 1] - 1 are sequence b's; None:
    one token of each. Any strides whose rows are 16-byte aligned; bfloat16 or float32."""
    dev = _device(cache.k, q, k, v, start, q_out)
    N, dt = k.shape[0], k.dtype
    kv = (N, cache.n_kv, cache.dh)
    rq = ro = None
    n_q = 0
    if q is not None:
        n_q = q.shape[1]
        shape = (N, n_q, cache.dh)
        rq = _packed(q, shape, dt, "q")
        if q_out is None:
            q_out = _like(q, stream) if q.is_contiguous() else _empty(shape, dt, q.device, stream)
            ro = _dense(q_out, 0, n_q * cache.dh, cache.dh)
        else:
            ro = _packed(q_out, shape, dt, "q_out")
    _launch(B.tasp_page_append, dev, stream, cache.struct, layer, None if rope is None else rope.struct, cache._start(start),
            N, _SEQ_TYPES[dt], rq, _packed(k, kv, dt, "k"), _packed(v, kv, dt, "v"), n_q, ro)
    return q_out


def page_read(cache, layer, n, first=None, dtype=torch.bfloat16, out=None, stream=None):
    """(k, v) ``[B][Hkv][n][dh]``: rows first .. first + n - 1 (device int32 [B]; None: 0) as values."""
    shape = (cache.batch, cache.n_kv, n, cache.dh)
    if out is not None:
        k, v = out
        dev, dt = _device(cache.k, first, k, v), k.dtype
        rk, rv = _rows(k, shape, dt, "k", 2, 1), _rows(v, shape, dt, "v", 2, 1)
    else:
        dev, dt = _device(cache.k, first), dtype
        k = _empty(shape, dt, cache.k.device, stream)
        v = _like(k, stream)
        strides = cache.n_kv * n * cache.dh, cache.dh, n * cache.dh
        rk, rv = _dense(k, *strides), _dense(v, *strides)
    _launch(B.tasp_page_read, dev, stream, cache.struct, layer, _ptr(first, (cache.batch,), torch.int32, "first"), n,
            _SEQ_TYPES[dt], rk, rv)
    return k, v


def _expected(n_tokens, max_new):
    """The numbers of new tokens that calls expect of a sequence where max_new is None: all of the call's, or, without start, one."""
    return (1, n_tokens) if max_new is None else (max_new,)


def page_attention_workspace(cache, n_q_heads, n_tokens, max_len=None, max_new=None, stream=None):
    """A workspace for page_attention calls of this shape (any layer; max_new None: with start and without)."""
    n = max(B.tasp_page_attention_workspace_bytes(cache.struct, n_q_heads, n_tokens, cache.max_seq if max_len is None else max_len, m)
            for m in _expected(n_tokens, max_new))
    return _workspace(n, cache.k.device, stream)


def page_attention(cache, layer, q, start=None, scale=None, max_len=None, max_new=None, out=None, workspace=None, stream=None):
    """Causal attention of the appended tokens' queries ``[N][Hq][dh]`` over their sequences' pages; start as page_append.
    max_len, max_new: the largest length and number of new tokens of a sequence that are expected; workspace: of
    page_attention_workspace with the same arguments (else one of the call's own). Rows of tokens that are no sequence's are
    not written."""
    dev, dt = _device(cache.k, q, start, out), q.dtype
    N, n_q = q.shape[:2]
    shape = (N, n_q, cache.dh)
    rq = _packed(q, shape, dt, "q")
    if out is None:
        out = _like(q, stream) if q.is_contiguous() else _empty(shape, dt, q.device, stream)
        ro = _dense(out, 0, n_q * cache.dh, cache.dh)
    else:
        ro = _packed(out, shape, dt, "out")
    if max_len is None:
        max_len = cache.max_seq
    if max_new is None:
        max_new = 1 if start is None else N
    ws = _on(dev, workspace) if workspace is not None else page_attention_workspace(cache, n_q, N, max_len, max_new, stream)
    _launch(B.tasp_page_attention, dev, stream, cache.struct, layer, cache._start(start), N, _SEQ_TYPES[dt], rq, n_q,
            cache.dh ** -0.5 if scale is None else scale, max_len, max_new, ro, ws[1], ws[2])
    return out


def page_advance(cache, n_tokens, start=None, stream=None):
    """Lengths grow by the tokens of a step (start as page_append), behind its last layer. Returns them."""
    dev = _device(cache.k, start)
    _launch(B.tasp_page_advance, dev, stream, cache.struct, cache._start(start), n_tokens)
    return cache.len


class TokenLogprobs(NamedTuple):
    """Of every row: the token's log probability, the entropy, the token's rank, the first tokens in the order of logits and
    their log probabilities; of every sequence of rows the mean log probability (None without ``start``)."""
    logprob: torch.Tensor
    entropy: torch.Tensor
    rank: torch.Tensor
    top_ids: torch.Tensor
    top_logprobs: torch.Tensor
    mean: Optional[torch.Tensor]


def token_logprobs_workspace(rows, vocab, n_top=0, device="cuda", stream=None):
    """A workspace for token_logprobs calls of this shape."""
    return _workspace(B.tasp_token_logprobs_workspace_bytes(rows, vocab, n_top), device, stream)


def token_logprobs(logits, tokens, n_top=0, temperature=1.0, start=None, workspace=None, stream=None):
    """Scores of tokens int32 ``[R]`` (outside the vocabulary: padding) against logits ``[R][V]`` (float32 or bfloat16, rows
    that do not overlap). start int32 ``[S + 1]``: rows start[i] .. start[i + 1] - 1 are sequence i's."""
    dev = _device(logits, tokens, start)
    if logits.dim() != 2 or logits.dtype not in (torch.float32, torch.bfloat16) or (logits.shape[1] > 1 and logits.stride(1) != 1):
        raise ValueError(f"logits must be a float32 or bfloat16 tensor [R][V] with contiguous rows, not {logits.dtype} {tuple(logits.shape)}")
    R, V = logits.shape
    S = 0
    if start is not None:
        if start.dim() != 1 or start.shape[0] < 2:
            raise ValueError(f"start must be [S + 1], not {tuple(start.shape)}")
        S = start.shape[0] - 1
    # one allocation for the outputs of a type
    top = R * n_top
    numbers, whole = _empty((2 * R + top + S,), torch.float32, logits.device, stream), _empty((R + top,), torch.int32, logits.device, stream)
    logprob, entropy, top_lp, mean = numbers.split((R, R, top, S))
    rank, ids = whole.split((R, top))
    at, to = numbers.data_ptr(), whole.data_ptr()
    ws = _on(dev, workspace) if workspace is not None else token_logprobs_workspace(R, V, n_top, logits.device, stream)
    _launch(B.tasp_token_logprobs, dev, stream, logits.data_ptr(), _SEQ_TYPES[logits.dtype], logits.stride(0) if R > 1 else V,
            _ptr(tokens, (R,), torch.int32, "tokens"), R, V, temperature, n_top, at, at + 4 * R, to, to + 4 * R,
            at + 8 * R, _ptr(start, (S + 1,), torch.int32, "start"), S, at + 8 * R + 4 * top if S else None, ws[1], ws[2])
    return TokenLogprobs(logprob, entropy, rank, ids.view(R, n_top), top_lp.view(R, n_top), mean if S else None)
