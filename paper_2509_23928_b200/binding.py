"""ctypes binding of include/hivis.h.  Argument marshalling only."""
from __future__ import annotations

import ctypes as C
import os
from typing import Dict, NamedTuple, Optional, Sequence

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libhivis.so")

HIVIS_F32, HIVIS_BF16, HIVIS_BF16_KV4 = 0, 1, 2
HIVIS_MAX_BATCH, HIVIS_MAX_K = 64, 16
TAPS = {"u": 0, "attn": 1, "y": 2, "act": 3, "g": 4, "q": 5}
ERRORS = {0: "OK", -1: "ARG", -2: "SHAPE", -3: "DTYPE", -4: "STATE", -5: "CAPACITY", -6: "CUDA",
          -7: "TIMEOUT", -8: "NOMEM"}

EXPORTS = ("hivis_init", "hivis_destroy", "hivis_prefill", "hivis_draft", "hivis_verify", "hivis_reset",
           "hivis_get_kv_len", "hivis_set_kv_len", "hivis_read_kv", "hivis_debug_tap", "hivis_step_bytes",
           "hivis_launch_count", "hivis_last_error", "hivis_profile_begin", "hivis_profile_end", "hivis_set_option",
           "hivis_status", "hivis_verify_noalloc", "hivis_read_phase_times", "hivis_draft_tree", "hivis_verify_tree", "hivis_verify_sampled", "hivis_draft_sampled",
           "hivis_set_kv_len_batch", "hivis_kv4_append", "hivis_kv4_read", "hivis_kv4_attention",
           "hivis_logprobs")
HIVIS_KV4_GROUP, HIVIS_KV4_MAX_QUERIES, HIVIS_KV4_MAX_MASK = 32, 64, 1024
HIVIS_OPT_CHAIN_KERNEL = 0
HIVIS_OPT_TC_KERNEL = 1
HIVIS_OPT_WAIT_LIMIT_US = 2
HIVIS_OPT_DEBUG_MISS_BARRIER = 3
HIVIS_OPT_PHASE_TIMES = 4
HIVIS_OPT_L2_KEEP = 5
HIVIS_OPT_TC_PREFILL = 6
HIVIS_PHASE_EVENTS = 24
PROFILE_CLASSES = ("fuse_fc", "qkv", "attention", "o_proj", "gate_up", "down", "lm_head_argmax", "setup_finish",
                   "draft_chain")


class HivisError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"HIVIS_ERR_{ERRORS.get(code, code)} ({code}): {msg}")
        self.code = code


class hivis_config(C.Structure):
    _fields_ = [("struct_size", C.c_uint32), ("dtype", C.c_int), ("d", C.c_int), ("n_q_heads", C.c_int),
                ("n_kv_heads", C.c_int), ("head_dim", C.c_int), ("ffn", C.c_int), ("vocab", C.c_int),
                ("rms_eps", C.c_float), ("rope_base", C.c_float), ("max_batch", C.c_int),
                ("max_len", C.c_int), ("max_k", C.c_int)]


_WNAMES = ("embed", "lm_head", "fc", "norm1", "wq", "wk", "wv", "bq", "bk", "bv", "wo", "norm2", "w_gate",
           "w_up", "w_down", "resid_proj")


class hivis_weights(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in _WNAMES]


class hivis_kv4_cache(C.Structure):
    _fields_ = [("struct_size", C.c_uint32), ("n_slots", C.c_int), ("n_kv_heads", C.c_int), ("head_dim", C.c_int),
                ("max_len", C.c_int), ("data", C.c_void_p)]


def _load() -> C.CDLL:
    if not os.path.exists(LIB_PATH):
        from . import build as _b          # nvcc is part of the toolchain image; build in-tree once
        _b.build()
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is missing and could not be built: the CUDA library is required")
    L = C.CDLL(LIB_PATH)
    vp, ip, i32 = C.c_void_p, C.POINTER(C.c_int), C.c_int
    L.hivis_init.argtypes = [C.POINTER(vp), C.POINTER(hivis_config), C.POINTER(hivis_weights), vp]
    L.hivis_destroy.argtypes = [vp]
    L.hivis_prefill.argtypes = [vp, i32, ip, vp, vp, ip, ip, vp, vp]
    L.hivis_draft.argtypes = [vp, i32, ip, i32, vp, i32, vp, vp, vp, vp]
    L.hivis_verify.argtypes = [vp, i32, ip, i32, vp, vp, i32, vp, vp, vp, vp]
    L.hivis_reset.argtypes = [vp, i32, vp]
    L.hivis_get_kv_len.argtypes = [vp, i32, ip, ip, vp]
    L.hivis_set_kv_len.argtypes = [vp, i32, i32, i32, vp]
    L.hivis_set_kv_len_batch.argtypes = [vp, i32, ip, ip, i32, vp]
    L.hivis_read_kv.argtypes = [vp, i32, i32, i32, vp, vp, vp]
    L.hivis_debug_tap.argtypes = [vp, i32, vp, vp]
    L.hivis_step_bytes.argtypes = [vp, i32, ip]
    L.hivis_step_bytes.restype = C.c_int64
    L.hivis_launch_count.argtypes = [vp]
    L.hivis_launch_count.restype = C.c_int64
    L.hivis_set_option.argtypes = [vp, i32, i32]
    L.hivis_status.argtypes = [vp, vp]
    L.hivis_profile_begin.argtypes = [vp]
    L.hivis_profile_end.argtypes = [vp, C.POINTER(C.c_float), C.POINTER(C.c_int64)]
    L.hivis_verify_noalloc.argtypes = [i32, i32, i32, vp, vp, i32, vp, vp, vp, vp, vp]
    L.hivis_verify_sampled.argtypes = [vp, i32, ip, i32, vp, vp, vp, i32, C.c_float, vp, vp, vp, vp, vp, vp]
    L.hivis_draft_sampled.argtypes = [vp, i32, ip, i32, vp, i32, C.c_float, vp, vp, vp, vp]
    L.hivis_draft_tree.argtypes = [vp, i32, i32, i32, i32, vp, i32, vp, vp, vp, vp, vp]
    L.hivis_verify_tree.argtypes = [vp, i32, vp, i32, vp, vp, vp, vp, vp]
    L.hivis_read_phase_times.argtypes = [vp, vp, C.c_longlong, ip, ip, vp]
    cp = C.POINTER(hivis_kv4_cache)
    L.hivis_kv4_append.argtypes = [cp, i32, ip, ip, vp, vp, vp, i32, C.c_int64, vp]
    L.hivis_kv4_read.argtypes = [cp, i32, ip, ip, vp, vp, vp, vp]
    L.hivis_kv4_attention.argtypes = [cp, i32, ip, vp, i32, i32, vp, i32, C.c_int64, C.c_float, vp, i32, vp, C.c_int64, vp]
    L.hivis_logprobs.argtypes = [i32, i32, vp, i32, C.c_int64, C.c_float, vp, i32, i32, vp, vp, vp, vp, vp]
    L.hivis_last_error.argtypes = [vp]
    L.hivis_last_error.restype = C.c_char_p
    for n in EXPORTS:
        getattr(L, n)
    return L


lib = _load()


def _ints(seq: Optional[Sequence[int]]):
    if seq is None:
        return None
    seq = [int(x) for x in seq]
    return (C.c_int * len(seq))(*seq)


def _ptr(t) -> Optional[int]:
    """Device address of a torch tensor (None stays None); plain ints pass through."""
    if t is None:
        return None
    if isinstance(t, int):
        return t
    assert t.is_cuda and t.is_contiguous(), "expected a contiguous CUDA tensor"
    return t.data_ptr()


def _row_ptr(t) -> Optional[int]:
    """As _ptr, for a tensor whose rows (first dimension) may lie apart."""
    if t is None or isinstance(t, int):
        return t
    assert t.is_cuda and (t.is_contiguous() or t[0].is_contiguous()), "expected a CUDA tensor with contiguous rows"
    return t.data_ptr()


def _stream(stream) -> int:
    if stream is None:
        import torch
        return torch.cuda.current_stream().cuda_stream
    return stream if isinstance(stream, int) else stream.cuda_stream


def hivis_last_error(ctx=None) -> str:
    return (lib.hivis_last_error(ctx) or b"").decode()


def _check(rc: int, ctx=None):
    if rc != 0:
        raise HivisError(rc, hivis_last_error(ctx))


# ------------------------------------------------------------------ functions named as in hivis.h
def hivis_init(cfg: hivis_config, weights: hivis_weights, stream=None) -> int:
    out = C.c_void_p()
    _check(lib.hivis_init(C.byref(out), C.byref(cfg), C.byref(weights), _stream(stream)))
    return out.value


def hivis_destroy(ctx) -> None:
    _check(lib.hivis_destroy(ctx))


def hivis_prefill(ctx, B, seq_slots, ids, hidden, cu_seqlens, start_pos=None, resid0=None, stream=None):
    _check(lib.hivis_prefill(ctx, int(B), _ints(seq_slots), _ptr(ids), _ptr(hidden), _ints(cu_seqlens),
                             _ints(start_pos), _ptr(resid0), _stream(stream)), ctx)


def hivis_draft(ctx, B, seq_slots, k, resid, n_resid, out_ids, forced_ids=None, out_logits=None, stream=None):
    _check(lib.hivis_draft(ctx, int(B), _ints(seq_slots), int(k), _ptr(resid), int(n_resid), _ptr(out_ids),
                           _ptr(forced_ids), _ptr(out_logits), _stream(stream)), ctx)


def hivis_draft_sampled(ctx, B, seq_slots, k, resid, n_resid, temperature, uniforms, out_ids, out_logits=None, stream=None):
    _check(lib.hivis_draft_sampled(ctx, int(B), _ints(seq_slots), int(k), _ptr(resid), int(n_resid), float(temperature),
                                   _ptr(uniforms), _ptr(out_ids), _ptr(out_logits), _stream(stream)), ctx)


def hivis_verify(ctx, B, seq_slots, k, draft_ids, target_logits, logits_dtype, out_accept, out_next,
                 out_kv_len=None, stream=None):
    _check(lib.hivis_verify(ctx, int(B), _ints(seq_slots), int(k), _ptr(draft_ids), _ptr(target_logits),
                            int(logits_dtype), _ptr(out_accept), _ptr(out_next), _ptr(out_kv_len),
                            _stream(stream)), ctx)


def hivis_verify_sampled(ctx, B, seq_slots, k, draft_ids, draft_logits, target_logits, logits_dtype, temperature, u_accept,
                         u_sample, out_accept, out_next, out_kv_len=None, stream=None):
    _check(lib.hivis_verify_sampled(ctx, int(B), _ints(seq_slots), int(k), _ptr(draft_ids), _ptr(draft_logits),
                                    _ptr(target_logits), int(logits_dtype), float(temperature), _ptr(u_accept), _ptr(u_sample),
                                    _ptr(out_accept), _ptr(out_next), _ptr(out_kv_len), _stream(stream)), ctx)


def hivis_draft_tree(ctx, slot, topk, depth, keep, resid, n_resid, out_tokens, out_parents, out_scores, out_count,
                     stream=None):
    _check(lib.hivis_draft_tree(ctx, int(slot), int(topk), int(depth), int(keep), _ptr(resid), int(n_resid),
                                _ptr(out_tokens), _ptr(out_parents), _ptr(out_scores), _ptr(out_count), _stream(stream)), ctx)


def hivis_verify_tree(ctx, slot, target_logits, logits_dtype, out_accept, out_path, out_next, out_kv_len=None, stream=None):
    _check(lib.hivis_verify_tree(ctx, int(slot), _ptr(target_logits), int(logits_dtype), _ptr(out_accept), _ptr(out_path),
                                 _ptr(out_next), _ptr(out_kv_len), _stream(stream)), ctx)


def hivis_verify_noalloc(B, k, vocab, draft_ids, target_logits, logits_dtype, rows_before, out_accept,
                         out_next, out_kv_len=None, stream=None):
    """Context-free greedy verification for callers that must not allocate device memory: the
    argmax keys sit in a fixed array inside the library (at most 64 sequences, k <= 16)."""
    _check(lib.hivis_verify_noalloc(int(B), int(k), int(vocab), _ptr(draft_ids), _ptr(target_logits),
                                    int(logits_dtype), _ptr(rows_before), _ptr(out_accept), _ptr(out_next),
                                    _ptr(out_kv_len), _stream(stream)))


def hivis_kv4_append(cache, B, seq_slots, cu_seqlens, start_rows, k, v, dtype, ld, stream=None):
    _check(lib.hivis_kv4_append(C.byref(cache), int(B), _ints(seq_slots), _ints(cu_seqlens), _ptr(start_rows), _row_ptr(k),
                                _row_ptr(v), int(dtype), int(ld), _stream(stream)))


def hivis_kv4_read(cache, B, seq_slots, cu_seqlens, start_rows, out_k, out_v, stream=None):
    _check(lib.hivis_kv4_read(C.byref(cache), int(B), _ints(seq_slots), _ints(cu_seqlens), _ptr(start_rows), _ptr(out_k),
                              _ptr(out_v), _stream(stream)))


def hivis_kv4_attention(cache, B, seq_slots, rows, n_q, n_q_heads, q, dtype, q_ld, scale, mask, mask_rows, out, out_ld,
                        stream=None):
    _check(lib.hivis_kv4_attention(C.byref(cache), int(B), _ints(seq_slots), _ptr(rows), int(n_q), int(n_q_heads), _row_ptr(q),
                                   int(dtype), int(q_ld), float(scale), _ptr(mask), int(mask_rows), _row_ptr(out), int(out_ld),
                                   _stream(stream)))


def hivis_logprobs(n_rows, vocab, logits, logits_dtype, ld, temperature, ids, n_ids, top_n, out_logprobs, out_entropy=None,
                   out_top_ids=None, out_top_logprobs=None, stream=None):
    _check(lib.hivis_logprobs(int(n_rows), int(vocab), _row_ptr(logits), int(logits_dtype), int(ld), float(temperature), _ptr(ids),
                              int(n_ids), int(top_n), _ptr(out_logprobs), _ptr(out_entropy), _ptr(out_top_ids),
                              _ptr(out_top_logprobs), _stream(stream)))


def hivis_reset(ctx, slot, stream=None):
    _check(lib.hivis_reset(ctx, int(slot), _stream(stream)), ctx)


def hivis_get_kv_len(ctx, slot, stream=None):
    n, p = C.c_int(), C.c_int()
    _check(lib.hivis_get_kv_len(ctx, int(slot), C.byref(n), C.byref(p), _stream(stream)), ctx)
    return n.value, bool(p.value)


def hivis_set_kv_len(ctx, slot, n_rows, restore_pending=False, stream=None):
    _check(lib.hivis_set_kv_len(ctx, int(slot), int(n_rows), int(bool(restore_pending)), _stream(stream)), ctx)


def hivis_set_kv_len_batch(ctx, B, seq_slots, n_rows, restore_pending=False, stream=None):
    _check(lib.hivis_set_kv_len_batch(ctx, int(B), _ints(seq_slots), _ints(n_rows), 1 if restore_pending else 0,
                                      _stream(stream)), ctx)


def hivis_read_kv(ctx, slot, row0, n, out_k, out_v, stream=None):
    _check(lib.hivis_read_kv(ctx, int(slot), int(row0), int(n), _ptr(out_k), _ptr(out_v), _stream(stream)), ctx)


def hivis_debug_tap(ctx, which, out, stream=None):
    _check(lib.hivis_debug_tap(ctx, int(which), _ptr(out), _stream(stream)), ctx)


def hivis_step_bytes(ctx, kv_rows: Sequence[int]) -> int:
    return int(lib.hivis_step_bytes(ctx, len(kv_rows), _ints(kv_rows)))


def hivis_set_option(ctx, option: int, value: int) -> None:
    _check(lib.hivis_set_option(ctx, int(option), int(value)), ctx)


def hivis_status(ctx, stream=None) -> None:
    """Synchronise and raise HivisError(TIMEOUT) if a kernel gave up on a bounded wait."""
    _check(lib.hivis_status(ctx, _stream(stream)), ctx)


def hivis_profile_begin(ctx) -> None:
    _check(lib.hivis_profile_begin(ctx), ctx)


def hivis_profile_end(ctx):
    """-> {class name: (device ms, launches)} accumulated since hivis_profile_begin."""
    ms = (C.c_float * len(PROFILE_CLASSES))()
    n = (C.c_int64 * len(PROFILE_CLASSES))()
    _check(lib.hivis_profile_end(ctx, ms, n), ctx)
    return {name: (float(ms[i]), int(n[i])) for i, name in enumerate(PROFILE_CLASSES)}


def hivis_read_phase_times(ctx, stream=None):
    """-> uint64 array [k, HIVIS_PHASE_EVENTS, grid] of the last recorded tensor-core chain launch (ns; 0 = no event)."""
    import numpy as np
    k, g = C.c_int(), C.c_int()
    rc = lib.hivis_read_phase_times(ctx, None, 0, C.byref(k), C.byref(g), _stream(stream))
    if rc != -5:
        _check(rc, ctx)
    out = np.zeros((k.value, HIVIS_PHASE_EVENTS, g.value), dtype=np.uint64)
    _check(lib.hivis_read_phase_times(ctx, out.ctypes.data_as(C.c_void_p), out.size, C.byref(k), C.byref(g),
                                      _stream(stream)), ctx)
    return out


def hivis_launch_count(ctx) -> int:
    return int(lib.hivis_launch_count(ctx))


# ------------------------------------------------------------------ convenience wrapper (torch tensors)
class Drafter:
    """Owns one hivis context.  `weights`: name -> CUDA tensor in the context dtype, [out, in]."""

    def __init__(self, dims, weights: Dict[str, "object"], max_batch: int, max_len: int, max_k: int = 8,
                 stream=None, kv_bits: Optional[int] = None):
        """kv_bits: None keeps the cache in the weights' type; 4 (bf16 weights) holds it in 4 bits (HIVIS_BF16_KV4)."""
        import torch
        self.torch = torch
        self.dims = dims
        self.dtype = HIVIS_BF16 if dims.dtype == "bf16" else HIVIS_F32
        self.tdtype = torch.bfloat16 if self.dtype == HIVIS_BF16 else torch.float32
        if kv_bits is not None:
            if kv_bits != 4 or self.dtype != HIVIS_BF16:
                raise ValueError("kv_bits takes 4, for drafters with bf16 weights")
            self.dtype = HIVIS_BF16_KV4
        cfg = hivis_config(C.sizeof(hivis_config), self.dtype, dims.d, dims.n_q_heads, dims.n_kv_heads,
                           dims.head_dim, dims.ffn, dims.vocab, float(dims.rms_eps), float(dims.rope_base),
                           int(max_batch), int(max_len), int(max_k))
        w = hivis_weights(*[_ptr(weights.get(n)) for n in _WNAMES])
        self.ctx = hivis_init(cfg, w, stream)
        torch.cuda.current_stream().synchronize()      # the caller may now drop its weight tensors
        self.max_batch, self.max_len, self.max_k = max_batch, max_len, max_k
        self.dev = torch.device("cuda", torch.cuda.current_device())

    def close(self):
        if getattr(self, "ctx", None):
            hivis_destroy(self.ctx)
            self.ctx = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def prefill(self, ids, hidden, cu_seqlens, slots=None, start_pos=None, resid0=None):
        B = len(cu_seqlens) - 1
        hivis_prefill(self.ctx, B, slots, ids, hidden, cu_seqlens, start_pos, resid0)

    def draft(self, B, k, resid=None, slots=None, forced_ids=None, want_logits=False, out_ids=None):
        t = self.torch
        if out_ids is None:
            out_ids = t.empty((B, k), dtype=t.int32, device=self.dev)
        logits = t.empty((B, k, self.dims.vocab), dtype=t.float32, device=self.dev) if want_logits else None
        n_resid = 0 if resid is None else int(resid.shape[0])
        hivis_draft(self.ctx, B, slots, k, resid, n_resid, out_ids, forced_ids, logits)
        return (out_ids, logits) if want_logits else out_ids

    def draft_sampled(self, B, k, temperature, uniforms, resid=None, slots=None, want_logits=True):
        """Chained drafting with every token drawn from softmax(logits / temperature); uniforms fp32 [B, k, vocab]."""
        t = self.torch
        out_ids = t.empty((B, k), dtype=t.int32, device=self.dev)
        logits = t.empty((B, k, self.dims.vocab), dtype=t.float32, device=self.dev) if want_logits else None
        hivis_draft_sampled(self.ctx, B, slots, k, resid, 0 if resid is None else int(resid.shape[0]), temperature, uniforms,
                            out_ids, logits)
        return (out_ids, logits) if want_logits else out_ids

    def verify(self, draft_ids, target_logits, slots=None):
        t = self.torch
        B, k = draft_ids.shape
        ldt = HIVIS_BF16 if target_logits.dtype == t.bfloat16 else HIVIS_F32
        acc = t.empty(B, dtype=t.int32, device=self.dev)
        nxt = t.empty(B, dtype=t.int32, device=self.dev)
        kv = t.empty(B, dtype=t.int32, device=self.dev)
        hivis_verify(self.ctx, B, slots, k, draft_ids, target_logits, ldt, acc, nxt, kv)
        return acc, nxt, kv

    def verify_sampled(self, draft_ids, draft_logits, target_logits, temperature, u_accept, u_sample, slots=None):
        t = self.torch
        B, k = draft_ids.shape
        ldt = HIVIS_BF16 if target_logits.dtype == t.bfloat16 else HIVIS_F32
        acc = t.empty((B + 3) // 4 * 4, dtype=t.int32, device=self.dev)
        nxt = t.empty_like(acc)
        kv = t.empty_like(acc)
        hivis_verify_sampled(self.ctx, B, slots, k, draft_ids, draft_logits, target_logits, ldt, temperature, u_accept,
                             u_sample, acc, nxt, kv)
        return acc[:B], nxt[:B], kv[:B]

    def draft_tree(self, slot, topk, depth, keep, resid=None):
        """-> (tokens, parents, scores, count) of the draft tree of one sequence; count is a 1-element tensor."""
        t = self.torch
        tokens = t.full((keep,), -1, dtype=t.int32, device=self.dev)
        parents = t.full((keep,), -2, dtype=t.int32, device=self.dev)
        scores = t.zeros((keep,), dtype=t.float32, device=self.dev)
        count = t.zeros((4,), dtype=t.int32, device=self.dev)
        hivis_draft_tree(self.ctx, slot, topk, depth, keep, resid, 0 if resid is None else int(resid.shape[0]), tokens,
                         parents, scores, count)
        return tokens, parents, scores, count

    def verify_tree(self, slot, depth, target_logits):
        """-> (n accepted, path [depth], next token, rows) tensors."""
        t = self.torch
        ldt = HIVIS_BF16 if target_logits.dtype == t.bfloat16 else HIVIS_F32
        acc = t.zeros((4,), dtype=t.int32, device=self.dev)
        path = t.full(((depth + 3) // 4 * 4,), -2, dtype=t.int32, device=self.dev)
        nxt = t.zeros((4,), dtype=t.int32, device=self.dev)
        kv = t.zeros((4,), dtype=t.int32, device=self.dev)
        hivis_verify_tree(self.ctx, slot, target_logits, ldt, acc, path, nxt, kv)
        return acc, path, nxt, kv

    def kv_len(self, slot):
        return hivis_get_kv_len(self.ctx, slot)

    def set_kv_len(self, slot, n_rows, restore_pending=False):
        hivis_set_kv_len(self.ctx, slot, n_rows, restore_pending)

    def set_kv_len_batch(self, n_rows, slots=None, restore_pending=False):
        hivis_set_kv_len_batch(self.ctx, len(n_rows), slots, [int(x) for x in n_rows], restore_pending)

    def reset(self, slot):
        hivis_reset(self.ctx, slot)

    def read_kv(self, slot, row0, n):
        t = self.torch
        kvw = self.dims.n_kv_heads * self.dims.head_dim
        k = t.empty((n, kvw), dtype=t.float32, device=self.dev)
        v = t.empty((n, kvw), dtype=t.float32, device=self.dev)
        hivis_read_kv(self.ctx, slot, row0, n, k, v)
        return k, v

    def tap(self, name, B):
        t = self.torch
        width = {"u": self.dims.d, "attn": self.dims.n_q_heads * self.dims.head_dim, "y": self.dims.d,
                 "act": self.dims.ffn, "g": self.dims.d, "q": self.dims.n_q_heads * self.dims.head_dim}[name]
        out = t.empty((B, width), dtype=t.float32, device=self.dev)
        hivis_debug_tap(self.ctx, TAPS[name], out)
        return out

    def set_chain_kernel(self, on: bool):
        hivis_set_option(self.ctx, HIVIS_OPT_CHAIN_KERNEL, 1 if on else 0)

    def set_tc_kernel(self, on):
        """False/0: never; True: for every batch size it supports (2 in the C API); "auto"/1: the default."""
        v = 1 if on == "auto" else (2 if on is True else int(on))
        hivis_set_option(self.ctx, HIVIS_OPT_TC_KERNEL, v)

    def set_wait_limit_us(self, us: int):
        hivis_set_option(self.ctx, HIVIS_OPT_WAIT_LIMIT_US, int(us))

    def miss_next_barrier(self):
        """Test aid: the grid barriers of the next draft cannot complete, so its waits run out."""
        hivis_set_option(self.ctx, HIVIS_OPT_DEBUG_MISS_BARRIER, 1)

    def set_tc_prefill(self, on):
        """False: hivis_prefill always works in passes of 16 pairs; True: the default threshold; an int n > 1:
        calls of n pairs or more take the tensor-core path."""
        hivis_set_option(self.ctx, HIVIS_OPT_TC_PREFILL, int(on))

    def set_l2_keep(self, mask: int):
        """Bit p set: the tensor-core chain kernel asks L2 to keep the weights of matrix p (0 FC .. 5 LM head)."""
        hivis_set_option(self.ctx, HIVIS_OPT_L2_KEEP, int(mask))

    def record_phase_times(self, on: bool = True):
        hivis_set_option(self.ctx, HIVIS_OPT_PHASE_TIMES, 1 if on else 0)

    def phase_times(self):
        return hivis_read_phase_times(self.ctx)

    def status(self):
        hivis_status(self.ctx)

    def step_bytes(self, kv_rows):
        return hivis_step_bytes(self.ctx, kv_rows)

    def launch_count(self):
        return hivis_launch_count(self.ctx)


_DTYPES = {}


def _dtype(t) -> int:
    """HIVIS_F32 or HIVIS_BF16, whichever a tensor's element type is."""
    if not _DTYPES:
        import torch
        _DTYPES.update({torch.float32: HIVIS_F32, torch.bfloat16: HIVIS_BF16})
    if t.dtype not in _DTYPES:
        raise TypeError(f"expected a bfloat16 or float32 tensor, not {t.dtype}")
    return _DTYPES[t.dtype]


def _aligned(t):
    """A tensor that is only read, starting on 16 bytes as the library wants it: itself, or a copy of a view that starts elsewhere."""
    return t if t.data_ptr() % 16 == 0 else t.new_empty(t.shape).copy_(t)


def _slots(slots, B):
    if slots is None:
        return None
    if len(slots) != B:
        raise ValueError(f"{len(slots)} slots for {B} sequences")
    return _ints(slots)


def _raw_stream(index: int) -> int:
    """The current stream of a device, without a Stream object around it."""
    import torch
    return torch._C._cuda_getCurrentRawStream(index)


class Kv4Cache:
    """A key/value cache held in 4 bits (include/hivis.h: hivis_kv4_cache) for `n_slots` sequences of up to `max_len` rows
    (rounded up to a multiple of 32).  Rows hold [n_kv_heads, head_dim] keys and values.  Keys, values, queries and outputs start on 16 bytes;
    lists of counts and masks may start anywhere (a view that does not start on 16 bytes is copied)."""

    def __init__(self, n_slots: int, n_kv_heads: int, head_dim: int, max_len: int, device=None):
        import torch
        self.torch = torch
        self.dev = torch.device("cuda", torch.cuda.current_device()) if device is None else torch.device(device)
        if self.dev.index is None:
            self.dev = torch.device("cuda", torch.cuda.current_device())
        self.n_slots, self.n_kv_heads, self.head_dim = int(n_slots), int(n_kv_heads), int(head_dim)
        self.max_len = (int(max_len) + 31) // 32 * 32
        if self.n_slots < 1 or self.n_kv_heads < 1 or self.max_len < 32 or self.head_dim not in (64, 128):
            raise ValueError("a cache has at least one slot, KV head and row, and a head_dim of 64 or 128")
        self.data = torch.zeros(self.n_slots * self.n_kv_heads * self.max_len * self.head_dim * 5 // 4, dtype=torch.uint8, device=self.dev)
        self.c = hivis_kv4_cache(C.sizeof(hivis_kv4_cache), self.n_slots, self.n_kv_heads, self.head_dim, self.max_len,
                                 self.data.data_ptr())
        self._ref, self._scale = C.byref(self.c), self.head_dim ** -0.5

    # (The checks below are written for few Python operations: on short sequences the host is what a call waits for.)
    def _elsewhere(self, *tensors):
        """Whether the cache's device is not the current one; every tensor has to be on it."""
        for t in tensors:
            if t is not None and t.get_device() != self.dev.index:
                raise ValueError(f"the cache is on {self.dev}, a tensor on {t.device}")
        return self.torch.cuda.current_device() != self.dev.index

    def _row_stride(self, t, n_heads, n_rows, name):
        """[n_rows, n_heads, head_dim] with rows that may lie apart -> elements from one row to the next."""
        shape, stride = t.shape, t.stride()
        if len(shape) != 3 or shape[0] != n_rows or shape[1] != n_heads or shape[2] != self.head_dim:
            raise ValueError(f"{name} has shape {tuple(shape)}, expected {(n_rows, n_heads, self.head_dim)}")
        if stride[2] != 1 or (n_heads > 1 and stride[1] != self.head_dim):
            if t.numel():
                raise ValueError(f"the rows of {name} are not contiguous")
        return stride[0] if n_rows > 1 else n_heads * self.head_dim

    def _counts(self, t, B, name):
        if t.dtype is not self.torch.int32 or t.shape != (B,) or (B > 1 and t.stride(0) != 1):
            raise ValueError(f"{name} must be a contiguous int32 tensor of {B} entries")
        return _aligned(t)

    def append(self, k, v, cu_seqlens, start_rows, slots=None):
        """Rows [cu_seqlens[b], cu_seqlens[b + 1]) of k and v ([total, n_kv_heads, head_dim], bf16 or fp32) become rows
        start_rows[b].. (int32 tensor) of slot slots[b] (default b)."""
        if self._elsewhere(k, v, start_rows):
            with self.torch.cuda.device(self.dev):
                return self.append(k, v, cu_seqlens, start_rows, slots)
        B, total = len(cu_seqlens) - 1, int(cu_seqlens[-1])
        ld = self._row_stride(k, self.n_kv_heads, total, "k")
        if self._row_stride(v, self.n_kv_heads, total, "v") != ld or v.dtype is not k.dtype:
            raise ValueError("k and v must have the same type and row stride")
        first = self._counts(start_rows, B, "start_rows")
        _check(lib.hivis_kv4_append(self._ref, B, _slots(slots, B), _ints(cu_seqlens), first.data_ptr(), k.data_ptr(),
                                    v.data_ptr(), _dtype(k), ld, _raw_stream(self.dev.index)))

    def read(self, cu_seqlens, start_rows, slots=None):
        """-> (k, v) fp32 [total, n_kv_heads, head_dim]: what rows start_rows[b].. of the slots stand for.  (Places whose row would lie
        outside the cache are not written: they hold what the allocator left there.)"""
        if self._elsewhere(start_rows):
            with self.torch.cuda.device(self.dev):
                return self.read(cu_seqlens, start_rows, slots)
        t, B = self.torch, len(cu_seqlens) - 1
        shape = (int(cu_seqlens[-1]), self.n_kv_heads, self.head_dim)
        k = t.empty(shape, dtype=t.float32, device=self.dev)
        v = k.new_empty(shape)
        first = self._counts(start_rows, B, "start_rows")
        _check(lib.hivis_kv4_read(self._ref, B, _slots(slots, B), _ints(cu_seqlens), first.data_ptr(), k.data_ptr(),
                                  v.data_ptr(), _raw_stream(self.dev.index)))
        return k, v

    def attention(self, q, rows, n_q=1, scale=None, mask=None, mask_rows=0, slots=None, out=None):
        """q [B * n_q, n_q_heads, head_dim] (bf16 or fp32) over the slots' first rows[b] rows (int32 tensor) -> the same shape
        and type.  Causal over the last n_q rows, or by `mask` (int32 [B, n_q, ceil(mask_rows / 32)]) over the last mask_rows."""
        if self._elsewhere(q, rows, mask, out):
            with self.torch.cuda.device(self.dev):
                return self.attention(q, rows, n_q, scale, mask, mask_rows, slots, out)
        t, B = self.torch, rows.shape[0]
        heads = q.shape[1] if q.dim() == 3 else 0
        q_ld = self._row_stride(q, heads, B * n_q, "q")
        mask_ptr = None
        if mask is not None:
            if mask_rows < 1:
                raise ValueError("a mask covers at least one row: mask_rows says how many")
            if mask.dtype is not t.int32 or tuple(mask.shape) != (B, n_q, (mask_rows + 31) // 32) or not mask.is_contiguous():
                raise ValueError("mask must be a contiguous int32 tensor [B, n_q, ceil(mask_rows / 32)]")
            mask = _aligned(mask)
            mask_ptr = mask.data_ptr()
        counts = self._counts(rows, B, "rows")
        if out is None:
            out = q.new_empty(q.shape)
            out_ld = heads * self.head_dim
        else:
            if out.dtype is not q.dtype:
                raise ValueError("out must have the type of q")
            out_ld = self._row_stride(out, heads, B * n_q, "out")
        _check(lib.hivis_kv4_attention(self._ref, B, _slots(slots, B), counts.data_ptr(), n_q, heads, q.data_ptr(), _dtype(q), q_ld,
                                       self._scale if scale is None else scale, mask_ptr, mask_rows, out.data_ptr(), out_ld,
                                       _raw_stream(self.dev.index)))
        return out


class Logprobs(NamedTuple):
    """What `logprobs` returns; fields that were not asked for are None."""
    logprobs: "object" = None       # fp32 [n_rows, n_ids]
    entropy: "object" = None        # fp32 [n_rows]
    top_ids: "object" = None        # int32 [n_rows, top_n]
    top_logprobs: "object" = None   # fp32 [n_rows, top_n]


def logprobs(logits, ids=None, temperature: float = 1.0, top_n: int = 0, entropy: bool = True) -> Logprobs:
    """Log-probabilities of `ids` (int32 [n_rows, n_ids]) under softmax(logits / temperature), the rows' entropy and their
    `top_n` most probable tokens; logits [n_rows, vocab], bf16 or fp32, rows may lie apart.  include/hivis.h: hivis_logprobs.
    Views may start anywhere; one that does not start on 16 bytes (logits[1:] of an odd vocabulary, say) is copied first."""
    import torch
    shape, stride, index = logits.shape, logits.stride(), logits.get_device()
    if len(shape) != 2 or (stride[1] != 1 and shape[1] > 1):
        raise ValueError(f"logits must be [n_rows, vocab] with contiguous rows, not {tuple(shape)}")
    if index < 0:
        raise ValueError("logits must be a CUDA tensor")
    if torch.cuda.current_device() != index:
        with torch.cuda.device(index):
            return logprobs(logits, ids, temperature, top_n, entropy)
    n, vocab = shape
    n_ids = 0
    if ids is not None:
        if ids.dtype is not torch.int32 or ids.dim() != 2 or ids.shape[0] != n or ids.get_device() != index or not ids.is_contiguous():
            raise ValueError("ids must be a contiguous int32 tensor [n_rows, n_ids] beside the logits")
        n_ids = ids.shape[1]
        ids = _aligned(ids)
    logits = _aligned(logits)
    stride = logits.stride()
    lp = h = top = top_lp = None
    p_lp = p_h = p_top = p_top_lp = None
    f32 = torch.float32
    if n_ids:
        lp = logits.new_empty((n, n_ids), dtype=f32)
        p_lp = lp.data_ptr()
    if entropy:
        h = logits.new_empty((n,), dtype=f32)
        p_h = h.data_ptr()
    if top_n > 0:
        top = logits.new_empty((n, top_n), dtype=torch.int32)
        top_lp = logits.new_empty((n, top_n), dtype=f32)
        p_top, p_top_lp = top.data_ptr(), top_lp.data_ptr()
    _check(lib.hivis_logprobs(n, vocab, logits.data_ptr(), _dtype(logits), stride[0] if n > 1 else vocab, temperature,
                              ids.data_ptr() if n_ids else None, n_ids, top_n, p_lp, p_h, p_top, p_top_lp, _raw_stream(index)))
    return Logprobs(lp, h, top, top_lp)
