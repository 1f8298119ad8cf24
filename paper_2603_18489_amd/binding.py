"""Thin ctypes binding of libec.so (include/ec.h).  Argument marshalling only: every step of the
denoising path runs in the library's HIP kernels.  PyTorch supplies device memory and the stream.
"""
from __future__ import annotations

import ctypes as C
import os
from typing import Dict, List, NamedTuple, Optional, Sequence

import numpy as np

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libec.so")

EC_MAX_N = 32
EC_MAX_BLOCK = 128
EC_MAX_BATCH = 64
EC_F32, EC_BF16, EC_FP8W, EC_MXFP4W = 0, 1, 2, 3
EC_FULL, EC_PARTIAL, EC_AUTO = 0, 1, 2
EC_GATE_MAX_ENTROPY, EC_GATE_ENTROPY_SUM, EC_GATE_MAX_CONFIDENCE = 0, 1, 2
EC_SCHED_BLOCKS, EC_SCHED_SLIDING = 0, 1
EC_OK, EC_ERR_ARG, EC_ERR_CONFIG, EC_ERR_WORKSPACE, EC_ERR_STATE, EC_ERR_HIP = 0, -1, -2, -3, -4, -5
EC_ERR_HOST_MEMORY = -6
EC_ERR_NONFINITE = -7
(EC_K_EMBED, EC_K_NORM, EC_K_QKV, EC_K_ROPE_KV, EC_K_ATTN, EC_K_OPROJ, EC_K_GATEUP, EC_K_SWIGLU,
 EC_K_DOWN, EC_K_LMHEAD, EC_K_VOCAB_REDUCE, EC_K_DECIDE, EC_K_COUNT) = range(13)
EC_T_F32, EC_T_BF16, EC_T_MXFP4, EC_T_E4M3 = 0, 1, 2, 3
KERNEL_CLASS_NAMES = ["embed", "norm", "qkv", "rope_kv", "attn", "oproj", "gateup", "swiglu",
                      "down", "lmhead", "vocab_reduce", "decide"]
(EC_DBG_LOGITS, EC_DBG_KCACHE, EC_DBG_VCACHE, EC_DBG_X, EC_DBG_MASKED, EC_DBG_HIST, EC_DBG_ROWS,
 EC_DBG_ROW_STATS) = range(8)

EXPORTS = ["ec_workspace_bytes", "ec_init", "ec_reset", "ec_step", "ec_step_forced", "ec_debug_keep_logits",
           "ec_step_forced_batch", "ec_generate", "ec_profile_enable", "ec_profile_read",
           "ec_debug_read", "ec_debug_read_seq", "ec_debug_block_shape", "ec_debug_attn_tiles", "ec_debug_meeting",
           "ec_debug_mx_blocks", "ec_destroy", "ec_strerror", "ec_last_error",
           "ec_row_entropy_workspace_bytes", "ec_row_entropy", "ec_row_entropy_noalloc",
           "ec_row_sample_workspace_bytes", "ec_row_sample", "ec_mx_quantize", "ec_mx_dequantize",
           "ec_mx_packed_bytes", "ec_mx_pack", "ec_mx_linear_workspace_bytes", "ec_mx_linear",
           "ec_rotary_frequencies", "ec_rotary", "ec_kv_bytes", "ec_kv_write", "ec_kv_read",
           "ec_kv_attention_workspace_bytes", "ec_kv_attention"]


class ec_model_cfg(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("n_layers", "d_model", "n_heads", "n_kv_heads",
                                         "head_dim", "d_ffn", "vocab", "mask_id")] + \
               [(n, C.c_float) for n in ("rms_eps", "rope_base", "logit_scale")] + \
               [("dtype", C.c_int32)]


QUANT_MATRICES = ("wq", "wk", "wv", "wo", "w_gate", "w_up", "w_down")


class ec_weights(C.Structure):
    _fields_ = [("tok_emb", C.c_void_p), ("lm_head", C.c_void_p), ("final_norm", C.c_void_p)] + \
               [(n, C.POINTER(C.c_void_p)) for n in ("attn_norm", "wq", "wk", "wv", "wo",
                                                      "mlp_norm", "w_gate", "w_up", "w_down")] + \
               [("lm_head_scale", C.c_void_p)] + \
               [(n + "_scale", C.POINTER(C.c_void_p)) for n in QUANT_MATRICES] + \
               [("lm_head_mx", C.c_void_p)] + [(n + "_mx", C.POINTER(C.c_void_p)) for n in QUANT_MATRICES]


class ec_decode_cfg(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("batch", "gen_len", "block", "k_recent",
                                         "tokens_per_step")] + \
               [("tau", C.c_float), ("conf_threshold", C.c_float), ("gate_metric", C.c_int32),
                ("schedule", C.c_int32)]


class ec_step_result(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("n_unmasked", "done", "mode_run", "next_mode",
                                         "n_query_rows", "step_index", "n_block_rows",
                                         "n_recent_next")] + \
               [("max_entropy", C.c_float),
                ("positions", C.c_int32 * EC_MAX_N), ("tokens", C.c_int32 * EC_MAX_N),
                ("entropy", C.c_float * EC_MAX_N), ("confidence", C.c_float * EC_MAX_N)]

    def as_dict(self) -> dict:
        n = self.n_unmasked
        return {"n_unmasked": n, "done": bool(self.done), "mode_run": self.mode_run,
                "next_mode": self.next_mode, "n_query_rows": self.n_query_rows,
                "step_index": self.step_index, "n_block_rows": self.n_block_rows,
                "n_recent_next": self.n_recent_next, "max_entropy": float(self.max_entropy),
                "positions": list(self.positions[:n]), "tokens": list(self.tokens[:n]),
                "entropy": list(self.entropy[:n]), "confidence": list(self.confidence[:n])}


class ec_sample_cfg(C.Structure):
    _fields_ = [("temperature", C.c_float), ("top_k", C.c_int32), ("top_p", C.c_float), ("min_p", C.c_float)]


class ec_rotary_cfg(C.Structure):
    _fields_ = [("dim", C.c_int32)] + [(n, C.c_double) for n in ("base", "factor", "original", "low", "high")]


class ec_kv_cache(C.Structure):
    _fields_ = [("data", C.c_void_p)] + [(n, C.c_int32) for n in ("type", "pages", "page", "kv_heads", "head_dim")]


class ec_kv_attention_cfg(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("rows", "heads", "seqs", "max_rows", "max_keys", "table_pages", "prefix_pages",
                                         "prefix_len", "causal")] + [("scale", C.c_float), ("table_ld", C.c_size_t)]


class ec_gen_stats(C.Structure):
    _fields_ = [("steps", C.c_int32), ("full_steps", C.c_int32), ("partial_steps", C.c_int32),
                ("tokens", C.c_int32), ("rows_recomputed", C.c_int64), ("ms_total", C.c_double)]


class ec_profile(C.Structure):
    _fields_ = [("ms", C.c_double * EC_K_COUNT), ("launches", C.c_int64 * EC_K_COUNT),
                ("steps", C.c_int64)]


_lib = None


def load_library() -> C.CDLL:
    """Loads libec.so; raises if it has not been built (there is no fallback path)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} is missing: run `python -m paper_2603_18489_amd.build` "
                           "(or __graft_entry__.build()) first")
    lib = C.CDLL(LIB_PATH)
    vp, i32p = C.c_void_p, C.POINTER(C.c_int32)
    lib.ec_workspace_bytes.restype = C.c_size_t
    lib.ec_workspace_bytes.argtypes = [C.POINTER(ec_model_cfg), C.POINTER(ec_decode_cfg), i32p]
    lib.ec_init.restype = C.c_int
    lib.ec_init.argtypes = [C.POINTER(vp), C.POINTER(ec_model_cfg), C.POINTER(ec_weights),
                            C.POINTER(ec_decode_cfg), i32p, i32p, vp, C.c_size_t, vp]
    lib.ec_reset.restype = C.c_int
    lib.ec_reset.argtypes = [vp, i32p]
    lib.ec_step.restype = C.c_int
    lib.ec_step.argtypes = [vp, C.c_int, C.POINTER(ec_step_result)]
    lib.ec_step_forced.restype = C.c_int
    lib.ec_step_forced.argtypes = [vp, C.c_int, C.c_int32, i32p, i32p, C.POINTER(ec_step_result)]
    lib.ec_step_forced_batch.restype = C.c_int
    lib.ec_step_forced_batch.argtypes = [vp, i32p, i32p, i32p, i32p, C.POINTER(ec_step_result)]
    lib.ec_generate.restype = C.c_int
    lib.ec_generate.argtypes = [vp, i32p, C.POINTER(ec_gen_stats)]
    lib.ec_profile_enable.restype = C.c_int
    lib.ec_profile_enable.argtypes = [vp, C.c_int]
    lib.ec_profile_read.restype = C.c_int
    lib.ec_profile_read.argtypes = [vp, C.POINTER(ec_profile)]
    lib.ec_debug_keep_logits.restype = C.c_int
    lib.ec_debug_keep_logits.argtypes = [vp, C.c_int]
    lib.ec_debug_meeting.restype = C.c_int
    lib.ec_debug_meeting.argtypes = [vp, C.c_int32, C.c_int]
    lib.ec_debug_read.restype = C.c_int
    lib.ec_debug_read.argtypes = [vp, C.c_int, C.c_int, vp, C.c_size_t]
    lib.ec_debug_read_seq.restype = C.c_int
    lib.ec_debug_read_seq.argtypes = [vp, C.c_int, C.c_int, C.c_int, vp, C.c_size_t]
    lib.ec_debug_block_shape.restype = C.c_int
    lib.ec_debug_block_shape.argtypes = [C.POINTER(ec_model_cfg), C.c_int, C.c_int32, C.c_int32,
                                         C.POINTER(C.c_int32 * 3)]
    lib.ec_debug_attn_tiles.restype = C.c_int
    lib.ec_debug_attn_tiles.argtypes = [C.POINTER(ec_model_cfg), C.c_int32, i32p, i32p, i32p]
    lib.ec_row_entropy_workspace_bytes.restype = C.c_size_t
    lib.ec_row_entropy_workspace_bytes.argtypes = [C.c_int32, C.c_int32]
    lib.ec_row_entropy.restype = C.c_int
    lib.ec_row_entropy.argtypes = [vp, C.c_int32, C.c_int32, C.c_size_t, vp, vp, C.c_size_t, vp]
    lib.ec_row_entropy_noalloc.restype = C.c_int
    lib.ec_row_entropy_noalloc.argtypes = [vp, C.c_int32, C.c_int32, C.c_size_t, vp, vp]
    lib.ec_row_sample_workspace_bytes.restype = C.c_size_t
    lib.ec_row_sample_workspace_bytes.argtypes = [C.c_int32, C.c_int32]
    lib.ec_row_sample.restype = C.c_int
    lib.ec_row_sample.argtypes = [vp, C.c_int32, C.c_int32, C.c_int32, C.c_size_t, vp, C.POINTER(ec_sample_cfg),
                                  vp, vp, vp, C.c_size_t, vp]
    lib.ec_mx_quantize.restype = C.c_int
    lib.ec_mx_quantize.argtypes = [vp, C.c_int32, C.c_int64, C.c_int32, C.c_size_t, vp, vp, vp]
    lib.ec_mx_dequantize.restype = C.c_int
    lib.ec_mx_dequantize.argtypes = [vp, vp, C.c_int64, C.c_int32, vp, C.c_int32, C.c_size_t, vp]
    lib.ec_mx_packed_bytes.restype = C.c_size_t
    lib.ec_mx_packed_bytes.argtypes = [C.c_int32, C.c_int32]
    lib.ec_mx_pack.restype = C.c_int
    lib.ec_mx_pack.argtypes = [vp, vp, C.c_int32, C.c_int32, vp, C.c_size_t, vp]
    lib.ec_mx_linear_workspace_bytes.restype = C.c_size_t
    lib.ec_mx_linear_workspace_bytes.argtypes = [C.c_int32, C.c_int64, C.c_int32, C.c_int32]
    lib.ec_debug_mx_blocks.restype = C.c_int
    lib.ec_debug_mx_blocks.argtypes = [C.c_int32, C.c_int64, C.c_int32, C.c_int32, i32p]
    lib.ec_mx_linear.restype = C.c_int
    lib.ec_mx_linear.argtypes = [vp, vp, C.c_int32, C.c_int64, C.c_size_t, vp, C.c_int32, C.c_int32, vp, C.c_int32,
                                 C.c_size_t, vp, C.c_size_t, vp]
    lib.ec_rotary_frequencies.restype = C.c_int
    lib.ec_rotary_frequencies.argtypes = [C.POINTER(ec_rotary_cfg), vp]
    lib.ec_rotary.restype = C.c_int
    lib.ec_rotary.argtypes = [vp, C.c_int32, C.c_int64, C.c_int32, C.c_int32, C.c_size_t, C.c_size_t, vp, vp, C.c_int32, C.c_int32,
                              C.c_float, C.c_int32, vp, C.c_size_t, C.c_size_t, vp]
    lib.ec_kv_bytes.restype = C.c_size_t
    lib.ec_kv_bytes.argtypes = [C.POINTER(ec_kv_cache)]
    lib.ec_kv_write.restype = C.c_int
    lib.ec_kv_write.argtypes = [C.POINTER(ec_kv_cache), vp, vp, C.c_int32, C.c_int32] + [C.c_size_t] * 4 + [vp, vp]
    lib.ec_kv_read.restype = C.c_int
    lib.ec_kv_read.argtypes = [C.POINTER(ec_kv_cache), vp, C.c_int32, vp, vp, C.c_int32] + [C.c_size_t] * 4 + [vp]
    lib.ec_kv_attention_workspace_bytes.restype = C.c_size_t
    lib.ec_kv_attention_workspace_bytes.argtypes = [C.POINTER(ec_kv_cache), C.POINTER(ec_kv_attention_cfg)]
    lib.ec_kv_attention.restype = C.c_int
    lib.ec_kv_attention.argtypes = [C.POINTER(ec_kv_cache), C.POINTER(ec_kv_attention_cfg), vp, C.c_size_t, C.c_size_t, vp, vp, vp, vp,
                                    vp, C.c_size_t, C.c_size_t, vp, C.c_size_t, vp]
    lib.ec_destroy.restype = None
    lib.ec_destroy.argtypes = [vp]
    lib.ec_strerror.restype = C.c_char_p
    lib.ec_strerror.argtypes = [C.c_int]
    lib.ec_last_error.restype = C.c_char_p
    lib.ec_last_error.argtypes = [vp]
    _lib = lib
    return lib


class EcError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"ec error {code} ({load_library().ec_strerror(code).decode()}): {msg}")
        self.code = code


def model_cfg_struct(cfg) -> ec_model_cfg:
    return ec_model_cfg(cfg.n_layers, cfg.d_model, cfg.n_heads, cfg.n_kv_heads, cfg.head_dim,
                        cfg.d_ffn, cfg.vocab, cfg.mask_id, cfg.rms_eps, cfg.rope_base,
                        cfg.logit_scale, {"f32": EC_F32, "bf16": EC_BF16, "fp8w": EC_FP8W,
                                          "mxfp4w": EC_MXFP4W}[cfg.dtype])


def decode_cfg_struct(dec) -> ec_decode_cfg:
    return ec_decode_cfg(dec.batch, dec.gen_len, dec.block, dec.k_recent, dec.tokens_per_step,
                         dec.tau, getattr(dec, "conf_threshold", 0.0),
                         getattr(dec, "gate_metric", 0), getattr(dec, "schedule", 0))


def _i32(a) -> np.ndarray:
    return np.ascontiguousarray(np.asarray(a, dtype=np.int32))


def _i32p(a: np.ndarray):
    return a.ctypes.data_as(C.POINTER(C.c_int32))


def weights_to_device(cfg, w: Dict[str, object], device="cuda:0") -> Dict[str, object]:
    """Uploads host weights (float32, uint16 bfloat16 bit patterns, or matrices as codes and scales) as
    torch device tensors; a matrix `name` in e4m3 becomes the uint8 tensor `name` and the float32 tensor
    `name_scale`, one in 4 bits the uint8 tensors `name` and `name_mx`.  For a model whose `dtype` is "mxfp4w"
    matrices that are still float32 or bfloat16 are brought to 4 bits on the device (mxfp4_quantize)."""
    import torch

    def up(a: np.ndarray):
        if a.dtype == np.uint16:
            return torch.from_numpy(a.view(np.int16)).to(device).view(torch.bfloat16)
        return torch.from_numpy(a).to(device)

    out: Dict[str, object] = {}
    for k, v in w.items():
        items = v if isinstance(v, list) else [v]
        if cfg.dtype == "mxfp4w" and (k in QUANT_MATRICES or k == "lm_head"):
            pairs = [(up(x.codes), up(x.scales)) if hasattr(x, "codes") else mxfp4_quantize(up(x)) for x in items]
            out[k] = [c for c, _ in pairs] if isinstance(v, list) else pairs[0][0]
            out[k + "_mx"] = [s for _, s in pairs] if isinstance(v, list) else pairs[0][1]
        elif hasattr(items[0], "codes"):
            codes, scales = [up(x.codes) for x in items], [up(x.scale) for x in items]
            out[k] = codes if isinstance(v, list) else codes[0]
            out[k + "_scale"] = scales if isinstance(v, list) else scales[0]
        else:
            out[k] = [up(x) for x in v] if isinstance(v, list) else up(v)
    return out


def block_shape(cfg, product: int, list_rows: int, rows: int):
    """ec_debug_block_shape: (rows, output features, K ranges) of the blocks of a many-row product."""
    mc, shape = model_cfg_struct(cfg), (C.c_int32 * 3)()
    rc = load_library().ec_debug_block_shape(C.byref(mc), product, list_rows, rows, C.byref(shape))
    if rc != EC_OK:
        raise EcError(rc, load_library().ec_last_error(None).decode())
    return tuple(shape)


def attn_tiles(cfg, rows: Sequence[int], positions: Sequence[int]) -> int:
    """ec_debug_attn_tiles: row tiles to a block of the attention of sequences with so many rows and positions."""
    mc, tiles = model_cfg_struct(cfg), C.c_int32()
    rc = load_library().ec_debug_attn_tiles(C.byref(mc), len(rows), _i32p(_i32(rows)), _i32p(_i32(positions)),
                                            C.byref(tiles))
    if rc != EC_OK:
        raise EcError(rc, load_library().ec_last_error(None).decode())
    return tiles.value


def mx_blocks(x_type: int, rows: int, n: int, k: int):
    """ec_debug_mx_blocks: (rows, features, ranges of K) of the blocks of a 4-bit product."""
    shape = (C.c_int32 * 3)()
    rc = load_library().ec_debug_mx_blocks(x_type, rows, n, k, shape)
    if rc != EC_OK:
        raise EcError(rc, load_library().ec_last_error(None).decode())
    return tuple(shape)


def _raw_stream(torch, stream, device: int) -> int:
    """hipStream_t of `stream`, or of `device`'s current stream (where torch has the lookup that makes
    no stream object: 0.4 us instead of 2.7, in a call of about 8)."""
    if stream is None:
        lookup = getattr(torch._C, "_cuda_getCurrentRawStream", None)
        if lookup is not None:
            return lookup(device)
        stream = torch.cuda.current_stream(device)
    return stream.cuda_stream


def row_entropy(logits, stream=None):
    """ec_row_entropy on a float32 CUDA tensor [rows, vocab] (row stride = logits.stride(0)):
    returns a float32 CUDA tensor [rows, 4] (token, confidence, entropy, max logit).  The
    workspace is a torch allocation.  Without `stream` the call is ordered on the current stream
    like any torch operation; with one it is enqueued there and waited for."""
    import torch
    dev, current = logits.get_device(), torch.cuda.current_device()
    if 0 <= dev != current:   # (the kernels run where the logits are)
        with torch.cuda.device(dev):
            return row_entropy(logits, stream)
    if stream is not None:
        # Result and workspace come from the pool of the stream that the kernels run on: the current
        # stream's pool may hand out the workspace of an earlier call whose kernels are still pending.
        here = torch.cuda.current_stream()
        with torch.cuda.stream(stream):
            stats = row_entropy(logits)
        stream.synchronize()
        if stats.shape[0] and stream != here:
            stats.record_stream(here)    # the caller goes on with it there
        return stats
    lib = _lib or load_library()
    rows, vocab = logits.shape
    assert logits.dtype == torch.float32 and logits.stride(1) == 1
    stats = torch.empty((rows, 4), dtype=torch.float32, device=logits.device)
    if rows == 0:
        return stats         # (an empty tensor has no address to hand over)
    need = lib.ec_row_entropy_workspace_bytes(rows, vocab)
    # (both belong to the current stream: the allocator hands their memory on behind this call only)
    ws = torch.empty(max(need, 256), dtype=torch.uint8, device=logits.device)
    rc = lib.ec_row_entropy(logits.data_ptr(), rows, vocab, logits.stride(0) if rows > 1 else vocab,
                            stats.data_ptr(), ws.data_ptr(), need, _raw_stream(torch, None, current))
    if rc != EC_OK:
        raise EcError(rc, lib.ec_last_error(None).decode())
    return stats


def row_entropy_noalloc(logits, stats, stream=None):
    """ec_row_entropy_noalloc: `stats` is a caller-provided float32 CUDA tensor [rows, 4]; the
    call itself allocates nothing.  Enqueued on `stream` (default: current), not synchronised."""
    import torch
    dev, current = logits.get_device(), torch.cuda.current_device()
    if 0 <= dev != current:
        with torch.cuda.device(dev):
            return row_entropy_noalloc(logits, stats, stream)
    lib = _lib or load_library()
    rows, vocab = logits.shape
    assert logits.dtype == torch.float32 and logits.stride(1) == 1
    assert stats.dtype == torch.float32 and stats.is_contiguous() and stats.shape == (rows, 4)
    rc = lib.ec_row_entropy_noalloc(logits.data_ptr(), rows, vocab,
                                    logits.stride(0) if rows > 1 else vocab, stats.data_ptr(),
                                    _raw_stream(torch, stream, current))
    if rc != EC_OK:
        raise EcError(rc, lib.ec_last_error(None).decode())


_INT_MAX = 2 ** 31 - 1


def _need(ok: bool, what: str) -> None:
    if not ok:
        raise ValueError(what)


def _place(stream, call, first, *others):
    """Runs call() where the tensors are: on their device, and on `stream` if one is given, whose pool then owns what it
    allocates and which is waited for (as row_entropy does); on the device's current stream otherwise."""
    import torch
    dev = first.get_device()
    if dev < 0:
        raise ValueError("tensors must be on one GPU")
    for t in others:
        if t.get_device() != dev:
            raise ValueError("tensors must be on one GPU")
    if dev != torch.cuda.current_device():
        with torch.cuda.device(dev):
            return _place(stream, call, first, *others)
    if stream is None:
        return call(_raw_stream(torch, None, dev))
    here = torch.cuda.current_stream()
    with torch.cuda.stream(stream):
        out = call(_raw_stream(torch, None, dev))
    stream.synchronize()
    if stream != here:
        for t in out if isinstance(out, tuple) else (out,):
            if hasattr(t, "record_stream"):
                t.record_stream(here)    # the caller goes on with it there
    return out


def _workspace(torch, size: int, device):
    """Workspace and its address, which belong to the current stream; none where none is needed."""
    if not size:
        return None, None
    ws = torch.empty((size,), dtype=torch.uint8, device=device)
    return ws, ws.data_ptr()


def _done(lib, rc: int) -> None:
    if rc != EC_OK:
        raise EcError(rc, lib.ec_last_error(None).decode())


def _plain_type(dtype) -> int:
    import torch
    _need(dtype in (torch.float32, torch.bfloat16), "float32 or bfloat16 is needed")
    return EC_T_F32 if dtype == torch.float32 else EC_T_BF16


def _rows_of(x):
    """rows, columns and row stride of a matrix whose columns are next to each other"""
    _need(x.dim() == 2, "a matrix is needed")
    rows, cols = x.shape
    _need(x.stride(1) == 1 or cols <= 1, "the columns of a row must be next to each other")
    ld = x.stride(0) if rows > 1 else cols
    _need(ld >= cols, "rows must not overlap")
    _need(max(rows, cols) <= _INT_MAX, "at most 2^31 - 1 rows and columns")   # (what the calls' arguments hold)
    return rows, cols, ld


def row_sample(logits, uniforms, temperature: float = 1.0, top_k: int = 0, top_p: float = 1.0, min_p: float = 0.0,
               stream=None):
    """ec_row_sample: a token drawn from each row of a float32 or bfloat16 CUDA matrix [rows, vocab], from the numbers
    `uniforms` (float32 [rows], in [0, 1)).  Returns an int32 tensor [rows] of tokens and a float32 tensor [rows, 4]
    (probability among the kept tokens, among all, number kept, share of the probability kept).  Mask logits with -inf rather than with
    low finite numbers: long rows with filters cost less so.  `stream` as for row_entropy; no gradients."""
    import torch
    kind = _plain_type(logits.dtype)
    rows, vocab, ld = _rows_of(logits)
    _need(uniforms.dtype == torch.float32 and uniforms.shape == (rows,) and (rows <= 1 or uniforms.stride(0) == 1),
          "uniforms must be float32 [rows]")
    lib = _lib or load_library()
    cfg = ec_sample_cfg(temperature, max(-1, min(top_k, _INT_MAX)), top_p, min_p)

    def call(raw):
        tokens = torch.empty((rows,), dtype=torch.int32, device=logits.device)
        stats = torch.empty((rows, 4), dtype=torch.float32, device=logits.device)
        size = lib.ec_row_sample_workspace_bytes(rows, vocab)
        ws, at = _workspace(torch, size, logits.device)
        _done(lib, lib.ec_row_sample(logits.data_ptr(), kind, rows, vocab, ld, uniforms.data_ptr(), C.byref(cfg),
                                     tokens.data_ptr(), stats.data_ptr(), at, size, raw))
        return tokens, stats
    return _place(stream, call, logits, uniforms)


class Mxfp4(NamedTuple):
    """A matrix in microscaled 4-bit floating point: uint8 codes [rows, k/2] (an even k in the low four bits) and uint8
    scales [rows, k/32] (2^(s - 127) for 32 values; 255: NaN)."""
    codes: object
    scales: object


class Mxfp4Matrix(NamedTuple):
    """An n x k matrix as mxfp4_linear reads it."""
    data: object
    n: int
    k: int


def _mx_of(q):
    import torch
    codes, scales = q
    _need(codes.dtype == torch.uint8 and scales.dtype == torch.uint8, "codes and scales must be uint8")
    _need(codes.dim() == 2 and scales.dim() == 2 and codes.shape[0] == scales.shape[0] and
          codes.shape[1] == 16 * scales.shape[1], "codes [rows, k/2] and scales [rows, k/32] are needed")
    _need(codes.is_contiguous() and scales.is_contiguous(), "codes and scales must be contiguous")
    _need(max(codes.shape[0], 2 * codes.shape[1]) <= _INT_MAX, "at most 2^31 - 1 rows and columns")
    return codes, scales, codes.shape[0], 2 * codes.shape[1]


def mxfp4_quantize(x, stream=None) -> Mxfp4:
    """ec_mx_quantize: a float32 or bfloat16 CUDA matrix [rows, k] (k a multiple of 32) in 4 bits."""
    import torch
    kind = _plain_type(x.dtype)
    rows, k, ld = _rows_of(x)
    lib = _lib or load_library()

    def call(raw):
        codes = torch.empty((rows, k // 2), dtype=torch.uint8, device=x.device)
        scales = torch.empty((rows, k // 32), dtype=torch.uint8, device=x.device)
        _done(lib, lib.ec_mx_quantize(x.data_ptr(), kind, rows, k, ld, codes.data_ptr(), scales.data_ptr(), raw))
        return Mxfp4(codes, scales)
    return _place(stream, call, x)


def mxfp4_dequantize(q: Mxfp4, dtype=None, stream=None):
    """ec_mx_dequantize: the values of a 4-bit matrix, float32 (the default) or bfloat16; exact in either."""
    import torch
    dtype = torch.float32 if dtype is None else dtype
    kind = _plain_type(dtype)
    codes, scales, rows, k = _mx_of(q)
    lib = _lib or load_library()

    def call(raw):
        out = torch.empty((rows, k), dtype=dtype, device=codes.device)
        _done(lib, lib.ec_mx_dequantize(codes.data_ptr(), scales.data_ptr(), rows, k, out.data_ptr(), kind, k, raw))
        return out
    return _place(stream, call, codes, scales)


def mxfp4_pack(q: Mxfp4, stream=None) -> Mxfp4Matrix:
    """ec_mx_pack: lays a 4-bit matrix [n, k] out for mxfp4_linear, once."""
    import torch
    codes, scales, n, k = _mx_of(q)
    lib = _lib or load_library()

    def call(raw):
        size = lib.ec_mx_packed_bytes(n, k)
        data = torch.empty((max(size, 256),), dtype=torch.uint8, device=codes.device)
        _done(lib, lib.ec_mx_pack(codes.data_ptr(), scales.data_ptr(), n, k, data.data_ptr(), size, raw))
        return Mxfp4Matrix(data, n, k)
    return _place(stream, call, codes, scales)


def mxfp4_linear(x, w: Mxfp4Matrix, dtype=None, stream=None):
    """ec_mx_linear: x W^T, float32 or bfloat16 (the default), for x a bfloat16 CUDA matrix [rows, k] (row stride a multiple
    of 8 elements) or one in 4 bits (Mxfp4).  For inference: the result carries no gradient, whatever x requires."""
    import torch
    dtype = torch.bfloat16 if dtype is None else dtype
    kind = _plain_type(dtype)
    if isinstance(x, tuple):
        codes, scales, rows, k = _mx_of(x)
        tensors, x_kind, ld, x_scales = (codes, scales, w.data), EC_T_MXFP4, k, scales.data_ptr()
    else:
        _need(x.dtype == torch.bfloat16, "x must be bfloat16 or Mxfp4")
        rows, k, ld = _rows_of(x)
        ld = ld if rows > 1 else (k + 7) // 8 * 8
        tensors, x_kind, x_scales = (x, w.data), EC_T_BF16, None
    _need(k == w.k, "x has another k than the matrix")
    _need(w.data.dtype == torch.uint8 and w.data.is_contiguous(), "data must be contiguous uint8, as mxfp4_pack makes it")
    lib = _lib or load_library()

    def call(raw):
        # (groups of 64 rows x 128 k, as ec_mx_packed_bytes counts them, without another call)
        _need(w.data.numel() >= (w.n + 63) // 64 * ((k + 127) // 128) * 4352, "data is not a matrix [n, k] of mxfp4_pack")
        y = torch.empty((rows, w.n), dtype=dtype, device=w.data.device)
        size = lib.ec_mx_linear_workspace_bytes(x_kind, rows, w.n, k)
        ws, at = _workspace(torch, size, w.data.device)
        _done(lib, lib.ec_mx_linear(tensors[0].data_ptr(), x_scales, x_kind, rows, ld, w.data.data_ptr(), w.n, k,
                                    y.data_ptr(), kind, w.n, at, size, raw))
        return y
    return _place(stream, call, *tensors)


def _heads_of(x, what: str):
    """rows, heads, components and the two strides of a tensor [rows, heads, head_dim] whose components are next to each other"""
    if x.dim() != 3:
        raise ValueError(f"{what} must be [rows, heads, head_dim]")
    rows, heads, dim = x.shape
    ld, ld_head, one = x.stride()
    if rows > _INT_MAX or heads > _INT_MAX or dim > _INT_MAX:
        raise ValueError("at most 2^31 - 1 rows, heads and components")
    if one != 1 and dim > 1 and rows > 0:
        raise ValueError("the components of a head must be next to each other")
    return rows, heads, dim, ld if rows > 1 else 0, ld_head if heads > 1 else 0


def _ints(torch, t, size, what: str):
    if t.dtype != torch.int32 or t.shape != size or not t.is_contiguous():
        raise ValueError(f"{what} must be contiguous int32 {list(size)}")


class RotaryPlan(NamedTuple):
    """How rotary() turns rows: turns (float64 [dim/2], on the GPU) of each pair a position."""
    turns: object
    dim: int
    interleaved: bool
    amplitude: float


def rotary_plan(dim: int, base: float = 10000.0, interleaved: bool = False, factor: float = 1.0, original: float = 0.0,
                low: float = 1.0, high: float = 32.0, amplitude: float = 1.0, device="cuda") -> RotaryPlan:
    """ec_rotary_frequencies: theta_i = base^(-2 i / dim) for the first `dim` components of a head, divided by `factor` for a longer
    context - all of them (original 0), or those that turn fewer than `high` times over `original` positions (wholly below `low` turns)."""
    import torch
    _need(0 < dim <= _INT_MAX, "dim must be positive")
    lib = _lib or load_library()
    turns = np.zeros(dim // 2 + 1)
    _done(lib, lib.ec_rotary_frequencies(C.byref(ec_rotary_cfg(dim, base, factor, original, low, high)), turns.ctypes.data))
    return RotaryPlan(torch.from_numpy(turns[:-1].copy()).to(device), dim, bool(interleaved), float(amplitude))


def rotary(x, positions, plan: RotaryPlan, inverse: bool = False, out=None, stream=None):
    """ec_rotary: a float32 or bfloat16 CUDA tensor [rows, heads, head_dim] (queries and keys beside each other, say) turned by the rows'
    positions (int32 [rows]).  `out` may be x itself.  The result carries no gradient, whatever x requires: rotary(gradient, positions, plan,
    inverse=True) is x's."""
    import torch
    kind = _plain_type(x.dtype)
    rows, heads, dim, ld, ld_head = _heads_of(x, "x")
    _ints(torch, positions, (rows,), "positions")
    turns, turning, interleaved, amplitude = plan
    if turns.dtype != torch.float64 or turns.shape != (turning // 2,) or not turns.is_contiguous():
        raise ValueError("turns must be contiguous float64 [dim/2], as rotary_plan makes them")
    if out is not None:
        _need(out.dtype == x.dtype and out.shape == x.shape, "out must have x's shape and type")
    lib = _lib or load_library()

    def call(raw):
        if out is None:
            y, to, to_head = torch.empty((rows, heads, dim), dtype=x.dtype, device=x.device), heads * dim, dim
        else:
            y = out
            _, _, _, to, to_head = _heads_of(y, "out")
        _done(lib, lib.ec_rotary(x.data_ptr(), kind, rows, heads, dim, ld, ld_head, positions.data_ptr(), turns.data_ptr(), turning,
                                 interleaved, amplitude, inverse, y.data_ptr(), to, to_head, raw))
        return y
    if out is None:
        return _place(stream, call, x, positions, turns)
    return _place(stream, call, x, positions, turns, out)


class KvCache(NamedTuple):
    """A paged cache of keys and values of one layer (ec_kv_cache): `data` uint8 on the GPU, laid out by the library; token t of page p is
    slot p * page + t."""
    data: object
    kind: int
    pages: int
    page: int
    kv_heads: int
    head_dim: int


def kv_cache(pages: int, kv_heads: int, head_dim: int, page: int = 64, dtype=None, device="cuda") -> KvCache:
    """A cache of zeros for pages * page tokens, in e4m3 with a power of two to a token and head (torch.float8_e4m3fn, the default) or in
    torch.bfloat16."""
    import torch
    _need(dtype in (None, torch.float8_e4m3fn, torch.bfloat16), "a cache is float8_e4m3fn or bfloat16")
    _need(max(pages, kv_heads, head_dim, page) <= _INT_MAX, "at most 2^31 - 1 tokens")
    lib = _lib or load_library()
    kind = EC_T_BF16 if dtype == torch.bfloat16 else EC_T_E4M3
    size = lib.ec_kv_bytes(C.byref(ec_kv_cache(None, kind, pages, page, kv_heads, head_dim)))
    _need(size > 0, "page must be 32, 64, 128 or 256, head_dim 64 or 128, kv_heads at most 1024, and the tokens fewer than 2^31")
    return KvCache(torch.zeros((size,), dtype=torch.uint8, device=device), kind, pages, page, kv_heads, head_dim)


def _cache_struct(torch, cache: KvCache):
    data, kind, pages, page, heads, dim = cache
    # (bytes as ec_kv_bytes counts them, without another call, which the library refuses limits for)
    _need(data.dtype == torch.uint8 and data.is_contiguous() and
          0 < 2 * pages * page * heads * (dim * (2 if kind == EC_T_BF16 else 1) + 1) <= data.numel(), "data is not a cache of kv_cache")
    return ec_kv_cache(data.data_ptr(), kind, pages, page, heads, dim)


def kv_write(cache: KvCache, k, v, slots, stream=None) -> None:
    """ec_kv_write: float32 or bfloat16 CUDA tensors [rows, kv_heads, head_dim] into the slots (int32 [rows]) of a cache.  A row whose slot is
    not in the cache (-1) is left out; of rows that name the same slot the last one is stored."""
    import torch
    kind = _plain_type(k.dtype)
    rows, heads, dim, k_ld, k_head = _heads_of(k, "k")
    _need(v.dtype == k.dtype and v.shape == k.shape, "v must have k's shape and type")
    _, _, _, v_ld, v_head = _heads_of(v, "v")
    _need((heads, dim) == (cache.kv_heads, cache.head_dim), "k and v have other heads than the cache")
    _ints(torch, slots, (rows,), "slots")
    lib = _lib or load_library()

    def call(raw):
        c = _cache_struct(torch, cache)
        _done(lib, lib.ec_kv_write(C.byref(c), k.data_ptr(), v.data_ptr(), kind, rows, k_ld, k_head, v_ld, v_head, slots.data_ptr(), raw))
    return _place(stream, call, cache.data, k, v, slots)


def kv_read(cache: KvCache, slots, dtype=None, stream=None):
    """ec_kv_read: keys and values [rows, kv_heads, head_dim] of the slots (int32 [rows]), bfloat16 (the default) or float32.  A slot that is
    not in the cache reads zeros."""
    import torch
    dtype = torch.bfloat16 if dtype is None else dtype
    kind = _plain_type(dtype)
    if slots.dim() != 1 or slots.shape[0] > _INT_MAX:
        raise ValueError("slots must be contiguous int32 [rows], at most 2^31 - 1")
    rows = slots.shape[0]
    _ints(torch, slots, (rows,), "slots")
    lib = _lib or load_library()

    def call(raw):
        c = _cache_struct(torch, cache)
        head, ld = cache.head_dim, cache.kv_heads * cache.head_dim
        k = torch.empty((rows, cache.kv_heads, head), dtype=dtype, device=cache.data.device)
        v = torch.empty_like(k)
        _done(lib, lib.ec_kv_read(C.byref(c), slots.data_ptr(), rows, k.data_ptr(), v.data_ptr(), kind, ld, head, ld, head, raw))
        return k, v
    return _place(stream, call, cache.data, slots)


def kv_attention(q, cache: KvCache, table, lengths, starts=None, max_rows: Optional[int] = None, max_keys: Optional[int] = None,
                 prefix=None, prefix_len: int = 0, causal: bool = False, scale: Optional[float] = None, out=None, stream=None):
    """ec_kv_attention: bfloat16 queries [rows, heads, head_dim] (strides multiples of 8) of a batch of sequences over a cache.  Sequence b has
    the pages table[b] (int32 [seqs, pages]), lengths[b] keys (int32 [seqs]) and the rows starts[b] .. starts[b + 1] - 1 (int32 [seqs + 1];
    without it as many rows each).  prefix: pages (int32) whose first prefix_len tokens all sequences see before their own.  causal: row i of n
    sees its sequence's keys before lengths[b] - n + i + 1.  max_rows, max_keys: the most of any sequence, where that is known on
    the host to be less than all rows and the whole table; what is beyond is not computed.  scale: 1 / sqrt(head_dim) by default.  Without `out`
    the rows of no sequence are zeros; with it they are left as they were.  No gradients."""
    import torch
    if q.dtype != torch.bfloat16:
        raise ValueError("q must be bfloat16")
    rows, heads, dim, ld, ld_head = _heads_of(q, "q")
    if dim != cache.head_dim:
        raise ValueError("q has another head_dim than the cache")
    if table.dim() != 2 or table.dtype != torch.int32 or (table.shape[1] > 1 and table.stride(1) != 1):
        raise ValueError("table must be int32 [seqs, pages]")
    seqs, width = table.shape
    _ints(torch, lengths, (seqs,), "lengths")
    tensors = [cache.data, q, table, lengths]
    if starts is not None:
        _ints(torch, starts, (seqs + 1,), "starts")
        tensors.append(starts)
        max_rows = rows if max_rows is None else min(max_rows, rows)
    else:
        each = rows // max(seqs, 1)
        if rows != each * seqs or max_rows not in (None, each):
            raise ValueError("without starts every sequence has rows / seqs rows")
        max_rows = each
    prefix_pages = 0
    if prefix is not None:
        _need(prefix.dim() == 1, "prefix must be contiguous int32 [pages]")
        prefix_pages = prefix.shape[0]
        _ints(torch, prefix, (prefix_pages,), "prefix")
        tensors.append(prefix)
    if out is not None:
        _need(out.dtype == q.dtype and out.shape == q.shape, "out must have q's shape and type")
        tensors.append(out)
    if max_keys is None:
        max_keys = min(width * cache.page, _INT_MAX)
    if not (0 <= max_rows and 0 <= max_keys <= _INT_MAX and 0 <= prefix_len <= _INT_MAX and prefix_pages <= _INT_MAX and seqs <= _INT_MAX and width <= _INT_MAX):
        raise ValueError("sizes and lengths must be in [0, 2^31)")
    lib = _lib or load_library()
    cfg = ec_kv_attention_cfg(rows, heads, seqs, max_rows, max_keys, width, prefix_pages, prefix_len, causal,
                              dim ** -0.5 if scale is None else scale, table.stride(0) if seqs > 1 else width)

    def call(raw):
        c = _cache_struct(torch, cache)
        if out is None:
            y = (torch.empty if starts is None else torch.zeros)((rows, heads, dim), dtype=q.dtype, device=q.device)
            to, to_head = heads * dim, dim
        else:
            y = out
            _, _, _, to, to_head = _heads_of(y, "out")
        if seqs == 0:
            return y         # (no row is of a sequence)
        size = lib.ec_kv_attention_workspace_bytes(C.byref(c), C.byref(cfg))
        ws, at = _workspace(torch, size, q.device)
        _done(lib, lib.ec_kv_attention(C.byref(c), C.byref(cfg), q.data_ptr(), ld, ld_head, table.data_ptr(), lengths.data_ptr(),
                                       None if starts is None else starts.data_ptr(), prefix.data_ptr() if prefix_pages else None,
                                       y.data_ptr(), to, to_head, at, size, raw))
        return y
    return _place(stream, call, *tensors)


class EntropyCache:
    """One context: holds the torch tensors the library borrows (weights, workspace).
    With dec.batch > 1, `prompt` is a list of dec.batch prompts and the per-sequence results
    come back as lists in sequence order."""

    def __init__(self, cfg, dev_weights: Dict[str, object], dec, prompt, stream=None):
        import torch
        self.lib = load_library()
        self.cfg, self.dec = cfg, dec
        self.B = dec.batch
        prompts = [list(prompt)] if self.B == 1 else [list(p) for p in prompt]
        assert len(prompts) == self.B
        self.Ps = [len(p) for p in prompts]
        self.N = dec.gen_len
        self.Ts = [p + self.N for p in self.Ps]
        self.P, self.T = self.Ps[0], self.Ts[0]
        self._w = dev_weights  # keep alive
        self._mc, self._dc = model_cfg_struct(cfg), decode_cfg_struct(dec)
        L = cfg.n_layers
        ws = ec_weights()
        ws.tok_emb = dev_weights["tok_emb"].data_ptr()
        ws.lm_head = dev_weights["lm_head"].data_ptr()
        ws.final_norm = dev_weights["final_norm"].data_ptr()
        self._ptr_arrays = {}
        for name in ("attn_norm", "wq", "wk", "wv", "wo", "mlp_norm", "w_gate", "w_up", "w_down"):
            arr = (C.c_void_p * L)(*[t.data_ptr() for t in dev_weights[name]])
            self._ptr_arrays[name] = arr
            setattr(ws, name, C.cast(arr, C.POINTER(C.c_void_p)))
        of_scales = {"fp8w": "_scale", "mxfp4w": "_mx"}.get(cfg.dtype)
        if of_scales:
            setattr(ws, "lm_head" + of_scales, dev_weights["lm_head" + of_scales].data_ptr())
            for name in QUANT_MATRICES:
                arr = (C.c_void_p * L)(*[t.data_ptr() for t in dev_weights[name + of_scales]])
                self._ptr_arrays[name + of_scales] = arr
                setattr(ws, name + of_scales, C.cast(arr, C.POINTER(C.c_void_p)))
        self._ws = ws
        plen = _i32(self.Ps)
        need = self.lib.ec_workspace_bytes(C.byref(self._mc), C.byref(self._dc), _i32p(plen))
        if need == 0:
            # let ec_init produce the message
            need = 256
        self.workspace_bytes = need
        self._workspace = torch.empty(need, dtype=torch.uint8, device=dev_weights["tok_emb"].device)
        self._stream = stream if stream is not None else torch.cuda.current_stream()
        ctx = C.c_void_p()
        pr = _i32([t for p in prompts for t in p])
        rc = self.lib.ec_init(C.byref(ctx), C.byref(self._mc), C.byref(self._ws),
                              C.byref(self._dc), _i32p(pr), _i32p(plen),
                              C.c_void_p(self._workspace.data_ptr()), need,
                              C.c_void_p(self._stream.cuda_stream))
        if rc != EC_OK:
            raise EcError(rc, self.lib.ec_last_error(None).decode())
        self.ctx = ctx

    def _check(self, rc: int):
        if rc != EC_OK:
            raise EcError(rc, self.lib.ec_last_error(self.ctx).decode())

    def reset(self, prompt):
        prompts = [list(prompt)] if self.B == 1 else [list(p) for p in prompt]
        assert [len(p) for p in prompts] == self.Ps
        pr = _i32([t for p in prompts for t in p])
        self._check(self.lib.ec_reset(self.ctx, _i32p(pr)))

    def step(self, mode: int = EC_AUTO):
        r = (ec_step_result * self.B)()
        self._check(self.lib.ec_step(self.ctx, mode, r))
        return r[0].as_dict() if self.B == 1 else [x.as_dict() for x in r]

    def step_forced_batch(self, modes: Sequence[int], positions, tokens) -> List[dict]:
        """positions / tokens: one list per sequence (ignored for finished sequences)."""
        r = (ec_step_result * self.B)()
        n = _i32([len(p) for p in positions])
        p = _i32([v for q in positions for v in q] or [0])
        t = _i32([v for q in tokens for v in q] or [0])
        self._check(self.lib.ec_step_forced_batch(self.ctx, _i32p(_i32(modes)), _i32p(n), _i32p(p),
                                                  _i32p(t), r))
        return [x.as_dict() for x in r]

    def step_forced(self, mode: int, positions: Sequence[int], tokens: Sequence[int]) -> dict:
        r = ec_step_result()
        p, t = _i32(positions), _i32(tokens)
        self._check(self.lib.ec_step_forced(self.ctx, mode, len(p), _i32p(p), _i32p(t), C.byref(r)))
        return r.as_dict()

    def generate(self):
        out = np.zeros(self.B * self.N, dtype=np.int32)
        st = ec_gen_stats()
        self._check(self.lib.ec_generate(self.ctx, _i32p(out), C.byref(st)))
        stats = {k: getattr(st, k) for k, _ in ec_gen_stats._fields_}
        return (out if self.B == 1 else out.reshape(self.B, self.N)), stats

    def keep_logits(self, on: bool = True):
        """Makes the following steps store their logits so that EC_DBG_LOGITS can read them."""
        self._check(self.lib.ec_debug_keep_logits(self.ctx, int(on)))

    def debug_meeting(self, polls: int, apart: bool = False):
        """Blocks that share a tile wait this many polls for each other; apart: as if on different XCDs."""
        self._check(self.lib.ec_debug_meeting(self.ctx, polls, int(apart)))

    def profile_enable(self, on: bool):
        self._check(self.lib.ec_profile_enable(self.ctx, int(on)))

    def profile_read(self) -> dict:
        p = ec_profile()
        self._check(self.lib.ec_profile_read(self.ctx, C.byref(p)))
        return {"steps": p.steps,
                "ms": {n: p.ms[i] for i, n in enumerate(KERNEL_CLASS_NAMES)},
                "launches": {n: p.launches[i] for i, n in enumerate(KERNEL_CLASS_NAMES)}}

    def debug_read(self, what: int, layer: int = 0, count: Optional[int] = None,
                   seq: int = 0) -> np.ndarray:
        cfg = self.cfg
        T = self.Ts[seq]
        kvw = cfg.n_kv_heads * cfg.head_dim
        if what == EC_DBG_LOGITS:
            n = self.dec.block if count is None else count
            out = np.empty((n, cfg.vocab), dtype=np.float32)
        elif what in (EC_DBG_KCACHE, EC_DBG_VCACHE):
            out = np.empty((T, cfg.n_kv_heads, cfg.head_dim),
                           dtype=np.float32 if cfg.dtype == "f32" else np.uint16)
        elif what == EC_DBG_X:
            out = np.empty(T, dtype=np.int32)
        elif what == EC_DBG_MASKED:
            out = np.empty(T, dtype=np.uint8)
        elif what == EC_DBG_HIST:
            out = np.empty(self.N, dtype=np.int32)
        elif what == EC_DBG_ROWS:
            out = np.empty(int(count), dtype=np.int32)
        elif what == EC_DBG_ROW_STATS:
            n = self.dec.block if count is None else count
            out = np.empty((n, 4), dtype=np.float32)
        else:
            raise ValueError("unknown debug item")
        self._check(self.lib.ec_debug_read_seq(self.ctx, seq, what, layer,
                                               out.ctypes.data_as(C.c_void_p), out.nbytes))
        return out

    def close(self):
        if getattr(self, "ctx", None):
            self.lib.ec_destroy(self.ctx)
            self.ctx = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
