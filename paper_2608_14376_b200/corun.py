"""ctypes binding of the C ABI in ``include/corun.h`` (argument marshalling only).

Every step of the hot path runs in the CUDA kernels of ``libcorun.so``; there
is no CPU or PyTorch fallback: if the library is missing or the call fails, an
exception is raised.
"""
from __future__ import annotations

import ctypes as C
import os

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libcorun.so")

OK, EINVAL, ESLOT, ENOSPACE, ECTX, ECUDA, ETIMEOUT, ENOMEM, ELIMIT = 0, -1, -2, -3, -4, -5, -6, -7, -8

EXPORTS = [
    "corun_init", "corun_init_moe", "corun_init_mla", "corun_prefill", "corun_prefill_batch", "corun_decode_step", "corun_decode_enqueue", "corun_decode_wait",
    "corun_release", "corun_destroy", "corun_get_logits", "corun_force_token", "corun_context_len",
    "corun_free_blocks", "corun_debug_kv_read", "corun_debug_kv_write", "corun_debug_adopt",
    "corun_debug_set_eager", "corun_debug_read", "corun_debug_kv_fill", "corun_debug_time_kernel", "corun_decode_launches", "corun_debug_gemm", "corun_debug_gemm_pair", "corun_debug_gemm_experts", "corun_debug_prefill_attention", "corun_debug_variate",
    "corun_debug_sample", "corun_debug_wait_probe", "corun_debug_microbench", "corun_debug_check_index", "corun_gemm_static", "corun_strerror", "corun_last_cuda_error", "corun_engine_info",
    "corun_sched_create", "corun_sched_create_for_engine", "corun_sched_destroy", "corun_sched_submit",
    "corun_sched_step", "corun_sched_poll", "corun_sched_slot_of", "corun_sched_counts",
    "corun_sched_enable_batched_prefill", "corun_prefill_geometry", "corun_prefill_class",
    "corun_moe_create", "corun_moe_destroy", "corun_moe_forward", "corun_moe_sync", "corun_moe_weight_bytes",
    "corun_moe_launches", "corun_mla_attend", "corun_mla_workspace_floats", "corun_mla_sync",
    "corun_rope_create", "corun_rope_destroy", "corun_rope_apply", "corun_kv8_append", "corun_kv8_attend", "corun_kv8_attend_bytes",
    "corun_kv8_sync", "corun_kv8_evict", "corun_kv8_evict_bytes",
]


# kernel timelines: present only in a library built with CORUN_BUILD_DEBUG=1 (include/corun_debug.h)
DEBUG_EXPORTS = ["corun_debug_gemm_trace", "corun_debug_attn_trace", "corun_debug_step_trace"]


def _need_debug_build():
    if not hasattr(lib(), "corun_debug_step_trace"):
        raise RuntimeError("kernel timelines need a library built with CORUN_BUILD_DEBUG=1 "
                           "(CORUN_BUILD_DEBUG=1 python -m paper_2608_14376_b200.build --force)")


class MoeShape(C.Structure):
    _fields_ = [("hidden", C.c_int32), ("n_experts", C.c_int32), ("top_k", C.c_int32), ("expert_ffn", C.c_int32),
                ("n_shared", C.c_int32), ("renormalize", C.c_int32)]


class MoeLayers(C.Structure):
    """``corun_moe_layers``."""
    _fields_ = [("n_experts", C.c_int32), ("top_k", C.c_int32), ("expert_ffn", C.c_int32), ("n_shared", C.c_int32),
                ("renormalize", C.c_int32), ("router", C.POINTER(C.c_void_p)), ("gate_up", C.POINTER(C.c_void_p)),
                ("down", C.POINTER(C.c_void_p))]


class MlaLayers(C.Structure):
    """``corun_mla_layers``."""
    _fields_ = [("kv_lora_rank", C.c_int32), ("qk_nope", C.c_int32), ("qk_rope", C.c_int32), ("v_head", C.c_int32),
                ("first_dense", C.c_int32), ("kv_norm", C.POINTER(C.c_void_p)), ("wkv_b", C.POINTER(C.c_void_p))]


class RopeConfig(C.Structure):
    """``corun_rope_config``."""
    _fields_ = [("rot_dim", C.c_int32), ("interleaved", C.c_int32), ("scaling", C.c_int32), ("original_context", C.c_int32),
                ("theta", C.c_double), ("factor", C.c_double), ("low", C.c_double), ("high", C.c_double), ("magnitude", C.c_double)]


class Heads(C.Structure):
    """``corun_heads``."""
    _fields_ = [("p", C.c_void_p), ("token_stride", C.c_int64), ("head_stride", C.c_int64)]


class Kv8CacheArgs(C.Structure):
    """``corun_kv8_cache``."""
    _fields_ = [("pool", C.c_void_p), ("exps", C.c_void_p), ("pages", C.c_int64), ("block", C.c_int32), ("n_kv", C.c_int32),
                ("head_dim", C.c_int32)]


class Kv8Rows(C.Structure):
    """``corun_kv8_rows``."""
    _fields_ = [("block_table", C.c_void_p), ("max_blocks", C.c_int32), ("ctx", C.c_void_p), ("cu", C.c_void_p), ("B", C.c_int32),
                ("T", C.c_int32)]


class CorunError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        msg = lib().corun_strerror(status).decode()
        extra = f" (cuda error {lib().corun_last_cuda_error()})" if status == ECUDA else ""
        super().__init__(f"{where}: {msg}{extra} [{status}]")


class Shape(C.Structure):
    _fields_ = [(n, C.c_int32) for n in
                ("n_layers", "hidden", "n_q_heads", "n_kv_heads", "head_dim", "ffn", "vocab")] + [
        ("rms_eps", C.c_float), ("rope_theta", C.c_float), ("arch", C.c_int32)]


_PP = C.POINTER(C.c_void_p)


class Weights(C.Structure):
    _fields_ = [("embed", C.c_void_p), ("lm_head", C.c_void_p), ("final_norm", C.c_void_p),
                ("attn_norm", _PP), ("wqkv", _PP), ("wo", _PP), ("mlp_norm", _PP), ("wgate_up", _PP), ("wdown", _PP)]


class Sampling(C.Structure):
    _fields_ = [("temperature", C.c_float), ("top_p", C.c_float)]


PREFILL_FN = C.CFUNCTYPE(C.c_int, C.c_void_p, C.c_int32, C.POINTER(C.c_int32), C.c_int32, C.c_int32, C.POINTER(Sampling),
                         C.c_uint64, C.POINTER(C.c_int32))
DECODE_FN = C.CFUNCTYPE(C.c_int, C.c_void_p, C.POINTER(C.c_uint8), C.POINTER(C.c_uint64), C.POINTER(C.c_int32))
RELEASE_FN = C.CFUNCTYPE(C.c_int, C.c_void_p, C.c_int32)
FREE_BLOCKS_FN = C.CFUNCTYPE(C.c_int64, C.c_void_p)
PREFILL_BATCH_FN = C.CFUNCTYPE(C.c_int, C.c_void_p, C.c_int32, C.POINTER(C.c_int32), C.POINTER(C.c_int32),
                               C.POINTER(C.c_int32), C.POINTER(C.c_int32), C.POINTER(Sampling), C.POINTER(C.c_uint64),
                               C.POINTER(C.c_int32))


class SchedOps(C.Structure):
    """``corun_sched_ops``: the four engine calls the scheduler makes."""
    _fields_ = [("prefill", PREFILL_FN), ("decode_step", DECODE_FN), ("release", RELEASE_FN),
                ("free_blocks", FREE_BLOCKS_FN)]

SCHED_IDLE, SCHED_PREFILL, SCHED_DECODE = 0, 1, 2


_lib = None


def lib():
    """Loads libcorun.so (built in-tree by ``paper_2608_14376_b200.build``); fails loudly if absent."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: run `python -m paper_2608_14376_b200.build` "
                               "(there is no fallback path)")
        L = C.CDLL(LIB_PATH)
        vp, i32, i64, u64 = C.c_void_p, C.c_int32, C.c_int64, C.c_uint64
        L.corun_init.argtypes = [C.POINTER(Shape), C.POINTER(Weights), i32, i32, i32, i64, vp, C.POINTER(vp)]
        L.corun_prefill.argtypes = [vp, i32, vp, i32, i32, C.POINTER(Sampling), u64, C.POINTER(i32)]
        L.corun_prefill_batch.argtypes = [vp, i32, vp, vp, vp, vp, vp, vp, vp]
        L.corun_decode_step.argtypes = [vp, vp, vp, vp]
        L.corun_decode_enqueue.argtypes = [vp, vp, vp]
        L.corun_decode_wait.argtypes = [vp, vp]
        L.corun_release.argtypes = [vp, i32]
        L.corun_destroy.argtypes = [vp]
        L.corun_destroy.restype = None
        L.corun_get_logits.argtypes = [vp, i32, vp]
        L.corun_force_token.argtypes = [vp, i32, i32]
        L.corun_context_len.argtypes = [vp, i32]
        L.corun_free_blocks.argtypes = [vp]
        L.corun_free_blocks.restype = i64
        L.corun_debug_kv_read.argtypes = [vp, i32, i32, i32, i32, vp, vp]
        L.corun_debug_kv_write.argtypes = [vp, i32, i32, i32, i32, vp, vp]
        L.corun_debug_adopt.argtypes = [vp, i32, i32, i32, i32, C.POINTER(Sampling), i32]
        L.corun_debug_set_eager.argtypes = [vp, i32]
        L.corun_debug_read.argtypes = [vp, i32, vp, i64]
        if hasattr(L, "corun_debug_step_trace"):              # a library built with CORUN_BUILD_DEBUG=1
            L.corun_debug_gemm_trace.argtypes = [vp, i32, i32, vp, C.POINTER(i32)]
            L.corun_debug_attn_trace.argtypes = [vp, i32, vp, C.POINTER(i32)]
            L.corun_debug_step_trace.argtypes = [vp, vp, i64]
        L.corun_debug_kv_fill.argtypes = [vp, i32, i32, C.c_float, u64]
        L.corun_debug_time_kernel.argtypes = [vp, i32, i32, C.POINTER(C.c_float)]
        L.corun_decode_launches.argtypes = [vp]
        L.corun_debug_gemm.argtypes = [vp, i32, i32, vp, i32, vp, vp]
        L.corun_prefill_class.argtypes = [vp, i32, C.POINTER(i32), C.POINTER(i32), C.POINTER(i32)]
        L.corun_debug_gemm_pair.argtypes = [i32, vp, i32, i32, vp, i32, vp, vp]
        L.corun_debug_gemm_experts.argtypes = [i32, vp, i32, i32, i32, vp, vp, vp, vp, vp]
        L.corun_debug_prefill_attention.argtypes = [vp, i32, i32, i32, i32, vp, vp]
        L.corun_debug_variate.argtypes = [u64, u64, C.POINTER(C.c_uint32)]
        L.corun_debug_sample.argtypes = [vp, i32, i32, C.POINTER(Sampling), vp, vp]
        L.corun_gemm_static.argtypes = [vp, i32, i32, vp, i32, vp, vp]
        L.corun_strerror.argtypes = [C.c_int]
        L.corun_strerror.restype = C.c_char_p
        L.corun_last_cuda_error.argtypes = []
        L.corun_engine_info.argtypes = [vp, C.POINTER(i32), C.POINTER(i32), C.POINTER(i32), C.POINTER(i64)]
        L.corun_sched_create.argtypes = [C.POINTER(SchedOps), vp, i32, i32, i32, C.POINTER(vp)]
        L.corun_sched_create_for_engine.argtypes = [vp, C.POINTER(vp)]
        L.corun_sched_destroy.argtypes = [vp]
        L.corun_sched_destroy.restype = None
        L.corun_sched_submit.argtypes = [vp, vp, i32, i32, C.POINTER(Sampling), u64, C.POINTER(i64)]
        L.corun_sched_step.argtypes = [vp, C.POINTER(i32), C.POINTER(i64), C.POINTER(i32)]
        L.corun_sched_poll.argtypes = [vp, i64, vp, i32, C.POINTER(i32), C.POINTER(i32)]
        L.corun_sched_slot_of.argtypes = [vp, i64, C.POINTER(i32)]
        L.corun_sched_counts.argtypes = [vp, C.POINTER(i32), C.POINTER(i32)]
        L.corun_moe_create.argtypes = [C.POINTER(MoeShape), vp, vp, vp, i32, vp, C.POINTER(vp)]
        L.corun_moe_destroy.argtypes = [vp]
        L.corun_moe_destroy.restype = None
        L.corun_moe_forward.argtypes = [vp, vp, vp, vp, vp]
        L.corun_moe_sync.argtypes = [vp]
        L.corun_moe_weight_bytes.argtypes = [vp]
        L.corun_moe_weight_bytes.restype = i64
        L.corun_moe_launches.argtypes = [vp]
        pp = C.POINTER
        L.corun_rope_create.argtypes = [pp(RopeConfig), pp(vp)]
        L.corun_rope_destroy.argtypes = [vp]
        L.corun_rope_destroy.restype = None
        L.corun_rope_apply.argtypes = [vp, pp(Heads), pp(Heads), i32, vp, i64, i32, i32, vp]
        L.corun_kv8_append.argtypes = [pp(Kv8CacheArgs), pp(Kv8Rows), pp(Heads), pp(Heads), i32, vp, vp, pp(Heads), pp(Heads), i32, vp, vp]
        L.corun_kv8_attend_bytes.argtypes = [i32] * 9
        L.corun_kv8_attend_bytes.restype = i64
        L.corun_kv8_attend.argtypes = [pp(Kv8CacheArgs), pp(Kv8Rows), i32, pp(Heads), pp(Heads), i32, i32, C.c_float, i32, vp, vp, i64, vp]
        L.corun_kv8_sync.argtypes = [vp, vp]
        L.corun_kv8_evict_bytes.argtypes = [i32] * 3
        L.corun_kv8_evict_bytes.restype = i64
        L.corun_kv8_evict.argtypes = [pp(Kv8CacheArgs), vp, i32, i32, vp, vp, vp, vp, i32, i32, i32, vp, vp, i64, vp]
        for n in EXPORTS:
            getattr(L, n)
        _lib = L
    return _lib


def _check(rc: int, where: str):
    if rc != OK:
        raise CorunError(rc, where)


class Engine:
    """One engine = one fixed decode shape (B, max_context) on the current CUDA device.

    ``weights``: dict of torch bf16 CUDA tensors laid out as ``corun_weights``
    describes (see ``synth.make_weights_*``); they are borrowed, keep them alive.
    """

    def __init__(self, shape, weights: dict, B: int, max_context: int, kv_pool_blocks: int = 0, stream=None, moe: dict = None,
                 mla: dict = None, kv_block: int = 16):
        """``moe``: Mixture-of-Experts feed-forward layers instead of the dense ones: a dict with n_experts, top_k,
        expert_ffn, n_shared, renormalize and lists of L CUDA bf16 tensors router [E, H], gate_up [(E+S)*2F, H],
        down [H, (E+S)*F] (``weights`` then needs no wgate_up / wdown).
        ``mla``: multi-head latent attention layers (``corun_init_mla``): a dict with kv_lora_rank, qk_nope, qk_rope,
        v_head, first_dense and lists of L CUDA bf16 tensors kv_norm [rank], wkv_b [nh*(nope+v), rank]; wqkv / wo of
        ``weights`` then have the MLA shapes, layers below first_dense are dense (wgate_up / wdown entries; None for
        the other layers), the others take ``moe`` (its entries below first_dense may be None).
        ``kv_block``: tokens per cache block: 16, or (``mla`` only) 64: the 16-token pages of a slot then come in aligned
        runs of four and the latent attention fetches a run with one TMA box; ``kv_pool_blocks`` counts these blocks."""
        import torch

        self._torch = torch
        self.shape, self.B, self.max_context = shape, B, max_context
        self._weights = weights
        d = shape.dict() if hasattr(shape, "dict") else dict(shape)
        self._cs = Shape(d["n_layers"], d["hidden"], d["n_q_heads"], d["n_kv_heads"], d["head_dim"], d["ffn"],
                         d["vocab"], d["rms_eps"], d["rope_theta"], 0)
        cw = Weights()
        self._arrs = {}
        for k in ("embed", "lm_head", "final_norm"):
            t = weights[k]
            assert t.is_cuda and t.dtype == torch.bfloat16 and t.is_contiguous()
            setattr(cw, k, t.data_ptr())
        def ptr_array(ts):
            assert len(ts) == d["n_layers"]
            for t in ts:
                assert t is None or (t.is_cuda and t.dtype == torch.bfloat16 and t.is_contiguous())
            return (C.c_void_p * len(ts))(*[(t.data_ptr() if t is not None else None) for t in ts])

        dense_needed = (not moe) or (mla is not None and mla["first_dense"] > 0)
        for k in ("attn_norm", "wqkv", "wo", "mlp_norm") + (("wgate_up", "wdown") if dense_needed else ()):
            arr = ptr_array(weights[k])
            self._arrs[k] = arr
            setattr(cw, k, C.cast(arr, _PP))
        self._cw = cw
        torch.cuda.synchronize()
        h = C.c_void_p()
        cm = None
        if moe:
            cm = MoeLayers(moe["n_experts"], moe["top_k"], moe["expert_ffn"], moe["n_shared"], 1 if moe.get("renormalize") else 0)
            self._moe = moe
            for k in ("router", "gate_up", "down"):
                arr = ptr_array(moe[k])
                self._arrs["moe_" + k] = arr
                setattr(cm, k, C.cast(arr, _PP))
        if mla is not None:
            cl = MlaLayers(mla["kv_lora_rank"], mla["qk_nope"], mla["qk_rope"], mla["v_head"], mla["first_dense"])
            self._mla = mla
            for k in ("kv_norm", "wkv_b"):
                arr = ptr_array(mla[k])
                self._arrs["mla_" + k] = arr
                setattr(cl, k, C.cast(arr, _PP))
            L = lib()
            L.corun_init_mla.argtypes = [C.POINTER(Shape), C.POINTER(Weights), C.POINTER(MlaLayers), C.POINTER(MoeLayers), C.c_int32,
                                         C.c_int32, C.c_int32, C.c_int64, C.c_void_p, C.POINTER(C.c_void_p)]
            _check(L.corun_init_mla(C.byref(self._cs), C.byref(cw), C.byref(cl), C.byref(cm) if cm is not None else None, B,
                                    max_context, kv_block, kv_pool_blocks, C.c_void_p(stream) if stream else None, C.byref(h)),
                   "corun_init_mla")
        elif moe:
            L = lib()
            L.corun_init_moe.argtypes = [C.POINTER(Shape), C.POINTER(Weights), C.POINTER(MoeLayers), C.c_int32, C.c_int32,
                                         C.c_int32, C.c_int64, C.c_void_p, C.POINTER(C.c_void_p)]
            _check(L.corun_init_moe(C.byref(self._cs), C.byref(cw), C.byref(cm), B, max_context, 16, kv_pool_blocks,
                                    C.c_void_p(stream) if stream else None, C.byref(h)), "corun_init_moe")
        else:
            _check(lib().corun_init(C.byref(self._cs), C.byref(cw), B, max_context, 16, kv_pool_blocks,
                                    C.c_void_p(stream) if stream else None, C.byref(h)), "corun_init")
        self._h = h
        self.vocab = d["vocab"]

    def close(self):
        if getattr(self, "_h", None):
            lib().corun_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # -- the four calls of the boundary
    def prefill(self, slot: int, tokens, reserve_len: int, temperature: float = 0.0, top_p: float = 1.0,
                seed: int = 0) -> int:
        t = np.ascontiguousarray(tokens, dtype=np.int32)
        s = Sampling(temperature, top_p)
        first = C.c_int32(-1)
        _check(lib().corun_prefill(self._h, slot, t.ctypes.data, t.shape[0], reserve_len, C.byref(s),
                                   seed & (2**64 - 1), C.byref(first)), "corun_prefill")
        return int(first.value)

    def prefill_batch(self, slots, prompts, reserve_lens, temperature: float = 0.0, top_p: float = 1.0, seeds=None) -> np.ndarray:
        """Prefill of several requests in shared chunks; returns their first tokens."""
        n = len(slots)
        sl = np.ascontiguousarray(slots, dtype=np.int32)
        lens = np.ascontiguousarray([len(p) for p in prompts], dtype=np.int32)
        toks = np.ascontiguousarray(np.concatenate([np.asarray(p, dtype=np.int32) for p in prompts]), dtype=np.int32)
        res = np.ascontiguousarray(reserve_lens, dtype=np.int32)
        smp = (Sampling * n)(*[Sampling(temperature, top_p) for _ in range(n)])
        sd = np.ascontiguousarray(seeds if seeds is not None else np.zeros(n), dtype=np.uint64)
        out = np.full(n, -1, np.int32)
        assert sl.shape == lens.shape == res.shape == sd.shape == (n,)
        _check(lib().corun_prefill_batch(self._h, n, sl.ctypes.data, toks.ctypes.data, lens.ctypes.data, res.ctypes.data,
                                         C.cast(smp, C.c_void_p), sd.ctypes.data, out.ctypes.data), "corun_prefill_batch")
        return out

    def decode_step(self, active, seeds) -> np.ndarray:
        a = np.ascontiguousarray(active, dtype=np.uint8)
        s = np.ascontiguousarray(seeds, dtype=np.uint64)
        assert a.shape == (self.B,) and s.shape == (self.B,)
        out = np.empty(self.B, np.int32)
        _check(lib().corun_decode_step(self._h, a.ctypes.data, s.ctypes.data, out.ctypes.data), "corun_decode_step")
        return out

    def decode_enqueue(self, active, seeds):
        a = np.ascontiguousarray(active, dtype=np.uint8)
        s = np.ascontiguousarray(seeds, dtype=np.uint64)
        _check(lib().corun_decode_enqueue(self._h, a.ctypes.data, s.ctypes.data), "corun_decode_enqueue")

    def decode_wait(self) -> np.ndarray:
        out = np.empty(self.B, np.int32)
        _check(lib().corun_decode_wait(self._h, out.ctypes.data), "corun_decode_wait")
        return out

    def release(self, slot: int):
        _check(lib().corun_release(self._h, slot), "corun_release")

    # -- accessors
    def logits(self, slot: int) -> np.ndarray:
        out = np.empty(self.vocab, np.float32)
        _check(lib().corun_get_logits(self._h, slot, out.ctypes.data), "corun_get_logits")
        return out

    def force_token(self, slot: int, token: int):
        _check(lib().corun_force_token(self._h, slot, int(token)), "corun_force_token")

    def prefill_class(self, n_tokens: int):
        """(class, rows to count as a chunk, tile rows) of prompts of that length (``corun_prefill_class``)."""
        c, ch, t = C.c_int32(-1), C.c_int32(-1), C.c_int32(-1)
        _check(lib().corun_prefill_class(self._h, n_tokens, C.byref(c), C.byref(ch), C.byref(t)), "corun_prefill_class")
        return c.value, ch.value, t.value

    def context_len(self, slot: int) -> int:
        rc = lib().corun_context_len(self._h, slot)
        if rc < 0:
            raise CorunError(rc, "corun_context_len")
        return rc

    def free_blocks(self) -> int:
        return int(lib().corun_free_blocks(self._h))

    def kv_read(self, slot: int, layer: int, pos0: int, n: int):
        if getattr(self, "_mla", None):                   # latent cache: rows of rank + rope values, no second array
            k = np.empty((n, self._mla["kv_lora_rank"] + self._mla["qk_rope"]), np.float32)
            _check(lib().corun_debug_kv_read(self._h, slot, layer, pos0, n, k.ctypes.data, None), "kv_read")
            return k, None
        kd = self._cs.n_kv_heads * self._cs.head_dim
        k = np.empty((n, kd), np.float32)
        v = np.empty((n, kd), np.float32)
        _check(lib().corun_debug_kv_read(self._h, slot, layer, pos0, n, k.ctypes.data, v.ctypes.data), "kv_read")
        return k, v

    def kv_write(self, slot: int, layer: int, pos0: int, k, v):
        k = np.ascontiguousarray(k, dtype=np.float32)
        if v is None:                                     # latent cache
            _check(lib().corun_debug_kv_write(self._h, slot, layer, pos0, k.shape[0], k.ctypes.data, None), "kv_write")
            return
        v = np.ascontiguousarray(v, dtype=np.float32)
        _check(lib().corun_debug_kv_write(self._h, slot, layer, pos0, k.shape[0], k.ctypes.data, v.ctypes.data),
               "kv_write")

    def adopt(self, slot: int, n_ctx: int, reserve_len: int, pending: int, temperature=0.0, top_p=1.0, step=1):
        s = Sampling(temperature, top_p)
        _check(lib().corun_debug_adopt(self._h, slot, n_ctx, reserve_len, pending, C.byref(s), step), "adopt")

    def kv_fill(self, slot: int, n_ctx: int, std: float, seed: int):
        _check(lib().corun_debug_kv_fill(self._h, slot, n_ctx, std, seed & (2**64 - 1)), "kv_fill")

    KERNEL_KINDS = ("gemm_qkv", "gemm_o", "gemm_gate_up", "gemm_down", "gemm_lm_head", "attention",
                    "resid_norm", "rope_kv_append", "swiglu", "sampler")
    # further kinds of corun_debug_time_kernel: engines with multi-head latent attention / with expert layers
    MLA_KERNEL_KINDS = {"mla_up_k": 10, "mla_up_v": 11}
    MOE_KERNEL_KINDS = {"moe_router": 12}
    MOE_GROUPED_KERNEL_KINDS = {"moe_group_gather": 13}   # decode programs with more than 64 padded rows

    def time_kernel(self, kind: int, reps: int) -> float:
        ms = C.c_float(0.0)
        _check(lib().corun_debug_time_kernel(self._h, kind, reps, C.byref(ms)), "time_kernel")
        return float(ms.value)

    def gemm_trace(self, kind: int, layer: int = 0) -> np.ndarray:
        """Per-CTA timeline [n_ctas, 8] (ns, relative to the earliest kernel entry) of one GEMM launch."""
        st = np.zeros(8 * 256, np.uint64)
        n = C.c_int32(0)
        _need_debug_build()
        _check(lib().corun_debug_gemm_trace(self._h, kind, layer, st.ctypes.data, C.byref(n)), "gemm_trace")
        t = st[:8 * n.value].reshape(n.value, 8).astype(np.int64)
        return t - t[:, 0].min()

    def step_trace(self, n_sms: int = 148) -> np.ndarray:
        """GEMM timelines of the last decode step, [4 * n_layers, n_sms, 8] ns (engine made with CORUN_TRACE_STEP=1)."""
        n = 4 * self._cs.n_layers * n_sms * 8
        st = np.zeros(n, np.uint64)
        _need_debug_build()
        _check(lib().corun_debug_step_trace(self._h, st.ctypes.data, n), "step_trace")
        return st.reshape(4 * self._cs.n_layers, n_sms, 8).astype(np.int64)

    def attn_trace(self, layer: int = 0) -> np.ndarray:
        """Per-CTA, per-item attention timeline [n_ctas, 64, 8] in ns (0 where an item does not exist)."""
        st = np.zeros(256 * 64 * 8, np.uint64)
        n = C.c_int32(0)
        _need_debug_build()
        _check(lib().corun_debug_attn_trace(self._h, layer, st.ctypes.data, C.byref(n)), "attn_trace")
        return st[:n.value * 512].reshape(n.value, 64, 8).astype(np.int64)

    def debug_read(self, which: int, n: int) -> np.ndarray:
        out = np.empty(n, np.float32)
        _check(lib().corun_debug_read(self._h, which, out.ctypes.data, n), "corun_debug_read")
        return out

    def prefill_attention(self, slot: int, layer: int, pos0: int, q) -> np.ndarray:
        """The long prompts' attention kernel for query rows q [n, heads, dims] at positions pos0 .."""
        q = np.ascontiguousarray(q, dtype=np.float32)
        out = np.empty(q.shape[:2] + (self._mla["v_head"] if getattr(self, "_mla", None) else q.shape[2],), np.float32)
        _check(lib().corun_debug_prefill_attention(self._h, slot, layer, pos0, q.shape[0], q.ctypes.data, out.ctypes.data),
               "corun_debug_prefill_attention")
        return out

    def set_eager(self, eager: bool):
        _check(lib().corun_debug_set_eager(self._h, int(eager)), "set_eager")

    def decode_launches(self) -> int:
        return int(lib().corun_decode_launches(self._h))


class Scheduler:
    """Host scheduler (isolated prefill in front of the padded decode iteration) around an
    ``Engine``, or around a table of callbacks standing in for one (``ops``: a ``SchedOps`` whose
    callbacks the caller keeps alive, with ``B``, ``kv_block`` and ``max_context``)."""

    def __init__(self, engine: "Engine" = None, ops: SchedOps = None, B: int = 0, kv_block: int = 16,
                 max_context: int = 0):
        h = C.c_void_p()
        if engine is not None:
            _check(lib().corun_sched_create_for_engine(engine._h, C.byref(h)), "corun_sched_create_for_engine")
        else:
            _check(lib().corun_sched_create(C.byref(ops), None, B, kv_block, max_context, C.byref(h)), "corun_sched_create")
        self._h, self._keep = h, (engine, ops)

    def close(self):
        if self._h:
            lib().corun_sched_destroy(self._h)
            self._h = None

    def enable_batched_prefill(self, fn=None, chunk_rows: int = 0, tile_rows: int = 0):
        """Prefill decisions take the requests behind the head that fit into the padding of the head's chunks
        (``fn``: a PREFILL_BATCH_FN for a stand-in engine; None = the engine's corun_prefill_batch)."""
        self._batch_fn = fn                                   # keep the callback alive
        L = lib()
        L.corun_sched_enable_batched_prefill.argtypes = [C.c_void_p, C.c_void_p, C.c_int32, C.c_int32]
        _check(L.corun_sched_enable_batched_prefill(self._h, C.cast(fn, C.c_void_p) if fn is not None else None,
                                                    chunk_rows, tile_rows), "corun_sched_enable_batched_prefill")

    def submit(self, prompt, max_new_tokens: int, temperature: float = 0.0, top_p: float = 1.0, seed: int = 0) -> int:
        t = np.ascontiguousarray(prompt, dtype=np.int32)
        s = Sampling(temperature, top_p)
        rid = C.c_int64(-1)
        _check(lib().corun_sched_submit(self._h, t.ctypes.data, t.shape[0], max_new_tokens, C.byref(s),
                                        seed & (2**64 - 1), C.byref(rid)), "corun_sched_submit")
        return int(rid.value)

    def step(self):
        """One scheduling decision -> (action, request id of a prefill or -1, requests that took part)."""
        a, rid, n = C.c_int32(0), C.c_int64(-1), C.c_int32(0)
        _check(lib().corun_sched_step(self._h, C.byref(a), C.byref(rid), C.byref(n)), "corun_sched_step")
        return int(a.value), int(rid.value), int(n.value)

    def poll(self, rid: int):
        """-> (tokens produced so far, finished?)"""
        n, fin = C.c_int32(0), C.c_int32(0)
        _check(lib().corun_sched_poll(self._h, rid, None, 0, C.byref(n), C.byref(fin)), "corun_sched_poll")
        out = np.empty(max(1, n.value), np.int32)
        _check(lib().corun_sched_poll(self._h, rid, out.ctypes.data, n.value, C.byref(n), C.byref(fin)), "corun_sched_poll")
        return out[:n.value].copy(), bool(fin.value)

    def slot_of(self, rid: int) -> int:
        s = C.c_int32(-1)
        _check(lib().corun_sched_slot_of(self._h, rid, C.byref(s)), "corun_sched_slot_of")
        return int(s.value)

    def counts(self):
        w, r = C.c_int32(0), C.c_int32(0)
        _check(lib().corun_sched_counts(self._h, C.byref(w), C.byref(r)), "corun_sched_counts")
        return int(w.value), int(r.value)


def debug_gemm(W, X):
    """out[r, n] = sum_k W[n, k] X[r, k]; W torch bf16 [N, K] cuda, X torch fp32 [R, K] cuda."""
    import torch

    N, K = W.shape
    R = X.shape[0]
    out = torch.empty((R, N), dtype=torch.float32, device=X.device)
    torch.cuda.synchronize()
    _check(lib().corun_debug_gemm(W.data_ptr(), N, K, X.data_ptr(), R, out.data_ptr(), None), "corun_debug_gemm")
    return out


def debug_gemm_pair(form, W, X):
    """The GEMM on pairs of SMs (``corun_debug_gemm_pair``): form 0 plain, 1 with SwiGLU (result [R, N / 2]), 2 keys and
    values; 3, 4: 0, 1 as a decode step runs them."""
    import torch

    N, K = W.shape
    R = X.shape[0]
    out = torch.empty((R, N // 2 if form in (1, 4) else N), dtype=torch.float32, device=X.device)
    torch.cuda.synchronize()
    _check(lib().corun_debug_gemm_pair(form, W.data_ptr(), N, K, X.data_ptr(), R, out.data_ptr(), None), "corun_debug_gemm_pair")
    return out


def debug_gemm_experts(form, W, rows, X, row_w=None):
    """The GEMMs of a prompt's experts (``corun_debug_gemm_experts``), rows[e] rows of X through expert e: form 0 W [N, E K], 1 gate / up
    with SwiGLU, W [E, 2F, K]."""
    import torch

    E, K = len(rows), X.shape[1]
    N = W.shape[1] if form else W.shape[0]
    out = torch.empty((X.shape[0], N // 2 if form else N), dtype=torch.float32, device=X.device)
    counts = np.asarray(rows, np.int32)
    torch.cuda.synchronize()
    _check(lib().corun_debug_gemm_experts(form, W.data_ptr(), E, N, K, counts.ctypes.data, X.data_ptr(),
                                          row_w.data_ptr() if row_w is not None else None, out.data_ptr(), None), "corun_debug_gemm_experts")
    return out


def gemm_static(W, X):
    """Same product as ``debug_gemm`` through ``corun_gemm_static``: the library's own fixed scratch
    array is used instead of fresh allocations (for callers that must not allocate device memory).
    The output tensor is the caller's; rows <= 16, K <= 4096, N <= 8192."""
    import torch

    N, K = W.shape
    R = X.shape[0]
    out = torch.empty((R, N), dtype=torch.float32, device=X.device)
    torch.cuda.synchronize()
    _check(lib().corun_gemm_static(W.data_ptr(), N, K, X.data_ptr(), R, out.data_ptr(), None), "corun_gemm_static")
    return out


def debug_variate(seed: int, t: int) -> int:
    o = C.c_uint32(0)
    _check(lib().corun_debug_variate(seed & (2**64 - 1), t, C.byref(o)), "corun_debug_variate")
    return int(o.value)


def debug_sample(logits, temperature: float, top_p: float, u24) -> np.ndarray:
    lg = np.ascontiguousarray(logits, dtype=np.float32)
    if lg.ndim == 1:
        lg = lg[None]
    u = np.ascontiguousarray(u24, dtype=np.uint32).reshape(-1)
    assert u.shape[0] == lg.shape[0]
    out = np.empty(lg.shape[0], np.int32)
    s = Sampling(temperature, top_p)
    _check(lib().corun_debug_sample(lg.ctypes.data, lg.shape[0], lg.shape[1], C.byref(s), u.ctypes.data,
                                    out.ctypes.data), "corun_debug_sample")
    return out


class MoeFfn:
    """Mixture-of-Experts feed-forward block (``include/corun_moe.h``).  Weights are CUDA bf16 tensors:
    router [E, H], gate_up [(E + S) * 2F, H], down [H, (E + S) * F]; B padded rows per call."""

    def __init__(self, hidden: int, n_experts: int, top_k: int, expert_ffn: int, n_shared: int, router, gate_up, down,
                 B: int, renormalize: bool = False):
        import torch

        self._torch = torch
        self.B, self.H, self.top_k = B, hidden, top_k
        self._w = (router, gate_up, down)                     # keep the borrowed tensors alive
        for t in self._w:
            assert t.is_cuda and t.dtype == torch.bfloat16 and t.is_contiguous()
        assert tuple(router.shape) == (n_experts, hidden)
        assert tuple(gate_up.shape) == ((n_experts + n_shared) * 2 * expert_ffn, hidden)
        assert tuple(down.shape) == (hidden, (n_experts + n_shared) * expert_ffn)
        sh = MoeShape(hidden, n_experts, top_k, expert_ffn, n_shared, 1 if renormalize else 0)
        h = C.c_void_p()
        self._stream = torch.cuda.current_stream()
        _check(lib().corun_moe_create(C.byref(sh), router.data_ptr(), gate_up.data_ptr(), down.data_ptr(), B,
                                      self._stream.cuda_stream, C.byref(h)), "corun_moe_create")
        self._h = h

    def forward(self, x, want_routing: bool = True):
        """x: CUDA fp32 [B, H] -> (y fp32 [B, H], experts int32 [B, top_k], probs fp32 [B, top_k]); asynchronous."""
        torch = self._torch
        assert x.is_cuda and x.dtype == torch.float32 and tuple(x.shape) == (self.B, self.H) and x.is_contiguous()
        y = torch.empty_like(x)
        ex = torch.empty((self.B, self.top_k), dtype=torch.int32, device=x.device) if want_routing else None
        pr = torch.empty((self.B, self.top_k), dtype=torch.float32, device=x.device) if want_routing else None
        _check(lib().corun_moe_forward(self._h, x.data_ptr(), y.data_ptr(), ex.data_ptr() if want_routing else None,
                                       pr.data_ptr() if want_routing else None), "corun_moe_forward")
        return y, ex, pr

    def sync(self):
        _check(lib().corun_moe_sync(self._h), "corun_moe_sync")

    def weight_bytes(self) -> int:
        return int(lib().corun_moe_weight_bytes(self._h))

    def launches(self) -> int:
        return int(lib().corun_moe_launches(self._h))

    def close(self):
        if self._h:
            lib().corun_moe_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class MlaAttention:
    """Absorbed multi-head latent attention for one query token per row over a paged latent cache
    (``include/corun_mla.h``) with its workspace and output allocated once: ``run`` only enqueues."""

    def __init__(self, B: int, n_heads: int, d_latent: int, d_rope: int, max_blocks: int, device="cuda"):
        import torch

        L = lib()
        L.corun_mla_workspace_floats.restype = C.c_int64
        L.corun_mla_workspace_floats.argtypes = [C.c_int32] * 4
        L.corun_mla_attend.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_int64, C.c_void_p, C.c_int32, C.c_void_p] + \
            [C.c_int32] * 4 + [C.c_float, C.c_void_p, C.c_void_p, C.c_void_p]
        L.corun_mla_sync.argtypes = [C.c_void_p, C.c_void_p]
        self.shape = (B, n_heads, d_latent, d_rope, max_blocks)
        self.ws = torch.empty(int(L.corun_mla_workspace_floats(B, n_heads, d_latent, max_blocks * 16)), dtype=torch.float32, device=device)
        self.out = torch.zeros((B, n_heads, d_latent), dtype=torch.float32, device=device)

    def run(self, q_lat, q_rope, pool, block_table, ctx, scale: float):
        """q_lat fp32 [B, n_heads, d_c], q_rope fp32 [B, n_heads, d_r], pool fp16 [pool_pages, 16, d_c + d_r],
        block_table int32 [B, max_blocks], ctx int32 [B] (contiguous CUDA tensors) -> o_lat fp32 [B, n_heads, d_c]
        (rows with ctx 0 keep what they held).  Asynchronous on torch's current stream."""
        import torch

        B, nh, dc, dr, mb = self.shape
        assert tuple(q_lat.shape) == (B, nh, dc) and q_lat.dtype == torch.float32 and q_lat.is_contiguous() and q_lat.is_cuda
        assert tuple(q_rope.shape) == (B, nh, dr) and q_rope.dtype == torch.float32 and q_rope.is_contiguous()
        assert pool.dtype == torch.float16 and pool.is_contiguous() and tuple(pool.shape[1:]) == (16, dc + dr)
        assert block_table.dtype == torch.int32 and block_table.is_contiguous() and tuple(block_table.shape) == (B, mb)
        assert ctx.dtype == torch.int32 and ctx.is_contiguous() and tuple(ctx.shape) == (B,)
        st = torch.cuda.current_stream().cuda_stream
        _check(lib().corun_mla_attend(q_lat.data_ptr(), q_rope.data_ptr(), pool.data_ptr(), pool.shape[0], block_table.data_ptr(),
                                      mb, ctx.data_ptr(), B, nh, dc, dr, float(scale), self.out.data_ptr(), self.ws.data_ptr(), st),
               "corun_mla_attend")
        return self.out

    def sync(self):
        """Waits for the stream; raises if a bounded device-side wait expired."""
        import torch

        _check(lib().corun_mla_sync(self.ws.data_ptr(), torch.cuda.current_stream().cuda_stream), "corun_mla_sync")


def mla_attend(q_lat, q_rope, pool, block_table, ctx, scale: float):
    """One call of ``MlaAttention`` with fresh buffers (rows with ctx 0 come back as zeros); waits for the result."""
    op = MlaAttention(q_lat.shape[0], q_lat.shape[1], q_lat.shape[2], q_rope.shape[2], block_table.shape[1], q_lat.device)
    out = op.run(q_lat, q_rope, pool, block_table, ctx, scale)
    op.sync()
    return out


ROPE_SCALINGS = ("none", "linear", "base", "parts", "bands")


_torch_mod = None


def _torch():
    """torch, looked up once (an import statement in a call costs it half a microsecond)."""
    global _torch_mod
    if _torch_mod is None:
        import torch

        _torch_mod = torch
    return _torch_mod


def _stream_of(index: int) -> int:
    """torch's current stream on device ``index``, as a ``cudaStream_t``."""
    T = _torch()
    raw = getattr(T._C, "_cuda_getCurrentRawStream", None)
    return raw(index) if raw is not None else T.cuda.current_stream(index).cuda_stream


def _launch(fn, where: str, device, *args):
    """``fn(*args, stream)`` with ``device`` as the current one, on torch's current stream there."""
    T, index = _torch(), device.index
    if device.type != "cuda":
        raise ValueError(f"CUDA tensors are needed, not tensors on {device}")
    if T.cuda.current_device() != index:
        with T.cuda.device(index):
            rc = fn(*args, _stream_of(index))
    else:
        rc = fn(*args, _stream_of(index))
    if rc:
        raise CorunError(rc, where)


def _dtype_code(t, what, f32=True):
    T, d = _torch(), t.dtype
    if d is T.bfloat16:
        return 1
    if d is T.float16:
        return 2
    if f32 and d is T.float32:
        return 0
    raise ValueError(f"{what}: {'float32, ' if f32 else ''}bfloat16 or float16 is needed, not {d}")


def _heads(t, shape, dtype, device, what):
    """[tokens, heads, dims] with contiguous dims as a ``corun_heads``."""
    st = t.stride()
    if t.shape != shape or t.dtype is not dtype or t.device != device or (st[2] != 1 and shape[2] > 1):
        raise ValueError(f"{what}: {tuple(shape)} {dtype} on {device} with contiguous dims is needed, "
                         f"not {tuple(t.shape)} {t.dtype} on {t.device}, strides {st}")
    return Heads(t.data_ptr(), st[0], st[1])


def _plain(t, shape, dtype, device, what):
    """A contiguous tensor's address."""
    if t.shape != shape or t.dtype is not dtype or t.device != device or not t.is_contiguous():
        raise ValueError(f"{what}: contiguous {tuple(shape)} {dtype} on {device} is needed, not {tuple(t.shape)} {t.dtype} on {t.device}")
    return t.data_ptr()


class Rope:
    """Rotary positions (``include/corun_rope.h``) of the first ``rot_dim`` values of every head.

    ``interleaved``: pairs (2i, 2i + 1) instead of (i, i + rot_dim / 2); ``scaling``: one of ``ROPE_SCALINGS`` ("base" is known as
    NTK-aware, "parts" as YaRN, "bands" goes by wavelength), with ``factor`` and, for "parts" (beta_slow, beta_fast) and "bands"
    (low_freq_factor, high_freq_factor), ``original_context``, ``low`` and ``high``; ``magnitude`` 0: the scaling's own."""

    def __init__(self, rot_dim: int, theta: float = 10000.0, interleaved: bool = False, scaling: str = "none", factor: float = 1.0,
                 original_context: int = 0, low: float = 1.0, high: float = 32.0, magnitude: float = 0.0):
        if scaling not in ROPE_SCALINGS:
            raise ValueError(f"scaling: one of {ROPE_SCALINGS} is needed, not {scaling!r}")
        c = RopeConfig(rot_dim, int(interleaved), ROPE_SCALINGS.index(scaling), original_context, theta, factor, low, high, magnitude)
        h = C.c_void_p()
        self._h = None
        _check(lib().corun_rope_create(C.byref(c), C.byref(h)), "corun_rope_create")
        self._h, self.rot_dim = h, rot_dim

    def _handle(self):
        if self._h is None:                                     # (to append, no handle means no rotation)
            raise ValueError("the Rope is closed")
        return self._h

    def apply(self, x, positions, out=None):
        """x [tokens, heads, dims] (fp32, bf16 or fp16, any strides of tokens and heads), positions int32 [tokens] -> rotated
        values in ``out`` (default: a new tensor; may be x).  Asynchronous on torch's current stream."""
        if x.dim() != 3:
            raise ValueError(f"x: [tokens, heads, dims] is needed, not {tuple(x.shape)}")
        h = self._handle()
        T, code, dev = _torch(), _dtype_code(x, "x"), x.device
        n, heads, dims = shape = x.shape
        xh = _heads(x, shape, x.dtype, dev, "x")
        y = out if out is not None else T.empty(shape, dtype=x.dtype, device=dev)
        yh = _heads(y, shape, x.dtype, dev, "out")
        pos = _plain(positions, (n,), T.int32, dev, "positions")
        if n and heads and dims:
            _launch(lib().corun_rope_apply, "corun_rope_apply", dev, h, xh, yh, code, pos, n, heads, dims)
        return y

    def close(self):
        if self._h:
            lib().corun_rope_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class Kv8Cache:
    """One layer's keys and values in 8 bits with a power-of-two scale per page, kind and head (``include/corun_kv8.h``):
    ``pool`` float8_e4m3fn [pages, 2, n_kv, block, head_dim] and ``exps`` int8 [pages, 2, n_kv], a value being pool * 2^exps.
    Which pages belong to whom is the caller's to say (block tables)."""

    def __init__(self, pages: int, n_kv: int, head_dim: int, block: int = 16, pool=None, exps=None, device="cuda"):
        torch, shape = _torch(), (pages, 2, n_kv, block, head_dim)
        self.pool = pool if pool is not None else torch.zeros(shape, dtype=torch.float8_e4m3fn, device=device)
        self.exps = exps if exps is not None else torch.zeros(shape[:3], dtype=torch.int8, device=self.pool.device)
        self.pages, self.n_kv, self.head_dim, self.block = pages, n_kv, head_dim, block
        self.device = self.pool.device
        self._c = Kv8CacheArgs(_plain(self.pool, shape, torch.float8_e4m3fn, self.device, "pool"),
                               _plain(self.exps, shape[:3], torch.int8, self.device, "exps"), pages, block, n_kv, head_dim)

    def _rows(self, ctx, block_table, cu, tokens):
        i32, dev, B = _torch().int32, self.device, ctx.shape[0]
        if block_table.dim() != 2:
            raise ValueError(f"block_table: [rows, blocks] is needed, not {tuple(block_table.shape)}")
        blocks = block_table.shape[1]
        return Kv8Rows(_plain(block_table, (B, blocks), i32, dev, "block_table"), blocks, _plain(ctx, (B,), i32, dev, "ctx"),
                       _plain(cu, (B + 1,), i32, dev, "cu") if cu is not None else None, B, tokens)

    def _mass(self, mass, block_table):
        if mass is None:
            return None
        rows, blocks = block_table.shape
        return _plain(mass, (rows, self.n_kv, blocks * self.block), _torch().float32, self.device, "mass")

    def append(self, k, v, ctx, block_table, cu=None, positions=None, rope: "Rope" = None, q=None, q_out=None, mass=None):
        """Appends k, v [tokens, n_kv, head_dim]: ``ctx`` int32 [rows] counts every row's cached tokens with the new ones, ``cu``
        int32 [rows + 1] says which tokens are whose (None: one each).  ``rope`` rotates keys and q [tokens, n_q, head_dim] at
        ``positions`` int32 [tokens].  Returns the queries (``q_out``, or a new tensor, zeros for tokens of no row), None without q; ``mass`` float32
        [rows, n_kv, blocks * block]: the new tokens' accumulated weights become 0.  Asynchronous on torch's current stream."""
        T, code, dt, dev = _torch(), _dtype_code(k, "k"), k.dtype, self.device
        n, n_kv, hd = k.shape[0], self.n_kv, self.head_dim
        kh = _heads(k, (n, n_kv, hd), dt, dev, "k")
        vh = _heads(v, (n, n_kv, hd), dt, dev, "v")
        rows = self._rows(ctx, block_table, cu, n)
        qh = oh = None
        n_q = 0
        if q is not None:
            n_q = q.shape[1]
            qh = _heads(q, (n, n_q, hd), dt, dev, "q")
            if q_out is None:
                q_out = T.zeros((n, n_q, hd), dtype=dt, device=dev)
            oh = _heads(q_out, (n, n_q, hd), dt, dev, "q_out")
        rh = rope._handle() if rope is not None else None
        if rope is not None and positions is None:
            raise ValueError("rope needs positions")
        pos = _plain(positions, (n,), T.int32, dev, "positions") if positions is not None else None
        _launch(lib().corun_kv8_append, "corun_kv8_append", dev, self._c, rows, kh, vh, code, rh, pos, qh, oh, n_q,
                self._mass(mass, block_table))
        return q_out if q is not None else None

    def evict(self, ctx, block_table, mass, keep, max_keep: int, sinks: int = 4, recent: int = 64, new_ctx=None):
        """Shortens every row to its first ``sinks``, its last ``recent`` and its heaviest other tokens, ``keep`` int32 [rows] (at
        most ``max_keep``) in all, for each key head on its own.  Returns (kept int32 [rows, n_kv, max_keep]: where the tokens
        that stayed had been, then -1; new_ctx int32 [rows]).  Asynchronous on torch's current stream."""
        T, dev, B = _torch(), self.device, ctx.shape[0]
        rows = self._rows(ctx, block_table, None, B)
        if mass is None:
            raise ValueError("mass is needed")
        if sinks >> 31 not in (0, -1) or recent >> 31 not in (0, -1):
            raise ValueError(f"sinks {sinks}, recent {recent}: 0 or more is needed, max_keep together at most")
        m = self._mass(mass, block_table)
        kp = _plain(keep, (B,), T.int32, dev, "keep")
        if new_ctx is None:
            new_ctx = T.empty_like(ctx)
        nc = _plain(new_ctx, (B,), T.int32, dev, "new_ctx")
        n_ws = lib().corun_kv8_evict_bytes(B, self.n_kv, max_keep)
        kept = T.empty((B, self.n_kv, max(max_keep, 0)), dtype=T.int32, device=dev)
        # a workspace of the call's own: torch hands its memory out again in stream order, and to no other captured graph
        ws = T.empty(max(n_ws, 1), dtype=T.uint8, device=dev)
        _launch(lib().corun_kv8_evict, "corun_kv8_evict", dev, self._c, rows.block_table, rows.max_blocks, B, rows.ctx, nc, m, kp, max_keep, sinks,
                recent, kept.data_ptr(), ws.data_ptr(), n_ws)
        return kept, new_ctx


class Kv8Attention:
    """Attention over a ``Kv8Cache`` for calls of at most ``tokens`` query tokens of ``rows`` rows, ``max_new`` a row."""

    def __init__(self, rows: int, n_q: int, n_kv: int, head_dim: int, max_blocks: int, block: int = 16, tokens: int = 0, max_new: int = 1):
        self.shape = (rows, n_q, n_kv, head_dim, max_blocks, block)
        self.tokens, self.max_new = tokens or rows, max_new
        self._bytes, self._last = {}, None                       # workspace sizes; the last call's workspace and stream

    def run(self, q, cache: "Kv8Cache", ctx, block_table, scale: float, cu=None, window: int = 0, mass=None, out=None):
        """q [tokens, n_q, head_dim] (bf16 or fp16) -> out (default: a new tensor, zeros where no row writes): the rows' last cached
        tokens' own queries, ``cu`` int32 [rows + 1] saying which are whose (None: one each).  ``window`` > 0: a query sees that
        many tokens back, itself among them.  ``mass`` float32 [rows, n_kv, blocks * block] receives the weights.
        Asynchronous on torch's current stream."""
        rows, n_q, n_kv, hd, max_blocks, block = self.shape
        T, code, dt, dev, n = _torch(), _dtype_code(q, "q", f32=False), q.dtype, cache.device, q.shape[0]
        if n > self.tokens or ctx.shape != (rows,) or block_table.shape != (rows, max_blocks) or \
                (cache.n_kv, cache.head_dim, cache.block) != (n_kv, hd, block):
            raise ValueError(f"made for {self.tokens} tokens, {rows} rows of {max_blocks} blocks of {block} tokens, {n_kv} key heads of {hd}")
        qh = _heads(q, (n, n_q, hd), dt, dev, "q")
        if out is None:
            out = T.zeros((n, n_q, hd), dtype=dt, device=dev)
        oh = _heads(out, (n, n_q, hd), dt, dev, "out")
        r = cache._rows(ctx, block_table, cu, n)
        m = cache._mass(mass, block_table)
        max_new = max(min(self.max_new, n), 1) if cu is not None else 1   # (no row has more tokens than the call)
        if window >> 31:                                        # beyond 32 bits: wider than any cache, as all of 2^30 and above, or refused
            window = 0 if window > 0 else -1
        key = (n, max_new, m is not None)
        n_ws = self._bytes.get(key)
        if n_ws is None:
            n_ws = self._bytes[key] = lib().corun_kv8_attend_bytes(rows, n, max_new, n_q, n_kv, hd, block, max_blocks, int(key[2]))
        # a workspace of the call's own: torch hands its memory out again in stream order, and to no other captured graph; the last
        # call's may be this one's
        self._last = None
        ws = T.empty(max(n_ws, 1), dtype=T.uint8, device=dev)
        _launch(lib().corun_kv8_attend, "corun_kv8_attend", dev, cache._c, r, max_new, qh, oh, code, n_q, scale, window, m, ws.data_ptr(), n_ws)
        # (a call without tokens has no status)
        self._last = (ws, _stream_of(dev.index)) if n else None
        return out

    def sync(self):
        """Waits for the last call's stream and for the current one (a captured call may have been replayed on it); raises if a
        bounded device-side wait of the last call expired.  Threads that look at their own calls take an object each."""
        last = self._last
        if last is not None:
            ws, stream = last
            if stream != _stream_of(ws.device.index):
                T = _torch()
                (T.cuda.ExternalStream(stream, device=ws.device) if stream else T.cuda.default_stream(ws.device)).synchronize()
            _launch(lib().corun_kv8_sync, "corun_kv8_sync", ws.device, ws.data_ptr())


MICROBENCH_KINDS = ("rmsnorm", "softmax", "column_sum")


def microbench(kind: int, variant: int, x, reps: int = 20):
    """``corun_debug_microbench`` on a CUDA fp32 matrix x [R, N]: (y, microseconds per launch, tiling used).
    kind: index into MICROBENCH_KINDS; variant 0 = tiling fixed for every R, 1 = adapted to R."""
    import torch

    assert x.is_cuda and x.dtype == torch.float32 and x.is_contiguous() and x.dim() == 2
    R, N = x.shape
    y = torch.empty((N,) if kind == 2 else (R, N), dtype=torch.float32, device=x.device)
    us, til = C.c_float(0.0), C.c_int32(0)
    L = lib()
    L.corun_debug_microbench.argtypes = [C.c_int32, C.c_int32, C.c_void_p, C.c_int32, C.c_int32, C.c_void_p, C.c_int32,
                                         C.POINTER(C.c_float), C.POINTER(C.c_int32), C.c_void_p]
    _check(L.corun_debug_microbench(kind, variant, x.data_ptr(), R, N, y.data_ptr(), reps, C.byref(us), C.byref(til),
                                    torch.cuda.current_stream().cuda_stream), "corun_debug_microbench")
    return y, float(us.value), int(til.value)
