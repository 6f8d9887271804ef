"""ctypes binding for libspd (include/spd.h): argument marshalling only.

PyTorch appears here solely as the owner of device memory and of the HIP stream; every
step of the decoding path runs inside the library's kernels.  There is no fallback: if the
library has not been built this module raises on first use.
"""
from __future__ import annotations

import ctypes as C
import math
import os

import numpy as np

HERE = os.path.dirname(os.path.abspath(__file__))
SPD_K_MAX, SPD_TAIL, SPD_N_ORDERS = 16, 5, 5
SPD_EHIP = -6
SPD_DTYPE = {"fp32": 0, "bf16": 1, "fp16": 2, "int8": 3}   # fp16: key/value cache only; int8: paged cache of chunks of new tokens only
_lib = None


class SpdError(RuntimeError):
    def __init__(self, code, where, detail=""):
        self.code = code
        super().__init__(f"{where}: {spd_strerror(code)} ({code}) {detail}".strip())


class SpdModelCfg(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("n_layers", "d_model", "n_heads", "n_kv_heads", "d_ffn", "vocab",
                                          "max_ctx", "k_max", "dtype")] + [("rms_eps", C.c_float), ("rope_theta", C.c_float),
                                                                      ("kv_dtype", C.c_int32)]


class SpdLayerWeights(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("attn_norm", "wqkv", "wo", "ffn_norm", "w_gate", "w_up", "w_down")]


class SpdWeightPtrs(C.Structure):
    _fields_ = [("embed", C.c_void_p), ("layers", C.POINTER(SpdLayerWeights)), ("final_norm", C.c_void_p),
                ("lm_head", C.c_void_p)]


class SpdNgramHostTables(C.Structure):
    _fields_ = [("keys", C.c_void_p * SPD_N_ORDERS), ("counts", C.c_void_p * SPD_N_ORDERS),
                ("n_entries", C.c_int64 * SPD_N_ORDERS), ("lambda_", C.c_float * SPD_N_ORDERS)]


class SpdDecodeCfg(C.Structure):
    _fields_ = [("k", C.c_int32), ("alpha", C.c_float), ("tau", C.c_float), ("delta", C.c_float)]


class SpdSampleCfg(C.Structure):
    _fields_ = [("top_p", C.c_float), ("tau", C.c_float)]


def library_path() -> str:
    return os.environ.get("SPD_LIBRARY", os.path.join(HERE, "libspd.so"))


def lib():
    """The loaded C-ABI library.  Fails loudly when it has not been built."""
    global _lib
    if _lib is None:
        path = library_path()
        if not os.path.exists(path):
            raise ImportError(f"{path} is missing: build it first (python -m paper_2405_18400_amd.build)")
        L = C.CDLL(path)
        vp, i32, i64, f32, sz = C.c_void_p, C.c_int32, C.c_int64, C.c_float, C.c_size_t
        sig = {
            "spd_workspace_bytes": [C.POINTER(SpdModelCfg), C.POINTER(sz)],
            "spd_create": [C.POINTER(SpdModelCfg), C.POINTER(SpdWeightPtrs), vp, sz, vp, C.POINTER(vp)],
            "spd_ngram_table_bytes": [C.POINTER(SpdNgramHostTables), C.POINTER(sz)],
            "spd_load_ngrams": [vp, C.POINTER(SpdNgramHostTables), vp, sz],
            "spd_prefill": [vp, vp, i32],
            "spd_step": [vp, C.POINTER(SpdDecodeCfg), vp, vp, vp],
            "spd_nucleus_step": [vp, C.POINTER(SpdSampleCfg), C.c_float, vp, vp],
            "spd_get_nucleus_info": [vp, vp, vp, vp],
            "spd_commit": [vp, C.c_float, vp, vp, i32, vp],
            "spd_set_dense_prefill": [vp, i32],
            "spd_get_dense_prefill": [vp, C.POINTER(i32)],
            "spd_nucleus_sample": [vp, C.POINTER(SpdSampleCfg), C.c_float, vp, i32],
            "spd_generate": [vp, vp, i32, C.POINTER(SpdDecodeCfg), i32, vp, vp],
            "spd_get_state": [vp, C.POINTER(i32), vp, vp, vp],
            "spd_set_state": [vp, i32, vp, vp],
            "spd_read_logits": [vp, vp],
            "spd_get_step_info": [vp, vp, vp, vp, vp, vp],
            "spd_expand_prune": [vp, C.POINTER(SpdDecodeCfg), vp, i32],
            "spd_position": [vp, C.POINTER(i32)],
            "spd_set_graph": [vp, i32],
            "spd_set_kernel_timing": [vp, i32],
            "spd_get_phase_clock": [vp, i32, C.POINTER(C.c_int64), C.POINTER(i32), C.POINTER(i32)],
            "spd_set_fused": [vp, i32],
            "spd_get_fused": [vp, C.POINTER(i32)],
            "spd_get_kernel_timing": [vp, i32, C.POINTER(C.c_char_p), C.POINTER(f32), C.POINTER(C.c_int64), C.POINTER(i32)],
            "spd_test_state_layout": [C.POINTER(sz), C.POINTER(sz)],
            "spd_test_state_status": [vp, sz],
            "spd_test_poke_err": [vp, i32],
            "spd_test_ngram_table": [C.POINTER(SpdNgramHostTables), i32, vp, sz, C.POINTER(i32)],
            "spd_test_attention_shared_cut": [i32] * 8 + [vp],
            "spd_test_beam_select_cut": [i32] * 4 + [vp],
            "spd_test_prefill_cut": [C.POINTER(SpdModelCfg), i32, i32, i32, vp],
            "spd_test_prefill_attention": [i32, vp, vp, vp, vp, vp, i32, i32, i32, i32, i32, i32, vp],
            "spd_test_force_prefill_cut": [vp, i32, i32, i32, i32, vp],
            "spd_test_force_last_query": [vp, i32, i32, C.POINTER(i32)],
            "spd_op_gemv": [i32, vp, vp, f32, vp, vp, vp, i32, i32, vp],
            "spd_op_swiglu": [i32, vp, vp, vp, f32, vp, vp, i32, i32, vp],
            "spd_op_attention": [i32, vp, vp, vp, vp, vp, i32, i32, i32, i32, i32, vp],
            "spd_op_attention_static": [i32, vp, vp, vp, vp, i32, i32, i32, i32, i32, vp],
            "spd_op_append_paged": [i32, vp, vp, vp] + [i32] * 6 + [vp, i64, vp, vp, i64, vp, vp, i32, i32, f32, vp, vp, vp],
            "spd_op_attention_shared": [i32, vp, vp, vp, vp] + [i32] * 6 + [vp, vp, i32, i32, i32, i32, vp, vp, sz, vp, vp],
            "spd_op_beam_select": [i32, vp, i64, i32, i32, i32, i32, vp, vp, i32, f32, vp, vp, vp, vp, vp, sz, vp],
            "spd_op_beam_reorder": [i32, vp, vp, vp] + [i32] * 7 + [i64, i32, vp, vp, vp, vp, vp],
            "spd_op_beam_reorder_shared": [i32, vp, vp, vp] + [i32] * 7 + [i64, i32, vp, vp, vp, vp, vp, vp],
            "spd_op_append_paged_q8": [vp] * 5 + [i32] * 6 + [vp, i64, vp, vp, i64, vp, vp, i32, i32, f32, vp, vp, vp],
            "spd_op_read_paged": [i32] + [vp] * 5 + [i32] * 6 + [vp, vp, i32, i32, vp, vp, vp, vp],
            "spd_op_attention_paged": [i32, i32, vp, i64] + [vp] * 5 + [i32] * 6 + [vp, vp, i32, i32, i32, i32, vp, vp, sz, vp, vp],
            "spd_op_verify_drafts": [i32, vp, i64, vp, i64, vp, vp, vp, i32, i32, i32, C.c_double, C.c_double, vp, vp, vp, vp, sz, vp, vp],
        }
        for name, args in sig.items():
            fn = getattr(L, name)
            fn.argtypes, fn.restype = args, C.c_int
        L.spd_destroy.argtypes, L.spd_destroy.restype = [vp], None
        L.spd_last_error.argtypes, L.spd_last_error.restype = [vp], C.c_char_p
        L.spd_strerror.argtypes, L.spd_strerror.restype = [C.c_int], C.c_char_p
        L.spd_op_attention_scratch_bytes.argtypes, L.spd_op_attention_scratch_bytes.restype = [i32, i32, i32], sz
        L.spd_op_attention_shared_scratch_bytes.argtypes, L.spd_op_attention_shared_scratch_bytes.restype = [i32] * 7, sz
        L.spd_op_attention_paged_scratch_bytes.argtypes, L.spd_op_attention_paged_scratch_bytes.restype = [i32] * 9, sz
        L.spd_op_verify_drafts_scratch_bytes.argtypes, L.spd_op_verify_drafts_scratch_bytes.restype = [i32] * 3, sz
        L.spd_op_beam_select_scratch_bytes.argtypes, L.spd_op_beam_select_scratch_bytes.restype = [i32] * 4, sz
        L.hipStreamSynchronize.argtypes, L.hipStreamSynchronize.restype = [vp], C.c_int   # (the runtime that libspd is linked to)
        _lib = L
    return _lib


def spd_strerror(code: int) -> str:
    return lib().spd_strerror(int(code)).decode()


def _np_ptr(a):
    """An array's address.  The buffer protocol takes 0.4 us where `a.ctypes.data_as` takes 2.5 (a call has up to five of
    them: spd_get_state 22.6 -> 14.2 us, spd_get_step_info 19.1 -> 14.3); it wants a writable array with an element, others go by `a.ctypes`."""
    if a is None:
        return None
    try:
        return C.addressof(C.c_char.from_buffer(a))
    except (TypeError, ValueError):
        return a.ctypes.data


def model_cfg(shape, max_ctx: int, k_max: int, kv_dtype: str = "fp32") -> SpdModelCfg:
    return SpdModelCfg(shape.n_layers, shape.d_model, shape.n_heads, shape.n_kv_heads, shape.d_ffn, shape.vocab,
                       max_ctx, k_max, SPD_DTYPE[shape.dtype], shape.rms_eps, shape.rope_theta, SPD_DTYPE[kv_dtype])


def spd_workspace_bytes(cfg: SpdModelCfg) -> int:
    out = C.c_size_t(0)
    rc = lib().spd_workspace_bytes(C.byref(cfg), C.byref(out))
    if rc:
        raise SpdError(rc, "spd_workspace_bytes")
    return out.value


def ngram_struct(tables: dict, lambdas) -> tuple[SpdNgramHostTables, list]:
    """{n: (keys int32 [N, n], counts uint32 [N])} -> the C struct (+ the arrays kept alive)."""
    t, keep = SpdNgramHostTables(), []
    for o in range(SPD_N_ORDERS):
        keys, counts = tables.get(o + 2, (None, None))
        n = 0 if keys is None else len(keys)
        if n:
            keys = np.ascontiguousarray(keys, dtype=np.int32)
            counts = np.ascontiguousarray(counts, dtype=np.uint32)
            keep += [keys, counts]
            t.keys[o], t.counts[o] = keys.ctypes.data, counts.ctypes.data
        t.n_entries[o] = n
        t.lambda_[o] = float(lambdas[o])
    return t, keep


def spd_ngram_table_bytes(tables: dict, lambdas=(0, 0, 0, 0, 0)) -> int:
    t, _keep = ngram_struct(tables, lambdas)
    out = C.c_size_t(0)
    rc = lib().spd_ngram_table_bytes(C.byref(t), C.byref(out))
    if rc:
        raise SpdError(rc, "spd_ngram_table_bytes")
    return out.value


def _torch():
    import torch
    return torch


def to_device(arr, dtype: str, device="cuda"):
    """Host array -> device tensor holding the same bits (uint16 patterns become bfloat16).
    Tensors already on the device pass through."""
    torch = _torch()
    if isinstance(arr, torch.Tensor):
        assert arr.dtype == (torch.bfloat16 if dtype == "bf16" else torch.float32)
        return arr.to(device).contiguous()
    if dtype == "bf16":
        assert arr.dtype == np.uint16
        return torch.from_numpy(arr.view(np.int16)).to(device).view(torch.bfloat16)
    return torch.from_numpy(np.ascontiguousarray(arr, dtype=np.float32)).to(device)


class Session:
    """Owns the device tensors (weights, workspace, n-gram buffer), the stream and the spd_ctx.
    Methods carry the C function names and only marshal arguments."""

    def __init__(self, shape, weights: dict, max_ctx: int, k_max: int = 8, device="cuda", stream=None, kv_dtype: str = "fp32"):
        torch = _torch()
        if not torch.cuda.is_available():
            raise RuntimeError("libspd needs a GPU: no HIP device is visible")
        self.shape, self.device, self.L = shape, device, lib()
        self.stream = stream if stream is not None else torch.cuda.Stream(device=device)
        self.cfg = model_cfg(shape, max_ctx, k_max, kv_dtype)
        dev = lambda a: to_device(a, shape.dtype, device)
        self.t = {"embed": dev(weights["embed"]), "final_norm": dev(weights["final_norm"]), "lm_head": dev(weights["lm_head"])}
        self.layers = (SpdLayerWeights * max(shape.n_layers, 1))()
        for l in range(shape.n_layers):
            p = f"layers.{l}."
            qkv = weights.get(p + "wqkv")
            if qkv is None:
                qkv = np.concatenate([weights[p + "wq"], weights[p + "wk"], weights[p + "wv"]], axis=0)
            names = {"attn_norm": weights[p + "attn_norm"], "wqkv": qkv, "wo": weights[p + "wo"],
                     "ffn_norm": weights[p + "ffn_norm"], "w_gate": weights[p + "w_gate"],
                     "w_up": weights[p + "w_up"], "w_down": weights[p + "w_down"]}
            for nm, arr in names.items():
                self.t[p + nm] = dev(arr)
                setattr(self.layers[l], nm, self.t[p + nm].data_ptr())
        self.wp = SpdWeightPtrs(self.t["embed"].data_ptr(), self.layers, self.t["final_norm"].data_ptr(),
                                self.t["lm_head"].data_ptr())
        self.workspace = torch.empty(spd_workspace_bytes(self.cfg) + 256, dtype=torch.uint8, device=device)
        ws_ptr = (self.workspace.data_ptr() + 255) // 256 * 256
        torch.cuda.synchronize()
        self.ctx = C.c_void_p()
        rc = self.L.spd_create(C.byref(self.cfg), C.byref(self.wp), ws_ptr, self.workspace.numel() - 256,
                               self.stream.cuda_stream, C.byref(self.ctx))
        if rc:
            self.ctx = None
            raise SpdError(rc, "spd_create")
        self.ngram_buf = None

    # -- error plumbing
    def _chk(self, rc, where):
        if rc:
            raise SpdError(rc, where, self.L.spd_last_error(self.ctx).decode())

    def close(self):
        if getattr(self, "ctx", None):
            self.L.spd_destroy(self.ctx)
            self.ctx = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # -- the boundary, one method per C entry point
    def spd_load_ngrams(self, tables: dict, lambdas):
        torch = _torch()
        t, _keep = ngram_struct(tables, lambdas)
        need = C.c_size_t(0)
        self._chk(self.L.spd_ngram_table_bytes(C.byref(t), C.byref(need)), "spd_ngram_table_bytes")
        buf = torch.empty(need.value + 256, dtype=torch.uint8, device=self.device)
        ptr = (buf.data_ptr() + 255) // 256 * 256
        torch.cuda.synchronize()
        self._chk(self.L.spd_load_ngrams(self.ctx, C.byref(t), ptr, need.value), "spd_load_ngrams")
        self.ngram_buf = buf      # the previous buffer (if any) is released only now

    def spd_prefill(self, prefix):
        p = np.ascontiguousarray(prefix, dtype=np.int32)
        self._chk(self.L.spd_prefill(self.ctx, _np_ptr(p), len(p)), "spd_prefill")

    def spd_step(self, dc: SpdDecodeCfg, fetch: bool = True):
        if not fetch:
            self._chk(self.L.spd_step(self.ctx, C.byref(dc), None, None, None), "spd_step")
            return None
        tok, par, sc = np.zeros(dc.k, np.int32), np.zeros(dc.k, np.int32), np.zeros(dc.k, np.float32)
        self._chk(self.L.spd_step(self.ctx, C.byref(dc), _np_ptr(tok), _np_ptr(par), _np_ptr(sc)), "spd_step")
        return tok, par, sc

    def spd_commit(self, u: float):
        """-> (index of the sampled draft, its tokens since the last prefill / commit)."""
        cap = self.cfg.max_ctx
        chosen, n = C.c_int32(0), C.c_int32(0)
        toks = np.zeros(cap, np.int32)
        self._chk(self.L.spd_commit(self.ctx, float(u), C.byref(chosen), _np_ptr(toks), cap, C.byref(n)), "spd_commit")
        return chosen.value, toks[:n.value].copy()

    def spd_set_dense_prefill(self, enable: bool):
        self._chk(self.L.spd_set_dense_prefill(self.ctx, int(enable)), "spd_set_dense_prefill")

    def spd_get_dense_prefill(self) -> bool:
        out = C.c_int32(0)
        self._chk(self.L.spd_get_dense_prefill(self.ctx, C.byref(out)), "spd_get_dense_prefill")
        return bool(out.value)

    def spd_nucleus_step(self, sc: SpdSampleCfg, u: float, fetch: bool = True):
        if not fetch:
            self._chk(self.L.spd_nucleus_step(self.ctx, C.byref(sc), float(u), None, None), "spd_nucleus_step")
            return None
        tok, lp = C.c_int32(0), C.c_float(0)
        self._chk(self.L.spd_nucleus_step(self.ctx, C.byref(sc), float(u), C.byref(tok), C.byref(lp)), "spd_nucleus_step")
        return tok.value, lp.value

    def spd_nucleus_sample(self, sc: SpdSampleCfg, u: float, dev_logits, first: bool):
        assert dev_logits.is_cuda and dev_logits.dtype == _torch().float32 and dev_logits.numel() == self.shape.vocab
        self._chk(self.L.spd_nucleus_sample(self.ctx, C.byref(sc), float(u), dev_logits.data_ptr(), int(first)),
                  "spd_nucleus_sample")

    def spd_get_nucleus_info(self):
        size, mass, total = C.c_int32(0), C.c_float(0), C.c_float(0)
        self._chk(self.L.spd_get_nucleus_info(self.ctx, C.byref(size), C.byref(mass), C.byref(total)), "spd_get_nucleus_info")
        return size.value, mass.value, total.value

    def spd_generate(self, prefix, dc: SpdDecodeCfg, n_tokens: int):
        p = np.ascontiguousarray(prefix, dtype=np.int32)
        drafts, sc = np.zeros((dc.k, n_tokens), np.int32), np.zeros(dc.k, np.float32)
        self._chk(self.L.spd_generate(self.ctx, _np_ptr(p), len(p), C.byref(dc), n_tokens, _np_ptr(drafts), _np_ptr(sc)),
                  "spd_generate")
        return drafts, sc

    def spd_get_state(self):
        k = C.c_int32(0)
        tails, sc, g = np.zeros((SPD_K_MAX, SPD_TAIL), np.int32), np.zeros(SPD_K_MAX, np.float32), np.zeros(SPD_K_MAX, np.float32)
        self._chk(self.L.spd_get_state(self.ctx, C.byref(k), _np_ptr(tails), _np_ptr(sc), _np_ptr(g)), "spd_get_state")
        return tails[:k.value].copy(), sc[:k.value].copy(), g[:k.value].copy()

    def spd_set_state(self, tails, logscores):
        t = np.ascontiguousarray(tails, dtype=np.int32)
        s = np.ascontiguousarray(logscores, dtype=np.float32)
        self._chk(self.L.spd_set_state(self.ctx, len(s), _np_ptr(t), _np_ptr(s)), "spd_set_state")

    def spd_read_logits(self):
        out = np.zeros(self.shape.vocab, np.float32)
        self._chk(self.L.spd_read_logits(self.ctx, _np_ptr(out)), "spd_read_logits")
        return out

    def spd_get_step_info(self, k: int):
        ids, lp = np.zeros(k, np.int32), np.zeros(k, np.float32)
        cs, cv, cp = np.zeros((k, k), np.float32), np.zeros((k, k), np.int32), np.zeros((k, k), np.float32)
        self._chk(self.L.spd_get_step_info(self.ctx, _np_ptr(ids), _np_ptr(lp), _np_ptr(cs), _np_ptr(cv), _np_ptr(cp)),
                  "spd_get_step_info")
        return ids, lp, cs, cv, cp

    def spd_expand_prune(self, dc: SpdDecodeCfg, dev_logits, first: bool):
        assert dev_logits.is_cuda and dev_logits.dtype == _torch().float32 and dev_logits.numel() == self.shape.vocab
        self._chk(self.L.spd_expand_prune(self.ctx, C.byref(dc), dev_logits.data_ptr(), int(first)), "spd_expand_prune")

    def spd_test_poke_err(self, value: int):
        self._chk(self.L.spd_test_poke_err(self.ctx, int(value)), "spd_test_poke_err")

    def spd_test_force_prefill_cut(self, product: int, tile: int, splits: int, n_tokens: int):
        """-> (tokens and columns of a tile, blocks that share a tile's k range, epilogue in the product)."""
        out = np.zeros(4, np.int32)
        self._chk(self.L.spd_test_force_prefill_cut(self.ctx, product, tile, splits, n_tokens, _np_ptr(out)), "spd_test_force_prefill_cut")
        return int(out[0]), int(out[1]), int(out[2]), bool(out[3])

    def spd_test_force_last_query(self, mode: int, n_tokens: int) -> bool:
        """-> whether the last layer's query has a product of its own in a chunk of n_tokens."""
        out = C.c_int32(0)
        self._chk(self.L.spd_test_force_last_query(self.ctx, mode, n_tokens, C.byref(out)), "spd_test_force_last_query")
        return bool(out.value)

    def spd_position(self) -> int:
        out = C.c_int32(0)
        self._chk(self.L.spd_position(self.ctx, C.byref(out)), "spd_position")
        return out.value

    def spd_set_graph(self, enable: bool):
        self._chk(self.L.spd_set_graph(self.ctx, int(enable)), "spd_set_graph")

    def spd_set_fused(self, enable: bool):
        self._chk(self.L.spd_set_fused(self.ctx, int(enable)), "spd_set_fused")

    def spd_get_fused(self) -> bool:
        out = C.c_int32(0)
        self._chk(self.L.spd_get_fused(self.ctx, C.byref(out)), "spd_get_fused")
        return bool(out.value)

    def spd_set_kernel_timing(self, enable: bool):
        self._chk(self.L.spd_set_kernel_timing(self.ctx, int(enable)), "spd_set_kernel_timing")

    def spd_get_kernel_timing(self) -> dict:
        cap = 32
        names, ms, cnt, n = (C.c_char_p * cap)(), (C.c_float * cap)(), (C.c_int64 * cap)(), C.c_int32(0)
        self._chk(self.L.spd_get_kernel_timing(self.ctx, cap, names, ms, cnt, C.byref(n)), "spd_get_kernel_timing")
        return {names[i].decode(): (ms[i], cnt[i]) for i in range(n.value)}

    def spd_get_phase_clock(self):
        """Clock stamps [blocks, 2 (5 n_layers + 2)] of the most recent fused forward."""
        cap = 2 * (5 * self.shape.n_layers + 2) * 2048
        out, n, nb = np.zeros(cap, dtype=np.int64), C.c_int32(0), C.c_int32(0)
        self._chk(self.L.spd_get_phase_clock(self.ctx, cap, out.ctypes.data_as(C.POINTER(C.c_int64)), C.byref(n),
                                             C.byref(nb)), "spd_get_phase_clock")
        return out[:n.value * nb.value].reshape(nb.value, n.value).copy()

    def synchronize(self):
        self.stream.synchronize()


# ---- stand-alone operators (device tensors in, device tensors out; caller's current stream)
def _stream_ptr(device=None):
    """The calling thread's current stream on its current device, without the Stream object around it: building that
    took 2.9 of the 7.2 us such a call took the host (now 0.4 of 4.7)."""
    torch = _torch()
    raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)      # (private to torch: a build may lack it)
    return raw(torch.cuda.current_device() if device is None else device) if raw is not None else torch.cuda.current_stream().cuda_stream


def spd_op_gemv(dtype: str, W, x, y, gain=None, eps=0.0, residual=None):
    rows, cols = W.shape
    rc = lib().spd_op_gemv(SPD_DTYPE[dtype], W.data_ptr(), gain.data_ptr() if gain is not None else None, eps,
                           x.data_ptr(), residual.data_ptr() if residual is not None else None, y.data_ptr(),
                           rows, cols, _stream_ptr())
    if rc:
        raise SpdError(rc, "spd_op_gemv")


def spd_op_swiglu(dtype: str, Wg, Wu, x, u, gain=None, eps=0.0):
    rows, cols = Wg.shape
    rc = lib().spd_op_swiglu(SPD_DTYPE[dtype], Wg.data_ptr(), Wu.data_ptr(), gain.data_ptr() if gain is not None else None,
                             eps, x.data_ptr(), u.data_ptr(), rows, cols, _stream_ptr())
    if rc:
        raise SpdError(rc, "spd_op_swiglu")


def spd_op_attention(dtype: str, q, K, V, out, n_ctx: int):
    L, stream = lib(), _stream_ptr()
    n_heads, d_head = q.shape
    n_kv, cap_ctx, _ = K.shape
    scratch = _torch().empty(L.spd_op_attention_scratch_bytes(n_heads, d_head, cap_ctx) + 256, dtype=_torch().uint8, device=q.device)
    ptr = (scratch.data_ptr() + 255) // 256 * 256
    rc = L.spd_op_attention(SPD_DTYPE[dtype], q.data_ptr(), K.data_ptr(), V.data_ptr(), out.data_ptr(), ptr,
                            n_heads, n_kv, d_head, n_ctx, cap_ctx, stream)
    if rc:
        raise SpdError(rc, "spd_op_attention")
    if L.hipStreamSynchronize(stream):   # the call returns with its result in place (no Stream object for it: 3 us)
        raise SpdError(SPD_EHIP, "spd_op_attention")


def spd_op_attention_static(dtype: str, q, K, V, out, n_ctx: int):
    """The same on the library's static scratch: no allocation here or in the library."""
    n_heads, d_head = q.shape
    n_kv, cap_ctx, _ = K.shape
    rc = lib().spd_op_attention_static(SPD_DTYPE[dtype], q.data_ptr(), K.data_ptr(), V.data_ptr(), out.data_ptr(),
                                       n_heads, n_kv, d_head, n_ctx, cap_ctx, _stream_ptr())
    if rc:
        raise SpdError(rc, "spd_op_attention_static")


# ---- several sequences over one prompt, on a paged cache: K, V [pages, n_kv_heads, page_size, d_head], table int32 [n_seq, entries].
# Nothing here waits for the GPU; `err`, an int32 tensor of one element, is set to 1 by what only the kernels can see (spd.h).
# A decoding step makes a few such calls per layer, so each looks its arguments over in one expression and names what is wrong
# only where something is (append / attention / selection / reordering: 4.8 / 4.2 / 5.0 / 3.5 us of host time in front of a call's
# launch, 0.2 to 0.3 more with err; with a check per tensor 2.1 to 2.6 us more).
def _refuse(where, device, **tensors):
    """Says what is wrong with tensors given as (tensor, type, shape): they have to be whole, on `device`, and of as many elements (None: not looked at)."""
    for name, (t, dtype, shape) in tensors.items():
        if t is None:
            continue
        if t.get_device() != device:
            raise ValueError(f"{where}: {name} is not on the current device")
        if t.dtype is not dtype:
            raise ValueError(f"{where}: {name} is {t.dtype}, not {dtype}")
        if not t.is_contiguous():
            raise ValueError(f"{where}: {name} is not contiguous")
        if shape is not None and (t.numel() != math.prod(shape) or (name == "V" and t.shape != shape)):
            raise ValueError(f"{where}: {name} has shape {tuple(t.shape)}, not {shape}")


_INT32 = 2 ** 31 - 1      # (ctypes cuts larger numbers off without a word)


def _kv_type(where, torch, dtype):
    kv = torch.float16 if dtype == "fp16" else torch.bfloat16 if dtype == "bf16" else torch.float32 if dtype == "fp32" else None
    if kv is None:
        raise ValueError(f"{where}: no element type {dtype!r}")
    return kv


def _rows(where, device, name, t, heads, d, torch):
    """The stride of the tokens of t [tokens, heads, d], which may lie apart (parts of one product's rows)."""
    stride, between, within = t.stride()
    if t.dtype is not torch.float32 or t.get_device() != device:
        raise ValueError(f"{where}: {name} has to be float32 on the current device")
    if (within != 1 and d > 1) or (between != d and heads > 1):
        raise ValueError(f"{where}: the heads of {name}'s tokens have to lie one behind the other")
    return stride


def _scratch(torch, n_bytes, like):
    """Memory for one call.  It goes back to torch's pool when the call has been enqueued: that pool hands it out again in the order of the
    stream the call runs on, the current one.  (The pool's blocks start at multiples of 512 bytes.)"""
    return torch.empty(n_bytes, dtype=torch.uint8, device=like.device)


def _new_rows(where, torch, device, k, v, q, q_out, n, n_kv, d):
    """The rows of n new tokens: k, v [n, n_kv, d] and q [n, heads, d] -> q_out."""
    if k.shape != (n, n_kv, d) or v.shape != (n, n_kv, d):
        raise ValueError(f"{where}: k and v have to be [{n}, {n_kv}, {d}]")
    kv_stride, q_stride, heads, q_ptr, out_ptr = _rows(where, device, "k", k, n_kv, d, torch), 0, 0, None, None
    if _rows(where, device, "v", v, n_kv, d, torch) != kv_stride and n > 1:
        raise ValueError(f"{where}: k and v differ in their tokens' stride")
    if q is not None:
        heads = q.shape[1]
        if q_out is None or q.shape != (n, heads, d):
            raise ValueError(f"{where}: q has to be [{n}, heads, {d}], and comes with q_out")
        q_stride, q_ptr, out_ptr = _rows(where, device, "q", q, heads, d, torch), q.data_ptr(), q_out.data_ptr()
        if not (q_out.dtype is torch.float32 and q_out.numel() == n * heads * d and q_out.is_contiguous() and q_out.get_device() == device):
            _refuse(where, device, q_out=(q_out, torch.float32, (n, heads, d)))
    elif q_out is not None:
        raise ValueError(f"{where}: q_out comes with q")
    if n <= 1:                          # (a single token's stride may be anything)
        kv_stride, q_stride = n_kv * d, heads * d
    return kv_stride, q_ptr, q_stride, heads, out_ptr


def spd_op_append_paged(dtype: str, K, V, table, k, v, seq, pos, rope_theta: float, q=None, q_out=None, err=None):
    """k, v [tokens, n_kv_heads, d_head] (and q [tokens, n_heads, d_head] -> q_out), rotated by pos, to the rows of their sequences; seq < 0: padding."""
    torch, where = _torch(), "spd_op_append_paged"
    kv, i32, device = _kv_type(where, torch, dtype), torch.int32, torch.cuda.current_device()
    shape = K.shape
    n_pages, n_kv, page_size, d = shape
    n_seq, entries = table.shape
    n = seq.numel()
    if not (K.dtype is kv and V.dtype is kv and table.dtype is i32 and seq.dtype is i32 and pos.dtype is i32 and V.shape == shape and pos.numel() == n
            and K.is_contiguous() and V.is_contiguous() and table.is_contiguous() and seq.is_contiguous() and pos.is_contiguous()
            and K.get_device() == device and V.get_device() == device and table.get_device() == device and seq.get_device() == device and pos.get_device() == device
            and (err is None or (err.dtype is i32 and err.numel() == 1 and err.get_device() == device))):
        _refuse(where, device, K=(K, kv, None), V=(V, kv, shape), table=(table, i32, None), seq=(seq, i32, (n,)), pos=(pos, i32, (n,)), err=(err, i32, (1,)))
    kv_stride, q_ptr, q_stride, heads, out_ptr = _new_rows(where, torch, device, k, v, q, q_out, n, n_kv, d)
    rc = lib().spd_op_append_paged(SPD_DTYPE[dtype], K.data_ptr(), V.data_ptr(), table.data_ptr(), n_pages, n_kv, page_size, d, n_seq, entries, q_ptr, q_stride,
                                   k.data_ptr(), v.data_ptr(), kv_stride, seq.data_ptr(), pos.data_ptr(), n, heads, rope_theta, out_ptr,
                                   None if err is None else err.data_ptr(), _stream_ptr(device))
    if rc:
        raise SpdError(rc, where)


def spd_op_attention_shared(dtype: str, q, K, V, table, shared, length, out, width: int, max_shared: int, max_own: int, err=None):
    """q, out [n_seq, n_heads, d_head]; shared int32 [n_seq / width], length int32 [n_seq]."""
    torch, where = _torch(), "spd_op_attention_shared"
    kv, i32, f32, device = _kv_type(where, torch, dtype), torch.int32, torch.float32, torch.cuda.current_device()
    shape, rows = K.shape, q.shape
    n_pages, n_kv, page_size, d = shape
    n_seq, heads, q_d = rows
    entries = table.shape[-1]
    if width < 1 or n_seq % width:
        raise ValueError(f"{where}: {n_seq} sequences are no groups of {width}")
    groups = n_seq // width
    if max_shared > _INT32 or max_own > _INT32:
        raise ValueError(f"{where}: max_shared or max_own is no 32-bit number")
    if not (q.dtype is f32 and out.dtype is f32 and K.dtype is kv and V.dtype is kv and table.dtype is i32 and shared.dtype is i32 and length.dtype is i32 and q_d == d
            and out.numel() == q.numel() and V.shape == shape and table.numel() == n_seq * entries and shared.numel() == groups and length.numel() == n_seq
            and q.is_contiguous() and out.is_contiguous() and K.is_contiguous() and V.is_contiguous() and table.is_contiguous() and shared.is_contiguous()
            and length.is_contiguous() and q.get_device() == device and out.get_device() == device and K.get_device() == device and V.get_device() == device
            and table.get_device() == device and shared.get_device() == device and length.get_device() == device
            and (err is None or (err.dtype is i32 and err.numel() == 1 and err.get_device() == device))):
        _refuse(where, device, q=(q, f32, (n_seq, heads, d)), K=(K, kv, None), V=(V, kv, shape), table=(table, i32, (n_seq, entries)), shared=(shared, i32, (groups,)),
                length=(length, i32, (n_seq,)), out=(out, f32, (n_seq, heads, d)), err=(err, i32, (1,)))
    L = lib()
    n_bytes, scratch = L.spd_op_attention_shared_scratch_bytes(n_seq, width, heads, n_kv, d, max_shared, max_own), None
    if n_bytes:
        buf = _scratch(torch, n_bytes, q)
        scratch = buf.data_ptr()
    rc = L.spd_op_attention_shared(SPD_DTYPE[dtype], q.data_ptr(), K.data_ptr(), V.data_ptr(), table.data_ptr(), n_pages, n_kv, page_size, d, n_seq, entries,
                                   shared.data_ptr(), length.data_ptr(), width, heads, max_shared, max_own, out.data_ptr(), scratch, n_bytes,
                                   None if err is None else err.data_ptr(), _stream_ptr(device))
    if rc:
        raise SpdError(rc, where)


def spd_op_beam_select(dtype: str, logits, scores, out_scores, out_tokens, out_parents, tau: float = 1.0, ended=None, end_token: int = -1, out_ended=None):
    """logits [n_groups, n_in, vocab] (rows may lie apart), scores [n_groups, n_in] -> out_* [n_groups, n_out]."""
    torch, where = _torch(), "spd_op_beam_select"
    kind, i32, f32, device = _kv_type(where, torch, dtype), torch.int32, torch.float32, torch.cuda.current_device()
    groups, n_in, vocab = logits.shape
    n_out = out_scores.shape[-1]
    n = groups * n_out
    if not -_INT32 <= end_token <= _INT32:
        raise ValueError(f"{where}: end_token is no 32-bit number")
    if logits.dtype is not kind:
        raise ValueError(f"{where}: logits are {logits.dtype}, not {dtype}")
    of_group, of_row, of_entry = logits.stride()
    stride = of_row if n_in > 1 else of_group if groups > 1 else vocab
    if (of_entry != 1 and vocab > 1) or (groups > 1 and of_group != n_in * stride) or logits.get_device() != device:
        raise ValueError(f"{where}: logits have to be rows of one stride on the current device")
    if not (scores.dtype is f32 and out_scores.dtype is f32 and out_tokens.dtype is i32 and out_parents.dtype is i32 and scores.numel() == groups * n_in
            and out_scores.numel() == n and out_tokens.numel() == n and out_parents.numel() == n and scores.is_contiguous() and out_scores.is_contiguous()
            and out_tokens.is_contiguous() and out_parents.is_contiguous() and scores.get_device() == device and out_scores.get_device() == device
            and out_tokens.get_device() == device and out_parents.get_device() == device
            and (ended is None or (ended.dtype is i32 and ended.numel() == groups * n_in and ended.is_contiguous() and ended.get_device() == device))
            and (out_ended is None or (out_ended.dtype is i32 and out_ended.numel() == n and out_ended.is_contiguous() and out_ended.get_device() == device))):
        ins, outs = (groups, n_in), (groups, n_out)
        _refuse(where, device, scores=(scores, f32, ins), out_scores=(out_scores, f32, outs), out_tokens=(out_tokens, i32, outs), out_parents=(out_parents, i32, outs),
                ended=(ended, i32, ins), out_ended=(out_ended, i32, outs))
    L = lib()
    n_bytes, scratch = L.spd_op_beam_select_scratch_bytes(groups, n_in, n_out, vocab), None
    if n_bytes:
        buf = _scratch(torch, n_bytes, logits)
        scratch = buf.data_ptr()
    rc = L.spd_op_beam_select(SPD_DTYPE[dtype], logits.data_ptr(), stride, groups, n_in, n_out, vocab, scores.data_ptr(), None if ended is None else ended.data_ptr(),
                              end_token, tau, out_scores.data_ptr(), out_tokens.data_ptr(), out_parents.data_ptr(),
                              None if out_ended is None else out_ended.data_ptr(), scratch, n_bytes, _stream_ptr(device))
    if rc:
        raise SpdError(rc, where)


def spd_op_beam_reorder(dtype: str, K, V, table, parents, length, table_out, width: int, err=None, shared=None):
    """K, V [pages, ...] or [layers, pages, n_kv_heads, page_size, d_head]; parents int32 [n_seq / width, width], length int32 [n_seq]; table -> table_out.
    shared, int32 [n_seq / width]: positions that only a group's first row holds, as for the attention; without it every row has to hold all of its own (spd.h)."""
    torch, where = _torch(), "spd_op_beam_reorder"
    kv, i32, device = _kv_type(where, torch, dtype), torch.int32, torch.cuda.current_device()
    shape, rows = K.shape, table.shape
    n_pages, n_kv, page_size, d = shape[-4:]
    if len(shape) > 5:
        raise ValueError(f"{where}: K has shape {tuple(shape)}, not [(layers,) pages, heads, page size, d_head]")
    layers = shape[0] if len(shape) == 5 else 1
    n_seq, entries = rows
    if width < 1 or n_seq % width:
        raise ValueError(f"{where}: {n_seq} sequences are no groups of {width}")
    groups = (n_seq // width, width)
    if not (K.dtype is kv and V.dtype is kv and table.dtype is i32 and parents.dtype is i32 and length.dtype is i32 and table_out.dtype is i32 and V.shape == shape
            and parents.numel() == n_seq and length.numel() == n_seq and table_out.numel() == n_seq * entries and K.is_contiguous() and V.is_contiguous() and table.is_contiguous()
            and parents.is_contiguous() and length.is_contiguous() and table_out.is_contiguous() and K.get_device() == device and V.get_device() == device
            and table.get_device() == device and parents.get_device() == device and length.get_device() == device and table_out.get_device() == device
            and (shared is None or (shared.dtype is i32 and shared.numel() == groups[0] and shared.is_contiguous() and shared.get_device() == device))
            and (err is None or (err.dtype is i32 and err.numel() == 1 and err.get_device() == device))):
        _refuse(where, device, K=(K, kv, None), V=(V, kv, shape), table=(table, i32, None), parents=(parents, i32, groups), length=(length, i32, (n_seq,)),
                table_out=(table_out, i32, rows), shared=(shared, i32, groups[:1]), err=(err, i32, (1,)))
    name, of_group = (where, ()) if shared is None else (where + "_shared", (shared.data_ptr(),))
    rc = getattr(lib(), name)(SPD_DTYPE[dtype], K.data_ptr(), V.data_ptr(), table.data_ptr(), n_pages, n_kv, page_size, d, n_seq, entries, layers,
                              n_pages * n_kv * page_size * d, width, parents.data_ptr(), length.data_ptr(), *of_group, table_out.data_ptr(),
                              None if err is None else err.data_ptr(), _stream_ptr(device))
    if rc:
        raise SpdError(rc, where)


# ---- chunks of new tokens through a paged cache, which may hold codes of 8 bits with a scale per row: K, V int8 [pages, n_kv_heads, page_size, d_head], scales float32
# [pages, n_kv_heads, page_size].  Sequence s has the new tokens first[s] .. first[s + 1] - 1.
def _cache_type(where, torch, dtype):
    return torch.int8 if dtype == "int8" else _kv_type(where, torch, dtype)


def _io_type(where, torch, dtype):
    kind = "fp32" if dtype is torch.float32 else "fp16" if dtype is torch.float16 else "bf16" if dtype is torch.bfloat16 else None
    if kind is None:
        raise ValueError(f"{where}: rows are {dtype}, not float32, float16 or bfloat16")
    return kind


def _scales(where, torch, dtype, device, shape, K_scale, V_scale):
    """Addresses of an 8-bit cache's scales (None, None for other caches)."""
    if (K_scale is not None) != (dtype == "int8") or (V_scale is not None) != (dtype == "int8"):
        raise ValueError(f"{where}: an int8 cache comes with K_scale and V_scale, others without")
    if K_scale is None:
        return None, None
    f32, rows = torch.float32, shape[:3]
    if not (K_scale.dtype is f32 and V_scale.dtype is f32 and K_scale.shape == rows and V_scale.shape == rows and K_scale.is_contiguous() and V_scale.is_contiguous()
            and K_scale.get_device() == device and V_scale.get_device() == device):
        _refuse(where, device, K_scale=(K_scale, f32, rows), V_scale=(V_scale, f32, rows))
        raise ValueError(f"{where}: scales have to be {tuple(rows)}")
    return K_scale.data_ptr(), V_scale.data_ptr()


def spd_op_append_paged_q8(K, V, K_scale, V_scale, table, k, v, seq, pos, rope_theta: float, q=None, q_out=None, err=None):
    """spd_op_append_paged into an int8 cache: codes to K and V, a scale per row to K_scale and V_scale."""
    torch, where = _torch(), "spd_op_append_paged_q8"
    i8, i32, device = torch.int8, torch.int32, torch.cuda.current_device()
    shape = K.shape
    n_pages, n_kv, page_size, d = shape
    n_seq, entries = table.shape
    n = seq.numel()
    if not (K.dtype is i8 and V.dtype is i8 and table.dtype is i32 and seq.dtype is i32 and pos.dtype is i32 and V.shape == shape and pos.numel() == n
            and K.is_contiguous() and V.is_contiguous() and table.is_contiguous() and seq.is_contiguous() and pos.is_contiguous()
            and K.get_device() == device and V.get_device() == device and table.get_device() == device and seq.get_device() == device and pos.get_device() == device
            and (err is None or (err.dtype is i32 and err.numel() == 1 and err.get_device() == device))):
        _refuse(where, device, K=(K, i8, None), V=(V, i8, shape), table=(table, i32, None), seq=(seq, i32, (n,)), pos=(pos, i32, (n,)), err=(err, i32, (1,)))
    scales = _scales(where, torch, "int8", device, shape, K_scale, V_scale)
    kv_stride, q_ptr, q_stride, heads, out_ptr = _new_rows(where, torch, device, k, v, q, q_out, n, n_kv, d)
    rc = lib().spd_op_append_paged_q8(K.data_ptr(), V.data_ptr(), *scales, table.data_ptr(), n_pages, n_kv, page_size, d, n_seq, entries, q_ptr, q_stride, k.data_ptr(),
                                      v.data_ptr(), kv_stride, seq.data_ptr(), pos.data_ptr(), n, heads, rope_theta, out_ptr, None if err is None else err.data_ptr(), _stream_ptr(device))
    if rc:
        raise SpdError(rc, where)


def spd_op_read_paged(dtype: str, K, V, table, seq, pos, k_out, v_out, K_scale=None, V_scale=None, err=None):
    """Cached rows back: k_out, v_out [tokens, n_kv_heads, d_head], float32, float16 or bfloat16; seq < 0: padding."""
    torch, where = _torch(), "spd_op_read_paged"
    kv, i32, device = _cache_type(where, torch, dtype), torch.int32, torch.cuda.current_device()
    shape = K.shape
    n_pages, n_kv, page_size, d = shape
    n_seq, entries = table.shape
    n, kind = seq.numel(), k_out.dtype
    if not (K.dtype is kv and V.dtype is kv and table.dtype is i32 and seq.dtype is i32 and pos.dtype is i32 and V.shape == shape and pos.numel() == n and v_out.dtype is kind
            and k_out.numel() == n * n_kv * d and v_out.numel() == n * n_kv * d and K.is_contiguous() and V.is_contiguous() and table.is_contiguous() and seq.is_contiguous()
            and pos.is_contiguous() and k_out.is_contiguous() and v_out.is_contiguous() and K.get_device() == device and V.get_device() == device and table.get_device() == device
            and seq.get_device() == device and pos.get_device() == device and k_out.get_device() == device and v_out.get_device() == device
            and (err is None or (err.dtype is i32 and err.numel() == 1 and err.get_device() == device))):
        _refuse(where, device, K=(K, kv, None), V=(V, kv, shape), table=(table, i32, None), seq=(seq, i32, (n,)), pos=(pos, i32, (n,)), k_out=(k_out, kind, (n, n_kv, d)),
                v_out=(v_out, kind, (n, n_kv, d)), err=(err, i32, (1,)))
    scales = _scales(where, torch, dtype, device, shape, K_scale, V_scale)
    rc = lib().spd_op_read_paged(SPD_DTYPE[dtype], K.data_ptr(), V.data_ptr(), *scales, table.data_ptr(), n_pages, n_kv, page_size, d, n_seq, entries, seq.data_ptr(), pos.data_ptr(),
                                 n, SPD_DTYPE[_io_type(where, torch, kind)], k_out.data_ptr(), v_out.data_ptr(), None if err is None else err.data_ptr(), _stream_ptr(device))
    if rc:
        raise SpdError(rc, where)


def spd_op_attention_paged(dtype: str, q, K, V, table, first, length, out, max_new: int, max_len: int, K_scale=None, V_scale=None, err=None):
    """q [tokens, n_heads, d_head] (tokens may lie apart) -> out, both float32 or both the cache's type (int8 cache: float16 or bfloat16); first int32 [n_seq + 1], length int32 [n_seq]."""
    torch, where = _torch(), "spd_op_attention_paged"
    kv, i32, device, kind = _cache_type(where, torch, dtype), torch.int32, torch.cuda.current_device(), q.dtype
    shape = K.shape
    n_pages, n_kv, page_size, d = shape
    n_seq, entries = table.shape
    n, heads, q_d = q.shape
    q_stride, between, within = q.stride()
    if n <= 1:                          # (a single token's stride may be anything)
        q_stride = heads * d
    if max_new > _INT32 or max_len > _INT32:
        raise ValueError(f"{where}: max_new or max_len is no 32-bit number")
    if q_d != d or within != 1 or (between != d and heads > 1) or q.get_device() != device:
        raise ValueError(f"{where}: q has to be [tokens, heads, {d}] on the current device, a token's heads one behind the other")
    if not (out.dtype is kind and K.dtype is kv and V.dtype is kv and table.dtype is i32 and first.dtype is i32 and length.dtype is i32 and out.numel() == n * heads * d
            and V.shape == shape and first.numel() == n_seq + 1 and length.numel() == n_seq and out.is_contiguous() and K.is_contiguous() and V.is_contiguous()
            and table.is_contiguous() and first.is_contiguous() and length.is_contiguous() and out.get_device() == device and K.get_device() == device and V.get_device() == device
            and table.get_device() == device and first.get_device() == device and length.get_device() == device
            and (err is None or (err.dtype is i32 and err.numel() == 1 and err.get_device() == device))):
        _refuse(where, device, K=(K, kv, None), V=(V, kv, shape), table=(table, i32, None), first=(first, i32, (n_seq + 1,)), length=(length, i32, (n_seq,)), out=(out, kind, (n, heads, d)),
                err=(err, i32, (1,)))
    scales = _scales(where, torch, dtype, device, shape, K_scale, V_scale)
    L, kinds = lib(), (SPD_DTYPE[dtype], SPD_DTYPE[_io_type(where, torch, kind)])
    n_bytes, scratch = L.spd_op_attention_paged_scratch_bytes(*kinds, n_seq, n, heads, n_kv, d, max_new, max_len), None
    if n_bytes:
        buf = _scratch(torch, n_bytes, q)
        scratch = buf.data_ptr()
    rc = L.spd_op_attention_paged(*kinds, q.data_ptr(), q_stride, K.data_ptr(), V.data_ptr(), *scales, table.data_ptr(), n_pages, n_kv, page_size, d, n_seq, entries, first.data_ptr(),
                                  length.data_ptr(), n, heads, max_new, max_len, out.data_ptr(), scratch, n_bytes, None if err is None else err.data_ptr(), _stream_ptr(device))
    if rc:
        raise SpdError(rc, where)


def spd_op_verify_drafts(dtype: str, logits, tokens, first, u, out_tokens, out_logprobs, out_accepted, tau: float = 1.0, draft_logits=None, draft_tau: float = 1.0, err=None):
    """logits, draft_logits [tokens, vocab] (rows may lie apart), tokens int32 and u float32 [tokens], first int32 [n_seq + 1] -> out_tokens, out_logprobs [tokens], out_accepted [n_seq]."""
    torch, where = _torch(), "spd_op_verify_drafts"
    kind, i32, f32, device = _kv_type(where, torch, dtype), torch.int32, torch.float32, torch.cuda.current_device()
    n, vocab = logits.shape
    n_seq = first.numel() - 1

    def rows(name, t):
        stride, within = t.stride()
        if t.dtype is not kind or t.shape != (n, vocab) or (within != 1 and vocab > 1) or t.get_device() != device:
            raise ValueError(f"{where}: {name} has to be {dtype} [{n}, {vocab}] on the current device, whole rows")
        return stride if n > 1 else vocab

    stride, draft_stride = rows("logits", logits), rows("draft_logits", draft_logits) if draft_logits is not None else 0
    if not (tokens.dtype is i32 and first.dtype is i32 and u.dtype is f32 and out_tokens.dtype is i32 and out_logprobs.dtype is f32 and out_accepted.dtype is i32 and n_seq >= 0
            and tokens.numel() == n and u.numel() == n and out_tokens.numel() == n and out_logprobs.numel() == n and out_accepted.numel() == n_seq
            and tokens.is_contiguous() and first.is_contiguous() and u.is_contiguous() and out_tokens.is_contiguous() and out_logprobs.is_contiguous() and out_accepted.is_contiguous()
            and tokens.get_device() == device and first.get_device() == device and u.get_device() == device and out_tokens.get_device() == device
            and out_logprobs.get_device() == device and out_accepted.get_device() == device and (err is None or (err.dtype is i32 and err.numel() == 1 and err.get_device() == device))):
        if n_seq < 0:
            raise ValueError(f"{where}: first has one element more than there are sequences")
        _refuse(where, device, tokens=(tokens, i32, (n,)), first=(first, i32, None), u=(u, f32, (n,)), out_tokens=(out_tokens, i32, (n,)), out_logprobs=(out_logprobs, f32, (n,)),
                out_accepted=(out_accepted, i32, (n_seq,)), err=(err, i32, (1,)))
    L = lib()
    n_bytes, scratch = L.spd_op_verify_drafts_scratch_bytes(n_seq, n, vocab), None
    if n_bytes:
        buf = _scratch(torch, n_bytes, logits)
        scratch = buf.data_ptr()
    rc = L.spd_op_verify_drafts(SPD_DTYPE[dtype], logits.data_ptr(), stride, None if draft_logits is None else draft_logits.data_ptr(), draft_stride, tokens.data_ptr(), first.data_ptr(),
                                u.data_ptr(), n_seq, n, vocab, tau, draft_tau, out_tokens.data_ptr(), out_logprobs.data_ptr(), out_accepted.data_ptr(), scratch, n_bytes,
                                None if err is None else err.data_ptr(), _stream_ptr(device))
    if rc:
        raise SpdError(rc, where)


def spd_test_state_layout():
    words, err_word = C.c_size_t(0), C.c_size_t(0)
    rc = lib().spd_test_state_layout(C.byref(words), C.byref(err_word))
    if rc:
        raise SpdError(rc, "spd_test_state_layout")
    return words.value, err_word.value


def spd_test_state_status(state_words) -> int:
    a = np.ascontiguousarray(state_words, dtype=np.int32)
    return lib().spd_test_state_status(_np_ptr(a), a.size)


def spd_test_ngram_table(tables: dict, vocab: int):
    """-> (slots [n, 8] int32: six token ids, count as two words; longest displacement)."""
    t, _keep = ngram_struct(tables, (0, 0, 0, 0, 0))
    slots, probe = np.zeros((spd_ngram_table_bytes(tables) // 32, 8), np.int32), C.c_int32(0)
    rc = lib().spd_test_ngram_table(C.byref(t), vocab, _np_ptr(slots), slots.nbytes, C.byref(probe))
    if rc:
        raise SpdError(rc, "spd_test_ngram_table")
    return slots, probe.value


def spd_test_prefill_cut(cfg: SpdModelCfg, num_cu: int, n_tokens: int, product: int):
    """-> (tokens and columns of a tile, blocks that share a tile's k range, epilogue in the product)."""
    out = np.zeros(4, np.int32)
    rc = lib().spd_test_prefill_cut(C.byref(cfg), num_cu, n_tokens, product, _np_ptr(out))
    if rc:
        raise SpdError(rc, "spd_test_prefill_cut")
    return int(out[0]), int(out[1]), int(out[2]), bool(out[3])


def spd_test_attention_shared_cut(dtype: str, n_seq: int, width: int, n_heads: int, n_kv_heads: int, d_head: int, max_shared: int, max_own: int):
    """-> (shared chunks, positions of one, own chunks, rows of a shared block, shared blocks, keys of a stage, stages)."""
    out = np.zeros(7, np.int32)
    rc = lib().spd_test_attention_shared_cut(SPD_DTYPE[dtype], n_seq, width, n_heads, n_kv_heads, d_head, max_shared, max_own, _np_ptr(out))
    if rc:
        raise SpdError(rc, "spd_test_attention_shared_cut")
    return tuple(int(x) for x in out)


def spd_test_beam_select_cut(n_groups: int, n_in: int, n_out: int, vocab: int):
    """-> (logits per lane of a slice, 0 where there is one launch; slices of a row)."""
    out = np.zeros(2, np.int32)
    rc = lib().spd_test_beam_select_cut(n_groups, n_in, n_out, vocab, _np_ptr(out))
    if rc:
        raise SpdError(rc, "spd_test_beam_select_cut")
    return int(out[0]), int(out[1])


def spd_test_prefill_attention(kv_dtype: str, q, K, V, pos: int):
    """Causal attention of a prefix chunk's queries [tokens, heads, d_head] over the cache: (hi, lo), two bfloat16 tensors."""
    torch = _torch()
    n_tokens, n_heads, d_head = q.shape
    n_kv, cap_ctx, _ = K.shape
    hi, lo = (torch.empty(q.shape, dtype=torch.bfloat16, device=q.device) for _ in range(2))
    rc = lib().spd_test_prefill_attention(SPD_DTYPE[kv_dtype], q.data_ptr(), K.data_ptr(), V.data_ptr(), hi.data_ptr(), lo.data_ptr(),
                                          n_tokens, pos, n_heads, n_kv, d_head, cap_ctx, _stream_ptr())
    if rc:
        raise SpdError(rc, "spd_test_prefill_attention")
    return hi, lo
