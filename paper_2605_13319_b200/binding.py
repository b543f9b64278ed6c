"""ctypes binding of libpipesd.so (include/pipesd.h): argument marshalling only.

PyTorch is used for device memory and streams; every step of the verify pass runs in the CUDA
kernels behind the C ABI.  There is no CPU or library fallback: if the shared library is missing
or fails to load, importing a symbol from here raises.
"""
from __future__ import annotations

import ctypes
from pathlib import Path

import numpy as np

_HERE = Path(__file__).resolve().parent
LIB_PATH = _HERE / "libpipesd.so"
_lib = None

OK, E_INVALID, E_FULL, E_OOM_PAGES, E_STATE, E_RANGE, E_CUDA, E_NOMEM = 0, -1, -2, -3, -4, -5, -6, -7
E_TOO_LARGE = -8
STATIC_SCRATCH_BYTES = 8 << 20
MODE_STOCHASTIC, MODE_GREEDY = 0, 1
Q_HOST, AUTOCOMMIT, CHAIN = 1, 2, 4
TOKEN_PENDING = -1
F32, BF16 = 0, 1
DISCARDED = 1

i32, u32, u64, f32, vp = ctypes.c_int32, ctypes.c_uint32, ctypes.c_uint64, ctypes.c_float, ctypes.c_void_p
i64 = ctypes.c_int64


class ModelCfg(ctypes.Structure):
    _fields_ = [(n, i32) for n in ("n_layers", "d_model", "n_q_heads", "n_kv_heads", "head_dim", "d_ffn", "vocab")] \
        + [("rms_eps", f32), ("rope_base", f32)] \
        + [(n, i32) for n in ("page_size", "n_pages", "max_requests", "max_draft", "max_rows", "max_seq", "device", "reserved")]


class LayerWeights(ctypes.Structure):
    _fields_ = [(n, vp) for n in ("wq", "wk", "wv", "wo", "wg", "wu", "wd", "attn_norm", "ffn_norm")]


class Weights(ctypes.Structure):
    _fields_ = [("tok_emb", vp), ("lm_head", vp), ("final_norm", vp), ("layers", ctypes.POINTER(LayerWeights))]


class Sizes(ctypes.Structure):
    _fields_ = [("weights_bytes", u64), ("kv_bytes", u64), ("workspace_bytes", u64)]


class Mem(ctypes.Structure):
    _fields_ = [("weights", vp), ("weights_bytes", u64), ("kv", vp), ("kv_bytes", u64),
                ("workspace", vp), ("workspace_bytes", u64)]


class VerifyItem(ctypes.Structure):
    _fields_ = [("req", i32), ("k", i32), ("mode", i32), ("reserved", i32),
                ("tokens", vp), ("q", vp), ("u", vp)]


class VerifyResult(ctypes.Structure):
    _fields_ = [("n_accepted", i32), ("next_token", i32), ("status", i32), ("reserved", i32)]


class ProfileInfo(ctypes.Structure):
    _fields_ = [("kernel_launches", ctypes.c_int64), ("gemm_launches", ctypes.c_int64),
                ("gemm_ms", ctypes.c_double), ("gemm_bytes", ctypes.c_double)]


class Kv4Cfg(ctypes.Structure):
    _fields_ = [(n, i32) for n in ("n_kv_heads", "head_dim", "page_size", "n_pages", "max_pages", "reserved")]


class Kv16Cfg(ctypes.Structure):
    _fields_ = [(n, i32) for n in ("n_layers", "n_kv_heads", "head_dim", "page_size", "n_pages", "max_pages", "reserved")]


# name -> (restype, argtypes); mirrors include/pipesd.h one to one
_SIGNATURES = {
    "pipesd_strerror": (ctypes.c_char_p, [i32]),
    "pipesd_last_error": (ctypes.c_char_p, [vp]),
    "pipesd_query_sizes": (i32, [ctypes.POINTER(ModelCfg), ctypes.POINTER(Sizes)]),
    "pipesd_ctx_create": (i32, [ctypes.POINTER(ModelCfg), ctypes.POINTER(Weights), ctypes.POINTER(Mem), vp,
                                ctypes.POINTER(vp)]),
    "pipesd_ctx_destroy": (i32, [vp]),
    "pipesd_ctx_sync": (i32, [vp]),
    "pipesd_req_open": (i32, [vp, ctypes.POINTER(i32)]),
    "pipesd_req_close": (i32, [vp, i32]),
    "pipesd_req_len": (i32, [vp, i32, ctypes.POINTER(i32)]),
    "pipesd_prefill": (i32, [vp, i32, vp, i32, vp]),
    "pipesd_verify": (i32, [vp, i32, ctypes.POINTER(VerifyItem), ctypes.POINTER(VerifyResult), u32]),
    "pipesd_kv_rollback": (i32, [vp, i32, vp, vp, vp]),
    "pipesd_debug_get_logits": (i32, [vp, vp, i32]),
    "pipesd_debug_read_kv": (i32, [vp, i32, i32, i32, i32, vp, vp]),
    "pipesd_debug_write_kv": (i32, [vp, i32, i32, i32, i32, vp, vp]),
    "pipesd_reject_from_logits": (i32, [vp, i32, i32, vp, vp, vp, vp, ctypes.POINTER(VerifyResult)]),
    "pipesd_debug_set_len": (i32, [vp, i32, i32]),
    "pipesd_profile_enable": (i32, [vp, i32]),
    "pipesd_profile_read": (i32, [vp, ctypes.POINTER(ProfileInfo)]),
    "pipesd_gemm_packed_bytes": (u64, [i32, i32]),
    "pipesd_gemm_scratch_bytes": (u64, [i32, i32, i32]),
    "pipesd_gemm_pack": (i32, [vp, vp, i32, i32, vp]),
    "pipesd_gemm_run": (i32, [vp, vp, vp, vp, i32, i32, i32, vp]),
    "pipesd_gemm_run_static": (i32, [vp, vp, vp, i32, i32, i32, vp]),
    "pipesd_sample": (i32, [vp, i32, i64, i32, i32, vp, vp, vp, vp, i64, vp]),
    "pipesd_accept_scratch_bytes": (u64, [i32]),
    "pipesd_accept": (i32, [vp, i32, i64, i32, i32, i32, vp, vp, vp, i64, vp, vp, vp, vp, vp, vp]),
    "pipesd_kv4_pool_bytes": (u64, [ctypes.POINTER(Kv4Cfg)]),
    "pipesd_kv4_append": (i32, [ctypes.POINTER(Kv4Cfg), vp, vp, vp, i32, i64, i64, i32, i32, vp, vp, vp, vp]),
    "pipesd_kv4_read": (i32, [ctypes.POINTER(Kv4Cfg), vp, vp, vp, i32, i32, vp, vp, vp, vp]),
    "pipesd_kv4_attend_scratch_bytes": (u64, [ctypes.POINTER(Kv4Cfg)]),
    "pipesd_kv4_attend": (i32, [ctypes.POINTER(Kv4Cfg), vp, vp, vp, i32, i64, i64, i32, f32, i32, i32, vp, vp, vp, vp, vp]),
    "pipesd_attend_packed": (i32, [vp, vp, vp, vp, i64, i64, i64, i64, i32, i32, i32, f32, i32, i32, vp, vp]),
    "pipesd_tree_mask": (i32, [i32, i32, vp, vp, i32, vp, vp, vp]),
    "pipesd_debug_attend_gives_up": (i32, [i32]),
    "pipesd_kv16_pool_bytes": (u64, [ctypes.POINTER(Kv16Cfg)]),
    "pipesd_kv16_append": (i32, [ctypes.POINTER(Kv16Cfg), vp, i32, vp, vp, i32, i64, i64, i32, i32, vp, vp, vp, vp]),
    "pipesd_kv16_read": (i32, [ctypes.POINTER(Kv16Cfg), vp, i32, vp, vp, i32, i32, vp, vp, vp, vp]),
    "pipesd_kv16_attend_scratch_bytes": (u64, [ctypes.POINTER(Kv16Cfg), i32, i32]),
    "pipesd_kv16_attend": (i32, [ctypes.POINTER(Kv16Cfg), vp, i32, vp, vp, i32, i64, i64, i32, f32, i32, i32, vp, vp, vp, vp, i32, vp, vp]),
    "pipesd_kv16_plan_scratch_bytes": (u64, [ctypes.POINTER(Kv16Cfg), i32]),
    "pipesd_kv16_reserve": (i32, [ctypes.POINTER(Kv16Cfg), i32, vp, vp, vp, vp, vp, vp]),
    "pipesd_kv16_fork": (i32, [ctypes.POINTER(Kv16Cfg), vp, i32, vp, vp, vp, vp, i32, vp, vp, vp, vp, vp]),
    "pipesd_kv16_compact": (i32, [ctypes.POINTER(Kv16Cfg), vp, i32, vp, i32, vp, vp, vp, vp]),
    "pipesd_kv16_release": (i32, [ctypes.POINTER(Kv16Cfg), i32, vp, vp, vp, vp]),
    "pipesd_sched_round_time": (i32, [i32, ctypes.c_double, ctypes.c_double, ctypes.c_double, vp, i32,
                                      ctypes.POINTER(ctypes.c_double)]),
    "pipesd_sched_optimal_batching": (i32, [i32, ctypes.c_double, ctypes.c_double, ctypes.c_double, vp,
                                            ctypes.POINTER(i32), ctypes.POINTER(ctypes.c_double)]),
    "pipesd_sched_trigger_step": (i32, [ctypes.POINTER(ctypes.c_double), ctypes.c_double, ctypes.c_double,
                                        ctypes.c_double, ctypes.POINTER(i32)]),
    "pipesd_debug_force_dense": (i32, [vp, i32]),
    "pipesd_share_device": (i32, [vp, i32]),
    "pipesd_debug_merge_polls": (i32, [vp, i32]),
    "pipesd_debug_stack_ctas": (i32, [vp, i32]),
    "pipesd_debug_stack_looks": (i32, [vp, i32]),
    "pipesd_debug_prefill_chunk": (i32, [ctypes.POINTER(ModelCfg), i32, i32, ctypes.POINTER(ctypes.c_int32), ctypes.POINTER(ctypes.c_int32)]),
    "pipesd_debug_gemm_dense_scratch_bytes": (u64, [i32, i32, i32]),
    "pipesd_debug_gemm_dense": (i32, [vp, vp, vp, vp, i32, i32, i32, i32, i32, vp]),
    "pipesd_debug_attn_slots": (i32, [vp, i32, ctypes.POINTER(ctypes.c_int32)]),
    "pipesd_debug_attn_split": (i32, [i32, i32, ctypes.POINTER(ctypes.c_int32), i32, ctypes.POINTER(ctypes.c_int32)]),
    "pipesd_debug_req_state": (i32, [vp, i32, ctypes.POINTER(ctypes.c_int32)]),
    "pipesd_debug_wait_timeout": (i32, [vp, i32]),
}


def lib():
    """Load libpipesd.so (no fallback: a missing library is an error)."""
    global _lib
    if _lib is None:
        if not LIB_PATH.exists():
            raise RuntimeError(f"{LIB_PATH} is missing: build it with paper_2605_13319_b200.build.build_cuda(); "
                               "there is no CPU path")
        L = ctypes.CDLL(str(LIB_PATH))
        for name, (res, args) in _SIGNATURES.items():
            fn = getattr(L, name)
            fn.restype, fn.argtypes = res, args
        _lib = L
    return _lib


class PipesdError(RuntimeError):
    def __init__(self, code, where, detail=""):
        self.code = code
        msg = lib().pipesd_strerror(code).decode()
        super().__init__(f"{where}: {msg} ({code}) {detail}")


def _np_ptr(a):
    return a.ctypes.data if a is not None else None


class Context:
    """One verification context: a Llama-style target model, its paged KV pool and workspace.

    Method names follow the C entry points (pipesd_<name>)."""

    def __init__(self, shape, weights: dict, *, n_pages: int, max_requests: int = 1, max_draft: int = 16,
                 max_rows: int | None = None, max_seq: int = 4096, page_size: int = 16, device: int = 0,
                 stream=None, poison: bool = False):
        import torch
        if not torch.cuda.is_available():
            raise RuntimeError("a CUDA device is required: the verify pass has no CPU path")
        self.torch = torch
        self.shape = shape
        self.device = torch.device("cuda", device)
        torch.cuda.set_device(self.device)
        self.stream = stream if stream is not None else torch.cuda.current_stream(self.device)
        if max_rows is None:
            max_rows = max(max_draft + 1, 32)
        self.cfg = ModelCfg(shape.n_layers, shape.d_model, shape.n_q_heads, shape.n_kv_heads, shape.head_dim,
                            shape.d_ffn, shape.vocab, shape.rms_eps, shape.rope_base, page_size, n_pages,
                            max_requests, max_draft, max_rows, max_seq, device, 0)
        L = lib()
        sz = Sizes()
        rc = L.pipesd_query_sizes(ctypes.byref(self.cfg), ctypes.byref(sz))
        if rc != OK:
            raise PipesdError(rc, "pipesd_query_sizes")
        self.sizes = sz
        with torch.cuda.stream(self.stream):
            self._wbuf = torch.empty(sz.weights_bytes, dtype=torch.uint8, device=self.device)
            self._kvbuf = torch.empty(sz.kv_bytes, dtype=torch.uint8, device=self.device)
            self._wsbuf = torch.zeros(sz.workspace_bytes, dtype=torch.uint8, device=self.device)
            if poison:
                # Every byte 0xFF: NaN as bf16 and as fp32, -1 as an index.  A read of a K/V row or of a workspace
                # element that this library did not write first then shows up in the results instead of passing
                # silently (pipesd_ctx_create initialises what it relies on itself).
                self._kvbuf.fill_(0xFF)
                self._wsbuf.fill_(0xFF)
            # upload the caller's row-major bf16 tensors; they are released after the repack
            up = lambda a: torch.from_numpy(a).to(self.device, non_blocking=False)
            lw = (LayerWeights * shape.n_layers)()
            keep = []
            for i, l in enumerate(weights["layers"]):
                for name in ("wq", "wk", "wv", "wo", "wg", "wu", "wd"):
                    t = up(l[name].view(np.int16))
                    keep.append(t)
                    setattr(lw[i], name, t.data_ptr())
                for name in ("attn_norm", "ffn_norm"):
                    t = up(l[name])
                    keep.append(t)
                    setattr(lw[i], name, t.data_ptr())
            te, lh, fn = up(weights["tok_emb"].view(np.int16)), up(weights["lm_head"].view(np.int16)), \
                up(weights["final_norm"])
            w = Weights(te.data_ptr(), lh.data_ptr(), fn.data_ptr(), lw)
            mem = Mem(self._wbuf.data_ptr(), sz.weights_bytes, self._kvbuf.data_ptr(), sz.kv_bytes,
                      self._wsbuf.data_ptr(), sz.workspace_bytes)
            h = vp()
            rc = L.pipesd_ctx_create(ctypes.byref(self.cfg), ctypes.byref(w), ctypes.byref(mem),
                                     vp(self.stream.cuda_stream), ctypes.byref(h))
            if rc != OK:
                raise PipesdError(rc, "pipesd_ctx_create")
            self._h = h
            self.ctx_sync()
            del keep, te, lh, fn
        self._alive = []   # host arrays referenced by an in-flight verify

    # -- helpers
    def _check(self, rc, where):
        if rc != OK:
            raise PipesdError(rc, where, lib().pipesd_last_error(self._h).decode())

    def close(self):
        if getattr(self, "_h", None):
            lib().pipesd_ctx_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # -- C entry points
    def ctx_sync(self):
        self._check(lib().pipesd_ctx_sync(self._h), "pipesd_ctx_sync")
        self._alive = []

    def share_device(self, share: bool = True):
        """Other work shares the device: no pass takes all of its SMs at once."""
        self._check(lib().pipesd_share_device(self._h, int(share)), "pipesd_share_device")

    def req_open(self) -> int:
        r = i32()
        self._check(lib().pipesd_req_open(self._h, ctypes.byref(r)), "pipesd_req_open")
        return r.value

    def req_close(self, req: int):
        self._check(lib().pipesd_req_close(self._h, req), "pipesd_req_close")

    def req_len(self, req: int) -> int:
        n = i32()
        self._check(lib().pipesd_req_len(self._h, req, ctypes.byref(n)), "pipesd_req_len")
        return n.value

    def prefill(self, req: int, tokens, want_last_logits: bool = False):
        t = np.ascontiguousarray(tokens, np.int32)
        out = np.empty(self.shape.vocab, np.float32) if want_last_logits else None
        self._check(lib().pipesd_prefill(self._h, req, _np_ptr(t), t.size, _np_ptr(out)), "pipesd_prefill")
        return out

    def verify(self, items, flags: int = 0, sync: bool = True):
        """items: list of dict(req, tokens[k+1], q (torch cuda tensor / numpy with Q_HOST / None), u[k+1], mode).
        Returns a list of (n_accepted, next_token) when sync, else the ctypes result array (filled by ctx_sync)."""
        n = len(items)
        arr = (VerifyItem * n)()
        res = (VerifyResult * n)()
        alive = [arr, res]
        for i, it in enumerate(items):
            tok = np.ascontiguousarray(it["tokens"], np.int32)
            k = tok.size - 1
            u = it.get("u")
            u = np.ascontiguousarray(u, np.float32) if u is not None else None
            q = it.get("q")
            if q is None:
                qp = None
            elif isinstance(q, np.ndarray):
                assert flags & Q_HOST, "numpy q needs the Q_HOST flag"
                q = np.ascontiguousarray(q, np.float32)
                assert q.shape == (k, self.shape.vocab)
                qp = q.ctypes.data
            else:
                assert q.is_cuda and q.dtype == self.torch.float32 and q.is_contiguous()
                assert tuple(q.shape) == (k, self.shape.vocab)
                qp = q.data_ptr()
            alive += [tok, u, q]
            arr[i] = VerifyItem(it["req"], k, it.get("mode", MODE_STOCHASTIC), 0, tok.ctypes.data, qp,
                                u.ctypes.data if u is not None else None)
        self._alive = self._alive + alive if (flags & CHAIN) else alive
        self._check(lib().pipesd_verify(self._h, n, arr, res, flags), "pipesd_verify")
        if not sync:
            return res
        self.ctx_sync()
        return [(r.n_accepted, r.next_token) for r in res]

    def kv_rollback(self, reqs, n_accepted, next_token=None):
        r = np.ascontiguousarray(reqs, np.int32)
        a = np.ascontiguousarray(n_accepted, np.int32)
        t = np.ascontiguousarray(next_token, np.int32) if next_token is not None else None
        self._check(lib().pipesd_kv_rollback(self._h, r.size, _np_ptr(r), _np_ptr(a), _np_ptr(t)), "pipesd_kv_rollback")

    def debug_req_state(self, req: int):
        out = (ctypes.c_int32 * 3)()
        self._check(lib().pipesd_debug_req_state(self._h, req, out), "pipesd_debug_req_state")
        return tuple(out)

    def debug_force_dense(self, on: int):
        """0: off; 1: every pass on the dense kernel; n > 1: planned like a pass of n rows."""
        self._check(lib().pipesd_debug_force_dense(self._h, int(on)), "pipesd_debug_force_dense")

    def debug_merge_polls(self, polls: int):
        self._check(lib().pipesd_debug_merge_polls(self._h, polls), "pipesd_debug_merge_polls")

    def debug_stack_ctas(self, ctas: int):
        """CTAs of the layer-stack kernel; 0: one per SM."""
        self._check(lib().pipesd_debug_stack_ctas(self._h, ctas), "pipesd_debug_stack_ctas")

    def debug_stack_looks(self, looks: int):
        """Looks after which a CTA of the layer-stack kernel no longer waits for the others; 0: its own limit."""
        self._check(lib().pipesd_debug_stack_looks(self._h, looks), "pipesd_debug_stack_looks")

    def debug_attn_slots(self, rows_per_kv_head: int):
        out = (ctypes.c_int32 * 2)()
        self._check(lib().pipesd_debug_attn_slots(self._h, rows_per_kv_head, out), "pipesd_debug_attn_slots")
        return tuple(out)

    def debug_wait_timeout(self, limit_us: int):
        self._check(lib().pipesd_debug_wait_timeout(self._h, limit_us), "pipesd_debug_wait_timeout")

    def debug_get_logits(self, rows: int) -> np.ndarray:
        out = np.empty((rows, self.shape.vocab), np.float32)
        self._check(lib().pipesd_debug_get_logits(self._h, _np_ptr(out), rows), "pipesd_debug_get_logits")
        return out

    def debug_read_kv(self, req: int, layer: int, pos0: int, n_pos: int):
        w = self.shape.n_kv_heads * self.shape.head_dim
        k = np.empty((n_pos, w), np.uint16)
        v = np.empty((n_pos, w), np.uint16)
        self._check(lib().pipesd_debug_read_kv(self._h, req, layer, pos0, n_pos, _np_ptr(k), _np_ptr(v)),
                    "pipesd_debug_read_kv")
        return k, v

    def debug_write_kv(self, req: int, layer: int, pos0: int, k_bf16, v_bf16):
        k = np.ascontiguousarray(k_bf16, np.uint16)
        v = np.ascontiguousarray(v_bf16, np.uint16)
        self._check(lib().pipesd_debug_write_kv(self._h, req, layer, pos0, k.shape[0], _np_ptr(k), _np_ptr(v)),
                    "pipesd_debug_write_kv")

    def debug_set_len(self, req: int, new_len: int):
        self._check(lib().pipesd_debug_set_len(self._h, req, new_len), "pipesd_debug_set_len")

    def profile_enable(self, time_gemms: bool = False):
        self._check(lib().pipesd_profile_enable(self._h, int(time_gemms)), "pipesd_profile_enable")

    def profile_read(self) -> dict:
        info = ProfileInfo()
        self._check(lib().pipesd_profile_read(self._h, ctypes.byref(info)), "pipesd_profile_read")
        return dict(kernel_launches=info.kernel_launches, gemm_launches=info.gemm_launches,
                    gemm_ms=info.gemm_ms, gemm_bytes=info.gemm_bytes)

    def reject_from_logits(self, logits, q, drafts, u, mode: int = MODE_STOCHASTIC):
        logits = np.ascontiguousarray(logits, np.float32)
        k = logits.shape[0] - 1
        q = np.ascontiguousarray(q, np.float32) if q is not None else None
        drafts = np.ascontiguousarray(drafts, np.int32)
        u = np.ascontiguousarray(u, np.float32)
        res = VerifyResult()
        self._check(lib().pipesd_reject_from_logits(self._h, k, mode, _np_ptr(logits), _np_ptr(q), _np_ptr(drafts),
                                                    _np_ptr(u), ctypes.byref(res)), "pipesd_reject_from_logits")
        return res.n_accepted, res.next_token


# ---- stand-alone GEMM entry points
def gemm_pack(W, stream=None):
    """W: torch cuda int16/bfloat16 tensor [N,K] (bf16 bit patterns) -> packed torch uint8 tensor."""
    import torch
    N, K = W.shape
    packed = torch.empty(lib().pipesd_gemm_packed_bytes(N, K), dtype=torch.uint8, device=W.device)
    st = stream if stream is not None else torch.cuda.current_stream(W.device)
    rc = lib().pipesd_gemm_pack(W.data_ptr(), packed.data_ptr(), N, K, vp(st.cuda_stream))
    if rc != OK:
        raise PipesdError(rc, "pipesd_gemm_pack")
    return packed


def gemm_scratch(M, N, K, device):
    import torch
    return torch.empty(max(int(lib().pipesd_gemm_scratch_bytes(M, N, K)), 16), dtype=torch.uint8, device=device)


def gemm_run(packed, x, y, scratch, N, K, stream=None):
    import torch
    M = x.shape[0]
    assert x.dtype == torch.float32 and y.dtype == torch.float32 and x.is_contiguous() and y.is_contiguous()
    assert x.shape[1] == K and tuple(y.shape) == (M, N)
    st = stream if stream is not None else torch.cuda.current_stream(x.device)
    rc = lib().pipesd_gemm_run(packed.data_ptr(), x.data_ptr(), y.data_ptr(), scratch.data_ptr(), M, N, K,
                               vp(st.cuda_stream))
    if rc != OK:
        raise PipesdError(rc, "pipesd_gemm_run")


def gemm_run_static(packed, x, y, N, K, stream=None):
    """pipesd_gemm_run_static: the GEMM with its split-K scratch inside the library, for callers that may
    not allocate device memory.  Same arguments as gemm_run minus the scratch tensor; nothing is allocated
    here either (the tensors are the caller's).  Raises PipesdError(E_TOO_LARGE) beyond the built-in limit."""
    import torch
    M = x.shape[0]
    assert x.dtype == torch.float32 and y.dtype == torch.float32 and x.is_contiguous() and y.is_contiguous()
    assert x.shape[1] == K and tuple(y.shape) == (M, N)
    st = stream if stream is not None else torch.cuda.current_stream(x.device)
    rc = lib().pipesd_gemm_run_static(packed.data_ptr(), x.data_ptr(), y.data_ptr(), M, N, K, vp(st.cuda_stream))
    if rc != OK:
        raise PipesdError(rc, "pipesd_gemm_run_static")


def debug_gemm_dense(packed, x, y, scratch, N, K, tokens_per_cta, slices):
    """The dense projection kernel alone, in a given plan.  scratch: uint8 tensor of at least
    pipesd_debug_gemm_dense_scratch_bytes(M, K, tokens_per_cta) bytes."""
    import torch
    M = x.shape[0]
    assert x.dtype == torch.float32 and y.dtype == torch.float32 and x.is_contiguous() and y.is_contiguous()
    assert x.shape[1] == K and tuple(y.shape) == (M, N)
    assert scratch.numel() * scratch.element_size() >= lib().pipesd_debug_gemm_dense_scratch_bytes(M, K, tokens_per_cta)
    st = torch.cuda.current_stream(x.device)
    rc = lib().pipesd_debug_gemm_dense(packed.data_ptr(), x.data_ptr(), y.data_ptr(), scratch.data_ptr(), M, N, K,
                                       tokens_per_cta, slices, vp(st.cuda_stream))
    if rc != OK:
        raise PipesdError(rc, "pipesd_debug_gemm_dense")


def debug_attn_split(total_keys: int, page_size: int, resident_ctas, units: int):
    """(key splits, keys per split, cut-down ring?) of one request: host arithmetic only."""
    res = (ctypes.c_int32 * 2)(*[int(x) for x in resident_ctas])
    out = (ctypes.c_int32 * 3)()
    rc = lib().pipesd_debug_attn_split(total_keys, page_size, res, units, out)
    if rc != 0:
        raise PipesdError(rc, "pipesd_debug_attn_split")
    return tuple(out)


# ---- shaped sampling and acceptance, on device tensors (no context)
class _on:
    """The device as the current one, and `stream` (None: its current stream) as the one that allocations belong to.  With a stream of
    its own, a call keeps the memory of its tensors from being given out again while that stream may still use it: those that it is
    given, and, for the current stream, those that it makes."""

    __slots__ = ("index", "stream", "tensors", "scopes", "home")

    def __init__(self, device, stream, *tensors):
        self.index, self.stream, self.tensors, self.scopes, self.home = device.index, stream, tensors, None, None
        assert stream is None or stream.device == device, f"stream: one of {device} expected"

    def __enter__(self):
        import torch
        if self.stream is None and torch.cuda.current_device() == self.index:        # (the usual call: nothing to switch)
            return torch._C._cuda_getCurrentRawStream(self.index)
        import contextlib
        self.scopes = contextlib.ExitStack()
        self.scopes.enter_context(torch.cuda.device(self.index))
        if self.stream is not None:
            self.home = torch.cuda.current_stream(self.index)
            for t in self.tensors:
                if t is not None and t.is_cuda:
                    t.record_stream(self.stream)
            self.scopes.enter_context(torch.cuda.stream(self.stream))
        return torch.cuda.current_stream(self.index).cuda_stream

    def __exit__(self, *exc):
        if self.scopes is not None:
            self.scopes.close()

    def made(self, *tensors):
        if self.home is not None:
            for t in tensors:
                t.record_stream(self.home)


def _rows_of(t, name):
    """Elements between the rows of a CUDA tensor whose rows (all dimensions but the first) are contiguous."""
    assert t.is_cuda and t.dim() >= 2, f"{name}: a CUDA tensor of rows"
    if t.is_contiguous():
        return t.numel() // max(t.shape[0], 1)
    inner = 1
    for d in range(t.dim() - 1, 0, -1):
        assert t.shape[d] == 1 or t.stride(d) == inner, f"{name}: rows must be contiguous"
        inner *= t.shape[d]
    assert t.shape[0] <= 1 or t.stride(0) >= inner, f"{name}: rows overlap"
    return t.stride(0) if t.shape[0] > 1 else inner


def _dtype_of(t, name):
    import torch
    if t.dtype is torch.float32:
        return F32
    assert t.dtype is torch.bfloat16, f"{name}: fp32 or bf16"
    return BF16


def _vector(t, n, dtype, device, name):
    assert t.get_device() == device.index and t.dtype is dtype and t.numel() == n and t.is_contiguous(), f"{name}: {n} contiguous {dtype} on {device} expected"
    return t.data_ptr()


def shaping(n: int, *, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, device="cuda"):
    """Settings of n rows (sample) or requests (accept), each given as one number or n of them: an int32 tensor [n, 4] that
    holds pipesd_shaping entries."""
    import torch
    a = np.empty((n, 4), np.int32)
    t, p, m = (np.broadcast_to(np.asarray(x, np.float32), (n,)) for x in (temperature, top_p, min_p))
    if not ((t >= 0) & (t <= 1e30)).all():
        raise ValueError("temperature: numbers of [0, 1e30]")
    if not (p > 0).all():
        raise ValueError("top_p: numbers > 0")
    if not ((m >= 0) & (m <= 1)).all():
        raise ValueError("min_p: numbers of [0, 1]")
    a[:, 0], a[:, 1], a[:, 2], a[:, 3] = t.view(np.int32), np.broadcast_to(np.asarray(top_k, np.int32), (n,)), p.view(np.int32), m.view(np.int32)
    return torch.from_numpy(a).to(device)


def sample(logits, shaping, u, *, probs=None, tokens=None, stream=None):
    """pipesd_sample: one token per row of logits [rows, vocab] (fp32 or bf16, any row stride), settings from shaping(),
    uniforms u [rows] (fp32).  probs: an fp32 tensor [rows, vocab] that receives the distributions.  Returns the tokens (int32)."""
    import torch
    rows, vocab = logits.shape
    dev = logits.device
    ld = _rows_of(logits, "logits")
    pl = 0
    if probs is not None:
        assert probs.dtype is torch.float32 and probs.shape == (rows, vocab) and probs.device == dev
        pl = _rows_of(probs, "probs")
    on = _on(dev, stream, logits, shaping, u, probs, tokens)
    with on as st:
        if tokens is None:
            tokens = torch.empty(rows, dtype=torch.int32, device=dev)
            on.made(tokens)
        rc = lib().pipesd_sample(logits.data_ptr(), _dtype_of(logits, "logits"), ld, rows, vocab, _vector(shaping, 4 * rows, torch.int32, dev, "shaping"),
                                 _vector(u, rows, torch.float32, dev, "u"), _vector(tokens, rows, torch.int32, dev, "tokens"),
                                 probs.data_ptr() if probs is not None else None, pl, st)
    if rc != OK:
        raise PipesdError(rc, "pipesd_sample")
    return tokens


def accept(logits, row0, shaping, q, drafts, u, *, stream=None):
    """pipesd_accept: the acceptance rule for shaped targets.  row0: int32 [n_req + 1]; shaping: of the requests; q: fp32
    [rows - n_req, vocab]; drafts: int32 [rows - n_req]; u: fp32 [rows].  Returns (n_accepted, next_token), int32 [n_req] each."""
    import torch
    rows, vocab = logits.shape
    dev = logits.device
    n_req = row0.numel() - 1
    assert n_req >= 1, "row0: a request at least"
    ld = _rows_of(logits, "logits")
    ql, qp, dp = 0, None, None
    if rows > n_req:
        assert q is not None and drafts is not None, "q, drafts: of the rows beyond one per request"
        assert q.dtype is torch.float32 and q.shape == (rows - n_req, vocab) and q.device == dev
        ql, qp, dp = _rows_of(q, "q"), q.data_ptr(), _vector(drafts, rows - n_req, torch.int32, dev, "drafts")
    on = _on(dev, stream, logits, row0, shaping, q, drafts, u)
    with on as st:
        n_accepted = torch.empty(n_req, dtype=torch.int32, device=dev)
        next_token = torch.empty_like(n_accepted)
        on.made(n_accepted, next_token)
        scratch = torch.empty(int(lib().pipesd_accept_scratch_bytes(rows)), dtype=torch.uint8, device=dev)
        rc = lib().pipesd_accept(logits.data_ptr(), _dtype_of(logits, "logits"), ld, n_req, rows, vocab, _vector(row0, n_req + 1, torch.int32, dev, "row0"),
                                 _vector(shaping, 4 * n_req, torch.int32, dev, "shaping"), qp, ql, dp, _vector(u, rows, torch.float32, dev, "u"),
                                 n_accepted.data_ptr(), next_token.data_ptr(), scratch.data_ptr(), st)
    if rc != OK:
        raise PipesdError(rc, "pipesd_accept")
    return n_accepted, next_token


class Kv4Cache:
    """One layer's paged K/V cache in 4 bits (pipesd_kv4_*).  The pool is a uint8 tensor [pages, KV heads, units, bytes], the
    caller's or one of n_pages pages made here; requests, positions and page tables are the caller's, as device tensors:

      row0   int32 [n_req + 1]            request r has rows row0[r] .. row0[r+1]-1 of the call
      base   int32 [n_req]                position of its first row
      table  int32 [n_req, max_pages]     its pages; -1 where there is none
    """

    def __init__(self, n_kv_heads: int, head_dim: int, *, n_pages: int | None = None, pool=None, page_size: int = 16, device="cuda"):
        import torch
        if pool is None:
            cfg = Kv4Cfg(n_kv_heads, head_dim, page_size, n_pages or 0, 1, 0)
            size = int(lib().pipesd_kv4_pool_bytes(ctypes.byref(cfg)))
            if size == 0:
                raise PipesdError(E_INVALID, "pipesd_kv4_pool_bytes")
            pool = torch.zeros(size, dtype=torch.uint8, device=device)
        elif n_pages is None:
            n_pages = pool.shape[0]
        cfg = Kv4Cfg(n_kv_heads, head_dim, page_size, n_pages, 1, 0)
        size = int(lib().pipesd_kv4_pool_bytes(ctypes.byref(cfg)))
        if size == 0:
            raise PipesdError(E_INVALID, "pipesd_kv4_pool_bytes")
        assert pool.is_cuda and pool.dtype == torch.uint8 and pool.is_contiguous() and pool.numel() == size, f"pool: {size} contiguous bytes expected"
        self.pool, self.n_kv_heads, self.head_dim, self.page_size, self.n_pages = pool, n_kv_heads, head_dim, page_size, n_pages
        self._scratch_bytes = int(lib().pipesd_kv4_attend_scratch_bytes(ctypes.byref(cfg)))
        self._cfgs = {}        # by the width of the page table

    def _where(self, rows, row0, base, table):
        import torch
        n_req, dev = base.numel(), self.pool.device
        assert table.dim() == 2 and table.shape[0] == n_req, "table: [n_req, max_pages]"
        cfg = self._cfgs.get(table.shape[1])
        if cfg is None:
            cfg = self._cfgs[table.shape[1]] = Kv4Cfg(self.n_kv_heads, self.head_dim, self.page_size, self.n_pages, table.shape[1], 0)
        return cfg, (n_req, rows, _vector(row0, n_req + 1, torch.int32, dev, "row0"), _vector(base, n_req, torch.int32, dev, "base"),
                     _vector(table, table.numel(), torch.int32, dev, "table"))

    def append(self, k, v, row0, base, table, *, stream=None):
        """Quantises the rows k, v [rows, KV heads, head_dim] (fp32 or bf16) into their positions."""
        dev = self.pool.device
        shape = (k.shape[0], self.n_kv_heads, self.head_dim)
        assert k.shape == shape == v.shape and k.dtype is v.dtype and k.get_device() == dev.index == v.get_device(), f"k, v: two alike of {shape} on {dev}"
        cfg, where = self._where(k.shape[0], row0, base, table)
        with _on(dev, stream, self.pool, k, v, row0, base, table) as st:
            rc = lib().pipesd_kv4_append(ctypes.byref(cfg), self.pool.data_ptr(), k.data_ptr(), v.data_ptr(), _dtype_of(k, "k"), _rows_of(k, "k"), _rows_of(v, "v"),
                                         *where, st)
        if rc != OK:
            raise PipesdError(rc, "pipesd_kv4_append")

    def read(self, rows: int, row0, base, table, *, stream=None):
        """The values at the rows' positions, fp32 [rows, KV heads, head_dim] of K and of V."""
        import torch
        dev = self.pool.device
        cfg, where = self._where(rows, row0, base, table)
        on = _on(dev, stream, self.pool, row0, base, table)
        with on as st:
            k = torch.empty((rows, self.n_kv_heads, self.head_dim), dtype=torch.float32, device=dev)
            v = torch.empty_like(k)
            on.made(k, v)
            rc = lib().pipesd_kv4_read(ctypes.byref(cfg), self.pool.data_ptr(), k.data_ptr(), v.data_ptr(), *where, st)
        if rc != OK:
            raise PipesdError(rc, "pipesd_kv4_read")
        return k, v

    def attend(self, q, row0, base, table, *, scale=None, out=None, stream=None):
        """Attention of the rows q [rows, query heads, head_dim] (fp32 or bf16; appended before) over their requests' positions.
        scale: head_dim ** -0.5 unless given."""
        import torch
        dev = self.pool.device
        assert q.dim() == 3 and q.shape[2] == self.head_dim and q.get_device() == dev.index, f"q: [rows, query heads, {self.head_dim}] on {dev}"
        cfg, where = self._where(q.shape[0], row0, base, table)
        on = _on(dev, stream, self.pool, q, row0, base, table, out)
        with on as st:
            if out is None:
                out = torch.empty_like(q, memory_format=torch.contiguous_format)
                on.made(out)
            else:
                assert out.shape == q.shape and out.dtype is q.dtype and out.get_device() == dev.index, "out: like q"
            scratch = torch.empty(self._scratch_bytes, dtype=torch.uint8, device=dev)
            rc = lib().pipesd_kv4_attend(ctypes.byref(cfg), self.pool.data_ptr(), q.data_ptr(), out.data_ptr(), _dtype_of(q, "q"), _rows_of(q, "q"), _rows_of(out, "out"),
                                         q.shape[1], self.head_dim ** -0.5 if scale is None else scale, *where, scratch.data_ptr(), st)
        if rc != OK:
            raise PipesdError(rc, "pipesd_kv4_attend")
        return out


# ---- trees of drafts: prompts, a bf16 cache and its pages, on device tensors (no context)
def attend_packed(q, k, v, row0, *, scale=None, out=None, stream=None):
    """pipesd_attend_packed: causal attention of prompts packed one behind the other.  q [rows, query heads, head_dim], k, v [rows, KV
    heads, head_dim] in bf16, row strides of their own (views of a fused projection will do); row0: int32 [prompts + 1].  scale: head_dim ** -0.5
    unless given.  Returns out, like q (made here: rows of no prompt are not written)."""
    import torch
    dev = q.device
    assert q.dim() == 3 and k.dim() == 3 and k.shape == v.shape and k.shape[0] == q.shape[0] and k.shape[2] == q.shape[2], "q, k, v: [rows, heads, head_dim]"
    assert q.dtype is k.dtype is v.dtype is torch.bfloat16 and k.device == dev == v.device, "q, k, v: bf16 on one device"
    rows, heads, hd = q.shape
    n_req = row0.numel() - 1
    on = _on(dev, stream, q, k, v, row0, out)
    with on as st:
        if out is None:
            out = torch.empty_like(q, memory_format=torch.contiguous_format)
            on.made(out)
        else:
            assert out.shape == q.shape and out.dtype is q.dtype and out.device == dev, "out: like q"
        rc = lib().pipesd_attend_packed(q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(), _rows_of(q, "q"), _rows_of(k, "k"), _rows_of(v, "v"),
                                        _rows_of(out, "out"), heads, k.shape[1], hd, hd ** -0.5 if scale is None else scale, n_req, rows,
                                        _vector(row0, n_req + 1, torch.int32, dev, "row0"), st)
    if rc != OK:
        raise PipesdError(rc, "pipesd_attend_packed")
    return out


def tree_mask(parent, row0, words: int, *, stream=None):
    """pipesd_tree_mask: (mask int32 [rows, words], depth int32 [rows]) of drafted trees.  parent: int32 [rows], indices within the request, -1
    below the prefix; row0: int32 [n_req + 1].  Rows of no request: no bits, depth 0."""
    import torch
    dev, rows, n_req = parent.device, parent.numel(), row0.numel() - 1
    on = _on(dev, stream, parent, row0)
    with on as st:
        mask, depth = torch.empty((rows, words), dtype=torch.int32, device=dev), torch.empty(rows, dtype=torch.int32, device=dev)
        on.made(mask, depth)
        rc = lib().pipesd_tree_mask(n_req, rows, _vector(row0, n_req + 1, torch.int32, dev, "row0"), _vector(parent, rows, torch.int32, dev, "parent"), words,
                                    mask.data_ptr(), depth.data_ptr(), st)
    if rc != OK:
        raise PipesdError(rc, "pipesd_tree_mask")
    return mask, depth


class Kv16Cache:
    """A paged K/V cache in bf16 (pipesd_kv16_*), all layers of it.  The pool is a bf16 tensor [layers, pages, 2, KV heads, page_size / 8,
    head_dim / 8, 8, 8], the caller's or one of n_pages pages made here; requests, positions, tables and references are the caller's, as int32
    device tensors: row0, base and table as for Kv4Cache, and

      refs   [n_pages]      entries of tables that hold a page; zeros at first
      keep   [n_req, words] rows of tree_mask
    """

    def __init__(self, n_kv_heads: int, head_dim: int, *, n_layers: int | None = None, n_pages: int | None = None, pool=None, page_size: int = 16, device="cuda"):
        import torch
        if pool is not None:
            assert pool.is_cuda and pool.dtype is torch.bfloat16 and pool.is_contiguous(), "pool: contiguous bf16 on a CUDA device"
            if pool.dim() == 8:
                shape = (2, n_kv_heads, page_size // 8, head_dim // 8, 8, 8)
                assert tuple(pool.shape[2:]) == shape, f"pool: [layers, pages, {', '.join(map(str, shape))}] expected"
                n_layers, n_pages = n_layers or pool.shape[0], n_pages or pool.shape[1]
        self.n_kv_heads, self.head_dim, self.page_size = n_kv_heads, head_dim, page_size
        self.n_layers, self.n_pages = 1 if n_layers is None else n_layers, n_pages or 0
        self._cfgs = {}        # by the width of the page table
        size = int(lib().pipesd_kv16_pool_bytes(ctypes.byref(self._cfg(1))))
        if size == 0:
            raise PipesdError(E_INVALID, "pipesd_kv16_pool_bytes")
        if pool is None:
            pool = torch.zeros((self.n_layers, self.n_pages, 2, n_kv_heads, page_size // 8, head_dim // 8, 8, 8), dtype=torch.bfloat16, device=device)
        assert pool.numel() * 2 == size, f"pool: {size} bytes expected"
        self.pool = pool

    def _cfg(self, max_pages):
        cfg = self._cfgs.get(max_pages)
        if cfg is None:
            cfg = self._cfgs[max_pages] = Kv16Cfg(self.n_layers, self.n_kv_heads, self.head_dim, self.page_size, self.n_pages, max_pages, 0)
        return cfg

    def _ints(self, t, n, name):
        import torch
        return _vector(t, n, torch.int32, self.pool.device, name)

    def _where(self, rows, row0, base, table):
        n_req = base.numel()
        assert table.dim() == 2 and table.shape[0] == n_req, "table: [n_req, max_pages]"
        return self._cfg(table.shape[1]), (n_req, rows, self._ints(row0, n_req + 1, "row0"), self._ints(base, n_req, "base"),
                                           self._ints(table, table.numel(), "table"))

    def append(self, k, v, row0, base, table, *, layer: int = 0, stream=None):
        """Writes the rows k, v [rows, KV heads, head_dim] (fp32 or bf16) into their positions of a layer."""
        dev = self.pool.device
        shape = (k.shape[0], self.n_kv_heads, self.head_dim)
        assert k.shape == shape == v.shape and k.dtype is v.dtype and k.get_device() == dev.index == v.get_device(), f"k, v: two alike of {shape} on {dev}"
        cfg, where = self._where(k.shape[0], row0, base, table)
        with _on(dev, stream, self.pool, k, v, row0, base, table) as st:
            rc = lib().pipesd_kv16_append(ctypes.byref(cfg), self.pool.data_ptr(), layer, k.data_ptr(), v.data_ptr(), _dtype_of(k, "k"), _rows_of(k, "k"),
                                          _rows_of(v, "v"), *where, st)
        if rc != OK:
            raise PipesdError(rc, "pipesd_kv16_append")

    def read(self, rows: int, row0, base, table, *, layer: int = 0, stream=None):
        """The rows' positions of a layer, bf16 [rows, KV heads, head_dim] of K and of V."""
        import torch
        dev = self.pool.device
        cfg, where = self._where(rows, row0, base, table)
        on = _on(dev, stream, self.pool, row0, base, table)
        with on as st:
            k = torch.empty((rows, self.n_kv_heads, self.head_dim), dtype=torch.bfloat16, device=dev)
            v = torch.empty_like(k)
            on.made(k, v)
            rc = lib().pipesd_kv16_read(ctypes.byref(cfg), self.pool.data_ptr(), layer, k.data_ptr(), v.data_ptr(), *where, st)
        if rc != OK:
            raise PipesdError(rc, "pipesd_kv16_read")
        return k, v

    def attend(self, q, row0, base, table, *, mask=None, layer: int = 0, scale=None, out=None, stream=None):
        """Attention of the rows q [rows, query heads, head_dim] (fp32 or bf16; appended before): over their requests' positions below base,
        and the new rows that mask (int32 [rows, words], from tree_mask) names, or, without one, those up to themselves.  scale: head_dim ** -0.5
        unless given."""
        import torch
        dev = self.pool.device
        assert q.dim() == 3 and q.shape[2] == self.head_dim and q.get_device() == dev.index, f"q: [rows, query heads, {self.head_dim}] on {dev}"
        rows, heads = q.shape[:2]
        cfg, where = self._where(rows, row0, base, table)
        words, bits = 0, None
        if mask is not None:
            assert mask.dim() == 2 and mask.shape[0] == rows, "mask: [rows, words]"
            words, bits = mask.shape[1], self._ints(mask, mask.numel(), "mask")
        on = _on(dev, stream, self.pool, q, row0, base, table, mask, out)
        with on as st:
            if out is None:
                out = torch.empty_like(q, memory_format=torch.contiguous_format)
                on.made(out)
            else:
                assert out.shape == q.shape and out.dtype is q.dtype and out.get_device() == dev.index, "out: like q"
            scratch = torch.empty(int(lib().pipesd_kv16_attend_scratch_bytes(ctypes.byref(cfg), rows, heads)) or 16, dtype=torch.uint8, device=dev)
            rc = lib().pipesd_kv16_attend(ctypes.byref(cfg), self.pool.data_ptr(), layer, q.data_ptr(), out.data_ptr(), _dtype_of(q, "q"), _rows_of(q, "q"),
                                          _rows_of(out, "out"), heads, self.head_dim ** -0.5 if scale is None else scale, *where, bits, words, scratch.data_ptr(), st)
        if rc != OK:
            raise PipesdError(rc, "pipesd_kv16_attend")
        return out

    def _plan(self, n, table, refs, stream, *given):
        """(configuration, addresses of table and refs, a stream scope and what makes pages and scratch within it)."""
        import torch
        dev = self.pool.device
        assert table.dim() == 2, "table: [requests, max_pages]"
        cfg, on = self._cfg(table.shape[1]), _on(dev, stream, self.pool, table, refs, *given)

        def room():
            pages = torch.empty(n, dtype=torch.int32, device=dev)
            on.made(pages)
            return pages, torch.empty(int(lib().pipesd_kv16_plan_scratch_bytes(ctypes.byref(cfg), n)) or 16, dtype=torch.uint8, device=dev)

        return cfg, self._ints(table, table.numel(), "table"), self._ints(refs, self.n_pages, "refs"), on, room

    def reserve(self, length, table, refs, *, stream=None):
        """Pages for the positions below length [n_req] where the requests' rows of table have none.  Returns how many pages each then has there,
        -1 where there were not enough (int32 [n_req])."""
        n = length.numel()
        assert table.shape[0] == n, "table: [n_req, max_pages]"
        cfg, tab, ref, on, room = self._plan(n, table, refs, stream, length)
        with on as st:
            pages, scratch = room()
            rc = lib().pipesd_kv16_reserve(ctypes.byref(cfg), n, self._ints(length, n, "length"), tab, ref, pages.data_ptr(), scratch.data_ptr(), st)
        if rc != OK:
            raise PipesdError(rc, "pipesd_kv16_reserve")
        return pages

    def fork(self, src, dst, length, own, table, refs, *, stream=None):
        """Rows dst of table become continuations of rows src, which hold length positions: pages of positions below own are shared, the others
        copied.  All int32 [n].  Returns the pages that each has, -1 where there were not enough (int32 [n])."""
        n = src.numel()
        cfg, tab, ref, on, room = self._plan(n, table, refs, stream, src, dst, length, own)
        with on as st:
            pages, scratch = room()
            rc = lib().pipesd_kv16_fork(ctypes.byref(cfg), self.pool.data_ptr(), n, *(self._ints(t, n, name) for t, name in
                                        ((src, "src"), (dst, "dst"), (length, "length"), (own, "own"))), table.shape[0], tab, ref, pages.data_ptr(),
                                        scratch.data_ptr(), st)
        if rc != OK:
            raise PipesdError(rc, "pipesd_kv16_fork")
        return pages

    def compact(self, keep, base, table, *, stream=None):
        """Of the rows behind base [n_req], those whose bits are set in keep [n_req, words] move together to base, base + 1, ..., in all layers.
        Returns how many there are (int32 [n_req])."""
        import torch
        dev, n = self.pool.device, base.numel()
        assert table.dim() == 2 and table.shape[0] == n and keep.dim() == 2 and keep.shape[0] == n, "keep: [n_req, words], table: [n_req, max_pages]"
        on = _on(dev, stream, self.pool, keep, base, table)
        with on as st:
            kept = torch.empty(n, dtype=torch.int32, device=dev)
            on.made(kept)
            rc = lib().pipesd_kv16_compact(ctypes.byref(self._cfg(table.shape[1])), self.pool.data_ptr(), n, self._ints(keep, keep.numel(), "keep"), keep.shape[1],
                                           self._ints(base, n, "base"), self._ints(table, table.numel(), "table"), kept.data_ptr(), st)
        if rc != OK:
            raise PipesdError(rc, "pipesd_kv16_compact")
        return kept

    def release(self, length, table, refs, *, stream=None):
        """Pages that hold only positions from length [n_req] on leave their rows of table."""
        n = length.numel()
        assert table.dim() == 2 and table.shape[0] == n, "table: [n_req, max_pages]"
        with _on(self.pool.device, stream, self.pool, length, table, refs) as st:
            rc = lib().pipesd_kv16_release(ctypes.byref(self._cfg(table.shape[1])), n, self._ints(length, n, "length"), self._ints(table, table.numel(), "table"),
                                           self._ints(refs, self.n_pages, "refs"), st)
        if rc != OK:
            raise PipesdError(rc, "pipesd_kv16_release")


# ---- the edge-side scheduling model (host code of the library)
def sched_round_time(N: int, alpha: float, beta: float, gamma: float, boundaries) -> float:
    b = np.ascontiguousarray(boundaries, np.int32)
    T = ctypes.c_double()
    rc = lib().pipesd_sched_round_time(N, alpha, beta, gamma, _np_ptr(b), b.size, ctypes.byref(T))
    if rc != OK:
        raise PipesdError(rc, "pipesd_sched_round_time")
    return T.value


def sched_optimal_batching(N: int, alpha: float, beta: float, gamma: float):
    """(boundaries b_1..b_K as a tuple, minimal T)."""
    b = np.zeros(max(N, 1), np.int32)
    K = i32()
    T = ctypes.c_double()
    rc = lib().pipesd_sched_optimal_batching(N, alpha, beta, gamma, _np_ptr(b), ctypes.byref(K), ctypes.byref(T))
    if rc != OK:
        raise PipesdError(rc, "pipesd_sched_optimal_batching")
    return tuple(int(x) for x in b[:K.value]), T.value


def sched_trigger_step(c1: float, R1: float, R2: float, p: float):
    """(triggered?, C1 after the step)."""
    c = ctypes.c_double(c1)
    fire = i32()
    rc = lib().pipesd_sched_trigger_step(ctypes.byref(c), R1, R2, p, ctypes.byref(fire))
    if rc != OK:
        raise PipesdError(rc, "pipesd_sched_trigger_step")
    return bool(fire.value), c.value
