"""ctypes binding of libcllm.so (C ABI in include/cllm.h). Argument marshalling only: every
step of the decode runs in the library's HIP kernels. Importing this module fails loudly when
the library has not been built; there is no fallback path.
"""
import ctypes
import os

import numpy as np

from .configs import ModelConfig

_HERE = os.path.dirname(os.path.abspath(__file__))
# CLLM_HOST_SANITIZE=1 selects the build with address and undefined-behaviour checks on the host
# code (build.py --host-sanitize), for runs of the CPU tests under the sanitizer runtime.
HOST_SANITIZE = os.environ.get("CLLM_HOST_SANITIZE") == "1"
LIB_PATH = os.path.join(_HERE, "libcllm.hostsan.so" if HOST_SANITIZE else "libcllm.so")

CLLM_OK = 0
STATUS_NAMES = {0: "OK", 1: "ERR_ARG", 2: "ERR_STATE", 3: "ERR_CAPACITY", 4: "ERR_OOM", 5: "ERR_IO",
                6: "ERR_FORMAT", 7: "ERR_DEVICE", 8: "ERR_NUMERIC"}
KT = {"qkv": 0, "attn": 1, "o": 2, "gate_up": 3, "down": 4, "lm_head": 5, "scan": 6, "attn_combine": 7,
      "embed": 8, "loss_logits": 9, "loss_rows": 10, "loss_dh": 11, "loss_dw": 12}

_i32, _i64, _u64, _f32, _dbl, _vp = (ctypes.c_int32, ctypes.c_int64, ctypes.c_uint64, ctypes.c_float,
                                     ctypes.c_double, ctypes.c_void_p)


class cllm_config(ctypes.Structure):
    _fields_ = [("n_layers", _i32), ("d_model", _i32), ("n_heads", _i32), ("head_dim", _i32),
                ("ffn_dim", _i32), ("vocab", _i32), ("rms_eps", _f32), ("rope_base", _f32), ("dtype", _i32)]


class cllm_runtime_opts(ctypes.Structure):
    _fields_ = [("max_ctx", _i32), ("max_block", _i32), ("max_new", _i32), ("device", _i32), ("stream", _vp),
                ("max_batch", _i32), ("prefill_chunk", _i32), ("workspace", _vp), ("workspace_bytes", ctypes.c_size_t)]


class cllm_guess_spec(ctypes.Structure):
    _fields_ = [("policy", _i32), ("block_policy", _i32), ("stream", _vp), ("stream_len", _i32),
                ("thr53", _u64), ("seed", _u64)]


class cllm_decode_stats(ctypes.Structure):
    _fields_ = [("steps", _i64), ("blocks", _i64), ("tokens", _i64), ("accept_hist", _i64 * 65),
                ("prefill_ms", _dbl), ("decode_ms", _dbl), ("rows", _i64), ("iter_ms_p10", _dbl),
                ("iter_ms_p50", _dbl), ("iter_ms_p90", _dbl), ("iter_ms_full_p50", _dbl), ("iter_ms_full_p10", _dbl),
                ("iter_ms_full_p90", _dbl)]


class cllm_trace_stats(ctypes.Structure):
    _fields_ = [("iterations", _i64), ("fast_forward_mean", _dbl), ("stationary", _i64), ("windows", _i64),
                ("stationary_per_window", _dbl)]


class cllm_paged_config(ctypes.Structure):
    _fields_ = [("n_heads", _i32), ("n_kv_heads", _i32), ("head_dim", _i32), ("dtype", _i32), ("page_size", _i32),
                ("n_pages", _i32), ("max_seqs", _i32), ("max_ctx", _i32), ("max_rows", _i32), ("rope_base", _f32),
                ("device", _i32), ("stream", _vp), ("workspace", _vp), ("workspace_bytes", ctypes.c_size_t)]


class cllm_paged_views(ctypes.Structure):
    _fields_ = [("block_table", _vp), ("seq_pages", _vp), ("free_list", _vp), ("row_start", _vp), ("row_slot", _vp),
                ("row_pos", _vp), ("max_pages", _i32)]


TRACE_STRIDE = 5 + 2 * 64  # CLLM_TRACE_STRIDE

EXPORTS = ["cllm_model_create", "cllm_model_set_weights", "cllm_model_init_random", "cllm_model_load", "cllm_model_free", "cllm_prefill",
           "cllm_jacobi_step", "cllm_jacobi_decode", "cllm_ar_decode", "cllm_jacobi_step_batch",
           "cllm_jacobi_decode_batch", "cllm_reset", "cllm_debug_logits", "cllm_trace_enable", "cllm_trace_read",
           "cllm_trace_count", "cllm_collect_states", "cllm_loss_head", "cllm_loss_head_device", "cllm_hidden_rows", "cllm_hidden_rows_noalloc", "cllm_seq_state", "cllm_timing_enable", "cllm_timing_read",
           "cllm_paged_workspace_bytes", "cllm_paged_create", "cllm_paged_free", "cllm_paged_views_get", "cllm_paged_plan",
           "cllm_paged_append", "cllm_paged_attn", "cllm_paged_status", "cllm_paged_last_error",
           "cllm_streamed_weight_bytes", "cllm_workspace_bytes", "cllm_status_string", "cllm_last_error"]

_lib = None


def lib():
    """Load libcllm.so (raises if it is not built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is not built; run `python -m paper_2403_00835_amd.build`")
        # PyTorch wheels carry their own HIP runtime. Loaded first, it is the one libcllm.so binds
        # to, so torch's device memory and streams are valid in the library's calls; loaded after
        # the system runtime has opened the GPU, it finds no GPU. Import it first when installed.
        try:
            import torch  # noqa: F401
        except ImportError:
            pass
        L = ctypes.CDLL(LIB_PATH)
        P = ctypes.POINTER
        L.cllm_model_create.argtypes = [P(cllm_config), P(cllm_runtime_opts), P(_vp)]
        L.cllm_model_set_weights.argtypes = [_vp, _vp, _i32]
        L.cllm_model_load.argtypes = [ctypes.c_char_p, P(cllm_runtime_opts), P(_vp)]
        L.cllm_model_init_random.argtypes = [P(cllm_config), _u64, P(cllm_runtime_opts), P(_vp)]
        L.cllm_model_free.argtypes = [_vp]
        L.cllm_model_free.restype = None
        L.cllm_prefill.argtypes = [_vp, _i32, _vp, _i32, P(_i32)]
        L.cllm_jacobi_step.argtypes = [_vp, _i32, _vp, _i32, _vp, P(_i32)]
        L.cllm_jacobi_decode.argtypes = [_vp, _i32, _vp, _i32, _i32, _i32, P(cllm_guess_spec), _vp,
                                         P(cllm_decode_stats)]
        L.cllm_ar_decode.argtypes = [_vp, _i32, _vp, _i32, _i32, _vp, P(cllm_decode_stats)]
        L.cllm_jacobi_step_batch.argtypes = [_vp, _i32, _vp, _vp, _vp, _vp, _vp]
        L.cllm_jacobi_decode_batch.argtypes = [_vp, _i32, _vp, _vp, _vp, _i32, _i32, _vp, _vp, _vp]
        L.cllm_reset.argtypes = [_vp, _i32]
        L.cllm_debug_logits.argtypes = [_vp, _i32, _vp, ctypes.c_size_t]
        L.cllm_seq_state.argtypes = [_vp, _i32, P(_i32), P(_i32)]
        L.cllm_trace_enable.argtypes = [_vp, _i32]
        L.cllm_trace_read.argtypes = [_vp, _i32, _vp, _i64, P(_i64)]
        L.cllm_trace_count.argtypes = [_vp, _i64, _vp, _i64, _i32, _i32, P(cllm_trace_stats)]
        L.cllm_loss_head.argtypes = [_vp, _vp, _vp, _i32, _vp, _vp, _i32, _f32, _vp, _vp, _vp, _vp, _vp, P(_dbl)]
        L.cllm_loss_head_device.argtypes = [_vp, _vp, _vp, _i32, _vp, _vp, _i32, _f32, _vp, _vp, _vp, _vp, _vp, _vp]
        L.cllm_hidden_rows.argtypes = [_vp, _i32, _vp, _i32, _vp]
        L.cllm_hidden_rows_noalloc.argtypes = [_vp, _i32, _vp, _i32, _vp]
        L.cllm_collect_states.argtypes = [_vp, _i64, _vp, _i64, _i32, _dbl, ctypes.c_uint64, _vp, _vp, _vp, _i64,
                                          P(_i64)]
        L.cllm_timing_enable.argtypes = [_vp, _i32, _i32, _i32]
        L.cllm_timing_read.argtypes = [_vp, P(_i64), P(_dbl)]
        L.cllm_workspace_bytes.argtypes = [P(cllm_config), P(cllm_runtime_opts), P(ctypes.c_size_t)]
        L.cllm_streamed_weight_bytes.argtypes = [_vp]
        L.cllm_streamed_weight_bytes.restype = _i64
        L.cllm_status_string.argtypes = [_i32]
        L.cllm_status_string.restype = ctypes.c_char_p
        L.cllm_last_error.argtypes = [_vp]
        L.cllm_last_error.restype = ctypes.c_char_p
        L.cllm_paged_workspace_bytes.argtypes = [P(cllm_paged_config), P(ctypes.c_size_t)]
        L.cllm_paged_create.argtypes = [P(cllm_paged_config), P(_vp)]
        L.cllm_paged_free.argtypes = [_vp]
        L.cllm_paged_free.restype = None
        L.cllm_paged_views_get.argtypes = [_vp, P(cllm_paged_views)]
        L.cllm_paged_plan.argtypes = [_vp, _i32, _vp, _vp, _vp, _i32, _i32, _i32]
        L.cllm_paged_append.argtypes = [_vp, _vp, _i64, _vp, _i64, _vp, _i64, _vp, _i64, _vp, _vp]
        L.cllm_paged_attn.argtypes = [_vp, _vp, _i64, _vp, _vp, _f32, _vp, _i64, _vp]
        L.cllm_paged_status.argtypes = [_vp, P(_i32), P(_i32)]
        L.cllm_paged_last_error.argtypes = [_vp]
        L.cllm_paged_last_error.restype = ctypes.c_char_p
        for name in EXPORTS:
            if name not in ("cllm_paged_free", "cllm_paged_last_error", "cllm_model_free", "cllm_streamed_weight_bytes", "cllm_status_string",
                            "cllm_last_error"):
                getattr(L, name).restype = _i32
        _lib = L
    return _lib


class CllmError(RuntimeError):
    def __init__(self, status, msg):
        super().__init__(f"{STATUS_NAMES.get(status, status)}: {msg}")
        self.status = status


def _p(a):
    return a.ctypes.data


def make_config(cfg: ModelConfig):
    return cllm_config(cfg.n_layers, cfg.d_model, cfg.n_heads, cfg.head_dim, cfg.ffn_dim, cfg.vocab,
                       cfg.rms_eps, cfg.rope_base, cfg.dtype_code)


def thr53(p):
    return int(round(min(max(float(p), 0.0), 1.0) * float(1 << 53)))


def workspace_bytes(cfg: ModelConfig, max_ctx, max_block=16, max_new=256, max_batch=1, prefill_chunk=0):
    """Bytes of caller-owned workspace a context of these options takes (cllm_workspace_bytes)."""
    opts = cllm_runtime_opts(max_ctx, max_block, max_new, 0, None, max_batch, prefill_chunk, None, 0)
    n = ctypes.c_size_t(0)
    st = lib().cllm_workspace_bytes(ctypes.byref(make_config(cfg)), ctypes.byref(opts), ctypes.byref(n))
    if st != CLLM_OK:
        raise CllmError(st, "cllm_workspace_bytes failed")
    return int(n.value)


class Model:
    """One context of libcllm.so: model weights, KV cache and workspace on one GPU."""

    def __init__(self, cfg: ModelConfig, max_ctx, max_block=16, max_new=256, device=0, stream=None,
                 weights=None, path=None, max_batch=1, random_seed=None, prefill_chunk=0, workspace=None):
        """weights: host tensors (cllm_model_set_weights); path: a weight file (cllm_model_load);
        random_seed: seeded synthetic weights drawn on the GPU (cllm_model_init_random);
        workspace: (device pointer, bytes) of caller-owned device memory for the iteration
        workspace (see workspace_bytes), kept alive by the caller until close()."""
        self.cfg = cfg
        self.L = lib()
        self.max_block = max_block
        self.max_batch = max_batch
        ws_ptr, ws_bytes = workspace if workspace is not None else (None, 0)
        opts = cllm_runtime_opts(max_ctx, max_block, max_new, device, stream, max_batch, prefill_chunk, ws_ptr,
                                 ws_bytes)
        h = _vp()
        if path is not None:
            st = self.L.cllm_model_load(os.fsencode(path), ctypes.byref(opts), ctypes.byref(h))
        elif random_seed is not None:
            st = self.L.cllm_model_init_random(ctypes.byref(make_config(cfg)), int(random_seed), ctypes.byref(opts),
                                               ctypes.byref(h))
        else:
            st = self.L.cllm_model_create(ctypes.byref(make_config(cfg)), ctypes.byref(opts), ctypes.byref(h))
        if st != CLLM_OK:
            raise CllmError(st, "model creation failed")
        self.h = h
        self._dbg = None
        if weights is not None:
            self.set_weights(weights)

    def close(self):
        if getattr(self, "h", None):
            self.L.cllm_model_free(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _check(self, st):
        if st != CLLM_OK:
            msg = self.L.cllm_last_error(self.h)
            raise CllmError(st, msg.decode() if msg else "")

    def set_weights(self, tensors):
        ts = [np.ascontiguousarray(t) for t in tensors]
        arr = (_vp * len(ts))(*[_p(t) for t in ts])
        self._check(self.L.cllm_model_set_weights(self.h, ctypes.cast(arr, _vp), len(ts)))

    def streamed_weight_bytes(self):
        return int(self.L.cllm_streamed_weight_bytes(self.h))

    def prefill(self, prompt, seq=0):
        p = np.ascontiguousarray(prompt, dtype=np.int32)
        y0 = _i32(0)
        self._check(self.L.cllm_prefill(self.h, seq, _p(p), p.size, ctypes.byref(y0)))
        return int(y0.value)

    def jacobi_step(self, block_in, seq=0):
        b = np.ascontiguousarray(block_in, dtype=np.int32)
        out = np.empty(b.size, dtype=np.int32)
        a = _i32(0)
        self._check(self.L.cllm_jacobi_step(self.h, seq, _p(b), b.size, _p(out), ctypes.byref(a)))
        return out, int(a.value)

    def jacobi_decode(self, prompt, n, max_new, policy=0, block_policy=0, stream=None, p=0.0, seed=0, seq=0):
        pr = np.ascontiguousarray(prompt, dtype=np.int32)
        out = np.empty(max_new, dtype=np.int32)
        st = cllm_decode_stats()
        s_arr = None if stream is None else np.ascontiguousarray(stream, dtype=np.int32)
        g = cllm_guess_spec(policy, block_policy, None if s_arr is None else _p(s_arr),
                            0 if s_arr is None else s_arr.size, thr53(p), seed)
        self._check(self.L.cllm_jacobi_decode(self.h, seq, _p(pr), pr.size, n, max_new, ctypes.byref(g), _p(out),
                                              ctypes.byref(st)))
        return out, _stats(st)

    def ar_decode(self, prompt, max_new, seq=0):
        pr = np.ascontiguousarray(prompt, dtype=np.int32)
        out = np.empty(max_new, dtype=np.int32)
        st = cllm_decode_stats()
        self._check(self.L.cllm_ar_decode(self.h, seq, _p(pr), pr.size, max_new, _p(out), ctypes.byref(st)))
        return out, _stats(st)

    def jacobi_step_batch(self, seq_ids, blocks):
        """One batched iteration: blocks[b] is the block of slot seq_ids[b]. Returns the list of
        (block_out, accepted) per entry."""
        B = len(seq_ids)
        ids = np.ascontiguousarray(seq_ids, dtype=np.int32)
        zin = np.zeros((B, self.max_block), dtype=np.int32)
        m = np.zeros(B, dtype=np.int32)
        for b, blk in enumerate(blocks):
            blk = np.asarray(blk, dtype=np.int32)
            zin[b, :blk.size] = blk
            m[b] = blk.size
        out = np.zeros((B, self.max_block), dtype=np.int32)
        acc = np.zeros(B, dtype=np.int32)
        self._check(self.L.cllm_jacobi_step_batch(self.h, B, _p(ids), _p(zin), _p(m), _p(out), _p(acc)))
        return [(out[b, :m[b]].copy(), int(acc[b])) for b in range(B)]

    def jacobi_decode_batch(self, seq_ids, prompts, n, max_new, specs=None):
        """Batched decode. specs: per entry dict(policy, block_policy, stream, p, seed) or None.
        Returns (out [B, max_new], list of stats dicts)."""
        B = len(seq_ids)
        ids = np.ascontiguousarray(seq_ids, dtype=np.int32)
        lens = np.array([len(p) for p in prompts], dtype=np.int32)
        cat = np.ascontiguousarray(np.concatenate([np.asarray(p, dtype=np.int32) for p in prompts]))
        out = np.zeros((B, max_new), dtype=np.int32)
        stats = (cllm_decode_stats * B)()
        gs_arr, keep = None, []
        if specs is not None:
            gs_arr = (cllm_guess_spec * B)()
            for b, sp in enumerate(specs):
                st = sp.get("stream")
                s_arr = None if st is None else np.ascontiguousarray(st, dtype=np.int32)
                keep.append(s_arr)
                gs_arr[b] = cllm_guess_spec(sp.get("policy", 0), sp.get("block_policy", 0),
                                            None if s_arr is None else _p(s_arr),
                                            0 if s_arr is None else s_arr.size, thr53(sp.get("p", 0.0)),
                                            sp.get("seed", 0))
        self._check(self.L.cllm_jacobi_decode_batch(self.h, B, _p(ids), _p(cat), _p(lens), n, max_new,
                                                    None if gs_arr is None else ctypes.cast(gs_arr, _vp), _p(out),
                                                    ctypes.cast(stats, _vp)))
        return out, [_stats(stats[b]) for b in range(B)]

    def reset(self, seq=0):
        self._check(self.L.cllm_reset(self.h, seq))

    def debug_logits(self, enable, rows=None):
        if enable:
            rows = rows or max(64, -(-self.max_batch * self.max_block // 64) * 64)
            self._dbg = np.zeros((rows, self.cfg.vocab), dtype=np.float32)
            self._check(self.L.cllm_debug_logits(self.h, 1, _p(self._dbg), self._dbg.size))
        else:
            self._check(self.L.cllm_debug_logits(self.h, 0, None, 0))
            self._dbg = None

    def last_logits(self, m):
        return self._dbg[:m].copy()

    def seq_state(self, seq=0):
        L, pend = _i32(0), _i32(0)
        self._check(self.L.cllm_seq_state(self.h, seq, ctypes.byref(L), ctypes.byref(pend)))
        return int(L.value), int(pend.value)

    def loss_head(self, teacher, student, ar_rows, ar_targets, omega, want_dw=False):
        """CLLM loss at the LM head and its gradients (cllm_loss_head): dict kl, nll, loss,
        d_student, d_ar and, with want_dw, d_W."""
        d, V = self.cfg.d_model, self.cfg.vocab
        T = np.ascontiguousarray(teacher, dtype=np.float32).reshape(-1, d)
        S = np.ascontiguousarray(student, dtype=np.float32).reshape(-1, d)
        Ar = np.ascontiguousarray(ar_rows, dtype=np.float32).reshape(-1, d)
        tg = np.ascontiguousarray(ar_targets, dtype=np.int32)
        P, A = T.shape[0], Ar.shape[0]
        kl, nll = np.zeros(max(P, 1), np.float32), np.zeros(max(A, 1), np.float32)
        ds, da = np.zeros((max(P, 1), d), np.float32), np.zeros((max(A, 1), d), np.float32)
        dw = np.zeros((V, d), np.float32) if want_dw else None
        loss = _dbl(0.0)
        self._check(self.L.cllm_loss_head(self.h, _p(T) if P else None, _p(S) if P else None, P,
                                          _p(Ar) if A else None, _p(tg) if A else None, A, float(omega),
                                          _p(kl), _p(nll), _p(ds), _p(da), None if dw is None else _p(dw),
                                          ctypes.byref(loss)))
        out = {"kl": kl[:P], "nll": nll[:A], "loss": float(loss.value), "d_student": ds[:P], "d_ar": da[:A]}
        if want_dw:
            out["d_W"] = dw
        return out

    def loss_head_device(self, n_pairs, n_ar, omega, teacher, student, ar_rows, ar_targets, row_kl, row_nll,
                         d_student, d_ar, d_weight=None, loss=None):
        """cllm_loss_head_device: enqueue the loss head on device arrays (torch tensors on the
        context's GPU, or raw addresses) and return without waiting. A tensor argument must be
        contiguous, of the entry point's type (float32; int32 targets; float64 loss) and hold at
        least its rows."""
        d, V = self.cfg.d_model, self.cfg.vocab
        P, A = int(n_pairs), int(n_ar)
        args = [(teacher, P * d, "float32"), (student, P * d, "float32"), (ar_rows, A * d, "float32"),
                (ar_targets, A, "int32"), (row_kl, P, "float32"), (row_nll, A, "float32"),
                (d_student, P * d, "float32"), (d_ar, A * d, "float32"), (d_weight, V * d, "float32"),
                (loss, 1, "float64")]
        ptrs = [_dev_ptr(x, n, t) if n else None for x, n, t in args]
        self._check(self.L.cllm_loss_head_device(self.h, ptrs[0], ptrs[1], P, ptrs[2], ptrs[3], A, float(omega),
                                                 *ptrs[4:]))

    def hidden_rows(self, block, seq=0):
        """cllm_hidden_rows: the LM-head input rows [m, d] of an iteration over block at the slot's
        committed length (nothing committed)."""
        b = np.ascontiguousarray(block, dtype=np.int32)
        out = np.empty((b.size, self.cfg.d_model), dtype=np.float32)
        self._check(self.L.cllm_hidden_rows(self.h, seq, _p(b), b.size, _p(out)))
        return out

    def hidden_rows_noalloc(self, block, seq=0):
        """cllm_hidden_rows_noalloc: hidden_rows with the staging rows in the library's fixed
        per-GPU scratch (no allocation)."""
        b = np.ascontiguousarray(block, dtype=np.int32)
        out = np.empty((b.size, self.cfg.d_model), dtype=np.float32)
        self._check(self.L.cllm_hidden_rows_noalloc(self.h, seq, _p(b), b.size, _p(out)))
        return out

    def trace_enable(self, enable=True):
        self._check(self.L.cllm_trace_enable(self.h, 1 if enable else 0))

    def trace_read(self, seq=0):
        """Records of the slot's last recorded decode, as dicts (L, e, b0, m, a, z, pred)."""
        n = _i64(0)
        self._check(self.L.cllm_trace_read(self.h, seq, None, 0, ctypes.byref(n)))
        raw = np.zeros((max(int(n.value), 1), TRACE_STRIDE), dtype=np.int32)
        self._check(self.L.cllm_trace_read(self.h, seq, _p(raw), int(n.value), ctypes.byref(n)))
        return records_to_dicts(raw[:int(n.value)])

    def timing_enable(self, kernel_class, max_rows=0, every=1):
        cls = KT[kernel_class] if isinstance(kernel_class, str) else int(kernel_class)
        self._check(self.L.cllm_timing_enable(self.h, cls, max_rows, every))

    def timing_read(self):
        n, ms = _i64(0), _dbl(0.0)
        self._check(self.L.cllm_timing_read(self.h, ctypes.byref(n), ctypes.byref(ms)))
        return int(n.value), float(ms.value)


def _dev_ptr(x, count, dtype):
    """Device address of x (None, an int address, or a tensor with data_ptr(): checked to be
    contiguous, of dtype and holding at least count elements)."""
    if x is None:
        return None
    if isinstance(x, int):
        return x
    if not x.is_contiguous() or str(x.dtype).split(".")[-1] != dtype or x.numel() < count:
        raise ValueError(f"device array: need a contiguous {dtype} tensor of >= {count} elements, got "
                         f"{x.dtype} {tuple(x.shape)}")
    return x.data_ptr()


_increment_version = None


def _changed(*tensors):
    """Tells autograd that a call has written the tensors (through their addresses, which it does not see)."""
    global _increment_version
    if _increment_version is None:
        from torch.autograd.graph import increment_version
        _increment_version = increment_version
    _increment_version(tensors)


class PagedCache:
    """A paged KV cache (cllm_paged_*): the books of a page pool that the requests of a server share,
    and the operators of a step on it, on PyTorch tensors of the cache's GPU:

        cache.plan(seq_ids, ctx_lens, new_lens, rows)      # pages and rows of the step
        per layer: cache.append(q, k, v, q, k_pages, v_pages); cache.attn(q, k_pages, v_pages, out)

    The operators have no backward: a tensor that requires grad is refused unless gradients are off
    (torch.no_grad(), torch.inference_mode()).

    Work is queued on the stream given at creation (None: PyTorch's current one), which has to be
    PyTorch's current stream in every call. block_table, seq_pages, free_list, row_start, row_slot and
    row_pos are int32 tensors over the cache's own books, to be read in that stream's order."""

    def __init__(self, n_heads, n_kv_heads, head_dim, page_size, n_pages, max_seqs, max_ctx, max_rows, dtype="bf16",
                 rope_base=0.0, device=0, stream=None):
        import torch
        if dtype not in ("bf16", "f32"):
            raise ValueError("dtype must be 'bf16' or 'f32'")
        self.L = lib()
        self.h = None
        self.n_heads, self.n_kv_heads, self.head_dim = n_heads, n_kv_heads, head_dim
        self.max_rows, self.rows = max_rows, 0
        self.dtype = torch.bfloat16 if dtype == "bf16" else torch.float32
        self._int32, self._float32 = torch.int32, torch.float32
        self.pool_shape = (n_pages, n_kv_heads, page_size, head_dim)
        cfg = cllm_paged_config(n_heads, n_kv_heads, head_dim, 1 if dtype == "bf16" else 0, page_size, n_pages, max_seqs,
                                max_ctx, max_rows, rope_base, device, None, None, 0)
        n = ctypes.c_size_t(0)
        st = self.L.cllm_paged_workspace_bytes(ctypes.byref(cfg), ctypes.byref(n))
        if st != CLLM_OK:
            raise CllmError(st, "cllm_paged_workspace_bytes failed")
        self.device = torch.device("cuda", device)
        # the address of the current stream (2 us less per call than by a Stream object)
        raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
        self._current = (lambda: raw(device)) if raw else (lambda: torch.cuda.current_stream(self.device).cuda_stream)
        cur = torch.cuda.current_stream(self.device)
        self.stream = cur.cuda_stream if stream is None else stream
        self._ws = torch.empty(n.value, dtype=torch.uint8, device=self.device)
        if self.stream != cur.cuda_stream:
            cur.synchronize()  # the memory's last user in the allocator's order
            # (an ExternalStream of address 0 would be a new stream)
            self._ws.record_stream(torch.cuda.ExternalStream(self.stream, device=self.device) if self.stream else
                                   torch.cuda.default_stream(self.device))
        cfg.stream, cfg.workspace, cfg.workspace_bytes = self.stream, self._ws.data_ptr(), n.value
        h = _vp()
        st = self.L.cllm_paged_create(ctypes.byref(cfg), ctypes.byref(h))
        if st != CLLM_OK:
            raise CllmError(st, "cllm_paged_create failed")
        self.h = h
        v = cllm_paged_views()
        self._check(self.L.cllm_paged_views_get(h, ctypes.byref(v)))

        def view(ptr, *shape):
            o, count = ptr - self._ws.data_ptr(), 1
            for x in shape:
                count *= x
            return self._ws[o:o + 4 * count].view(torch.int32).view(*shape)

        self.block_table = view(v.block_table, max_seqs, v.max_pages)
        self.seq_pages, self.free_list = view(v.seq_pages, max_seqs), view(v.free_list, n_pages)
        self.row_start, self.row_slot = view(v.row_start, max_seqs + 1), view(v.row_slot, max_rows)
        self.row_pos = view(v.row_pos, max_rows)

    def close(self):
        """Ends the cache. Waits for nothing (a graph may be in capture): work in flight has the books until PyTorch's
        allocator gives their memory to another user, in the stream's order."""
        if getattr(self, "h", None):
            self.L.cllm_paged_free(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _check(self, st):
        if st != CLLM_OK:
            msg = self.L.cllm_paged_last_error(self.h)
            raise CllmError(st, msg.decode() if msg else "")

    def _on_stream(self):
        if not self.h:
            raise ValueError("the cache is closed")
        if self._current() != self.stream:
            raise ValueError("PyTorch's current stream is not the cache's")

    def _no_backward(self, name):
        import torch
        if torch.is_grad_enabled():
            raise ValueError(f"{name} requires grad, and the paged operators have no backward: call them under torch.no_grad()")

    def _lens(self, x, n):
        if x.dtype != self._int32 or x.dim() != 1 or x.numel() != n or not x.is_contiguous() or x.device != self.device:
            raise ValueError(f"lengths: contiguous int32 tensors of one size on {self.device}, got {x.dtype} "
                             f"{tuple(x.shape)} on {x.device}")
        return x.data_ptr()

    def _rows(self, x, heads, name):
        """Address and row stride of rows [>= the plan's rows][heads][head_dim] (or [..][heads * head_dim])."""
        s, t = x.shape, x.stride()
        whole = (len(s) == 3 and s[1] == heads and s[2] == self.head_dim and t[2] == 1 and (heads == 1 or t[1] == self.head_dim)
                 ) or (len(s) == 2 and s[1] == heads * self.head_dim and t[1] == 1)
        if not whole or s[0] < self.rows or x.dtype != self.dtype or x.device != self.device:
            raise ValueError(f"{name}: at least {self.rows} rows of {heads} x {self.head_dim} {self.dtype} with contiguous "
                             f"heads on {self.device}, got {x.dtype} {tuple(s)} strides {tuple(t)} on {x.device}")
        if x.requires_grad:
            self._no_backward(name)
        return x.data_ptr(), (t[0] if s[0] > 1 else heads * self.head_dim)

    def _pool(self, x, name):
        if x.shape != self.pool_shape or x.dtype != self.dtype or x.device != self.device or not x.is_contiguous():
            raise ValueError(f"{name}: a contiguous {self.dtype} tensor {self.pool_shape} on {self.device}, got {x.dtype} "
                             f"{tuple(x.shape)} on {x.device}")
        if x.requires_grad:
            self._no_backward(name)
        return x.data_ptr()

    def plan(self, seq_ids, ctx_lens, new_lens, rows, max_new=0, max_len=0):
        """cllm_paged_plan: int32 tensors of one size; rows, max_new, max_len: the host's bounds."""
        self._on_stream()
        n = seq_ids.numel()
        self._check(self.L.cllm_paged_plan(self.h, n, self._lens(seq_ids, n), self._lens(ctx_lens, n),
                                           self._lens(new_lens, n), rows, max_new, max_len))
        self.rows = rows
        _changed(self._ws)

    def append(self, q, k, v, q_out, k_pages, v_pages):
        """cllm_paged_append: rows q [.., n_heads, head_dim] (or None, with q_out), k and v
        [.., n_kv_heads, head_dim], of any row stride, into pools of pool_shape."""
        self._on_stream()
        if (q is None) != (q_out is None):
            raise ValueError("q and q_out go together")
        none = (None, 0)
        qa = none if q is None else self._rows(q, self.n_heads, "q")
        qo = none if q_out is None else self._rows(q_out, self.n_heads, "q_out")
        self._check(self.L.cllm_paged_append(self.h, *qa, *self._rows(k, self.n_kv_heads, "k"),
                                             *self._rows(v, self.n_kv_heads, "v"), *qo, self._pool(k_pages, "k_pages"),
                                             self._pool(v_pages, "v_pages")))
        if q_out is None:
            _changed(k_pages, v_pages)
        else:
            _changed(q_out, k_pages, v_pages)

    def attn(self, q, k_pages, v_pages, out, scale=None, lse=None):
        """cllm_paged_attn: rows q [.., n_heads, head_dim] over the pools into out (of q's shape); lse: a
        contiguous float32 [.., n_heads]. scale None: 1 / sqrt(head_dim)."""
        self._on_stream()
        if scale is not None and not _f32(scale).value:
            raise ValueError(f"scale {scale} is 0 in float32")
        if lse is not None:
            if lse.dtype != self._float32 or lse.dim() != 2 or lse.shape[1] != self.n_heads or lse.shape[0] < self.rows or \
                    not lse.is_contiguous() or lse.device != self.device:
                raise ValueError(f"lse: a contiguous float32 tensor of at least {self.rows} x {self.n_heads} on {self.device}")
            if lse.requires_grad:
                self._no_backward("lse")
        self._check(self.L.cllm_paged_attn(self.h, *self._rows(q, self.n_heads, "q"), self._pool(k_pages, "k_pages"),
                                           self._pool(v_pages, "v_pages"), 0.0 if scale is None else scale,
                                           *self._rows(out, self.n_heads, "out"),
                                           None if lse is None else lse.data_ptr()))
        if lse is None:
            _changed(out)
        else:
            _changed(out, lse)

    def status(self):
        """cllm_paged_status: (rows of the last plan, free pages); raises when it was refused."""
        rows, free = _i32(0), _i32(0)
        self._check(self.L.cllm_paged_status(self.h, ctypes.byref(rows), ctypes.byref(free)))
        return int(rows.value), int(free.value)


def records_to_dicts(raw):
    out = []
    for r in raw:
        m = int(r[3])
        out.append({"L": int(r[0]), "e": int(r[1]), "b0": int(r[2]), "m": m, "a": int(r[4]),
                    "z": r[5:5 + m].copy(), "pred": r[5 + 64:5 + 64 + m].copy()})
    return out


def dicts_to_records(traj):
    raw = np.zeros((max(len(traj), 1), TRACE_STRIDE), dtype=np.int32)
    for t, r in enumerate(traj):
        raw[t, :5] = [r["L"], r["e"], r["b0"], r["m"], r["a"]]
        raw[t, 5:5 + r["m"]] = r["z"]
        raw[t, 5 + 64:5 + 64 + r["m"]] = r["pred"]
    return raw[:len(traj)]


def trace_count(traj, tokens, n, block_policy):
    """Fast-forward and stationary counts of a trajectory (cllm_trace_count)."""
    raw = dicts_to_records(traj) if isinstance(traj, list) else np.ascontiguousarray(traj, dtype=np.int32)
    tok = np.ascontiguousarray(tokens, dtype=np.int32)
    st = cllm_trace_stats()
    rc = lib().cllm_trace_count(_p(raw) if raw.size else None, raw.shape[0], _p(tok) if tok.size else None,
                                tok.size, n, block_policy, ctypes.byref(st))
    if rc:
        raise CllmError(rc, "cllm_trace_count")
    return {"iterations": int(st.iterations), "fast_forward_mean": float(st.fast_forward_mean),
            "stationary": int(st.stationary), "windows": int(st.windows),
            "stationary_per_window": float(st.stationary_per_window)}


def collect_states(traj, tokens, n, rate, seed):
    """Trajectory states and their augmented copies (cllm_collect_states): arrays
    states[S, n], augmented[S, n] (-1 past a short block) and block_start[S]."""
    raw = dicts_to_records(traj) if isinstance(traj, list) else np.ascontiguousarray(traj, dtype=np.int32)
    tok = np.ascontiguousarray(tokens, dtype=np.int32)
    cnt = _i64(0)
    args = (_p(raw) if raw.size else None, raw.shape[0], _p(tok) if tok.size else None, tok.size, n, float(rate),
            int(seed) & ((1 << 64) - 1))
    rc = lib().cllm_collect_states(*args, None, None, None, 0, ctypes.byref(cnt))
    if rc:
        raise CllmError(rc, "cllm_collect_states")
    S = int(cnt.value)
    st = np.zeros((max(S, 1), n), dtype=np.int32)
    au = np.zeros((max(S, 1), n), dtype=np.int32)
    bs = np.zeros(max(S, 1), dtype=np.int32)
    rc = lib().cllm_collect_states(*args, _p(st), _p(au), _p(bs), S, ctypes.byref(cnt))
    if rc:
        raise CllmError(rc, "cllm_collect_states")
    return st[:S], au[:S], bs[:S]


def _stats(st):
    return {"steps": int(st.steps), "blocks": int(st.blocks), "tokens": int(st.tokens),
            "accept_hist": [int(x) for x in st.accept_hist], "prefill_ms": float(st.prefill_ms),
            "decode_ms": float(st.decode_ms), "rows": int(st.rows), "iter_ms_p10": float(st.iter_ms_p10),
            "iter_ms_p50": float(st.iter_ms_p50), "iter_ms_p90": float(st.iter_ms_p90),
            "iter_ms_full_p50": float(st.iter_ms_full_p50), "iter_ms_full_p10": float(st.iter_ms_full_p10),
            "iter_ms_full_p90": float(st.iter_ms_full_p90)}


def write_weight_file(path, cfg: ModelConfig, tensors):
    """Write the weight-file format of cllm_model_load: 64-byte header, then the tensors."""
    import struct
    hdr = b"CLLMWTS1" + struct.pack("<i6i2fi", 1, cfg.n_layers, cfg.d_model, cfg.n_heads, cfg.head_dim,
                                    cfg.ffn_dim, cfg.vocab, cfg.rms_eps, cfg.rope_base, cfg.dtype_code)
    hdr = hdr + b"\0" * (64 - len(hdr))
    with open(path, "wb") as f:
        f.write(hdr)
        for t in tensors:
            f.write(np.ascontiguousarray(t).tobytes())
