"""Thin ctypes binding of ``libpacer.so`` (C ABI declared in ``include/pacer.h``).

Argument marshalling only: every step of the decoding loop runs in the CUDA
library.  PyTorch is used for device memory (the workspace and the weights are
torch tensors owned by the caller) and for the stream.  Importing this module
fails loudly when the library has not been built; there is no CPU fallback.
"""
from __future__ import annotations

import array
import contextlib
import ctypes as C
import math
import os
import threading
import weakref
from typing import Dict, Optional

import numpy as np
import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libpacer.so")

if not os.path.exists(LIB_PATH):
    raise ImportError(
        f"{LIB_PATH} is missing: build it with `python -m paper_2602_01274_b200.build` "
        "(nvcc, sm_100a). There is no fallback path.")

_lib = C.CDLL(LIB_PATH)

PACER_TARGET, PACER_DRAFT, PACER_PREVERIFY = 0, 1, 2
PACER_GREEDY, PACER_SAMPLE = 0, 1
(BUF_TOKENS, BUF_DRAFTS, BUF_ALPHA, BUF_VERIFY_LOGITS, BUF_DRAFT_LOGITS, BUF_HPEND, BUF_DRAFT_LEN, BUF_ACCEPT_LEN,
 BUF_KCACHE_T, BUF_VCACHE_T, BUF_KCACHE_D, BUF_VCACHE_D, BUF_KCACHE_B, BUF_VCACHE_B, BUF_PHASE_NS) = range(15)


class ModelCfg(C.Structure):
    _fields_ = [("n_layers", C.c_int32), ("d_model", C.c_int32), ("n_heads", C.c_int32), ("n_kv_heads", C.c_int32),
                ("d_ffn", C.c_int32), ("vocab", C.c_int32), ("rope_theta", C.c_float), ("rms_eps", C.c_float)]


class Cfg(C.Structure):
    _fields_ = [("target", ModelCfg), ("draft", ModelCfg), ("max_batch", C.c_int32), ("max_ctx", C.c_int32),
                ("gamma_cap", C.c_int32), ("block_b", C.c_int32), ("rho", C.c_float), ("criterion", C.c_int32),
                ("succ_bias", C.c_float), ("use_posemb", C.c_int32), ("mb_scope", C.c_int32)]


class Tensor(C.Structure):
    _fields_ = [("name", C.c_char_p), ("dev_ptr", C.c_void_p), ("numel", C.c_int64)]


class AdamwCfg(C.Structure):
    _fields_ = [("lr", C.c_double), ("beta_one", C.c_double), ("beta_two", C.c_double), ("eps", C.c_double), ("weight_decay", C.c_double),
                ("max_norm", C.c_double), ("step", C.c_int64), ("seed", C.c_uint64), ("norm", C.c_void_p), ("lr_device", C.c_void_p),
                ("step_device", C.c_void_p), ("state_bits", C.c_int32), ("seeded", C.c_int32)]


class Stats(C.Structure):
    _fields_ = [("n_draft_fwd", C.c_int64), ("n_mb_calls", C.c_int64), ("n_target_fwd", C.c_int64),
                ("n_steps", C.c_int64), ("n_generated", C.c_int64), ("n_kernel_launches", C.c_int64),
                ("ms_prefill", C.c_float), ("ms_decode", C.c_float)]

    def as_dict(self):
        return {k: getattr(self, k) for k, _ in self._fields_}


class SeqState(C.Structure):
    _fields_ = [("P", C.c_int32), ("len_T", C.c_int32), ("len_D", C.c_int32), ("len_B", C.c_int32),
                ("gamma", C.c_int32), ("k_round", C.c_int32), ("t_k", C.c_float), ("drafting", C.c_int32),
                ("finished", C.c_int32), ("n_steps", C.c_int32), ("last_n", C.c_int32), ("last_next", C.c_int32),
                ("n_pend", C.c_int32), ("err", C.c_int32), ("n_draft_fwd", C.c_int64), ("n_mb_calls", C.c_int64),
                ("n_target_fwd", C.c_int64)]

    def as_dict(self):
        return {k: getattr(self, k) for k, _ in self._fields_}


_P = C.c_void_p
_lib.pacer_strerror.restype = C.c_char_p
_lib.pacer_strerror.argtypes = [C.c_int]
_lib.pacer_last_error.restype = C.c_char_p
_lib.pacer_last_error.argtypes = [_P]
_lib.pacer_workspace_bytes.restype = C.c_size_t
_lib.pacer_workspace_bytes.argtypes = [C.POINTER(Cfg)]
_lib.pacer_create.argtypes = [C.POINTER(Cfg), _P, C.c_size_t, _P, C.POINTER(_P)]
_lib.pacer_destroy.argtypes = [_P]
_lib.pacer_load_weights.argtypes = [_P, C.c_int, C.POINTER(Tensor), C.c_int, _P]
_lib.pacer_prefill.argtypes = [_P, _P, C.c_int, C.c_int, C.c_int, C.c_int, C.c_float, C.c_int, C.c_uint64]
for _n in ("pacer_draft_step", "pacer_preverify", "pacer_verify", "pacer_accept_rollback"):
    getattr(_lib, _n).argtypes = [_P]
_lib.pacer_debug_set_device_status.argtypes = [_P, C.c_int, C.c_int, C.c_int, C.c_int]
_lib.pacer_read_state.argtypes = [_P, C.POINTER(SeqState), C.c_int]
_lib.pacer_read_buffer.argtypes = [_P, C.c_int, _P, C.c_size_t]
_lib.pacer_generate.argtypes = [_P, _P, C.c_int, C.c_int, C.c_int, C.c_int, C.c_float, C.c_int, C.c_uint64,
                                _P, _P, _P, _P, C.POINTER(Stats)]
_lib.pacer_generate_sched.argtypes = [_P, _P, C.c_int, C.c_int, C.c_int, _P, C.c_int, C.c_int, C.c_uint64,
                                      _P, _P, _P, _P, C.POINTER(Stats)]
_lib.pacer_generate_ar.argtypes = [_P, _P, C.c_int, C.c_int, C.c_int, C.c_int, C.c_uint64, _P, C.POINTER(Stats)]
_lib.pacer_profile_begin.argtypes = [_P]
_lib.pacer_profile_end.argtypes = [_P, C.POINTER(C.c_double), C.POINTER(C.c_double), C.POINTER(C.c_int64)]
_lib.pacer_linear_scratch_bytes.restype = C.c_size_t
_lib.pacer_linear_scratch_bytes.argtypes = [C.c_int, C.c_int, C.c_int]
_lib.pacer_linear.argtypes = [_P, _P, _P, C.c_int, C.c_int, C.c_int, _P, C.c_size_t, _P]
_lib.pacer_linear_static.argtypes = [_P, _P, _P, C.c_int, C.c_int, C.c_int, _P]
PACER_LINEAR_STATIC_BYTES = 4 << 20
_I, _L, _F = C.c_int, C.c_int64, C.c_float
_lib.pacer_logprobs.argtypes = [_P, _I, _L, _I, _I, _P, _I, _P, _P, _P, _P, _P, _P]
_lib.pacer_batch.argtypes = [_P]
_lib.pacer_verify_logprobs.argtypes = [_P, _I, _P, _P, _P, _P]
_lib.pacer_logprobs_backward.argtypes = [_P, _I, _L, _I, _I, _P, _P, _P, _P, _P, _P, _P, _L, _P]
_lib.pacer_distill.argtypes = [_P, _I, _L, _I, _I, _P, _P, _I, _I, _P, _F, _P, _P, _P, _P, _P, _L, _P]
_lib.pacer_distill_backward.argtypes = [_P, _I, _L, _I, _I, _P, _P, _I, _I, _P, _F, _P, _P, _P, _P, _L, _P]
_lib.pacer_head_logprobs_scratch_bytes.restype = C.c_size_t
_lib.pacer_head_logprobs_scratch_bytes.argtypes = [_I, _I]
_lib.pacer_head_logprobs.argtypes = [_P, _L, _P, _L, _I, _I, _I, _P, _P, _F, _P, _P, _P, _P, C.c_size_t, _P]
for _n, _a in (("pacer_head_logprobs_backward", [_P] * 6 + [_P, _L, _P, _L]), ("pacer_head_nll_grad", [_P] * 2 + [_P, _L, _P, _L])):
    getattr(_lib, _n).argtypes = [_P, _L, _P, _L, _I, _I, _I, _P, _P, _F, *_a, _P, C.c_size_t, _P]
    getattr(_lib, _n + "_scratch_bytes").restype = C.c_size_t
    getattr(_lib, _n + "_scratch_bytes").argtypes = [_I, _I, _I]
_lib.pacer_adamw.argtypes = [_P, _I, C.POINTER(AdamwCfg), _P]
_lib.pacer_adamw_states.argtypes = [_P, _I, _P, _P, _P]
_lib.pacer_grad_norm.argtypes = [_P, _I, _P, _P, C.c_size_t, _P]
_lib.pacer_grad_norm_scratch_bytes.restype = C.c_size_t
_lib.pacer_grad_norm_scratch_bytes.argtypes = [_I]
PACER_F32, PACER_BF16, PACER_F16 = 0, 1, 2
PACER_MAX_VOCAB = 393216
_DTYPES = {torch.float32: PACER_F32, torch.bfloat16: PACER_BF16, torch.float16: PACER_F16}


class PacerError(RuntimeError):
    pass


def exported_symbols():
    """The C entry points this binding resolved (all declared in pacer.h)."""
    return ["pacer_strerror", "pacer_last_error", "pacer_workspace_bytes", "pacer_create", "pacer_destroy",
            "pacer_load_weights", "pacer_prefill", "pacer_draft_step", "pacer_preverify", "pacer_verify",
            "pacer_accept_rollback", "pacer_read_state", "pacer_batch", "pacer_read_buffer", "pacer_generate", "pacer_generate_sched",
            "pacer_generate_ar", "pacer_debug_set_device_status",
            "pacer_profile_begin", "pacer_profile_end", "pacer_linear_scratch_bytes", "pacer_linear", "pacer_linear_static",
            "pacer_logprobs", "pacer_verify_logprobs", "pacer_logprobs_backward", "pacer_distill", "pacer_distill_backward",
            "pacer_head_logprobs_scratch_bytes", "pacer_head_logprobs", "pacer_head_logprobs_backward_scratch_bytes",
            "pacer_head_logprobs_backward", "pacer_head_nll_grad_scratch_bytes", "pacer_head_nll_grad",
            "pacer_adamw", "pacer_adamw_states", "pacer_grad_norm_scratch_bytes", "pacer_grad_norm"]


def _model_cfg(s) -> ModelCfg:
    return ModelCfg(s.n_layers, s.d_model, s.n_heads, s.n_kv_heads, s.d_ffn, s.vocab, s.rope_theta, s.rms_eps)


def make_cfg(target, draft, max_batch, max_ctx, gamma_cap, block_b=4, rho=1.05, criterion=0, succ_bias=8.0,
             use_posemb=1, mb_scope=0) -> Cfg:
    """target/draft: objects with n_layers, d_model, n_heads, n_kv_heads, d_ffn, vocab, rope_theta, rms_eps."""
    return Cfg(_model_cfg(target), _model_cfg(draft), max_batch, max_ctx, gamma_cap, block_b, rho, criterion,
               succ_bias, use_posemb, mb_scope)


def pacer_workspace_bytes(cfg: Cfg) -> int:
    return _lib.pacer_workspace_bytes(C.byref(cfg))


def _i32(a) -> np.ndarray:
    return np.ascontiguousarray(np.asarray(a, dtype=np.int32))


# Logits of a window are read into page-locked memory, which is filled at the link's rate: fresh pageable memory took 0.33 ms
# for 3.2 MB, a twelfth of the forward that made them.  A program may keep what it reads, so the total alive is bounded.
_PINNED_MAX = 64 << 20
_pinned_lock = threading.Lock()
_pinned_alive: list = []                        # weak references to the arrays (every view keeps its array alive)


def _pinned_array(nbytes: int) -> Optional[np.ndarray]:
    """A page-locked byte array, or None where it would exceed the bound."""
    global _pinned_alive
    with _pinned_lock:
        alive = [a for a in (r() for r in _pinned_alive) if a is not None]
        if sum(a.nbytes for a in alive) + nbytes > _PINNED_MAX:
            return None
        out = torch.empty(nbytes, dtype=torch.uint8, pin_memory=True).numpy()
        _pinned_alive = [weakref.ref(a) for a in alive] + [weakref.ref(out)]
    return out


class Context:
    """One pacer_ctx.  Methods carry the names of the C entry points."""

    def __init__(self, cfg: Cfg, device="cuda:0", stream: Optional[torch.cuda.Stream] = None):
        self.cfg = cfg
        self.device = torch.device(device)
        nbytes = pacer_workspace_bytes(cfg)
        if nbytes == 0:
            raise PacerError("bad configuration")
        with torch.cuda.device(self.device):
            self.workspace = torch.empty(nbytes + 256, dtype=torch.uint8, device=self.device)
            base = self.workspace.data_ptr()
            self._ws_ptr = (base + 255) // 256 * 256
            # a stream of its own (the legacy default stream cannot be captured into the per-step CUDA graph)
            self.stream = stream if stream is not None else torch.cuda.Stream(self.device)
            h = _P()
            rc = _lib.pacer_create(C.byref(cfg), self._ws_ptr, nbytes, self.stream.cuda_stream, C.byref(h))
        self._h = h
        self._keep = []
        self._check(rc)

    def _check(self, rc):
        if rc != 0:
            msg = _lib.pacer_last_error(self._h if self._h else None)
            raise PacerError(f"{_lib.pacer_strerror(rc).decode()} ({rc}): {msg.decode() if msg else ''}")

    def close(self):
        if getattr(self, "_h", None):
            _lib.pacer_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def pacer_load_weights(self, which: int, tensors: Dict[str, torch.Tensor], succ: Optional[torch.Tensor] = None):
        arr = (Tensor * len(tensors))()
        for i, (k, t) in enumerate(tensors.items()):
            assert t.is_cuda and t.dtype == torch.bfloat16 and t.is_contiguous(), k
            arr[i] = Tensor(k.encode(), t.data_ptr(), t.numel())
            self._keep.append(t)
        sp = None
        if succ is not None:
            assert succ.is_cuda and succ.dtype == torch.int32 and succ.is_contiguous()
            self._keep.append(succ)
            sp = succ.data_ptr()
        with torch.cuda.device(self.device):
            self.stream.wait_stream(torch.cuda.current_stream(self.device))     # the tensors may still be being written
            self._check(_lib.pacer_load_weights(self._h, which, arr, len(tensors), sp))
            torch.cuda.current_stream(self.device).wait_stream(self.stream)     # later torch work sees the copy done

    def pacer_prefill(self, prompt, max_new, gamma_max, threshold, mode=PACER_GREEDY, seed=0):
        p = _i32(prompt)
        if p.ndim == 1:
            p = p[None]
        with torch.cuda.device(self.device):
            self._check(_lib.pacer_prefill(self._h, p.ctypes.data, p.shape[0], p.shape[1], max_new, gamma_max,
                                           threshold, mode, seed))

    def pacer_draft_step(self):
        with torch.cuda.device(self.device):
            self._check(_lib.pacer_draft_step(self._h))

    def pacer_preverify(self):
        with torch.cuda.device(self.device):
            self._check(_lib.pacer_preverify(self._h))

    def pacer_verify(self):
        with torch.cuda.device(self.device):
            self._check(_lib.pacer_verify(self._h))

    def pacer_verify_logprobs(self, top: int = 0):
        """Between pacer_verify and the next stage call: (logp, entropy f32 [batch][gamma_cap + 1], top_ids int32 and top_logp f32
        [batch][gamma_cap + 1][top]) of the target's distributions behind every row of the window, on the device.  Row j's token
        is draft j + 1; rows past a sequence's window are NaN (ids -1).  batch: the current run's, whichever call began it."""
        rows = (_lib.pacer_batch(self._h), self.cfg.gamma_cap + 1)     # (the library writes that many)
        with torch.cuda.device(self.device):
            logp, entropy = (torch.full(rows, math.nan, device=self.device) for _ in range(2))
            ids = torch.full((*rows, max(top, 0)), -1, dtype=torch.int32, device=self.device)
            top_logp = torch.full((*rows, max(top, 0)), math.nan, device=self.device)
            current = torch.cuda.current_stream(self.device)
            self.stream.wait_stream(current)                        # the outputs are being filled there
            self._check(_lib.pacer_verify_logprobs(self._h, top, logp.data_ptr(), entropy.data_ptr(), ids.data_ptr(), top_logp.data_ptr()))
            current.wait_stream(self.stream)
        return logp, entropy, ids, top_logp

    def pacer_accept_rollback(self):
        with torch.cuda.device(self.device):
            self._check(_lib.pacer_accept_rollback(self._h))

    def pacer_debug_set_device_status(self, code, block=0, warp=0, detail=0):
        with torch.cuda.device(self.device):
            self._check(_lib.pacer_debug_set_device_status(self._h, code, block, warp, detail))

    def pacer_read_state(self, batch=1):
        arr = (SeqState * batch)()
        with torch.cuda.device(self.device):
            self._check(_lib.pacer_read_state(self._h, arr, batch))
        return [a.as_dict() for a in arr]

    def pacer_read_buffer(self, which: int, dtype, count: int) -> np.ndarray:
        """The first `count` elements of a device buffer.  Arrays of 256 KB to 64 MB are page-locked while at most 64 MB of
        such arrays are alive in the process (their memory goes back to PyTorch's host cache, which reuses it); others are
        ordinary memory.  As with any page-locked array, keep it until an asynchronous copy out of a part of it has ended."""
        nbytes = count * np.dtype(dtype).itemsize
        out = _pinned_array(nbytes) if (256 << 10) <= nbytes <= _PINNED_MAX else None
        out = np.empty(count, dtype=dtype) if out is None else out.view(dtype)
        with torch.cuda.device(self.device):
            self._check(_lib.pacer_read_buffer(self._h, which, out.ctypes.data, out.nbytes))
        return out

    def pacer_profile_begin(self):
        self._check(_lib.pacer_profile_begin(self._h))

    def pacer_profile_end(self):
        """Returns (summed GEMM device ms, weight bytes streamed, launches)."""
        ms, by, n = C.c_double(0), C.c_double(0), C.c_int64(0)
        with torch.cuda.device(self.device):
            self._check(_lib.pacer_profile_end(self._h, C.byref(ms), C.byref(by), C.byref(n)))
        return ms.value, by.value, n.value

    def pacer_generate(self, prompt, max_new, gamma_max, threshold, mode=PACER_GREEDY, seed=0):
        """Returns (tokens [batch][max_new], n_steps [batch], draft_len, accept_len [batch][max_new], stats dict)."""
        p = _i32(prompt)
        if p.ndim == 1:
            p = p[None]
        B = p.shape[0]
        tok = np.zeros((B, max_new), np.int32)
        ns = np.zeros(B, np.int32)
        dl = np.zeros((B, max_new), np.int32)
        al = np.zeros((B, max_new), np.int32)
        st = Stats()
        with torch.cuda.device(self.device):
            self._check(_lib.pacer_generate(self._h, p.ctypes.data, B, p.shape[1], max_new, gamma_max, threshold, mode,
                                            seed, tok.ctypes.data, ns.ctypes.data, dl.ctypes.data, al.ctypes.data,
                                            C.byref(st)))
        return tok, ns, dl, al, st.as_dict()

    def pacer_generate_sched(self, prompt, max_new, windows, mode=PACER_GREEDY, seed=0):
        """Speculative decoding with prescribed windows (int32 [batch][n_windows] or [n_windows]); returns like
        pacer_generate."""
        p = _i32(prompt)
        if p.ndim == 1:
            p = p[None]
        w = _i32(windows)
        if w.ndim == 1:
            w = w[None]
        B = p.shape[0]
        assert w.shape[0] == B
        tok = np.zeros((B, max_new), np.int32)
        ns = np.zeros(B, np.int32)
        dl = np.zeros((B, max_new), np.int32)
        al = np.zeros((B, max_new), np.int32)
        st = Stats()
        with torch.cuda.device(self.device):
            self._check(_lib.pacer_generate_sched(self._h, p.ctypes.data, B, p.shape[1], max_new, w.ctypes.data,
                                                  w.shape[1], mode, seed, tok.ctypes.data, ns.ctypes.data,
                                                  dl.ctypes.data, al.ctypes.data, C.byref(st)))
        return tok, ns, dl, al, st.as_dict()

    def pacer_generate_ar(self, prompt, max_new, mode=PACER_GREEDY, seed=0):
        p = _i32(prompt)
        if p.ndim == 1:
            p = p[None]
        tok = np.zeros((p.shape[0], max_new), np.int32)
        st = Stats()
        with torch.cuda.device(self.device):
            self._check(_lib.pacer_generate_ar(self._h, p.ctypes.data, p.shape[0], p.shape[1], max_new, mode, seed,
                                               tok.ctypes.data, C.byref(st)))
        return tok, st.as_dict()


def pacer_linear(x: torch.Tensor, w: torch.Tensor) -> torch.Tensor:
    """y = x @ w.T through the library's skinny GEMM. x bf16 [rows<=32][K], w bf16 [N][K] -> f32 [rows][N]."""
    assert x.is_cuda and w.is_cuda and x.dtype == torch.bfloat16 and w.dtype == torch.bfloat16
    x, w = x.contiguous(), w.contiguous()
    rows, K = x.shape
    N = w.shape[0]
    nbytes = _lib.pacer_linear_scratch_bytes(rows, N, K)
    if nbytes == 0:
        raise PacerError("pacer_linear: unsupported shape")
    dev = x.device
    y = torch.empty(rows, N, dtype=torch.float32, device=dev)
    # (switching the current device costs more than the product of a small shape, and so does an allocation: the product reads no
    # scratch, and where the entry point without it takes the shape it is the one called)
    with contextlib.nullcontext() if dev.index == torch.cuda.current_device() else torch.cuda.device(dev):
        stream = torch.cuda.current_stream(dev).cuda_stream
        if nbytes <= PACER_LINEAR_STATIC_BYTES:
            rc = _lib.pacer_linear_static(x.data_ptr(), w.data_ptr(), y.data_ptr(), rows, N, K, stream)
        else:
            scratch = torch.empty(nbytes + 256, dtype=torch.uint8, device=dev)
            rc = _lib.pacer_linear(x.data_ptr(), w.data_ptr(), y.data_ptr(), rows, N, K, (scratch.data_ptr() + 255) // 256 * 256,
                                   nbytes, stream)
    if rc != 0:
        raise PacerError(f"pacer_linear: {_lib.pacer_strerror(rc).decode()}: {_lib.pacer_last_error(None).decode()}")
    return y


def pacer_linear_static(x: torch.Tensor, w: torch.Tensor, out: torch.Tensor) -> torch.Tensor:
    """y = x @ w.T written into the caller's `out` (f32 [rows][N]) without scratch: the call itself
    allocates nothing on the device, for callers whose device memory is all spoken for.  Shapes whose
    pacer_linear_scratch_bytes exceeds PACER_LINEAR_STATIC_BYTES raise PacerError."""
    assert x.is_cuda and w.is_cuda and out.is_cuda and x.dtype == torch.bfloat16 and w.dtype == torch.bfloat16
    assert x.is_contiguous() and w.is_contiguous() and out.is_contiguous() and out.dtype == torch.float32
    rows, K = x.shape
    N = w.shape[0]
    assert tuple(out.shape) == (rows, N)
    with torch.cuda.device(x.device):
        rc = _lib.pacer_linear_static(x.data_ptr(), w.data_ptr(), out.data_ptr(), rows, N, K,
                                      torch.cuda.current_stream(x.device).cuda_stream)
    if rc != 0:
        raise PacerError(f"pacer_linear_static: {_lib.pacer_strerror(rc).decode()}: {_lib.pacer_last_error(None).decode()}")
    return out


# ----------------------------------------------------------------------------- operators on rows of logits


def _rows(t: torch.Tensor, name: str = "logits") -> torch.Tensor:
    """`t` as the library takes it: on the GPU, [rows][vocab], one of three types, elements of a row side by side."""
    if not (t.is_cuda and t.dim() == 2 and t.dtype in _DTYPES):
        raise AssertionError(f"{name}: f32, bf16 or f16 [rows][vocab] on the GPU")
    return t if t.is_contiguous() or (t.stride(1) == 1 and t.stride(0) >= t.shape[1]) else t.contiguous()


def _vec(t: Optional[torch.Tensor], name: str, like: torch.Tensor, dtype, *more) -> Optional[torch.Tensor]:
    """A side input: [rows] or [rows][more], of the given type, contiguous, beside the logits.  None stays None."""
    if t is None:
        return None
    if t.dtype != dtype or t.shape != (like.shape[0], *more) or t.device != like.device:
        raise AssertionError(f"{name}: {dtype} of shape {(like.shape[0], *more)} on {like.device}")
    return t.contiguous()


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else t.data_ptr()


def _ld(t: torch.Tensor) -> int:
    """Elements from row to row (a single row's stride says nothing)."""
    return t.shape[1] if t.is_contiguous() else t.stride(0)


def _layout(z: torch.Tensor):
    """The C arguments that describe rows of logits."""
    return z.data_ptr(), _DTYPES[z.dtype], _ld(z), *z.shape


def _gradient_like(z: torch.Tensor) -> torch.Tensor:
    """Rows that lie as the logits' do (so that they are written 16 bytes at a time), where those are padded by little."""
    rows, vocab = z.shape
    if vocab < z.stride(0) <= vocab + 1024 and rows > 1:
        return torch.empty(rows, z.stride(0), dtype=z.dtype, device=z.device)[:, :vocab]
    return torch.empty(rows, vocab, dtype=z.dtype, device=z.device)


def _out_like(z: torch.Tensor, out: Optional[torch.Tensor]) -> torch.Tensor:
    if out is None:
        return _gradient_like(z)
    assert out.device == z.device and out.dtype == z.dtype and out.shape == z.shape and out.stride(1) == 1 and \
        (out.shape[0] <= 1 or out.stride(0) >= out.shape[1]), "out: like the logits, rows apart"
    return out


def _written(*outputs: Optional[torch.Tensor]):
    """Tensors of the caller that a call has written: autograd has to know, as of torch's own in-place functions, so that a backward
    pass which saved them (or what they are views of) says so instead of computing with what is there now."""
    changed = [t for t in outputs if t is not None]
    if changed:
        torch.autograd.graph.increment_version(changed)


# torch.cuda.current_stream(..).cuda_stream, where torch has it without the object that costs 2 us a call
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda dev: torch.cuda.current_stream(dev).cuda_stream)


def _call(fn, like: torch.Tensor, *args):
    """The C entry point on the tensors' device and torch's current stream there."""
    dev = like.device.index
    if dev == torch.cuda.current_device():
        rc = fn(*args, _raw_stream(dev))
    else:
        with torch.cuda.device(dev):
            rc = fn(*args, _raw_stream(dev))
    if rc != 0:
        raise PacerError(f"{fn.__name__}: {_lib.pacer_strerror(rc).decode()}: {_lib.pacer_last_error(None).decode()}")


def pacer_logprobs(logits: torch.Tensor, tokens: torch.Tensor, top: int = 0, out=None):
    """Log probabilities of given tokens under rows of logits [rows][vocab] (f32, bf16 or f16): returns
    (logp [rows], entropy [rows], lse [rows], top_ids int32 [rows][top], top_logp [rows][top]).  tokens int32 [rows]; one outside
    the vocabulary (-1, say) has logp 0.  Alternatives: larger logit first, of equal ones the lower id.  `out`: five such tensors
    to write (contiguous; else they are made, views of one allocation).  No gradient: see pacer_logprobs_backward, and
    losses.token_logprobs for autograd."""
    z = _rows(logits)
    tokens = _vec(tokens, "tokens", z, torch.int32)
    rows, dev, n = z.shape[0], z.device, max(top, 0)
    if out is None:
        logp, entropy, lse, top_logp = torch.empty((3 + n) * rows, dtype=torch.float32, device=dev).split_with_sizes((rows, rows, rows, n * rows))
        ids, top_logp = torch.empty((rows, n), dtype=torch.int32, device=dev), top_logp.view(rows, n)
    else:
        logp, entropy, lse, ids, top_logp = out
        for t in out:
            shape, dtype = ((rows, n) if t is ids or t is top_logp else (rows,)), (torch.int32 if t is ids else torch.float32)
            assert t.shape == shape and t.dtype == dtype and t.device == dev and t.is_contiguous(), f"out: contiguous {dtype} {shape} on {dev}"
    _call(_lib.pacer_logprobs, z, *_layout(z), _ptr(tokens), top, logp.data_ptr(), entropy.data_ptr(), lse.data_ptr(), ids.data_ptr(),
          top_logp.data_ptr())
    if out is not None:
        _written(*out)
    return logp, entropy, lse, ids, top_logp


def pacer_logprobs_backward(logits, tokens, lse, entropy, grad_logp, grad_entropy=None, grad_lse=None, out=None):
    """The gradient of pacer_logprobs' logp, entropy and lse with respect to the logits, in their type.  Each incoming gradient
    (f32 [rows]) may be None; `out` may be the logits themselves."""
    z = _rows(logits)
    f32 = torch.float32
    tokens, lse, entropy = _vec(tokens, "tokens", z, torch.int32), _vec(lse, "lse", z, f32), _vec(entropy, "entropy", z, f32)
    gl, gh, gs = _vec(grad_logp, "grad_logp", z, f32), _vec(grad_entropy, "grad_entropy", z, f32), _vec(grad_lse, "grad_lse", z, f32)
    given, out = out, _out_like(z, out)
    _call(_lib.pacer_logprobs_backward, z, *_layout(z), _ptr(tokens), _ptr(lse), _ptr(entropy), _ptr(gl), _ptr(gh), _ptr(gs), out.data_ptr(),
          _ld(out))
    _written(given)
    return out


def _teacher(z, ids, teacher, teacher_lse):
    k = ids.shape[-1] if ids.dim() == 2 else -1
    ids = _vec(ids, "ids", z, torch.int32, k)
    assert teacher.dtype in _DTYPES, "teacher: f32, bf16 or f16"
    return ids, _vec(teacher, "teacher", z, teacher.dtype, k), _vec(teacher_lse, "teacher_lse", z, torch.float32), k


def pacer_distill(logits, ids, teacher, temperature: float = 1.0, teacher_lse=None):
    """Distillation from a teacher's top logits: per row KL(q || p) with p = softmax(logits / temperature) and q over the listed
    tokens ids int32 [rows][k] with logits teacher [rows][k] (f32, bf16 or f16), renormalised; with teacher_lse f32 [rows] (the
    teacher's log-sum-exp over its whole row, at this temperature) the tokens outside the list are one further class.  An id
    outside the vocabulary is no entry.  Returns (loss [rows], lse [rows], tail_lse [rows] or None)."""
    z = _rows(logits)
    ids, teacher, teacher_lse, k = _teacher(z, ids, teacher, teacher_lse)
    loss, lse = torch.empty(2, z.shape[0], dtype=torch.float32, device=z.device).unbind(0)
    tail = None if teacher_lse is None else torch.empty_like(teacher_lse)
    _call(_lib.pacer_distill, z, *_layout(z), ids.data_ptr(), teacher.data_ptr(), _DTYPES[teacher.dtype], k, _ptr(teacher_lse), temperature,
          loss.data_ptr(), lse.data_ptr(), _ptr(tail), None, None, 0)
    return loss, lse, tail


def pacer_distill_grad(logits, ids, teacher, weight, temperature: float = 1.0, teacher_lse=None, out=None):
    """pacer_distill's loss [rows] and, in the same pass, weight[row] times its gradient with respect to the logits (in their
    type; `out` may be the logits themselves): (loss, dlogits)."""
    z = _rows(logits)
    ids, teacher, teacher_lse, k = _teacher(z, ids, teacher, teacher_lse)
    weight = _vec(weight, "weight", z, torch.float32)
    given, out = out, _out_like(z, out)
    loss = torch.empty(z.shape[0], dtype=torch.float32, device=z.device)
    _call(_lib.pacer_distill, z, *_layout(z), ids.data_ptr(), teacher.data_ptr(), _DTYPES[teacher.dtype], k, _ptr(teacher_lse), temperature,
          loss.data_ptr(), None, None, _ptr(weight), out.data_ptr(), _ld(out))
    _written(given)
    return loss, out


def pacer_distill_backward(logits, ids, teacher, lse, tail_lse, grad_loss, temperature: float = 1.0, teacher_lse=None, out=None):
    """The gradient of pacer_distill's loss from what that call left (lse, tail_lse) and f32 [rows] grad_loss."""
    z = _rows(logits)
    ids, teacher, teacher_lse, k = _teacher(z, ids, teacher, teacher_lse)
    f32 = torch.float32
    lse, tail_lse, grad_loss = _vec(lse, "lse", z, f32), _vec(tail_lse, "tail_lse", z, f32), _vec(grad_loss, "grad_loss", z, f32)
    given, out = out, _out_like(z, out)
    _call(_lib.pacer_distill_backward, z, *_layout(z), ids.data_ptr(), teacher.data_ptr(), _DTYPES[teacher.dtype], k, _ptr(teacher_lse),
          temperature, _ptr(lse), _ptr(tail_lse), _ptr(grad_loss), out.data_ptr(), _ld(out))
    _written(given)
    return out


def pacer_head_logprobs(hidden, head, tokens, bias_ids=None, bias: float = 0.0):
    """pacer_logprobs of the rows hidden @ head.T without writing those logits: hidden bf16 [rows][d], head bf16 [vocab][d]
    (rows of 16-byte multiples), tokens int32 [rows]; bias_ids int32 [rows]: tokens whose logit gets `bias` added.
    Returns (logp [rows], entropy [rows], lse [rows])."""
    h, w = _rows(hidden, "hidden"), _rows(head, "head")
    assert h.dtype == w.dtype == torch.bfloat16 and h.device == w.device and h.shape[1] == w.shape[1], "bf16 [rows][d] and [vocab][d]"
    tokens, bias_ids = _vec(tokens, "tokens", h, torch.int32), _vec(bias_ids, "bias_ids", h, torch.int32)
    rows, d = h.shape
    vocab = w.shape[0]
    nbytes = _lib.pacer_head_logprobs_scratch_bytes(rows, vocab)
    logp, entropy, lse = torch.empty(3 * rows, dtype=torch.float32, device=h.device).split_with_sizes((rows, rows, rows))
    scratch = torch.empty(nbytes, dtype=torch.uint8, device=h.device)      # (torch aligns an allocation to 512 bytes)
    _call(_lib.pacer_head_logprobs, h, h.data_ptr(), _ld(h), w.data_ptr(), _ld(w), rows, vocab, d, _ptr(tokens),
          _ptr(bias_ids), bias, logp.data_ptr(), entropy.data_ptr(), lse.data_ptr(), scratch.data_ptr(), nbytes)
    return logp, entropy, lse


def _head(hidden, head):
    h, w = _rows(hidden, "hidden"), _rows(head, "head")
    assert h.dtype == w.dtype == torch.bfloat16 and h.device == w.device and h.shape[1] == w.shape[1], "bf16 [rows][d] and [vocab][d]"
    return h, w


def _head_gradients(h, w, grads, out):
    """(dhidden or None, dhead or None, those of the caller)"""
    given = [None, None] if out is None else list(out)
    made = []
    for t, want, mine in zip((h, w), grads, given):
        if mine is not None:
            assert mine.device == t.device and mine.dtype == t.dtype and mine.shape == t.shape and mine.stride(1) == 1 and \
                (mine.shape[0] <= 1 or mine.stride(0) >= mine.shape[1]), "out: like hidden and head, rows apart"
        made.append((torch.empty(t.shape, dtype=t.dtype, device=t.device) if mine is None else mine) if want else None)
    return (*made, [g for g, want in zip(given, grads) if want])


def _ld_or_0(t: Optional[torch.Tensor]) -> int:
    return 0 if t is None else _ld(t)


def pacer_head_logprobs_backward(hidden, head, tokens, logp, lse, entropy, grad_logp, grad_entropy=None, grad_lse=None, bias_ids=None,
                                 bias: float = 0.0, grads=(True, True), out=None):
    """The gradients of pacer_head_logprobs' logp, entropy and lse (what that call returned for the same arguments) with respect to
    hidden and head, bf16: (dhidden [rows][d], dhead [vocab][d]).  Each incoming gradient (f32 [rows]) may be None, not all three;
    tokens and logp may be None where grad_logp is, entropy where grad_entropy is.  grads: which of the two are wanted (the other is None);
    out: a pair of tensors to write (each may be None)."""
    h, w = _head(hidden, head)
    f32, i32 = torch.float32, torch.int32
    tokens, bias_ids = _vec(tokens, "tokens", h, i32), _vec(bias_ids, "bias_ids", h, i32)
    logp, lse, entropy = _vec(logp, "logp", h, f32), _vec(lse, "lse", h, f32), _vec(entropy, "entropy", h, f32)
    gl, gh, gs = _vec(grad_logp, "grad_logp", h, f32), _vec(grad_entropy, "grad_entropy", h, f32), _vec(grad_lse, "grad_lse", h, f32)
    dh, dw, given = _head_gradients(h, w, grads, out)
    (rows, d), vocab = h.shape, w.shape[0]
    nbytes = _lib.pacer_head_logprobs_backward_scratch_bytes(rows, vocab, d)
    scratch = torch.empty(nbytes, dtype=torch.uint8, device=h.device)
    _call(_lib.pacer_head_logprobs_backward, h, h.data_ptr(), _ld(h), w.data_ptr(), _ld(w), rows, vocab, d, _ptr(tokens), _ptr(bias_ids), bias,
          _ptr(logp), _ptr(lse), _ptr(entropy), _ptr(gl), _ptr(gh), _ptr(gs), _ptr(dh), _ld_or_0(dh), _ptr(dw), _ld_or_0(dw), scratch.data_ptr(), nbytes)
    _written(*given)
    return dh, dw


def pacer_head_nll_grad(hidden, head, tokens, weight, bias_ids=None, bias: float = 0.0, grads=(True, True), out=None):
    """Softmax cross entropy of int32 tokens [rows] under the rows hidden @ head.T without keeping those logits (the call's scratch has 16 bits for each,
    32 up to 128 rows, 2 GB at most), and in the same call the gradients of sum(weight * loss): (loss f32 [rows], dhidden bf16 [rows][d], dhead bf16 [vocab][d]).  A token outside the vocabulary
    (-1, say) has loss 0 and passes no gradient.  bias_ids, bias: as pacer_head_logprobs; grads, out: as
    pacer_head_logprobs_backward."""
    h, w = _head(hidden, head)
    tokens, bias_ids, weight = _vec(tokens, "tokens", h, torch.int32), _vec(bias_ids, "bias_ids", h, torch.int32), _vec(weight, "weight", h, torch.float32)
    dh, dw, given = _head_gradients(h, w, grads, out)
    (rows, d), vocab = h.shape, w.shape[0]
    loss = torch.empty(rows, dtype=torch.float32, device=h.device)
    nbytes = _lib.pacer_head_nll_grad_scratch_bytes(rows, vocab, d)
    scratch = torch.empty(nbytes, dtype=torch.uint8, device=h.device)
    _call(_lib.pacer_head_nll_grad, h, h.data_ptr(), _ld(h), w.data_ptr(), _ld(w), rows, vocab, d, _ptr(tokens), _ptr(bias_ids), bias, _ptr(weight),
          loss.data_ptr(), _ptr(dh), _ld_or_0(dh), _ptr(dw), _ld_or_0(dw), scratch.data_ptr(), nbytes)
    _written(*given)
    return loss, dh, dw


# ----------------------------------------------------------------------------- AdamW over many tensors


def _adamw_fits(tensors, numel, device):
    """Whether all is as it has to be (_check_adamw says what is not, ten times as slowly)."""
    params, copies, exp_avg, exp_avg_sq, scales = tensors
    if any(x is not None and len(x) != len(params) for x in tensors) or (params and device.type != "cuda"):
        return False
    types, state = {p.dtype for p in params}, torch.float32 if scales is None else torch.uint8
    given = [x for x in (params, exp_avg, exp_avg_sq, scales) if x is not None]
    if copies is not None:
        given.append([c for c in copies if c is not None])
    return types <= {torch.float32, torch.bfloat16} and {t.dtype for x in (exp_avg, exp_avg_sq) for t in x} <= {state} and \
        all(list(map(torch.Tensor.numel, x)) == numel for x in (params, exp_avg, exp_avg_sq)) and \
        (copies is None or all(c is None or (c.dtype == torch.bfloat16 and c.numel() == n and p.dtype == torch.float32) for c, n, p in zip(copies, numel, params))) and \
        (scales is None or all(x.dtype == torch.float32 and x.shape == (-(-n // 256), 2) for x, n in zip(scales, numel))) and \
        all(all(map(torch.Tensor.is_contiguous, x)) and set(map(torch.Tensor.get_device, x)) <= {device.index} for x in given if x)


def _check_adamw(tensors, numel, device):
    if _adamw_fits(tensors, numel, device):
        return
    params, copies, exp_avg, exp_avg_sq, scales = tensors
    if any(x is not None and len(x) != len(params) for x in tensors):
        raise AssertionError("AdamwTensors: lists of one length")
    state = torch.float32 if scales is None else torch.uint8
    for i, (p, n) in enumerate(zip(params, numel)):
        if not (p.is_cuda and p.dtype in (torch.float32, torch.bfloat16)):
            raise AssertionError(f"param {i}: f32 or bf16 on the GPU")
        if p.numel() != n:
            raise AssertionError(f"param {i}: has another size than when it was given")
        for t, dtype, name in ((exp_avg[i], state, "exp_avg"), (exp_avg_sq[i], state, "exp_avg_sq"), (copies[i] if copies else None, torch.bfloat16, "copy")):
            if (t is not None or name != "copy") and (t.dtype != dtype or t.numel() != n):
                raise AssertionError(f"{name} {i}: {dtype} of the param's size")
        if copies and copies[i] is not None and p.dtype != torch.float32:
            raise AssertionError(f"copy {i}: only of an f32 param")
        if scales is not None and (scales[i].dtype != torch.float32 or scales[i].shape != (-(-n // 256), 2)):
            raise AssertionError(f"scales {i}: torch.float32 [{-(-n // 256)}][2]")
        for x in tensors:
            if x is not None and x[i] is not None and not (x[i].is_contiguous() and x[i].device == device):
                raise AssertionError(f"tensors of param {i}: contiguous, on {device}")


class AdamwTensors:
    """The tensors of an optimiser as the library takes them, checked once and kept: params f32 or bf16, exp_avg and exp_avg_sq of the same
    sizes (f32; with `scales` uint8 codes, scales f32 [ceil(numel / 256)][2]), copies (bf16, with f32 params) or None; all contiguous, on
    one GPU.  roots: the codes of exp_avg_sq hold the second moments' roots.  Holds references to the tensors."""

    def __init__(self, params, exp_avg, exp_avg_sq, scales=None, copies=None, roots: bool = False):
        self.tensors = tuple(None if x is None else list(x) for x in (params, copies, exp_avg, exp_avg_sq, scales))
        params = self.tensors[0]
        self.state_bits, n = 32 if scales is None else 8, len(params)
        self.device = params[0].device if n else None
        self.numel = list(map(torch.Tensor.numel, params))
        _check_adamw(self.tensors, self.numel, self.device)
        self.all = [t for x in self.tensors if x is not None for t in x]
        self.changed = [t for t in self.all if t is not None]
        self._gaps = len(self.changed) < len(self.all)                  # (copies may be missing)
        # pacer_adamw_tensor: param, copy, grad, exp_avg, exp_avg_sq, scales, numel, (param_type, grad_type, v_code)
        self._code = 1 << 48 if roots and scales is not None else 0
        self._types = np.array([_DTYPES[p.dtype] for p in params], dtype=np.int64)
        self.table = np.zeros((n, 8), dtype=np.int64)
        self.table[:, 6], self.table[:, 7] = self.numel, self._types | self._code
        self._address = self.table.ctypes.data
        self._at = self._grads_at = self._grads_types = None
        self._place()

    def _place(self):
        """The addresses, as they are now: a program may exchange a tensor's storage (which is then looked at again)."""
        at = [0 if t is None else t.data_ptr() for t in self.all] if self._gaps else list(map(torch.Tensor.data_ptr, self.all))
        if at != self._at:
            if self._at is not None:
                _check_adamw(self.tensors, self.numel, self.device)
            self._at, n = at, len(self.numel)
            self._types = np.array([_DTYPES[p.dtype] for p in self.tensors[0]], dtype=np.int64)
            self._grads_types = None
            for i, col in enumerate(c for c, x in zip((0, 1, 3, 4, 5), self.tensors) if x is not None):
                self.table[:, col] = at[i * n:(i + 1) * n]

    def with_grads(self, grads):
        """The table's address."""
        if not self.numel:
            raise AssertionError("grads: one for each param")
        types, at = _gradients(grads, self.device)
        if list(map(torch.Tensor.numel, grads)) != self.numel:
            raise AssertionError("grads: one of each param's size")
        self._place()
        if at != self._grads_at:
            self._grads_at = at
            self.table[:, 2] = _words(at)
        if types != self._grads_types:
            self._grads_types = types
            self.table[:, 7] = self._types | (np.array(types, dtype=np.int64) << 32) | self._code
        return self._address


def _words(x) -> np.ndarray:
    """A list of whole numbers as int64 (numpy takes three times as long)."""
    return np.frombuffer(array.array("q", x), dtype=np.int64)


def _gradients(grads, device):
    """Types (one for all, where they are alike) and addresses of gradients."""
    dtypes = {g.dtype for g in grads}
    if not dtypes <= _DTYPES.keys() or not all(map(torch.Tensor.is_contiguous, grads)) or set(map(torch.Tensor.get_device, grads)) - {device.index} or \
            device.type != "cuda":
        raise AssertionError(f"grads: f32, bf16 or f16, contiguous, on one GPU ({device})")
    return _DTYPES[dtypes.pop()] if len(dtypes) == 1 else [_DTYPES[g.dtype] for g in grads], list(map(torch.Tensor.data_ptr, grads))


def pacer_grad_norm(grads) -> torch.Tensor:
    """The global 2-norm of a list of gradients (f32, bf16 or f16, contiguous, on one GPU) as an f32 scalar on the device, summed in 64
    bits; infinite where a gradient is infinite or NaN.  Nothing is read back."""
    grads = list(grads)
    if not grads:
        raise AssertionError("grads: at least one")
    dev, n = grads[0].device, len(grads)
    types, at = _gradients(grads, dev)
    rows = array.array("q", bytes(24 * n))                                       # pacer_gradient: address, size, type
    rows[0::3], rows[1::3] = array.array("q", at), array.array("q", map(torch.Tensor.numel, grads))
    rows[2::3] = array.array("q", types if isinstance(types, list) else (types,) * n)
    nbytes = _lib.pacer_grad_norm_scratch_bytes(n)
    buf = torch.empty(nbytes // 4 + 2, dtype=torch.float32, device=dev)          # the result, then the scratch
    out = buf.data_ptr()
    _call(_lib.pacer_grad_norm, buf, rows.buffer_info()[0], n, out, out + 8, nbytes)
    return buf.select(0, 0)


def pacer_adamw(tensors, grads, *args, **more):
    """An AdamW step over all of `tensors`, in place, in one launch for up to 480 of them.  Called as

        pacer_adamw(tensors, grads, step, lr, betas=(0.9, 0.999), eps=1e-8, weight_decay=0.01, seed=None, norm=None, max_norm=0.0)
        pacer_adamw(params, grads, exp_avg, exp_avg_sq, step, lr, betas=(0.9, 0.999), eps=1e-8, weight_decay=0.01, scales=None, copies=None,
                    seed=None, norm=None, max_norm=0.0, roots=True)

    with AdamwTensors, or with lists of tensors as AdamwTensors takes them, which are then checked in every call.  (As to codes of second
    moments, lists hold their roots unless roots=False, AdamwTensors hold them as they are unless roots=True.)  step (1 for the first) and lr:
    numbers, or int32 and f32 scalars on the device (for a call that is captured into a graph).  seed: 8-bit states and bf16 params are
    rounded at random with a hash of it, the step and the element (None: to nearest).  norm: the gradients' global norm
    (pacer_grad_norm); they are scaled to at most max_norm (0: not at all), and where it is not finite nothing is changed.  max_norm
    takes a norm: without one AdamwTensors are refused, lists stepped without scaling."""
    return (_adamw if isinstance(tensors, AdamwTensors) else _adamw_lists)(tensors, grads, *args, **more)


def _adamw(tensors, grads, step, lr, betas=(0.9, 0.999), eps=1e-8, weight_decay=0.01, seed=None, norm=None, max_norm=0.0):
    if tensors.numel or len(grads):
        _step(tensors, tensors.with_grads(grads), len(tensors.numel), tensors.state_bits, step, lr, betas, eps, weight_decay, seed, norm, max_norm)
        torch.autograd.graph.increment_version(tensors.changed)         # (as _written)


def _adamw_lists(params, grads, exp_avg, exp_avg_sq, step, lr, betas=(0.9, 0.999), eps=1e-8, weight_decay=0.01, scales=None, copies=None, seed=None,
                 norm=None, max_norm=0.0, roots=True):
    tensors = params, copies, exp_avg, exp_avg_sq, scales = tuple(None if x is None else list(x) for x in (params, copies, exp_avg, exp_avg_sq, scales))
    grads, n = list(grads), len(params)
    states = _Lists(params, list(map(torch.Tensor.numel, params)))
    _check_adamw(tensors, states.numel, states.device)
    if not n and not grads:
        return
    if list(map(torch.Tensor.numel, grads)) != states.numel:
        raise AssertionError("grads: one for each param, of its size")
    types, at = _gradients(grads, states.device)
    states.put(2, at)
    for col, x in ((0, params), (3, exp_avg), (4, exp_avg_sq), (5, scales)):
        if x is not None:
            states.put(col, map(torch.Tensor.data_ptr, x))
    if copies is not None:
        states.put(1, (0 if c is None else c.data_ptr() for c in copies))
    code = 1 << 48 if roots and scales is not None else 0
    states.put(7, (_DTYPES[p.dtype] | t << 32 | code for p, t in zip(params, types if isinstance(types, list) else (types,) * n)))
    _step(states, states.address, n, 32 if scales is None else 8, step, lr, betas, eps, weight_decay, seed, norm, 0.0 if norm is None else max_norm)
    _written(*(t for x in tensors if x is not None for t in x))


def _step(like, table, n, bits, step, lr, betas, eps, weight_decay, seed, norm, max_norm):
    cfg = AdamwCfg(beta_one=betas[0], beta_two=betas[1], eps=eps, weight_decay=weight_decay, max_norm=max_norm, state_bits=bits,
                   seeded=seed is not None, seed=0 if seed is None else seed & ((1 << 64) - 1))
    for name, x, dtype in (("step", step, torch.int32), ("lr", lr, torch.float32)):
        if torch.is_tensor(x):
            assert x.dtype == dtype and x.numel() == 1 and x.device == like.device, f"{name}: one {dtype} on {like.device}"
            setattr(cfg, name + "_device", x.data_ptr())
        else:
            setattr(cfg, name, x)
    if norm is not None:
        assert norm.dtype == torch.float32 and norm.numel() == 1 and norm.device == like.device, f"norm: one torch.float32 on {like.device}"
        cfg.norm = norm.data_ptr()
    _call(_lib.pacer_adamw, like, table, n, C.byref(cfg))


class _Lists:
    """A table of pacer_adamw_tensor for one call, columns as AdamwTensors has them."""

    def __init__(self, like, numel):
        self.device, self.numel = like[0].device if like else None, numel
        self.rows = array.array("q", bytes(64 * len(numel)))
        self.address = self.rows.buffer_info()[0]
        self.put(6, numel)

    def put(self, col, x):
        self.rows[col::8] = array.array("q", x)


def pacer_adamw_states(tensors, *args, **more):
    """What 8-bit states stand for: (exp_avg, exp_avg_sq), lists of f32 tensors of the params' sizes, or written to `out` (two lists;
    contiguous, of those sizes).  Called as

        pacer_adamw_states(tensors, out=None)
        pacer_adamw_states(exp_avg, exp_avg_sq, scales, out=None, roots=True)

    with AdamwTensors or with lists (see pacer_adamw)."""
    return (_adamw_states if isinstance(tensors, AdamwTensors) else _adamw_states_lists)(tensors, *args, **more)


def _adamw_states_lists(exp_avg, exp_avg_sq, scales, out=None, roots=True):
    exp_avg, exp_avg_sq, scales = list(exp_avg), list(exp_avg_sq), list(scales)
    if not len(exp_avg) == len(exp_avg_sq) == len(scales):
        raise AssertionError("exp_avg, exp_avg_sq, scales: lists of one length")
    states = _Lists(exp_avg, list(map(torch.Tensor.numel, exp_avg)))
    for i, (m, v, x, n) in enumerate(zip(exp_avg, exp_avg_sq, scales, states.numel)):
        if not (m.dtype == v.dtype == torch.uint8 and v.numel() == n and x.dtype == torch.float32 and x.shape == (-(-n // 256), 2)):
            raise AssertionError(f"states {i}: torch.uint8 of one size, scales torch.float32 [{-(-n // 256)}][2]")
        if not all(t.is_cuda and t.device == states.device and t.is_contiguous() for t in (m, v, x)):
            raise AssertionError(f"states {i}: contiguous, on one GPU ({states.device})")
    for col, x in ((3, exp_avg), (4, exp_avg_sq), (5, scales)):
        states.put(col, map(torch.Tensor.data_ptr, x))
    states.put(7, [1 << 48 if roots else 0] * len(exp_avg))
    return _read_states(states, states.address, exp_avg, out)


def _adamw_states(tensors, out=None):
    assert tensors.state_bits == 8, "8-bit states"
    if tensors.numel:
        tensors._place()
    return _read_states(tensors, tensors._address, tensors.tensors[0], out)


def _read_states(states, table, like, out):
    if out is None:
        out = tuple([torch.empty(p.shape, dtype=torch.float32, device=p.device) for p in like] for _ in range(2))
    for x in out:
        if len(x) != len(states.numel):
            raise AssertionError("out: one for each param")
        for t, n in zip(x, states.numel):
            if t.dtype != torch.float32 or t.numel() != n or not t.is_contiguous() or t.device != states.device:
                raise AssertionError(f"out: f32 of the params' sizes, contiguous, on {states.device}")
    if states.numel:
        m, v = (np.array([t.data_ptr() for t in x], dtype=np.int64) for x in out)
        _call(_lib.pacer_adamw_states, states, table, len(m), m.ctypes.data, v.ctypes.data)
        _written(*out[0], *out[1])
    return out


def load_pair(ctx: Context, pair: dict):
    """Registers the three models of a synthetic pair (tensors already on the context's device)."""
    ctx.pacer_load_weights(PACER_TARGET, pair["target"], pair["succ_T"])
    ctx.pacer_load_weights(PACER_DRAFT, pair["draft"], pair["succ_D"])
    ctx.pacer_load_weights(PACER_PREVERIFY, pair["preverify"])
