"""ctypes binding of libkforcing.so (include/kforcing.h).

`lib()` returns the loaded library with typed signatures for every kf_*
entry point (same names as the C ABI).  `KForcing` wraps one context: it
allocates the state buffer with torch on a CUDA (HIP) device, passes device
pointers and the current stream, and turns error codes into KfError.  No
computation happens here.  If the shared library is missing the import of
`lib()` fails loudly: there is no CPU fallback.
"""
from __future__ import annotations

import contextlib
import ctypes
import os
from typing import NamedTuple, Optional

_PKG = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_PKG, "libkforcing.so")

KF_OK, KF_EINVAL, KF_ESTATE, KF_ECTX, KF_ENOMEM, KF_EHIP = 0, -1, -2, -3, -4, -5
KF_FP32, KF_BF16, KF_FP16 = 0, 1, 2
KF_FLAG_DEBUG_LOGITS = 1
KF_FLAG_TEMPERATURE = 2
KF_FLAG_TEACHER = 4
KF_FLAG_ROLLOUT = 8
KF_FLAG_RMS_ROPE = 16
KF_FLAG_SERVING = 32
KF_PAGE = 128  # positions per KV page
KF_MASK_SINGLE, KF_MASK_DOUBLE = 0, 1
KF_NORM_LAYER, KF_NORM_RMS = 0, 1
KF_MAX_TOP = 64
KF_KC_NAMES = ["embed", "noise", "norm", "qkv", "attn", "oproj", "mlp_up", "mlp_down", "head",
               "select"]
KF_TIMING_ALL = (1 << len(KF_KC_NAMES)) - 1

_lib = None


class KfConfig(ctypes.Structure):
    _fields_ = [
        ("n_layer", ctypes.c_int), ("d_model", ctypes.c_int), ("n_head", ctypes.c_int),
        ("d_mlp", ctypes.c_int), ("vocab", ctypes.c_int), ("n_ctx", ctypes.c_int),
        ("dtype", ctypes.c_int), ("max_batch", ctypes.c_int), ("max_k", ctypes.c_int),
        ("max_prompt", ctypes.c_int), ("flags", ctypes.c_uint), ("kv_pages", ctypes.c_int),
    ]


class KfGrad(ctypes.Structure):
    _fields_ = [("src", ctypes.c_void_p), ("dst", ctypes.c_void_p), ("n", ctypes.c_int64),
                ("src_dtype", ctypes.c_int), ("dst_dtype", ctypes.c_int)]


class KfGradPlan(ctypes.Structure):
    _fields_ = [("dev", ctypes.c_void_p), ("chunks", ctypes.c_int64), ("has_dst", ctypes.c_int)]


class KfError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"kforcing error {code}: {msg}")
        self.code = code


def lib_path() -> str:
    return _LIB_PATH


def lib():
    """Load libkforcing.so and declare every entry point of include/kforcing.h."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(_LIB_PATH):
        raise ImportError(f"{_LIB_PATH} is missing: build it with "
                          "`python -m paper_2606_10820_amd.build` (there is no CPU fallback)")
    L = ctypes.CDLL(_LIB_PATH)
    P, I, U64, SZ = ctypes.c_void_p, ctypes.c_int, ctypes.c_uint64, ctypes.c_size_t
    I64, F = ctypes.c_int64, ctypes.c_float
    CP = ctypes.POINTER(KfConfig)
    IP = ctypes.POINTER(ctypes.c_int)
    sigs = {
        "kf_create": (I, [CP, P, ctypes.POINTER(P)]),
        "kf_state_bytes": (SZ, [CP]),
        "kf_bind_state": (I, [P, P, SZ]),
        "kf_load_weights": (I, [P, P, SZ, I]),
        "kf_prefill": (I, [P, I, I, P, I, P, P]),
        "kf_decode_block": (I, [P, I, I, P, P]),
        "kf_decode_block_noalloc": (I, [P, I, I, P, P]),
        "kf_generate": (I, [P, I, I, P, I, I, U64, P]),
        "kf_prefill_ar": (I, [P, I, I, P, P, P]),
        "kf_decode_ar": (I, [P, I, P, P]),
        "kf_generate_ar": (I, [P, I, I, P, I, U64, P]),
        "kf_debug_logits": (I, [P, P, SZ]),
        "kf_fill_noise": (I, [P, U64, I, I, I, P]),
        "kf_set_temperature": (I, [P, P, I]),
        "kf_teacher_targets": (I, [P, I, I, P, P, P, P]),
        "kf_selfforcing_targets": (I, [P, I, I, I, P, P, P, P, P]),
        "kf_get_state": (I, [P, IP, IP, IP]),
        "kf_device_errors": (I, [P, IP]),
        "kf_set_graphs": (I, [P, I]),
        "kf_set_timing": (I, [P, I]),
        "kf_kernel_time": (I, [P, I, ctypes.POINTER(ctypes.c_double), IP]),
        "kf_destroy": (None, [P]),
        "kf_last_error": (ctypes.c_char_p, [P]),
        "kf_strerror": (ctypes.c_char_p, [I]),
        "kf_training_attention": (I, [P, I, I, I, I, I, I, P, P, P, P, ctypes.c_float]),
        "kf_training_attention_lse": (I, [P, I, I, I, I, I, I, P, P, P, P, P, F]),
        "kf_training_attention_backward_bytes": (SZ, [I, I, I, I, I, I]),
        "kf_training_attention_backward": (I, [P, I, I, I, I, I, I] + [P] * 9 + [F, P, SZ]),
        "kf_layer_norm": (I, [P, I, I, I, I64, I, P, I64, P, P, F, P, I64, P]),
        "kf_layer_norm_backward_bytes": (SZ, [I64, I]),
        "kf_layer_norm_backward": (I, [P, I, I, I, I64, I, P, I64, P, P, P, I64, P, I64, P, I64,
                                       P, P, P, SZ]),
        "kf_token_logprobs": (I, [P, I, I64, I, P, I64, P, I, P, P, P, P, P]),
        "kf_token_logprobs_backward": (I, [P, I, I64, I, P, I64, P, P, P, P, P, P, P, I64]),
        "kf_grad_plan_bytes": (SZ, [I, P]),
        "kf_grad_plan_init": (I, [P, I, P, P, SZ, ctypes.POINTER(KfGradPlan)]),
        "kf_grad_norm": (I, [P, ctypes.POINTER(KfGradPlan), P]),
        "kf_grad_clip": (I, [P, ctypes.POINTER(KfGradPlan), F, P]),
        "kf_serve_admit": (I, [P, I, P, I, P, I, P, P]),
        "kf_serve_step": (I, [P, I, P, I, P, P]),
        "kf_serve_release": (I, [P, I, P]),
        "kf_serve_state": (I, [P, I, IP, IP, IP]),
        "kf_serve_pages": (I, [P, IP, IP]),
    }
    for name, (res, args) in sigs.items():
        f = getattr(L, name)
        f.restype = res
        f.argtypes = args
    _lib = L
    return L


def make_config(n_layer, d_model, n_head, d_mlp, vocab, n_ctx, dtype, max_batch, max_k,
                max_prompt, flags=0, kv_pages=0) -> KfConfig:
    return KfConfig(n_layer, d_model, n_head, d_mlp, vocab, n_ctx, dtype, max_batch, max_k,
                    max_prompt, flags, kv_pages)


class KForcing:
    """One library context with its device state buffer (allocated by torch)."""

    def __init__(self, cfg: KfConfig, device: str = "cuda:0", stream=None):
        import torch
        self.torch = torch
        self.L = lib()
        self.cfg = cfg
        self.device = torch.device(device)
        self.stream = stream if stream is not None else torch.cuda.current_stream(self.device)
        h = ctypes.c_void_p()
        rc = self.L.kf_create(ctypes.byref(cfg), ctypes.c_void_p(self.stream.cuda_stream),
                              ctypes.byref(h))
        if rc != KF_OK:
            raise KfError(rc, "kf_create rejected the configuration")
        self.h = h
        nbytes = self.L.kf_state_bytes(ctypes.byref(cfg))
        self.state = torch.empty(nbytes + 256, dtype=torch.uint8, device=self.device)
        base = self.state.data_ptr()
        aligned = (base + 255) // 256 * 256
        self._check(self.L.kf_bind_state(self.h, ctypes.c_void_p(aligned), nbytes))

    # -- plumbing -------------------------------------------------------
    def _check(self, rc: int):
        if rc != KF_OK:
            raise KfError(rc, self.L.kf_last_error(self.h).decode())

    @staticmethod
    def _p(t) -> ctypes.c_void_p:
        return ctypes.c_void_p(t.data_ptr()) if t is not None else ctypes.c_void_p(0)

    def _i32(self, x):
        return self.torch.as_tensor(x, dtype=self.torch.int32, device=self.device).contiguous()

    def _f32(self, x):
        return self.torch.as_tensor(x, dtype=self.torch.float32, device=self.device).contiguous()

    def close(self):
        if getattr(self, "h", None):
            self.L.kf_destroy(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # -- entry points ----------------------------------------------------
    def load_weights(self, blob, on_device: bool = True):
        """blob: numpy float32 array (header + tensors), copied as given."""
        import numpy as np
        arr = np.ascontiguousarray(blob, dtype=np.float32)
        if on_device:
            t = self.torch.from_numpy(arr).to(self.device)
            self._check(self.L.kf_load_weights(self.h, self._p(t), arr.nbytes, 1))
            self.torch.cuda.synchronize(self.device)
        else:
            self._check(self.L.kf_load_weights(self.h, ctypes.c_void_p(arr.ctypes.data),
                                               arr.nbytes, 0))

    def prefill(self, prompt, k: int, noise, out=None):
        prompt = self._i32(prompt)
        noise = self._f32(noise)
        B, N = prompt.shape
        if out is None:
            out = self.torch.empty((B, k), dtype=self.torch.int32, device=self.device)
        self._check(self.L.kf_prefill(self.h, B, N, self._p(prompt), k, self._p(noise),
                                      self._p(out)))
        return out

    def decode_block(self, noise, out=None):
        noise = self._f32(noise)
        B, k = noise.shape
        if out is None:
            out = self.torch.empty((B, k), dtype=self.torch.int32, device=self.device)
        self._check(self.L.kf_decode_block(self.h, B, k, self._p(noise), self._p(out)))
        return out

    def decode_block_noalloc(self, noise, out=None):
        """kf_decode_block with the step's partial results in the library's
        device scratch (no allocation inside the call)."""
        noise = self._f32(noise)
        B, k = noise.shape
        if out is None:
            out = self.torch.empty((B, k), dtype=self.torch.int32, device=self.device)
        self._check(self.L.kf_decode_block_noalloc(self.h, B, k, self._p(noise), self._p(out)))
        return out

    def generate(self, prompt, L: int, k: int, seed: int, out=None):
        prompt = self._i32(prompt)
        B, N = prompt.shape
        if out is None:
            out = self.torch.empty((B, L), dtype=self.torch.int32, device=self.device)
        self._check(self.L.kf_generate(self.h, B, N, self._p(prompt), L, k, seed, self._p(out)))
        return out

    def prefill_ar(self, prompt, u, out=None):
        prompt = self._i32(prompt)
        u = self._f32(u)
        B, N = prompt.shape
        if out is None:
            out = self.torch.empty((B,), dtype=self.torch.int32, device=self.device)
        self._check(self.L.kf_prefill_ar(self.h, B, N, self._p(prompt), self._p(u), self._p(out)))
        return out

    def decode_ar(self, u, out=None):
        u = self._f32(u)
        B = u.shape[0]
        if out is None:
            out = self.torch.empty((B,), dtype=self.torch.int32, device=self.device)
        self._check(self.L.kf_decode_ar(self.h, B, self._p(u), self._p(out)))
        return out

    def generate_ar(self, prompt, L: int, seed: int, out=None):
        prompt = self._i32(prompt)
        B, N = prompt.shape
        if out is None:
            out = self.torch.empty((B, L), dtype=self.torch.int32, device=self.device)
        self._check(self.L.kf_generate_ar(self.h, B, N, self._p(prompt), L, seed, self._p(out)))
        return out

    def debug_logits(self, rows: int):
        out = self.torch.empty((rows, self.cfg.vocab), dtype=self.torch.float32,
                               device=self.device)
        self._check(self.L.kf_debug_logits(self.h, self._p(out), out.numel()))
        return out

    def set_temperature(self, tau):
        """Per-sequence temperatures tau [B] (temperature-conditioned models)."""
        t = self._f32(tau).reshape(-1)
        self._check(self.L.kf_set_temperature(self.h, self._p(t), int(t.numel())))
        self.torch.cuda.synchronize(self.device)  # t is read during the call's kernels

    def teacher_targets(self, tokens, tau, u, out=None):
        """Stage-1 teacher targets: tokens [B][N] int32, tau [B], u [B][N]
        (device tensors or array-likes); returns targets [B][N] int32."""
        tk = self._i32(tokens)
        B, N = tk.shape
        t = self._f32(tau).reshape(-1)
        uu = self._f32(u).reshape(B, N)
        if out is None:
            out = self.torch.empty((B, N), dtype=self.torch.int32, device=self.device)
        self._check(self.L.kf_teacher_targets(self.h, B, N, self._p(tk), self._p(t), self._p(uu),
                                              self._p(out)))
        self.torch.cuda.synchronize(self.device)  # the inputs may be temporaries
        return out

    def selfforcing_targets(self, tokens, k: int, z1, z2):
        """Stage-2 teacher rollout: tokens [B][N], z1/z2 [B][N][k]; returns (x1, x2),
        each int32 [B][N][k]."""
        tk = self._i32(tokens)
        B, N = tk.shape
        a = self._f32(z1).reshape(B, N, k)
        b = self._f32(z2).reshape(B, N, k)
        x1 = self.torch.empty((B, N, k), dtype=self.torch.int32, device=self.device)
        x2 = self.torch.empty((B, N, k), dtype=self.torch.int32, device=self.device)
        self._check(self.L.kf_selfforcing_targets(self.h, B, N, k, self._p(tk), self._p(a),
                                                  self._p(b), self._p(x1), self._p(x2)))
        self.torch.cuda.synchronize(self.device)  # the inputs may be temporaries
        return x1, x2

    # -- continuous batching (KF_FLAG_SERVING) ---------------------------
    @staticmethod
    def _slots(slots):
        import numpy as np
        arr = np.ascontiguousarray(slots, dtype=np.int32)
        return arr, ctypes.c_void_p(arr.ctypes.data)

    def serve_admit(self, slots, prompts, k: int, noise, out=None):
        """Start len(slots) sequences: prompts [n][N], noise [n][k] -> out [n][k]."""
        arr, sp = self._slots(slots)
        prompts = self._i32(prompts).reshape(len(arr), -1)
        noise = self._f32(noise)
        n, N = prompts.shape
        if out is None:
            out = self.torch.empty((n, k), dtype=self.torch.int32, device=self.device)
        self._check(self.L.kf_serve_admit(self.h, n, sp, N, self._p(prompts), k, self._p(noise),
                                          self._p(out)))
        return out

    def serve_step(self, slots, noise, out=None):
        """One decode block for the listed slots: noise [n][k] -> out [n][k]."""
        arr, sp = self._slots(slots)
        noise = self._f32(noise)
        n, k = noise.shape
        if out is None:
            out = self.torch.empty((n, k), dtype=self.torch.int32, device=self.device)
        self._check(self.L.kf_serve_step(self.h, n, sp, k, self._p(noise), self._p(out)))
        return out

    def serve_release(self, slots):
        arr, sp = self._slots(slots)
        self._check(self.L.kf_serve_release(self.h, len(arr), sp))

    def serve_state(self, slot: int):
        C, p, g = ctypes.c_int(), ctypes.c_int(), ctypes.c_int()
        self._check(self.L.kf_serve_state(self.h, slot, ctypes.byref(C), ctypes.byref(p),
                                          ctypes.byref(g)))
        return C.value, p.value, g.value

    def serve_pages(self):
        f, t = ctypes.c_int(), ctypes.c_int()
        self._check(self.L.kf_serve_pages(self.h, ctypes.byref(f), ctypes.byref(t)))
        return f.value, t.value

    def fill_noise(self, seed: int, B: int, p0: int, n: int):
        out = self.torch.empty((B, n), dtype=self.torch.float32, device=self.device)
        self._check(self.L.kf_fill_noise(self.h, seed, B, p0, n, self._p(out)))
        return out

    def get_state(self):
        C, p, B = ctypes.c_int(), ctypes.c_int(), ctypes.c_int()
        self._check(self.L.kf_get_state(self.h, ctypes.byref(C), ctypes.byref(p), ctypes.byref(B)))
        return C.value, p.value, B.value

    def device_errors(self) -> int:
        f = ctypes.c_int()
        self._check(self.L.kf_device_errors(self.h, ctypes.byref(f)))
        return f.value

    def set_graphs(self, enable: bool):
        self._check(self.L.kf_set_graphs(self.h, int(enable)))

    def set_timing(self, class_mask: int = KF_TIMING_ALL):
        """Bracket launches of the selected kernel classes (bit mask) with HIP events."""
        self._check(self.L.kf_set_timing(self.h, int(class_mask)))

    def kernel_time(self, cls: int):
        ms, n = ctypes.c_double(), ctypes.c_int()
        self._check(self.L.kf_kernel_time(self.h, cls, ctypes.byref(ms), ctypes.byref(n)))
        return ms.value, n.value


def training_attention_shapes(mask: int, N: int, k: int):
    """(query rows, keys) of one sequence under a training mask."""
    if mask == KF_MASK_SINGLE:
        return N + N * k, N + N * k
    return 2 * N * k, N + 2 * N * k


def training_attention_entries(mask: int, N: int, k: int) -> int:
    """Visible (query, key) pairs of one sequence under a training mask: the
    algorithmic work (4 * d_head flops each) of kf_training_attention."""
    ctx = N * (N + 1) // 2                      # context rows, causal
    noise = k * N * (N + 1) // 2 + N * k * (k + 1) // 2   # staircase + in-group causal
    if mask == KF_MASK_SINGLE:
        return ctx + noise
    # Future-1 rows as the noise rows above; Future-2 rows add all k Future-1 keys
    return 2 * noise + N * k * k


def training_attention(mask: int, q, k_, v, N: int, k: int, scale: Optional[float] = None,
                       out=None, stream=None):
    """Attention of the training masks (kf_training_attention).

    q [B][H][rows][dh], k_/v [B][H][keys][dh]: contiguous bf16 device tensors.
    Returns out (allocated like q when None).  The call is asynchronous on
    `stream` (default: torch's current stream)."""
    import torch
    B, H, rows, dh = q.shape
    if (rows, k_.shape[2]) != training_attention_shapes(mask, N, k):
        raise ValueError("q/k rows do not match the mask's layout")
    for t in (q, k_, v):
        if t.dtype != torch.bfloat16 or not t.is_contiguous() or not t.is_cuda:
            raise ValueError("q, k, v must be contiguous bf16 device tensors")
    if k_.shape != v.shape or k_.shape[:2] != (B, H) or k_.shape[3] != dh:
        raise ValueError("k and v must be [B][H][keys][dh] like q")
    if out is None:
        out = torch.empty_like(q)
    if scale is None:
        scale = dh ** -0.5
    s = stream if stream is not None else torch.cuda.current_stream(q.device)
    rc = lib().kf_training_attention(
        ctypes.c_void_p(s.cuda_stream), mask, B, H, N, k, dh, ctypes.c_void_p(q.data_ptr()),
        ctypes.c_void_p(k_.data_ptr()), ctypes.c_void_p(v.data_ptr()),
        ctypes.c_void_p(out.data_ptr()), float(scale))
    if rc != KF_OK:
        raise KfError(rc, lib().kf_strerror(rc).decode())
    return out


# ------------------------------------------------ operators of the training step
# Each call runs on `stream` (default: torch's current stream of the tensors'
# device) and allocates its results there.  The calls are no part of autograd:
# their results carry no graph, also where an argument requires gradients, and
# the *_backward functions are called by the training loop itself.

_NOTHING = contextlib.nullcontext()


def _ok(rc: int):
    if rc != KF_OK:
        raise KfError(rc, lib().kf_strerror(rc).decode())


def _ptr(t):
    return t.data_ptr() if t is not None else None


_current_raw = _current_device = None  # torch's, looked up on the first call


def _on(device, stream, used):
    """(raw stream, context to allocate and launch in) for tensors on `device`; the
    caching allocator learns which tensors another stream uses."""
    global _current_raw, _current_device
    if device.type != "cuda":
        raise ValueError("tensors must be on a GPU")
    if stream is not None and stream.device != device:  # (every device's default stream has handle 0)
        raise ValueError("the stream is another device's")
    import torch
    if _current_device is None:
        _current_device = torch.cuda.current_device
        # the stream's handle without a Stream object (2 us a call), where torch has it
        _current_raw = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (
            lambda i: torch.cuda.current_stream(i).cuda_stream)
    raw = _current_raw(device.index)
    if stream is not None and stream.cuda_stream != raw:
        for t in used:
            if t is not None:
                t.record_stream(stream)
        return stream.cuda_stream, torch.cuda.stream(stream)
    if _current_device() == device.index:
        return raw, _NOTHING
    return raw, torch.cuda.device(device)


_CODES = {"torch.float32": KF_FP32, "torch.bfloat16": KF_BF16, "torch.float16": KF_FP16}
_type_codes = {}  # the same by torch.dtype


def _type(t, what: str) -> int:
    code = _type_codes.get(t)
    if code is None:
        code = _CODES.get(str(t))
        if code is None:
            raise ValueError(f"{what} must be float32, bfloat16 or float16")
        _type_codes[t] = code
    return code


def _rows(t, what: str, shape=None):
    """(rows, ld) of t [..., d] seen as rows of d consecutive elements."""
    if t.dim() < 1:
        raise ValueError(f"{what} must have at least one dimension")
    if shape is not None and t.shape != shape:
        raise ValueError(f"{what} must have shape {tuple(shape)}")
    d = t.shape[-1]
    if t.dim() != 2:
        try:
            t = t.view(-1, d) if t.numel() else t.new_empty((0, d))
        except RuntimeError:
            raise ValueError(f"{what}'s rows must be evenly spaced") from None
    if d > 1 and t.stride(1) != 1 and t.numel():
        raise ValueError(f"{what}'s last dimension must be contiguous")
    return t.shape[0], (t.stride(0) if t.shape[0] > 1 else d)


def _check(t, what: str, device, dtype, n: int):
    """t (or None) holds n consecutive elements of dtype on device."""
    if t is not None and (t.device != device or t.dtype != dtype or t.numel() != n
                          or not t.is_contiguous()):
        raise ValueError(f"{what} must be {n} contiguous {dtype} elements on {device}")


def _attention_args(mask, q, k_, v, N, k, *more):
    import torch
    B, H, rows, dh = q.shape
    if (rows, k_.shape[2]) != training_attention_shapes(mask, N, k):
        raise ValueError("q/k rows do not match the mask's layout")
    if k_.shape != v.shape or k_.shape[:2] != (B, H) or k_.shape[3] != dh:
        raise ValueError("k and v must be [B][H][keys][dh] like q")
    for t in (q, k_, v, *more):
        if t.dtype != torch.bfloat16 or not t.is_contiguous() or t.device != q.device:
            raise ValueError("tensors must be contiguous bf16 on one device")
    for t in more:
        if t.shape != q.shape:
            raise ValueError("out and dout must have q's shape")
    return B, H, rows, dh


def training_attention_lse(mask: int, q, k_, v, N: int, k: int, scale: Optional[float] = None,
                           stream=None):
    """training_attention that also returns each query row's log of the sum of exponentials,
    (out, lse [B][H][rows] fp32), for training_attention_backward (no autograd graph)."""
    import torch
    B, H, rows, dh = _attention_args(mask, q, k_, v, N, k)
    s, ctx = _on(q.device, stream, (q, k_, v))
    with ctx:
        out = torch.empty_like(q)
        lse = torch.empty((B, H, rows), dtype=torch.float32, device=q.device)
        _ok(lib().kf_training_attention_lse(s, mask, B, H, N, k, dh, q.data_ptr(), k_.data_ptr(),
                                            v.data_ptr(), out.data_ptr(), lse.data_ptr(),
                                            dh ** -0.5 if scale is None else scale))
    return out, lse


def training_attention_backward(mask: int, q, k_, v, out, lse, dout, N: int, k: int,
                                scale: Optional[float] = None, stream=None):
    """Gradients (dq, dk, dv) of training_attention from the gradient dout of its output, with
    out and lse of training_attention_lse (kf_training_attention_backward)."""
    import torch
    B, H, rows, dh = _attention_args(mask, q, k_, v, N, k, out, dout)
    _check(lse, "lse", q.device, torch.float32, B * H * rows)
    s, ctx = _on(q.device, stream, (q, k_, v, out, lse, dout))
    with ctx:
        dq, dk, dv = torch.empty_like(q), torch.empty_like(k_), torch.empty_like(v)
        n = lib().kf_training_attention_backward_bytes(mask, B, H, N, k, dh)
        ws = torch.empty(n, dtype=torch.uint8, device=q.device)
        _ok(lib().kf_training_attention_backward(
            s, mask, B, H, N, k, dh, q.data_ptr(), k_.data_ptr(), v.data_ptr(), out.data_ptr(),
            lse.data_ptr(), dout.data_ptr(), dq.data_ptr(), dk.data_ptr(), dv.data_ptr(),
            dh ** -0.5 if scale is None else scale, ws.data_ptr(), n))
    return dq, dk, dv


def layer_norm(x, gain, shift=None, eps: float = 1e-5, rms: bool = False, out_dtype=None,
               out=None, stream=None):
    """LayerNorm (or with rms RMSNorm) of the rows of x [..., d] (kf_layer_norm).

    gain, shift [d] fp32.  Returns (y, stats): y like x in out_dtype (default x's;
    another only for fp32 x), stats [rows][2] fp32 for layer_norm_backward (no autograd
    graph)."""
    import torch
    rows, ldx = _rows(x, "x")
    d, dev = x.shape[-1], x.device
    _check(gain, "gain", dev, torch.float32, d)
    _check(shift, "shift", dev, torch.float32, d)
    s, ctx = _on(dev, stream, (x, gain, shift, out))
    with ctx:
        if out is None:
            y, ldy = torch.empty(x.shape, dtype=out_dtype or x.dtype, device=dev), d
        else:
            y, (_, ldy) = out, _rows(out, "out", x.shape)
            if y.device != dev or (out_dtype or y.dtype) != y.dtype:
                raise ValueError("out must be on x's device and of out_dtype")
        stats = torch.empty((rows, 2), dtype=torch.float32, device=dev)
        _ok(lib().kf_layer_norm(s, KF_NORM_RMS if rms else KF_NORM_LAYER, _type(x.dtype, "x"),
                                _type(y.dtype, "out"), rows, d, x.data_ptr(), ldx, _ptr(gain),
                                _ptr(shift), eps, y.data_ptr(), ldy, stats.data_ptr()))
    return y, stats


def layer_norm_backward(dy, x, gain, stats, rms: bool = False, dres=None, stream=None):
    """Gradients of layer_norm (kf_layer_norm_backward): (dx, dgain, dshift), dx like x,
    with dres (the gradient along the residual path, like x) added when given; dgain and
    dshift [d] fp32, dshift None with rms."""
    import torch
    rows, ldx = _rows(x, "x")
    _, lddy = _rows(dy, "dy", x.shape)
    d, dev = x.shape[-1], x.device
    lddres = d
    if dres is not None:
        _, lddres = _rows(dres, "dres", x.shape)
        if dres.dtype != x.dtype or dres.device != dev:
            raise ValueError("dres must be of x's type and device")
    if dy.device != dev:
        raise ValueError("dy must be on x's device")
    _check(gain, "gain", dev, torch.float32, d)
    _check(stats, "stats", dev, torch.float32, 2 * rows)
    s, ctx = _on(dev, stream, (dy, x, gain, stats, dres))
    with ctx:
        dx = torch.empty(x.shape, dtype=x.dtype, device=dev)
        dgain = torch.empty(d, dtype=torch.float32, device=dev)
        dshift = None if rms else torch.empty(d, dtype=torch.float32, device=dev)
        n = lib().kf_layer_norm_backward_bytes(rows, d)
        ws = torch.empty(n, dtype=torch.uint8, device=dev)
        _ok(lib().kf_layer_norm_backward(
            s, KF_NORM_RMS if rms else KF_NORM_LAYER, _type(x.dtype, "x"), _type(dy.dtype, "dy"),
            rows, d, x.data_ptr(), ldx, _ptr(gain), stats.data_ptr(), dy.data_ptr(), lddy,
            _ptr(dres), lddres, dx.data_ptr(), d, dgain.data_ptr(), _ptr(dshift), ws.data_ptr(), n))
    return dx, dgain, dshift


class TokenLogprobs(NamedTuple):
    logp: "torch.Tensor"
    entropy: "Optional[torch.Tensor]" = None
    lse: "Optional[torch.Tensor]" = None
    top_ids: "Optional[torch.Tensor]" = None
    top_logp: "Optional[torch.Tensor]" = None


def token_logprobs(logits, tokens=None, n_top: int = 0, entropy: bool = True, lse: bool = False,
                   stream=None) -> TokenLogprobs:
    """Log probabilities of tokens [...] int32 under softmax(logits [..., vocab]), with the
    rows' entropies, log-sums (lse) and n_top most probable ids (kf_token_logprobs; no
    autograd graph)."""
    import torch
    rows, ld = _rows(logits, "logits")
    lead, V, dev = logits.shape[:-1], logits.shape[-1], logits.device
    _check(tokens, "tokens", dev, torch.int32, rows)
    s, ctx = _on(dev, stream, (logits, tokens))
    with ctx:
        logp = torch.empty(lead, dtype=torch.float32, device=dev)
        H = torch.empty_like(logp) if entropy else None
        ls = torch.empty_like(logp) if lse else None
        ids = top = None
        if n_top > 0:
            ids = torch.empty((*lead, n_top), dtype=torch.int32, device=dev)
            top = torch.empty((*lead, n_top), dtype=torch.float32, device=dev)
        _ok(lib().kf_token_logprobs(s, _type(logits.dtype, "logits"), rows, V, logits.data_ptr(),
                                    ld, _ptr(tokens), n_top, logp.data_ptr(), _ptr(H), _ptr(ls),
                                    _ptr(ids), _ptr(top)))
    return TokenLogprobs(logp, H, ls, ids, top)


def token_logprobs_backward(logits, tokens, d_logp=None, d_entropy=None, out=None,
                            entropy: bool = False, lse: bool = False, stream=None):
    """Gradient of logits [..., vocab] from the gradients d_logp and d_entropy [...] fp32 of
    token_logprobs (kf_token_logprobs_backward; no forward call is needed before).  Returns
    (d_logits, TokenLogprobs); out may be logits itself."""
    import torch
    rows, ld = _rows(logits, "logits")
    lead, V, dev = logits.shape[:-1], logits.shape[-1], logits.device
    _check(tokens, "tokens", dev, torch.int32, rows)
    _check(d_logp, "d_logp", dev, torch.float32, rows)
    _check(d_entropy, "d_entropy", dev, torch.float32, rows)
    s, ctx = _on(dev, stream, (logits, tokens, d_logp, d_entropy, out))
    with ctx:
        logp = torch.empty(lead, dtype=torch.float32, device=dev)
        H = torch.empty_like(logp) if entropy else None
        ls = torch.empty_like(logp) if lse else None
        if out is None:
            out, ldd = torch.empty(logits.shape, dtype=logits.dtype, device=dev), V
        else:
            _, ldd = _rows(out, "out", logits.shape)
            if out.dtype != logits.dtype or out.device != dev:
                raise ValueError("out must be of logits' type and device")
        _ok(lib().kf_token_logprobs_backward(
            s, _type(logits.dtype, "logits"), rows, V, logits.data_ptr(), ld, _ptr(tokens),
            _ptr(d_logp), _ptr(d_entropy), logp.data_ptr(), _ptr(H), _ptr(ls), out.data_ptr(), ldd))
    return out, TokenLogprobs(logp, H, ls)


class GradClip:
    """The norm of a list of gradients as a whole, and their clipping (kf_grad_norm,
    kf_grad_clip): a plan over the tensors `grads`, which it keeps.

    out: where the scaled gradients go, a tensor for each (of its type or fp32); default the
    gradients themselves.  The plan is built on `stream` and used on one stream at a time; it
    may be dropped while calls still run, but not while a graph that captured one is in use."""

    def __init__(self, grads, out=None, stream=None):
        import torch
        self.grads = list(grads)
        self.out = self.grads if out is None else list(out)
        if len(self.out) != len(self.grads) or not self.grads:
            raise ValueError("a plan takes one or more gradients and an out for each")
        self.device = self.grads[0].device
        arr = (KfGrad * len(self.grads))()
        for i, (a, b) in enumerate(zip(self.grads, self.out)):
            if a.device != self.device or b.device != self.device or a.numel() != b.numel():
                raise ValueError("gradients and outs must match in size, on one device")
            if not a.is_contiguous() or not b.is_contiguous():
                raise ValueError("gradients and outs must be contiguous")
            arr[i] = KfGrad(a.data_ptr(), b.data_ptr(), a.numel(), _type(a.dtype, "a gradient"),
                            _type(b.dtype, "an out"))
        n = lib().kf_grad_plan_bytes(len(self.grads), arr)
        if n == 0:
            raise KfError(KF_EINVAL, "kf_grad_plan_bytes rejected the tensors")
        self.plan = KfGradPlan()
        s, ctx = _on(self.device, stream, ())
        self.stream = s  # whose memory buf is
        with ctx:
            self.buf = torch.empty(n + 256, dtype=torch.uint8, device=self.device)
            _ok(lib().kf_grad_plan_init(s, len(self.grads), arr,
                                        (self.buf.data_ptr() + 255) // 256 * 256, n,
                                        ctypes.byref(self.plan)))

    def _call(self, stream, f, *more):
        import torch
        s, ctx = _on(self.device, stream, (*self.grads, *self.out) if stream else ())
        if s != self.stream:  # buf may go back to its own stream while this one still reads it
            self.buf.record_stream(stream or torch.cuda.current_stream(self.device))
        with ctx:
            norm = torch.empty((), dtype=torch.float32, device=self.device)
            _ok(f(s, self.plan, *more, norm.data_ptr()))
        return norm

    def norm(self, stream=None):
        """The norm of all gradients, a 0-dimensional fp32 tensor."""
        return self._call(stream, lib().kf_grad_norm)

    def clip(self, max_norm: float, stream=None):
        """Scale the gradients to at most max_norm into `out`; returns the norm before."""
        return self._call(stream, lib().kf_grad_clip, max_norm)
