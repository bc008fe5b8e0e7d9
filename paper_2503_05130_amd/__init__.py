"""Python binding of libiefwd (include/iefwd.h): argument marshalling only.

Every step of the forward pass runs in the library's HIP kernels; this module
converts Python arguments to C ones and turns non-zero status codes into
``IefwdError``.  torch supplies device memory and streams (``tensor.data_ptr()``,
``torch.cuda.Stream.cuda_stream``).

torch is imported before the library is loaded so that the library binds to the
HIP runtime torch already loaded (one runtime per process).  There is no CPU
fallback: if ``libiefwd.so`` is missing, loading raises.
"""
from __future__ import annotations

import ctypes
import os

import numpy as np
import torch  # noqa: F401  (must be loaded before libiefwd.so)

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libiefwd.so")

ABI_VERSION = 1
OK, EINVAL, ENODEV, ENOMEM, EHIP, ESTATE, EVERSION = 0, -1, -2, -3, -4, -5, -6
K_QKV, K_ATTN, K_OUTPROJ, K_FFN1, K_FFN2, K_LN, K_BWD_GEMM, K_BWD, K_OPTIM = range(9)
TRAIN_MASTER, TRAIN_GRAD, TRAIN_MOMENT1, TRAIN_MOMENT2 = range(4)
EPI_BIAS_BF16, EPI_BIAS_GELU_BF16, EPI_BIAS_RESID_F32 = 0, 1, 2
KV_BF16, KV_E4M3, KV_MX4 = 0, 1, 3
BF16, F32 = 0, 1
EPI_LN_RESID_F32, EPI_F32, EPI_GELU_BWD_BF16, EPI_GELU2_BF16 = 4, 5, 6, 7

_u32, _u64, _i32, _f32, _vp, _sz = (ctypes.c_uint32, ctypes.c_uint64, ctypes.c_int, ctypes.c_float,
                                    ctypes.c_void_p, ctypes.c_size_t)

# every function the header declares, with its C signature
SIGNATURES = {
    "iefwd_config_init": (None, [_vp]),
    "iefwd_device_info": (_i32, [_i32, ctypes.POINTER(_u32), ctypes.POINTER(_u32)]),
    "iefwd_build_cu_mask": (_i32, [_u32, _u32, _u32, _u32, ctypes.POINTER(_u32), _u32]),
    "iefwd_create": (_i32, [_vp, _i32, ctypes.POINTER(_vp)]),
    "iefwd_destroy": (_i32, [_vp]),
    "iefwd_set_quota": (_i32, [_vp, _u32]),
    "iefwd_set_quota_at": (_i32, [_vp, _u32, _u32]),
    "iefwd_decode": (_i32, [_vp, _vp, _u32, _u32, _i32]),
    "iefwd_prepare_quota_at": (_i32, [_vp, _u32, _u32]),
    "iefwd_set_stream_cache": (_i32, [_vp, _u32]),
    "iefwd_kernels_launched": (_i32, [_vp, ctypes.POINTER(ctypes.c_uint64)]),
    "iefwd_ctl_params_init": (_i32, [_vp]),
    "iefwd_ctl_create": (_i32, [_vp, ctypes.POINTER(_vp)]),
    "iefwd_ctl_destroy": (_i32, [_vp]),
    "iefwd_ctl_add": (_i32, [_vp, ctypes.c_double, ctypes.c_double, ctypes.c_int, ctypes.POINTER(_u32)]),
    "iefwd_ctl_report": (_i32, [_vp, _u32, ctypes.c_uint64, ctypes.c_double]),
    "iefwd_ctl_issue": (_i32, [_vp, ctypes.POINTER(ctypes.c_double), ctypes.POINTER(_u32), ctypes.POINTER(_u32),
                                _u32]),
    "iefwd_ctl_state": (_i32, [_vp, ctypes.POINTER(ctypes.c_int32)]),
    "iefwd_set_cu_mask": (_i32, [_vp, ctypes.POINTER(_u32), _u32]),
    "iefwd_get_cu_mask": (_i32, [_vp, ctypes.POINTER(_u32), _u32]),
    "iefwd_submit": (_i32, [_vp, _vp, _u32, _u32, _i32]),
    "iefwd_wait": (_i32, [_vp]),
    "iefwd_read_logits": (_i32, [_vp, _vp, _sz, _i32]),
    "iefwd_last_batch_ms": (_i32, [_vp, ctypes.POINTER(_f32)]),
    "iefwd_get_stream": (_i32, [_vp, ctypes.POINTER(_vp)]),
    "iefwd_time_kernel": (_i32, [_vp, _u32, _i32]),
    "iefwd_kernel_time": (_i32, [_vp, _u32, ctypes.POINTER(ctypes.c_double), ctypes.POINTER(_u64)]),
    "iefwd_export_tensor": (_i32, [_vp, _u32, _u32, _vp, _sz]),
    "iefwd_train_params_init": (None, [_vp]),
    "iefwd_train_create": (_i32, [_vp, _vp, _i32, ctypes.POINTER(_vp)]),
    "iefwd_train_step": (_i32, [_vp, _vp, _vp, _u32, _u32, _i32]),
    "iefwd_train_loss": (_i32, [_vp, ctypes.POINTER(_f32)]),
    "iefwd_train_steps": (_i32, [_vp, ctypes.POINTER(_u64)]),
    "iefwd_train_export": (_i32, [_vp, _u32, _u32, _u32, _vp, _sz]),
    "iefwd_last_error": (ctypes.c_char_p, []),
    "iefwd_status_string": (ctypes.c_char_p, [_i32]),
    "iefwd_test_gemm": (_i32, [_u32, _vp, _vp, _vp, _vp, _vp, _u32, _u32, _u32, _vp]),
    "iefwd_test_gemm_on": (_i32, [_u32, _u32] + [_vp] * 10 + [_u32] * 3 + [_vp]),
    "iefwd_test_gemm_group": (_i32, [_u32, _u32] + [_vp] * 5 + [_u32] + [ctypes.POINTER(_u32)] * 2 + [_vp]),
    "iefwd_test_gemm_qkv_on": (_i32, [_u32] + [_vp] * 6 + [_u32] * 4 + [_vp]),
    "iefwd_test_gemm_plan": (_i32, [_u32, _u32, _u32, _u32, _u32, _u32, ctypes.POINTER(_u32), ctypes.POINTER(_u32),
                                     ctypes.POINTER(_u32), ctypes.POINTER(_u32)]),
    "iefwd_test_gemm_skinny": (_i32, [_u32, _vp, _vp, _vp, _vp, _vp, _u32, _u32, _u32, _vp, _vp, _vp, _f32, _vp]),
    "iefwd_test_skinny_pack": (_i32, [_vp, _vp, _u32, _u32, _u32, _vp]),
    "iefwd_test_gemm_skinny_packed": (_i32, [_u32, _vp, _vp, _u32, _vp, _vp, _vp, _u32, _u32, _u32, _vp, _vp, _vp,
                                             _f32, _vp]),
    "iefwd_test_gemm_skinny_shared": (_i32, [_u32, _vp, _vp, _u32, _vp, _vp, _vp, _u32, _u32, _u32, _vp, _vp, _vp,
                                             _f32, _vp]),
    "iefwd_test_skinny_groups": (_i32, [_u32, _u32, _u32, _i32, ctypes.POINTER(_u32)]),
    "iefwd_test_gemm_qkv": (_i32, [_vp, _vp, _vp, _vp, _vp, _vp, _u32, _u32, _u32, _u32, _vp]),
    "iefwd_test_attention": (_i32, [_vp, _vp, _vp, _vp, _u32, _u32, _u32, _u32, _i32, _vp]),
    "iefwd_test_attention_place": (_i32, [_u32, _u32, _i32, _u32, _vp, _sz]),
    "iefwd_test_layernorm": (_i32, [_vp, _vp, _vp, _vp, _vp, _u32, _u32, _f32, _vp]),
    "iefwd_test_ln_head": (_i32, [_vp, _vp, _vp, _vp, _vp, _vp, _u32, _u32, _u32, _f32, _vp]),
    "iefwd_test_cu_probe": (_i32, [_vp, _u32, _vp]),
    "iefwd_test_decode_attention": (_i32, [_vp, _vp, _vp, _vp, _u32, _u32, _u32, _u32, _u32, _u32, _vp]),
    "iefwd_paged_plan": (_i32, [_u32, _u32, _vp, _vp, _vp, _u32, _u32, _vp, _u32, _vp, _vp, _vp, _vp, _u32, _vp, _vp, _vp]),
    "iefwd_paged_append": (_i32, [_vp, _vp, _vp, _vp, _u32, _u64, _u64, _vp]),
    "iefwd_paged_attention_workspace": (_i32, [_vp, _u32, _u32, _u32, ctypes.POINTER(_sz)]),
    "iefwd_paged_attention": (_i32, [_vp, _vp, _u64, _u32, _vp, _u32, _u32, _vp, _u32, _f32, _vp, _vp, _sz, _vp]),
    "iefwd_paged_attention_scored": (_i32, [_vp, _vp, _u64, _u32, _vp, _u32, _u32, _vp, _u32, _f32, _f32, _vp, _vp, _vp, _sz, _vp]),
    "iefwd_paged_read": (_i32, [_vp, _vp, _vp, _vp, _u32, _u64, _u64, _vp]),
    "iefwd_test_paged_split": (_i32, [_u32, _u32, _u32, _u32, ctypes.POINTER(_u32)]),
    "iefwd_q4_packed_bytes": (_i32, [_u32, _u32, _u32, ctypes.POINTER(_sz)]),
    "iefwd_q4_pack": (_i32, [_vp, _vp, _vp, _vp, _u32, _u32, _u32, _vp]),
    "iefwd_q4_gemm": (_i32, [_u32, _vp, _vp, _vp, _vp, _vp, _u32, _u32, _u32, _u32, _vp]),
    "iefwd_mx4_bytes": (_i32, [_u32, _u32, ctypes.POINTER(_sz)]),
    "iefwd_mx4_quantize": (_i32, [_u32, _vp, _u64, _vp, _u32, _u32, _vp]),
    "iefwd_mx4_pack": (_i32, [_vp, _vp, _vp, _u32, _u32, _vp]),
    "iefwd_mx4_values": (_i32, [_vp, _u32, _vp, _u64, _u32, _u32, _vp]),
    "iefwd_mx4_gemm": (_i32, [_u32, _vp, _vp, _vp, _vp, _vp, _u32, _u32, _u32, _vp]),
    "iefwd_mx4_gemm_bf16": (_i32, [_u32, _vp, _vp, _vp, _vp, _vp, _u32, _u32, _u32, _vp]),
    "iefwd_token_logprobs_workspace": (_i32, [_u32, _u32, _u32, ctypes.POINTER(_sz)]),
    "iefwd_token_logprobs": (_i32, [_u32, _vp, _u64, _u32, _u32, _vp, _f32, _vp, _vp, _vp, _u32, _vp, _vp, _vp, _sz, _vp]),
    "iefwd_token_logprobs_grad": (_i32, [_u32, _vp, _u64, _u32, _u32, _vp, _f32, _vp, _vp, _vp, _vp, _vp, _u64, _vp]),
    "iefwd_decode_attention_noalloc": (_i32, [_vp, _vp, _vp, _vp, _u32, _u32, _u32, _u32, _u32, _u32, _vp]),
}


class Config(ctypes.Structure):
    """Mirror of ``iefwd_config``."""
    _fields_ = [
        ("abi_version", _u32), ("n_layers", _u32), ("d_model", _u32), ("n_heads", _u32),
        ("d_ff", _u32), ("max_batch", _u32), ("max_seq", _u32), ("n_out", _u32),
        ("pre_ln", _u32), ("causal", _u32), ("kv_cache", _u32),
        ("ln_eps", _f32), ("w_std", _f32), ("b_std", _f32), ("ln_std", _f32), ("qk_std", _f32),
        ("seed", _u64),
    ]


class IefwdError(RuntimeError):
    def __init__(self, status: int, func: str, msg: str):
        super().__init__(f"{func}: {status_string(status)} ({status}): {msg}")
        self.status = status


_lib = None


def lib() -> ctypes.CDLL:
    """The loaded library (raises if it has not been built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with `python -m paper_2503_05130_amd.build`")
        handle = ctypes.CDLL(LIB_PATH)
        for name, (res, args) in SIGNATURES.items():
            fn = getattr(handle, name)
            fn.restype = res
            fn.argtypes = args
        _lib = handle
    return _lib


def status_string(status: int) -> str:
    return lib().iefwd_status_string(status).decode()


def last_error() -> str:
    return lib().iefwd_last_error().decode()


def _check(status: int, func: str) -> None:
    if status != OK:
        raise IefwdError(status, func, last_error())


def _ptr(x) -> int | None:
    """Device/host address of a tensor or array (None stays NULL)."""
    if x is None:
        return None
    if isinstance(x, torch.Tensor):
        return x.data_ptr()
    if isinstance(x, np.ndarray):
        return x.ctypes.data
    return int(x)


def _stream(s) -> int | None:
    if s is None:
        return None
    if isinstance(s, torch.cuda.Stream):
        return s.cuda_stream
    return int(s)


# ------------------------------------------------------------------------------------ device
def device_info(device: int = 0) -> tuple[int, int]:
    n_cu, n_xcd = _u32(), _u32()
    _check(lib().iefwd_device_info(device, ctypes.byref(n_cu), ctypes.byref(n_xcd)), "iefwd_device_info")
    return n_cu.value, n_xcd.value


def build_cu_mask(n_cu: int, n_xcd: int, quota: int, first: int = 0, n_words: int | None = None) -> list[int]:
    n_words = n_words if n_words is not None else (n_cu + 31) // 32
    buf = (_u32 * n_words)()
    _check(lib().iefwd_build_cu_mask(n_cu, n_xcd, quota, first, buf, n_words), "iefwd_build_cu_mask")
    return list(buf)


def make_config(**kw) -> Config:
    cfg = Config()
    lib().iefwd_config_init(ctypes.byref(cfg))
    for k, v in kw.items():
        if not hasattr(cfg, k):
            raise KeyError(f"unknown config field {k}")
        setattr(cfg, k, v)
    return cfg


# ---------------------------------------------------------------------------------- instance
class Instance:
    """One serverless DL instance: its model, workspace and CU-masked stream."""

    def __init__(self, device: int = 0, **config):
        self._h = None
        self.cfg = make_config(**config)
        h = _vp()
        _check(lib().iefwd_create(ctypes.byref(self.cfg), device, ctypes.byref(h)), "iefwd_create")
        self._h = h
        self.device = device

    @property
    def out_width(self) -> int:
        return self.cfg.n_out if self.cfg.n_out > 0 else self.cfg.d_model

    def close(self) -> None:
        if self._h is not None:
            _check(lib().iefwd_destroy(self._h), "iefwd_destroy")
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        self.close()

    def set_quota(self, n_cu: int, first: int = 0) -> None:
        _check(lib().iefwd_set_quota_at(self._h, n_cu, first), "iefwd_set_quota_at")

    def prepare_quota(self, n_cu: int, first: int = 0) -> None:
        """Create the masked stream for (n_cu, first) ahead of time; may be called
        from another thread while this instance serves."""
        _check(lib().iefwd_prepare_quota_at(self._h, n_cu, first), "iefwd_prepare_quota_at")

    def set_stream_cache(self, capacity: int) -> None:
        """Number of masked streams (hardware queues) the instance keeps cached."""
        _check(lib().iefwd_set_stream_cache(self._h, capacity), "iefwd_set_stream_cache")

    def set_cu_mask(self, mask) -> None:
        buf = (_u32 * len(mask))(*mask)
        _check(lib().iefwd_set_cu_mask(self._h, buf, len(mask)), "iefwd_set_cu_mask")

    def get_cu_mask(self, n_words: int = 8) -> list[int]:
        buf = (_u32 * n_words)()
        _check(lib().iefwd_get_cu_mask(self._h, buf, n_words), "iefwd_get_cu_mask")
        return list(buf)

    def submit(self, x, batch: int | None = None, seq: int | None = None) -> None:
        """x: fp32 [batch, seq, d_model] -- a CUDA tensor (kept alive by the caller
        until wait/read) or a host array/tensor (copied before return)."""
        if isinstance(x, torch.Tensor):
            if x.dtype != torch.float32 or not x.is_contiguous():
                raise ValueError("x must be a contiguous float32 tensor")
            is_dev = 1 if x.is_cuda else 0
        else:
            x = np.ascontiguousarray(x, dtype=np.float32)
            is_dev = 0
        b = batch if batch is not None else x.shape[0]
        s = seq if seq is not None else x.shape[1]
        if int(np.prod(x.shape)) != b * s * self.cfg.d_model:
            raise ValueError("x does not have batch * seq * d_model elements")
        self._x_keep = x
        _check(lib().iefwd_submit(self._h, _ptr(x), b, s, is_dev), "iefwd_submit")
        self._last_shape = (b, s)

    def decode(self, x, pos: int) -> None:
        """One decode step (kv_cache instances): x fp32 [batch, d_model] -- the new
        tokens' embeddings -- appended at position `pos`."""
        if isinstance(x, torch.Tensor):
            if x.dtype != torch.float32 or not x.is_contiguous():
                raise ValueError("x must be a contiguous float32 tensor")
            is_dev = 1 if x.is_cuda else 0
        else:
            x = np.ascontiguousarray(x, dtype=np.float32)
            is_dev = 0
        b = x.shape[0]
        if int(np.prod(x.shape)) != b * self.cfg.d_model:
            raise ValueError("x does not have batch * d_model elements")
        self._x_keep = x
        _check(lib().iefwd_decode(self._h, _ptr(x), b, pos, is_dev), "iefwd_decode")
        self._last_shape = (b, 1)

    def wait(self) -> None:
        _check(lib().iefwd_wait(self._h), "iefwd_wait")

    def read_logits(self, out=None):
        """Waits and returns the last batch's output (numpy fp32 unless `out`
        -- a CUDA tensor or host array of the right size -- is given)."""
        b, s = getattr(self, "_last_shape", (0, 0))
        if out is None:
            out = np.empty((b, s, self.out_width), dtype=np.float32)
        is_dev = 1 if isinstance(out, torch.Tensor) and out.is_cuda else 0
        n = out.numel() if isinstance(out, torch.Tensor) else out.size
        _check(lib().iefwd_read_logits(self._h, _ptr(out), n, is_dev), "iefwd_read_logits")
        return out

    def last_batch_ms(self) -> float:
        v = _f32()
        _check(lib().iefwd_last_batch_ms(self._h, ctypes.byref(v)), "iefwd_last_batch_ms")
        return v.value

    def kernels_launched(self) -> int:
        v = _u64()
        _check(lib().iefwd_kernels_launched(self._h, ctypes.byref(v)), "iefwd_kernels_launched")
        return v.value

    def stream_handle(self) -> int:
        v = _vp()
        _check(lib().iefwd_get_stream(self._h, ctypes.byref(v)), "iefwd_get_stream")
        return v.value or 0

    def time_kernel(self, kind: int, enable: bool = True) -> None:
        _check(lib().iefwd_time_kernel(self._h, kind, 1 if enable else 0), "iefwd_time_kernel")

    def kernel_time(self, kind: int) -> tuple[float, int]:
        ms, n = ctypes.c_double(), _u64()
        _check(lib().iefwd_kernel_time(self._h, kind, ctypes.byref(ms), ctypes.byref(n)), "iefwd_kernel_time")
        return ms.value, n.value

    def export_tensor(self, layer: int, slot: int) -> np.ndarray:
        """Stored tensor in its logical layout: bf16 tensors as uint16 bit
        patterns, LN parameters as float32."""
        c = self.cfg
        d, F, n_out = c.d_model, c.d_ff, c.n_out
        shapes = {0: (d, 3 * d), 1: (3 * d,), 2: (d, d), 3: (d,), 4: (d,), 5: (d,), 6: (d, F), 7: (F,),
                  8: (F, d), 9: (d,), 10: (d,), 11: (d,), 12: (d,), 13: (d,), 14: (d, n_out), 15: (n_out,)}
        f32_slots = {4, 5, 10, 11, 12, 13}
        out = np.empty(shapes[slot], dtype=np.float32 if slot in f32_slots else np.uint16)
        _check(lib().iefwd_export_tensor(self._h, layer, slot, out.ctypes.data, out.nbytes),
               "iefwd_export_tensor")
        return out


# ---------------------------------------------------------------------- per-kernel entry points
def test_gemm(epilogue, a, w, bias, resid, out, M, N, K, stream=None) -> None:
    _check(lib().iefwd_test_gemm(epilogue, _ptr(a), _ptr(w), _ptr(bias), _ptr(resid), _ptr(out), M, N, K,
                                 _stream(stream)), "iefwd_test_gemm")


def test_gemm_on(n_cu, epilogue, a, w, out, M, N, K, bias=None, resid=None, stats=None, gamma=None, beta=None, aux=None,
                 out2=None, stream=None) -> None:
    """test_gemm with the tile chosen for n_cu CUs, and with the epilogues of a post-LN block and of training."""
    _check(lib().iefwd_test_gemm_on(n_cu, epilogue, _ptr(a), _ptr(w), _ptr(bias), _ptr(resid), _ptr(stats), _ptr(gamma),
                                    _ptr(beta), _ptr(aux), _ptr(out), _ptr(out2), M, N, K, _stream(stream)),
           "iefwd_test_gemm_on")


def test_gemm_group(n_cu, shapes, K, a=None, w=None, out=None, stream=None) -> tuple[int, int]:
    """Products [M, K] x [N, K]^T for (M, N) in shapes in one launch (none without operands); the output tile."""
    n = len(shapes)
    sizes = [(_u32 * n)(*[s[i] for s in shapes]) for i in (0, 1)]
    ptrs = [None if t is None else (_vp * n)(*[_ptr(x) for x in t]) for t in (a, w, out)]
    tile = [_u32(), _u32()]
    _check(lib().iefwd_test_gemm_group(n_cu, n, *ptrs, *sizes, K, *[ctypes.byref(t) for t in tile], _stream(stream)),
           "iefwd_test_gemm_group")
    return tile[0].value, tile[1].value


def test_gemm_skinny(epilogue, a, w, bias, resid, out, M, N, K, ln=None, stream=None) -> None:
    """ln: None, or (z, gamma, beta, eps) to take the activations as LayerNorm(z)."""
    z, g, b, eps = ln if ln is not None else (None, None, None, 0.0)
    _check(lib().iefwd_test_gemm_skinny(epilogue, _ptr(a), _ptr(w), _ptr(bias), _ptr(resid), _ptr(out), M, N, K,
                                        _ptr(z), _ptr(g), _ptr(b), eps, _stream(stream)), "iefwd_test_gemm_skinny")


def test_skinny_pack(w, dst, N, K, groups, stream=None) -> None:
    """dst (N * K bf16, device) = W [N, K] in the decode product's packed layout for `groups` K-groups."""
    _check(lib().iefwd_test_skinny_pack(_ptr(w), _ptr(dst), N, K, groups, _stream(stream)), "iefwd_test_skinny_pack")


def test_gemm_skinny_packed(epilogue, a, w_packed, groups, bias, resid, out, M, N, K, ln=None, stream=None) -> None:
    """test_gemm_skinny reading the packed copy of W (test_skinny_pack)."""
    z, g, b, eps = ln if ln is not None else (None, None, None, 0.0)
    _check(lib().iefwd_test_gemm_skinny_packed(epilogue, _ptr(a), _ptr(w_packed), groups, _ptr(bias), _ptr(resid),
                                               _ptr(out), M, N, K, _ptr(z), _ptr(g), _ptr(b), eps, _stream(stream)),
           "iefwd_test_gemm_skinny_packed")


def test_gemm_skinny_shared(epilogue, a, w_packed, groups, bias, resid, out, M, N, K, ln=None, stream=None) -> None:
    """test_gemm_skinny reading a packed copy of W made for `groups` K-groups, a multiple of the product's own."""
    z, g, b, eps = ln if ln is not None else (None, None, None, 0.0)
    _check(lib().iefwd_test_gemm_skinny_shared(epilogue, _ptr(a), _ptr(w_packed), groups, _ptr(bias), _ptr(resid),
                                               _ptr(out), M, N, K, _ptr(z), _ptr(g), _ptr(b), eps, _stream(stream)),
           "iefwd_test_gemm_skinny_shared")


def test_skinny_groups(M, N, K, ln) -> int:
    """The K-group count the decode product uses for (M, N, K), with or without the LayerNorm prologue."""
    g = _u32()
    _check(lib().iefwd_test_skinny_groups(M, N, K, 1 if ln else 0, ctypes.byref(g)), "iefwd_test_skinny_groups")
    return g.value


def test_gemm_qkv(a, w, bias, q, k, vt, batch, seq, d_model, n_heads, stream=None) -> None:
    _check(lib().iefwd_test_gemm_qkv(_ptr(a), _ptr(w), _ptr(bias), _ptr(q), _ptr(k), _ptr(vt), batch, seq,
                                     d_model, n_heads, _stream(stream)), "iefwd_test_gemm_qkv")


def test_gemm_qkv_on(n_cu, a, w, bias, q, k, vt, batch, seq, d_model, n_heads, stream=None) -> None:
    """test_gemm_qkv with the tile chosen for n_cu CUs."""
    _check(lib().iefwd_test_gemm_qkv_on(n_cu, _ptr(a), _ptr(w), _ptr(bias), _ptr(q), _ptr(k), _ptr(vt), batch, seq,
                                        d_model, n_heads, _stream(stream)), "iefwd_test_gemm_qkv_on")


def test_attention(q, k, vt, ctx, batch, n_heads, seq, head_dim, causal, stream=None) -> None:
    _check(lib().iefwd_test_attention(_ptr(q), _ptr(k), _ptr(vt), _ptr(ctx), batch, n_heads, seq, head_dim,
                                      1 if causal else 0, _stream(stream)), "iefwd_test_attention")


def test_attention_place(pairs: int, groups: int, causal: bool, n_cu: int = 256) -> np.ndarray:
    """int32 [pairs * groups, 2]: the (query group, batch * head pair) of each workgroup of the attention grid."""
    out = np.empty((pairs * groups, 2), dtype=np.int32)
    _check(lib().iefwd_test_attention_place(pairs, groups, 1 if causal else 0, n_cu, out.ctypes.data, out.size),
           "iefwd_test_attention_place")
    return out


def test_layernorm(z, gamma, beta, out_f32, out_bf16, rows, d, eps, stream=None) -> None:
    _check(lib().iefwd_test_layernorm(_ptr(z), _ptr(gamma), _ptr(beta), _ptr(out_f32), _ptr(out_bf16), rows,
                                      d, eps, _stream(stream)), "iefwd_test_layernorm")


def test_ln_head(z, gamma, beta, wh, bh, logits, rows, d, n_out, eps, stream=None) -> None:
    _check(lib().iefwd_test_ln_head(_ptr(z), _ptr(gamma), _ptr(beta), _ptr(wh), _ptr(bh), _ptr(logits), rows,
                                    d, n_out, eps, _stream(stream)), "iefwd_test_ln_head")


def test_decode_attention(q, k, vt, ctx, batch, n_heads, n_keys, head_dim, k_rows, vt_stride, stream=None) -> None:
    _check(lib().iefwd_test_decode_attention(_ptr(q), _ptr(k), _ptr(vt), _ptr(ctx), batch, n_heads, n_keys,
                                             head_dim, k_rows, vt_stride, _stream(stream)),
           "iefwd_test_decode_attention")


def test_gemm_plan(M: int, N: int, K: int, align: int, n_cu: int, ln_residual: bool = False) -> tuple[int, int, int, int]:
    """(k_order, tile_order, tile_m, tile_n) of an M x N x K product on n_cu CUs (ln_residual: the
    post-LN residual epilogue)."""
    o = [_u32() for _ in range(4)]
    _check(lib().iefwd_test_gemm_plan(M, N, K, align, n_cu, 1 if ln_residual else 0, *[ctypes.byref(v) for v in o]),
           "iefwd_test_gemm_plan")
    return tuple(v.value for v in o)


def decode_attention_noalloc(q, k, vt, ctx, batch, n_heads, n_keys, head_dim, k_rows, vt_stride,
                             stream=None) -> None:
    _check(lib().iefwd_decode_attention_noalloc(_ptr(q), _ptr(k), _ptr(vt), _ptr(ctx), batch, n_heads, n_keys,
                                                head_dim, k_rows, vt_stride, _stream(stream)),
           "iefwd_decode_attention_noalloc")


def test_cu_probe(n_groups: int, out, stream=None) -> None:
    _check(lib().iefwd_test_cu_probe(_stream(stream), n_groups, _ptr(out)), "iefwd_test_cu_probe")


# ------------------------------------------------------------------ token generation over a paged cache
class PagedCacheDesc(ctypes.Structure):
    """Mirror of ``iefwd_paged_cache``."""
    _fields_ = [("abi_version", _u32), ("kv_type", _u32), ("n_pages", _u32), ("page_size", _u32), ("n_kv_heads", _u32),
                ("head_dim", _u32), ("k", _vp), ("v", _vp), ("k_scale", _vp), ("v_scale", _vp)]


def _is(t, dtype, device: int, shape) -> bool:
    """Whether t is a contiguous tensor of this type, shape and GPU.  The calls of a decode step take a few
    microseconds on the GPU, so their checks are one expression here and explained only when they fail."""
    try:
        return t.dtype is dtype and t.get_device() == device and t.shape == shape and t.is_contiguous()
    except AttributeError:
        return False


def _need(name: str, t, dtype, device: int | None = None, shape=None):
    """Raises unless t is a tensor of this type on the GPU and, if given, `device` and of `shape` and contiguous."""
    if not isinstance(t, torch.Tensor) or t.dtype is not dtype or not t.is_cuda:
        raise ValueError(f"{name} must be a {dtype} tensor on the GPU")
    if device is not None and t.get_device() != device:
        raise ValueError(f"{name} is on {t.device}, not on cuda:{device}")
    if shape is not None and (t.shape != tuple(shape) or not t.is_contiguous()):
        raise ValueError(f"{name} must be contiguous with shape {tuple(shape)}")
    return t


def _rows(name: str, t, device: int, rows: int, heads: int, head_dim: int) -> int:
    """Checks rows of heads (bf16 [rows, heads, head_dim], or the last two as one) that may be
    slices of wider rows; returns their stride in elements."""
    if not isinstance(t, torch.Tensor) or t.dtype is not torch.bfloat16 or t.get_device() != device:
        _need(name, t, torch.bfloat16, device)
    shape, stride = t.shape, t.stride()
    if not (shape == (rows, heads, head_dim) and stride[2] == 1 and (heads == 1 or stride[1] == head_dim) or
            shape == (rows, heads * head_dim) and stride[1] == 1):
        raise ValueError(f"{name} must be [{rows}, {heads}, {head_dim}] with each row contiguous")
    return stride[0] if rows > 1 else heads * head_dim


def _table(table, device: int, batch: int) -> tuple[int, int]:
    """Checks int32 [batch, max_pages] with contiguous rows; returns the rows' stride and max_pages."""
    if not isinstance(table, torch.Tensor) or table.dtype is not torch.int32 or table.get_device() != device:
        _need("table", table, torch.int32, device)
    if table.dim() != 2 or table.shape[0] != batch or (table.shape[1] > 1 and table.stride(1) != 1):
        raise ValueError("table must be [batch, max_pages] with each row contiguous")
    cols = table.shape[1]
    return (table.stride(0) if batch > 1 else cols), cols


# torch's current device, and the handle of its current stream of a device: torch.cuda.current_device() and
# torch.cuda.current_stream(device).cuda_stream without the objects around them, which take longer (1.9 us) than a launch.
_current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)
_current_stream = getattr(torch._C, "_cuda_getCurrentRawStream", lambda device: torch.cuda.current_stream(device).cuda_stream)


def _call(device: int, stream, name: str, *args) -> None:
    """Calls a library function with `device` current, on `stream` or else torch's current stream of it."""
    handle = _current_stream(device) if stream is None else _stream(stream)
    fn = getattr(_lib or lib(), name)
    if _current_device() == device:
        status = fn(*args, handle)
    else:
        with torch.cuda.device(device):
            status = fn(*args, handle)
    if status != OK:
        _check(status, name)


class PagedCache:
    """A pool of pages of keys and values (``iefwd_paged_cache``) in the caller's tensors:
    k [n_pages, n_kv_heads, head_dim // E, page_size, E] and v [n_pages, n_kv_heads, page_size // 4,
    head_dim, 4], bfloat16 (E = 8) or float8_e4m3fn (E = 16; then with fp32 k_scale and v_scale
    [n_kv_heads]); or, in microscaled 4 bits, uint8 k [n_pages, n_kv_heads, 17, head_dim // 32, page_size] and v
    [n_pages, n_kv_heads, 17, page_size // 4, head_dim // 8], per head of a page 16 parts codes and one of scales.
    ``PagedCache.empty`` makes them.  Calls run on `stream`, by default torch's
    current stream of the cache's GPU; they neither wait for another stream nor keep the tensors given alive."""

    def __init__(self, k, v, k_scale=None, v_scale=None):
        dtype = k.dtype if isinstance(k, torch.Tensor) and k.dtype in (torch.float8_e4m3fn, torch.uint8) else torch.bfloat16
        e4m3, mx4, e = dtype is torch.float8_e4m3fn, dtype is torch.uint8, 16 if dtype is torch.float8_e4m3fn else 8
        _need("k", k, dtype)
        if k.dim() != 5 or (k.shape[2] != 17 if mx4 else k.shape[4] != e):
            raise ValueError("k must be [n_pages, n_kv_heads, 17, head_dim // 32, page_size]" if mx4 else
                             f"k must be [n_pages, n_kv_heads, head_dim // {e}, page_size, {e}]")
        n_pages, heads, pieces, page, _ = k.shape
        if mx4:
            pieces, page = k.shape[3:]
        self.device, self._dev = k.device, k.get_device()
        self.page_size, self.n_kv_heads, self.head_dim = page, heads, pieces * (32 if mx4 else e)
        _need("k", k, dtype, shape=k.shape)
        _need("v", v, dtype, self._dev, (n_pages, heads, 17, page // 4, self.head_dim // 8) if mx4 else
              (n_pages, heads, page // 4, self.head_dim, 4))
        if e4m3:
            _need("k_scale", k_scale, torch.float32, self._dev, (heads,))
            _need("v_scale", v_scale, torch.float32, self._dev, (heads,))
        elif k_scale is not None or v_scale is not None:
            raise ValueError("scales belong to a float8_e4m3fn cache")
        self.k, self.v, self.k_scale, self.v_scale = k, v, k_scale, v_scale
        kind = KV_E4M3 if e4m3 else KV_MX4 if mx4 else KV_BF16
        self.desc = PagedCacheDesc(ABI_VERSION, kind, n_pages, page, heads, self.head_dim, _ptr(k), _ptr(v), _ptr(k_scale),
                                   _ptr(v_scale))
        self._ref = ctypes.byref(self.desc)

    @classmethod
    def empty(cls, n_pages: int, page_size: int, n_kv_heads: int, head_dim: int, k_scale=None, v_scale=None,
              device="cuda:0", mx4: bool = False) -> "PagedCache":
        """A pool in new, unset memory; 8-bit if scales are given, in microscaled 4 bits with mx4."""
        if mx4:
            if page_size % 4 or head_dim % 32:
                raise ValueError("page_size must be a multiple of 4 and head_dim of 32")
            return cls(torch.empty((n_pages, n_kv_heads, 17, head_dim // 32, page_size), dtype=torch.uint8, device=device),
                       torch.empty((n_pages, n_kv_heads, 17, page_size // 4, head_dim // 8), dtype=torch.uint8, device=device),
                       k_scale, v_scale)
        dtype, e = (torch.bfloat16, 8) if k_scale is None else (torch.float8_e4m3fn, 16)
        return cls(torch.empty((n_pages, n_kv_heads, head_dim // e, page_size, e), dtype=dtype, device=device),
                   torch.empty((n_pages, n_kv_heads, page_size // 4, head_dim, 4), dtype=dtype, device=device), k_scale,
                   v_scale)

    def append(self, k, v, slots, stream=None) -> None:
        """Writes new tokens' keys and values, bf16 [tokens, n_kv_heads, head_dim] (rows may lie apart), to
        their slots (int64 [tokens], from ``paged_plan``; outside the pool: skipped)."""
        dev = self._dev
        n = _count(slots)
        if not _is(slots, torch.int64, dev, (n,)):
            _need("slots", slots, torch.int64, dev, (n,))
        ks = _rows("k", k, dev, n, self.n_kv_heads, self.head_dim)
        vs = _rows("v", v, dev, n, self.n_kv_heads, self.head_dim)
        _call(dev, stream, "iefwd_paged_append", self._ref, k.data_ptr(), v.data_ptr(), slots.data_ptr(), n, ks, vs)

    def read(self, slots, k, v, stream=None) -> None:
        """k and v, bf16 [tokens, n_kv_heads, head_dim] (rows may lie apart) = what the cache holds at slots (int64 [tokens];
        outside the pool: zeros)."""
        dev = self._dev
        n = _count(slots)
        if not _is(slots, torch.int64, dev, (n,)):
            _need("slots", slots, torch.int64, dev, (n,))
        ks = _rows("k", k, dev, n, self.n_kv_heads, self.head_dim)
        vs = _rows("v", v, dev, n, self.n_kv_heads, self.head_dim)
        _call(dev, stream, "iefwd_paged_read", self._ref, slots.data_ptr(), k.data_ptr(), v.data_ptr(), n, ks, vs)

    def workspace(self, batch: int, n_heads: int, max_pages: int) -> torch.Tensor:
        """A workspace for ``attention`` on a batch of up to this size (a smaller one may need more, and has it) and a table of
        up to max_pages columns, in memory of torch's current stream: calls on another one have to be ordered behind it, and the
        workspace to live until they have run."""
        n, most = _sz(), 0
        # requests are cut into fewer parts at each power of two of batch x key-value heads x tiles of 16 heads, up to 256
        rows = max(self.n_kv_heads * -(-n_heads // (16 * self.n_kv_heads)), 1)
        for b in {batch, *(min(batch, (1 << i) // rows) for i in range(9))} - {0} or {0}:
            _check(lib().iefwd_paged_attention_workspace(self._ref, b, n_heads, max_pages, ctypes.byref(n)),
                   "iefwd_paged_attention_workspace")
            most = max(most, n.value)
        return torch.empty(most, dtype=torch.uint8, device=self.device)

    def attention(self, q, table, lens, out, workspace, scale: float | None = None, stream=None, cap: float = 0.0,
                  slopes=None) -> None:
        """out bf16 [batch, n_heads, head_dim] = attention of one query per request and head, q of that
        shape (rows may lie apart), over the pages in `table` (int32 [batch, max_pages], rows may lie apart) of
        lens (int32 [batch]) cached tokens.  scale: 1 / sqrt(head_dim) by default.  A score s becomes cap tanh(s / cap) unless
        cap is 0, and loses slopes[head] (fp32 [n_heads]) times the key's distance from the newest one."""
        dev, d = self._dev, self.head_dim
        batch = len(lens)
        if not _is(lens, torch.int32, dev, (batch,)):
            _need("lens", lens, torch.int32, dev, (batch,))
        stride, cols = _table(table, dev, batch)
        heads = out.numel() // (batch * d) if batch else 0
        if not (_is(out, torch.bfloat16, dev, (batch, heads, d)) or _is(out, torch.bfloat16, dev, (batch, heads * d))):
            _need("out", out, torch.bfloat16, dev, (batch, heads, d))
        qs = _rows("q", q, dev, batch, heads, d)
        if workspace.dtype is not torch.uint8 or workspace.get_device() != dev or not workspace.is_contiguous():
            _need("workspace", workspace, torch.uint8, dev, (workspace.numel(),))
        scale = d ** -0.5 if scale is None else scale
        if cap == 0.0 and slopes is None:
            _call(dev, stream, "iefwd_paged_attention", self._ref, q.data_ptr(), qs, heads, table.data_ptr(), stride, cols,
                  lens.data_ptr(), batch, scale, out.data_ptr(), workspace.data_ptr(), workspace.numel())
            return
        if slopes is not None and not _is(slopes, torch.float32, dev, (heads,)):
            _need("slopes", slopes, torch.float32, dev, (heads,))
        _call(dev, stream, "iefwd_paged_attention_scored", self._ref, q.data_ptr(), qs, heads, table.data_ptr(), stride, cols,
              lens.data_ptr(), batch, scale, cap, None if slopes is None else slopes.data_ptr(), out.data_ptr(),
              workspace.data_ptr(), workspace.numel())


def paged_plan(page_size: int, lens, new_lens, table, ring, counters, lens_out, counters_out, slots, starts, refused,
               stream=None) -> None:
    """Pages and slots of a step (``iefwd_paged_plan``): requests of lens cached tokens come to new_lens ones.
    int32 lens, new_lens, lens_out [batch], table [batch, max_pages] (rows may lie apart), ring [pages of the pool],
    starts [batch + 1], refused [1]; int64 counters, counters_out [2], slots [most new tokens].  Runs on `stream`, by
    default torch's current stream of lens' GPU."""
    dev = _need("lens", lens, torch.int32).get_device()
    n, n_pages, room = len(lens), len(ring), len(slots)
    i32, i64 = torch.int32, torch.int64
    if not (_is(lens, i32, dev, (n,)) and _is(new_lens, i32, dev, (n,)) and _is(lens_out, i32, dev, (n,)) and
            _is(ring, i32, dev, (n_pages,)) and _is(counters, i64, dev, (2,)) and _is(counters_out, i64, dev, (2,)) and
            _is(slots, i64, dev, (room,)) and _is(starts, i32, dev, (n + 1,)) and _is(refused, i32, dev, (1,))):
        for name, t, dtype, count in (("lens", lens, i32, n), ("new_lens", new_lens, i32, n), ("lens_out", lens_out, i32, n),
                                      ("ring", ring, i32, n_pages), ("counters", counters, i64, 2),
                                      ("counters_out", counters_out, i64, 2), ("slots", slots, i64, room),
                                      ("starts", starts, i32, n + 1), ("refused", refused, i32, 1)):
            _need(name, t, dtype, dev, (count,))
    stride, cols = _table(table, dev, n)
    _call(dev, stream, "iefwd_paged_plan", n, page_size, lens.data_ptr(), new_lens.data_ptr(), table.data_ptr(), stride, cols,
          ring.data_ptr(), n_pages, counters.data_ptr(), lens_out.data_ptr(), counters_out.data_ptr(), slots.data_ptr(), room,
          starts.data_ptr(), refused.data_ptr())


def test_paged_split(batch: int, n_heads: int, n_kv_heads: int, n_keys: int) -> int:
    """The keys in each part that ``PagedCache.attention`` splits a request of n_keys into."""
    keys = _u32()
    _check(lib().iefwd_test_paged_split(batch, n_heads, n_kv_heads, n_keys, ctypes.byref(keys)), "iefwd_test_paged_split")
    return keys.value


class Q4Weight:
    """A weight matrix [N, K] in 4 bits, laid out for ``product`` once: codes uint8 [N, K / 2] (weight 2 i in
    the low half of byte i), scales bf16 [N, K / group], zeros uint8 [N, K / group] or None (8 everywhere);
    W = scales (codes - zeros).  Calls run on `stream`, by default torch's current stream of the weight's GPU.
    The constructor allocates on the current stream and packs on `stream`: the one waits for the other before and
    after, so that the tensors given, which are not kept, may be freed or overwritten at once on the current stream,
    and the weight used there.  A weight that is used on another stream lives until its last call there has run."""

    def __init__(self, codes, scales, zeros=None, stream=None):
        _need("codes", codes, torch.uint8)
        if codes.dim() != 2 or not isinstance(scales, torch.Tensor) or scales.dim() != 2 or not scales.shape[1]:
            raise ValueError("codes must be [N, K / 2] and scales [N, K / group]")
        self.device, self._dev, self.N, self.K = codes.device, codes.get_device(), codes.shape[0], 2 * codes.shape[1]
        self.group = self.K // scales.shape[1]
        shape = (self.N, self.K // self.group if self.group else 0)
        _need("codes", codes, torch.uint8, shape=codes.shape)
        _need("scales", scales, torch.bfloat16, self._dev, shape)
        if zeros is not None:
            _need("zeros", zeros, torch.uint8, self._dev, shape)
        n = _sz()
        _check(lib().iefwd_q4_packed_bytes(self.N, self.K, self.group, ctypes.byref(n)), "iefwd_q4_packed_bytes")
        home = torch.cuda.current_stream(self._dev)
        self.packed = torch.empty(n.value, dtype=torch.uint8, device=self.device)
        self._at = self.packed.data_ptr()
        side = home if stream is None else torch.cuda.ExternalStream(_stream(stream), device=self.device)
        apart = side.cuda_stream != home.cuda_stream
        if apart:      # home's earlier work may still use the memory of `packed`
            side.wait_stream(home)
        _call(self._dev, side, "iefwd_q4_pack", codes.data_ptr(), scales.data_ptr(), _ptr(zeros), self._at, self.N, self.K,
              self.group)
        if apart:
            home.wait_stream(side)
        for t in (codes, scales, zeros):      # of a third stream, perhaps: not handed out again before they are read
            if t is not None:
                t.record_stream(home)

    def product(self, a, out, epilogue: int = EPI_BIAS_BF16, bias=None, resid=None, stream=None) -> None:
        """out [M, N] = epilogue(a W^T + bias), a bf16 [M, K], M <= 16; out bf16, or fp32 (as resid) for
        EPI_BIAS_RESID_F32; bias bf16 [N] or None."""
        dev, m, n, k = self._dev, len(a), self.N, self.K
        f32 = epilogue == EPI_BIAS_RESID_F32
        kind = torch.float32 if f32 else torch.bfloat16
        if not (_is(a, torch.bfloat16, dev, (m, k)) and _is(out, kind, dev, (m, n)) and
                (bias is None or _is(bias, torch.bfloat16, dev, (n,))) and (not f32 or _is(resid, kind, dev, (m, n)))):
            _need("a", a, torch.bfloat16, dev, (m, k))
            _need("out", out, kind, dev, (m, n))
            if bias is not None:
                _need("bias", bias, torch.bfloat16, dev, (n,))
            _need("resid", resid, kind, dev, (m, n))
        _call(dev, stream, "iefwd_q4_gemm", epilogue, a.data_ptr(), self._at,
              None if bias is None else bias.data_ptr(), resid.data_ptr() if f32 else None, out.data_ptr(), m, n, k, self.group)


# ------------------------------------------------------------------ matrices in microscaled 4 bits
_FLOATS = {torch.bfloat16: BF16, torch.float32: F32}


def _float_rows(name: str, t, device: int, cols: int) -> tuple[int, int, int]:
    """Checks bf16 or fp32 [rows, cols] whose rows are contiguous and may lie apart; returns its type, the rows' stride in
    elements and the number of rows."""
    try:
        kind, shape, stride = _FLOATS.get(t.dtype), t.shape, t.stride()
        if kind is not None and t.get_device() == device and len(shape) == 2 and shape[1] == cols and (cols == 1 or stride[1] == 1):
            return kind, (stride[0] if shape[0] > 1 else cols), shape[0]
    except AttributeError:
        pass
    raise ValueError(f"{name} must be a bfloat16 or float32 tensor [rows, {cols}] on cuda:{device} with each row contiguous")


def _count(t) -> int:
    """len(t) of a tensor in a third of its time; 0 for what is none."""
    try:
        return t.shape[0]
    except (AttributeError, IndexError):
        return 0


class Mx4Matrix:
    """A matrix [rows, K] in microscaled 4 bits (``iefwd_mx4_*``), in new, unset memory of torch's current stream: weights, or
    activations for a product.  Calls run on `stream`, by default torch's current stream of the matrix's GPU; they neither
    wait for another stream nor keep the tensors given alive."""

    def __init__(self, rows: int, K: int, device="cuda:0"):
        if rows >> 32 or K >> 32:      # ctypes would cut them to 32 bits
            raise ValueError("a matrix has 1 to 2^24 rows and 1 to 2^20 columns")
        n = _sz()
        _check(lib().iefwd_mx4_bytes(rows, K, ctypes.byref(n)), "iefwd_mx4_bytes")
        self.rows, self.K = rows, K
        self.packed = torch.empty(n.value, dtype=torch.uint8, device=device)
        if not self.packed.is_cuda:
            raise ValueError("device must be a GPU")
        self.device, self._dev, self._at = self.packed.device, self.packed.get_device(), self.packed.data_ptr()

    def quantize(self, x, stream=None) -> None:
        """The first len(x) rows (and the rest of their 16 as zeros) = x, bf16 or fp32 [at most rows, K], whose rows may lie
        apart."""
        kind, stride, n = _float_rows("x", x, self._dev, self.K)
        if n > self.rows:
            raise ValueError(f"x has {n} rows, the matrix {self.rows}")
        _call(self._dev, stream, "iefwd_mx4_quantize", kind, x.data_ptr(), stride, self._at, n, self.K)

    def load(self, codes, scales, stream=None) -> None:
        """All rows from codes uint8 [rows, K / 2] (column 2 i in the low half of byte i) and scale bytes uint8
        [rows, K / 32], as checkpoints hold them; K a multiple of 32."""
        if self.K % 32:
            raise ValueError("K must be a multiple of 32")
        _need("codes", codes, torch.uint8, self._dev, (self.rows, self.K // 2))
        _need("scales", scales, torch.uint8, self._dev, (self.rows, self.K // 32))
        _call(self._dev, stream, "iefwd_mx4_pack", codes.data_ptr(), scales.data_ptr(), self._at, self.rows, self.K)

    def values(self, out, stream=None) -> None:
        """out, bf16 or fp32 [at most rows, K], whose rows may lie apart, = the values of the first rows."""
        kind, stride, n = _float_rows("out", out, self._dev, self.K)
        if n > self.rows:
            raise ValueError(f"out has {n} rows, the matrix {self.rows}")
        _call(self._dev, stream, "iefwd_mx4_values", self._at, kind, out.data_ptr(), stride, n, self.K)

    def product(self, a, out, epilogue: int = EPI_BIAS_BF16, bias=None, resid=None, stream=None) -> None:
        """out [M, N] = epilogue(a W^T + bias) with this matrix as W [N, K]: a another Mx4Matrix, of which the first M
        rows are taken, or bf16 [M, K], M <= 16 and K a multiple of 8, which is quantised on the way; out bf16, or fp32 (as resid)
        for EPI_BIAS_RESID_F32; bias bf16 [N] or None."""
        dev, m, n, k = self._dev, _count(out), self.rows, self.K
        f32 = epilogue == EPI_BIAS_RESID_F32
        kind = torch.float32 if f32 else torch.bfloat16
        if not (_is(out, kind, dev, (m, n)) and (bias is None or _is(bias, torch.bfloat16, dev, (n,))) and
                (not f32 or _is(resid, kind, dev, (m, n)))):
            _need("out", out, kind, dev, (m, n))
            if bias is not None:
                _need("bias", bias, torch.bfloat16, dev, (n,))
            _need("resid", resid, kind, dev, (m, n))
        if isinstance(a, Mx4Matrix):
            if a.K != k or a.rows < m or a._dev != dev:
                raise ValueError(f"a must have at least {m} rows, {k} columns and be on cuda:{dev}")
            name, at = "iefwd_mx4_gemm", a._at
        else:
            if m >> 32 or not _is(a, torch.bfloat16, dev, (m, k)):
                _need("a", a, torch.bfloat16, dev, (m, k))
                raise ValueError("a in bf16 has at most 16 rows")
            name, at = "iefwd_mx4_gemm_bf16", a.data_ptr()
        _call(dev, stream, name, epilogue, at, self._at, None if bias is None else bias.data_ptr(),
              resid.data_ptr() if f32 else None, out.data_ptr(), m, n, k)


# ------------------------------------------------------------------ log probabilities of tokens
def token_logprobs_workspace(rows: int, vocab: int, n_top: int = 0, device="cuda:0") -> torch.Tensor:
    """A workspace for ``token_logprobs`` on up to this many rows and most probable tokens (fewer rows may need more than these, and
    have it), in memory of torch's current stream: calls on another one have to be ordered behind it, and the workspace to live
    until they have run."""
    if rows >> 32 or vocab >> 32 or n_top >> 32:
        raise ValueError("sizes must be below 2^32")
    n = _sz()
    for r in (rows, 1):
        _check(lib().iefwd_token_logprobs_workspace(r, vocab, n_top, ctypes.byref(n)), "iefwd_token_logprobs_workspace")
    # where a row alone is not cut into parts, none are; else the most of any number of rows
    return torch.empty(min(64 * rows, 2048) * (12 + 8 * n_top) if n.value else 0, dtype=torch.uint8, device=device)


def _logits(name: str, t) -> tuple[int, int, int, int, int]:
    """Checks bf16 or fp32 [rows, vocab] with contiguous rows; returns its GPU, type, sizes and row stride."""
    if not isinstance(t, torch.Tensor) or t.dtype not in _FLOATS or not t.is_cuda:
        raise ValueError(f"{name} must be a bfloat16 or float32 tensor on the GPU")
    if t.dim() != 2 or (t.shape[1] > 1 and t.stride(1) != 1):
        raise ValueError(f"{name} must be [rows, vocab] with each row contiguous")
    rows, vocab = t.shape
    if rows >> 32 or vocab >> 32:      # ctypes would cut them to 32 bits
        raise ValueError(f"{name} must have at most 2^22 rows and 2^24 columns")
    return t.get_device(), _FLOATS[t.dtype], rows, vocab, t.stride(0) if rows > 1 else vocab


def token_logprobs(logits, tokens, logprobs, workspace, entropy=None, stats=None, top_ids=None, top_logprobs=None,
                   scale: float = 1.0, stream=None) -> None:
    """Log probabilities under softmax(scale * logits) (``iefwd_token_logprobs``): logits bf16 or fp32 [rows, vocab], whose rows
    may lie apart, tokens int64 [rows] (outside the vocabulary: 0); fp32 logprobs and, if given, entropy [rows], stats [rows, 2]
    for ``token_logprobs_grad``, and the most probable tokens, int32 top_ids and fp32 top_logprobs [rows, n].  Runs on
    `stream`, by default torch's current stream of the logits' GPU."""
    dev, kind, rows, vocab, stride = _logits("logits", logits)
    f32 = torch.float32
    n = top_ids.shape[-1] if isinstance(top_ids, torch.Tensor) and top_ids.dim() else 0
    if n >> 32:
        raise ValueError("at most 32 most probable tokens")
    if not (_is(tokens, torch.int64, dev, (rows,)) and _is(logprobs, f32, dev, (rows,)) and
            (entropy is None or _is(entropy, f32, dev, (rows,))) and (stats is None or _is(stats, f32, dev, (rows, 2))) and
            (top_ids is None or _is(top_ids, torch.int32, dev, (rows, n))) and
            (top_logprobs is None if top_ids is None else _is(top_logprobs, f32, dev, (rows, n))) and
            _is(workspace, torch.uint8, dev, (workspace.numel(),) if isinstance(workspace, torch.Tensor) else ())):
        _need("tokens", tokens, torch.int64, dev, (rows,))
        _need("logprobs", logprobs, f32, dev, (rows,))
        for name, t, shape in (("entropy", entropy, (rows,)), ("stats", stats, (rows, 2))):
            if t is not None:
                _need(name, t, f32, dev, shape)
        if (top_ids is None) != (top_logprobs is None):
            raise ValueError("top_ids and top_logprobs come together")
        if top_ids is not None:
            _need("top_ids", top_ids, torch.int32, dev, (rows, n))
            _need("top_logprobs", top_logprobs, f32, dev, (rows, n))
        _need("workspace", workspace, torch.uint8, dev)
        _need("workspace", workspace, torch.uint8, dev, (workspace.numel(),))
    _call(dev, stream, "iefwd_token_logprobs", kind, logits.data_ptr(), stride, rows, vocab, tokens.data_ptr(), scale,
          logprobs.data_ptr(), None if entropy is None else entropy.data_ptr(), None if stats is None else stats.data_ptr(), n,
          top_ids.data_ptr() if n else None, top_logprobs.data_ptr() if n else None, workspace.data_ptr(), workspace.numel())


def token_logprobs_grad(logits, tokens, stats, out, grad_logprobs=None, entropy=None, grad_entropy=None, scale: float = 1.0,
                        stream=None) -> None:
    """out [rows, vocab] = the gradient by the logits of sum(grad_logprobs * logprobs + grad_entropy * entropy) (fp32 [rows], at
    least one), with the arguments, stats and entropy of ``token_logprobs``; out as logits, whose rows may lie apart, or logits
    themselves."""
    dev, kind, rows, vocab, stride = _logits("logits", logits)
    out_dev, out_kind, out_rows, out_vocab, out_stride = _logits("out", out)
    if (out_dev, out_kind, out_rows, out_vocab) != (dev, kind, rows, vocab):
        raise ValueError("out must be as logits")
    f32 = torch.float32
    given = (("grad_logprobs", grad_logprobs), ("entropy", entropy), ("grad_entropy", grad_entropy))
    if not (_is(tokens, torch.int64, dev, (rows,)) and _is(stats, f32, dev, (rows, 2)) and
            all(t is None or _is(t, f32, dev, (rows,)) for _, t in given)):
        _need("tokens", tokens, torch.int64, dev, (rows,))
        _need("stats", stats, f32, dev, (rows, 2))
        for name, t in given:
            if t is not None:
                _need(name, t, f32, dev, (rows,))
    _call(dev, stream, "iefwd_token_logprobs_grad", kind, logits.data_ptr(), stride, rows, vocab, tokens.data_ptr(), scale,
          stats.data_ptr(), *[None if t is None else t.data_ptr() for t in (entropy, grad_logprobs, grad_entropy)],
          out.data_ptr(), out_stride)


# ------------------------------------------------------------------ quota controller
CTL_NONE, CTL_EMERGENCY, CTL_RECOVERY, CTL_CONTENTION = 0, 1, 2, 3


class TrainParams(ctypes.Structure):
    """Mirror of ``iefwd_train_params``."""
    _fields_ = [("abi_version", _u32), ("reserved0", _u32), ("lr", _f32), ("beta1", _f32), ("beta2", _f32),
                ("eps", _f32), ("weight_decay", _f32), ("reserved1", _f32)]


def train_params(**kw) -> TrainParams:
    tp = TrainParams()
    lib().iefwd_train_params_init(ctypes.byref(tp))
    for k, v in kw.items():
        if k not in ("lr", "beta1", "beta2", "eps", "weight_decay"):
            raise ValueError(f"unknown training parameter {k}")
        setattr(tp, k, v)
    return tp


class Trainer(Instance):
    """A training instance (post-LN encoder, softmax cross-entropy, AdamW): the
    same quota calls as an inference instance, plus whole training steps."""

    def __init__(self, device: int = 0, train: dict | None = None, **config):
        self._h = None
        self.cfg = make_config(**config)
        self.tp = train_params(**(train or {}))
        h = _vp()
        _check(lib().iefwd_train_create(ctypes.byref(self.cfg), ctypes.byref(self.tp), device, ctypes.byref(h)),
               "iefwd_train_create")
        self._h = h
        self.device = device

    def step(self, x, labels) -> None:
        """One asynchronous training step.  x fp32 [B, S, d], labels int32 [B, S]:
        both CUDA tensors (kept alive until the step completes) or both host arrays."""
        if isinstance(x, torch.Tensor) and x.is_cuda:
            if not (isinstance(labels, torch.Tensor) and labels.is_cuda):
                raise ValueError("x and labels must both be on the device or both on the host")
            if x.dtype != torch.float32 or not x.is_contiguous():
                raise ValueError("x must be a contiguous float32 tensor")
            if labels.dtype != torch.int32 or not labels.is_contiguous():
                raise ValueError("labels must be a contiguous int32 tensor")
            is_dev = 1
        else:
            x = np.ascontiguousarray(x.cpu().numpy() if isinstance(x, torch.Tensor) else x, dtype=np.float32)
            labels = np.ascontiguousarray(labels.cpu().numpy() if isinstance(labels, torch.Tensor) else labels,
                                          dtype=np.int32)
            is_dev = 0
        b, s_ = x.shape[0], x.shape[1]
        _check(lib().iefwd_train_step(self._h, _ptr(x), _ptr(labels), b, s_, is_dev), "iefwd_train_step")
        self._last_shape = (b, s_)
        self._keep = (x, labels)

    def loss(self) -> float:
        v = _f32()
        _check(lib().iefwd_train_loss(self._h, ctypes.byref(v)), "iefwd_train_loss")
        return float(v.value)

    def steps(self) -> int:
        v = _u64()
        _check(lib().iefwd_train_steps(self._h, ctypes.byref(v)), "iefwd_train_steps")
        return int(v.value)

    def export(self, layer: int, slot: int, what: int, shape) -> np.ndarray:
        out = np.empty(shape, dtype=np.float32)
        _check(lib().iefwd_train_export(self._h, layer, slot, what, out.ctypes.data, out.size), "iefwd_train_export")
        return out


CTL_TEMPORARY_YIELD = 1


class CtlParams(ctypes.Structure):
    _fields_ = [("abi_version", _u32), ("max_tokens", _u32), ("window", _u32), ("granule", _u32),
                ("min_quota", _u32), ("flags", _u32), ("eta_violation", ctypes.c_double),
                ("eta_increase", ctypes.c_double)]


class Controller:
    """The fast scale-up/down quota controller (iefwd_ctl_*): report each
    instance's kernels and last batch time once per control period, then
    issue() returns (tokens, quotas, first mask bits) in id order.
    temporary_yield=True sets IEFWD_CTL_TEMPORARY_YIELD."""

    def __init__(self, temporary_yield: bool = False, **params):
        p = CtlParams()
        _check(lib().iefwd_ctl_params_init(ctypes.byref(p)), "iefwd_ctl_params_init")
        for k, v in params.items():
            setattr(p, k, v)
        if temporary_yield:
            p.flags |= CTL_TEMPORARY_YIELD
        h = _vp()
        _check(lib().iefwd_ctl_create(ctypes.byref(p), ctypes.byref(h)), "iefwd_ctl_create")
        self._h = h.value
        self.n = 0

    def add(self, request: float, limit: float, slo_sensitive: bool) -> int:
        i = _u32()
        _check(lib().iefwd_ctl_add(self._h, request, limit, 1 if slo_sensitive else 0, ctypes.byref(i)),
               "iefwd_ctl_add")
        self.n += 1
        return i.value

    def report(self, i: int, kernels: int, klc_ms: float) -> None:
        _check(lib().iefwd_ctl_report(self._h, i, kernels, klc_ms), "iefwd_ctl_report")

    def issue(self) -> tuple[list[float], list[int], list[int]]:
        t, q, f = (ctypes.c_double * max(self.n, 1))(), (_u32 * max(self.n, 1))(), (_u32 * max(self.n, 1))()
        _check(lib().iefwd_ctl_issue(self._h, t, q, f, self.n), "iefwd_ctl_issue")
        return list(t)[:self.n], list(q)[:self.n], list(f)[:self.n]

    def state(self) -> int:
        v = ctypes.c_int32()
        _check(lib().iefwd_ctl_state(self._h, ctypes.byref(v)), "iefwd_ctl_state")
        return v.value

    def close(self) -> None:
        if getattr(self, "_h", None):
            lib().iefwd_ctl_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:   # interpreter shutdown
            pass

