"""ctypes binding of librr.so: argument marshalling only, every step runs in the HIP kernels.

Function names and argument order follow include/rr.h.  Tensors are torch CUDA tensors (torch is
used for device memory and streams only); calls are enqueued on torch's current stream.
"""
from __future__ import annotations

import ctypes as C
import os
from dataclasses import dataclass

RR_F32, RR_BF16 = 0, 1
RR_ACT_GELU, RR_ACT_SWIGLU, RR_ACT_NONE = 0, 1, 2
RR_INTRA_GPU, RR_FILL_IN, RR_POLICY_ARRIVAL, RR_QUOTA_PER_GROUP = 1, 2, 4, 8
RR_GRAD_STRAIGHT_THROUGH, RR_GRAD_ACCUMULATE = 1, 2

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB = None


class RRError(RuntimeError):
    pass


class _Config(C.Structure):
    _fields_ = [("T", C.c_int32), ("d_model", C.c_int32), ("d_ff", C.c_int32), ("E", C.c_int32),
                ("k", C.c_int32), ("G", C.c_int32), ("capacity_factor", C.c_float),
                ("dtype", C.c_int32), ("act", C.c_int32), ("flags", C.c_uint32)]


class _LinearConfig(C.Structure):
    _fields_ = [("M", C.c_int32), ("K", C.c_int32), ("N", C.c_int32), ("dtype", C.c_int32), ("act", C.c_int32)]


_TABLE_FIELDS = ("rank_expert", "slot", "slot_token", "fill_topk", "fill_total",
                 "ir_expert", "ir_row", "ir_offset", "ir_token", "combine_w")


class _Tables(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in _TABLE_FIELDS]


class _KernelTime(C.Structure):
    _fields_ = [("name", C.c_char_p), ("launches", C.c_int32), ("total_ms", C.c_float)]


@dataclass
class RRConfig:
    T: int
    d_model: int
    d_ff: int
    E: int
    k: int
    G: int
    capacity_factor: float
    dtype: int = RR_BF16
    act: int = RR_ACT_SWIGLU
    flags: int = RR_INTRA_GPU | RR_FILL_IN

    def c(self) -> _Config:
        return _Config(self.T, self.d_model, self.d_ff, self.E, self.k, self.G, self.capacity_factor,
                       self.dtype, self.act, self.flags)


@dataclass
class RRLinearConfig:
    M: int
    K: int
    N: int
    dtype: int = RR_BF16
    act: int = RR_ACT_NONE

    @property
    def rows(self) -> int:
        """Rows of the weight matrix, columns of the pre-activations."""
        return 2 * self.N if self.act == RR_ACT_SWIGLU else self.N

    def c(self) -> _LinearConfig:
        return _LinearConfig(self.M, self.K, self.N, self.dtype, self.act)


def library_path() -> str:
    return os.path.join(_HERE, "librr.so")


def load_library():
    """Loads librr.so; raises if it has not been built (there is no fallback path)."""
    global _LIB
    if _LIB is not None:
        return _LIB
    path = library_path()
    if not os.path.exists(path):
        raise RRError(f"{path} is missing: build it with `python -m paper_2402_12399_amd.build`")
    lib = C.CDLL(path)
    vp, i32, sz = C.c_void_p, C.c_int32, C.c_size_t
    lib.rr_capacity.restype = i32
    lib.rr_capacity.argtypes = [i32, i32, C.c_float]
    lib.rr_slots_per_expert.restype = i32
    lib.rr_slots_per_expert.argtypes = [C.POINTER(_Config)]
    lib.rr_workspace_bytes.restype = C.c_int
    lib.rr_workspace_bytes.argtypes = [C.POINTER(_Config), C.POINTER(sz)]
    lib.rr_router_scores.restype = C.c_int
    lib.rr_router_scores.argtypes = [C.POINTER(_Config), vp, vp, vp, vp, vp, vp, vp]
    lib.rr_rectified_dispatch.restype = C.c_int
    lib.rr_rectified_dispatch.argtypes = [C.POINTER(_Config), vp, C.POINTER(_Tables), vp, sz, vp]
    lib.rr_rectified_dispatch_static.restype = C.c_int
    lib.rr_rectified_dispatch_static.argtypes = [C.POINTER(_Config), vp, C.POINTER(_Tables), vp]
    lib.rr_moe_forward.restype = C.c_int
    lib.rr_moe_forward.argtypes = [C.POINTER(_Config), vp, vp, vp, vp, vp, vp, vp, C.POINTER(_Tables), vp, vp, sz, vp]
    lib.rr_router_backward.restype = C.c_int
    lib.rr_router_backward.argtypes = [C.POINTER(_Config), vp, vp, C.POINTER(_Tables), vp, sz, C.c_uint32, vp, vp, vp]
    f32, i64, u64, u32 = C.c_float, C.c_int64, C.c_uint64, C.c_uint32
    lib.rr_balance_workspace_bytes.restype = C.c_int
    lib.rr_balance_workspace_bytes.argtypes = [C.POINTER(_Config), C.POINTER(sz)]
    lib.rr_balance_loss.restype = C.c_int
    lib.rr_balance_loss.argtypes = [C.POINTER(_Config), vp, vp, vp, f32, vp, vp, vp, vp, sz, vp]
    lib.rr_balance_loss_backward.restype = C.c_int
    lib.rr_balance_loss_backward.argtypes = [C.POINTER(_Config), vp, vp, vp, f32, vp, u32, vp, vp]
    lib.rr_dropout.restype = C.c_int
    lib.rr_dropout.argtypes = [i64, i32, vp, vp, f32, u64, u64, vp, vp, vp]
    lib.rr_dropout_backward.restype = C.c_int
    lib.rr_dropout_backward.argtypes = [i64, i32, vp, f32, u64, u64, vp, vp, vp]
    lib.rr_linear_workspace_bytes.restype = C.c_int
    lib.rr_linear_workspace_bytes.argtypes = [C.POINTER(_LinearConfig), i32, C.POINTER(sz)]
    lib.rr_linear.restype = C.c_int
    lib.rr_linear.argtypes = [C.POINTER(_LinearConfig), vp, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.rr_linear_backward.restype = C.c_int
    lib.rr_linear_backward.argtypes = [C.POINTER(_LinearConfig), vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.rr_init.restype = C.c_int
    lib.rr_init.argtypes = []
    lib.rr_profile_enable.restype = C.c_int
    lib.rr_profile_enable.argtypes = [C.c_int]
    lib.rr_profile_read.restype = C.c_int
    lib.rr_profile_read.argtypes = [C.POINTER(_KernelTime), i32, C.POINTER(i32)]
    lib.rr_strerror.restype = C.c_char_p
    lib.rr_strerror.argtypes = [C.c_int]
    _LIB = lib
    return lib


def rr_strerror(code: int) -> str:
    return load_library().rr_strerror(code).decode()


def _check(code: int, what: str):
    if code != 0:
        raise RRError(f"{what} failed: {rr_strerror(code)} ({code})")


def _ptr(t):
    return None if t is None else C.c_void_p(t.data_ptr())


def _stream():
    import torch
    return C.c_void_p(torch.cuda.current_stream().cuda_stream)


def rr_init():
    _check(load_library().rr_init(), "rr_init")


def rr_capacity(T: int, E: int, capacity_factor: float) -> int:
    return int(load_library().rr_capacity(T, E, capacity_factor))


def rr_slots_per_expert(cfg: RRConfig) -> int:
    cc = cfg.c()
    n = int(load_library().rr_slots_per_expert(C.byref(cc)))
    if n < 0:
        raise RRError("rr_slots_per_expert: invalid or unsupported configuration")
    return n


def rr_workspace_bytes(cfg: RRConfig) -> int:
    n = C.c_size_t(0)
    cc = cfg.c()
    _check(load_library().rr_workspace_bytes(C.byref(cc), C.byref(n)), "rr_workspace_bytes")
    return int(n.value)


def alloc_workspace(cfg: RRConfig, device="cuda"):
    import torch
    return torch.empty(rr_workspace_bytes(cfg), dtype=torch.uint8, device=device)


class Tables:
    """Device tensors of rr_tables plus the C struct that points at them."""

    def __init__(self, cfg: RRConfig, device="cuda"):
        import torch
        C_ = rr_slots_per_expert(cfg)
        i32 = dict(dtype=torch.int32, device=device)
        self.capacity = C_
        self.rank_expert = torch.empty((cfg.T, cfg.k + 1), **i32)
        self.slot = torch.empty((cfg.T, cfg.k + 1), **i32)
        self.slot_token = torch.empty((cfg.E, C_), **i32)
        self.fill_topk = torch.empty(cfg.E, **i32)
        self.fill_total = torch.empty(cfg.E, **i32)
        self.ir_expert = torch.empty(cfg.T, **i32)
        self.ir_row = torch.empty(cfg.T, **i32)
        self.ir_offset = torch.empty(cfg.E + 1, **i32)
        self.ir_token = torch.empty(cfg.T, **i32)
        self.combine_w = torch.empty((cfg.T, cfg.k + 2), dtype=torch.float32, device=device)

    def c(self) -> _Tables:
        return _Tables(*[getattr(self, n).data_ptr() for n in _TABLE_FIELDS])

    def to_host(self) -> dict:
        out = {n: getattr(self, n).cpu().numpy() for n in _TABLE_FIELDS}
        out["ir_token"] = out["ir_token"][:int(out["ir_offset"][-1])]
        return out


def alloc_tables(cfg: RRConfig, device="cuda") -> Tables:
    return Tables(cfg, device)


def rr_router_scores(cfg: RRConfig, x, w_router, bias, logits, probs=None, rank_expert=None):
    cc = cfg.c()
    _check(load_library().rr_router_scores(C.byref(cc), _ptr(x), _ptr(w_router), _ptr(bias), _ptr(logits),
                                           _ptr(probs), _ptr(rank_expert), _stream()), "rr_router_scores")


def rr_rectified_dispatch(cfg: RRConfig, logits, tables: Tables, workspace):
    cc, tc = cfg.c(), tables.c()
    _check(load_library().rr_rectified_dispatch(C.byref(cc), _ptr(logits), C.byref(tc), _ptr(workspace),
                                                workspace.numel(), _stream()), "rr_rectified_dispatch")


def rr_rectified_dispatch_static(cfg: RRConfig, logits, tables: Tables):
    """rr_rectified_dispatch with the library's own static scratch buffer (allocates nothing)."""
    cc, tc = cfg.c(), tables.c()
    _check(load_library().rr_rectified_dispatch_static(C.byref(cc), _ptr(logits), C.byref(tc), _stream()),
           "rr_rectified_dispatch_static")


def rr_moe_forward(cfg: RRConfig, x, w_router, bias, w1, w3, w2, out, tables: Tables | None, logits, workspace):
    cc = cfg.c()
    tc = tables.c() if tables is not None else None
    _check(load_library().rr_moe_forward(C.byref(cc), _ptr(x), _ptr(w_router), _ptr(bias), _ptr(w1), _ptr(w3),
                                         _ptr(w2), _ptr(out), C.byref(tc) if tc is not None else None,
                                         _ptr(logits), _ptr(workspace), workspace.numel(), _stream()),
           "rr_moe_forward")


def rr_router_backward(cfg: RRConfig, dout, logits, tables: Tables | None, workspace, dlogits, dcombine_w=None,
                       straight_through: bool = True):
    cc = cfg.c()
    tc = tables.c() if tables is not None else None
    _check(load_library().rr_router_backward(C.byref(cc), _ptr(dout), _ptr(logits),
                                             C.byref(tc) if tc is not None else None, _ptr(workspace),
                                             workspace.numel(), RR_GRAD_STRAIGHT_THROUGH if straight_through else 0,
                                             _ptr(dcombine_w), _ptr(dlogits), _stream()), "rr_router_backward")


class _Args:
    """Addresses of the tensors of one call of the operators around the layer, checked: dense, as large as the call takes them to
    be, of their type, and on the current device, where the call is enqueued.  (A few tenths of a microsecond per tensor: small
    calls are bound by what the host does.)"""

    __slots__ = ("what", "device")

    def __init__(self, what: str):
        import torch
        self.what = what
        self.device = torch.cuda.current_device() if torch.cuda.is_initialized() else None

    def __call__(self, name, t, numel, dtype):
        """Address of t, or None for None."""
        if t is None:
            return None
        if not t.is_cuda or t.get_device() != self.device:
            self._refuse_device(name, t)
        if t.numel() != numel or t.dtype is not dtype or not t.is_contiguous():
            raise RRError(f"{self.what}: {name} must be dense, {numel} elements of {dtype}; got {tuple(t.shape)} {t.dtype}, "
                          f"{'dense' if t.is_contiguous() else 'not dense'}")
        return t.data_ptr()

    def workspace(self, t):
        """Address and bytes of a workspace (None, 0 for None)."""
        if t is None:
            return None, 0
        import torch
        n = t.numel()
        return self("workspace", t, n, torch.uint8), n

    def mask(self, t, numel):
        import torch
        return self("token_mask", t, numel, torch.bool if t is not None and t.dtype is torch.bool else torch.uint8)

    def stream(self):
        import torch
        return torch._C._cuda_getCurrentRawStream(self.device)

    def _refuse_device(self, name, t):
        import torch
        # (a tensor on a GPU, though the module says that it has not been initialised: initialise it and look again)
        if t.is_cuda and self.device is None:
            self.device = torch.cuda.current_device()
        if not t.is_cuda or t.get_device() != self.device:
            raise RRError(f"{self.what}: {name} is on {t.device}, not on the current GPU")


def _torch_type(dtype: int):
    import torch
    if dtype not in (RR_F32, RR_BF16):
        raise RRError(f"unsupported dtype {dtype}")
    return torch.float32 if dtype == RR_F32 else torch.bfloat16


def rr_balance_workspace_bytes(cfg: RRConfig) -> int:
    n, cc = C.c_size_t(0), cfg.c()
    _check(load_library().rr_balance_workspace_bytes(C.byref(cc), C.byref(n)), "rr_balance_workspace_bytes")
    return int(n.value)


def alloc_balance_workspace(cfg: RRConfig, device="cuda"):
    import torch
    return torch.empty(rr_balance_workspace_bytes(cfg), dtype=torch.uint8, device=device)


def rr_balance_loss(cfg: RRConfig, logits, rank_expert, coef: float, loss, counts, workspace, mean_prob=None, token_mask=None):
    """loss [1], counts [E + 1] (int32: choices per expert, then the tokens that count), mean_prob [E] or None.
    token_mask [T], uint8 or bool, or None: 0 = padding."""
    import torch
    a, f32, T, E = _Args("rr_balance_loss"), torch.float32, cfg.T, cfg.E
    args = (a("logits", logits, T * E, f32), a("rank_expert", rank_expert, T * (cfg.k + 1), torch.int32), a.mask(token_mask, T), coef,
            a("loss", loss, 1, f32), a("counts", counts, E + 1, torch.int32), a("mean_prob", mean_prob, E, f32), *a.workspace(workspace))
    cc = cfg.c()
    _check(load_library().rr_balance_loss(C.byref(cc), *args, a.stream()), "rr_balance_loss")


def rr_balance_loss_backward(cfg: RRConfig, logits, counts, coef: float, dlogits, dloss=None, token_mask=None,
                             accumulate: bool = False):
    """dlogits [T, E], written or (accumulate) added to; dloss [1] or None for 1."""
    import torch
    a, f32, T, E = _Args("rr_balance_loss_backward"), torch.float32, cfg.T, cfg.E
    args = (a("logits", logits, T * E, f32), a("counts", counts, E + 1, torch.int32), a.mask(token_mask, T), coef,
            a("dloss", dloss, 1, f32), RR_GRAD_ACCUMULATE if accumulate else 0, a("dlogits", dlogits, T * E, f32))
    cc = cfg.c()
    _check(load_library().rr_balance_loss_backward(C.byref(cc), *args, a.stream()), "rr_balance_loss_backward")


def _dropout_type(t):
    import torch
    dtype = t.dtype
    if dtype is not torch.float32 and dtype is not torch.bfloat16:
        raise RRError(f"dropout: unsupported type {dtype}")
    return RR_F32 if dtype is torch.float32 else RR_BF16


def rr_dropout(x, p: float, seed: int, offset: int, out, residual=None, device_offset=None):
    """out = residual + dropout(x), any shape; out may be x or residual.  device_offset: None or one int64 on the GPU, added to
    `offset` when the kernel runs (captured graphs).  A call uses up (x.numel() + 7) // 8 counters from `offset` on."""
    import torch
    a, dtype, n, t = _Args("rr_dropout"), _dropout_type(x), x.numel(), x.dtype
    _check(load_library().rr_dropout(n, dtype, a("x", x, n, t), a("residual", residual, n, t), p, seed, offset,
                                     a("device_offset", device_offset, 1, torch.int64), a("out", out, n, t), a.stream()), "rr_dropout")


def rr_dropout_backward(dout, p: float, seed: int, offset: int, dx, device_offset=None):
    """dx from dout with the mask of the forward call of the same p, seed and offset; dx may be dout."""
    import torch
    a, dtype, n, t = _Args("rr_dropout_backward"), _dropout_type(dout), dout.numel(), dout.dtype
    _check(load_library().rr_dropout_backward(n, dtype, a("dout", dout, n, t), p, seed, offset,
                                              a("device_offset", device_offset, 1, torch.int64), a("dx", dx, n, t), a.stream()),
           "rr_dropout_backward")


def rr_linear_workspace_bytes(cfg: RRLinearConfig, backward: bool = False) -> int:
    n, cc = C.c_size_t(0), cfg.c()
    _check(load_library().rr_linear_workspace_bytes(C.byref(cc), 1 if backward else 0, C.byref(n)), "rr_linear_workspace_bytes")
    return int(n.value)


def alloc_linear_workspace(cfg: RRLinearConfig, backward: bool = False, device="cuda"):
    import torch
    return torch.empty(rr_linear_workspace_bytes(cfg, backward), dtype=torch.uint8, device=device)


def rr_linear(cfg: RRLinearConfig, x, w, bias, residual, y, pre, workspace):
    """y = residual + act(x W^T + bias); bias, residual and pre (the pre-activations, an output) may be None."""
    import torch
    a, t, M, N, R = _Args("rr_linear"), _torch_type(cfg.dtype), cfg.M, cfg.N, cfg.rows
    args = (a("x", x, M * cfg.K, t), a("w", w, R * cfg.K, t), a("bias", bias, R, torch.float32), a("residual", residual, M * N, t),
            a("y", y, M * N, t), a("pre", pre, M * R, t), *a.workspace(workspace))
    cc = cfg.c()
    _check(load_library().rr_linear(C.byref(cc), *args, a.stream()), "rr_linear")


def rr_linear_backward(cfg: RRLinearConfig, x, w, pre, dy, dx, dw, dbias, workspace):
    """dx, dw and dbias (None: not wanted) from dy and the pre-activations of the forward call (None without an activation)."""
    import torch
    a, t, M, K, N, R = _Args("rr_linear_backward"), _torch_type(cfg.dtype), cfg.M, cfg.K, cfg.N, cfg.rows
    args = (a("x", x, M * K, t), a("w", w, R * K, t), a("pre", pre, M * R, t), a("dy", dy, M * N, t), a("dx", dx, M * K, t),
            a("dw", dw, R * K, t), a("dbias", dbias, R, torch.float32), *a.workspace(workspace))
    cc = cfg.c()
    _check(load_library().rr_linear_backward(C.byref(cc), *args, a.stream()), "rr_linear_backward")


def rr_profile_enable(on: bool):
    _check(load_library().rr_profile_enable(1 if on else 0), "rr_profile_enable")


def rr_profile_read() -> dict:
    arr = (_KernelTime * 32)()
    n = C.c_int32(0)
    _check(load_library().rr_profile_read(arr, 32, C.byref(n)), "rr_profile_read")
    return {arr[i].name.decode(): (int(arr[i].launches), float(arr[i].total_ms)) for i in range(n.value)}
