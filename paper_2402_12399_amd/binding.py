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


def _no_wrap(cfg, fields: int):
    """Refuses what the C structure would cut to 32 bits.  `fields`: all of them or-ed together; one that is negative, which may hide
    others, the library refuses itself."""
    if fields >> 31 not in (0, -1):
        raise RRError(f"{cfg}: a field does not fit in 32 bits")


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
        _no_wrap(self, self.M | self.K | self.N | self.dtype | self.act)
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


# The operators around the layer check their tensors: dense, as large as the call takes them to be, of their type, and on the current
# device, where the call is enqueued.  Small calls are bound by what the host does, hence the plain functions below (2 us a call).
_TORCH = None


def _torch():
    global _TORCH
    if _TORCH is None:
        import torch
        _TORCH = torch
    return _TORCH


def _device(what: str, t) -> int:
    """The current device; t, a tensor that the call cannot do without, must be on a GPU."""
    if t is None or not t.is_cuda:
        raise RRError(f"{what}: {'a tensor is missing' if t is None else f'a tensor is on {t.device}, not on the current GPU'}")
    return _torch()._C._cuda_getDevice()


def _addr(what: str, name: str, t, numel: int, dtype, device: int):
    """Address of t, checked, or None for None."""
    if t is None:
        return None
    if t.get_device() != device:
        raise RRError(f"{what}: {name} is on {t.device}, not on the current GPU")
    if t.numel() != numel or t.dtype is not dtype or not t.is_contiguous():
        raise RRError(f"{what}: {name} must be dense, {numel} elements of {dtype}; got {tuple(t.shape)} {t.dtype}, "
                      f"{'dense' if t.is_contiguous() else 'not dense'}")
    return t.data_ptr()


def _mask_addr(what: str, t, numel: int, device: int):
    torch = _torch()
    return _addr(what, "token_mask", t, numel, torch.bool if t is not None and t.dtype is torch.bool else torch.uint8, device)


def _work(what: str, t, device: int):
    """Address and bytes of a workspace (None, 0 for None)."""
    if t is None:
        return None, 0
    n = t.numel()
    return _addr(what, "workspace", t, n, _torch().uint8, device), n


def _stream_of(device: int) -> int:
    return _torch()._C._cuda_getCurrentRawStream(device)


def _torch_type(dtype: int):
    if dtype not in (RR_F32, RR_BF16):
        raise RRError(f"unsupported dtype {dtype}")
    return _torch().float32 if dtype == RR_F32 else _torch().bfloat16


def _balance_config(cfg: RRConfig) -> _Config:
    _no_wrap(cfg, cfg.T | cfg.E | cfg.k)
    return cfg.c()


def rr_balance_workspace_bytes(cfg: RRConfig) -> int:
    n, cc = C.c_size_t(0), _balance_config(cfg)
    _check(load_library().rr_balance_workspace_bytes(C.byref(cc), C.byref(n)), "rr_balance_workspace_bytes")
    return int(n.value)


def alloc_balance_workspace(cfg: RRConfig, device="cuda"):
    import torch
    return torch.empty(rr_balance_workspace_bytes(cfg), dtype=torch.uint8, device=device)


def rr_balance_loss(cfg: RRConfig, logits, rank_expert, coef: float, loss, counts, workspace, mean_prob=None, token_mask=None):
    """loss [1], counts [E + 1] (int32: choices per expert, then the tokens that count), mean_prob [E] or None.
    token_mask [T], uint8 or bool, or None: 0 = padding."""
    me, f32, i32, T, E = "rr_balance_loss", _torch().float32, _torch().int32, cfg.T, cfg.E
    d = _device(me, logits)
    ws, size = _work(me, workspace, d)
    cc = _balance_config(cfg)
    _check(load_library().rr_balance_loss(
        C.byref(cc), _addr(me, "logits", logits, T * E, f32, d), _addr(me, "rank_expert", rank_expert, T * (cfg.k + 1), i32, d),
        _mask_addr(me, token_mask, T, d), coef, _addr(me, "loss", loss, 1, f32, d), _addr(me, "counts", counts, E + 1, i32, d),
        _addr(me, "mean_prob", mean_prob, E, f32, d), ws, size, _stream_of(d)), me)


def rr_balance_loss_backward(cfg: RRConfig, logits, counts, coef: float, dlogits, dloss=None, token_mask=None,
                             accumulate: bool = False):
    """dlogits [T, E], written or (accumulate) added to; dloss [1] or None for 1."""
    me, f32, T, E = "rr_balance_loss_backward", _torch().float32, cfg.T, cfg.E
    d = _device(me, logits)
    cc = _balance_config(cfg)
    _check(load_library().rr_balance_loss_backward(
        C.byref(cc), _addr(me, "logits", logits, T * E, f32, d), _addr(me, "counts", counts, E + 1, _torch().int32, d),
        _mask_addr(me, token_mask, T, d), coef, _addr(me, "dloss", dloss, 1, f32, d), RR_GRAD_ACCUMULATE if accumulate else 0,
        _addr(me, "dlogits", dlogits, T * E, f32, d), _stream_of(d)), me)


def _dropout_type(what: str, t):
    dtype = t.dtype
    if dtype is not _torch().float32 and dtype is not _torch().bfloat16:
        raise RRError(f"{what}: unsupported type {dtype}")
    return dtype, RR_F32 if dtype is _torch().float32 else RR_BF16


def _check_seed(what: str, seed: int):
    """Refuses what the C call would cut to 64 bits.  (A negative number that fits is the unsigned one of the same bits.)"""
    if not -1 << 63 <= seed < 1 << 64:
        raise RRError(f"{what}: seed {seed} does not fit in 64 bits")


def rr_dropout(x, p: float, seed: int, offset: int, out, residual=None, device_offset=None):
    """out = residual + dropout(x), any shape; out may be x or residual.  device_offset: None or one int64 on the GPU, added to
    `offset` when the kernel runs (captured graphs).  A call uses up (x.numel() + 7) // 8 counters from `offset` on.  A seed has
    64 bits, or is refused; counters, and `offset` with them, are taken modulo 2^64."""
    me, n = "rr_dropout", x.numel()
    t, dtype = _dropout_type(me, x)
    _check_seed(me, seed)
    d = _device(me, x)
    _check(load_library().rr_dropout(
        n, dtype, _addr(me, "x", x, n, t, d), _addr(me, "residual", residual, n, t, d), p, seed, offset,
        _addr(me, "device_offset", device_offset, 1, _torch().int64, d), _addr(me, "out", out, n, t, d), _stream_of(d)), me)


def rr_dropout_backward(dout, p: float, seed: int, offset: int, dx, device_offset=None):
    """dx from dout with the mask of the forward call of the same p, seed and offset; dx may be dout."""
    me, n = "rr_dropout_backward", dout.numel()
    t, dtype = _dropout_type(me, dout)
    _check_seed(me, seed)
    d = _device(me, dout)
    _check(load_library().rr_dropout_backward(
        n, dtype, _addr(me, "dout", dout, n, t, d), p, seed, offset,
        _addr(me, "device_offset", device_offset, 1, _torch().int64, d), _addr(me, "dx", dx, n, t, d), _stream_of(d)), me)


def rr_linear_workspace_bytes(cfg: RRLinearConfig, backward: bool = False) -> int:
    n, cc = C.c_size_t(0), cfg.c()
    _check(load_library().rr_linear_workspace_bytes(C.byref(cc), 1 if backward else 0, C.byref(n)), "rr_linear_workspace_bytes")
    return int(n.value)


def alloc_linear_workspace(cfg: RRLinearConfig, backward: bool = False, device="cuda"):
    import torch
    return torch.empty(rr_linear_workspace_bytes(cfg, backward), dtype=torch.uint8, device=device)


def rr_linear(cfg: RRLinearConfig, x, w, bias, residual, y, pre, workspace):
    """y = residual + act(x W^T + bias); bias, residual and pre (the pre-activations, an output) may be None."""
    me, t, M, K, N, R = "rr_linear", _torch_type(cfg.dtype), cfg.M, cfg.K, cfg.N, cfg.rows
    d = _device(me, x)
    ws, size = _work(me, workspace, d)
    cc = cfg.c()
    _check(load_library().rr_linear(
        C.byref(cc), _addr(me, "x", x, M * K, t, d), _addr(me, "w", w, R * K, t, d), _addr(me, "bias", bias, R, _torch().float32, d),
        _addr(me, "residual", residual, M * N, t, d), _addr(me, "y", y, M * N, t, d), _addr(me, "pre", pre, M * R, t, d), ws, size,
        _stream_of(d)), me)


def rr_linear_backward(cfg: RRLinearConfig, x, w, pre, dy, dx, dw, dbias, workspace):
    """dx, dw and dbias (None: not wanted) from dy and the pre-activations of the forward call (None without an activation)."""
    me, t, M, K, N, R = "rr_linear_backward", _torch_type(cfg.dtype), cfg.M, cfg.K, cfg.N, cfg.rows
    d = _device(me, dy)
    ws, size = _work(me, workspace, d)
    cc = cfg.c()
    _check(load_library().rr_linear_backward(
        C.byref(cc), _addr(me, "x", x, M * K, t, d), _addr(me, "w", w, R * K, t, d), _addr(me, "pre", pre, M * R, t, d),
        _addr(me, "dy", dy, M * N, t, d), _addr(me, "dx", dx, M * K, t, d), _addr(me, "dw", dw, R * K, t, d),
        _addr(me, "dbias", dbias, R, _torch().float32, d), ws, size, _stream_of(d)), me)


def rr_profile_enable(on: bool):
    _check(load_library().rr_profile_enable(1 if on else 0), "rr_profile_enable")


def rr_profile_read() -> dict:
    arr = (_KernelTime * 32)()
    n = C.c_int32(0)
    _check(load_library().rr_profile_read(arr, 32, C.byref(n)), "rr_profile_read")
    return {arr[i].name.decode(): (int(arr[i].launches), float(arr[i].total_ms)) for i in range(n.value)}
