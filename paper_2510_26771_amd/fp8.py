"""8-bit floating point layers with block scales, dense and by expert, the router and the experts' MLP (include/stamp.h).

Like binding.StampPlan: argument checks and marshalling only, no fallback; all tensors of a call live on the plan's (the routing's) GPU,
which is the current one, and calls are asynchronous on the given stream of it (default: torch's current one)."""
from __future__ import annotations

import ctypes as C
from dataclasses import dataclass

from .binding import STAMP_BF16, STAMP_F32, _check, _ptr, _stream, load_library

STAMP_E4M3 = 2
STAMP_SCALE_F32, STAMP_SCALE_POW2 = 0, 1
BLOCK = 128
FP8_ROUTES = {1: "rows", 2: "tiles_64", 3: "tiles_128", 4: "tiles_256"}  # stamp_fp8_route_t


class _Desc(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("d_in", "d_out", "experts", "gated", "x_dtype", "y_dtype", "w_dtype", "w_is_out_by_in", "scale_format")]


class _Routing(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("tokens", "experts", "top_k")] + [
        (n, C.c_void_p) for n in ("ids", "weights", "offsets", "token_of_row", "row_of_slot")]


@dataclass
class Fp8Desc:
    d_in: int
    d_out: int
    experts: int = 0          # 0: one layer
    gated: int = 0            # 1: gate and up matrices, for experts_forward
    x_dtype: int = STAMP_BF16
    y_dtype: int = STAMP_BF16
    w_dtype: int = STAMP_E4M3
    w_is_out_by_in: int = 1
    scale_format: int = STAMP_SCALE_F32

    def to_c(self) -> _Desc:
        return _Desc(**{n: int(getattr(self, n)) for n, _ in _Desc._fields_})


def _torch_dtype(code):
    import torch
    return torch.bfloat16 if code == STAMP_BF16 else torch.float32


# gpu: index of the plan's (the routing's) GPU; get_device() is -1 for tensors of the host
def _matrix(t, name, rows, cols, dtype, gpu):
    """A [rows, cols] tensor of that type on that GPU whose rows are contiguous; returns the distance of its rows in elements."""
    if t.get_device() != gpu or t.shape != (rows, cols):
        raise ValueError(f"{name} must be a tensor of shape ({rows}, {cols}) on GPU {gpu}")
    if t.dtype != dtype:
        raise ValueError(f"{name} must be {dtype}, not {t.dtype}")
    if cols > 1 and t.stride(1) != 1:
        raise ValueError(f"{name}'s rows must be contiguous")
    return t.stride(0) if rows > 1 else cols


def _flat(t, name, numel, dtype, gpu):
    if t.get_device() != gpu or t.dtype != dtype or t.numel() != numel or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous tensor of {numel} {dtype} on GPU {gpu}")


def _room(t, gpu):
    """Bytes of a workspace."""
    if t is None or t.get_device() != gpu or not t.is_contiguous():
        raise ValueError(f"workspace must be a contiguous tensor on GPU {gpu}")
    return t.nbytes


class Fp8Plan:
    """Owns a stamp_fp8_plan_t: the weights of one layer, or of all experts of one layer.  W, w_scales and bias are read on the stream: with
    a stream of one's own they have to live until it has drained."""

    def __init__(self, desc: Fp8Desc, W, w_scales=None, bias=None, stream=None):
        import torch
        self.lib = load_library()
        self.desc = d = desc
        self._h = C.c_void_p()
        mats = max(d.experts, 1) * (2 if d.gated else 1)
        kinds = {STAMP_F32: (torch.float32,), STAMP_BF16: (torch.bfloat16,), STAMP_E4M3: (torch.float8_e4m3fn, torch.uint8)}
        if W is None or not W.is_cuda or not W.is_contiguous():
            raise ValueError("W must be a contiguous GPU tensor: the library has no host path")
        if W.dtype not in kinds.get(d.w_dtype, (W.dtype,)):
            raise ValueError(f"W is {W.dtype}, the description says otherwise")
        if W.numel() != mats * d.d_in * d.d_out or W.dim() < 2 or tuple(W.shape[-2:]) != ((d.d_out, d.d_in) if d.w_is_out_by_in else (d.d_in, d.d_out)):
            raise ValueError("W's shape is not the description's")
        self.gpu = W.get_device()
        if w_scales is not None:
            _flat(w_scales, "w_scales", mats * -(-d.d_out // BLOCK) * -(-d.d_in // BLOCK), torch.float32, self.gpu)
        if bias is not None:
            _flat(bias, "bias", max(d.experts, 1) * d.d_out, torch.float32, self.gpu)
        _check(self.lib.stamp_fp8_plan_create(C.byref(d.to_c()), _ptr(W), _ptr(w_scales), _ptr(bias), _stream(stream, self.gpu), C.byref(self._h)),
               "stamp_fp8_plan_create")
        self._x_dtype, self._y_dtype = _torch_dtype(d.x_dtype), _torch_dtype(d.y_dtype)

    def destroy(self):
        if self._h:
            self.lib.stamp_fp8_plan_destroy(self._h)
            self._h = C.c_void_p()

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass

    # -- queries --
    def workspace_bytes(self, rows: int) -> int:
        return int(self.lib.stamp_fp8_workspace_bytes(self._h, int(rows)))

    def alloc_workspace(self, rows: int, device="cuda"):
        import torch
        return torch.empty(max(self.workspace_bytes(rows), 256), dtype=torch.uint8, device=device)

    def route(self, rows: int) -> str:
        """Name (FP8_ROUTES) of the kernel that a call with so many rows runs."""
        return FP8_ROUTES[int(self.lib.stamp_fp8_debug_route(self._h, int(rows)))]

    def cut(self, rows: int) -> tuple:
        """(columns of the first of two launches or 0, parts of the depth in the first, in the second) of a call in tiles; zeros else."""
        out = (C.c_int32 * 3)()
        _check(self.lib.stamp_fp8_debug_cut(self._h, int(rows), out), "stamp_fp8_debug_cut")
        return tuple(out)

    def set_route(self, route: str = ""):
        """For tests and measurements: that kernel for every call ("": by rule)."""
        code = {n: c for c, n in FP8_ROUTES.items()}[route] if route else 0
        _check(self.lib.stamp_fp8_debug_set_route(self._h, code), "stamp_fp8_debug_set_route")

    # -- compute (asynchronous on the stream) --
    def alloc_act_buffers(self, rows: int, device="cuda"):
        """Codes [rows, d_in rounded up to 128] and scales [blocks, rows rounded up to 4] for quantize_act."""
        import torch
        kb = -(-self.desc.d_in // BLOCK)
        return (torch.empty((rows, kb * BLOCK), dtype=torch.uint8, device=device),
                torch.empty((kb, -(-max(rows, 1) // 4) * 4), dtype=torch.float32, device=device))

    def _act_buffers(self, codes, scales, rows):
        import torch
        kb = -(-self.desc.d_in // BLOCK)
        _flat(codes, "codes", rows * kb * BLOCK, torch.uint8, self.gpu)
        if scales.get_device() != self.gpu or scales.dtype != torch.float32 or scales.dim() != 2 or scales.shape[0] != kb or not scales.is_contiguous():
            raise ValueError(f"scales must be a contiguous tensor of {kb} rows of float32 on GPU {self.gpu}")
        return scales.shape[1]

    def _x(self, X, rows):
        return _matrix(X, "X", rows, self.desc.d_in, self._x_dtype, self.gpu)

    def _y(self, Y, rows):
        return _matrix(Y, "Y", rows, self.desc.d_out, self._y_dtype, self.gpu)

    def quantize_act(self, X, codes, scales, stream=None):
        ld = self._x(X, X.shape[0])
        lds = self._act_buffers(codes, scales, X.shape[0])
        _check(self.lib.stamp_fp8_quantize_act(self._h, X.shape[0], _ptr(X), ld, _ptr(codes), _ptr(scales), lds, _stream(stream, self.gpu)),
               "stamp_fp8_quantize_act")

    def linear_forward(self, X, Y, workspace, stream=None):
        rows = X.shape[0]
        ld_x, ld_y, room = self._x(X, rows), self._y(Y, rows), _room(workspace, self.gpu)
        _check(self.lib.stamp_fp8_linear_forward(self._h, rows, _ptr(X), ld_x, _ptr(Y), ld_y, _ptr(workspace), room, _stream(stream, self.gpu)),
               "stamp_fp8_linear_forward")

    def linear_forward_q(self, codes, scales, Y, workspace, stream=None):
        rows = Y.shape[0]
        lds, ld_y, room = self._act_buffers(codes, scales, rows), self._y(Y, rows), _room(workspace, self.gpu)
        _check(self.lib.stamp_fp8_linear_forward_q(self._h, rows, _ptr(codes), _ptr(scales), lds, _ptr(Y), ld_y, _ptr(workspace),
                                                   room, _stream(stream, self.gpu)), "stamp_fp8_linear_forward_q")

    def grouped_forward(self, X, offsets, Y, workspace, stream=None):
        """Rows offsets[e] .. offsets[e + 1] - 1 of X times expert e's weights."""
        import torch
        rows = X.shape[0]
        ld_x, ld_y, room = self._x(X, rows), self._y(Y, rows), _room(workspace, self.gpu)
        _flat(offsets, "offsets", self.desc.experts + 1, torch.int32, self.gpu)
        _check(self.lib.stamp_fp8_grouped_forward(self._h, rows, _ptr(offsets), _ptr(X), ld_x, _ptr(Y), ld_y, _ptr(workspace),
                                                  room, _stream(stream, self.gpu)), "stamp_fp8_grouped_forward")

    def debug_weight_codes(self):
        """Codes (bytes) [experts][2 if gated][d_out][d_in] and scales [..][blocks of d_out][blocks of d_in], on the host."""
        import numpy as np
        d = self.desc
        lead = ((d.experts,) if d.experts else ()) + ((2,) if d.gated else ())
        codes = np.empty(lead + (d.d_out, d.d_in), dtype=np.uint8)
        scales = np.empty(lead + (-(-d.d_out // BLOCK), -(-d.d_in // BLOCK)), dtype=np.float32)
        _check(self.lib.stamp_fp8_debug_weight_codes(self._h, codes.ctypes.data, scales.ctypes.data), "stamp_fp8_debug_weight_codes")
        return codes, scales


class Routing:
    """What route_topk writes (stamp_routing_t) and its workspace; one object serves any number of calls of its sizes."""

    def __init__(self, tokens: int, experts: int, top_k: int, device="cuda"):
        import torch
        if torch.device(device).type != "cuda":
            raise ValueError("a routing lives on a GPU")
        self.lib = load_library()
        self.tokens, self.experts, self.top_k = int(tokens), int(experts), int(top_k)
        need = int(self.lib.stamp_route_workspace_bytes(self.tokens, self.experts, self.top_k))
        if need == 0:
            raise ValueError("tokens, experts or top_k out of range")

        def ints(*shape):
            return torch.empty(shape, dtype=torch.int32, device=device)
        self.ids, self.row_of_slot = ints(tokens, top_k), ints(tokens, top_k)
        self.weights = torch.empty((tokens, top_k), dtype=torch.float32, device=device)
        self.offsets, self.token_of_row = ints(experts + 1), ints(tokens * top_k)
        self.workspace = torch.empty(need, dtype=torch.uint8, device=device)
        self.gpu = self.workspace.get_device()
        self._c = _Routing(self.tokens, self.experts, self.top_k, _ptr(self.ids), _ptr(self.weights), _ptr(self.offsets), _ptr(self.token_of_row),
                           _ptr(self.row_of_slot))


def route_topk(logits, routing: Routing, renormalize: bool = True, stream=None):
    """The top_k experts of every token, their weights, and the order of the rows by expert -> routing."""
    import torch
    if logits.dtype not in (torch.float32, torch.bfloat16):
        raise ValueError("logits must be float32 or bfloat16")
    ld = _matrix(logits, "logits", routing.tokens, routing.experts, logits.dtype, routing.gpu)
    _check(routing.lib.stamp_route_topk(C.byref(routing._c), _ptr(logits), STAMP_BF16 if logits.dtype == torch.bfloat16 else STAMP_F32, ld,
                                        int(bool(renormalize)), _ptr(routing.workspace), routing.workspace.numel(), _stream(stream, routing.gpu)), "stamp_route_topk")


def experts_workspace(up: Fp8Plan, down: Fp8Plan, tokens: int, top_k: int, device="cuda"):
    import torch
    n = int(up.lib.stamp_experts_workspace_bytes(up._h, down._h, int(tokens), int(top_k)))
    return torch.empty(max(n, 256), dtype=torch.uint8, device=device)


def experts_forward(up: Fp8Plan, down: Fp8Plan, X, routing: Routing, Y, workspace, stream=None):
    """The gated MLP of the chosen experts of every token, summed with their weights."""
    if down.gpu != up.gpu or routing.gpu != up.gpu:
        raise ValueError("both plans and the routing must lie on one GPU")
    ld_x, ld_y, room = up._x(X, routing.tokens), down._y(Y, routing.tokens), _room(workspace, up.gpu)
    _check(up.lib.stamp_experts_forward(up._h, down._h, C.byref(routing._c), _ptr(X), ld_x, _ptr(Y), ld_y, _ptr(workspace), room,
                                        _stream(stream, up.gpu)), "stamp_experts_forward")
