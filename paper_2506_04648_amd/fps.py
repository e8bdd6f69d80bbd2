"""Thin ctypes binding over libfps (argument marshalling only; every step runs in the HIP kernels).

PyTorch is used for device memory and streams.  There is no CPU fallback: if the shared library
has not been built (see `paper_2506_04648_amd.build`), loading fails with an error.
"""
from __future__ import annotations

import ctypes
import os

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libfps.so")

FPS_OK = 0
FPS_ERR_INVALID_ARG = -1
FPS_ERR_UNSUPPORTED = -2
FPS_ERR_WORKSPACE = -3
FPS_ERR_HIP = -4

PREC_BF16, PREC_FP8 = 0, 1
VSCALE_TILE, VSCALE_CHANNEL = 0, 1
ROLE_Q, ROLE_K, ROLE_V = 0, 1, 2
OUT_BF16, OUT_F32 = 0, 1
PAIRS_ADJACENT, PAIRS_HALVES = 0, 1
LAYOUT_TILED, LAYOUT_RASTER = 0, 1
EDGE_TRUNCATE, EDGE_SHIFT = 0, 1

EXPORTS = ("fps_last_error", "fps_schedule_select", "fps_num_tiles", "fps_num_groups", "fps_tile_slots",
           "fps_block_slots", "fps_packed_bytes",
           "fps_tile_mask_host", "fps_tile_order", "fps_tile_unorder", "fps_quantize_tiles",
           "fps_quantize_raster",
           "fps_pack_tiles_bf16", "fps_pack_raster_bf16", "fps_debug_unpack_q8", "fps_debug_copy", "fps_debug_scores_q8",
           "fps_debug_scores_block_q8", "fps_debug_mfma_rate", "fps_debug_issue_mix",
           "fps_attn_fwd", "fps_rotation_floats", "fps_rotation_table_host", "fps_norm_rotate", "fps_norm_rotate_operand",
           "fps_norm_rotate_bwd_bytes", "fps_norm_rotate_bwd", "fps_dequantize", "fps_mx4_bytes", "fps_mx4_quantize",
           "fps_mx4_dequantize", "fps_mx4_matmul", "fps_mx4_linear_bytes", "fps_mx4_linear")
SIZES = ("fps_num_tiles", "fps_num_groups", "fps_tile_slots", "fps_block_slots", "fps_packed_bytes", "fps_rotation_floats",
         "fps_norm_rotate_bwd_bytes", "fps_mx4_bytes", "fps_mx4_linear_bytes")                      # exports that return a size, 0 for a refusal


class Shape(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int) for n in ("B", "heads", "head_dim", "T", "H", "W", "Tt", "Th", "Tw",
                                            "Qt", "Qh", "Qw")]


class Window(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int) for n in ("wt", "wh", "ww", "edge")]


class Regime(ctypes.Structure):
    _fields_ = [("prec", ctypes.c_int), ("win", Window)] + [(n, ctypes.c_int) for n in
                                                            ("Tt", "Th", "Tw", "Qt", "Qh", "Qw")]


class StepCfg(ctypes.Structure):
    _fields_ = [("step", ctypes.c_int), ("num_steps", ctypes.c_int), ("alpha1", ctypes.c_float),
                ("alpha2", ctypes.c_float), ("regime", Regime * 3)]


class View(ctypes.Structure):
    _fields_ = ([("data", ctypes.c_void_p)] + [(n, ctypes.c_int) for n in ("dt", "B", "heads", "rows", "cols")]
                + [(n, ctypes.c_int64) for n in ("stride_b", "stride_h", "stride_r")])


class Norm(ctypes.Structure):
    _fields_ = [("weight", ctypes.c_void_p), ("per_head", ctypes.c_int), ("eps", ctypes.c_float)]


class Rotation(ctypes.Structure):
    _fields_ = ([("table", ctypes.c_void_p), ("stride_b", ctypes.c_int64)]
                + [(n, ctypes.c_int) for n in ("pairs_t", "pairs_h", "pairs_w", "pairing")])


class FpsError(RuntimeError):
    def __init__(self, status, text):
        super().__init__(f"libfps status {status}: {text}")
        self.status = status


_lib = None
_torch = None                                  # the module, once a device entry point has needed it
_written = None                                # marks what a call has written into: autograd then takes it no longer for what it saved
_codes = {}                                    # of torch's types, from then on


def _import_torch():
    global _torch, _written
    if _torch is None:
        import torch
        _torch, _written = torch, torch.autograd.graph.increment_version
    return _torch


def lib():
    """Load libfps.so (once).  Raises if it is not built: the product path has no fallback."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise FileNotFoundError(
                f"{LIB_PATH} not found: build it with `python -c 'import __graft_entry__ as g; g.build()'`")
        L = ctypes.CDLL(LIB_PATH)
        vp, ip, fp = ctypes.c_void_p, ctypes.c_int, ctypes.POINTER(ctypes.c_float)
        L.fps_last_error.restype = ctypes.c_char_p
        L.fps_last_error.argtypes = []
        L.fps_schedule_select.argtypes = [ctypes.POINTER(StepCfg), ctypes.POINTER(Regime)]
        L.fps_num_tiles.argtypes = [ctypes.POINTER(Shape)]
        L.fps_num_groups.argtypes = [ctypes.POINTER(Shape)]
        L.fps_tile_slots.argtypes = [ctypes.POINTER(Shape)]
        L.fps_block_slots.argtypes = [ctypes.POINTER(Shape)]
        L.fps_packed_bytes.argtypes = [ctypes.POINTER(Shape), ip]
        L.fps_tile_mask_host.argtypes = [ctypes.POINTER(Shape), ctypes.POINTER(Window), vp,
                                         ctypes.POINTER(ctypes.c_uint64)]
        L.fps_tile_order.argtypes = [ctypes.POINTER(Shape), vp, vp, vp]
        L.fps_tile_unorder.argtypes = [ctypes.POINTER(Shape), vp, ip, vp, vp]
        L.fps_quantize_tiles.argtypes = [ctypes.POINTER(Shape), vp, ip, ip, vp, vp, vp]
        L.fps_quantize_raster.argtypes = [ctypes.POINTER(Shape), vp, ip, ip, vp, vp, vp]
        L.fps_pack_tiles_bf16.argtypes = [ctypes.POINTER(Shape), vp, ip, vp, vp, vp]
        L.fps_pack_raster_bf16.argtypes = [ctypes.POINTER(Shape), vp, ip, vp, vp, vp]
        L.fps_debug_unpack_q8.argtypes = [ctypes.POINTER(Shape), vp, ip, vp, vp]
        L.fps_debug_copy.argtypes = [vp, vp, ctypes.c_size_t, vp]
        L.fps_debug_scores_q8.argtypes = [ctypes.POINTER(Shape), vp, vp, ip, ip, ip, vp, vp]
        L.fps_debug_scores_block_q8.argtypes = [ctypes.POINTER(Shape), vp, vp, ip, ip, ip, ip, ip, vp,
                                                ctypes.POINTER(ctypes.c_int), vp]
        L.fps_debug_mfma_rate.argtypes = [ip, ip, vp, vp]
        L.fps_debug_issue_mix.argtypes = [ip, ip, ip, ip, ip, ip, vp, vp, vp]
        L.fps_attn_fwd.argtypes = [ctypes.POINTER(Shape), ctypes.POINTER(Window), ip,
                                   ctypes.POINTER(StepCfg), vp, vp, vp, vp, vp, vp, ip, vp, ip, ip, vp, vp]
        shape, view, norm, rot = (ctypes.POINTER(t) for t in (Shape, View, Norm, Rotation))
        L.fps_rotation_floats.argtypes = [shape, rot]
        L.fps_rotation_table_host.argtypes = [shape, rot, ctypes.POINTER(ctypes.c_int64), ctypes.c_double, vp]
        L.fps_norm_rotate.argtypes = [shape, view, norm, rot, view, vp]
        L.fps_norm_rotate_operand.argtypes = [shape, view, norm, rot, ip, ip, vp, vp, vp]
        L.fps_norm_rotate_bwd_bytes.argtypes = [shape, norm]
        L.fps_norm_rotate_bwd.argtypes = [shape, view, norm, rot, view, view, vp, vp, ctypes.c_size_t, vp]
        L.fps_dequantize.argtypes = [shape, vp, vp, ip, ip, ip, vp, vp]
        L.fps_mx4_bytes.argtypes = L.fps_mx4_linear_bytes.argtypes = [ctypes.c_int64, ctypes.c_int64]
        L.fps_mx4_quantize.argtypes = [view, vp, vp]
        L.fps_mx4_dequantize.argtypes = [vp, view, vp]
        L.fps_mx4_matmul.argtypes = [ctypes.c_int64, vp, vp, vp, view, vp]
        L.fps_mx4_linear.argtypes = [view, vp, vp, view, vp, ctypes.c_size_t, vp]
        for name in EXPORTS:
            if name != "fps_last_error":
                getattr(L, name).restype = ctypes.c_size_t if name in SIZES else ctypes.c_int
        _lib = L
    return _lib


def last_error() -> str:
    return lib().fps_last_error().decode()


def _check(status):
    if status != FPS_OK:
        raise FpsError(status, last_error())


def make_shape(heads, grid, tile, B=1, head_dim=128, qtile=None) -> Shape:
    """qtile: quantisation sub-tile (it must divide the tile); None = one scale per tile."""
    q = (0, 0, 0) if qtile is None else tuple(qtile)
    return Shape(B, heads, head_dim, grid[0], grid[1], grid[2], tile[0], tile[1], tile[2], q[0], q[1], q[2])


def make_step_cfg(step, num_steps, alpha1, alpha2, regimes) -> StepCfg:
    """regimes: three (prec, (wt, wh, ww[, edge])[, (Tt, Th, Tw)[, (Qt, Qh, Qw)]]) entries for the
    early, mid and late steps (Eq. 6); the optional items are the regime's granularity g(t): its
    tile and its quantisation sub-tile."""
    cfg = StepCfg()
    cfg.step, cfg.num_steps, cfg.alpha1, cfg.alpha2 = step, num_steps, alpha1, alpha2
    for i, reg in enumerate(regimes):
        cfg.regime[i].prec = reg[0]
        cfg.regime[i].win = Window(*reg[1])
        if len(reg) > 2 and reg[2] is not None:
            cfg.regime[i].Tt, cfg.regime[i].Th, cfg.regime[i].Tw = reg[2]
        if len(reg) > 3 and reg[3] is not None:
            cfg.regime[i].Qt, cfg.regime[i].Qh, cfg.regime[i].Qw = reg[3]
    return cfg


def _stream(device=None):
    # the handle alone: building a Stream object around it takes 3 us, as long as the launch itself
    torch = _torch or _import_torch()
    raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)      # not in torch's documented interface
    return raw(torch.cuda.current_device() if device is None else device) if raw else torch.cuda.current_stream().cuda_stream


def _ptr(t):
    return t.data_ptr() if t is not None else None


# ---- host helpers ---------------------------------------------------------------------------
def schedule_select(cfg: StepCfg, with_tile=False):
    """(prec, window) of the step's regime; with_tile=True appends its tile (Tt, Th, Tw) or None,
    and its quantisation sub-tile if it names one."""
    out = Regime()
    _check(lib().fps_schedule_select(ctypes.byref(cfg), ctypes.byref(out)))
    win = (out.win.wt, out.win.wh, out.win.ww) + ((out.win.edge,) if out.win.edge else ())
    if with_tile:
        tile = (out.Tt, out.Th, out.Tw) if out.Tt else None
        if out.Qt:
            return out.prec, win, tile, (out.Qt, out.Qh, out.Qw)
        return out.prec, win, tile
    return out.prec, win


def num_tiles(shape: Shape) -> int:
    return int(lib().fps_num_tiles(ctypes.byref(shape)))


def num_groups(shape: Shape) -> int:
    """Quantisation groups (scales) per head: one per tile, or per sub-tile of each tile."""
    return int(lib().fps_num_groups(ctypes.byref(shape)))


def tile_slots(shape: Shape) -> int:
    """Slots one tile occupies in tiled and packed tensors (its tokens rounded up to whole blocks)."""
    return int(lib().fps_tile_slots(ctypes.byref(shape)))


def packed_bytes(shape: Shape, prec: int) -> int:
    return int(lib().fps_packed_bytes(ctypes.byref(shape), prec))


def tile_mask_host(shape: Shape, window):
    import numpy as np
    M = num_tiles(shape)
    if M == 0:
        raise FpsError(FPS_ERR_INVALID_ARG, last_error())
    mask = np.zeros((M, M), dtype=np.uint8)
    pairs = ctypes.c_uint64(0)
    win = Window(*window)
    _check(lib().fps_tile_mask_host(ctypes.byref(shape), ctypes.byref(win),
                                    mask.ctypes.data_as(ctypes.c_void_p), ctypes.byref(pairs)))
    return mask, int(pairs.value)


# ---- device entry points (torch tensors on the current device) --------------------------------
def _tiled_len(shape: Shape) -> int:
    n = num_tiles(shape) * tile_slots(shape)
    if n == 0:
        raise FpsError(FPS_ERR_INVALID_ARG, last_error())
    return n


def tile_order(shape: Shape, x_raster, out=None):
    import torch
    assert x_raster.dtype == torch.bfloat16 and x_raster.is_cuda and x_raster.is_contiguous()
    if out is None:
        out = torch.empty((shape.B, shape.heads, _tiled_len(shape), shape.head_dim),
                          dtype=torch.bfloat16, device=x_raster.device)
    _check(lib().fps_tile_order(ctypes.byref(shape), _ptr(x_raster), _ptr(out), _stream()))
    return out


def tile_unorder(shape: Shape, o_tiled, out=None):
    import torch
    assert o_tiled.is_cuda and o_tiled.is_contiguous()
    dt = OUT_F32 if o_tiled.dtype == torch.float32 else OUT_BF16
    if out is None:
        out = torch.empty((shape.B, shape.heads, shape.T, shape.H, shape.W, shape.head_dim),
                          dtype=o_tiled.dtype, device=o_tiled.device)
    _check(lib().fps_tile_unorder(ctypes.byref(shape), _ptr(o_tiled), dt, _ptr(out), _stream()))
    return out


def quantize_tiles(shape: Shape, x_tiled, role, vscale=VSCALE_TILE, out=None, scales=None,
                   raster=False):
    """Per-tile FP8 quantisation of a tile-ordered tensor, or (raster=True) of a raster tensor with
    the tile ordering fused in.  Returns (packed codes, scales)."""
    torch = _torch or _import_torch()
    assert x_tiled.dtype == torch.bfloat16 and x_tiled.is_cuda and x_tiled.is_contiguous()
    if out is None:
        out = torch.empty(packed_bytes(shape, PREC_FP8), dtype=torch.uint8, device=x_tiled.device)
    if scales is None:
        n = shape.head_dim if (role == ROLE_V and vscale == VSCALE_CHANNEL) else num_groups(shape)
        scales = torch.empty((shape.B, shape.heads, n), dtype=torch.float32, device=x_tiled.device)
    fn = lib().fps_quantize_raster if raster else lib().fps_quantize_tiles
    _check(fn(shape, x_tiled.data_ptr(), role, vscale, out.data_ptr(), scales.data_ptr(), _stream()))
    return out, scales


def pack_tiles_bf16(shape: Shape, x_tiled, role, out=None, vscale=None, raster=False):
    """BF16-mode operand packing of a tile-ordered tensor, or (raster=True) of a raster tensor with
    the tile ordering fused in.  Returns (packed tensor, per-group V scales or None)."""
    torch = _torch or _import_torch()
    assert x_tiled.dtype == torch.bfloat16 and x_tiled.is_cuda and x_tiled.is_contiguous()
    if out is None:
        out = torch.empty(packed_bytes(shape, PREC_BF16), dtype=torch.uint8, device=x_tiled.device)
    if role == ROLE_V and vscale is None:
        vscale = torch.empty((shape.B, shape.heads, num_groups(shape)), dtype=torch.float32,
                             device=x_tiled.device)
    fn = lib().fps_pack_raster_bf16 if raster else lib().fps_pack_tiles_bf16
    _check(fn(shape, x_tiled.data_ptr(), role, out.data_ptr(), _ptr(vscale), _stream()))
    return out, vscale


def debug_unpack_q8(shape: Shape, xq, role):
    import torch
    out = torch.empty((shape.B, shape.heads, _tiled_len(shape), shape.head_dim), dtype=torch.uint8,
                      device=xq.device)
    _check(lib().fps_debug_unpack_q8(ctypes.byref(shape), _ptr(xq), role, _ptr(out), _stream()))
    return out


def debug_copy(src, dst):
    assert src.is_cuda and dst.is_cuda and src.is_contiguous() and dst.is_contiguous()
    nbytes = src.numel() * src.element_size()
    assert nbytes == dst.numel() * dst.element_size()
    _check(lib().fps_debug_copy(_ptr(src), _ptr(dst), nbytes, _stream()))
    return dst


def debug_mfma_rate(workgroups, iters, sink):
    """Launch the MFMA-only kernel; returns the FLOPs it executes (the caller times it)."""
    assert sink.is_cuda and sink.numel() >= workgroups * 256
    _check(lib().fps_debug_mfma_rate(workgroups, iters, _ptr(sink), _stream()))
    return workgroups * 4 * iters * 8 * 65536.0


def debug_issue_mix(matrix_kind, valu_per_mfma, valu_kind, workgroups_per_cu, workgroups, iters, sink, cycles):
    """One launch of the matrix/vector issue-mix kernel; cycles (int64, workgroups*4) receives each
    wave's shader clocks for iters*8 groups."""
    _check(lib().fps_debug_issue_mix(matrix_kind, valu_per_mfma, valu_kind, workgroups_per_cu, workgroups,
                                     iters, _ptr(sink), _ptr(cycles), _stream()))


def debug_scores_q8(shape: Shape, q8, k8, bh, u, v):
    import torch
    ts = tile_slots(shape)
    out = torch.empty((ts, ts), dtype=torch.float32, device=q8.device)
    _check(lib().fps_debug_scores_q8(ctypes.byref(shape), _ptr(q8), _ptr(k8), bh, u, v, _ptr(out),
                                     _stream()))
    return out


def block_slots(shape: Shape) -> int:
    """BS, the slots of one block, as the library lays tensors out (128 or 32)."""
    n = lib().fps_block_slots(ctypes.byref(shape))
    if n == 0:
        raise FpsError(FPS_ERR_INVALID_ARG, last_error())
    return int(n)


def debug_scores_block_q8(shape: Shape, q8, k8, bh, u, jq, v, jk, out=None):
    """Raw score accumulators of one (query block, key block) pair; returns a [BS, BS] tensor."""
    import torch
    bs = block_slots(shape)
    if out is None:
        out = torch.empty((bs, bs), dtype=torch.float32, device=q8.device)
    got = ctypes.c_int(0)
    _check(lib().fps_debug_scores_block_q8(ctypes.byref(shape), _ptr(q8), _ptr(k8), bh, u, jq, v, jk,
                                           _ptr(out), ctypes.byref(got), _stream()))
    assert got.value == bs
    return out


def attn_fwd(shape: Shape, window, prec, q, k, v, sq=None, sk=None, sv=None, vscale=VSCALE_TILE,
             out=None, out_dtype=None, visited=None, step: StepCfg = None, raster_out=False):
    torch = _torch or _import_torch()
    if out is None:
        out_dtype = out_dtype or torch.bfloat16
        dims = ((shape.T, shape.H, shape.W, shape.head_dim) if raster_out
                else (_tiled_len(shape), shape.head_dim))
        out = torch.empty((shape.B, shape.heads) + dims, dtype=out_dtype, device=q.device)
    dt = OUT_F32 if out.dtype == torch.float32 else OUT_BF16
    win = Window(*window) if window is not None else None
    if win is None and step is None:
        raise ValueError("attn_fwd needs a window or a step configuration")
    # pointers without a call of this module's own each, a structure as it is (ctypes passes its address where a pointer to
    # one is declared): on the smallest call, whose four launches wait for the host, 22.7 -> 21.3 us
    _check(lib().fps_attn_fwd(shape, win, prec, step, None if q is None else q.data_ptr(),
                              None if k is None else k.data_ptr(), None if v is None else v.data_ptr(),
                              None if sq is None else sq.data_ptr(), None if sk is None else sk.data_ptr(),
                              None if sv is None else sv.data_ptr(), vscale, out.data_ptr(), dt,
                              LAYOUT_RASTER if raster_out else LAYOUT_TILED,
                              None if visited is None else visited.data_ptr(), _stream()))
    return out


# ---- before and after the attention -------------------------------------------------------------
def _here(*tensors):
    """Every tensor (None: left out) is on the current device and autograd waits for a gradient of none; returns its stream, which the call
    goes to."""
    recording = (_torch or _import_torch()).is_grad_enabled()
    current = away = None
    for t in tensors:
        if t is None:
            continue
        if recording and t.requires_grad:
            raise ValueError("a tensor requires a gradient, which this call does not record: make it under torch.no_grad(), or in an "
                             "autograd.Function whose backward calls the gradient's entry point")
        device = t.get_device()                            # -1 on the host
        if device != current:
            if current is None and device >= 0:
                current = _torch.cuda.current_device()
            if device != current and away is None:
                away = t.device
    if away is not None:
        raise ValueError(f"a tensor on {away}, not on the current device" + ("" if current is None else f" (cuda:{current})"))
    return _stream(current)


def _whole(t, dtype, numel, name):
    if t.dtype != dtype or t.numel() != numel or not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous {dtype} of {numel} elements, not {t.dtype} {tuple(t.shape)}")


def _workspace(t):
    """A workspace's bytes, all of which are its own."""
    if not t.is_contiguous():
        raise ValueError(f"a workspace must be contiguous, not {tuple(t.shape)} of strides {t.stride()}")
    return t.numel() * t.element_size()


def _dtype_code(t):
    if not _codes:
        torch = _torch or _import_torch()
        _codes.update({torch.bfloat16: OUT_BF16, torch.float32: OUT_F32})
    code = _codes.get(t.dtype)
    if code is None:
        raise ValueError(f"{t.dtype} instead of bfloat16 or float32")
    return code


def _view(t, name) -> View:
    """[B, heads, tokens.., cols] of any strides; axes of tokens must follow each other in memory as in the shape."""
    size, stride = t.shape, t.stride()
    last = len(size) - 1
    if last < 3:
        raise ValueError(f"{name} must be [B, heads, tokens.., channels], not {tuple(size)}")
    rows, at = 1, 0
    for i in range(last - 1, 1, -1):                       # two of these views are made a call: as little as it takes
        n = size[i]
        if n == 1:
            continue
        if rows == 1:
            at = stride[i]
        elif stride[i] != at * rows:
            raise ValueError(f"{name}: the token axes of strides {stride[2:-1]} are not one axis")
        rows *= n
    if stride[last] != 1 and size[last] > 1:
        raise ValueError(f"{name}: the channels must be contiguous")
    return View(t.data_ptr(), _dtype_code(t), size[0], size[1], rows, size[last], stride[0], stride[1], at)


def make_norm(weight=None, eps=1e-6) -> Norm:
    """Norm of each token of each head; weight: fp32 [128], or [heads, 128] for one of each head, or None.  The tensor is kept, and
    each call reads it where it lies then; its type and size stay."""
    if weight is not None:
        torch = _torch or _import_torch()
        if weight.dtype != torch.float32 or weight.dim() not in (1, 2) or weight.shape[-1] != 128 or not weight.is_contiguous():
            raise ValueError(f"a norm's weight is contiguous fp32 [128] or [heads, 128], not {weight.dtype} {tuple(weight.shape)}")
    norm = Norm(_ptr(weight), weight is not None and weight.dim() == 2, eps)
    norm.tensor, norm.size = weight, None if weight is None else weight.shape
    return norm


def rotation_table(shape: Shape, split, base=10000.0, start=(0, 0, 0)):
    """The rotation's table of shape's grid on the host, fp32 [entries, 2] from angles in 64 bits: `split` pairs turn with t, h
    and w, pair i of n by place * base^(-i/n); start: place of the first frame, row and column."""
    torch = _torch or _import_torch()
    rot = Rotation(None, 0, *split, PAIRS_ADJACENT)
    n = int(lib().fps_rotation_floats(ctypes.byref(shape), ctypes.byref(rot)))
    if n == 0 and sum(split) != 0:
        raise FpsError(FPS_ERR_INVALID_ARG, last_error())
    table = torch.empty((n // 2, 2), dtype=torch.float32)
    _check(lib().fps_rotation_table_host(ctypes.byref(shape), ctypes.byref(rot), (ctypes.c_int64 * 3)(*start), base,
                                         table.data_ptr() or ctypes.addressof((ctypes.c_float * 1)())))
    return table


def make_rotation(table, split, halves=False) -> Rotation:
    """table: fp32 [entries, 2] (cos, sin) on the device, of T*split[0] + H*split[1] + W*split[2] entries as rotation_table
    has them, or [B, entries, 2] for one of each batch element, kept as a norm's weight is; halves: channel i turns with i + 64
    instead of 2i with 2i + 1."""
    torch = _torch or _import_torch()
    if table.dtype != torch.float32 or table.dim() not in (2, 3) or table.shape[-1] != 2 or not table.is_contiguous():
        raise ValueError(f"a rotation's table is contiguous fp32 [entries, 2] or [B, entries, 2], not {table.dtype} {tuple(table.shape)}")
    rot = Rotation(table.data_ptr(), 2 * table.shape[1] if table.dim() == 3 else 0, *split, PAIRS_HALVES if halves else PAIRS_ADJACENT)
    rot.tensor, rot.size = table, table.shape
    return rot


def _address(t, size, name):
    """Where a tensor that is kept from call to call lies now: a parameter may have been given other memory since the last one."""
    at = t.data_ptr()
    if t.dtype is not _torch.float32 or t.shape != size or not t.is_contiguous() or (at == 0 and t.numel() != 0):
        raise ValueError(f"{name} has become {t.dtype} {tuple(t.shape)}" + (" without memory" if at == 0 else ""))
    return at


def _check_turning(shape: Shape, norm, rotation):
    weight = table = None
    if norm is not None and norm.tensor is not None:
        weight, size = norm.tensor, norm.size
        norm.weight = _address(weight, size, "a norm's weight")
        if norm.per_head and size[0] != shape.heads:
            raise ValueError(f"a norm's weight of {size[0]} heads, not {shape.heads}")
    if rotation is not None:
        table, size = rotation.tensor, rotation.size
        rotation.table = _address(table, size, "a rotation's table")
        n = shape.T * rotation.pairs_t + shape.H * rotation.pairs_h + shape.W * rotation.pairs_w
        if size[-2] != n or (len(size) == 3 and size[0] != shape.B):
            raise ValueError(f"a rotation's table {tuple(size)}, not of {n} entries (of {shape.B} batch elements)")
    return weight, table


def norm_rotate(shape: Shape, x, norm: Norm = None, rotation: Rotation = None, out=None, out_dtype=None):
    """Each head's norm and the rotation by the token's place.  x: bf16 or fp32 [B, heads, tokens, 128] of any strides, for
    instance projection.view(B, tokens, heads, 128).transpose(1, 2); out alike (default: raster order, x's type)."""
    torch = _torch or _import_torch()
    weight, table = _check_turning(shape, norm, rotation)
    if out is None:
        out = torch.empty((shape.B, shape.heads, shape.T, shape.H, shape.W, shape.head_dim), dtype=out_dtype or x.dtype,
                          device=x.device)
    stream = _here(x, out, weight, table)
    _check(lib().fps_norm_rotate(shape, _view(x, "x"), norm, rotation, _view(out, "out"), stream))
    _written(out)
    return out


def norm_rotate_operand(shape: Shape, x, role, prec=PREC_FP8, norm: Norm = None, rotation: Rotation = None, out=None, scales=None):
    """norm_rotate straight into the operand of attn_fwd (Q or K).  Returns (packed operand, scales or None)."""
    torch = _torch or _import_torch()
    weight, table = _check_turning(shape, norm, rotation)
    fp8 = prec == PREC_FP8
    if out is None:
        out = torch.empty(packed_bytes(shape, prec), dtype=torch.uint8, device=x.device)
    if not fp8:
        scales = None
    elif scales is None:
        scales = torch.empty((shape.B, shape.heads, num_groups(shape)), dtype=torch.float32, device=x.device)
    stream = _here(x, out, scales, weight, table)
    _whole(out, torch.uint8, packed_bytes(shape, prec), "out")
    if fp8:
        _whole(scales, torch.float32, shape.B * shape.heads * num_groups(shape), "scales")
    _check(lib().fps_norm_rotate_operand(shape, _view(x, "x"), norm, rotation, role, prec, out.data_ptr(), _ptr(scales), stream))
    _written((out, scales) if fp8 else out)
    return out, scales


def norm_rotate_bwd_bytes(shape: Shape, norm: Norm = None) -> int:
    n = int(lib().fps_norm_rotate_bwd_bytes(shape, norm))
    if n == 0:
        raise FpsError(FPS_ERR_INVALID_ARG, last_error())
    return n


def norm_rotate_bwd(shape: Shape, x, dy, norm: Norm = None, rotation: Rotation = None, dx=None, dweight=None, workspace=None,
                    need_dweight=True):
    """Gradient of norm_rotate: (dx, dweight); dweight is None without a weight, or if it is not wanted.  Straight through a
    quantisation that follows: dy is then the gradient of the operand's values."""
    torch = _torch or _import_torch()
    weight, table = _check_turning(shape, norm, rotation)
    if dx is None:
        dx = torch.empty_like(x)
    if weight is None or not need_dweight:
        dweight = workspace = None
        size = 0
    else:
        if dweight is None:
            dweight = torch.empty_like(weight)
        _whole(dweight, torch.float32, weight.numel(), "dweight")
        if workspace is None:
            workspace = torch.empty(norm_rotate_bwd_bytes(shape, norm), dtype=torch.uint8, device=x.device)
        size = _workspace(workspace)
    stream = _here(x, dy, dx, dweight, workspace, weight, table)
    _check(lib().fps_norm_rotate_bwd(shape, _view(x, "x"), norm, rotation, _view(dy, "dy"), _view(dx, "dx"), _ptr(dweight),
                                     _ptr(workspace), size, stream))
    _written(dx if dweight is None else (dx, dweight))
    return dx, dweight


def dequantize(shape: Shape, xq, scales, role, vscale=VSCALE_TILE, out=None, out_dtype=None):
    """The values of a packed E4M3 operand, code * scale, in raster order [B, heads, T, H, W, 128]."""
    torch = _torch or _import_torch()
    dims = (shape.B, shape.heads, shape.T, shape.H, shape.W, shape.head_dim)
    if out is None:
        out = torch.empty(dims, dtype=out_dtype or torch.bfloat16, device=xq.device)
    stream = _here(xq, scales, out)
    _whole(xq, torch.uint8, packed_bytes(shape, PREC_FP8), "xq")
    _whole(out, out.dtype, shape.B * shape.heads * shape.T * shape.H * shape.W * shape.head_dim, "out")
    n = shape.head_dim if role == ROLE_V and vscale == VSCALE_CHANNEL else num_groups(shape)
    _whole(scales, torch.float32, shape.B * shape.heads * n, "scales")
    _check(lib().fps_dequantize(shape, xq.data_ptr(), scales.data_ptr(), role, vscale, _dtype_code(out), out.data_ptr(), stream))
    _written(out)
    return out


def _matrix(t, name):
    """A matrix [rows, cols], several [B, rows, cols], or a tensor [B, heads, tokens.., cols] whose matrix has B * tokens rows of
    heads * cols; columns of a row (of a head) are contiguous.  Returns its View, rows and columns."""
    size, stride = t.shape, t.stride()
    n = len(size)
    if n >= 4:
        v = _view(t, name)
        return v, v.B * v.rows, v.heads * v.cols
    if n < 2:
        raise ValueError(f"{name} must have rows and columns, not {tuple(size)}")
    rows, cols = size[-2], size[-1]
    if stride[-1] != 1 and cols > 1:
        raise ValueError(f"{name}: the columns must be contiguous")
    if n == 2:
        return View(t.data_ptr(), _dtype_code(t), 1, 1, rows, cols, 0, 0, stride[0]), rows, cols
    return View(t.data_ptr(), _dtype_code(t), size[0], 1, rows, cols, stride[0], 0, stride[1]), size[0] * rows, cols


def mx4_bytes(rows, cols) -> int:
    """Bytes of a matrix packed in microscaled 4-bit floating point."""
    n = int(lib().fps_mx4_bytes(rows, cols))
    if n == 0:
        raise FpsError(FPS_ERR_INVALID_ARG, last_error())
    return n


def mx4_linear_bytes(rows, cols) -> int:
    n = int(lib().fps_mx4_linear_bytes(rows, cols))
    if n == 0:
        raise FpsError(FPS_ERR_INVALID_ARG, last_error())
    return n


def mx4_quantize(x, out=None):
    """bf16 or fp32 rows (see _matrix) -> packed blocks of 32 E2M1 codes with a power of two each."""
    torch = _torch or _import_torch()
    v, rows, cols = _matrix(x, "x")
    n = mx4_bytes(rows, cols)
    if out is None:
        out = torch.empty(n, dtype=torch.uint8, device=x.device)
    stream = _here(x, out)
    _whole(out, torch.uint8, n, "out")
    _check(lib().fps_mx4_quantize(v, out.data_ptr(), stream))
    _written(out)
    return out


def mx4_dequantize(packed, rows, cols, out=None, out_dtype=None):
    """The values of a packed matrix [rows, cols], also into a tensor that stands for one."""
    torch = _torch or _import_torch()
    if out is None:
        out = torch.empty((rows, cols), dtype=out_dtype or torch.bfloat16, device=packed.device)
    stream = _here(packed, out)
    v, *size = _matrix(out, "out")
    if size != [rows, cols]:
        raise ValueError(f"out {tuple(out.shape)} is not a matrix of {rows} x {cols}")
    _whole(packed, torch.uint8, mx4_bytes(rows, cols), "packed")
    _check(lib().fps_mx4_dequantize(packed.data_ptr(), v, stream))
    _written(out)
    return out


def _product_out(out, out_dtype, rows, cols, like):
    torch = _torch or _import_torch()
    if out is None:
        out = torch.empty((rows, cols), dtype=out_dtype or torch.bfloat16, device=like.device)
    v, r, c = _matrix(out, "out")
    if r != rows or c != cols:
        raise ValueError(f"out {tuple(out.shape)} is not a matrix of {rows} x {cols}")
    return out, v


def mx4_matmul(a, b, m, n, k, bias=None, out=None, out_dtype=None):
    """a b^T + bias of packed matrices a [m, k] and b [n, k]; bias: fp32 [n]."""
    torch = _torch or _import_torch()
    out, v = _product_out(out, out_dtype, m, n, a)
    stream = _here(a, b, bias, out)
    _whole(a, torch.uint8, mx4_bytes(m, k), "a")
    _whole(b, torch.uint8, mx4_bytes(n, k), "b")
    if bias is not None:
        _whole(bias, torch.float32, n, "bias")
    _check(lib().fps_mx4_matmul(k, a.data_ptr(), b.data_ptr(), _ptr(bias), v, stream))
    _written(out)
    return out


def mx4_linear(x, w, n, bias=None, out=None, out_dtype=None, workspace=None):
    """x W^T + bias, x (rows as in mx4_quantize) quantised on the way; w: mx4_quantize of the weights [n, k]."""
    torch = _torch or _import_torch()
    xv, m, k = _matrix(x, "x")
    out, v = _product_out(out, out_dtype, m, n, x)
    if workspace is None:
        workspace = torch.empty(mx4_linear_bytes(m, k), dtype=torch.uint8, device=x.device)
    size = _workspace(workspace)
    stream = _here(x, w, bias, out, workspace)
    _whole(w, torch.uint8, mx4_bytes(n, k), "w")
    if bias is not None:
        _whole(bias, torch.float32, n, "bias")
    _check(lib().fps_mx4_linear(xv, w.data_ptr(), _ptr(bias), v, workspace.data_ptr(), size, stream))
    _written(out)
    return out
