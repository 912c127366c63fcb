"""Torch-facing wrappers of the C ABI (argument marshalling only).

Every step of the layer runs in the HIP kernels of libcs.so; these functions
check tensor placement/dtype/shape, allocate outputs with torch and pass raw
device pointers plus torch's current HIP stream.  They never compute on the
host and have no fallback.
"""
from __future__ import annotations

import ctypes
import math
from dataclasses import dataclass

import numpy as np
import torch

from . import _lib
from ._lib import CS_BF16, CS_F16, CS_F32, CS_I8, CS_I32, check, lib

_TORCH_DT = {torch.int8: CS_I8, torch.int32: CS_I32, torch.float32: CS_F32}
_NP_DT = {np.dtype(np.int8): CS_I8, np.dtype(np.float32): CS_F32}


def _dt(t: torch.Tensor) -> int:
    try:
        return _TORCH_DT[t.dtype]
    except KeyError:
        raise TypeError(f"unsupported dtype {t.dtype}") from None


def _dev(t: torch.Tensor, name: str) -> int:
    if not t.is_cuda:
        raise ValueError(f"{name} must be a GPU tensor")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return t.data_ptr()


def _opt(t: torch.Tensor | None, name: str):
    return None if t is None else _dev(t, name)


def _stream() -> int:
    return torch.cuda.current_stream().cuda_stream


# ------------------------------------------------------------------ pack (host)
def pack(W: np.ndarray, n: int):
    """Combine on the host: W [d_out][r] (int8 or float32) -> (aug, holes).

    aug is the augmented packed tensor [r][G] (G = d_out / n): for int8
    weights a uint16 array, entry = uint8(value) | kid << 8; for float32
    weights a uint32 array [r][G][2] holding (value bits, kid).  Raises
    CSError(CS_ERR_COLLISION) with .bad = (g, i) when two kernels of a set
    share a slot."""
    W = np.ascontiguousarray(W)
    if W.ndim != 2:
        raise ValueError("W must be [d_out][r]")
    d_out, r = W.shape
    wt = _NP_DT.get(W.dtype)
    if wt is None:
        raise TypeError(f"unsupported weight dtype {W.dtype}")
    G = d_out // n if n > 0 else 0
    if wt == CS_I8:
        aug = np.zeros((r, max(G, 1)), dtype=np.uint16)
    else:
        aug = np.zeros((r, max(G, 1), 2), dtype=np.uint32)
    holes = ctypes.c_int64(0)
    bg, bi = ctypes.c_int(0), ctypes.c_int(0)
    st = lib().cs_pack(wt, W.ctypes.data, d_out, r, n, aug.ctypes.data,
                       ctypes.byref(holes), ctypes.byref(bg), ctypes.byref(bi))
    if st != _lib.CS_OK:
        err = _lib.CSError("cs_pack", st)
        err.bad = (bg.value, bi.value)
        raise err
    return aug, int(holes.value)


def unpack_aug(aug: np.ndarray):
    """Split a host augmented tensor into (values [r][G], kernel IDs [r][G])."""
    if aug.dtype == np.uint16:
        return (aug & 0xFF).astype(np.uint8).view(np.int8), (aug >> 8).astype(np.int64)
    if aug.dtype == np.uint32 and aug.ndim == 3 and aug.shape[2] == 2:
        return aug[..., 0].copy().view(np.float32), aug[..., 1].astype(np.int64)
    raise TypeError("not an augmented tensor")


def aug_to_device(aug: np.ndarray, device="cuda") -> torch.Tensor:
    """Upload an augmented tensor: int16 [r][G] (int8 weights) or int32
    [r][G][2] (float32 weights), bit patterns unchanged."""
    if aug.dtype == np.uint16:
        return torch.from_numpy(aug.view(np.int16)).to(device)
    if aug.dtype == np.uint32:
        return torch.from_numpy(aug.view(np.int32)).to(device)
    raise TypeError("not an augmented tensor")


def _aug(aug: torch.Tensor, xdt: torch.dtype, n: int):
    """Device pointer and c_out of an augmented tensor that matches activations of dtype xdt."""
    ok = (xdt == torch.int8 and aug.dtype == torch.int16 and aug.dim() == 2) or \
         (xdt == torch.float32 and aug.dtype == torch.int32 and aug.dim() == 3 and
          aug.shape[2] == 2)
    if not ok:
        raise TypeError(f"augmented tensor {aug.dtype}{tuple(aug.shape)} does not match {xdt}")
    return _dev(aug, "aug"), aug.shape[1] * n


# ------------------------------------------------------------------ device ops
def compact(x: torch.Tensor):
    """x [rows][c] (int8/float32) -> (idx uint16-as-int16 [rows][c], val, cnt int32).
    Only idx[r, :cnt[r]] and val[r, :cnt[r]] are defined."""
    if x.dim() != 2:
        raise ValueError("x must be [rows][c]")
    rows, c = x.shape
    idx = torch.empty((rows, c), dtype=torch.int16, device=x.device)
    val = torch.empty_like(x)
    cnt = torch.empty((rows,), dtype=torch.int32, device=x.device)
    check("cs_compact", lib().cs_compact(_dt(x), _dev(x, "x"), rows, c, _dev(idx, "idx"),
                                         _dev(val, "val"), _dev(cnt, "cnt"), _stream()))
    return idx, val, cnt


def compact_into(x: torch.Tensor, idx: torch.Tensor, val: torch.Tensor, cnt: torch.Tensor) -> None:
    """cs_compact into caller-provided buffers (idx int16 [rows][c], val like x, cnt int32)."""
    rows, c = x.shape
    if idx.shape != (rows, c) or val.shape != (rows, c) or cnt.shape != (rows,):
        raise ValueError("buffer shapes do not match x")
    if idx.dtype != torch.int16 or val.dtype != x.dtype or cnt.dtype != torch.int32:
        raise TypeError("buffer dtypes do not match")
    check("cs_compact", lib().cs_compact(_dt(x), _dev(x, "x"), rows, c, _dev(idx, "idx"),
                                         _dev(val, "val"), _dev(cnt, "cnt"), _stream()))


def conv_out(h: int, k: int, stride: int, pad: int) -> int:
    return (h + 2 * pad - k) // stride + 1


def mrs_conv2d(idx: torch.Tensor, lval: torch.Tensor, cnt: torch.Tensor, in_shape, aug,
               kh: int, kw: int, n: int, stride: int = 1, pad: int = 0, bias=None, pool: int = 1,
               out: torch.Tensor | None = None) -> torch.Tensor:
    """Multiply/route/sum on compacted lists of the b*h*w input pixels."""
    b, h, w, c_in = in_shape
    pa, c_out = _aug(aug, lval.dtype, n)
    ho, wo = conv_out(h, kh, stride, pad), conv_out(w, kw, stride, pad)
    ydt = torch.int32 if lval.dtype == torch.int8 else torch.float32
    if out is None:
        out = torch.empty((b, ho // pool, wo // pool, c_out), dtype=ydt, device=lval.device)
    check("cs_mrs_conv2d", lib().cs_mrs_conv2d(
        _dt(lval), _dev(idx, "idx"), _dev(lval, "lval"), _dev(cnt, "cnt"), idx.shape[-1],
        b, h, w, c_in, kh, kw, stride, pad, pa, c_out, n,
        _opt(bias, "bias"), pool, _dev(out, "out"), _stream()))
    return out


def mrs_kwta_conv2d(idx: torch.Tensor, lval: torch.Tensor, cnt: torch.Tensor, in_shape, aug,
                    kh: int, kw: int, n: int, stride: int = 1, pad: int = 0, bias=None,
                    pool: int = 1, *, k: int, out_dtype: torch.dtype | None = None,
                    shift: int = 0, y: torch.Tensor | None = None, keep_sums: bool = True,
                    cap: int | None = None, lists=None, out: torch.Tensor | None = None):
    """One layer: multiply/route/sum (+ bias, pool) and k-WTA over each output
    pixel's channels.  Returns (y, result) where y holds the sums (when
    keep_sums) and result is the dense masked output, or the (idx, val, cnt)
    lists when `cap` or `lists` is given."""
    b, h, w, c_in = in_shape
    pa, c_out = _aug(aug, lval.dtype, n)
    ho, wo = conv_out(h, kh, stride, pad), conv_out(w, kw, stride, pad)
    acc_dt = torch.int32 if lval.dtype == torch.int8 else torch.float32
    odt = acc_dt if out_dtype is None else out_dtype
    oshape = (b, max(ho, 0) // pool, max(wo, 0) // pool, c_out)
    rows = oshape[0] * oshape[1] * oshape[2]
    if y is None:
        y = torch.empty(oshape, dtype=acc_dt, device=lval.device)
    if lists is None and cap is not None:
        lists = (torch.empty((rows, cap), dtype=torch.int16, device=lval.device),
                 torch.empty((rows, cap), dtype=odt, device=lval.device),
                 torch.empty((rows,), dtype=torch.int32, device=lval.device))
    if lists is not None:
        oi, ov, oc = lists
        if oi.dtype != torch.int16 or ov.dtype != odt or oc.dtype != torch.int32:
            raise TypeError("list buffer dtypes do not match")
        if oi.shape != ov.shape or oi.dim() != 2 or oi.shape[0] != rows or oc.shape != (rows,):
            raise ValueError("list buffer shapes do not match the output")
        args = (None, _dev(oi, "oidx"), _dev(ov, "oval"), _dev(oc, "ocnt"), oi.shape[1])
        result = lists
    else:
        if out is None:
            out = torch.empty(oshape, dtype=odt, device=lval.device)
        if out.dtype != odt or out.numel() != rows * c_out:
            raise ValueError("out does not match the output")
        args = (_dev(out, "out"), None, None, None, 0)
        result = out
    check("cs_mrs_kwta_conv2d", lib().cs_mrs_kwta_conv2d(
        _dt(lval), _dev(idx, "idx"), _dev(lval, "lval"), _dev(cnt, "cnt"), idx.shape[-1],
        b, h, w, c_in, kh, kw, stride, pad, pa, c_out, n, _opt(bias, "bias"), pool,
        _dev(y, "y"), 1 if keep_sums else 0, k, _TORCH_DT[odt], shift, *args, _stream()))
    return y, result


def mrs_kwta_units_conv2d(idx: torch.Tensor, lval: torch.Tensor, cnt: torch.Tensor, in_shape,
                          aug, kh: int, kw: int, n: int, stride: int = 1, pad: int = 0,
                          bias=None, pool: int = 1, *, k: int, unit: int,
                          y: torch.Tensor | None = None, keep_sums: bool = True,
                          cap: int | None = None, lists=None, out: torch.Tensor | None = None):
    """One fp32 layer with k-WTA in units (cs_mrs_kwta_units_conv2d): every
    `unit` consecutive channels of an output pixel keep their own k winners.
    Returns (y, result) as mrs_kwta_conv2d."""
    b, h, w, c_in = in_shape
    pa, c_out = _aug(aug, lval.dtype, n)
    ho, wo = conv_out(h, kh, stride, pad), conv_out(w, kw, stride, pad)
    acc_dt = torch.int32 if lval.dtype == torch.int8 else torch.float32
    oshape = (b, max(ho, 0) // pool, max(wo, 0) // pool, c_out)
    rows = oshape[0] * oshape[1] * oshape[2]
    if y is None:
        y = torch.empty(oshape, dtype=acc_dt, device=lval.device)
    if lists is None and cap is not None:
        lists = (torch.empty((rows, cap), dtype=torch.int16, device=lval.device),
                 torch.empty((rows, cap), dtype=acc_dt, device=lval.device),
                 torch.empty((rows,), dtype=torch.int32, device=lval.device))
    if lists is not None:
        oi, ov, oc = lists
        if oi.dtype != torch.int16 or ov.dtype != acc_dt or oc.dtype != torch.int32:
            raise TypeError("list buffer dtypes do not match")
        if oi.shape != ov.shape or oi.dim() != 2 or oi.shape[0] != rows or oc.shape != (rows,):
            raise ValueError("list buffer shapes do not match the output")
        args = (None, _dev(oi, "oidx"), _dev(ov, "oval"), _dev(oc, "ocnt"), oi.shape[1])
        result = lists
    else:
        if out is None:
            out = torch.empty(oshape, dtype=acc_dt, device=lval.device)
        if out.dtype != acc_dt or out.numel() != rows * c_out:
            raise ValueError("out does not match the output")
        args = (_dev(out, "out"), None, None, None, 0)
        result = out
    check("cs_mrs_kwta_units_conv2d", lib().cs_mrs_kwta_units_conv2d(
        _dt(lval), _dev(idx, "idx"), _dev(lval, "lval"), _dev(cnt, "cnt"), idx.shape[-1],
        b, h, w, c_in, kh, kw, stride, pad, pa, c_out, n, _opt(bias, "bias"), pool,
        _dev(y, "y"), 1 if keep_sums else 0, k, unit, *args, _stream()))
    return y, result


def mrs_kwta_chain2(idx: torch.Tensor, lval: torch.Tensor, cnt: torch.Tensor, in_shape, aug,
                    kh: int, kw: int, n: int, stride: int = 1, pad: int = 0, bias=None,
                    pool: int = 1, *, k: int, shift: int, aug2, n2: int, bias2=None,
                    y: torch.Tensor | None = None, keep_sums: bool = True, cap: int | None = None,
                    lists=None, y2: torch.Tensor | None = None):
    """An int8 layer with k-WTA (one output vector per sample) and the linear
    layer on its requantised winners (cs_mrs_kwta_chain2).  Returns
    (y, lists, y2): the first layer's sums (when keep_sums), its winners'
    lists and the second layer's int32 sums [b][c_out2]."""
    if lval.dtype != torch.int8:
        raise TypeError("mrs_kwta_chain2 takes int8 lists")
    b, h, w, c_in = in_shape
    pa, c_out = _aug(aug, lval.dtype, n)
    pa2, c_out2 = _aug(aug2, torch.int8, n2)
    ho, wo = conv_out(h, kh, stride, pad), conv_out(w, kw, stride, pad)
    oshape = (b, max(ho, 0) // pool, max(wo, 0) // pool, c_out)
    rows = oshape[0] * oshape[1] * oshape[2]
    if y is None:
        y = torch.empty(oshape, dtype=torch.int32, device=lval.device)
    if lists is None:
        cap = list_capacity(k) if cap is None else cap
        lists = (torch.empty((rows, cap), dtype=torch.int16, device=lval.device),
                 torch.empty((rows, cap), dtype=torch.int8, device=lval.device),
                 torch.empty((rows,), dtype=torch.int32, device=lval.device))
    oi, ov, oc = lists
    if oi.dtype != torch.int16 or ov.dtype != torch.int8 or oc.dtype != torch.int32:
        raise TypeError("list buffer dtypes do not match")
    if oi.shape != ov.shape or oi.dim() != 2 or oi.shape[0] != rows or oc.shape != (rows,):
        raise ValueError("list buffer shapes do not match the output")
    if y2 is None:
        y2 = torch.empty((b, c_out2), dtype=torch.int32, device=lval.device)
    if y2.dtype != torch.int32 or y2.numel() != b * c_out2:
        raise ValueError("y2 does not match the second layer's output")
    check("cs_mrs_kwta_chain2", lib().cs_mrs_kwta_chain2(
        CS_I8, _dev(idx, "idx"), _dev(lval, "lval"), _dev(cnt, "cnt"), idx.shape[-1],
        b, h, w, c_in, kh, kw, stride, pad, pa, c_out, n, _opt(bias, "bias"), pool,
        _dev(y, "y"), 1 if keep_sums else 0, k, CS_I8, shift, _dev(oi, "oidx"), _dev(ov, "oval"),
        _dev(oc, "ocnt"), oi.shape[1], pa2, c_out2, n2, _opt(bias2, "bias2"), _dev(y2, "y2"),
        _stream()))
    return y, lists, y2


def _list_buffers(rows: int, cap: int, device, lists=None):
    if lists is None:
        lists = (torch.empty((rows, cap), dtype=torch.int16, device=device),
                 torch.empty((rows, cap), dtype=torch.int8, device=device),
                 torch.empty((rows,), dtype=torch.int32, device=device))
    oi, ov, oc = lists
    if oi.dtype != torch.int16 or ov.dtype != torch.int8 or oc.dtype != torch.int32:
        raise TypeError("list buffer dtypes do not match")
    if oi.shape != ov.shape or oi.dim() != 2 or oi.shape[0] != rows or oc.shape != (rows,):
        raise ValueError("list buffer shapes do not match the output")
    return lists


def mrs_kwta_chain3(idx: torch.Tensor, lval: torch.Tensor, cnt: torch.Tensor, in_shape, aug,
                    kh: int, kw: int, n: int, stride: int = 1, pad: int = 0, bias=None,
                    pool: int = 1, *, k: int, shift: int, aug2, n2: int, bias2=None, k2: int,
                    shift2: int, aug3, n3: int, bias3=None, keep_sums: bool = True,
                    y: torch.Tensor | None = None, cap: int | None = None, lists=None,
                    y2: torch.Tensor | None = None, cap2: int | None = None, lists2=None,
                    y3: torch.Tensor | None = None):
    """An int8 conv layer with k-WTA and lists, a layer with k-WTA over its
    whole pooled map, and a linear layer on the second one's winners
    (cs_mrs_kwta_chain3).  aug2 packs [c_out2][hp*wp*c_out] weights in the
    (y, x, channel) slot order of the first layer's NHWC output.  Returns
    (y, lists, y2, lists2, y3)."""
    if lval.dtype != torch.int8:
        raise TypeError("mrs_kwta_chain3 takes int8 lists")
    b, h, w, c_in = in_shape
    pa, c_out = _aug(aug, lval.dtype, n)
    pa2, c_out2 = _aug(aug2, torch.int8, n2)
    pa3, c_out3 = _aug(aug3, torch.int8, n3)
    ho, wo = conv_out(h, kh, stride, pad), conv_out(w, kw, stride, pad)
    oshape = (b, max(ho, 0) // pool, max(wo, 0) // pool, c_out)
    rows = oshape[0] * oshape[1] * oshape[2]
    dev = lval.device
    if y is None:
        y = torch.empty(oshape, dtype=torch.int32, device=dev)
    lists = _list_buffers(rows, list_capacity(k) if cap is None else cap, dev, lists)
    if y2 is None:
        y2 = torch.empty((b, c_out2), dtype=torch.int32, device=dev)
    lists2 = _list_buffers(b, list_capacity(k2) if cap2 is None else cap2, dev, lists2)
    if y3 is None:
        y3 = torch.empty((b, c_out3), dtype=torch.int32, device=dev)
    for t, nm, m in ((y2, "y2", c_out2), (y3, "y3", c_out3)):
        if t.dtype != torch.int32 or t.numel() != b * m:
            raise ValueError(f"{nm} does not match its layer's output")
    oi, ov, oc = lists
    oi2, ov2, oc2 = lists2
    check("cs_mrs_kwta_chain3", lib().cs_mrs_kwta_chain3(
        CS_I8, _dev(idx, "idx"), _dev(lval, "lval"), _dev(cnt, "cnt"), idx.shape[-1],
        b, h, w, c_in, kh, kw, stride, pad, pa, c_out, n, _opt(bias, "bias"), pool,
        _dev(y, "y"), 1 if keep_sums else 0, k, CS_I8, shift, _dev(oi, "oidx"), _dev(ov, "oval"),
        _dev(oc, "ocnt"), oi.shape[1], pa2, c_out2, n2, _opt(bias2, "bias2"), _dev(y2, "y2"),
        k2, shift2, _dev(oi2, "oidx2"), _dev(ov2, "oval2"), _dev(oc2, "ocnt2"), oi2.shape[1],
        pa3, c_out3, n3, _opt(bias3, "bias3"), _dev(y3, "y3"), _stream()))
    return y, lists, y2, lists2, y3


def conv2d_dense_kwta_chain3(x: torch.Tensor, aug, kh: int, kw: int, n: int, stride: int = 1,
                             pad: int = 0, bias=None, pool: int = 1, *, k: int, shift: int,
                             aug2, kh2: int, kw2: int, n2: int, stride2: int = 1, pad2: int = 0,
                             bias2=None, pool2: int = 1, k2: int, shift2: int, aug3, n3: int,
                             bias3=None, k3: int, shift3: int, aug4, n4: int, bias4=None,
                             keep_sums: bool = True, y=None, lists=None, y2=None, lists2=None,
                             y3=None, lists3=None, y4=None):
    """The dense-input int8 first layer with k-WTA lists, then the three layers
    of mrs_kwta_chain3 on them (cs_conv2d_dense_kwta_chain3).  Returns
    (y, lists, y2, lists2, y3, lists3, y4)."""
    if x.dim() != 4 or x.dtype != torch.int8:
        raise ValueError("x must be int8 NHWC")
    b, h, w, c_in = x.shape
    dev = x.device
    pa, c_out = _aug(aug, torch.int8, n)
    pa2, c_out2 = _aug(aug2, torch.int8, n2)
    pa3, c_out3 = _aug(aug3, torch.int8, n3)
    pa4, c_out4 = _aug(aug4, torch.int8, n4)
    ho, wo = conv_out(h, kh, stride, pad), conv_out(w, kw, stride, pad)
    s1 = (b, max(ho, 0) // pool, max(wo, 0) // pool, c_out)
    ho2, wo2 = conv_out(s1[1], kh2, stride2, pad2), conv_out(s1[2], kw2, stride2, pad2)
    s2 = (b, max(ho2, 0) // pool2, max(wo2, 0) // pool2, c_out2)
    r1, r2 = s1[0] * s1[1] * s1[2], s2[0] * s2[1] * s2[2]
    y = torch.empty(s1, dtype=torch.int32, device=dev) if y is None else y
    y2 = torch.empty(s2, dtype=torch.int32, device=dev) if y2 is None else y2
    y3 = torch.empty((b, c_out3), dtype=torch.int32, device=dev) if y3 is None else y3
    y4 = torch.empty((b, c_out4), dtype=torch.int32, device=dev) if y4 is None else y4
    for t, nm, m in ((y, "y", r1 * c_out), (y2, "y2", r2 * c_out2), (y3, "y3", b * c_out3),
                     (y4, "y4", b * c_out4)):
        if t.dtype != torch.int32 or t.numel() != m:
            raise ValueError(f"{nm} does not match its layer's output")
    lists = _list_buffers(r1, list_capacity(k), dev, lists)
    lists2 = _list_buffers(r2, list_capacity(k2), dev, lists2)
    lists3 = _list_buffers(b, list_capacity(k3), dev, lists3)
    (oi, ov, oc), (oi2, ov2, oc2), (oi3, ov3, oc3) = lists, lists2, lists3
    check("cs_conv2d_dense_kwta_chain3", lib().cs_conv2d_dense_kwta_chain3(
        CS_I8, _dev(x, "x"), b, h, w, c_in, kh, kw, stride, pad, pa, c_out, n, _opt(bias, "bias"),
        pool, _dev(y, "y"), 1 if keep_sums else 0, k, CS_I8, shift, _dev(oi, "oidx"),
        _dev(ov, "oval"), _dev(oc, "ocnt"), oi.shape[1],
        kh2, kw2, stride2, pad2, pa2, c_out2, n2, _opt(bias2, "bias2"), pool2, _dev(y2, "y2"),
        k2, shift2, _dev(oi2, "oidx2"), _dev(ov2, "oval2"), _dev(oc2, "ocnt2"), oi2.shape[1],
        pa3, c_out3, n3, _opt(bias3, "bias3"), _dev(y3, "y3"), k3, shift3, _dev(oi3, "oidx3"),
        _dev(ov3, "oval3"), _dev(oc3, "ocnt3"), oi3.shape[1],
        pa4, c_out4, n4, _opt(bias4, "bias4"), _dev(y4, "y4"), _stream()))
    return y, lists, y2, lists2, y3, lists3, y4


def mrs_plan(dtype: torch.dtype, cap: int, in_shape, kh: int, kw: int, stride: int, pad: int,
             c_out: int, n: int, pool: int = 1, k: int = -1) -> dict:
    """The launch plan the library picks for a layer (host only)."""
    b, h, w, c_in = in_shape
    info = (ctypes.c_int64 * 11)()
    check("cs_mrs_plan", lib().cs_mrs_plan(_TORCH_DT[dtype], cap, b, h, w, c_in, kh, kw, stride,
                                           pad, c_out, n, pool, k, info))
    path = ("simple", "tiled", "fused", "sample", "scatter", "rows", "blocks")[info[0]]
    kwta = None if k < 0 else ("separate" if info[10] else "fused")
    if path == "blocks":
        return {"path": path, "kwta": kwta, "select": info[1], "rows_per_block": info[2],
                "table_blocks": info[3], "slices": info[4], "list_parts": 1 << info[5],
                "blocks": info[6], "lds": info[7], "sets_per_lane": info[8]}
    if path == "rows":
        return {"path": path, "kwta": kwta, "blocks": info[6], "lds": info[7],
                "channels_per_lane": info[8]}
    if path == "scatter":
        return {"path": path, "kwta": kwta, "band_rows": info[2], "blocks": info[6],
                "lds": info[7], "sets_per_lane": info[8]}
    if path == "sample":
        return {"path": path, "kwta": kwta, "blocks": info[6], "lds": info[7],
                "slices": info[8]}
    if path != "fused":
        return {"path": path, "kwta": kwta}
    return {"path": path, "tile_mode": info[1], "tile": info[2], "tile_cols": info[3],
            "list_cap": info[4], "npix_cap": info[5], "blocks": info[6], "lds": info[7],
            "log2_slices": info[8], "select": info[9], "kwta": kwta}


def workspace_bytes(op: int, dtype: torch.dtype, rows: int, c_in: int) -> int:
    return int(lib().cs_workspace_bytes(op, _TORCH_DT[dtype], rows, c_in))


def workspace(op: int, dtype: torch.dtype, rows: int, c_in: int, device) -> torch.Tensor:
    nbytes = workspace_bytes(op, dtype, rows, c_in)
    if nbytes == 0:
        raise ValueError("invalid workspace request")
    return torch.empty((nbytes,), dtype=torch.uint8, device=device)


def conv2d_noalloc(x: torch.Tensor, aug: torch.Tensor, kh: int, kw: int, n: int,
                   stride: int = 1, pad: int = 0, bias: torch.Tensor | None = None,
                   pool: int = 1, out: torch.Tensor | None = None) -> torch.Tensor:
    """conv2d without a workspace argument: the library's own scratch holds the
    compaction lists (cs_conv2d_noalloc; nothing is allocated when `out` is
    given).  Calls that overlap on one GPU race on that scratch."""
    if x.dim() != 4:
        raise ValueError("x must be NHWC")
    b, h, w, c_in = x.shape
    pa, c_out = _aug(aug, x.dtype, n)
    ho, wo = conv_out(h, kh, stride, pad), conv_out(w, kw, stride, pad)
    ydt = torch.int32 if x.dtype == torch.int8 else torch.float32
    if out is None:
        out = torch.empty((b, max(ho, 0) // pool, max(wo, 0) // pool, c_out), dtype=ydt,
                          device=x.device)
    check("cs_conv2d_noalloc", lib().cs_conv2d_noalloc(
        _dt(x), _dev(x, "x"), b, h, w, c_in, kh, kw, stride, pad, pa, c_out, n,
        _opt(bias, "bias"), pool, _dev(out, "out"), _stream()))
    return out


def conv2d(x: torch.Tensor, aug: torch.Tensor, kh: int, kw: int, n: int,
           stride: int = 1, pad: int = 0, bias: torch.Tensor | None = None, pool: int = 1,
           ws: torch.Tensor | None = None, out: torch.Tensor | None = None) -> torch.Tensor:
    """Sparse-sparse conv of NHWC x with packed OHWI kernels (aug [kh*kw*c_in][G])."""
    if x.dim() != 4:
        raise ValueError("x must be NHWC")
    b, h, w, c_in = x.shape
    pa, c_out = _aug(aug, x.dtype, n)
    ho, wo = conv_out(h, kh, stride, pad), conv_out(w, kw, stride, pad)
    ydt = torch.int32 if x.dtype == torch.int8 else torch.float32
    if out is None:
        out = torch.empty((b, max(ho, 0) // pool, max(wo, 0) // pool, c_out), dtype=ydt,
                          device=x.device)
    if ws is None:
        ws = workspace(1, x.dtype, b * h * w, c_in, x.device)
    check("cs_conv2d", lib().cs_conv2d(
        _dt(x), _dev(x, "x"), b, h, w, c_in, kh, kw, stride, pad, pa, c_out, n,
        _opt(bias, "bias"), pool, _dev(out, "out"), _dev(ws, "ws"), ws.numel(), _stream()))
    return out


def conv2d_dense_blocks(x: torch.Tensor, aug: torch.Tensor, kidb: torch.Tensor, kh: int,
                        kw: int, n: int, stride: int = 1, pad: int = 0,
                        bias: torch.Tensor | None = None,
                        out: torch.Tensor | None = None) -> torch.Tensor:
    """Sparse-dense int8 conv with block CS, a block being one pixel's c_in <= 4
    channels (cs_conv2d_dense_blocks); aug and kidb as ops.pack_blocks gives
    them with b = c_in (on the device)."""
    if x.dim() != 4 or x.dtype != torch.int8:
        raise ValueError("x must be int8 NHWC")
    b, h, w, c_in = x.shape
    pa, c_out = _aug(aug, x.dtype, n)
    if kidb.dtype != torch.uint8 or tuple(kidb.shape) != (kh * kw, c_out // n):
        raise ValueError("kidb must be uint8 [kh*kw][c_out/n]")
    ho, wo = conv_out(h, kh, stride, pad), conv_out(w, kw, stride, pad)
    if out is None:
        out = torch.empty((b, max(ho, 0), max(wo, 0), c_out), dtype=torch.int32,
                          device=x.device)
    check("cs_conv2d_dense_blocks", lib().cs_conv2d_dense_blocks(
        _dev(x, "x"), b, h, w, c_in, kh, kw, stride, pad, pa, _dev(kidb, "kidb"), c_out, n,
        _opt(bias, "bias"), _dev(out, "out"), _stream()))
    return out


def conv2d_dense_blocks_plan(in_shape, kh: int, kw: int, c_out: int, n: int, stride: int = 1,
                             pad: int = 0) -> dict | None:
    """How conv2d_dense_blocks runs on the matrix cores, None on the routed kernel
    (host only)."""
    b, h, w, c_in = in_shape
    info = (ctypes.c_int64 * 8)()
    check("cs_conv2d_dense_blocks_plan", lib().cs_conv2d_dense_blocks_plan(
        b, h, w, c_in, kh, kw, stride, pad, c_out, n, info))
    if not info[0]:
        return None
    return {"rows": info[1], "groups": info[2], "segments": info[3], "tiles": info[4],
            "workgroups": info[5], "slices": info[6], "steps": info[7]}


def conv2d_dense(x: torch.Tensor, aug: torch.Tensor, kh: int, kw: int, n: int,
                 stride: int = 1, pad: int = 0, bias: torch.Tensor | None = None, pool: int = 1,
                 out: torch.Tensor | None = None) -> torch.Tensor:
    """Sparse-dense conv (dense NHWC input, no compaction); see cs_conv2d_dense for the
    supported shapes."""
    if x.dim() != 4:
        raise ValueError("x must be NHWC")
    b, h, w, c_in = x.shape
    pa, c_out = _aug(aug, x.dtype, n)
    ho, wo = conv_out(h, kh, stride, pad), conv_out(w, kw, stride, pad)
    ydt = torch.int32 if x.dtype == torch.int8 else torch.float32
    if out is None:
        out = torch.empty((b, max(ho, 0) // pool, max(wo, 0) // pool, c_out), dtype=ydt,
                          device=x.device)
    check("cs_conv2d_dense", lib().cs_conv2d_dense(
        _dt(x), _dev(x, "x"), b, h, w, c_in, kh, kw, stride, pad, pa, c_out, n,
        _opt(bias, "bias"), pool, _dev(out, "out"), _stream()))
    return out


def conv2d_dense_kwta(x: torch.Tensor, aug: torch.Tensor, kh: int, kw: int, n: int,
                      stride: int = 1, pad: int = 0, bias: torch.Tensor | None = None,
                      pool: int = 1, *, k: int, out_dtype: torch.dtype | None = None,
                      shift: int = 0, y: torch.Tensor | None = None, keep_sums: bool = True,
                      cap: int | None = None, lists=None, out: torch.Tensor | None = None):
    """The dense-input first layer with k-WTA (cs_conv2d_dense_kwta).  Returns
    (y, result) as mrs_kwta_conv2d does."""
    if x.dim() != 4:
        raise ValueError("x must be NHWC")
    b, h, w, c_in = x.shape
    pa, c_out = _aug(aug, x.dtype, n)
    ho, wo = conv_out(h, kh, stride, pad), conv_out(w, kw, stride, pad)
    acc_dt = torch.int32 if x.dtype == torch.int8 else torch.float32
    odt = acc_dt if out_dtype is None else out_dtype
    oshape = (b, max(ho, 0) // pool, max(wo, 0) // pool, c_out)
    rows = oshape[0] * oshape[1] * oshape[2]
    if y is None:
        y = torch.empty(oshape, dtype=acc_dt, device=x.device)
    if lists is None and cap is not None:
        lists = (torch.empty((rows, cap), dtype=torch.int16, device=x.device),
                 torch.empty((rows, cap), dtype=odt, device=x.device),
                 torch.empty((rows,), dtype=torch.int32, device=x.device))
    if lists is not None:
        oi, ov, oc = lists
        if oi.dtype != torch.int16 or ov.dtype != odt or oc.dtype != torch.int32:
            raise TypeError("list buffer dtypes do not match")
        if oi.shape != ov.shape or oi.dim() != 2 or oi.shape[0] != rows or oc.shape != (rows,):
            raise ValueError("list buffer shapes do not match the output")
        args = (None, _dev(oi, "oidx"), _dev(ov, "oval"), _dev(oc, "ocnt"), oi.shape[1])
        result = lists
    else:
        if out is None:
            out = torch.empty(oshape, dtype=odt, device=x.device)
        if out.dtype != odt or out.numel() != rows * c_out:
            raise ValueError("out does not match the output")
        args = (_dev(out, "out"), None, None, None, 0)
        result = out
    check("cs_conv2d_dense_kwta", lib().cs_conv2d_dense_kwta(
        _dt(x), _dev(x, "x"), b, h, w, c_in, kh, kw, stride, pad, pa, c_out, n,
        _opt(bias, "bias"), pool, _dev(y, "y"), 1 if keep_sums else 0, k, _TORCH_DT[odt], shift,
        *args, _stream()))
    return y, result


def reorder_table(aug: np.ndarray, kh: int, kw: int, c_in: int, c_out: int, n: int) -> np.ndarray:
    """cs_reorder_table: the fp32 packed kernel (host, from pack) in Kernel-ID
    order, int32 [c_out][smax][2] (tile byte offset, value bits), smax the
    longest support rounded up to a multiple of 8."""
    if not (aug.dtype == np.uint32 and aug.ndim == 3 and aug.shape[2] == 2):
        raise TypeError("reorder_table takes an fp32 packed kernel (uint32 [r][G][2])")
    aug = np.ascontiguousarray(aug)
    smax = ctypes.c_int(0)
    check("cs_reorder_table", lib().cs_reorder_table(aug.ctypes.data, kh, kw, c_in, c_out, n,
                                                     ctypes.byref(smax), None))
    smax.value = (smax.value + 7) // 8 * 8           # the kernel reads 8 entries at a time
    table = np.zeros((c_out, smax.value, 2), dtype=np.int32)
    check("cs_reorder_table", lib().cs_reorder_table(aug.ctypes.data, kh, kw, c_in, c_out, n,
                                                     ctypes.byref(smax), table.ctypes.data))
    return table


def pack_blocks(W: np.ndarray, n: int, b: int):
    """Combine with blocks of b slots on the host (cs_pack_blocks): W [d_out][r]
    int8/float32 -> (aug as pack gives it, kidb uint8 [r/b][G], holes).
    Raises CSError with .bad = (kernel or set, block) when a support splits a
    block (CS_ERR_SHAPE) or two kernels of a set share one (CS_ERR_COLLISION)."""
    W = np.ascontiguousarray(W)
    if W.ndim != 2:
        raise ValueError("W must be [d_out][r]")
    d_out, r = W.shape
    wt = _NP_DT.get(W.dtype)
    if wt is None:
        raise TypeError(f"unsupported weight dtype {W.dtype}")
    G = d_out // n if n > 0 else 0
    aug = (np.zeros((r, max(G, 1)), dtype=np.uint16) if wt == CS_I8
           else np.zeros((r, max(G, 1), 2), dtype=np.uint32))
    kidb = np.zeros((max(r // b, 1) if b > 0 else 1, max(G, 1)), dtype=np.uint8)
    holes = ctypes.c_int64(0)
    bg, bi = ctypes.c_int(0), ctypes.c_int(0)
    st = lib().cs_pack_blocks(wt, W.ctypes.data, d_out, r, n, b, aug.ctypes.data,
                              kidb.ctypes.data, ctypes.byref(holes), ctypes.byref(bg),
                              ctypes.byref(bi))
    if st != _lib.CS_OK:
        err = _lib.CSError("cs_pack_blocks", st)
        err.bad = (bg.value, bi.value)
        raise err
    return aug, kidb, int(holes.value)


def pack_channels(W4: np.ndarray, n: int):
    """Combine along the channel dimension on the host (cs_pack_channels):
    W4 [c_out][kh][kw][c_in] fp32 -> (packed uint32 [c_out][c_in/n][kh][kw][2]
    holding (value bits, channel ID), holes); int8 -> packed uint16
    [c_out][c_in/n][kh][kw] (value byte | channel ID << 8).  Raises CSError
    (CS_ERR_COLLISION) with .bad = (o, slot) on a collision."""
    i8 = np.asarray(W4).dtype == np.int8
    W4 = np.ascontiguousarray(W4, dtype=np.int8 if i8 else np.float32)
    if W4.ndim != 4:
        raise ValueError("W4 must be [c_out][kh][kw][c_in]")
    c_out, kh, kw, c_in = W4.shape
    q = c_in // n if n > 0 else 0
    if i8:
        packed = np.zeros((c_out, max(q, 1), kh, kw), dtype=np.uint16)
    else:
        packed = np.zeros((c_out, max(q, 1), kh, kw, 2), dtype=np.uint32)
    holes = ctypes.c_int64(0)
    bo, bi = ctypes.c_int(0), ctypes.c_int(0)
    st = lib().cs_pack_channels(CS_I8 if i8 else CS_F32, W4.ctypes.data, c_out, kh, kw, c_in, n,
                                packed.ctypes.data, ctypes.byref(holes), ctypes.byref(bo),
                                ctypes.byref(bi))
    if st != _lib.CS_OK:
        err = _lib.CSError("cs_pack_channels", st)
        err.bad = (bo.value, bi.value)
        raise err
    return packed, int(holes.value)


def channel_table(packed: np.ndarray, kh: int, kw: int, c_in: int, c_out: int, n: int,
                  stride: int = 1) -> np.ndarray:
    """cs_channel_table: an int8 channel-overlaid layer's table for
    conv2d_channels at this stride, int32 [c_out][5 * ceil((c_in/n)*kh*kw / 4)]."""
    packed = np.ascontiguousarray(packed, dtype=np.uint16)
    s4 = ((c_in // n) * kh * kw + 3) // 4
    table = np.zeros((c_out, 5 * s4), dtype=np.int32)
    check("cs_channel_table", lib().cs_channel_table(packed.ctypes.data, kh, kw, c_in, c_out, n,
                                                      stride, table.ctypes.data))
    return table


def conv2d_channels(x: torch.Tensor, table: torch.Tensor, kh: int, kw: int, c_out: int, n: int,
                    stride: int = 1, pad: int = 0, bias: torch.Tensor | None = None,
                    out: torch.Tensor | None = None) -> torch.Tensor:
    """int8 dense-input conv with the channel-dimension overlay (cs_conv2d_channels);
    table: device copy of channel_table(...) for this stride."""
    if x.dim() != 4 or x.dtype != torch.int8:
        raise ValueError("x must be int8 NHWC")
    b, h, w, c_in = x.shape
    ho, wo = conv_out(h, kh, stride, pad), conv_out(w, kw, stride, pad)
    if out is None:
        out = torch.empty((b, max(ho, 0), max(wo, 0), c_out), dtype=torch.int32, device=x.device)
    check("cs_conv2d_channels", lib().cs_conv2d_channels(
        _dev(x, "x"), b, h, w, c_in, kh, kw, stride, pad, _dev(table, "table"), c_out, n,
        _opt(bias, "bias"), _dev(out, "out"), _stream()))
    return out


def reorder_table_channels(packed: np.ndarray, kh: int, kw: int, c_in: int, c_out: int,
                           n: int) -> np.ndarray:
    """cs_reorder_table_channels: a channel-overlaid layer's table for
    conv2d_reorder_kwta, int32 [c_out][smax][2] (smax a multiple of 8)."""
    packed = np.ascontiguousarray(packed)
    smax = ctypes.c_int(0)
    check("cs_reorder_table_channels", lib().cs_reorder_table_channels(
        packed.ctypes.data, kh, kw, c_in, c_out, n, ctypes.byref(smax), None))
    smax.value = (smax.value + 7) // 8 * 8
    table = np.zeros((c_out, smax.value, 2), dtype=np.int32)
    check("cs_reorder_table_channels", lib().cs_reorder_table_channels(
        packed.ctypes.data, kh, kw, c_in, c_out, n, ctypes.byref(smax), table.ctypes.data))
    return table


def conv2d_reorder_kwta(x: torch.Tensor, table: torch.Tensor, kh: int, kw: int, pad: int = 0,
                        bias: torch.Tensor | None = None, *, k: int,
                        y: torch.Tensor | None = None, keep_sums: bool = True,
                        cap: int | None = None, lists=None, out: torch.Tensor | None = None):
    """A dense-input fp32 conv layer by reordering (cs_conv2d_reorder_kwta);
    table is reorder_table's result on the device.  Returns (y, result) as
    mrs_kwta_conv2d does."""
    if x.dim() != 4:
        raise ValueError("x must be NHWC")
    if table.dim() != 3 or table.dtype != torch.int32 or table.shape[2] != 2:
        raise ValueError("table must be int32 [c_out][smax][2]")
    b, h, w, c_in = x.shape
    c_out, smax = table.shape[0], table.shape[1]
    ho, wo = conv_out(h, kh, 1, pad), conv_out(w, kw, 1, pad)
    oshape = (b, max(ho, 0), max(wo, 0), c_out)
    rows = oshape[0] * oshape[1] * oshape[2]
    if y is None:
        y = torch.empty(oshape, dtype=torch.float32, device=x.device)
    if lists is None and cap is not None:
        lists = (torch.empty((rows, cap), dtype=torch.int16, device=x.device),
                 torch.empty((rows, cap), dtype=torch.float32, device=x.device),
                 torch.empty((rows,), dtype=torch.int32, device=x.device))
    if lists is not None:
        oi, ov, oc = lists
        if oi.dtype != torch.int16 or ov.dtype != torch.float32 or oc.dtype != torch.int32:
            raise TypeError("list buffer dtypes do not match")
        if oi.shape != ov.shape or oi.dim() != 2 or oi.shape[0] != rows or oc.shape != (rows,):
            raise ValueError("list buffer shapes do not match the output")
        args = (None, _dev(oi, "oidx"), _dev(ov, "oval"), _dev(oc, "ocnt"), oi.shape[1])
        result = lists
    else:
        if out is None:
            out = torch.empty(oshape, dtype=torch.float32, device=x.device)
        if out.dtype != torch.float32 or out.numel() != rows * c_out:
            raise ValueError("out does not match the output")
        args = (_dev(out, "out"), None, None, None, 0)
        result = out
    check("cs_conv2d_reorder_kwta", lib().cs_conv2d_reorder_kwta(
        _dt(x), _dev(x, "x"), b, h, w, c_in, kh, kw, pad, _dev(table, "table"), smax, c_out,
        _opt(bias, "bias"), _dev(y, "y"), 1 if keep_sums else 0, k, CS_F32, *args, _stream()))
    return y, result


def linear(x: torch.Tensor, aug: torch.Tensor, n: int,
           bias: torch.Tensor | None = None, ws: torch.Tensor | None = None,
           out: torch.Tensor | None = None) -> torch.Tensor:
    """Sparse-sparse linear layer: x [batch][d_in], packed aug [d_in][G]."""
    if x.dim() != 2:
        raise ValueError("x must be [batch][d_in]")
    batch, d_in = x.shape
    pa, d_out = _aug(aug, x.dtype, n)
    ydt = torch.int32 if x.dtype == torch.int8 else torch.float32
    if out is None:
        out = torch.empty((batch, d_out), dtype=ydt, device=x.device)
    if ws is None:
        ws = workspace(0, x.dtype, batch, d_in, x.device)
    check("cs_linear", lib().cs_linear(
        _dt(x), _dev(x, "x"), batch, d_in, pa, d_out, n,
        _opt(bias, "bias"), _dev(out, "out"), _dev(ws, "ws"), ws.numel(), _stream()))
    return out


def conv2d_kwta(x: torch.Tensor, aug: torch.Tensor, kh: int, kw: int, n: int, stride: int = 1,
                pad: int = 0, bias: torch.Tensor | None = None, pool: int = 1, *, k: int, ws,
                y: torch.Tensor, out_dtype: torch.dtype | None = None, shift: int = 0,
                keep_sums: bool = True, lists=None, out: torch.Tensor | None = None):
    """A layer with k-WTA on its dense NHWC input (cs_conv2d_kwta); a linear
    layer is a 1x1 layer on 1x1 images.  ws: (idx, val, cnt) buffers
    [pixels][c_in] as compact returns them (cnt holds the non-zero counts
    afterwards, the others are scratch).  Returns (y, result) as
    mrs_kwta_conv2d."""
    if x.dim() != 4:
        raise ValueError("x must be NHWC")
    b, h, w, c_in = x.shape
    pa, c_out = _aug(aug, x.dtype, n)
    if aug.shape[0] != kh * kw * c_in:
        raise ValueError("aug does not match x")
    ho, wo = conv_out(h, kh, stride, pad), conv_out(w, kw, stride, pad)
    rows = b * (max(ho, 0) // pool) * (max(wo, 0) // pool)
    acc_dt = torch.int32 if x.dtype == torch.int8 else torch.float32
    odt = acc_dt if out_dtype is None else out_dtype
    li, lv, lc = ws
    if li.shape != (b * h * w, c_in) or lv.shape != li.shape or lc.shape != (b * h * w,):
        raise ValueError("list buffer shapes do not match x")
    if li.dtype != torch.int16 or lv.dtype != x.dtype or lc.dtype != torch.int32:
        raise TypeError("list buffer dtypes do not match")
    if y.dtype != acc_dt or y.numel() != rows * c_out:
        raise ValueError("y does not match the output")
    if lists is not None:
        oi, ov, oc = lists
        if oi.dtype != torch.int16 or ov.dtype != odt or oc.dtype != torch.int32:
            raise TypeError("list buffer dtypes do not match")
        if oi.shape != ov.shape or oi.dim() != 2 or oi.shape[0] != rows or oc.shape != (rows,):
            raise ValueError("list buffer shapes do not match the output")
        args = (None, _dev(oi, "oidx"), _dev(ov, "oval"), _dev(oc, "ocnt"), oi.shape[1])
        result = lists
    else:
        if out is None:
            out = torch.empty((rows, c_out), dtype=odt, device=x.device)
        if out.dtype != odt or out.numel() != rows * c_out:
            raise ValueError("out does not match the output")
        args = (_dev(out, "out"), None, None, None, 0)
        result = out
    check("cs_conv2d_kwta", lib().cs_conv2d_kwta(
        _dt(x), _dev(x, "x"), b, h, w, c_in, kh, kw, stride, pad, pa, c_out, n,
        _opt(bias, "bias"), pool, _dev(y, "y"), 1 if keep_sums else 0, k, _TORCH_DT[odt], shift,
        *args, _dev(li, "lidx"), _dev(lv, "lval"), _dev(lc, "lcnt"), _stream()))
    return y, result


def kwta(x: torch.Tensor, k: int, out_dtype: torch.dtype | None = None, shift: int = 0,
         out: torch.Tensor | None = None) -> torch.Tensor:
    """k-WTA along the last axis.  out_dtype=torch.int8 on int32 input
    requantises the winners with `shift`."""
    c = x.shape[-1]
    rows = x.numel() // c if c else 0
    odt = x.dtype if out_dtype is None else out_dtype
    if out is None:
        out = torch.empty(x.shape, dtype=odt, device=x.device)
    check("cs_kwta", lib().cs_kwta(_dt(x), _dev(x, "x"), rows, c, k, _TORCH_DT[odt], shift,
                                   _dev(out, "out"), _stream()))
    return out


def list_capacity(k: int) -> int:
    """Row stride for k-entry lists: k rounded up to a multiple of 4 (vector reads)."""
    return max(4, (k + 3) // 4 * 4)


def kwta_lists(x: torch.Tensor, k: int, out_dtype: torch.dtype | None = None, shift: int = 0,
               cap: int | None = None, out=None):
    """k-WTA along the last axis, winners emitted as (idx, val, cnt) lists of
    capacity `cap` (default: list_capacity(k)).  Rows are all leading axes."""
    c = x.shape[-1]
    rows = x.numel() // c if c else 0
    odt = x.dtype if out_dtype is None else out_dtype
    cap = list_capacity(k) if cap is None else cap
    if out is None:
        idx = torch.empty((rows, cap), dtype=torch.int16, device=x.device)
        val = torch.empty((rows, cap), dtype=odt, device=x.device)
        cnt = torch.empty((rows,), dtype=torch.int32, device=x.device)
    else:
        idx, val, cnt = out
    check("cs_kwta_lists", lib().cs_kwta_lists(
        _dt(x), _dev(x, "x"), rows, c, k, _TORCH_DT[odt], shift, _dev(idx, "idx"),
        _dev(val, "val"), _dev(cnt, "cnt"), cap, _stream()))
    return idx, val, cnt


# ------------------------------------------------- 8-bit attention-layer operators
_FLOAT_DT = {torch.float32: CS_F32, torch.float16: CS_F16, torch.bfloat16: CS_BF16}


def _float_dt(t: torch.dtype) -> int:
    try:
        return _FLOAT_DT[t]
    except KeyError:
        raise TypeError(f"unsupported dtype {t}") from None


_INT_MAX = 2 ** 31 - 1           # ctypes would pass on the low 32 bits of a larger number
_current_gpu = torch._C._cuda_getDevice
_current_stream = torch._C._cuda_getCurrentRawStream


def _call(name: str, gpu: int, fn, *args) -> None:
    """fn(*args, stream) on torch's current stream of this GPU, whichever GPU is current.  (The raw
    handle, not _stream()'s Stream object, which costs as much as a launch.)"""
    if gpu == _current_gpu():
        st = fn(*args, _current_stream(gpu))
    else:
        with torch.cuda.device(gpu):
            st = fn(*args, _current_stream(gpu))
    if st:
        check(name, st)


def _gpu(t: torch.Tensor, name: str) -> int:
    gpu = t.get_device()
    if gpu < 0:
        raise ValueError(f"{name} must be a GPU tensor")
    return gpu


def _on(t: torch.Tensor, name: str, gpu: int) -> None:
    if t.get_device() != gpu:
        raise ValueError(f"{name} must be on GPU {gpu}, as the call's other tensors")


def _rows(t: torch.Tensor, name: str, gpu: int):
    """Device pointer, row stride and shape of a matrix on this GPU whose rows are contiguous."""
    shape = t.shape
    _on(t, name, gpu)
    if len(shape) != 2:
        raise ValueError(f"{name} must be a matrix")
    ld, e = t.stride()
    rows, c = shape
    if e != 1 and c > 1:
        raise ValueError(f"{name}'s rows must be contiguous")
    if c > _INT_MAX:
        raise ValueError(f"{name}'s rows have more than 2^31 - 1 elements")
    return t.data_ptr(), ld if rows > 1 else max(ld, c), rows, c


def _heads(t: torch.Tensor, name: str, gpu: int):
    """Device pointer, token stride and head stride of a tensor [tokens][heads][d] on this GPU."""
    _on(t, name, gpu)
    if t.dim() != 3:
        raise ValueError(f"{name} must be [tokens][heads][d]")
    tokens, heads, d = t.shape
    ts, hs, e = t.stride()
    if e != 1 and d > 1:
        raise ValueError(f"{name}'s heads must be contiguous")
    if heads <= 1:
        hs = d
    return t.data_ptr(), ts if tokens > 1 else heads * hs, hs


def _dense(t: torch.Tensor, name: str, gpu: int) -> int:
    _on(t, name, gpu)
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return t.data_ptr()


def _vector(t: torch.Tensor | None, name: str, dtype: torch.dtype, n: int, gpu: int):
    if t is None:
        return None
    if t.dtype != dtype or t.shape != (n,):
        raise ValueError(f"{name} must be {dtype} [{n}]")
    return _dense(t, name, gpu)


def _ws(ws: torch.Tensor | None, need, device, gpu: int):
    """A workspace, its pointer and size; one of need() bytes made for the call where the caller
    keeps none (torch's allocator orders its reuse on the stream)."""
    if ws is None:
        ws = torch.empty((need(),), dtype=torch.uint8, device=device)
    return ws, _dense(ws, "ws", gpu), ws.numel() * ws.element_size()


def quantise_rows(x: torch.Tensor, q: torch.Tensor | None = None,
                  scale: torch.Tensor | None = None):
    """Codes int8 [rows][c] and scales float32 [rows] of the rows of x (float32, float16 or
    bfloat16 [rows][c]): cs_quantise_rows.  Codes made here have a row stride that is a multiple
    of 16, which cs_linear_q8 reads fastest."""
    gpu = _gpu(x, "x")
    px, ldx, rows, c = _rows(x, "x", gpu)
    if q is None:
        q = torch.empty((rows, (c + 15) // 16 * 16), dtype=torch.int8, device=x.device)[:, :c]
    if q.dtype != torch.int8 or q.shape != x.shape:
        raise ValueError("q must be int8 of x's shape")
    if scale is None:
        scale = torch.empty((rows,), dtype=torch.float32, device=x.device)
    pq, ldq, _, _ = _rows(q, "q", gpu)
    _call("cs_quantise_rows", gpu, lib().cs_quantise_rows, _float_dt(x.dtype), px, ldx, rows, c, pq,
          ldq, _vector(scale, "scale", torch.float32, rows, gpu))
    return q, scale


def linear_q8_workspace(dtype: torch.dtype, rows: int, k: int, d_out: int,
                        device="cuda") -> torch.Tensor:
    """Workspace of linear_q8 for inputs of up to `rows` rows of this dtype."""
    dt = CS_I8 if dtype == torch.int8 else _float_dt(dtype)
    return torch.empty((int(lib().cs_linear_q8_workspace_bytes(dt, rows, k, d_out)),),
                       dtype=torch.uint8, device=device)


def linear_q8(x: torch.Tensor, w: torch.Tensor, sw: torch.Tensor, sx: torch.Tensor | None = None,
              bias: torch.Tensor | None = None, out_dtype: torch.dtype | None = None,
              ws: torch.Tensor | None = None, out: torch.Tensor | None = None) -> torch.Tensor:
    """y = (x @ w.T) * sx * sw + bias on 8-bit codes (cs_linear_q8).  w int8 [d_out][k] with
    scales sw (quantise_rows of the weight matrix gives both).  x [rows][k] is int8 with scales
    sx, or a float tensor that the call quantises row by row.  out_dtype: x's by default, float32
    for int8 x."""
    gpu = _gpu(x, "x")
    px, ldx, rows, k = _rows(x, "x", gpu)
    pw, ldw, d_out, kw = _rows(w, "w", gpu)
    xdt = x.dtype
    if w.dtype != torch.int8 or kw != k:
        raise ValueError(f"w must be int8 [d_out][{k}]")
    if d_out > _INT_MAX:
        raise ValueError("w has more than 2^31 - 1 rows")
    codes = xdt == torch.int8
    xt = CS_I8 if codes else _float_dt(xdt)
    if codes != (sx is not None):
        raise ValueError("sx goes with int8 x")
    if out_dtype is None:
        out_dtype = torch.float32 if codes else xdt
    if out is None:
        out = x.new_empty((rows, d_out), dtype=out_dtype)
        py, ldy = out.data_ptr(), d_out
    else:
        py, ldy, yr, yc = _rows(out, "out", gpu)
        if out.dtype != out_dtype or yr != rows or yc != d_out:
            raise ValueError(f"out must be {out_dtype} [{rows}][{d_out}]")
    L = lib()
    ws, pws, nws = _ws(ws, lambda: L.cs_linear_q8_workspace_bytes(xt, rows, k, d_out), x.device,
                       gpu)
    _call("cs_linear_q8", gpu, L.cs_linear_q8,
          xt, px, ldx, _vector(sx, "sx", torch.float32, rows, gpu), rows, k, pw, ldw,
          _vector(sw, "sw", torch.float32, d_out, gpu), d_out,
          _vector(bias, "bias", torch.float32, d_out, gpu), _float_dt(out_dtype), py, ldy, pws,
          nws)
    return out


@dataclass(frozen=True)
class PagedCache:
    """Keys and values of many sequences in 8 bits (cs_q8_cache): codes int8
    [pages][heads][page][d], scales float32 [pages][heads][page]."""
    k: torch.Tensor
    v: torch.Tensor
    k_scale: torch.Tensor
    v_scale: torch.Tensor

    def __post_init__(self):
        if self.k.dim() != 4:
            raise ValueError("codes must be [pages][heads][page][d]")
        for t, dt, shape, name in ((self.k, torch.int8, self.k.shape, "k"),
                                   (self.v, torch.int8, self.k.shape, "v"),
                                   (self.k_scale, torch.float32, self.k.shape[:3], "k_scale"),
                                   (self.v_scale, torch.float32, self.k.shape[:3], "v_scale")):
            if t.dtype != dt or t.shape != shape:
                raise ValueError(f"{name} must be {dt} {list(shape)}")
            if not t.is_contiguous():
                raise ValueError(f"{name} must be contiguous")
            if t.device != self.k.device:
                raise ValueError(f"{name} must be on {self.k.device}, as k is")
        c = _lib.Q8Cache(self.k.data_ptr(), self.v.data_ptr(), self.k_scale.data_ptr(),
                         self.v_scale.data_ptr(), *self.k.shape)
        for name, value in (("_c", c), ("_ref", ctypes.byref(c)),
                            *zip(("pages", "heads", "page", "d"), self.k.shape)):
            object.__setattr__(self, name, value)

    @classmethod
    def empty(cls, pages: int, heads: int, page: int, d: int, device="cuda") -> "PagedCache":
        def codes():
            return torch.empty((pages, heads, page, d), dtype=torch.int8, device=device)

        def scales():
            return torch.empty((pages, heads, page), dtype=torch.float32, device=device)
        return cls(codes(), codes(), scales(), scales())

    def _ptr(self, gpu: int):
        _on(self.k, "the cache", gpu)
        return self._ref


def cache_write(cache: PagedCache, k: torch.Tensor, v: torch.Tensor, slots: torch.Tensor) -> None:
    """Quantise k and v (float [tokens][heads][d]) into the cache's slots (int64 [tokens], slot =
    page number * page + offset; one outside the cache leaves its token out): cs_cache_write."""
    gpu = _gpu(k, "k")
    pk, ldk, hsk = _heads(k, "k", gpu)
    pv, ldv, hsv = _heads(v, "v", gpu)
    shape = k.shape
    if k.dtype != v.dtype or v.shape != shape or shape[1] != cache.heads or shape[2] != cache.d:
        raise ValueError(f"k and v must be of one type and [tokens][{cache.heads}][{cache.d}]")
    _call("cs_cache_write", gpu, lib().cs_cache_write,
          cache._ptr(gpu), _float_dt(k.dtype), pk, ldk, hsk, pv, ldv, hsv,
          _vector(slots, "slots", torch.int64, shape[0], gpu), shape[0])


def cache_read(cache: PagedCache, slots: torch.Tensor, dtype: torch.dtype,
               out: tuple | None = None):
    """(k, v), each [tokens][heads][d] of `dtype`, of the slots' tokens: cs_cache_read."""
    gpu = _gpu(slots, "slots")
    shape = (slots.shape[0], cache.heads, cache.d)
    if out is None:
        out = (slots.new_empty(shape, dtype=dtype), slots.new_empty(shape, dtype=dtype))
    else:
        for t in out:
            if t.dtype != dtype or t.shape != shape:
                raise ValueError(f"out must be {dtype} {list(shape)}")
    _call("cs_cache_read", gpu, lib().cs_cache_read,
          cache._ptr(gpu), _vector(slots, "slots", torch.int64, shape[0], gpu), shape[0],
          _float_dt(dtype), _dense(out[0], "out", gpu), _dense(out[1], "out", gpu))
    return out


def _attention_args(q: torch.Tensor, cache: PagedCache, table: torch.Tensor, max_len: int | None):
    """q's dtype and the sizes of a call, as cs_paged_attention_workspace_bytes takes them."""
    shape, pages = q.shape, table.shape
    if len(shape) != 3 or shape[2] != cache.d:
        raise ValueError(f"q must be [tokens][q_heads][{cache.d}]")
    if table.dtype != torch.int32 or len(pages) != 2:
        raise ValueError("table must be int32 [batch][pages]")
    tokens, q_heads, _ = shape
    batch, width = pages
    if tokens | q_heads | batch | width > _INT_MAX:           # none is negative
        raise ValueError("q or table has a dimension over 2^31 - 1")
    ml = 0 if max_len is None else int(max_len)
    return _float_dt(q.dtype), tokens, q_heads, batch, width, ml if ml < _INT_MAX else _INT_MAX


def paged_attention_workspace(q: torch.Tensor, cache: PagedCache, table: torch.Tensor,
                              max_len: int | None = None) -> torch.Tensor:
    """Workspace of paged_attention for arguments of these shapes."""
    n = lib().cs_paged_attention_workspace_bytes(
        cache._ref, *_attention_args(q, cache, table, max_len))
    return torch.empty((int(n),), dtype=torch.uint8, device=q.device)


def paged_attention_plan(dtype: torch.dtype, heads: int, page: int, d: int, tokens: int,
                         q_heads: int, batch: int, table_width: int, max_len: int | None = None,
                         window: int = 0) -> dict:
    """How paged_attention runs these sizes (host only): cs_paged_attention_plan."""
    # the cache's arrays are not touched; any aligned address stands for them
    cache = _lib.Q8Cache(16, 16, 16, 16, 1, heads, page, d)
    info = (ctypes.c_int64 * 6)()
    check("cs_paged_attention_plan", lib().cs_paged_attention_plan(
        ctypes.byref(cache), _float_dt(dtype), tokens, q_heads, batch, table_width,
        0 if max_len is None else min(int(max_len), _INT_MAX), min(window, _INT_MAX), info))
    return dict(zip(("rows", "parts", "part", "wavefronts", "workgroups", "bytes"), info))


def paged_attention(q: torch.Tensor, cache: PagedCache, table: torch.Tensor, lens: torch.Tensor,
                    starts: torch.Tensor, *, scale: float | None = None, window: int = 0,
                    max_len: int | None = None, ws: torch.Tensor | None = None,
                    out: torch.Tensor | None = None) -> torch.Tensor:
    """Causal attention of each sequence's new tokens over the cache that already holds them
    (cs_paged_attention).  q float [tokens][q_heads][d]; table int32 [batch][pages] page numbers;
    lens int32 [batch] positions with the new ones; starts int32 [batch + 1] first new token of
    each sequence in q.  scale: 1 / sqrt(d) by default.  window: positions seen, 0 for all.
    max_len: the longest of lens if the caller knows it (a hint for how the work is split)."""
    qt, tokens, q_heads, b, width, ml = _attention_args(q, cache, table, max_len)
    if window > _INT_MAX:                                     # hides nothing either
        window = _INT_MAX
    gpu = _gpu(q, "q")
    pq, ldq, hsq = _heads(q, "q", gpu)
    if out is None:
        out = q.new_empty(q.shape)
    elif out.dtype != q.dtype or out.shape != q.shape:
        raise ValueError("out must be of q's type and shape")
    L = lib()
    ws, pws, nws = _ws(ws, lambda: L.cs_paged_attention_workspace_bytes(
        cache._ref, qt, tokens, q_heads, b, width, ml), q.device, gpu)
    _call("cs_paged_attention", gpu, L.cs_paged_attention,
          cache._ptr(gpu), qt, pq, ldq, hsq, tokens, q_heads, b, _dense(table, "table", gpu), width,
          _vector(lens, "lens", torch.int32, b, gpu),
          _vector(starts, "starts", torch.int32, b + 1, gpu), ml,
          1.0 / math.sqrt(cache.d) if scale is None else scale, window, _dense(out, "out", gpu),
          pws, nws)
    return out
