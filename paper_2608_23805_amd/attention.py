"""Binding of the attention block's operators: projection with its epilogue
(``linear``, with 4-bit weights ``linear_q4``), the paged cache of keys and
values in 8 bits (``KvCache``, ``KvSeqs``, ``kv_append``, ``kv_read``, with
rotation by positions ``KvRotary``, ``kv_append_rotary``), the attention that
reads it (``kv_attention``, over pages that sequences share ``KvGroups``,
``kv_attention_shared``) and its eviction (``kv_evict``); see ``include/msi.h``.
``AttentionBlock`` runs them in a row as the attention block of a stacked layer.

A decode step makes several of these calls a layer, each a few microseconds
of GPU time, so a call checks its tensors with few attribute reads and packs
its argument struct in one step.  Calls run on the device that holds the
tensors; a call whose tensors lie on several devices is refused."""
from __future__ import annotations

import ctypes
import math
import struct
from typing import Optional

import torch

from . import (ACTIVATIONS, KV_ALL_ROWS, KV_FORMATS, MSI_BF16, MSI_E_INVALID_ARG, MSI_E_NOMEM, MSI_F32, MSI_KV_BLOCK,
               MSI_OK, MsiError, lib, msi_kv_append_rotary_args, msi_kv_attention_args, msi_kv_cache, msi_kv_evict_args,
               msi_kv_groups, msi_kv_seqs, msi_linear_args, msi_linear_q4_args, _check)

_BF16 = (torch.bfloat16, torch.int16)            # bf16 tensors, or their bits
_F16 = (torch.float16, torch.int16)              # likewise fp16
_F32, _I32 = torch.float32, torch.int32
_pack_linear = struct.Struct("<5Q6I3Q")
_pack_q4 = struct.Struct("<Q2I")
_pack_attention = struct.Struct("<4QIfIf3Q")
_pack_rotary = struct.Struct("<8Q4I5Q")
_pack_evict = struct.Struct("<4I4Q")
for _s, _c in ((_pack_linear, msi_linear_args), (_pack_attention, msi_kv_attention_args), (_pack_evict, msi_kv_evict_args),
               (_pack_rotary, msi_kv_append_rotary_args)):
    assert _s.size == ctypes.sizeof(_c)
assert _pack_linear.size + _pack_q4.size == ctypes.sizeof(msi_linear_q4_args)


def _refuse(msg: str):
    raise MsiError(MSI_E_INVALID_ARG, msg)


# the current device without the public call's look whether HIP is initialised: a tensor on a device shows that it is
_current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)


def _call(device, fn, *args):
    """The library call, with the tensors' device current."""
    index = device.index
    if index is None:
        _refuse(f"tensors must be on a HIP device, got {device}")
    if index == _current_device():
        st = fn(*args)
    else:
        with torch.cuda.device(device):
            st = fn(*args)
    if st != MSI_OK:
        _check(st)


def _stream(s, device) -> Optional[int]:
    """The handle of a stream (torch's, or a handle already); torch's tell their device, which must be the tensors'."""
    if s is None:
        return None
    if getattr(s, "device_index", device.index) != device.index:
        _refuse(f"the stream is on device {s.device_index}, the tensors are on {device}")
    return getattr(s, "cuda_stream", s)


def _dense(name: str, t, dtype, device, shape=None):
    if t.dtype != dtype or t.device != device or not t.is_contiguous():
        _refuse(f"{name} must be contiguous {dtype} on {device}")
    if shape is not None and t.shape != shape:
        _refuse(f"{name} must have shape {tuple(shape)}, got {tuple(t.shape)}")


def _status(status, device) -> int:
    if status is None:
        return 0
    _dense("status", status, _I32, device)
    if status.numel() < 1:
        _refuse("status must hold a word")
    return status.data_ptr()


def _matrix(name: str, t, M: int, N: int, device, dtypes) -> int:
    """Row stride of an [M, N] tensor with contiguous rows (of a single row: any that is a multiple of 8)."""
    if t.shape != (M, N) or t.dtype not in dtypes or t.device != device:
        _refuse(f"{name} must be [{M}, {N}] {' or '.join(map(str, dtypes))} on {device}, "
                f"got {tuple(t.shape)} {t.dtype} on {t.device}")
    return _row_stride(name, t, M, N)


def _row_stride(name: str, t, M: int, N: int) -> int:
    """Row stride of a tensor of shape [M, N]."""
    if M == 0:
        return (N + 7) // 8 * 8              # (a tensor without elements may have any strides)
    rs, cs = t.stride()
    if (cs != 1 and N > 1) or (rs < N and M > 1):
        _refuse(f"{name}: rows must be contiguous in themselves and must not overlap")
    return rs if M > 1 else (N + 7) // 8 * 8


_ANY = _BF16 + (_F32,)
_F32_MOST = torch.finfo(_F32).max


def _scale(scale: float):
    """The factor of the scores: as a power of two's exponent it has to be a number of fp32."""
    if not abs(scale) * 1.4426950408889634 <= _F32_MOST:
        _refuse(f"scale must be finite, under 2^127, got {scale}")


def _decay(mass_decay: float):
    if not 0.0 <= mass_decay <= _F32_MOST:
        _refuse(f"mass_decay must be finite in fp32 and not negative, got {mass_decay}")


def _pack(x, dev, M: int, K: int, w, N: int, out, bias, act: str, residual) -> bytes:
    """The arguments of a projection (msi_linear_args) of x [M, K] whose weights w [N, ...] have been checked."""
    if x.dtype not in _BF16:
        _refuse(f"x must be {' or '.join(map(str, _BF16))}, got {x.dtype}")
    xs = _row_stride("x", x, M, K)
    code = ACTIVATIONS.get(act)
    if code is None:
        _refuse(f"unknown activation {act!r}")
    if bias is not None:
        _dense("bias", bias, _F32, dev, (N,))
    os_ = _matrix("out", out, M, N, dev, _ANY)
    rp = rs = rt = 0
    if residual is not None:
        rs = _matrix("residual", residual, M, N, dev, _ANY)
        rp, rt = residual.data_ptr(), MSI_F32 if residual.dtype == _F32 else MSI_BF16
    return _pack_linear.pack(x.data_ptr(), w.data_ptr(), 0 if bias is None else bias.data_ptr(), rp, out.data_ptr(),
                             M, N, K, code, rt, MSI_F32 if out.dtype == _F32 else MSI_BF16, xs, rs, os_)


def linear(x, w, out, bias=None, act: str = "none", residual=None, stream=None):
    """out = act(x w^T + bias) + residual (msi_linear).

    x [M, K] and w [N, K] bf16 (x's rows may be strided), bias [N] float32,
    residual and out [M, N] bf16 or float32 with strided rows; residual may be out."""
    dev, xshape, wshape = x.device, x.shape, w.shape
    if len(xshape) != 2 or len(wshape) != 2:
        _refuse("x and w must be matrices")
    if w.dtype not in _BF16:
        _refuse(f"w must be bf16 (or its bits in int16), got {w.dtype}")
    (M, K), N = xshape, wshape[0]
    _dense("w", w, w.dtype, dev, (N, K))
    _call(dev, lib.msi_linear, _pack(x, dev, M, K, w, N, out, bias, act, residual), _stream(stream, dev))


def linear_q4(x, w, scales, out, bias=None, act: str = "none", residual=None, stream=None):
    """out = act(x W^T + bias) + residual with 4-bit weights W[n, k] = scales[n, k / group] * q[n, k] (msi_linear_q4).

    w [N, K / 2] uint8: the codes q = -8 .. 7, element 2j in the low nibble of byte j; scales [N, K / group] float16 (or
    its bits in int16), group 32, 64 or 128; the others as ``linear``'s.  It takes less time than ``linear`` up to some 256
    rows (half of it for single tokens), more from 512 on."""
    dev, xshape, sshape = x.device, x.shape, scales.shape
    if len(xshape) != 2 or len(sshape) != 2 or w.dim() != 2:
        _refuse("x, w and scales must be matrices")
    (M, K), (N, groups) = xshape, sshape
    group = K // groups if groups else 0
    if group not in (32, 64, 128) or group * groups != K:
        _refuse(f"scales must be [N, K / 32], [N, K / 64] or [N, K / 128], got {tuple(sshape)} for K = {K}")
    _dense("w", w, torch.uint8, dev, (N, K // 2))
    if scales.dtype not in _F16 or scales.device != dev or not scales.is_contiguous():
        _refuse(f"scales must be contiguous float16 (or its bits in int16) on {dev}, got {scales.dtype} on {scales.device}")
    _call(dev, lib.msi_linear_q4,
          _pack(x, dev, M, K, w, N, out, bias, act, residual) + _pack_q4.pack(scales.data_ptr(), group, 0), _stream(stream, dev))


class KvCache:
    """One layer's pages of keys and values in 8 bits (msi_kv_cache).

    data [n_pages, n_heads, 2, 64, head_dim] uint8, scales [n_pages, n_heads, 2]
    float32, mass [n_pages, n_heads, 64] float32 or None; ``alloc`` makes them.
    Memory that no append or eviction has written holds no tokens: its contents do not matter."""

    def __init__(self, data, scales, mass=None, fmt: str = "e4m3"):
        if fmt not in KV_FORMATS:
            _refuse(f"unknown cache format {fmt!r}")
        if data.dim() != 5 or data.shape[2] != 2 or data.shape[3] != MSI_KV_BLOCK:
            _refuse("data must be [n_pages, n_heads, 2, 64, head_dim]")
        P, H, _, _, D = data.shape
        _dense("data", data, torch.uint8, data.device)
        _dense("scales", scales, _F32, data.device, (P, H, 2))
        if mass is not None:
            _dense("mass", mass, _F32, data.device, (P, H, MSI_KV_BLOCK))
        self.data, self.scales, self.mass, self.fmt = data, scales, mass, fmt
        self.n_pages, self.n_heads, self.head_dim, self.device = P, H, D, data.device
        self.c = msi_kv_cache(KV_FORMATS[fmt], P, H, D, data.data_ptr(), scales.data_ptr(),
                              None if mass is None else mass.data_ptr())
        self._ref = ctypes.byref(self.c)

    @staticmethod
    def alloc(n_pages: int, n_heads: int, head_dim: int, fmt: str = "e4m3", mass: bool = True, device="cuda") -> "KvCache":
        data = torch.empty((n_pages, n_heads, 2, MSI_KV_BLOCK, head_dim), dtype=torch.uint8, device=device)
        scales = torch.empty((n_pages, n_heads, 2), dtype=_F32, device=device)
        m = torch.zeros((n_pages, n_heads, MSI_KV_BLOCK), dtype=_F32, device=device) if mass else None
        return KvCache(data, scales, m, fmt)


class KvSeqs:
    """The sequences of a call (msi_kv_seqs): page table [n_seqs, max_blocks],
    token counts [n_seqs] and row offsets [n_seqs + 1] in device int32 tensors,
    whose contents may change between calls, and the host's bounds on them."""

    def __init__(self, table, lens, cu_rows=None, *, n_rows: int = 0, max_rows: int = 0, max_len: Optional[int] = None):
        dev = lens.device
        if table.dim() != 2:
            _refuse("table must be [n_seqs, max_blocks]")
        S, nb = table.shape
        _dense("table", table, _I32, dev)
        _dense("lens", lens, _I32, dev, (S,))
        if cu_rows is not None:
            _dense("cu_rows", cu_rows, _I32, dev, (S + 1,))
        self.table, self.lens, self.cu_rows = table, lens, cu_rows
        self.n_rows, self.max_rows = int(n_rows), int(max_rows)
        self.max_len = nb * MSI_KV_BLOCK if max_len is None else int(max_len)
        self.n_seqs, self.max_blocks, self.device = S, nb, dev
        if min(self.n_rows, self.max_rows, self.max_len) < 0 or max(self.n_rows, self.max_rows, self.max_len) >= 1 << 31:
            _refuse("n_rows, max_rows and max_len must be 0 .. 2^31 - 1")
        self.c = msi_kv_seqs(S, nb, self.n_rows, self.max_rows, self.max_len, 0, table.data_ptr(), lens.data_ptr(),
                             None if cu_rows is None else cu_rows.data_ptr())
        self._ref = ctypes.byref(self.c)


def _rows(cache: KvCache, seqs: KvSeqs, name: str, t, heads: int) -> int:
    """Row stride of a [n_rows, heads, head_dim] tensor whose rows are contiguous in themselves."""
    n, D = seqs.n_rows, cache.head_dim
    if t.shape != (n, heads, D) or t.dtype not in _BF16 or t.device != cache.device:
        _refuse(f"{name} must be [{n}, {heads}, {D}] bf16 (or its bits in int16) on {cache.device}, "
                f"got {tuple(t.shape)} {t.dtype} on {t.device}")
    if n == 0:
        return heads * D
    rs, hs, ds = t.stride()
    if ds != 1 or (hs != D and heads > 1) or (rs < heads * D and n > 1):
        _refuse(f"{name}: rows must be contiguous in themselves and must not overlap")
    return rs if n > 1 else heads * D


def _same_device(cache: KvCache, seqs: KvSeqs):
    if seqs.device != cache.device:
        _refuse("cache and sequences must be on one device")


def kv_append(cache: KvCache, seqs: KvSeqs, k, v, status=None, stream=None):
    """Write the last rows of every sequence into its pages (msi_kv_append); k, v [n_rows, n_heads, head_dim] bf16."""
    _same_device(cache, seqs)
    H, dev = cache.n_heads, cache.device
    ks, vs = _rows(cache, seqs, "k", k, H), _rows(cache, seqs, "v", v, H)
    _call(dev, lib.msi_kv_append, cache._ref, seqs._ref, k.data_ptr(), v.data_ptr(), ks, vs, _status(status, dev),
          _stream(stream, dev))


def _arctan_of(n: int, one: int) -> int:
    """arctan(1 / n) in units of 1 / one, by its power series."""
    power = total = one // n
    k = 1
    while power:
        power //= -n * n
        k += 2
        total += power // k
    return total


# 2 pi (Machin's formula): a double reaches 2^1024, whose fraction of a turn to 2^-65 takes 2 pi to 2^-1090 of itself
_PI_BITS = 1200
_TWO_PI = 8 * (4 * _arctan_of(5, 1 << _PI_BITS) - _arctan_of(239, 1 << _PI_BITS))


def _turns(x: float) -> int:
    """An angle's fraction of a turn in units of 2^-64, to the nearest."""
    n, d = x.as_integer_ratio()
    d *= _TWO_PI
    return ((n << _PI_BITS + 65) + d) // (2 * d) % 2 ** 64


class KvRotary:
    """How positions rotate queries and keys (the constant part of msi_kv_append_rotary's arguments).

    inv_freq: the frequencies, radians for each position; pair i of a head's first 2 len(inv_freq) elements turns by
    position * inv_freq[i], the pairs being (i, i + len(inv_freq)) or, ``interleaved``, (2 i, 2 i + 1).  ``axes`` gives
    the pairs' axes for rows with several positions (time, height, width): a list as long as inv_freq, of 0 .. 3."""

    def __init__(self, inv_freq, axes=None, interleaved: bool = False, device="cuda"):
        f = [float(x) for x in inv_freq]
        if len(f) % 8 or not 8 <= len(f) <= 128:
            _refuse(f"inv_freq must hold a multiple of 8 frequencies, 8 .. 128, got {len(f)}")
        if not all(math.isfinite(x) for x in f):
            _refuse("inv_freq must be finite")
        a = None if axes is None else [int(x) for x in axes]
        if a is not None and (len(a) != len(f) or min(a) < 0 or max(a) > 3):
            _refuse("axes must be as many as the frequencies, 0 .. 3")
        turns = [_turns(x) for x in f]
        self.rot_dim, self.interleaved = 2 * len(f), bool(interleaved)
        self.n_axes = 1 if a is None else max(a) + 1
        self.freq = torch.tensor([t - (t >> 63 << 64) for t in turns], dtype=torch.int64).to(device)
        self.axis = None if self.n_axes == 1 else torch.tensor(a, dtype=torch.uint8).to(device)
        self.device = self.freq.device
        self._freq, self._axis = self.freq.data_ptr(), 0 if self.axis is None else self.axis.data_ptr()


def _positions(rotary: KvRotary, positions, n: int, device) -> int:
    """Stride from one axis of the positions to the next."""
    if positions is None:
        _refuse("positions are needed")
    axes, shape = rotary.n_axes, positions.shape
    if (shape != (axes, n) and (axes > 1 or shape != (n,))) or positions.dtype != _I32 or positions.device != device or \
            rotary.device != device:
        _refuse(f"positions must be int32 [{axes}, {n}] on {device}, as rotary, got {tuple(shape)} {positions.dtype} on "
                f"{positions.device} and rotary on {rotary.device}")
    strides = positions.stride()
    if n > 1 and strides[-1] != 1:
        _refuse("an axis of positions must be contiguous")
    if axes == 1:
        return n
    if strides[0] < n:
        _refuse("axes of positions must not overlap")
    return strides[0]


def kv_append_rotary(cache: KvCache, seqs: KvSeqs, rotary: KvRotary, positions, q, q_out, k, v, status=None, stream=None):
    """kv_append with queries and keys rotated by their positions on the way (msi_kv_append_rotary).

    positions int32 [rotary.n_axes, n_rows], or [n_rows] for one axis; q [n_rows, n_q_heads, head_dim] bf16 is rotated
    into q_out (which may be q), or None; k, v [n_rows, n_heads, head_dim] bf16."""
    _same_device(cache, seqs)
    H, dev, n = cache.n_heads, cache.device, seqs.n_rows
    step = _positions(rotary, positions, n, dev)
    if rotary.rot_dim > cache.head_dim:
        _refuse(f"{rotary.rot_dim} elements rotate, heads have {cache.head_dim}")
    qp = op = qs = os_ = Hq = 0
    if (q is None) != (q_out is None):
        _refuse("q and q_out go together")
    if q is not None:
        shape = q.shape
        if len(shape) != 3:
            _refuse("q must be [n_rows, n_q_heads, head_dim]")
        Hq = shape[1]
        qs, os_ = _rows(cache, seqs, "q", q, Hq), _rows(cache, seqs, "q_out", q_out, Hq)
        qp, op = q.data_ptr(), q_out.data_ptr()
    ks, vs = _rows(cache, seqs, "k", k, H), _rows(cache, seqs, "v", v, H)
    _call(dev, lib.msi_kv_append_rotary, cache._ref, seqs._ref,
          _pack_rotary.pack(qp, op, k.data_ptr(), v.data_ptr(), qs, os_, ks, vs, Hq, rotary.rot_dim, rotary.n_axes,
                            rotary.interleaved, rotary._freq, rotary._axis, positions.data_ptr(), step, _status(status, dev)),
          _stream(stream, dev))


def kv_read(cache: KvCache, seqs: KvSeqs, k, v, status=None, stream=None):
    """The last rows of every sequence as bf16 into k, v [n_rows, n_heads, head_dim] (msi_kv_read)."""
    _same_device(cache, seqs)
    H, dev = cache.n_heads, cache.device
    ks, vs = _rows(cache, seqs, "k", k, H), _rows(cache, seqs, "v", v, H)
    _call(dev, lib.msi_kv_read, cache._ref, seqs._ref, k.data_ptr(), v.data_ptr(), ks, vs, _status(status, dev),
          _stream(stream, dev))


def kv_attention_workspace_size(cache: KvCache, seqs: KvSeqs, n_q_heads: int, mass_rows: int = 0) -> int:
    """Bytes of workspace of kv_attention calls with these bounds."""
    n = ctypes.c_uint64()
    if n_q_heads < 0 or mass_rows < 0:
        _refuse("n_q_heads and mass_rows must not be negative")
    _check(lib.msi_kv_attention_workspace(cache._ref, seqs._ref, n_q_heads, min(mass_rows, 1 << 30), ctypes.byref(n)))
    return n.value


def kv_attention_workspace(cache: KvCache, seqs: KvSeqs, n_q_heads: int, mass_rows: int = 0):
    """Workspace of kv_attention calls with these bounds (a uint8 tensor)."""
    return torch.empty(kv_attention_workspace_size(cache, seqs, n_q_heads, mass_rows), dtype=torch.uint8,
                       device=cache.device)


def _attention(cache: KvCache, seqs: KvSeqs, q, out, scale: float, mass_rows: int, mass_decay: float, workspace, status,
               all_rows: bool):
    """The sequences and arguments of an attention call."""
    if q.dim() != 3:
        _refuse("q must be [n_rows, n_q_heads, head_dim]")
    if mass_rows < 0:
        _refuse("mass_rows must not be negative")
    _scale(scale)
    if mass_rows:
        _decay(mass_decay)
    Hq, dev = q.shape[1], cache.device
    qs, os_ = _rows(cache, seqs, "q", q, Hq), _rows(cache, seqs, "out", out, Hq)
    wp = wn = 0
    if workspace is not None:
        _dense("workspace", workspace, torch.uint8, dev)
        wp, wn = workspace.data_ptr(), workspace.numel()
    ref = seqs._ref
    if all_rows:
        c = msi_kv_seqs.from_buffer_copy(seqs.c)
        c.flags |= KV_ALL_ROWS
        ref = ctypes.byref(c)
    return ref, _pack_attention.pack(q.data_ptr(), out.data_ptr(), qs, os_, Hq, scale, min(mass_rows, 1 << 30),
                                     mass_decay if mass_rows else 0.0, wp, wn, _status(status, dev))


def kv_attention(cache: KvCache, seqs: KvSeqs, q, out, scale: float, mass_rows: int = 0, mass_decay: float = 1.0,
                 workspace=None, status=None, stream=None, all_rows: bool = False):
    """Attention of q [n_rows, n_q_heads, head_dim] bf16 over the sequences' pages into out (msi_kv_attention).

    all_rows: every row of out is written, with zeros where no sequence answers for it (MSI_KV_ALL_ROWS)."""
    _same_device(cache, seqs)
    ref, args = _attention(cache, seqs, q, out, scale, mass_rows, mass_decay, workspace, status, all_rows)
    _call(cache.device, lib.msi_kv_attention, cache._ref, ref, args, _stream(stream, cache.device))


class KvGroups:
    """Groups of neighbouring sequences that hold the same first pages (msi_kv_groups): first sequence of every group
    [n_groups + 1] and shared blocks [n_groups] in device int32 tensors, whose contents may change between calls, and the
    host's bounds: ``max_rows`` rows of a group, ``max_blocks`` shared blocks.  A sequence whose rows do not all stand behind
    the shared blocks is attended by itself, with a table of its own."""

    def __init__(self, cu_seqs, blocks, *, max_rows: int, max_blocks: int):
        dev = blocks.device
        if blocks.dim() != 1:
            _refuse("blocks must be [n_groups]")
        n = blocks.shape[0]
        _dense("blocks", blocks, _I32, dev)
        _dense("cu_seqs", cu_seqs, _I32, dev, (n + 1,))
        self.cu_seqs, self.blocks, self.n_groups, self.device = cu_seqs, blocks, n, dev
        self.max_rows, self.max_blocks = int(max_rows), int(max_blocks)
        if min(self.max_rows, self.max_blocks) < 0 or max(self.max_rows, self.max_blocks) >= 1 << 31:
            _refuse("max_rows and max_blocks must be 0 .. 2^31 - 1")
        self.c = msi_kv_groups(n, self.max_rows, self.max_blocks, 0, cu_seqs.data_ptr(), blocks.data_ptr())
        self._ref = ctypes.byref(self.c)


def kv_attention_shared_workspace_size(cache: KvCache, seqs: KvSeqs, groups: KvGroups, n_q_heads: int) -> int:
    """Bytes of workspace of kv_attention_shared calls with these bounds."""
    n = ctypes.c_uint64()
    if n_q_heads < 0:
        _refuse("n_q_heads must not be negative")
    _check(lib.msi_kv_attention_shared_workspace(cache._ref, seqs._ref, groups._ref, n_q_heads, ctypes.byref(n)))
    return n.value


def kv_attention_shared_workspace(cache: KvCache, seqs: KvSeqs, groups: KvGroups, n_q_heads: int):
    """Workspace of kv_attention_shared calls with these bounds (a uint8 tensor)."""
    return torch.empty(kv_attention_shared_workspace_size(cache, seqs, groups, n_q_heads), dtype=torch.uint8,
                       device=cache.device)


def kv_attention_shared(cache: KvCache, seqs: KvSeqs, groups: KvGroups, q, out, scale: float, workspace=None, status=None,
                        stream=None, all_rows: bool = False):
    """kv_attention of sequences that share their first pages, each of which is read once for its group
    (msi_kv_attention_shared).  The workspace is kv_attention_shared_workspace's."""
    _same_device(cache, seqs)
    if groups.device != cache.device:
        _refuse("cache and groups must be on one device")
    ref, args = _attention(cache, seqs, q, out, scale, 0, 0.0, workspace, status, all_rows)
    _call(cache.device, lib.msi_kv_attention_shared, cache._ref, ref, groups._ref, args, _stream(stream, cache.device))


def kv_evict(cache: KvCache, seqs: KvSeqs, dst_table, new_lens, keep, *, budget: int, sinks: int = 0, recent: int = 0,
             status=None, stream=None):
    """Cut every sequence back to ``budget`` tokens a head into the pages of dst_table [n_seqs, blocks]
    (msi_kv_evict); new_lens [n_seqs] and keep [n_seqs, n_heads, budget] int32 receive what was kept."""
    _same_device(cache, seqs)
    dev, S = cache.device, seqs.n_seqs
    if min(budget, sinks, recent) < 0 or max(budget, sinks, recent) >= 1 << 31:
        _refuse("budget, sinks and recent must be 0 .. 2^31 - 1")
    if dst_table.dim() != 2 or dst_table.shape[0] != S:
        _refuse("dst_table must be [n_seqs, blocks]")
    _dense("dst_table", dst_table, _I32, dev)
    _dense("new_lens", new_lens, _I32, dev, (S,))
    _dense("keep", keep, _I32, dev, (S, cache.n_heads, budget))
    _call(dev, lib.msi_kv_evict, cache._ref, seqs._ref,
          _pack_evict.pack(budget, sinks, recent, dst_table.shape[1], dst_table.data_ptr(), new_lens.data_ptr(),
                           keep.data_ptr(), _status(status, dev)), _stream(stream, dev))


def _block_width(name: str, w) -> int:
    """K of a block's matrix: bf16, or a pair of 4-bit codes and scales."""
    if not isinstance(w, torch.Tensor) and not (isinstance(w, tuple) and len(w) == 2 and
                                                all(isinstance(t, torch.Tensor) for t in w)):
        _refuse(f"{name} must be a matrix or a pair (codes, scales)")
    m = w[0] if isinstance(w, tuple) else w
    K = 0 if m.dim() != 2 else m.shape[1] * (2 if isinstance(w, tuple) else 1)
    if K < 8 or K % 8:
        _refuse(f"{name} must be a matrix whose rows are a multiple of 8")
    return K


def _block_weights(name: str, w, N: int, K: int, dev):
    """What a projection would refuse of a block's matrix."""
    m = w
    if isinstance(w, tuple):
        if w[1].dim() != 2 or w[1].shape[1] < 1 or K % w[1].shape[1] or \
                K // w[1].shape[1] not in (32, 64, 128):
            _refuse(f"{name} must be a pair (codes, scales) with a scale for each 32, 64 or 128 of {K} weights")
        m, scales = w
        _dense(f"{name}'s codes", m, torch.uint8, dev, (N, K // 2))
        _dense(f"{name}'s scales", scales, scales.dtype if scales.dtype in _F16 else torch.float16, dev, (N, scales.shape[1]))
    else:
        _dense(name, m, m.dtype if m.dtype in _BF16 else torch.bfloat16, dev, (N, K))
    if m.data_ptr() % 16:
        _refuse(f"{name} must be 16-byte aligned")


def _block_linear(x, w, out, bias, stream):
    if isinstance(w, tuple):
        linear_q4(x, *w, out, bias=bias, stream=stream)
    else:
        linear(x, w, out, bias=bias, stream=stream)


class AttentionBlock:
    """The attention block of one stacked layer on fixed buffers: with the layer's normalised input x (bf16) and the
    residual stream h (fp32),

        q, k, v = x wqkv^T + bias;  rotate q, k;  append k, v;  a = attention(q);  h += a wo^T;  x = bf16(rmsnorm(h))

    wqkv [(n_q_heads + 2 n_kv_heads) head_dim, d] and wo [d, n_q_heads head_dim] bf16, or either a pair (codes, scales) of
    4-bit weights as ``linear_q4`` takes them; bias float32 or None.  With ``rotary`` (KvRotary) queries and keys turn by the
    ``positions`` of the step's rows on their way into the cache.  With ``groups`` (KvGroups) the step's sequences share their
    first pages.  ``step`` runs it whole; ``project`` and ``attend`` are its halves, for a model that normalises (or rotates
    in another way) queries and keys between them.  Holds the buffers for up to max_rows rows and, from ``reserve`` on, the
    attention's workspace, unless one is handed in.  Steps allocate nothing and can be captured; those of one block share its
    buffers, so they must not overlap.  Rows below n_rows that no sequence brings, and those of a sequence that breaks a
    bound or has more rows than tokens, get nothing added to h."""

    def __init__(self, wqkv, wo, cache: KvCache, n_q_heads: int, max_rows: int, bias=None, scale: Optional[float] = None,
                 rotary: Optional[KvRotary] = None):
        D, H, dev = cache.head_dim, cache.n_heads, cache.device
        if n_q_heads < 1 or n_q_heads % H:
            _refuse("n_q_heads must be a multiple of the cache's n_heads")
        self.rows_qkv, inner = (n_q_heads + 2 * H) * D, n_q_heads * D
        self.d = _block_width("wqkv", wqkv)
        _block_width("wo", wo)
        for name, w, N, K in (("wqkv", wqkv, self.rows_qkv, self.d), ("wo", wo, self.d, inner)):
            _block_weights(name, w, N, K, dev)
        if rotary is not None and (rotary.device != dev or rotary.rot_dim > D):
            _refuse(f"rotary must be on {dev} and rotate at most {D} elements")
        if bias is not None:
            _dense("bias", bias, _F32, dev, (self.rows_qkv,))
        if max_rows < 0:
            _refuse("max_rows must not be negative")
        self.wqkv, self.wo, self.bias, self.cache, self.n_q_heads = wqkv, wo, bias, cache, n_q_heads
        self.rotary = rotary
        self.scale = D ** -0.5 if scale is None else scale
        _scale(self.scale)
        self.qkv = torch.empty((max_rows, n_q_heads + 2 * H, D), dtype=torch.bfloat16, device=dev)
        self.attn = torch.empty((max_rows, n_q_heads, D), dtype=torch.bfloat16, device=dev)
        self.out = torch.empty((max_rows, self.d), dtype=_F32, device=dev)
        self._kept = []                   # every workspace so far: captured steps go on using theirs
        self.workspace = None
        self._settle()

    def _settle(self):
        """Memory the allocator hands out may have work of the current stream pending; steps may run on any."""
        if self.cache.device.type == "cuda":
            torch.cuda.current_stream(self.cache.device).synchronize()

    def _need(self, seqs: KvSeqs, mass_rows: int, groups: Optional[KvGroups]) -> int:
        """Bytes of workspace of a step."""
        if groups is None:
            return kv_attention_workspace_size(self.cache, seqs, self.n_q_heads, mass_rows)
        if mass_rows:
            _refuse("mass_rows must be 0 with groups: a shared page has several sequences' weights")
        return kv_attention_shared_workspace_size(self.cache, seqs, groups, self.n_q_heads)

    def reserve(self, seqs: KvSeqs, mass_rows: int = 0, groups: Optional[KvGroups] = None):
        """Workspace for steps with these bounds (of the largest ones asked for so far).  Captured steps go on using the one
        they were captured with, so earlier ones are kept; each is at least twice the one before."""
        need = self._need(seqs, mass_rows, groups)
        have = 0 if self.workspace is None else self.workspace.numel()
        if self.workspace is None or have < need:
            self.workspace = torch.empty(max(need, 2 * have), dtype=torch.uint8, device=self.cache.device)
            self._kept.append(self.workspace)
            self._settle()

    def _check_x(self, x, seqs: KvSeqs):
        if seqs.n_rows > self.qkv.shape[0]:
            _refuse(f"{seqs.n_rows} rows, buffers for {self.qkv.shape[0]}")
        _same_device(self.cache, seqs)
        _dense("x", x, x.dtype if x.dtype in _BF16 else torch.bfloat16, self.cache.device, (seqs.n_rows, self.d))

    def _check_rest(self, h, seqs: KvSeqs, mass_rows: int, mass_decay: float, status, workspace, positions, groups):
        """The workspace of a step whose other arguments are right."""
        dev = self.cache.device
        _dense("h", h, _F32, dev, (seqs.n_rows, self.d))
        _status(status, dev)
        if mass_rows:
            _decay(mass_decay)
        if self.rotary is not None:
            _positions(self.rotary, positions, seqs.n_rows, dev)
        elif positions is not None:
            _refuse("positions need a block with rotary")
        if groups is not None and groups.device != dev:
            _refuse("cache and groups must be on one device")
        need = self._need(seqs, mass_rows, groups)
        if workspace is None:
            workspace = self.workspace
        else:
            _dense("workspace", workspace, torch.uint8, dev)
            if workspace.data_ptr() % 16:
                _refuse("workspace must be 16-byte aligned")
        if need > (0 if workspace is None else workspace.numel()):
            raise MsiError(MSI_E_NOMEM, "reserve(seqs, mass_rows, groups) comes before a step, or a workspace of "
                                        f"{need} bytes is handed in")
        return workspace

    def _project(self, x, n: int, stream):
        qkv = self.qkv[:n]
        _block_linear(x, self.wqkv, qkv.view(n, self.rows_qkv), self.bias, stream)
        return qkv

    def _attend(self, x, h, seqs: KvSeqs, mass_rows: int, mass_decay: float, workspace, status, stream, positions, groups):
        n, Hq, H = seqs.n_rows, self.n_q_heads, self.cache.n_heads
        qkv, attn, out = self.qkv[:n], self.attn[:n], self.out[:n]
        q, k, v = qkv[:, :Hq], qkv[:, Hq:Hq + H], qkv[:, Hq + H:]
        if self.rotary is None:
            kv_append(self.cache, seqs, k, v, status=status, stream=stream)
        else:
            kv_append_rotary(self.cache, seqs, self.rotary, positions, q, q, k, v, status=status, stream=stream)
        if groups is None:
            kv_attention(self.cache, seqs, q, attn, self.scale, mass_rows=mass_rows, mass_decay=mass_decay,
                         workspace=workspace, status=status, stream=stream, all_rows=True)
        else:
            kv_attention_shared(self.cache, seqs, groups, q, attn, self.scale, workspace=workspace, status=status,
                                stream=stream, all_rows=True)
        _block_linear(attn.view(n, Hq * self.cache.head_dim), self.wo, out, None, stream)
        if n:
            _call(h.device, lib.msi_residual_add, out.data_ptr(), h.data_ptr(), x.data_ptr(), n, h.shape[1],
                  _stream(stream, h.device))

    def project(self, x, seqs: KvSeqs, stream=None):
        """First half: queries, keys and values of the rows x, [n_rows, n_q_heads + 2 n_kv_heads, head_dim] bf16 in the block's
        buffer, where the caller may change them (on ``stream``) before ``attend``."""
        self._check_x(x, seqs)
        return self._project(x, seqs.n_rows, stream)

    def attend(self, x, h, seqs: KvSeqs, mass_rows: int = 0, mass_decay: float = 1.0, status=None, stream=None, workspace=None,
               positions=None, groups: Optional[KvGroups] = None):
        """Second half, with what ``project`` left: rotates, appends, attends, and updates h and x as a step does."""
        self._check_x(x, seqs)
        workspace = self._check_rest(h, seqs, mass_rows, mass_decay, status, workspace, positions, groups)
        self._attend(x, h, seqs, mass_rows, mass_decay, workspace, status, stream, positions, groups)

    def step(self, x, h, seqs: KvSeqs, mass_rows: int = 0, mass_decay: float = 1.0, status=None, stream=None, workspace=None,
             positions=None, groups: Optional[KvGroups] = None):
        """x [n_rows, d] (bf16) and h [n_rows, d] (float32) of the call's rows, both updated in place.  What is refused is
        refused before the cache, x or h change.  ``workspace`` (uint8, kv_attention_workspace_size bytes, with groups
        kv_attention_shared_workspace_size) takes the place of the block's own: blocks whose steps run one after another can
        share one.  ``positions``: as kv_append_rotary's, of a block with rotary."""
        self._check_x(x, seqs)
        workspace = self._check_rest(h, seqs, mass_rows, mass_decay, status, workspace, positions, groups)
        self._project(x, seqs.n_rows, stream)
        self._attend(x, h, seqs, mass_rows, mass_decay, workspace, status, stream, positions, groups)
