"""Windowed attention and its 8-bit cache: binding of vsa_window_* and vsa_cache_* (include/vsa.h has the contract).

Argument marshalling only, as in `vsa.py`: shapes, types, strides and devices are checked here, everything else happens in
libvsa.so's kernels.  Calls run on the current stream of the tensors' device; scratch comes from torch's allocator, call by
call, unless a workspace is handed over.

    pb = WindowProblem(B=1, H=12, Hkv=12, d=128, max_q=32760, max_k=32760, left=6, right=0, sinks=1, unit=1560)
    buf = WindowBuffers(pb)                       # outputs, log-sum-exps, gradients, workspace
    buf.forward(q, k, v)                          # buf.out; q [B, max_q, H, d], k, v [B, max_k, Hkv, d]
    buf.backward(q, k, v, dout)                   # buf.dq, buf.dk, buf.dv

    cache = PagedCache(pages, Hkv=12, d=128)
    cache.append(k_new, v_new, table, lens)       # lens: tokens there before
    out = cache.attend(q, table, lens_now, left=6, right=0, sinks=1, unit=1560)
"""
import ctypes as C
from dataclasses import dataclass

import torch

from .vsa import VsaError, lib

PAGE = 64
# the current stream's handle, without the object around it where torch offers that
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda index: torch.cuda.current_stream(index).cuda_stream)
_DTYPES = {torch.bfloat16: 0, torch.float16: 1}


class VsaStrides(C.Structure):
    _fields_ = [("batch", C.c_int64), ("token", C.c_int64), ("head", C.c_int64)]


class VsaWindow(C.Structure):
    _fields_ = [("B", C.c_int32), ("H", C.c_int32), ("Hkv", C.c_int32), ("d", C.c_int32), ("max_q", C.c_int32), ("max_k", C.c_int32),
                ("total_q", C.c_int64), ("total_k", C.c_int64), ("unit", C.c_int32), ("left", C.c_int32), ("right", C.c_int32),
                ("sinks", C.c_int32), ("softmax_scale", C.c_float), ("dtype", C.c_int32)] + [
                    (n, VsaStrides) for n in ("q", "k", "v", "out", "dout", "dq", "dk", "dv")]


class VsaCache(C.Structure):
    _fields_ = [("B", C.c_int32), ("H", C.c_int32), ("Hkv", C.c_int32), ("d", C.c_int32), ("max_q", C.c_int32), ("total_q", C.c_int64),
                ("pages", C.c_int32), ("max_pages", C.c_int32), ("unit", C.c_int32), ("left", C.c_int32), ("right", C.c_int32),
                ("sinks", C.c_int32), ("softmax_scale", C.c_float), ("dtype", C.c_int32)] + [
                    (n, VsaStrides) for n in ("q", "out", "k", "v")]


@dataclass
class WindowProblem:
    """Shape and mask of one call; mirrors vsa_window_t.  Packed tensors: total_q, total_k rows in all, max_q and max_k the
    longest sequences (or more)."""
    B: int
    H: int
    Hkv: int
    d: int
    max_q: int
    max_k: int
    left: int = -1
    right: int = 0
    sinks: int = 0
    unit: int = 1
    softmax_scale: float = 0.0
    dtype: torch.dtype = torch.bfloat16
    total_q: int = 0
    total_k: int = 0

    def params(self):
        if self.dtype not in _DTYPES:
            raise ValueError(f"dtype is bfloat16 or float16, not {self.dtype}")
        return VsaWindow(self.B, self.H, self.Hkv, self.d, self.max_q, self.max_k, self.total_q, self.total_k, self.unit, self.left,
                         self.right, self.sinks, self.softmax_scale, _DTYPES[self.dtype])


def _strides(t, name):
    if t.shape[-1] > 1 and t.stride(-1) != 1:
        raise ValueError(f"{name}: the elements of a row must be contiguous")
    s = [step if n > 1 else 0 for n, step in zip(t.shape, t.stride())]  # (of a dimension with one entry it may be anything)
    return VsaStrides(s[0] if t.dim() == 4 else 0, s[-3], s[-2])


def _want(t, name, shape, dtype, device):
    if not isinstance(t, torch.Tensor) or tuple(t.shape) != tuple(shape) or t.dtype != dtype or t.device != device:
        have = f"{t.dtype} {tuple(t.shape)} on {t.device}" if isinstance(t, torch.Tensor) else type(t).__name__
        raise ValueError(f"{name} must be {dtype} {tuple(shape)} on {device}, not {have}")
    return t


def _whole(t, name, shape, dtype, device):
    if not _want(t, name, shape, dtype, device).is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return t


def _shapes(pb, packed):
    if packed:
        return (pb.total_q, pb.H, pb.d), (pb.total_k, pb.Hkv, pb.d)
    return (pb.B, pb.max_q, pb.H, pb.d), (pb.B, pb.max_k, pb.Hkv, pb.d)


def _run(device, name, *args):
    """The entry point `name` on the device's current stream."""
    index = device.index
    if index is None:
        raise ValueError(f"tensors must be on a GPU, not on {device}")
    f = getattr(lib(), name)
    if index == torch.cuda.current_device():
        rc = f(*args, _raw_stream(index))
    else:
        with torch.cuda.device(index):
            rc = f(*args, _raw_stream(index))
    if rc:
        raise VsaError(name, rc)


_known = {}  # parameters of calls by their shapes, strides, types and mask: building them takes longer than a launch
_NAMES = ("q", "k", "v", "out", "dout", "dq", "dk", "dv")


def _window_call(pb, tensors, lse, cu_q, cu_k):
    """Address of the parameters of a call, its tensors checked: q, k, v, out and, backward, dout, dq, dk, dv."""
    q = tensors[0]
    device = q.device
    if (cu_q is None) != (cu_k is None):
        raise ValueError("cu_q and cu_k: both or neither")
    packed = cu_q is not None
    key = (*pb.__dict__.values(), packed, *[x for t in tensors for x in (t.shape, t.stride())])
    known = _known.get(key)
    if known is None:
        sq, sk = _shapes(pb, packed)
        p = pb.params()
        for n, t in zip(_NAMES, tensors):
            setattr(p, n, _strides(_want(t, n, sk if n in ("k", "v", "dk", "dv") else sq, pb.dtype, device), n))
        if len(_known) >= 1024:
            _known.clear()
        known = _known[key] = (p, C.addressof(p), (pb.H, sq[0] if packed else sq[0] * sq[1]), *(int(lib().vsa_window_workspace_bytes(C.byref(p), backward)) for backward in (0, 1)))
    for n, t in zip(_NAMES, tensors):
        if t.dtype is not pb.dtype or t.device != device:
            raise ValueError(f"{n} must be {pb.dtype} on {device}, not {t.dtype} on {t.device}")
    if packed:
        _whole(cu_q, "cu_q", (pb.B + 1,), torch.int32, device)
        _whole(cu_k, "cu_k", (pb.B + 1,), torch.int32, device)
    if lse is not None:
        _whole(lse, "lse", known[2], torch.float32, device)
    return known


def _at(t):
    return None if t is None else t.data_ptr()


def vsa_window_workspace_bytes(pb: WindowProblem, backward: bool) -> int:
    return int(lib().vsa_window_workspace_bytes(C.byref(pb.params()), int(backward)))


def _bytes(t):
    return 0 if t is None else t.numel() * t.element_size()


def _workspace(t, need, device):
    """The one given, or a new one."""
    if t is None:
        return torch.empty(need, dtype=torch.uint8, device=device)
    if t.device != device or not t.is_contiguous():
        raise ValueError("the workspace must be contiguous and on the tensors' device")
    return t


def vsa_window_forward(pb: WindowProblem, q, k, v, out, lse=None, cu_q=None, cu_k=None, workspace=None):
    """out, lse (or None: not wanted) are written; lse is fp32 [H, rows].  Without a workspace one is allocated."""
    call = _window_call(pb, (q, k, v, out), lse, cu_q, cu_k)
    workspace = _workspace(workspace, call[3], q.device)
    _run(q.device, "vsa_window_forward", call[1], q.data_ptr(), k.data_ptr(), v.data_ptr(), _at(cu_q), _at(cu_k), out.data_ptr(), _at(lse),
         workspace.data_ptr(), _bytes(workspace))


def vsa_window_backward(pb: WindowProblem, q, k, v, out, dout, lse, dq, dk, dv, workspace=None, cu_q=None, cu_k=None):
    """dq, dk, dv are written; out, lse as the forward wrote them.  Without a workspace one is allocated."""
    call = _window_call(pb, (q, k, v, out, dout, dq, dk, dv), lse, cu_q, cu_k)
    workspace = _workspace(workspace, call[4], q.device)
    _run(q.device, "vsa_window_backward", call[1], q.data_ptr(), k.data_ptr(), v.data_ptr(), _at(cu_q), _at(cu_k), out.data_ptr(),
         dout.data_ptr(), lse.data_ptr(), dq.data_ptr(), dk.data_ptr(), dv.data_ptr(), workspace.data_ptr(),
         _bytes(workspace))


class WindowBuffers:
    """Convenience holder: allocates every output, saved tensor and the workspace of a WindowProblem once.  packed: by default
    where the problem gives total rows; to be said where packed tensors have none at all."""

    def __init__(self, pb: WindowProblem, device="cuda", backward=True, packed=None):
        self.pb = pb
        need = max(vsa_window_workspace_bytes(pb, False), vsa_window_workspace_bytes(pb, True) if backward else 0)
        if need == 0:
            raise ValueError(f"not a problem the library takes: {pb}")
        device = torch.empty(0, device=device).device
        packed = pb.total_q > 0 or pb.total_k > 0 if packed is None else packed
        sq, sk = _shapes(pb, packed)
        new = lambda s: torch.empty(s, dtype=pb.dtype, device=device)
        self.out = new(sq)
        self.lse = torch.empty((pb.H, sq[0] if packed else sq[0] * sq[1]), dtype=torch.float32, device=device)
        if backward:
            self.dq, self.dk, self.dv = new(sq), new(sk), new(sk)
        self.workspace = torch.empty(need, dtype=torch.uint8, device=device)

    def forward(self, q, k, v, cu_q=None, cu_k=None):
        vsa_window_forward(self.pb, q, k, v, self.out, self.lse, cu_q, cu_k, self.workspace)

    def backward(self, q, k, v, dout, cu_q=None, cu_k=None):
        """Behind forward() on the same inputs."""
        vsa_window_backward(self.pb, q, k, v, self.out, dout, self.lse, self.dq, self.dk, self.dv, self.workspace, cu_q, cu_k)


def vsa_cache_workspace_bytes(p: VsaCache) -> int:
    return int(lib().vsa_cache_workspace_bytes(C.byref(p)))


class PagedCache:
    """Keys and values of many sequences in pages of 64 tokens, e4m3 with a scale per page and head.

    k [pages, Hkv, 64, d] and v [pages, Hkv, d, 64] (torch.float8_e4m3fn), k_scale and v_scale [pages, Hkv] (fp32).  Which page
    belongs to whom is the caller's: `table` (int32 [B, max_pages]) names the pages of a sequence in order."""

    def __init__(self, pages: int, Hkv: int, d: int, device="cuda"):
        self._own(torch.zeros((pages, Hkv, PAGE, d), dtype=torch.float8_e4m3fn, device=device),
                  torch.zeros((pages, Hkv, d, PAGE), dtype=torch.float8_e4m3fn, device=device),
                  torch.ones((pages, Hkv), device=device), torch.ones((pages, Hkv), device=device))

    @classmethod
    def of(cls, k, v, k_scale, v_scale):
        """A cache over tensors that are there."""
        self = cls.__new__(cls)
        self._own(k, v, k_scale, v_scale)
        return self

    def _own(self, k, v, k_scale, v_scale):
        pages, heads, _, d = k.shape
        _whole(k, "k", (pages, heads, PAGE, d), torch.float8_e4m3fn, k.device)
        _whole(v, "v", (pages, heads, d, PAGE), torch.float8_e4m3fn, k.device)
        _whole(k_scale, "k_scale", (pages, heads), torch.float32, k.device)
        _whole(v_scale, "v_scale", (pages, heads), torch.float32, k.device)
        self.k, self.v, self.k_scale, self.v_scale = k, v, k_scale, v_scale
        self.pages, self.Hkv, self.d, self.device = pages, heads, d, k.device
        self._pool = (k.data_ptr(), v.data_ptr(), k_scale.data_ptr(), v_scale.data_ptr())
        self._params = {}  # of calls by their shapes, strides, types and mask: building them takes longer than the launch

    def _call(self, x, table, lens, cu, most, name):
        """The parameters of a call whose tokens are x: [B, n, heads, d], or packed [rows, heads, d] with offsets `cu`."""
        if x.dtype not in _DTYPES:
            raise ValueError(f"{name} is bfloat16 or float16, not {x.dtype}")
        if x.dim() != (4 if cu is None else 3) or x.shape[-1] != self.d:
            raise ValueError(f"{name} is [B, n, heads, {self.d}], or [rows, heads, {self.d}] with offsets, not {tuple(x.shape)}")
        B = table.shape[0] if table.dim() == 2 else -1
        if B < 1:
            raise ValueError("table is int32 [B, max_pages]")
        if tuple(lens.shape) != (B,):
            raise ValueError(f"lens is int32 [{B}], not {tuple(lens.shape)}")
        if cu is None:
            if x.shape[0] != B:
                raise ValueError(f"{name} has {x.shape[0]} sequences, table has {B}")
            most, rows = x.shape[1], 0
        else:
            if tuple(cu.shape) != (B + 1,):
                raise ValueError(f"cu is int32 [{B + 1}], not {tuple(cu.shape)}")
            rows = x.shape[0]
            most = rows if most is None else min(most, rows)
        if len(self._params) >= 256:
            self._params.clear()
        return VsaCache(B=B, H=x.shape[-2], Hkv=self.Hkv, d=self.d, max_q=most, total_q=rows, pages=self.pages, max_pages=table.shape[1],
                        unit=1, left=-1, right=0, dtype=_DTYPES[x.dtype])

    def _check(self, tokens, table, lens, cu):
        """What a call's tensors have to be besides their shapes and strides."""
        here = self.device
        for t in tokens:
            if t.device != here:
                raise ValueError(f"tensors must be on the cache's device, {here}, not on {t.device}")
        for t in (table, lens) if cu is None else (table, lens, cu):
            if t.dtype is not torch.int32 or not t.is_contiguous() or t.device != here:
                raise ValueError(f"table, lens and cu are contiguous int32 tensors on {here}, not {t.dtype} on {t.device}")

    def append(self, k, v, table, lens, cu=None, max_new=None):
        """New tokens k, v behind the `lens` (int32 [B]) tokens that each sequence has: [B, n, Hkv, d], or packed
        [rows, Hkv, d] with offsets `cu` (int32 [B+1]) and at most `max_new` tokens a sequence (None: as many as there are rows)."""
        packed = cu is not None
        key = (k.shape, k.stride(), v.shape, v.stride(), k.dtype, v.dtype, table.shape, lens.shape, packed and cu.shape, max_new)
        known = self._params.get(key)
        if known is None:
            p = self._call(k, table, lens, cu, max_new, "k")
            if k.shape[-2] != self.Hkv:
                raise ValueError(f"k has {k.shape[-2]} heads, the cache has {self.Hkv}")
            _want(v, "v", k.shape, k.dtype, v.device)
            p.k, p.v = _strides(k, "k"), _strides(v, "v")
            known = self._params[key] = (p, C.addressof(p))
        self._check((k, v), table, lens, cu)
        _run(self.device, "vsa_cache_append", known[1], k.data_ptr(), v.data_ptr(), cu.data_ptr() if packed else None, lens.data_ptr(), table.data_ptr(),
                  *self._pool)

    def attend(self, q, table, lens, cu=None, max_q=None, *, left=-1, right=0, sinks=0, unit=1, softmax_scale=0.0, out=None, lse=None,
               workspace=None):
        """Attention of q over the first `lens` tokens of each sequence, of which the queries are the last: q [B, n, H, d], or packed
        [rows, H, d] with offsets `cu` and at most `max_q` queries a sequence (None: as many as there are rows; where all have
        few, saying so is faster).  Returns out (a new tensor, or the one given); rows
        that belong to no sequence are not written."""
        packed = cu is not None
        if out is None:
            out = torch.empty_like(q, memory_format=torch.contiguous_format)
        elif out.shape != q.shape or out.dtype != q.dtype:
            raise ValueError(f"out must be {q.dtype} {tuple(q.shape)}, not {out.dtype} {tuple(out.shape)}")
        key = (q.shape, q.stride(), out.stride(), q.dtype, table.shape, lens.shape, packed and cu.shape, max_q, left, right, sinks, unit,
               softmax_scale)
        known = self._params.get(key)
        if known is None:
            p = self._call(q, table, lens, cu, max_q, "q")
            p.unit, p.left, p.right, p.sinks, p.softmax_scale = unit, left, right, sinks, softmax_scale
            p.q, p.out = _strides(q, "q"), _strides(out, "out")
            known = self._params[key] = (p, C.addressof(p), vsa_cache_workspace_bytes(p))
        self._check((q, out), table, lens, cu)
        if lse is not None:
            _whole(lse, "lse", (q.shape[-2], q.shape[0] if packed else q.shape[0] * q.shape[1]), torch.float32, self.device)
        workspace = _workspace(workspace, known[2], self.device)
        _run(self.device, "vsa_cache_attention", known[1], q.data_ptr(), cu.data_ptr() if packed else None, lens.data_ptr(), table.data_ptr(), *self._pool,
                  out.data_ptr(), None if lse is None else lse.data_ptr(), workspace.data_ptr(), _bytes(workspace))
        return out

    def workspace_bytes(self, B, H, max_q, max_pages):
        """Scratch that attend() needs for calls of at most this size; 0 if there is none such."""
        return vsa_cache_workspace_bytes(VsaCache(B=B, H=H, Hkv=self.Hkv, d=self.d, max_q=max_q, total_q=0, pages=self.pages,
                                                  max_pages=max_pages, unit=1, left=-1, right=0))


def vsa_host_window_walk(pb: WindowProblem, nq: int, nk: int):
    """Host-only: replays how blocks walk a sequence of nq queries and nk keys; returns the number of wrong pairs."""
    wrong = C.c_int64(-1)
    rc = lib().vsa_host_window_walk(C.byref(pb.params()), nq, nk, C.byref(wrong))
    if rc and wrong.value < 0:
        raise VsaError("vsa_host_window_walk", rc)
    return wrong.value
