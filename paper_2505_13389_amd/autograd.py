"""Video Sparse Attention as a differentiable PyTorch op (App. B: tile -> sparse attention -> untile).

Marshalling only: the token permutation, the forward and the backward all run in libvsa.so's
kernels; torch supplies device memory, the current stream and the autograd graph.  Tensors are in
the layout a video DiT holds them in, token-major raster order: bf16 [B, L, H, d] with
L = T*Hh*W and n = t*Hh*W + h*W + w (Sec. 2.1).

    out = video_sparse_attention(q, k, v, gate_c, gate_f, grid=(T, Hh, W), topk=K)

gate_f may be None (a fine gate of ones, Sec. 2.3).  No gradient flows through the top-K selection.
A model that keeps its activations in tiled order across layers (App. B caption) should call the
vsa_* entry points directly and skip the permutations.

    out = window_attention(q, k, v, left=6, right=0, sinks=1, unit=Hh * W)

is attention over a window of units (frames) and the first few, for models that generate a clip piece by piece: q [B, Lq, H, d],
k, v [B, Lk, Hkv, d] in bf16 or fp16 with any strides, or packed [rows, heads, d] with offsets cu_q, cu_k (int32 [B+1]).
"""
import torch
from torch.autograd.graph import get_gradient_edge

from . import vsa, window


class _VideoSparseAttention(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, gate_c, gate_f, grid, topk, cube, softmax_scale, flags):
        B, L, H, d = q.shape
        T, Hh, W = grid
        assert L == T * Hh * W, "q is [B, T*Hh*W, H, d]"
        pb = vsa.Problem(B, H, T, Hh, W, d, topk, tuple(cube), float(softmax_scale or 0.0), int(flags))
        Np, Nc = vsa.vsa_padded_tokens(pb)
        shape = (B, H, Np, d)
        bf = dict(dtype=torch.bfloat16, device=q.device)
        f32 = dict(dtype=torch.float32, device=q.device)

        raster = [x.contiguous() for x in (q, k, v, gate_c, gate_f) if x is not None]
        tiled = [torch.empty(shape, **bf) for _ in raster]
        vsa.vsa_tile_permute_many(pb, raster, tiled, inverse=False, blhd=True)
        tq, tk, tv, tgc, tgf = tiled if gate_f is not None else tiled + [None]
        # the attention writes raster tokens and, in the backward, reads and writes them: no permutation on that side
        pb = vsa.Problem(B, H, T, Hh, W, d, topk, tuple(cube), float(softmax_scale or 0.0),
                         int(flags) | vsa.VSA_FLAG_RASTER_IO)
        out = torch.empty_like(q, memory_format=torch.contiguous_format)
        rows = Nc // 4 if pb.flags & vsa.VSA_FLAG_SELECT_POOLED_2X2 else Nc
        idx = torch.empty((B, H, rows, pb.topk), dtype=torch.int32, device=q.device)
        out_fine, lse_fine = torch.empty(shape, **bf), torch.empty((B, H, Np), **f32)
        out_coarse, lse_coarse = torch.empty((B, H, Nc, d), **f32), torch.empty((B, H, Nc), **f32)
        workspace = torch.empty(vsa.vsa_workspace_bytes(pb, False), dtype=torch.uint8, device=q.device)
        vsa.vsa_forward(pb, tq, tk, tv, tgc, tgf, out, idx, out_fine, lse_fine, out_coarse, lse_coarse, workspace)
        ctx.pb, ctx.kept = pb, (idx, out_fine, lse_fine, out_coarse, lse_coarse)
        ctx.save_for_backward(tq, tk, tv, tgc, tgf)
        return out

    @staticmethod
    def backward(ctx, dout):
        pb = ctx.pb
        tq, tk, tv, tgc, tgf = ctx.saved_tensors
        idx, out_fine, lse_fine, out_coarse, lse_coarse = ctx.kept
        dout = dout.contiguous()
        dq, dk, dv, dgc = (torch.empty_like(dout) for _ in range(4))
        dgf = None if tgf is None else torch.empty_like(dout)
        workspace = torch.empty(vsa.vsa_workspace_bytes(pb, True), dtype=torch.uint8, device=dout.device)
        vsa.vsa_backward(pb, tq, tk, tv, tgc, tgf, dout, idx, out_fine, lse_fine, out_coarse, lse_coarse, dq, dk, dv, dgc,
                         dgf, workspace)
        return dq, dk, dv, dgc, dgf, None, None, None, None, None


def video_sparse_attention(q, k, v, gate_c, gate_f=None, *, grid, topk, cube=(4, 4, 4), softmax_scale=None, flags=0):
    """q, k, v, gate_c, gate_f (or None): bf16 [B, T*Hh*W, H, d] on the GPU; returns bf16 of the same shape."""
    return _VideoSparseAttention.apply(q, k, v, gate_c, gate_f, tuple(grid), int(topk), tuple(cube), softmax_scale, flags)


class _WindowAttention(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, cu_q, cu_k, pb):
        packed = cu_q is not None
        rows = q.shape[0] if packed else q.shape[0] * q.shape[1]
        out = torch.empty_like(q, memory_format=torch.contiguous_format)  # (rows of no sequence: written by nobody)
        if packed:
            out.zero_()
        lse = torch.empty((pb.H, rows), dtype=torch.float32, device=q.device)
        window.vsa_window_forward(pb, q, k, v, out, lse, cu_q, cu_k)
        ctx.pb = pb
        ctx.save_for_backward(q, k, v, out, lse, cu_q, cu_k)
        return out

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dout):
        q, k, v, out, lse, cu_q, cu_k = ctx.saved_tensors
        dout = _rows_of_16_bytes(dout)
        new = torch.empty if cu_q is None else torch.zeros
        dq, dk, dv = (new(x.shape, dtype=x.dtype, device=x.device) for x in (q, k, v))
        window.vsa_window_backward(ctx.pb, q, k, v, out, dout, lse, dq, dk, dv, None, cu_q, cu_k)
        return dq, dk, dv, None, None, None


def _refuse_held_leaves(*leaves):
    """A backward captured into a graph joins the stream on which the gradient node of a leaf was made, and an eager graph of that
    leaf that lives keeps the node of its own, uncaptured stream: the capture breaks, which ends the process.  So such a call is
    refused.  (A node that nobody holds is made anew, without the metadata written to it here.)  Returns the nodes, to be held
    until the call's own graph does."""
    nodes, stream = [], torch.cuda.current_stream().cuda_stream
    for x in leaves:
        if not (x.requires_grad and x.is_leaf and torch.is_grad_enabled()):
            continue
        get_gradient_edge(x).node.metadata["vsa_seen"] = True
        node = get_gradient_edge(x).node
        if "vsa_seen" in node.metadata and node.metadata.get("vsa_captured_on") != stream:
            del node, nodes  # (a traceback holds what this frame holds)
            raise RuntimeError("window_attention is captured into a graph while another autograd graph of one of its leaves lives: let "
                               "that graph go first (or pass a view, if it belongs to the same capture)")
        node.metadata["vsa_captured_on"] = stream
        nodes.append(node)
    return nodes


def _rows_of_16_bytes(x):
    """x itself where the kernels can read it in place, else a contiguous copy."""
    ok = x.stride(-1) == 1 and all(s % 8 == 0 for s in x.stride()[:-1]) and x.data_ptr() % 16 == 0 and x.stride(-3) <= 1 << 24
    return x if ok else x.contiguous()


def window_attention(q, k, v, *, left=-1, right=0, sinks=0, unit=1, softmax_scale=None, cu_q=None, cu_k=None, max_q=None, max_k=None):
    """softmax(scale q k^T over the visible keys) v.  Packed sequences: max_q and max_k bound their lengths (None: the rows of
    the tensor).  Returns a tensor of q's shape; packed, the rows of no sequence are zeros, and so are their gradients."""
    packed = cu_q is not None
    if q.dim() != (3 if packed else 4) or k.dim() != q.dim() or v.dim() != q.dim():
        raise ValueError("q, k, v are [B, L, heads, d], or [rows, heads, d] with cu_q and cu_k")
    held = _refuse_held_leaves(q, k, v) if q.is_cuda and torch.cuda.is_current_stream_capturing() else None  # noqa: F841 (kept to the end)
    q, k, v = (_rows_of_16_bytes(x) for x in (q, k, v))
    B = cu_q.numel() - 1 if packed else q.shape[0]
    longest = lambda most, x: x.shape[-3] if most is None else min(most, x.shape[-3]) if packed else x.shape[-3]
    pb = window.WindowProblem(B, q.shape[-2], k.shape[-2], q.shape[-1], longest(max_q, q), longest(max_k, k), left, right, sinks, unit,
                              float(softmax_scale or 0.0), q.dtype, q.shape[0] if packed else 0, k.shape[0] if packed else 0)
    return _WindowAttention.apply(q, k, v, cu_q, cu_k, pb)
