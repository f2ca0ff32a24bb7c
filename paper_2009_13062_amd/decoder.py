"""Binding of the decoders' operators: attention of prompts, of trees of drafted tokens over a cache, and the cache.

Argument marshalling only, as in the package's ``__init__``, which exports these functions.  Rows (Q, K, V) are [M, B*N, heads*d]
tensors whose last dimension is contiguous: dense, or column blocks of one packed projection (``qkv[..., :heads*d]``).  Caches,
lengths and every other operand are contiguous; integers are int32, slopes, weights and lse float32.  All operands live on the
current device.  With ``stream=`` a call runs there and takes its own memory there: that stream has to be behind whatever writes the
operands, and operands are to be kept, and results not read elsewhere, until it has passed the call.
"""
from __future__ import annotations

from typing import Optional, Tuple

import torch

import paper_2009_13062_amd as nf


def _current_device() -> int:
    return nf._device() if nf._device is not None else torch.cuda.current_device()


def _on_current(t: torch.Tensor) -> None:
    if not t.is_cuda:
        raise ValueError("netfuse operands must be CUDA tensors")
    if t.device.index != _current_device():
        raise ValueError("operand on %s, but the current device is cuda:%d" % (t.device, _current_device()))


def _dense(t: Optional[torch.Tensor], name: str, shape, dtype: torch.dtype):
    """Address of a contiguous operand of this shape and type; None stays None."""
    if t is None:
        return None
    if t.dtype != dtype:
        raise TypeError("%s must be %s, got %s" % (name, dtype, t.dtype))
    if tuple(t.shape) != tuple(shape):
        raise ValueError("%s must be %s, got %s" % (name, list(shape), list(t.shape)))
    if not t.is_contiguous():
        raise ValueError("%s must be contiguous" % name)
    _on_current(t)
    return t.data_ptr()


def _rows(t: torch.Tensor, name: str, M: int, N: int, width: int, dtype: torch.dtype) -> Tuple[int, int, int]:
    """Address, model stride and row stride of rows whose last dimension is contiguous."""
    if t.dtype != dtype:
        raise TypeError("%s must be %s, got %s" % (name, dtype, t.dtype))
    if tuple(t.shape) != (M, N, width):
        raise ValueError("%s must be %s, got %s" % (name, [M, N, width], list(t.shape)))
    if width > 1 and t.stride(2) != 1:
        raise ValueError("the last dimension of %s must be contiguous" % name)
    _on_current(t)
    row = t.stride(1) if N > 1 else width                    # the stride of a dimension of one element says nothing
    return t.data_ptr(), (t.stride(0) if M > 1 else (N - 1) * row + width), row


def _key_value_rows(K, V, M, N, width, dtype):
    k, km, kr = _rows(K, "K", M, N, width, dtype)
    v, vm, vr = _rows(V, "V", M, N, width, dtype)
    if (km, kr) != (vm, vr):
        raise ValueError("K and V must have the same strides")
    return k, v, km, kr


def _head_size(width: int, heads: int) -> int:
    if heads <= 0 or width <= 0 or width % heads:
        raise ValueError("%d features do not make %d heads" % (width, heads))
    return width // heads


def _cache_shape(Kc, Vc, dtype):
    if Kc.dim() != 5:
        raise ValueError("a cache is [M, B, kv_heads, C, d]")
    return tuple(Kc.shape), _dense(Kc, "Kc", Kc.shape, dtype), _dense(Vc, "Vc", Kc.shape, dtype)


def _own(stream, shape, dtype, device):
    """Memory of a call's own: from the pool of the stream that the call runs on.  A block of the current stream's pool may still be in use by work
    that is queued there, which nothing would hold the given stream back from."""
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    with torch.cuda.stream(stream):
        return torch.empty(shape, dtype=dtype, device=device)


def _output(stream, shape, dtype, device):
    """The same for a result, which the caller goes on to use on the current stream: freed, it is not handed out again before that stream has passed."""
    t = _own(stream, shape, dtype, device)
    if stream is not None:
        t.record_stream(torch.cuda.current_stream())
    return t


def attention_prompt(Q, K, V, B, S, heads, kv_heads=None, causal=True, scale=None, cap=0.0, slope=None, length=None, prefix=None, doc=None, out=None, stream=None):
    """Attention of prompts: Q[M, B*S, heads*d], K and V[M, B*S, kv_heads*d] -> [M, B*S, heads*d].

    Scores are cap*tanh(scale*qk/cap) (cap 0: scale*qk) minus slope[m, head] * distance.  Row i sees key j if both lie below length[m, b], and, where
    causal, j <= i or j < prefix[m, b], and, with doc[m, b, S], both belong to the same document >= 0.  Rows that see nothing are 0."""
    if nf._native is not None and stream is None and type(Q) is nf._Tensor and Q.is_cuda:
        device = nf._device()
        O = nf._native.attention_prompt(Q, K, V, B, S, heads, kv_heads, causal, scale, cap, slope, length, prefix, doc, out, device, nf._raw_stream(device))
        if O is not None:
            return O
    if Q.dim() != 3:
        raise ValueError("Q must be [M, B*S, heads*d]")
    kv_heads = heads if kv_heads is None else kv_heads
    M, d, dt = Q.shape[0], _head_size(Q.shape[2], heads), nf._dt(Q)
    q, qm, qr = _rows(Q, "Q", M, B * S, heads * d, Q.dtype)
    k, v, km, kr = _key_value_rows(K, V, M, B * S, kv_heads * d, Q.dtype)
    small = (_dense(slope, "slope", (M, heads), torch.float32), _dense(length, "length", (M, B), torch.int32), _dense(prefix, "prefix", (M, B), torch.int32),
             _dense(doc, "doc", (M, B, S), torch.int32))
    O = _output(stream, (M, B * S, heads * d), Q.dtype, Q.device) if out is None else out
    nf._check("netfuse_attention_prompt", nf.lib.netfuse_attention_prompt(
        q, k, v, *small, _dense(O, "out", (M, B * S, heads * d), Q.dtype), M, B, S, heads, kv_heads, d, qm, qr, km, kr, int(bool(causal)),
        float(d ** -0.5 if scale is None else scale), float(cap), dt, nf._stream(stream)))
    return O


def attention_tree_workspace(M, B, T, C, heads, kv_heads, d, dtype=torch.bfloat16) -> int:
    """Bytes of workspace of attention_tree (0: none needed)."""
    n = nf.lib.netfuse_attention_tree_workspace(M, B, T, C, heads, kv_heads, d, nf.NF_BF16 if dtype == torch.bfloat16 else nf.NF_F32)
    if n < 0:
        raise nf.NetFuseError("netfuse_attention_tree_workspace", nf.NF_EUNSUPPORTED)
    return n


def _workspace(workspace, need, device, stream):
    """The caller's workspace, or one of this call; its address and size."""
    if workspace is None:
        workspace = _own(stream, need, torch.uint8, device) if need else None
    else:
        _on_current(workspace)
        if not workspace.is_contiguous():
            raise ValueError("workspace must be contiguous")
    return workspace, (workspace.data_ptr() if workspace is not None else None), (workspace.numel() * workspace.element_size() if workspace is not None else 0)


def attention_tree(Q, K, V, Kc, Vc, length, start=None, parent=None, nodes=None, pos=None, slope=None, scale=None, cap=0.0, out=None, lse=None, workspace=None, stream=None):
    """Attention of T <= 64 drafted tokens per sequence over caches: Q[M, B*T, heads*d], K and V[M, B*T, kv_heads*d], Kc and Vc[M, B, kv_heads, C, d]
    -> [M, B*T, heads*d].

    Node t sees the length[m, b] entries of its cache, itself and its ancestors by parent[m, b, T] (None: a chain; T = 1: a single token); its position is
    start[m, b] (None: length) plus the number of its ancestors, an entry's is pos[m, b, kv_heads, C] (None: its slot).  nodes[m, b]: how many nodes there
    are; rows past it are 0.  lse: a float32 [M, B*T, heads] tensor that receives the logarithms of the sums, for cache_weigh.
    workspace: attention_tree_workspace(...) bytes, a call's own if None."""
    if nf._native is not None and stream is None and type(Q) is nf._Tensor and Q.is_cuda:
        device = nf._device()
        O = nf._native.attention_tree(Q, K, V, Kc, Vc, length, start, parent, nodes, pos, slope, scale, cap, out, lse, workspace, device, nf._raw_stream(device))
        if O is not None:
            return O
    (M, B, kv_heads, C, d), kc, vc = _cache_shape(Kc, Vc, Q.dtype)
    if Q.dim() != 3 or Q.shape[0] != M or Q.shape[1] % B or Q.shape[2] % d:
        raise ValueError("Q must be [M, B*T, heads*d]")
    T, heads, dt = Q.shape[1] // B, Q.shape[2] // d, nf._dt(Q)
    q, qm, qr = _rows(Q, "Q", M, B * T, heads * d, Q.dtype)
    k, v, km, kr = _key_value_rows(K, V, M, B * T, kv_heads * d, Q.dtype)
    if length is None:
        raise ValueError("length is required")
    small = (_dense(pos, "pos", (M, B, kv_heads, C), torch.int32), _dense(length, "length", (M, B), torch.int32), _dense(start, "start", (M, B), torch.int32),
             _dense(parent, "parent", (M, B, T), torch.int32), _dense(nodes, "nodes", (M, B), torch.int32), _dense(slope, "slope", (M, heads), torch.float32))
    z = _dense(lse, "lse", (M, B * T, heads), torch.float32)
    O = _output(stream, (M, B * T, heads * d), Q.dtype, Q.device) if out is None else out
    o = _dense(O, "out", (M, B * T, heads * d), Q.dtype)
    need = max(0, nf.lib.netfuse_attention_tree_workspace(M, B, T, C, heads, kv_heads, d, dt))
    ws, ws_ptr, ws_bytes = _workspace(workspace, need, Q.device, stream)
    nf._check("netfuse_attention_tree", nf.lib.netfuse_attention_tree(
        q, k, v, kc, vc, *small, o, z, ws_ptr, ws_bytes, M, B, T, C, heads, kv_heads, d, qm, qr, km, kr, float(d ** -0.5 if scale is None else scale), float(cap), dt, nf._stream(stream)))
    return O


def cache_append(K, V, Kc, Vc, pos, weight, length, start=None, index=None, count=None, stream=None):
    """Entry length + i of each cache takes row index[m, b, i] (None: row i) of K and V[M, B*T, kv_heads*d], position start + i and weight 0, for
    i < count[m, b] (None: all).  pos int32 and weight float32 [M, B, kv_heads, C], or None where they are not kept.  `length` stays as it is."""
    if nf._native is not None and stream is None and type(K) is nf._Tensor and K.is_cuda:
        device = nf._device()
        if nf._native.cache_append(K, V, Kc, Vc, pos, weight, length, start, index, count, device, nf._raw_stream(device)) is not None:
            return
    (M, B, kv_heads, C, d), kc, vc = _cache_shape(Kc, Vc, K.dtype)
    if K.dim() != 3 or K.shape[0] != M or K.shape[1] % B:
        raise ValueError("K must be [M, B*T, kv_heads*d]")
    T = K.shape[1] // B
    k, v, km, kr = _key_value_rows(K, V, M, B * T, kv_heads * d, K.dtype)
    n = T if index is None else index.shape[-1]
    if length is None:
        raise ValueError("length is required")
    nf._check("netfuse_cache_append", nf.lib.netfuse_cache_append(
        k, v, _dense(index, "index", (M, B, n), torch.int32), _dense(count, "count", (M, B), torch.int32), _dense(length, "length", (M, B), torch.int32),
        _dense(start, "start", (M, B), torch.int32), kc, vc, _dense(pos, "pos", (M, B, kv_heads, C), torch.int32), _dense(weight, "weight", (M, B, kv_heads, C), torch.float32),
        M, B, T, n, C, kv_heads, d, km, kr, nf._dt(K), nf._stream(stream)))


def cache_weigh(Q, lse, Kc, weight, length, start=None, index=None, count=None, pos=None, slope=None, scale=None, cap=0.0, out=None, stream=None):
    """weight[M, B, kv_heads, C] plus the attention weight that the appended tokens gave to each entry (length, start, index and count as they were for
    cache_append; Q and lse as of attention_tree, with its pos, slope, scale and cap).  out may be weight."""
    if nf._native is not None and stream is None and type(Q) is nf._Tensor and Q.is_cuda:
        device = nf._device()
        W = nf._native.cache_weigh(Q, lse, Kc, weight, length, start, index, count, pos, slope, scale, cap, out, device, nf._raw_stream(device))
        if W is not None:
            return W
    if Kc.dim() != 5:
        raise ValueError("a cache is [M, B, kv_heads, C, d]")
    M, B, kv_heads, C, d = Kc.shape
    if Q.dim() != 3 or Q.shape[0] != M or Q.shape[1] % B or Q.shape[2] % d:
        raise ValueError("Q must be [M, B*T, heads*d]")
    T, heads = Q.shape[1] // B, Q.shape[2] // d
    n = T if index is None else index.shape[-1]
    if lse is None or weight is None or length is None:
        raise ValueError("lse, weight and length are required")
    q, qm, qr = _rows(Q, "Q", M, B * T, heads * d, Q.dtype)
    small = (_dense(lse, "lse", (M, B * T, heads), torch.float32), _dense(index, "index", (M, B, n), torch.int32), _dense(count, "count", (M, B), torch.int32),
             _dense(Kc, "Kc", Kc.shape, Q.dtype), _dense(pos, "pos", (M, B, kv_heads, C), torch.int32), _dense(length, "length", (M, B), torch.int32),
             _dense(start, "start", (M, B), torch.int32), _dense(slope, "slope", (M, heads), torch.float32), _dense(weight, "weight", (M, B, kv_heads, C), torch.float32))
    W = _output(stream, (M, B, kv_heads, C), torch.float32, Q.device) if out is None else out
    nf._check("netfuse_cache_weigh", nf.lib.netfuse_cache_weigh(
        q, *small, _dense(W, "out", (M, B, kv_heads, C), torch.float32), M, B, T, n, C, heads, kv_heads, d, qm, qr, float(d ** -0.5 if scale is None else scale), float(cap),
        nf._dt(Q), nf._stream(stream)))
    return W


def cache_evict_workspace(M, B, C, kv_heads, budget) -> int:
    """Bytes of workspace of cache_evict."""
    n = nf.lib.netfuse_cache_evict_workspace(M, B, C, kv_heads, budget)
    if n < 0:
        raise nf.NetFuseError("netfuse_cache_evict_workspace", nf.NF_EINVAL)
    return n


def cache_evict(Kc, Vc, pos, weight, length, budget, start=None, recent=0, pos_out=None, weight_out=None, workspace=None, stream=None):
    """Cuts every cache that holds more than `budget` entries back to it: the entries of lowest weight leave (the lower slot among equals), those at positions
    start - recent and later last, and the free slots below budget take the entries that stay above it.  Keys and values move in place; position and
    weight too, or into pos_out and weight_out, which are returned.  `length` stays as it is: the caller takes length.clamp_(max=budget)."""
    pos_out, weight_out = (pos if pos_out is None else pos_out), (weight if weight_out is None else weight_out)
    if nf._native is not None and stream is None and workspace is None and type(Kc) is nf._Tensor and Kc.is_cuda:
        device = nf._device()
        if nf._native.cache_evict(Kc, Vc, pos, weight, length, budget, start, recent, pos_out, weight_out, device, nf._raw_stream(device)) is not None:
            return pos_out, weight_out
    if weight is None or length is None:
        raise ValueError("weight and length are required")
    (M, B, kv_heads, C, d), kc, vc = _cache_shape(Kc, Vc, Kc.dtype)
    shape = (M, B, kv_heads, C)
    small = (_dense(pos, "pos", shape, torch.int32), _dense(weight, "weight", shape, torch.float32), _dense(length, "length", (M, B), torch.int32),
             _dense(start, "start", (M, B), torch.int32), _dense(pos_out, "pos_out", shape, torch.int32), _dense(weight_out, "weight_out", shape, torch.float32))
    need = max(0, nf.lib.netfuse_cache_evict_workspace(M, B, C, kv_heads, budget))
    ws, ws_ptr, ws_bytes = _workspace(workspace, max(need, 4), Kc.device, stream)
    nf._check("netfuse_cache_evict", nf.lib.netfuse_cache_evict(
        kc, vc, *small, ws_ptr, ws_bytes, M, B, C, kv_heads, d, int(budget), int(recent), nf._dt(Kc), nf._stream(stream)))
    return pos_out, weight_out
