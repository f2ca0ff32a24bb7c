"""Binding of what surrounds the decoders' attention in a step: heads normed and rotated, a cache of 4 bits and attention over it, log probabilities of tokens.

Argument marshalling only, with the conventions of ``decoder.py``: rows are [M, B*N, heads*d] tensors whose last dimension is contiguous, everything else is
contiguous, integers are int32, weights and results of statistics float32; all operands live on the current device.  A cache of 4 bits is two uint8 tensors, codes
[M, B, kv_heads, C, 16*G] and scales [M, B, kv_heads, C, G or G + 1], G groups of 32 features (layout of include/netfuse.h; ``cache_fp4`` makes one).
"""
from __future__ import annotations

import ctypes
from typing import Optional, Tuple

import torch

import paper_2009_13062_amd as nf
from .decoder import _dense, _head_size, _key_value_rows, _output, _rows, _workspace


def _rows_out(out: Optional[torch.Tensor], name, M, N, width, dtype, device, stream, whole):
    """The given rows or new ones (0 where not all of them are written), their address and strides."""
    if out is None:
        out = _output(stream, (M, N, width), dtype, device)
        if not whole:
            if stream is None:
                out.zero_()
            else:
                with torch.cuda.stream(stream):
                    out.zero_()
    return (out,) + _rows(out, name, M, N, width, dtype)


def rotate_heads(Q, K, B, S, heads, kv_heads=None, freq=None, gamma_q=None, gamma_k=None, pos=None, start=None, length=None, sections=None, interleaved=False, eps=1e-6, out_q=None, out_k=None,
                 stream=None):
    """Queries and keys of Q[M, B*S, heads*d] and K[M, B*S, kv_heads*d] (K may be None) normed head by head where a weight gamma[M, d] is given,
    x / sqrt(mean(x^2) + eps) * gamma, then rotated: pair i of the first 2*len(freq) features -- (i, i + len(freq)), or (2i, 2i + 1) where interleaved -- by
    position * freq[i].  -> (rotated Q, rotated K); out_q may be Q, out_k may be K.

    Positions are pos[M, B, S], or start[m, b] + s (None: s), or pos[M, B, S, axes] with sections = the number of pairs of each axis, in order.  Rows at and past
    length[m, b] are left as they are in out_q and out_k (0 in new ones)."""
    if nf._native is not None and stream is None and type(Q) is nf._Tensor and Q.is_cuda:
        device = nf._device()
        done = nf._native.rotate_heads(Q, K, B, S, heads, kv_heads, freq, gamma_q, gamma_k, pos, start, length, sections, interleaved, eps, out_q, out_k, device, nf._raw_stream(device))
        if done is not None:
            return done
    if Q.dim() != 3:
        raise ValueError("Q must be [M, B*S, heads*d]")
    kv_heads = 0 if K is None else heads if kv_heads is None else kv_heads
    M, d, dt = Q.shape[0], _head_size(Q.shape[2], heads), nf._dt(Q)
    if K is None and out_k is not None:
        raise ValueError("out_k without K")
    if K is not None and kv_heads <= 0:
        raise ValueError("K has kv_heads heads, one at least")
    q, qm, qr = _rows(Q, "Q", M, B * S, heads * d, Q.dtype)
    k, km, kr = (None, 0, 0) if K is None else _rows(K, "K", M, B * S, kv_heads * d, Q.dtype)
    pairs = 0 if freq is None else freq.numel()
    axes, parts = 1, None
    if sections is not None:
        sections = [int(x) for x in sections]
        axes = len(sections)
        if axes == 0:
            raise ValueError("sections names at least one axis")
        parts = (ctypes.c_int * axes)(*sections)
    if axes > 1 and pos is None:
        raise ValueError("several axes need pos")
    shape = (M, B, S) if pos is None or pos.dim() == 3 and axes == 1 else (M, B, S, axes)
    small = (_dense(gamma_q, "gamma_q", (M, d), torch.float32), _dense(gamma_k, "gamma_k", (M, d), torch.float32), _dense(freq, "freq", (pairs,), torch.float32),
             _dense(pos, "pos", shape, torch.int32), _dense(start, "start", (M, B), torch.int32), _dense(length, "length", (M, B), torch.int32))
    Qo, qo, qom, qor = _rows_out(out_q, "out_q", M, B * S, heads * d, Q.dtype, Q.device, stream, length is None)
    Ko, ko, kom, kor = (None, None, 0, 0) if K is None else _rows_out(out_k, "out_k", M, B * S, kv_heads * d, Q.dtype, Q.device, stream, length is None)
    nf._check("netfuse_rotate_heads", nf.lib.netfuse_rotate_heads(
        q, k, *small, parts, qo, ko, M, B, S, heads, kv_heads, d, 2 * pairs, axes, qm, qr, km, kr, qom, qor, kom, kor, float(eps), int(bool(interleaved)), dt, nf._stream(stream)))
    return Qo, Ko


def _groups(d: int) -> Tuple[int, int]:
    """Bytes of a row's codes and of its scales."""
    G = (d + 31) // 32
    return 16 * G, G + G % 2


def cache_fp4(M, B, kv_heads, C, d, device="cuda"):
    """An empty cache of 4 bits for heads of d features: (Kc, Ks, Vc, Vs)."""
    codes, scales = _groups(d)
    new = lambda n: torch.zeros((M, B, kv_heads, C, n), dtype=torch.uint8, device=device)  # noqa: E731
    return new(codes), new(scales), new(codes), new(scales)


def _fp4_shape(Kc, Ks, Vc, Vs, d):
    if Kc.dim() != 5:
        raise ValueError("a cache of 4 bits is codes [M, B, kv_heads, C, 16*G] and scales [M, B, kv_heads, C, G or G + 1]")
    M, B, kv_heads, C = Kc.shape[:4]
    codes, scales = _groups(d)
    u8 = torch.uint8
    return (M, B, kv_heads, C), (_dense(Kc, "Kc", (M, B, kv_heads, C, codes), u8), _dense(Ks, "Ks", (M, B, kv_heads, C, scales), u8),
                                 _dense(Vc, "Vc", (M, B, kv_heads, C, codes), u8), _dense(Vs, "Vs", (M, B, kv_heads, C, scales), u8))


def cache_append_fp4(K, V, Kc, Ks, Vc, Vs, pos, weight, length, start=None, index=None, count=None, stream=None):
    """cache_append into a cache of 4 bits: rows of K and V[M, B*T, kv_heads*d] are quantised as they are written (include/netfuse.h says how)."""
    if nf._native is not None and stream is None and type(K) is nf._Tensor and K.is_cuda:
        device = nf._device()
        if nf._native.cache_append_fp4(K, V, Kc, Ks, Vc, Vs, pos, weight, length, start, index, count, device, nf._raw_stream(device)) is not None:
            return
    if Kc.dim() != 5 or K.dim() != 3:
        raise ValueError("K must be [M, B*T, kv_heads*d] and Kc [M, B, kv_heads, C, 16*G]")
    d = _head_size(K.shape[2], Kc.shape[2])
    (M, B, kv_heads, C), held = _fp4_shape(Kc, Ks, Vc, Vs, d)
    if K.shape[0] != M or K.shape[1] % B:
        raise ValueError("K must be [M, B*T, kv_heads*d]")
    T = K.shape[1] // B
    k, v, km, kr = _key_value_rows(K, V, M, B * T, kv_heads * d, K.dtype)
    n = T if index is None else index.shape[-1]
    if length is None or any(x is None for x in held):
        raise ValueError("length and the four parts of the cache are required")
    nf._check("netfuse_cache_append_fp4", nf.lib.netfuse_cache_append_fp4(
        k, v, _dense(index, "index", (M, B, n), torch.int32), _dense(count, "count", (M, B), torch.int32), _dense(length, "length", (M, B), torch.int32),
        _dense(start, "start", (M, B), torch.int32), *held, _dense(pos, "pos", (M, B, kv_heads, C), torch.int32), _dense(weight, "weight", (M, B, kv_heads, C), torch.float32),
        M, B, T, n, C, kv_heads, d, km, kr, nf._dt(K), nf._stream(stream)))


def cache_read_fp4(Kc, Ks, Vc, Vs, d, n=None, first=None, count=None, dtype=torch.bfloat16, out_k=None, out_v=None, stream=None):
    """Entries first[m, b] + i (None: i), i < n (None: C), of a cache of 4 bits as K, V[M, B, kv_heads, n, d] (bfloat16 or float32, exact in either but for bfloat16's range);
    those at and past count[m, b], and past the cache, are 0.  Vc and Vs may be None together: keys alone, V is None then."""
    if nf._native is not None and stream is None and type(Kc) is nf._Tensor and Kc.is_cuda and out_k is not None:
        device = nf._device()
        if nf._native.cache_read_fp4(Kc, Ks, Vc, Vs, d, n, first, count, out_k, out_v, device, nf._raw_stream(device)) is not None:
            return out_k, out_v
    (M, B, kv_heads, C), held = _fp4_shape(Kc, Ks, Vc, Vs, d)
    if Ks is None or (Vc is None) != (Vs is None) or (Vc is None and out_v is not None):
        raise ValueError("keys, or keys and values: codes and scales of each")
    n = C if n is None else n
    dtype = dtype if out_k is None else out_k.dtype
    shape = (M, B, kv_heads, n, d)
    K = _output(stream, shape, dtype, Kc.device) if out_k is None else out_k
    V = None if Vc is None else _output(stream, shape, dtype, Kc.device) if out_v is None else out_v
    nf._check("netfuse_cache_read_fp4", nf.lib.netfuse_cache_read_fp4(
        *held, _dense(first, "first", (M, B), torch.int32), _dense(count, "count", (M, B), torch.int32), _dense(K, "out_k", shape, dtype), _dense(V, "out_v", shape, dtype), M, B, n, C, kv_heads, d,
        nf._dt(K), nf._stream(stream)))
    return K, V


def attention_tree_fp4_workspace(M, B, T, C, heads, kv_heads, d, dtype=torch.bfloat16) -> int:
    """Bytes of workspace of attention_tree_fp4 (0: none needed)."""
    n = nf.lib.netfuse_attention_tree_fp4_workspace(M, B, T, C, heads, kv_heads, d, nf.NF_BF16 if dtype == torch.bfloat16 else nf.NF_F32)
    if n < 0:
        raise nf.NetFuseError("netfuse_attention_tree_fp4_workspace", nf.NF_EUNSUPPORTED)
    return n


def attention_tree_fp4(Q, K, V, Kc, Ks, Vc, Vs, length, start=None, parent=None, nodes=None, pos=None, slope=None, scale=None, cap=0.0, out=None, lse=None, workspace=None, stream=None):
    """attention_tree over a cache of 4 bits: Q[M, B*T, heads*d], the new tokens' K and V[M, B*T, kv_heads*d] -> [M, B*T, heads*d]."""
    if nf._native is not None and stream is None and type(Q) is nf._Tensor and Q.is_cuda:
        device = nf._device()
        O = nf._native.attention_tree_fp4(Q, K, V, Kc, Ks, Vc, Vs, length, start, parent, nodes, pos, slope, scale, cap, out, lse, workspace, device, nf._raw_stream(device))
        if O is not None:
            return O
    if Kc.dim() != 5 or Q.dim() != 3 or K.dim() != 3:
        raise ValueError("Q must be [M, B*T, heads*d], K [M, B*T, kv_heads*d] and Kc [M, B, kv_heads, C, 16*G]")
    d = _head_size(K.shape[2], Kc.shape[2])
    (M, B, kv_heads, C), held = _fp4_shape(Kc, Ks, Vc, Vs, d)
    if Q.shape[0] != M or Q.shape[1] % B or Q.shape[2] % d:
        raise ValueError("Q must be [M, B*T, heads*d]")
    T, heads, dt = Q.shape[1] // B, Q.shape[2] // d, nf._dt(Q)
    q, qm, qr = _rows(Q, "Q", M, B * T, heads * d, Q.dtype)
    k, v, km, kr = _key_value_rows(K, V, M, B * T, kv_heads * d, Q.dtype)
    if length is None or any(x is None for x in held):
        raise ValueError("length and the four parts of the cache are required")
    small = (_dense(pos, "pos", (M, B, kv_heads, C), torch.int32), _dense(length, "length", (M, B), torch.int32), _dense(start, "start", (M, B), torch.int32),
             _dense(parent, "parent", (M, B, T), torch.int32), _dense(nodes, "nodes", (M, B), torch.int32), _dense(slope, "slope", (M, heads), torch.float32))
    z = _dense(lse, "lse", (M, B * T, heads), torch.float32)
    O = _output(stream, (M, B * T, heads * d), Q.dtype, Q.device) if out is None else out
    o = _dense(O, "out", (M, B * T, heads * d), Q.dtype)
    need = max(0, nf.lib.netfuse_attention_tree_fp4_workspace(M, B, T, C, heads, kv_heads, d, dt))
    ws, ws_ptr, ws_bytes = _workspace(workspace, need, Q.device, stream)
    nf._check("netfuse_attention_tree_fp4", nf.lib.netfuse_attention_tree_fp4(
        q, k, v, *held, *small, o, z, ws_ptr, ws_bytes, M, B, T, C, heads, kv_heads, d, qm, qr, km, kr, float(d ** -0.5 if scale is None else scale), float(cap), dt, nf._stream(stream)))
    return O


def token_logprobs_workspace(M, B, T, V, k) -> int:
    """Bytes of workspace of token_logprobs."""
    n = nf.lib.netfuse_token_logprobs_workspace(M, B, T, V, k)
    if n < 0:
        raise nf.NetFuseError("netfuse_token_logprobs_workspace", nf.NF_EINVAL)
    return n


def token_logprobs(logits, token=None, k=0, vocab=None, nodes=None, scale=1.0, cap=0.0, out=None, workspace=None, stream=None):
    """Log probabilities of the tokens token[M, N, n] under logits[M, N, V] (N = B*T rows per model, last dimension contiguous), of cap*tanh(scale*logit/cap) (cap 0:
    scale*logit): -> (logp[M, N, n], entropy[M, N], top[M, N, k], top_logp[M, N, k]); logp is None without token, the last two with k = 0.

    top: the k <= 32 tokens of the largest logits, the lower first among equals, -1 where there are no more.  vocab[m]: tokens that model m has (None: V).
    A temperature t is scale 1/t; where the model caps its logits at c before they are divided by it, scale 1/t and cap c/t.
    nodes[M, B]: how many of the T rows of a sequence are there; the others are as rows without tokens.  out: the four results to write into.
    workspace: token_logprobs_workspace(...) bytes, a call's own if None."""
    if nf._native is not None and stream is None and type(logits) is nf._Tensor and logits.is_cuda:
        device = nf._device()
        done = nf._native.token_logprobs(logits, token, k, vocab, nodes, scale, cap, out, workspace, device, nf._raw_stream(device))
        if done is not None:
            return done
    if logits.dim() != 3:
        raise ValueError("logits must be [M, N, V]")
    M, N, V = logits.shape
    dt = nf._dt(logits)
    p, sm, sr = _rows(logits, "logits", M, N, V, logits.dtype)
    B = 1
    if nodes is not None:
        if nodes.dim() != 2 or nodes.shape[1] == 0 or N % nodes.shape[1]:
            raise ValueError("nodes must be [M, B], N a multiple of B")
        B = nodes.shape[1]
    n = 0
    if token is not None:
        if token.dim() != 3 or token.shape[2] == 0:
            raise ValueError("token must be [M, N, n], n at least 1")
        n = token.shape[2]
    if out is None:
        f32, dev = torch.float32, logits.device
        out = (_output(stream, (M, N, n), f32, dev) if n else None, _output(stream, (M, N), f32, dev), _output(stream, (M, N, k), torch.int32, dev) if k else None,
               _output(stream, (M, N, k), f32, dev) if k else None)
    logp, entropy, top, top_logp = out
    need = max(16, nf.lib.netfuse_token_logprobs_workspace(M, B, N // B, V, k))
    ws, ws_ptr, ws_bytes = _workspace(workspace, need, logits.device, stream)
    nf._check("netfuse_token_logprobs", nf.lib.netfuse_token_logprobs(
        p, _dense(token, "token", (M, N, n), torch.int32), _dense(vocab, "vocab", (M,), torch.int32), _dense(nodes, "nodes", (M, B), torch.int32), _dense(logp, "logp", (M, N, n), torch.float32),
        _dense(entropy, "entropy", (M, N), torch.float32), _dense(top, "top", (M, N, k), torch.int32), _dense(top_logp, "top_logp", (M, N, k), torch.float32), ws_ptr, ws_bytes, M, B, N // B, V, n, k,
        sm, sr, float(scale), float(cap), dt, nf._stream(stream)))
    return out
