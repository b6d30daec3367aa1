"""torch.autograd glue over the C-ABI library: a differentiable function and a drop-in module.

Nothing here computes: tensors are allocated with torch, their addresses are handed to
dma_mask_gen / dma_fwd / dma_bwd_scores, and the results are returned to autograd.
The paper names this integration as its own future work (Section 7); the operations are
those of Section 4: Eq. 3-6 forward, Eq. 7-10 backward, and the chain rule of Eq. 3 that
carries the bias gradient on to the score parameters (Section 6).

Layout: packed tokens, Q [T, H_q, d], K, V [T, H_kv, d] (bf16 or fp32, contiguous), W [H_q, d]
and A [H_q] fp32, cu_seqlens [n_docs + 1] int32 on the same device.  A W of shape
[H_q, H_kv * d] selects the paper's full cross-head sampling tensor (Eq. 3: the score of a head
contracts the token's values of all heads; dma_scores_xhead and its chain rule).  The selection of
the kept keys is piecewise constant, so no gradient flows through it (Section 6).
"""
from __future__ import annotations

import math

import torch

from . import binding as B
from .paged_cache import PagedCache


def _dtype_code(t):
    if t.dtype == torch.bfloat16:
        return B.DMA_BF16
    if t.dtype == torch.float32:
        return B.DMA_F32
    raise TypeError(f"Q/K/V must be bfloat16 or float32, got {t.dtype}")


def _check_inputs(Q, K, V, W, A, cu_seqlens):
    for name, t in (("Q", Q), ("K", K), ("V", V), ("W", W), ("A", A), ("cu_seqlens", cu_seqlens)):
        if not t.is_cuda:
            raise RuntimeError(f"{name} must live on the GPU: this library has no CPU path")
    if Q.dim() != 3 or K.dim() != 3 or K.shape != V.shape or Q.shape[0] != K.shape[0] or Q.shape[2] != K.shape[2]:
        raise ValueError("expected Q [T, H_q, d] and K, V [T, H_kv, d]")
    if K.dtype != Q.dtype or V.dtype != Q.dtype:
        raise TypeError("Q, K, V must share one dtype")
    H_q, d = Q.shape[1], Q.shape[2]
    if W.shape not in ((H_q, d), (H_q, K.shape[1] * d)) or A.shape != (H_q,):
        raise ValueError("expected W [H_q, d] (per head) or [H_q, H_kv * d] (cross-head) and A [H_q]")
    if W.dtype != torch.float32 or A.dtype != torch.float32 or cu_seqlens.dtype != torch.int32:
        raise TypeError("W, A must be float32 and cu_seqlens int32")


def _row_bytes(H_q, T):
    """Bytes of an [H_q, T] buffer of 32-bit values, to the next whole 256."""
    return (H_q * T * 4 + 255) // 256 * 256


class DynamicMaskAttentionFunction(torch.autograd.Function):
    """O = DMA(Q, K, V; W, A) on packed variable-length documents; differentiable in Q, K, V, W, A."""

    @staticmethod
    def forward(ctx, Q, K, V, W, A, cu_seqlens, k, max_seqlen=0, softmax_scale=0.0, bias=None):
        _check_inputs(Q, K, V, W, A, cu_seqlens)
        Q, K, V, W, A = (t.contiguous() for t in (Q, K, V, W, A))
        T, H_q, d = Q.shape
        bias_heads, bias_per_token = 0, True
        if bias is not None:
            # one value per key, broadcast over the query rows: [H_q or 1, T] (packed like the tokens) or
            # [H_q or 1, max_seqlen] (by position in the document, shared by all documents)
            if (not bias.is_cuda or bias.dtype != torch.float32 or bias.dim() != 2 or bias.shape[0] not in (1, H_q)
                    or bias.shape[1] not in (T, max_seqlen)):
                raise ValueError("bias must be a float32 GPU tensor [H_q or 1, T] or [H_q or 1, max_seqlen]")
            bias = bias.contiguous()
            bias_heads, bias_per_token = bias.shape[0], bias.shape[1] == T
        shape = B.make_shape(T, cu_seqlens.numel() - 1, H_q, K.shape[1], d, k, causal=True,
                             dtype=_dtype_code(Q), softmax_scale=softmax_scale, max_seqlen=max_seqlen)
        dev = Q.device
        # z, expiry, LSE and the mask plan live in one allocation (a short call's time is the host's)
        per_row = _row_bytes(H_q, T)
        state = torch.empty(3 * per_row + B.dma_mask_bytes(shape), dtype=torch.uint8, device=dev)
        z, expiry, LSE, mask = (state.data_ptr() + i * per_row for i in range(4))
        O = torch.empty_like(Q)
        xhead = K.shape[1] > 1 and W.shape[1] == K.shape[1] * d
        if xhead:
            B.dma_scores_xhead(shape, V, W, A, z)
        Wm, Am = (None, None) if xhead else (W, A)          # cross-head: the scores are supplied to dma_mask_gen
        if bias is None:
            B.dma_mask_gen(shape, V, Wm, Am, cu_seqlens, z, expiry, None, mask)
        else:
            B.dma_mask_gen_bias(shape, V, Wm, Am, cu_seqlens, bias, bias_heads, bias_per_token, z, expiry, None, mask)
        B.dma_fwd(shape, Q, K, V, z, expiry, mask, cu_seqlens, O, LSE, None, 0)
        ctx.save_for_backward(Q, K, V, W, A, cu_seqlens, state, O)
        ctx.shape, ctx.xhead = shape, xhead
        ctx.bias_form = None if bias is None else (bias_heads, bias_per_token, tuple(bias.shape))
        return O

    @staticmethod
    def backward(ctx, dO):
        Q, K, V, W, A, cu_seqlens, state, O = ctx.saved_tensors
        shape = ctx.shape
        dO = dO.contiguous()
        per_row, ws_bytes = _row_bytes(Q.shape[1], Q.shape[0]), B.dma_workspace_bytes(shape)
        z, expiry, LSE, mask = (state.data_ptr() + i * per_row for i in range(4))
        dQ, dK, dV = torch.empty_like(Q), torch.empty_like(K), torch.empty_like(V)
        dW, dA = torch.empty_like(W), torch.empty_like(A)
        scratch = torch.empty(per_row + ws_bytes, dtype=torch.uint8, device=Q.device)   # dz, then the workspace
        dz = scratch.data_ptr()
        ws = dz + per_row
        # dz -> dW, dA, and the part of dV that flows through the content scores, added in place
        if ctx.xhead:
            B.dma_bwd(shape, Q, K, V, O, dO, LSE, z, expiry, mask, cu_seqlens, dQ, dK, dV, dz, ws, ws_bytes)
            B.dma_scores_xhead_bwd(shape, V, W, A, dz, dW, dA, dV, True)
        else:
            B.dma_bwd_scores(shape, Q, K, V, O, dO, LSE, z, expiry, mask, cu_seqlens, W, A, dQ, dK, dV, dz, dW, dA,
                             ws, ws_bytes)
        dbias = None
        if ctx.bias_form is not None:   # the bias enters the score like z: its gradient is dz, reduced over what shares it
            bias_heads, bias_per_token, bshape = ctx.bias_form
            dbias = torch.empty(bshape, dtype=torch.float32, device=Q.device)
            B.dma_bias_bwd(shape, dz, cu_seqlens, bias_heads, bias_per_token, dbias)
        return dQ, dK, dV, dW, dA, None, None, None, None, dbias


def dynamic_mask_attention(Q, K, V, W, A, cu_seqlens, k, max_seqlen=0, softmax_scale=0.0, bias=None):
    """Functional form; see DynamicMaskAttentionFunction.  bias (optional, differentiable): a further
    additive attention bias per key, [H_q or 1, T] or [H_q or 1, max_seqlen] (Section 1: biases with
    batch, head and query broadcasting); it does not take part in the selection of the kept keys."""
    return DynamicMaskAttentionFunction.apply(Q, K, V, W, A, cu_seqlens, k, max_seqlen, softmax_scale, bias)


def rotary_freqs(dim, base=10000.0, device=None):
    """base^(-2 i / dim) for the dim / 2 pairs of dim rotated channels (float32)."""
    i = torch.arange(dim // 2, dtype=torch.float64, device="cpu")    # (the same numbers for every device)
    return (float(base) ** (-2.0 * i / dim)).float().to(device)


class RotaryFunction(torch.autograd.Function):
    """Q and K turned to their positions, or back (dma_rope); their gradients go the other way.  Differentiable in Q and K, any number of times."""

    @staticmethod
    def forward(ctx, Q, K, freqs, cu_seqlens, positions, interleaved, inverse):
        T = Q.shape[0]
        for name, t in (("Q", Q), ("K", K), ("freqs", freqs), ("cu_seqlens", cu_seqlens), ("positions", positions)):
            if t is not None and not t.is_cuda:
                raise RuntimeError(f"{name} must live on the GPU: this library has no CPU path")
            if t is not None and t.device != Q.device:
                raise RuntimeError(f"{name} must be on {Q.device}, got {t.device}")
        if Q.dim() != 3 or K.dim() != 3 or K.shape[0] != T or K.shape[2] != Q.shape[2]:
            raise ValueError("expected Q [T, H_q, d] and K [T, H_kv, d]")
        if (cu_seqlens is None) == (positions is None):
            raise ValueError("positions are those in the documents of cu_seqlens, or given: one of the two")
        if ctx.needs_input_grad[2]:
            raise ValueError("freqs get no gradient")
        if positions is not None and positions.shape != (T,):
            raise ValueError(f"expected positions [{T}], got {list(positions.shape)}")
        if K.dtype != Q.dtype or freqs.dtype != torch.float32 or freqs.dim() != 1 or (cu_seqlens if positions is None else positions).dtype != torch.int32:
            raise TypeError("Q and K must share one dtype, freqs [m] be float32, cu_seqlens or positions int32")
        freqs, cu_seqlens, positions = (None if t is None else t.contiguous() for t in (freqs, cu_seqlens, positions))
        shape = B.make_shape(T, 1 if cu_seqlens is None else cu_seqlens.numel() - 1, Q.shape[1], K.shape[1], Q.shape[2], 1, dtype=_dtype_code(Q))
        Qi, Ki = PagedCache._rows(Q), PagedCache._rows(K)     # (where they lie, if rows can be read there)
        Qo, Ko = (torch.empty(x.shape, dtype=x.dtype, device=x.device) for x in (Q, K))
        with torch.cuda.device(Q.device):
            B.dma_rope(shape, Qi, Qi.stride(0), Ki, Ki.stride(0), cu_seqlens, positions, freqs, 2 * freqs.numel(), interleaved, inverse, Qo,
                       Qo.stride(0), Ko, Ko.stride(0))
        ctx.save_for_backward(freqs, cu_seqlens, positions)
        ctx.way = bool(interleaved), not inverse
        return Qo, Ko

    @staticmethod
    def backward(ctx, dQ, dK):
        return (*RotaryFunction.apply(dQ, dK, *ctx.saved_tensors, *ctx.way), None, None, None, None, None)


def rotary(Q, K, freqs, cu_seqlens=None, positions=None, interleaved=False):
    """Q [T, H_q, d] and K [T, H_kv, d] with their first 2 * len(freqs) channels turned in pairs, pair i by position * freqs[i]: the
    channels (i, i + len(freqs)), or (2 i, 2 i + 1) if interleaved.  A token's position is its place in its document (cu_seqlens), or
    positions [T] (int32).  Differentiable in Q and K, which may be parts of one projection's output."""
    return RotaryFunction.apply(Q, K, freqs, cu_seqlens, positions, interleaved, False)


class DynamicMaskAttention(torch.nn.Module):
    """The attention core of a DMA layer (the part between the QKV projections and the output
    projection).  Parameters: the score projection `W` [H_q, d] (the paper's Delta taken per head;
    [H_q, H_kv * d], the full tensor, with cross_head=True) and the gate `A` [H_q].  Their
    initialisation is a choice of this module, not the paper's: W ~ N(0, 1 / fan-in), A = -1, which
    keeps the initial scores in (0, 1) and close together.

    forward(q, k, v): [B, L, H, d] batches (each sequence its own document), or packed [T, H, d]
    tensors with cu_seqlens.  rotary_dim > 0: q and k are turned to their positions first (rotary), in that many
    channels; positions [T] (int32, [B, L] with batches) replace those in the documents.  Frequencies other than those of
    rotary_base go into the buffer rotary_freqs (float32), which moves with the module and keeps its values and type.
    """

    def __init__(self, num_heads, num_kv_heads, head_dim, keep_window, softmax_scale=None, device=None,
                 cross_head=False, rotary_dim=0, rotary_base=10000.0, rotary_interleaved=False):
        super().__init__()
        if num_heads % num_kv_heads:
            raise ValueError("num_heads must be a multiple of num_kv_heads")
        self.num_heads, self.num_kv_heads, self.head_dim = num_heads, num_kv_heads, head_dim
        self.keep_window = int(keep_window)
        self.softmax_scale = 0.0 if softmax_scale is None else float(softmax_scale)
        fan_in = head_dim * (num_kv_heads if cross_head else 1)   # cross_head: the full Delta of Eq. 3
        self.W = torch.nn.Parameter(torch.randn(num_heads, fan_in, dtype=torch.float32, device=device)
                                    / math.sqrt(fan_in))
        if rotary_dim % 16 or not 0 <= rotary_dim <= head_dim:
            raise ValueError("rotary_dim must be a multiple of 16 of at most head_dim")
        self.rotary_interleaved = bool(rotary_interleaved)
        self.rotary_dim, self.rotary_base = rotary_dim, rotary_base
        freqs = rotary_freqs(rotary_dim, rotary_base, device) if rotary_dim else None
        self.register_buffer("rotary_freqs", freqs, persistent=False)
        self.A = torch.nn.Parameter(torch.full((num_heads,), -1.0, dtype=torch.float32, device=device))

    def _apply(self, fn, *args, **kwargs):
        held = self.rotary_freqs
        super()._apply(fn, *args, **kwargs)
        if held is not None:   # (a change of type does not round them, and where the device stays, so does the tensor: a graph may read it)
            device = self.rotary_freqs.device
            if held.is_meta and device.type != "meta":
                self.rotary_freqs = rotary_freqs(self.rotary_dim, self.rotary_base, device)
            else:
                self.rotary_freqs = held.to(device)
        return self

    def forward(self, q, k, v, cu_seqlens=None, max_seqlen=0, positions=None):
        if q.dim() == 4:
            if cu_seqlens is not None:
                raise ValueError("cu_seqlens goes with packed [T, H, d] inputs")
            Bsz, L = q.shape[0], q.shape[1]
            cu = torch.arange(0, (Bsz + 1) * L, L, dtype=torch.int32, device=q.device)
            packed = (x.reshape(Bsz * L, *x.shape[2:]) for x in (q, k, v))
            o = self._attend(*packed, cu, L, None if positions is None else positions.reshape(-1))
            return o.view(Bsz, L, *q.shape[2:])
        if cu_seqlens is None:
            raise ValueError("packed inputs need cu_seqlens")
        return self._attend(q, k, v, cu_seqlens, max_seqlen, positions)

    def _attend(self, q, k, v, cu_seqlens, max_seqlen, positions):
        if self.rotary_freqs is not None:
            q, k = rotary(q, k, self.rotary_freqs, cu_seqlens if positions is None else None, positions, self.rotary_interleaved)
        elif positions is not None:
            raise ValueError("positions go with rotary_dim")
        return dynamic_mask_attention(q, k, v, self.W, self.A, cu_seqlens, self.keep_window, max_seqlen,
                                      self.softmax_scale)

    def step(self, q, k, v, cache, rows, max_len=0, prefixes=None, max_prefix=0):
        """A decoding step over a paged cache (paged_cache.PagedCache): k, v [n, H_kv, d] of the step's new rows go to their places
        with this module's scores, then q [n, H_q, d] attends from them.  rows: what cache.assign returned; max_len: as for
        cache.decode; prefixes, max_prefix: as for cache.decode_prefix.  With rotary_dim, k and q are turned on the way, to their places in
        the requests, behind the prefixes.  Without gradients; o [n, H_q, d].  What cannot be done is refused before the cache is changed."""
        with torch.no_grad():
            W, A = self.W.detach(), self.A.detach()
            checked = cache._check_decode(q, self.keep_window, rows, self.softmax_scale, max_len, prefixes, max_prefix)   # (before the rows go in)
            freqs = self.rotary_freqs
            if freqs is not None:
                cache._check_rotary(rows, q, freqs, prefixes)
            if W.shape[1] == self.head_dim:
                if freqs is None:
                    cache.append(rows.slots, k, v, W=W, A=A)
                else:
                    q = cache.append_rotary(rows, q, k, v, freqs, W=W, A=A, prefixes=prefixes, interleaved=self.rotary_interleaved)
            else:                                    # the cross-head scores have an entry point of their own
                s, n = cache.shape, rows.slots.numel()
                cache._check_values(rows.slots, k, v)         # (all that append checks: a kernel reads v, W and A before it)
                cache._check("W", W, (s.H_q, s.H_kv * s.d), torch.float32)
                cache._check("A", A, (s.H_q,), torch.float32)
                z = torch.empty((s.H_q, n), dtype=torch.float32, device=v.device)
                if n:
                    shape = B.make_shape(n, 1, s.H_q, s.H_kv, s.d, 1, dtype=_dtype_code(v))
                    cache._call_with(shape, B.dma_scores_xhead, cache._rows(v).contiguous(), cache._aligned(W), A, z)
                if freqs is None:
                    cache._append(rows.slots, k, v, None, None, z)
                else:
                    q = cache._append_rotary(rows, q, k, v, freqs, None, None, z, prefixes, self.rotary_interleaved)
            if prefixes is not None:
                return cache._attend_prefix(q, *checked, self.softmax_scale, prefixes, max_prefix)[0]
            return cache._attend(q, *checked, self.softmax_scale)[0]
