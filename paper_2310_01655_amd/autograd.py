"""torch.autograd glue over the C ABI, for callers that train.

Only marshalling happens here: the forward is psf_causal_attn_fwd_save where the library keeps
the forward state for the backward pass (psf_fwd_save_bytes(desc) > 0), psf_causal_attn_fwd
elsewhere; the backward is psf_causal_attn_bwd_saved / psf_causal_attn_bwd.  The Gaussian
sketch matrices G are constants of the layer (Algorithm 1 draws them once): they receive no
gradient.  With learned sketches (Algorithm 2) G holds the networks' parameters, which are
trained with the model: when G requires a gradient the backward is
psf_causal_attn_bwd_saved_learned / psf_causal_attn_bwd_learned and G receives the parameter gradient (accumulated in fp32 by the library, returned in G's dtype).
layer_norm and causal_window_attention are the differentiable forms of psf_layer_norm_* and psf_window_attn_*.
"""
import torch

from . import binding as psf


class _CausalPolysketchAttention(torch.autograd.Function):
    @staticmethod
    def forward(ctx, Q, K, V, G, desc):
        Q, K, V = Q.contiguous(), K.contiguous(), V.contiguous()
        stream = torch.cuda.current_stream(Q.device)
        if psf.fwd_save_bytes(desc) > 0:
            O, save = psf.psf_causal_attn_fwd_save(desc, Q, K, V, G, stream=stream)
        else:
            O, save = psf.psf_causal_attn_fwd(desc, Q, K, V, G, stream=stream), None
        ctx.desc, ctx.save = desc, save
        ctx.g_grad = bool(desc.learned) and G is not None and G.requires_grad
        ctx.save_for_backward(Q, K, V, G if G is not None else Q.new_empty(0), O)
        return O

    @staticmethod
    def backward(ctx, dO):
        Q, K, V, G, O = ctx.saved_tensors
        G = G if G.numel() else None
        dO = dO.contiguous()
        stream = torch.cuda.current_stream(Q.device)
        if ctx.g_grad:
            if ctx.save is not None:
                dQ, dK, dV, dG = psf.psf_causal_attn_bwd_saved_learned(ctx.desc, Q, K, V, G, O, dO, ctx.save,
                                                                       stream=stream)
            else:
                dQ, dK, dV, dG = psf.psf_causal_attn_bwd_learned(ctx.desc, Q, K, V, G, dO, stream=stream)
            return dQ, dK, dV, dG.to(G.dtype), None
        if ctx.save is not None:
            dQ, dK, dV = psf.psf_causal_attn_bwd_saved(ctx.desc, Q, K, V, G, O, dO, ctx.save, stream=stream)
        else:
            dQ, dK, dV = psf.psf_causal_attn_bwd(ctx.desc, Q, K, V, G, dO, stream=stream)
        return dQ, dK, dV, None, None


def causal_polysketch_attention(Q, K, V, G, p, r, b, local=psf.LOCAL_EXACT, per_head=False, learned=False, q_norm=None,
                                k_norm=None):
    """Differentiable causal Polysketch attention (Sections 3, 3.1, 3.2 of the paper) of
    Q, K [batch, heads, n, d] and V [batch, heads, n, dv] on the GPU; G as for
    psf_causal_attn_fwd ([1 or heads, g_len(d, r, p)], None for p = 2; with learned = True the
    networks' parameters of Algorithm 2, [1 or heads, learned_len(d, r, p)]).  Gradients flow to
    Q, K and V, and to G when it holds learned parameters that require a gradient.  q_norm, k_norm: (weight, bias or None)
    of a layer normalisation of the query or key rows before the attention (Section 2.1), whose parameters get
    gradients too."""
    Q, K = _normed(Q, q_norm), _normed(K, k_norm)
    B, H, n, d = Q.shape
    dtype = {torch.float32: "f32", torch.bfloat16: "bf16"}[Q.dtype]
    desc = psf.make_desc(B, H, n, d, p, r, b, dtype, dv=V.shape[-1], local=local, per_head=per_head,
                         learned=learned)
    return _CausalPolysketchAttention.apply(Q, K, V, G, desc)


def _first_order_only():
    # (what torch's once_differentiable does, at a tenth of its time: a backward pass with gradients enabled is one
    # that is to be differentiated again)
    if torch.is_grad_enabled():
        raise RuntimeError("no second derivatives: call backward without create_graph")


class _LayerNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, eps):
        x = x.contiguous()
        y, stats = psf.psf_layer_norm_fwd(x, weight, bias, eps, want_stats=True)
        ctx.save_for_backward(x, weight, stats)
        ctx.has_bias = bias is not None
        return y

    @staticmethod
    def backward(ctx, dy):
        _first_order_only()
        x, weight, stats = ctx.saved_tensors
        dx, dweight, dbias = psf.psf_layer_norm_bwd(x, weight, stats, dy.contiguous(), want_bias=ctx.has_bias)
        return dx, dweight, dbias, None


def layer_norm(x, weight, bias=None, eps=1e-6):
    """Differentiable layer normalisation over the last axis of x (at most 8192 long), float32 or bfloat16: the step the
    paper puts before the attention (Section 2.1), for Q and K rows or a model's tokens.  weight and
    bias [width] in x's dtype."""
    return _LayerNorm.apply(x, weight.contiguous(), None if bias is None else bias.contiguous(), eps)


class _CausalWindowAttention(torch.autograd.Function):
    @staticmethod
    def forward(ctx, Q, K, V, lengths, desc):
        Q, K, V = Q.contiguous(), K.contiguous(), V.contiguous()
        O, lse = psf.psf_window_attn_fwd(desc, Q, K, V, lengths=lengths, want_lse=True)
        ctx.desc = desc
        ctx.save_for_backward(Q, K, V, lengths, O, lse)
        return O

    @staticmethod
    def backward(ctx, dO):
        _first_order_only()
        Q, K, V, lengths, O, lse = ctx.saved_tensors
        dQ, dK, dV = psf.psf_window_attn_bwd(ctx.desc, Q, K, V, O, lse, dO.contiguous(), lengths=lengths)
        return dQ, dK, dV, None, None


def _normed(x, norm):
    return x if norm is None else layer_norm(x, *norm)


def causal_window_attention(Q, K, V, window=None, sinks=0, lengths=None, scale=None, tokens_first=False, q_norm=None,
                            k_norm=None):
    """Differentiable softmax attention in which row i sees its last `window` tokens (None: all) and the first `sinks`
    tokens of the sequence.  Q [batch, heads, n, d], K and V [batch, kv_heads, n, d], heads a multiple of kv_heads,
    or with tokens_first all of them [batch, n, heads, d]; d a multiple of 8, at most 128.  lengths: int32 [batch] on the
    GPU, tokens of each sequence (rows behind them give zeros and get zero gradients).  q_norm, k_norm as for
    causal_polysketch_attention."""
    if Q.dim() != 4 or K.dim() != 4:
        raise ValueError("Q, K, V must have four axes")
    Q, K = _normed(Q, q_norm), _normed(K, k_norm)
    at = 2 if tokens_first else 1
    dtype = {torch.float32: "f32", torch.bfloat16: "bf16"}[Q.dtype]
    desc = psf.make_window_desc(Q.shape[0], Q.shape[at], Q.shape[3 - at], Q.shape[3], window, sinks, dtype,
                                kv_heads=K.shape[at], tokens_first=tokens_first, scale=scale)
    return _CausalWindowAttention.apply(Q, K, V, lengths, desc)
