"""The attention layer and the operators around it as differentiable torch operations (marshalling only: forward =
basp_layer_fwd, backward = basp_layer_bwd, or with fused=True basp_layer_fwd_fused and basp_layer_bwd_seq; nothing is
computed in Python).

    q_seq, k_seq = basp_qk_norm_rope(plan, q_seq, k_seq, w_q, w_k, cos, sin)   # head norms and rotation
    o_seq = basp_attention(plan, q_seq, k_seq, v_seq)          # lists of n_ranks sequence-sharded bf16 tensors
    loss = basp_lm_loss(plan, x_seq, w, labels)                # cross entropy over the vocabulary, a scalar
    loss.backward()                                            # gradients arrive on the inputs

The forward keeps its workspace (head-sharded Q, K, V, O) and the log-sum-exp for the backward, as a training step of the
paper's setting does between the two passes; the backward needs a second workspace (basp_layer_bwd_workspace_bytes).
Both are allocated through torch's caching allocator on the current device.  With fused=True the forward is the one
fused kernel and keeps nothing but its output and the log-sum-exp (no head-sharded copies live between the passes: for
the 128K-token training shape that is 2.5 GiB less); the backward then redoes the exchanges of Q, K, V and O itself.  With
fused=True and checkpoint8=True what is kept of Q, K, V and O are 8-bit checkpoints (basp_ckpt_pack), saved as any tensors that
hooks may move away; the backward reads them back with the exchanges (basp_layer_bwd_ckpt).  With 32/8 heads of 128 that is 10.6 KB
per token in place of 20.5 where nothing else keeps the bf16 tensors.  It is little where something does: the output O that a
projection keeps for its own backward stays in bf16, and then the two forms hold 18.8 and 20.5 KB.  The head norms keep their
own inputs (10.2 KB) in either case.

The operations run on the current stream with the tensors' device current, and may be captured into a CUDA graph, forward and
backward, as torch prescribes: warmed up on a side stream, and with no eager graph of the same leaves alive during the capture.
"""
from __future__ import annotations

import torch
from torch.autograd.function import once_differentiable

from . import binding


class _BaspAttention(torch.autograd.Function):
    @staticmethod
    def forward(ctx, plan, softmax_scale, fused, checkpoint8, grads, *shards):
        n = plan.N
        if checkpoint8 and not fused:
            raise ValueError("checkpoint8 goes with fused=True (the other form keeps its head-sharded copies)")
        if len(shards) != 3 * n:
            raise ValueError(f"expected {3 * n} shards (q, k, v of {n} ranks), got {len(shards)}")
        q_seq, k_seq, v_seq = shards[:n], shards[n:2 * n], shards[2 * n:]
        for t in shards:
            if t.dtype != torch.bfloat16 or not t.is_cuda or not t.is_contiguous():
                raise ValueError("shards must be contiguous bf16 CUDA tensors")
        dev = q_seq[0].device
        o_seq = [torch.empty_like(t) for t in q_seq]
        lse = [torch.empty((plan.Bl, plan.Hq_l, plan.S), dtype=torch.float32, device=dev) for _ in range(n)]
        if fused:
            binding.basp_layer_fwd_fused(plan, list(q_seq), list(k_seq), list(v_seq), o_seq, lse, softmax_scale=softmax_scale)
            ws = None
            if checkpoint8 and grads and any(ctx.needs_input_grad):
                ckpt = [torch.empty(binding.basp_ckpt_bytes(plan, r), dtype=torch.uint8, device=dev) for r in range(n)]
                binding.basp_ckpt_pack(plan, q_seq, k_seq, v_seq, o_seq, ckpt)
                ctx.save_for_backward(*ckpt)
            elif not checkpoint8:
                ctx.save_for_backward(*shards, *o_seq)
        else:
            ws = torch.empty(binding.basp_workspace_bytes(plan), dtype=torch.uint8, device=dev)
            binding.basp_layer_fwd(plan, list(q_seq), list(k_seq), list(v_seq), o_seq, ws, lse_shards=lse,
                                   softmax_scale=softmax_scale)
        ctx.plan, ctx.softmax_scale, ctx.ws, ctx.lse, ctx.fused, ctx.checkpoint8 = plan, softmax_scale, ws, lse, fused, checkpoint8
        ctx.shapes = [t.shape for t in shards]
        return tuple(o_seq)

    @staticmethod
    @once_differentiable
    def backward(ctx, *do_seq):
        plan, n = ctx.plan, ctx.plan.N
        dev = ctx.lse[0].device
        do_seq = [torch.zeros(s, dtype=torch.bfloat16, device=dev) if g is None else g.contiguous()
                  for g, s in zip(do_seq, ctx.shapes)]
        grads = [torch.empty(s, dtype=torch.bfloat16, device=dev) for s in ctx.shapes]
        if ctx.checkpoint8:
            ws2 = torch.empty(binding.basp_layer_bwd_seq_workspace_bytes(plan), dtype=torch.uint8, device=dev)
            binding.basp_layer_bwd_ckpt(plan, ctx.saved_tensors, ctx.lse, do_seq, grads[:n], grads[n:2 * n], grads[2 * n:], ws2,
                                        softmax_scale=ctx.softmax_scale)
            return (None, None, None, None, None, *grads)
        if ctx.fused:
            saved = ctx.saved_tensors
            q_seq, k_seq, v_seq, o_seq = (list(saved[i * n:(i + 1) * n]) for i in range(4))
            ws2 = torch.empty(binding.basp_layer_bwd_seq_workspace_bytes(plan), dtype=torch.uint8, device=dev)
            binding.basp_layer_bwd_seq(plan, q_seq, k_seq, v_seq, o_seq, ctx.lse, do_seq, grads[:n], grads[n:2 * n],
                                       grads[2 * n:], ws2, softmax_scale=ctx.softmax_scale)
            return (None, None, None, None, None, *grads)
        qh, kh, vh, oh = (binding.as_shards(a) for a in binding.basp_layer_workspace_shards(plan, ctx.ws))
        ws2 = torch.empty(binding.basp_layer_bwd_workspace_bytes(plan), dtype=torch.uint8, device=dev)
        binding.basp_layer_bwd(plan, qh, kh, vh, oh, ctx.lse, do_seq, grads[:n], grads[n:2 * n], grads[2 * n:], ws2,
                               softmax_scale=ctx.softmax_scale)
        return (None, None, None, None, None, *grads)


def basp_attention(plan, q_seq, k_seq, v_seq, softmax_scale: float = 0.0, fused: bool = False, checkpoint8: bool = False):
    """Causal (or, per the plan, unmasked) attention over the group-sharded sequences of `plan`: the two group-local
    all-to-alls and the attention of Section IV-C, differentiable.  Returns the list of n_ranks output shards in the
    layout of q_seq.  checkpoint8 (with fused): keep Q, K, V and O in 8 bits for the backward; O besides what others keep of it.
    Second derivatives are refused."""
    return list(_BaspAttention.apply(plan, float(softmax_scale), bool(fused), bool(checkpoint8), torch.is_grad_enabled(), *q_seq,
                                     *k_seq, *v_seq))


class _QkNormRope(torch.autograd.Function):
    @staticmethod
    def forward(ctx, plan, eps, cos, sin, w_q, w_k, *shards):
        n = plan.N
        if len(shards) != 2 * n:
            raise ValueError(f"expected {2 * n} shards (q, k of {n} ranks), got {len(shards)}")
        out = [torch.empty_like(t) for t in shards]
        with torch.cuda.device(w_q.device):
            binding.basp_qk_norm_rope(plan, shards[:n], shards[n:], w_q, w_k, cos, sin, out[:n], out[n:], eps=eps)
        ctx.plan, ctx.eps = plan, eps
        ctx.save_for_backward(cos, sin, w_q, w_k, *shards)
        return tuple(out)

    @staticmethod
    @once_differentiable
    def backward(ctx, *d_out):
        plan, n = ctx.plan, ctx.plan.N
        cos, sin, w_q, w_k, *shards = ctx.saved_tensors
        d_out = [torch.zeros_like(t) if g is None else g.contiguous() for g, t in zip(d_out, shards)]
        grads = [torch.empty_like(t) for t in shards]
        dw_q, dw_k = (torch.empty(plan.D, dtype=torch.float32, device=w_q.device) for _ in range(2))
        ws = torch.empty(binding.basp_qk_norm_rope_bwd_workspace_bytes(plan), dtype=torch.uint8, device=w_q.device)
        with torch.cuda.device(w_q.device):
            binding.basp_qk_norm_rope_bwd(plan, shards[:n], shards[n:], w_q, w_k, cos, sin, d_out[:n], d_out[n:], grads[:n],
                                          grads[n:], dw_q, dw_k, ws, eps=ctx.eps)
        return (None, None, None, None, dw_q.to(w_q.dtype), dw_k.to(w_k.dtype), *grads)


def basp_qk_norm_rope(plan, q_seq, k_seq, w_q, w_k, rope_cos, rope_sin, eps: float = 1e-6):
    """Root-mean-square norm of every query and key head (weights w_q, w_k [D], bf16) with the rotary embedding, on
    sequence-sharded Q and K; differentiable in the shards and the weights, not in the tables.  Returns (q shards, k shards)."""
    if rope_cos.requires_grad or rope_sin.requires_grad:
        raise ValueError("rope_cos and rope_sin are not differentiable")
    out = _QkNormRope.apply(plan, float(eps), rope_cos, rope_sin, w_q, w_k, *q_seq, *k_seq)
    return list(out[:plan.N]), list(out[plan.N:])


class _LmLoss(torch.autograd.Function):
    @staticmethod
    def forward(ctx, plan, labels, token_weights, piece_rows, grads, w, *x_seq):
        vocab, hidden = w.shape
        dev = w.device
        # needs_input_grad goes by requires_grad alone; `grads`: whether there will be a backward at all
        want_w, want_x = grads and ctx.needs_input_grad[5], grads and any(ctx.needs_input_grad[6:])
        loss = [torch.empty(t.shape[:-1], dtype=torch.float32, device=dev) for t in x_seq]
        dx = [torch.empty_like(t) for t in x_seq] if want_x else None
        dw = torch.empty_like(w) if want_w else None
        with torch.cuda.device(dev):
            if want_w or want_x:
                ws = torch.empty(binding.basp_lm_loss_grad_workspace_bytes(plan, hidden, vocab, piece_rows), dtype=torch.uint8,
                                 device=dev)
                binding.basp_lm_loss_grad(plan, hidden, vocab, x_seq, w, labels, token_weights, loss, None, dx, dw, ws,
                                          piece_rows=piece_rows)
            else:
                ws = torch.empty(binding.basp_lm_loss_fwd_workspace_bytes(plan, vocab), dtype=torch.uint8, device=dev)
                binding.basp_lm_loss_fwd(plan, hidden, vocab, x_seq, w, labels, loss, None, ws)
        ctx.n, ctx.want = len(x_seq), (want_w, want_x)
        ctx.save_for_backward(*([dw] if want_w else []), *(dx if want_x else []))
        every = torch.cat([t.reshape(-1) for t in loss])
        if token_weights is not None:
            weight = torch.cat([t.reshape(-1) for t in token_weights])
            label = torch.cat([t.reshape(-1) for t in labels])
            # a token of weight 0 has no part, whatever its loss, and one without a label none, whatever its weight
            every = torch.where((weight != 0) & (label >= 0) & (label < vocab), every * weight, 0.0)
        return every.sum()

    @staticmethod
    @once_differentiable
    def backward(ctx, d_loss):
        saved = list(ctx.saved_tensors)
        want_w, want_x = ctx.want
        dw = saved.pop(0) * d_loss if want_w else None
        return (None, None, None, None, None, dw, *((t * d_loss for t in saved) if want_x else [None] * ctx.n))


def basp_lm_loss(plan, x_seq, w, labels, token_weights=None, piece_rows: int = 0):
    """sum over the tokens of token_weights * (ln sum_v exp(x . w_v) - x . w_label): the language-model loss on the ranks'
    sequence shards x_seq (bf16 [..., hidden]) with the head w (bf16 [vocab, hidden]), without keeping the logits;
    differentiable in x_seq and w.  labels: int64 shards, a value outside [0, vocab) marks a token without a loss;
    token_weights: fp32 shards or None (1 each), for a mean 1 / (number of tokens with a label); not differentiable.
    The gradients are formed together with the loss (they need the same products) and kept for the backward, which
    scales them by the incoming gradient; under torch.no_grad() or inference_mode() the loss alone is computed."""
    if token_weights is not None and any(t.requires_grad for t in token_weights):
        raise ValueError("token_weights are not differentiable")
    return _LmLoss.apply(plan, list(labels), None if token_weights is None else list(token_weights), int(piece_rows),
                         torch.is_grad_enabled(), w, *x_seq)
