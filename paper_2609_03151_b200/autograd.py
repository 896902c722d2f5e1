"""The attention layer and the operators around it as differentiable torch operations (marshalling only: forward =
basp_layer_fwd, backward = basp_layer_bwd, or with fused=True basp_layer_fwd_fused and basp_layer_bwd_seq; nothing is
computed in Python).

    q_seq, k_seq = basp_qk_norm_rope(plan, q_seq, k_seq, w_q, w_k, cos, sin)   # head norms and rotation
    q_seq, k_seq = basp_rope(plan, rope, q_seq, k_seq, positions)              # or the rotation alone, positions of packed documents
    o_seq = basp_attention(plan, q_seq, k_seq, v_seq)          # lists of n_ranks sequence-sharded bf16 tensors
    o_seq = basp_attention(plan, q_seq, k_seq, v_seq, score=score)             # capped, biased, masked (binding.basp_score)
    h_seq, n_seq = basp_block_norm(plan, x_seq, y_seq, w_post, gate, w_pre)    # norms, gate and sum between two blocks
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
    def forward(ctx, plan, softmax_scale, fused, checkpoint8, score, grads, *shards):
        n = plan.N
        if score is not None and fused:
            raise ValueError("score goes without fused (the fused kernel has the plan's own mask)")
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
            if score is not None:
                with torch.cuda.device(dev):
                    binding.basp_layer_masked_fwd(plan, score, q_seq, k_seq, v_seq, o_seq, ws, lse_shards=lse, softmax_scale=softmax_scale)
            else:
                binding.basp_layer_fwd(plan, list(q_seq), list(k_seq), list(v_seq), o_seq, ws, lse_shards=lse,
                                       softmax_scale=softmax_scale)
        if score is not None:
            # the backward reads them again: as saved tensors, so that one which was written in between is refused (raw addresses and
            # tensors of an inference mode have no record of that)
            tensors = (score.slopes, score.mask)
            kept = [isinstance(t, torch.Tensor) and not t.is_inference() for t in tensors]
            ctx.score = (score.softcap, *(None if keep else t for t, keep in zip(tensors, kept)))
            ctx.save_for_backward(*(t if keep else None for t, keep in zip(tensors, kept)))
        ctx.has_score = score is not None
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
            return (None, None, None, None, None, None, *grads)
        if ctx.fused:
            saved = ctx.saved_tensors
            q_seq, k_seq, v_seq, o_seq = (list(saved[i * n:(i + 1) * n]) for i in range(4))
            ws2 = torch.empty(binding.basp_layer_bwd_seq_workspace_bytes(plan), dtype=torch.uint8, device=dev)
            binding.basp_layer_bwd_seq(plan, q_seq, k_seq, v_seq, o_seq, ctx.lse, do_seq, grads[:n], grads[n:2 * n],
                                       grads[2 * n:], ws2, softmax_scale=ctx.softmax_scale)
            return (None, None, None, None, None, None, *grads)
        qh, kh, vh, oh = (binding.as_shards(a) for a in binding.basp_layer_workspace_shards(plan, ctx.ws))
        size = binding.basp_layer_masked_bwd_workspace_bytes if ctx.has_score else binding.basp_layer_bwd_workspace_bytes
        ws2 = torch.empty(size(plan), dtype=torch.uint8, device=dev)
        if ctx.has_score:
            softcap, *given = ctx.score
            score = binding.basp_score(softcap, *(t if saved is None else saved for saved, t in zip(ctx.saved_tensors, given)))
            with torch.cuda.device(dev):
                binding.basp_layer_masked_bwd(plan, score, qh, kh, vh, oh, ctx.lse, do_seq, grads[:n], grads[n:2 * n], grads[2 * n:],
                                              ws2, softmax_scale=ctx.softmax_scale)
        else:
            binding.basp_layer_bwd(plan, qh, kh, vh, oh, ctx.lse, do_seq, grads[:n], grads[n:2 * n], grads[2 * n:], ws2,
                                   softmax_scale=ctx.softmax_scale)
        return (None, None, None, None, None, None, *grads)


def basp_attention(plan, q_seq, k_seq, v_seq, softmax_scale: float = 0.0, fused: bool = False, checkpoint8: bool = False, score=None):
    """Causal (or, per the plan, unmasked) attention over the group-sharded sequences of `plan`: the two group-local
    all-to-alls and the attention of Section IV-C, differentiable.  Returns the list of n_ranks output shards in the
    layout of q_seq.  checkpoint8 (with fused): keep Q, K, V and O in 8 bits for the backward; O besides what others keep of it.
    score (without fused): a binding.basp_score, for capped scores, a bias by distance and masks of documents, prefixes, windows or
    any key ranges; its tensors are read again by the backward, which is refused where they were written in between (a mask refilled for the
    next batch among it: a mask for each batch whose backward is to come), and get no gradients.  Second derivatives are refused."""
    if score is not None and getattr(score.slopes, "requires_grad", False):
        raise ValueError("the slopes of a score are not differentiable")
    return list(_BaspAttention.apply(plan, float(softmax_scale), bool(fused), bool(checkpoint8), score, torch.is_grad_enabled(), *q_seq,
                                     *k_seq, *v_seq))


class _Rope(torch.autograd.Function):
    @staticmethod
    def forward(ctx, plan, rope, positions, *shards):
        n = plan.N
        if len(shards) != 2 * n:
            raise ValueError(f"expected {2 * n} shards (q, k of {n} ranks), got {len(shards)}")
        out = [torch.empty_like(t) for t in shards]
        with torch.cuda.device(shards[0].device):
            binding.basp_rope(plan, rope, shards[:n], shards[n:], out[:n], out[n:], positions=positions)
        ctx.plan, ctx.rope, ctx.has_positions = plan, rope, positions is not None
        ctx.shapes = [t.shape for t in shards]
        if positions is not None:
            ctx.save_for_backward(positions)
        return tuple(out)

    @staticmethod
    @once_differentiable
    def backward(ctx, *d_out):
        plan, n = ctx.plan, ctx.plan.N
        positions = ctx.saved_tensors[0] if ctx.has_positions else None
        dev = next(g.device for g in d_out if g is not None)
        d_out = [torch.zeros(s, dtype=torch.bfloat16, device=dev) if g is None else g.contiguous() for g, s in zip(d_out, ctx.shapes)]
        grads = [torch.empty_like(t) for t in d_out]
        with torch.cuda.device(dev):
            binding.basp_rope(plan, ctx.rope, d_out[:n], d_out[n:], grads[:n], grads[n:], positions=positions, inverse=True)
        return (None, None, None, *grads)


def basp_rope(plan, rope, q_seq, k_seq, positions=None):
    """Rotary positions on sequence-sharded Q and K (rope: of binding.basp_rope_make; positions: int32 [B, S], None: the place in the
    sequence); differentiable in the shards.  Returns (q shards, k shards)."""
    out = _Rope.apply(plan, rope, positions, *q_seq, *k_seq)
    return list(out[:plan.N]), list(out[plan.N:])


class _BlockNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, plan, res_scale, eps, w_post, gate, w_pre, *shards):
        n, has_y = plan.N, len(shards) == 2 * plan.N
        if len(shards) not in (n, 2 * n):
            raise ValueError(f"expected {n} or {2 * n} shards (x, and y where there is a block before, of {n} ranks), got {len(shards)}")
        x, y = shards[:n], shards[n:] if has_y else None
        hidden = x[0].shape[-1]
        h = [torch.empty_like(t) for t in x] if has_y else None
        after = [torch.empty_like(t) for t in x] if w_pre is not None else None
        with torch.cuda.device(x[0].device):
            binding.basp_block_norm(plan, hidden, x, y, h, after, w_post=w_post, gate=gate, w_pre=w_pre, res_scale=res_scale, eps=eps)
        ctx.plan, ctx.res_scale, ctx.eps, ctx.hidden, ctx.has_y = plan, res_scale, eps, hidden, has_y
        ctx.has = [t is not None for t in (w_post, gate, w_pre)]
        ctx.shapes, ctx.y_shapes = [t.shape for t in x], [t.shape for t in y or ()]
        ctx.weight_shapes = [None if t is None else t.shape for t in (w_post, gate, w_pre)]
        ctx.save_for_backward(*[t for t in (w_post, gate, w_pre) if t is not None], *((h if has_y else x) if w_pre is not None else ()),
                              *(y if w_post is not None or gate is not None else ()))
        return tuple((h or []) + (after or []))

    @staticmethod
    @once_differentiable
    def backward(ctx, *d_out):
        plan, n = ctx.plan, ctx.plan.N
        saved = list(ctx.saved_tensors)
        w_post, gate, w_pre = [saved.pop(0) if there else None for there in ctx.has]
        h = [saved.pop(0) for _ in range(n)] if w_pre is not None else None
        y = saved if w_post is not None or gate is not None else None
        dev = next(g.device for g in d_out if g is not None)
        fill = lambda gs: [torch.zeros(s, dtype=torch.bfloat16, device=dev) if g is None else g.contiguous() for g, s in zip(gs, ctx.shapes)]
        dh, dn = (d_out[:n], d_out[n:]) if ctx.has_y else ([], d_out)
        dn = fill(dn) if w_pre is not None else None
        # the stream's own gradient may be missing (the last sum's) where that through the norm is there
        dh = None if dn is not None and all(g is None for g in dh) else fill(dh)
        dx = [torch.empty(s, dtype=torch.bfloat16, device=dev) for s in ctx.shapes]
        dy = [torch.empty(s, dtype=torch.bfloat16, device=dev) for s in ctx.y_shapes] if ctx.has_y else None
        sums = [torch.empty(ctx.hidden, dtype=torch.float32, device=dev) if there else None for there in ctx.has]
        ws = torch.empty(binding.basp_block_norm_bwd_workspace_bytes(plan, ctx.hidden), dtype=torch.uint8, device=dev)
        with torch.cuda.device(dev):
            binding.basp_block_norm_bwd(plan, ctx.hidden, h, y, dh, dn, dx, dy, *sums, ws, w_post=w_post, gate=gate, w_pre=w_pre,
                                        res_scale=ctx.res_scale, eps=ctx.eps)
        return (None, None, None, *[None if s is None else s.to(torch.bfloat16).reshape(shape) for s, shape in zip(sums, ctx.weight_shapes)],
                *dx, *(dy or []))


def basp_block_norm(plan, x_seq, y_seq=None, w_post=None, gate=None, w_pre=None, res_scale: float = 1.0, eps: float = 1e-6):
    """h = x + res_scale gate norm(y; w_post) and n = norm(h; w_pre) on the ranks' rows (bf16 [..., hidden]): the edge between two blocks.
    Without y_seq (the first block) h is x itself; without w_pre (the last one) n is None.  Returns (h shards, n shards);
    differentiable in the shards and the weights."""
    n = plan.N
    out = _BlockNorm.apply(plan, float(res_scale), float(eps), w_post, gate, w_pre, *x_seq, *(y_seq or []))
    if y_seq is None:
        return list(x_seq), list(out)
    return list(out[:n]), list(out[n:]) or None


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
