"""The operators as a training step runs them: QKV projection, head norms with rotation, attention layer with 8-bit
checkpoints, output projection, language-model loss, and back, on sequence shards; the whole against the same chain in fp64."""
import numpy as np
import pytest
import torch

import oracle
from helpers import make_plan
from paper_2609_03151_b200 import synth

pytestmark = pytest.mark.gpu


def f64(t):
    return t.detach().double().cpu()


class Linear(torch.autograd.Function):
    """x W^T per shard by the library's projection, gradients by plain products."""

    @staticmethod
    def forward(ctx, call, w, *x):
        ctx.save_for_backward(w, *x)
        return tuple(call(list(x), w))

    @staticmethod
    def backward(ctx, *dy):
        w, *x = ctx.saved_tensors
        dy = [g.reshape(g.shape[0], -1) for g in dy]
        dw = sum(g.float().t() @ t.float() for g, t in zip(dy, x))
        return (None, dw.to(w.dtype), *[(g.float() @ w.float()).to(t.dtype) for g, t in zip(dy, x)])


@pytest.mark.parametrize("checkpoint8", [False, True])
def test_step(basp, checkpoint8):
    from paper_2609_03151_b200.autograd import basp_attention, basp_lm_loss, basp_qk_norm_rope
    w = synth.Workload("step", N=4, B=2, S=256, Hq=4, Hkv=2, D=128)
    hidden, vocab, T = 256, 1000, 128
    pl = make_plan(basp, w)
    g = torch.Generator().manual_seed(1)
    x = [synth.randn_bf16(g, (T, hidden)) for _ in range(4)]
    wq = (torch.randn(((4 + 4) * 128, hidden), generator=g) / hidden ** 0.5).to(torch.bfloat16)
    wo = (torch.randn((hidden, 512), generator=g) / 512 ** 0.5).to(torch.bfloat16)
    wv = (torch.randn((vocab, hidden), generator=g) / hidden ** 0.5).to(torch.bfloat16)
    nq, nk = ((1 + 0.2 * torch.randn(128, generator=g)).to(torch.bfloat16) for _ in range(2))
    labels = [torch.randint(0, vocab, (T,), generator=g) for _ in range(4)]
    labels[1][5] = -100
    cos, sin = synth.rope_tables(256, 128)

    # ---- the library, bf16
    X = [t.cuda().requires_grad_() for t in x]
    P = [t.cuda().requires_grad_() for t in (wq, wo, wv, nq, nk)]
    tables = [t.t().contiguous().cuda() for t in (cos, sin)]

    def qkv(xs, wt):
        out = [torch.empty((T, h, 128), dtype=torch.bfloat16, device="cuda") for h in (4,) * 4 + (2,) * 8]
        basp.basp_qkv_proj(pl, hidden, xs, wt, out[:4], out[4:8], out[8:])
        return [torch.cat([out[r], out[4 + r], out[8 + r]], dim=1) for r in range(4)]

    def back_out(os, wt):
        y = [torch.empty((T, hidden), dtype=torch.bfloat16, device="cuda") for _ in range(4)]
        basp.basp_out_proj(pl, hidden, os, wt, y)
        return y

    basp.basp_clear_status()
    rows = Linear.apply(qkv, P[0], *X)
    q, k, v = ([t[:, a:b].contiguous() for t in rows] for a, b in ((0, 4), (4, 6), (6, 8)))
    q, k = basp_qk_norm_rope(pl, q, k, P[3], P[4], *tables)
    o = basp_attention(pl, q, k, v, fused=True, checkpoint8=checkpoint8)
    y = Linear.apply(back_out, P[1], *[t.reshape(T, 512) for t in o])
    weight = [torch.full((T,), 1.0 / 511, device="cuda") for _ in range(4)]
    loss = basp_lm_loss(pl, y, P[2], [t.cuda() for t in labels], weight)
    loss.backward()
    basp.basp_get_status()

    # ---- the chain in fp64 by torch's autograd (group g: ranks 2g, 2g + 1 hold the halves of sequence g)
    X8 = torch.cat(x).double().requires_grad_()
    P8 = [t.double().requires_grad_() for t in (wq, wo, wv, nq, nk)]
    c, s = (t.double().repeat(2, 1)[:, None, :] for t in (cos, sin))

    def norm_rope(t, wt):
        z = t / torch.sqrt(t.square().mean(-1, keepdim=True) + 1e-6) * wt
        lo, hi = z.chunk(2, -1)
        return torch.cat([lo * c - hi * s, hi * c + lo * s], -1)
    r8 = (X8 @ P8[0].t()).view(512, 8, 128)
    q8, k8, v8 = norm_rope(r8[:, :4], P8[3]), norm_rope(r8[:, 4:6], P8[4]), r8[:, 6:]
    sp = lambda t, n: t.view(2, 256, n, 128).transpose(1, 2)
    k8, v8 = (sp(t, 2).repeat_interleave(2, 1) for t in (k8, v8))
    a = (sp(q8, 4) @ k8.transpose(-1, -2) / 128 ** 0.5).masked_fill(~torch.ones(256, 256).tril().bool(), float("-inf")).softmax(-1)
    o8 = (a @ v8).transpose(1, 2).reshape(512, 512)
    z = (o8 @ P8[1].t()) @ P8[2].t()
    lab = torch.cat(labels)
    ok = lab >= 0
    loss8 = ((torch.logsumexp(z, -1) - z.gather(1, lab.clamp(min=0)[:, None])[:, 0]) * ok).sum() / 511
    loss8.backward()

    assert abs(loss.item() - loss8.item()) <= 5e-3 * abs(loss8.item())
    # every tensor between the steps is rounded to bf16 (2^-9 in the mean): a dozen roundings in a row give about 1 %; the
    # checkpoints' step of a 127th of a vector's largest element is about 0.6 % of each of Q, K, V, O and enters the scores twice
    bound = 0.05 if checkpoint8 else 0.03
    for name, got, ref in [("x", torch.cat([t.grad for t in X]), X8.grad)] + [(n, t.grad, r.grad) for n, t, r in
                                                                              zip(("wqkv", "wo", "head", "w_q", "w_k"), P, P8)]:
        off = (f64(got) - ref).norm() / ref.norm()
        assert off <= bound, (name, float(off))
