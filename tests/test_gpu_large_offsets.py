"""Sizes whose element offsets pass 2^31, and losses of many pieces, on samples: head norms and their gradients, checkpoints, the
language-model loss.  References in fp64 on the sampled rows (on the GPU where a sum runs over all of them)."""
import numpy as np
import pytest
import torch

import oracle
from paper_2609_03151_b200 import synth

pytestmark = pytest.mark.gpu


def rough(n, seed, scale=1.0):
    """n bf16 values of about unit size without a generator's cost: a hash of the index."""
    out = torch.empty(n, dtype=torch.bfloat16, device="cuda")
    for a in range(0, n, 1 << 28):
        i = torch.arange(a, min(n, a + (1 << 28)), device="cuda", dtype=torch.int64)
        h = (i * 2654435761 + seed * 40503) & 0xffff
        out[a:a + i.numel()] = ((h.float() / 32768.0 - 1.0) * (1.7 * scale)).to(torch.bfloat16)
    return out


def test_norm_and_checkpoint_past_32_bits(basp):
    S, Hq, Hkv, D = 530001, 32, 1, 128                      # 2.17e9 elements of Q in one shard
    pl = basp.basp_plan_create(1, 1, S, Hq, Hkv, D)
    rows = [0, 1, 524287, 524288, 524289, S - 2, S - 1]     # 524288 rows of 4096: 2^31 elements
    q, k, dy = rough(S * Hq * D, 1), rough(S * Hkv * D, 2), rough(S * Hq * D, 3)
    w = rough(D, 4)
    cos, sin = synth.rope_tables(S, D)
    tables = [t.t().contiguous().cuda() for t in (cos, sin)]
    pick = lambda t, h: t.view(S, h, D)[rows].double().cpu().numpy()
    out, outk = torch.zeros_like(q), torch.zeros_like(k)
    basp.basp_qk_norm_rope(pl, [q], [k], w, w, *tables, [out], [outk], eps=1e-5)
    want = oracle.qk_norm_rope(pick(q, Hq), w.double().cpu().numpy(), cos.numpy(), sin.numpy(), rows, 1e-5)
    assert np.abs(pick(out, Hq) - want).max() <= 2.0 ** -8 * np.abs(want).max()
    dw = [torch.zeros(D, device="cuda") for _ in range(2)]
    ws = torch.empty(basp.basp_qk_norm_rope_bwd_workspace_bytes(pl), dtype=torch.uint8, device="cuda")
    basp.basp_qk_norm_rope_bwd(pl, [q], [k], w, w, *tables, [dy], [k], [out], [outk], *dw, ws, eps=1e-5)
    want, _ = oracle.qk_norm_rope_bwd(pick(q, Hq), w.double().cpu().numpy(), cos.numpy(), sin.numpy(), rows, 1e-5, pick(dy, Hq))
    assert np.abs(pick(out, Hq) - want).max() <= 2.0 ** -8 * np.abs(want).max()
    del dy, outk, tables
    ck = [torch.zeros(basp.basp_ckpt_bytes(pl, 0), dtype=torch.uint8, device="cuda")]
    basp.basp_ckpt_pack(pl, [q], [k], [k], [q], ck)
    ko, vo, oo = torch.zeros_like(k), torch.zeros_like(k), torch.zeros_like(q)
    basp.basp_ckpt_reshard_s2h(pl, ck, [out], [ko], [vo], [oo])
    want = torch.from_numpy(oracle.ckpt_values(*oracle.ckpt_codes(pick(q, Hq).astype(np.float32)))).to(torch.bfloat16).double().numpy()
    assert np.array_equal(pick(out, Hq), want) and np.array_equal(pick(oo, Hq), want)


@pytest.mark.parametrize("rows,hidden,vocab,piece", [
    (8200, 64, 264193, 0),             # 8200 x 264193: the 16-bit logits pass 2^31 elements; two pieces
    (8192, 128, 262400, 8192),         # in one piece
    (30001, 72, 1100, 0),              # four pieces, the last one short
    (40000, 64, 700, 32768),
])
def test_loss_of_many_logits_and_pieces(basp, rows, hidden, vocab, piece):
    pl = basp.basp_plan_create(1, 1, rows, 1, 1, 64)
    x = rough(rows * hidden, 5).view(rows, hidden)
    w = rough(vocab * hidden, 6, 2.0 / hidden ** 0.5).view(vocab, hidden)
    y = (torch.arange(rows, device="cuda") * 7919 + 3) % vocab
    y[::17] = -100
    g = torch.rand(rows, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda")
    loss, lse = torch.zeros(rows, device="cuda"), torch.zeros(rows, device="cuda")
    dx, dw = torch.zeros_like(x), torch.zeros_like(w)
    ws = torch.empty(basp.basp_lm_loss_grad_workspace_bytes(pl, hidden, vocab, piece), dtype=torch.uint8, device="cuda")
    basp.basp_clear_status()
    basp.basp_lm_loss_grad(pl, hidden, vocab, [x], w, [y], [g], [loss], [lse], [dx], dw, ws, piece_rows=piece)
    basp.basp_get_status()
    x8, w8, g8 = x.double(), w.double(), torch.where(y >= 0, g, 0.0).double()
    # every row's statistics in fp64, some thousand rows at a time
    exact = torch.cat([torch.logsumexp(x8[a:a + 1024] @ w8.t(), -1) for a in range(0, rows, 1024)])
    target = (x8 * w8[y.clamp(min=0)]).sum(-1)
    assert (lse - exact).abs().max().item() <= 1e-4
    assert (loss - torch.where(y >= 0, exact - target, 0.0)).abs().max().item() <= 1e-4
    some = torch.tensor([0, 1, 17, 127, 128, rows // 2, rows - 2, rows - 1], device="cuda")
    dz = torch.exp(x8[some] @ w8.t() - exact[some, None])
    dz[torch.arange(some.numel()), y[some].clamp(min=0)] -= 1.0
    want = (dz * g8[some, None]) @ w8
    assert (dx[some].double() - want).norm().item() <= 2.0 ** -8 * want.norm().item()
    assert (dx[y < 0] == 0).all().item()
    words = torch.unique(torch.cat([y[-40:].clamp(min=0), torch.tensor([0, 1, 255, 256, vocab - 2, vocab - 1], device="cuda")]))
    dz = torch.exp(x8 @ w8[words].t() - exact[:, None]) - (y[:, None] == words[None, :]).double()
    want = (dz * g8[:, None]).t() @ x8
    assert (dw[words].double() - want).norm().item() <= 2.0 ** -8 * want.norm().item()
