"""8-bit checkpoints of Q, K, V and O: the codes, scales and values brought back bit for bit against the definition's fp32
arithmetic, the exchange against the oracle's, and the layer's backward from checkpoints against the fp64 formula at the
values brought back."""
import numpy as np
import pytest
import torch

import oracle
from helpers import make_plan
from paper_2609_03151_b200 import synth

pytestmark = pytest.mark.gpu

CASES = [
    synth.Workload("one_token", N=1, B=1, S=1, Hq=1, Hkv=1, D=128),
    synth.Workload("d16", N=2, B=2, S=70, Hq=4, Hkv=2, D=16),
    synth.Workload("d32", N=2, B=1, S=131, Hq=6, Hkv=2, D=32),
    synth.Workload("d48", N=1, B=3, S=45, Hq=5, Hkv=5, D=48),
    synth.Workload("d64_two_seqs", N=4, B=4, S=100, Hq=8, Hkv=4, D=64, G=2),
    synth.Workload("d80", N=4, B=2, S=203, Hq=20, Hkv=4, D=80),
    synth.Workload("d96_uneven_two_seqs", N=4, B=2, S=77, Hq=8, Hkv=4, D=96, G=1),
    synth.Workload("d112", N=2, B=2, S=65, Hq=7, Hkv=7, D=112),
    synth.Workload("d128_uneven", N=4, B=1, S=1021, Hq=32, Hkv=8, D=128),
    synth.Workload("replicated_kv", N=8, B=1, S=264, Hq=16, Hkv=2, D=128),
    synth.Workload("replicated_uneven", N=4, B=1, S=1022, Hq=8, Hkv=2, D=96),
    synth.Workload("many_ranks", N=32, B=4, S=160, Hq=8, Hkv=8, D=64),
]


def shards(pl, w, seed=0):
    """Q, K, V, O per rank; among them a zero vector, a tiny one, ones with an infinity and a NaN, and an exact half step."""
    g = torch.Generator().manual_seed(seed + w.S)
    out = []
    for i, h in enumerate((w.Hq, w.Hkv, w.Hkv, w.Hq)):
        ts = []
        for r in range(pl.N):
            t = synth.randn_bf16(g, (pl.Bl, pl.rank_tokens(r), h, w.D)).float() * torch.exp(2 * torch.randn((1, 1, h, 1), generator=g))
            t = t.to(torch.bfloat16)
            if t.shape[1] > 8:
                t[0, 0, 0] = 0.0
                t[0, 1, 0] = 1e-36
                t[0, 2, 0, 3] = float("inf")
                t[0, 3, 0, w.D - 1] = float("nan")
                t[0, 4, 0] = 63.5
                t[0, 4, 0, 0] = 127.0                                  # scale 1: 63.5 rounds to the even 64
                t[0, 5, 0] = 3e38
            ts.append(t)
        out.append(ts)
    return out


def parts_of(pl, w, r, buf):
    """Codes and scales of rank r's checkpoint, by the documented layout."""
    raw, at, T = buf.cpu().numpy(), 0, pl.rank_tokens(r)
    up = lambda n: (n + 15) // 16 * 16
    codes, scales = [], []
    for h in (w.Hq, w.Hkv, w.Hkv, w.Hq):
        n = pl.Bl * T * h * w.D
        codes.append(raw[at:at + n].view(np.int8).reshape(pl.Bl, T, h, w.D))
        at += up(n)
    for h in (w.Hq, w.Hkv, w.Hkv, w.Hq):
        n = pl.Bl * T * h * 4
        scales.append(raw[at:at + n].copy().view(np.float32).reshape(pl.Bl, T, h))
        at += up(n)
    assert at == raw.size
    return codes, scales


def to_heads(pl, per_rank):
    """Sequence shards [Bl, T, H, D] to the head shards of all ranks (numpy, any element type)."""
    out = []
    for r in range(pl.N):
        g, m = r // pl.K, r % pl.K
        x = np.concatenate([per_rank[g * pl.K + i] for i in range(pl.K)], axis=1)
        h = x.shape[2]
        out.append(x[:, :, m * h // pl.K:(m + 1) * h // pl.K] if h % pl.K == 0 else x[:, :, m * h // pl.K:m * h // pl.K + 1])
    return out


@pytest.mark.parametrize("aligned", [True, False])
@pytest.mark.parametrize("w", CASES, ids=lambda w: w.name)
def test_codes_and_way_back(basp, w, aligned):
    pl = make_plan(basp, w)
    host = shards(pl, w)

    def place(t):                                          # on a multiple of 32 bytes, or 16 bytes beside one
        big = torch.full((t.numel() + 8,), 7.0, dtype=torch.bfloat16, device="cuda")
        at = big[0 if aligned else 8:][:t.numel()].view(t.shape)
        assert (at.data_ptr() % 32 == 0) == aligned
        return at
    dev = [[place(t).copy_(t) for t in ts] for ts in host]
    ckpt = [torch.full((basp.basp_ckpt_bytes(pl, r) + 16,), 201, dtype=torch.uint8, device="cuda") for r in range(pl.N)]
    views = [c[:-16] for c in ckpt]
    basp.basp_ckpt_pack(pl, *dev, views)
    want = [[], [], [], []]
    for r in range(pl.N):
        codes, scales = parts_of(pl, w, r, views[r])
        for i in range(4):
            c, s = oracle.ckpt_codes(host[i][r].float().numpy())
            assert np.array_equal(scales[i], s, equal_nan=True), (i, r)
            ok = np.isfinite(s)
            assert np.array_equal(codes[i][ok], c[ok]), (i, r)
            want[i].append(torch.from_numpy(oracle.ckpt_values(c, s)).to(torch.bfloat16).float().numpy())
        assert (ckpt[r][-16:] == 201).all()
    heads = [[place(torch.empty((pl.Bl, pl.S, h, w.D), dtype=torch.bfloat16)).fill_(float("nan")) for _ in range(pl.N)]
             for h in (pl.Hq_l, pl.Hkv_l, pl.Hkv_l, pl.Hq_l)]
    basp.basp_ckpt_reshard_s2h(pl, views, *heads)
    for i in range(4):
        for got, ref in zip(heads[i], to_heads(pl, want[i])):
            assert np.array_equal(got.float().cpu().numpy(), ref, equal_nan=True), i


def test_every_code_and_tie(basp):
    """All bf16 magnitudes that share a scale with 127: every code and every half step, both signs."""
    w = synth.Workload("codes", N=1, B=1, S=64, Hq=2, Hkv=2, D=128)
    pl = make_plan(basp, w)
    vals = torch.arange(-127, 127.5, 0.5).to(torch.bfloat16)           # 509 values, the ones bf16 can hold
    x = torch.cat([vals, vals.flip(0)]).repeat(17)[:64 * 2 * 128].view(1, 64, 2, 128).clone()
    x[..., 0] = 127.0
    y = (x.float() * 1.7).to(torch.bfloat16)                           # a scale that is no power of two
    dev = [[t.cuda()] for t in (x, y, x, y)]
    ck = [torch.empty(basp.basp_ckpt_bytes(pl, 0), dtype=torch.uint8, device="cuda")]
    basp.basp_ckpt_pack(pl, *dev, ck)
    codes, scales = parts_of(pl, w, 0, ck[0])
    for t, c, s in zip((x, y, x, y), codes, scales):
        wc, ws = oracle.ckpt_codes(t.float().numpy())
        assert np.array_equal(c, wc) and np.array_equal(s, ws)


def f64(t):
    return t.float().cpu().numpy().astype(np.float64)


@pytest.mark.parametrize("w,autograd", [
    (synth.Workload("b64", N=4, B=2, S=512, Hq=4, Hkv=4, D=64), False),
    (synth.Workload("b128", N=4, B=2, S=512, Hq=8, Hkv=4, D=128), True),
    (synth.Workload("b80_uneven", N=2, B=1, S=301, Hq=4, Hkv=2, D=80), False),
    (synth.Workload("b_replicated", N=4, B=1, S=256, Hq=8, Hkv=2, D=64), False),
], ids=lambda x: getattr(x, "name", str(x)))
def test_layer_backward_from_checkpoints(basp, w, autograd):
    """Gradients against the fp64 formula at the values brought back, with the forward's log-sum-exp.  Tolerance as for the
    layer's backward from bf16 shards: 2e-2 absolute and the rounding of the result.  Where a group has more ranks than KV
    heads, dK and dV are sums of copies that each rank first rounds to bf16: |round(a) + round(b) - (a + b)| <= 2^-8 (|a| + |b|)
    comes on top (the sum's own rounding is the 2^-8 of the result)."""
    from paper_2609_03151_b200.autograd import basp_attention
    pl = make_plan(basp, w)
    op = oracle.plan_uneven(w.N, w.B, w.S, w.G)
    ts = synth.make_qkv(w, 4, with_dO=True)
    split = lambda t: [synth.from_bits(np.ascontiguousarray(a)).cuda() for a in oracle.partition_uneven(synth.bits(t), op)]
    q, k, v, do = (split(t) for t in ts)
    o = [torch.empty_like(t) for t in q]
    lse = [torch.empty((pl.Bl, pl.Hq_l, pl.S), dtype=torch.float32, device="cuda") for _ in range(w.N)]
    basp.basp_clear_status()
    space = torch.empty(basp.basp_workspace_bytes(pl), dtype=torch.uint8, device="cuda")
    basp.basp_layer_fwd(pl, q, k, v, o, space, lse_shards=lse)
    ck = [torch.empty(basp.basp_ckpt_bytes(pl, r), dtype=torch.uint8, device="cuda") for r in range(w.N)]
    basp.basp_ckpt_pack(pl, q, k, v, o, ck)
    grads = [[torch.full_like(t, float("nan")) for t in x] for x in (q, k, v)]
    space = torch.empty(basp.basp_layer_bwd_seq_workspace_bytes(pl), dtype=torch.uint8, device="cuda")
    basp.basp_layer_bwd_ckpt(pl, ck, lse, do, *grads, space)
    basp.basp_get_status()
    if autograd:
        leaves = [[t.clone().requires_grad_() for t in x] for x in (q, k, v)]
        out = basp_attention(pl, *leaves, fused=True, checkpoint8=True)
        torch.autograd.backward(out, do)
        basp.basp_get_status()
        grads = [[t.grad for t in x] for x in leaves]
        with pytest.raises(ValueError, match="fused"):
            basp_attention(pl, *leaves, checkpoint8=True)
    # the values brought back, head-sharded, through the oracle's own arithmetic
    kept = []
    for x in (q, k, v, o):
        back = [oracle.ckpt_values(*oracle.ckpt_codes(t.float().cpu().numpy())) for t in x]
        kept.append([torch.from_numpy(b).to(torch.bfloat16).float().numpy().astype(np.float64) for b in to_heads(pl, back)])
    doh = to_heads(pl, [f64(t) for t in do])
    zeros = lambda: [[np.zeros((pl.Bl, pl.rank_tokens(r), h, w.D)) for r in range(w.N)] for h in (w.Hq, w.Hkv, w.Hkv)]
    want, copies = zeros(), zeros()
    for r in range(w.N):
        for b in range(pl.Bl):
            g = oracle.attn_bwd_given(*(kept[i][r][b] for i in range(4)), f64(lse[r][b]), doh[r][b])
            info = basp.basp_plan_get_rank(pl, r)
            for i, (n, lo, hi) in enumerate((("dQ", "q_head_begin", "q_head_end"), ("dK", "kv_head_begin", "kv_head_end"),
                                             ("dV", "kv_head_begin", "kv_head_end"))):
                for l in range(pl.K):
                    dst, T = r // pl.K * pl.K + l, pl.rank_tokens(l)
                    want[i][dst][b][:, info[lo]:info[hi]] += g[n][l * pl.T:l * pl.T + T]
                    if i > 0 and pl.K > w.Hkv:
                        copies[i][dst][b][:, info[lo]:info[hi]] += np.abs(g[n][l * pl.T:l * pl.T + T])
    for name, got, ref, several in zip(("dq", "dk", "dv"), grads, want, copies):
        for a, b, c in zip(got, ref, several):
            err = np.abs(f64(a).reshape(b.shape) - b)
            assert (err <= 2e-2 + 2.0 ** -8 * (np.abs(b) + c)).all(), (w.name, name, float(err.max()))


@pytest.mark.parametrize("mode", ["no_grad", "inference_mode", "no leaf"])
def test_an_evaluation_packs_no_checkpoints(basp, mode):
    """Where no backward will come, the layer with checkpoint8 is the fused forward alone."""
    from contextlib import nullcontext

    from paper_2609_03151_b200.autograd import basp_attention
    w = synth.Workload("eval", N=4, B=2, S=512, Hq=4, Hkv=2, D=64)
    pl = make_plan(basp, w)
    g = torch.Generator(device="cuda").manual_seed(3)
    q, k, v = ([torch.randn((pl.Bl, pl.T, h, w.D), generator=g, device="cuda").to(torch.bfloat16) for _ in range(4)]
               for h in (w.Hq, w.Hkv, w.Hkv))
    basp.basp_clear_status()
    before = basp.basp_launch_count()
    plain = basp_attention(pl, q, k, v, fused=True)
    alone = basp.basp_launch_count() - before
    if mode != "no leaf":
        q, k, v = ([t.clone().requires_grad_() for t in ts] for ts in (q, k, v))
    with nullcontext() if mode == "no leaf" else getattr(torch, mode)():
        before = basp.basp_launch_count()
        out = basp_attention(pl, q, k, v, fused=True, checkpoint8=True)
    basp.basp_get_status()
    assert basp.basp_launch_count() - before == alone
    assert all(torch.equal(a, b) for a, b in zip(plain, out))


def test_checkpoints_are_saved_tensors(basp):
    """Saved-tensor hooks (offloading between the passes) see the checkpoints and nothing of the shards in bf16; a backward from
    what they give back has the gradients of one without them.  dK and dV bit for bit, dQ comes from a reduction in whatever order its blocks
    finish (fp32, rounded to bf16: neighbours at most)."""
    from paper_2609_03151_b200.autograd import basp_attention
    w = synth.Workload("hooks", N=4, B=2, S=512, Hq=4, Hkv=2, D=64)
    pl = make_plan(basp, w)
    g = torch.Generator(device="cuda").manual_seed(4)
    q, k, v, do = ([torch.randn((pl.Bl, pl.T, h, w.D), generator=g, device="cuda").to(torch.bfloat16) for _ in range(4)]
                   for h in (w.Hq, w.Hkv, w.Hkv, w.Hq))
    seen, grads = [], []

    def away(t):
        seen.append((t.dtype, t.numel()))
        return t.cpu()
    for hooks in (False, True):
        leaves = [[t.clone().requires_grad_() for t in ts] for ts in (q, k, v)]
        basp.basp_clear_status()
        if hooks:
            with torch.autograd.graph.saved_tensors_hooks(away, lambda t: t.cuda()):
                out = basp_attention(pl, *leaves, fused=True, checkpoint8=True)
        else:
            out = basp_attention(pl, *leaves, fused=True, checkpoint8=True)
        torch.autograd.backward(out, do)
        basp.basp_get_status()
        grads.append([[t.grad for t in ts] for ts in leaves])
    assert seen == [(torch.uint8, basp.basp_ckpt_bytes(pl, r)) for r in range(4)]
    for a, b in zip(*(x[0] for x in grads)):
        assert ((a.float() - b.float()).abs() <= 2.0 ** -7 * b.float().abs() + 1e-6).all()
    for i in (1, 2):
        assert all(torch.equal(a, b) for a, b in zip(grads[0][i], grads[1][i]))


def test_what_is_held_between_the_passes(basp):
    """With checkpoints the layer holds them and the log-sum-exp, without them Q, K, V, O and the log-sum-exp in place of them (to the
    allocator's 512 bytes a tensor)."""
    from paper_2609_03151_b200.autograd import basp_attention
    w = synth.Workload("held", N=4, B=2, S=2048, Hq=8, Hkv=4, D=128)
    pl = make_plan(basp, w)
    ones = lambda h: [torch.ones((pl.Bl, pl.T, h, w.D), dtype=torch.bfloat16, device="cuda").requires_grad_() for _ in range(4)]
    leaves = [ones(h) for h in (w.Hq, w.Hkv, w.Hkv)]
    bf16 = 4 * pl.Bl * pl.T * (2 * w.Hq + 2 * w.Hkv) * w.D * 2
    lse = 4 * pl.Bl * pl.Hq_l * pl.S * 4
    want = {False: bf16 + lse, True: sum(basp.basp_ckpt_bytes(pl, r) for r in range(4)) + lse}
    assert want[True] < 0.55 * want[False]
    for ckpt in (False, True):
        before = torch.cuda.memory_allocated()
        x = [[t * 1.0 for t in ts] for ts in leaves]       # activations that nothing else keeps
        out = basp_attention(pl, *x, fused=True, checkpoint8=ckpt)
        loss = sum(t.float().sum() for t in out)           # holds the graph, and nothing of the outputs
        del x, out
        held = torch.cuda.memory_allocated() - before
        assert want[ckpt] <= held <= want[ckpt] + 32 * 512, (ckpt, held, want[ckpt])
        del loss
