"""Attention with masked and shaped scores, forward and backward, against the fp64 oracle, element by element.

Tolerances.  A score is an fp32 sum of D products (cut off or rounded by 2^-23 of the running sum each, at most) and, capped, a tanh of
an absolute error of a few 2^-23: with m the largest sum of magnitudes scale |q||k| of a head, dz = (D / 8 + 4) 2^-23 m + 2^-21 cap
+ 2^-20 (1 + the largest bias met with a weight, which fp32 holds to 2^-24).  exp(dz) - 1 < 2 dz here.
  O    P rounded to bf16 (2^-8 of each term), normaliser and exponentials (2 dz each), the result rounded (2^-8)
  LSE  dz, and the logarithm's and the sums' own 2^-20 (1 + |LSE|)
  dV   as O, with its own magnitudes
  dQ   dS rounded to bf16 (2^-8 of each term), its P (2 dz), an absolute error of dO.v - dO.O of 2^-16 of the sums of magnitudes of
       D products in every row's share, the result rounded (2^-8), the sum of fp32 terms in any order 2^-18 of the magnitudes
  dK   as dQ; in rows of up to eight keys Delta is summed from P that are 2 dz off themselves, which adds as much of the sum of magnitudes
and 1e-30 besides, which nothing of these magnitudes is told from zero by (a saturated cap has a derivative of zero in fp64 and 2^-118 in
fp32).  The cap's derivative 1 - tanh^2(s / c) is good to 2^-20 of itself at the score it is given (four roundings and two approximations of
2^-22), within dQ's 2^-18; its logarithm changes by at most 2 / c for each unit of the score, so the score's own error ds (dz without
the cap's part) moves it by up to exp(2 ds / c) - 1 of itself, which is what counts for a cap of 1e-4."""
import numpy as np
import pytest
import torch

import oracle
from helpers import make_plan
from paper_2609_03151_b200 import synth

pytestmark = pytest.mark.gpu

W = lambda **kw: synth.Workload("m", **kw)
SHAPES = {
    "one token": W(N=1, B=1, S=1, Hq=1, Hkv=1, D=128),
    "two tokens d16": W(N=2, B=1, S=2, Hq=2, Hkv=2, D=16),
    "a tile less one": W(N=1, B=2, S=127, Hq=2, Hkv=1, D=64, G=1),
    "a tile": W(N=2, B=1, S=128, Hq=4, Hkv=2, D=128),
    "a tile and one": W(N=1, B=1, S=129, Hq=3, Hkv=3, D=48),
    "five tiles d80": W(N=4, B=2, S=515, Hq=8, Hkv=4, D=80),
    "seven tiles": W(N=2, B=2, S=800, Hq=4, Hkv=2, D=128),
    "seven tiles d64": W(N=4, B=4, S=801, Hq=4, Hkv=2, D=64, G=2),
    "replicated kv": W(N=4, B=1, S=300, Hq=8, Hkv=2, D=96),
    "many ranks": W(N=16, B=4, S=260, Hq=8, Hkv=4, D=32),
}
KINDS = ["causal", "plan without a mask", "docs", "prefix", "window", "ranges", "all", "nothing"]
SHAPING = {"plain": (0.0, False), "cap": (30.0, False), "tight cap": (1.5, False), "wide cap": (200.0, False), "bias": (0.0, True),
           "cap bias": (20.0, True), "wide cap bias": (120.0, True), "tiny cap": (1e-4, False), "huge cap": (1e6, False)}


def documents(rng, B, S, pad):
    """Positions of packed documents, and for every token its document's length."""
    pos, length = np.full((B, S), -1, dtype=np.int32), np.ones((B, S), dtype=np.int32)
    for b in range(B):
        at, stop = 0, S - pad
        while at < stop:
            n = min(stop - at, int(rng.choice([1, 2, 17, 64, 128, 130, 300])))
            pos[b, at:at + n] = np.arange(n)
            length[b, at:at + n] = n
            at += n
    return pos, length


def mask_of(basp, pl, kind, rng):
    """(mask object or None, begin, end [B, S])"""
    B, S = pl.cfg.micro_batch, pl.S
    at = np.tile(np.arange(S), (B, 1))
    if kind == "causal":
        return None, 0 * at, at + 1
    if kind == "plan without a mask":
        return None, 0 * at, 0 * at + S
    mask = torch.full((basp.basp_mask_bytes(pl) + 32,), 255, dtype=torch.uint8, device="cuda")
    cu = lambda a: torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()
    if kind in ("docs", "prefix", "window"):
        pos, length = documents(rng, B, S, S // 9)
        prefix = np.minimum(length, rng.integers(0, 200)) if kind == "prefix" else None
        window = int(rng.integers(1, 200)) if kind == "window" else 0
        basp.basp_mask_packed(pl, cu(pos), mask, None if prefix is None else cu(prefix), window)
        begin, end = oracle.packed_ranges(pos, prefix, window)
    else:
        if kind == "ranges":                 # anything: empty, past the ends, backwards
            begin, end = rng.integers(-20, S + 20, (B, S)), rng.integers(-20, S + 20, (B, S))
            whole = rng.random((B, S)) < 0.2
            begin, end = np.where(whole, -5, begin), np.where(whole, S + 9, end)
        elif kind == "all":
            begin, end = 0 * at, 0 * at + S
        else:
            begin, end = at + 1, at
        basp.basp_mask_ranges(pl, cu(begin), cu(end), mask)
    return mask, np.clip(begin, 0, S), np.clip(end, 0, S)


def head_shards(x, pl, heads, rep):
    """[B, S, H, D] as the ranks' head shards; rep: ranks that share a head."""
    per = max(1, x.shape[2] // pl.K)
    out = []
    for r in range(pl.N):
        g, l = r // pl.K, r % pl.K
        first = l // rep if rep > 1 else l * per
        out.append(x[g * pl.Bl:(g + 1) * pl.Bl, :, first:first + per].contiguous().cuda())
    return out


def f64(t):
    return t.float().cpu().numpy().astype(np.float64)


def run(basp, w, kind, shaping, seed=0, backward=True, spread=1.0):
    rng = np.random.default_rng(seed + w.S)
    cap, bias = SHAPING[shaping]
    pl = make_plan(basp, w, causal=kind not in ("all", "plan without a mask"))
    g = torch.Generator().manual_seed(seed)
    mk = lambda h: (spread * torch.randn((w.B, w.S, h, w.D), generator=g) * torch.exp(0.3 * torch.randn((h, 1), generator=g))).to(torch.bfloat16)
    q, k, v, do = mk(w.Hq), mk(w.Hkv), mk(w.Hkv), mk(w.Hq)
    rep = max(1, pl.K // w.Hkv)
    dq, dk, dv, ddo = (head_shards(t, pl, t.shape[2], rep if t.shape[2] == w.Hkv and w.Hkv < pl.K else 1) for t in (q, k, v, do))
    mask, begin, end = mask_of(basp, pl, kind, rng)
    slopes = (2.0 ** (-8.0 * (torch.arange(w.Hq) + 1.0) / w.Hq)) if bias else None
    if bias and w.Hq > 1:
        slopes[0], slopes[-1] = 2.0, 0.0
    score = basp.basp_score(cap, None if slopes is None else slopes.cuda(), mask)
    o = [torch.full_like(t, float("nan")) for t in dq]
    lse = [torch.full((pl.Bl, pl.Hq_l, pl.S), float("nan"), device="cuda") for _ in range(pl.N)]
    basp.basp_clear_status()
    basp.basp_attn_masked_fwd(pl, score, dq, dk, dv, o, lse)
    basp.basp_get_status()
    grads = None
    ref = [[None] * w.B for _ in range(2)]
    refs = [oracle.attn_shaped(f64(q[b]), f64(k[b]), f64(v[b]), begin[b], end[b], cap, None if slopes is None else slopes.double().numpy())
            for b in range(w.B)]
    # the backward pass by itself: at the oracle's O and LSE (the O of rows of up to eight keys is not used: Delta is the sum of P dO.v there,
    # which is dO.O of the unrounded O)
    if backward:
        O = torch.from_numpy(np.stack([r["o"] for r in refs])).to(torch.bfloat16)
        short = (end - begin <= 8)[..., None, None]
        L = torch.from_numpy(np.stack([r["lse"] for r in refs])).float()
        o_in = head_shards(O, pl, w.Hq, 1)
        l_in = [L[r // pl.K * pl.Bl:(r // pl.K + 1) * pl.Bl, r % pl.K * pl.Hq_l:(r % pl.K + 1) * pl.Hq_l].contiguous().cuda() for r in range(pl.N)]
        grads = [[torch.full_like(t, float("nan")) for t in x] for x in (dq, dk, dv)]
        ws = torch.full((basp.basp_attn_masked_bwd_workspace_bytes(pl),), 255, dtype=torch.uint8, device="cuda")
        basp.basp_attn_masked_bwd(pl, score, dq, dk, dv, o_in, ddo, l_in, *grads, ws)
        basp.basp_get_status()
        refs = [{**r, **{n: t for n, t in oracle.attn_shaped(f64(q[b]), f64(k[b]), f64(v[b]), begin[b], end[b], cap,
                                                              None if slopes is None else slopes.double().numpy(), do=f64(do[b]),
                                                              given=(np.where(short[b], r["o"], f64(O[b])), L[b].double().numpy())).items() if n not in ("o", "lse", "mag_o")}}
                for b, r in enumerate(refs)]
    return pl, refs, o, lse, grads, (cap, 0.0 if slopes is None else float(slopes.max()), (q, k, v, do))


def close(got, want, bound, what):
    bad = ~(np.abs(got - want) <= bound)
    assert not bad.any(), (what, int(bad.sum()), float(np.nanmax(np.abs(got - want) / bound)), bool(np.isnan(got).any()))


def check(w, pl, refs, o, lse, grads, info):
    cap, steepest, (q, k, v, do) = info
    H = w.Hq
    for r in range(pl.N):
        g, l = r // pl.K, r % pl.K
        hq = slice(l * pl.Hq_l, (l + 1) * pl.Hq_l)
        for bl in range(pl.Bl):
            ref = refs[g * pl.Bl + bl]
            # a key whose weight is above e^-20 lies within that much bias (beyond the cap) of the nearest
            dz = (w.D / 8 + 4) * 2.0 ** -23 * ref["top"] + 2.0 ** -21 * min(cap, ref["top"]) + 2.0 ** -20 * (1 + (20 + 2 * ref["top"]) * (steepest > 0) / 16)
            want = ref["lse"][hq]
            got = lse[r][bl].double().cpu().numpy()
            none = np.isneginf(want)
            assert np.array_equal(np.isneginf(got), none)
            far = w.S * steepest * 2.0 ** -23 if steepest else 0.0          # a row that sees far keys alone has its bias in the LSE
            close(got[~none], want[~none], dz + far + 2.0 ** -20 * (1 + np.abs(want[~none])), (r, bl, "lse"))
            p = 2 * dz + far
            close(f64(o[r][bl]), ref["o"][:, hq], (2.0 ** -8 + 2 * p) * ref["mag_o"][:, hq] + 2.0 ** -8 * np.abs(ref["o"][:, hq]), (r, bl, "o"))
            if grads is None:
                continue
            b = g * pl.Bl + bl
            G = H // w.Hkv
            bend = np.expm1(2 * (w.D / 8 + 4) * 2.0 ** -23 * ref["top"] / cap) if cap else 0.0
            dots = (2.0 ** -16 + p) * np.einsum("shd,shd->s", np.abs(f64(do[b])), np.abs(f64(v[b])).repeat(G, 1).max(0)[None] + np.abs(ref["o"])).max()
            unit = lambda n: (2.0 ** -8 + 2 * p + 2.0 ** -18 + bend) * ref["mag_" + n] + dots * ref["row_" + n] + 2.0 ** -8 * np.abs(ref[n]) + 1e-30
            close(f64(grads[0][r][bl]), ref["dq"][:, hq], unit("dq")[:, hq], (r, bl, "dq"))
            # a rank with a shared KV head holds its own query heads' part: summed over the sharing ranks
            if w.Hkv < pl.K:
                rep = pl.K // w.Hkv
                if l % rep:
                    continue
                dk, dv = (sum(f64(x[r + i][bl]) for i in range(rep)) for x in grads[1:])
                hk, extra = slice(l // rep, l // rep + 1), rep
            else:
                dk, dv = (f64(x[r][bl]) for x in grads[1:])
                hk, extra = slice(l * pl.Hkv_l, (l + 1) * pl.Hkv_l), 1
            bound_dv = (2.0 ** -8 + 2 * p) * ref["mag_dv"] + 2.0 ** -8 * (np.abs(ref["dv"]) if extra == 1 else ref["mag_dv"])
            close(dv, ref["dv"][:, hk], bound_dv[:, hk], (r, bl, "dv"))
            close(dk, ref["dk"][:, hk], (unit("dk") + (extra > 1) * 2.0 ** -8 * ref["mag_dk"])[:, hk], (r, bl, "dk"))


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("shape", ["one token", "a tile less one", "a tile and one", "five tiles d80", "seven tiles d64"])
def test_masks(basp, shape, kind):
    w = SHAPES[shape]
    check(w, *run(basp, w, kind, "plain", 1))


@pytest.mark.parametrize("shaping", [s for s in SHAPING if s != "plain"])
@pytest.mark.parametrize("kind,shape", [("causal", "seven tiles"), ("docs", "seven tiles d64"), ("ranges", "five tiles d80"), ("all", "a tile and one"),
                                        ("prefix", "seven tiles")])
def test_shapings(basp, kind, shape, shaping):
    w = SHAPES[shape]
    check(w, *run(basp, w, kind, shaping, 2))


@pytest.mark.parametrize("shape", ["two tokens d16", "a tile", "replicated kv", "many ranks"])
def test_plans(basp, shape):
    w = SHAPES[shape]
    check(w, *run(basp, w, "docs", "cap bias", 3))
    check(w, *run(basp, w, "causal", "plain", 4))


def test_large_scores(basp):
    """Scores of hundreds: the softmax is one key almost everywhere, the cap is reached almost everywhere."""
    w = SHAPES["five tiles d80"]
    for shaping in ("plain", "cap", "cap bias"):
        check(w, *run(basp, w, "docs", shaping, 5, backward=False, spread=6.0))


def test_many_tiles_against_the_causal_kernel(basp):
    """Sixty tiles, one document: the causal kernel's results within both kernels' roundings, and the mask's order over launches of
    three steps."""
    pl = basp.basp_plan_create(2, 1, 7600, 8, 4, 128)
    g = torch.Generator(device="cuda").manual_seed(1)
    mk = lambda h: [torch.randn((1, 7600, h // 2, 128), generator=g, device="cuda").to(torch.bfloat16) for _ in range(2)]
    q, k, v, do = mk(8), mk(4), mk(4), mk(8)
    mask = torch.empty(basp.basp_mask_bytes(pl), dtype=torch.uint8, device="cuda")
    basp.basp_mask_packed(pl, torch.arange(7600, dtype=torch.int32, device="cuda")[None].contiguous(), mask)
    basp.basp_clear_status()
    res = []
    for score in (None, basp.basp_score(mask=mask), basp.basp_score()):
        o, lse = [torch.full_like(t, float("nan")) for t in q], [torch.empty((1, 4, 7600), device="cuda") for _ in range(2)]
        grads = [[torch.full_like(t, float("nan")) for t in x] for x in (q, k, v)]
        size = basp.basp_attn_bwd_workspace_bytes if score is None else basp.basp_attn_masked_bwd_workspace_bytes
        ws = torch.empty(size(pl), dtype=torch.uint8, device="cuda")
        if score is None:
            basp.basp_attn_fwd(pl, q, k, v, o, lse)
            basp.basp_attn_bwd(pl, q, k, v, o, do, lse, *grads, ws)
        else:
            basp.basp_attn_masked_fwd(pl, score, q, k, v, o, lse)
            basp.basp_attn_masked_bwd(pl, score, q, k, v, o, do, lse, *grads, ws)
        res.append([torch.cat([t.double().flatten() for t in x]) for x in (o, lse, *grads)])
    basp.basp_get_status()
    for other in res[1:]:
        for a, b, n in zip(res[0], other, ("o", "lse", "dq", "dk", "dv")):
            assert ((a - b).norm() / a.norm()).item() <= (1e-6 if n == "lse" else 2.0 ** -8), n     # two roundings of 2^-9 rms each at most


def test_rows_behind_the_last_document(basp):
    """Padding: its rows come out as zeros and -inf, its keys get zeros, and a neighbour's memory behind the shard stays."""
    pl = basp.basp_plan_create(1, 1, 300, 2, 1, 64)
    g = torch.Generator(device="cuda").manual_seed(2)
    mk = lambda h: torch.randn((1, 300, h, 64), generator=g, device="cuda").to(torch.bfloat16)
    q, k, v, do = mk(2), mk(1), mk(1), mk(2)
    pos = torch.cat([torch.arange(70), torch.arange(90), torch.full((140,), -1)]).int()[None].cuda()
    mask = torch.empty(basp.basp_mask_bytes(pl), dtype=torch.uint8, device="cuda")
    basp.basp_mask_packed(pl, pos, mask)
    room = torch.full((5, 320 * 2 * 64), 7.0, dtype=torch.bfloat16, device="cuda")
    o, dq, dk, dv = (room[i, :300 * h * 64].view(1, 300, h, 64) for i, h in enumerate((2, 2, 1, 1)))
    lse = torch.full((2 * 300 + 20,), 7.0, device="cuda")
    score = basp.basp_score(mask=mask)
    ws = torch.empty(basp.basp_attn_masked_bwd_workspace_bytes(pl), dtype=torch.uint8, device="cuda")
    basp.basp_clear_status()
    basp.basp_attn_masked_fwd(pl, score, [q], [k], [v], [o], [lse[:600].view(1, 2, 300)])
    basp.basp_attn_masked_bwd(pl, score, [q], [k], [v], [o], [do], [lse[:600].view(1, 2, 300)], [dq], [dk], [dv], ws)
    basp.basp_get_status()
    assert all((t[0, 160:] == 0).all() for t in (o, dq, dk, dv)) and torch.isneginf(lse[:600].view(2, 300)[:, 160:]).all()
    assert all((room[i, 300 * h * 64:] == 7).all() for i, h in enumerate((2, 2, 1, 1))) and (lse[600:] == 7).all()
    assert all(torch.isfinite(t.float()).all() and (t[0, :160].float().abs().sum((1, 2)) > 0).sum() >= 155 for t in (o, dk, dv))


def test_past_two_billion_elements(basp):
    """A shard of more than 2^31 elements: the last document's rows against the same document alone."""
    S, H, D = 66000, 260, 128
    pl = basp.basp_plan_create(1, 1, S, H, 1, D)
    assert S * H * D > 2 ** 31
    g = torch.Generator(device="cuda").manual_seed(3)
    q = torch.zeros((1, S, H, D), dtype=torch.bfloat16, device="cuda")
    n = 200
    q[0, -n:] = torch.randn((n, H, D), generator=g, device="cuda").to(torch.bfloat16)
    k, v = (torch.randn((1, S, 1, D), generator=g, device="cuda").to(torch.bfloat16) for _ in range(2))
    pos = torch.arange(S, dtype=torch.int32, device="cuda") % 128
    pos[-n:] = torch.arange(n, device="cuda")
    mask = torch.empty(basp.basp_mask_bytes(pl), dtype=torch.uint8, device="cuda")
    basp.basp_mask_packed(pl, pos[None].contiguous(), mask)
    o, lse = torch.empty_like(q), torch.empty((1, H, S), device="cuda")
    basp.basp_clear_status()
    basp.basp_attn_masked_fwd(pl, basp.basp_score(mask=mask), [q], [k], [v], [o], [lse])
    basp.basp_get_status()
    small = basp.basp_plan_create(1, 1, n, H, 1, D)
    o2, lse2 = torch.empty((1, n, H, D), dtype=torch.bfloat16, device="cuda"), torch.empty((1, H, n), device="cuda")
    basp.basp_attn_masked_fwd(small, basp.basp_score(), [q[:, -n:].contiguous()], [k[:, -n:].contiguous()], [v[:, -n:].contiguous()], [o2], [lse2])
    # the same keys in other tiles: P's rounding (2^-8 of terms of up to |v|) and the result's
    assert (o[:, -n:].float() - o2.float()).abs().max().item() <= 2.0 ** -7 * v[:, -n:].float().abs().max().item()
    assert (lse[..., -n:] - lse2).abs().max().item() <= 1e-5
    assert torch.allclose(lse[0, :, 5], torch.log(torch.tensor(6.0)).cuda().expand(H), atol=1e-5)      # zero queries: a mean over the keys


@pytest.mark.parametrize("shaping", ["plain", "cap", "wide cap", "bias", "cap bias"])
@pytest.mark.parametrize("D", [64, 128])
def test_queries_that_see_one_key(basp, D, shaping):
    """P is 1 there whatever the score: O is the key's value and no gradient reaches Q and K, to the bit; dV is dO, rounded once."""
    S, H = 300, 2
    cap, bias = SHAPING[shaping]
    pl = make_plan(basp, W(N=1, B=1, S=S, Hq=H, Hkv=H, D=D))
    g = torch.Generator().manual_seed(D)
    q, k, v, do = ([torch.randn((1, S, H, D), generator=g).to(torch.bfloat16).cuda()] for _ in range(4))
    mask = torch.empty(basp.basp_mask_bytes(pl), dtype=torch.uint8, device="cuda")
    slopes = torch.tensor([0.5, 0.01], device="cuda") if bias else None
    o, dq, dk, dv = ([torch.full_like(t[0], float("nan"))] for t in (q, q, k, v))
    lse = [torch.empty((1, H, S), device="cuda")]
    ws = torch.empty(basp.basp_attn_masked_bwd_workspace_bytes(pl), dtype=torch.uint8, device="cuda")
    one = torch.arange(S, dtype=torch.int32)
    # documents of one token; a window of one; a first row of its own and whole documents behind it
    for pos, window in ((0 * one, 0), (one, 1), (one % 150, 0)):
        basp.basp_mask_packed(pl, pos.reshape(1, S).cuda(), mask, None, window)
        sc = basp.basp_score(softcap=cap, slopes=slopes, mask=mask)
        basp.basp_attn_masked_fwd(pl, sc, q, k, v, o, lse)
        basp.basp_attn_masked_bwd(pl, sc, q, k, v, o, do, lse, dq, dk, dv, ws)
        alone = torch.ones(S, dtype=torch.bool) if window or not pos.any() else pos == 0
        assert torch.equal(o[0][0, alone], v[0][0, alone])
        assert (dq[0][0, alone] == 0).all()
        if alone.all():
            assert (dk[0] == 0).all() and torch.equal(dv[0], do[0])
    assert basp.basp_get_status() == [0, 0, 0, 0]


@pytest.mark.parametrize("kind", ["two tokens", "window", "documents"])
@pytest.mark.parametrize("D", [16, 64, 128])
def test_gradients_of_rows_with_few_keys(basp, D, kind):
    """Forward and backward in a row, where dO.v - Delta is small against the roundings of O: the result's 2-norm is off by the roundings of
    dS and of the result, 2^-9 rms each at most, and by those of P (2^-9 of each term of Delta) in no row."""
    S, H = (2 if kind == "two tokens" else 300), 8
    pl = make_plan(basp, W(N=1, B=1, S=S, Hq=H, Hkv=H, D=D))
    g = torch.Generator().manual_seed(D)
    q, k, v, do = ([torch.randn((1, S, H, D), generator=g).to(torch.bfloat16).cuda()] for _ in range(4))
    pos = np.arange(S, dtype=np.int32)[None] % (5 if kind == "documents" else S)
    window = 3 if kind == "window" else 0
    mask = torch.empty(basp.basp_mask_bytes(pl), dtype=torch.uint8, device="cuda")
    basp.basp_mask_packed(pl, torch.from_numpy(pos).cuda(), mask, None, window)
    begin, end = oracle.packed_ranges(pos, None, window)
    for cap, slopes in ((0.0, None), (20.0, torch.linspace(0.01, 0.5, H))):
        sc = basp.basp_score(softcap=cap, slopes=None if slopes is None else slopes.cuda(), mask=mask)
        o, dq, dk, dv = ([torch.full_like(t[0], float("nan"))] for t in (q, q, k, v))
        lse = [torch.empty((1, H, S), device="cuda")]
        ws = torch.empty(basp.basp_attn_masked_bwd_workspace_bytes(pl), dtype=torch.uint8, device="cuda")
        basp.basp_attn_masked_fwd(pl, sc, q, k, v, o, lse)
        basp.basp_attn_masked_bwd(pl, sc, q, k, v, o, do, lse, dq, dk, dv, ws)
        ref = oracle.attn_shaped(*(f64(t[0][0]) for t in (q, k, v)), begin[0], end[0], cap, None if slopes is None else slopes.double().numpy(),
                                 do=f64(do[0][0]))
        for got, n in ((dq, "dq"), (dk, "dk")):
            assert np.linalg.norm(f64(got[0][0]) - ref[n]) <= 2.0 ** -8 * np.linalg.norm(ref[n]), (cap, n)


@pytest.mark.parametrize("S", [300, 8400])
def test_a_mask_rewritten_between_calls(basp, S):
    """One mask buffer filled for one batch after another, each read by the calls right behind it (which start under the mask's own launches: one
    block up to 64 tiles, three launches above): the results with a wait after every call."""
    pl = make_plan(basp, W(N=1, B=1, S=S, Hq=2, Hkv=1, D=64))
    g = torch.Generator(device="cuda").manual_seed(S)
    q, k, v = ([torch.randn((1, S, h, 64), generator=g, device="cuda").to(torch.bfloat16)] for h in (2, 1, 1))
    at = torch.arange(S, dtype=torch.int32, device="cuda")[None]
    batches = [(at % n).contiguous() for n in (S, 1, 130, 64, 257, 7)]
    mask = torch.zeros(basp.basp_mask_bytes(pl), dtype=torch.uint8, device="cuda")
    scores = [basp.basp_score(mask=mask), basp.basp_score(softcap=20.0, mask=mask)]
    fresh = lambda: [[([torch.empty_like(q[0])], [torch.empty((1, 2, S), device="cuda")]) for _ in scores] for _ in batches]

    def calls(pos, out, pause):
        basp.basp_mask_packed(pl, pos, mask)
        pause()
        for score, (o, lse) in zip(scores, out):
            basp.basp_attn_masked_fwd(pl, score, q, k, v, o, lse)
            pause()

    basp.basp_clear_status()
    want, got = fresh(), [fresh() for _ in range(8)]
    for pos, out in zip(batches, want):
        calls(pos, out, torch.cuda.synchronize)
    for turn in got:
        for pos, out in zip(batches, turn):
            calls(pos, out, lambda: None)
    basp.basp_get_status()
    for turn in got:
        for a, b in zip(want, turn):
            assert all(torch.equal(x[0], y[0]) for m, n in zip(a, b) for x, y in zip(m, n))


@pytest.mark.parametrize("shaping", ["cap", "cap bias", "wide cap"])
@pytest.mark.parametrize("D", [64, 128])
def test_capped_scores_beyond_fp32(basp, D, shaping):
    """Products of 1e60 are infinite as raw scores; capped they are the cap, with its sign, and keys at -cap keep the weight that the formula
    gives them: all of it where a row sees no others.  Tolerances as above, with the sums of magnitudes of the other features (where the
    first one is not zero it decides the score alone); dV takes the forward's LSE, so its P has that error too."""
    S, H = 300, 2
    cap, bias = SHAPING[shaping]
    pl = make_plan(basp, W(N=1, B=1, S=S, Hq=H, Hkv=H, D=D))
    g = torch.Generator().manual_seed(D)
    q, k, v, do = (torch.randn((1, S, H, D), generator=g) for _ in range(4))
    q[..., 0], k[..., 0] = 0.0, 0.0
    ordinary = float((q.abs().amax(1) * k.abs().amax(1)).sum(-1).max()) / D ** 0.5       # no sum of magnitudes without the first feature is larger
    q[0, ::2, :, 0] = 1e30
    kind = torch.arange(S) % 7
    kind[:5] = 0
    kind[128:256] = 0                                     # tile borders among keys at -cap, and a whole tile of them
    k[0, kind == 0, :, 0], k[0, kind == 1, :, 0] = -1e30, 1e30
    q, k, v, do = ([t.to(torch.bfloat16).cuda()] for t in (q, k, v, do))
    slopes = torch.tensor([0.01, 0.1]) if bias else None
    o, lse = [torch.full_like(q[0], float("nan"))], [torch.full((1, H, S), float("nan"), device="cuda")]
    grads = [[torch.full_like(t[0], float("nan"))] for t in (q, k, v)]
    mask = torch.empty(basp.basp_mask_bytes(pl), dtype=torch.uint8, device="cuda")
    ws = torch.empty(basp.basp_attn_masked_bwd_workspace_bytes(pl), dtype=torch.uint8, device="cuda")
    # causal rows; windows of four keys, which in the whole tile are all at -cap; documents of 60
    for pos, window in ((torch.arange(S), 0), (torch.arange(S), 4), (torch.arange(S) % 60, 0)):
        basp.basp_mask_packed(pl, pos.int()[None].cuda(), mask, None, window)
        begin, end = oracle.packed_ranges(pos[None].numpy(), None, window)
        sc = basp.basp_score(cap, None if slopes is None else slopes.cuda(), mask)
        basp.basp_clear_status()
        basp.basp_attn_masked_fwd(pl, sc, q, k, v, o, lse)
        basp.basp_attn_masked_bwd(pl, sc, q, k, v, o, do, lse, *grads, ws)
        basp.basp_get_status()
        ref = oracle.attn_shaped(*(f64(t[0][0]) for t in (q, k, v)), begin[0], end[0], cap, None if slopes is None else slopes.double().numpy(),
                                 do=f64(do[0][0]))
        dz = (D / 8 + 4) * 2.0 ** -23 * ordinary + 2.0 ** -21 * cap + (2.0 ** -22 * 0.1 * S if bias else 0.0)
        close(lse[0][0].double().cpu().numpy(), ref["lse"], dz + 2.0 ** -20 * (1 + np.abs(ref["lse"])), "lse")
        close(f64(o[0][0]), ref["o"], (2.0 ** -8 + 4 * dz) * ref["mag_o"] + 2.0 ** -8 * np.abs(ref["o"]), "o")
        close(f64(grads[2][0][0]), ref["dv"], (2.0 ** -8 + 8 * dz + 2.0 ** -19 * cap) * ref["mag_dv"] + 2.0 ** -8 * np.abs(ref["dv"]), "dv")
        assert all(torch.isfinite(t[0].float()).all() for t in grads)
