"""The forms of the masked attention that a plan's size and a score's numbers choose: the mask object of one launch and of three, the backward that
divides the query heads of a key head evenly, unevenly or not at all, slopes of either sign, wide caps over many tiles; and the layer around it
where ranks share key heads or have different numbers of tokens, and the backward on two streams.  Tolerances: those of
tests/test_gpu_masked_attn.py, the gradients at the kernel's own O and LSE."""
import numpy as np
import pytest
import torch

import oracle
from helpers import make_plan
from paper_2609_03151_b200 import synth
from test_gpu_masked_attn import check, close, documents, f64, head_shards, mask_of, run

pytestmark = pytest.mark.gpu

W = lambda **kw: synth.Workload("f", **kw)


def compare(basp, w, kind, cap=0.0, slopes=None, seed=0, sample=None):
    """Forward and backward against the oracle, in all key heads of all sequences or in `sample` of them."""
    rng = np.random.default_rng(seed + w.S)
    pl = make_plan(basp, w)
    assert w.Hkv >= pl.K
    g = torch.Generator().manual_seed(seed)
    mk = lambda h: (torch.randn((w.B, w.S, h, w.D), generator=g) * torch.exp(0.3 * torch.randn((h, 1), generator=g))).to(torch.bfloat16)
    q, k, v, do = mk(w.Hq), mk(w.Hkv), mk(w.Hkv), mk(w.Hq)
    dq, dk, dv, ddo = (head_shards(t, pl, t.shape[2], 1) for t in (q, k, v, do))
    mask, begin, end = mask_of(basp, pl, kind, rng)
    score = basp.basp_score(cap, None if slopes is None else slopes.float().cuda(), mask)
    o = [torch.full_like(t, float("nan")) for t in dq]
    lse = [torch.full((pl.Bl, pl.Hq_l, pl.S), float("nan"), device="cuda") for _ in range(pl.N)]
    grads = [[torch.full_like(t, float("nan")) for t in x] for x in (dq, dk, dv)]
    ws = torch.full((basp.basp_attn_masked_bwd_workspace_bytes(pl),), 255, dtype=torch.uint8, device="cuda")
    basp.basp_clear_status()
    basp.basp_attn_masked_fwd(pl, score, dq, dk, dv, o, lse)
    basp.basp_attn_masked_bwd(pl, score, dq, dk, dv, o, ddo, lse, *grads, ws)
    basp.basp_get_status()
    assert all(torch.isfinite(t.float()).all() for x in (o, *grads) for t in x)
    G = w.Hq // w.Hkv
    steep = 0.0 if slopes is None else float(slopes.abs().max())
    for b, hkv in sample or [(b, h) for b in range(w.B) for h in range(w.Hkv)]:
        r, bl, first = b // pl.Bl * pl.K + hkv // pl.Hkv_l, b % pl.Bl, hkv % pl.Hkv_l * G
        mine, hs, one = slice(first, first + G), slice(hkv * G, hkv * G + G), slice(hkv % pl.Hkv_l, hkv % pl.Hkv_l + 1)
        Q, K, V, DO = f64(q[b, :, hs]), f64(k[b, :, hkv:hkv + 1]), f64(v[b, :, hkv:hkv + 1]), f64(do[b, :, hs])
        args = (Q, K, V, begin[b], end[b], cap, None if slopes is None else slopes[hs].double().numpy())
        ref = oracle.attn_shaped(*args)
        top = ref["top"]
        dz = (w.D / 8 + 4) * 2.0 ** -23 * top + 2.0 ** -21 * min(cap, top) + 2.0 ** -20 * (1 + (20 + 2 * top) * (steep > 0) / 16)
        far = w.S * steep * 2.0 ** -23
        p = 2 * dz + far
        O, L = f64(o[r][bl])[:, mine], lse[r][bl][mine].double().cpu().numpy()
        none = np.isneginf(ref["lse"])
        assert np.array_equal(np.isneginf(L), none)
        close(L[~none], ref["lse"][~none], dz + far + 2.0 ** -20 * (1 + np.abs(ref["lse"][~none])), (b, hkv, "lse"))
        close(O, ref["o"], (2.0 ** -8 + 2 * p) * ref["mag_o"] + 2.0 ** -8 * np.abs(ref["o"]), (b, hkv, "o"))
        # rows of up to eight keys take Delta from the scores: dO.O of the unrounded O
        short = (end[b] - begin[b] <= 8)[:, None, None]
        ref.update({n: t for n, t in oracle.attn_shaped(*args, do=DO, given=(np.where(short, ref["o"], O), L)).items() if n not in ("o", "lse", "mag_o")})
        bend = np.expm1(2 * (w.D / 8 + 4) * 2.0 ** -23 * top / cap) if cap else 0.0
        dots = (2.0 ** -16 + p) * np.einsum("shd,shd->s", np.abs(DO), np.abs(V).repeat(G, 1).max(0)[None] + np.abs(ref["o"])).max()
        got = {"dq": f64(grads[0][r][bl])[:, mine], "dk": f64(grads[1][r][bl])[:, one], "dv": f64(grads[2][r][bl])[:, one]}
        for n in ("dq", "dk"):
            close(got[n], ref[n], (2.0 ** -8 + 2 * p + 2.0 ** -18 + bend) * ref["mag_" + n] + dots * ref["row_" + n] + 2.0 ** -8 * np.abs(ref[n]) + 1e-30,
                  (b, hkv, n))
        close(got["dv"], ref["dv"], (2.0 ** -8 + 2 * p) * ref["mag_dv"] + 2.0 ** -8 * np.abs(ref["dv"]), (b, hkv, "dv"))


def parts_of(basp, pl):
    """Into how many parts the backward divides the query heads of a key head, from the workspace it asks for: the fp32 accumulator of dQ, Delta
    rounded up to 256 bytes, and fp32 dK and dV for every part where there are several."""
    rows = pl.Bl * pl.S
    rest = basp.basp_attn_masked_bwd_workspace_bytes(pl) // pl.N - rows * pl.Hq_l * pl.D * 4 - (rows * pl.Hq_l * 4 + 255) // 256 * 256
    return max(1, rest // (rows * pl.Hkv_l * pl.D * 8))


# heads a key head has, and into how many parts they go
DIVIDED = {
    "whole": (W(N=4, B=4, S=1100, Hq=26, Hkv=13, D=64), 1),
    "whole, two ranks a sequence": (W(N=8, B=4, S=1100, Hq=28, Hkv=14, D=64), 1),
    "two and one": (W(N=4, B=4, S=1100, Hq=27, Hkv=9, D=64), 2),
    "two, two and one": (W(N=4, B=4, S=1100, Hq=30, Hkv=6, D=64), 3),
}


@pytest.mark.parametrize("kind,cap,biased", [("docs", 0.0, False), ("causal", 20.0, False), ("ranges", 0.0, True), ("docs", 30.0, True)])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("form", list(DIVIDED))
def test_query_heads_of_a_key_head(basp, form, D, kind, cap, biased):
    w, parts = DIVIDED[form]
    w = W(N=w.N, B=w.B, S=w.S, Hq=w.Hq, Hkv=w.Hkv, D=D)
    assert parts_of(basp, make_plan(basp, w)) == parts       # another rule needs other plans here
    slopes = 2.0 ** (-8.0 * (torch.arange(w.Hq) + 1.0) / w.Hq) if biased else None
    compare(basp, w, kind, cap, slopes, 11, sample=[(0, 0), (1, w.Hkv // 2), (w.B - 1, w.Hkv - 1)])


@pytest.mark.parametrize("kind", ["docs", "prefix", "window", "ranges"])
@pytest.mark.parametrize("w", [W(N=8, B=8, S=1100, Hq=4, Hkv=2, D=64), W(N=2, B=2, S=4200, Hq=2, Hkv=1, D=128)], ids=["72 tiles", "66 tiles"])
def test_masks_of_three_launches(basp, w, kind):
    compare(basp, w, kind, 0.0, None, 12)


def mask_tables(basp, pl, mask):
    """(ranges [B, S, 2], tiles [B, n, 4], seen [B, n, 2], forward's items, backward's items) of a mask object."""
    B, n = pl.cfg.micro_batch, -(-pl.S // 128)
    raw, at = mask.cpu().numpy(), 0

    def take(count, width):
        nonlocal at
        part = raw[at:at + count * width * 4].view(np.int32).reshape(count, width)
        at += count * width * 4
        return part
    ranges, tiles, seen = take(B * n * 128, 2), take(B * n, 4), take(B * n, 2)
    at = (at + 15) // 16 * 16
    fwd, bwd = take(B * ((n + 1) // 2), 12), take(B * n, 4)
    assert at == basp.basp_mask_bytes(pl)
    whole = ranges.reshape(B, n * 128, 2)
    assert (whole[:, pl.S:] == 0).all()
    return whole[:, :pl.S], tiles.reshape(B, n, 4), seen.reshape(B, n, 2), fwd, bwd


@pytest.mark.parametrize("kind", ["docs", "prefix", "window", "ranges", "nothing"])
@pytest.mark.parametrize("B,S", [(1, 8192), (1, 8193), (2, 4096), (5, 1600), (3, 130)], ids=lambda n: str(n))
def test_mask_tables(basp, B, S, kind):
    """What the kernels walk, at 64 tiles and 65 (one launch and three): every query's keys, every tile's, and both lists of work, longest first."""
    pl = basp.basp_plan_create(B, B, S, 2, 1, 64)
    rng = np.random.default_rng(S)
    mask, begin, end = mask_of(basp, pl, kind, rng)
    ranges, tiles, seen, fwd, bwd = mask_tables(basp, pl, mask[:basp.basp_mask_bytes(pl)])
    some = end > begin
    want = np.where(some[..., None], np.stack([begin, end], -1), 0)
    assert np.array_equal(ranges, want)
    n = tiles.shape[1]
    cost = np.zeros((B, n + 1), dtype=np.int64)
    sees = np.zeros((B, n, n), dtype=bool)
    for b in range(B):
        for m in range(n):
            rows, on = want[b, m * 128:(m + 1) * 128], some[b, m * 128:(m + 1) * 128]
            if not on.any():
                assert not tiles[b, m].any()
                continue
            lo, hi, full, full_end = tiles[b, m]
            assert lo == rows[on, 0].min() // 128 and hi == -(-rows[on, 1].max() // 128)
            cost[b, m] = hi - lo
            sees[b, m, lo:hi] = True
            # wholly visible tiles: all that there are, where every row sees some key
            for j in range(lo, hi):
                assert (full <= j < full_end) == bool((rows[:, 0] <= j * 128).all() and (rows[:, 1] >= (j + 1) * 128).all())
        for j in range(n):
            by = np.flatnonzero(sees[b, :, j])
            assert tuple(seen[b, j]) == ((by[0], by[-1] + 1) if len(by) else (0, 0))
    blocks = [(b, i) for b in range(B) for i in range((n + 1) // 2)]
    order = sorted(blocks, key=lambda e: -(cost[e[0], 2 * e[1]] + cost[e[0], 2 * e[1] + 1]))             # (stable: ties in order)
    assert [tuple(e[:2]) for e in fwd] == order
    for e in fwd:
        for t in range(2):
            at = 2 * e[1] + t
            assert np.array_equal(e[4 + 4 * t:8 + 4 * t], tiles[e[0], at] if at < n else np.zeros(4))
    order = sorted([(b, j) for b in range(B) for j in range(n)], key=lambda e: -(seen[e][1] - seen[e][0]))
    assert [tuple(e) for e in bwd] == [(*e, *seen[e]) for e in order]


@pytest.mark.parametrize("cap", [0.0, 20.0, 120.0])
@pytest.mark.parametrize("kind", ["causal", "docs", "prefix", "ranges"])
@pytest.mark.parametrize("D", [64, 128])
def test_slopes_of_either_sign(basp, D, kind, cap):
    """A negative slope favours far keys: the largest exponential of a row is another one's.  Small slopes and steep ones."""
    w = W(N=2, B=2, S=515, Hq=6, Hkv=3, D=D)
    compare(basp, w, kind, cap, torch.tensor([-0.5, -0.01, 0.03, -2.0, 2.0, -0.0]), 13)


@pytest.mark.parametrize("shaping", ["wide cap", "wide cap bias", "huge cap"])
@pytest.mark.parametrize("kind", ["causal", "docs"])
@pytest.mark.parametrize("D", [64, 128])
def test_wide_caps_over_many_tiles(basp, D, kind, shaping):
    w = W(N=2, B=1, S=1300, Hq=4, Hkv=2, D=D)
    check(w, *run(basp, w, kind, shaping, 14))


def rank_rows(x, pl):
    """[B, S, H, D] as the ranks' sequence shards [Bl, tokens, H, D]."""
    return [x[r // pl.K * pl.Bl:(r // pl.K + 1) * pl.Bl, r % pl.K * pl.T:r % pl.K * pl.T + pl.rank_tokens(r)].contiguous() for r in range(pl.N)]


def from_rank_rows(shards, pl, B):
    """The other way, in fp64."""
    groups = [torch.cat([t.double().cpu() for t in shards[g * pl.K:(g + 1) * pl.K]], 1) for g in range(pl.N // pl.K)]
    return torch.cat(groups).numpy()


LAYERS = {
    "shared key heads, uneven": W(N=4, B=1, S=301, Hq=8, Hkv=2, D=128),            # 76 x 3 + 73 tokens
    "two sequences a group, uneven": W(N=8, B=2, S=203, Hq=8, Hkv=8, D=80, G=1),   # 26 x 7 + 21
    "one key head": W(N=4, B=2, S=260, Hq=4, Hkv=1, D=128, G=2),
    "even": W(N=2, B=1, S=512, Hq=8, Hkv=2, D=128),
}


@pytest.mark.parametrize("shaping", ["plain", "cap bias"])
@pytest.mark.parametrize("name", list(LAYERS))
def test_layer(basp, name, shaping):
    """The layer on sequence shards against the whole attention.  2-norms: O has P's roundings and its own (2^-9 rms each at most); the gradients have
    those of dS, of O in Delta, of a shared head's parts and of the result, four of 2^-9."""
    w = LAYERS[name]
    pl = make_plan(basp, w)
    g = torch.Generator().manual_seed(w.S)
    q, k, v, do = (torch.randn((w.B, w.S, h, w.D), generator=g).to(torch.bfloat16) for h in (w.Hq, w.Hkv, w.Hkv, w.Hq))
    pos, _ = documents(np.random.default_rng(w.S), w.B, w.S, 20)
    begin, end = oracle.packed_ranges(pos)
    mask = torch.empty(basp.basp_mask_bytes(pl), dtype=torch.uint8, device="cuda")
    basp.basp_mask_packed(pl, torch.from_numpy(pos).cuda(), mask)
    cap, slopes = (20.0, 2.0 ** -torch.arange(1.0, w.Hq + 1)) if shaping == "cap bias" else (0.0, None)
    score = basp.basp_score(cap, None if slopes is None else slopes.cuda(), mask)
    Q, K, V, DO = ([t.cuda() for t in rank_rows(x, pl)] for x in (q, k, v, do))
    O, DQ, DK, DV = ([torch.full_like(t, float("nan")) for t in x] for x in (Q, Q, K, V))
    lse = [torch.empty((pl.Bl, pl.Hq_l, pl.S), device="cuda") for _ in range(pl.N)]
    ws = torch.full((basp.basp_workspace_bytes(pl),), 255, dtype=torch.uint8, device="cuda")
    ws2 = torch.full((basp.basp_layer_masked_bwd_workspace_bytes(pl),), 255, dtype=torch.uint8, device="cuda")
    basp.basp_clear_status()
    basp.basp_layer_masked_fwd(pl, score, Q, K, V, O, ws, lse_shards=lse)
    held = [basp.as_shards(a) for a in basp.basp_layer_workspace_shards(pl, ws)]
    basp.basp_layer_masked_bwd(pl, score, *held, lse, DO, DQ, DK, DV, ws2)
    basp.basp_get_status()
    got = [from_rank_rows(x, pl, w.B) for x in (O, DQ, DK, DV)]
    want = [oracle.attn_shaped(f64(q[b]), f64(k[b]), f64(v[b]), begin[b], end[b], cap, None if slopes is None else slopes.double().numpy(),
                               do=f64(do[b])) for b in range(w.B)]
    for n, x in zip(("o", "dq", "dk", "dv"), got):
        ref = np.stack([r[n] for r in want])
        assert np.linalg.norm(x - ref) <= (2.0 ** -8 if n in ("o", "dv") and w.Hkv >= pl.K else 2.0 ** -7) * np.linalg.norm(ref), n


def test_backward_on_two_streams(basp):
    """Masked backward passes of two sizes on two streams, a dozen times over, against each alone: dK and dV to the bit, dQ but for the order of
    its sums (one key tile: to the bit as well)."""
    jobs = []
    for S, Hq, Hkv, D, cap in ((900, 8, 4, 128, 0.0), (700, 12, 4, 64, 20.0), (100, 8, 2, 64, 0.0)):
        pl = basp.basp_plan_create(1, 1, S, Hq, Hkv, D)
        g = torch.Generator(device="cuda").manual_seed(S)
        q, k, v, do = (torch.randn((1, S, h, D), generator=g, device="cuda").to(torch.bfloat16) for h in (Hq, Hkv, Hkv, Hq))
        mask = torch.empty(basp.basp_mask_bytes(pl), dtype=torch.uint8, device="cuda")
        basp.basp_mask_packed(pl, (torch.arange(S, device="cuda") % 333).int()[None].contiguous(), mask)
        score = basp.basp_score(cap, None, mask)
        o, lse = torch.empty_like(q), torch.empty((1, Hq, S), device="cuda")
        basp.basp_attn_masked_fwd(pl, score, [q], [k], [v], [o], [lse])
        ws = torch.empty(basp.basp_attn_masked_bwd_workspace_bytes(pl), dtype=torch.uint8, device="cuda")

        def call(out, stream, pl=pl, score=score, x=(q, k, v, o, do, lse), ws=ws):
            basp.basp_attn_masked_bwd(pl, score, *[[t] for t in x], *[[t] for t in out], ws, stream=stream)
        jobs.append((call, [q, k, v], S))
    basp.basp_clear_status()
    alone, out = ([[torch.full_like(t, float("nan")) for t in x] for _, x, _ in jobs] for _ in range(2))
    for (call, _, _), o in zip(jobs, alone):
        call(o, None)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in jobs]
    for _ in range(12):
        for (call, _, _), o, s in zip(jobs, out, streams):
            call(o, s)
    torch.cuda.synchronize()
    basp.basp_get_status()
    for (_, _, S), a, b in zip(jobs, alone, out):
        assert torch.equal(a[1], b[1]) and torch.equal(a[2], b[2])
        assert torch.equal(a[0], b[0]) if S <= 128 else ((a[0].float() - b[0].float()).norm() / a[0].float().norm()).item() <= 2.0 ** -8


@pytest.mark.parametrize("cap,biased", [(0.0, False), (20.0, False), (0.0, True), (120.0, True)])
@pytest.mark.parametrize("D", [64, 128])
def test_scale_of_the_caller(basp, D, cap, biased):
    """Four times the default scale is the default on four times Q, to the bit (a power of two passes through every rounding); O without a place
    for the LSE has the same bits."""
    S, H = 300, 2
    pl = basp.basp_plan_create(1, 1, S, H, H, D)
    g = torch.Generator(device="cuda").manual_seed(D)
    q, k, v, do = (torch.randn((1, S, H, D), generator=g, device="cuda").to(torch.bfloat16) for _ in range(4))
    pos = (torch.arange(S, device="cuda") % 140).int()
    pos[-30:] = torch.arange(30, device="cuda") % 3                     # rows of up to eight keys too
    mask = torch.empty(basp.basp_mask_bytes(pl), dtype=torch.uint8, device="cuda")
    basp.basp_mask_packed(pl, pos[None].contiguous(), mask)
    score = basp.basp_score(cap, torch.tensor([0.5, 0.01], device="cuda") if biased else None, mask)
    ws = torch.empty(basp.basp_attn_masked_bwd_workspace_bytes(pl), dtype=torch.uint8, device="cuda")
    basp.basp_clear_status()
    got = []
    for Q, scale in ((q, float(np.float32(1.0) / np.sqrt(np.float32(D))) * 4.0), (q * 4, 0.0)):
        o, alone, lse = torch.full_like(q, float("nan")), torch.full_like(q, float("nan")), torch.empty((1, H, S), device="cuda")
        grads = [[torch.full_like(t, float("nan"))] for t in (q, k, v)]
        basp.basp_attn_masked_fwd(pl, score, [Q], [k], [v], [o], [lse], softmax_scale=scale)
        basp.basp_attn_masked_fwd(pl, score, [Q], [k], [v], [alone], None, softmax_scale=scale)
        basp.basp_attn_masked_bwd(pl, score, [Q], [k], [v], [o], [do], [lse], *grads, ws, softmax_scale=scale)
        assert torch.equal(o, alone)
        got.append((o, lse, *(t[0] for t in grads)))
    basp.basp_get_status()
    (o, lse, dq, dk, dv), (o4, lse4, dq4, dk4, dv4) = got
    # dS has the scale as a factor: four times as large in the first call, and multiplied by a quarter of the second one's Q for dK
    assert torch.equal(o, o4) and torch.equal(lse, lse4) and torch.equal(dv, dv4) and torch.equal(dk, dk4)
    assert ((dq.float() - 4 * dq4.float()).norm() / dq.float().norm()).item() <= 2.0 ** -8              # the order of dQ's sums
