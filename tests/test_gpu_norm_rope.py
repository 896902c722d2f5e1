"""Head norms with the rotary embedding, forward and backward, against the fp64 oracle.

Tolerances, per element: one rounding to bf16 (2^-8 of the value) and the fp32 arithmetic before it, bounded by its terms:
  y   the pair's two terms, each a product of four fp32 numbers of which r has a relative error below 2^-20 (the mean of D
      squares, at most 16 in a row per lane and three shuffles: 2^-24 x 19 / 2, and the reciprocal root's 2 ulp)
  dx  the terms r w u and x r^3 (x.w u) / D; the dot product adds 2^-24 x 19 of the sum of its terms' magnitudes, r^3 three
      times r's error: 2^-18 of the terms' magnitudes covers both
  dw  a sum over tokens and heads in fp32: a thread adds at most ~600 terms here, then 2 + 8 + 32 partial sums: 2^-24 x 700 < 2^-14
      of the sum of magnitudes, and u's and r's own errors 2^-19"""
import numpy as np
import pytest
import torch

import oracle
from helpers import make_plan
from paper_2609_03151_b200 import synth

pytestmark = pytest.mark.gpu

CASES = [
    synth.Workload("one_token", N=1, B=1, S=1, Hq=1, Hkv=1, D=128),
    synth.Workload("token_per_rank", N=4, B=1, S=4, Hq=8, Hkv=4, D=128),
    synth.Workload("d16", N=2, B=2, S=70, Hq=3, Hkv=1, D=16),
    synth.Workload("d32", N=2, B=1, S=131, Hq=6, Hkv=2, D=32),
    synth.Workload("d48", N=1, B=3, S=45, Hq=5, Hkv=5, D=48),
    synth.Workload("d64_two_seqs", N=4, B=4, S=100, Hq=8, Hkv=4, D=64, G=2),
    synth.Workload("d80", N=4, B=2, S=203, Hq=20, Hkv=4, D=80),
    synth.Workload("d96_uneven_two_seqs", N=4, B=2, S=77, Hq=8, Hkv=4, D=96, G=1),
    synth.Workload("d112", N=2, B=2, S=65, Hq=7, Hkv=7, D=112),
    synth.Workload("d128_uneven", N=4, B=1, S=1021, Hq=32, Hkv=8, D=128),
    synth.Workload("data_parallel", N=2, B=4, S=33, Hq=4, Hkv=2, D=128),
    synth.Workload("many_ranks", N=16, B=2, S=160, Hq=8, Hkv=8, D=64),
    synth.Workload("replicated_kv", N=8, B=1, S=264, Hq=16, Hkv=2, D=128),
]
EPS = 1e-5


def setup(basp, w, seed=0):
    """Plan, inputs per rank (device), weights, tables and the positions of every rank's rows."""
    pl = make_plan(basp, w)
    g = torch.Generator().manual_seed(seed + w.S * w.D)
    rows = [pl.Bl * pl.rank_tokens(r) for r in range(pl.N)]
    mk = lambda h: [(synth.randn_bf16(g, (n, h, w.D)).float() * torch.exp(torch.randn((1, h, 1), generator=g))).to(torch.bfloat16)
                    for n in rows]
    weights = [(1 + 0.3 * torch.randn(w.D, generator=g)).to(torch.bfloat16) for _ in range(2)]
    cos, sin = synth.rope_tables(w.S, w.D)
    pos = [np.tile(np.arange(pl.rank_tokens(r)), pl.Bl) + (r % pl.K) * pl.T for r in range(pl.N)]
    return pl, mk, weights, cos, sin, pos


def f64(t):
    return t.float().cpu().numpy().astype(np.float64)


def cuda(ts):
    return [t.cuda() for t in ts]


def blank(ts):
    return [torch.full_like(t, float("nan")) for t in ts]


def halves(a):
    lo, hi = np.split(np.abs(a), 2, axis=-1)
    return np.concatenate([lo + hi, lo + hi], axis=-1)


def check_fwd(x, w, cos, sin, pos, y, what):
    ref = oracle.qk_norm_rope(f64(x), f64(w), cos.numpy(), sin.numpy(), pos, EPS)
    z = f64(x) / np.sqrt((f64(x) ** 2).mean(-1, keepdims=True) + EPS) * f64(w)
    bad = np.abs(f64(y) - ref) > 2.0 ** -8 * np.abs(ref) + 2.0 ** -20 * halves(z)
    assert not bad.any(), (what, int(bad.sum()))


@pytest.mark.parametrize("w", CASES, ids=lambda w: w.name)
def test_forward(basp, w):
    pl, mk, (wq, wk), cos, sin, pos = setup(basp, w)
    q, k = mk(w.Hq), mk(w.Hkv)
    dq, dk = cuda(q), cuda(k)
    table = [t.t().contiguous().cuda() for t in (cos, sin)]
    oq, ok = blank(dq), blank(dk)
    basp.basp_qk_norm_rope(pl, dq, dk, wq.cuda(), wk.cuda(), *table, oq, ok, eps=EPS)
    for r in range(pl.N):
        check_fwd(q[r], wq, cos, sin, pos[r], oq[r], (w.name, "q", r))
        check_fwd(k[r], wk, cos, sin, pos[r], ok[r], (w.name, "k", r))
    # in place: the same bits
    basp.basp_qk_norm_rope(pl, dq, dk, wq.cuda(), wk.cuda(), *table, dq, dk, eps=EPS)
    assert all(torch.equal(a, b) for a, b in zip(dq + dk, oq + ok))


@pytest.mark.parametrize("w", CASES, ids=lambda w: w.name)
def test_backward(basp, w):
    pl, mk, ws, cos, sin, pos = setup(basp, w, 1)
    x, dy = [mk(w.Hq), mk(w.Hkv)], [mk(w.Hq), mk(w.Hkv)]
    table = [t.t().contiguous().cuda() for t in (cos, sin)]
    xd, dyd = [cuda(t) for t in x], [cuda(t) for t in dy]
    dx = [blank(t) for t in xd]
    dw = [torch.full((w.D,), float("nan"), device="cuda") for _ in range(2)]
    space = torch.full((basp.basp_qk_norm_rope_bwd_workspace_bytes(pl) // 4,), float("nan"), device="cuda")
    args = (pl, *xd, ws[0].cuda(), ws[1].cuda(), *table, *dyd)
    basp.basp_qk_norm_rope_bwd(*args, *dx, *dw, space, eps=EPS)
    for i in range(2):
        sum_dw, size_dw = 0.0, 0.0
        for r in range(pl.N):
            X, W, DY = f64(x[i][r]), f64(ws[i]), f64(dy[i][r])
            want, want_w = oracle.qk_norm_rope_bwd(X, W, cos.numpy(), sin.numpy(), pos[r], EPS, DY)
            s = (X * X).mean(-1, keepdims=True) + EPS
            u = halves(DY)                                            # bounds |R^T dy|
            terms = np.abs(W) * u / np.sqrt(s) + np.abs(X) * s ** -1.5 * (np.abs(X * W) * u).sum(-1, keepdims=True) / w.D
            bad = np.abs(f64(dx[i][r]) - want) > 2.0 ** -8 * np.abs(want) + 2.0 ** -18 * terms
            assert not bad.any(), (w.name, i, r, int(bad.sum()))
            sum_dw, size_dw = sum_dw + want_w, size_dw + (np.abs(X) / np.sqrt(s) * u).sum((0, 1))
        assert (np.abs(f64(dw[i]) - sum_dw) <= (2.0 ** -14 + 2.0 ** -19) * size_dw).all(), (w.name, i)
    # again: the same bits; and with the gradient written over the incoming one
    dx2, dw2 = [blank(t) for t in xd], [torch.empty_like(t) for t in dw]
    basp.basp_qk_norm_rope_bwd(*args, *dx2, *dw2, space, eps=EPS)
    assert all(torch.equal(a, b) for a, b in zip(dx[0] + dx[1] + dw, dx2[0] + dx2[1] + dw2))
    basp.basp_qk_norm_rope_bwd(*args, *dyd, *dw2, space, eps=EPS)
    assert all(torch.equal(a, b) for a, b in zip(dx[0] + dx[1], dyd[0] + dyd[1]))


def test_zero_and_special_vectors(basp):
    w = synth.Workload("special", N=1, B=1, S=3, Hq=4, Hkv=2, D=64)
    pl, mk, (wq, wk), cos, sin, pos = setup(basp, w)
    q, k = mk(4), mk(2)
    q[0][0, 0] = 0.0                                      # a zero vector stays zero
    q[0][1, 1] = 2.0 ** -60                               # far below eps: x / sqrt(eps)
    q[0][2, 2, 5] = float("inf")
    q[0][2, 3, 6] = float("nan")
    out, ok = blank(cuda(q)), blank(cuda(k))
    basp.basp_qk_norm_rope(pl, cuda(q), cuda(k), wq.cuda(), wk.cuda(), cos.t().contiguous().cuda(), sin.t().contiguous().cuda(),
                           out, ok, eps=EPS)
    y = f64(out[0])
    assert (y[0, 0] == 0).all() and np.isnan(y[2, 3]).all() and np.isnan(y[2, 2, 5])
    assert np.isfinite(y[:2]).all() and np.isfinite(y[2, :2]).all()      # the neighbours are untouched
    finite = [t.clone() for t in q]
    finite[0][2, 2:] = 1.0
    out[0][2, 2:] = torch.nan
    ref = oracle.qk_norm_rope(f64(finite[0][:2]), f64(wq), cos.numpy(), sin.numpy(), pos[0][:2], EPS)
    assert (np.abs(y[:2] - ref) <= 2.0 ** -8 * np.abs(ref) + 1e-5).all()


def test_backward_of_zeros_and_small_vectors_with_a_small_eps(basp):
    """eps = 1e-30: r = 10^15 of a zero vector leaves fp32 in its third power, but x r^3 (x . w u) / D is zero there; a vector
    of 2^-40 is far above eps.  The bounds are those of the other tests, in the vector's own units."""
    w, eps = synth.Workload("small_eps", N=1, B=1, S=4, Hq=4, Hkv=2, D=64), 1e-30
    pl, mk, ws, cos, sin, pos = setup(basp, w, 3)
    x, dy = [mk(4), mk(2)], [mk(4), mk(2)]
    x[0][0][1, 2], x[1][0][:] = 0.0, 0.0
    x[0][0][2] *= 2.0 ** -40                              # exact
    table = [t.t().contiguous().cuda() for t in (cos, sin)]
    dx = [blank(cuda(t)) for t in x]
    dw = [torch.full((w.D,), float("nan"), device="cuda") for _ in range(2)]
    space = torch.full((basp.basp_qk_norm_rope_bwd_workspace_bytes(pl) // 4,), float("nan"), device="cuda")
    basp.basp_qk_norm_rope_bwd(pl, cuda(x[0]), cuda(x[1]), ws[0].cuda(), ws[1].cuda(), *table, cuda(dy[0]), cuda(dy[1]), *dx,
                               *dw, space, eps=eps)
    for i in range(2):
        X, W, DY = f64(x[i][0]), f64(ws[i]), f64(dy[i][0])
        want, want_w = oracle.qk_norm_rope_bwd(X, W, cos.numpy(), sin.numpy(), pos[0], eps, DY)
        s, u = (X * X).mean(-1, keepdims=True) + eps, halves(DY)
        terms = np.abs(W) * u / np.sqrt(s) + np.abs(X) * s ** -1.5 * (np.abs(X * W) * u).sum(-1, keepdims=True) / w.D
        assert (np.abs(f64(dx[i][0]) - want) <= 2.0 ** -8 * np.abs(want) + 2.0 ** -18 * terms).all(), i
        size = (np.abs(X) / np.sqrt(s) * u).sum((0, 1))
        assert (np.abs(f64(dw[i]) - want_w) <= (2.0 ** -14 + 2.0 ** -19) * size).all(), i


def test_rows_behind_the_shard_are_left(basp):
    """A buffer longer than the shard keeps what lies behind it (tiles of 32 tokens, shards of 5)."""
    w = synth.Workload("tail", N=2, B=2, S=5, Hq=2, Hkv=2, D=128)
    pl, mk, (wq, wk), cos, sin, _ = setup(basp, w)
    q, k = cuda(mk(2)), cuda(mk(2))
    big = [torch.full((64, 2, 128), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(4)]
    basp.basp_qk_norm_rope(pl, q, k, wq.cuda(), wk.cuda(), cos.t().contiguous().cuda(), sin.t().contiguous().cuda(),
                           [t[:5] for t in big[:2]], [t[:5] for t in big[2:]])
    assert all((t[5:] == 7.0).all().item() for t in big)


def test_autograd_and_graph(basp):
    from paper_2609_03151_b200.autograd import basp_qk_norm_rope
    w = synth.Workload("auto", N=4, B=2, S=96, Hq=4, Hkv=2, D=64)
    pl, mk, ws, cos, sin, pos = setup(basp, w, 2)
    leaves = [[t.requires_grad_() for t in cuda(mk(h))] for h in (4, 2)]
    wl = [t.cuda().requires_grad_() for t in ws]
    dy = [cuda(mk(4)), cuda(mk(2))]
    table = [t.t().contiguous().cuda() for t in (cos, sin)]
    q, k = basp_qk_norm_rope(pl, *leaves, *wl, *table, eps=EPS)
    torch.autograd.backward(q + k, dy[0] + dy[1])
    for i in range(2):
        got_w = 0.0
        for r in range(pl.N):
            X, W = f64(leaves[i][r].detach()), f64(ws[i])
            want, want_w = oracle.qk_norm_rope_bwd(X, W, cos.numpy(), sin.numpy(), pos[r], EPS, f64(dy[i][r]))
            assert np.abs(f64(leaves[i][r].grad) - want).max() <= 2.0 ** -7 * np.abs(want).max()
            got_w = got_w + want_w
        assert np.abs(f64(wl[i].grad) - got_w).max() <= 2.0 ** -7 * np.abs(got_w).max()
    # the library's calls in a CUDA graph: replay on new inputs
    x = [t.detach().clone() for t in leaves[0]], [t.detach().clone() for t in leaves[1]]
    out = [[torch.empty_like(t) for t in s] for s in x]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        basp.basp_qk_norm_rope(pl, *x, wl[0].detach(), wl[1].detach(), *table, *out, eps=EPS)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        basp.basp_qk_norm_rope(pl, *x, wl[0].detach(), wl[1].detach(), *table, *out, eps=EPS)
    for a, b in zip(x[0] + x[1], cuda(mk(4)) + cuda(mk(2))):
        a.copy_(b)
    graph.replay()
    torch.cuda.synchronize()
    eager = [[torch.empty_like(t) for t in s] for s in x]
    basp.basp_qk_norm_rope(pl, *x, wl[0].detach(), wl[1].detach(), *table, *eager, eps=EPS)
    assert all(torch.equal(a, b) for a, b in zip(out[0] + out[1], eager[0] + eager[1]))
