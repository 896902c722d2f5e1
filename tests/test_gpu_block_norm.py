"""Norms around a block with gate and residual scale, forward and backward, against the fp64 oracle.

Tolerances, per element: one rounding to bf16 (2^-8 of the value) and the fp32 arithmetic before it.  A sum over a row adds at most 32
terms in a thread and then 5 + 16 sums: 2^-24 x 53 of the sum of magnitudes (of squares: of the sum itself), so r is good to 2^-19
and r^3 to 2^-17.
  h     2^-18 of its two terms' magnitudes
  n     r of h: 2^-18 of |n|, and h's own error times w r
  dx,dy 2^-16 of the magnitudes of the terms
  dw    a sum over rows in fp32: a thread adds up to 600 rows here, then 8 groups and partial rows by 32: 2^-24 x 700 < 2^-14 of the sum of
        magnitudes, and each term's own 2^-16"""
import numpy as np
import pytest
import torch

import oracle
from helpers import make_plan
from paper_2609_03151_b200 import synth

pytestmark = pytest.mark.gpu

SHAPES = {
    "one token": synth.Workload("s", N=1, B=1, S=1, Hq=1, Hkv=1, D=64),
    "uneven": synth.Workload("s", N=4, B=2, S=77, Hq=4, Hkv=4, D=64, G=1),
    "many ranks": synth.Workload("s", N=16, B=4, S=35, Hq=16, Hkv=16, D=64),
    "many rows": synth.Workload("s", N=2, B=1, S=2500, Hq=2, Hkv=2, D=64),
}
WEIGHTS = [(1, 1, 1), (1, 0, 1), (0, 1, 1), (0, 0, 1), (1, 1, 0), (0, 1, 0), (0, 0, 0)]
EPS = 1e-5


def f64(t):
    return t.float().cpu().numpy().astype(np.float64)


def setup(basp, w, hidden, seed=0):
    pl = make_plan(basp, w)
    g = torch.Generator().manual_seed(seed + w.S + hidden)
    rows = [pl.Bl * pl.rank_tokens(r) for r in range(pl.N)]
    feature = torch.exp(0.7 * torch.randn(hidden, generator=g))
    mk = lambda scale=1.0: [(scale * torch.randn((n, hidden), generator=g) * feature).to(torch.bfloat16) for n in rows]
    weights = [(m + 0.3 * torch.randn(hidden, generator=g)).to(torch.bfloat16) for m in (1.0, 0.5, 1.0)]
    return pl, mk, weights


def cuda(ts):
    return [t.cuda() for t in ts]


def blank(ts):
    return [torch.full_like(t, float("nan")) for t in ts]


def within(got, want, bound, what):
    bad = ~(np.abs(got - want) <= bound)
    assert not bad.any(), (what, int(bad.sum()), float(np.nanmax(np.abs(got - want) / bound)))


def rms(t):
    return np.sqrt((t * t).mean(-1, keepdims=True) + EPS)


@pytest.mark.parametrize("on", WEIGHTS, ids=lambda on: "%d%d%d" % on)
@pytest.mark.parametrize("hidden", [8, 264, 512, 520, 4096, 8200])
def test_forward_and_backward(basp, hidden, on):
    w = SHAPES["uneven"]
    pl, mk, weights = setup(basp, w, hidden)
    x, y, dh, dn = mk(2.0), mk(), mk(0.1), mk(0.1)
    ws = [t if o else None for t, o in zip(weights, on)]
    dev = [None if t is None else t.cuda() for t in ws]
    kw = dict(w_post=dev[0], gate=dev[1], w_pre=dev[2], res_scale=0.7, eps=EPS)
    h, n = blank(cuda(x)), blank(cuda(x)) if on[2] else None
    basp.basp_clear_status()
    basp.basp_block_norm(pl, hidden, cuda(x), cuda(y), h, n, **kw)
    W = [None if t is None else f64(t) for t in ws]
    for r in range(pl.N):
        want_h, want_n = oracle.block_norm(f64(x[r]), f64(y[r]), *W, 0.7, EPS)
        off = 2.0 ** -18 * (np.abs(f64(x[r])) + np.abs(want_h - f64(x[r])))
        within(f64(h[r]), want_h, 2.0 ** -8 * np.abs(want_h) + off, (r, "h"))
        if on[2]:
            within(f64(n[r]), want_n, (2.0 ** -8 + 2.0 ** -17) * np.abs(want_n) + off * np.abs(W[2]) / rms(want_h), (r, "n"))
    dx, dy = blank(cuda(x)), blank(cuda(x))
    sums = [torch.full((hidden,), float("nan"), device="cuda") if o else None for o in on]
    space = torch.full((basp.basp_block_norm_bwd_workspace_bytes(pl, hidden),), 255, dtype=torch.uint8, device="cuda")
    basp.basp_block_norm_bwd(pl, hidden, cuda(x) if on[2] else None, cuda(y) if on[0] or on[1] else None, cuda(dh), cuda(dn) if on[2] else None,
                             dx, dy, *sums, space, **kw)
    basp.basp_get_status()
    totals, mags = {}, {}
    for r in range(pl.N):
        X, Y, DH, DN = (f64(t[r]) for t in (x, y, dh, dn))
        ref = oracle.block_norm_bwd(X, Y, *W, 0.7, EPS, DH, DN if on[2] else None)
        mag = np.abs(DH)
        if on[2]:
            up = np.abs(DN * W[2])
            mag = mag + up / rms(X) + np.abs(X) * (up * np.abs(X)).mean(-1, keepdims=True) / rms(X) ** 3
            mags["dw_pre"] = mags.get("dw_pre", 0) + np.abs(DN * X / rms(X)).sum(0)
        within(f64(dx[r]), ref["dx"], 2.0 ** -8 * np.abs(ref["dx"]) + 2.0 ** -16 * mag, (r, "dx"))
        mag = 0.7 * mag
        if on[1]:
            mags["dgate"] = mags.get("dgate", 0) + (mag * np.abs(Y / rms(Y) * W[0] if on[0] else Y)).sum(0)
            mag = mag * np.abs(W[1])
        if on[0]:
            mags["dw_post"] = mags.get("dw_post", 0) + (mag * np.abs(Y) / rms(Y)).sum(0)
            up = mag * np.abs(W[0])
            mag = up / rms(Y) + np.abs(Y) * (up * np.abs(Y)).mean(-1, keepdims=True) / rms(Y) ** 3
        within(f64(dy[r]), ref["dy"], 2.0 ** -8 * np.abs(ref["dy"]) + 2.0 ** -16 * mag, (r, "dy"))
        for name in ("dw_post", "dgate", "dw_pre"):
            if name in ref:
                totals[name] = totals.get(name, 0) + ref[name]
    for name, t in zip(("dw_post", "dgate", "dw_pre"), sums):
        if t is not None:
            within(t.double().cpu().numpy(), totals[name], 2.0 ** -13 * mags[name], name)


@pytest.mark.parametrize("hidden", [64, 2048, 16384])
@pytest.mark.parametrize("shape", ["one token", "many ranks", "many rows"])
def test_rows(basp, shape, hidden):
    w = SHAPES[shape]
    if shape == "many rows" and hidden == 16384:
        w = synth.Workload("s", N=2, B=1, S=700, Hq=2, Hkv=2, D=64)
    pl, mk, (wp, g, wn) = setup(basp, w, hidden)
    x, y, dh, dn = mk(2.0), mk(), mk(0.1), mk(0.1)
    kw = dict(w_post=wp.cuda(), gate=g.cuda(), w_pre=wn.cuda(), eps=EPS)
    h, n, dx, dy = (blank(cuda(x)) for _ in range(4))
    sums = [torch.empty(hidden, device="cuda") for _ in range(3)]
    space = torch.empty(basp.basp_block_norm_bwd_workspace_bytes(pl, hidden), dtype=torch.uint8, device="cuda")
    basp.basp_clear_status()
    basp.basp_block_norm(pl, hidden, cuda(x), cuda(y), h, n, **kw)
    basp.basp_block_norm_bwd(pl, hidden, cuda(x), cuda(y), cuda(dh), cuda(dn), dx, dy, *sums, space, **kw)
    basp.basp_get_status()
    W = [f64(t) for t in (wp, g, wn)]
    X, Y, DH, DN = (np.concatenate([f64(t) for t in s]) for s in (x, y, dh, dn))
    ref_h, ref_n = oracle.block_norm(X, Y, *W, 1.0, EPS)
    ref = oracle.block_norm_bwd(X, Y, *W, 1.0, EPS, DH, DN)
    off = 2.0 ** -18 * (np.abs(X) + np.abs(ref_h - X))
    cat = lambda ts: np.concatenate([f64(t) for t in ts])
    within(cat(h), ref_h, 2.0 ** -8 * np.abs(ref_h) + off, "h")
    within(cat(n), ref_n, (2.0 ** -8 + 2.0 ** -17) * np.abs(ref_n) + off * np.abs(W[2]) / rms(ref_h), "n")
    up = np.abs(DN * W[2])
    mag = np.abs(DH) + up / rms(X) + np.abs(X) * (up * np.abs(X)).mean(-1, keepdims=True) / rms(X) ** 3
    within(cat(dx), ref["dx"], 2.0 ** -8 * np.abs(ref["dx"]) + 2.0 ** -16 * mag, "dx")
    within(sums[2].double().cpu().numpy(), ref["dw_pre"], 2.0 ** -13 * np.abs(DN * X / rms(X)).sum(0), "dw_pre")
    within(sums[1].double().cpu().numpy(), ref["dgate"], 2.0 ** -13 * (mag * np.abs(Y / rms(Y) * W[0])).sum(0), "dgate")
    mag = mag * np.abs(W[1])
    within(sums[0].double().cpu().numpy(), ref["dw_post"], 2.0 ** -13 * (mag * np.abs(Y) / rms(Y)).sum(0), "dw_post")
    up = mag * np.abs(W[0])
    mag = up / rms(Y) + np.abs(Y) * (up * np.abs(Y)).mean(-1, keepdims=True) / rms(Y) ** 3
    within(cat(dy), ref["dy"], 2.0 ** -8 * np.abs(ref["dy"]) + 2.0 ** -16 * mag, "dy")


def test_first_norm_and_missing_gradients(basp):
    """Without a block before: n of x alone and its gradients; with one but without a gradient of the stream."""
    w, hidden = SHAPES["uneven"], 264
    pl, mk, (wp, g, wn) = setup(basp, w, hidden)
    x, y, dn = mk(2.0), mk(), mk()
    n, dx, dy = (blank(cuda(x)) for _ in range(3))
    dw = [torch.empty(hidden, device="cuda") for _ in range(3)]
    space = torch.empty(basp.basp_block_norm_bwd_workspace_bytes(pl, hidden), dtype=torch.uint8, device="cuda")
    basp.basp_block_norm(pl, hidden, cuda(x), None, None, n, w_pre=wn.cuda(), eps=EPS)
    basp.basp_block_norm_bwd(pl, hidden, cuda(x), None, None, cuda(dn), dx, None, None, None, dw[2], space, w_pre=wn.cuda(), eps=EPS)
    for r in range(pl.N):
        want = oracle.block_norm(f64(x[r]), None, None, None, f64(wn), 1.0, EPS)[1]
        within(f64(n[r]), want, (2.0 ** -8 + 2.0 ** -17) * np.abs(want), r)
        ref = oracle.block_norm_bwd(f64(x[r]), None, None, None, f64(wn), 1.0, EPS, None, f64(dn[r]))
        up = np.abs(f64(dn[r]) * f64(wn))
        mag = up / rms(f64(x[r])) + np.abs(f64(x[r])) * (up * np.abs(f64(x[r]))).mean(-1, keepdims=True) / rms(f64(x[r])) ** 3
        within(f64(dx[r]), ref["dx"], 2.0 ** -8 * np.abs(ref["dx"]) + 2.0 ** -16 * mag, r)
    zeros = [torch.zeros_like(t) for t in x]
    kw = dict(w_post=wp.cuda(), gate=g.cuda(), w_pre=wn.cuda(), eps=EPS)
    got = []
    for dh in (None, cuda(zeros)):
        a, b = blank(cuda(x)), blank(cuda(x))
        sums = [torch.empty(hidden, device="cuda") for _ in range(3)]
        basp.basp_block_norm_bwd(pl, hidden, cuda(x), cuda(y), dh, cuda(dn), a, b, *sums, space, **kw)
        got.append(a + b + sums)
    assert all(torch.equal(p, q) for p, q in zip(*got))


@pytest.mark.parametrize("hidden", [328, 4096])
def test_in_place_and_zero_rows(basp, hidden):
    """h over x or y, n over the other; dx over dh or dn, dy over y; the same bits.  Rows of zeros stay finite."""
    w = SHAPES["uneven"]
    pl, mk, (wp, g, wn) = setup(basp, w, hidden)
    x, y, dh, dn = mk(), mk(), mk(), mk()
    for t in (x, y):
        t[0][3] = 0
    kw = dict(w_post=wp.cuda(), gate=g.cuda(), w_pre=wn.cuda(), eps=1e-30)
    space = torch.empty(basp.basp_block_norm_bwd_workspace_bytes(pl, hidden), dtype=torch.uint8, device="cuda")
    h, n = blank(cuda(x)), blank(cuda(x))
    basp.basp_block_norm(pl, hidden, cuda(x), cuda(y), h, n, **kw)
    assert all(torch.isfinite(t.float()).all() for t in h + n)
    for swap in (False, True):
        a, b = cuda(x), cuda(y)
        basp.basp_block_norm(pl, hidden, a, b, *((b, a) if swap else (a, b)), **kw)
        for p, q in zip(h + n, (b + a) if swap else (a + b)):
            assert torch.equal(p, q)
    dx, dy = blank(cuda(x)), blank(cuda(x))
    s0 = [torch.empty(hidden, device="cuda") for _ in range(3)]
    basp.basp_block_norm_bwd(pl, hidden, cuda(x), cuda(y), cuda(dh), cuda(dn), dx, dy, *s0, space, **kw)
    for over in (0, 1):
        X, Y, a, b = cuda(x), cuda(y), cuda(dh), cuda(dn)
        s1 = [torch.empty(hidden, device="cuda") for _ in range(3)]
        basp.basp_block_norm_bwd(pl, hidden, X, Y, a, b, (a, b)[over], Y, *s1, space, **kw)
        assert all(torch.equal(p, q) or (torch.isnan(p) == torch.isnan(q)).all() for p, q in zip(dx + dy + s0, (a, b)[over] + Y + s1))
    assert all(torch.isfinite(t.float()).all() for t in dx + dy + s0)


@pytest.mark.parametrize("hidden", [64, 520, 4096])
def test_no_weights_no_workspace(basp, hidden):
    """Without weights there are no sums: the workspace may be missing, small, or full of someone else's data, which stays."""
    w = SHAPES["uneven"]
    pl, mk, _ = setup(basp, w, hidden)
    dh = mk()
    guard = torch.full((64 + 148 * 16 * 3 * hidden * 4,), 7, dtype=torch.uint8, device="cuda")       # more than any number of blocks could write
    want = [(0.5 * f64(t), f64(t)) for t in dh]
    basp.basp_clear_status()
    for space in (None, guard[16:32], guard[17:18]):
        dx, dy = blank(cuda(dh)), blank(cuda(dh))
        basp.basp_block_norm_bwd(pl, hidden, None, None, cuda(dh), None, dx, dy, None, None, None, space, res_scale=0.5, eps=EPS)
        basp.basp_get_status()
        for r in range(pl.N):
            assert np.array_equal(f64(dx[r]), want[r][1]) and np.array_equal(f64(dy[r]), want[r][0])       # a power of two: exact
        assert (guard == 7).all()


@pytest.mark.parametrize("hidden", [64, 328, 4096, 16384])
@pytest.mark.parametrize("shape", ["uneven", "many rows"])
def test_backward_in_place_to_the_bit(basp, shape, hidden):
    """dx over dh_out or over dn, dy over y: every gradient has the bits that separate outputs get."""
    w = SHAPES[shape]
    pl, mk, (wp, g, wn) = setup(basp, w, hidden)
    x, y, dh, dn = (cuda(mk()) for _ in range(4))
    copy = lambda ts: [t.clone() for t in ts]
    kw = dict(w_post=wp.cuda(), gate=g.cuda(), w_pre=wn.cuda(), res_scale=0.7, eps=EPS)
    space = torch.empty(basp.basp_block_norm_bwd_workspace_bytes(pl, hidden), dtype=torch.uint8, device="cuda")
    dx, dy, sums = blank(x), blank(x), [torch.empty(hidden, device="cuda") for _ in range(3)]
    basp.basp_clear_status()
    basp.basp_block_norm_bwd(pl, hidden, x, y, dh, dn, dx, dy, *sums, space, **kw)
    want = dx + dy + sums
    assert all(torch.isfinite(t.float()).all() and (t != 0).any() for t in want)
    for over in (0, 1):
        a, b, Y = copy(dh), copy(dn), copy(y)
        s1 = [torch.full((hidden,), float("nan"), device="cuda") for _ in range(3)]
        basp.basp_block_norm_bwd(pl, hidden, x, Y, a, b, (a, b)[over], Y, *s1, space, **kw)
        for p, q in zip(want, (a, b)[over] + Y + s1):
            assert torch.equal(p, q)
        assert all(torch.equal(p, q) for p, q in zip((b, a)[over], (dn, dh)[over]))       # the other input stays
    basp.basp_get_status()
