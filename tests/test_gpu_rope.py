"""Rotary positions of any token order against the fp64 oracle.  Tolerance: one rounding to bf16 (2^-8 of the value) and the fp32
arithmetic before it: angle, sine and cosine to 2^-22, two products: 2^-21 of the pair's magnitudes (times the factor)."""
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
    synth.Workload("many_heads", N=1, B=1, S=19, Hq=67, Hkv=1, D=128),
    synth.Workload("many_ranks", N=16, B=2, S=160, Hq=8, Hkv=8, D=64),
]


def f64(t):
    return t.float().cpu().numpy().astype(np.float64)


def rows_of(pl, r, positions):
    """Positions of rank r's rows in order."""
    g, l = r // pl.K, r % pl.K
    n = pl.rank_tokens(r)
    return np.concatenate([positions[g * pl.Bl + b, l * pl.T:l * pl.T + n] for b in range(pl.Bl)])


def call(basp, w, rotary, positions=None, interleaved=False, scaling="none", inverse=False, in_place=False, theta=10000.0):
    pl = make_plan(basp, w)
    g = torch.Generator().manual_seed(w.S + rotary)
    mk = lambda h: [torch.randn((pl.Bl * pl.rank_tokens(r), h, w.D), generator=g).to(torch.bfloat16) for r in range(pl.N)]
    q, k = mk(w.Hq), mk(w.Hkv)
    rope = basp.basp_rope_make(rotary, theta, interleaved, scaling, 8.0, 64.0)
    x = [[t.cuda() for t in s] for s in (q, k)]
    y = x if in_place else [[torch.full_like(t, float("nan")) for t in s] for s in x]
    pos = None if positions is None else torch.from_numpy(positions.astype(np.int32)).cuda()
    basp.basp_rope(pl, rope, *x, *y, positions=pos, inverse=inverse)
    f, size = oracle.rope_frequencies(rotary, theta, scaling, 8.0, 64.0)
    where = np.tile(np.arange(w.S), (w.B, 1)) if positions is None else positions
    for s, out in zip((q, k), y):
        for r in range(pl.N):
            args = (rows_of(pl, r, where), f, size, interleaved, inverse)
            want = oracle.rope_any(f64(s[r]), *args)
            mag = np.abs(f64(s[r]))
            pair = mag[..., :rotary].reshape(*mag.shape[:-1], rotary // 2, 2) if interleaved else \
                np.stack([mag[..., :rotary // 2], mag[..., rotary // 2:rotary]], -1)
            pair = np.repeat(pair.sum(-1), 2, -1) if interleaved else np.concatenate([pair.sum(-1)] * 2, -1)
            bound = 2.0 ** -8 * np.abs(want)
            bound[..., :rotary] += 2.0 ** -21 * size * pair
            bound[..., rotary:] = 0.0                                        # copied bit for bit
            assert (np.abs(f64(out[r]) - want) <= bound).all(), r
    return y


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("w", CASES, ids=lambda w: w.name)
def test_positions(basp, w, interleaved):
    rng = np.random.default_rng(w.S)
    call(basp, w, w.D, None, interleaved)
    pos = rng.integers(-50, 200, (w.B, w.S))
    call(basp, w, w.D, pos, interleaved, inverse=True)
    for rotary in sorted({16, max(16, w.D // 32 * 16)}):
        call(basp, w, rotary, pos, interleaved, in_place=True)


@pytest.mark.parametrize("scaling", ["linear", "yarn", "wavelength"])
def test_scalings(basp, scaling):
    w = CASES[6]
    for inverse in (False, True):
        call(basp, w, 64, np.random.default_rng(1).integers(0, 4000, (w.B, w.S)), False, scaling, inverse)


def test_far_positions(basp):
    """To the ends of int32: the oracle's own angle (a double's 2^-53 of it) is good to 2^-22 radian there."""
    w = CASES[3]
    rng = np.random.default_rng(2)
    call(basp, w, 32, rng.choice([-2 ** 31, 2 ** 31 - 1, 10 ** 9, -10 ** 6, 123456789], (w.B, w.S)), True)
    call(basp, w, 32, rng.integers(0, 2 ** 24, (w.B, w.S)), False, theta=500000.0)


def test_rotation_and_back(basp):
    """The gradient is the transpose: turning back gives the input within two roundings."""
    w = CASES[9]
    pl = make_plan(basp, w)
    g = torch.Generator(device="cuda").manual_seed(1)
    q, k = (torch.randn((19, h, 128), generator=g, device="cuda").to(torch.bfloat16) for h in (67, 1))
    pos = torch.randint(0, 10 ** 6, (1, 19), generator=g, device="cuda", dtype=torch.int32)
    rope = basp.basp_rope_make(96, 10000.0, True)
    a, b, c, d = (torch.empty_like(t) for t in (q, k, q, k))
    basp.basp_rope(pl, rope, [q], [k], [a], [b], positions=pos)
    basp.basp_rope(pl, rope, [a], [b], [c], [d], positions=pos, inverse=True)
    for x, y in ((q, c), (k, d)):
        size = x.float()[..., :96].unflatten(-1, (48, 2)).norm(dim=-1, keepdim=True).expand(-1, -1, -1, 2).flatten(-2)
        # each of the two roundings moves a feature by at most 2^-8 of the pair's length, and the turn mixes two of them
        assert ((x.float() - y.float())[..., :96].abs() <= 3 * 2.0 ** -8 * size).all() and torch.equal(x[..., 96:], y[..., 96:])


def test_past_two_billion_elements(basp):
    S, H = 66000, 256
    pl = basp.basp_plan_create(1, 1, S, H, 8, 128)
    q = torch.ones((S, H, 128), dtype=torch.bfloat16, device="cuda")
    k = torch.ones((S, 8, 128), dtype=torch.bfloat16, device="cuda")
    assert q.numel() > 2 ** 31
    basp.basp_rope(pl, basp.basp_rope_make(128), [q], [k], [q], [k])
    for r in (0, 1, S // 2, S - 1):
        want = oracle.rope_any(np.ones((1, 1, 128)), [r], oracle.rope_frequencies(128, 10000.0)[0])[0, 0]
        for t in (q[r, 0], q[r, -1], k[r, -1]):
            assert (np.abs(f64(t) - want) <= 2.0 ** -8 * np.abs(want) + 2.0 ** -20).all()
