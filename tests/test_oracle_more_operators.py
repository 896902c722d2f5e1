"""Pins of the oracle's masked and shaped attention, rotations of any positions and block norms: against loops over single elements,
known cases and difference quotients."""
import math

import numpy as np
import pytest

import oracle
from paper_2609_03151_b200 import synth


def quotient(f, x, at, h=1e-5):
    hi, lo = x.copy(), x.copy()
    hi[at] += h
    lo[at] -= h
    return (f(hi) - f(lo)) / (2 * h)


def test_packed_ranges_of_a_known_batch():
    pos = np.array([[0, 1, 2, 0, 1, -1]])
    begin, end = oracle.packed_ranges(pos)
    assert begin.tolist() == [[0, 0, 0, 3, 3, 0]] and end.tolist() == [[1, 2, 3, 4, 5, 0]]
    begin, end = oracle.packed_ranges(pos, np.array([[2, 2, 2, 1, 1, 0]]))
    assert end.tolist() == [[2, 2, 3, 4, 5, 0]]
    begin, end = oracle.packed_ranges(pos, None, 2)
    assert begin.tolist() == [[0, 0, 1, 3, 3, 0]]


def test_shaped_attention_by_elements():
    rng = np.random.default_rng(0)
    S, H, D, cap = 7, 4, 16, 3.0
    q, k, v = rng.normal(size=(S, H, D)), rng.normal(size=(S, 2, D)), rng.normal(size=(S, 2, D))
    begin, end = rng.integers(0, S, S), rng.integers(0, S + 1, S)
    begin[3], end[3] = 2, 2
    slopes = np.array([0.5, 0.25, 0.0, 1.0])
    out = oracle.attn_shaped(q, k, v, begin, end, cap, slopes)
    for i in range(S):
        for h in range(H):
            keys = range(int(begin[i]), int(end[i]))
            w = [math.exp(cap * math.tanh(q[i, h] @ k[j, h // 2] / math.sqrt(D) / cap) - slopes[h] * abs(i - j)) for j in keys]
            want = sum(a * v[j, h // 2] for a, j in zip(w, keys)) / sum(w) if w else np.zeros(D)
            assert np.allclose(out["o"][i, h], want)
            assert np.isclose(out["lse"][h, i], math.log(sum(w))) if w else out["lse"][h, i] == -np.inf


def test_shaped_attention_reduces_to_the_causal_one():
    w = synth.Workload("r", N=1, B=1, S=20, Hq=4, Hkv=2, D=16)
    ts = synth.make_qkv(w, 2, with_dO=True)
    bits = [synth.bits(t) for t in ts]
    q, k, v, do = (oracle.bf16_bits_to_f64(b)[0] for b in bits)
    O, lse = oracle.attn_fwd(bits[0], bits[1], bits[2])
    out = oracle.attn_shaped(q, k, v, np.zeros(20, dtype=int), np.arange(20) + 1, do=do)
    assert np.allclose(out["o"], O[0]) and np.allclose(out["lse"], lse[0])
    ref = oracle.attn_bwd(*bits)
    dq, dk, dv = ref["dQ"], ref["dK"], ref["dV"]
    assert np.allclose(out["dq"], dq[0]) and np.allclose(out["dk"], dk[0]) and np.allclose(out["dv"], dv[0])
    given = oracle.attn_shaped(q, k, v, np.zeros(20, dtype=int), np.arange(20) + 1, do=do, given=(O[0], lse[0]))
    assert np.allclose(given["dq"], dq[0]) and np.allclose(given["dk"], dk[0])


@pytest.mark.parametrize("cap,bias", [(0.0, False), (2.0, False), (0.0, True), (1.0, True)])
def test_shaped_gradients_against_differences(cap, bias):
    rng = np.random.default_rng(1)
    S, H, D = 9, 4, 16
    x = {"q": rng.normal(size=(S, H, D)), "k": rng.normal(size=(S, 2, D)), "v": rng.normal(size=(S, 2, D))}
    do = rng.normal(size=(S, H, D))
    begin = np.array([0, 0, 0, 3, 3, 0, 5, 5, 0])
    end = np.array([3, 3, 3, 4, 6, 0, 9, 8, 9])
    slopes = np.array([0.5, 0.1, 0.7, 0.0]) if bias else None
    out = oracle.attn_shaped(x["q"], x["k"], x["v"], begin, end, cap, slopes, do=do)
    for n in "qkv":
        for at in [(0, 0, 0), (4, 1, 7), (8, 0, 15), (5, 1, 3)]:
            f = lambda t: (oracle.attn_shaped(*(t if m == n else x[m] for m in "qkv"), begin, end, cap, slopes)["o"] * do).sum()
            want = quotient(f, x[n], at)
            assert abs(out["d" + n][at] - want) < 1e-7 * (1 + abs(want))


def test_frequencies_of_known_cases():
    f, size = oracle.rope_frequencies(64, 10000.0)
    assert np.allclose(f[:2], [1.0, 10000.0 ** (-1 / 32)]) and size == 1.0
    assert np.allclose(oracle.rope_frequencies(64, 10000.0, "linear", 4.0)[0], f / 4)
    for scaling in ("yarn", "wavelength"):
        g, size = oracle.rope_frequencies(128, 500000.0, scaling, 8.0, 8192.0)
        base = oracle.rope_frequencies(128, 500000.0)[0]
        assert g[0] == base[0] and np.isclose(g[-1], base[-1] / 8) and (np.diff(g) < 0).all()
        assert np.isclose(size, 0.1 * math.log(8) + 1 if scaling == "yarn" else 1.0)


@pytest.mark.parametrize("interleaved", [False, True])
def test_rotation_keeps_lengths_and_turns_back(interleaved):
    rng = np.random.default_rng(2)
    x, pos = rng.normal(size=(5, 3, 48)), np.array([0, 1, 77, -3, 100000])
    f, _ = oracle.rope_frequencies(32, 10000.0)
    y = oracle.rope_any(x, pos, f, 1.0, interleaved)
    assert np.array_equal(y[0], x[0]) and np.array_equal(y[..., 32:], x[..., 32:])
    assert np.allclose(np.linalg.norm(y, axis=-1), np.linalg.norm(x, axis=-1))
    assert np.allclose(oracle.rope_any(y, pos, f, 1.0, interleaved, inverse=True), x)
    # a score depends on the distance alone
    a, b = (oracle.rope_any(x[:1], [p], f, 1.0, interleaved) for p in (10, 1010))
    c, d = (oracle.rope_any(x[1:2], [p], f, 1.0, interleaved) for p in (3, 1003))
    assert np.allclose((a * c).sum(-1), (b * d).sum(-1))
    if not interleaved:
        tables = [t.numpy().astype(np.float64) for t in synth.rope_tables(90, 32)]
        assert np.allclose(oracle.rope(x[:3, :, :32], *tables, [0, 1, 77]),
                           oracle.rope_any(x[:3, :, :32], [0, 1, 77], oracle.rope_frequencies(32, synth_base(tables))[0]), atol=1e-5)


def synth_base(tables):
    """The base of synth's tables from the second pair's angle at position 1."""
    return float(math.atan2(tables[1][1, 1], tables[0][1, 1]) ** -16)


@pytest.mark.parametrize("post,gated,pre", [(1, 1, 1), (1, 0, 1), (0, 1, 1), (0, 0, 1), (1, 1, 0), (0, 0, 0)])
def test_block_norm_gradients_against_differences(post, gated, pre):
    rng = np.random.default_rng(3)
    x, y = rng.normal(size=(4, 24)), 2 * rng.normal(size=(4, 24))
    w = [1 + 0.2 * rng.normal(size=24) if on else None for on in (post, gated, pre)]
    dh, dn = rng.normal(size=(4, 24)), rng.normal(size=(4, 24)) if pre else None

    def loss(x, y, *w):
        h, n = oracle.block_norm(x, y, *w, 0.7, 1e-3)
        return (h * dh).sum() + (0.0 if n is None else (n * dn).sum())
    h, _ = oracle.block_norm(x, y, *w, 0.7, 1e-3)
    out = oracle.block_norm_bwd(h, y, *w, 0.7, 1e-3, dh, dn)
    for at in [(0, 0), (3, 23), (1, 11)]:
        assert abs(out["dx"][at] - quotient(lambda t: loss(t, y, *w), x, at)) < 1e-6
        assert abs(out["dy"][at] - quotient(lambda t: loss(x, t, *w), y, at)) < 1e-6
    for i, n in enumerate(("dw_post", "dgate", "dw_pre")):
        assert (n in out) == (w[i] is not None)
        if n in out:
            for j in (0, 7, 23):
                assert abs(out[n][j] - quotient(lambda t: loss(x, y, *(t if m == i else w[m] for m in range(3))), w[i], j)) < 1e-6
