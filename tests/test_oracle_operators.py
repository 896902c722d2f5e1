"""Pins of the oracle's head norms, 8-bit codes and language-model loss: against difference quotients, known cases and
loops over single elements."""
import numpy as np
import pytest

import oracle
from paper_2609_03151_b200 import synth


def quotient(f, x, at, h=1e-5):
    hi, lo = x.copy(), x.copy()
    hi[at] += h
    lo[at] -= h
    return (f(hi) - f(lo)) / (2 * h)


@pytest.mark.parametrize("D", [16, 80, 128])
def test_norm_rope_gradients_against_differences(D):
    rng = np.random.default_rng(D)
    x, dy, w = rng.normal(size=(3, 2, D)), rng.normal(size=(3, 2, D)), 1 + 0.2 * rng.normal(size=D)
    cos, sin = (t.numpy().astype(np.float64) for t in synth.rope_tables(7, D))
    pos = np.array([0, 3, 6])
    dx, dw = oracle.qk_norm_rope_bwd(x, w, cos, sin, pos, 1e-3, dy)
    for at in [(0, 0, 0), (1, 1, D // 2), (2, 0, D - 1), (2, 1, D // 2 - 1)]:
        want = quotient(lambda v: (oracle.qk_norm_rope(v, w, cos, sin, pos, 1e-3) * dy).sum(), x, at)
        assert abs(dx[at] - want) < 1e-7 * (1 + abs(want))
    for j in (0, D // 2, D - 1):
        want = quotient(lambda v: (oracle.qk_norm_rope(x, v, cos, sin, pos, 1e-3) * dy).sum(), w, j)
        assert abs(dw[j] - want) < 1e-7 * (1 + abs(want))


def test_norm_of_known_vectors():
    cos, sin = np.ones((1, 8)), np.zeros((1, 8))                 # no turn
    x = np.full((1, 1, 16), 3.0)
    assert np.allclose(oracle.qk_norm_rope(x, np.ones(16), cos, sin, [0], 0.0), 1.0)
    assert np.allclose(oracle.qk_norm_rope(0 * x, np.ones(16), cos, sin, [0], 1e-6), 0.0)


def test_codes_by_elements():
    rng = np.random.default_rng(3)
    x = synth.from_bits(synth.bits(synth.randn_bf16(__import__("torch").Generator().manual_seed(1), (5, 3, 16)))).float().numpy()
    x[0, 0] = 0.0
    x[0, 1] = 2.0 ** -101
    x[1, 0, 5] = np.inf
    x[1, 1, 6] = np.nan
    codes, scales = oracle.ckpt_codes(x)
    back = oracle.ckpt_values(codes, scales)
    assert (back[0, :2] == 0).all() and np.isnan(back[1, :2]).all()
    for t, h in [(2, 0), (3, 2), (4, 1)]:
        top = max(abs(float(v)) for v in x[t, h])
        assert max(abs(int(c)) for c in codes[t, h]) == 127
        assert all(abs(float(b) - float(v)) <= top / 127 * 0.500001 for b, v in zip(back[t, h], x[t, h]))


def test_gradients_at_given_values_reduce_to_the_attention_backward():
    w = synth.Workload("g", N=1, B=1, S=24, Hq=4, Hkv=2, D=16)
    ts = synth.make_qkv(w, 2, with_dO=True)
    bits = [synth.bits(t) for t in ts]
    q, k, v, do = (oracle.bf16_bits_to_f64(b)[0] for b in bits)
    O, lse = oracle.attn_fwd(bits[0], bits[1], bits[2])
    want = oracle.attn_bwd(*bits)
    got = oracle.attn_bwd_given(q, k, v, O[0], lse[0], do)
    for n in ("dQ", "dK", "dV"):
        assert np.abs(got[n] - want[n][0]).max() < 1e-10


def test_loss_against_differences_and_known_cases():
    rng = np.random.default_rng(5)
    x, w = rng.normal(size=(4, 6)), rng.normal(size=(9, 6))
    labels, g = np.array([0, 8, -100, 9]), np.array([0.5, 2.0, 3.0, 1.0])
    r = oracle.lm_loss(x, w, labels, g)
    assert (r["loss"][2:] == 0).all() and (r["dx"][2:] == 0).all()      # no label; label beyond the vocabulary
    f = lambda a, b: (oracle.lm_loss(a, b, labels)["loss"] * g).sum()
    for at in [(0, 0), (1, 5), (2, 3)]:
        assert abs(r["dx"][at] - quotient(lambda v: f(v, w), x, at)) < 1e-8
    for at in [(0, 0), (8, 5), (4, 2)]:
        assert abs(r["dw"][at] - quotient(lambda v: f(x, v), w, at)) < 1e-8
    flat = oracle.lm_loss(np.zeros((2, 6)), w, np.array([1, 2]), np.ones(2))
    assert np.allclose(flat["loss"], np.log(9)) and np.allclose(flat["dz"][0], np.where(np.arange(9) == 1, 1 / 9 - 1, 1 / 9))
    one = oracle.lm_loss(x, w[:1], np.zeros(4, dtype=int), np.ones(4))
    assert np.allclose(one["loss"], 0) and np.allclose(one["dx"], 0)
