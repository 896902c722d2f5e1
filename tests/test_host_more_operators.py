"""What the masked attention, the rotation and the block norms refuse, the sizes they report and the frequencies that are made on the
host: no GPU needed (every refusal comes before the first launch; the addresses are made up)."""
import ctypes
import math
import os

import numpy as np
import pytest
import torch

import oracle
from paper_2609_03151_b200 import build

N = 4
P = lambda xs: None if xs is None else (ctypes.c_void_p * len(xs))(*xs)


def table(base, step=0x1000000):
    return [(base << 32) + i * step for i in range(N)]


@pytest.fixture
def plan(basp):
    return basp.basp_plan_create(N, 2, 1024, 8, 4, 64)            # K = 2, T = 512


def test_mask_sizes_and_refusals(basp, plan):
    need = basp.basp_mask_bytes(plan)
    # ranges, tiles, the tiles' sweeps, and the two lists of work items
    assert need == 2 * 1024 * 8 + 16 * 16 + 16 * 8 + 2 * 4 * 48 + 16 * 16 and basp.lib.basp_mask_bytes(None) == 0
    at, other, mask = 0x10_0000_0000, 0x11_0000_0000, 0x12_0000_0000
    ranges = lambda b=at, e=other, m=mask, n=need: basp.lib.basp_mask_ranges(plan.handle, b, e, m, n, None)
    packed = lambda pos=at, pre=other, window=0, m=mask, n=need, pl=plan: basp.lib.basp_mask_packed(pl.handle, pos, pre, window, m, n, None)
    assert basp.lib.basp_mask_ranges(None, at, other, mask, need, None) == basp.lib.basp_mask_packed(None, at, None, 0, mask, need, None) \
        == basp.BASP_ERR_NULL
    assert ranges(b=None) == ranges(e=None) == ranges(m=None) == packed(pos=None) == packed(m=None) == basp.BASP_ERR_NULL
    assert ranges(b=at + 2) == ranges(m=mask + 8) == packed(pre=other + 1) == basp.BASP_ERR_ALIGN
    assert ranges(n=need - 1) == packed(n=need - 1) == basp.BASP_ERR_WORKSPACE
    assert ranges(m=at) == packed(m=other) == basp.BASP_ERR_ALIAS
    assert packed(window=-1) == basp.BASP_ERR_INVALID
    assert packed(pl=basp.basp_plan_create(N, 2, 1024, 8, 4, 64, causal=False)) == basp.BASP_ERR_INVALID


def attn(basp, plan, softcap=0.0, slopes=None, mask=None, mask_bytes=0, scale=0.0, **kw):
    a = dict(q=table(0x10), k=table(0x11), v=table(0x12), o=table(0x13), lse=table(0x14))
    a.update(kw)
    return basp.lib.basp_attn_masked_fwd(plan.handle, ctypes.byref(basp._Score(softcap, slopes, mask, mask_bytes)), P(a["q"]), P(a["k"]),
                                         P(a["v"]), P(a["o"]), P(a["lse"]), scale, None)


def attn_bwd(basp, plan, bytes_less=0, **kw):
    a = dict(q=table(0x10), k=table(0x11), v=table(0x12), o=table(0x13), do=table(0x14), lse=table(0x15), dq=table(0x16), dk=table(0x17),
             dv=table(0x18), ws=0x19_0000_0000, softcap=0.0)
    a.update(kw)
    return basp.lib.basp_attn_masked_bwd(plan.handle, ctypes.byref(basp._Score(a["softcap"], None, None, 0)),
                                         *[P(a[n]) for n in ("q", "k", "v", "o", "do", "lse", "dq", "dk", "dv")], a["ws"],
                                         basp.basp_attn_masked_bwd_workspace_bytes(plan) - bytes_less, 0.0, None)


def test_masked_attention_refusals(basp, plan):
    need = basp.basp_mask_bytes(plan)
    assert basp.lib.basp_attn_masked_fwd(plan.handle, None, *[P(table(0x10))] * 5, 0.0, None) == basp.BASP_ERR_NULL
    for name, base in (("q", 0x10), ("k", 0x11), ("v", 0x12), ("o", 0x13)):
        t = table(base)
        assert attn(basp, plan, **{name: None}) == attn(basp, plan, **{name: t[:3] + [None]}) == basp.BASP_ERR_NULL
        assert attn(basp, plan, **{name: t[:3] + [t[3] + 8]}) == basp.BASP_ERR_ALIGN
    assert attn(basp, plan, lse=table(0x14)[:3] + [None]) == basp.BASP_ERR_NULL
    for cap in (-1.0, math.nan, math.inf, 1e13, 1e-13):
        assert attn(basp, plan, softcap=cap) == attn_bwd(basp, plan, softcap=cap) == basp.BASP_ERR_INVALID
    assert attn(basp, plan, softcap=1e9) == attn(basp, plan, softcap=1e-8) == attn(basp, plan, scale=-1.0) == basp.BASP_ERR_INVALID
    assert attn(basp, plan, slopes=0x20_0000_0002) == attn(basp, plan, mask=0x20_0000_0008, mask_bytes=need) == basp.BASP_ERR_ALIGN
    assert attn(basp, plan, mask=0x20_0000_0000, mask_bytes=need - 1) == basp.BASP_ERR_WORKSPACE
    assert attn(basp, plan, o=table(0x10)) == attn(basp, plan, o=table(0x11)) == attn(basp, plan, lse=table(0x13)) == basp.BASP_ERR_ALIAS
    assert attn(basp, plan, mask=table(0x13)[0], mask_bytes=need) == attn(basp, plan, slopes=table(0x14)[1]) == basp.BASP_ERR_ALIAS
    for D in (40, 144):
        assert attn(basp, basp.basp_plan_create(N, 2, 1024, 8, 4, D)) == basp.BASP_ERR_UNSUPPORTED
    for name, base in (("q", 0x10), ("o", 0x13), ("do", 0x14), ("lse", 0x15), ("dq", 0x16), ("dk", 0x17), ("dv", 0x18)):
        assert attn_bwd(basp, plan, **{name: None}) == attn_bwd(basp, plan, **{name: table(base)[:3] + [None]}) == basp.BASP_ERR_NULL
        assert attn_bwd(basp, plan, **{name: table(base)[:3] + [table(base)[3] + 4]}) == basp.BASP_ERR_ALIGN
    assert attn_bwd(basp, plan, bytes_less=1) == basp.BASP_ERR_WORKSPACE
    assert attn_bwd(basp, plan, ws=None) == basp.BASP_ERR_NULL
    assert attn_bwd(basp, plan, dq=table(0x10)) == attn_bwd(basp, plan, dk=table(0x18)) == attn_bwd(basp, plan, ws=table(0x17)[0]) == basp.BASP_ERR_ALIAS


def test_masked_layer_refusals(basp, plan):
    need = basp.basp_workspace_bytes(plan)
    score = ctypes.byref(basp._Score(0.0, None, None, 0))
    fwd = lambda ws=0x20_0000_0000, n=need, scale=0.0: basp.lib.basp_layer_masked_fwd(
        plan.handle, score, P(table(0x10)), P(table(0x11)), P(table(0x12)), P(table(0x13)), None, ws, n, scale, None)
    assert fwd(ws=None) == basp.BASP_ERR_NULL
    assert fwd(ws=0x20_0000_0008) == basp.BASP_ERR_ALIGN
    assert fwd(n=need - 1) == basp.BASP_ERR_WORKSPACE
    assert fwd(scale=-1.0) == basp.BASP_ERR_INVALID
    n = basp.basp_layer_masked_bwd_workspace_bytes(plan)
    assert n > basp.basp_attn_masked_bwd_workspace_bytes(plan) and basp.lib.basp_layer_masked_bwd_workspace_bytes(None) == 0
    bwd = lambda ws=0x20_0000_0000, n=n: basp.lib.basp_layer_masked_bwd(plan.handle, score, *[P(table(0x10 + i)) for i in range(9)], ws, n, 0.0, None)
    assert bwd(ws=None) == basp.BASP_ERR_NULL
    assert bwd(n=n - 1) == basp.BASP_ERR_WORKSPACE


def test_masked_layer_refuses_before_its_first_launch(basp, plan):
    """What the attention in the middle of the layer refuses, and what the exchange behind it would, is refused before the exchange in front of it
    (whose launch fails here, without a GPU, with another code); the score's tensors lie in nothing that the layer writes."""
    need, size = basp.basp_workspace_bytes(plan), basp.basp_mask_bytes(plan)
    ws, mask, slopes = 0x20_0000_0000, 0x21_0000_0000, 0x22_0000_0000

    def score(cap=0.0, slopes=None, mask=None, mask_bytes=size):
        return ctypes.byref(basp._Score(cap, slopes, mask, mask_bytes))

    def fwd(sc=score(), lse=table(0x14), **kw):
        a = dict(q=table(0x10), k=table(0x11), v=table(0x12), o=table(0x13))
        a.update(kw)
        return basp.lib.basp_layer_masked_fwd(plan.handle, sc, P(a["q"]), P(a["k"]), P(a["v"]), P(a["o"]), P(lse), ws, need, 0.0, None)

    bytes_bwd = basp.basp_layer_masked_bwd_workspace_bytes(plan)

    def bwd(sc=score(), **kw):
        a = {n: table(0x40 + i) for i, n in enumerate(("q", "k", "v", "o", "lse", "do", "dq", "dk", "dv"))}
        a.update(kw)
        return basp.lib.basp_layer_masked_bwd(plan.handle, sc, *[P(t) for t in a.values()], ws, bytes_bwd, 0.0, None)

    for call in (fwd, bwd):
        if not torch.cuda.is_available():
            assert call() == call(score(30.0, slopes, mask)) == basp.BASP_ERR_CUDA               # nothing to refuse: the launch
        assert call(None) == basp.BASP_ERR_NULL
        assert call(score(-1.0)) == call(score(math.nan)) == call(score(1e-13)) == basp.BASP_ERR_INVALID
        assert call(score(slopes=slopes + 2)) == call(score(mask=mask + 8)) == basp.BASP_ERR_ALIGN
        assert call(score(mask=mask, mask_bytes=size - 1)) == basp.BASP_ERR_WORKSPACE
        # in the workspace's first shard (an input of the attention) and in its last bytes
        n = need if call is fwd else bytes_bwd
        for at in (ws, ws + n - 16):
            assert call(score(mask=at)) == call(score(slopes=at)) == basp.BASP_ERR_ALIAS
        missing, odd = {"lse": table(0x14)[:3] + [None]}, {"lse": table(0x14)[:3] + [table(0x14)[3] + 2]}
        assert call(**missing) == basp.BASP_ERR_NULL and call(**odd) == basp.BASP_ERR_ALIGN
    outs = {fwd: {"o": 0x13}, bwd: {"dq": 0x46, "dk": 0x47, "dv": 0x48}}
    for call, named in outs.items():
        for name, base in named.items():
            t = table(base)
            assert call(**{name: None}) == call(**{name: t[:3] + [None]}) == basp.BASP_ERR_NULL
            assert call(**{name: t[:3] + [t[3] + 8]}) == basp.BASP_ERR_ALIGN
            assert call(score(mask=t[1] + 64)) == call(score(slopes=t[2])) == basp.BASP_ERR_ALIAS
    assert fwd(score(mask=table(0x14)[0])) == basp.BASP_ERR_ALIAS                                 # LSE is written too
    for name in ("q", "k", "v", "o"):
        assert bwd(**{name: table(0x10)[:3] + [None]}) == basp.BASP_ERR_NULL
    for D in (40, 144):
        other = basp.basp_plan_create(N, 2, 1024, 8, 4, D)
        assert basp.lib.basp_layer_masked_fwd(other.handle, score(), P(table(0x10)), P(table(0x11)), P(table(0x12)), P(table(0x13)), None, ws,
                                              basp.basp_workspace_bytes(other), 0.0, None) == basp.BASP_ERR_UNSUPPORTED


def test_score_structure(basp):
    """What the binding packs is the library's structure."""
    m = type("M", (), {"space": lambda self, mask: (0x1234567890, 77)})()
    packed = basp.basp_score(2.5, None, object()).pack(m, 0x9876543210)
    s = basp._Score.from_buffer_copy(packed)
    assert len(packed) == ctypes.sizeof(basp._Score) and (s.softcap, s.slopes, s.mask, s.mask_bytes) == (2.5, 0x9876543210, 0x1234567890, 77)


@pytest.mark.parametrize("scaling", ["none", "linear", "yarn", "wavelength"])
@pytest.mark.parametrize("rotary,theta,factor,trained", [(128, 500000.0, 16.0, 8192.0), (32, 10000.0, 1.0, 2048.0), (16, 10000.0, 40.0, 4096.0)])
def test_frequencies(basp, scaling, rotary, theta, factor, trained):
    t = basp.basp_rope_make(rotary, theta, scaling=scaling, factor=factor, original_len=trained)
    f, size = oracle.rope_frequencies(rotary, theta, scaling, factor, trained)
    got = np.array(list(t.turns[:rotary // 2]), dtype=np.float64) * 2.0 ** -64 * 2 * np.pi
    # half a step of 2^-64 turns (the lowest frequencies are 2^-25 of a turn: a relative 10^-12), the roundings of doubles, and of one float
    assert (np.abs(got - f) <= 2.0 ** -65 * 2 * np.pi + 1e-14 * f).all() and abs(t.factor - size) <= 2.0 ** -24 * size
    assert not any(t.turns[rotary // 2:]) and t.rotary_dim == rotary and t.interleaved == 0
    assert basp.basp_rope_make(rotary, theta, attention_factor=0.5).factor == 0.5


def test_rope_refusals(basp, plan):
    bad = lambda code, **kw: pytest.raises(basp.BaspError, match=r"\(%d\)" % code)
    for kw, code in (({"rotary_dim": 24}, basp.BASP_ERR_UNSUPPORTED), ({"rotary_dim": 144}, basp.BASP_ERR_UNSUPPORTED),
                     ({"theta": 1.0}, basp.BASP_ERR_INVALID), ({"theta": math.nan}, basp.BASP_ERR_INVALID),
                     ({"scaling": "linear", "factor": 0.5}, basp.BASP_ERR_INVALID), ({"scaling": "yarn", "factor": 4.0}, basp.BASP_ERR_INVALID),
                     ({"scaling": "wavelength", "factor": 4.0, "original_len": 100.0, "slow": 3.0, "fast": 2.0}, basp.BASP_ERR_INVALID),
                     ({"attention_factor": -1.0}, basp.BASP_ERR_INVALID)):
        with bad(code):
            basp.basp_rope_make(**{"rotary_dim": 64, **kw})
    with pytest.raises(ValueError):
        basp.basp_rope_make(64, scaling="ntk")
    assert basp.lib.basp_rope_make(None, None) == basp.BASP_ERR_NULL

    def call(rotary=64, pl=plan, **kw):
        a = dict(q=table(0x10), k=table(0x11), pos=0x12_0000_0000, qo=table(0x13), ko=table(0x14))
        a.update(kw)
        return basp.lib.basp_rope(pl.handle, ctypes.byref(basp.basp_rope_make(rotary)), P(a["q"]), P(a["k"]), a["pos"], 0, P(a["qo"]),
                                  P(a["ko"]), None)
    for name, base in (("q", 0x10), ("k", 0x11), ("qo", 0x13), ("ko", 0x14)):
        assert call(**{name: None}) == call(**{name: table(base)[:3] + [None]}) == basp.BASP_ERR_NULL
        assert call(**{name: table(base)[:3] + [table(base)[3] + 8]}) == basp.BASP_ERR_ALIGN
    assert call(pos=0x12_0000_0001) == basp.BASP_ERR_ALIGN
    assert call(rotary=80) == call(pl=basp.basp_plan_create(N, 2, 1024, 8, 4, 40)) == basp.BASP_ERR_UNSUPPORTED
    assert call(qo=[table(0x10)[1]] + table(0x13)[1:]) == call(ko=table(0x13)) == call(qo=table(0x11)) == basp.BASP_ERR_ALIAS
    assert call(qo=[table(0x10)[0] + 16] + table(0x13)[1:]) == call(pos=table(0x13)[2]) == basp.BASP_ERR_ALIAS


def test_block_norm_refusals(basp, plan):
    A = lambda n: (n << 32)

    def fwd(hidden=256, eps=1e-6, scale=1.0, **kw):
        a = dict(x=table(0x10), y=table(0x11), wp=A(0x12), g=A(0x13), wn=A(0x14), h=table(0x15), n=table(0x16))
        a.update(kw)
        return basp.lib.basp_block_norm(plan.handle, hidden, P(a["x"]), P(a["y"]), a["wp"], a["g"], a["wn"], scale, eps, P(a["h"]), P(a["n"]), None)
    assert fwd(x=None) == fwd(y=None) == fwd(h=None) == fwd(n=None) == fwd(wn=None) == basp.BASP_ERR_NULL
    assert fwd(y=None, h=None) == basp.BASP_ERR_NULL                                          # a gate without a block's output
    assert fwd(y=None, h=None, wp=None, g=None, wn=None, n=None) == basp.BASP_ERR_NULL        # nothing to do
    for name, base in (("x", 0x10), ("y", 0x11), ("h", 0x15), ("n", 0x16)):
        assert fwd(**{name: table(base)[:3] + [None]}) == basp.BASP_ERR_NULL
        assert fwd(**{name: table(base)[:3] + [table(base)[3] + 2]}) == basp.BASP_ERR_ALIGN
    assert fwd(wp=A(0x12) + 2) == fwd(g=A(0x13) + 8) == basp.BASP_ERR_ALIGN
    assert fwd(hidden=0) == fwd(hidden=-8) == basp.BASP_ERR_INVALID
    assert fwd(hidden=12) == fwd(hidden=16392) == basp.BASP_ERR_UNSUPPORTED
    for eps in (0.0, -1.0, math.nan, math.inf):
        assert fwd(eps=eps) == basp.BASP_ERR_INVALID
    assert fwd(scale=math.nan) == fwd(scale=math.inf) == basp.BASP_ERR_INVALID
    assert fwd(n=table(0x15)) == fwd(h=[table(0x10)[1]] + table(0x15)[1:]) == fwd(n=[table(0x11)[0] + 16] + table(0x16)[1:]) == basp.BASP_ERR_ALIAS
    assert fwd(wn=table(0x15)[0]) == basp.BASP_ERR_ALIAS

    need = basp.basp_block_norm_bwd_workspace_bytes(plan, 256)
    assert need > 0 and basp.basp_block_norm_bwd_workspace_bytes(plan, 12) == basp.lib.basp_block_norm_bwd_workspace_bytes(None, 256) == 0

    def bwd(n=need, **kw):
        a = dict(h=table(0x10), y=table(0x11), wp=A(0x12), g=A(0x13), wn=A(0x14), dh=table(0x15), dn=table(0x16), dx=table(0x17),
                 dy=table(0x18), dwp=A(0x19), dg=A(0x1a), dwn=A(0x1b), ws=A(0x1c))
        a.update(kw)
        return basp.lib.basp_block_norm_bwd(plan.handle, 256, P(a["h"]), P(a["y"]), a["wp"], a["g"], a["wn"], 1.0, 1e-6, P(a["dh"]), P(a["dn"]),
                                            P(a["dx"]), P(a["dy"]), a["dwp"], a["dg"], a["dwn"], a["ws"], n, None)
    for name in ("h", "y", "dn", "dx", "dy", "dwp", "dg", "dwn", "ws", "wp", "g", "wn"):
        assert bwd(**{name: None}) == basp.BASP_ERR_NULL, name
    assert bwd(dh=None, dn=None, wn=None, dwn=None) == basp.BASP_ERR_NULL                     # no gradient comes in
    assert bwd(n=need - 1) == basp.BASP_ERR_WORKSPACE
    assert bwd(dwp=A(0x19) + 2) == bwd(ws=A(0x1c) + 4) == basp.BASP_ERR_ALIGN
    assert bwd(dx=table(0x10)) == bwd(dx=table(0x11)) == bwd(dy=table(0x15)) == bwd(dy=table(0x17)) == bwd(dwp=A(0x1a)) == basp.BASP_ERR_ALIAS


def test_loads_of_what_an_overlapping_kernel_writes():
    """The forward kernels start under the launch before them, which may be the one that writes the mask object: no load of theirs is one
    that wants memory which nothing writes while the kernel runs."""
    for name in ("attn_masked_fwd.cu", "attn_shaped_fwd.cuh"):
        with open(os.path.join(build.CSRC, name)) as f:
            code = f.read()
        assert "__ldg" not in code and "ld.global.nc" not in code, name
        assert name != "attn_masked_fwd.cu" or "launch_early_smem(attn_masked_fwd_kernel" in code


def test_marshalling_refusals(basp, plan):
    """Tensors that the library would misread are refused before it sees them."""
    cpu = lambda *s, dtype=torch.bfloat16: torch.zeros(s, dtype=dtype)
    with pytest.raises(ValueError):
        basp.basp_mask_packed(plan, cpu(2, 1024, dtype=torch.int64), cpu(basp.basp_mask_bytes(plan), dtype=torch.uint8))
    with pytest.raises(ValueError):
        basp.basp_rope(plan, basp.basp_rope_make(64), [cpu(512, 8, 64)] * 3, [cpu(512, 4, 64)] * 4, [cpu(512, 8, 64)] * 4, [cpu(512, 4, 64)] * 4)
    with pytest.raises(ValueError):
        basp.basp_block_norm(plan, 64, [cpu(512, 64)] * 4, [cpu(512, 64)] * 4, [cpu(512, 64)] * 4, [cpu(512, 32)] * 4, w_pre=cpu(64))
