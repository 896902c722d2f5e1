"""What the head norms, 8-bit checkpoints and language-model loss refuse, and the sizes they report: no GPU needed (every
refusal comes before the first launch; the addresses are made up)."""
import ctypes

import pytest
import torch

N = 4
P = lambda xs: (ctypes.c_void_p * len(xs))(*xs)


def table(base, step=0x1000000):
    return [base + i * step for i in range(N)]


@pytest.fixture
def plan(basp):
    return basp.basp_plan_create(N, 2, 1024, 8, 4, 64)            # K = 2, T = 512


def norm_args(basp, plan, **kw):
    a = dict(q=table(0x10_0000_0000), k=table(0x11_0000_0000), wq=0x12_0000_0000, wk=0x12_0000_1000, cos=0x13_0000_0000,
             sin=0x14_0000_0000, eps=1e-6, qo=table(0x15_0000_0000), ko=table(0x16_0000_0000))
    a.update(kw)
    return basp.lib.basp_qk_norm_rope(plan.handle, P(a["q"]), P(a["k"]), a["wq"], a["wk"], a["cos"], a["sin"], a["eps"],
                                      P(a["qo"]), P(a["ko"]), None)


def test_norm_rope_refusals(basp, plan):
    q, qo = table(0x10_0000_0000), table(0x15_0000_0000)
    assert basp.lib.basp_qk_norm_rope(None, *[None] * 6, 1e-6, None, None, None) == basp.BASP_ERR_NULL
    for name in ("wq", "wk", "cos", "sin"):
        assert norm_args(basp, plan, **{name: None}) == basp.BASP_ERR_NULL
    for name, base in (("q", 0x10), ("k", 0x11), ("qo", 0x15), ("ko", 0x16)):
        t = table(base << 32)
        assert norm_args(basp, plan, **{name: t[:3] + [None]}) == basp.BASP_ERR_NULL
        assert norm_args(basp, plan, **{name: t[:3] + [t[3] + 8]}) == basp.BASP_ERR_ALIGN
    assert norm_args(basp, plan, cos=0x13_0000_0002) == basp.BASP_ERR_ALIGN
    for eps in (0.0, -1e-6, float("nan"), float("inf")):
        assert norm_args(basp, plan, eps=eps) == basp.BASP_ERR_INVALID
    shard = 512 * 8 * 64 * 2
    assert norm_args(basp, plan, qo=[q[1]] + qo[1:]) == basp.BASP_ERR_ALIAS          # another rank's input
    assert norm_args(basp, plan, qo=[q[0] + 16] + qo[1:]) == basp.BASP_ERR_ALIAS     # its own, shifted
    assert norm_args(basp, plan, qo=[qo[0], qo[0] + shard - 16] + qo[2:]) == basp.BASP_ERR_ALIAS
    assert norm_args(basp, plan, ko=[q[0]] + table(0x16_0000_0000)[1:]) == basp.BASP_ERR_ALIAS
    odd = basp.basp_plan_create(N, 2, 1024, 8, 4, 40)
    wide = basp.basp_plan_create(N, 2, 1024, 8, 4, 256)
    assert norm_args(basp, odd) == norm_args(basp, wide) == basp.BASP_ERR_UNSUPPORTED


def test_norm_rope_bwd_refusals(basp, plan):
    need = basp.basp_qk_norm_rope_bwd_workspace_bytes(plan)
    assert need > 0 and need % 4 == 0 and basp.lib.basp_qk_norm_rope_bwd_workspace_bytes(None) == 0

    def call(**kw):
        a = dict(q=table(0x10_0000_0000), k=table(0x11_0000_0000), dy=table(0x15_0000_0000), dyk=table(0x16_0000_0000),
                 dq=table(0x17_0000_0000), dk=table(0x18_0000_0000), dwq=0x19_0000_0000, dwk=0x19_0000_1000,
                 ws=0x1a_0000_0000, n=need, eps=1e-6)
        a.update(kw)
        return basp.lib.basp_qk_norm_rope_bwd(plan.handle, P(a["q"]), P(a["k"]), 0x12_0000_0000, 0x12_0000_1000, 0x13_0000_0000,
                                              0x14_0000_0000, a["eps"], P(a["dy"]), P(a["dyk"]), P(a["dq"]), P(a["dk"]), a["dwq"],
                                              a["dwk"], a["ws"], a["n"], None)
    assert call(n=need - 1) == basp.BASP_ERR_WORKSPACE
    assert call(ws=None) == call(dwq=None) == call(dwk=None) == basp.BASP_ERR_NULL
    assert call(ws=0x1a_0000_0008) == call(dwq=0x19_0000_0002) == basp.BASP_ERR_ALIGN
    assert call(eps=0.0) == basp.BASP_ERR_INVALID
    assert call(dq=table(0x10_0000_0000)) == basp.BASP_ERR_ALIAS                     # the norm's inputs are still needed
    assert call(dwk=0x19_0000_0000) == call(dwq=0x1a_0000_0000) == basp.BASP_ERR_ALIAS


def test_checkpoint_sizes_and_refusals(basp, plan):
    for D, S, K in ((64, 1024, 2), (16, 203, 2), (96, 1021, 1)):
        pl = basp.basp_plan_create(2 * K, 2, S, 8, 4, D)
        for r in range(pl.N):
            T = pl.rank_tokens(r)
            up = lambda n: (n + 15) // 16 * 16
            want = 2 * (up(T * 8 * D) + up(T * 4 * D)) + 2 * (up(T * 8 * 4) + up(T * 4 * 4))
            assert basp.basp_ckpt_bytes(pl, r) == want
    assert basp.basp_ckpt_bytes(plan, -1) == basp.basp_ckpt_bytes(plan, N) == 0
    seq = [table(b << 32) for b in (0x10, 0x11, 0x12, 0x13)]
    ck = table(0x14_0000_0000)
    pack = lambda s, c: basp.lib.basp_ckpt_pack(plan.handle, *[P(t) for t in s], P(c), None)
    back = lambda c, h: basp.lib.basp_ckpt_reshard_s2h(plan.handle, P(c), *[P(t) for t in h], None)
    for i in range(4):
        bad = [list(t) for t in seq]
        bad[i][2] = None
        assert pack(bad, ck) == back(ck, bad) == basp.BASP_ERR_NULL
        bad[i][2] = seq[i][2] + 8
        assert pack(bad, ck) == back(ck, bad) == basp.BASP_ERR_ALIGN
    assert pack(seq, ck[:3] + [None]) == back(ck[:3] + [None], seq) == basp.BASP_ERR_NULL
    assert pack(seq, ck[:3] + [ck[3] + 8]) == basp.BASP_ERR_ALIGN
    assert pack(seq, [seq[0][0]] + ck[1:]) == back([seq[0][0]] + ck[1:], seq) == basp.BASP_ERR_ALIAS
    assert pack(seq, [ck[0], ck[0] + 16] + ck[2:]) == basp.BASP_ERR_ALIAS
    L = basp.lib
    assert L.basp_ckpt_pack(plan.handle, P(seq[0]), None, P(seq[2]), P(seq[3]), P(ck), None) == basp.BASP_ERR_NULL
    assert L.basp_ckpt_pack(plan.handle, *[P(t) for t in seq], None, None) == basp.BASP_ERR_NULL
    wide = basp.basp_plan_create(N, 2, 1024, 8, 4, 256)
    assert L.basp_ckpt_pack(wide.handle, *[P(t) for t in seq], P(ck), None) == basp.BASP_ERR_UNSUPPORTED
    # the layer's backward from checkpoints: the checks of the form on bf16 shards, then the checkpoints'
    lse, do, dq, dk, dv = (table(b << 32) for b in (0x15, 0x16, 0x17, 0x18, 0x19))
    need = basp.basp_layer_bwd_seq_workspace_bytes(plan)
    bwd = lambda c, n, scale: L.basp_layer_bwd_ckpt(plan.handle, P(c), P(lse), P(do), P(dq), P(dk), P(dv), 0x20_0000_0000, n, scale, None)
    assert bwd(ck, need - 1, 0.0) == basp.BASP_ERR_WORKSPACE
    assert bwd(ck, need, -1.0) == basp.BASP_ERR_INVALID
    assert bwd(ck[:3] + [None], need, 0.0) == basp.BASP_ERR_NULL


def loss_args(basp, plan, grad, hidden=256, vocab=1000, **kw):
    need = basp.basp_lm_loss_grad_workspace_bytes(plan, hidden, vocab) if grad else basp.basp_lm_loss_fwd_workspace_bytes(plan, vocab)
    a = dict(x=table(0x10_0000_0000), w=0x11_0000_0000, y=table(0x12_0000_0000), g=table(0x13_0000_0000), loss=table(0x14_0000_0000),
             lse=table(0x15_0000_0000), dx=table(0x16_0000_0000), dw=0x17_0000_0000, ws=0x18_0000_0000, n=need, piece=0)
    a.update(kw)
    t = lambda n: None if a[n] is None else P(a[n])
    if grad:
        return basp.lib.basp_lm_loss_grad(plan.handle, hidden, vocab, t("x"), a["w"], t("y"), t("g"), t("loss"), t("lse"), t("dx"),
                                          a["dw"], a["piece"], a["ws"], a["n"], None)
    return basp.lib.basp_lm_loss_fwd(plan.handle, hidden, vocab, t("x"), a["w"], t("y"), t("loss"), t("lse"), a["ws"], a["n"], None)


@pytest.mark.parametrize("grad", [False, True])
def test_loss_refusals(basp, plan, grad):
    call = lambda **kw: loss_args(basp, plan, grad, **kw)
    for name in ("x", "w", "y", "loss", "ws"):
        assert call(**{name: None}) == basp.BASP_ERR_NULL
    for name, base in (("x", 0x10), ("y", 0x12), ("loss", 0x14), ("lse", 0x15)):
        t = table(base << 32)
        assert call(**{name: t[:3] + [None]}) == basp.BASP_ERR_NULL
        assert call(**{name: t[:3] + [t[3] + 2]}) == basp.BASP_ERR_ALIGN
    assert call(w=0x11_0000_0008) == call(ws=0x18_0000_0008) == basp.BASP_ERR_ALIGN
    assert call(n=15) == basp.BASP_ERR_WORKSPACE
    assert call(hidden=0) == call(vocab=0) == call(hidden=-8) == basp.BASP_ERR_INVALID
    assert call(hidden=252) == call(hidden=65544) == call(vocab=(1 << 24) + 1) == basp.BASP_ERR_UNSUPPORTED
    assert call(loss=table(0x15_0000_0000)) == call(ws=0x11_0000_0000) == call(loss=table(0x10_0000_0000)) == basp.BASP_ERR_ALIAS
    if grad:
        assert call(dx=None, dw=None) == basp.BASP_ERR_NULL
        assert call(dx=table(0x10_0000_0000)) == call(dw=0x11_0000_0000) == basp.BASP_ERR_ALIAS
        assert call(g=table(0x13_0000_0000)[:3] + [None]) == basp.BASP_ERR_NULL
        assert call(piece=-1) == basp.BASP_ERR_INVALID
        assert call(piece=40000) == basp.BASP_ERR_UNSUPPORTED


def test_loss_workspace_sizes(basp, plan):
    one = basp.basp_lm_loss_grad_workspace_bytes(plan, 256, 1000)
    many = basp.basp_lm_loss_grad_workspace_bytes(plan, 256, 1000, piece_rows=128)
    assert one > 2048 * 1024 * 2                                    # 2048 rows, pitch 1024, 16 bits each, in one piece
    assert 1000 * 256 * 4 < many < one                              # pieces: a running sum of dw, fewer rows
    assert basp.basp_lm_loss_grad_workspace_bytes(plan, 256, 1000, piece_rows=1) == many
    assert basp.basp_lm_loss_grad_workspace_bytes(plan, 252, 1000) == basp.basp_lm_loss_grad_workspace_bytes(plan, 256, 0) == 0
    assert 0 < basp.basp_lm_loss_fwd_workspace_bytes(plan, 1000) < many
    big = basp.basp_plan_create(8, 1, 131072, 32, 8, 128)           # 128K tokens: bounded by the piece, not by the rows
    assert basp.basp_lm_loss_grad_workspace_bytes(big, 4096, 128256) < 6 << 30
    assert basp.basp_lm_loss_fwd_workspace_bytes(big, 128256) < 64 << 20


@pytest.mark.parametrize("rows,hidden,vocab", [(524416, 8192, 128256), (516224, 1024, 32000), (8193, 4096, 128256), (2043, 2560, 50257)])
def test_loss_workspace_is_what_the_header_says(basp, rows, hidden, vocab):
    """A short last piece splits its vocabulary often; its partial sums have its own rows, not a whole piece's."""
    pl = basp.basp_plan_create(1, 1, rows, 8, 8, 64)
    up = lambda n, m: (n + m - 1) // m * m
    piece = min(up(rows, 128), 8192)
    logits = piece * up(vocab, 256)
    several = rows > 8192
    least = logits * 2 + logits // 16 + piece * hidden * 2 + several * vocab * hidden * 4
    got = basp.basp_lm_loss_grad_workspace_bytes(pl, hidden, vocab)
    # 36 bytes a row for statistics of rows, sections on multiples of 256 bytes; several pieces share the rows evenly
    assert got <= least + 768e6 + piece * 36 + 8 * 256
    assert got >= least * (0.5 if several else 1.0)


def test_binding_refuses_tensors_it_would_misread(basp, plan):
    q = [torch.zeros((512, 8, 64), dtype=torch.bfloat16) for _ in range(N)]
    with pytest.raises(ValueError, match="q_seq"):
        basp.basp_qk_norm_rope(plan, [t.float() for t in q], q, None, None, None, None, q, q)
    with pytest.raises(ValueError, match="q_seq"):
        basp.basp_qk_norm_rope(plan, [t[:511] for t in q], q, None, None, None, None, q, q)
    with pytest.raises(ValueError, match="not contiguous"):
        basp.basp_ckpt_pack(plan, [t.transpose(0, 1) for t in q], q, q, q, q)
    with pytest.raises(ValueError, match="device memory"):
        basp.basp_ckpt_pack(plan, q, q, q, q, q)
    with pytest.raises(ValueError, match="expected 4 shards"):
        basp.basp_ckpt_pack(plan, q[:0], q, q, q, q)


def test_marshalling_passes_on_what_it_cannot_vouch_for(basp):
    """The quick look at a call's tensors answers with addresses or not at all; what it does not know (raw addresses, wrong
    tensors, wrong arguments) is left to the binding's own checks."""
    from paper_2609_03151_b200._marshal import addresses
    t = torch.zeros(8, dtype=torch.bfloat16)
    assert addresses(0, (("a", torch.bfloat16, [t], (8,)),)) is None                 # not in device memory
    assert addresses(0, (("a", torch.bfloat16, [123], (8,)),)) is None
    assert addresses(0, (("a", torch.bfloat16, [t, t], (8,)),)) is None
    assert addresses(0, (("a", torch.bfloat16, t, "8"),)) is None
    assert addresses(0, (("a", torch.bfloat16, None, (8,)), ("b", torch.float32, None, 3)))[1] == [None, None]
    assert addresses(0, ())[1] == []
    with pytest.raises(TypeError):
        addresses(0)
    m = basp._Marshal()
    table, one, none = m.addresses(("a", torch.bfloat16, [16, None, 48], (8, 8, 8)), ("b", torch.float32, 4096, 3), ("c", torch.int64, None, 1))
    assert list((ctypes.c_void_p * 3).from_address(table)) == [16, None, 48] and one == 4096 and none is None


def test_the_rotation_tables_are_not_differentiable():
    from paper_2609_03151_b200.autograd import basp_qk_norm_rope
    t = torch.zeros(4, 8)
    for cos, sin in ((t.clone().requires_grad_(), t), (t, t.clone().requires_grad_())):
        with pytest.raises(ValueError, match="not differentiable"):
            basp_qk_norm_rope(None, [], [], t, t, cos, sin)
