"""Head norms, checkpoints and loss as programs call them: captured into CUDA graphs and replayed on new inputs, on two streams at
once, on raw addresses, with graphs that share nothing; and the ends of their ranges (no token with a label, weights all zero,
the same label everywhere)."""
import numpy as np
import pytest
import torch

import oracle
from helpers import make_plan
from paper_2609_03151_b200 import synth

pytestmark = pytest.mark.gpu


def capture(call):
    """The call as a graph, after an eager run."""
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        call()
    return graph


def normal(g, *shape):
    return torch.randn(shape, generator=g, device="cuda").to(torch.bfloat16)


@pytest.mark.parametrize("op", ["norm_bwd", "ckpt", "loss"])
def test_two_graphs_and_eager(basp, op):
    """Two graphs of the same operator with workspaces of their own, replayed in turn on inputs written after the capture, give the
    eager results bit for bit (the layer backward's dQ: the attention's own reduction order, within its rounding)."""
    w = synth.Workload("g", N=4, B=2, S=512, Hq=4, Hkv=2, D=128)
    pl = make_plan(basp, w)
    g = torch.Generator(device="cuda").manual_seed(1)
    rows, T = 4, 256
    cos, sin = (t.t().contiguous().cuda() for t in synth.rope_tables(512, 128))

    def make():
        if op == "norm_bwd":
            ins = [normal(g, T, h, 128) for h in (4,) * 4 + (2,) * 4 + (4,) * 4 + (2,) * 4] + [normal(g, 128) for _ in range(2)]
            outs = [torch.empty_like(t) for t in ins[8:16]] + [torch.empty(128, device="cuda") for _ in range(2)]
            ws = torch.empty(basp.basp_qk_norm_rope_bwd_workspace_bytes(pl), dtype=torch.uint8, device="cuda")
            return ins, outs, lambda: basp.basp_qk_norm_rope_bwd(pl, ins[:4], ins[4:8], ins[16], ins[17], cos, sin, ins[8:12],
                                                                 ins[12:16], outs[:4], outs[4:8], outs[8], outs[9], ws)
        if op == "ckpt":
            ins = [normal(g, T, h, 128) for h in (4,) * 4 + (2,) * 8 + (4,) * 8]
            ck = [torch.empty(basp.basp_ckpt_bytes(pl, r), dtype=torch.uint8, device="cuda") for r in range(4)]
            lse = [torch.full((1, 2, 512), 3.0, device="cuda") for _ in range(4)]
            outs = [torch.empty_like(t) for t in ins[:12]]
            ws = torch.empty(basp.basp_layer_bwd_seq_workspace_bytes(pl), dtype=torch.uint8, device="cuda")

            def call():
                basp.basp_ckpt_pack(pl, ins[:4], ins[4:8], ins[8:12], ins[12:16], ck)
                basp.basp_layer_bwd_ckpt(pl, ck, lse, ins[16:], outs[:4], outs[4:8], outs[8:], ws)
            return ins, outs, call
        ins = [normal(g, T, 128) for _ in range(4)] + [(torch.randn((900, 128), generator=g, device="cuda") * 0.1).to(torch.bfloat16)]
        labels = [torch.randint(0, 900, (T,), generator=g, device="cuda") for _ in range(4)]
        outs = [torch.empty(T, device="cuda") for _ in range(8)] + [torch.empty_like(t) for t in ins]
        ws = torch.empty(basp.basp_lm_loss_grad_workspace_bytes(pl, 128, 900, 512), dtype=torch.uint8, device="cuda")
        return ins, outs, lambda: basp.basp_lm_loss_grad(pl, 128, 900, ins[:4], ins[4], labels, None, outs[:4], outs[4:8], outs[8:12],
                                                         outs[12], ws, piece_rows=512)
    basp.basp_clear_status()
    sets = [make(), make()]
    graphs = [capture(call) for _, _, call in sets]
    for ins, outs, _ in sets:
        for t in ins:
            t.copy_(normal(g, *t.shape) * 0.3)
        for t in outs:
            t.fill_(float("nan"))
    for _ in range(2):
        for graph in graphs:
            graph.replay()
    torch.cuda.synchronize()
    basp.basp_get_status()
    for ins, outs, call in sets:
        got = [t.clone() for t in outs]
        for t in outs:
            t.fill_(float("nan"))
        call()
        for i, (a, b) in enumerate(zip(got, outs)):
            if op == "ckpt" and i < 4:
                assert (a.float() - b.float()).abs().max().item() <= 2e-2 + 2.0 ** -7 * b.float().abs().max().item()
            else:
                assert torch.equal(a, b), i


def test_captured_training_step(basp):
    """Head norms, attention with checkpoints and the loss, forward and backward by torch's autograd, captured as one graph and
    replayed on new inputs: the gradients of an eager step on them."""
    from paper_2609_03151_b200.autograd import basp_attention, basp_lm_loss, basp_qk_norm_rope
    pl = basp.basp_plan_create(4, 2, 256, 4, 2, 128)
    g = torch.Generator(device="cuda").manual_seed(7)
    tables = [t.t().contiguous().cuda() for t in synth.rope_tables(256, 128)]
    labels = [torch.randint(0, 500, (128,), generator=g, device="cuda") for _ in range(4)]
    weight = [torch.full((128,), 1.0 / 512, device="cuda") for _ in range(4)]
    make = lambda: [normal(g, 128, h, 128) for h in (4,) * 4 + (2,) * 8] + [normal(g, 128) * 0.1 + 1, normal(g, 128) * 0.1 + 1,
                                                                             normal(g, 500, 512) * 0.05]
    leaves = [t.to(torch.bfloat16).requires_grad_() for t in make()]

    def step():
        q, k = basp_qk_norm_rope(pl, leaves[:4], leaves[4:8], leaves[12], leaves[13], *tables)
        o = basp_attention(pl, q, k, leaves[8:12], fused=True, checkpoint8=True)
        loss = basp_lm_loss(pl, [t.reshape(128, 512) for t in o], leaves[14], labels, weight)
        loss.backward()
        return loss.detach()

    basp.basp_clear_status()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    for t in leaves:
        t.grad = None
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        loss = step()
    fresh = make()
    with torch.no_grad():
        for t, f in zip(leaves, fresh):
            t.copy_(f)
    graph.replay()
    torch.cuda.synchronize()
    got, got_loss = [t.grad.clone() for t in leaves], loss.clone()
    for t in leaves:
        t.grad = None
    eager_loss = step()
    basp.basp_get_status()
    assert torch.equal(got_loss, eager_loss)
    for i, (a, t) in enumerate(zip(got, leaves)):
        off = (a.float() - t.grad.float()).norm() / t.grad.float().norm()
        assert off <= 2.0 ** -8, (i, off.item())          # dQ comes from a reduction in whatever order its blocks finish


def test_two_streams_at_once(basp):
    """Two losses of different sizes on two streams, a dozen times over, against each alone."""
    g = torch.Generator(device="cuda").manual_seed(2)
    jobs = []
    for S, hidden, vocab in ((700, 256, 3000), (90, 512, 5000)):
        pl = basp.basp_plan_create(2, 1, S, 8, 8, 64)
        rows = [pl.rank_tokens(r) for r in range(2)]
        x = [normal(g, n, hidden) for n in rows]
        w = (torch.randn((vocab, hidden), generator=g, device="cuda") * hidden ** -0.5).to(torch.bfloat16)
        y = [torch.randint(0, vocab, (n,), generator=g, device="cuda") for n in rows]
        ws = torch.empty(basp.basp_lm_loss_grad_workspace_bytes(pl, hidden, vocab), dtype=torch.uint8, device="cuda")
        make = lambda rows=rows, x=x, w=w: ([torch.empty(n, device="cuda") for n in rows], [torch.empty_like(t) for t in x], torch.empty_like(w))
        call = lambda o, stream, pl=pl, hidden=hidden, vocab=vocab, x=x, w=w, y=y, ws=ws: basp.basp_lm_loss_grad(
            pl, hidden, vocab, x, w, y, None, o[0], None, o[1], o[2], ws, stream=stream)
        jobs.append((make, call))
    basp.basp_clear_status()
    alone = []
    for make, call in jobs:
        o = make()
        call(o, None)
        alone.append(o)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in jobs]
    out = [make() for make, _ in jobs]
    torch.cuda.synchronize()
    for _ in range(12):
        for (_, call), o, s in zip(jobs, out, streams):
            call(o, s)
    torch.cuda.synchronize()
    basp.basp_get_status()
    for a, b in zip(alone, out):
        assert all(torch.equal(p, q) for p, q in zip(a[0] + a[1] + [a[2]], b[0] + b[1] + [b[2]]))


def test_raw_addresses(basp):
    w = synth.Workload("raw", N=2, B=2, S=64, Hq=2, Hkv=2, D=64)
    pl = make_plan(basp, w)
    g = torch.Generator(device="cuda").manual_seed(3)
    q, k = ([normal(g, 64, 2, 64) for _ in range(2)] for _ in range(2))
    wq = normal(g, 64)
    tables = [t.t().contiguous().cuda() for t in synth.rope_tables(64, 64)]
    outs = [[[torch.empty_like(t) for t in x] for x in (q, k)] for _ in range(2)]
    basp.basp_qk_norm_rope(pl, q, k, wq, wq, *tables, *outs[0])
    at = lambda ts: [t.data_ptr() for t in ts]
    basp.basp_qk_norm_rope(pl, at(q), basp.as_shards(at(k)), wq.data_ptr(), wq, *[t.data_ptr() for t in tables], at(outs[1][0]), at(outs[1][1]))
    for a, b in zip(outs[0], outs[1]):
        assert all(torch.equal(x, y) for x, y in zip(a, b))


@pytest.mark.parametrize("case", ["no_labels", "zero_weights", "one_label", "one_row_counts"])
def test_ends_of_the_loss(basp, case):
    pl = basp.basp_plan_create(2, 1, 300, 8, 8, 64)
    hidden, vocab = 128, 700
    g = torch.Generator().manual_seed(4)
    x = [synth.randn_bf16(g, (150, hidden)) for _ in range(2)]
    w = (torch.randn((vocab, hidden), generator=g) / hidden ** 0.5).to(torch.bfloat16)
    y = [torch.randint(0, vocab, (150,), generator=g) for _ in range(2)]
    wt = [torch.rand(150, generator=g) for _ in range(2)]
    if case == "no_labels":
        y = [torch.full_like(t, -100) for t in y]
    elif case == "zero_weights":
        wt = [torch.zeros_like(t) for t in wt]
    elif case == "one_label":
        y = [torch.full_like(t, vocab - 1) for t in y]           # every row adds to the same word's gradient
    else:
        y = [torch.full_like(t, -1) for t in y]
        y[1][149] = 0
    c = lambda ts: [t.cuda() for t in ts]
    loss, lse = ([torch.full((150,), float("nan"), device="cuda") for _ in range(2)] for _ in range(2))
    dx, dw = [torch.full_like(t, float("nan")) for t in c(x)], torch.full_like(w, float("nan")).cuda()
    ws = torch.full((basp.basp_lm_loss_grad_workspace_bytes(pl, hidden, vocab),), 255, dtype=torch.uint8, device="cuda")
    basp.basp_clear_status()
    basp.basp_lm_loss_grad(pl, hidden, vocab, c(x), w.cuda(), c(y), c(wt), loss, lse, dx, dw, ws)
    basp.basp_get_status()
    f64 = lambda t: t.double().cpu().numpy()
    ref = oracle.lm_loss(f64(torch.cat(x)), f64(w), torch.cat(y).numpy(), f64(torch.cat(wt)))
    tz = (hidden / 16 + 16) * 2.0 ** -23 * (np.abs(f64(torch.cat(x))) @ np.abs(f64(w)).T).max()      # of a logit
    assert (np.abs(f64(torch.cat(loss)) - ref["loss"]) <= 2 * tz + 2.0 ** -20 * (1 + np.abs(ref["lse"]))).all()
    assert (np.abs(f64(torch.cat(lse)) - ref["lse"]) <= 2 * tz + 2.0 ** -20 * (1 + np.abs(ref["lse"]))).all()
    for got, want in ((f64(torch.cat(dx)), ref["dx"]), (f64(dw), ref["dw"])):
        if case in ("no_labels", "zero_weights"):
            assert (got == 0).all()
        else:
            assert np.linalg.norm(got - want) <= 2.0 ** -8 * np.linalg.norm(want)


def test_second_derivatives_are_refused(basp):
    from paper_2609_03151_b200.autograd import basp_lm_loss
    pl = basp.basp_plan_create(1, 1, 8, 1, 1, 64)
    g = torch.Generator(device="cuda").manual_seed(5)
    x, w = normal(g, 8, 64).requires_grad_(), normal(g, 100, 64)
    loss = basp_lm_loss(pl, [x], w, [torch.zeros(8, dtype=torch.int64, device="cuda")])
    (dx,) = torch.autograd.grad(loss, x, create_graph=True)
    with pytest.raises(RuntimeError):
        dx.float().sum().backward()


@pytest.mark.parametrize("op", ["attention", "attention fused", "attention checkpoint8", "head norms"])
def test_no_second_derivative_is_lost(basp, op):
    """The gradients carry no graph of their own: asking for one through them is refused, and not answered with the other paths'
    terms alone (here a penalty on the gradient beside the loss itself)."""
    from paper_2609_03151_b200.autograd import basp_attention, basp_qk_norm_rope
    pl = basp.basp_plan_create(2, 1, 256, 2, 2, 64)           # 128 tokens per rank: the fused form's unit
    g = torch.Generator(device="cuda").manual_seed(6)
    leaves = [normal(g, 128, 2, 64).requires_grad_() for _ in range(6)]
    one = torch.ones(64, dtype=torch.bfloat16, device="cuda")
    tables = [t.t().contiguous().cuda() for t in synth.rope_tables(256, 64)]

    def call(x):
        if op == "head norms":
            return sum(basp_qk_norm_rope(pl, x[:2], x[2:4], one, one, *tables), [])
        return basp_attention(pl, x[:2], x[2:4], x[4:], fused=op != "attention", checkpoint8="8" in op)
    x = [t * 1.5 for t in leaves]                          # a graph of its own in front of the operation
    loss = sum(t.float().square().sum() for t in call(x))
    (dx,) = torch.autograd.grad(loss, leaves[0], create_graph=True)
    with pytest.raises(RuntimeError, match="once_differentiable"):
        (dx.float().square().sum() + loss).backward()
