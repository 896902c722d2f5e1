"""A block of a model trained on packed documents: norms, rotation, masked attention together through torch's autograd, against the same
block written out in fp64; captured into graphs, on two streams at once, on raw addresses, and what autograd refuses."""
import pytest
import torch

import oracle

pytestmark = pytest.mark.gpu

PLAN = (4, 2, 210, 4, 2, 64)          # ranks, sequences, tokens (105 per rank), heads, key heads, head dimension
HIDDEN = 256


def positions():
    """Packed documents of two sequences, padding behind the second one's."""
    rows = [torch.cat([torch.arange(n) for n in ns]) for ns in ((100, 7, 103), (1, 128, 60))]
    return torch.stack([torch.nn.functional.pad(r, (0, 210 - len(r)), value=-1) for r in rows]).int().cuda()


def normal(g, *shape):
    return torch.randn(shape, generator=g, device="cuda").to(torch.bfloat16)


def make_leaves(seed):
    """x and the last block's y of every rank, a projection, and the weights of the norms."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    x, y = ([normal(g, 105, HIDDEN) for _ in range(4)] for _ in range(2))
    w_qkv = (torch.randn((HIDDEN, (4 + 2 + 2) * 64), generator=g, device="cuda") * HIDDEN ** -0.5).to(torch.bfloat16)
    norms = [(1 + 0.2 * torch.randn(HIDDEN, generator=g, device="cuda")).to(torch.bfloat16) for _ in range(3)]
    return x + y + [w_qkv] + norms


def block(basp, plan, leaves, rope, score, pos, up):
    """sum of up * o + h over the block's outputs"""
    from paper_2609_03151_b200.autograd import basp_attention, basp_block_norm, basp_rope
    x, y, w_qkv, (wp, g, wn) = leaves[:4], leaves[4:8], leaves[8], leaves[9:]
    h, n = basp_block_norm(plan, x, y, wp, g, wn, res_scale=0.5)
    qkv = [(t @ w_qkv).reshape(105, 8, 64) for t in n]
    q, k, v = ([t[:, a:b].contiguous() for t in qkv] for a, b in ((0, 4), (4, 6), (6, 8)))
    q, k = basp_rope(plan, rope, q, k, pos)
    o = basp_attention(plan, q, k, v, score=score)
    return sum((a.reshape(105, -1).float() * u[:, :HIDDEN].float()).sum() + (b.float() * u[:, HIDDEN:].float()).sum()
               for a, b, u in zip(o, h, up))


def plain(leaves, pos, slopes, cap, up):
    """The same in fp64 on all tokens."""
    leaves = [t.detach().double().requires_grad_() for t in leaves]
    x, y, w_qkv, (wp, g, wn) = torch.cat(leaves[:4]), torch.cat(leaves[4:8]), leaves[8], leaves[9:]
    norm = lambda t, w: t / (t.square().mean(-1, keepdim=True) + 1e-6).sqrt() * w
    h = x + 0.5 * g * norm(y, wp)
    qkv = (norm(h, wn) @ w_qkv).reshape(2, 210, 8, 64)
    angle = pos.double()[..., None, None] * 10000.0 ** (-torch.arange(32, device="cuda", dtype=torch.float64) / 32)
    turn = lambda t: torch.cat([t[..., :32] * angle.cos() - t[..., 32:] * angle.sin(), t[..., 32:] * angle.cos() + t[..., :32] * angle.sin()], -1)
    q, k, v = (t.transpose(1, 2) for t in (turn(qkv[:, :, :4]), turn(qkv[:, :, 4:6]).repeat_interleave(2, 2), qkv[:, :, 6:].repeat_interleave(2, 2)))
    at = torch.arange(210, device="cuda")
    begin, end = (torch.from_numpy(t).cuda() for t in oracle.packed_ranges(pos.cpu().numpy()))
    see = ((at >= begin[..., None]) & (at < end[..., None]))[:, None]
    z = cap * torch.tanh(q @ k.mT / 8.0 / cap) - slopes.double()[:, None, None] * (at[:, None] - at).abs()
    p = torch.softmax(z.masked_fill(~see, -1e9), -1) * see
    o = (p @ v).transpose(1, 2).reshape(420, 256)
    u = torch.cat(up).double()
    loss = (o * u[:, :HIDDEN]).sum() + (h * u[:, HIDDEN:]).sum()
    return loss, torch.autograd.grad(loss, leaves)


@pytest.fixture
def setting(basp):
    plan = basp.basp_plan_create(*PLAN)
    pos, slopes = positions(), 2.0 ** -torch.arange(1.0, 5.0, device="cuda")
    mask = torch.empty(basp.basp_mask_bytes(plan), dtype=torch.uint8, device="cuda")
    basp.basp_mask_packed(plan, pos, mask)
    g = torch.Generator(device="cuda").manual_seed(9)
    return plan, pos, slopes, mask, basp.basp_rope_make(64), [normal(g, 105, 2 * HIDDEN) for _ in range(4)]


def test_training_step(basp, setting):
    plan, pos, slopes, mask, rope, up = setting
    leaves = [t.requires_grad_() for t in make_leaves(1)]
    basp.basp_clear_status()
    loss = block(basp, plan, leaves, rope, basp.basp_score(8.0, slopes, mask), pos, up)
    loss.backward()
    basp.basp_get_status()
    want, grads = plain(leaves, pos, slopes, 8.0, up)
    # some ten roundings to bf16 in a row, each within 2^-8 of its tensor's norm and most of them 2^-9.5 (rms): 2^-6
    for i, (t, ref) in enumerate(zip(leaves, grads)):
        off = ((t.grad.double() - ref).norm() / ref.norm()).item()
        assert off <= 2.0 ** -6, (i, off)
    # the terms' own roundings, 2^-8 of each, with random signs: far below 2^-8 of the sum of their norms
    assert abs(loss.item() - want.item()) <= 2.0 ** -6 * torch.cat(up).double().norm().item() * 3


def test_captured_step(basp, setting):
    """The whole step captured, its mask built inside the graph, replayed on new inputs and new documents: an eager step's gradients."""
    plan, pos, slopes, mask, rope, up = setting
    pos = pos.clone()
    leaves = [t.requires_grad_() for t in make_leaves(2)]

    def step():
        basp.basp_mask_packed(plan, pos, mask)
        loss = block(basp, plan, leaves, rope, basp.basp_score(8.0, slopes, mask), pos, up)
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
    with torch.no_grad():
        for t, f in zip(leaves, make_leaves(3)):
            t.copy_(f)
    pos.copy_(pos.flip(0))
    graph.replay()
    torch.cuda.synchronize()
    got, got_loss = [t.grad.clone() for t in leaves], loss.clone()
    for t in leaves:
        t.grad = None
    eager = step()
    basp.basp_get_status()
    assert torch.equal(got_loss, eager)
    for i, (a, t) in enumerate(zip(got, leaves)):
        off = (a.float() - t.grad.float()).norm() / t.grad.float().norm()
        assert off <= 2.0 ** -8, (i, off.item())          # dQ comes from a reduction in whatever order its blocks finish


def test_two_streams_at_once(basp):
    """Masked attention and block norms of two sizes on two streams, a dozen times over, against each alone."""
    jobs = []
    for i, (S, hidden) in enumerate(((900, 512), (333, 2048))):
        plan = basp.basp_plan_create(1, 1, S, 8, 4, 128)
        g = torch.Generator(device="cuda").manual_seed(20 + i)
        q, k, v = (normal(g, 1, S, h, 128) for h in (8, 4, 4))
        x, y, dn = (normal(g, S, hidden) for _ in range(3))
        w = normal(g, hidden)
        pos = (torch.arange(S, device="cuda") % (150 + 60 * i)).int()[None].contiguous()
        mask = torch.empty(basp.basp_mask_bytes(plan), dtype=torch.uint8, device="cuda")
        ws = torch.empty(basp.basp_block_norm_bwd_workspace_bytes(plan, hidden), dtype=torch.uint8, device="cuda")
        make = lambda q=q, x=x, S=S, hidden=hidden: [torch.empty_like(q), torch.empty((1, 8, S), device="cuda")] + [torch.empty_like(x) for _ in range(4)] + \
            [torch.empty(hidden, device="cuda") for _ in range(2)]

        def call(o, stream, plan=plan, q=q, k=k, v=v, x=x, y=y, dn=dn, w=w, pos=pos, mask=mask, ws=ws, hidden=hidden):
            basp.basp_mask_packed(plan, pos, mask, stream=stream)
            basp.basp_attn_masked_fwd(plan, basp.basp_score(20.0, None, mask), [q], [k], [v], [o[0]], [o[1]], stream=stream)
            basp.basp_block_norm(plan, hidden, [x], [y], [o[2]], [o[3]], gate=w, w_pre=w, stream=stream)
            basp.basp_block_norm_bwd(plan, hidden, [o[2]], [y], None, [dn], [o[4]], [o[5]], None, o[6], o[7], ws, gate=w, w_pre=w, stream=stream)
        jobs.append((make, call))
    basp.basp_clear_status()
    alone = []
    for make, call in jobs:
        o = make()
        call(o, None)
        alone.append(o)
    torch.cuda.synchronize()
    streams, out = [torch.cuda.Stream() for _ in jobs], [make() for make, _ in jobs]
    torch.cuda.synchronize()
    for _ in range(12):
        for (_, call), o, s in zip(jobs, out, streams):
            call(o, s)
    torch.cuda.synchronize()
    basp.basp_get_status()
    for a, b in zip(alone, out):
        assert all(torch.equal(p, q) for p, q in zip(a, b))


def test_raw_addresses(basp):
    plan = basp.basp_plan_create(2, 2, 64, 2, 2, 64)
    g = torch.Generator(device="cuda").manual_seed(3)
    q, k = ([normal(g, 64, 2, 64) for _ in range(2)] for _ in range(2))
    outs = [[[torch.empty_like(t) for t in x] for x in (q, k)] for _ in range(2)]
    rope, at = basp.basp_rope_make(32), lambda ts: [t.data_ptr() for t in ts]
    basp.basp_rope(plan, rope, q, k, *outs[0])
    basp.basp_rope(plan, rope, at(q), basp.as_shards(at(k)), at(outs[1][0]), at(outs[1][1]))
    assert all(torch.equal(a, b) for x, y in zip(*outs) for a, b in zip(x, y))


def test_what_autograd_refuses(basp, setting):
    from paper_2609_03151_b200.autograd import basp_attention, basp_block_norm, basp_rope
    plan, pos, slopes, mask, rope, up = setting
    g = torch.Generator(device="cuda").manual_seed(4)
    q, k, v = ([normal(g, 105, h, 64).requires_grad_() for _ in range(4)] for h in (4, 2, 2))
    with pytest.raises(ValueError):
        basp_attention(plan, q, k, v, score=basp.basp_score(mask=mask), fused=True)
    with pytest.raises(ValueError):
        basp_attention(plan, q, k, v, score=basp.basp_score(slopes=slopes.clone().requires_grad_(), mask=mask))
    with pytest.raises(ValueError):
        basp_block_norm(plan, [normal(g, 105, 64)] * 4, [normal(g, 105, 64)] * 3, w_pre=normal(g, 64))
    calls = (lambda: basp_attention(plan, q, k, v, score=basp.basp_score(mask=mask)), lambda: sum(basp_rope(plan, rope, q, k, pos), []),
             lambda: basp_block_norm(plan, [t.reshape(105, -1) for t in q], w_pre=normal(g, 256))[1])
    for call in calls:
        loss = sum(t.float().square().sum() for t in call())
        (d,) = torch.autograd.grad(loss, q[0], create_graph=True)
        with pytest.raises(RuntimeError):
            d.float().sum().backward()


@pytest.mark.parametrize("form", ["first", "last", "middle, one output unused"])
def test_block_norm_forms_through_autograd(basp, form):
    from paper_2609_03151_b200.autograd import basp_block_norm
    plan = basp.basp_plan_create(1, 1, 50, 1, 1, 64)
    g = torch.Generator(device="cuda").manual_seed(5)
    x, y, w = normal(g, 50, 128).requires_grad_(), normal(g, 50, 128).requires_grad_(), normal(g, 128).requires_grad_()
    u = normal(g, 50, 128)
    X, Y, V = (t.detach().double().requires_grad_() for t in (x, y, w))
    norm = lambda t, s: t / (t.square().mean(-1, keepdim=True) + 1e-6).sqrt() * s
    if form == "first":
        out, ref, pairs = basp_block_norm(plan, [x], w_pre=w)[1][0], norm(X, V), ((x, X), (w, V))
    elif form == "last":
        h, n = basp_block_norm(plan, [x], [y], w_post=w, res_scale=0.3)
        assert n is None
        out, ref, pairs = h[0], X + 0.3 * norm(Y, V), ((x, X), (y, Y), (w, V))
    else:
        out = basp_block_norm(plan, [x], [y], gate=w, w_pre=w.detach())[1][0]
        ref, pairs = norm(X + Y * V, V.detach()), ((x, X), (y, Y), (w, V))
    (out.float() * u.float()).sum().backward()
    (ref * u.double()).sum().backward()
    for a, b in pairs:          # the sum h and the result rounded once each: 2^-8 of the norm and what a norm makes of it
        assert ((a.grad.double() - b.grad).norm() / b.grad.norm()).item() <= 2.0 ** -6


def test_a_score_changed_between_the_passes(basp, setting):
    """The backward reads the mask and the slopes again: one that was refilled in between is refused, as torch refuses any saved tensor that was
    written; another mask or cap put into the score object changes nothing."""
    from paper_2609_03151_b200.autograd import basp_attention
    plan, pos, slopes, mask, rope, up = setting
    g = torch.Generator(device="cuda").manual_seed(6)
    q, k, v = ([normal(g, 105, h, 64).requires_grad_() for _ in range(4)] for h in (4, 2, 2))
    u = [normal(g, 105, 4, 64) for _ in range(4)]
    begin = torch.zeros((2, 210), dtype=torch.int32, device="cuda")

    def forward():
        for t in q + k + v:
            t.grad = None
        score = basp.basp_score(8.0, slopes, mask)
        return score, sum((o.float() * t.float()).sum() for o, t in zip(basp_attention(plan, q, k, v, score=score), u))

    basp.basp_clear_status()
    forward()[1].backward()
    want = [t.grad.clone() for t in q + k + v]
    for write in (lambda: basp.basp_mask_packed(plan, pos, mask), lambda: basp.basp_mask_ranges(plan, begin, begin + 1, mask), lambda: mask.zero_(),
                  lambda: slopes.mul_(2.0)):
        basp.basp_mask_packed(plan, pos, mask)
        loss = forward()[1]
        write()
        with pytest.raises(RuntimeError, match="inplace"):
            loss.backward()
    slopes.div_(2.0)
    basp.basp_mask_packed(plan, pos, mask)
    score, loss = forward()
    score.mask, score.slopes, score.softcap = None, None, 0.0
    loss.backward()
    basp.basp_get_status()
    for t, ref in zip(q + k + v, want):
        assert ((t.grad.float() - ref.float()).norm() / ref.float().norm()).item() <= 2.0 ** -8        # dQ's sums in another order
    with torch.no_grad():                                  # no backward comes: the buffer is free for the next batch
        basp_attention(plan, q, k, v, score=basp.basp_score(8.0, slopes, mask))
        basp.basp_mask_packed(plan, pos, mask)
    with torch.inference_mode():                           # a mask without a record of its writes serves as well
        mask = torch.empty_like(mask)
        basp.basp_mask_packed(plan, pos, mask)
    forward()[1].backward()
    basp.basp_get_status()
    for t, ref in zip(q + k + v, want):
        assert ((t.grad.float() - ref.float()).norm() / ref.float().norm()).item() <= 2.0 ** -8


def test_block_norm_takes_the_attention_output_as_it_is(basp):
    """y in the attention's [tokens, heads, features], a weight of [1, hidden]: gradients in the inputs' own shapes, the bits of flat ones."""
    from paper_2609_03151_b200.autograd import basp_block_norm
    plan = basp.basp_plan_create(2, 1, 210, 4, 2, 64)
    g = torch.Generator(device="cuda").manual_seed(7)
    x, up = ([normal(g, 105, HIDDEN) for _ in range(2)] for _ in range(2))
    y = [normal(g, 105, 4, 64) for _ in range(2)]
    w = [normal(g, HIDDEN) for _ in range(3)]
    grads = []
    for shape, row in (((105, 4, 64), (1, HIDDEN)), ((105, HIDDEN), (HIDDEN,))):
        leaves = [t.clone().requires_grad_() for t in x + [t.reshape(shape) for t in y] + [t.reshape(row) for t in w]]
        h, n = basp_block_norm(plan, leaves[:2], leaves[2:4], *leaves[4:])
        torch.autograd.backward(h + n, up + up)
        assert all(t.grad.shape == t.shape for t in leaves)
        grads.append([t.grad.flatten() for t in leaves])
    assert all(torch.equal(a, b) for a, b in zip(*grads))
