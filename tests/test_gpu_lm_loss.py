"""The language-model loss and its gradients against the fp64 oracle.

Tolerances.  A logit is a sum of `hidden` exact products that the tensor cores add up in fp32, 16 at a time: at most
(hidden / 16 + 16) steps, each off by at most 2^-23 of the sum of magnitudes:  tz = (hidden/16 + 16) 2^-23 max sum |x w|.
  loss, lse   2 tz and 2^-20 (1 + |lse|) for the statistics (fp32 exponentials and logarithms, sums of positive terms)
  dz          2^-8 (bf16) + 2^-11 (the 16-bit distance, 2^-11 ln 2, and the approximate exponential) + 4 tz (its exponent), relative;
              probabilities below 2^-64 of a tile's largest may be zero
  dx, dw      dz's error through the products' magnitudes, their own fp32 sums (K/16 + 16) 2^-23, one rounding 2^-8 of the result.
These bound the worst case; independent roundings also keep the 2-norm of dx and dw within 2^-8 of the result's (two bf16
roundings, each at most 2^-8 / sqrt(3) in the mean, give 0.82 x 2^-8)."""
import numpy as np
import pytest
import torch

import oracle
from helpers import make_plan
from paper_2609_03151_b200 import synth

pytestmark = pytest.mark.gpu

L = lambda name, N, B, S, hidden, vocab, G=0: (synth.Workload(name, N=N, B=B, S=S, Hq=8, Hkv=8, D=64, G=G), hidden, vocab)
CASES = [
    L("one_token", 1, 1, 1, 64, 300),
    L("one_word", 1, 1, 3, 8, 1),
    L("two_words", 1, 1, 5, 16, 2),
    L("small_hidden", 2, 2, 9, 40, 257),
    L("token_per_rank", 8, 1, 8, 128, 1000),
    L("slots_of_16", 4, 2, 24, 264, 511),              # 12 tokens per rank: several ranks in a tile
    L("slots_of_32_uneven", 4, 1, 77, 192, 1025),      # 20, 20, 20, 17 tokens
    L("slots_of_64", 2, 1, 100, 520, 768),
    L("slots_of_128", 2, 2, 200, 256, 3001),           # 200 tokens per rank: 128 + 72
    L("uneven_two_seqs", 4, 2, 301, 320, 1500, 1),     # two sequences per rank, 76, 76, 76, 73 tokens each
    L("several_tiles", 2, 1, 1021, 512, 2048),
    L("many_ranks", 16, 2, 80, 128, 777),
    L("long_vocabulary", 1, 1, 130, 128, 50257),
    L("data_parallel", 2, 4, 33, 96, 640),
]


def inputs(pl, hidden, vocab, seed=0, sure=12.0):
    g = torch.Generator().manual_seed(seed + hidden + vocab)
    w = (torch.randn((vocab, hidden), generator=g) / hidden ** 0.5).to(torch.bfloat16)
    x, labels, weights = [], [], []
    for r in range(pl.N):
        n = pl.Bl * pl.rank_tokens(r)
        y = torch.randint(0, vocab, (n,), generator=g)
        t = torch.randn((n, hidden), generator=g) + sure * torch.rand((n, 1), generator=g) * w[y].float()
        u = torch.rand(n, generator=g)
        y = torch.where(u < 0.1, -100, torch.where(u < 0.15, vocab, torch.where(u < 0.18, -(1 << 40), y)))
        x.append(t.to(torch.bfloat16)); labels.append(y)
        weights.append(torch.rand(n, generator=g) + 0.1)
    if pl.Bl * pl.T > 4:
        weights[0][1] = 0.0
        weights[0][2] = -2.0
    return w, x, labels, weights


def f64(t):
    return t.float().cpu().numpy().astype(np.float64)


def cat(ts):
    return torch.cat([t.reshape(-1, *t.shape[1:]) for t in ts])


def run(basp, pl, hidden, vocab, w, x, labels, weights, piece_rows=0, dx=True, dw=True):
    c = lambda ts: [t.cuda() for t in ts]
    x, w = c(x), w.cuda()
    loss, lse = ([torch.full((t.shape[0],), float("nan"), device="cuda") for t in x] for _ in range(2))
    dx = [torch.full_like(t, float("nan")) for t in x] if dx else None
    dw = torch.full_like(w, float("nan")) if dw else None
    ws = torch.full((basp.basp_lm_loss_grad_workspace_bytes(pl, hidden, vocab, piece_rows),), 255, dtype=torch.uint8, device="cuda")
    basp.basp_clear_status()
    basp.basp_lm_loss_grad(pl, hidden, vocab, x, w, c(labels), None if weights is None else c(weights), loss, lse, dx, dw, ws,
                           piece_rows=piece_rows)
    basp.basp_get_status()
    return loss, lse, dx, dw


def check(got, ref, x, w, hidden, vocab, what):
    loss, lse, dx, dw = got
    X, W = f64(cat(x)), f64(w)
    tz = (hidden / 16 + 16) * 2.0 ** -23 * (np.abs(X) @ np.abs(W).T).max()
    tol = 2 * tz + 2.0 ** -20 * (1 + np.abs(ref["lse"]))
    assert (np.abs(f64(cat(loss)) - ref["loss"]) <= tol).all(), (what, "loss", np.abs(f64(cat(loss)) - ref["loss"]).max())
    if lse is not None:
        assert (np.abs(f64(cat(lse)) - ref["lse"]) <= tol).all(), (what, "lse")
    rel = 2.0 ** -8 + 2.0 ** -11 + 4 * tz
    adz = np.abs(ref["dz"])
    for name, out, want, terms, k in (("dx", dx, ref["dx"], adz @ np.abs(W), vocab), ("dw", dw, ref["dw"], adz.T @ np.abs(X), X.shape[0])):
        if out is None:
            continue
        have = f64(cat(out) if isinstance(out, list) else out)
        err = np.abs(have - want)
        assert (err <= 2.0 ** -8 * np.abs(want) + (rel + (k / 16 + 16) * 2.0 ** -23) * terms + 1e-37).all(), (what, name, float(err.max()))
        if want.size >= 4096 and np.linalg.norm(want) > 0:
            assert np.linalg.norm(err) <= 2.0 ** -8 * np.linalg.norm(want), (what, name, np.linalg.norm(err) / np.linalg.norm(want))


@pytest.mark.parametrize("w,hidden,vocab", CASES, ids=lambda x: getattr(x, "name", ""))
def test_loss_and_gradients(basp, w, hidden, vocab):
    pl = make_plan(basp, w)
    W, x, labels, weights = inputs(pl, hidden, vocab)
    ref = oracle.lm_loss(f64(cat(x)), f64(W), cat(labels).numpy(), cat(weights).numpy().astype(np.float64))
    got = run(basp, pl, hidden, vocab, W, x, labels, weights)
    check(got, ref, x, W, hidden, vocab, w.name)
    # the loss alone: the same bits
    c = lambda ts: [t.cuda() for t in ts]
    loss, lse = ([torch.full((t.shape[0],), float("nan"), device="cuda") for t in x] for _ in range(2))
    ws = torch.full((basp.basp_lm_loss_fwd_workspace_bytes(pl, vocab),), 255, dtype=torch.uint8, device="cuda")
    basp.basp_lm_loss_fwd(pl, hidden, vocab, c(x), W.cuda(), c(labels), loss, lse, ws)
    basp.basp_get_status()
    assert torch.equal(cat(loss), cat(got[0])) and torch.equal(cat(lse), cat(got[1]))
    # one gradient alone, no log-sum-exp: the same bits
    again = run(basp, pl, hidden, vocab, W, x, labels, weights, dw=False)
    assert torch.equal(cat(again[2]), cat(got[2]))
    again = run(basp, pl, hidden, vocab, W, x, labels, weights, dx=False)
    assert torch.equal(again[3], got[3])
    basp.basp_lm_loss_fwd(pl, hidden, vocab, c(x), W.cuda(), c(labels), loss, None, ws)
    assert torch.equal(cat(loss), cat(got[0]))


@pytest.mark.parametrize("piece_rows", [1, 256, 384, 512])
def test_pieces(basp, piece_rows):
    w, hidden, vocab = L("pieces", 4, 2, 500, 320, 1111)
    pl = make_plan(basp, w)
    W, x, labels, weights = inputs(pl, hidden, vocab, 1)
    ref = oracle.lm_loss(f64(cat(x)), f64(W), cat(labels).numpy(), cat(weights).numpy().astype(np.float64))
    got = run(basp, pl, hidden, vocab, W, x, labels, weights, piece_rows=piece_rows)
    check(got, ref, x, W, hidden, vocab, piece_rows)
    again = run(basp, pl, hidden, vocab, W, x, labels, weights, piece_rows=piece_rows)
    for a, b in zip(got[0] + got[1] + got[2] + [got[3]], again[0] + again[1] + again[2] + [again[3]]):
        assert torch.equal(a, b)


@pytest.mark.parametrize("rows,piece_rows", [(300, 256), (1100, 512), (700, 640)])
def test_short_last_piece_with_a_split_vocabulary(basp, rows, piece_rows):
    """The last piece has fewer row tiles than the others, so its dx splits the vocabulary more often: its partial sums stay clear of
    the running sum of dw."""
    w, hidden, vocab = L("short_last", 1, 1, rows, 64, 20000)
    pl = make_plan(basp, w)
    W, x, labels, weights = inputs(pl, hidden, vocab, 6)
    ref = oracle.lm_loss(f64(cat(x)), f64(W), cat(labels).numpy(), cat(weights).numpy().astype(np.float64))
    check(run(basp, pl, hidden, vocab, W, x, labels, weights, piece_rows=piece_rows), ref, x, W, hidden, vocab, (rows, piece_rows))


def test_weights_of_one_and_confident_predictions(basp):
    """No weight table; the target 60 above the others: a loss far below fp32's spacing at the logit's size."""
    w, hidden, vocab = L("sure", 2, 1, 64, 256, 700)
    pl = make_plan(basp, w)
    W, x, labels, _ = inputs(pl, hidden, vocab, 2, sure=0.0)
    g = torch.Generator().manual_seed(9)
    labels = [torch.randint(0, vocab, y.shape, generator=g) for y in labels]
    x = [(t.float() * 0.2 + 20 * W[y].float()).to(torch.bfloat16) for t, y in zip(x, labels)]
    ref = oracle.lm_loss(f64(cat(x)), f64(W), cat(labels).numpy(), np.ones(64))
    got = run(basp, pl, hidden, vocab, W, x, labels, None)
    check(got, ref, x, W, hidden, vocab, "sure")
    # relative: others / target's probability is exp of a difference of logits, off by 2 tz
    X = f64(cat(x))
    tz = (hidden / 16 + 16) * 2.0 ** -23 * (np.abs(X) @ np.abs(f64(W)).T).max()
    z = X @ f64(W).T
    y = cat(labels).numpy()
    others = np.log(np.where(np.arange(vocab) == y[:, None], 0.0, np.exp(z - z.max(1, keepdims=True))).sum(1)) + z.max(1)
    exact = np.log1p(np.exp(others - z[np.arange(64), y]))
    assert exact.min() < 1e-5
    assert (np.abs(f64(cat(got[0])) - exact) <= (4 * tz + 2.0 ** -18) * exact).all()


def far_from_zero(rows, vocab, seed):
    """Logits that are exact in fp32 and up to 6e4 off zero, all words of a row alike: x = (+-2^k, 1, 0, ...), a word's first weight is
    1.171875 for all, its second a multiple of 1/8.  Four words stand above the others, within 2 of one another; labels are elsewhere."""
    hidden = 64
    g = torch.Generator().manual_seed(seed)
    W = torch.zeros((vocab, hidden))
    W[:, 0] = 1.171875
    W[:, 1] = torch.randint(-32, 33, (vocab,), generator=g) / 8
    for i, word in enumerate((7, vocab // 2, vocab // 2 + 1, vocab - 3)):
        W[word, 1] = 10 + i / 2
    x = torch.zeros((rows, hidden))
    x[:, 0] = 2.0 ** (10 + torch.arange(rows) % 6) * (1 - 2 * (torch.arange(rows) // 6 % 2))
    x[:, 1] = 1 + torch.randint(0, 3, (rows,), generator=g) / 4
    y = 8 + torch.randint(0, vocab // 2 - 8, (rows,), generator=g)
    return hidden, W.to(torch.bfloat16), x.to(torch.bfloat16), y, torch.rand(rows, generator=g) + 0.5


@pytest.mark.parametrize("rows", [100, 520])           # single CTAs, pairs
def test_top_words_of_logits_far_from_zero(basp, rows):
    """A logit's distance below its group's largest is zero for the largest whatever the rounding of large numbers.  Here the
    logits are exact, so what is left of the tolerances above is dz's 2^-8 + 2^-11 and the log-sum-exp, which is rounded twice
    at its size: 2 x 2^-24 |lse| of every probability."""
    vocab = 700
    hidden, W, x, y, weights = far_from_zero(rows, vocab, 11)
    pl = make_plan(basp, L("far", 1, 1, rows, hidden, vocab)[0])
    ref = oracle.lm_loss(f64(x), f64(W), y.numpy(), weights.numpy().astype(np.float64))
    size = np.abs(ref["lse"]).max()
    assert size > 3e4 and np.sort(np.abs(ref["dz"]), 1)[:, -3].min() > 0.02
    loss, lse, dx, dw = run(basp, pl, hidden, vocab, W, [x], [y], [weights])
    off = 2.0 ** -23 * size
    assert (np.abs(f64(loss[0]) - ref["loss"]) <= off + 2.0 ** -20 * (1 + ref["loss"])).all()
    assert (np.abs(f64(lse[0]) - ref["lse"]) <= off + 2.0 ** -20).all()
    adz, X8, W8 = np.abs(ref["dz"]), f64(x), f64(W)
    for name, got, want, terms, k in (("dx", dx[0], ref["dx"], adz @ np.abs(W8), vocab), ("dw", dw, ref["dw"], adz.T @ np.abs(X8), rows)):
        err = np.abs(f64(got) - want)
        tol = 2.0 ** -8 * np.abs(want) + (2.0 ** -8 + 2.0 ** -11 + off + (k / 16 + 16) * 2.0 ** -23) * terms + 1e-37
        assert (err <= tol).all(), (name, float(err.max()), float((err / tol).max()))


@pytest.mark.parametrize("target", ["elsewhere", "top", "only"])
@pytest.mark.parametrize("rows", [100, 520])           # single CTAs, pairs
def test_losses_and_probabilities_do_not_depend_on_the_offset(basp, rows, target):
    """softmax(z + c) = softmax(z): nothing of the loss or the gradients is rounded at the size of the logits, only lse itself is
    (half a step, 2^-24 of it).  The label is a word far below the top, one of the top, or the one word far above all others."""
    vocab = 700
    hidden, W, x, y, weights = far_from_zero(rows, vocab, 12)
    if target != "elsewhere":
        y[:] = vocab // 2
    if target == "only":
        W[vocab // 2, 1] = 24
    pl = make_plan(basp, L("far", 1, 1, rows, hidden, vocab)[0])
    ref = oracle.lm_loss(f64(x), f64(W), y.numpy(), weights.numpy().astype(np.float64))
    loss, lse, dx, dw = run(basp, pl, hidden, vocab, W, [x], [y], [weights])
    assert (np.abs(f64(loss[0]) - ref["loss"]) <= 2.0 ** -20 * (1 + ref["loss"])).all()
    assert (np.abs(f64(lse[0]) - ref["lse"]) <= 2.0 ** -24 * np.abs(ref["lse"]) + 2.0 ** -19).all()
    adz, X8, W8 = np.abs(ref["dz"]), f64(x), f64(W)
    for name, got, want, terms, k in (("dx", dx[0], ref["dx"], adz @ np.abs(W8), vocab), ("dw", dw, ref["dw"], adz.T @ np.abs(X8), rows)):
        err = np.abs(f64(got) - want)
        tol = 2.0 ** -8 * np.abs(want) + (2.0 ** -8 + 2.0 ** -11 + (k / 16 + 16) * 2.0 ** -23) * terms + 1e-37
        assert (err <= tol).all(), (name, float(err.max()), float((err / tol).max()))


@pytest.mark.parametrize("rows", [100, 520])           # single CTAs, pairs
@pytest.mark.parametrize("hidden", [2048, 8192])
def test_lse_is_not_short_of_what_the_products_cut_off(basp, rows, hidden):
    """The tensor cores cut a running sum off towards zero, up to 2^-23 of it in each of hidden / 16 steps; on such values
    that is 2^-30 hidden of a logit in the mean (2^-3 of the bound), by which lse = ln sum exp z is short by as much of
    sum p z.  The kernel makes up for it: at least half has to be gone from the mean over the tokens, besides 2^-21 for the
    statistics (fp32 of about 9: half a step of 2^-21)."""
    w, hidden, vocab = L("short", 1, 1, rows, hidden, 4096)
    pl = make_plan(basp, w)
    W, x, labels, weights = inputs(pl, hidden, vocab, 7, sure=0.0)
    z = x[0].cuda().double() @ W.cuda().double().T
    exact = torch.logsumexp(z, -1)
    spread = (torch.softmax(z, -1) * z).sum(-1)
    _, lse, _, _ = run(basp, pl, hidden, vocab, W, x, labels, weights, dw=False)
    short = (exact - lse[0].double()).mean().abs().item()
    assert short <= 2.0 ** -31 * hidden * spread.mean().item() + 2.0 ** -21, short


@pytest.mark.parametrize("rows", [100, 520])           # single CTAs, pairs
@pytest.mark.parametrize("hidden,features", [(4096, 1), (4096, 16), (65536, 2), (65536, 16)])
def test_rows_of_few_features_are_exact(basp, hidden, features, rows):
    """Rows of x with few features other than zero lose nothing in the products: logits (up to 60) exact in fp32, so the loss and
    lse have the statistics' errors alone."""
    w, hidden, vocab = L("few", 1, 1, rows, hidden, 500)
    pl = make_plan(basp, w)
    g = torch.Generator().manual_seed(hidden + features)
    at = torch.rand((rows, hidden), generator=g).topk(features, 1).indices
    x = torch.zeros((rows, hidden)).scatter_(1, at, 2.0 ** torch.randint(-1, 2, (rows, features), generator=g).float())
    W = torch.randint(-32, 33, (vocab, hidden), generator=g) / 8 * (4.0 if features == 1 else 1.0)
    x, W = x.to(torch.bfloat16), W.to(torch.bfloat16)
    y = torch.randint(0, vocab, (rows,), generator=g)
    y[::7] = -100
    ref = oracle.lm_loss(f64(x), f64(W), y.numpy(), np.ones(rows))
    assert ref["lse"].max() > 8
    loss, lse, _, _ = run(basp, pl, hidden, vocab, W, [x], [y], None, dw=False)
    for got, want in ((loss, ref["loss"]), (lse, ref["lse"])):
        err = np.abs(f64(got[0]) - want)
        assert (err <= 2.0 ** -20 * (1 + np.abs(ref["lse"]))).all(), float(err.max())


@pytest.mark.parametrize("features", [512, 2048])
def test_what_is_made_up_for_goes_by_the_features_of_the_row(basp, features):
    """As test_lse_is_not_short_of_what_the_products_cut_off, on rows whose features behind the first ones are zero: the shortfall is
    that of the shorter sum, in every rank's rows."""
    w, hidden, vocab = L("padded", 2, 1, 200, 8192, 4096)
    pl = make_plan(basp, w)
    W, x, labels, weights = inputs(pl, hidden, vocab, 9, sure=0.0)
    for t in x:
        t[:, features:] = 0.0
        t.mul_(2.0 if features == 2048 else 4.0)            # logits of about unit size again, an exact factor
    z = cat(x).cuda().double() @ W.cuda().double().T
    exact = torch.logsumexp(z, -1)
    spread = (torch.softmax(z, -1) * z).sum(-1)
    _, lse, _, _ = run(basp, pl, hidden, vocab, W, x, labels, weights, dw=False)
    short = (exact - cat(lse).double()).mean().abs().item()
    assert short <= 2.0 ** -31 * features * spread.mean().item() + 2.0 ** -21, short


def test_special_rows_and_words(basp):
    """Infinities and NaN: a row that has them is NaN and no other row is; a row without a label or a weight leaves the
    gradients alone; a word whose weights make its logit -inf has probability zero."""
    w, hidden, vocab = L("special", 2, 1, 40, 64, 600)
    pl = make_plan(basp, w)
    W, x, labels, weights = inputs(pl, hidden, vocab, 3)
    labels = [torch.where((y < 0) | (y >= vocab), 5, y) for y in labels]
    x[0][3, 7] = float("nan")
    x[0][4, 7] = float("inf")
    labels[0][3] = -100                                     # no label: its NaN reaches nothing but its lse
    weights[0][4] = 0.0
    clean = [t.clone() for t in x]
    clean[0][3:5] = 0.0
    ref = oracle.lm_loss(f64(cat(clean)), f64(W), cat(labels).numpy(), cat(weights).numpy().astype(np.float64))
    loss, lse, dx, dw = run(basp, pl, hidden, vocab, W, x, labels, weights)
    keep = np.ones(40, dtype=bool)
    keep[3:5] = False
    assert loss[0][3].item() == 0.0 and not np.isfinite(f64(loss[0])[4]) and not np.isfinite(f64(lse[0])[3:5]).any()
    assert (f64(dx[0])[3:5] == 0).all()
    sub = lambda a: a[keep]
    refk = dict(loss=sub(ref["loss"]), lse=sub(ref["lse"]), dz=sub(ref["dz"]), dx=sub(ref["dx"]), dw=ref["dw"])
    xk = [torch.from_numpy(sub(f64(cat(clean)))).to(torch.bfloat16)]
    pick = lambda ts: [cat(ts)[torch.from_numpy(keep).cuda()]]
    zk = refk["dz"]
    check((pick(loss), pick(lse), pick(dx), dw), refk, xk, W, hidden, vocab, "special")
    # the NaN row has a label and a weight: its own dx and the whole of dw are NaN, the other rows are not touched
    labels[0][3] = 5
    loss2, _, dx2, dw2 = run(basp, pl, hidden, vocab, W, x, labels, weights)
    assert np.isnan(f64(dx2[0])[3]).all() and torch.isnan(dw2).all().item()
    assert torch.equal(pick(loss2)[0], pick(loss)[0]) and torch.equal(pick(dx2)[0], pick(dx)[0])
    # a logit of -inf everywhere but at the target, and words at -inf in every tile
    x2 = [torch.ones_like(t) for t in x]
    W2 = W.clone()
    W2[100:] = float("-inf")
    lab2 = [torch.full_like(y, 3) for y in labels]
    ref2 = oracle.lm_loss(f64(cat(x2)), f64(W2[:100]), cat(lab2).numpy(), np.ones(40))
    loss, lse, dx, dw = run(basp, pl, hidden, vocab, W2, x2, lab2, None, dx=False)
    assert (np.abs(f64(cat(loss)) - ref2["loss"]) <= 1e-4).all()
    assert (f64(dw)[100:] == 0).all() and np.linalg.norm(f64(dw)[:100] - ref2["dw"]) <= 2.0 ** -8 * np.linalg.norm(ref2["dw"])


@pytest.mark.parametrize("value", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("N,S", [(2, 40), (1, 700)])
def test_a_weight_that_is_no_number_stays_with_its_token(basp, value, N, S):
    """A NaN or infinite token weight makes its own row of dx and dw no numbers (dz = g (p - onehot)); the losses and the
    other tokens' dx are those of the call without it."""
    w, hidden, vocab = L("odd_weight", N, 1, S, 64, 600)
    pl = make_plan(basp, w)
    W, x, labels, weights = inputs(pl, hidden, vocab, 6)
    labels = [torch.where((y < 0) | (y >= vocab), 5, y) for y in labels]
    weights[0][5] = 0.5                                     # not the largest: the others' unit does not change
    weights[0][6] = 1.25
    loss, lse, dx, _ = run(basp, pl, hidden, vocab, W, x, labels, weights)
    weights[0][5] = value
    loss2, lse2, dx2, dw2 = run(basp, pl, hidden, vocab, W, x, labels, weights)
    assert torch.equal(cat(loss), cat(loss2)) and torch.equal(cat(lse), cat(lse2))
    keep = torch.ones(S, dtype=torch.bool, device="cuda")
    keep[5] = False
    assert torch.equal(cat(dx)[keep], cat(dx2)[keep]) and torch.isfinite(cat(dx2)[keep]).all().item()
    assert not torch.isfinite(cat(dx2)[5]).any().item() and not torch.isfinite(dw2).any().item()
    # no finite weight at all
    none = [torch.full_like(t, value) for t in weights]
    loss3, _, dx3, dw3 = run(basp, pl, hidden, vocab, W, x, labels, none)
    assert torch.equal(cat(loss), cat(loss3))
    assert not torch.isfinite(cat(dx3)).any().item() and not torch.isfinite(dw3).any().item()


def test_rows_and_words_behind_the_ends_are_left(basp):
    w, hidden, vocab = L("ends", 2, 1, 20, 72, 300)
    pl = make_plan(basp, w)
    W, x, labels, weights = inputs(pl, hidden, vocab, 4)
    c = lambda ts: [t.cuda() for t in ts]
    big = [torch.full((64, hidden), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    bigw = torch.full((vocab + 300, hidden), 7.0, dtype=torch.bfloat16, device="cuda")
    bigl = [torch.full((140,), 7.0, device="cuda") for _ in range(4)]
    need = basp.basp_lm_loss_grad_workspace_bytes(pl, hidden, vocab)
    ws = torch.full((need + 4096,), 201, dtype=torch.uint8, device="cuda")
    basp.basp_lm_loss_grad(pl, hidden, vocab, c(x), W.cuda(), c(labels), c(weights), [t[:10] for t in bigl[:2]],
                           [t[:10] for t in bigl[2:]], [t[:10] for t in big], bigw[:vocab], ws[:need])
    basp.basp_get_status()
    assert all((t[10:] == 7.0).all().item() for t in big + bigl)
    assert (bigw[vocab:] == 7.0).all().item() and (ws[need:] == 201).all().item()


def test_autograd_pieces_of_it_and_graph(basp):
    from paper_2609_03151_b200.autograd import basp_lm_loss
    w, hidden, vocab = L("auto", 4, 2, 60, 128, 900)
    pl = make_plan(basp, w)
    W, x, labels, weights = inputs(pl, hidden, vocab, 5)
    ref = oracle.lm_loss(f64(cat(x)), f64(W), cat(labels).numpy(), cat(weights).numpy().astype(np.float64))
    c = lambda ts: [t.cuda() for t in ts]
    xl, wl, yl, gl = [t.requires_grad_() for t in c(x)], W.cuda().requires_grad_(), c(labels), c(weights)
    loss = basp_lm_loss(pl, xl, wl, yl, gl)
    want = (ref["loss"] * cat(weights).numpy()).sum()
    assert abs(loss.item() - want) <= 1e-4 * (1 + abs(want))
    (3 * loss).backward()
    for name, got, exact in (("dx", cat([t.grad for t in xl]), ref["dx"]), ("dw", wl.grad, ref["dw"])):
        assert np.linalg.norm(f64(got) - 3 * exact) <= 1.5 * 2.0 ** -8 * np.linalg.norm(3 * exact), name     # one more rounding
    # only one side wants a gradient; none does
    half = basp_lm_loss(pl, [t.detach() for t in xl], wl, yl, gl)
    (g,) = torch.autograd.grad(half, wl)
    assert torch.equal(half, loss) and np.linalg.norm(f64(g) - ref["dw"]) <= 2.0 ** -8 * np.linalg.norm(ref["dw"])
    (g,) = torch.autograd.grad(basp_lm_loss(pl, xl, wl.detach(), yl, gl), [xl[1]])
    assert np.linalg.norm(f64(g) - ref["dx"][60 // 2:60]) <= 2.0 ** -8 * np.linalg.norm(ref["dx"][30:60])
    with torch.no_grad():
        assert torch.equal(basp_lm_loss(pl, xl, wl, yl, gl), loss)
    with pytest.raises(ValueError, match="differentiable"):
        basp_lm_loss(pl, xl, wl, yl, [t.clone().requires_grad_() for t in gl])
    # captured and replayed on new inputs
    xs, ws = [t.detach().clone() for t in xl], wl.detach()
    space = torch.empty(basp.basp_lm_loss_grad_workspace_bytes(pl, hidden, vocab), dtype=torch.uint8, device="cuda")
    out = [torch.empty(t.shape[0], device="cuda") for t in xs], [torch.empty_like(t) for t in xs], torch.empty_like(ws)
    call = lambda o, sp: basp.basp_lm_loss_grad(pl, hidden, vocab, xs, ws, yl, gl, o[0], None, o[1], o[2], sp)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call(out, space)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        call(out, space)
    for t in xs:
        t.mul_(-0.5)
    graph.replay()
    torch.cuda.synchronize()
    eager = [torch.empty_like(t) for t in out[0]], [torch.empty_like(t) for t in out[1]], torch.empty_like(ws)
    call(eager, torch.empty_like(space))
    basp.basp_get_status()
    assert all(torch.equal(a, b) for a, b in zip(out[0] + out[1] + [out[2]], eager[0] + eager[1] + [eager[2]]))


def test_the_weight_of_a_token_without_a_label_has_no_part(basp):
    """1 / (number of labels) is infinite where a shard's tokens have none: the summed loss and its gradients leave them out."""
    from paper_2609_03151_b200.autograd import basp_lm_loss
    w, hidden, vocab = L("no_label", 2, 1, 40, 64, 600)
    pl = make_plan(basp, w)
    W, x, labels, weights = inputs(pl, hidden, vocab, 8)
    labels[0][3], labels[0][4], labels[1][:] = -100, vocab, -100
    c = lambda ts: [t.cuda() for t in ts]
    grads = []
    for odd in (1.0, float("inf"), float("nan")):
        weights[0][3] = weights[0][4] = odd
        weights[1][:] = odd
        xl, wl = [t.requires_grad_() for t in c(x)], W.cuda().requires_grad_()
        loss = basp_lm_loss(pl, xl, wl, c(labels), c(weights))
        grads.append((loss.detach(), *torch.autograd.grad(loss, [*xl, wl])))
    assert all(torch.isfinite(t).all().item() for t in grads[0])
    assert all(torch.equal(a, b) for other in grads[1:] for a, b in zip(grads[0], other))


@pytest.mark.parametrize("mode", [torch.no_grad, torch.inference_mode])
def test_an_evaluation_computes_the_loss_alone(basp, mode):
    """Without a backward to come there are no gradients, whatever the head's requires_grad: the launches are those of
    basp_lm_loss_fwd, and nothing of the gradients' size is allocated."""
    from paper_2609_03151_b200.autograd import basp_lm_loss
    w, hidden, vocab = L("eval", 2, 1, 300, 256, 20000)
    pl = make_plan(basp, w)
    W, x, labels, weights = inputs(pl, hidden, vocab, 10)
    c = lambda ts: [t.cuda() for t in ts]
    xl, wl, yl, gl = [t.requires_grad_() for t in c(x)], W.cuda().requires_grad_(), c(labels), c(weights)
    loss = basp_lm_loss(pl, xl, wl, yl, gl)
    out = [torch.empty(t.shape[0], device="cuda") for t in x]
    ws = torch.empty(basp.basp_lm_loss_fwd_workspace_bytes(pl, vocab), dtype=torch.uint8, device="cuda")
    before = basp.basp_launch_count()
    basp.basp_lm_loss_fwd(pl, hidden, vocab, [t.detach() for t in xl], wl.detach(), yl, out, None, ws)
    alone = basp.basp_launch_count() - before
    del ws
    torch.cuda.synchronize()
    torch.cuda.reset_peak_memory_stats()
    held, before = torch.cuda.memory_allocated(), basp.basp_launch_count()
    with mode():
        value = basp_lm_loss(pl, xl, wl, yl, gl)
    assert basp.basp_launch_count() - before == alone
    assert torch.cuda.max_memory_allocated() - held < wl.numel() * 2
    assert torch.equal(value, loss) and not value.requires_grad


def test_weights_far_apart(basp):
    """Weights down to 2^-100 of the largest keep their token's dx to the same share of itself: of dz only what is below 2^-26 of a row's
    largest passes into numbers of fewer bits."""
    w, hidden, vocab = L("apart", 1, 1, 96, 128, 900)
    pl = make_plan(basp, w)
    W, x, labels, _ = inputs(pl, hidden, vocab, 13)
    labels = [torch.where((y < 0) | (y >= vocab), 5, y) for y in labels]
    weights = [2.0 ** -torch.tensor([0.0, 40.0, 80.0, 100.0]).repeat(24)]
    ref = oracle.lm_loss(f64(x[0]), f64(W), labels[0].numpy(), weights[0].numpy().astype(np.float64))
    _, _, dx, _ = run(basp, pl, hidden, vocab, W, x, labels, weights)
    off = np.linalg.norm(f64(dx[0]) - ref["dx"], axis=1)
    assert (off <= 2.0 ** -7 * np.linalg.norm(ref["dx"], axis=1)).all()       # one row: two roundings at most, 2^-8 each
