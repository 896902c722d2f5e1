"""Sizes, inputs, plain forms and 64-bit values of the operators of a block that is trained on packed documents.

  attn   attention whose scores are capped, biased by distance and masked by documents, prefixes or a window, on head
         shards: forward alone, or forward and backward (basp_mask_packed, basp_attn_masked_fwd, basp_attn_masked_bwd)
  rope   rotary positions that restart in every document: half or interleaved pairs, part of the head, frequencies scaled
         for long contexts; the inverse rotation is the gradient (basp_rope)
  norm   norms after and before a block with its gate and residual scale, forward and backward
         (basp_block_norm, basp_block_norm_bwd)

`run` computes the plain form with elementary torch operations, or makes the library's calls where `own` is true.
Every case uses the BASP grouping (one sequence per group), so the ranks' sequence shards, one after another, are the
tokens of the micro-batch in order.  A sequence is filled with documents; the lengths follow from the case, their order from
the seed.  `pad` tokens at the end of a sequence belong to no document: position -1.
"""
import math

import numpy as np
import torch

own = False

EPS = 1e-6
THETA = 500000.0          # base of the rotary frequencies
TRAINED = 8192            # context length before it was extended


# ---------------------------------------------------------------------------------------------- cases
def _attn(name, N, B, S, Hq, Hkv, D, docs, **more):
    """docs: documents in a sequence (0: no mask object, the plan's causal mask); prefix: share of every document that all its
    tokens see; window: keys that a token sees at most (0: all); cap: of the scores (0: none); bias: slopes by distance."""
    case = {"op": "attn", "name": name, "N": N, "B": B, "S": S, "Hq": Hq, "Hkv": Hkv, "D": D, "docs": docs, "pad": 0,
            "prefix": 0.0, "window": 0, "cap": 0.0, "bias": False, "train": False}
    return {**case, **more}


def _rope(name, N, B, S, Hq, Hkv, D, rotary, **more):
    """rotary: features that are rotated; start: position of every document's first token (tokens before it are in a cache)."""
    case = {"op": "rope", "name": name, "N": N, "B": B, "S": S, "Hq": Hq, "Hkv": Hkv, "D": D, "rotary": rotary, "docs": 1,
            "start": 0, "pad": 0, "interleaved": False, "scaling": "none", "factor": 1.0, "inverse": False}
    return {**case, **more}


def _norm(name, N, B, S, hidden, **more):
    """post, gate, pre: whether the block's output has a norm of its own, a gate, and the next block a norm."""
    case = {"op": "norm", "name": name, "N": N, "B": B, "S": S, "Hq": N, "Hkv": N, "D": 64, "hidden": hidden, "post": True,
            "gate": True, "pre": True, "scale": 1.0, "backward": False}
    return {**case, **more}


def listed():
    return [
        # two short packed sequences of a tiny model: latency of the mask's and the attention's call
        _attn("attn fwd 2x777 D64", 2, 2, 777, 8, 8, 64, 5, pad=9),
        # evaluation of one packed 32K sequence of an 8B model
        _attn("attn fwd docs 32K", 8, 1, 32768, 32, 8, 128, 24, pad=500),
        # two 4K sequences of a model with capped scores and a window in every other layer
        _attn("attn fwd cap window 2x4K", 8, 2, 4096, 16, 8, 128, 1, window=2048, cap=50.0),
        # odd length and head dimension, prompts that are seen whole, bias by distance
        _attn("attn fwd prefix bias odd D80", 4, 2, 2501, 20, 4, 80, 7, prefix=0.3, bias=True),
        # training step of an 8B model on packed 16K sequences
        _attn("attn train docs 16K", 8, 1, 16384, 32, 8, 128, 12, train=True),
        # odd length, capped and biased scores under the plan's own causal mask, small heads
        _attn("attn train cap bias odd D64", 2, 2, 3001, 12, 4, 64, 0, cap=30.0, bias=True, train=True),
        # one token: latency alone
        _rope("rope 1 token", 1, 1, 1, 32, 8, 128, 128, start=6007, interleaved=True),
        # gradient at an odd length, a head dimension that is no power of two, interleaved pairs in part of the head
        _rope("rope inverse odd D80", 4, 2, 5001, 20, 4, 80, 32, docs=9, interleaved=True, inverse=True),
        # one 64K sequence of an 8B model extended by a factor of 16
        _rope("rope 64K scaled", 8, 1, 65536, 32, 8, 128, 128, docs=40, scaling="yarn", factor=16.0),
        # one token: latency alone
        _norm("norm fwd 1 token", 1, 1, 1, 4096),
        # two 8K sequences of a 1B model without gate
        _norm("norm fwd 2x8K", 8, 2, 8192, 2048, gate=False),
        # training step of an 8B model on 64K tokens
        _norm("norm bwd 64K", 8, 1, 65536, 4096, scale=0.5, backward=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _length(rng, K, hi):
    """A sequence length of at least one token for each of K ranks, odd ones among them."""
    while True:
        S = max(K, _log(rng, 1, max(2, hi)))
        if (K - 1) * (-(-S // K)) < S:
            return S


def draw(rng):
    op = rng.choice(["attn", "attn", "rope", "norm"])
    B = rng.choice([1, 1, 2, 4])
    K = rng.choice([1, 2, 4])
    N = B * K
    Hkv = rng.choice([4, 8, 12])
    Hq = Hkv * rng.choice([1, 2, 4, 5])
    if op == "attn":
        D = rng.choice([16, 32, 48, 64, 80, 96, 112, 128, 128])
        train = rng.random() < 0.5
        most = (16384 ** 2 if train else 32768 ** 2) * 32 * 128
        S = _length(rng, K, min(16384 if train else 32768, int(math.sqrt(most / (B * Hq * 128)))))
        cap, bias = rng.choice([0.0, 0.0, 20.0, 50.0]), rng.random() < 0.4
        docs = 0 if (cap or bias) and rng.random() < 0.3 else max(1, S // _log(rng, min(32, S), S))
        return _attn("", N, B, S, Hq, Hkv, D, docs, pad=rng.choice([0, 0, S // 20]) if docs else 0, cap=cap, bias=bias,
                     prefix=rng.choice([0.0, 0.0, 0.25]) if docs else 0.0,
                     window=rng.choice([0, 0, _log(rng, 1, S)]) if docs else 0, train=train)
    if op == "rope":
        D = rng.choice([16, 32, 48, 64, 80, 96, 112, 128, 128])
        S = _length(rng, K, min(65536, 65536 * 40 * 128 // (B * (Hq + Hkv) * D)))
        scaling = rng.choice(["none", "linear", "yarn", "wavelength"])
        return _rope("", N, B, S, Hq, Hkv, D, 16 * rng.randint(1, D // 16), docs=max(1, S // _log(rng, min(32, S), S)),
                     start=rng.choice([0, _log(rng, 1, 100000)]), pad=rng.choice([0, S // 20]), interleaved=rng.random() < 0.5, scaling=scaling,
                     factor=1.0 if scaling == "none" else rng.choice([2.0, 8.0, 32.0]), inverse=rng.random() < 0.4)
    hidden = 8 * _log(rng, 8, 1024)
    S = _length(rng, K, min(65536, 65536 * 4096 // (B * hidden)))
    post, pre = rng.choice([(True, True), (True, True), (False, True), (True, False)])
    return _norm("", N, B, S, hidden, post=post, pre=pre, gate=rng.random() < 0.5, scale=rng.choice([1.0, 0.5, 0.22]),
                 backward=rng.random() < 0.5)


# --------------------------------------------------------------------------------------------- inputs
def _lengths(c):
    """Lengths of a sequence's documents: log-normal, as the documents of a corpus are, at least one token each."""
    n, total = max(1, c["docs"]), c["S"] - c["pad"]
    n = min(n, total)
    share = np.exp(1.2 * np.array([_normal_quantile((i + 0.5) / n) for i in range(n)]))
    ends = np.floor(np.cumsum(share) / share.sum() * (total - n) + 0.5).astype(np.int64)
    return np.diff(ends, prepend=0) + 1


def _normal_quantile(p):
    """Logistic stand-in for the quantile of a normal distribution."""
    return math.log(p / (1.0 - p)) / 1.702


def _documents(c, g):
    """Positions [B, S] (int32, -1 in the padding) and, for every token, its document's length."""
    lengths = torch.from_numpy(_lengths(c))
    order = torch.randperm(len(lengths) * c["B"], generator=g, device="cuda").cpu()
    pos = torch.full((c["B"], c["S"]), -1, dtype=torch.int32)
    own_length = torch.ones((c["B"], c["S"]), dtype=torch.int64)
    for b in range(c["B"]):
        mine = lengths[order[order // len(lengths) == b] % len(lengths)]
        n = int(mine.sum())
        start = torch.repeat_interleave(torch.cumsum(mine, 0) - mine, mine)
        pos[b, :n] = (torch.arange(n) - start).int()
        own_length[b, :n] = torch.repeat_interleave(mine, mine)
    return pos.cuda(), own_length.cuda()


def _tokens(c):
    """Tokens of every rank in order."""
    K = c["N"] // c["B"]
    T = -(-c["S"] // K)
    return [min(T, c["S"] - l * T) for _ in range(c["B"]) for l in range(K)]


def _shards(t, c):
    """The ranks' sequence shards of a tensor over all tokens [B*S, ...]."""
    return list(torch.split(t, _tokens(c)))


def _rope_shape(c):
    return {"rotary_dim": c["rotary"], "theta": THETA, "interleaved": c["interleaved"], "scaling": c["scaling"],
            "factor": c["factor"], "original_len": TRAINED}


def _library(c):
    """What a program that uses the library keeps between calls: the plan, the workspaces, the rotation's frequencies."""
    from paper_2609_03151_b200 import binding as lib
    plan = lib.basp_plan_create(c["N"], c["B"], c["S"], c["Hq"], c["Hkv"], c["D"])
    h, need, mask = {"lib": lib, "plan": plan}, 0, 0
    if c["op"] == "attn":
        mask = lib.basp_mask_bytes(plan)
        need = lib.basp_attn_masked_bwd_workspace_bytes(plan) if c["train"] else 0
    elif c["op"] == "rope":
        h["rope"] = lib.basp_rope_make(**_rope_shape(c))
    elif c["backward"]:
        need = lib.basp_block_norm_bwd_workspace_bytes(plan, c["hidden"])
    h["mask"], h["workspace"] = (torch.empty(max(16, n), dtype=torch.uint8, device="cuda") for n in (mask, need))
    return h


def prepare(case, seed):
    c = case
    g = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32)

    def heads(*shape):
        """Activations [..., heads, D]: every head at its own scale."""
        return (normal(*shape) * torch.exp(0.3 * normal(shape[-2], 1))).to(torch.bfloat16)

    s = {"case": c, "library": _library(c) if own else None}
    if c["op"] == "attn":
        K = c["N"] // c["B"]
        hq, hkv = c["Hq"] // K, max(1, c["Hkv"] // K)
        shape = {"q": hq, "k": hkv, "v": hkv, **({"do": hq} if c["train"] else {})}
        for n, h in shape.items():
            s[n] = [heads(1, c["S"], h, c["D"]) for _ in range(c["N"])]
        s["o"] = [torch.empty_like(t) for t in s["q"]]
        s["lse"] = [torch.empty((1, hq, c["S"]), device="cuda") for _ in range(c["N"])]
        if c["train"]:
            s["dq"], s["dk"], s["dv"] = ([torch.empty_like(t) for t in s[n]] for n in "qkv")
        s["positions"], length = _documents(c, g)
        s["prefix"] = (length * c["prefix"]).int() if c["prefix"] else None
        s["slopes"] = 2.0 ** (-8.0 * (torch.arange(c["Hq"], device="cuda") + 1.0) / c["Hq"]) if c["bias"] else None
    elif c["op"] == "rope":
        s["q"], s["k"] = (_shards(heads(c["B"] * c["S"], h, c["D"]), c) for h in (c["Hq"], c["Hkv"]))
        s["q_res"], s["k_res"] = ([torch.empty_like(t) for t in s[n]] for n in "qk")
        s["positions"] = _documents(c, g)[0]
        s["positions"] += c["start"] * (s["positions"] >= 0)
    else:
        rows, wide = c["B"] * c["S"], c["hidden"]

        def stream(scale):
            """Activations of the residual stream: a few features much larger than the others."""
            return _shards((scale * normal(rows, wide) * torch.exp(0.5 * normal(wide))).to(torch.bfloat16), c)

        def weight(want, middle):
            return (middle + 0.2 * normal(wide)).to(torch.bfloat16) if want else None

        s["x"], s["y"] = stream(4.0), stream(1.0)
        s["w_post"], s["gate"], s["w_pre"] = weight(c["post"], 1.0), weight(c["gate"], 0.5), weight(c["pre"], 1.0)
        if c["backward"]:
            s["dh"], s["dn"] = stream(1e-3), stream(1e-3) if c["pre"] else None
            s["dx"], s["dy"] = ([torch.empty_like(t) for t in s["x"]] for _ in range(2))
            for n, want in (("dw_post", c["post"]), ("dgate", c["gate"]), ("dw_pre", c["pre"])):
                s[n] = torch.empty(wide, device="cuda") if want else None
        else:
            s["h"] = [torch.empty_like(t) for t in s["x"]]
            s["n"] = [torch.empty_like(t) for t in s["x"]] if c["pre"] else None
    return s


# ------------------------------------------------------------------------------------------ one pass
def run(state):
    if own:
        return _own(state)
    return {"attn": _plain_attn, "rope": _plain_rope, "norm": _plain_norm}[state["case"]["op"]](state)


def _own(s):
    c, h = s["case"], s["library"]
    lib, plan = h["lib"], h["plan"]
    if c["op"] == "attn":
        if c["docs"]:
            lib.basp_mask_packed(plan, s["positions"], h["mask"], prefix=s["prefix"], window=c["window"])
        score = lib.basp_score(softcap=c["cap"], slopes=s["slopes"], mask=h["mask"] if c["docs"] else None)
        lib.basp_attn_masked_fwd(plan, score, s["q"], s["k"], s["v"], s["o"], s["lse"])
        out = {"o": s["o"], "lse": s["lse"]}
        if c["train"]:
            lib.basp_attn_masked_bwd(plan, score, s["q"], s["k"], s["v"], s["o"], s["do"], s["lse"], s["dq"], s["dk"], s["dv"],
                                     h["workspace"])
            out.update(dq=s["dq"], dk=s["dk"], dv=s["dv"])
        return out
    if c["op"] == "rope":
        lib.basp_rope(plan, h["rope"], s["q"], s["k"], s["q_res"], s["k_res"], positions=s["positions"], inverse=c["inverse"])
        return {"q": s["q_res"], "k": s["k_res"]}
    weights = {"w_post": s["w_post"], "gate": s["gate"], "w_pre": s["w_pre"], "res_scale": c["scale"], "eps": EPS}
    if not c["backward"]:
        lib.basp_block_norm(plan, c["hidden"], s["x"], s["y"], s["h"], s["n"], **weights)
        return {"h": s["h"], **({"n": s["n"]} if c["pre"] else {})}
    lib.basp_block_norm_bwd(plan, c["hidden"], s["x"], s["y"], s["dh"], s["dn"], s["dx"], s["dy"], s["dw_post"], s["dgate"],
                            s["dw_pre"], h["workspace"], **weights)
    return {"dx": s["dx"], "dy": s["dy"], **{n: s[n] for n in ("dw_post", "dgate", "dw_pre") if s[n] is not None}}


def _visible(s, b):
    """Which keys [S, S] the queries of sequence b see."""
    c = s["case"]
    at = torch.arange(c["S"], device="cuda")
    if not c["docs"]:
        return at[None, :] <= at[:, None]
    pos = s["positions"][b].long()
    first = at - pos
    end = at + 1
    if s["prefix"] is not None:
        end = torch.maximum(end, first + s["prefix"][b].long())
    if c["window"]:
        first = torch.maximum(first, at - c["window"] + 1)
    return (at[None, :] >= first[:, None]) & (at[None, :] < end[:, None]) & (pos >= 0)[:, None]


def _plain_attn(s):
    c = s["case"]
    K, scale, cap = c["N"] // c["B"], c["D"] ** -0.5, c["cap"]
    out = {n: [torch.empty_like(t) for t in s[n]] for n in ("o", "lse")}
    if c["train"]:
        out.update(dq=[torch.empty_like(t) for t in s["q"]],
                   **{"d" + n: [torch.zeros_like(t, dtype=torch.float32) for t in s[n]] for n in "kv"})
    at = torch.arange(c["S"], device="cuda", dtype=torch.float32)
    # one head of one rank at a time: its scores are [S, S]
    for r in range(c["N"]):
        see, group = _visible(s, r // K), s["q"][r].shape[2] // s["k"][r].shape[2]
        for h in range(s["q"][r].shape[2]):
            q, k, v = (s[n][r][0, :, i].float() for n, i in (("q", h), ("k", h // group), ("v", h // group)))
            z = (q @ k.t()).mul_(scale)
            if cap:
                z = z.div_(cap).tanh_()
                slope = 1.0 - z.square() if c["train"] else None
                z.mul_(cap)
            if c["bias"]:
                z -= s["slopes"][(r % K) * s["q"][r].shape[2] + h] * (at[:, None] - at[None, :]).abs_()
            z.masked_fill_(~see, -math.inf)
            top = z.amax(-1, keepdim=True)
            top = torch.where(top == -math.inf, 0.0, top)
            p = z.sub_(top).exp_()
            total = p.sum(-1, keepdim=True)
            p.div_(torch.where(total == 0, 1.0, total))
            o = p @ v
            out["o"][r][0, :, h] = o.to(torch.bfloat16)
            out["lse"][r][0, h] = (top + total.log())[:, 0]
            if c["train"]:
                do = s["do"][r][0, :, h].float()
                out["dv"][r][0, :, h // group] += p.t() @ do
                d = p.mul_((do @ v.t()).sub_((do * o).sum(-1, keepdim=True))).mul_(scale)
                if cap:
                    d.mul_(slope)
                out["dq"][r][0, :, h] = (d @ k).to(torch.bfloat16)
                out["dk"][r][0, :, h // group] += d.t() @ q
    if c["train"]:
        out["dk"], out["dv"] = ([t.to(torch.bfloat16) for t in out[n]] for n in ("dk", "dv"))
    return out


def _frequencies(c):
    """Frequencies of the pairs in radians a token and the factor on the rotated features."""
    half, L, n = c["rotary"] // 2, float(TRAINED), c["factor"]
    f = THETA ** (-torch.arange(half, dtype=torch.float64, device="cuda") / half)
    if c["scaling"] == "linear":
        return f / n, 1.0
    if c["scaling"] == "yarn":
        # pairs that turn over 32 times in the trained length stay, those that turn less than once are stretched
        low, high = (half * math.log(L / (turns * 2 * math.pi)) / math.log(THETA) for turns in (32.0, 1.0))
        low, high = max(math.floor(low), 0), min(math.ceil(high), 2 * half - 1)
        ramp = ((torch.arange(half, device="cuda", dtype=torch.float64) - low) / max(high - low, 0.001)).clamp(0, 1)
        return f / n * ramp + f * (1 - ramp), 0.1 * math.log(n) + 1.0
    if c["scaling"] == "wavelength":
        # the same by the wave's length: shorter than a quarter of the trained length, or longer than all of it
        keep = ((L * f / (2 * math.pi) - 1.0) / (4.0 - 1.0)).clamp(0, 1)
        return f / n * (1 - keep) + f * keep, 1.0
    return f, 1.0


def _plain_rope(s):
    c = s["case"]
    half = c["rotary"] // 2
    f, factor = _frequencies(c)
    angle = s["positions"].reshape(-1, 1).double() * f
    cos, sin = ((factor * fn(angle)).float()[:, None, :] for fn in (torch.cos, torch.sin))
    if c["inverse"]:
        sin = -sin

    def turned(shards):
        x = torch.cat(shards).float()
        a, b = (x[..., 0:2 * half:2], x[..., 1:2 * half:2]) if c["interleaved"] else (x[..., :half], x[..., half:2 * half])
        a, b = a * cos - b * sin, b * cos + a * sin
        head = torch.stack([a, b], -1).flatten(-2) if c["interleaved"] else torch.cat([a, b], -1)
        return _shards(torch.cat([head, x[..., 2 * half:]], -1).to(torch.bfloat16), c)

    return {"q": turned(s["q"]), "k": turned(s["k"])}


def _plain_norm(s):
    c = s["case"]
    y = torch.cat(s["y"]).float()
    ry = torch.rsqrt(y.square().mean(-1, keepdim=True) + EPS)
    w_post, gate, w_pre = (None if s[n] is None else s[n].float() for n in ("w_post", "gate", "w_pre"))
    z = y * ry * w_post if c["post"] else y
    if not c["backward"]:
        h = torch.cat(s["x"]).float() + c["scale"] * (z * gate if c["gate"] else z)
        out = {"h": _shards(h.to(torch.bfloat16), c)}
        if c["pre"]:
            r = torch.rsqrt(h.square().mean(-1, keepdim=True) + EPS)
            out["n"] = _shards((h * r * w_pre).to(torch.bfloat16), c)
        return out
    dh, sums = torch.cat(s["dh"]).float(), {}
    if c["pre"]:
        h, dn = torch.cat(s["x"]).float(), torch.cat(s["dn"]).float()
        r = torch.rsqrt(h.square().mean(-1, keepdim=True) + EPS)
        n, up = h * r, dn * w_pre
        sums["dw_pre"] = (dn * n).sum(0, dtype=torch.float64).float()
        dh = dh + r * (up - n * (up * n).mean(-1, keepdim=True))
    dz = c["scale"] * dh
    if c["gate"]:
        sums["dgate"] = (dz * z).sum(0, dtype=torch.float64).float()
        dz = dz * gate
    dy = dz
    if c["post"]:
        n = y * ry
        sums["dw_post"] = (dz * n).sum(0, dtype=torch.float64).float()
        dy = dz * w_post
        dy = ry * (dy - n * (dy * n).mean(-1, keepdim=True))
    return {"dx": _shards(dh.to(torch.bfloat16), c), "dy": _shards(dy.to(torch.bfloat16), c),
            **{n: sums[n] for n in ("dw_post", "dgate", "dw_pre") if n in sums}}


# ------------------------------------------------------------------------------------------- 64 bits
def exact(case, seed):
    c, s = case, prepare(case, seed)
    return {"attn": _exact_attn, "rope": _exact_rope, "norm": _exact_norm}[c["op"]](s, c)


def _exact_attn(s, c):
    """Softmax and its gradients by automatic differentiation, document by document where nothing crosses their borders."""
    f8, K = torch.float64, c["N"] // c["B"]
    names = ("o", "lse") + (("dq", "dk", "dv") if c["train"] else ())
    like = {"o": "q", "lse": "lse", "dq": "q", "dk": "k", "dv": "v"}
    out = {n: [torch.zeros_like(t, dtype=f8) for t in s[like[n]]] for n in names}
    for r in range(c["N"]):
        out["lse"][r].fill_(-math.inf)
        pos = s["positions"][r // K].cpu()
        starts = (pos == 0).nonzero()[:, 0].tolist() if c["docs"] else [0]
        stops = starts[1:] + [int((pos >= 0).sum()) if c["docs"] else c["S"]]
        heads, group = s["q"][r].shape[2], s["q"][r].shape[2] // s["k"][r].shape[2]
        for a, b in zip(starts, stops):
            i = torch.arange(a, b, device="cuda", dtype=f8)
            ahead = i[None, :] - i[:, None]                                  # key minus query
            hide = ahead > 0
            if s["prefix"] is not None:
                hide &= (i - a >= s["prefix"][r // K, a])[None, :]
            if c["docs"] and c["window"]:
                hide |= ahead <= -c["window"]
            for h in range(heads):
                leaf = [s[n][r][0, a:b, j].to(f8).requires_grad_(c["train"]) for n, j in (("q", h), ("k", h // group), ("v", h // group))]
                z = torch.matmul(leaf[0], leaf[1].mT) / math.sqrt(c["D"])
                if c["cap"]:
                    z = torch.tanh(z / c["cap"]) * c["cap"]
                if c["bias"]:
                    z = z - ahead.abs() * s["slopes"][(r % K) * heads + h].to(f8)
                z = z.masked_fill(hide, -math.inf)
                o = torch.matmul(torch.softmax(z, -1), leaf[2])
                out["o"][r][0, a:b, h] = o.detach()
                out["lse"][r][0, h, a:b] = torch.logsumexp(z.detach(), -1)
                if c["train"]:
                    dq, dk, dv = torch.autograd.grad(o, leaf, s["do"][r][0, a:b, h].to(f8))
                    out["dq"][r][0, a:b, h] = dq
                    out["dk"][r][0, a:b, h // group] += dk
                    out["dv"][r][0, a:b, h // group] += dv
    return out


def _exact_rope(s, c):
    """Pairs as complex numbers, multiplied by a complex number of the position."""
    half, n = c["rotary"] // 2, c["factor"]
    angle, size = [], 1.0
    for j in range(half):
        w = math.exp(-j / half * math.log(THETA))
        turns = TRAINED * w / (2 * math.pi)
        if c["scaling"] == "linear":
            w /= n
        elif c["scaling"] == "wavelength":
            w = w if turns > 4 else w / n if turns < 1 else (turns - 1) / 3 * w + (4 - turns) / 3 * w / n
        elif c["scaling"] == "yarn":
            of = [half * (math.log(TRAINED / 2 / math.pi) - math.log(t)) / math.log(THETA) for t in (32, 1)]
            first, last = max(0, math.floor(of[0])), min(2 * half - 1, math.ceil(of[1]))
            part = min(1.0, max(0.0, (j - first) / max(1e-3, last - first)))
            w, size = w * (1 - part + part / n), 1 + math.log(n) / 10
        angle.append(w)
    turn = torch.polar(torch.tensor(size, dtype=torch.float64, device="cuda"),
                       s["positions"].reshape(-1, 1, 1).double() * torch.tensor(angle, dtype=torch.float64, device="cuda"))
    turn = turn.conj() if c["inverse"] else turn
    out = {}
    for name in "qk":
        x = torch.cat(s[name]).double()
        part = x[..., :2 * half]
        pair = part.unflatten(-1, (half, 2)) if c["interleaved"] else part.unflatten(-1, (2, half)).mT
        part = torch.view_as_real(torch.view_as_complex(pair.contiguous()) * turn)
        part = part.flatten(-2) if c["interleaved"] else part.mT.flatten(-2)
        out[name] = _shards(torch.cat([part, x[..., 2 * half:]], -1), c)
    return out


def _exact_norm(s, c):
    """Gradients from the definition by automatic differentiation; the backward pass takes the stream behind the block as given."""
    f8 = torch.float64
    rows = max(1, (1 << 27) // c["hidden"])
    leaf = {n: None if s[n] is None else s[n].to(f8).requires_grad_(c["backward"]) for n in ("w_post", "gate", "w_pre")}

    def norm(t, w):
        return t / torch.sqrt(torch.mean(t * t, -1, keepdim=True) + EPS) * w

    def added(y):
        z = y if leaf["w_post"] is None else norm(y, leaf["w_post"])
        return c["scale"] * (z if leaf["gate"] is None else z * leaf["gate"])

    part = {n: torch.split(torch.cat(s[n]), rows) for n in ("x", "y", *(("dh", "dn") if c["backward"] else ())) if s[n] is not None}
    out, sums = {}, {n: 0.0 for n, v in leaf.items() if v is not None}
    for i in range(len(part["x"])):
        x, y = part["x"][i].to(f8), part["y"][i].to(f8)
        if not c["backward"]:
            h = x + added(y)
            got = {"h": h, **({"n": norm(h, leaf["w_pre"])} if c["pre"] else {})}
        else:
            x.requires_grad_(), y.requires_grad_()
            dh = part["dh"][i].to(f8)
            if c["pre"]:
                more, dw = torch.autograd.grad(norm(x, leaf["w_pre"]), (x, leaf["w_pre"]), part["dn"][i].to(f8))
                dh, sums["w_pre"] = dh + more, sums["w_pre"] + dw
            wanted = [n for n in ("w_post", "gate") if leaf[n] is not None]
            dy, *dw = torch.autograd.grad(added(y), (y, *(leaf[n] for n in wanted)), dh)
            for n, v in zip(wanted, dw):
                sums[n] = sums[n] + v
            got = {"dx": dh, "dy": dy}
        for n, t in got.items():
            out.setdefault(n, []).append(t.detach())
    out = {n: _shards(torch.cat(t), c) for n, t in out.items()}
    if c["backward"]:
        out.update({to: sums[n] for n, to in (("w_post", "dw_post"), ("gate", "dgate"), ("w_pre", "dw_pre")) if n in sums})
    return out


# ---------------------------------------------------------------------------------------------- work
def _pairs(c):
    """Visible (query, key) pairs of one head of one sequence."""
    if not c["docs"]:
        return c["S"] * (c["S"] + 1) // 2
    total = 0
    for n in _lengths(c):
        i = np.arange(n)
        end = np.maximum(i + 1, int(n * c["prefix"]))
        total += int((end - (np.maximum(0, i - c["window"] + 1) if c["window"] else 0)).sum())
    return total


def work(case):
    c = case
    rows = c["B"] * c["S"]
    if c["op"] == "attn":
        # q, k, v read, o and lse written; a training step reads do and writes dq, dk and dv besides
        K = c["N"] // c["B"]
        q, kv = rows * c["Hq"] * c["D"], rows * max(K, c["Hkv"]) * c["D"]
        moved = 2 * (2 * q + 2 * kv) + 4 * rows * c["Hq"] + 4 * rows
        moved += 2 * (2 * q + 2 * kv) if c["train"] else 0
        return {"bytes": moved, "flops": (14 if c["train"] else 4) * c["D"] * c["Hq"] * c["B"] * _pairs(c)}
    if c["op"] == "rope":
        e = rows * (c["Hq"] + c["Hkv"])
        return {"bytes": 4 * e * c["D"] + 4 * rows, "flops": 3 * e * c["rotary"]}
    e, used = rows * c["hidden"], c["post"] + c["gate"] + c["pre"]
    if not c["backward"]:
        return {"bytes": (6 + 2 * c["pre"]) * e + 2 * used * c["hidden"], "flops": (3 + 5 * c["post"] + 4 * c["pre"]) * e}
    # the stream is read for the norm before the next block alone, the block's output for its own norm or the gate
    read = 2 * c["pre"] * 2 + 2 + 2 * (c["post"] or c["gate"])
    return {"bytes": (read + 4) * e + 6 * used * c["hidden"], "flops": (4 + 9 * c["post"] + 2 * c["gate"] + 9 * c["pre"]) * e}
