"""Sizes, inputs, plain forms and 64-bit values of the operators around the attention layer of a training step.

  norm_rope   RMS norm of every query and key head with the rotary position embedding, forward and backward
              (basp_qk_norm_rope, basp_qk_norm_rope_bwd)
  ckpt        activations of the layer kept in 8 bits between the passes and brought back head-sharded
              (basp_ckpt_pack, basp_ckpt_reshard_s2h)
  loss        softmax cross entropy of the language-model head over the whole vocabulary, without keeping the logits,
              alone and with its gradients (basp_lm_loss_fwd, basp_lm_loss_grad)

`run` computes the plain form with elementary torch operations, or makes the library's calls where `own` is true.
Every case uses the BASP grouping (one sequence per group), so the ranks' sequence shards, one after another, are the
tokens of the micro-batch in order.
"""
import math

import torch

own = False

EPS = 1e-6                # of the head norms
CODE_MAX = 127.0          # largest magnitude of an 8-bit code
ROW_ZERO = 2.0 ** -100    # a head vector whose largest magnitude is below this is stored as zeros
IGNORED = -100            # label of a token without a loss (prompt or padding)


# ---------------------------------------------------------------------------------------------- cases
def _layer(op, name, N, B, S, Hq, Hkv, D, **more):
    return {"op": op, "name": name, "N": N, "B": B, "S": S, "Hq": Hq, "Hkv": Hkv, "D": D, **more}


def listed():
    return [
        # one token on one rank: the smallest call, latency only
        _layer("norm_rope", "norm_rope fwd 1 token", 1, 1, 1, 32, 8, 128, backward=False),
        # a micro-batch of two 8K sequences on 8 ranks, as many key heads as query heads
        _layer("norm_rope", "norm_rope fwd 2x8K", 8, 2, 8192, 32, 32, 128, backward=False),
        # a length the group size does not divide, a head dimension that is no power of two
        _layer("norm_rope", "norm_rope bwd odd D80", 4, 2, 5001, 20, 4, 80, backward=True),
        # the 128K-token training step
        _layer("norm_rope", "norm_rope bwd 128K", 8, 1, 131072, 32, 8, 128, backward=True),
        # a tiny layer: latency of the two calls
        _layer("ckpt", "ckpt 2x1K D64", 4, 2, 1024, 8, 8, 64),
        # more ranks in a group than key heads (replicated key heads), odd length, odd head dimension
        _layer("ckpt", "ckpt odd D96", 8, 1, 10007, 16, 4, 96),
        # two 32K sequences of an 8B model
        _layer("ckpt", "ckpt 2x32K", 8, 2, 32768, 32, 8, 128),
        # one token's loss against a small vocabulary: a pass over the weights
        _layer("loss", "loss fwd 1 token", 1, 1, 1, 32, 8, 128, hidden=2048, vocab=32000, grad=False),
        # evaluation of two 8K sequences of a 1B model
        _layer("loss", "loss fwd 2x8K", 8, 2, 8192, 32, 8, 64, hidden=2048, vocab=128256, grad=False),
        # a short fine-tuning batch: few rows against the whole weight matrix, forward and backward
        _layer("loss", "loss grad 48 tokens", 2, 2, 24, 32, 8, 128, hidden=4096, vocab=32000, grad=True),
        # odd length, odd vocabulary
        _layer("loss", "loss grad odd", 4, 1, 2043, 20, 4, 128, hidden=2560, vocab=50257, grad=True),
        # training step of an 8B model on 8K tokens
        _layer("loss", "loss grad 8K", 8, 1, 8192, 32, 8, 128, hidden=4096, vocab=128256, grad=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _length(rng, K, hi):
    """A sequence length of at least one token for each of K ranks, odd ones among them."""
    while True:
        S = max(K, _log(rng, 1, hi))
        if (K - 1) * (-(-S // K)) < S:
            return S


def draw(rng):
    op = rng.choice(["norm_rope", "ckpt", "loss"])
    B = rng.choice([1, 1, 2, 4])
    K = rng.choice([1, 2, 4])
    N = B * K
    group = rng.choice([1, 2, 4, 5])
    Hkv = rng.choice([4, 8, 12])
    Hq = Hkv * group
    if op == "norm_rope":
        D = rng.choice([16, 32, 48, 64, 80, 96, 112, 128, 128])
        S = _length(rng, K, min(131072, 131072 * 40 * 128 // (B * (Hq + Hkv) * D)))
        return {"op": op, "N": N, "B": B, "S": S, "Hq": Hq, "Hkv": Hkv, "D": D, "backward": rng.random() < 0.5}
    if op == "ckpt":
        D = rng.choice([16, 32, 64, 80, 96, 112, 128, 128])
        S = _length(rng, K, min(65536, 2 * 32768 * 80 * 128 // (B * 2 * (Hq + Hkv) * D)))
        return {"op": op, "N": N, "B": B, "S": S, "Hq": Hq, "Hkv": Hkv, "D": D}
    hidden = 8 * _log(rng, 32, 512)
    vocab = _log(rng, 1000, 131072)
    S = _length(rng, K, max(K, min(8192, 8192 * 4096 * 128256 // (hidden * vocab)) // B))
    return {"op": op, "N": N, "B": B, "S": S, "Hq": Hq, "Hkv": Hkv, "D": 64, "hidden": hidden, "vocab": vocab,
            "grad": rng.random() < 0.6}


def _geometry(c):
    """Ranks of a group, tokens of a rank, and the tokens of every rank in order."""
    K = c["N"] // c["B"]
    T = -(-c["S"] // K)
    return K, T, [min(T, c["S"] - l * T) for _ in range(c["B"]) for l in range(K)]


# --------------------------------------------------------------------------------------------- inputs
def _shards(t, c):
    """The ranks' sequence shards of a tensor over all tokens [B*S, ...]."""
    return list(torch.split(t, _geometry(c)[2]))


def _library(c):
    """What a program that uses the library keeps between calls: the plan and the workspaces."""
    from paper_2609_03151_b200 import binding as lib
    plan = lib.basp_plan_create(c["N"], c["B"], c["S"], c["Hq"], c["Hkv"], c["D"])
    need = {
        "norm_rope": lambda: lib.basp_qk_norm_rope_bwd_workspace_bytes(plan) if c["backward"] else 0,
        "ckpt": lambda: 0,
        "loss": lambda: (lib.basp_lm_loss_grad_workspace_bytes(plan, c["hidden"], c["vocab"]) if c["grad"]
                         else lib.basp_lm_loss_fwd_workspace_bytes(plan, c["vocab"])),
    }[c["op"]]()
    ckpt = [torch.empty(lib.basp_ckpt_bytes(plan, r), dtype=torch.uint8, device="cuda") for r in range(c["N"])] \
        if c["op"] == "ckpt" else None
    return {"lib": lib, "plan": plan, "ckpt": ckpt, "workspace": torch.empty(max(16, need), dtype=torch.uint8, device="cuda")}


def prepare(case, seed):
    c = case
    g = torch.Generator(device="cuda").manual_seed(seed)
    rows = c["B"] * c["S"]

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32)

    def heads(h):
        """Activations of h heads: every head at its own scale."""
        return (normal(rows, h, c["D"]) * torch.exp(0.5 * normal(1, h, 1))).to(torch.bfloat16)

    s = {"case": c, "library": _library(c) if own else None}
    if c["op"] == "norm_rope":
        s["q"], s["k"] = _shards(heads(c["Hq"]), c), _shards(heads(c["Hkv"]), c)
        s["w_q"], s["w_k"] = ((1.0 + 0.2 * normal(c["D"])).to(torch.bfloat16) for _ in range(2))
        j = torch.arange(c["D"] // 2, dtype=torch.float64, device="cuda")
        angle = (500000.0 ** (-2.0 * j / c["D"]))[:, None] * torch.arange(c["S"], dtype=torch.float64, device="cuda")
        s["cos"], s["sin"] = torch.cos(angle).float(), torch.sin(angle).float()          # [D/2, S], feature-major
        if c["backward"]:
            s["dq_out"], s["dk_out"] = _shards(heads(c["Hq"]), c), _shards(heads(c["Hkv"]), c)
            s["dw_q"], s["dw_k"] = (torch.empty(c["D"], device="cuda") for _ in range(2))
        s["q_res"], s["k_res"] = ([torch.empty_like(t) for t in s[n]] for n in ("q", "k"))
    elif c["op"] == "ckpt":
        s["q"], s["k"], s["v"], s["o"] = (_shards(heads(h), c) for h in (c["Hq"], c["Hkv"], c["Hkv"], c["Hq"]))
        K = _geometry(c)[0]
        shape = {n: (1, c["S"], max(1, h // K), c["D"]) for n, h in (("q", c["Hq"]), ("k", c["Hkv"]))}
        s["head"] = [[torch.empty(shape[n], dtype=torch.bfloat16, device="cuda") for _ in range(c["N"])] for n in "qkkq"]
    else:
        w = normal(c["vocab"], c["hidden"]).mul_(c["hidden"] ** -0.5).to(torch.bfloat16)
        labels = torch.randint(0, c["vocab"], (rows,), generator=g, device="cuda")
        # the final norm's output: noise, and a share of the target's own direction, from none to a confident prediction
        sure = 16.0 * torch.rand((rows, 1), generator=g, device="cuda")
        x = (normal(rows, c["hidden"]) + sure * w[labels].float()).to(torch.bfloat16)
        labels = torch.where(torch.rand(rows, generator=g, device="cuda") < 0.1, IGNORED, labels)
        weight = (labels >= 0) / (labels >= 0).sum().clamp(min=1).float()                # the mean over the tokens with a label
        s["x"], s["labels"], s["weight"] = _shards(x, c), _shards(labels, c), _shards(weight, c)
        s["w"] = w
        s["loss"], s["lse"] = ([torch.empty(t.shape[0], device="cuda") for t in s["x"]] for _ in range(2))
        if c["grad"]:
            s["dx"], s["dw"] = [torch.empty_like(t) for t in s["x"]], torch.empty_like(w)
    return s


# ------------------------------------------------------------------------------------------ one pass
def run(state):
    if own:
        return _own(state)
    c = state["case"]
    if c["op"] == "norm_rope":
        return _plain_norm_rope(state, torch.float32)
    if c["op"] == "ckpt":
        return _plain_ckpt(state, c)
    return _plain_loss(state, c)


def _own(s):
    c, h = s["case"], s["library"]
    lib, plan = h["lib"], h["plan"]
    if c["op"] == "norm_rope":
        args = (plan, s["q"], s["k"], s["w_q"], s["w_k"], s["cos"], s["sin"])
        if not c["backward"]:
            lib.basp_qk_norm_rope(*args, s["q_res"], s["k_res"], eps=EPS)
            return {"q": s["q_res"], "k": s["k_res"]}
        lib.basp_qk_norm_rope_bwd(*args, s["dq_out"], s["dk_out"], s["q_res"], s["k_res"], s["dw_q"], s["dw_k"],
                                  h["workspace"], eps=EPS)
        return {"dq": s["q_res"], "dk": s["k_res"], "dw_q": s["dw_q"], "dw_k": s["dw_k"]}
    if c["op"] == "ckpt":
        lib.basp_ckpt_pack(plan, s["q"], s["k"], s["v"], s["o"], h["ckpt"])
        lib.basp_ckpt_reshard_s2h(plan, h["ckpt"], *s["head"])
        return s["head"]
    args = (plan, c["hidden"], c["vocab"], s["x"], s["w"], s["labels"])
    if not c["grad"]:
        lib.basp_lm_loss_fwd(*args, s["loss"], s["lse"], h["workspace"])
        return {"loss": s["loss"], "lse": s["lse"]}
    lib.basp_lm_loss_grad(*args, s["weight"], s["loss"], s["lse"], s["dx"], s["dw"], h["workspace"])
    return {"loss": s["loss"], "lse": s["lse"], "dx": s["dx"], "dw": s["dw"]}


def _rotate(x, cos, sin):
    lo, hi = x.chunk(2, dim=-1)
    return torch.cat([lo * cos - hi * sin, hi * cos + lo * sin], dim=-1)


def _plain_norm_rope(s, t):
    c = s["case"]
    cos, sin = (s[n].to(t).t().repeat(c["B"], 1)[:, None, :] for n in ("cos", "sin"))    # [B*S, 1, D/2]

    def forward(x, w):
        x = torch.cat(x).to(t)
        return _rotate(x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * w.to(t), cos, sin)

    def backward(x, w, dy):
        x, w = torch.cat(x).to(t), w.to(t)
        r = torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS)
        n = x * r
        dz = _rotate(torch.cat(dy).to(t), cos, -sin)                                     # the rotation's transpose
        dw = (dz * n).sum((0, 1), dtype=torch.float64)
        dn = dz * w
        return r * (dn - n * (dn * n).mean(-1, keepdim=True)), dw

    down = torch.bfloat16 if t == torch.float32 else t
    if not c["backward"]:
        return {"q": _shards(forward(s["q"], s["w_q"]).to(down), c), "k": _shards(forward(s["k"], s["w_k"]).to(down), c)}
    dq, dw_q = backward(s["q"], s["w_q"], s["dq_out"])
    dk, dw_k = backward(s["k"], s["w_k"], s["dk_out"])
    return {"dq": _shards(dq.to(down), c), "dk": _shards(dk.to(down), c), "dw_q": dw_q.to(t), "dw_k": dw_k.to(t)}


def _to_heads(x, c):
    """All tokens [B*S, H, D] as the ranks' head shards [1, S, H/K, D] (a group with more ranks than heads: one head each,
    the same for K/H ranks in a row)."""
    K, h = c["N"] // c["B"], x.shape[1]
    x = x.reshape(c["B"], c["S"], h, c["D"])
    if h < K:
        x = x.repeat_interleave(K // h, dim=2)
    per = x.shape[2] // K
    return [x[r // K:r // K + 1, :, (r % K) * per:(r % K + 1) * per].contiguous() for r in range(c["N"])]


def _plain_ckpt(s, c):
    def kept(x):
        x = torch.cat(x).float()
        top = x.abs().amax(-1, keepdim=True)
        code = torch.where(top < ROW_ZERO, torch.zeros_like(x), torch.round(x * (CODE_MAX / top)))
        return (code * torch.where(top < ROW_ZERO, torch.zeros_like(top), top / CODE_MAX)).to(torch.bfloat16)

    return [_to_heads(kept(s[n]), c) for n in "qkvo"]


def _plain_loss(s, c):
    x, w = torch.cat(s["x"]).float(), s["w"].float()
    labels = torch.cat(s["labels"])
    valid, at = labels >= 0, labels.clamp(min=0)[:, None]
    z = x @ w.t()
    top = z.amax(-1, keepdim=True)
    e = torch.exp(z - top)
    # the target apart from the others: lse - z[target] of a confident prediction would cancel
    others = e.scatter(1, at, torch.where(valid[:, None], 0.0, e.gather(1, at))).sum(-1, keepdim=True).log() + top
    away = others - z.gather(1, at)
    loss = torch.where(valid[:, None], away.clamp(min=0) + torch.log1p(torch.exp(-away.abs())), 0.0)
    lse = torch.where(valid[:, None], z.gather(1, at) + loss, others)
    out = {"loss": _shards(loss[:, 0], c), "lse": _shards(lse[:, 0], c)}
    if c["grad"]:
        d = torch.exp(z - lse)
        d.scatter_(1, at, -torch.sigmoid(away))
        d *= torch.where(valid, torch.cat(s["weight"]), 0.0)[:, None]
        out["dx"] = _shards((d @ w).to(torch.bfloat16), c)
        out["dw"] = (d.t() @ x).to(torch.bfloat16)
    return out


# ------------------------------------------------------------------------------------------- 64 bits
def exact(case, seed):
    c, s = case, prepare(case, seed)
    f8 = torch.float64
    if c["op"] == "norm_rope":
        # y = A z with z = x w / sqrt(mean x^2 + eps) and A the rotation; written with complex numbers, the pair
        # (j, j + D/2) of a head as one number
        half = c["D"] // 2
        turn = torch.complex(s["cos"].to(f8), s["sin"].to(f8)).t()                       # [S, D/2]

        def pairs(x):
            x = torch.cat(x).to(f8).reshape(c["B"], c["S"], -1, c["D"])
            return torch.complex(x[..., :half].contiguous(), x[..., half:].contiguous())

        def flat(z):
            return _shards(torch.cat([z.real, z.imag], -1).reshape(c["B"] * c["S"], -1, c["D"]), c)

        def weights(w):
            return torch.complex(w[:half].to(f8), torch.zeros_like(w[:half].to(f8))), \
                torch.complex(w[half:].to(f8), torch.zeros_like(w[half:].to(f8)))

        def scaled(z, w):
            (a, b) = weights(w)
            return torch.complex(z.real * a.real, z.imag * b.real)

        def size(z):
            return (z.real.square() + z.imag.square()).sum(-1, keepdim=True) / c["D"] + EPS

        if not c["backward"]:
            return {n: flat(scaled(pairs(s[n]) / size(pairs(s[n])).sqrt(), s["w_" + n]) * turn[:, None]) for n in "qk"}
        out = {}
        for n in "qk":
            z, up = pairs(s[n]), pairs(s["d%s_out" % n]) * turn.conj()[:, None]
            m = size(z)
            grad_w = torch.cat([(up.real * z.real / m.sqrt()).sum((0, 1, 2)), (up.imag * z.imag / m.sqrt()).sum((0, 1, 2))])
            up = scaled(up, s["w_" + n])
            along = (up.real * z.real + up.imag * z.imag).sum(-1, keepdim=True)
            # d/dx of x m^(-1/2): m^(-1/2) up - x (x . up) m^(-3/2) / D
            out["d" + n], out["dw_" + n] = flat(up * m.rsqrt() - z * (along * m ** -1.5 / c["D"])), grad_w
        return out
    if c["op"] == "ckpt":
        # whole steps of a 127th of the vector's largest magnitude, the nearest one
        def kept(x):
            x = torch.cat(x).to(f8)
            step = x.abs().amax(-1, keepdim=True) / CODE_MAX
            return torch.where(step * CODE_MAX < ROW_ZERO, torch.zeros_like(x), torch.round(x / step) * step)

        return [_to_heads(kept(s[n]), c) for n in "qkvo"]
    x, w, labels = torch.cat(s["x"]).to(f8), s["w"].to(f8), torch.cat(s["labels"])
    if 6.0 * x.shape[0] * w.numel() > 4e13:
        return None
    z = torch.matmul(x, w.mT)
    lse = torch.logsumexp(z, -1)
    keep = (labels != IGNORED).to(f8)
    rows = torch.arange(x.shape[0], device="cuda")
    target = labels.clamp(min=0)
    out = {"loss": _shards((lse - z[rows, target]) * keep, c), "lse": _shards(lse, c)}
    if c["grad"]:
        p = z.sub_(lse[:, None]).exp_()
        p[rows, target] -= 1.0
        p.mul_((keep * torch.cat(s["weight"]).to(f8))[:, None])
        out["dx"], out["dw"] = _shards(torch.matmul(p, w), c), torch.matmul(p.mT, x)
    return out


# ---------------------------------------------------------------------------------------------- work
def work(case):
    c = case
    rows = c["B"] * c["S"]
    if c["op"] == "norm_rope":
        e = rows * (c["Hq"] + c["Hkv"]) * c["D"]
        tables = 4 * c["S"] * c["D"] + 4 * c["D"]
        return {"bytes": e * (6 if c["backward"] else 4) + tables, "flops": e * (20 if c["backward"] else 8)}
    if c["op"] == "ckpt":
        # the activations read, codes and scales written by one call and read by the other, the head shards written
        K = c["N"] // c["B"]
        e, v = rows * 2 * (c["Hq"] + c["Hkv"]) * c["D"], rows * 2 * (c["Hq"] + c["Hkv"])
        written = rows * 2 * (c["Hq"] + max(K, c["Hkv"])) * c["D"]
        return {"bytes": 2 * e + 2 * (e + 4 * v) + 2 * written, "flops": 5 * e}
    x, w, z = rows * c["hidden"], c["vocab"] * c["hidden"], rows * c["hidden"] * c["vocab"]
    per_token = 8 * rows + 8 * rows
    if not c["grad"]:
        return {"bytes": 2 * x + 2 * w + per_token, "flops": 2 * z}
    return {"bytes": 4 * x + 4 * w + per_token + 4 * rows, "flops": 6 * z}
