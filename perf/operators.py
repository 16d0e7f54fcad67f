"""Performance cases of the operators around the attention: token norms, rotary positions, differential attention.

A case is one use of an operator as a video-DiT layer (or a causal model's layer over a cache) makes it:

* ``norm``: layer norm or RMS norm of the rows of a [B, H, N, C] tensor; hidden rows (H = 1, C the model's width, with
  adaptive weights per sample) or heads (C = d); ``norm_train`` is the forward pass with its statistics and the backward
  pass with the gradients of the weights.
* ``rope``: rotary positions of Q and K in one call, over the latent grid or at given positions; ``inverse`` is the
  transposed rotation, which takes gradients back.
* ``diff``: differential attention O = (softmax(Q1 K1') - lam softmax(Q2 K2')) V, where the maps use the two halves of a
  head's channels: prompts, and few tokens over a padded cache; ``diff_train`` is the forward pass with what the backward
  pass needs, and the backward pass.

Fields of a case: ``op``, batch ``B``, heads ``H`` (and ``Hk`` of K and V), tokens ``N`` (and ``M`` keys), width ``C`` or
head width ``d``, ``dtype``, and the switches of the operator.
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


def _norm(name, B, H, N, C, dtype="bf16", kind="layer", affine="none", wide=False, train=False, token_major=False):
    """``affine``: none, shared (weight and bias [C]), or adaptive (1 + scale and shift [B, C]); ``wide``: float32 weights."""
    c = dict(op="norm_train" if train else "norm", B=B, H=H, N=N, C=C, dtype=dtype, kind=kind, affine=affine, wide=wide,
             token_major=token_major)
    return c if name is None else dict(name=name, **c)


def _rope(name, B, H, Hk, d, T=0, Hg=0, Wg=0, N=0, dtype="bf16", layout="interleaved", block=0, rot=0, scaling="none",
          base=10000.0, factor=1.0, orig_len=4096, first=0, inverse=False, token_major=False):
    """Positions are the latent grid T x Hg x Wg, or N tokens a sample, from position ``first`` on."""
    block = block or d
    c = dict(op="rope", B=B, H=H, Hk=Hk, d=d, T=T, Hg=Hg, Wg=Wg, N=N or T * Hg * Wg, dtype=dtype, layout=layout, block=block,
             rot=rot or block, scaling=scaling, base=base, factor=factor, orig_len=orig_len, first=first, inverse=inverse,
             token_major=token_major)
    return c if name is None else dict(name=name, **c)


def _diff(name, B, H, Hk, d, N, M=0, dtype="bf16", causal=False, ragged=False, train=False, token_major=False):
    """``ragged``: sample b has M - b M / (2 B) valid keys (a padded cache or batch)."""
    c = dict(op="diff_train" if train else "diff", B=B, H=H, Hk=Hk, d=d, N=N, M=M or N, dtype=dtype, causal=causal,
             ragged=ragged, token_major=token_major)
    return c if name is None else dict(name=name, **c)


def listed():
    return [
        # norm of the heads of Q for single tokens of a small batch: launch and latency are the time
        _norm("norm-heads-single", 8, 12, 1, 128, kind="rms", affine="shared"),
        # adaptive layer norm of the hidden rows before a mid-size layer: 32,760 tokens, 12 heads of 128
        _norm("norm-adaptive-mid", 1, 1, 32760, 1536, affine="adaptive"),
        # a training step's norm over a short clip's rows with a learned weight and bias, both passes
        _norm("norm-train-wide", 2, 1, 8190, 5120, affine="shared", wide=True, train=True),
        # rows of an odd width in float32, whose starts are on no vector's boundary, both passes
        _norm("norm-train-odd", 3, 1, 2111, 1283, dtype="fp32", affine="adaptive", train=True),
        # rotary positions of a mid-size layer's Q and K over its latent grid, as the QKV projection leaves them
        _rope("rope-grid-mid", 1, 12, 12, 128, 21, 30, 52, token_major=True),
        # single tokens of many requests at far positions, shared key heads, half of the head, long-context scaling
        _rope("rope-single-far", 32, 32, 8, 128, N=1, layout="half", rot=64, scaling="yarn", factor=16.0, first=50000),
        # the gradient of the rotation of both halves of float32 heads
        _rope("rope-gradient", 2, 20, 20, 128, N=6001, dtype="fp32", layout="half", block=64, inverse=True),
        # differential attention over the whole clip at half the mid layer's frame rate and height
        _diff("diff-clip", 1, 12, 12, 128, 16380, token_major=True),
        # one request's single token over a short cache: latency
        _diff("diff-single-short", 1, 12, 4, 64, 1, 1000, dtype="fp16", causal=True),
        # single tokens of a batch over a padded cache of up to 16,384 keys: the cache has to be read
        _diff("diff-single-long", 16, 32, 8, 128, 1, 16384, causal=True, ragged=True),
        # a causal training step, shared key heads
        _diff("diff-train-causal", 2, 12, 4, 128, 2048, causal=True, train=True),
        # a training step over a padded batch of odd length, narrow heads
        _diff("diff-train-ragged", 3, 6, 6, 64, 777, dtype="fp16", ragged=True, train=True, token_major=True),
    ]


def draw(rng):
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    while True:
        op = rng.choice(["norm", "norm", "norm_train", "norm_train", "rope", "rope", "rope", "diff", "diff", "single",
                         "single", "diff_train", "diff_train"])
        major = rng.random() < 0.5
        if op in ("norm", "norm_train"):
            heads = rng.random() < 0.3
            C = rng.choice([64, 128]) if heads else log(1, 10000) if rng.random() < 0.4 else 8 * log(8, 1250)
            c = _norm(None, rng.randint(1, 8), rng.randint(1, 40) if heads else 1, log(1, 40000), C,
                      dtype=rng.choice(["bf16", "bf16", "fp16", "fp32"]), kind=rng.choice(["layer", "layer", "rms"]),
                      affine=rng.choice(["none", "shared", "adaptive"]), wide=rng.random() < 0.5, train=op == "norm_train",
                      token_major=major)
            if c["B"] * c["H"] * c["N"] * C > 9e7:
                continue
        elif op == "rope":
            d, H = rng.choice([64, 128]), log(1, 40)
            same = dict(dtype=rng.choice(["bf16", "bf16", "fp16", "fp32"]), layout=rng.choice(["interleaved", "half"]),
                        block=rng.choice([d, d, d // 2]), inverse=rng.random() < 0.3, token_major=major)
            Hk = rng.choice([h for h in range(1, H + 1) if H % h == 0])
            if rng.random() < 0.5:
                c = _rope(None, rng.choice([1, 1, 2]), H, Hk, d, log(1, 33), log(2, 45), log(2, 80), **same)
            else:
                scaling = rng.choice(["none", "linear", "ntk", "yarn"])
                c = _rope(None, log(1, 64), H, Hk, d, N=log(1, 16000), rot=same["block"] // rng.choice([1, 1, 2]),
                          scaling=scaling, base=rng.choice([10000.0, 500000.0]),
                          factor=1.0 if scaling == "none" else rng.choice([2.0, 8.0, 40.0]), first=log(1, 120000), **same)
            if c["B"] * (H + Hk) * c["N"] * d > 1.2e8:
                continue
        else:
            H = log(1, 40)
            Hk = rng.choice([h for h in range(1, H + 1) if H % h == 0 and H <= 16 * h])
            N = {"single": rng.choice([1, 1, 2, 5]), "diff": log(1, 9000), "diff_train": log(1, 4000)}[op]
            M = N if op == "diff_train" else N + log(1, 20000) if op == "single" else rng.choice([N, N, N + log(1, 5000)])
            c = _diff(None, log(1, 32), H, Hk, rng.choice([64, 128]), N, M, dtype=rng.choice(["bf16", "bf16", "fp16"]),
                      causal=rng.random() < 0.5, ragged=rng.random() < 0.5, train=op == "diff_train", token_major=major)
            # the scores of a plain pass stay within the largest listed case's, and so do the keys and values
            if c["B"] * H * N * c["M"] > (0.8e9 if op == "diff_train" else 2.4e9) or c["B"] * Hk * c["M"] * c["d"] > 2.6e8:
                continue
        return c


# ---- inputs ------------------------------------------------------------------
def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _empty(c, H, N, C):
    """A [B, H, N, C] tensor, or such a view of [B, N, H, C] storage."""
    dt = DTYPES[c["dtype"]]
    if c["token_major"]:
        return torch.empty((c["B"], N, H, C), dtype=dt, device="cuda").transpose(1, 2)
    return torch.empty((c["B"], H, N, C), dtype=dt, device="cuda")


def _normal(c, g, H, N, C, scale=1.0, shift=0.0):
    """Normal values around a shift of each head and channel."""
    x = _empty(c, H, N, C)
    x.normal_(generator=g)
    x *= scale
    if shift:
        x += shift * torch.randn(c["B"], H, 1, C, generator=g, device="cuda").to(x.dtype)
    return x


def _lens(c):
    return [c["M"] - (b * c["M"]) // (2 * c["B"]) if c["ragged"] else c["M"] for b in range(c["B"])]


def _rot_axis(c):
    if not c["T"]:
        return (c["rot"],)
    side = 2 * (c["rot"] // 6)
    return (c["rot"] - 2 * side, side, side)


def _turns(c):
    """Turns per position of every rotated pair (float64), the axis after axis, and the factor of cosine and sine."""
    turns, scale = [], 1.0
    for D in _rot_axis(c):
        i = torch.arange(0, D, 2, dtype=torch.float64)
        base = c["base"] * (c["factor"] ** (D / (D - 2)) if c["scaling"] == "ntk" and D > 2 else 1.0)
        f = base ** (-i / D)
        if c["scaling"] == "linear":
            f = f / c["factor"]
        if c["scaling"] == "yarn":
            at = [D * math.log(c["orig_len"] / (n * 2 * math.pi)) / (2 * math.log(base)) for n in (32.0, 1.0)]
            lo, hi = max(math.floor(at[0]), 0), min(math.ceil(at[1]), D - 1)
            ramp = ((i / 2 - lo) / max(hi - lo, 0.001)).clamp(0, 1)
            f = f / c["factor"] * ramp + f * (1 - ramp)
            scale = 0.1 * math.log(c["factor"]) + 1.0
        turns.append(f / (2 * math.pi))
    return torch.cat(turns), scale


def prepare(case, seed):
    c, g = case, _gen(seed)
    s = dict(c=c)
    if c["op"] in ("norm", "norm_train"):
        B, H, N, C = c["B"], c["H"], c["N"], c["C"]
        s["X"] = _normal(c, g, H, N, C, 1.5, 0.5)
        s["Y"] = _empty(c, H, N, C)
        s["w"] = s["b"] = None
        if c["affine"] != "none":
            shape = (B, C) if c["affine"] == "adaptive" else (C,)
            wt = torch.float32 if c["wide"] else DTYPES[c["dtype"]]
            s["w"] = (0.2 * torch.randn(shape, generator=g, device="cuda") + (c["affine"] == "shared")).to(wt)
            s["b"] = (0.2 * torch.randn(shape, generator=g, device="cuda")).to(wt)
        if c["op"] == "norm_train":
            s["dY"], s["dX"] = _normal(c, g, H, N, C), _empty(c, H, N, C)
            s["stats"] = torch.empty((B, H, N, 2), device="cuda")
            s["dw"], s["db"] = (None, None) if s["w"] is None else (torch.empty_like(s["w"]), torch.empty_like(s["b"]))
    elif c["op"] == "rope":
        s["Q"], s["K"] = _normal(c, g, c["H"], c["N"], c["d"]), _normal(c, g, c["Hk"], c["N"], c["d"])
        s["Qo"], s["Ko"] = _empty(c, c["H"], c["N"], c["d"]), _empty(c, c["Hk"], c["N"], c["d"])
        turns, s["scale"] = _turns(c)
        s["turns"], s["rot_axis"], s["pos"] = turns.cuda(), _rot_axis(c), None
        if not c["T"]:
            start = c["first"] + torch.randint(0, 1000, (c["B"], 1, 1), generator=g, device="cuda")
            s["pos"] = (start + torch.arange(c["N"], device="cuda")[None, :, None]).to(torch.int32)
    else:
        H, Hk, N, M, d = c["H"], c["Hk"], c["N"], c["M"], c["d"]
        s["Q"], s["K"] = _normal(c, g, H, N, d, 1.5, 0.3), _normal(c, g, Hk, M, d, 1.0, 0.5)
        s["V"] = _normal(c, g, Hk, M, d, 1.0, 0.5)
        s["lam"] = 0.2 + 0.6 * torch.rand(H, generator=g, device="cuda")
        s["O"] = _empty(c, H, N, d)
        s["kv_lens"] = torch.tensor(_lens(c), dtype=torch.int32, device="cuda") if c["ragged"] else None
        # a prompt's first query is its first token; few tokens are the last ones of their cache
        s["q_start"] = torch.zeros(c["B"], dtype=torch.int32, device="cuda") if c["ragged"] and N == M else None
        if c["op"] == "diff_train":
            s["dO"], s["O2"] = _normal(c, g, H, N, d), _empty(c, H, N, d)
            s["dQ"], s["dK"], s["dV"] = _empty(c, H, N, d), _empty(c, Hk, M, d), _empty(c, Hk, M, d)
            s["lse"] = torch.empty((c["B"], H, 2, N), device="cuda")
            s["dlam"] = torch.empty(H, device="cuda")
    return s


# ---- plain forms -----------------------------------------------------------------
def _affine(s, dt):
    """Weight and bias as [B or 1, 1, 1, C] factors."""
    c = s["c"]
    if s["w"] is None:
        return torch.ones(1, 1, 1, 1, dtype=dt, device="cuda"), torch.zeros(1, 1, 1, 1, dtype=dt, device="cuda")
    w, b = (x.to(dt).reshape(-1, 1, 1, c["C"]) for x in (s["w"], s["b"]))
    return (w + 1.0 if c["affine"] == "adaptive" else w), b


def _norm_stats(x, kind, eps):
    mean = x.mean(-1, keepdim=True) if kind == "layer" else torch.zeros_like(x[..., :1])
    var = ((x - mean) * (x - mean)).mean(-1, keepdim=True)
    return mean, 1.0 / torch.sqrt(var + eps)


EPS = 1e-6


def _plain_norm(s):
    c = s["c"]
    dt = DTYPES[c["dtype"]]
    x = s["X"].float()
    w, b = _affine(s, torch.float32)
    mean, r = _norm_stats(x, c["kind"], EPS)
    xh = (x - mean) * r
    out = {"Y": (xh * w + b).to(dt)}
    if c["op"] == "norm_train":
        dy = s["dY"].float()
        gy = dy * w
        m1 = gy.mean(-1, keepdim=True) if c["kind"] == "layer" else 0.0
        out["dX"] = (r * (gy - m1 - xh * (gy * xh).mean(-1, keepdim=True))).to(dt)
        out["stats"] = torch.cat([mean, r], -1)
        if s["w"] is not None:
            over = (1, 2) if c["affine"] == "adaptive" else (0, 1, 2)
            out["dw"], out["db"] = (dy * xh).sum(over).to(s["w"].dtype), dy.sum(over).to(s["b"].dtype)
    return out


def _cos_sin(s):
    """Cosine and sine of every token and pair, float64 [B or 1, 1, N, rot / 2]."""
    c = s["c"]
    if s["pos"] is None:
        n = torch.arange(c["N"], device="cuda")
        pos = torch.stack([n // (c["Hg"] * c["Wg"]), n // c["Wg"] % c["Hg"], n % c["Wg"]], -1)[None]
    else:
        pos = s["pos"]
    axis = torch.cat([torch.full((D // 2,), a, dtype=torch.int64) for a, D in enumerate(s["rot_axis"])]).cuda()
    t = pos.double()[..., axis] * s["turns"]
    angle = ((t - torch.round(t)) * (2 * math.pi))[:, None]
    sign = -1.0 if c["inverse"] else 1.0
    return torch.cos(angle) * s["scale"], torch.sin(angle) * (sign * s["scale"])


def _rotate(x, cos, sin, c):
    """x [B, H, N, d] rotated; cos and sin [.., 1, N, rot / 2]."""
    y = x.reshape(x.shape[:-1] + (c["d"] // c["block"], c["block"]))
    cos, sin = cos[..., None, :], sin[..., None, :]
    r, rest = y[..., :c["rot"]], y[..., c["rot"]:]
    if c["layout"] == "interleaved":
        a, b = r[..., 0::2], r[..., 1::2]
        r = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    else:
        a, b = r[..., :c["rot"] // 2], r[..., c["rot"] // 2:]
        r = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    return torch.cat([r, rest], -1).reshape(x.shape)


def _plain_rope(s):
    c = s["c"]
    cos, sin = (x.float() for x in _cos_sin(s))
    return {"Qo": _rotate(s["Q"].float(), cos, sin, c).to(s["Q"].dtype),
            "Ko": _rotate(s["K"].float(), cos, sin, c).to(s["K"].dtype)}


def _visible(s):
    """Which keys each query sees: [B, 1, 1, 1, N, M]."""
    c = s["c"]
    j = torch.arange(c["M"], device="cuda")[None, None, :]
    lens = torch.tensor(_lens(c), device="cuda")[:, None, None]
    see = (j < lens).expand(-1, c["N"], -1)
    if c["causal"]:
        start = lens - c["N"] if s["q_start"] is None else s["q_start"].long()[:, None, None]
        see = see & (j <= start + torch.arange(c["N"], device="cuda")[None, :, None])
    return see[:, None, None, None]


def _plain_diff(s):
    c = s["c"]
    B, H, Hk, N, M, d = c["B"], c["H"], c["Hk"], c["N"], c["M"], c["d"]
    G, dt, scale = H // Hk, s["Q"].dtype, 1.0 / math.sqrt(d // 2)
    q = s["Q"].float().reshape(B, Hk, G, N, 2, d // 2).transpose(3, 4)           # [B, Hk, G, 2, N, d/2]
    k = s["K"].float().reshape(B, Hk, 1, M, 2, d // 2).transpose(3, 4)           # [B, Hk, 1, 2, M, d/2]
    v = s["V"].float().reshape(B, Hk, 1, M, d)
    lam = s["lam"].reshape(1, Hk, G, 1, 1)
    x = torch.where(_visible(s), torch.matmul(q, k.transpose(-1, -2)) * scale, -math.inf)
    top = x.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    e = torch.exp(x - top)
    total = e.sum(-1, keepdim=True)
    P = e / torch.where(total == 0, 1.0, total)
    del x, e
    C = P[:, :, :, 0] - lam * P[:, :, :, 1]
    out = {"O": torch.matmul(C, v).reshape(B, H, N, d).to(dt)}
    if c["op"] == "diff_train":
        dO = s["dO"].float().reshape(B, Hk, G, N, d)
        out["lse"] = (top + torch.log(total)).reshape(B, H, 2, N)
        out["dV"] = torch.matmul(C.transpose(-1, -2), dO).sum(2).to(dt)
        dP = torch.matmul(dO, v.transpose(-1, -2))[:, :, :, None]
        delta = (P * dP).sum(-1, keepdim=True)
        dS = P * (dP - delta)
        dS = torch.stack([dS[:, :, :, 0], -lam * dS[:, :, :, 1]], 3) * scale
        out["dQ"] = torch.matmul(dS, k).transpose(3, 4).reshape(B, H, N, d).to(dt)
        out["dK"] = torch.matmul(dS.transpose(-1, -2), q).sum(2).transpose(2, 3).reshape(B, Hk, M, d).to(dt)
        out["dlam"] = -delta[:, :, :, 1].sum((0, 3, 4)).reshape(H)
    return out


# ---- the framework's calls ----------------------------------------------------------
def _own_norm(s):
    from paper_2609_32628_amd import api
    c = s["c"]
    plus, out = c["affine"] == "adaptive", {"Y": s["Y"]}
    if c["op"] == "norm":
        api.da2_norm(s["X"], s["Y"], s["w"], s["b"], kind=c["kind"], eps=EPS, plus_one=plus)
        return out
    if "ws" not in s:
        s["ws"] = torch.empty(api.da2_norm_ws_bytes(s["X"], s["w"]), dtype=torch.uint8, device="cuda")
    api.da2_norm(s["X"], s["Y"], s["w"], s["b"], kind=c["kind"], eps=EPS, plus_one=plus, stats=s["stats"])
    api.da2_norm_bwd(s["dY"], s["X"], s["stats"], s["dX"], s["w"], s["dw"], s["db"], kind=c["kind"], plus_one=plus, ws=s["ws"])
    out.update(dX=s["dX"], stats=s["stats"])
    if s["w"] is not None:
        out.update(dw=s["dw"], db=s["db"])
    return out


def _own_rope(s):
    from paper_2609_32628_amd import api
    c = s["c"]
    if "rope" not in s:
        s["rope"] = api.Rope(layout=c["layout"], block=c["block"], rot_axis=s["rot_axis"], turns=s["turns"], scale=s["scale"])
    api.da2_rope(s["rope"], s["Q"], s["Qo"], s["K"], s["Ko"], pos=s["pos"], grid=(c["Hg"], c["Wg"]) if c["T"] else None,
                 inverse=c["inverse"])
    return {"Qo": s["Qo"], "Ko": s["Ko"]}


def _own_diff(s):
    from paper_2609_32628_amd import api
    c = s["c"]
    train = c["op"] == "diff_train"
    if "ws" not in s:
        s["ws"] = torch.empty(api.da2_diff_ws_bytes(s["Q"], s["K"], train), dtype=torch.uint8, device="cuda")
    how = dict(kv_lens=s["kv_lens"], q_start=s["q_start"], causal=c["causal"])
    if not train:
        api.da2_diff_attn(s["Q"], s["K"], s["V"], s["lam"], s["O"], s["ws"], **how)
        return {"O": s["O"]}
    api.da2_diff_attn(s["Q"], s["K"], s["V"], s["lam"], s["O"], s["ws"], lse=s["lse"], **how)
    api.da2_diff_attn_bwd(s["Q"], s["K"], s["V"], s["lam"], s["lse"], s["dO"], s["dQ"], s["dK"], s["dV"], s["dlam"],
                          s["ws"], **how)
    return {n: s[n] for n in ("O", "lse", "dV", "dQ", "dK", "dlam")}


def run(state):
    op = state["c"]["op"]
    if op in ("norm", "norm_train"):
        return _own_norm(state) if own else _plain_norm(state)
    if op == "rope":
        return _own_rope(state) if own else _plain_rope(state)
    return _own_diff(state) if own else _plain_diff(state)


def work(case):
    c = case
    e = 4 if c["dtype"] == "fp32" else 2
    if c["op"] in ("norm", "norm_train"):
        n = c["B"] * c["H"] * c["N"] * c["C"]
        w = 0 if c["affine"] == "none" else 2 * c["C"] * (c["B"] if c["affine"] == "adaptive" else 1) * (4 if c["wide"] else e)
        if c["op"] == "norm":
            return {"bytes": 2 * n * e + w, "flops": 8 * n}
        return {"bytes": 4 * n * e + 2 * w + 8 * n // c["C"], "flops": 22 * n}
    if c["op"] == "rope":
        n = c["B"] * (c["H"] + c["Hk"]) * c["N"] * c["d"]
        return {"bytes": 2 * n * e, "flops": 3 * n * c["rot"] // c["block"]}
    lens, N, d = _lens(c), c["N"], c["d"]
    pairs = sum(n * N for n in lens)
    if c["causal"]:
        start = [0 if c["ragged"] and N == c["M"] else n - N for n in lens]
        pairs = sum(_triangle(n, N, a) for n, a in zip(lens, start))
    q, kv = c["B"] * c["H"] * N * d * e, 2 * sum(lens) * c["Hk"] * d * e
    # multiply-adds of a pair: both maps d, their values 2 d; the backward pass d for each of dP, dV, dK, dQ and the maps
    if c["op"] == "diff":
        return {"bytes": 2 * q + kv, "flops": 2 * 3 * d * pairs * c["H"]}
    return {"bytes": 4 * q + 2 * kv, "flops": 2 * 8 * d * pairs * c["H"]}


def _triangle(n, N, start):
    """Visible pairs of N causal queries from position start on over n keys."""
    return sum(min(max(start + i + 1, 0), n) for i in range(N))


# ---- the same in 64 bits -----------------------------------------------------------
def _exact_norm(s):
    c = s["c"]
    x, B, C = s["X"].double(), c["B"], c["C"]
    mu = x.sum(-1, keepdim=True) / C if c["kind"] == "layer" else x.new_zeros(x.shape[:-1] + (1,))
    r = ((x - mu).square().sum(-1, keepdim=True) / C + EPS).rsqrt()
    xh = (x - mu) * r
    w = b = None
    y = xh
    if s["w"] is not None:
        w = s["w"].double().view(-1, 1, 1, C) + (1 if c["affine"] == "adaptive" else 0)
        b = s["b"].double().view(-1, 1, 1, C)
        y = xh * w + b
    out = {"Y": y}
    if c["op"] == "norm_train":
        dy = s["dY"].double()
        gx = dy if w is None else dy * w
        # dx = J' g for y = xh(x): r (I - 1 1'/C - xh xh'/C) g (without the mean's part for an RMS norm)
        dx = gx - xh * ((gx * xh).sum(-1, keepdim=True) / C)
        if c["kind"] == "layer":
            dx = dx - gx.sum(-1, keepdim=True) / C
        out["dX"] = dx * r
        out["stats"] = torch.cat([mu, r], -1)
        if w is not None:
            per = (dy * xh).flatten(1, 2).sum(1), dy.flatten(1, 2).sum(1)        # [B, C]
            out["dw"], out["db"] = per if c["affine"] == "adaptive" else (per[0].sum(0), per[1].sum(0))
    return out


def _exact_rope(s):
    c = s["c"]
    half, B, N = c["rot"] // 2, c["B"], c["N"]
    dev = "cuda"
    pos = torch.zeros(B, N, half, dtype=torch.float64, device=dev)
    at = 0
    for a, D in enumerate(s["rot_axis"]):
        if s["pos"] is not None:
            p = s["pos"][..., a].double()
        else:
            p = torch.cartesian_prod(*(torch.arange(n, device=dev, dtype=torch.float64) for n in (c["T"], c["Hg"], c["Wg"])))[:, a]
            p = p.expand(B, N)
        pos[..., at:at + D // 2] = p[..., None]
        at += D // 2
    turn = torch.remainder(pos * s["turns"], 1.0)
    z = torch.polar(torch.full_like(turn, s["scale"]), 2 * math.pi * turn)
    if c["inverse"]:
        z = z.conj()
    out = {}
    for name in ("Q", "K"):
        x = s[name].double().clone()
        for o in range(0, c["d"], c["block"]):
            first = slice(o, o + c["rot"], 2) if c["layout"] == "interleaved" else slice(o, o + half)
            second = slice(o + 1, o + c["rot"], 2) if c["layout"] == "interleaved" else slice(o + half, o + c["rot"])
            y = torch.complex(x[..., first].contiguous(), x[..., second].contiguous()) * z[:, None]
            x[..., first], x[..., second] = y.real, y.imag
        out[name + "o"] = x
    return out


def _exact_diff(s):
    c = s["c"]
    B, H, Hk, N, M, d = c["B"], c["H"], c["Hk"], c["N"], c["M"], c["d"]
    train, G, h = c["op"] == "diff_train", H // Hk, d // 2
    root = math.sqrt(h)
    new = lambda *n: torch.zeros(n, dtype=torch.float64, device="cuda")  # noqa: E731
    out = {"O": new(B, H, N, d)}
    if train:
        out.update(lse=torch.full((B, H, 2, N), -math.inf, dtype=torch.float64, device="cuda"), dV=new(B, Hk, M, d),
                   dQ=new(B, H, N, d), dK=new(B, Hk, M, d), dlam=new(H))
    step = max(1, 2 ** 27 // M)
    for b, n in enumerate(_lens(c)):
        start = 0 if s["q_start"] is not None else n - N
        for hq in range(H):
            kh = hq // G
            lam = float(s["lam"][hq])
            K, V = s["K"][b, kh, :n].double(), s["V"][b, kh, :n].double()
            for i in range(0, N, step):
                Q = s["Q"][b, hq, i:i + step].double()
                A = []
                for m in (0, 1):
                    z = Q[:, m * h:(m + 1) * h] @ K[:, m * h:(m + 1) * h].T.contiguous() / root
                    if c["causal"]:
                        last = start + i + torch.arange(Q.shape[0], device="cuda")[:, None]
                        z.masked_fill_(torch.arange(n, device="cuda")[None] > last, -math.inf)
                    if train:
                        out["lse"][b, hq, m, i:i + step] = torch.logsumexp(z, -1)
                    A.append(torch.nan_to_num(torch.softmax(z, -1), nan=0.0))
                out["O"][b, hq, i:i + step] = A[0] @ V - lam * (A[1] @ V)
                if train:
                    dO = s["dO"][b, hq, i:i + step].double()
                    out["dV"][b, kh, :n] += (A[0] - lam * A[1]).T.contiguous() @ dO
                    g = dO @ V.T.contiguous()
                    out["dlam"][hq] -= (A[1] * g).sum()
                    for m, f in ((0, 1.0), (1, -lam)):
                        dz = f * A[m] * (g - (A[m] * g).sum(-1, keepdim=True)) / root
                        out["dQ"][b, hq, i:i + step, m * h:(m + 1) * h] = dz @ K[:, m * h:(m + 1) * h]
                        out["dK"][b, kh, :n, m * h:(m + 1) * h] += dz.T.contiguous() @ Q[:, m * h:(m + 1) * h]
    return out


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] in ("norm", "norm_train"):
        return _exact_norm(s)
    if case["op"] == "rope":
        return _exact_rope(s)
    # float64 products of the scores and values at some tens of TFLOP/s, and a loop over samples and heads
    if case["B"] * case["H"] > 1500 or case["B"] * case["H"] * case["N"] * case["M"] > 4e9:
        return None
    return _exact_diff(s)
