"""More operators of token models, as cases that can be timed and compared: plain torch, and the kernel-level entry points.

A case is a dict of plain values; ``kind`` says which operator it is about:

  rotary   ``cdp_k_head_norm_rotary``, ``cdp_k_head_norm_rotary_backward``: norms of each query and key head and the rotation by position, in one pass
  gated    ``cdp_k_gated_linear``, ``cdp_k_gated_linear_backward``: act(x wg^T) * (x wu^T), the first half of a gated feed-forward block
  linear   ``cdp_k_linear``, ``cdp_k_linear_backward``: act(x w^T + bias) + residual, the projections around it
  logprob  ``cdp_k_token_logprob``, ``cdp_k_token_logprob_backward``: log probabilities of given tokens, entropy and the likeliest tokens of each row

Where ``own`` is false, ``run`` is elementary torch operations in 32 bits (angles in 64), rounded once; ``exact`` is the same from the definitions in 64.
"""
import math
import random

import torch

own = False

DTYPES = {"f32": (0, torch.float32, 4), "bf16": (1, torch.bfloat16, 2)}
ACTS = {"silu": 0, "gelu": 1, "sigmoid": 2, "none": 3}
EPS = 1e-6


def listed():
    return [
        # A few tokens of a toy model, fp32, forward and backward: what the calls cost when there is next to nothing to do.
        dict(name="rotary_small_f32", kind="rotary", dtype="f32", tokens=64, sequences=3, split=1, far=0, heads=4, kv_heads=2, width=16, rotary=16, interleaved=False,
             norm=True, backward=True),
        # Whole prompts of a large model, four query heads to a key head, far from the start of their documents: training, forward and backward.
        dict(name="rotary_long_bf16", kind="rotary", dtype="bf16", tokens=16384, sequences=4, split=2, far=500_000, heads=32, kv_heads=8, width=128, rotary=128,
             interleaved=False, norm=True, backward=True),
        # Odd lengths and head width, pairs beside each other, half of each head rotated, fp32.
        dict(name="rotary_odd_f32", kind="rotary", dtype="f32", tokens=2501, sequences=7, split=3, far=1000, heads=8, kv_heads=8, width=80, rotary=40, interleaved=True,
             norm=True, backward=True),
        # One new token of a large model: the weights are read once.
        dict(name="gated_token_bf16", kind="gated", dtype="bf16", rows=1, inputs=4096, hidden=12288, act="silu", backward=False),
        # 32 x 196 tokens of ViT-B's width, a training step.
        dict(name="gated_vit_bf16", kind="gated", dtype="bf16", rows=6272, inputs=768, hidden=2048, act="gelu", backward=True),
        # A long prompt of a large model, a training step.
        dict(name="gated_large_bf16", kind="gated", dtype="bf16", rows=8192, inputs=4096, hidden=12288, act="silu", backward=True),
        # One micro-batch of the smallest width, fp32, forward and backward.
        dict(name="linear_small_f32", kind="linear", dtype="f32", rows=8, inputs=64, outputs=64, act="silu", bias=True, residual=False, backward=True),
        # A large model's projection back to its width, with the residual, a training step.
        dict(name="linear_wide_bf16", kind="linear", dtype="bf16", rows=8192, inputs=4096, outputs=4096, act="none", bias=False, residual=True, backward=True),
        # Ragged sizes in fp32, a training step.
        dict(name="linear_odd_f32", kind="linear", dtype="f32", rows=1999, inputs=520, outputs=1368, act="gelu", bias=True, residual=True, backward=True),
        # The next token of 16 sequences from a large vocabulary, a tenth of it ruled out, with twenty alternatives.
        dict(name="logprob_sampling_bf16", kind="logprob", dtype="bf16", rows=16, vocab=128000, pitch=128000, top=20, padding=0.0, masked=0.1, scale=1.25, backward=False),
        # The loss of 4096 tokens over a large vocabulary, a quarter of them prompts that are not learnt; its gradient in both directions.
        dict(name="logprob_train_bf16", kind="logprob", dtype="bf16", rows=4096, vocab=128000, pitch=128000, top=0, padding=0.25, masked=0.0, scale=1.0, backward=True),
        # A vocabulary of no round size, rows that begin at any element, with alternatives, fp32.
        dict(name="logprob_words_f32", kind="logprob", dtype="f32", rows=1500, vocab=50257, pitch=50257, top=8, padding=0.1, masked=0.0, scale=0.8, backward=True),
    ]


def _log(rng, lo, hi, step=1):
    """Log-uniform multiple of `step` in [lo, hi]."""
    v = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    return int(min(hi // step * step, max(-(-lo // step) * step, round(v / step) * step)))


def draw(rng):
    kind = rng.choice(["rotary", "gated", "linear", "logprob"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    e = DTYPES[dtype][2]
    if kind == "rotary":
        kv_heads = rng.choice([1, 2, 4, 8])
        heads = kv_heads * rng.choice([1, 2, 3, 4])
        width = rng.choice([16, 32, 40, 64, 64, 80, 96, 128, 128])
        tokens = _log(rng, 1, 190_000_000 // e // ((heads + 2 * kv_heads) * width))
        return dict(kind=kind, dtype=dtype, tokens=tokens, sequences=min(tokens, _log(rng, 1, 64)), split=rng.randint(0, 1000), far=rng.choice([0, 0, 4000, 1_000_000]),
                    heads=heads, kv_heads=kv_heads, width=width, rotary=rng.choice([width, width, width // 2, 2 * rng.randint(1, width // 2)]),
                    interleaved=rng.random() < 0.4, norm=rng.random() < 0.7, backward=rng.random() < 0.6)
    if kind in ("gated", "linear"):
        inputs, width = _log(rng, 32, 4096, 8), _log(rng, 32, 12288, 8)
        most = (400_000_000_000 if dtype == "bf16" else 20_000_000_000) // (inputs * width)
        rows = _log(rng, 1, max(2, min(8192, most)))
        c = dict(kind=kind, dtype=dtype, rows=rows, inputs=inputs, backward=rng.random() < 0.6)
        if kind == "gated":
            return dict(c, hidden=width, act=rng.choice(["silu", "silu", "gelu", "sigmoid"]))
        return dict(c, outputs=width, act=rng.choice(["none", "none", "silu", "gelu"]), bias=rng.random() < 0.5, residual=rng.random() < 0.5)
    vocab = _log(rng, 2, 128000)
    pitch = vocab + rng.choice([0, 0, 1, -vocab % 64])
    rows = _log(rng, 1, min(8192, 1_000_000_000 // e // pitch))
    return dict(kind=kind, dtype=dtype, rows=rows, vocab=vocab, pitch=pitch, top=min(vocab, rng.choice([0, 0, 1, 5, 20, 50])) if rows * vocab < 50_000_000 else 0,
                padding=rng.choice([0.0, 0.1, 0.5]), masked=rng.choice([0.0, 0.0, 0.3]), scale=rng.choice([1.0, 1.0, 1.25, 0.5]), backward=rng.random() < 0.6)


def _positions(case):
    """Tokens of packed sequences of a spread of 1 to 20, each counted from a first position of its own."""
    n, total = case["sequences"], case["tokens"]
    rng = random.Random(case["split"])
    far, res = sorted(rng.randint(0, total) for _ in range(n - 1)), []
    for a, b in zip([0] + far, far + [total]):
        first = rng.randint(0, case["far"])
        res.extend(range(first, first + b - a))
    return res


def prepare(case, seed):
    code, t, e = DTYPES[case["dtype"]]
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    normal = lambda *shape: torch.randn(shape, generator=g, device="cuda")  # noqa: E731
    empty = lambda *shape: torch.empty(shape, dtype=t, device="cuda")  # noqa: E731
    f32 = lambda *shape: torch.empty(shape, device="cuda")  # noqa: E731
    s = dict(case=case, code=code, dtype=t)
    if case["kind"] == "rotary":
        T, H, K, W, R = case["tokens"], case["heads"], case["kv_heads"], case["width"], case["rotary"]
        C = (H + 2 * K) * W
        s.update(qkv=normal(T, C).to(t), positions=torch.tensor(_positions(case), dtype=torch.int32, device="cuda"),
                 freqs=(10000.0 ** (-torch.arange(0, R, 2, device="cuda", dtype=torch.float64) / R)).float(), out=empty(T, C),
                 gamma_q=1 + 0.1 * normal(W) if case["norm"] else None, gamma_k=1 + 0.1 * normal(W) if case["norm"] else None)
        if case["backward"]:
            s.update(dout=normal(T, C).to(t), dqkv=empty(T, C), dgamma_q=f32(W) if case["norm"] else None, dgamma_k=f32(W) if case["norm"] else None,
                     ws=torch.empty(8 * W * min(T, 1024) + 256, dtype=torch.uint8, device="cuda"))
    elif case["kind"] == "gated":
        R, I, H = case["rows"], case["inputs"], case["hidden"]
        s.update(x=normal(R, I).to(t), wg=(normal(H, I) / math.sqrt(I)).to(t), wu=(normal(H, I) / math.sqrt(I)).to(t), h=empty(R, H), g=None, u=None)
        planes = 6 * (R * I + 2 * H * I) + 1024 if e == 4 else 0
        if case["backward"]:
            s.update(g=empty(R, H), u=empty(R, H), dh=normal(R, H).to(t), dx=empty(R, I), dwg=empty(H, I), dwu=empty(H, I))
            planes += (12 if e == 4 else 4) * R * H + 1024 + min(512 << 20, 32 * max(R, 2 * H) * I)  # and room for shared sums
        s["ws"] = torch.empty(planes, dtype=torch.uint8, device="cuda")
    elif case["kind"] == "linear":
        R, I, O = case["rows"], case["inputs"], case["outputs"]
        s.update(x=normal(R, I).to(t), w=(normal(O, I) / math.sqrt(I)).to(t), bias=(0.1 * normal(O)).to(t) if case["bias"] else None,
                 residual=normal(R, O).to(t) if case["residual"] else None, y=empty(R, O), z=None)
        planes = 6 * (R * I + O * I) + 1024 if e == 4 else 0
        if case["backward"]:
            s.update(z=empty(R, O) if case["act"] != "none" else None, dy=normal(R, O).to(t), dx=empty(R, I), dw=empty(O, I), dbias=empty(O) if case["bias"] else None)
            planes += (6 if e == 4 else 2) * R * O + 4 * O * min(R, 256) + 1024 + min(512 << 20, 32 * max(R, O) * I)  # and room for shared sums
        s["ws"] = torch.empty(planes, dtype=torch.uint8, device="cuda")
    else:
        R, V, P = case["rows"], case["vocab"], case["pitch"]
        logits = 2.5 * normal(R, P)
        logits[torch.rand(R, P, generator=g, device="cuda") < case["masked"]] = -math.inf
        # words come by rank, and a model has learnt a little of them
        targets = ((torch.exp(torch.rand(R, generator=g, device="cuda") * math.log(V + 1)).floor() - 1).clamp(0, V - 1)).long()
        logits[torch.arange(R, device="cuda"), targets] = 4 + 3 * normal(R)
        s.update(logits=logits.to(t), logprob=f32(R), entropy=f32(R), lse=f32(R))
        s["targets"] = torch.where(torch.rand(R, generator=g, device="cuda") < case["padding"], torch.full_like(targets, -100), targets).to(torch.int32)
        if case["top"]:
            s.update(top_ids=torch.empty((R, case["top"]), dtype=torch.int32, device="cuda"), top_logprobs=f32(R, case["top"]))
        if case["backward"]:
            s.update(dlogprob=normal(R) / R, dentropy=0.1 * normal(R) / R, dlogits=torch.zeros((R, P), dtype=t, device="cuda"))
        s["ws"] = torch.empty(1 << 20, dtype=torch.uint8, device="cuda")
    return s


def run(s):
    if own:
        return {"rotary": _rotary_own, "gated": _gated_own, "linear": _linear_own, "logprob": _logprob_own}[s["case"]["kind"]](s)
    return {"rotary": _rotary, "gated": _gated, "linear": _linear, "logprob": _logprob}[s["case"]["kind"]](s)


# ---- plain forms ------------------------------------------------------------------------------------------------------
def _turned(c, a, cos, sin):
    """Rows of heads a[T, heads, W] with their pairs turned by the angle of cos, sin [T, 1, rotary / 2]."""
    R = c["rotary"]
    if c["interleaved"]:
        x, y = a[:, :, 0:R:2], a[:, :, 1:R:2]
        turned = torch.stack([x * cos - y * sin, y * cos + x * sin], 3).flatten(2)
    else:
        x, y = a[:, :, :R // 2], a[:, :, R // 2:R]
        turned = torch.cat([x * cos - y * sin, y * cos + x * sin], 2)
    return torch.cat([turned, a[:, :, R:]], 2)


def _rotary(s):
    c, t = s["case"], s["dtype"]
    T, H, K, W = c["tokens"], c["heads"], c["kv_heads"], c["width"]
    angle = s["positions"].double()[:, None, None] * s["freqs"].double()
    cos, sin = torch.cos(angle).float(), torch.sin(angle).float()
    a = s["qkv"].float().reshape(T, H + 2 * K, W)
    x, v = a[:, :H + K], a[:, H + K:]
    gamma = torch.cat([s["gamma_q"].expand(H, W), s["gamma_k"].expand(K, W)]) if c["norm"] else None
    if c["norm"]:
        rho = (x.square().mean(2, keepdim=True) + EPS).rsqrt()
        hat = x * rho
        n = hat * gamma
    else:
        n = x
    res = {"out": torch.cat([_turned(c, n, cos, sin), v], 1).reshape(T, -1).to(t)}
    if c["backward"]:
        d = s["dout"].float().reshape(T, H + 2 * K, W)
        dn = _turned(c, d[:, :H + K], cos, -sin)
        if c["norm"]:
            b = dn * gamma
            dx = rho * (b - hat * (b * hat).mean(2, keepdim=True))
            dgamma = (dn * hat).sum(0)
            res.update(dgamma_q=dgamma[:H].sum(0), dgamma_k=dgamma[H:].sum(0))
        else:
            dx = dn
        res["dqkv"] = torch.cat([dx, d[:, H + K:]], 1).reshape(T, -1).to(t)
    return res


def _act(name, g):
    """An activation and its derivative."""
    if name == "none":
        return g, torch.ones_like(g)
    sig = 1 / (1 + torch.exp(-g))
    if name == "silu":
        return g * sig, sig * (1 + g * (1 - sig))
    if name == "sigmoid":
        return sig, sig * (1 - sig)
    phi = 0.5 * (1 + torch.erf(g * math.sqrt(0.5)))
    return g * phi, phi + g * torch.exp(-0.5 * g * g) * (1 / math.sqrt(2 * math.pi))


def _gated(s):
    c, t = s["case"], s["dtype"]
    x, wg, wu = s["x"].float(), s["wg"].float(), s["wu"].float()
    g, u = torch.matmul(x, wg.t()), torch.matmul(x, wu.t())
    a, da = _act(c["act"], g)
    res = {"h": (a * u).to(t)}
    if c["backward"]:
        dh = s["dh"].float()
        dg, du = dh * u * da, dh * a
        res.update(g=g.to(t), u=u.to(t), dx=(torch.matmul(dg, wg) + torch.matmul(du, wu)).to(t), dwg=torch.matmul(dg.t(), x).to(t), dwu=torch.matmul(du.t(), x).to(t))
    return res


def _linear(s):
    c, t = s["case"], s["dtype"]
    x, w = s["x"].float(), s["w"].float()
    z = torch.matmul(x, w.t())
    if c["bias"]:
        z += s["bias"].float()
    a, da = _act(c["act"], z)
    res = {"y": (a + s["residual"].float() if c["residual"] else a).to(t)}
    if c["backward"]:
        dz = s["dy"].float() * da
        if c["act"] != "none":
            res["z"] = z.to(t)
        res.update(dx=torch.matmul(dz, w).to(t), dw=torch.matmul(dz.t(), x).to(t))
        if c["bias"]:
            res["dbias"] = dz.sum(0).to(t)
    return res


def _logprob(s):
    c, t = s["case"], s["dtype"]
    R, V = c["rows"], c["vocab"]
    used = s["targets"] >= 0
    at = torch.where(used, s["targets"], 0).long()[:, None]
    raw = s["logits"][:, :V].float()
    z = raw * c["scale"]
    m = z.amax(1, keepdim=True)
    ez = (z - m).exp()
    total = ez.sum(1, keepdim=True)
    lse = m + torch.log(total)
    p = ez / total
    zero = torch.zeros((), device="cuda")
    logp = z - lse
    entropy = -torch.where(p > 0, p * logp, zero).sum(1)
    res = {"logprob": torch.where(used, logp.gather(1, at)[:, 0], zero), "entropy": torch.where(used, entropy, zero), "lse": torch.where(used, lse[:, 0], zero)}
    if c["top"]:
        order = torch.sort(raw, dim=1, descending=True, stable=True).indices[:, :c["top"]]
        res["top_ids"] = torch.where(used[:, None], order, -1).to(torch.int32)
        res["top_logprobs"] = torch.where(used[:, None], logp.gather(1, order), zero)
    if c["backward"]:
        dl, de = (torch.where(used, s[k], zero)[:, None] for k in ("dlogprob", "dentropy"))
        d = p * (-dl - de * (torch.where(p > 0, logp, zero) + entropy[:, None]))
        d.scatter_add_(1, at, dl)
        dlogits = torch.zeros((R, c["pitch"]), dtype=t, device="cuda")
        dlogits[:, :V] = d * c["scale"]
        res["dlogits"] = dlogits
    return res


# ---- the framework's calls --------------------------------------------------------------------------------------------
def _at(x):
    return 0 if x is None else x.data_ptr()


def _rotary_own(s):
    from paper_2403_08837_amd import binding as cdp
    c = s["case"]
    sizes = (c["tokens"], c["heads"], c["kv_heads"], c["width"], c["rotary"])
    given = (_at(s["qkv"]), _at(s["positions"]), _at(s["freqs"]), _at(s["gamma_q"]), _at(s["gamma_k"]))
    cdp.cdp_k_head_norm_rotary(s["code"], *given, _at(s["out"]), EPS, int(c["interleaved"]), *sizes)
    res = {"out": s["out"]}
    if c["backward"]:
        cdp.cdp_k_head_norm_rotary_backward(s["code"], 0, *given, _at(s["dout"]), _at(s["dqkv"]), _at(s["dgamma_q"]), _at(s["dgamma_k"]), EPS, int(c["interleaved"]),
                                            _at(s["ws"]), s["ws"].numel(), *sizes)
        if c["norm"]:
            res.update(dgamma_q=s["dgamma_q"], dgamma_k=s["dgamma_k"])
        res["dqkv"] = s["dqkv"]
    return res


def _gated_own(s):
    from paper_2403_08837_amd import binding as cdp
    c = s["case"]
    sizes = (_at(s["ws"]), s["ws"].numel(), c["rows"], c["inputs"], c["hidden"])
    cdp.cdp_k_gated_linear(s["code"], ACTS[c["act"]], _at(s["x"]), _at(s["wg"]), _at(s["wu"]), _at(s["h"]), _at(s["g"]), _at(s["u"]), *sizes)
    res = {"h": s["h"]}
    if c["backward"]:
        cdp.cdp_k_gated_linear_backward(s["code"], ACTS[c["act"]], _at(s["x"]), _at(s["wg"]), _at(s["wu"]), _at(s["g"]), _at(s["u"]), _at(s["dh"]), _at(s["dx"]),
                                        _at(s["dwg"]), _at(s["dwu"]), *sizes)
        res.update(g=s["g"], u=s["u"], dx=s["dx"], dwg=s["dwg"], dwu=s["dwu"])
    return res


def _linear_own(s):
    from paper_2403_08837_amd import binding as cdp
    c = s["case"]
    sizes = (_at(s["ws"]), s["ws"].numel(), c["rows"], c["inputs"], c["outputs"])
    cdp.cdp_k_linear(s["code"], ACTS[c["act"]], _at(s["x"]), _at(s["w"]), _at(s["bias"]), _at(s["residual"]), _at(s["y"]), _at(s["z"]), *sizes)
    res = {"y": s["y"]}
    if c["backward"]:
        cdp.cdp_k_linear_backward(s["code"], ACTS[c["act"]], _at(s["x"]), _at(s["w"]), _at(s["z"]), _at(s["dy"]), _at(s["dx"]), _at(s["dw"]), _at(s["dbias"]), *sizes)
        if c["act"] != "none":
            res["z"] = s["z"]
        res.update(dx=s["dx"], dw=s["dw"])
        if c["bias"]:
            res["dbias"] = s["dbias"]
    return res


def _logprob_own(s):
    from paper_2403_08837_amd import binding as cdp
    c = s["case"]
    given = (s["code"], _at(s["logits"]), c["pitch"], _at(s["targets"]), c["scale"])
    cdp.cdp_k_token_logprob(*given, _at(s["logprob"]), _at(s["entropy"]), _at(s["lse"]), _at(s.get("top_ids")), _at(s.get("top_logprobs")), c["top"], _at(s["ws"]),
                            s["ws"].numel(), c["rows"], c["vocab"])
    res = {k: s[k] for k in ("logprob", "entropy", "lse")}
    if c["top"]:
        res.update(top_ids=s["top_ids"], top_logprobs=s["top_logprobs"])
    if c["backward"]:
        cdp.cdp_k_token_logprob_backward(*given, _at(s["lse"]), _at(s["entropy"]), _at(s["dlogprob"]), _at(s["dentropy"]), _at(s["dlogits"]), c["rows"], c["vocab"])
        res["dlogits"] = s["dlogits"]
    return res


# ---- what a pass cannot do without ------------------------------------------------------------------------------------
def work(case):
    e = DTYPES[case["dtype"]][2]
    if case["kind"] == "rotary":
        T, H, K, W = case["tokens"], case["heads"], case["kv_heads"], case["width"]
        n, v = T * (H + K) * W, T * K * W
        return {"bytes": e * (2 * n + 2 * v) + 4 * T + (e * ((3 if case["norm"] else 2) * n + 2 * v) if case["backward"] else 0), "flops": n * (10 + (25 if case["backward"] else 0))}
    if case["kind"] == "gated":
        R, I, H = case["rows"], case["inputs"], case["hidden"]
        b = e * (R * I + 2 * H * I + R * H)
        if case["backward"]:
            b += e * (2 * R * H + 2 * R * I + 4 * H * I + 3 * R * H)
        return {"bytes": b, "flops": (12 if case["backward"] else 4) * R * I * H}
    if case["kind"] == "linear":
        R, I, O = case["rows"], case["inputs"], case["outputs"]
        z = int(case["act"] != "none")
        b = e * (R * I + O * I + R * O * (1 + int(case["residual"])))
        if case["backward"]:
            b += e * (2 * R * I + 2 * O * I + R * O * (1 + 2 * z))
        return {"bytes": b, "flops": (6 if case["backward"] else 2) * R * I * O}
    R, V = case["rows"], case["vocab"]
    used = round(R * (1 - case["padding"]))
    return {"bytes": e * used * V + 16 * R + 8 * R * case["top"] + (e * (used + R) * V if case["backward"] else 0), "flops": used * V * (6 + (8 if case["backward"] else 0))}


# ---- the definitions in 64 bits ---------------------------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    return {"rotary": _rotary_exact, "gated": _gated_exact, "linear": _linear_exact, "logprob": _logprob_exact}[case["kind"]](s)


def _rotary_exact(s):
    """A pair is a complex number, its rotation a product; gradients by the chain rule."""
    c = s["case"]
    T, H, K, W, R = c["tokens"], c["heads"], c["kv_heads"], c["width"], c["rotary"]
    angle = s["positions"].double()[:, None] * s["freqs"].double()[None, :]
    turn = torch.polar(torch.ones_like(angle), angle)[:, None, :]
    qkv = s["qkv"].double().requires_grad_(c["backward"])
    leaves = [s[k].double().requires_grad_(c["backward"]) if c["norm"] else None for k in ("gamma_q", "gamma_k")]
    q, k, v = (a.reshape(T, -1, W) for a in qkv.split([H * W, K * W, K * W], 1))
    parts = []
    for a, gamma in zip((q, k), leaves):
        if gamma is not None:
            a = a / torch.sqrt((a * a).sum(2, keepdim=True) / W + EPS) * gamma
        pairs = a[:, :, :R].reshape(T, -1, R // 2, 2) if c["interleaved"] else a[:, :, :R].reshape(T, -1, 2, R // 2).transpose(2, 3)
        pairs = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turn)
        if not c["interleaved"]:
            pairs = pairs.transpose(2, 3)
        parts += [torch.cat([pairs.reshape(T, -1, R), a[:, :, R:]], 2).reshape(T, -1)]
    out = torch.cat(parts + [v.reshape(T, -1)], 1)
    res = {"out": out.detach()}
    if c["backward"]:
        out.backward(s["dout"].double())
        if c["norm"]:
            res.update(dgamma_q=leaves[0].grad, dgamma_k=leaves[1].grad)
        res["dqkv"] = qkv.grad
    return res


def _gated_exact(s):
    c = s["case"]
    x, wg, wu = (s[k].double().requires_grad_(c["backward"]) for k in ("x", "wg", "wu"))
    g, u = x @ wg.t(), x @ wu.t()
    act = {"silu": torch.nn.functional.silu, "gelu": torch.nn.functional.gelu, "sigmoid": torch.sigmoid}[c["act"]]
    h = act(g) * u
    res = {"h": h.detach()}
    if c["backward"]:
        h.backward(s["dh"].double())
        res.update(g=g.detach(), u=u.detach(), dx=x.grad, dwg=wg.grad, dwu=wu.grad)
    return res


def _linear_exact(s):
    c = s["case"]
    x, w = (s[k].double().requires_grad_(c["backward"]) for k in ("x", "w"))
    bias = s["bias"].double().requires_grad_(c["backward"]) if c["bias"] else None
    z = torch.nn.functional.linear(x, w, bias)
    act = {"silu": torch.nn.functional.silu, "gelu": torch.nn.functional.gelu, "none": lambda v: v}[c["act"]]
    y = act(z)
    res = {"y": (y + s["residual"].double() if c["residual"] else y).detach()}
    if c["backward"]:
        y.backward(s["dy"].double())
        if c["act"] != "none":
            res["z"] = z.detach()
        res.update(dx=x.grad, dw=w.grad)
        if c["bias"]:
            res["dbias"] = bias.grad
    return res


def _logprob_exact(s):
    """Row blocks one after the other, gradients by the chain rule."""
    c = s["case"]
    R, V = c["rows"], c["vocab"]
    parts = []
    for rows in torch.arange(R, device="cuda").split(max(1, 100_000_000 // V)):
        logits = s["logits"][rows].double()
        z = (logits[:, :V] * c["scale"]).requires_grad_(c["backward"])
        target = s["targets"][rows].long()
        learnt = target >= 0
        lse = torch.logsumexp(z, 1)
        p = torch.softmax(z, 1)
        entropy = lse - torch.where(p > 0, p * z.clamp(min=-1e300), 0.0).sum(1)
        logprob = z[torch.arange(len(rows), device="cuda"), target.clamp(min=0)] - lse
        res = {k: torch.where(learnt, v, 0.0).detach() for k, v in (("logprob", logprob), ("entropy", entropy), ("lse", lse))}
        if c["top"]:
            best = torch.sort(z.detach(), 1, descending=True).values[:, :c["top"]] - lse.detach()[:, None]
            res["top_ids"], res["top_logprobs"] = None, torch.where(learnt[:, None], best, 0.0)
        if c["backward"]:
            (torch.where(learnt, s["dlogprob"][rows].double() * logprob, 0.0).sum() + torch.where(learnt, s["dentropy"][rows].double() * entropy, 0.0).sum()).backward()
            d = torch.zeros_like(logits)
            d[:, :V] = z.grad * c["scale"]
            res["dlogits"] = d
        parts.append(res)
    return {k: torch.cat([q[k] for q in parts]) if parts[0][k] is not None else None for k in parts[0]}
