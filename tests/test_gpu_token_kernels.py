"""Operators of token models (embedding, norms around a block, packed causal attention, gradient clipping) against their formulas in 64 bits.

Tolerances count roundings: u = 2^-24 is half a step of fp32, `half(t)` that of the element type (bf16 2^-8 relative to the value, fp32 2^-24).  A
value that is a sum of terms is off by at most (roundings on the longest way from an input to it) * u * (sum of the terms' sizes), plus
half a step of its own type.  The references compute those sizes beside the values."""
import math

import numpy as np
import pytest

from paper_2403_08837_amd import binding as b

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

U = 2.0 ** -24
F32, BF16 = 0, 1
TYPES = {F32: torch.float32, BF16: torch.bfloat16}
GUARD = 7  # elements (of the type's own size) or rows past an output that have to stay as they are


def half(dtype):
    return 2.0 ** -8 if dtype == BF16 else U


def randn(seed, *shape, scale=1.0):
    g = torch.Generator()
    g.manual_seed(seed)
    return scale * torch.randn(shape, generator=g, dtype=torch.float64)


class Held:
    """Device tensors with `shift` elements before them and GUARD behind, which `check` finds untouched."""

    def __init__(self):
        self.all = []

    def __call__(self, value, t, shift=0):
        value = value.to(t)
        whole = torch.full((shift + value.numel() + GUARD,), 7.0, dtype=t, device="cuda")
        whole[shift:shift + value.numel()] = value.reshape(-1).cuda()
        self.all.append((whole, shift, value.numel()))
        return whole[shift:shift + value.numel()].view(value.shape)

    def out(self, t, *shape, shift=0):
        return self(torch.full(shape, float("nan")), t, shift)

    def check(self):
        torch.cuda.synchronize()
        for whole, shift, n in self.all:
            assert bool((whole[:shift] == 7).all()) and bool((whole[shift + n:] == 7).all())


def p(x):
    return 0 if x is None else x.data_ptr()


def workspace(n):
    return torch.full((n // 4 + 1,), float("nan"), device="cuda")


def near(got, want, tol, what):
    got, tol = got.detach().cpu().double(), torch.as_tensor(tol, dtype=torch.float64)
    assert got.shape == want.shape
    if not got.numel():
        return
    fine = (got - want).abs() <= tol
    fine |= torch.isnan(got) & torch.isnan(want) | (got == want)
    worst = ((got - want).abs() / tol.clamp(min=1e-300)).flatten().argmax()
    assert bool(fine.all()), (what, int((~fine).sum()), got.numel(), got.flatten()[worst].item(), want.flatten()[worst].item(), tol.expand(got.shape).flatten()[worst].item())


# ---- embedding --------------------------------------------------------------------------------------------------------
def ids_of(kind, rows, vocab, seed):
    g = np.random.default_rng(seed)
    if kind == "one":
        return np.full(rows, vocab - 1, dtype=np.int32)
    if kind == "outside":
        return g.choice(np.array([-1, vocab, -2 ** 31, 2 ** 31 - 1]), rows).astype(np.int32)
    ids = g.integers(0, vocab, rows) if kind == "even" else np.minimum((vocab + 1) ** g.random(rows) - 1, vocab - 1).astype(np.int64)
    if kind == "padded":
        ids = np.where(g.random(rows) < 0.3, g.choice(np.array([-1, vocab, vocab + 1, -7]), rows), ids)
    return ids.astype(np.int32)


EMBEDDINGS = [("even", 1, 1, 1), ("even", 1, 5, 8), ("words", 31, 7, 3), ("words", 33, 40, 64), ("padded", 200, 50, 20), ("one", 1000, 3, 24), ("outside", 65, 9, 16),
              ("even", 64, 4000, 257), ("words", 2048, 300, 8), ("words", 2049, 70000, 12), ("padded", 5000, 1000, 33), ("one", 4097, 2, 5), ("even", 300, 20, 1032),
              ("words", 40000, 128000, 4), ("words", 9000, 2000, 128)]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("kind,rows,vocab,C", EMBEDDINGS)
@pytest.mark.parametrize("shift", [0, 1])
def test_embedding(dtype, kind, rows, vocab, C, shift):
    """Lookup and both forms of the gradient; `shift`: tensors that begin one element past a 16-byte border.  Forward: one product.  Backward: a
    row's n terms in any order, one product, one addition: (n + 2) roundings."""
    t, scale, hold = TYPES[dtype], 1.7, Held()
    ids = torch.from_numpy(ids_of(kind, rows, vocab, rows + C))
    table, dout, base = randn(1, vocab, C).to(t), randn(2, rows, C).to(t), randn(3, vocab, C).float()
    inside = (ids >= 0) & (ids < vocab)
    at = torch.where(inside, ids, 0).long()
    scale32 = float(np.float32(scale))
    tab, ids_d, dout_d = hold(table, t, shift), hold(ids, torch.int32, shift), hold(dout, t, shift)
    out, dt, acc = hold.out(t, rows, C, shift=shift), hold.out(torch.float32, vocab, C, shift=shift), hold(base, torch.float32, shift)
    need = 16 * rows + 8 * C * -(-rows // 32) + 512
    ws = workspace(need)
    b.cdp_k_embedding(dtype, 0, p(tab), p(ids_d), 0, p(out), scale, 0, 0, rows, vocab, C)
    b.cdp_k_embedding(dtype, 1, 0, p(ids_d), p(dout_d), p(dt), scale, p(ws), need, rows, vocab, C)
    b.cdp_k_embedding(dtype, 2, 0, p(ids_d), p(dout_d), p(acc), scale, p(ws), need, rows, vocab, C)
    want = scale32 * table[at].double() * inside[:, None]
    near(out, want, (half(dtype) + 2 * U) * want.abs(), "out")
    d = dout.double() * scale32 * inside[:, None]
    grad = torch.zeros((vocab, C), dtype=torch.float64).index_add_(0, at, d)
    size = torch.zeros((vocab, C), dtype=torch.float64).index_add_(0, at, d.abs())
    n = torch.zeros(vocab, dtype=torch.float64).index_add_(0, at, inside.double())[:, None]
    near(dt, grad, (n + 2) * U * size, "dtable")
    near(acc, grad + base, (n + 3) * U * (size + base.abs() * (n > 0)), "dtable, added to")
    assert torch.equal(acc[n[:, 0].cuda() == 0].cpu(), base[n[:, 0] == 0])
    hold.check()


@pytest.mark.parametrize("rows", [700, 6000])
def test_embedding_gradient_is_the_same_every_time(rows):
    ids = torch.from_numpy(ids_of("padded", rows, 90, 4)).cuda()
    dout = randn(5, rows, 96).float().cuda()
    need = 16 * rows + 8 * 96 * -(-rows // 32) + 512
    got = []
    for _ in range(3):
        got.append(torch.full((90, 96), float("nan"), device="cuda"))
        b.cdp_k_embedding(F32, 1, 0, p(ids), p(dout), p(got[-1]), 0.3, p(workspace(need)), need, rows, 90, 96)
        torch.cuda.synchronize()
    assert all(torch.equal(g, got[0]) for g in got[1:])


def test_embedding_of_what_is_not_finite():
    """Rows of other tokens do not see it; padding is zero, not zero times it."""
    ids = torch.tensor([0, 2, -1, 1], dtype=torch.int32, device="cuda")
    table = torch.tensor([[1.0, 2.0], [float("inf"), -3.0], [float("nan"), 4.0]], device="cuda")
    dout = torch.tensor([[1.0, 1.0], [float("nan"), 1.0], [float("inf"), float("nan")], [float("inf"), 2.0]], device="cuda")
    out, dt, ws = torch.empty(4, 2, device="cuda"), torch.empty(3, 2, device="cuda"), workspace(1024)
    b.cdp_k_embedding(F32, 0, p(table), p(ids), 0, p(out), 1.0, 0, 0, 4, 3, 2)
    b.cdp_k_embedding(F32, 1, 0, p(ids), p(dout), p(dt), 1.0, p(ws), 1024, 4, 3, 2)
    assert np.array_equal(out.cpu().numpy(), [[1, 2], [np.nan, 4], [0, 0], [np.inf, -3]], equal_nan=True)
    assert np.array_equal(dt.cpu().numpy(), [[1, 1], [np.inf, 2], [np.nan, 1]], equal_nan=True)


def test_embedding_table_past_2_to_the_31():
    """Offsets in 64 bits: the last rows of a table of 2^31 elements and more."""
    V, C, rows = (1 << 22) + 3, 520, 5
    table = torch.zeros((V, C), dtype=torch.bfloat16, device="cuda")
    ids = torch.tensor([V - 1, 0, V - 2, V - 1, V], dtype=torch.int32, device="cuda")
    table[V - 1], table[V - 2] = 3.0, 5.0
    out, dout = torch.empty((rows, C), dtype=torch.bfloat16, device="cuda"), torch.ones((rows, C), dtype=torch.bfloat16, device="cuda")
    b.cdp_k_embedding(BF16, 0, p(table), p(ids), 0, p(out), 2.0, 0, 0, rows, V, C)
    assert out[:, 0].tolist() == [6, 0, 10, 6, 0] and torch.equal(out, out[:, :1].expand(rows, C))
    need = 16 * rows + 8 * C + 512
    grad = torch.full((V, C), 9.0, device="cuda")
    b.cdp_k_embedding(BF16, 1, 0, p(ids), p(dout), p(grad), 2.0, p(workspace(need)), need, rows, V, C)
    sums = grad.sum(1)
    assert sums[V - 1].item() == 4 * C and sums[V - 2].item() == 2 * C and sums[0].item() == 2 * C and int((sums != 0).sum()) == 3


# ---- norms around a block ---------------------------------------------------------------------------------------------
def norm_reference(x, h, gate, post, pre, dr, dy, scale, eps):
    """Values and sizes of the terms."""
    res, size = {}, {}
    if h is not None:
        eta = (h.square().mean(1, keepdim=True) + eps).rsqrt() if post is not None else torch.ones_like(h[:, :1])
        n = h * eta
        u = n * post if post is not None else h
        sig = torch.sigmoid(gate) if gate is not None else torch.ones_like(h)
        term = scale * sig * u
        r = x + term
        size["r"] = x.abs() + term.abs()
    else:
        r, size["r"] = x, 0 * x
    res["r"] = r
    if pre is not None:
        rho = (r.square().mean(1, keepdim=True) + eps).rsqrt()
        res["y"] = r * rho * pre
        # r's error moves every y of the row through rho, and its own
        size["y"] = (size["r"] + r.abs() * (1 + size["r"].norm(dim=1, keepdim=True) / r.norm(dim=1, keepdim=True).clamp(min=1e-30))) * rho * pre.abs()
    d, d_size = torch.zeros_like(r), torch.zeros_like(r)
    if dr is not None:
        d, d_size = d + dr, d_size + dr.abs()
    if pre is not None:
        rhat, a = r * rho, dy * pre
        # the size of a value of rhat: r's own terms, and what the whole row's do to rho
        rhat_size = size["y"] / pre.abs().clamp(min=1e-30)
        d = d + rho * (a - rhat * (a * rhat).mean(1, keepdim=True))
        d_size = d_size + rho * (a.abs() * (1 + size["r"].norm(dim=1, keepdim=True) / r.norm(dim=1, keepdim=True).clamp(min=1e-30)) + 2 * rhat_size * (a.abs() * rhat_size).mean(1, keepdim=True))
        res["dpre"], size["dpre"] = (dy * rhat).sum(0), (dy.abs() * rhat_size).sum(0)
    res["dx"], size["dx"] = d, d_size
    if h is not None:
        du, du_size = scale * sig * d, scale * sig * d_size
        if gate is not None:
            res["dgate"], size["dgate"] = scale * u * d * sig * (1 - sig), scale * u.abs() * d_size * sig
        if post is not None:
            c, c_size = du * post, du_size * post.abs()
            res["dh"] = eta * (c - n * (c * n).mean(1, keepdim=True))
            size["dh"] = eta * (c_size + n.abs() * (c_size * n.abs()).mean(1, keepdim=True))
            res["dpost"], size["dpost"] = (du * n).sum(0), (du_size * n.abs()).sum(0)
        else:
            res["dh"], size["dh"] = du, du_size
    return res, size


def norm_tolerance(name, res, size, dtype, rows):
    """What `size` holds is the sum of the terms' sizes.  A sum over a row is at most 16 values in a lane, then a tree of at most 10 levels: 27 roundings with the squares; eta and rho are roots of such
    sums (half their relative error), with an error of the reciprocal root of 2 units and one product with 1/C; sigmoid costs 6 units.  r: 14 + 3 +
    6 + 4 < 32.  y: twice that and its own 20: < 96.  The gradients chain two norms and their means, each mean another 27: < 160.  Column sums: rows
    of a workgroup one after the other, then its share with the others', at most rows + 16 more."""
    k = {"r": 32, "y": 96}.get(name, 160) + (rows + 16 if name in ("dpre", "dpost") else 0)
    own = half(dtype) if name not in ("dpre", "dpost") else U
    return k * U * size[name] + own * res[name].abs() * (1 + 1e-3)


NORMS = [(1, 1), (3, 7), (5, 64), (64, 64), (33, 250), (7, 768), (40, 1000), (9, 1024), (6, 1025), (5, 2048), (3, 2056), (600, 96), (4, 4096), (3, 5003), (2, 8192),
         (2, 11111), (3, 16384), (1030, 520)]
FORMS = ["all", "no post", "no gate", "h alone", "norm alone", "end", "no dr"]


def norm_case(form, rows, C, t, seed=0):
    v = {k: randn(seed + i, rows, C).to(t) for i, k in enumerate(("x", "gate", "dr", "dy"))}
    v["h"] = randn(seed + 9, rows, C, scale=3.0).to(t)
    v["post"], v["pre"] = ((1 + randn(seed + i, C, scale=0.2)).float() for i in (20, 30))
    if form in ("no post", "h alone", "norm alone"):
        v["post"] = None
    if form in ("no gate", "h alone", "norm alone"):
        v["gate"] = None
    if form == "norm alone":
        v["h"] = None
    if form == "end":
        v["pre"] = v["dy"] = None
    if form == "no dr":
        v["dr"] = None
    return v


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,C", NORMS)
@pytest.mark.parametrize("form", FORMS)
def test_residual_norm(dtype, rows, C, form):
    """Forward and both forms of the backward; even numbers of rows also on tensors that begin one element past a 16-byte border."""
    t, hold, scale, eps, shift = TYPES[dtype], Held(), 0.75, 1e-5, 1 - rows % 2
    v = norm_case(form, rows, C, t, C)
    dbl = lambda x: None if x is None else x.double()  # noqa: E731
    dev = {k: None if x is None else hold(x, x.dtype, shift) for k, x in v.items()}
    r = hold.out(t, rows, C, shift=shift)
    y = hold.out(t, rows, C, shift=shift) if v["pre"] is not None else None
    b.cdp_k_residual_norm(dtype, p(dev["x"]), p(dev["h"]), p(dev["gate"]), p(dev["post"]), p(dev["pre"]), p(r), p(y), scale, eps, rows, C)
    got = {"r": r, "y": y, "dx": hold.out(t, rows, C, shift=shift)}
    got["dh"] = hold.out(t, rows, C, shift=shift) if v["h"] is not None else None
    got["dgate"] = hold.out(t, rows, C, shift=shift) if v["gate"] is not None else None
    base = {k: randn(77, C).float() for k in ("post", "pre")}
    grads = [{k: hold(base[k], torch.float32, shift) if v[k] is not None else None for k in base} for _ in range(2)]
    need = 8 * C * min(rows, 512) + 256
    ws = workspace(need)
    for accumulate in (0, 1):
        b.cdp_k_residual_norm_backward(dtype, accumulate, p(dev["x"]) if v["pre"] is not None else 0, p(dev["h"]), p(dev["gate"]), p(dev["post"]), p(dev["pre"]), p(dev["dr"]),
                                       p(dev["dy"]), p(got["dx"]), p(got["dh"]), p(got["dgate"]), p(grads[accumulate]["post"]), p(grads[accumulate]["pre"]), scale, eps,
                                       p(ws), need, rows, C)
    args = [dbl(v[k]) for k in ("x", "h", "gate", "post", "pre", "dr", "dy")]
    eps = float(np.float32(eps))
    res, size = norm_reference(*args, scale, eps)
    for k in got:
        if got[k] is not None:
            near(got[k], res[k], norm_tolerance(k, res, size, dtype, rows), k)
    for k in base:
        if v[k] is not None:
            name = "d" + k
            tol = norm_tolerance(name, res, size, dtype, rows)
            near(grads[0][k], res[name], tol, name)
            near(grads[1][k], res[name] + base[k], tol + 2 * U * (base[k].abs() + res[name].abs()), name + ", added to")
    hold.check()


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_residual_norm_in_place_without_r_and_of_zeros(dtype):
    """r over x and dx over dr give the same bits; y without r; rows of zeros have finite norms and gradients."""
    t, rows, C = TYPES[dtype], 37, 776
    v = {k: None if x is None else x.cuda() for k, x in norm_case("all", rows, C, t, 5).items()}
    v["x"][3] = 0
    v["h"][3] = 0
    r, y, y2 = (torch.empty((rows, C), dtype=t, device="cuda") for _ in range(3))
    fwd = lambda x, r, y: b.cdp_k_residual_norm(dtype, p(x), p(v["h"]), p(v["gate"]), p(v["post"]), p(v["pre"]), p(r), p(y), 0.5, 1e-6, rows, C)  # noqa: E731
    fwd(v["x"], r, y)
    fwd(v["x"], None, y2)
    assert torch.equal(y, y2) and not y[3].any() and not r[3].any()
    x = v["x"].clone()
    fwd(x, x, y2)
    assert torch.equal(x, r) and torch.equal(y, y2)
    need = 8 * C * rows + 256
    results = []
    for inplace in (False, True):
        dr = v["dr"].clone()
        outs = [dr if inplace else torch.empty_like(dr), torch.empty_like(dr), torch.empty_like(dr), torch.empty(C, device="cuda"), torch.empty(C, device="cuda")]
        b.cdp_k_residual_norm_backward(dtype, 0, p(v["x"]), p(v["h"]), p(v["gate"]), p(v["post"]), p(v["pre"]), p(dr), p(v["dy"]), *[p(o) for o in outs[:3]], p(outs[3]),
                                       p(outs[4]), 0.5, 1e-6, p(workspace(need)), need, rows, C)
        results.append(outs)
    for one, two in zip(*results):
        assert torch.isfinite(one.float()).all() and torch.equal(one, two)


def test_residual_norm_of_extreme_gates():
    """sigmoid of far values is 0 or 1 and its derivative 0: no NaN."""
    gate = torch.tensor([[-1e30, -200.0, -88.0, 0.0, 88.0, 200.0, 1e30, -float("inf")]], device="cuda")
    x, h = torch.ones_like(gate), 2 * torch.ones_like(gate)
    r, dx, dh, dg = (torch.empty_like(gate) for _ in range(4))
    b.cdp_k_residual_norm(F32, p(x), p(h), p(gate), 0, 0, p(r), 0, 1.0, 1e-6, 1, 8)
    b.cdp_k_residual_norm_backward(F32, 0, 0, p(h), p(gate), 0, 0, p(x), 0, p(dx), p(dh), p(dg), 0, 0, 1.0, 1e-6, 0, 0, 1, 8)
    sig = torch.sigmoid(gate.double())
    near(r, (1 + 2 * sig).cpu(), 16 * U * 3, "r")
    near(dh, sig.cpu(), 16 * U, "dh")
    near(dg, (2 * sig * (1 - sig)).cpu(), 16 * U * 2, "dgate")


# ---- packed causal attention --------------------------------------------------------------------------------------------
def attention_reference(qkv, at, heads, kv_heads, width, scale, dtype, dout=None, out_given=None, lse_given=None):
    """Outputs and their tolerances, head by head and sequence by sequence.  Backward: from the given out and lse, as documented.

    Scores: a score's error, relative to 1 as an exponent, is e_s = scale * (width + 4) u sum |q| |k| plus 4 units of the exponent's own arithmetic (its
    size in units: 2 u |x|).  out: that error on every term twice (numerator, denominator), the type's rounding of a probability (bf16: half a step), sums of n
    terms and at most n rescalings.  What fp32 cannot hold is lost: a probability below 2^-126, which reaches a result through at most 2^12 terms of factors below 2^20 in
    all, so 2^-94.  lse: the largest e_s, the sum's rounding, its own."""
    T, g, ht = qkv.shape[0], heads // kv_heads, half(dtype)
    rounded = ht if dtype == BF16 else 0.0   # what is held in the element type between two products
    x = qkv.reshape(T, heads + 2 * kv_heads, width)
    res = {"out": torch.zeros(T, heads, width, dtype=torch.float64), "lse": torch.zeros(heads, T, dtype=torch.float64), "dqkv": torch.zeros_like(x)}
    tol = {k: torch.zeros_like(v) for k, v in res.items()}
    used = torch.zeros(T, dtype=torch.bool)
    for s0, s1 in zip(at, at[1:]):
        n = s1 - s0
        if not n:
            continue
        used[s0:s1] = True
        rows = slice(s0, s1)
        later = torch.ones(n, n, dtype=torch.bool).triu(1)
        for h in range(heads):
            k, v = x[rows, heads + h // g], x[rows, heads + kv_heads + h // g]
            q = x[rows, h]
            s = scale * (q @ k.T)
            e = abs(scale) * (width + 4) * U * (q.abs() @ k.abs().T) + 4 * U * (1 + s.abs())
            s, e = s.masked_fill(later, -math.inf), e.masked_fill(later, 0.0)
            lse = torch.logsumexp(s, 1)
            e_max = e.max(1, keepdim=True).values
            if dout is None:
                P = torch.exp(s - lse[:, None])
                res["out"][rows, h], res["lse"][h, rows] = P @ v, lse
                size = P @ v.abs()
                tol["out"][rows, h] = (rounded + 2 * e_max + (2 * n + 16) * U) * size + ht * (P @ v).abs()
                tol["lse"][h, rows] = e_max[:, 0] + (n + 8) * U + 4 * U * (lse.abs() + s.masked_fill(later, 0).abs().max(1).values)
                continue
            P = torch.exp(s - lse_given[h, rows, None])
            e_p = e + 4 * U * (1 + lse_given[h, rows, None].abs()) + 8 * U
            do, o = dout[rows, h * width:(h + 1) * width], out_given[rows, h * width:(h + 1) * width]
            dp, delta = do @ v.T, (do * o).sum(1, keepdim=True)
            e_dp = (width + 4) * U * (do.abs() @ v.abs().T + (do * o).abs().sum(1, keepdim=True))
            ds = P * (dp - delta)
            e_ds = P * (e_dp + (e_p + 4 * U) * (dp - delta).abs()) + rounded * ds.abs()
            q_, k_, v_ = h, heads + h // g, heads + kv_heads + h // g
            sums = (n * g + 16) * U
            res["dqkv"][rows, q_] = scale * ds @ k
            tol["dqkv"][rows, q_] = abs(scale) * (e_ds + sums * ds.abs()) @ k.abs()
            res["dqkv"][rows, k_] += scale * ds.T @ q
            tol["dqkv"][rows, k_] += abs(scale) * (e_ds + sums * ds.abs()).T @ q.abs()
            res["dqkv"][rows, v_] += P.T @ do
            tol["dqkv"][rows, v_] += (P * (e_p + rounded + sums)).T @ do.abs()
    tol["dqkv"] += ht * res["dqkv"].abs() + 2.0 ** -94
    tol["out"] += 2.0 ** -94
    for k in ("out", "dqkv"):
        res[k], tol[k] = res[k].reshape(T, -1), tol[k].reshape(T, -1)
    return res, tol, used


ATTENTION = [  # lengths (before them and behind them rows of no sequence), heads, key heads, width
    (0, [1], 0, 1, 1, 8), (0, [2], 0, 2, 1, 16), (0, [31], 1, 1, 1, 64), (0, [32], 0, 2, 2, 32), (0, [33], 0, 4, 2, 40), (0, [64], 3, 3, 3, 64), (0, [65], 0, 2, 1, 128),
    (0, [127, 1], 0, 2, 2, 24), (0, [128, 128], 0, 4, 1, 64), (0, [129], 0, 2, 2, 96), (2, [1, 0, 0, 5, 1, 130], 7, 6, 2, 64), (0, [0, 0], 4, 2, 2, 16), (0, [257], 0, 3, 1, 128),
    (5, [300, 17, 1, 1, 64], 9, 8, 2, 64), (0, [515], 0, 2, 2, 80), (0, [700], 0, 4, 1, 128), (0, [1] * 70, 3, 2, 1, 64), (0, [3, 0, 40] * 25, 0, 5, 1, 56),
    (0, [1000, 24], 0, 1, 1, 104), (0, [200, 333], 11, 12, 4, 112), (1, [640, 383], 0, 8, 1, 32), (0, [1300], 0, 1, 1, 64)]


def attention_call(dtype, qkv, at, heads, kv_heads, width, scale, dout, parts, stream=0, hold=None):
    t, T = qkv.dtype, qkv.shape[0]
    hold = hold or Held()
    q = hold(qkv, t)
    offsets = hold(torch.tensor(at, dtype=torch.int32), torch.int32, 1)
    out, lse, dqkv = hold.out(t, T, heads * width), hold.out(torch.float32, heads, T), hold.out(t, *qkv.shape)
    need = 4 * heads * T + 512 + parts * 8 * kv_heads * T * width
    ws, sizes = workspace(need), (T, len(at) - 1, heads, kv_heads, width, scale)
    b.cdp_k_attention_packed(dtype, 0, p(q), p(offsets), p(out), p(lse), 0, 0, 0, 0, *sizes, stream)
    if dout is not None:
        b.cdp_k_attention_packed(dtype, 1, p(q), p(offsets), p(out), p(lse), p(hold(dout, t)), p(dqkv), p(ws), need, *sizes, stream)
    hold.check()
    return out, lse, dqkv


def attention_case(before, lengths, behind, heads, kv_heads, width, t, seed=0, size=1.0):
    at = [before]
    for n in lengths:
        at.append(at[-1] + n)
    T = at[-1] + behind
    qkv = randn(seed, T, (heads + 2 * kv_heads) * width, scale=size).to(t)
    return at, qkv, randn(seed + 1, T, heads * width).to(t)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("before,lengths,behind,heads,kv_heads,width", ATTENTION, ids=lambda v: str(v) if not isinstance(v, list) or len(v) < 7 else "many")
@pytest.mark.parametrize("parts", [0, 8])
def test_packed_attention(dtype, before, lengths, behind, heads, kv_heads, width, parts):
    t, scale = TYPES[dtype], 1.3 * width ** -0.5
    at, qkv, dout = attention_case(before, lengths, behind, heads, kv_heads, width, t, width)
    # what lies outside the sequences is not read for another's sake
    outside = torch.ones(qkv.shape[0], dtype=torch.bool)
    outside[at[0]:at[-1]] = False
    qkv[outside], dout[outside] = float("nan"), float("nan")
    out, lse, dqkv = attention_call(dtype, qkv, at, heads, kv_heads, width, scale, dout, parts)
    scale = float(np.float32(scale))
    clean = lambda v: torch.where(outside[:, None], 0.0, v.double())  # noqa: E731
    res, tol, used = attention_reference(clean(qkv), at, heads, kv_heads, width, scale, dtype)
    near(out[used.cuda()], res["out"][used], tol["out"][used], "out")
    near(lse[:, used.cuda()], res["lse"][:, used], tol["lse"][:, used], "lse")
    assert bool(torch.isnan(out[~used.cuda()]).all()) and bool(torch.isnan(lse[:, ~used.cuda()]).all()) and bool(torch.isnan(dqkv[~used.cuda()]).all())
    res, tol, _ = attention_reference(clean(qkv), at, heads, kv_heads, width, scale, dtype, clean(dout), clean(out.cpu()), torch.where(outside, 0.0, lse.cpu().double()))
    near(dqkv[used.cuda()], res["dqkv"][used], tol["dqkv"][used], "dqkv")


# launches of many workgroups (test_gpu_token_ranges.py has a case for every kernel); 63 and 64 sequences, which are put in order in different ways
CROWDED = [(0, [37] * 62 + [200], 5, 12, 4, 64), (3, [37, 0, 90, 1] * 16, 0, 12, 12, 32), (0, [300, 700, 129, 64, 500], 0, 32, 8, 128), (0, [511, 2, 640], 0, 64, 64, 96),
           (0, [900, 800], 1, 56, 8, 80), (0, [640, 33], 3, 64, 16, 104), (0, [129] * 40, 1, 16, 16, 16), (2, [1500], 0, 72, 24, 48)]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("before,lengths,behind,heads,kv_heads,width", CROWDED, ids=lambda v: str(v) if not isinstance(v, list) or len(v) < 7 else "many")
def test_packed_attention_of_many_workgroups(dtype, before, lengths, behind, heads, kv_heads, width):
    for parts in (0, 8):
        test_packed_attention(dtype, before, lengths, behind, heads, kv_heads, width, parts)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("size", [12.0, 1e-3])
def test_packed_attention_of_large_and_small_scores(dtype, size):
    """Scores of several hundred, whose maximum moves from tile to tile, and scores that are all but equal."""
    at, qkv, dout = attention_case(0, [450, 61], 0, 4, 2, 64, TYPES[dtype], 3, size)
    out, lse, dqkv = attention_call(dtype, qkv, at, 4, 2, 64, 0.125, dout, 0)
    res, tol, _ = attention_reference(qkv.double(), at, 4, 2, 64, 0.125, dtype)
    near(out, res["out"], tol["out"], "out")
    near(lse, res["lse"], tol["lse"], "lse")
    res, tol, _ = attention_reference(qkv.double(), at, 4, 2, 64, 0.125, dtype, dout.double(), out.cpu().double(), lse.cpu().double())
    near(dqkv, res["dqkv"], tol["dqkv"], "dqkv")


@pytest.mark.parametrize("scale", [0.0, -0.2])
def test_packed_attention_of_other_scales(scale):
    """No scale (means of the values) and a negative one."""
    at, qkv, dout = attention_case(0, [100, 3], 0, 2, 1, 32, torch.float32, 4)
    out, lse, dqkv = attention_call(F32, qkv, at, 2, 1, 32, scale, dout, 0)
    scale = float(np.float32(scale))
    res, tol, _ = attention_reference(qkv.double(), at, 2, 1, 32, scale, F32)
    near(out, res["out"], tol["out"], "out")
    near(lse, res["lse"], tol["lse"], "lse")
    res, tol, _ = attention_reference(qkv.double(), at, 2, 1, 32, scale, F32, dout.double(), out.cpu().double(), lse.cpu().double())
    near(dqkv, res["dqkv"], tol["dqkv"], "dqkv")


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_packed_attention_is_the_same_every_time_and_for_a_sequence_alone(dtype):
    """The same bits again; and a sequence's results do not depend on what it is packed with (no parts: nothing is shared)."""
    at, qkv, dout = attention_case(0, [77, 300, 130], 0, 4, 2, 64, TYPES[dtype], 6)
    first = attention_call(dtype, qkv, at, 4, 2, 64, 0.125, dout, 0)
    again = attention_call(dtype, qkv, at, 4, 2, 64, 0.125, dout, 0)
    alone = attention_call(dtype, qkv[77:377].contiguous(), [0, 300], 4, 2, 64, 0.125, dout[77:377].contiguous(), 0)
    for i, (x, y, z) in enumerate(zip(first, again, alone)):
        assert torch.equal(x, y)
        assert torch.equal(x[:, 77:377] if i == 1 else x[77:377], z)


def test_packed_attention_of_broken_offsets_stays_inside():
    """Offsets that descend, are negative or pass the end: whatever comes out, nothing outside the outputs is written (Held.check) and nothing hangs."""
    _, qkv, dout = attention_case(0, [200], 0, 2, 1, 64, torch.bfloat16, 8)
    for at in ([0, 500], [-50, 100, 250], [150, 20, 200], [300, 400], [2 ** 31 - 1, -2 ** 31, 7], [-9, -5]):
        attention_call(BF16, qkv, at, 2, 1, 64, 0.125, dout, 2)


@pytest.mark.parametrize("sequences", [2, 40, 63, 64, 300])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_packed_attention_of_many_broken_offsets_stays_inside(dtype, sequences):
    for heads in (2, 24):
        _, qkv, dout = attention_case(0, [700], 0, heads, 2, 64, TYPES[dtype], 8)
        g = torch.Generator().manual_seed(sequences)
        for low, high in ((-100, 1000), (0, 701), (-2 ** 31, 2 ** 31 - 1)):
            at = torch.randint(low, high, (sequences + 1,), generator=g).tolist()
            attention_call(dtype, qkv, at, heads, 2, 64, 0.125, dout, 2)


def test_packed_attention_gradient_against_differences():
    """fp64 differences of the formula's forward: what the references above call the gradient is one."""
    at, qkv, dout = attention_case(0, [9, 4], 0, 4, 2, 8, torch.float32, 12)
    out, lse, dqkv = attention_call(F32, qkv, at, 4, 2, 8, 0.35, dout, 0)
    scale = float(np.float32(0.35))
    f = lambda x: (attention_reference(x, at, 4, 2, 8, scale, F32)[0]["out"] * dout.double()).sum().item()  # noqa: E731
    x = qkv.double()
    for i in range(0, x.numel(), 5):
        step = torch.zeros(x.numel(), dtype=torch.float64)
        step[i] = 1e-5
        d = (f(x + step.view(x.shape)) - f(x - step.view(x.shape))) / 2e-5
        assert abs(d - dqkv.flatten()[i].item()) <= 2e-5 * max(1.0, abs(d)), (i, d)


# ---- gradient clipping -----------------------------------------------------------------------------------------------
def clip_call(dtype, grads, outs, max_norm, stream=0):
    at = np.array([p(g) if g.numel() else 0 for g in grads], dtype=np.int64)
    out_at = np.array([p(o) if o.numel() else 0 for o in outs], dtype=np.int64) if outs is not None else None
    counts = np.array([g.numel() for g in grads], dtype=np.int64)
    norm, ws = torch.full((1,), -1.0, device="cuda"), workspace(65536)
    b.cdp_k_grad_clip(dtype, len(grads), at.ctypes.data, 0 if outs is None else out_at.ctypes.data, counts.ctypes.data, max_norm, p(norm), p(ws), 65536, stream)
    at[:], counts[:] = 0, 0   # the arrays are read during the call
    return norm


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("counts", [[1], [7], [0, 5, 0], [1000, 3, 64], [100003], [4096] * 130, [1, 70000, 33] * 90, [3_000_001, 12]])
@pytest.mark.parametrize("max_norm", [1.0, 1e9])
def test_grad_clip(dtype, counts, max_norm):
    """The norm: squares summed in 64 bits, rounded once.  The gradients: the factor (two roundings) and the product's, or untouched."""
    t, hold = TYPES[dtype], Held()
    values = [randn(i + len(counts), n, scale=2.0).to(t) for i, n in enumerate(counts)]
    grads = [hold(v, t, i % 3) for i, v in enumerate(values)]
    outs = [hold.out(t, n, shift=(i + len(counts)) % 2) for i, n in enumerate(counts)]
    norm = clip_call(dtype, grads, outs, max_norm)
    want = math.sqrt(sum(float(v.double().square().sum()) for v in values))
    near(norm, torch.tensor([want], dtype=torch.float64), 2 * U * want, "norm")
    factor = max_norm / want if want > max_norm else 1.0
    for v, o in zip(values, outs):
        if factor == 1.0:
            assert torch.equal(o.cpu(), v)
        else:
            near(o, v.double() * factor, (half(dtype) + 4 * U) * (v.double() * factor).abs(), "out")
    hold.check()
    kept = clip_call(dtype, grads, None, max_norm)
    assert torch.equal(kept, norm) and all(torch.equal(g.cpu(), v) for g, v in zip(grads, values))
    clip_call(dtype, grads, grads, max_norm)   # in place
    assert all(torch.equal(g, o) for g, o in zip(grads, outs))
    hold.check()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("counts", [[7] * 160, [1025] * 161, [0] * 100 + [50000] + [0] * 59, [0] * 200 + [5], [16384, 0, 8192, 16385, 8193] * 33, [1024] * 16 + [0] + [2048] * 16 + [3]],
                         ids=lambda c: "%d of %d" % (len(c), sum(c)))
def test_grad_clip_of_whole_tables_and_units(dtype, counts):
    test_grad_clip(dtype, counts, 1.0)


def test_grad_clip_of_what_is_not_finite_or_zero():
    g = torch.tensor([1.0, 2.0, float("nan")], device="cuda")
    assert torch.isnan(clip_call(F32, [g], [g], 0.5)) and torch.equal(g[:2], torch.tensor([1.0, 2.0], device="cuda"))
    g = torch.tensor([1.0, 2.0, float("inf")], device="cuda")
    assert torch.isinf(clip_call(F32, [g], [g], 0.5)) and not g[:2].any() and torch.isnan(g[2])
    g = torch.zeros(9, device="cuda")
    assert clip_call(F32, [g], [g], 0.0).item() == 0 and not g.any()
    g = torch.full((4,), 1e30, device="cuda")   # squares past fp32
    assert abs(clip_call(F32, [g], [g], 2.0).item() / 2e30 - 1) <= 2 * U and bool(((g - 1).abs() <= 4 * U).all())
    g = torch.full((4,), 1e-30, device="cuda")  # and below it
    assert abs(clip_call(F32, [g], [g], 2.0).item() / 2e-30 - 1) <= 2 * U
    g = torch.full((3,), 5.0, device="cuda")
    clip_call(F32, [g], [g], float("inf"))
    assert bool((g == 5).all())


# ---- together, on streams and in graphs --------------------------------------------------------------------------------
class Step:
    """One training step of a one-block token model from the entry points, fp32: embedding, norm, q|k|v map, packed attention, output map, gated
    residual and norm, the squared error to a target as loss; all gradients, clipped together."""
    V, C, H, K, W, EPS = 50, 48, 4, 2, 16, 1e-5

    def __init__(self, lengths, seed):
        self.at = [0]
        for n in lengths:
            self.at.append(self.at[-1] + n)
        T, C, Q = self.at[-1], self.C, (self.H + 2 * self.K) * self.W
        self.T, self.Q, self.A = T, Q, self.H * self.W
        self.ids = torch.from_numpy(ids_of("words", T, self.V, seed))
        self.value = {"table": randn(seed, self.V, C), "g1": 1 + randn(seed + 1, C, scale=0.1), "wqkv": randn(seed + 2, Q, C, scale=0.2), "wo": randn(seed + 3, C, self.A, scale=0.2),
                      "wg": randn(seed + 4, C, C, scale=0.2), "post": 1 + randn(seed + 5, C, scale=0.1), "g2": 1 + randn(seed + 6, C, scale=0.1)}
        self.value = {k: v.float() for k, v in self.value.items()}
        self.target = randn(seed + 7, T, C).float()
        self.w = {k: v.cuda() for k, v in self.value.items()}
        self.ids_d, self.target_d = self.ids.cuda(), self.target.cuda()
        self.offsets = torch.tensor(self.at, dtype=torch.int32, device="cuda")
        f = lambda *n: torch.full(n, float("nan"), device="cuda")  # noqa: E731
        self.buf = dict(x=f(T, C), n1=f(T, C), qkv=f(T, Q), att=f(T, self.A), lse=f(self.H, T), h=f(T, C), gate=f(T, C), r=f(T, C), y=f(T, C), dy=f(T, C), dx=f(T, C), dh=f(T, C),
                        dgate=f(T, C), datt=f(T, self.A), dqkv=f(T, Q), dn1=f(T, C), dn1b=f(T, C), dx0=f(T, C))
        self.grad = {k: f(*v.shape) for k, v in self.value.items()}
        self.clipped = {k: f(*v.shape) for k, v in self.value.items()}
        self.norm = f(1)
        self.ws = {"emb": workspace(16 * T + 8 * C * (T // 32 + 1) + 512), "norm": workspace(8 * C * T + 256), "att": workspace(4 * self.H * T + 512), "clip": workspace(65536)}
        self.lists = [np.array([p(d[k]) for k in self.value], dtype=np.int64) for d in (self.grad, self.clipped)]
        self.lists.append(np.array([v.numel() for v in self.value.values()], dtype=np.int64))

    def run(self, stream=0):
        T, C, Q, A, B, w, g, ws = self.T, self.C, self.Q, self.A, self.buf, self.w, self.grad, self.ws
        gemm = lambda a_k, b_k, x, y, out, M, N, K, lda, ldb: b.cdp_k_gemm(F32, 0, a_k, b_k, p(x), p(y), p(out), M, N, K, lda, ldb, stream)  # noqa: E731
        size = lambda k: ws[k].numel() * 4  # noqa: E731
        b.cdp_k_embedding(F32, 0, p(w["table"]), p(self.ids_d), 0, p(B["x"]), 1.5, 0, 0, T, self.V, C, stream)
        b.cdp_k_residual_norm(F32, p(B["x"]), 0, 0, 0, p(w["g1"]), 0, p(B["n1"]), 1.0, self.EPS, T, C, stream)
        gemm(1, 1, B["n1"], w["wqkv"], B["qkv"], T, Q, C, C, C)
        att = (T, len(self.at) - 1, self.H, self.K, self.W, 0.25, stream)
        b.cdp_k_attention_packed(F32, 0, p(B["qkv"]), p(self.offsets), p(B["att"]), p(B["lse"]), 0, 0, 0, 0, *att)
        gemm(1, 1, B["att"], w["wo"], B["h"], T, C, A, A, A)
        gemm(1, 1, B["n1"], w["wg"], B["gate"], T, C, C, C, C)
        b.cdp_k_residual_norm(F32, p(B["x"]), p(B["h"]), p(B["gate"]), p(w["post"]), p(w["g2"]), p(B["r"]), p(B["y"]), 0.5, self.EPS, T, C, stream)
        torch.sub(B["y"], self.target_d, out=B["dy"])   # the gradient of half the squared error
        b.cdp_k_residual_norm_backward(F32, 0, p(B["x"]), p(B["h"]), p(B["gate"]), p(w["post"]), p(w["g2"]), 0, p(B["dy"]), p(B["dx"]), p(B["dh"]), p(B["dgate"]), p(g["post"]),
                                       p(g["g2"]), 0.5, self.EPS, p(ws["norm"]), size("norm"), T, C, stream)
        gemm(0, 0, B["dh"], B["att"], g["wo"], C, A, T, C, A)
        gemm(0, 0, B["dgate"], B["n1"], g["wg"], C, C, T, C, C)
        gemm(1, 0, B["dh"], w["wo"], B["datt"], T, A, C, C, A)
        b.cdp_k_attention_packed(F32, 1, p(B["qkv"]), p(self.offsets), p(B["att"]), p(B["lse"]), p(B["datt"]), p(B["dqkv"]), p(ws["att"]), size("att"), *att)
        gemm(0, 0, B["dqkv"], B["n1"], g["wqkv"], Q, C, T, Q, C)
        gemm(1, 0, B["dqkv"], w["wqkv"], B["dn1"], T, C, Q, Q, C)
        gemm(1, 0, B["dgate"], w["wg"], B["dn1b"], T, C, C, C, C)
        B["dn1"].add_(B["dn1b"])
        b.cdp_k_residual_norm_backward(F32, 0, p(B["x"]), 0, 0, 0, p(w["g1"]), p(B["dx"]), p(B["dn1"]), p(B["dx0"]), 0, 0, 0, p(g["g1"]), 1.0, self.EPS, p(ws["norm"]),
                                       size("norm"), T, C, stream)
        b.cdp_k_embedding(F32, 1, 0, p(self.ids_d), p(B["dx0"]), p(g["table"]), 1.5, p(ws["emb"]), size("emb"), T, self.V, C, stream)
        b.cdp_k_grad_clip(F32, len(g), *[v.ctypes.data for v in self.lists], 1.0, p(self.norm), p(ws["clip"]), 65536, stream)

    def reference(self):
        w = {k: v.double().requires_grad_() for k, v in self.value.items()}
        rms = lambda v, g: v / torch.sqrt(v.square().mean(1, keepdim=True) + self.EPS) * g  # noqa: E731
        T, H, K, W = self.T, self.H, self.K, self.W
        x = 1.5 * w["table"][self.ids.long()]
        n1 = rms(x, w["g1"])
        q, k, v = (n1 @ w["wqkv"].T).split([H * W, K * W, K * W], 1)
        row = torch.arange(T)
        s = torch.tensor([sum(a <= i for a in self.at[1:]) for i in range(T)])
        seen = (s[:, None] == s[None]) & (row[:, None] >= row[None])
        outs = []
        for h in range(H):
            sl = lambda m, i: m[:, i * W:(i + 1) * W]  # noqa: E731
            a = (0.25 * sl(q, h) @ sl(k, h * K // H).T).masked_fill(~seen, -math.inf).softmax(1)
            outs.append(a @ sl(v, h * K // H))
        r = x + 0.5 * torch.sigmoid(n1 @ w["wg"].T) * rms(torch.cat(outs, 1) @ w["wo"].T, w["post"])
        y = rms(r, w["g2"])
        (0.5 * (y - self.target.double()).square().sum()).backward()
        return y.detach(), {k: v.grad for k, v in w.items()}

    def state(self):
        return [self.buf["y"], self.norm] + list(self.grad.values()) + list(self.clipped.values())


def test_training_step_of_a_token_model():
    """Against autograd in 64 bits.  The step is some 20 contractions of at most 128 terms in a row; each passes on an error of its operands enlarged by
    no more than a few times its own, so that 1e-4 of a gradient's largest value (1700 units) is over ten times what roundings can
    make of it, and a wrong term in any operator is a hundredth at least."""
    step = Step([30, 1, 64, 0, 33], 40)
    step.run()
    torch.cuda.synchronize()
    y, grads = step.reference()
    near(step.buf["y"], y, 1e-5 * y.abs().max(), "y")
    for k, v in grads.items():
        near(step.grad[k], v, 1e-4 * v.abs().max(), k)
    norm = math.sqrt(sum(float(v.square().sum()) for v in grads.values()))
    assert norm > 1 and abs(step.norm.item() / norm - 1) <= 1e-4
    for k in grads:
        near(step.clipped[k], step.grad[k].cpu().double() / step.norm.item(), 8 * U * step.grad[k].cpu().double().abs(), k)


def test_training_step_on_a_stream_and_in_graphs():
    """On a stream of its own, captured, and replayed among eager runs, in turn with a second captured step: every time the same bits."""
    one, two = Step([30, 1, 64, 0, 33], 40), Step([5, 200], 41)
    want = []
    for s in (one, two):
        s.run()
        torch.cuda.synchronize()
        want.append([v.clone() for v in s.state()])
    side = torch.cuda.Stream()
    graphs = []
    with torch.cuda.stream(side):
        for s in (one, two):
            s.run(side.cuda_stream)
    side.synchronize()
    for s in (one, two):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            s.run(side.cuda_stream)
        graphs.append(graph)
    for _ in range(4):
        for s, graph, values in zip((one, two), graphs, want):
            for v in s.state():
                v.fill_(float("nan"))
            graph.replay()
            torch.cuda.synchronize()
            for got, v in zip(s.state(), values):
                assert torch.equal(got, v)
            s.run()
            torch.cuda.synchronize()
            for got, v in zip(s.state(), values):
                assert torch.equal(got, v)
