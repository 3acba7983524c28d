"""More operators of token models (norms of heads with rotation, gated linear maps, token log probabilities) against their formulas in 64 bits.

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
GUARD = 16  # elements past an output that have to stay as they are


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
        return self(torch.full(shape, float("nan")) if t.is_floating_point else torch.full(shape, -77), t, shift)

    def workspace(self, n):
        """Exactly n bytes, of NaN."""
        whole = torch.full((n + 64,), 0xff, dtype=torch.uint8, device="cuda")
        whole[n:] = 7
        self.all.append((whole, 0, n))
        return whole[:n]

    def check(self):
        torch.cuda.synchronize()
        for whole, shift, n in self.all:
            assert bool((whole[:shift] == 7).all()) and bool((whole[shift + n:] == 7).all())


def p(x):
    return 0 if x is None else x.data_ptr()


def near(got, want, tol, what):
    got, tol = got.detach().cpu().double(), torch.as_tensor(tol, dtype=torch.float64)
    want = want.detach()
    assert got.shape == want.shape
    if not got.numel():
        return
    fine = (got - want).abs() <= tol
    fine |= torch.isnan(got) & torch.isnan(want) | (got == want)
    worst = ((got - want).abs() / tol.clamp(min=1e-300)).expand(got.shape).flatten().argmax()
    assert bool(fine.all()), (what, int((~fine).sum()), got.numel(), got.flatten()[worst].item(), want.flatten()[worst].item(), tol.expand(got.shape).flatten()[worst].item())


# ---- norms of heads and rotation --------------------------------------------------------------------------------------
EPS = 1e-6


def angles(positions, freqs):
    """Cosines and sines in 64 bits: the product of a position and an fp32 number fits the 64 bits of a long double's fraction."""
    a = positions.numpy().astype(np.longdouble)[:, None] * freqs.numpy().astype(np.longdouble)[None, :]
    return (torch.from_numpy(f(a).astype(np.float64))[:, None, :] for f in (np.cos, np.sin))


def turn(a, cos, sin, R, inter):
    x, y = (a[:, :, 0:R:2], a[:, :, 1:R:2]) if inter else (a[:, :, :R // 2], a[:, :, R // 2:R])
    t = torch.stack([x * cos - y * sin, y * cos + x * sin], 3)
    return torch.cat([t.flatten(2) if inter else t.transpose(2, 3).flatten(2), a[:, :, R:]], 2)


def size_of_pairs(a, R, inter):
    """|x| + |y| at both places of a pair, |x| elsewhere."""
    one = torch.ones((), dtype=torch.float64)
    return turn(a.abs(), one, -one, R, inter).clamp(min=0) * 0 + torch.cat([_pair_sum(a.abs(), R, inter), a[:, :, R:].abs()], 2)


def _pair_sum(a, R, inter):
    x, y = (a[:, :, 0:R:2], a[:, :, 1:R:2]) if inter else (a[:, :, :R // 2], a[:, :, R // 2:R])
    s = torch.stack([x + y, x + y], 3)
    return s.flatten(2) if inter else s.transpose(2, 3).flatten(2)


def rotary_reference(qkv, positions, freqs, gq, gk, dout, eps, inter, T, H, K, W, R):
    """Values and the sizes of the terms that they are sums of, in 64 bits."""
    a, d = (x.double().reshape(T, H + 2 * K, W) for x in (qkv, dout))
    x, v = a[:, :H + K], a[:, H + K:]
    cos, sin = angles(positions, freqs) if R else (torch.ones((T, 1, 0), dtype=torch.float64),) * 2
    gamma = torch.cat([(g if g is not None else torch.ones(W)).double().expand(n, W) for g, n in ((gq, H), (gk, K))])
    normed = torch.cat([torch.full((n, 1), 1.0 if g is not None else 0.0, dtype=torch.float64) for g, n in ((gq, H), (gk, K))])
    rho = torch.where(normed > 0, (x.square().mean(2, keepdim=True) + eps).rsqrt(), 1.0)
    hat = x * rho
    n = hat * gamma
    res = {"out": torch.cat([turn(n, cos, sin, R, inter), v], 1), "out_size": torch.cat([size_of_pairs(n, R, inter), 0 * v], 1)}
    dn, dn_size = turn(d[:, :H + K], cos, -sin, R, inter), size_of_pairs(d[:, :H + K], R, inter)
    e, e_size = dn * gamma, dn_size * gamma.abs()
    dx = rho * (e - normed * hat * (e * hat).mean(2, keepdim=True))
    dx_size = rho * (e_size + normed * hat.abs() * (e_size * hat.abs()).mean(2, keepdim=True))
    res.update(dqkv=torch.cat([dx, d[:, H + K:]], 1), dqkv_size=torch.cat([dx_size, 0 * v], 1))
    g, g_size = (dn * hat).sum(0), (dn_size * hat.abs()).sum(0)
    res.update(dgq=g[:H].sum(0), dgk=g[H:].sum(0), dgq_size=g_size[:H].sum(0), dgk_size=g_size[H:].sum(0))
    return {k: x.reshape(T, -1) if x.dim() == 3 else x for k, x in res.items()}


#      T, H, K, W, R, interleaved, gammas, positions up to
ROTARY = [(1, 1, 1, 8, 8, False, "qk", 0), (1, 4, 2, 128, 128, False, "qk", 2 ** 31 - 1), (3, 2, 1, 16, 16, True, "qk", 100), (65, 4, 2, 64, 64, False, "qk", 10000),
          (5, 3, 3, 40, 40, False, "qk", 7), (33, 8, 8, 80, 40, True, "qk", 1000), (7, 6, 2, 96, 12, False, "qk", 50), (9, 4, 4, 128, 2, False, "qk", 50), (4, 2, 1, 24, 22, False, "", 9),
          (130, 12, 4, 64, 64, True, "q", 2 ** 20), (17, 2, 2, 128, 126, True, "k", -2 ** 31), (600, 32, 8, 128, 128, False, "qk", 8192), (20, 2, 1, 48, 0, False, "qk", 0), (2, 40, 8, 112, 56, False, "k", 5),
          (2100, 1, 1, 8, 4, True, "q", 3), (1030, 5, 1, 32, 32, False, "", 2 ** 24), (6, 4000, 1, 8, 8, False, "qk", 3)]


def rotary_inputs(case, dtype, seed):
    T, H, K, W, R, inter, gammas, far = case
    C, t = (H + 2 * K) * W, TYPES[dtype]
    rng = np.random.default_rng(seed)
    positions = torch.from_numpy(rng.integers(min(0, far), max(0, far) + 1, T).astype(np.int32))
    freqs = torch.from_numpy((10000.0 ** (-np.arange(0, R, 2) / max(R, 1))).astype(np.float32))
    gq, gk = (1 + randn(seed + i, W, scale=0.3).float() if c in gammas else None for i, c in enumerate("qk"))
    return randn(seed + 3, T, C).to(t), positions, freqs, gq, gk, randn(seed + 4, T, C).to(t)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("case", ROTARY, ids=str)
def test_head_norm_rotary(dtype, case):
    """A norm's root: W squares and their sum, a root and its factors, W / 2 + 6 roundings; cosine and sine 3; two products and a sum 3.  Backward the
    same norm, the pair (6), the two sums over W: 2 W + 20.  Gammas: n terms and those."""
    T, H, K, W, R, inter, gammas, far = case
    t, hold = TYPES[dtype], Held()
    qkv, positions, freqs, gq, gk, dout = rotary_inputs(case, dtype, T + W)
    want = rotary_reference(qkv, positions, freqs, gq, gk, dout, float(np.float32(EPS)), inter, T, H, K, W, R)
    dev = [hold(qkv, t), hold(positions, torch.int32), hold(freqs, torch.float32), *(hold(g, torch.float32, 1) if g is not None else None for g in (gq, gk))]
    given = [p(x) for x in dev]
    if not R:
        given[1] = given[2] = 0
    out, sizes = hold.out(t, *qkv.shape), (T, H, K, W, R)
    b.cdp_k_head_norm_rotary(dtype, *given, p(out), EPS, int(inter), *sizes)
    near(out, want["out"], half(dtype) * want["out"].abs() + (W / 2 + 12) * U * want["out_size"], "out")
    dout_d, dqkv = hold(dout, t), hold.out(t, *qkv.shape)
    dg = [hold.out(torch.float32, W, shift=1) if g is not None else None for g in (gq, gk)]
    need = 8 * W * min(T, 1024) + 256
    ws = hold.workspace(need)
    b.cdp_k_head_norm_rotary_backward(dtype, 0, *given, p(dout_d), p(dqkv), p(dg[0]), p(dg[1]), EPS, int(inter), p(ws), need, *sizes)
    near(dqkv, want["dqkv"], half(dtype) * want["dqkv"].abs() + (2 * W + 20) * U * want["dqkv_size"], "dqkv")
    for g, name, n in ((dg[0], "dgq", T * H), (dg[1], "dgk", T * K)):
        if g is not None:
            near(g, want[name], (n + W / 2 + 16) * U * want[name + "_size"], name)
    # added to, in place of dout, and again: the same bits
    again = [g.clone() if g is not None else None for g in dg]
    same = dout_d.clone()
    b.cdp_k_head_norm_rotary_backward(dtype, 1, *given, p(same), p(same), p(again[0]), p(again[1]), EPS, int(inter), p(ws), need, *sizes)
    assert torch.equal(same, dqkv)
    for g, h in zip(again, dg):
        if g is not None:
            assert torch.equal(g, h + h)
    same = dev[0].clone()
    b.cdp_k_head_norm_rotary(dtype, p(same), *given[1:], p(same), EPS, int(inter), *sizes)
    assert torch.equal(same, out)
    hold.check()


# ---- gated linear -----------------------------------------------------------------------------------------------------
def act_of(act, g):
    s = torch.sigmoid(g)
    if act == 3:
        return g, torch.ones_like(g)
    if act == 0:
        return g * s, s * (1 + g * torch.sigmoid(-g))
    if act == 2:
        return s, s * torch.sigmoid(-g)
    phi = 0.5 * torch.erfc(-g * math.sqrt(0.5))
    return g * phi, phi + g * torch.exp(-0.5 * g * g) / math.sqrt(2 * math.pi)


GATED = [(2, 16, 8, 3), (70, 96, 40, 3), (1, 8, 8, 0), (1, 4096, 64, 0), (3, 24, 16, 1), (16, 72, 40, 2), (17, 8, 8, 0), (33, 64, 64, 1), (64, 200, 136, 0), (65, 136, 72, 2), (129, 72, 264, 0), (130, 520, 128, 1), (300, 64, 1000, 0),
         (257, 328, 520, 0), (20, 2048, 24, 0), (700, 40, 32, 2), (513, 1032, 264, 1)]


def planes(dtype):
    return 2.0 ** -24 if dtype == F32 else 0.0  # of a product: what the cut factors and the products left out come to, twice


def gated_workspace(dtype, backward, R, I, H):
    return (8 if dtype == F32 else 4) * R * H + 1024 if backward else 0


@pytest.mark.parametrize("shared", [0, 3])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("R,I,H,act", GATED)
def test_gated_linear(R, I, H, act, dtype, shared):
    """Sums of I terms: 2 I + 8 roundings (the matrix units' own and the sums').  An activation is within 32 roundings of its argument's size and has slopes
    up to 1.2.  Backward from the forward's own g and u: dg and du within 64 roundings and half a step of what the products take."""
    t, hold = TYPES[dtype], Held()
    x, wg, wu, dh = randn(1, R, I).to(t), randn(2, H, I, scale=I ** -0.5).to(t), randn(3, H, I, scale=I ** -0.5).to(t), randn(4, R, H).to(t)
    xd, wgd, wud, dhd = (v.double() for v in (x, wg, wu, dh))
    dev = [hold(v, t) for v in (x, wg, wu)]
    h, g, u, h2 = (hold.out(t, R, H) for _ in range(4))
    need = gated_workspace(dtype, False, R, I, H) + shared * 8 * R * H
    ws = hold.workspace(need) if need else None
    b.cdp_k_gated_linear(dtype, act, *map(p, dev), p(h), p(g), p(u), p(ws), need, R, I, H)
    b.cdp_k_gated_linear(dtype, act, *map(p, dev), p(h2), 0, 0, p(ws), need, R, I, H)
    assert torch.equal(h, h2)
    wantg, wantu = xd @ wgd.t(), xd @ wud.t()
    eg, eu = (((2 * I + 8) * U + planes(dtype)) * (xd.abs() @ w.abs().t()) for w in (wgd, wud))
    near(g, wantg, eg + half(dtype) * wantg.abs(), "g")
    near(u, wantu, eu + half(dtype) * wantu.abs(), "u")
    a, _ = act_of(act, wantg)
    want = a * wantu
    near(h, want, half(dtype) * want.abs() + 1.2 * eg * wantu.abs() + (a.abs() + 1.2 * eg) * eu + 32 * U * (wantg.abs() + 1) * wantu.abs(), "h")

    dx, dwg, dwu = hold.out(t, R, I), hold.out(t, H, I), hold.out(t, H, I)
    need = gated_workspace(dtype, True, R, I, H) + shared * max(4 * R * I, 8 * H * I)
    ws, dhc = hold.workspace(need), hold(dh, t)
    b.cdp_k_gated_linear_backward(dtype, act, *map(p, dev), p(g), p(u), p(dhc), p(dx), p(dwg), p(dwu), p(ws), need, R, I, H)
    gd, ud = g.cpu().double(), u.cpu().double()
    a, da = act_of(act, gd)
    dg, du = dhd * ud * da, dhd * a
    mid = 2.0 ** -8 if dtype == BF16 else 0.0
    sg, su = ((mid * v.abs() + 64 * U * (gd.abs() + 1) * s) for v, s in ((dg, (dhd * ud).abs()), (du, dhd.abs())))
    wantx = dg @ wgd + du @ wud
    sizex = (dg.abs() + sg) @ wgd.abs() + (du.abs() + su) @ wud.abs()
    # both, and one of the two alone
    dx2, dwg2, dwu2 = hold.out(t, R, I), hold.out(t, H, I), hold.out(t, H, I)
    b.cdp_k_gated_linear_backward(dtype, act, *map(p, dev), p(g), p(u), p(dhc), p(dx2), 0, 0, p(ws), need, R, I, H)
    b.cdp_k_gated_linear_backward(dtype, act, *map(p, dev), p(g), p(u), p(dhc), 0, p(dwg2), p(dwu2), p(ws), need, R, I, H)
    for got in (dx, dx2):
        near(got, wantx, half(dtype) * wantx.abs() + sg @ wgd.abs() + su @ wud.abs() + ((4 * H + 8) * U + planes(dtype)) * sizex, "dx")
    for got, v, s, what in ((dwg, dg, sg, "dwg"), (dwu, du, su, "dwu"), (dwg2, dg, sg, "dwg"), (dwu2, du, su, "dwu")):
        want = v.t() @ xd
        near(got, want, half(dtype) * want.abs() + s.t() @ xd.abs() + ((2 * R + 8) * U + planes(dtype)) * ((v.abs() + s).t() @ xd.abs()), what)
    hold.check()


# ---- linear -----------------------------------------------------------------------------------------------------------
LINEARS = [(1, 8, 8, 3, "br"), (1, 4096, 72, 0, ""), (3, 24, 16, 1, "b"), (16, 72, 40, 2, "r"), (17, 8, 8, 3, "br"), (33, 64, 64, 1, ""), (64, 200, 136, 0, "br"), (65, 136, 72, 3, "r"), (129, 72, 264, 0, "b"),
           (130, 520, 128, 1, "br"), (300, 64, 1000, 3, "b"), (257, 328, 520, 3, ""), (20, 2048, 24, 0, "br"), (700, 40, 32, 2, "br"), (513, 1032, 264, 1, "b"), (9000, 16, 24, 0, "b"), (2050, 4104, 4104, 3, "br")]


@pytest.mark.parametrize("shared", [0, 3])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("R,I,O,act,extra", LINEARS)
def test_linear(R, I, O, act, extra, dtype, shared):
    """As of a gated map; bias and residual one rounding each.  dbias: R terms of dz before its rounding."""
    t, hold = TYPES[dtype], Held()
    x, w, dy = randn(1, R, I).to(t), randn(2, O, I, scale=I ** -0.5).to(t), randn(4, R, O).to(t)
    bias = randn(5, O).to(t) if "b" in extra else None
    residual = randn(6, R, O).to(t) if "r" in extra else None
    big = R * I * O > 2 ** 31
    work = (lambda v: v.cuda()) if big else (lambda v: v)  # (the references, in 64 bits either way)
    xd, wd, dyd = (work(v.double()) for v in (x, w, dy))
    dev = [hold(v, t) for v in (x, w)] + [hold(v, t) if v is not None else None for v in (bias, residual)]
    y, z, y2 = (hold.out(t, R, O) for _ in range(3))
    need = shared * 4 * R * O
    ws = hold.workspace(need) if need else None
    b.cdp_k_linear(dtype, act, *map(p, dev), p(y), p(z), p(ws), need, R, I, O)
    if residual is not None:
        y2.copy_(dev[3])
    b.cdp_k_linear(dtype, act, *map(p, dev[:3]), p(y2) if residual is not None else 0, p(y2), 0, p(ws), need, R, I, O)
    assert torch.equal(y, y2)
    bd = work(bias.double()) if bias is not None else torch.zeros((), dtype=torch.float64)
    want = xd @ wd.t() + bd
    e = ((2 * I + 8) * U + planes(dtype)) * (xd.abs() @ wd.abs().t() + bd.abs())
    near(z, want.cpu(), (e + half(dtype) * want.abs()).cpu(), "z")
    if act == 3:
        a, slope = want, 1.0
    else:
        a, slope = act_of(act, want)[0], 1.2
    rd = work(residual.double()) if residual is not None else torch.zeros((), dtype=torch.float64)
    near(y, (a + rd).cpu(), (half(dtype) * (a + rd).abs() + slope * e + 32 * U * (want.abs() + 1) + 2 * U * rd.abs()).cpu(), "y")

    dx, dw, dbias = hold.out(t, R, I), hold.out(t, O, I), hold.out(t, O)
    need = (4 if dtype == F32 else 2) * R * O + 4 * O * min(R, 256) + 1024 + shared * 4 * max(R, O) * I
    ws, dyc = hold.workspace(need), hold(dy, t)
    zin = p(z) if act != 3 else 0
    b.cdp_k_linear_backward(dtype, act, p(dev[0]), p(dev[1]), zin, p(dyc), p(dx), p(dw), p(dbias), p(ws), need, R, I, O)
    zd = work(z.cpu().double())
    da = act_of(act, zd)[1] if act != 3 else torch.ones_like(zd)
    dz = dyd * da
    close = (64 * U * (zd.abs() + 1) * dyd.abs()) if act != 3 else 0 * dyd
    s = (2.0 ** -8 if dtype == BF16 and act != 3 else 0.0) * dz.abs() + close
    alone = [hold.out(t, *v.shape) for v in (dx, dw, dbias)]
    for one in range(3):
        b.cdp_k_linear_backward(dtype, act, p(dev[0]) if one == 1 else 0, p(dev[1]) if one == 0 else 0, zin, p(dyc), *(p(v) if k == one else 0 for k, v in enumerate(alone)),
                                p(ws), need, R, I, O)
    for got, v, sv, o, n, what in ((dx, dz, s, wd, O, "dx"), (dw, dz.t(), s.t(), xd, R, "dw"), (alone[0], dz, s, wd, O, "dx alone"), (alone[1], dz.t(), s.t(), xd, R, "dw alone")):
        want = v @ o
        near(got, want.cpu(), (half(dtype) * want.abs() + sv @ o.abs() + ((2 * n + 8) * U + planes(dtype)) * ((v.abs() + sv) @ o.abs())).cpu(), what)
    want = dz.sum(0)
    for got in (dbias, alone[2]):
        near(got, want.cpu(), (half(dtype) * want.abs() + close.sum(0) + R * U * dz.abs().sum(0)).cpu(), "dbias")
    hold.check()


# ---- token log probabilities ------------------------------------------------------------------------------------------
def logprob_reference(logits, targets, scale, top):
    z = logits.double() * scale
    V = z.shape[1]
    used = (targets >= 0) & (targets < V) if targets is not None else torch.ones(len(z), dtype=torch.bool)
    lse = torch.logsumexp(z, 1)
    none = torch.isinf(lse)
    logp = torch.where(none[:, None], torch.full_like(z, -math.inf), z - lse[:, None])
    prob = torch.exp(logp)
    plogp = torch.where(prob > 0, prob * logp, torch.where(torch.isnan(prob), prob, 0.0))
    entropy = -plogp.sum(1)
    order = torch.sort(torch.where(torch.isnan(logits.double()), -math.inf, logits.double()), dim=1, descending=True, stable=True).indices[:, :top]
    return dict(z=z, used=used, lse=lse, logp=logp, prob=prob, entropy=entropy, order=order, top=logp.gather(1, order))


#          rows, vocab, pitch, top, kind
LOGPROBS = [(1, 1, 1, 1, "even"), (1, 2, 5, 2, "even"), (3, 7, 7, 3, "masked"), (5, 8, 8, 8, "ties"), (4, 63, 64, 20, "even"), (2, 1000, 1003, 64, "ties"), (9, 2049, 2049, 5, "masked"), (2, 50257, 50257, 20, "even"),
            (1, 128000, 128000, 64, "even"), (3, 131073, 131075, 50, "ties"), (2, 65536, 65536, 64, "rising"), (1200, 300, 301, 4, "padded"), (1100, 5000, 5000, 0, "padded"), (40, 17000, 17000, 1, "equal"),
            (6, 70000, 70000, 33, "equal"), (1030, 9001, 9001, 64, "rising"), (3, 20000, 20001, 20, "block")]


def logits_of(kind, rows, vocab, pitch, dtype, seed):
    x = randn(seed, rows, pitch, scale=3.0)
    g = np.random.default_rng(seed)
    if kind == "masked":
        x[torch.from_numpy(g.random((rows, pitch)) < 0.6)] = -math.inf
        x[0] = -math.inf
        x[-1, :vocab] = -math.inf
        x[-1, vocab // 2] = 1.5
    if kind == "ties":
        x = (x * 2).round() / 2
        x[x == 0] = torch.where(torch.rand(int((x == 0).sum())) < 0.5, -0.0, 0.0).double()
    if kind == "rising":
        x = x.sort(1).values
    if kind == "equal":
        x = torch.full_like(x, 1.25)
    if kind == "block":
        x[:, vocab // 3:vocab // 3 + 5000] += 30
    return x.to(TYPES[dtype])


@pytest.mark.parametrize("shared", [False, True])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("case", LOGPROBS, ids=str)
def test_token_logprob(case, dtype, shared):
    """A sum of V exponentials in lanes: V / 64 + 64 roundings, and each exponential's argument two of its size, up to the largest |z| twice.  Backward: the
    argument's roundings, of |z| and |lse|, and ten more.  The argument log p is a difference of those two, off by `left` whatever is left of it, so p (log p + H)
    is by p (left + left (|log p| + H)): the 1 in its size."""
    rows, V, pitch, top, kind = case
    t, hold, scale = TYPES[dtype], Held(), 0.75
    logits = logits_of(kind, rows, V, pitch, dtype, rows + V)
    g = np.random.default_rng(V)
    targets = torch.from_numpy(g.integers(0, V, rows).astype(np.int32))
    if kind == "padded":
        targets[torch.from_numpy(g.random(rows) < 0.4)] = -1
        targets[0], targets[-1] = V, 2 ** 31 - 1
    shift = rows % 3
    dev, tg = hold(logits, t, shift), hold(targets, torch.int32, 1)
    logprob, entropy, lse = (hold.out(torch.float32, rows, shift=1) for _ in range(3))
    ids, best = hold.out(torch.int32, rows, top, shift=1), hold.out(torch.float32, rows, top, shift=1)
    ws = hold.workspace(1 << 20) if shared else None
    given = (dtype, p(dev), pitch, p(tg), scale)
    b.cdp_k_token_logprob(*given, p(logprob), p(entropy), p(lse), p(ids) if top else 0, p(best) if top else 0, top, p(ws), 1 << 20 if shared else 0, rows, V)
    want = logprob_reference(logits[:, :V], targets, scale, top)
    used = want["used"]
    finite = torch.where(torch.isfinite(want["z"]), want["z"], 0.0)
    most = finite.abs().amax(1)
    tol = U * (V / 64 + 64 + 4 * most + want["lse"].abs().nan_to_num(posinf=0))
    at = targets.long().clamp(0, V - 1)[:, None]
    zero = torch.zeros((), dtype=torch.float64)
    near(lse, torch.where(used, want["lse"], zero), tol, "lse")
    near(logprob, torch.where(used, want["logp"].gather(1, at)[:, 0], zero), 2 * tol, "logprob")
    far = (want["lse"] - want["z"].amax(1)).nan_to_num() + 20 + math.log(V)
    near(entropy, torch.where(used, want["entropy"], zero), 4 * tol * far, "entropy")
    if top:
        order = torch.where(used[:, None], want["order"], -1)
        assert torch.equal(ids.cpu().long(), order), (ids.cpu().long() != order).nonzero()[:5]
        near(best, torch.where(used[:, None], want["top"], zero), 2 * tol[:, None], "top")
    dl, de = randn(8, rows).float(), randn(9, rows, scale=0.3).float()
    dld, ded = hold(dl, torch.float32), hold(de, torch.float32, 1)
    dlogits = hold(torch.full((rows, pitch), 5.0), t, shift)
    b.cdp_k_token_logprob_backward(*given, p(lse), p(entropy), p(dld), p(ded), p(dlogits), rows, V)
    prob, logp = want["prob"], torch.where(want["prob"] > 0, want["logp"], zero)
    H = want["entropy"][:, None]
    one = torch.zeros_like(prob).scatter_(1, at, 1.0)
    some = (used & ~torch.isinf(want["lse"]))[:, None]
    d = scale * (dl.double()[:, None] * (one - prob) - de.double()[:, None] * prob * (logp + H))
    size = scale * (dl.double().abs()[:, None] * (one + prob) + de.double().abs()[:, None] * prob * (logp.abs() + H + 1))
    left = U * (4 * most + 4 * want["lse"].abs().nan_to_num(posinf=0))[:, None] + (4 * tol * far)[:, None] + 16 * U
    near(dlogits[:, :V], torch.where(some, d, zero), half(dtype) * d.abs() + 2 * left * size + 1e-37, "dlogits")
    assert bool((dlogits[:, V:] == 5).all())
    # in place, and either gradient alone
    same = dev.clone()
    b.cdp_k_token_logprob_backward(dtype, p(same), *given[2:], p(lse), p(entropy), p(dld), p(ded), p(same), rows, V)
    assert torch.equal(same[:, :V], dlogits[:, :V]) and torch.equal(same[:, V:].nan_to_num(), dev[:, V:].nan_to_num())
    # at another alignment than the logits
    other = hold(torch.full((rows, pitch), 5.0), t, shift + 1)
    b.cdp_k_token_logprob_backward(*given, p(lse), p(entropy), p(dld), p(ded), p(other), rows, V)
    assert torch.equal(other, dlogits)
    b.cdp_k_token_logprob_backward(*given, p(lse), 0, p(dld), 0, p(dlogits), rows, V)
    d1, s1 = scale * dl.double()[:, None] * (one - prob), scale * dl.double().abs()[:, None] * (one + prob)
    near(dlogits[:, :V], torch.where(some, d1, zero), half(dtype) * d1.abs() + left * s1 + 1e-37, "from logprob")
    b.cdp_k_token_logprob_backward(dtype, p(dev), pitch, 0, scale, p(lse), p(entropy), 0, p(ded), p(dlogits), rows, V)
    d2, s2 = -scale * de.double()[:, None] * prob * (logp + H), scale * de.double().abs()[:, None] * prob * (logp.abs() + H + 1)
    keep = ~torch.isinf(want["lse"]) & used  # (rows that were not wanted have no lse)
    near(dlogits[keep][:, :V], d2[keep], half(dtype) * d2[keep].abs() + 2 * left[keep] * s2[keep] + 1e-37, "from entropy")
    hold.check()
