"""More operators of token models over the ranges that they are offered for: tiles of every size, shared sums, offsets past 32 bits.

Against their formulas in 64 bits, tolerances as in test_gpu_more_token_kernels.py."""
import math

import numpy as np
import pytest

from paper_2403_08837_amd import binding as b
from test_gpu_more_token_kernels import BF16, EPS, F32, TYPES, U, act_of, gated_workspace, half, p, planes

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


def normal(seed, *shape, scale=1.0, t=torch.float32):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return (scale * torch.randn(shape, generator=g, device="cuda")).to(t)


def near(got, want, tol, what):
    worst = ((got.double() - want).abs() / tol).max()
    assert got.shape == want.shape and bool(worst <= 1), (what, float(worst))


def check_linear(R, I, O, act, dtype, room):
    t = TYPES[dtype]
    x, w, dy, bias, res = normal(1, R, I, t=t), normal(2, O, I, scale=I ** -0.5, t=t), normal(3, R, O, t=t), normal(4, O, t=t), normal(5, R, O, t=t)
    y, z, dx, dw, db = (torch.full(s, float("nan"), dtype=t, device="cuda") for s in ((R, O), (R, O), (R, I), (O, I), (O,)))
    need = (4 if dtype == F32 else 2) * R * O + 4 * O * min(R, 256) + 1024
    ws = torch.full((need + room,), 0xff, dtype=torch.uint8, device="cuda")
    b.cdp_k_linear(dtype, act, p(x), p(w), p(bias), p(res), p(y), p(z), p(ws) if room else 0, room, R, I, O)
    b.cdp_k_linear_backward(dtype, act, p(x), p(w), p(z), p(dy), p(dx), p(dw), p(db), p(ws), ws.numel(), R, I, O)
    xd, wd, dyd = x.double(), w.double(), dy.double()
    want = xd @ wd.t() + bias.double()
    e = ((2 * I + 8) * U + planes(dtype)) * (xd.abs() @ wd.abs().t() + bias.double().abs())
    near(z, want, e + half(dtype) * want.abs(), "z")
    a = act_of(act, want)[0]
    near(y, a + res.double(), half(dtype) * (a + res.double()).abs() + 1.2 * e + 32 * U * (want.abs() + 1) + 2 * U * res.double().abs(), "y")
    zd = z.double()
    dz = dyd * act_of(act, zd)[1]
    s = (2.0 ** -8 if dtype == BF16 and act != 3 else 0.0) * dz.abs() + (64 * U * (zd.abs() + 1) * dyd.abs() if act != 3 else 0.0)
    for got, v, sv, o, n, what in ((dx, dz, s, wd, O, "dx"), (dw, dz.t(), s.t(), xd, R, "dw")):
        want = v @ o
        near(got, want, half(dtype) * want.abs() + sv @ o.abs() + ((2 * n + 8) * U + planes(dtype)) * ((v.abs() + sv) @ o.abs()), what)
    near(db, dz.sum(0), half(dtype) * dz.sum(0).abs() + s.sum(0) + R * U * dz.abs().sum(0), "dbias")


def check_gated(R, I, H, act, dtype, room):
    t = TYPES[dtype]
    x, wg, wu, dh = normal(1, R, I, t=t), normal(2, H, I, scale=I ** -0.5, t=t), normal(3, H, I, scale=I ** -0.5, t=t), normal(4, R, H, t=t)
    h, g, u, dx, dwg, dwu = (torch.full(s, float("nan"), dtype=t, device="cuda") for s in ((R, H),) * 3 + ((R, I), (H, I), (H, I)))
    ws = torch.full((gated_workspace(dtype, True, R, I, H) + room,), 0xff, dtype=torch.uint8, device="cuda")
    b.cdp_k_gated_linear(dtype, act, p(x), p(wg), p(wu), p(h), p(g), p(u), p(ws) if room else 0, room, R, I, H)
    b.cdp_k_gated_linear_backward(dtype, act, p(x), p(wg), p(wu), p(g), p(u), p(dh), p(dx), p(dwg), p(dwu), p(ws), ws.numel(), R, I, H)
    xd, wgd, wud, dhd = (v.double() for v in (x, wg, wu, dh))
    wantg, wantu = xd @ wgd.t(), xd @ wud.t()
    eg, eu = (((2 * I + 8) * U + planes(dtype)) * (xd.abs() @ w.abs().t()) for w in (wgd, wud))
    near(g, wantg, eg + half(dtype) * wantg.abs(), "g")
    near(u, wantu, eu + half(dtype) * wantu.abs(), "u")
    a = act_of(act, wantg)[0]
    near(h, a * wantu, half(dtype) * (a * wantu).abs() + 1.2 * eg * wantu.abs() + (a.abs() + 1.2 * eg) * eu + 32 * U * (wantg.abs() + 1) * wantu.abs(), "h")
    gd, ud = g.double(), u.double()
    a, da = act_of(act, gd)
    dg, du = dhd * ud * da, dhd * a
    mid = 2.0 ** -8 if dtype == BF16 else 0.0
    sg, su = (mid * v.abs() + 64 * U * (gd.abs() + 1) * s for v, s in ((dg, (dhd * ud).abs()), (du, dhd.abs())))
    want = dg @ wgd + du @ wud
    near(dx, want, half(dtype) * want.abs() + sg @ wgd.abs() + su @ wud.abs() + ((4 * H + 8) * U + planes(dtype)) * ((dg.abs() + sg) @ wgd.abs() + (du.abs() + su) @ wud.abs()), "dx")
    for got, v, s, what in ((dwg, dg, sg, "dwg"), (dwu, du, su, "dwu")):
        want = v.t() @ xd
        near(got, want, half(dtype) * want.abs() + s.t() @ xd.abs() + ((2 * R + 8) * U + planes(dtype)) * ((v.abs() + s).t() @ xd.abs()), what)


# enough for 256 x 256 tiles in bf16 and 128 x 128 in fp32, ragged and whole; long sums of few results; wide and narrow
LARGE = [(4096, 1024, 4096), (4100, 1032, 3080), (2000, 776, 2056), (8200, 64, 1024), (64, 8192, 128), (9000, 40, 48), (300, 4104, 1000), (1500, 3000, 704), (4090, 4104, 2048)]


@pytest.mark.parametrize("room", [0, 64 << 20])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("R,I,O", LARGE)
def test_linear_of_large_sizes(R, I, O, dtype, room):
    check_linear(R, I, O, 1, dtype, room)


@pytest.mark.parametrize("room", [0, 64 << 20])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("R,I,H", [(4096, 1024, 2048), (4100, 1032, 2056), (2000, 776, 1032), (8200, 64, 512), (64, 8192, 72), (9000, 40, 24), (300, 4104, 1000), (4090, 4104, 1024)])
def test_gated_linear_of_large_sizes(R, I, H, dtype, room):
    check_gated(R, I, H, 0, dtype, room)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("seed", range(24))
def test_linear_maps_of_any_size(seed, dtype):
    """Sizes over the logarithm of the range, room for shared sums or part of it, every activation."""
    g = np.random.default_rng(seed)
    R = int(np.exp(g.uniform(0, math.log(3000))))
    I, O = (8 * int(np.exp(g.uniform(0, math.log(300)))) for _ in range(2))
    room = int(g.choice([0, 4096, 1 << 18, 1 << 24]))
    check_linear(R, I, O, int(g.integers(4)), dtype, room)
    check_gated(R, I, O, int(g.integers(4)), dtype, room)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("R,I,O", [(16, 1032, 4096), (16, 1024, 4104), (17, 520, 1000), (31, 136, 40), (32, 1032, 2816), (33, 72, 24), (50, 264, 2824), (64, 1000, 1000), (64, 24, 5000), (65, 520, 1000), (9, 64, 20000),
                                   (30, 64, 20008), (60, 64, 20008)])
def test_linear_maps_of_some_rows(R, I, O, dtype):
    """One to four groups of 16 rows, whole and not, with one and two groups of columns."""
    check_linear(R, I, O, 0, dtype, 0)
    check_linear(R, I, O, 3, dtype, 1 << 22)
    check_gated(R, I, O, 1, dtype, 0)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("act", range(4))
@pytest.mark.parametrize("R,I,O", [(1, 8, 8), (3, 72, 248), (16, 64, 256), (16, 136, 264), (15, 200, 512), (1, 1000, 520), (17, 72, 256)])
def test_linear_maps_of_few_rows(R, I, O, act, dtype):
    """Around the sizes from which a backward pass is more than one launch."""
    check_linear(R, I, O, act, dtype, 0)
    check_gated(R, I, O, act, dtype, 0)


# ---- offsets past 32 bits ---------------------------------------------------------------------------------------------
def test_logprob_of_rows_far_apart():
    """Rows 2^31 elements apart, the third 8 GiB behind the first."""
    rows, V, ld, t = 3, 5001, 1 << 31, torch.bfloat16
    logits, dlogits = (torch.empty((rows - 1) * ld + V, dtype=t, device="cuda") for _ in range(2))
    x = normal(1, rows, V, scale=3, t=t)
    for r in range(rows):
        logits[r * ld:r * ld + V] = x[r]
        dlogits[r * ld + V:r * ld + V + 64] = 5
    targets = torch.tensor([7, 5000, 0], dtype=torch.int32, device="cuda")
    f = [torch.empty((2, rows), device="cuda") for _ in range(3)]
    ids, best = torch.empty((2, rows, 4), dtype=torch.int32, device="cuda"), torch.empty((2, rows, 4), device="cuda")
    dl, small = normal(2, rows), torch.empty((rows, V), dtype=t, device="cuda")
    for k, (a, pitch, d) in enumerate(((logits, ld, dlogits), (x, V, small))):
        b.cdp_k_token_logprob(BF16, p(a), pitch, p(targets), 1.0, *(p(v[k]) for v in f), p(ids[k]), p(best[k]), 4, 0, 0, rows, V)
        b.cdp_k_token_logprob_backward(BF16, p(a), pitch, p(targets), 1.0, p(f[2][k]), p(f[1][k]), p(dl), p(dl), p(d), rows, V)
    want = torch.log_softmax(x.double(), 1).gather(1, targets.long()[:, None])[:, 0]
    near(f[0][0], want, U * (V / 64 + 200) * torch.ones_like(want), "logprob")
    for v in (*f, ids, best):  # (rows that begin elsewhere in a 16-byte piece add up in another order)
        assert torch.equal(v[0], v[1]) or float((v[0] - v[1]).abs().max()) < U * (V / 64 + 200)
    for r in range(rows):
        assert float((dlogits[r * ld:r * ld + V].float() - small[r].float()).abs().max()) <= 2.0 ** -8
        if r < rows - 1:
            assert bool((dlogits[r * ld + V:r * ld + V + 64] == 5).all())


def test_rotary_of_many_tokens():
    """More than 2^31 elements: the last tokens as they come out of a call of their own."""
    T, H, K, W, n = 360000, 32, 8, 128, 50
    t, C = torch.bfloat16, (H + 2 * K) * W
    assert T * C > 2 ** 31
    x, d = (torch.empty((T, C), dtype=t, device="cuda") for _ in range(2))
    for v, s in ((x, 1), (d, 2)):
        v.fill_(0.5)
        v[-n:] = normal(s, n, C, t=t)
    pos = torch.arange(T, device="cuda", dtype=torch.int32)
    freqs, gamma = torch.rand(W // 2, device="cuda"), 1 + 0.1 * normal(3, 2, W)
    out, dx, dg = torch.empty_like(x), torch.empty_like(x), torch.empty((2, W), device="cuda")
    ws = torch.empty(8 * W * 1024 + 256, dtype=torch.uint8, device="cuda")
    few = [torch.empty((n, C), dtype=t, device="cuda") for _ in range(2)]
    for q, e, ps, o, g, m in ((x, d, pos, out, dx, T), (x[-n:], d[-n:], pos[-n:].clone(), few[0], few[1], n)):
        given = (p(q), p(ps), p(freqs), p(gamma), p(gamma[1]))
        b.cdp_k_head_norm_rotary(BF16, *given, p(o), EPS, 0, m, H, K, W, W)
        b.cdp_k_head_norm_rotary_backward(BF16, 0, *given, p(e), p(g), p(dg), p(dg[1]), EPS, 0, p(ws), ws.numel(), m, H, K, W, W)
    assert torch.equal(out[-n:], few[0]) and torch.equal(dx[-n:], few[1])


@pytest.mark.parametrize("R,I,O", [(1050000, 2056, 64), (40, 2056, 1048576), (4, 2056, 1048576), (1050000, 16, 2056)])
def test_linear_of_many_elements(R, I, O):
    """More than 2^31 elements of x, of w (and dw), of y: rows at either end, and the other operand's gradient."""
    t = torch.bfloat16
    assert max(R * I, I * O, R * O) > 2 ** 31
    x, w, y = torch.empty((R, I), dtype=t, device="cuda"), torch.empty((O, I), dtype=t, device="cuda"), torch.full((R, O), float("nan"), dtype=t, device="cuda")
    for v, n, s in ((x, R, 1), (w, O, I ** -0.5)):
        for k in range(0, n, 65536):
            v[k:k + 65536] = normal(k, *v[k:k + 65536].shape, scale=s, t=t)
    b.cdp_k_linear(BF16, 3, p(x), p(w), 0, 0, p(y), 0, 0, 0, R, I, O)
    rows, cols = (torch.cat([torch.arange(min(n, 40)), torch.arange(max(0, n - 40), n)]).unique().cuda() for n in (R, O))

    def sums(v, o, n):
        want = v @ o
        return want, 2.0 ** -8 * want.abs() + (2 * n + 8) * U * (v.abs() @ o.abs())
    near(y[rows][:, cols], *sums(x[rows].double(), w[cols].double().t(), I), "y")
    dy = y  # (any numbers)
    dx, dw = torch.full_like(x, float("nan")), torch.full_like(w, float("nan"))
    ws = torch.empty(2 * R * O + 4 * O * min(R, 256) + 1024 + (64 << 20), dtype=torch.uint8, device="cuda")
    b.cdp_k_linear_backward(BF16, 3, p(x), p(w), 0, p(dy), p(dx), p(dw), 0, p(ws), ws.numel(), R, I, O)
    some = torch.arange(0, I, max(1, I // 50)).cuda()

    def long(a, c, n):  # a[:, n] c[n, :] in pieces of n
        want = torch.zeros((a.shape[0], c.shape[1]), dtype=torch.float64, device="cuda")
        size = torch.zeros_like(want)
        for k in range(0, n, 65536):
            v, o = a[:, k:k + 65536].double(), c[k:k + 65536].double()
            want += v @ o
            size += v.abs() @ o.abs()
        # (sums of a million terms: those of 2^16 in a row, whose roundings are of either sign, are off by far less than their number of them)
        return want, 2.0 ** -8 * want.abs() + min(2 * n + 8, 2 ** 15) * U * size
    near(dx[rows][:, some], *long(dy[rows], w[:, some], O), "dx")
    near(dw[cols][:, some], *long(dy[:, cols].t(), x[:, some], R), "dw")
