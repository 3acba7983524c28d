"""Operators of token models over the ranges that they are offered for: far magnitudes, open gates, launches of many rows, every kernel of packed attention.

Against their formulas in 64 bits, tolerances as in test_gpu_token_kernels.py: U = 2^-24 and half(t) are half a step of fp32 and of the element type."""
import math

import numpy as np
import pytest

from paper_2403_08837_amd import binding as b
from test_gpu_token_kernels import (BF16, F32, TYPES, U, Held, Step, attention_call, attention_case, attention_reference, clip_call, half, near, norm_case, norm_reference, norm_tolerance,
                                    p, randn, workspace)

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


# ---- norms around a block ---------------------------------------------------------------------------------------------
def norm_calls(v, dtype, scale, eps, shift=0):
    """Both directions on tensors that begin `shift` elements past a 16-byte border: everything that is written, by name."""
    rows, C = v["x"].shape
    t, hold = TYPES[dtype], Held()
    dev = {k: None if x is None else hold(x, x.dtype, shift) for k, x in v.items()}
    made = lambda there: hold.out(t, rows, C, shift=shift) if there is not None else None  # noqa: E731
    got = {"r": made(v["x"]), "y": made(v["pre"]), "dx": made(v["x"]), "dh": made(v["h"]), "dgate": made(v["gate"])}
    for k in ("post", "pre"):
        got["d" + k] = hold.out(torch.float32, C, shift=shift) if v[k] is not None else None
    b.cdp_k_residual_norm(dtype, p(dev["x"]), p(dev["h"]), p(dev["gate"]), p(dev["post"]), p(dev["pre"]), p(got["r"]), p(got["y"]), scale, eps, rows, C)
    need = 8 * C * min(rows, 512) + 256
    b.cdp_k_residual_norm_backward(dtype, 0, p(dev["x"]) if v["pre"] is not None else 0, p(dev["h"]), p(dev["gate"]), p(dev["post"]), p(dev["pre"]), p(dev["dr"]), p(dev["dy"]),
                                   p(got["dx"]), p(got["dh"]), p(got["dgate"]), p(got["dpost"]), p(got["dpre"]), scale, eps, p(workspace(need)), need, rows, C)
    hold.check()
    return {k: x for k, x in got.items() if x is not None}


def norm_check(v, dtype, scale, eps, shift=0):
    rows = v["x"].shape[0]
    got = norm_calls(v, dtype, scale, eps, shift)
    args = [None if v[k] is None else v[k].cuda().double() for k in ("x", "h", "gate", "post", "pre", "dr", "dy")]
    res, size = norm_reference(*args, scale, float(np.float32(eps)))
    for k, x in got.items():
        near(x, res[k].cpu(), norm_tolerance(k, res, size, dtype, rows).cpu(), k)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("form", ["all", "no post", "norm alone", "end", "no dr"])
@pytest.mark.parametrize("x_size,h_size", [(1e13, 1.0), (1e15, 1e-12), (1e17, 1e17), (1.0, 1e13), (1.0, 1e15), (1e-12, 1e17), (1e-12, 1e-12)])
@pytest.mark.parametrize("C", [776, 250])
def test_residual_norm_of_large_and_small_rows(dtype, form, x_size, h_size, C):
    """Magnitudes whose squares fp32 holds (and whose cubes it does not)."""
    v = norm_case(form, 21, C, TYPES[dtype], C)
    for k, size in (("x", x_size), ("h", h_size)):
        v[k] = None if v[k] is None else (v[k].double() * size).to(v[k].dtype)
    norm_check(v, dtype, 0.75, 1e-5)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("eps", [1e-24, 1e-30])
def test_residual_norm_of_zeros_with_a_small_eps(dtype, eps):
    """Rows of zeros among others: their reciprocal roots are 1e12 and 1e15, what they make of dy is finite."""
    v = norm_case("all", 12, 264, TYPES[dtype], 3)
    v["x"][2], v["h"][2], v["h"][7] = 0, 0, 0
    norm_check(v, dtype, 0.75, eps)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_residual_norm_of_open_gates(dtype):
    """dgate of gates that are nearly open or shut is as exact as its factor sig (1 - sig) is small.  exp(-|g|): the exponent in units of 2 is rounded
    twice, 2 |g| U, and the power is 2 U off; one addition, a reciprocal of 2 U, their product, and four more products: (2 |g| + 16) U."""
    t = TYPES[dtype]
    gate = torch.tensor([[g * s for g in (0.5, 3.0, 5.0, 10.0, 12.0, 15.0, 17.0, 20.0, 40.0, 60.0, 0.0, 1.0) for s in (1, -1)]])
    h, dr = randn(1, *gate.shape).to(t), randn(2, *gate.shape).to(t)
    got = norm_calls({"x": h, "h": h, "gate": gate.to(t), "post": None, "pre": None, "dr": dr, "dy": None}, dtype, 0.75, 1e-5)
    g = gate.to(t).double()
    q, e = 1 / (1 + torch.exp(-g.abs())), torch.exp(-g.abs())
    sig = torch.where(g < 0, e * q, q)
    want = 0.75 * h.double() * dr.double() * e * q * q
    near(got["dgate"], want, ((2 * g.abs() + 16) * U + half(dtype)) * want.abs(), "dgate")
    near(got["dh"], 0.75 * sig * dr.double(), ((2 * g.abs() + 16) * U + half(dtype)) * (0.75 * sig * dr.double()).abs(), "dh")


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("gated", [False, True])
def test_residual_of_what_is_not_finite(dtype, gated):
    """Without norms nothing but its own place sees an infinite or missing value of h, and there only what the formula says does."""
    t, rows, C = TYPES[dtype], 3, 16
    v = norm_case("end", rows, C, t, 4)
    v["post"] = None
    if not gated:
        v["gate"] = None
    v["h"][1, 3], v["h"][2, 5] = float("inf"), float("nan")
    got = norm_calls(v, dtype, 0.75, 1e-5)
    sig = torch.sigmoid(v["gate"].double()) if gated else torch.ones(rows, C, dtype=torch.float64)
    dr, h = v["dr"].double(), v["h"].double()
    near(got["dx"], dr, 0.0, "dx")
    near(got["dh"], 0.75 * sig * dr, (half(dtype) + 32 * U) * (0.75 * sig * dr).abs(), "dh")
    want = v["x"].double() + 0.75 * sig * h
    near(got["r"], want, torch.nan_to_num((half(dtype) + 32 * U) * (v["x"].double().abs() + (0.75 * sig * h).abs()), nan=0.0, posinf=0.0), "r")
    if gated:
        want = 0.75 * h * dr * sig * (1 - sig)
        near(got["dgate"], want, torch.nan_to_num((half(dtype) + 32 * U) * want.abs(), nan=0.0, posinf=0.0), "dgate")
    v["post"] = norm_case("end", rows, C, t, 4)["post"]  # (a row of h without a norm has no gradient; r has)
    near(norm_calls(v, dtype, 0.75, 1e-5)["dx"], dr, 0.0, "dx, with a norm of h")


# more row groups than workgroups backward (512), so that every one has a second and third, of one wavefront's lanes or several, on aligned tensors and others
MANY_ROWS = [(20000, 64), (6272, 192), (2100, 768), (1700, 1000), (1300, 2056), (1100, 4096), (1037, 8192), (515, 16384), (700, 1500)]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,C", MANY_ROWS)
@pytest.mark.parametrize("form,shift", [("all", 0), ("all", 1), ("norm alone", 0), ("no dr", 0)])
def test_residual_norm_of_many_rows(dtype, rows, C, form, shift):
    norm_check(norm_case(form, rows, C, TYPES[dtype], C), dtype, 0.75, 1e-5, shift)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,C", [(2, 64), (64, 64), (34, 256), (600, 96), (4, 4096), (2, 8192), (4, 16384), (6, 768), (40, 1000), (1030, 520)])
def test_residual_norm_of_aligned_rows(dtype, rows, C):
    """Even numbers of rows on tensors of 16-byte borders."""
    for form in ("all", "no post", "no gate", "h alone", "norm alone", "end", "no dr"):
        norm_check(norm_case(form, rows, C, TYPES[dtype], C), dtype, 0.75, 1e-5)


# ---- packed causal attention --------------------------------------------------------------------------------------------
# Cases by which every kernel is compared, of every width: queries and keys, wavefronts that share 32 rows and those that have 32 each, equal heads and grouped
# ones, and those whose query heads are shared by workgroups (with room for their sums in the workspace).
PLACES = [(0, [2100], 2, 54, 6, 16), (0, [2090], 0, 54, 6, 32), (1, [2060], 0, 54, 6, 40), (0, [2100], 0, 54, 6, 64), (0, [2050], 0, 54, 6, 72), (0, [2077], 3, 45, 5, 96)]
PLACES += [(0, [130, 131] * 4, 1, 54, 54, w) for w in (16, 32, 40, 64, 80, 88, 112, 128)]
PLACES += [(0, [300, 290], 11, 2, 2, w) for w in (8, 32, 48, 64, 80, 96, 104, 128)]
PLACES += [(2, [600, 95], 0, 4, 2, w) for w in (16, 24, 48, 64, 72, 96, 112, 120)]
PLACES += [(0, [60, 39], 1, 2, 2, w) for w in (80, 104)] + [(0, [33, 60], 0, 4, 2, w) for w in (72, 112)]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("before,lengths,behind,heads,kv_heads,width", PLACES, ids=str)
def test_packed_attention_by_every_kernel(dtype, before, lengths, behind, heads, kv_heads, width):
    t, scale = TYPES[dtype], 1.3 * width ** -0.5
    at, qkv, dout = attention_case(before, lengths, behind, heads, kv_heads, width, t, width)
    outside = torch.ones(qkv.shape[0], dtype=torch.bool)
    outside[at[0]:at[-1]] = False
    qkv[outside], dout[outside] = float("nan"), float("nan")
    used = ~outside
    scale32 = float(np.float32(scale))
    with torch.device("cuda"):  # (the references' products of long sequences)
        clean = lambda v: torch.where(outside.cuda()[:, None], 0.0, v.cuda().double())  # noqa: E731
        res, tol, _ = attention_reference(clean(qkv), at, heads, kv_heads, width, scale32, dtype)
    for parts in (0, 8) if heads > kv_heads else (0,):
        out, lse, dqkv = attention_call(dtype, qkv, at, heads, kv_heads, width, scale, dout, parts)
        near(out.cpu()[used], res["out"].cpu()[used], tol["out"].cpu()[used], "out")
        near(lse.cpu()[:, used], res["lse"].cpu()[:, used], tol["lse"].cpu()[:, used], "lse")
        with torch.device("cuda"):
            back, back_tol, _ = attention_reference(clean(qkv), at, heads, kv_heads, width, scale32, dtype, clean(dout), clean(out), torch.where(outside.cuda(), 0.0, lse.double()))
        near(dqkv.cpu()[used], back["dqkv"].cpu()[used], back_tol["dqkv"].cpu()[used], "dqkv, %d parts" % parts)
        for v in (out, lse.T, dqkv):
            assert bool(torch.isnan(v[outside.cuda()]).all())


def test_packed_attention_products_of_fp32():
    """A score of two products that all but cancel, a b - fl(a b), enlarged 2^20 times: one token per sequence, whose lse is that score.  A product is
    that of three planes of 8 bits of either operand without the three smallest of nine: with 2^-7 and 2^-15 at most behind the first and the second plane, 2 x 2^-22 + 2^-30 of the
    product.  The last of its sums, whose terms are as large, has U; what the five sums before it have is 2^-6 at most.  Then 8 U of lse itself."""
    g = np.random.default_rng(5)
    T, H, W = 200, 8, 8
    a, c = ((1 + g.random((T, H))).astype(np.float32) for _ in range(2))
    a[0], c[0] = 1 + 2.0 ** -7 - 2.0 ** -23, 1 + 2.0 ** -7 - 2.0 ** -23
    a[1], c[1] = 1 + 2.0 ** -7 - 2.0 ** -15, 1 + 2.0 ** -6 - 2.0 ** -22
    qkv = torch.zeros(T, 3, H, W)
    qkv[:, 0, :, 0], qkv[:, 1, :, 0] = torch.from_numpy(a), torch.from_numpy(c)
    qkv[:, 0, :, 1], qkv[:, 1, :, 1] = torch.from_numpy(-(a * c)), 1.0
    out, lse, _ = attention_call(F32, qkv.reshape(T, 3 * H * W), list(range(T + 1)), H, H, W, 2.0 ** 20, None, 0)
    product = a.astype(np.float64) * c
    want = torch.from_numpy((product - (a * c)).T * 2.0 ** 20)
    near(lse, want, 2.0 ** 20 * ((2.0 ** -21 + 2.0 ** -30 + U) * torch.from_numpy(product.T) + 5 * U * 2.0 ** -6) + 8 * U * want.abs(), "lse")


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("heads,kv_heads,width,lengths", [(2, 1, 16, [20, 33, 9]), (4, 4, 64, [40, 100, 31]), (4, 2, 72, [300, 321, 65]), (54, 54, 64, [130, 129, 140])])
def test_packed_attention_of_what_is_not_finite_stays_in_its_sequence(dtype, heads, kv_heads, width, lengths):
    """Rows of q, k, v and dout in the middle sequence, its first and last among them: the other two have the same bits as without."""
    at, qkv, dout = attention_case(1, lengths, 2, heads, kv_heads, width, TYPES[dtype], 7)
    clean = attention_call(dtype, qkv, at, heads, kv_heads, width, 0.2, dout, 0)
    qkv, dout = qkv.clone(), dout.clone()
    x = qkv.view(qkv.shape[0], heads + 2 * kv_heads, width)
    for row, what in ((at[1], float("inf")), (at[1] + 3, float("nan")), (at[2] - 1, -float("inf"))):
        x[row, ::2], dout[row, 5:] = what, what
    got = attention_call(dtype, qkv, at, heads, kv_heads, width, 0.2, dout, 0)
    for a, b_ in ((at[0], at[1]), (at[2], at[3])):
        for i, (one, two) in enumerate(zip(clean, got)):
            one, two = (v.T[a:b_] if i == 1 else v[a:b_] for v in (one, two))
            assert torch.equal(one, two) and bool(torch.isfinite(one).all())


def test_packed_attention_of_the_largest_values():
    """Finite values that round to an infinite one in fewer bits are finite: one key, whose value is the result."""
    big = torch.finfo(torch.float32).max
    qkv = torch.zeros(2, 24)
    qkv[0, 16:], qkv[1, 16:] = big, torch.tensor([big, -big, 2.0 ** 127, 3.39e38, 3.397e38, -3.4e38, 1.0, 0.0])
    out, lse, _ = attention_call(F32, qkv, [0, 1, 2], 1, 1, 8, 1.0, None, 0)
    assert torch.equal(out.cpu(), qkv[:, 16:]) and not lse.any()


# ---- gradient clipping -----------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n", [5, 60001, 3000017])
@pytest.mark.parametrize("max_norm", [1.0, 1e-6, 1e-20])
def test_grad_clip_by_small_factors(dtype, n, max_norm):
    """Factors that are subnormal or smaller in fp32: what is left of the gradients is not."""
    t = TYPES[dtype]
    v = (1 + randn(n, n).abs().clamp(max=2)).mul(1e38).to(t)
    grads, outs = [v.cuda()], [torch.full((n,), float("nan"), dtype=t, device="cuda")]
    norm = clip_call(dtype, grads, outs, max_norm)
    want = math.sqrt(float((v.double() / 1e38).square().sum())) * 1e38
    if want < 3.4e38:
        near(norm, torch.tensor([want], dtype=torch.float64), 2 * U * want, "norm")
    want = v.double() * (max_norm / want)
    near(outs[0], want, (half(dtype) + 4 * U) * want.abs(), "out")


# ---- more than 32 bits --------------------------------------------------------------------------------------------------
FAR = 540_000, 4096  # rows and columns: more than 2^31 elements, 4.4 GB in bf16


def far_tensor(seed, rows, C):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn((rows, C), generator=g, device="cuda", dtype=torch.bfloat16)


def test_embedding_of_rows_past_2_to_the_31():
    """Lookup and gradient; words are taken in turn, so that a word's tokens lie everywhere."""
    (rows, C), vocab = FAR, 1001
    table, ids = far_tensor(1, vocab, C), (torch.arange(rows, device="cuda") % vocab).to(torch.int32)
    out = torch.empty((rows, C), device="cuda", dtype=torch.bfloat16)
    b.cdp_k_embedding(BF16, 0, p(table), p(ids), 0, p(out), 1.0, 0, 0, rows, vocab, C)
    for at in range(0, rows, 50_000):
        assert torch.equal(out[at:at + 50_000], table[ids[at:at + 50_000].long()])
    need = 16 * rows + 8 * C * -(-rows // 32) + 512
    dtable, ws = torch.empty((vocab, C), device="cuda"), torch.empty(need, dtype=torch.uint8, device="cuda")
    b.cdp_k_embedding(BF16, 1, 0, p(ids), p(out), p(dtable), 1.0, p(ws), need, rows, vocab, C)
    n = torch.bincount(ids, minlength=vocab).double()[:, None]
    near(dtable, (n * table.double()).cpu(), ((n + 2) * U * n * table.double().abs()).cpu(), "dtable")


@pytest.mark.parametrize("rows,vocab", [(5000, (1 << 20) - 1), (5000, 1 << 20), (5000, (1 << 20) + 5), (600_000, 4001), (530_000, 3)])
def test_embedding_gradient_of_many_words_and_tokens(rows, vocab):
    """Keys of 32 and of 64 bits over several runs; three rounds of merges."""
    C = 4
    ids = torch.randint(-1, vocab + 1, (rows,), generator=torch.Generator().manual_seed(rows))
    ids[::7] = vocab - 1
    dout, need = randn(2, rows, C).float(), 16 * rows + 8 * C * -(-rows // 32) + 512
    got = torch.full((vocab, C), float("nan"), device="cuda")
    ids_d, dout_d = ids.to(torch.int32).cuda(), dout.cuda()
    b.cdp_k_embedding(F32, 1, 0, p(ids_d), p(dout_d), p(got), 1.0, p(workspace(need)), need, rows, vocab, C)
    inside = (ids >= 0) & (ids < vocab)
    at, d = torch.where(inside, ids, 0), dout.double() * inside[:, None]
    grad, size, n = (torch.zeros((vocab, k), dtype=torch.float64).index_add_(0, at, v) for k, v in ((C, d), (C, d.abs()), (1, inside.double()[:, None])))
    near(got, grad, (n + 2) * U * size, "dtable")


def test_residual_norm_of_rows_past_2_to_the_31():
    (rows, C), scale, eps = FAR, 0.75, 1e-5
    v = {k: far_tensor(i, rows, C) for i, k in enumerate(("x", "h", "gate", "dr", "dy"))}
    post, pre = ((1 + randn(i, C, scale=0.2)).float().cuda() for i in (8, 9))
    got = {k: torch.full((rows, C), float("nan"), device="cuda", dtype=torch.bfloat16) for k in ("r", "y", "dx", "dh", "dgate")}
    dpost, dpre, need = torch.empty(C, device="cuda"), torch.empty(C, device="cuda"), 8 * C * 512 + 256
    b.cdp_k_residual_norm(BF16, p(v["x"]), p(v["h"]), p(v["gate"]), p(post), p(pre), p(got["r"]), p(got["y"]), scale, eps, rows, C)
    b.cdp_k_residual_norm_backward(BF16, 0, p(v["x"]), p(v["h"]), p(v["gate"]), p(post), p(pre), p(v["dr"]), p(v["dy"]), p(got["dx"]), p(got["dh"]), p(got["dgate"]), p(dpost),
                                   p(dpre), scale, eps, p(workspace(need)), need, rows, C)
    at = torch.tensor([0, 1, 262_143, 262_144, 524_287, 524_288, 524_289, rows - 2, rows - 1], device="cuda")
    args = [v[k][at].double() for k in ("x", "h", "gate")] + [post.double(), pre.double()] + [v[k][at].double() for k in ("dr", "dy")]
    res, size = norm_reference(*args, scale, float(np.float32(eps)))
    for k, x in got.items():
        near(x[at], res[k].cpu(), norm_tolerance(k, res, size, BF16, rows).cpu(), k)
        assert not any(bool(torch.isnan(x[i:i + 90_000]).any()) for i in range(0, rows, 90_000))
    assert bool(torch.isfinite(dpost).all()) and bool(torch.isfinite(dpre).all())


def test_packed_attention_past_4_gib():
    """600 sequences of 1000 tokens, 30 heads over one: rows of 8 KB."""
    n, S, H, K, W, scale = 1000, 600, 30, 1, 128, 0.1
    T = n * S + 3
    qkv, dout = far_tensor(1, T, (H + 2 * K) * W), far_tensor(2, T, H * W)
    offsets = torch.arange(S + 1, device="cuda", dtype=torch.int32) * n
    out, dqkv = (torch.full_like(v, float("nan")) for v in (dout, qkv))
    lse, need = torch.full((H, T), float("nan"), device="cuda"), 4 * H * T + 512
    b.cdp_k_attention_packed(BF16, 0, p(qkv), p(offsets), p(out), p(lse), 0, 0, 0, 0, T, S, H, K, W, scale)
    b.cdp_k_attention_packed(BF16, 1, p(qkv), p(offsets), p(out), p(lse), p(dout), p(dqkv), p(workspace(need)), need, T, S, H, K, W, scale)
    for s in (0, 261, 524, 525, S - 1):
        rows = slice(n * s, n * (s + 1))
        with torch.device("cuda"):
            x, scale32 = qkv[rows].double(), float(np.float32(scale))
            res, tol, _ = attention_reference(x, [0, n], H, K, W, scale32, BF16)
            back, back_tol, _ = attention_reference(x, [0, n], H, K, W, scale32, BF16, dout[rows].double(), out[rows].double(), lse[:, rows].double())
        for got, k in ((out[rows], "out"), (lse[:, rows], "lse")):
            near(got, res[k].cpu(), tol[k].cpu(), k)
        near(dqkv[rows], back["dqkv"].cpu(), back_tol["dqkv"].cpu(), "dqkv")
    assert all(bool(torch.isnan(v[n * S:]).all()) for v in (out, lse.T, dqkv))


def test_grad_clip_of_more_than_2_to_the_32_elements():
    """Ones: the norm is the root of their number, whichever are lost is seen."""
    n = (1 << 32) + 12345
    g = torch.ones(n, dtype=torch.bfloat16, device="cuda")
    g[-1] = 3.0
    norm = clip_call(BF16, [g], [g], 64.0)
    want = math.sqrt(n + 8)
    near(norm, torch.tensor([want], dtype=torch.float64), 2 * U * want, "norm")
    one = torch.tensor(64.0 / want, dtype=torch.float64)
    near(g[:1], one.reshape(1), (2.0 ** -8 + 4 * U) * one, "first")
    near(g[-1:], 3 * one.reshape(1), 3 * (2.0 ** -8 + 4 * U) * one, "last")
    assert all(bool((g[i:min(i + (1 << 28), n - 1)] == g[0]).all()) for i in range(0, n - 1, 1 << 28))


# ---- together -------------------------------------------------------------------------------------------------------------
def test_steps_that_overlap_on_two_streams():
    """Two training steps, each with workspaces of its own, under way at once, and one of them replayed from a graph beside the other's calls: the same bits."""
    steps, streams = (Step([30, 1, 64, 0, 33], 40), Step([500, 90, 7], 41)), (torch.cuda.Stream(), torch.cuda.Stream())
    want = []
    for s in steps:
        s.run()
        torch.cuda.synchronize()
        want.append([v.clone() for v in s.state()])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=streams[0]):
        steps[0].run(streams[0].cuda_stream)
    for replayed in (False, True):
        for s in steps:
            for v in s.state():
                v.fill_(float("nan"))
        torch.cuda.synchronize()
        for _ in range(10):
            for i, (s, stream) in enumerate(zip(steps, streams)):
                with torch.cuda.stream(stream):
                    if replayed and i == 0:
                        graph.replay()
                    else:
                        s.run(stream.cuda_stream)
        torch.cuda.synchronize()
        for s, values in zip(steps, want):
            assert all(torch.equal(got, v) for got, v in zip(s.state(), values))
