"""More operators of token models at the edges of what they are documented to take."""
import math

import pytest

from paper_2403_08837_amd import binding as b
from test_gpu_more_token_kernels import BF16, EPS, F32, TYPES, U, half, p, planes

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.fixture(autouse=True)
def memory_goes_back():
    """(Some of these take tens of gigabytes.)"""
    yield
    torch.cuda.empty_cache()


def same_bits(x, y):
    i = {2: torch.int16, 4: torch.int32}[x.element_size()]
    return torch.equal(x.contiguous().view(i), y.contiguous().view(i))


# ---- norms of heads and rotation --------------------------------------------------------------------------------------
#      width, rotary: lanes of 8, 4, 2 and 1 pairs; pairs beside each other that end within a lane; none
TAILS = [(128, 64), (128, 32), (40, 16), (80, 40), (16, 12), (24, 22), (128, 126), (64, 2), (48, 0)]


@pytest.mark.parametrize("gammas", ["", "q", "k"])
@pytest.mark.parametrize("inter", [0, 1])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("W,R", TAILS)
def test_values_outside_the_rotation_stay(W, R, dtype, inter, gammas):
    """Of heads without a gamma what is not rotated comes out as it is, bit for bit, whatever its neighbours are: infinities, zeros of either sign, subnormal numbers."""
    if not R and not gammas:
        return
    t, H, K, n = TYPES[dtype], 3, 2, 5
    g = torch.Generator()
    g.manual_seed(W + R)
    x, d = (torch.randn((n, H + 2 * K, W), generator=g) for _ in range(2))
    for v in (x, d):
        v[1, :, R] = math.inf
        v[2, :, W - 1] = -math.inf
        v[3, :, R:] = -0.0
        v[4, :, R:] = 0.25 * torch.finfo(t).smallest_normal * torch.sign(v[4, :, R:])
    x, d = x.to(t).cuda(), d.to(t).cuda()
    pos, freqs, gamma = torch.arange(1, n + 1).int().cuda(), torch.rand(max(1, R // 2), generator=g).cuda(), torch.ones(W).cuda()
    out, dx, dg = torch.empty_like(x), torch.empty_like(x), torch.empty((2, W), device="cuda")
    ws = torch.empty(8 * W * n + 256, dtype=torch.uint8, device="cuda")
    q, k = ("q" in gammas), ("k" in gammas)
    given = (p(x), p(pos), p(freqs), p(gamma) if q else 0, p(gamma) if k else 0)
    b.cdp_k_head_norm_rotary(dtype, *given, p(out), EPS, inter, n, H, K, W, R)
    b.cdp_k_head_norm_rotary_backward(dtype, 0, *given, p(d), p(dx), p(dg) if q else 0, p(dg[1]) if k else 0, EPS, inter, p(ws), ws.numel(), n, H, K, W, R)
    for name, heads in (("q", slice(0, H)), ("k", slice(H, H + K))):
        if name not in gammas:
            assert same_bits(out[:, heads, R:], x[:, heads, R:]), name
            assert same_bits(dx[:, heads, R:], d[:, heads, R:]), name
            for v in (out, dx):  # and reaches nothing that is rotated
                assert bool(torch.isfinite(v[:, heads, :R].float()).all())
    assert same_bits(out[:, H + K:], x[:, H + K:]) and same_bits(dx[:, H + K:], d[:, H + K:])


@pytest.mark.parametrize("inter", [0, 1])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
def test_what_is_not_finite_reaches_its_own_head_and_stays_there(dtype, bad, inter):
    """In x or in dout, of a normed head, of one without a gamma, of a v head (copied, bit for bit): every value of the head, the pair's two, that value.  A norm of an
    infinite head is its values times 0, NaN where they are infinite."""
    t, n, (H, K, W) = TYPES[dtype], 8, (3, 1, 40)
    g = torch.Generator()
    g.manual_seed(1)
    x, d = (torch.randn((n, H + 2 * K, W), generator=g) for _ in range(2))
    x[2, 1, 7] = x[3, 4, 5] = x[4, 3, 2] = bad
    d[5, 1, 7] = d[6, 4, 5] = d[7, 3, 2] = bad
    pair = [2, 3] if inter else [2, 22]
    pos, freqs, gamma = torch.arange(1, n + 1).int().cuda(), torch.rand(W // 2, generator=g).cuda(), torch.ones(W).cuda()
    x, d = x.to(t).cuda(), d.to(t).cuda()
    out, dx, dg = torch.empty_like(x), torch.empty_like(x), torch.empty(W, device="cuda")
    ws = torch.empty(8 * W * n + 256, dtype=torch.uint8, device="cuda")
    given = (p(x), p(pos), p(freqs), p(gamma), 0)
    b.cdp_k_head_norm_rotary(dtype, *given, p(out), EPS, inter, n, H, K, W, W)
    b.cdp_k_head_norm_rotary_backward(dtype, 0, *given, p(d), p(dx), p(dg), 0, EPS, inter, p(ws), ws.numel(), n, H, K, W, W)
    assert same_bits(out[:, H + K:], x[:, H + K:]) and same_bits(dx[:, H + K:], d[:, H + K:])
    fine, fine_d = (torch.isfinite(v.float().cpu()) for v in (out, dx))
    for f, normed, plain in ((fine, 2, 4), (fine_d, 5, 7)):
        assert not bool(f[normed, 1].all()) and not bool(f[plain, 3, pair].any())
        if math.isnan(bad) or f is fine_d:
            assert not bool(f[normed, 1].any())
        f[normed, 1], f[plain, 3, pair] = True, True
    assert not bool(fine_d[2, 1].any())  # the gradient of a head that was not finite
    fine_d[2, 1] = True
    fine[3, 4, 5], fine_d[6, 4, 5] = True, True
    assert bool(fine.all()) and bool(fine_d.all())
    assert not bool(torch.isfinite(dg.cpu()).all())


# ---- linear maps of many rows -----------------------------------------------------------------------------------------
def fill(x, seed, scale=1.0):
    """Normal numbers, a piece at a time."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    for v in x.split(max(1, (1 << 27) // x.shape[1])):
        v.copy_(scale * torch.randn(v.shape, generator=g, device="cuda"))
    return x


def ends(n, m=40):
    return torch.cat([torch.arange(min(n, m)), torch.arange(max(0, n - m), n)]).unique().cuda()


def far(got, want, tol, what):
    worst = float(((got.double() - want).abs() / tol).max())
    assert got.shape == want.shape and worst <= 1, (what, worst)


def product(v, o, n, dtype):
    """v @ o with what its roundings come to: a result of n terms, and its own."""
    want = v @ o
    return want, half(dtype) * want.abs() + ((2 * n + 8) * U + planes(dtype)) * (v.abs() @ o.abs())


def test_linear_of_more_rows_than_small_tiles_can_be_launched_for():
    """2^29 rows and a few: rows at either end, and a gradient of the weights that only the last rows have."""
    R, I, O, n, t = (1 << 29) + 3, 8, 16, 300, torch.bfloat16
    empty = lambda *s: torch.empty(s, dtype=t, device="cuda")  # noqa: E731
    x, w, bias, y = fill(empty(R, I), 1), fill(empty(O, I), 2), fill(empty(1, O), 3), empty(R, O).fill_(math.nan)
    b.cdp_k_linear(BF16, 3, p(x), p(w), p(bias), 0, p(y), 0, 0, 0, R, I, O)
    rows = ends(R, 1000)
    want, tol = product(x[rows].double(), w.double().t(), I + 1, BF16)
    far(y[rows], want + bias.double(), tol + (half(BF16) + 20 * U) * bias.double().abs(), "y")
    dy = y.zero_()
    fill(dy[-n:], 4)
    dx, dw, db = empty(R, I).fill_(math.nan), empty(O, I).fill_(math.nan), empty(O).fill_(math.nan)
    ws = torch.empty(2 * R * O + 4 * O * 256 + 1024 + (1 << 20), dtype=torch.uint8, device="cuda")
    b.cdp_k_linear_backward(BF16, 3, p(x), p(w), 0, p(dy), p(dx), p(dw), p(db), p(ws), ws.numel(), R, I, O)
    far(dx[-n:], *product(dy[-n:].double(), w.double(), O, BF16), "dx")
    assert bool((dx[rows][:1000] == 0).all())
    far(dw, *product(dy[-n:].double().t(), x[-n:].double(), n, BF16), "dw")
    d = dy[-n:].double()
    far(db, d.sum(0), half(BF16) * d.sum(0).abs() + n * U * d.abs().sum(0), "dbias")


# rows, inputs, outputs: more than 2^31 elements of x, of w and dw, of y and dy
MANY = [(1050000, 2056, 64), (40, 2056, 1048576), (4, 2056, 1048576), (1050000, 16, 2056)]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("R,I,O", MANY)
def test_linear_gradients_from_behind_2_to_31_elements(R, I, O, dtype):
    """dy is zero but for its last rows, or columns, whose x, or weights, lie behind 2^31 elements: what of them is lost or read elsewhere is all of the result."""
    t, n = TYPES[dtype], 300
    empty = lambda *s: torch.empty(s, dtype=t, device="cuda")  # noqa: E731
    rows, cols = min(n, R), O if R > O else n  # where dy is not zero: its last so many
    x, w, dy = fill(empty(R, I), 1), fill(empty(O, I), 2, I ** -0.5), empty(R, O).zero_()
    d = torch.randn((rows, cols), generator=torch.Generator("cuda").manual_seed(3), device="cuda").to(t)
    dy[R - rows:, O - cols:] = d
    assert max((R - rows) * I if R > O else 0, (O - cols) * I if O > R else 0, (R - rows) * O if R > O else 0) > 2 ** 31
    dx, dw, db = empty(R, I).fill_(math.nan), empty(O, I).fill_(math.nan), empty(O).fill_(math.nan)
    ws = torch.empty((4 if dtype == F32 else 2) * R * O + 4 * O * min(R, 256) + 1024 + (64 << 20), dtype=torch.uint8, device="cuda")
    b.cdp_k_linear_backward(dtype, 3, p(x), p(w), 0, p(dy), p(dx), p(dw), p(db), p(ws), ws.numel(), R, I, O)
    d = d.double()
    far(dx[R - rows:], *product(d, w[O - cols:].double(), cols, dtype), "dx")
    far(dw[O - cols:], *product(d.t(), x[R - rows:].double(), rows, dtype), "dw")
    far(db[O - cols:], d.sum(0), half(dtype) * d.sum(0).abs() + (rows + 40) * U * d.abs().sum(0), "dbias")
    for v, kept in ((dx, R - rows), (dw, O - cols), (db, O - cols)):  # and zeros elsewhere
        for part in v[:kept].split(1 << 18):
            assert not bool(part.any())


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_gated_gradients_from_behind_2_to_31_elements(dtype):
    """The same of gated maps: dh behind 2^31 elements alone is not zero."""
    t, n, (R, I, H) = TYPES[dtype], 300, (1050000, 16, 2056)
    empty = lambda *s: torch.empty(s, dtype=t, device="cuda")  # noqa: E731
    x, wg, wu = fill(empty(R, I), 1), fill(empty(H, I), 2, I ** -0.5), fill(empty(H, I), 3, I ** -0.5)
    h, g, u = (empty(R, H).fill_(math.nan) for _ in range(3))
    b.cdp_k_gated_linear(dtype, 3, p(x), p(wg), p(wu), p(h), p(g), p(u), 0, 0, R, I, H)
    rows = ends(R, 1000)
    for v, w in ((g, wg), (u, wu)):
        far(v[rows], *product(x[rows].double(), w.double().t(), I, dtype), "g, u")
    dh = h.zero_()
    fill(dh[-n:], 4)
    dx, dwg, dwu = empty(R, I).fill_(math.nan), empty(H, I).fill_(math.nan), empty(H, I).fill_(math.nan)
    ws = torch.empty(2 * dh.element_size() * R * H + 1024 + (64 << 20), dtype=torch.uint8, device="cuda")
    b.cdp_k_gated_linear_backward(dtype, 3, p(x), p(wg), p(wu), p(g), p(u), p(dh), p(dx), p(dwg), p(dwu), p(ws), ws.numel(), R, I, H)
    gd, ud, d, xd = (v[-n:].double() for v in (g, u, dh, x))
    dg, du = d * ud, d * gd
    step = half(dtype) + 2 * U  # dg and du are rounded to the element type
    want = dg @ wg.double() + du @ wu.double()
    size = dg.abs() @ wg.double().abs() + du.abs() @ wu.double().abs()
    far(dx[-n:], want, half(dtype) * want.abs() + (step + (4 * H + 8) * U + planes(dtype)) * (1 + step) * size, "dx")
    for got, v, what in ((dwg, dg, "dwg"), (dwu, du, "dwu")):
        want, size = v.t() @ xd, v.t().abs() @ xd.abs()
        far(got, want, half(dtype) * want.abs() + (step + (2 * n + 8) * U + planes(dtype)) * (1 + step) * size, what)
    for part in dx[:R - n].split(1 << 18):
        assert not bool(part.any())


# ---- small and large fp32 values --------------------------------------------------------------------------------------
@pytest.mark.parametrize("R,I,O", [(5, 72, 136), (16, 200, 264), (40, 520, 136), (70, 264, 136), (300, 328, 520), (1030, 1032, 1544)])
@pytest.mark.parametrize("small", ["x", "w"])
@pytest.mark.parametrize("power", [100, 115, 125, 130])
def test_linear_of_small_fp32_values(power, small, R, I, O):
    """One factor of about 2^-power, the other of 2^power (2^125 at most): of a factor 2^-27 of itself and what is below 2^-133 may be left out, of a product 2^-26."""
    up = min(power, 125)

    def rand(seed, *shape, p):
        return torch.ldexp(torch.randn(shape, generator=torch.Generator("cuda").manual_seed(seed), device="cuda"), torch.tensor(p, device="cuda"))
    less, more = rand(1, R, I, p=-power), rand(2, O, I, p=up)
    if small == "w":
        less, more = rand(1, O, I, p=-power), rand(2, R, I, p=up)
    x, w = (less, more) if small == "x" else (more, less)
    dy = {k: rand(3, R, O, p=v) for k, v in (("dx", -power if small == "x" else up), ("dw", up if small == "x" else -power))}
    y, dx, dw = torch.empty((R, O), device="cuda"), torch.empty((R, I), device="cuda"), torch.empty((O, I), device="cuda")
    ws = torch.empty(4 * R * O + 4 * O * min(R, 256) + 1024 + (4 << 20), dtype=torch.uint8, device="cuda")
    b.cdp_k_linear(F32, 3, p(x), p(w), 0, 0, p(y), 0, 0, 0, R, I, O)
    b.cdp_k_linear_backward(F32, 3, 0, p(w), 0, p(dy["dx"]), p(dx), 0, 0, p(ws), ws.numel(), R, I, O)
    b.cdp_k_linear_backward(F32, 3, p(x), 0, 0, p(dy["dw"]), 0, p(dw), 0, p(ws), ws.numel(), R, I, O)
    x, w, dy = x.double(), w.double(), {k: v.double() for k, v in dy.items()}
    for got, v, o, n, what in ((y, x, w.t(), I, "y"), (dx, dy["dx"], w, O, "dx"), (dw, dy["dw"].t(), x, R, "dw")):
        want, tol = product(v, o, n, F32)
        far(got, want, tol + 2.0 ** -133 * (v.abs().sum(1)[:, None] + o.abs().sum(0)), what)


# ---- log probabilities ------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("shared", [0, 1 << 20])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_logprob_of_logits_whose_difference_overflows(dtype, shared):
    """Logits of +-2e38 with a scale of 1/2: |z| is within fp32, and so are the log probabilities, up to -2e38 (their rounding: that of scale * logit, and one step)."""
    t, V, top, scale = TYPES[dtype], 20011, 3, 0.5
    x = torch.full((4, V), -2e38, dtype=torch.float64)
    x[0, 5] = 2e38
    x[1, [7, 9000]] = 2e38
    x[2, 1] = 1e38
    x[2, 2] = -3e38
    x[3] = 2e38
    x[3, 11] = -1.5e38
    x = x.to(t)
    targets = torch.tensor([6, 8, 2, 11], dtype=torch.int32)
    xd, td = x.cuda(), targets.cuda()
    lp, en, lse, best = (torch.empty(s, device="cuda") for s in (4, 4, 4, (4, top)))
    ids, dx, ones, ws = torch.empty((4, top), dtype=torch.int32, device="cuda"), torch.empty_like(xd), torch.ones(4, device="cuda"), torch.empty(1 << 20, dtype=torch.uint8, device="cuda")
    b.cdp_k_token_logprob(dtype, p(xd), V, p(td), scale, p(lp), p(en), p(lse), p(ids), p(best), top, p(ws) if shared else 0, shared, 4, V)
    b.cdp_k_token_logprob_backward(dtype, p(xd), V, p(td), scale, p(lse), p(en), p(ones), p(ones), p(dx), 4, V)
    z = scale * x.double()
    z = z - z.amax(1, keepdim=True)  # (64 bits of 1e38 have no room for the logarithm beside it)
    logp = z - torch.log(torch.exp(z).sum(1, keepdim=True))
    want = logp.gather(1, targets.long()[:, None])[:, 0]
    assert bool(torch.isfinite(lp).all())
    far(lp.cpu(), want, 4 * U * want.abs(), "logprob")
    order = torch.sort(x, dim=1, descending=True, stable=True).indices[:, :top]
    assert torch.equal(ids.cpu().long(), order)
    wanted = logp.gather(1, order)
    far(best.cpu(), wanted, 4 * U * wanted.abs() + 40 * U, "top")
    entropy = torch.tensor([0.0, math.log(2), 0.0, math.log(V - 1)], dtype=torch.float64)
    far(en.cpu(), entropy, U * (V / 64 + 200) * torch.ones(4, dtype=torch.float64), "entropy")
    assert bool(torch.isfinite(dx.float()).all())


@pytest.mark.parametrize("scale", [1e-30, 1e-20, 1e30, 1e38])
def test_logprob_of_any_scale(scale):
    """The same z of logits that are that much larger or smaller."""
    V = 3001
    s = torch.tensor(scale).double()
    x = (3 * torch.randn((3, V), generator=torch.Generator().manual_seed(1), dtype=torch.float64) / s).clamp(-3e38, 3e38).float()
    targets = torch.tensor([0, 7, V - 1], dtype=torch.int32)
    xd, td = x.cuda(), targets.cuda()
    lp, en, lse = (torch.empty(3, device="cuda") for _ in range(3))
    b.cdp_k_token_logprob(F32, p(xd), V, p(td), scale, p(lp), p(en), p(lse), 0, 0, 0, 0, 0, 3, V)
    z = s * x.double()
    want = torch.log_softmax(z, 1)
    tol = U * (V / 64 + 200) * torch.ones(3, dtype=torch.float64)
    far(lp.cpu(), want.gather(1, targets.long()[:, None])[:, 0], tol, "logprob")
    far(lse.cpu(), torch.logsumexp(z, 1), tol, "lse")
    far(en.cpu(), -(want.exp() * want).sum(1), 8 * tol, "entropy")


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("R,C,V,top", [(1, 64, 50257, 5), (37, 64, 50, 3), (300, 128, 1001, 0)])
def test_a_vocabulary_of_no_multiple_of_8(R, C, V, top, dtype):
    """The projection with weights padded by rows of zeros, log probabilities of the vocabulary alone, and both gradients: nothing comes from the padding, and nothing goes to it."""
    t, P = TYPES[dtype], -(-V // 8) * 8
    g = torch.Generator().manual_seed(V)
    x, w = torch.randn((R, C), generator=g).to(t).cuda(), torch.zeros((P, C), dtype=t, device="cuda")
    w[:V] = torch.randn((V, C), generator=g).to(t).cuda() * C ** -0.5
    targets = torch.randint(V, (R,), generator=g, dtype=torch.int32).cuda()
    logits, dlogits = torch.empty((R, P), dtype=t, device="cuda"), torch.zeros((R, P), dtype=t, device="cuda")
    lp, lse, ones = torch.empty(R, device="cuda"), torch.empty(R, device="cuda"), torch.ones(R, device="cuda")
    ids, best = torch.empty((R, max(1, top)), dtype=torch.int32, device="cuda"), torch.empty((R, max(1, top)), device="cuda")
    dx, dw, ws = torch.empty_like(x), torch.empty_like(w), torch.empty(1 << 26, dtype=torch.uint8, device="cuda")
    b.cdp_k_linear(dtype, 3, p(x), p(w), 0, 0, p(logits), 0, p(ws), ws.numel(), R, C, P)
    b.cdp_k_token_logprob(dtype, p(logits), P, p(targets), 1.0, p(lp), 0, p(lse), p(ids) if top else 0, p(best) if top else 0, top, p(ws), ws.numel(), R, V)
    b.cdp_k_token_logprob_backward(dtype, p(logits), P, p(targets), 1.0, p(lse), 0, p(ones), 0, p(dlogits), R, V)
    b.cdp_k_linear_backward(dtype, 3, p(x), p(w), 0, p(dlogits), p(dx), p(dw), 0, p(ws), ws.numel(), R, C, P)
    far(logits[:, :V], *product(x.double(), w[:V].double().t(), C, dtype), "logits")
    z = logits[:, :V].double()
    logp = torch.log_softmax(z, 1)
    far(lp, logp.gather(1, targets.long()[:, None])[:, 0], U * (V / 64 + 200) * torch.ones(R, dtype=torch.float64, device="cuda"), "logprob")
    if top:
        assert torch.equal(ids.long(), torch.sort(z, dim=1, descending=True, stable=True).indices[:, :top])
    want = torch.zeros_like(z).scatter_(1, targets.long()[:, None], 1.0) - logp.exp()
    # (probabilities by lse's rounding, sums of V terms in it, and a product's and a difference's)
    far(dlogits[:, :V], want, half(dtype) * want.abs() + (U * (V / 64 + 200) + 2.0 ** -22 * 20) * logp.exp() + 2 * U, "dlogits")
    assert not bool(dlogits[:, V:].any()) and not bool(dw[V:].any())
    d = dlogits.double()
    far(dx, *product(d, w.double(), P, dtype), "dx")
    far(dw[:V], *product(d[:, :V].t(), x.double(), R, dtype), "dw")


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_alternatives_of_rows_whose_large_logits_are_a_few_lanes(dtype):
    """A quarter of a long row, what 64 lanes of a workgroup read, is large and ascending: nearly all of it is above the first border.  The time stays that of reading a few times (it had gone by the
    square of the row: 60 and 100 times a random one's here)."""
    t, V, top = TYPES[dtype], 1 << 24, 64
    j = torch.arange(V, device="cuda")
    x = torch.randn((2, V), generator=torch.Generator("cuda").manual_seed(1), device="cuda")
    x[1] = torch.where((j * x.to(t).element_size() // 16) % 256 < 64, 1000 + j / 64, x[1])
    x = x.to(t)
    lse, ids, best = torch.empty(1, device="cuda"), torch.empty((1, top), dtype=torch.int32, device="cuda"), torch.empty((1, top), device="cuda")
    us = []
    for row in x:
        events = [torch.cuda.Event(enable_timing=True) for _ in range(2)]
        for _ in range(2):
            events[0].record()
            b.cdp_k_token_logprob(dtype, p(row), V, 0, 1.0, 0, 0, p(lse), p(ids), p(best), top, 0, 0, 1, V)
            events[1].record()
        torch.cuda.synchronize()
        us.append(events[0].elapsed_time(events[1]) * 1e3)
        assert torch.equal(ids[0].long(), torch.sort(row, descending=True, stable=True).indices[:top])
    assert us[1] < 20 * us[0], us
