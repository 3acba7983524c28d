"""More operators of token models at the edges of what they are documented to take."""
import math

import pytest

from paper_2403_08837_amd import binding as b
from test_gpu_more_token_kernels import BF16, EPS, F32, TYPES, U, half, p, planes

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


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
