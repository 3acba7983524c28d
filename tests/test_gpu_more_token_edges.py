"""More operators of token models at the edges of what they are documented to take."""
import math

import pytest

from paper_2403_08837_amd import binding as b
from test_gpu_more_token_kernels import BF16, EPS, F32, TYPES, p

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
