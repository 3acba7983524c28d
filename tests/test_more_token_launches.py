"""Linear maps of tokens: what the header allows has a launch.  Pointers are made up, and without a GPU nothing is launched: a call whose launch was laid out ends with CDP_EHIP, one for which
there is none with CDP_EINVAL."""
import pytest
import torch

from paper_2403_08837_amd import binding as b

pytestmark = pytest.mark.skipif(torch.cuda.device_count() > 0, reason="made-up pointers: without a GPU only")

P, F32, BF16 = 4096, 0, 1
CDP_EHIP = -4


def code(name, *args):
    with pytest.raises(b.CdpError) as e:
        getattr(b, name)(*args)
    return e.value.code


# (results of up to 2^32 elements, which memory holds)
LONG = [(1 << 28, 8), (1 << 28, 16), (1 << 29, 8), (1 << 30, 8)]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,width", LONG + [(100, 8), (1 << 22, 1024), (4096, 1 << 20), (65, 1 << 20), (16, 1 << 20)])
def test_sizes_that_memory_holds_are_launched(rows, width, dtype):
    e, inputs = (4 if dtype == F32 else 2), 8
    for room in (0, 1 << 30):
        assert code("cdp_k_linear", dtype, 1, P, P, P, P, P, P, P if room else 0, room, rows, inputs, width) == CDP_EHIP
        assert code("cdp_k_gated_linear", dtype, 0, P, P, P, P, P, P, P if room else 0, room, rows, inputs, width) == CDP_EHIP
        need = e * rows * width + 4 * width * min(rows, 256) + 1024
        for dx, dw, db in ((P, P, P), (P, 0, 0), (0, P, 0), (0, 0, P)):
            assert code("cdp_k_linear_backward", dtype, 1, P, P, P, P, dx, dw, db, P, need + room, rows, inputs, width) == CDP_EHIP
        for dx, dw in ((P, P), (P, 0), (0, P)):
            assert code("cdp_k_gated_linear_backward", dtype, 0, P, P, P, P, P, P, dx, dw, dw, P, 2 * e * rows * width + 1024 + room, rows, inputs, width) == CDP_EHIP


@pytest.mark.parametrize("rows,inputs,hidden", [(1 << 28, 8, 72), (1 << 29, 8, 72), (1 << 28, 72, 8), (1 << 24, 1024, 2048)])
def test_sizes_of_several_tiles_a_row_are_launched(rows, inputs, hidden):
    for dtype in (F32, BF16):
        assert code("cdp_k_gated_linear", dtype, 0, P, P, P, P, 0, 0, 0, 0, rows, inputs, hidden) == CDP_EHIP
        assert code("cdp_k_linear", dtype, 3, P, P, 0, 0, P, 0, 0, 0, rows, inputs, hidden) == CDP_EHIP


def test_launches_of_too_many_threads_are_refused():
    """2^30 rows of 2^20 results have none."""
    for dtype in (F32, BF16):
        assert code("cdp_k_linear", dtype, 3, P, P, 0, 0, P, 0, 0, 0, 1 << 30, 8, 1 << 20) == b.CDP_EINVAL
        assert code("cdp_k_gated_linear", dtype, 0, P, P, P, P, 0, 0, 0, 0, 1 << 30, 8, 1 << 20) == b.CDP_EINVAL
        assert code("cdp_k_linear_backward", dtype, 3, P, P, 0, P, P, P, 0, P, 1 << 60, 1 << 30, 1 << 20, 1 << 20) == b.CDP_EINVAL
