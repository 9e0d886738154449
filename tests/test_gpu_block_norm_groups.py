"""Block norm gradients where one block adds several whole gate groups, at every number of threads
that hold a row: the checks of the other shapes, and that the shapes reach that form."""
import pytest

from paper_1704_04560_amd import mtx
from tests import test_gpu_block_norm as base
from tests.ops_ref import BF16, F32

pytestmark = pytest.mark.gpu

# rows, D, shards, rows of a gate, extra strides, offset (1: rows that are not 16-byte aligned)
DIMS = [(2400, 120, 2, 2, 0, 0), (2100, 300, 1, 1, 0, 0), (2400, 512, 2, 2, 0, 0),
        (1500, 1000, 3, 1, 8, 0), (1100, 2000, 2, 1, 0, 0), (1100, 2056, 1, 1, 0, 0), (1200, 4096, 2, 2, 0, 0),
        (1100, 8192, 1, 1, 0, 0), (600, 16384, 1, 1, 0, 0),
        (2100, 33, 1, 1, 1, 1), (2100, 150, 3, 2, 0, 1), (2100, 771, 1, 1, 5, 1),
        (2200, 1021, 2, 1, 3, 1), (1100, 3001, 1, 2, 0, 1), (1100, 5003, 1, 1, 1, 1),
        (600, 9001, 1, 1, 0, 1), (2100, 101, 1, 1, 0, 1), (2100, 390, 2, 1, 1, 1),
        (1100, 1501, 1, 1, 0, 1)]
FORMS = [(False, True), (True, True), (True, False)]   # layer norm, post norm


def _blocks(desc, D, R):
    """Blocks of a backward launch (of its aligned or its unaligned form, whichever has more): each
    keeps five rows of partial sums, D rounded up to a multiple of 4."""
    return mtx.mtx_block_norm_sizes(desc, R) // (5 * 4 * ((D + 3) // 4 * 4))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("layer,post", FORMS)
@pytest.mark.parametrize("N,D,R,group,extra,off", DIMS)
def test_blocks_of_several_groups(N, D, R, group, extra, off, layer, post, dtype):
    kind = mtx.MTX_NORM_LAYER if layer else mtx.MTX_NORM_RMS
    d = mtx.make_norm_desc(kind, base.MT[dtype], N, D, 1e-5, 0.75, group, 1 << 33 if post else None, None,
                           1 << 34, 1 << 35, None, D + extra, D + extra, D + extra)
    assert _blocks(d, D, R) < N // group, "one block to a group"
    base.test_forward_and_backward(N, D, R, group, extra, off, layer, post, True, True, dtype)
