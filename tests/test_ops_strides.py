"""Operands over the rows of one matrix are refused on the host where they share an element (these
calls need no device; the addresses are never read)."""
import pytest

from paper_1704_04560_amd import mtx
from tests.test_ops_refusals import A, Buf, F, code, desc

N, D = 12, 8


@pytest.mark.parametrize("ld,off", [(16, 7), (16, 9), (16, 16 * 11 + 7), (24, 24 * 5 - 7), (8, 16),
                                    (17, 17 * 12 - 10), (16, -7), (40, 40 * 3 + 4)])
def test_columns_that_share_an_element(ld, off):
    h, y = A[0] + 4096, A[0] + 4096 + 4 * off
    assert code(mtx.mtx_block_norm_forward, desc(rows=N, D=D, ld=(ld, ld, ld)), h, A[1], A[2], y,
                None) == mtx.MTX_EINVAL
    assert code(mtx.mtx_block_norm_backward, desc(rows=N, D=D, ld=(ld, ld, ld)), 1, h, A[1], A[2],
                A[3], A[4], y, A[5], None, None, None, None, None, D, Buf(A[7])) == mtx.MTX_EINVAL


@pytest.mark.parametrize("ldh,ldy,off", [(16, 24, 8), (24, 16, 12), (1 << 20, 24, (1 << 20) * 11 + 2),
                                         (16, 17, 8), (100, 101, 85)])
def test_rows_of_unequal_strides_that_meet(ldh, ldy, off):
    """Some row of one reaches into a row of the other, if only far from where they begin."""
    rows_h = [set(range(i * ldh, i * ldh + D)) for i in range(N)]
    assert any(r & set(range(off + j * ldy, off + j * ldy + D)) for r in rows_h for j in range(N))
    assert code(mtx.mtx_block_norm_forward, desc(rows=N, D=D, ld=(ldh, 0, ldy)), A[0], A[1], A[2],
                A[0] + 4 * off, None) == mtx.MTX_EINVAL


def test_embedding_and_average_between_rows():
    w, tok, y = A[0], A[1], A[2]
    for bad in (y + 4 * 31, y - 4, y + 4 * 79):   # rows of 8 columns, 24 apart
        assert code(mtx.mtx_embed_forward, w, F, 10, 8, bad, 4, -1, 1.0, y, F, 24) == mtx.MTX_EINVAL
    for avg in (9, 21, 31):   # rows of 10, 22 apart, and the average's 10
        assert code(mtx.mtx_average_clip, A[3], 3, 10, 22, 1.0, A[3] + 4 * avg, None,
                    Buf(A[5])) == mtx.MTX_EINVAL
    assert code(mtx.mtx_average_clip, A[3], 3, 10, 22, 1.0, A[4], A[3] + 4 * 53,
                Buf(A[5])) == mtx.MTX_EINVAL
