"""The embedding gradient where its launches come to the limit of 2^32 threads."""
import pytest
import torch

from paper_1704_04560_amd import mtx
from tests.ops_ref import BF16

pytestmark = pytest.mark.gpu


def test_many_shards_of_wide_rows():
    """65536 shards of one token and 65536 values: 2^23 blocks of 512 threads.  Small whole numbers, so
    the gradients are exact; every seventh token lies outside the table."""
    R, D = 65536, 65536
    print(f"[case] embed_bwd R={R} n=1 V=1 D={D} bf16", flush=True)
    r, d = torch.arange(R, device="cuda"), torch.arange(D, device="cuda")
    dy = (d % 251).to(BF16).expand(R, D).contiguous()
    dy += (r % 5).to(BF16)[:, None]
    tok = torch.where(r % 7 == 3, 1, 0).to(torch.int32)
    grads = torch.full((R, D), 9.0, device="cuda")
    ws = torch.empty(mtx.mtx_embed_sizes(1, R, 1, D), dtype=torch.uint8, device="cuda")
    mtx.mtx_embed_backward(tok, 1, R, dy, mtx.MTX_BF16, D, 1, D, -1, 2.0, grads, D, False, ws)
    for a in range(0, R, 8192):
        s = slice(a, a + 8192)
        want = torch.where((tok[s] == 0)[:, None], 2.0 * dy[s].float(), 0.0)
        assert torch.equal(grads[s], want), a
