"""A Clip keeps its list on the tensors' GPU: tensors in host memory are refused before anything is
made of them (no device is needed)."""
import pytest
import torch

from paper_1704_04560_amd import mtx


@pytest.mark.parametrize("pairs", [
    [(torch.zeros(8), None)], [(torch.zeros(8), torch.zeros(8))],
    [(torch.zeros(8, device="meta"), None)],
    [(torch.zeros(8), None), (torch.zeros(3, device="meta"), None)]])
def test_tensors_in_host_memory(pairs):
    with pytest.raises(ValueError):
        mtx.Clip(pairs)


def test_an_empty_list():
    with pytest.raises(mtx.MtxError) as e:
        mtx.Clip([])
    assert e.value.code == mtx.MTX_EINVAL
