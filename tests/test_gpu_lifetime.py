"""What a handle or a model gives back to its owner is no longer in use: freeing a clip handle
waits for the calls that still use its buffers, on whichever stream these run."""
import pytest
import torch

from paper_1704_04560_amd import mtx

pytestmark = pytest.mark.gpu

N = 70_001


def _busy(stream):
    """Work that keeps a stream from finishing while the host goes on."""
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        torch.cuda._sleep(200_000_000)


def _grad():
    return torch.ones(N, device="cuda")


def test_free_waits_for_the_handles_last_stream():
    a, out = _grad(), torch.zeros(N, device="cuda")
    tensors = mtx.make_tensor_list([(a, out)])
    ws = torch.empty(mtx.mtx_clip_sizes(tensors), dtype=torch.uint8, device="cuda")
    handle = mtx.mtx_init_clip(tensors, ws)
    s = torch.cuda.Stream()
    _busy(s)
    mtx.mtx_clip_grads(handle, 1.0, None, stream=s)
    assert not s.query()
    mtx.mtx_free_clip(handle)
    assert s.query()
    assert torch.equal(out, out[:1].expand(N)) and abs(out[0].item() * N ** 0.5 - 1) < 1e-6


def test_a_dropped_clip_leaves_its_workspace_unused():
    a, out = _grad(), torch.zeros(N, device="cuda")
    clip = mtx.Clip([(a, out)])
    s = torch.cuda.Stream()
    _busy(s)
    clip.clip(1.0, stream=s)
    size = clip.workspace.numel()
    del clip
    assert s.query()
    other = torch.full((size,), 255, dtype=torch.uint8, device="cuda")   # may take its place
    torch.cuda.synchronize()
    assert torch.equal(out, out[:1].expand(N)) and other.all()


def test_free_inside_a_capture_leaves_it_alone():
    """A handle whose last call is being captured: nothing of it runs, and nothing is waited for."""
    a, out = _grad(), torch.zeros(N, device="cuda")
    tensors = mtx.make_tensor_list([(a, out)])
    ws = torch.empty(mtx.mtx_clip_sizes(tensors), dtype=torch.uint8, device="cuda")
    handle = mtx.mtx_init_clip(tensors, ws)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        mtx.mtx_clip_grads(handle, 1.0)
        mtx.mtx_free_clip(handle)
    for k in range(3):   # the graph needs the workspace and the tensors, not the handle
        a.fill_(k + 1.0)
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, out[:1].expand(N)) and abs(out[0].item() * N ** 0.5 - 1) < 1e-6
