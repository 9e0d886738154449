"""What a handle or a model gives back to its owner is no longer in use: freeing a clip handle,
changing the clip option's buffers or the update rule's state waits for the calls that still use
them, on whichever stream these run."""
import pytest
import torch

from paper_1704_04560_amd import mtx
from paper_1704_04560_amd import workloads as wl

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


def _model():
    net = wl.MLP
    m = mtx.Model(net.in_shape, wl.layer_tuples(net), net.dtype, 2, 4, seed=1)
    x, y = (torch.from_numpy(t).cuda() for t in wl.make_batch(net, 8, seed=2))
    return m, x, y


def test_clip_option_waits_for_steps_with_the_old_buffers():
    m, x, y = _model()
    nrm = torch.zeros(1, device="cuda")
    s = torch.cuda.Stream()
    for last in (dict(max_norm=0), dict(max_norm=0.5, norm_out=torch.zeros(1, device="cuda"))):
        m.set_clip_norm(0.1, nrm)
        held = m._clip   # (keeps them while the wait is tested)
        _busy(s)
        m.train_step(x, y, 0.01, 0.9, stream=s)
        assert not s.query()
        m.set_clip_norm(**last)
        assert s.query(), last
        assert held[0].item() > 0.1
        m.set_clip_norm(0)
    m.close()


def test_another_bound_over_the_same_buffers_does_not_wait():
    m, x, y = _model()
    nrm = torch.zeros(1, device="cuda")
    s = torch.cuda.Stream()
    m.set_clip_norm(0.1, nrm)
    _busy(s)
    m.train_step(x, y, 0.0, 0.0, stream=s)
    m.set_clip_norm(0.2, nrm)
    m.train_step(x, y, 0.0, 0.0, stream=s)
    assert not s.query()
    torch.cuda.synchronize()
    assert abs(float(m.grad_avg.double().norm()) - 0.2) <= 1e-6
    m.close()


def test_update_rule_waits_for_steps_with_the_old_state():
    m, x, y = _model()
    s = torch.cuda.Stream()
    m.set_optimizer(mtx.MTX_OPT_ADAM)
    held = m.s2
    _busy(s)
    m.train_step(x, y, 0.001, 0.0, stream=s)
    assert not s.query()
    m.set_optimizer(mtx.MTX_OPT_MOMENTUM)
    assert s.query()
    assert held.any()
    m.close()


def test_a_refused_update_rule_keeps_the_present_state():
    m, x, y = _model()
    m.set_optimizer(mtx.MTX_OPT_ADAM)
    held = m.s2
    with pytest.raises(mtx.MtxError):
        m.set_optimizer(mtx.MTX_OPT_ADAM, beta1=2.0)
    assert m.s2 is held
    m.train_step(x, y, 0.001, 0.0)
    torch.cuda.synchronize()
    assert held.any()
    m.close()


def test_a_handle_made_inside_a_capture_is_refused():
    """... and the capture goes on."""
    a, out = _grad(), torch.zeros(N, device="cuda")
    other = _grad()
    b = mtx.make_tensor_list([(other, None)])
    ws = torch.empty(mtx.mtx_clip_sizes(b), dtype=torch.uint8, device="cuda")
    clip = mtx.Clip([(a, out)])
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        with pytest.raises(mtx.MtxError) as e:
            mtx.mtx_init_clip(b, ws)
        clip.clip(1.0)
    assert e.value.code == mtx.MTX_EINVAL
    for k in range(3):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, out[:1].expand(N)) and abs(out[0].item() * N ** 0.5 - 1) < 1e-6


@pytest.mark.parametrize("own_stream", [False, True])
@pytest.mark.parametrize("busy", [False, True])
def test_a_clip_dropped_while_another_stream_is_captured(own_stream, busy):
    """... waits for its own call and leaves the capture alone."""
    a, out = _grad(), torch.zeros(N, device="cuda")
    b, out_b = _grad(), torch.zeros(N, device="cuda")
    clip, other = mtx.Clip([(a, out)]), mtx.Clip([(b, out_b)])
    s = torch.cuda.Stream() if own_stream else torch.cuda.default_stream()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    if not busy:
        other.clip(1.0, stream=s)
    with torch.cuda.graph(graph):
        clip.clip(1.0)
        if busy:
            with torch.cuda.stream(s):
                torch.cuda._sleep(200_000_000)
            other.clip(1.0, stream=s)
        del other
    assert s.query()
    for k in range(3):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for t in (out, out_b):
            assert torch.equal(t, t[:1].expand(N)) and abs(t[0].item() * N ** 0.5 - 1) < 1e-6


def test_a_captured_call_does_not_hide_an_earlier_one():
    """Work on one stream, then a call captured on another: the free waits for the work."""
    a, out = _grad(), torch.zeros(N, device="cuda")
    tensors = mtx.make_tensor_list([(a, out)])
    ws = torch.empty(mtx.mtx_clip_sizes(tensors), dtype=torch.uint8, device="cuda")
    handle = mtx.mtx_init_clip(tensors, ws)
    s = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        with torch.cuda.stream(s):
            torch.cuda._sleep(200_000_000)
        mtx.mtx_clip_grads(handle, 1.0, stream=s)
        mtx.mtx_clip_grads(handle, 1.0)
    mtx.mtx_free_clip(handle)
    assert s.query()
    assert torch.equal(out, out[:1].expand(N)) and abs(out[0].item() * N ** 0.5 - 1) < 1e-6


@pytest.mark.parametrize("what", ["clip", "rule", "free"])
def test_a_captured_step_does_not_hide_an_earlier_one(what):
    m, x, y = _model()
    m.set_optimizer(mtx.MTX_OPT_ADAM)
    m.set_clip_norm(1.0)
    held = m._clip, m.s2, m.w, m.v, m.grads, m.grad_avg, m.workspace
    s = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        with torch.cuda.stream(s):
            torch.cuda._sleep(200_000_000)
        m.train_step(x, y, 0.01, 0.9, stream=s)
        m.train_step(x, y, 0.01, 0.9)
    if what == "clip":
        m.set_clip_norm(0)
    elif what == "rule":
        m.set_optimizer(mtx.MTX_OPT_MOMENTUM)
    else:
        m.close()
    assert s.query()
    del graph, held
    m.close()


@pytest.mark.parametrize("overlap", [False, True])
def test_a_model_closed_while_another_stream_is_captured(overlap):
    m, x, y = _model()
    n, _, _ = _model()
    want, _, _ = _model()
    mtx.mtx_set_overlap(n.handle, overlap)
    n.train_step(x, y, 0.01, 0.9)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        m.train_step(x, y, 0.01, 0.9)
        n.close()
    for k in range(3):
        graph.replay()
        want.train_step(x, y, 0.01, 0.9)
        torch.cuda.synchronize()
        assert torch.equal(m.w, want.w) and torch.equal(m.v, want.v), k
    m.close()
    want.close()
