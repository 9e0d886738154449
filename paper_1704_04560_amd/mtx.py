"""Python binding of the C ABI in include/mtx.h (argument marshalling only).

Every function named mtx_* calls the function of the same name in libmtx.so; all arithmetic of
the training step runs in the library's HIP kernels.  PyTorch is used only to allocate device
memory and to name the stream.  If libmtx.so is missing the import of the library raises; there
is no fallback.
"""
from __future__ import annotations

import ctypes as C
import os
from typing import Optional, Sequence, Tuple

import numpy as np

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libmtx.so")

MTX_OK, MTX_EINVAL, MTX_ENOMEM, MTX_EHIP, MTX_EUNSUPPORTED, MTX_ENONFINITE = 0, -1, -2, -3, -4, -5
MTX_F32, MTX_BF16 = 0, 1
MTX_FC, MTX_CONV, MTX_MAXPOOL, MTX_BN, MTX_ADD, MTX_ADDP = 0, 1, 2, 3, 4, 5
MTX_EMBED, MTX_NORM = 6, 7
MTX_OPT_MOMENTUM, MTX_OPT_ADAM, MTX_OPT_ADAGRAD = 0, 1, 2
MTX_NORM_RMS, MTX_NORM_LAYER = 0, 1
MTX_CLIP_WORKSPACE_BYTES = 32768

EXPORTS = ("mtx_model_sizes", "mtx_init_model", "mtx_init_model_static", "mtx_train_step", "mtx_average_grads",
           "mtx_sgd_update", "mtx_adam_update", "mtx_adagrad_update", "mtx_get_params",
           "mtx_set_params", "mtx_get_layer_output", "mtx_set_optimizer",
           "mtx_get_pool_argmax", "mtx_set_graph_replay", "mtx_set_overlap",
           "mtx_set_layerwise_update", "mtx_set_fused_update", "mtx_set_nonfinite_check",
           "mtx_set_timing",
           "mtx_get_timing", "mtx_get_launches", "mtx_free_model", "mtx_last_error",
           "mtx_embed_forward", "mtx_embed_sizes", "mtx_embed_backward",
           "mtx_block_norm_forward", "mtx_block_norm_sizes", "mtx_block_norm_backward",
           "mtx_average_clip", "mtx_clip_sizes", "mtx_init_clip", "mtx_clip_grads",
           "mtx_free_clip", "mtx_train_step_tokens", "mtx_set_embedding", "mtx_set_clip_norm")


class MtxError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"mtx error {code}: {msg}")
        self.code = code


class mtx_layer(C.Structure):
    _fields_ = [(n, C.c_int) for n in ("kind", "out", "k", "stride", "pad", "groups", "relu")]


class mtx_model_desc(C.Structure):
    _fields_ = [("in_c", C.c_int), ("in_h", C.c_int), ("in_w", C.c_int),
                ("n_layers", C.c_int), ("layers", C.POINTER(mtx_layer)), ("compute", C.c_int)]


class mtx_sizes(C.Structure):
    _fields_ = [("n_params", C.c_size_t), ("grad_stride", C.c_size_t),
                ("workspace_bytes", C.c_size_t)]


class mtx_kernel_time(C.Structure):
    _fields_ = [("name", C.c_char * 32), ("layer", C.c_int), ("launches", C.c_int),
                ("total_ms", C.c_double)]


class mtx_launch_info(C.Structure):
    _fields_ = [("site", C.c_char * 32), ("layer", C.c_int), ("tile_rows", C.c_int),
                ("tile_cols", C.c_int), ("k_tile", C.c_int), ("splits", C.c_int),
                ("flags", C.c_int)]


MTX_GEMM_INTERLEAVED, MTX_GEMM_DIRECT_LDS, MTX_GEMM_FUSED_UPDATE, MTX_GEMM_HALO = 1, 2, 4, 8


class mtx_buffers(C.Structure):
    _fields_ = [("w", C.c_void_p), ("v", C.c_void_p), ("grads", C.c_void_p),
                ("grad_avg", C.c_void_p), ("workspace", C.c_void_p),
                ("workspace_bytes", C.c_size_t)]


class mtx_norm_desc(C.Structure):
    _fields_ = [("kind", C.c_int), ("dtype", C.c_int), ("rows", C.c_size_t), ("D", C.c_int),
                ("eps", C.c_float), ("scale", C.c_float), ("gate_rows", C.c_size_t),
                ("post_w", C.c_void_p), ("post_b", C.c_void_p), ("gate", C.c_void_p),
                ("pre_w", C.c_void_p), ("pre_b", C.c_void_p),
                ("ld_h", C.c_size_t), ("ld_x", C.c_size_t), ("ld_y", C.c_size_t)]


class mtx_tensor(C.Structure):
    _fields_ = [("src", C.c_void_p), ("dst", C.c_void_p), ("n", C.c_size_t),
                ("src_type", C.c_int), ("dst_type", C.c_int)]


_lib = None


def lib() -> C.CDLL:
    """Load libmtx.so (built by paper_1704_04560_amd/build.py).  Raises if it is missing."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise ImportError(f"{LIB_PATH} is not built; run paper_1704_04560_amd/build.py")
        L = C.CDLL(LIB_PATH)
        vp, sz, i32, f32 = C.c_void_p, C.c_size_t, C.c_int, C.c_float
        sig = {
            "mtx_model_sizes": (i32, [C.POINTER(mtx_model_desc), i32, i32, C.POINTER(mtx_sizes)]),
            "mtx_init_model": (i32, [C.POINTER(mtx_model_desc), i32, i32, C.c_uint64,
                                     C.POINTER(mtx_buffers), vp, C.POINTER(vp)]),
            "mtx_init_model_static": (i32, [C.POINTER(mtx_model_desc), i32, i32, C.c_uint64,
                                            C.POINTER(mtx_buffers), vp, C.POINTER(vp)]),
            "mtx_train_step": (i32, [vp, vp, vp, f32, f32, vp, vp]),
            "mtx_average_grads": (i32, [vp, i32, sz, sz, vp, vp]),
            "mtx_sgd_update": (i32, [vp, vp, vp, i32, sz, sz, f32, f32, vp, vp]),
            "mtx_adam_update": (i32, [vp, vp, vp, vp, i32, sz, sz, f32, f32, f32, f32,
                                      C.c_longlong, vp, vp]),
            "mtx_adagrad_update": (i32, [vp, vp, vp, i32, sz, sz, f32, f32, vp, vp]),
            "mtx_get_params": (i32, [vp, vp, vp]),
            "mtx_set_params": (i32, [vp, vp, vp]),
            "mtx_get_layer_output": (i32, [vp, i32, vp, sz]),
            "mtx_get_pool_argmax": (i32, [vp, i32, vp, sz]),
            "mtx_set_graph_replay": (i32, [vp, i32]),
            "mtx_set_optimizer": (i32, [vp, i32, f32, f32, f32, vp]),
            "mtx_set_layerwise_update": (i32, [vp, i32]),
            "mtx_set_fused_update": (i32, [vp, i32]),
            "mtx_set_nonfinite_check": (i32, [vp, i32]),
            "mtx_set_overlap": (i32, [vp, i32]),
            "mtx_set_timing": (i32, [vp, i32]),
            "mtx_get_timing": (i32, [vp, C.POINTER(mtx_kernel_time), i32, C.POINTER(i32), i32]),
            "mtx_get_launches": (i32, [vp, C.POINTER(mtx_launch_info), i32, C.POINTER(i32)]),
            "mtx_free_model": (None, [vp]),
            "mtx_last_error": (C.c_char_p, []),
            "mtx_train_step_tokens": (i32, [vp, vp, vp, f32, f32, vp, vp]),
            "mtx_set_embedding": (i32, [vp, f32, i32]),
            "mtx_set_clip_norm": (i32, [vp, f32, vp, vp]),
            "mtx_embed_forward": (i32, [vp, i32, i32, i32, vp, sz, i32, f32, vp, i32, sz, vp]),
            "mtx_embed_sizes": (i32, [sz, i32, i32, i32, C.POINTER(sz)]),
            "mtx_embed_backward": (i32, [vp, sz, i32, vp, i32, sz, i32, i32, i32, f32, vp, sz,
                                         i32, vp, sz, vp]),
            "mtx_block_norm_forward": (i32, [C.POINTER(mtx_norm_desc), vp, vp, vp, vp, vp, vp]),
            "mtx_block_norm_sizes": (i32, [C.POINTER(mtx_norm_desc), i32, C.POINTER(sz)]),
            "mtx_block_norm_backward": (i32, [C.POINTER(mtx_norm_desc), i32, *[vp] * 12, sz, vp,
                                              sz, vp]),
            "mtx_average_clip": (i32, [vp, i32, sz, sz, f32, vp, vp, vp, sz, vp]),
            "mtx_clip_sizes": (i32, [C.POINTER(mtx_tensor), i32, C.POINTER(sz)]),
            "mtx_init_clip": (i32, [C.POINTER(mtx_tensor), i32, vp, sz, vp, C.POINTER(vp)]),
            "mtx_clip_grads": (i32, [vp, f32, vp, vp]),
            "mtx_free_clip": (None, [vp]),
        }
        for name, (res, args) in sig.items():
            fn = getattr(L, name)
            fn.restype = res
            fn.argtypes = args
        _lib = L
    return _lib


def _check(rc: int):
    if rc != MTX_OK:
        msg = lib().mtx_last_error()
        raise MtxError(rc, msg.decode() if msg else "")


def _ptr(t) -> Optional[int]:
    if t is None:
        return None
    if isinstance(t, int):
        return t
    if isinstance(t, np.ndarray):
        return t.ctypes.data
    return t.data_ptr()


_int32 = None   # torch.int32, once torch is there


def _ids(t, name: str) -> Optional[int]:
    """Address of tokens or labels, which the library reads as int32 one after the other (torch's own
    integers are int64, and a sequence without its last token is not contiguous)."""
    global _int32
    if t is None or isinstance(t, int):
        return t
    if isinstance(t, np.ndarray):
        ok = t.dtype == np.int32 and t.flags.c_contiguous
    else:
        if _int32 is None:
            import torch
            _int32 = torch.int32
        ok = t.dtype is _int32 and t.is_contiguous()
    if not ok:
        raise ValueError(f"{name} must be contiguous int32")
    return _ptr(t)


_raw_stream = None   # (): the current stream's handle


def _stream(stream) -> Optional[int]:
    global _raw_stream
    if stream is None:
        if _raw_stream is None:
            import torch
            get = getattr(torch._C, "_cuda_getCurrentRawStream", None)
            # (a Stream object costs more host time than a small kernel takes)
            _raw_stream = ((lambda: get(torch.cuda.current_device())) if get else
                           (lambda: torch.cuda.current_stream().cuda_stream))
        return _raw_stream() or None
    if isinstance(stream, int):
        return stream or None
    return stream.cuda_stream or None


def make_desc(in_shape: Sequence[int], layers: Sequence[Sequence[int]], compute: int):
    arr = (mtx_layer * len(layers))()
    for i, t in enumerate(layers):
        for name, val in zip(("kind", "out", "k", "stride", "pad", "groups", "relu"), t):
            setattr(arr[i], name, int(val))
    d = mtx_model_desc(int(in_shape[0]), int(in_shape[1]), int(in_shape[2]), len(layers),
                       C.cast(arr, C.POINTER(mtx_layer)), int(compute))
    d._keep = arr
    return d


# ---- the C ABI, one Python function per entry point -------------------------------------------

def mtx_model_sizes(desc, R: int, shard_batch: int) -> Tuple[int, int, int]:
    out = mtx_sizes()
    _check(lib().mtx_model_sizes(C.byref(desc), R, shard_batch, C.byref(out)))
    return out.n_params, out.grad_stride, out.workspace_bytes


def mtx_init_model(desc, R, shard_batch, seed, w, v, grads, grad_avg, workspace, stream=None):
    bufs = mtx_buffers(_ptr(w), _ptr(v), _ptr(grads), _ptr(grad_avg), _ptr(workspace),
                       workspace.numel() * workspace.element_size())
    handle = C.c_void_p()
    _check(lib().mtx_init_model(C.byref(desc), R, shard_batch, C.c_uint64(seed), C.byref(bufs),
                                _stream(stream), C.byref(handle)))
    return handle


def mtx_init_model_static(desc, R, shard_batch, seed, w, v, grads, grad_avg, stream=None):
    bufs = mtx_buffers(_ptr(w), _ptr(v), _ptr(grads), _ptr(grad_avg), None, 0)
    handle = C.c_void_p()
    _check(lib().mtx_init_model_static(C.byref(desc), R, shard_batch, C.c_uint64(seed),
                                       C.byref(bufs), _stream(stream), C.byref(handle)))
    return handle


def mtx_train_step(handle, x, labels, lr, momentum, loss_out=None, stream=None):
    _check(lib().mtx_train_step(handle, _ptr(x), _ids(labels, "labels"), lr, momentum,
                                _ptr(loss_out), _stream(stream)))


def mtx_train_step_tokens(handle, tokens, labels, lr, momentum, loss_out=None, stream=None):
    _check(lib().mtx_train_step_tokens(handle, _ids(tokens, "tokens"), _ids(labels, "labels"), lr,
                                       momentum, _ptr(loss_out), _stream(stream)))


def mtx_set_embedding(handle, scale=1.0, pad=-1):
    _check(lib().mtx_set_embedding(handle, scale, pad))


def mtx_set_clip_norm(handle, max_norm, norm_out=None, workspace=None):
    _check(lib().mtx_set_clip_norm(handle, max_norm, _ptr(norm_out), _ptr(workspace)))


def mtx_average_grads(grads, R, n, ld, avg, stream=None):
    _check(lib().mtx_average_grads(_ptr(grads), R, n, ld, _ptr(avg), _stream(stream)))


def mtx_sgd_update(w, v, grads, R, n, ld, lr, momentum, avg_out=None, stream=None):
    _check(lib().mtx_sgd_update(_ptr(w), _ptr(v), _ptr(grads), R, n, ld, lr, momentum,
                                _ptr(avg_out), _stream(stream)))


def mtx_adam_update(w, m, v, grads, R, n, ld, lr, beta1, beta2, eps, step, avg_out=None,
                    stream=None):
    _check(lib().mtx_adam_update(_ptr(w), _ptr(m), _ptr(v), _ptr(grads), R, n, ld, lr, beta1,
                                 beta2, eps, step, _ptr(avg_out), _stream(stream)))


def mtx_adagrad_update(w, acc, grads, R, n, ld, lr, eps, avg_out=None, stream=None):
    _check(lib().mtx_adagrad_update(_ptr(w), _ptr(acc), _ptr(grads), R, n, ld, lr, eps,
                                    _ptr(avg_out), _stream(stream)))


def mtx_set_optimizer(handle, kind, beta1=0.9, beta2=0.999, eps=1e-8, s2=None):
    _check(lib().mtx_set_optimizer(handle, kind, beta1, beta2, eps, _ptr(s2)))


def mtx_get_params(handle, w_host: np.ndarray, v_host: Optional[np.ndarray] = None):
    _check(lib().mtx_get_params(handle, _ptr(w_host), _ptr(v_host)))


def mtx_set_params(handle, w_host: np.ndarray, v_host: Optional[np.ndarray] = None):
    w_host = np.ascontiguousarray(w_host, dtype=np.float32)
    v_host = None if v_host is None else np.ascontiguousarray(v_host, dtype=np.float32)
    _check(lib().mtx_set_params(handle, _ptr(w_host), _ptr(v_host)))


def mtx_get_layer_output(handle, layer: int, dst: np.ndarray):
    _check(lib().mtx_get_layer_output(handle, layer, _ptr(dst), dst.size))


def mtx_get_pool_argmax(handle, layer: int, dst: np.ndarray):
    _check(lib().mtx_get_pool_argmax(handle, layer, _ptr(dst), dst.size))


def mtx_set_graph_replay(handle, enable: bool):
    _check(lib().mtx_set_graph_replay(handle, 1 if enable else 0))


def mtx_set_overlap(handle, enable: bool):
    _check(lib().mtx_set_overlap(handle, 1 if enable else 0))


def mtx_set_layerwise_update(handle, enable: bool):
    _check(lib().mtx_set_layerwise_update(handle, 1 if enable else 0))


def mtx_set_fused_update(handle, enable: bool):
    _check(lib().mtx_set_fused_update(handle, 1 if enable else 0))


def mtx_set_nonfinite_check(handle, enable: bool):
    _check(lib().mtx_set_nonfinite_check(handle, 1 if enable else 0))


def mtx_set_timing(handle, enable: bool):
    _check(lib().mtx_set_timing(handle, 1 if enable else 0))


def mtx_get_timing(handle, reset: bool = False):
    """[(name, layer, launches, total_ms)] per launch site of the training step."""
    cap = 256
    buf = (mtx_kernel_time * cap)()
    cnt = C.c_int()
    _check(lib().mtx_get_timing(handle, buf, cap, C.byref(cnt), 1 if reset else 0))
    return [(buf[i].name.decode(), buf[i].layer, buf[i].launches, buf[i].total_ms)
            for i in range(min(cnt.value, cap))]


def mtx_get_launches(handle):
    """[dict(site, layer, tile_rows, tile_cols, k_tile, splits, flags)] per matrix launch of the
    last enqueued training step."""
    cap = 1024
    buf = (mtx_launch_info * cap)()
    cnt = C.c_int()
    _check(lib().mtx_get_launches(handle, buf, cap, C.byref(cnt)))
    return [dict(site=buf[i].site.decode(), layer=buf[i].layer, tile_rows=buf[i].tile_rows,
                 tile_cols=buf[i].tile_cols, k_tile=buf[i].k_tile, splits=buf[i].splits,
                 flags=buf[i].flags) for i in range(min(cnt.value, cap))]


def mtx_free_model(handle):
    lib().mtx_free_model(handle)


def _bytes(t) -> int:
    return 0 if t is None else t.nbytes


def mtx_embed_forward(w, w_type, V, D, tokens, n, pad, scale, y, y_type, ldy, stream=None):
    _check(lib().mtx_embed_forward(_ptr(w), w_type, V, D, _ids(tokens, "tokens"), n, pad, scale,
                                   _ptr(y), y_type, ldy, _stream(stream)))


def mtx_embed_sizes(n, R, V, D) -> int:
    out = C.c_size_t()
    _check(lib().mtx_embed_sizes(n, R, V, D, C.byref(out)))
    return out.value


def mtx_embed_backward(tokens, n, R, dy, dy_type, lddy, V, D, pad, scale, grads, ld, accumulate,
                       workspace, stream=None):
    _check(lib().mtx_embed_backward(_ids(tokens, "tokens"), n, R, _ptr(dy), dy_type, lddy, V, D, pad,
                                    scale, _ptr(grads), ld, 1 if accumulate else 0, _ptr(workspace),
                                    _bytes(workspace), _stream(stream)))


def make_norm_desc(kind, dtype, rows, D, eps=1e-5, scale=1.0, gate_rows=0, post_w=None,
                   post_b=None, gate=None, pre_w=None, pre_b=None, ld_h=0, ld_x=0, ld_y=0):
    """mtx_norm_desc over the given weights, which it keeps alive."""
    d = mtx_norm_desc(kind, dtype, rows, D, eps, scale, gate_rows, _ptr(post_w), _ptr(post_b),
                      _ptr(gate), _ptr(pre_w), _ptr(pre_b), ld_h, ld_x, ld_y)
    d._keep = (post_w, post_b, gate, pre_w, pre_b)
    return d


def mtx_block_norm_forward(desc, h, x, h_out, y, stats=None, stream=None):
    _check(lib().mtx_block_norm_forward(C.byref(desc), _ptr(h), _ptr(x), _ptr(h_out), _ptr(y),
                                        _ptr(stats), _stream(stream)))


def mtx_block_norm_sizes(desc, R) -> int:
    out = C.c_size_t()
    _check(lib().mtx_block_norm_sizes(C.byref(desc), R, C.byref(out)))
    return out.value


def mtx_block_norm_backward(desc, R, h_out, x, stats, dy, dh_out, dh, dx, d_post_w, d_post_b,
                            d_gate, d_pre_w, d_pre_b, ld, workspace, stream=None):
    _check(lib().mtx_block_norm_backward(
        C.byref(desc), R, _ptr(h_out), _ptr(x), _ptr(stats), _ptr(dy), _ptr(dh_out), _ptr(dh),
        _ptr(dx), _ptr(d_post_w), _ptr(d_post_b), _ptr(d_gate), _ptr(d_pre_w), _ptr(d_pre_b), ld,
        _ptr(workspace), _bytes(workspace), _stream(stream)))


def mtx_average_clip(grads, R, n, ld, max_norm, avg, norm_out, workspace, stream=None):
    _check(lib().mtx_average_clip(_ptr(grads), R, n, ld, max_norm, _ptr(avg), _ptr(norm_out),
                                  _ptr(workspace), _bytes(workspace), _stream(stream)))


def make_tensor_list(pairs):
    """mtx_tensor array of (src, dst) torch tensors (contiguous, float32 or bfloat16; dst may be
    None, or src itself)."""
    import torch
    types = {torch.float32: MTX_F32, torch.bfloat16: MTX_BF16}
    arr = (mtx_tensor * len(pairs))()
    for a, (src, dst) in zip(arr, pairs):
        for t in (src, dst):
            if t is None:
                continue
            if t.dtype not in types or not t.is_contiguous():
                raise ValueError("tensors must be contiguous, float32 or bfloat16")
            if t.numel() != src.numel() or t.device != src.device:
                raise ValueError("src and dst must have the same length and device")
        a.src, a.n, a.src_type = src.data_ptr(), src.numel(), types[src.dtype]
        if dst is not None:
            a.dst, a.dst_type = dst.data_ptr(), types[dst.dtype]
    return arr


def mtx_clip_sizes(tensors) -> int:
    out = C.c_size_t()
    _check(lib().mtx_clip_sizes(tensors, len(tensors), C.byref(out)))
    return out.value


def mtx_init_clip(tensors, workspace, stream=None):
    handle = C.c_void_p()
    _check(lib().mtx_init_clip(tensors, len(tensors), _ptr(workspace), _bytes(workspace),
                               _stream(stream), C.byref(handle)))
    return handle


def mtx_clip_grads(handle, max_norm, norm_out=None, stream=None):
    _check(lib().mtx_clip_grads(handle, max_norm, _ptr(norm_out), _stream(stream)))


def mtx_free_clip(handle):
    lib().mtx_free_clip(handle)


class Clip:
    """A list of (src, dst) tensors whose global norm is clipped (mtx_clip_grads), with its
    workspace; keeps the tensors alive.  Closing or dropping it waits for its last call; keep it as
    long as a graph that holds its calls is replayed."""

    def __init__(self, pairs, stream=None):
        import torch
        self.handle = None
        self.pairs = list(pairs)
        tensors = make_tensor_list(self.pairs)
        if any(not src.is_cuda or src.device != self.pairs[0][0].device for src, _ in self.pairs):
            raise ValueError("the tensors must be on one GPU")
        self.workspace = torch.empty(mtx_clip_sizes(tensors), dtype=torch.uint8,
                                     device=self.pairs[0][0].device)
        self.handle = mtx_init_clip(tensors, self.workspace, stream)

    def clip(self, max_norm, norm_out=None, stream=None):
        mtx_clip_grads(self.handle, max_norm, norm_out, stream)

    def close(self):
        if self.handle:
            mtx_free_clip(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


# ---- convenience wrapper owning the device buffers --------------------------------------------

class Model:
    """A network bound to caller-owned device buffers (allocated here with torch)."""

    def __init__(self, in_shape, layers, compute, R, shard_batch, seed=0, stream=None,
                 static_workspace=False):
        import torch
        self.in_shape = tuple(in_shape)
        self.layers = [tuple(int(v) for v in t) for t in layers]
        self.compute = compute
        self.R, self.Nb = R, shard_batch
        self.B = R * shard_batch
        self.desc = make_desc(in_shape, layers, compute)
        self.P, self.ld, self.ws_bytes = mtx_model_sizes(self.desc, R, shard_batch)
        dev = torch.device("cuda")
        self.w = torch.empty(self.P, dtype=torch.float32, device=dev)
        self.v = torch.empty(self.P, dtype=torch.float32, device=dev)
        self.grads = torch.empty(R * self.ld, dtype=torch.float32, device=dev)
        self.grad_avg = torch.empty(self.P, dtype=torch.float32, device=dev)
        if static_workspace:  # the library's static array (mtx_init_model_static)
            self.workspace = None
            self.handle = mtx_init_model_static(self.desc, R, shard_batch, seed, self.w, self.v,
                                                self.grads, self.grad_avg, stream)
        else:
            self.workspace = torch.empty(max(self.ws_bytes, 256), dtype=torch.uint8, device=dev)
            self.handle = mtx_init_model(self.desc, R, shard_batch, seed, self.w, self.v,
                                         self.grads, self.grad_avg, self.workspace, stream)
        self._shapes = self._out_shapes()
        self._clip = (None, None)   # norm_out and workspace of set_clip_norm
        self.s2 = None              # second moment of set_optimizer

    def _out_shapes(self):
        c, h, w = self.in_shape
        out = []
        for (kind, o, k, s, p, g, relu) in self.layers:
            if kind == MTX_EMBED:
                c = o
            elif kind == MTX_CONV:
                c, h, w = o, (h + 2 * p - k) // s + 1, (w + 2 * p - k) // s + 1
            elif kind == MTX_FC:
                c, h, w = o, 1, 1
            elif kind in (MTX_BN, MTX_ADD, MTX_ADDP, MTX_NORM):
                pass
            else:
                h, w = (h - k) // s + 1, (w - k) // s + 1
            out.append((c, h, w))
        return out

    def train_step(self, x, labels, lr, momentum, loss_out=None, stream=None):
        """x: images, or the tokens (int32) of a network that begins with MTX_EMBED."""
        step = mtx_train_step_tokens if self.layers[0][0] == MTX_EMBED else mtx_train_step
        step(self.handle, x, labels, lr, momentum, loss_out, stream)

    def set_clip_norm(self, max_norm, norm_out=None):
        """Clip the averaged gradient's global norm in train_step (0: off); norm_out: a device
        float32 [1] that receives the norm of every step.  A graph that holds a clipped step is
        replayed only while the option stays on with the same norm_out."""
        import torch
        ws = self._clip[1] if max_norm > 0 else None
        if max_norm > 0 and ws is None:
            ws = torch.empty(MTX_CLIP_WORKSPACE_BYTES, dtype=torch.uint8, device=self.w.device)
        mtx_set_clip_norm(self.handle, max_norm, norm_out, ws)
        self._clip = (norm_out if max_norm > 0 else None, ws)

    def set_optimizer(self, kind, beta1=0.9, beta2=0.999, eps=1e-8):
        """Select the update rule of train_step; Adam gets a zeroed second-moment buffer."""
        import torch
        s2 = None
        if kind == MTX_OPT_ADAM:
            s2 = torch.zeros(self.P, dtype=torch.float32, device=self.w.device)
        mtx_set_optimizer(self.handle, kind, beta1, beta2, eps, s2)
        self.s2 = s2   # (a refused call keeps the present one in use)

    def get_params(self):
        w = np.empty(self.P, np.float32)
        v = np.empty(self.P, np.float32)
        mtx_get_params(self.handle, w, v)
        return w, v

    def set_params(self, w, v=None):
        mtx_set_params(self.handle, w, v)

    def grads_host(self):
        """Per-shard gradients [R, P] (device-to-host copy through torch)."""
        import torch
        torch.cuda.synchronize()
        return self.grads.view(self.R, self.ld)[:, :self.P].cpu().numpy()

    def layer_output(self, layer: int) -> np.ndarray:
        dst = np.empty(int(np.prod(self._shapes[layer])) * self.B, np.float32)
        mtx_get_layer_output(self.handle, layer, dst)
        return dst

    def pool_argmax(self, layer: int) -> np.ndarray:
        dst = np.empty(int(np.prod(self._shapes[layer])) * self.B, np.uint8)
        mtx_get_pool_argmax(self.handle, layer, dst)
        return dst

    def close(self):
        if self.handle:
            mtx_free_model(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
