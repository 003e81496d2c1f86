"""ctypes binding of libflmoe.so (the C ABI declared in include/flmoe.h).

Argument marshalling only: every step of the shuffle runs in the library's HIP
kernels.  torch is used for device memory and for the current HIP stream.
There is no CPU fallback: if the shared library is missing, importing the
functions fails with an error that says how to build it.
"""
import ctypes as C
import os

import torch

from . import build as _build

FL_OK = 0
FL_ERR_INVALID_ARG, FL_ERR_ALIGNMENT, FL_ERR_WORKSPACE, FL_ERR_HIP = -1, -2, -3, -4
FL_ERR_STATIC_LIMIT = -5
FL_STATIC_SCRATCH_BYTES = 8 << 20
FL_STATUS_BAD_INDEX, FL_STATUS_CAPACITY, FL_STATUS_TIMEOUT = 1, 2, 4
FL_DTYPE_BF16, FL_DTYPE_E4M3_BLOCK128 = 0, 1
FL_FLAG_ZERO_PAD = 1
FL_FLAG_STREAM_ORDERED = 2
FL_FLAG_PEER_PUSH = 4
FL_FLAG_PARTIAL_SUMS = 8
FL_FLAG_PROGRESSIVE_RECV = 16
FL_ACT_SILU, FL_ACT_GELU = 0, 1
FL_KERNEL_COUNT = 11


class fl_moe_config(C.Structure):
    _fields_ = [("n_ranks", C.c_int32), ("n_experts", C.c_int32), ("max_tokens", C.c_int32),
                ("top_k", C.c_int32), ("hidden", C.c_int32), ("dispatch_dtype", C.c_int32),
                ("expert_align", C.c_int32), ("flags", C.c_int32),
                ("recv_capacity_rows", C.c_int64), ("expert_capacity_rows", C.c_int64),
                ("spin_limit", C.c_int64), ("max_private_rows", C.c_int32),
                ("reserved", C.c_int32)]


class fl_moe_sizes(C.Structure):
    _fields_ = [("workspace_bytes", C.c_size_t), ("recv_capacity_rows", C.c_int64),
                ("expert_capacity_rows", C.c_int64), ("send_capacity_rows", C.c_int64),
                ("x_row_bytes", C.c_int64), ("wire_row_bytes", C.c_int64),
                ("expert_x_row_bytes", C.c_int64), ("scales_per_row", C.c_int64),
                ("combine_row_bytes", C.c_int64), ("private_rows", C.c_int64),
                ("recv_buffer_rows", C.c_int64)]


class fl_moe_layout_view(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in
                ("counts", "dedup_counts", "tokens_per_expert", "send_off", "recv_off",
                 "expert_off", "comb_off", "comb_pos", "plan_ok")]


LAYOUT_OUT_FIELDS = ("counts", "dedup_counts", "tokens_per_expert", "send_off", "recv_off",
                     "expert_off", "comb_off", "comb_pos", "plan_ok", "status")


class fl_moe_layout_out(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in LAYOUT_OUT_FIELDS]


class fl_moe_debug_view(C.Structure):
    _fields_ = [("buf_a", C.c_void_p), ("buf_b", C.c_void_p),
                ("buf_a_rank_bytes", C.c_int64), ("buf_b_rank_bytes", C.c_int64),
                ("arrive_route", C.c_void_p), ("epoch_route", C.c_void_p),
                ("arrive_disp", C.c_void_p), ("arrive_comb", C.c_void_p),
                ("expect_disp", C.c_void_p), ("expect_comb", C.c_void_p), ("status", C.c_void_p)]


class fl_moe_launch_plan(C.Structure):
    _fields_ = [("unpack_by_chunks", C.c_int32), ("replies_by_chunks", C.c_int32), ("replies_cached", C.c_int32),
                ("layout_blocks", C.c_int32), ("layout_tiles", C.c_int32),
                ("recv_grid_rows", C.c_int64), ("reply_grid_rows", C.c_int64)]


class fl_moe_ordering_plan(C.Structure):
    _fields_ = [("dispatch_announce_kernel", C.c_int32), ("replies_written_through", C.c_int32),
                ("combine_announce_kernel", C.c_int32), ("dispatch_gate_kernel", C.c_int32),
                ("combine_gate_kernel", C.c_int32)]


EXPORTS = ["fl_moe_query_sizes", "fl_moe_create", "fl_moe_destroy", "fl_moe_layout",
           "fl_moe_layout_static",
           "fl_moe_dispatch_send", "fl_moe_dispatch_send_weighted", "fl_moe_dispatch_send_e4m3",
           "fl_moe_dispatch_recv",
           "fl_moe_combine_send",
           "fl_moe_combine_reduce", "fl_moe_expert_gated", "fl_moe_expert_gated_backward", "fl_moe_expert_product",
           "fl_moe_expert_product_backward", "fl_moe_expert_gated_e4m3", "fl_moe_expert_product_e4m3",
           "fl_moe_status", "fl_moe_reset", "fl_moe_required_capacities",
           "fl_moe_strerror", "fl_moe_debug_views", "fl_moe_debug_row_strides",
           "fl_moe_debug_tune", "fl_moe_debug_launch_groups", "fl_moe_debug_launch_plan", "fl_moe_debug_ordering_plan",
           "fl_moe_debug_copy", "fl_moe_debug_fill", "fl_moe_debug_read", "fl_moe_profile_enable", "fl_moe_profile_collect", "fl_moe_profile_read",
           "fl_moe_kernel_name", "fl_moe_build_id"]

_lib = None


def lib():
    """The loaded shared library.  Loads what is built; builds only if nothing is.  A
    library built from other sources than the ones beside it is refused: tests and
    benchmarks must never run an older binary than the code they claim to measure."""
    global _lib
    if _lib is None:
        path = _build.lib_path()
        if not os.path.exists(path):
            _build.build()
        L = C.CDLL(path)
        L.fl_moe_build_id.restype = C.c_char_p
        built_from, tree = L.fl_moe_build_id().decode(), _build.source_hash()
        if built_from != tree:
            raise RuntimeError(f"{path} was built from other sources (build id {built_from}, the tree has "
                               f"{tree}): rebuild it with `python -m paper_2510_27656_amd.build`")
        vp, i32, i64 = C.c_void_p, C.c_int, C.c_int64
        L.fl_moe_query_sizes.argtypes = [C.POINTER(fl_moe_config), C.POINTER(fl_moe_sizes)]
        L.fl_moe_create.argtypes = [C.POINTER(fl_moe_config), vp, C.c_size_t, C.POINTER(vp)]
        L.fl_moe_destroy.argtypes = [vp]
        L.fl_moe_layout.argtypes = [vp, i32, i32, vp, vp, C.POINTER(fl_moe_layout_view), vp]
        L.fl_moe_layout_static.argtypes = [C.POINTER(fl_moe_config), vp, vp,
                                           C.POINTER(fl_moe_layout_out), vp]
        L.fl_moe_dispatch_send.argtypes = [vp, i32, i32, vp, vp]
        L.fl_moe_dispatch_send_weighted.argtypes = [vp, i32, i32, vp, vp, vp]
        L.fl_moe_dispatch_send_e4m3.argtypes = [vp, i32, i32, vp, vp, vp, vp]
        L.fl_moe_dispatch_recv.argtypes = [vp, i32, i32, vp, vp, vp, vp]
        L.fl_moe_combine_send.argtypes = [vp, i32, i32, vp, vp]
        L.fl_moe_combine_reduce.argtypes = [vp, i32, i32, vp, vp, vp]
        rows = [C.POINTER(fl_moe_config), i32, i32, vp, vp, i32, i32]      # ..., widths or width and activation
        L.fl_moe_expert_gated.argtypes = rows + [vp] * 6
        L.fl_moe_expert_gated_backward.argtypes = rows + [vp] * 10
        L.fl_moe_expert_product.argtypes = rows + [vp] * 4
        L.fl_moe_expert_product_backward.argtypes = rows + [vp] * 6
        L.fl_moe_expert_gated_e4m3.argtypes = rows + [vp] * 7
        L.fl_moe_expert_product_e4m3.argtypes = rows + [vp] * 6
        L.fl_moe_status.argtypes = [vp, C.POINTER(C.c_int32), vp]
        L.fl_moe_reset.argtypes = [vp, vp]
        L.fl_moe_required_capacities.argtypes = [vp, C.POINTER(C.c_int64), C.POINTER(C.c_int64), vp]
        L.fl_moe_strerror.argtypes = [i32]
        L.fl_moe_strerror.restype = C.c_char_p
        L.fl_moe_debug_views.argtypes = [vp, C.POINTER(fl_moe_debug_view)]
        L.fl_moe_debug_row_strides.argtypes = [C.POINTER(fl_moe_config), C.POINTER(C.c_int64), C.POINTER(C.c_int64)]
        L.fl_moe_debug_tune.argtypes = [vp, i32, i32]
        L.fl_moe_debug_launch_groups.argtypes = [C.POINTER(fl_moe_config), i32, i32, C.POINTER(C.c_int)]
        L.fl_moe_debug_launch_plan.argtypes = [C.POINTER(fl_moe_config), i32, C.POINTER(fl_moe_launch_plan)]
        L.fl_moe_debug_ordering_plan.argtypes = [C.POINTER(fl_moe_config), i32, i32, C.POINTER(fl_moe_ordering_plan)]
        L.fl_moe_debug_copy.argtypes = [vp, vp, C.c_size_t, vp]
        L.fl_moe_debug_fill.argtypes = [vp, C.c_size_t, vp]
        L.fl_moe_debug_read.argtypes = [vp, C.c_size_t, vp, vp]
        L.fl_moe_profile_enable.argtypes = [vp, i32]
        L.fl_moe_profile_collect.argtypes = [vp, vp]
        L.fl_moe_profile_read.argtypes = [vp, C.POINTER(C.c_double), C.POINTER(i64)]
        L.fl_moe_kernel_name.argtypes = [i32]
        L.fl_moe_kernel_name.restype = C.c_char_p
        L.fl_moe_build_id.argtypes = []
        for name in EXPORTS:
            getattr(L, name)                    # every declared symbol must be exported
        _lib = L
    return _lib


class FlMoeError(RuntimeError):
    def __init__(self, code, where):
        self.code = code
        super().__init__(f"{where}: {lib().fl_moe_strerror(code).decode()} ({code})")


def _check(code, where):
    if code != FL_OK:
        raise FlMoeError(code, where)


# Handles and addresses go to the library as plain integers (its argument types turn them into pointers), and
# the current stream's handle is read without building a stream object: the five calls of a small step are
# bound by what the host does between launches (2 ranks x 16 tokens: 56 -> 44 us of host time per step).
# A torch built without GPU support has neither function; the host-only queries work there.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_current_device = getattr(torch._C, "_cuda_getDevice", None)


def _stream(stream):
    if stream is None:
        if _raw_stream is None or _current_device is None:
            return torch.cuda.current_stream().cuda_stream
        return _raw_stream(_current_device())
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


def _ptr(t):
    if t is None:
        return None
    assert t.is_cuda and t.is_contiguous()
    return t.data_ptr()


# ------------------------------------------------------------------ the C calls, same names
def fl_moe_query_sizes(cfg: fl_moe_config) -> fl_moe_sizes:
    out = fl_moe_sizes()
    _check(lib().fl_moe_query_sizes(C.byref(cfg), C.byref(out)), "fl_moe_query_sizes")
    return out


def fl_moe_create(cfg: fl_moe_config, workspace: torch.Tensor):
    ctx = C.c_void_p()
    _check(lib().fl_moe_create(C.byref(cfg), _ptr(workspace),
                               workspace.numel() * workspace.element_size(), C.byref(ctx)),
           "fl_moe_create")
    return ctx


def fl_moe_destroy(ctx):
    _check(lib().fl_moe_destroy(ctx), "fl_moe_destroy")


def fl_moe_layout(ctx, rank_begin, rank_count, indices, num_tokens, stream=None):
    view = fl_moe_layout_view()
    _check(lib().fl_moe_layout(ctx, rank_begin, rank_count, _ptr(indices), _ptr(num_tokens),
                               C.byref(view), _stream(stream)), "fl_moe_layout")
    return view


def fl_moe_layout_static(cfg: fl_moe_config, indices, num_tokens, out: dict, stream=None):
    """out: int32 device tensors by the field names of fl_moe_layout_out (caller-owned)."""
    o = fl_moe_layout_out(*[_ptr(out[n]) for n in LAYOUT_OUT_FIELDS])
    _check(lib().fl_moe_layout_static(C.byref(cfg), _ptr(indices), _ptr(num_tokens), C.byref(o),
                                      _stream(stream)), "fl_moe_layout_static")


def fl_moe_dispatch_send(ctx, rank_begin, rank_count, x, stream=None):
    _check(lib().fl_moe_dispatch_send(ctx, rank_begin, rank_count, _ptr(x), _stream(stream)),
           "fl_moe_dispatch_send")


def fl_moe_dispatch_send_e4m3(ctx, rank_begin, rank_count, codes, scales, weights=None, stream=None):
    _check(lib().fl_moe_dispatch_send_e4m3(ctx, rank_begin, rank_count, _ptr(codes), _ptr(scales),
                                           _ptr(weights),
                                           _stream(stream)), "fl_moe_dispatch_send_e4m3")


def fl_moe_dispatch_send_weighted(ctx, rank_begin, rank_count, x, weights, stream=None):
    _check(lib().fl_moe_dispatch_send_weighted(ctx, rank_begin, rank_count, _ptr(x), _ptr(weights),
                                               _stream(stream)), "fl_moe_dispatch_send_weighted")


def fl_moe_dispatch_recv(ctx, rank_begin, rank_count, expert_x, expert_scales, tokens_per_expert,
                         stream=None):
    _check(lib().fl_moe_dispatch_recv(ctx, rank_begin, rank_count, _ptr(expert_x),
                                      _ptr(expert_scales), _ptr(tokens_per_expert),
                                      _stream(stream)), "fl_moe_dispatch_recv")


def fl_moe_combine_send(ctx, rank_begin, rank_count, expert_y, stream=None):
    _check(lib().fl_moe_combine_send(ctx, rank_begin, rank_count, _ptr(expert_y), _stream(stream)),
           "fl_moe_combine_send")


def fl_moe_combine_reduce(ctx, rank_begin, rank_count, weights, out, stream=None):
    _check(lib().fl_moe_combine_reduce(ctx, rank_begin, rank_count, _ptr(weights), _ptr(out),
                                       _stream(stream)), "fl_moe_combine_reduce")


# The experts' products take tensors of many shapes, so their types and sizes are checked here as well: the library
# sees addresses only.
_BF16, _F32, _I32 = (torch.bfloat16,), (torch.float32,), (torch.int32,)
_E4M3 = (torch.uint8, torch.float8_e4m3fn)


class _Tensors:
    """Addresses of one call's tensors; each of the given type, of at least so many elements, on the current device."""

    def __init__(self, cfg, where):
        self.where = where
        self.sizes = fl_moe_query_sizes(cfg)
        self.rows = cfg.n_ranks * self.sizes.expert_capacity_rows
        self.experts, self.ranks = cfg.n_experts, cfg.n_ranks

    def __call__(self, t, dtypes, count, optional=False):
        if t is None and optional:
            return None
        if (not isinstance(t, torch.Tensor) or not t.is_cuda or t.get_device() != _current_device() or t.dtype not in dtypes
                or t.numel() < count or not t.is_contiguous()):
            raise FlMoeError(FL_ERR_INVALID_ARG, f"{self.where}: a tensor of {count} or more {dtypes[0]} elements in a row on "
                             f"the current device is needed, got {_described(t)}")
        return t.data_ptr()

    def tables(self, expert_off, tokens_per_expert):
        if isinstance(expert_off, int) and isinstance(tokens_per_expert, int):      # of a fl_moe_layout_view
            return expert_off, tokens_per_expert
        return self(expert_off, _I32, self.experts + self.ranks), self(tokens_per_expert, _I32, self.experts)


def _described(t):
    return f"{t.dtype} {tuple(t.shape)} on {t.device}" if isinstance(t, torch.Tensor) else repr(t)


def fl_moe_expert_gated(cfg, rank_begin, rank_count, expert_off, tokens_per_expert, inter, activation, x, w, h, pre=None,
                        pre_scales=None, stream=None):
    t = _Tensors(cfg, "fl_moe_expert_gated")
    _check(lib().fl_moe_expert_gated(
        C.byref(cfg), rank_begin, rank_count, *t.tables(expert_off, tokens_per_expert), inter, activation,
        t(x, _BF16, t.rows * cfg.hidden), t(w, _BF16, t.experts * 2 * inter * cfg.hidden), t(h, _BF16, t.rows * inter),
        t(pre, _BF16 if pre_scales is None else _E4M3, t.rows * 2 * inter, True),
        t(pre_scales, _F32, t.rows * 2 * inter // 128, True), _stream(stream)), t.where)


def fl_moe_expert_gated_backward(cfg, rank_begin, rank_count, expert_off, tokens_per_expert, inter, activation, x, w, pre,
                                 pre_scales, dh, dpre, dx=None, dw=None, h=None, stream=None):
    t = _Tensors(cfg, "fl_moe_expert_gated_backward")
    weights = t.experts * 2 * inter * cfg.hidden
    _check(lib().fl_moe_expert_gated_backward(
        C.byref(cfg), rank_begin, rank_count, *t.tables(expert_off, tokens_per_expert), inter, activation,
        t(x, _BF16, t.rows * cfg.hidden, True), t(w, _BF16, weights, True),
        t(pre, _BF16 if pre_scales is None else _E4M3, t.rows * 2 * inter),
        t(pre_scales, _F32, t.rows * 2 * inter // 128, True), t(dh, _BF16, t.rows * inter),
        t(dpre, _BF16, t.rows * 2 * inter), t(dx, _BF16, t.rows * cfg.hidden, True), t(dw, _BF16, weights, True),
        t(h, _BF16, t.rows * inter, True), _stream(stream)), t.where)


def fl_moe_expert_product(cfg, rank_begin, rank_count, expert_off, tokens_per_expert, in_features, out_features, x, w, y,
                          stream=None):
    t = _Tensors(cfg, "fl_moe_expert_product")
    _check(lib().fl_moe_expert_product(
        C.byref(cfg), rank_begin, rank_count, *t.tables(expert_off, tokens_per_expert), in_features, out_features,
        t(x, _BF16, t.rows * in_features), t(w, _BF16, t.experts * in_features * out_features),
        t(y, _BF16, t.rows * out_features), _stream(stream)), t.where)


def fl_moe_expert_product_backward(cfg, rank_begin, rank_count, expert_off, tokens_per_expert, in_features, out_features, x,
                                   w, dy, dx=None, dw=None, stream=None):
    t = _Tensors(cfg, "fl_moe_expert_product_backward")
    weights = t.experts * in_features * out_features
    _check(lib().fl_moe_expert_product_backward(
        C.byref(cfg), rank_begin, rank_count, *t.tables(expert_off, tokens_per_expert), in_features, out_features,
        t(x, _BF16, t.rows * in_features, True), t(w, _BF16, weights, True), t(dy, _BF16, t.rows * out_features),
        t(dx, _BF16, t.rows * in_features, True), t(dw, _BF16, weights, True), _stream(stream)), t.where)


def fl_moe_expert_gated_e4m3(cfg, rank_begin, rank_count, expert_off, tokens_per_expert, inter, activation, x, x_scales, w,
                             w_scales, h, h_scales, stream=None):
    t = _Tensors(cfg, "fl_moe_expert_gated_e4m3")
    weights = t.experts * 2 * inter * cfg.hidden
    _check(lib().fl_moe_expert_gated_e4m3(
        C.byref(cfg), rank_begin, rank_count, *t.tables(expert_off, tokens_per_expert), inter, activation,
        t(x, _E4M3, t.rows * cfg.hidden), t(x_scales, _F32, t.rows * cfg.hidden // 128), t(w, _E4M3, weights),
        t(w_scales, _F32, weights // (128 * 128)), t(h, _E4M3, t.rows * inter), t(h_scales, _F32, t.rows * inter // 128),
        _stream(stream)), t.where)


def fl_moe_expert_product_e4m3(cfg, rank_begin, rank_count, expert_off, tokens_per_expert, in_features, out_features, x,
                               x_scales, w, w_scales, y, stream=None):
    t = _Tensors(cfg, "fl_moe_expert_product_e4m3")
    _check(lib().fl_moe_expert_product_e4m3(
        C.byref(cfg), rank_begin, rank_count, *t.tables(expert_off, tokens_per_expert), in_features, out_features,
        t(x, _E4M3, t.rows * in_features), t(x_scales, _F32, t.rows * in_features // 128),
        t(w, _E4M3, t.experts * in_features * out_features),
        t(w_scales, _F32, t.experts * ((out_features + 127) // 128) * (in_features // 128)),
        t(y, _BF16, t.rows * out_features), _stream(stream)), t.where)


def fl_moe_status(ctx, stream=None) -> int:
    v = C.c_int32(0)
    _check(lib().fl_moe_status(ctx, C.byref(v), _stream(stream)), "fl_moe_status")
    return v.value


def fl_moe_reset(ctx, stream=None):
    _check(lib().fl_moe_reset(ctx, _stream(stream)), "fl_moe_reset")


def fl_moe_required_capacities(ctx, stream=None):
    """(recv_capacity_rows, expert_capacity_rows) the last step needs."""
    recv, expert = C.c_int64(), C.c_int64()
    _check(lib().fl_moe_required_capacities(ctx, C.byref(recv), C.byref(expert), _stream(stream)),
           "fl_moe_required_capacities")
    return recv.value, expert.value


def fl_moe_debug_views(ctx) -> fl_moe_debug_view:
    out = fl_moe_debug_view()
    _check(lib().fl_moe_debug_views(ctx, C.byref(out)), "fl_moe_debug_views")
    return out


def fl_moe_debug_tune(ctx, knob, value):
    _check(lib().fl_moe_debug_tune(ctx, knob, value), "fl_moe_debug_tune")


def fl_moe_debug_launch_groups(cfg: fl_moe_config, rank_count: int, launch_mb: int = -1) -> int:
    out = C.c_int(0)
    _check(lib().fl_moe_debug_launch_groups(C.byref(cfg), rank_count, launch_mb, C.byref(out)),
           "fl_moe_debug_launch_groups")
    return out.value


def fl_moe_debug_launch_plan(cfg: fl_moe_config, rank_count: int) -> fl_moe_launch_plan:
    out = fl_moe_launch_plan()
    _check(lib().fl_moe_debug_launch_plan(C.byref(cfg), rank_count, C.byref(out)), "fl_moe_debug_launch_plan")
    return out


def fl_moe_debug_ordering_plan(cfg: fl_moe_config, rank_count: int, cached_mb: int = -1) -> fl_moe_ordering_plan:
    out = fl_moe_ordering_plan()
    _check(lib().fl_moe_debug_ordering_plan(C.byref(cfg), rank_count, cached_mb, C.byref(out)),
           "fl_moe_debug_ordering_plan")
    return out


def fl_moe_debug_row_strides(cfg: fl_moe_config):
    """(dispatch, combine): bytes from row to row of the receive buffers."""
    dispatch, combine = C.c_int64(), C.c_int64()
    _check(lib().fl_moe_debug_row_strides(C.byref(cfg), C.byref(dispatch), C.byref(combine)), "fl_moe_debug_row_strides")
    return dispatch.value, combine.value


def fl_moe_debug_copy(dst, src, nbytes, stream=None):
    _check(lib().fl_moe_debug_copy(_ptr(dst), _ptr(src), nbytes, _stream(stream)),
           "fl_moe_debug_copy")


def fl_moe_debug_fill(dst, nbytes, stream=None):
    _check(lib().fl_moe_debug_fill(_ptr(dst), nbytes, _stream(stream)), "fl_moe_debug_fill")


def fl_moe_debug_read(src, nbytes, sink, stream=None):
    _check(lib().fl_moe_debug_read(_ptr(src), nbytes, _ptr(sink), _stream(stream)), "fl_moe_debug_read")


def fl_moe_build_id() -> str:
    return lib().fl_moe_build_id().decode()


def fl_moe_profile_enable(ctx, on):
    _check(lib().fl_moe_profile_enable(ctx, int(on)), "fl_moe_profile_enable")


def fl_moe_profile_collect(ctx, stream=None):
    _check(lib().fl_moe_profile_collect(ctx, _stream(stream)), "fl_moe_profile_collect")


def fl_moe_profile_read(ctx):
    ms = (C.c_double * FL_KERNEL_COUNT)()
    n = (C.c_int64 * FL_KERNEL_COUNT)()
    _check(lib().fl_moe_profile_read(ctx, ms, n), "fl_moe_profile_read")
    return {lib().fl_moe_kernel_name(i).decode(): (ms[i], n[i]) for i in range(FL_KERNEL_COUNT)}


# ------------------------------------------------------------------ convenience wrapper
class MoEShuffle:
    """Owns the device memory of one context (workspace and outputs) and forwards
    to the C calls.  No arithmetic happens here."""

    def __init__(self, n_ranks, n_experts, max_tokens, top_k, hidden, dispatch_dtype="bf16",
                 expert_align=1, zero_pad=False, recv_capacity_rows=0, expert_capacity_rows=0,
                 spin_limit=0, stream_ordered=False, max_private_rows=0, peer_push=False,
                 partial_sums=False, progressive_recv=False, device="cuda:0"):
        self.device = torch.device(device)
        self.cfg = fl_moe_config(
            n_ranks, n_experts, max_tokens, top_k, hidden,
            FL_DTYPE_BF16 if dispatch_dtype == "bf16" else FL_DTYPE_E4M3_BLOCK128,
            expert_align, (FL_FLAG_ZERO_PAD if zero_pad else 0)
            | (FL_FLAG_STREAM_ORDERED if stream_ordered else 0)
            | (FL_FLAG_PEER_PUSH if peer_push else 0)
            | (FL_FLAG_PARTIAL_SUMS if partial_sums else 0)
            | (FL_FLAG_PROGRESSIVE_RECV if progressive_recv else 0),
            recv_capacity_rows, expert_capacity_rows, spin_limit, max_private_rows, 0)
        self.partial_sums = bool(partial_sums)
        self.sizes = fl_moe_query_sizes(self.cfg)
        self.N, self.E, self.T, self.K, self.H = n_ranks, n_experts, max_tokens, top_k, hidden
        self.El = n_experts // n_ranks
        self.workspace = torch.empty(self.sizes.workspace_bytes, dtype=torch.uint8,
                                     device=self.device)
        self.ctx = fl_moe_create(self.cfg, self.workspace)
        cap = self.sizes.expert_capacity_rows
        self.expert_capacity_rows = cap
        if dispatch_dtype == "bf16":
            self.expert_x = torch.empty((n_ranks, cap, hidden), dtype=torch.bfloat16,
                                        device=self.device)
            self.expert_scales = None
        else:
            self.expert_x = torch.empty((n_ranks, cap, hidden), dtype=torch.uint8,
                                        device=self.device)
            self.expert_scales = torch.empty((n_ranks, cap, hidden // 128), dtype=torch.float32,
                                             device=self.device)
        self.tokens_per_expert = torch.zeros((n_ranks, self.El), dtype=torch.int32,
                                             device=self.device)
        self.out = torch.empty((n_ranks, max_tokens, hidden), dtype=torch.bfloat16,
                               device=self.device)
        self.view = None

    def close(self):
        if self.ctx is not None:
            torch.cuda.synchronize(self.device)
            fl_moe_destroy(self.ctx)
            self.ctx = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _ranks(self, ranks):
        return (0, self.N) if ranks is None else ranks

    def layout(self, indices, num_tokens, ranks=None, stream=None):
        self._indices, self._num_tokens = indices, num_tokens      # keep alive for the step
        rb, rc = self._ranks(ranks)
        self.view = fl_moe_layout(self.ctx, rb, rc, indices, num_tokens, stream)
        return self.view

    def dispatch_send(self, x, ranks=None, stream=None, weights=None, scales=None):
        rb, rc = self._ranks(ranks)
        if scales is not None:          # x holds e4m3 codes the caller quantised itself
            fl_moe_dispatch_send_e4m3(self.ctx, rb, rc, x, scales, weights, stream)
        elif weights is None:
            fl_moe_dispatch_send(self.ctx, rb, rc, x, stream)
        else:
            fl_moe_dispatch_send_weighted(self.ctx, rb, rc, x, weights, stream)

    def dispatch_recv(self, ranks=None, stream=None):
        rb, rc = self._ranks(ranks)
        fl_moe_dispatch_recv(self.ctx, rb, rc, self.expert_x, self.expert_scales,
                             self.tokens_per_expert, stream)
        return self.expert_x

    def combine_send(self, expert_y, ranks=None, stream=None):
        rb, rc = self._ranks(ranks)
        fl_moe_combine_send(self.ctx, rb, rc, expert_y, stream)

    def combine_reduce(self, weights, ranks=None, stream=None, out=None):
        rb, rc = self._ranks(ranks)
        fl_moe_combine_reduce(self.ctx, rb, rc, weights, self.out if out is None else out, stream)
        return self.out if out is None else out

    def status(self):
        return fl_moe_status(self.ctx)

    def required_capacities(self):
        return fl_moe_required_capacities(self.ctx)

    def reset(self):
        fl_moe_reset(self.ctx)

    def table(self, ptr, shape, dtype=torch.int32):
        """A tensor view of a table inside the workspace (for parity checks)."""
        off = ptr - self.workspace.data_ptr()
        n = 1
        for s in shape:
            n *= s
        nbytes = n * torch.empty((), dtype=dtype).element_size()
        assert 0 <= off and off + nbytes <= self.workspace.numel()
        return self.workspace[off:off + nbytes].view(dtype).reshape(shape)

    def layout_tables(self):
        v, N, E, El, T, K = self.view, self.N, self.E, self.El, self.T, self.K
        return {
            "C": self.table(v.counts, (N, E)),
            "M": self.table(v.dedup_counts, (N, N)),
            "G": self.table(v.tokens_per_expert, (N, El)),
            "send_off": self.table(v.send_off, (N, N + 1)),
            "recv_off": self.table(v.recv_off, (N, N + 1)),
            "expert_off": self.table(v.expert_off, (N, El + 1)),
            "comb_off": self.table(v.comb_off, (N, N + 1)),
            "comb_pos": self.table(v.comb_pos, (N, T, K)),
            "plan_ok": self.table(v.plan_ok, (N,)),
        }

    def debug(self):
        dv = fl_moe_debug_views(self.ctx)
        N = self.N
        return {
            "arrive_route": self.table(dv.arrive_route, (N, N)),
            "arrive_disp": self.table(dv.arrive_disp, (N, N)),
            "arrive_comb": self.table(dv.arrive_comb, (N, N)),
            "epoch_route": self.table(dv.epoch_route, (N,)),
            "expect_disp": self.table(dv.expect_disp, (N, N)),
            "expect_comb": self.table(dv.expect_comb, (N, N)),
            "buf_a": self.table(dv.buf_a, (N, dv.buf_a_rank_bytes), torch.uint8),
            "buf_b": self.table(dv.buf_b, (N, dv.buf_b_rank_bytes), torch.uint8),
        }


class MoEExperts:
    """The experts of one layer between dispatch_recv and combine_send of a MoEShuffle: owns their rows' buffers and
    forwards to the C calls.  No arithmetic happens here.

    inter: width of the gated block; w_in [E][2 * inter][hidden] (gates, then ups), w_out [E][hidden][inter]; bf16, or for
    a shuffle with e4m3 dispatch e4m3 codes with the scales of their 128 x 128 blocks (inference only).
    training: keeps what the backward pass needs: the pre-activations in bf16 or, keep="e4m3", in 8-bit blocks (then the
    block's output is not kept either, but worked out again), and copies of the step's tables, so that other layers'
    steps may run in between.  The rows themselves (expert_x) are the caller's to keep."""

    def __init__(self, shuffle, inter, activation="silu", training=False, keep="bf16"):
        self.shuffle, self.inter, self.training, self.keep = shuffle, inter, training, keep
        if activation not in ("silu", "gelu"):
            raise FlMoeError(FL_ERR_INVALID_ARG, f"MoEExperts: activation is silu or gelu, got {activation!r}")
        self.activation = FL_ACT_SILU if activation == "silu" else FL_ACT_GELU
        self.e4m3 = shuffle.expert_scales is not None
        if keep not in ("bf16", "e4m3") or (training and self.e4m3):
            raise FlMoeError(FL_ERR_INVALID_ARG, "MoEExperts: rows of e4m3 have no backward pass; keep is bf16 or e4m3")

        def rows(width, dtype=torch.bfloat16):
            return torch.empty((shuffle.N, shuffle.expert_capacity_rows, width), dtype=dtype, device=shuffle.device)
        self.h = rows(inter, torch.uint8 if self.e4m3 else torch.bfloat16)
        self.h_scales = rows(inter // 128, torch.float32) if self.e4m3 else None
        self.y = rows(shuffle.H)
        self.pre = self.pre_scales = self.tables = None
        if training:
            eights = keep == "e4m3"
            self.pre = rows(2 * inter, torch.uint8 if eights else torch.bfloat16)
            self.pre_scales = rows(2 * inter // 128, torch.float32) if eights else None
            # the pre-activations' gradients take the place of what was kept where they fit
            self.dpre = rows(2 * inter) if eights else self.pre
            self.dh, self.dx = rows(inter), rows(shuffle.H)
            self.tables = [torch.zeros((shuffle.N, n), dtype=torch.int32, device=shuffle.device) for n in (shuffle.El + 1, shuffle.El)]
            # of each rank: whether there is something kept for a backward pass; None once a forward pass was captured, whose
            # replays are not seen here
            self._kept = [False] * shuffle.N

    def _stream(self, stream):
        if stream is None:
            return torch.cuda.current_stream(self.shuffle.device)
        return stream if hasattr(stream, "cuda_stream") else torch.cuda.ExternalStream(int(stream), device=self.shuffle.device)

    def _keep(self, rb, rc, kept):
        self._kept[rb:rb + rc] = [None if was is None or kept is None else kept for was in self._kept[rb:rb + rc]]

    def _at(self, ranks):
        rb, rc = self.shuffle._ranks(ranks)
        return (self.shuffle.cfg, rb, rc, *self.tables)

    def forward(self, w_in, w_out, in_scales=None, out_scales=None, x=None, ranks=None, stream=None, x_scales=None):
        """y of the rows that dispatch_recv left (x, and of e4m3 rows x_scales: of other rows in that layout)."""
        sh = self.shuffle
        if (x_scales is not None) != (x is not None and self.e4m3):
            raise FlMoeError(FL_ERR_INVALID_ARG, "MoEExperts.forward: other rows of e4m3 come with their scales")
        if self.training:
            rb, rc = sh._ranks(ranks)                    # only theirs: the others' may be on their way on other streams
            with torch.cuda.stream(self._stream(stream)):
                captured = torch.cuda.is_current_stream_capturing()
                self._keep(rb, rc, None if captured else False)
                for mine, now in zip(self.tables, (sh.layout_tables()[t] for t in ("expert_off", "G"))):
                    mine[rb:rb + rc].copy_(now[rb:rb + rc])
        else:
            self.tables = (sh.view.expert_off, sh.view.tokens_per_expert)
        at, x = self._at(ranks), sh.expert_x if x is None else x
        if self.e4m3:
            fl_moe_expert_gated_e4m3(*at, self.inter, self.activation, x, sh.expert_scales if x_scales is None else x_scales,
                                     w_in, in_scales, self.h, self.h_scales, stream)
            fl_moe_expert_product_e4m3(*at, self.inter, sh.H, self.h, self.h_scales, w_out, out_scales, self.y, stream)
        else:
            fl_moe_expert_gated(*at, self.inter, self.activation, x, w_in, self.h, self.pre, self.pre_scales, stream)
            fl_moe_expert_product(*at, self.inter, sh.H, self.h, w_out, self.y, stream)
        if self.training:
            self._keep(rb, rc, True)
        return self.y

    def backward(self, dy, w_in, w_out, dw_in, dw_out, x=None, ranks=None, stream=None):
        """The rows' gradient; the weights' go to dw_in and dw_out.  x: the rows that forward had.  Once per forward of these
        ranks with keep="bf16": the kept pre-activations are gone then, another call is refused.  (Calls captured into a graph,
        and those behind a captured forward, are not checked: their replays are the caller's to keep in turn.)"""
        if not self.training:
            raise FlMoeError(FL_ERR_INVALID_ARG, "MoEExperts.backward: nothing was kept, training was not asked for")
        sh, at = self.shuffle, self._at(ranks)
        rb, rc = at[1:3]
        with torch.cuda.stream(self._stream(stream)):
            captured = torch.cuda.is_current_stream_capturing()
        if not captured and False in self._kept[rb:rb + rc]:
            raise FlMoeError(FL_ERR_INVALID_ARG, "MoEExperts.backward: nothing is kept of these ranks' rows: no forward pass, or its "
                             "backward pass has been")
        x = sh.expert_x if x is None else x
        again = self.h if self.keep == "e4m3" else None
        fl_moe_expert_product_backward(*at, self.inter, sh.H, self.h, w_out, dy, self.dh, None if again is not None else dw_out,
                                       stream)
        fl_moe_expert_gated_backward(*at, self.inter, self.activation, x, w_in, self.pre, self.pre_scales, self.dh, self.dpre,
                                     self.dx, dw_in, again, stream)
        if not captured and self.dpre is self.pre:
            self._keep(rb, rc, False)
        if again is not None:
            fl_moe_expert_product_backward(*at, self.inter, sh.H, again, None, dy, None, dw_out, stream)
        return self.dx
