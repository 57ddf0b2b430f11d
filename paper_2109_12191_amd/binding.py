"""ctypes binding of libdp_privatise.so: same names as the C ABI, argument marshalling only."""
from __future__ import annotations

import ctypes as C
import os
from typing import Optional

DP_OK, DP_ERR_INVALID_ARG, DP_ERR_UNSUPPORTED, DP_ERR_WORKSPACE, DP_ERR_DEVICE = range(5)
DP_DENSE, DP_CONV2D, DP_GN_AFFINE = 0, 1, 2
DP_F32, DP_BF16 = 0, 1
DP_NCHW, DP_NHWC = 0, 1
DP_WS_PER_EXAMPLE_GRAD, DP_WS_RECOMPUTE = 0, 1
DP_VARIANT_SHARED = 2
DP_VARIANT_MATERIALISE = 4
DP_RECOMPUTE_BLOCKS = 8
DP_QUERIES_AT_END = -1

_STATUS_NAMES = {1: "DP_ERR_INVALID_ARG", 2: "DP_ERR_UNSUPPORTED", 3: "DP_ERR_WORKSPACE", 4: "DP_ERR_DEVICE"}
_KINDS = {"dense": DP_DENSE, "conv": DP_CONV2D, "gn": DP_GN_AFFINE}

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_HERE, "libdp_privatise.so")
_lib = None


class DpError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"{_STATUS_NAMES.get(status, status)}: {message}")
        self.status = status


class LayerDesc(C.Structure):
    """Mirror of dp_layer_desc."""
    _fields_ = [("kind", C.c_int), ("in_dtype", C.c_int), ("layout", C.c_int), ("n", C.c_int),
                ("cin", C.c_int), ("cout", C.c_int), ("h", C.c_int), ("w", C.c_int),
                ("kh", C.c_int), ("kw", C.c_int), ("stride", C.c_int), ("pad", C.c_int),
                ("has_bias", C.c_int), ("gn_groups", C.c_int), ("gn_eps", C.c_float)]


class BiasDesc(C.Structure):
    """Mirror of dp_bias_desc."""
    _fields_ = [("in_dtype", C.c_int), ("n", C.c_int), ("heads", C.c_int), ("queries", C.c_int), ("keys", C.c_int),
                ("buckets", C.c_int), ("max_distance", C.c_int), ("bidirectional", C.c_int), ("causal", C.c_int),
                ("query_offset", C.c_int), ("scale", C.c_float), ("row_stride", C.c_size_t)]


class NormDesc(C.Structure):
    """Mirror of dp_norm_desc."""
    _fields_ = [("in_dtype", C.c_int), ("n", C.c_int), ("tokens", C.c_int), ("features", C.c_int), ("rms", C.c_int), ("eps", C.c_float),
                ("row_stride", C.c_size_t)]


class LogprobDesc(C.Structure):
    """Mirror of dp_logprob_desc."""
    _fields_ = [("in_dtype", C.c_int), ("n", C.c_int), ("tokens", C.c_int), ("vocab", C.c_int), ("top", C.c_int), ("scale", C.c_float),
                ("row_stride", C.c_size_t)]


def lib_path() -> str:
    return _LIB_PATH


def load_library():
    """Load the HIP library.  Raises if it has not been built: there is no fallback path."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(_LIB_PATH):
        raise RuntimeError(f"{_LIB_PATH} is missing: build it with `python -m paper_2109_12191_amd.build` "
                           "(or __graft_entry__.build()); there is no CPU fallback")
    lib = C.CDLL(_LIB_PATH)
    vp, sz, u64, u32, fl, it = C.c_void_p, C.c_size_t, C.c_uint64, C.c_uint32, C.c_float, C.c_int
    dpp, dbp, dnp, dlp = C.POINTER(LayerDesc), C.POINTER(BiasDesc), C.POINTER(NormDesc), C.POINTER(LogprobDesc)
    sigs = {
        "dp_group_clip_bounds": (it, [fl, it, vp, vp]),
        "dp_weight_count": (sz, [dpp]),
        "dp_bias_count": (sz, [dpp]),
        "dp_workspace_bytes": (sz, [dpp, it]),
        "dp_kernel_variant": (C.c_char_p, [dpp, it]),
        "dp_per_example_grad": (it, [dpp, vp, vp, vp, vp, sz, vp, vp, sz, vp]),
        "dp_static_scratch_bytes": (sz, []),
        "dp_per_example_grad_static": (it, [dpp, vp, vp, vp, vp, sz, vp, vp]),
        "dp_norms": (it, [vp, vp, it, it, it, vp, vp]),
        "dp_norm_partial_count": (sz, [dpp, it]),
        "dp_unit_workspace_bytes": (sz, [dpp, it]),
        "dp_batch_workspace_bytes": (sz, [dpp, it, it]),
        "dp_unit_grad": (it, [dpp, it, vp, vp, vp, vp, sz, vp, vp, sz, vp]),
        "dp_unit_grad_batch": (it, [vp, it, vp, vp, vp, vp, sz, vp, vp, vp, it, vp]),
        "dp_per_example_grad_partials": (it, [dpp, vp, vp, vp, vp, sz, vp, sz, vp]),
        "dp_norms_from_partials": (it, [vp, vp, vp, it, it, it, vp, vp]),
        "dp_per_example_grad_batch": (it, [vp, vp, vp, vp, vp, sz, vp, vp, vp, vp, it, vp]),
        "dp_layer_norms_from_partials": (it, [vp, vp, vp, it, it, vp]),
        "dp_clip_accumulate_recompute_batch": (it, [vp, vp, vp, vp, vp, vp, vp, vp, vp, it, vp]),
        "dp_example_addresses": (it, [vp, vp, it, it, it, vp, vp]),
        "dp_per_example_grad_blocks_batch_at": (it, [vp, vp, vp, vp, vp, sz, vp, vp, vp, vp, it, vp]),
        "dp_per_example_grad_batch_at": (it, [vp, vp, vp, vp, vp, sz, vp, vp, vp, vp, it, vp]),
        "dp_clip_accumulate_recompute_batch_at": (it, [vp, vp, vp, vp, vp, vp, vp, vp, vp, it, vp]),
        "dp_clip_accumulate_recompute_blocks_batch_at": (it, [vp, vp, vp, vp, vp, vp, vp, vp, vp, it, vp]),
        "dp_unit_grad_batch_at": (it, [vp, it, vp, vp, vp, vp, sz, vp, vp, vp, it, vp]),
        "dp_clip_accumulate_columns": (it, [vp, sz, vp, it, vp, vp, vp, vp, it, it, it, sz, vp, vp]),
        "dp_clip_factors": (it, [vp, fl, it, vp, vp]),
        "dp_clip_accumulate": (it, [vp, sz, vp, fl, it, sz, vp, vp]),
        "dp_clip_accumulate_segments": (it, [vp, sz, vp, it, vp, vp, vp, it, it, sz, vp, vp]),
        "dp_clip_accumulate_recompute": (it, [dpp, vp, vp, vp, fl, vp, vp, vp, sz, vp]),
        "dp_add_noise_finalize": (it, [vp, vp, sz, fl, fl, u64, u64, u64, u32, vp]),
        "dp_add_example_noise": (it, [vp, sz, fl, fl, u64, u64, u64, u32, u64, it, vp, vp]),
        "dp_add_noise_finalize_update": (it, [vp, vp, vp, vp, sz, fl, fl, u64, u64, u64, u32, fl, fl, vp]),
        "dp_add_noise_finalize_flat": (it, [vp, vp, vp, vp, vp, vp, vp, it, fl, fl, u64, u64, u64, vp, fl, fl, vp]),
        "dp_philox_raw": (it, [vp, sz, u64, u64, u32, vp]),
        "dp_checkpoint_pitch": (it, [it]),
        "dp_checkpoint_write": (it, [vp, it, sz, it, sz, vp, vp, vp]),
        "dp_checkpoint_read": (it, [vp, vp, sz, it, vp, it, sz, vp]),
        "dp_checkpoint_workspace_bytes": (sz, [dpp, it]),
        "dp_checkpoint_example_grad": (it, [dpp, vp, vp, vp, vp, vp, vp, sz, vp, vp, sz, vp]),
        "dp_checkpoint_clip_accumulate": (it, [dpp, vp, vp, vp, vp, vp, fl, vp, vp, vp, sz, vp]),
        "dp_bias_bucket": (it, [dbp, it]),
        "dp_bias_softmax": (it, [dbp, vp, vp, vp, vp, vp, vp]),
        "dp_bias_workspace_bytes": (sz, [dbp]),
        "dp_bias_softmax_backward": (it, [dbp, vp, vp, vp, vp, vp, vp, sz, vp, vp, sz, vp]),
        "dp_layer_norm": (it, [dnp, vp, vp, vp, vp, vp, vp]),
        "dp_layer_norm_workspace_bytes": (sz, [dnp]),
        "dp_layer_norm_backward": (it, [dnp, vp, vp, vp, vp, vp, vp, vp, sz, vp, vp, sz, vp]),
        "dp_token_logprobs_workspace_bytes": (sz, [dlp]),
        "dp_token_logprobs": (it, [dlp, vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]),
        "dp_token_logprobs_backward": (it, [dlp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]),
        "dp_profile_next_contraction": (it, [vp, vp]),
        "dp_last_error": (C.c_char_p, []),
        "dp_version": (C.c_char_p, []),
    }
    for name, (res, args) in sigs.items():
        fn = getattr(lib, name)
        fn.restype = res
        fn.argtypes = args
    _lib = lib
    return lib


EXPORTED = ("dp_group_clip_bounds", "dp_weight_count", "dp_bias_count", "dp_workspace_bytes", "dp_kernel_variant", "dp_per_example_grad", "dp_norms",
            "dp_static_scratch_bytes", "dp_per_example_grad_static",
            "dp_unit_workspace_bytes", "dp_batch_workspace_bytes", "dp_unit_grad", "dp_unit_grad_batch",
            "dp_norm_partial_count", "dp_per_example_grad_partials", "dp_norms_from_partials",
            "dp_per_example_grad_batch", "dp_layer_norms_from_partials", "dp_clip_accumulate_recompute_batch",
            "dp_example_addresses", "dp_per_example_grad_batch_at", "dp_per_example_grad_blocks_batch_at", "dp_clip_accumulate_recompute_batch_at", "dp_clip_accumulate_recompute_blocks_batch_at", "dp_unit_grad_batch_at",
            "dp_clip_accumulate_columns",
            "dp_clip_factors", "dp_clip_accumulate", "dp_clip_accumulate_segments", "dp_clip_accumulate_recompute", "dp_add_noise_finalize", "dp_add_noise_finalize_update", "dp_add_example_noise",
            "dp_checkpoint_pitch", "dp_checkpoint_write", "dp_checkpoint_read", "dp_checkpoint_workspace_bytes", "dp_checkpoint_example_grad",
            "dp_checkpoint_clip_accumulate", "dp_bias_bucket", "dp_bias_softmax", "dp_bias_workspace_bytes", "dp_bias_softmax_backward",
            "dp_layer_norm", "dp_layer_norm_workspace_bytes", "dp_layer_norm_backward",
            "dp_token_logprobs_workspace_bytes", "dp_token_logprobs", "dp_token_logprobs_backward",
            "dp_add_noise_finalize_flat", "dp_philox_raw", "dp_profile_next_contraction", "dp_last_error", "dp_version")


def make_desc(layer, n: int, dtype: str = "f32", layout: int = DP_NCHW) -> LayerDesc:
    """dp_layer_desc from a workload layer (anything with kind/cin/cout/h/w/kh/kw/stride/pad/...)."""
    return LayerDesc(_KINDS[layer.kind], DP_BF16 if dtype == "bf16" else DP_F32, layout, n,
                     layer.cin, layer.cout, layer.h, layer.w, layer.kh, layer.kw, layer.stride, layer.pad,
                     int(bool(layer.has_bias)), layer.gn_groups, float(layer.gn_eps))


def _ptr(t) -> Optional[int]:
    if t is None:
        return None
    if isinstance(t, int):
        return t
    return t.data_ptr()


def _nbytes(t) -> int:
    return 0 if t is None else t.numel() * t.element_size()


def _stream(stream) -> Optional[int]:
    if stream is not None:
        return stream if isinstance(stream, int) else stream.cuda_stream
    import torch
    current = getattr(torch._C, "_cuda_getCurrentRawStream", None)      # the handle without a Stream object around it: 0.3 us for 2.8
    if current is not None:
        return current(torch.cuda.current_device())
    return torch.cuda.current_stream().cuda_stream


def _check(status: int):
    if status != DP_OK:
        raise DpError(status, dp_last_error())


def dp_last_error() -> str:
    return load_library().dp_last_error().decode()


def dp_version() -> str:
    return load_library().dp_version().decode()


def dp_group_clip_bounds(clip_c: float, n_groups: int):
    """(list of per-group bounds, bound on the whole clipped gradient), both computed by the library."""
    gc = (C.c_float * max(n_groups, 1))()
    tot = C.c_float()
    _check(load_library().dp_group_clip_bounds(clip_c, n_groups, C.cast(gc, C.c_void_p), C.cast(C.byref(tot), C.c_void_p)))
    return [float(v) for v in gc], float(tot.value)


def dp_weight_count(desc: LayerDesc) -> int:
    return int(load_library().dp_weight_count(C.byref(desc)))


def dp_bias_count(desc: LayerDesc) -> int:
    return int(load_library().dp_bias_count(C.byref(desc)))


def dp_workspace_bytes(desc: LayerDesc, use: int = DP_WS_PER_EXAMPLE_GRAD) -> int:
    return int(load_library().dp_workspace_bytes(C.byref(desc), use))


def dp_kernel_variant(desc: LayerDesc, use: int = DP_WS_PER_EXAMPLE_GRAD) -> str:
    return load_library().dp_kernel_variant(C.byref(desc), use).decode()


def dp_per_example_grad(desc, x, dy, g_w, g_b, sqnorm, ws, g_stride: int = 0, ws_bytes: Optional[int] = None,
                        stream=None):
    _check(load_library().dp_per_example_grad(C.byref(desc), _ptr(x), _ptr(dy), _ptr(g_w), _ptr(g_b), g_stride,
                                              _ptr(sqnorm), _ptr(ws),
                                              _nbytes(ws) if ws_bytes is None else ws_bytes, _stream(stream)))


def dp_static_scratch_bytes() -> int:
    return int(load_library().dp_static_scratch_bytes())


def dp_per_example_grad_static(desc, x, dy, g_w, g_b, sqnorm, g_stride: int = 0, stream=None):
    _check(load_library().dp_per_example_grad_static(C.byref(desc), _ptr(x), _ptr(dy), _ptr(g_w), _ptr(g_b), g_stride,
                                                     _ptr(sqnorm), _stream(stream)))


def dp_norm_partial_count(desc, materialise: bool) -> int:
    return int(load_library().dp_norm_partial_count(C.byref(desc), 1 if materialise else 0))


def dp_per_example_grad_partials(desc, x, dy, g_w, g_b, ws, g_stride: int = 0, ws_bytes: Optional[int] = None,
                                 stream=None):
    _check(load_library().dp_per_example_grad_partials(C.byref(desc), _ptr(x), _ptr(dy), _ptr(g_w), _ptr(g_b),
                                                       g_stride, _ptr(ws),
                                                       _nbytes(ws) if ws_bytes is None else ws_bytes, _stream(stream)))


class PartialTable:
    """Host arrays for dp_norms_from_partials, built once: device pointers of every layer's partial
    sums (the start of its workspace), their per-example counts and the layer -> group map."""

    def __init__(self, pointers, counts, groups):
        n = len(pointers)
        self.n_layers = n
        self.ptrs = (C.c_void_p * n)(*[int(p) for p in pointers])
        self.counts = (C.c_int32 * n)(*[int(c) for c in counts])
        self.groups = (C.c_int32 * n)(*[int(g) for g in groups])


def dp_norms_from_partials(table: "PartialTable", n: int, n_groups: int, group_sqnorm, stream=None):
    _check(load_library().dp_norms_from_partials(C.cast(table.ptrs, C.c_void_p), C.cast(table.counts, C.c_void_p),
                                                 C.cast(table.groups, C.c_void_p), table.n_layers, n, n_groups,
                                                 _ptr(group_sqnorm), _stream(stream)))


def dp_batch_workspace_bytes(desc: LayerDesc, use: int = DP_WS_PER_EXAMPLE_GRAD, clip_unit: int = 1) -> int:
    """Workspace with which a layer of a batch call runs its fastest route."""
    return int(load_library().dp_batch_workspace_bytes(C.byref(desc), use, clip_unit))


def dp_unit_workspace_bytes(desc: LayerDesc, clip_unit: int) -> int:
    return int(load_library().dp_unit_workspace_bytes(C.byref(desc), clip_unit))


def dp_unit_grad(desc: LayerDesc, clip_unit: int, x, dy, g_w, g_b, sqnorm, ws, g_stride: int = 0, stream=None):
    """Sums of the per-example gradients over clipping units of clip_unit consecutive examples, and the squared
    norms of the sums ([n / clip_unit])."""
    _check(load_library().dp_unit_grad(C.byref(desc), clip_unit, _ptr(x), _ptr(dy), _ptr(g_w), _ptr(g_b), g_stride,
                                       _ptr(sqnorm), _ptr(ws), _nbytes(ws), _stream(stream)))


class LayerBatch:
    """Host arrays for the batch calls over a fixed set of layers: descriptors, workspaces, and (re)settable
    pointer arrays.  Pointers are plain integers (device addresses); None becomes NULL.  scale_blocks: the calls on example addresses
    work on finished blocks (sums of squares as norms, clipped sums that scale blocks)."""

    def __init__(self, descs, ws_ptrs, ws_bytes, scale_blocks: bool = False):
        self.scale_blocks = scale_blocks
        k = len(descs)
        self.n_layers = k
        self.descs = (LayerDesc * k)(*descs)
        self.ws = (C.c_void_p * k)(*[int(p) for p in ws_ptrs])
        self.ws_bytes = (C.c_size_t * k)(*[int(b) for b in ws_bytes])
        self.partial_counts = (C.c_int32 * k)()          # written by dp_per_example_grad_batch
        self._kept = {}

    def fill(self, key, values):
        """An array of device addresses that is kept and overwritten by the next fill of the same key (the library reads it
        before its call returns)."""
        arr = self._kept.get(key)
        if arr is None:
            arr = self._kept[key] = (C.c_void_p * self.n_layers)()
        arr[:] = values
        return arr

    def ptrs(self, values):
        assert len(values) == self.n_layers
        return (C.c_void_p * self.n_layers)(*[(None if v is None else int(v)) for v in values])

    def floats(self, values):
        assert len(values) == self.n_layers
        return (C.c_float * self.n_layers)(*[float(v) for v in values])


def dp_example_addresses(tensors, example_bytes, n_operands: int, n_tensors: int, per_tensor: int, table, stream=None):
    """tensors: n_operands * n_tensors device addresses; example_bytes: n_operands integers; table: a device int64 tensor (or its
    address) that receives n_operands * n_tensors * per_tensor example addresses."""
    _check(load_library().dp_example_addresses((C.c_void_p * len(tensors))(*tensors), (C.c_size_t * len(example_bytes))(*example_bytes),
                                               n_operands, n_tensors, per_tensor, _ptr(table), _stream(stream)))


def dp_per_example_grad_batch(batch: "LayerBatch", x, dy, g_w, g_b, sqnorm, g_stride: int = 0, stream=None, addresses: bool = False):
    """x, dy: ctypes pointer arrays from batch.ptrs() (addresses=True: of arrays of example addresses); g_w, g_b, sqnorm: the
    same or None (sqnorm None: the per-layer reduction is left to dp_layer_norms_from_partials).  batch.partial_counts receives
    the number of partial sums per example each layer left at the start of its workspace."""
    lib = load_library()
    _check((lib.dp_per_example_grad_blocks_batch_at if addresses and batch.scale_blocks else
            lib.dp_per_example_grad_batch_at if addresses else lib.dp_per_example_grad_batch)(
        batch.descs, x, dy, g_w, g_b, g_stride, sqnorm, batch.ws, batch.ws_bytes, batch.partial_counts, batch.n_layers, _stream(stream)))


def dp_unit_grad_batch(batch: "LayerBatch", clip_unit: int, x, dy, g_w, g_b, sqnorm, g_stride: int = 0, stream=None,
                       addresses: bool = False):
    """dp_unit_grad for the layers of a LayerBatch; x, dy, sqnorm: ctypes pointer arrays from batch.ptrs()."""
    lib = load_library()
    _check((lib.dp_unit_grad_batch_at if addresses else lib.dp_unit_grad_batch)(
        batch.descs, clip_unit, x, dy, g_w, g_b, g_stride, sqnorm, batch.ws, batch.ws_bytes, batch.n_layers, _stream(stream)))


def dp_layer_norms_from_partials(partials, counts, sqnorm, n_layers: int, n: int, stream=None):
    """partials, sqnorm: ctypes arrays of n_layers device pointers; counts: ctypes int32 array."""
    _check(load_library().dp_layer_norms_from_partials(C.cast(partials, C.c_void_p), C.cast(counts, C.c_void_p),
                                                       C.cast(sqnorm, C.c_void_p), n_layers, n, _stream(stream)))


def dp_clip_accumulate_recompute_batch(batch: "LayerBatch", x, dy, sqnorm, clip_c, acc_w, acc_b, stream=None, addresses: bool = False):
    lib = load_library()
    if batch.scale_blocks and not addresses:
        raise ValueError("the clipped sum that scales finished blocks takes example addresses")
    _check((lib.dp_clip_accumulate_recompute_blocks_batch_at if batch.scale_blocks else
            lib.dp_clip_accumulate_recompute_batch_at if addresses else lib.dp_clip_accumulate_recompute_batch)(
        batch.descs, x, dy, sqnorm, clip_c, acc_w, acc_b, batch.ws, batch.ws_bytes, batch.n_layers, _stream(stream)))


def dp_norms(layer_sqnorm, group_of_layer, n_layers: int, n: int, n_groups: int, group_sqnorm, stream=None):
    _check(load_library().dp_norms(_ptr(layer_sqnorm), _ptr(group_of_layer), n_layers, n, n_groups,
                                   _ptr(group_sqnorm), _stream(stream)))


def dp_clip_factors(sqnorm, clip_c: float, n: int, f, stream=None):
    _check(load_library().dp_clip_factors(_ptr(sqnorm), clip_c, n, _ptr(f), _stream(stream)))


def dp_clip_accumulate(g, sqnorm, clip_c: float, n: int, p: int, acc, g_stride: int = 0, stream=None):
    _check(load_library().dp_clip_accumulate(_ptr(g), g_stride, _ptr(sqnorm), clip_c, n, p, _ptr(acc),
                                             _stream(stream)))


class SegmentTable:
    """Host arrays for dp_clip_accumulate_segments: column where each segment starts, its clipping group and bound, and (for
    dp_clip_accumulate_columns) where it lies in the accumulator."""

    def __init__(self, begins, groups, clips, places=None):
        k = len(begins)
        self.n_seg = k
        self.begin = (C.c_size_t * k)(*[int(b) for b in begins])
        self.group = (C.c_int32 * k)(*[int(g) for g in groups])
        self.clip = (C.c_float * k)(*[float(c) for c in clips])
        self.place = (C.c_size_t * k)(*[int(p) for p in (begins if places is None else places)])


def dp_clip_accumulate_segments(g, group_sqnorm, n_groups: int, table: "SegmentTable", n: int, p: int, acc,
                                g_stride: int = 0, stream=None):
    _check(load_library().dp_clip_accumulate_segments(_ptr(g), g_stride, _ptr(group_sqnorm), n_groups,
                                                      C.cast(table.begin, C.c_void_p), C.cast(table.group, C.c_void_p),
                                                      C.cast(table.clip, C.c_void_p), table.n_seg, n, p, _ptr(acc),
                                                      _stream(stream)))


def dp_clip_accumulate_columns(g, group_sqnorm, n_groups: int, table: "SegmentTable", n: int, run: int, p: int, acc, g_stride: int = 0,
                               stream=None):
    _check(load_library().dp_clip_accumulate_columns(_ptr(g), g_stride, _ptr(group_sqnorm), n_groups, table.begin, table.place, table.group,
                                                     table.clip, table.n_seg, n, run, p, _ptr(acc), _stream(stream)))


def dp_clip_accumulate_recompute(desc, x, dy, sqnorm, clip_c: float, acc_w, acc_b, ws,
                                 ws_bytes: Optional[int] = None, stream=None):
    _check(load_library().dp_clip_accumulate_recompute(C.byref(desc), _ptr(x), _ptr(dy), _ptr(sqnorm), clip_c,
                                                       _ptr(acc_w), _ptr(acc_b), _ptr(ws),
                                                       _nbytes(ws) if ws_bytes is None else ws_bytes,
                                                       _stream(stream)))


def dp_add_noise_finalize(acc, out, p: int, sigma: float, clip_total: float, total_batch: int, seed: int,
                          step: int, tensor_id: int, stream=None):
    _check(load_library().dp_add_noise_finalize(_ptr(acc), _ptr(out), p, sigma, clip_total, total_batch, seed,
                                                step, tensor_id, _stream(stream)))


def dp_add_example_noise(acc, p: int, sigma: float, clip_total: float, total_batch: int, seed: int, step: int,
                         tensor_id: int, first_example: int, n_examples: int, step_dev=None, stream=None):
    _check(load_library().dp_add_example_noise(_ptr(acc), p, sigma, clip_total, total_batch, seed, step, tensor_id,
                                               first_example, n_examples, _ptr(step_dev), _stream(stream)))


def dp_add_noise_finalize_update(acc, theta, velocity, out, p: int, sigma: float, clip_total: float, total_batch: int,
                                 seed: int, step: int, tensor_id: int, lr: float, momentum: float, stream=None):
    _check(load_library().dp_add_noise_finalize_update(_ptr(acc), _ptr(theta), _ptr(velocity), _ptr(out), p, sigma,
                                                       clip_total, total_batch, seed, step, tensor_id, lr, momentum,
                                                       _stream(stream)))


class TensorTable:
    """Host arrays for dp_add_noise_finalize_flat: where each tensor starts in the flat parameter vector,
    its size and its Philox tensor id."""

    def __init__(self, begins, sizes, tensor_ids):
        k = len(begins)
        self.n_seg = k
        self.begin = (C.c_uint64 * k)(*[int(b) for b in begins])
        self.size = (C.c_uint64 * k)(*[int(v) for v in sizes])
        self.tensor_id = (C.c_uint32 * k)(*[int(t) for t in tensor_ids])


def dp_add_noise_finalize_flat(acc, out, table: "TensorTable", sigma: float, clip_total: float, total_batch: int,
                               seed: int, step: int = 0, step_dev=None, theta=None, velocity=None, lr: float = 0.0,
                               momentum: float = 0.0, stream=None):
    _check(load_library().dp_add_noise_finalize_flat(_ptr(acc), _ptr(out), _ptr(theta), _ptr(velocity),
                                                     C.cast(table.begin, C.c_void_p), C.cast(table.size, C.c_void_p),
                                                     C.cast(table.tensor_id, C.c_void_p), table.n_seg, sigma, clip_total,
                                                     total_batch, seed, step, _ptr(step_dev), lr, momentum,
                                                     _stream(stream)))


def dp_profile_next_contraction(start_event, stop_event):
    """Arm (or, with None, cancel) event bracketing of the next contraction kernel.  The arguments are
    torch.cuda.Event objects that have been recorded once (that creates their HIP handles)."""
    a = start_event.cuda_event if start_event is not None else None
    b = stop_event.cuda_event if stop_event is not None else None
    _check(load_library().dp_profile_next_contraction(a, b))


def dp_philox_raw(raw, p: int, seed: int, step: int, tensor_id: int, stream=None):
    _check(load_library().dp_philox_raw(_ptr(raw), p, seed, step, tensor_id, _stream(stream)))


def _lengths(t, n: int, what: str) -> Optional[int]:
    """Address of int32 lengths of n examples (or None).  torch's integers from lists are int64 and on the host: neither is what kernels read."""
    if t is None or type(t) is int:
        return t
    if t.element_size() != 4 or t.is_floating_point() or t.numel() < n or not t.is_contiguous() or not (t.is_cuda or t.is_pinned()):
        raise DpError(DP_ERR_INVALID_ARG, f"{what} must be {n} contiguous int32 on the device, not {t.dtype} {list(t.shape)} on {t.device}")
    return t.data_ptr()


_TYPES = ()                                       # torch's float32 and bfloat16 by dp_dtype, once a call has needed them


def _types():
    global _TYPES
    import torch
    _TYPES = (torch.float32, torch.bfloat16)
    return _TYPES


# (The order of what is asked, and no more of it, because a tensor takes 0.1 us to answer and the smallest calls take 4.)
def _floats(t, n: int, what: str) -> Optional[int]:
    """Address of n fp32 numbers (or None)."""
    if t is None or type(t) is int:
        return t
    if t.dtype is not (_TYPES or _types())[DP_F32] or t.nbytes < 4 * n or not t.is_contiguous() or not (t.is_cuda or t.is_pinned()):
        raise DpError(DP_ERR_INVALID_ARG, f"{what} must be {n} contiguous float32 on the device, not {t.dtype} {list(t.shape)} on {t.device}")
    return t.data_ptr()


def _gradient_rows(t, n: int, width: int, spacing: int, what: str) -> Optional[int]:
    """Address of n examples' fp32 gradients of `width` values, one every `spacing` (or None)."""
    if t is None or type(t) is int:
        return t
    shape = t.shape
    plain = t.stride() == (spacing, 1) and shape[0] >= n and shape[1] >= width
    if t.dtype is not (_TYPES or _types())[DP_F32] or not (plain or _has_rows(t, n, width, spacing)) or not (t.is_cuda or t.is_pinned()):
        raise DpError(DP_ERR_INVALID_ARG, f"{what} must be {n} rows of {width} float32 on the device, one every {spacing}, not {t.dtype} {list(shape)} of strides "
                                          f"{list(t.stride())} on {t.device}")
    return t.data_ptr()


def _row_layout(desc, width: int):
    """Of a call's rows: type, their number, values, elements from one to the next, bytes of all values, and the shape and strides of a tensor of n, tokens and
    width where there is something between rows.  What is unknown is the library's to refuse."""
    dtype, n, tokens, spacing = 1 if desc.in_dtype == DP_BF16 else 0, desc.n, desc.tokens, desc.row_stride or width
    rows = n * tokens
    return dtype, rows, width, spacing, rows * width * (2 if dtype else 4), None if spacing == width else ((n, tokens, width), (tokens * spacing, spacing, 1))


def _has_rows(t, rows: int, width: int, spacing: int) -> bool:
    """Whether a tensor's leading dimensions are `rows` rows or more, one every `spacing` elements, its trailing ones `width` values or more of each.  One
    dimension alone is taken as memory."""
    shape, strides = t.shape, t.stride()
    dims = [(size, stride) for size, stride in zip(reversed(shape), reversed(strides)) if size != 1]          # (the stride of a dimension of one means nothing)
    if len(dims) == 1 and dims[0][1] == 1:
        return dims[0][0] >= (rows - 1) * spacing + width
    row, at = 1, 0
    while at < len(dims) and dims[at][1] == row and (row < width or row * dims[at][0] <= spacing):
        row *= dims[at][0]
        at += 1
    if row < width:
        return False
    found = 1
    while found < rows and at < len(dims) and dims[at][1] == spacing * found and row <= spacing:
        found *= dims[at][0]
        at += 1
    return found >= rows


def _token_rows(t, layout, what: str) -> Optional[int]:
    """Address of [n, tokens] rows, of the descriptor's type and where it says they are (or None)."""
    if t is None or type(t) is int:
        return t
    dtype, rows, width, spacing, size, gaps = layout
    kind = (_TYPES or _types())[dtype]
    plain = t.nbytes == size and t.is_contiguous() if gaps is None else t.shape == gaps[0] and t.stride() == gaps[1]
    if t.dtype is not kind or not (plain or _has_rows(t, rows, width, spacing)) or not (t.is_cuda or t.is_pinned()):
        raise DpError(DP_ERR_INVALID_ARG, f"{what} must be {rows} rows of {width} {kind} on the device, one every {spacing}, not {t.dtype} {list(t.shape)} of "
                                          f"strides {list(t.stride())} on {t.device}")
    return t.data_ptr()


# ---- 8-bit activation checkpoints ---------------------------------------------------------------------------------

def _rows_of(t):
    """(dtype code, rows, features, elements from row to row) of a tensor whose leading dimensions are evenly spaced rows."""
    import torch
    dtype = t.dtype
    if dtype is not torch.bfloat16 and dtype is not torch.float32:
        raise DpError(DP_ERR_UNSUPPORTED, f"activations are float32 or bfloat16, not {dtype}")
    shape, strides = t.shape, t.stride()
    features, rows, spacing = shape[-1] if shape else 0, 1, 0
    even = features > 0 and (features == 1 or strides[-1] == 1)
    for d in range(len(shape) - 2, -1, -1):          # from the innermost on; the stride of a dimension of one means nothing
        if shape[d] != 1:
            even = even and (strides[d] == rows * spacing if spacing else strides[d] >= features)
            spacing = spacing or strides[d]
            rows *= shape[d]
    if not even and (rows or features <= 0):
        raise DpError(DP_ERR_INVALID_ARG, f"not rows of consecutive values: shape {tuple(shape)}, strides {strides}")
    return (DP_BF16 if dtype is torch.bfloat16 else DP_F32), rows, features, max(spacing, features)


def _check_checkpoint(codes, scales, rows: int, features: int):
    blocks = (features + 31) // 32
    for t, need, what in ((codes, rows * blocks * 32, "codes"), (scales, rows * blocks, "scales")):
        if t.element_size() != 1 or t.numel() < need or not t.is_contiguous():
            raise DpError(DP_ERR_INVALID_ARG, f"{what} must be at least {need} contiguous bytes for {rows} rows of {features} features")


def dp_checkpoint_pitch(features: int) -> int:
    """Bytes of codes of a row: features rounded up to a multiple of 32."""
    pitch = int(load_library().dp_checkpoint_pitch(features))
    if not pitch:
        raise DpError(DP_ERR_INVALID_ARG, dp_last_error())
    return pitch


def dp_checkpoint_write(x, codes, scales, stream=None):
    """x [..., features] (rows evenly spaced, float32 or bfloat16) into codes [rows, pitch] and scales [rows, pitch / 32] (bytes)."""
    dtype, rows, features, stride = _rows_of(x)
    _check_checkpoint(codes, scales, rows, features)
    _check(load_library().dp_checkpoint_write(_ptr(x), dtype, rows, features, stride, _ptr(codes), _ptr(scales), _stream(stream)))


def dp_checkpoint_read(codes, scales, x, stream=None):
    """The values of a checkpoint into x [..., features] (rows evenly spaced, float32 or bfloat16)."""
    dtype, rows, features, stride = _rows_of(x)
    _check_checkpoint(codes, scales, rows, features)
    _check(load_library().dp_checkpoint_read(_ptr(codes), _ptr(scales), rows, features, _ptr(x), dtype, stride, _stream(stream)))


def dp_checkpoint_workspace_bytes(desc: LayerDesc, use: int = DP_WS_PER_EXAMPLE_GRAD) -> int:
    return int(load_library().dp_checkpoint_workspace_bytes(C.byref(desc), use))


def dp_checkpoint_example_grad(desc: LayerDesc, codes, scales, dy, g_w, g_b, sqnorm, ws, lengths=None, g_stride: int = 0,
                               ws_bytes: Optional[int] = None, stream=None):
    """dp_per_example_grad of a dense layer with its input activations from a checkpoint; lengths: int32 tokens of each example."""
    _check(load_library().dp_checkpoint_example_grad(C.byref(desc), _ptr(codes), _ptr(scales), _ptr(dy), _lengths(lengths, desc.n, "lengths"), _ptr(g_w), _ptr(g_b),
                                                     g_stride, _ptr(sqnorm), _ptr(ws), _nbytes(ws) if ws_bytes is None else ws_bytes,
                                                     _stream(stream)))


def dp_checkpoint_clip_accumulate(desc: LayerDesc, codes, scales, dy, sqnorm, clip_c: float, acc_w, acc_b, ws, lengths=None,
                                  ws_bytes: Optional[int] = None, stream=None):
    """dp_clip_accumulate_recompute of a dense layer with its input activations from a checkpoint."""
    _check(load_library().dp_checkpoint_clip_accumulate(C.byref(desc), _ptr(codes), _ptr(scales), _ptr(dy), _lengths(lengths, desc.n, "lengths"), _ptr(sqnorm), clip_c,
                                                        _ptr(acc_w), _ptr(acc_b), _ptr(ws), _nbytes(ws) if ws_bytes is None else ws_bytes,
                                                        _stream(stream)))


# ---- attention probabilities under a relative position bias ---------------------------------------------------------

def dp_bias_bucket(desc: BiasDesc, distance: int) -> int:
    """Row of the bias table that a distance (query position - key position) uses."""
    bucket = int(load_library().dp_bias_bucket(C.byref(desc), distance))
    if bucket < 0:
        raise DpError(DP_ERR_INVALID_ARG, dp_last_error())
    return bucket


def dp_bias_softmax(desc: BiasDesc, scores, table, probs, query_lengths=None, key_lengths=None, stream=None):
    _check(load_library().dp_bias_softmax(C.byref(desc), _ptr(scores), _ptr(table), _lengths(query_lengths, desc.n, "query_lengths"),
                                          _lengths(key_lengths, desc.n, "key_lengths"), _ptr(probs),
                                          _stream(stream)))


def dp_bias_workspace_bytes(desc: BiasDesc) -> int:
    return int(load_library().dp_bias_workspace_bytes(C.byref(desc)))


def dp_bias_softmax_backward(desc: BiasDesc, probs, dprobs, dscores, g_table, sqnorm, ws, query_lengths=None, key_lengths=None,
                             g_stride: int = 0, ws_bytes: Optional[int] = None, stream=None):
    """Gradient of the scores, and per example the gradient of the bias table and its squared norm."""
    _check(load_library().dp_bias_softmax_backward(C.byref(desc), _ptr(probs), _ptr(dprobs), _lengths(query_lengths, desc.n, "query_lengths"),
                                          _lengths(key_lengths, desc.n, "key_lengths"), _ptr(dscores),
                                                   _ptr(g_table), g_stride, _ptr(sqnorm), _ptr(ws),
                                                   _nbytes(ws) if ws_bytes is None else ws_bytes, _stream(stream)))


# ---- normalisation of tokens over their features ---------------------------------------------------------------------

def dp_layer_norm(desc: NormDesc, x, gamma, beta, y, lengths=None, stream=None):
    """Layer norm (desc.rms: RMS norm) of every token of x [n, tokens, features] into y."""
    f = desc.features
    rows = _row_layout(desc, f)
    _check(load_library().dp_layer_norm(C.byref(desc), _token_rows(x, rows, "x"), _floats(gamma, f, "gamma"), _floats(beta, f, "beta"),
                                        _lengths(lengths, desc.n, "lengths"), _token_rows(y, rows, "y"), _stream(stream)))


def dp_layer_norm_workspace_bytes(desc: NormDesc) -> int:
    return int(load_library().dp_layer_norm_workspace_bytes(C.byref(desc)))


def dp_layer_norm_backward(desc: NormDesc, x, gamma, dy, dx, g_w, g_b, sqnorm, ws, lengths=None, g_stride: int = 0,
                           ws_bytes: Optional[int] = None, stream=None):
    """Gradient of the tokens, and per example the gradients of gamma and beta and their squared norm."""
    f = desc.features
    rows, spacing = _row_layout(desc, f), g_stride or f
    _check(load_library().dp_layer_norm_backward(C.byref(desc), _token_rows(x, rows, "x"), _floats(gamma, f, "gamma"), _token_rows(dy, rows, "dy"),
                                                 _lengths(lengths, desc.n, "lengths"), _token_rows(dx, rows, "dx"), _gradient_rows(g_w, desc.n, f, spacing, "g_w"),
                                                 _gradient_rows(g_b, desc.n, f, spacing, "g_b"), g_stride, _floats(sqnorm, desc.n, "sqnorm"), _ptr(ws), _nbytes(ws) if ws_bytes is None else ws_bytes, _stream(stream)))


# ---- log probabilities of tokens -------------------------------------------------------------------------------------

def dp_token_logprobs_workspace_bytes(desc: LogprobDesc) -> int:
    return int(load_library().dp_token_logprobs_workspace_bytes(C.byref(desc)))


def dp_token_logprobs(desc: LogprobDesc, logits, targets, logprobs, entropy, stats, top_logprobs, top_tokens, ws, lengths=None,
                      ws_bytes: Optional[int] = None, stream=None):
    """Log probabilities of targets (int32 [n, tokens]) under rows of logits, entropies, statistics for the backward pass, the most likely tokens; any
    of the results may be None."""
    rows, layout = desc.n * desc.tokens, _row_layout(desc, desc.vocab)
    _check(load_library().dp_token_logprobs(C.byref(desc), _token_rows(logits, layout, "logits"), _lengths(targets, rows, "targets"),
                                            _lengths(lengths, desc.n, "lengths"), _floats(logprobs, rows, "logprobs"), _floats(entropy, rows, "entropy"),
                                            _floats(stats, 2 * rows, "stats"), _floats(top_logprobs, rows * desc.top, "top_logprobs"),
                                            _lengths(top_tokens, rows * desc.top, "top_tokens"), _ptr(ws), _nbytes(ws) if ws_bytes is None else ws_bytes,
                                            _stream(stream)))


def dp_token_logprobs_backward(desc: LogprobDesc, logits, targets, stats, d_logprobs, dlogits, ws, entropy=None, d_entropy=None, logprobs=None,
                               lengths=None, ws_bytes: Optional[int] = None, stream=None):
    """Gradient of the logits from those of log probabilities and entropies; stats None: worked out in the same call, with the log probabilities
    where there is a place for them."""
    rows, layout = desc.n * desc.tokens, _row_layout(desc, desc.vocab)
    _check(load_library().dp_token_logprobs_backward(C.byref(desc), _token_rows(logits, layout, "logits"), _lengths(targets, rows, "targets"),
                                                     _lengths(lengths, desc.n, "lengths"), _floats(stats, 2 * rows, "stats"), _floats(entropy, rows, "entropy"),
                                                     _floats(d_logprobs, rows, "d_logprobs"), _floats(d_entropy, rows, "d_entropy"),
                                                     _floats(logprobs, rows, "logprobs"), _token_rows(dlogits, layout, "dlogits"), _ptr(ws),
                                                     _nbytes(ws) if ws_bytes is None else ws_bytes, _stream(stream)))
