"""ctypes binding of libjenga.so: the same names as the C ABI, argument marshalling only.

Every step of the path runs in the library's HIP kernels.  If the library has not been built the
import of this module fails: there is no fallback.
"""
import ctypes
import os
import struct

PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(PKG, "libjenga.so")

JENGA_FLAG_ADJACENCY = 1
JENGA_FLAG_CONDITION = 2
JENGA_FLAG_CURVE = 4
JENGA_FLAG_PACED_WALK = 8

JENGA_BF16, JENGA_F16, JENGA_F32, JENGA_E4M3, JENGA_E2M1 = range(5)
JENGA_DENSE_CAUSAL = 1
JENGA_ROTARY_HALVES = 1
JENGA_ROTARY_INVERSE = 2

EXPORTS = ["jenga_plan_create", "jenga_plan_destroy", "jenga_plan_info", "jenga_plan_export", "jenga_plan_tables",
           "jenga_curve_permute", "jenga_curve_permute_qkv", "jenga_curve_permute_rows", "jenga_select_blocks",
           "jenga_select_blocks_static",
           "jenga_block_sparse_attn", "jenga_pack_kv",
           "jenga_block_sparse_attn_packed", "jenga_unpermute", "jenga_forward", "jenga_stage_switch",
           "jenga_quantize", "jenga_matmul", "jenga_layer_norm", "jenga_layer_norm_grad", "jenga_layer_norm_grad_workspace",
           "jenga_quantize_mx", "jenga_matmul_mx", "jenga_rms_norm", "jenga_rms_norm_grad", "jenga_rms_norm_grad_workspace",
           "jenga_dense_attn", "jenga_dense_attn_workspace", "jenga_dense_attn_workspace_up_to",
           "jenga_rotary_table", "jenga_rotary", "jenga_forward_rotary", "jenga_strerror"]


class jenga_config(ctypes.Structure):
    _fields_ = [("T", ctypes.c_int32), ("H", ctypes.c_int32), ("W", ctypes.c_int32),
                ("n_text", ctypes.c_int32), ("batch", ctypes.c_int32), ("heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("block", ctypes.c_int32),
                ("topk_ratio", ctypes.c_double), ("cum_prob", ctypes.c_double),
                ("text_bias", ctypes.c_float), ("flags", ctypes.c_uint32)]


class jenga_plan_info_t(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("N_v", "M_v", "M_c", "M", "N_pad", "pad_v", "pad_c", "K_top")] + \
               [("select_workspace_bytes", ctypes.c_uint64), ("attn_workspace_bytes", ctypes.c_uint64)]


class jenga_matmul_config(ctypes.Structure):
    _fields_ = [("m", ctypes.c_int64), ("out_stride", ctypes.c_int64), ("n", ctypes.c_int32), ("k", ctypes.c_int32),
                ("out_type", ctypes.c_int32), ("reserved", ctypes.c_int32)]


class jenga_norm_config(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_int64), ("group_rows", ctypes.c_int64), ("x_stride", ctypes.c_int64), ("y_stride", ctypes.c_int64),
                ("param_stride", ctypes.c_int64), ("cols", ctypes.c_int32), ("x_type", ctypes.c_int32), ("y_type", ctypes.c_int32),
                ("param_type", ctypes.c_int32), ("eps", ctypes.c_float), ("weight_offset", ctypes.c_float)]


class jenga_rms_config(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int64) for n in ("rows", "x_row", "x_head", "add_row", "add_head", "sum_row", "sum_head", "y_row", "y_head")] + \
               [(n, ctypes.c_int32) for n in ("heads", "cols", "x_type", "y_type", "param_type")] + \
               [("eps", ctypes.c_float), ("weight_offset", ctypes.c_float), ("reserved", ctypes.c_int32)]


class jenga_dense_config(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int64) for n in ("q_rows", "kv_rows", "q_row", "q_head", "k_row", "k_head", "v_row", "v_head", "out_row",
                                              "out_head")] + \
               [(n, ctypes.c_int32) for n in ("sequences", "heads", "kv_heads", "head_dim", "type")] + \
               [("flags", ctypes.c_uint32), ("scale", ctypes.c_float), ("reserved", ctypes.c_int32)]


class jenga_rotary_config(ctypes.Structure):
    _fields_ = [("T", ctypes.c_int32), ("H", ctypes.c_int32), ("W", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("dim", ctypes.c_int32 * 3), ("type", ctypes.c_int32), ("theta", ctypes.c_double),
                ("origin", ctypes.c_double * 3), ("step", ctypes.c_double * 3), ("flags", ctypes.c_uint32),
                ("reserved", ctypes.c_uint32)]


class jenga_rotary_tensor(ctypes.Structure):
    _fields_ = [("src", ctypes.c_void_p), ("dst", ctypes.c_void_p)] + \
               [(n, ctypes.c_int64) for n in ("src_batch", "src_token", "src_head", "dst_batch", "dst_token", "dst_head")] + \
               [("heads", ctypes.c_int32), ("reserved", ctypes.c_int32)]


class JengaError(RuntimeError):
    def __init__(self, status, what):
        super().__init__("%s: %s (%d)" % (what, _lib.jenga_strerror(status).decode(), status))
        self.status = status


def _load():
    if not os.path.exists(LIB_PATH):
        raise ImportError("libjenga.so is not built: run `python -c 'import __graft_entry__ as g; g.build()'` "
                          "or `python paper_2505_16864_amd/build.py` (needs hipcc)")
    lib = ctypes.CDLL(LIB_PATH)
    vp, i32p = ctypes.c_void_p, ctypes.POINTER(ctypes.c_int32)
    lib.jenga_plan_create.argtypes = [ctypes.POINTER(jenga_config), ctypes.POINTER(vp)]
    lib.jenga_plan_destroy.argtypes = [vp]
    lib.jenga_plan_info.argtypes = [vp, ctypes.POINTER(jenga_plan_info_t)]
    lib.jenga_plan_export.argtypes = [vp, vp, vp, vp]
    lib.jenga_plan_tables.argtypes = [ctypes.POINTER(jenga_config), ctypes.POINTER(jenga_plan_info_t), vp, vp, vp]
    lib.jenga_curve_permute.argtypes = [vp, vp, vp, vp]
    lib.jenga_curve_permute_qkv.argtypes = [vp] * 8
    lib.jenga_unpermute.argtypes = [vp, vp, vp, vp]
    lib.jenga_curve_permute_rows.argtypes = [vp, vp, vp, ctypes.c_int32, vp]
    lib.jenga_select_blocks.argtypes = [vp, vp, vp, vp, vp, vp, vp, ctypes.c_size_t, vp]
    lib.jenga_select_blocks_static.argtypes = [vp, vp, vp, vp, vp, vp, vp]
    lib.jenga_block_sparse_attn.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, vp, ctypes.c_size_t, vp]
    lib.jenga_pack_kv.argtypes = [vp, vp, vp, vp, ctypes.c_size_t, vp]
    lib.jenga_block_sparse_attn_packed.argtypes = [vp, vp, vp, ctypes.c_size_t, vp, vp, vp, vp, vp]
    lib.jenga_forward.argtypes = [vp] * 11 + [ctypes.c_size_t, vp, vp, vp, ctypes.c_size_t, vp, vp]
    lib.jenga_stage_switch.argtypes = [vp, vp, vp, vp] + [ctypes.c_int32] * 7 + [ctypes.c_float, vp]
    i32, i64, size = ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t
    lib.jenga_quantize.argtypes = [vp, i64, i32, i64, i32, i32, vp, vp, vp]
    # the structs of these calls are passed by address, as ctypes structures or packed
    lib.jenga_matmul.argtypes = [vp] * 8
    lib.jenga_layer_norm.argtypes = [vp] * 9
    lib.jenga_layer_norm_grad.argtypes = [vp] * 10 + [size, vp]
    lib.jenga_layer_norm_grad_workspace.argtypes = [vp, ctypes.POINTER(ctypes.c_uint64)]
    lib.jenga_quantize_mx.argtypes = [vp, i64, i32, i64, i32, vp, vp, vp]
    lib.jenga_matmul_mx.argtypes = [vp] * 8
    lib.jenga_rms_norm.argtypes = [vp] * 9
    lib.jenga_rms_norm_grad.argtypes = [vp] * 9 + [size, vp]
    lib.jenga_rms_norm_grad_workspace.argtypes = [vp, ctypes.POINTER(ctypes.c_uint64)]
    lib.jenga_dense_attn.argtypes = [vp] * 9 + [size, vp]
    lib.jenga_dense_attn_workspace.argtypes = lib.jenga_dense_attn_workspace_up_to.argtypes = [vp, ctypes.POINTER(ctypes.c_uint64)]
    lib.jenga_rotary_table.argtypes = [ctypes.POINTER(jenga_rotary_config), vp]
    lib.jenga_rotary.argtypes = [vp] * 5 + [i32, i64, i64, vp]
    lib.jenga_forward_rotary.argtypes = [vp, ctypes.POINTER(jenga_rotary_config)] + [vp] * 4 + [i64] + [vp] * 7 + [size, vp, vp, vp,
                                                                                                                size, vp, vp]
    lib.jenga_strerror.argtypes = [ctypes.c_int]
    lib.jenga_strerror.restype = ctypes.c_char_p
    for name in EXPORTS[:-1]:
        getattr(lib, name).restype = ctypes.c_int
    return lib


_lib = _load()


def _check(status, what):
    if status != 0:
        raise JengaError(status, what)


def _ptr(t):
    """Device (or host) address of a torch tensor / numpy array / None / int."""
    if t is None:
        return None
    if isinstance(t, int):
        return t
    if hasattr(t, "data_ptr"):
        return t.data_ptr()
    return t.ctypes.data


def make_config(T, H, W, n_text, batch, heads, head_dim, block, topk, p, text_bias=0.0, flags=7):
    return jenga_config(T, H, W, n_text, batch, heads, head_dim, block, float(topk), float(p),
                        float(text_bias), flags)


def jenga_plan_create(cfg):
    plan = ctypes.c_void_p()
    _check(_lib.jenga_plan_create(ctypes.byref(cfg), ctypes.byref(plan)), "jenga_plan_create")
    return plan


def jenga_plan_destroy(plan):
    _check(_lib.jenga_plan_destroy(plan), "jenga_plan_destroy")


def jenga_plan_info(plan):
    info = jenga_plan_info_t()
    _check(_lib.jenga_plan_info(plan, ctypes.byref(info)), "jenga_plan_info")
    return info


def jenga_plan_export(plan, perm=None, inv_perm=None, adja=None):
    """perm, inv_perm: int32 numpy arrays [N_v]; adja: uint8 numpy array [M_v*M_v] (host)."""
    _check(_lib.jenga_plan_export(plan, _ptr(perm), _ptr(inv_perm), _ptr(adja)), "jenga_plan_export")


def jenga_plan_tables(cfg, perm=None, inv_perm=None, adja=None):
    """Host-only tables of a config (no device): returns the info struct, fills the given host arrays."""
    info = jenga_plan_info_t()
    _check(_lib.jenga_plan_tables(ctypes.byref(cfg), ctypes.byref(info), _ptr(perm), _ptr(inv_perm), _ptr(adja)),
           "jenga_plan_tables")
    return info


def jenga_curve_permute(plan, src_thw, dst_curve, stream=None):
    _check(_lib.jenga_curve_permute(plan, _ptr(src_thw), _ptr(dst_curve), stream), "jenga_curve_permute")


def jenga_curve_permute_qkv(plan, q_thw, k_thw, v_thw, q_curve, k_curve, v_curve, stream=None):
    _check(_lib.jenga_curve_permute_qkv(plan, _ptr(q_thw), _ptr(k_thw), _ptr(v_thw), _ptr(q_curve), _ptr(k_curve),
                                        _ptr(v_curve), stream), "jenga_curve_permute_qkv")


def jenga_curve_permute_rows(plan, src_rows, dst_rows, row_bytes, stream=None):
    _check(_lib.jenga_curve_permute_rows(plan, _ptr(src_rows), _ptr(dst_rows), row_bytes, stream),
           "jenga_curve_permute_rows")


def jenga_unpermute(plan, src_curve, dst_thw, stream=None):
    _check(_lib.jenga_unpermute(plan, _ptr(src_curve), _ptr(dst_thw), stream), "jenga_unpermute")


def jenga_select_blocks(plan, q_curve, k_curve, sel_count, sel_index, mask, workspace, workspace_bytes,
                        stream=None):
    _check(_lib.jenga_select_blocks(plan, _ptr(q_curve), _ptr(k_curve), _ptr(sel_count), _ptr(sel_index),
                                    _ptr(mask), _ptr(workspace), workspace_bytes, stream), "jenga_select_blocks")


def jenga_select_blocks_static(plan, q_curve, k_curve, sel_count, sel_index, mask, stream=None):
    _check(_lib.jenga_select_blocks_static(plan, _ptr(q_curve), _ptr(k_curve), _ptr(sel_count), _ptr(sel_index),
                                           _ptr(mask), stream), "jenga_select_blocks_static")


def jenga_block_sparse_attn(plan, q, k, v, sel_count, sel_index, out_curve, lse, workspace, workspace_bytes,
                            stream=None):
    """lse: float32 device tensor [batch, heads, N_pad] or None."""
    _check(_lib.jenga_block_sparse_attn(plan, _ptr(q), _ptr(k), _ptr(v), _ptr(sel_count), _ptr(sel_index),
                                        _ptr(out_curve), _ptr(lse), _ptr(workspace), workspace_bytes, stream),
           "jenga_block_sparse_attn")


def jenga_pack_kv(plan, k, v, workspace, workspace_bytes, stream=None):
    _check(_lib.jenga_pack_kv(plan, _ptr(k), _ptr(v), _ptr(workspace), workspace_bytes, stream), "jenga_pack_kv")


def jenga_block_sparse_attn_packed(plan, q, workspace, workspace_bytes, sel_count, sel_index, out_curve, lse=None,
                                   stream=None):
    _check(_lib.jenga_block_sparse_attn_packed(plan, _ptr(q), _ptr(workspace), workspace_bytes, _ptr(sel_count),
                                               _ptr(sel_index), _ptr(out_curve), _ptr(lse), stream),
           "jenga_block_sparse_attn_packed")


def jenga_forward(plan, q_thw, k_thw, v_thw, q_curve, k_curve, v_curve, sel_count, sel_index, mask, select_workspace,
                  select_workspace_bytes, out_curve, lse, attn_workspace, attn_workspace_bytes, out_thw, stream=None):
    _check(_lib.jenga_forward(plan, _ptr(q_thw), _ptr(k_thw), _ptr(v_thw), _ptr(q_curve), _ptr(k_curve), _ptr(v_curve),
                              _ptr(sel_count), _ptr(sel_index), _ptr(mask), _ptr(select_workspace), select_workspace_bytes,
                              _ptr(out_curve), _ptr(lse), _ptr(attn_workspace), attn_workspace_bytes, _ptr(out_thw), stream),
           "jenga_forward")


def jenga_stage_switch(x_t, eps_t, eps_tilde, x_out, channels, in_shape, out_shape, sigma_t, stream=None):
    """in_shape = (T_in, H_in, W_in), out_shape = (T_out, H_out, W_out); float32 device tensors."""
    _check(_lib.jenga_stage_switch(_ptr(x_t), _ptr(eps_t), _ptr(eps_tilde), _ptr(x_out), channels,
                                   *[int(v) for v in in_shape], *[int(v) for v in out_shape], float(sigma_t), stream),
           "jenga_stage_switch")


# The calls around the attention take torch tensors and read sizes, strides and types from them.  What the C ABI cannot see is
# checked here: values next to each other in the last dimension, all tensors on the device that is current.  They go to torch's current
# stream of that device, where its own work on the tensors goes, unless `stream` names another (0: the null stream, which is
# what None means to the calls above).  No gradient is recorded: tensors that require one are taken like others.  Small calls cost
# little more than this code and a launch, so it is written without detours.

_EINVAL = -1
_TYPES = {}            # torch's element types to jenga_type, filled by the first call that needs them
_DTYPE = {}            # and by name
_current_device = _current_stream = None
_U8 = _F32 = _I32 = None
_MATMUL, _NORM, _TENSOR = struct.Struct("=2q4i"), struct.Struct("=5q4i2f"), struct.Struct("=2Q6q2i")   # as the structures above
_RMS, _DENSE = struct.Struct("=9q5i2fi"), struct.Struct("=10q5iIfi")


def _use_torch():
    import torch
    global _current_device, _current_stream, _U8, _F32, _I32
    _U8, _F32, _I32 = torch.uint8, torch.float32, torch.int32
    _current_device, _current_stream = torch._C._cuda_getDevice, torch._C._cuda_getCurrentRawStream
    _DTYPE.update(f32=torch.float32, i32=torch.int32, u8=torch.uint8, bf16=torch.bfloat16, e4m3=torch.float8_e4m3fn)
    _TYPES.update({torch.bfloat16: JENGA_BF16, torch.float16: JENGA_F16, torch.float32: JENGA_F32, torch.float8_e4m3fn: JENGA_E4M3,
                   torch.uint8: JENGA_E4M3})


def _refuse(what, why):
    raise JengaError(_EINVAL, "%s: %s" % (what, why))


def _pack(what, layout, *values):
    """A structure as bytes: a third of the time that ctypes takes to fill one."""
    try:
        return layout.pack(*values)
    except (struct.error, OverflowError):
        _refuse(what, "sizes or numbers out of range")


def _type(t, what):
    code = _TYPES.get(t.dtype)
    if code is None:
        if not _TYPES:
            _use_torch()
            return _type(t, what)
        _refuse(what, "element type %s" % t.dtype)
    return code


def _on_device(what, tensors, stream):
    """Refuses tensors that are not on the current device; returns the stream to go to."""
    device = tensors[0].get_device()
    for t in tensors:
        if t is not None and (t.get_device() != device or device < 0):
            _refuse(what, "tensors are not all on one GPU")
    if device != _current_device():
        _refuse(what, "tensors are not on the current device")
    return _current_stream(device) if stream is None else stream


def _matrix(t, what, rows=None, cols=None):
    """The row stride of a matrix; of a single row any stride will do."""
    shape = t.shape
    if len(shape) != 2 or (rows is not None and (shape[0] != rows or shape[1] != cols)):
        _refuse(what, "shape %s" % (tuple(shape),))
    stride = t.stride()
    if stride[1] != 1 and shape[1] != 1:
        _refuse(what, "values of a row are not next to each other")
    return stride[0] if shape[0] > 1 else max(stride[0], shape[1])


def _whole(t, what, shape, dtype):
    """Refuses anything but a tensor of this shape and type (a name in _DTYPE) without gaps."""
    if t.is_contiguous() and t.shape == shape:
        have = t.dtype
        if have is _DTYPE[dtype] or (dtype == "e4m3" and have is _DTYPE["u8"]):   # its bytes will do
            return
    _refuse(what, "shape %s, type %s" % (tuple(t.shape), t.dtype))


def _room(workspace, what):
    """Address and bytes of a workspace.  One with gaps or repeats has fewer bytes, or has them elsewhere, than its elements say."""
    if not workspace.is_contiguous():
        _refuse(what, "a workspace with gaps")
    return workspace.data_ptr(), workspace.numel() * workspace.element_size()


def scale_columns(cols):
    """Bytes of a row of scales of an 8-bit tensor with `cols` columns."""
    return -(-cols // 512) * 4


def padded_columns(cols):
    """Columns of an 8-bit tensor that holds `cols` columns."""
    return -(-cols // 128) * 128


def jenga_quantize(x, q, scale, block_rows=1, stream=None):
    """x [rows, cols] -> q e4m3 [rows, padded_columns(cols)], scale uint8 [rows or ceil(rows / 128), scale_columns(cols)]."""
    what = "jenga_quantize"
    stride, kind = _matrix(x, what), _type(x, what)
    rows, cols = x.shape
    if block_rows not in (1, 128):
        _refuse(what, "blocks of %s rows" % block_rows)
    _whole(q, what, (rows, padded_columns(cols)), "e4m3")
    _whole(scale, what, (-(-rows // block_rows), scale_columns(cols)), "u8")
    stream = _on_device(what, (x, q, scale), stream)
    if cols > 0x7FFFFFFF:
        _refuse(what, "%d columns" % cols)
    if rows:
        _check(_lib.jenga_quantize(x.data_ptr(), stride, kind, rows, cols, block_rows, q.data_ptr(), scale.data_ptr(), stream), what)


def jenga_matmul(a, a_scale, b, b_scale, out, bias=None, stream=None):
    """out [m, n] = a b^T + bias for 8-bit tensors a [m, k] (blocks of 1 x 128) and b [n, k] (128 x 128); bias float32 [n]."""
    what = "jenga_matmul"
    if len(a.shape) != 2 or len(b.shape) != 2:
        _refuse(what, "shapes %s, %s" % (tuple(a.shape), tuple(b.shape)))
    (m, k), n, kind = a.shape, b.shape[0], _type(out, what)
    stride = _matrix(out, what, m, n)
    scales = scale_columns(k)
    _whole(a, what, (m, k), "e4m3")
    _whole(b, what, (n, k), "e4m3")
    _whole(a_scale, what, (m, scales), "u8")
    _whole(b_scale, what, (-(-n // 128), scales), "u8")
    if bias is not None:
        _whole(bias, what, (n,), "f32")
    stream = _on_device(what, (a, a_scale, b, b_scale, out, bias), stream)
    if m:
        _check(_lib.jenga_matmul(_pack(what, _MATMUL, m, stride, n, k, kind, 0), a.data_ptr(), a_scale.data_ptr(),
                                 b.data_ptr(), b_scale.data_ptr(), None if bias is None else bias.data_ptr(), out.data_ptr(), stream), what)


def _norm_config(what, x, y, weight, bias, group_rows, weight_offset, eps):
    x_stride, x_type, y_type = _matrix(x, what), _type(x, what), _type(y, what)
    rows, cols = x.shape
    if group_rows < 0:
        _refuse(what, "groups of %d rows" % group_rows)
    group_rows = group_rows or rows or 1
    param_stride, param_type = cols, x_type
    for p in (bias, weight):
        if p is not None:
            shape, stride = p.shape, p.stride()
            groups = -(-rows // group_rows)
            if not 1 <= len(shape) <= 2 or shape[-1] != cols or stride[-1] != 1 and cols != 1 or (rows and (shape[0] if len(shape) == 2 else 1) != groups):
                _refuse(what, "weight or bias of shape %s" % (tuple(shape),))
            stride = stride[0] if groups > 1 else cols
            if p is weight and bias is not None and (stride != param_stride or p.dtype != bias.dtype):
                _refuse(what, "weight and bias differ in stride or type")
            param_stride, param_type = stride, _type(p, what)
    if y_type == JENGA_E4M3:
        y_stride = padded_columns(cols)
        _whole(y, what, (rows, y_stride), "e4m3")
    else:
        y_stride = _matrix(y, what, rows, cols)
    return _pack(what, _NORM, rows, group_rows, x_stride, y_stride, param_stride, cols, x_type, y_type, param_type, eps, weight_offset)


def jenga_layer_norm(x, y, weight=None, bias=None, y_scale=None, mean=None, rstd=None, group_rows=0, weight_offset=0.0,
                     eps=1e-6, stream=None):
    """x, y [rows, cols]; weight, bias [cols] or [groups, cols], a group for each group_rows rows (0: one for all); mean, rstd
    float32 [rows].  y in e4m3: [rows, padded_columns(cols)] with y_scale uint8 [rows, scale_columns(cols)]."""
    what = "jenga_layer_norm"
    cfg = _norm_config(what, x, y, weight, bias, group_rows, weight_offset, eps)
    rows, cols = x.shape
    if y_scale is not None:
        _whole(y_scale, what, (rows, scale_columns(cols)), "u8")
    if mean is not None:
        _whole(mean, what, (rows,), "f32")
    if rstd is not None:
        _whole(rstd, what, (rows,), "f32")
    stream = _on_device(what, (x, y, weight, bias, y_scale, mean, rstd), stream)
    if rows:
        _check(_lib.jenga_layer_norm(cfg, x.data_ptr(), None if weight is None else weight.data_ptr(),
                                     None if bias is None else bias.data_ptr(), y.data_ptr(),
                                     None if y_scale is None else y_scale.data_ptr(), None if mean is None else mean.data_ptr(),
                                     None if rstd is None else rstd.data_ptr(), stream), what)


def jenga_layer_norm_grad_workspace(rows, cols, group_rows=0):
    """Bytes of the workspace of jenga_layer_norm_grad."""
    bytes_ = ctypes.c_uint64()
    cfg = jenga_norm_config(rows, group_rows or max(rows, 1), cols, cols, cols, cols, JENGA_F32, JENGA_F32, JENGA_F32, 0.0, 0.0)
    _check(_lib.jenga_layer_norm_grad_workspace(ctypes.byref(cfg), ctypes.byref(bytes_)), "jenga_layer_norm_grad_workspace")
    return bytes_.value


def jenga_layer_norm_grad(x, dy, dx, weight, mean, rstd, dweight=None, dbias=None, workspace=None, group_rows=0,
                          weight_offset=0.0, stream=None):
    """Gradients of x [rows, cols] and of weight and bias, float32 [groups, cols], from dy and jenga_layer_norm's mean and rstd."""
    what = "jenga_layer_norm_grad"
    cfg = _norm_config(what, x, dy, weight, None, group_rows, weight_offset, 0.0)
    rows, cols = x.shape
    if dy.dtype != x.dtype or dx.dtype != x.dtype or _matrix(dx, what, rows, cols) != x.stride(0) and rows > 1:
        _refuse(what, "dy is not of x's type, or dx is not laid out as x is")
    if mean is None or rstd is None:
        _refuse(what, "mean and rstd of the forward pass are wanted")
    _whole(mean, what, (rows,), "f32")
    _whole(rstd, what, (rows,), "f32")
    groups = -(-rows // (group_rows or rows or 1))
    for t in (dweight, dbias):
        if t is not None:
            if t.numel() != groups * cols:
                _refuse(what, "gradients of %d groups" % groups)
            _whole(t, what, t.shape, "f32")
    stream = _on_device(what, (x, dy, dx, weight, mean, rstd, dweight, dbias, workspace), stream)
    at_room, room = (None, 0) if workspace is None else _room(workspace, what)
    if rows:
        _check(_lib.jenga_layer_norm_grad(cfg, x.data_ptr(), dy.data_ptr(), _ptr(weight), mean.data_ptr(), rstd.data_ptr(),
                                          dx.data_ptr(), _ptr(dweight), _ptr(dbias), at_room, room, stream), what)


# The calls below are written out where the ones above share helpers: a small one costs what its Python and a launch cost.

def _one_gpu(what, device):
    """Refuses a call whose tensors are on `device` as far as they have been compared; returns torch's current stream there."""
    if device < 0:
        _refuse(what, "tensors are not all on one GPU")
    if device != _current_device():
        _refuse(what, "tensors are not on the current device")
    return _current_stream(device)


def jenga_quantize_mx(x, q, scale, stream=None):
    """x [rows, cols] -> 4-bit tensor: q uint8 [rows, padded_columns(cols) / 2], scale uint8 [rows, padded_columns(cols) / 32]."""
    what = "jenga_quantize_mx"
    stride, kind = _matrix(x, what), _TYPES.get(x.dtype)
    if kind is None:
        kind = _type(x, what)
    rows, cols = x.shape
    blocks = (cols + 127) >> 7
    if not (q.dtype is scale.dtype is _U8 and q.shape == (rows, blocks << 6) and scale.shape == (rows, blocks << 2) and q.is_contiguous()
            and scale.is_contiguous()):
        _refuse(what, "shapes %s, %s for %d x %d" % (tuple(q.shape), tuple(scale.shape), rows, cols))
    device = x.get_device()
    current = _one_gpu(what, device if device == q.get_device() == scale.get_device() else -1)
    if cols > 0x7FFFFFFF:
        _refuse(what, "%d columns" % cols)
    if rows:
        status = _lib.jenga_quantize_mx(x.data_ptr(), stride, kind, rows, cols, q.data_ptr(), scale.data_ptr(),
                                        current if stream is None else stream)
        if status:
            raise JengaError(status, what)


def jenga_matmul_mx(a, a_scale, b, b_scale, out, bias=None, stream=None):
    """out [m, n] = a b^T + bias for 4-bit tensors, a uint8 [m, k / 2] and b uint8 [n, k / 2] with a scale for each 32 values; bias
    float32 [n]."""
    what = "jenga_matmul_mx"
    kind, of_a, of_b = _TYPES.get(out.dtype), a.shape, b.shape
    if kind is None:
        kind = _type(out, what)
    if len(of_a) != 2 or len(of_b) != 2:
        _refuse(what, "shapes %s, %s" % (tuple(of_a), tuple(of_b)))
    m, half = of_a
    n = of_b[0]
    stride = _matrix(out, what, m, n)
    if not (of_b[1] == half and a_scale.shape == (m, half >> 4) and b_scale.shape == (n, half >> 4)
            and a.dtype is b.dtype is a_scale.dtype is b_scale.dtype is _U8
            and a.is_contiguous() and b.is_contiguous() and a_scale.is_contiguous() and b_scale.is_contiguous()):
        _refuse(what, "operands of shapes %s, %s with scales %s, %s" % tuple(tuple(t.shape) for t in (a, b, a_scale, b_scale)))
    device = a.get_device()
    if not device == b.get_device() == a_scale.get_device() == b_scale.get_device() == out.get_device():
        device = -1
    at_bias = None
    if bias is not None:
        if not (bias.dtype is _F32 and bias.shape == (n,) and bias.is_contiguous()):
            _refuse(what, "bias of shape %s, type %s" % (tuple(bias.shape), bias.dtype))
        if bias.get_device() != device:
            device = -1
        at_bias = bias.data_ptr()
    current = _one_gpu(what, device)
    if m:
        status = _lib.jenga_matmul_mx(_pack(what, _MATMUL, m, stride, n, 2 * half, kind, 0), a.data_ptr(), a_scale.data_ptr(),
                                      b.data_ptr(), b_scale.data_ptr(), at_bias, out.data_ptr(), current if stream is None else stream)
        if status:
            raise JengaError(status, what)


def _apart(t, what, shape, dtype, whole):
    """Row and head stride of a tensor of this shape; `whole`: those of one without gaps.  Along an axis of one any stride will do."""
    if t.dtype is not dtype or t.shape != shape:
        _refuse(what, "shape %s, type %s" % (tuple(t.shape), t.dtype))
    if t.is_contiguous():
        return whole
    stride = t.stride()
    if stride[-1] != 1 and shape[-1] != 1:
        _refuse(what, "values of a row are not next to each other")
    return stride[0] if shape[0] > 1 else 0, stride[1] if len(shape) == 3 and shape[1] > 1 else 0


def _rms_sizes(x, what):
    shape = x.shape
    if len(shape) == 2:
        return shape, shape[0], 1, shape[1]
    if len(shape) != 3:
        _refuse(what, "shape %s" % (tuple(shape),))
    return shape, shape[0], shape[1], shape[2]


def _rms_weight(weight, what, cols):
    kind = _TYPES.get(weight.dtype)
    if kind is None:
        kind = _type(weight, what)
    if weight.shape != (cols,) or not weight.is_contiguous():
        _refuse(what, "weight of shape %s" % (tuple(weight.shape),))
    return kind


def jenga_rms_norm(x, y, weight=None, residual=None, total=None, y_scale=None, rstd=None, weight_offset=0.0, eps=1e-6, stream=None):
    """x, residual, total [rows, cols] or [rows, heads, cols] of one type, each with strides of its own; y the same, or of [rows, cols] an
    8-bit (e4m3; its bytes will not do here) or 4-bit (uint8) tensor with its scales in y_scale; weight [cols]; rstd float32 [rows] or [rows, heads].  total, or y,
    may be x or residual."""
    what = "jenga_rms_norm"
    dtype, device = x.dtype, x.get_device()
    kind = param_type = _TYPES.get(dtype)
    if kind is None:
        kind = param_type = _type(x, what)
    shape, rows, heads, cols = _rms_sizes(x, what)
    whole = heads * cols, cols
    x_row, x_head = _apart(x, what, shape, dtype, whole)
    add_row = add_head = sum_row = sum_head = y_row = y_head = 0
    at_add = at_sum = at_weight = at_scale = at_rstd = None
    if residual is not None:
        add_row, add_head = _apart(residual, what, shape, dtype, whole)
        at_add = residual.data_ptr()
        if residual.get_device() != device:
            device = -1
    if total is not None:
        sum_row, sum_head = _apart(total, what, shape, dtype, whole)
        at_sum = total.data_ptr()
        if total.get_device() != device:
            device = -1
    y_type = _TYPES.get(y.dtype)
    if y_type is None:
        y_type = _type(y, what)
    if y_type == JENGA_E4M3:
        padded = padded_columns(cols)
        if len(shape) != 2 or y_scale is None:
            _refuse(what, "results in 8 and 4 bits are of [rows, cols], with scales")
        if y.dtype is _U8:
            y_type = JENGA_E2M1
            _whole(y, what, (rows, padded >> 1), "u8")
            _whole(y_scale, what, (rows, padded >> 5), "u8")
        else:
            _whole(y, what, (rows, padded), "e4m3")
            _whole(y_scale, what, (rows, scale_columns(cols)), "u8")
        at_scale = y_scale.data_ptr()
        if y_scale.get_device() != device:
            device = -1
    else:
        y_row, y_head = _apart(y, what, shape, dtype, whole)
        if y_scale is not None:
            _refuse(what, "scales of a result that has none")
    if weight is not None:
        param_type = _rms_weight(weight, what, cols)
        at_weight = weight.data_ptr()
        if weight.get_device() != device:
            device = -1
    if rstd is not None:
        _whole(rstd, what, shape[:-1], "f32")
        at_rstd = rstd.data_ptr()
        if rstd.get_device() != device:
            device = -1
    current = _one_gpu(what, device if y.get_device() == device else -1)
    if rows and heads:
        cfg = _pack(what, _RMS, rows, x_row, x_head, add_row, add_head, sum_row, sum_head, y_row, y_head, heads, cols, kind, y_type, param_type,
                    eps, weight_offset, 0)
        status = _lib.jenga_rms_norm(cfg, x.data_ptr(), at_add, at_weight, at_sum, y.data_ptr(), at_scale, at_rstd,
                                     current if stream is None else stream)
        if status:
            raise JengaError(status, what)


def jenga_rms_norm_grad_workspace(rows, cols):
    """Bytes of the workspace of jenga_rms_norm_grad; rows: with their heads."""
    bytes_ = ctypes.c_uint64()
    cfg = _pack("jenga_rms_norm_grad_workspace", _RMS, rows, cols, cols, 0, 0, 0, 0, cols, cols, 1, cols, JENGA_F32, JENGA_F32, JENGA_F32,
                0.0, 0.0, 0)
    _check(_lib.jenga_rms_norm_grad_workspace(cfg, ctypes.byref(bytes_)), "jenga_rms_norm_grad_workspace")
    return bytes_.value


def jenga_rms_norm_grad(total, dy, dx, weight, rstd, dtotal=None, dweight=None, workspace=None, weight_offset=0.0, stream=None):
    """Gradients of total (what was normed; the same for x and residual) and of weight, float32 [cols], from dy, jenga_rms_norm's rstd and
    dtotal, the gradient that total has from elsewhere.  dx may be dtotal."""
    what = "jenga_rms_norm_grad"
    dtype, device = total.dtype, total.get_device()
    kind = param_type = _TYPES.get(dtype)
    if kind is None:
        kind = param_type = _type(total, what)
    shape, rows, heads, cols = _rms_sizes(total, what)
    whole = heads * cols, cols
    x_row, x_head = _apart(total, what, shape, dtype, whole)
    y_row, y_head = _apart(dy, what, shape, dtype, whole)
    sum_row, sum_head = _apart(dx, what, shape, dtype, whole)
    add_row = add_head = 0
    at_add = at_weight = at_dweight = at_room = None
    if dtotal is not None:
        add_row, add_head = _apart(dtotal, what, shape, dtype, whole)
        at_add = dtotal.data_ptr()
        if dtotal.get_device() != device:
            device = -1
    if weight is not None:
        param_type = _rms_weight(weight, what, cols)
        at_weight = weight.data_ptr()
        if weight.get_device() != device:
            device = -1
    if rstd is None:
        _refuse(what, "rstd of the forward pass is wanted")
    _whole(rstd, what, shape[:-1], "f32")
    room = 0
    if dweight is not None:
        _whole(dweight, what, (cols,), "f32")
        at_dweight = dweight.data_ptr()
        if dweight.get_device() != device:
            device = -1
    if workspace is not None:
        at_room, room = _room(workspace, what)
        if workspace.get_device() != device:
            device = -1
    current = _one_gpu(what, device if device == dy.get_device() == dx.get_device() == rstd.get_device() else -1)
    if rows and heads:
        cfg = _pack(what, _RMS, rows, x_row, x_head, add_row, add_head, sum_row, sum_head, y_row, y_head, heads, cols, kind, kind, param_type,
                    0.0, weight_offset, 0)
        status = _lib.jenga_rms_norm_grad(cfg, total.data_ptr(), dy.data_ptr(), at_weight, rstd.data_ptr(), at_add, dx.data_ptr(), at_dweight,
                                          at_room, room, current if stream is None else stream)
        if status:
            raise JengaError(status, what)


def _dense_bytes(call, q_rows, kv_rows, sequences, heads, kv_heads, head_dim):
    bytes_ = ctypes.c_uint64()
    cfg = _pack(call, _DENSE, q_rows, kv_rows, 0, 0, 0, 0, 0, 0, 0, 0, sequences, heads, kv_heads, head_dim, JENGA_BF16, 0, 1.0, 0)
    _check(getattr(_lib, call)(cfg, ctypes.byref(bytes_)), call)
    return bytes_.value


def jenga_dense_attn_workspace(q_rows, kv_rows, sequences, heads, kv_heads, head_dim):
    """Bytes of the workspace of jenga_dense_attn for just these numbers of rows, keys and sequences in all; fewer may need more."""
    return _dense_bytes("jenga_dense_attn_workspace", q_rows, kv_rows, sequences, heads, kv_heads, head_dim)


def jenga_dense_attn_workspace_up_to(q_rows, kv_rows, sequences, heads, kv_heads, head_dim):
    """Bytes that are enough for every call with no more rows, keys and sequences."""
    return _dense_bytes("jenga_dense_attn_workspace_up_to", q_rows, kv_rows, sequences, heads, kv_heads, head_dim)


def jenga_dense_attn(q, k, v, out, q_start, kv_start, kv_len=None, causal=False, scale=None, workspace=None, stream=None):
    """q, out [rows, heads, head_dim], k, v [keys, kv_heads, head_dim] (bf16 or fp16, any strides but the last); q_start, kv_start int32
    [sequences + 1], kv_len int32 [sequences], on the device: rows and keys of each sequence.  out may be q.  scale: 1 / sqrt(head_dim)."""
    what = "jenga_dense_attn"
    dtype, shape, keys, device = q.dtype, q.shape, k.shape, q.get_device()
    kind = _TYPES.get(dtype)
    if kind is None:
        kind = _type(q, what)
    if len(shape) != 3 or len(keys) != 3 or keys[2] != shape[2] or not shape[2]:
        _refuse(what, "shapes %s, %s" % (tuple(shape), tuple(keys)))
    rows, heads, dim = shape
    whole, whole_kv = (heads * dim, dim), (keys[1] * dim, dim)
    q_row, q_head = _apart(q, what, shape, dtype, whole)
    out_row, out_head = _apart(out, what, shape, dtype, whole)
    k_row, k_head = _apart(k, what, keys, dtype, whole_kv)
    v_row, v_head = _apart(v, what, keys, dtype, whole_kv)
    sequences = q_start.numel() - 1
    if not (sequences >= 0 and q_start.dtype is kv_start.dtype is _I32 and q_start.shape == kv_start.shape == (sequences + 1,)
            and q_start.is_contiguous() and kv_start.is_contiguous()):
        _refuse(what, "starts of shapes %s, %s, types %s, %s" % (tuple(q_start.shape), tuple(kv_start.shape), q_start.dtype, kv_start.dtype))
    at_len = None
    if kv_len is not None:
        _whole(kv_len, what, (sequences,), "i32")
        at_len = kv_len.data_ptr()
        if kv_len.get_device() != device:
            device = -1
    if workspace is None:
        _refuse(what, "a workspace is wanted")
    at_room, room = _room(workspace, what)
    if not device == k.get_device() == v.get_device() == out.get_device() == q_start.get_device() == kv_start.get_device() == \
            workspace.get_device():
        device = -1
    current = _one_gpu(what, device)
    if rows and heads:
        cfg = _pack(what, _DENSE, rows, keys[0], q_row, q_head, k_row, k_head, v_row, v_head, out_row, out_head, sequences, heads, keys[1], dim,
                    kind, JENGA_DENSE_CAUSAL if causal else 0, dim ** -0.5 if scale is None else scale, 0)
        # without keys there is nothing to read, but the call wants addresses
        here = q.data_ptr()
        status = _lib.jenga_dense_attn(cfg, here, k.data_ptr() or here, v.data_ptr() or here, q_start.data_ptr(), kv_start.data_ptr(), at_len,
                                       out.data_ptr(), at_room, room, current if stream is None else stream)
        if status:
            raise JengaError(status, what)


def make_rotary(T, H, W, head_dim, dims, theta=10000.0, origin=(0.0, 0.0, 0.0), step=(1.0, 1.0, 1.0), flags=0):
    """dims: channels of the three axes.  The element type is set by each call from its tensors."""
    return jenga_rotary_config(T, H, W, head_dim, (ctypes.c_int32 * 3)(*dims), JENGA_BF16, theta, (ctypes.c_double * 3)(*origin),
                               (ctypes.c_double * 3)(*step), flags, 0)


def jenga_rotary_table(cfg, table):
    """table: float32 numpy array or CPU tensor of T dim[0] + H dim[1] + W dim[2] values, in any shape."""
    want = cfg.T * cfg.dim[0] + cfg.H * cfg.dim[1] + cfg.W * cfg.dim[2]
    count = table.numel() if hasattr(table, "numel") else table.size
    contiguous = table.is_contiguous() if hasattr(table, "is_contiguous") else table.flags.c_contiguous
    if count != want or not str(table.dtype).endswith("float32") or not contiguous or getattr(table, "is_cuda", False):
        _refuse("jenga_rotary_table", "a table of %d float32 on the host is wanted" % want)
    _check(_lib.jenga_rotary_table(ctypes.byref(cfg), _ptr(table)), "jenga_rotary_table")


def _rotary_table(cfg, table, what):
    dim = cfg.dim
    if table.numel() != cfg.T * dim[0] + cfg.H * dim[1] + cfg.W * dim[2] or not table.is_contiguous() or _type(table, what) != JENGA_F32:
        _refuse(what, "not a table of this grid")


def _rotary_tensor(cfg, src, dst, what):
    shape, s, d = src.shape, src.stride(), dst.stride()
    if len(shape) != 4 or dst.shape != shape or shape[3] != cfg.head_dim:
        _refuse(what, "shapes %s, %s" % (tuple(shape), tuple(dst.shape)))
    if s[3] != 1 or d[3] != 1 or dst.dtype != src.dtype:
        _refuse(what, "types differ or the channels of a head are not next to each other")
    return _pack(what, _TENSOR, src.data_ptr(), dst.data_ptr(), s[0], s[1], s[2], d[0], d[1], d[2], shape[2], 0)


def jenga_rotary(cfg, table, q, q_out, k=None, k_out=None, cells=None, plan=None, stream=None):
    """q, k [batch, tokens, heads, head_dim] (heads may differ, any strides but the last) -> q_out, k_out, which may be q and k.
    plan: tokens in its curve order (a curve-side tensor transposed to this shape); cells: int32 [batch, tokens, 3]."""
    what = "jenga_rotary"
    kind = _type(q, what)
    if (k is None) != (k_out is None):
        _refuse(what, "k without k_out, or the other way round")
    if k is None:
        tensors = _rotary_tensor(cfg, q, q_out, what)
    else:
        tensors = _rotary_tensor(cfg, q, q_out, what) + _rotary_tensor(cfg, k, k_out, what)
        if k.dtype != q.dtype or k.shape[:2] != q.shape[:2]:
            _refuse(what, "q and k differ in type or tokens")
    batch, tokens = q.shape[0], q.shape[1]
    _rotary_table(cfg, table, what)
    if cells is not None:
        _whole(cells, what, (batch, tokens, 3), "i32")
    stream = _on_device(what, (q, q_out, k, k_out, table, cells), stream)
    if batch and tokens:
        if cfg.type != kind:
            cfg = jenga_rotary_config.from_buffer_copy(cfg)
            cfg.type = kind
        _check(_lib.jenga_rotary(ctypes.byref(cfg), plan, None if cells is None else cells.data_ptr(), table.data_ptr(), tensors,
                                 1 if k is None else 2, batch, tokens, stream), what)


def jenga_forward_rotary(plan, cfg, table, q_thw, k_thw, v_thw, q_curve, k_curve, v_curve, sel_count, sel_index, mask,
                         select_workspace, select_workspace_bytes, out_curve, lse, attn_workspace, attn_workspace_bytes, out_thw,
                         stream=None):
    """q_thw, k_thw, v_thw: [batch, N_v + N_c, heads, head_dim], tokens the same distance apart in all three."""
    what = "jenga_forward_rotary"
    if len(q_thw.shape) != 4:
        _refuse(what, "shape %s" % (tuple(q_thw.shape),))
    batch, tokens, heads, dim = q_thw.shape
    stride = q_thw.stride(1) if tokens > 1 else q_thw.stride(0) if batch > 1 else heads * dim
    for t in (q_thw, k_thw, v_thw):
        s = t.stride()
        if t.shape != q_thw.shape or _type(t, what) != JENGA_BF16 or s[3] != 1 or (heads > 1 and s[2] != dim) or \
                (tokens > 1 and s[1] != stride) or (batch > 1 and s[0] != stride * tokens):
            _refuse(what, "shape %s, strides %s, type %s" % (tuple(t.shape), s, t.dtype))
    _rotary_table(cfg, table, what)
    stream = _on_device(what, (table, q_thw, k_thw, v_thw), stream)
    _check(_lib.jenga_forward_rotary(plan, ctypes.byref(cfg), _ptr(table), _ptr(q_thw), _ptr(k_thw), _ptr(v_thw), stride, _ptr(q_curve),
                                     _ptr(k_curve), _ptr(v_curve), _ptr(sel_count), _ptr(sel_index), _ptr(mask),
                                     _ptr(select_workspace), select_workspace_bytes, _ptr(out_curve), _ptr(lse),
                                     _ptr(attn_workspace), attn_workspace_bytes, _ptr(out_thw), stream), what)


def raw():
    """The ctypes library object, for tests of the error paths."""
    return _lib
