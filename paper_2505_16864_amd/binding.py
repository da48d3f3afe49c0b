"""ctypes binding of libjenga.so: the same names as the C ABI, argument marshalling only.

Every step of the path runs in the library's HIP kernels.  If the library has not been built the
import of this module fails: there is no fallback.
"""
import ctypes
import os

PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(PKG, "libjenga.so")

JENGA_FLAG_ADJACENCY = 1
JENGA_FLAG_CONDITION = 2
JENGA_FLAG_CURVE = 4
JENGA_FLAG_PACED_WALK = 8

JENGA_BF16, JENGA_F16, JENGA_F32, JENGA_E4M3 = range(4)
JENGA_ROTARY_HALVES = 1
JENGA_ROTARY_INVERSE = 2

EXPORTS = ["jenga_plan_create", "jenga_plan_destroy", "jenga_plan_info", "jenga_plan_export", "jenga_plan_tables",
           "jenga_curve_permute", "jenga_curve_permute_qkv", "jenga_curve_permute_rows", "jenga_select_blocks",
           "jenga_select_blocks_static",
           "jenga_block_sparse_attn", "jenga_pack_kv",
           "jenga_block_sparse_attn_packed", "jenga_unpermute", "jenga_forward", "jenga_stage_switch",
           "jenga_quantize", "jenga_matmul", "jenga_layer_norm", "jenga_layer_norm_grad", "jenga_layer_norm_grad_workspace",
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
    lib.jenga_matmul.argtypes = [ctypes.POINTER(jenga_matmul_config)] + [vp] * 7
    norm = ctypes.POINTER(jenga_norm_config)
    lib.jenga_layer_norm.argtypes = [norm] + [vp] * 8
    lib.jenga_layer_norm_grad.argtypes = [norm] + [vp] * 9 + [size, vp]
    lib.jenga_layer_norm_grad_workspace.argtypes = [norm, ctypes.POINTER(ctypes.c_uint64)]
    lib.jenga_rotary_table.argtypes = [ctypes.POINTER(jenga_rotary_config), vp]
    lib.jenga_rotary.argtypes = [ctypes.POINTER(jenga_rotary_config), vp, vp, vp, ctypes.POINTER(jenga_rotary_tensor), i32, i64,
                                 i64, vp]
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
# checked here: values next to each other in the last dimension, all tensors on the device that is current.

_EINVAL = -1


def _types():
    import torch
    return {torch.bfloat16: JENGA_BF16, torch.float16: JENGA_F16, torch.float32: JENGA_F32, torch.float8_e4m3fn: JENGA_E4M3,
            torch.uint8: JENGA_E4M3}


_TYPES = {}


def _type(t, what):
    if not _TYPES:
        _TYPES.update(_types())
    code = _TYPES.get(t.dtype)
    if code is None:
        raise JengaError(_EINVAL, "%s: element type %s" % (what, t.dtype))
    return code


def _need(ok, what, why):
    if not ok:
        raise JengaError(_EINVAL, "%s: %s" % (what, why))


def _on_device(what, *tensors):
    import torch
    on = {t.get_device() for t in tensors if t is not None}
    _need(len(on) == 1 and on != {-1} and on == {torch._C._cuda_getDevice()}, what, "a tensor is not on the current device")


def _matrix(t, what, shape=None):
    """The row stride of a matrix; of a single row any stride will do."""
    _need(t.dim() == 2 and (shape is None or tuple(t.shape) == tuple(shape)), what, "shape %s" % (tuple(t.shape),))
    _need(t.stride(1) == 1 or t.shape[1] == 1, what, "values of a row are not next to each other")
    return t.stride(0) if t.shape[0] > 1 else max(t.stride(0), t.shape[1])


def _plain(t, what, shape, dtype):
    """A tensor of this shape and type without gaps, or None."""
    if t is not None:
        _need(tuple(t.shape) == tuple(shape) and str(t.dtype)[6:] in dtype and t.is_contiguous(), what,
              "shape %s, type %s" % (tuple(t.shape), t.dtype))


def scale_columns(cols):
    """Bytes of a row of scales of an 8-bit tensor with `cols` columns."""
    return -(-cols // 512) * 4


def padded_columns(cols):
    """Columns of an 8-bit tensor that holds `cols` columns."""
    return -(-cols // 128) * 128


_E4M3 = ("float8_e4m3fn", "uint8")


def jenga_quantize(x, q, scale, block_rows=1, stream=None):
    """x [rows, cols] -> q e4m3 [rows, padded_columns(cols)], scale uint8 [rows or ceil(rows / 128), scale_columns(cols)]."""
    what = "jenga_quantize"
    stride = _matrix(x, what)
    rows, cols = x.shape
    _plain(q, what, (rows, padded_columns(cols)), _E4M3)
    _need(block_rows in (1, 128), what, "blocks of %s rows" % block_rows)
    _plain(scale, what, (-(-rows // block_rows), scale_columns(cols)), ("uint8",))
    _on_device(what, x, q, scale)
    if rows == 0:
        return
    _check(_lib.jenga_quantize(_ptr(x), stride, _type(x, what), rows, cols, block_rows, _ptr(q), _ptr(scale), stream), what)


def jenga_matmul(a, a_scale, b, b_scale, out, bias=None, stream=None):
    """out [m, n] = a b^T + bias for 8-bit tensors a [m, k] (blocks of 1 x 128) and b [n, k] (128 x 128); bias float32 [n]."""
    what = "jenga_matmul"
    stride = _matrix(out, what, (a.shape[0], b.shape[0]))
    (m, n), k = out.shape, a.shape[1]
    _plain(a, what, (m, k), _E4M3)
    _plain(b, what, (n, k), _E4M3)
    _plain(a_scale, what, (m, scale_columns(k)), ("uint8",))
    _plain(b_scale, what, (-(-n // 128), scale_columns(k)), ("uint8",))
    _plain(bias, what, (n,), ("float32",))
    _on_device(what, a, a_scale, b, b_scale, out, bias)
    if m == 0:
        return
    cfg = jenga_matmul_config(m, stride, n, k, _type(out, what), 0)
    _check(_lib.jenga_matmul(ctypes.byref(cfg), _ptr(a), _ptr(a_scale), _ptr(b), _ptr(b_scale), _ptr(bias), _ptr(out), stream), what)


def _norm_config(what, x, y, weight, bias, group_rows, weight_offset, eps):
    x_stride = _matrix(x, what)
    rows, cols = x.shape
    group_rows = group_rows or max(rows, 1)
    _need(group_rows > 0, what, "groups of %d rows" % group_rows)
    groups = -(-rows // group_rows)
    params = [(p.unsqueeze(0) if p.dim() == 1 else p) for p in (weight, bias) if p is not None]
    strides = [_matrix(p, what, (groups, cols) if rows else None) for p in params]
    _need(len(set(strides)) < 2 and len({p.dtype for p in params}) < 2, what, "weight and bias differ in stride or type")
    e4m3 = _type(y, what) == JENGA_E4M3
    y_stride = _matrix(y, what, (rows, padded_columns(cols) if e4m3 else cols))
    return jenga_norm_config(rows, group_rows, x_stride, y_stride, strides[0] if strides else cols, cols, _type(x, what),
                             _type(y, what), _type(params[0], what) if params else JENGA_F32, eps, weight_offset)


def jenga_layer_norm(x, y, weight=None, bias=None, y_scale=None, mean=None, rstd=None, group_rows=0, weight_offset=0.0,
                     eps=1e-6, stream=None):
    """x, y [rows, cols]; weight, bias [cols] or [groups, cols], a group for each group_rows rows (0: one for all); mean, rstd
    float32 [rows].  y in e4m3: [rows, padded_columns(cols)] with y_scale uint8 [rows, scale_columns(cols)]."""
    what = "jenga_layer_norm"
    cfg = _norm_config(what, x, y, weight, bias, group_rows, weight_offset, eps)
    _plain(y_scale, what, (cfg.rows, scale_columns(cfg.cols)), ("uint8",))
    _plain(mean, what, (cfg.rows,), ("float32",))
    _plain(rstd, what, (cfg.rows,), ("float32",))
    _on_device(what, x, y, weight, bias, y_scale, mean, rstd)
    if cfg.rows == 0:
        return
    _check(_lib.jenga_layer_norm(ctypes.byref(cfg), _ptr(x), _ptr(weight), _ptr(bias), _ptr(y), _ptr(y_scale), _ptr(mean),
                                 _ptr(rstd), stream), what)


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
    _need(cfg.y_type == cfg.x_type, what, "dy is not of x's type")
    _need(_matrix(dx, what, x.shape) == cfg.x_stride and dx.dtype == x.dtype, what, "dx is not laid out as x is")
    groups = -(-cfg.rows // cfg.group_rows)
    for t in (mean, rstd):
        _need(t is not None, what, "mean and rstd of the forward pass are wanted")
        _plain(t, what, (cfg.rows,), ("float32",))
    for t in (dweight, dbias):
        _need(t is None or t.numel() == groups * cfg.cols, what, "gradients of %d groups" % groups)
        _plain(t, what, t.shape if t is not None else (), ("float32",))
    _on_device(what, x, dy, dx, weight, mean, rstd, dweight, dbias, workspace)
    if cfg.rows == 0:
        return
    room = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(_lib.jenga_layer_norm_grad(ctypes.byref(cfg), _ptr(x), _ptr(dy), _ptr(weight), _ptr(mean), _ptr(rstd), _ptr(dx),
                                      _ptr(dweight), _ptr(dbias), _ptr(workspace), room, stream), what)


def make_rotary(T, H, W, head_dim, dims, theta=10000.0, origin=(0.0, 0.0, 0.0), step=(1.0, 1.0, 1.0), flags=0):
    """dims: channels of the three axes.  The element type is set by each call from its tensors."""
    return jenga_rotary_config(T, H, W, head_dim, (ctypes.c_int32 * 3)(*dims), JENGA_BF16, theta, (ctypes.c_double * 3)(*origin),
                               (ctypes.c_double * 3)(*step), flags, 0)


def jenga_rotary_table(cfg, table):
    """table: float32 numpy array or CPU tensor of T dim[0] + H dim[1] + W dim[2] values, in any shape."""
    want = cfg.T * cfg.dim[0] + cfg.H * cfg.dim[1] + cfg.W * cfg.dim[2]
    count = table.numel() if hasattr(table, "numel") else table.size
    contiguous = table.is_contiguous() if hasattr(table, "is_contiguous") else table.flags.c_contiguous
    _need(count == want and str(table.dtype).endswith("float32") and contiguous and not getattr(table, "is_cuda", False),
          "jenga_rotary_table", "a table of %d float32 on the host is wanted" % want)
    _check(_lib.jenga_rotary_table(ctypes.byref(cfg), _ptr(table)), "jenga_rotary_table")


def _rotary_table(cfg, table, what):
    _need(table.numel() == cfg.T * cfg.dim[0] + cfg.H * cfg.dim[1] + cfg.W * cfg.dim[2] and table.is_contiguous() and
          str(table.dtype).endswith("float32"), what, "not a table of this grid")


def jenga_rotary(cfg, table, q, q_out, k=None, k_out=None, cells=None, plan=None, stream=None):
    """q, k [batch, tokens, heads, head_dim] (heads may differ, any strides but the last) -> q_out, k_out, which may be q and k.
    plan: tokens in its curve order (a curve-side tensor transposed to this shape); cells: int32 [batch, tokens, 3]."""
    what = "jenga_rotary"
    batch, tokens = q.shape[:2]
    tensors = (jenga_rotary_tensor * 2)()
    pairs = [(q, q_out)] if k is None else [(q, q_out), (k, k_out)]
    for t, (src, dst) in zip(tensors, pairs):
        _need(src.dim() == 4 and src.shape == dst.shape and src.shape[:2] == q.shape[:2] and src.shape[3] == cfg.head_dim, what,
              "shapes %s, %s" % (tuple(src.shape), tuple(dst.shape)))
        _need(src.dtype == q.dtype and dst.dtype == q.dtype and src.stride(3) == 1 and dst.stride(3) == 1, what,
              "types differ or the channels of a head are not next to each other")
        t.src, t.dst, t.heads = src.data_ptr(), dst.data_ptr(), src.shape[2]
        t.src_batch, t.src_token, t.src_head = src.stride()[:3]
        t.dst_batch, t.dst_token, t.dst_head = dst.stride()[:3]
    _rotary_table(cfg, table, what)
    _plain(cells, what, (batch, tokens, 3), ("int32",))
    _on_device(what, table, q, q_out, k, k_out, cells)
    if batch == 0 or tokens == 0:
        return
    mine = jenga_rotary_config.from_buffer_copy(cfg)
    mine.type = _type(q, what)
    _check(_lib.jenga_rotary(ctypes.byref(mine), plan, _ptr(cells), _ptr(table), tensors, len(pairs), batch, tokens, stream), what)


def jenga_forward_rotary(plan, cfg, table, q_thw, k_thw, v_thw, q_curve, k_curve, v_curve, sel_count, sel_index, mask,
                         select_workspace, select_workspace_bytes, out_curve, lse, attn_workspace, attn_workspace_bytes, out_thw,
                         stream=None):
    """q_thw, k_thw, v_thw: [batch, N_v + N_c, heads, head_dim], tokens the same distance apart in all three."""
    what = "jenga_forward_rotary"
    batch, tokens, heads, dim = q_thw.shape
    stride = q_thw.stride(1) if tokens > 1 else q_thw.stride(0) if batch > 1 else heads * dim
    for t in (q_thw, k_thw, v_thw):
        _need(t.shape == q_thw.shape and str(t.dtype) == "torch.bfloat16" and t.stride(3) == 1 and (heads == 1 or t.stride(2) == dim) and
              (tokens == 1 or t.stride(1) == stride) and (batch == 1 or t.stride(0) == stride * tokens), what,
              "shape %s, strides %s" % (tuple(t.shape), t.stride()))
    _rotary_table(cfg, table, what)
    _on_device(what, table, q_thw, k_thw, v_thw)
    _check(_lib.jenga_forward_rotary(plan, ctypes.byref(cfg), _ptr(table), _ptr(q_thw), _ptr(k_thw), _ptr(v_thw), stride, _ptr(q_curve),
                                     _ptr(k_curve), _ptr(v_curve), _ptr(sel_count), _ptr(sel_index), _ptr(mask),
                                     _ptr(select_workspace), select_workspace_bytes, _ptr(out_curve), _ptr(lse),
                                     _ptr(attn_workspace), attn_workspace_bytes, _ptr(out_thw), stream), what)


def raw():
    """The ctypes library object, for tests of the error paths."""
    return _lib
