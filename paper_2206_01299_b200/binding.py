"""ctypes binding of libaq_b200.so: the same names as include/aq_b200.h, argument
marshalling only.  Every operation runs in the CUDA library; there is no Python or CPU
implementation behind these calls, and a missing library is an error.

Pointer arguments accept a torch tensor (its data_ptr() is passed; the tensor must be
contiguous), a numpy array (host forms), an int address, or None.
"""
import ctypes as C
import os

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libaq_b200.so")

AQ_OK, AQ_EINVAL, AQ_ENOMEM, AQ_ECUDA, AQ_EUNSUPPORTED = 0, -1, -2, -3, -4
AQ_DTYPE, AQ_BATCH, AQ_STREAM, AQ_RAW, AQ_FIRST_FLAGS, AQ_ROWS_PER_CTA = 1, 2, 3, 4, 5, 6
AQ_L2_PREFETCH = 10
AQ_RAW_LIST = 11
AQ_ROUNDING, AQ_SEED, AQ_EPOCH = 7, 8, 9
AQ_FP16, AQ_BF16, AQ_FP32 = 0, 1, 2
AQ_ROUND_INTERVAL, AQ_ROUND_STOCHASTIC = 0, 1
AQ_ACT_SILU, AQ_ACT_GELU, AQ_ACT_GELU_TANH = 0, 1, 2
AQ_ST_BAD_ID, AQ_ST_DUP_ID, AQ_ST_NO_RAW, AQ_ST_STAGED, AQ_ST_BAD_PTR = 1, 2, 4, 8, 16
AQ_ST_STALLED = 32


class QkShape(C.Structure):
    """aq_qk_shape: the heads of aq_qk_norm_rope."""
    _fields_ = [("heads_q", C.c_int32), ("heads_k", C.c_int32), ("head_dim", C.c_int32), ("rot_dim", C.c_int32),
                ("interleaved", C.c_int32), ("eps", C.c_float), ("n_positions", C.c_int64)]


class AdamTensor(C.Structure):
    """aq_adam_tensor: one tensor of aq_adamw or aq_grad_norm; aq_adam_table makes an array of them."""
    _fields_ = [("param", C.c_void_p), ("master", C.c_void_p), ("grad", C.c_void_p), ("m", C.c_void_p), ("v", C.c_void_p),
                ("m_scale", C.c_void_p), ("v_scale", C.c_void_p), ("numel", C.c_int64), ("weight_decay", C.c_float), ("grad_dtype", C.c_int32)]


class AdamwConfig(C.Structure):
    """aq_adamw_config: the settings of aq_adamw."""
    _fields_ = [("lr", C.c_double), ("beta1", C.c_double), ("beta2", C.c_double), ("eps", C.c_double), ("step", C.c_int64),
                ("state_bits", C.c_int32)]


_P, _I, _L, _F, _D = C.c_void_p, C.c_int, C.c_int64, C.c_float, C.c_double

# name -> (restype, argtypes); the load test checks these against the header
SIGNATURES = {
    "aq_create": (C.c_void_p, [C.c_int64, C.c_int, C.c_int, C.c_int, C.c_int]),
    "aq_create_hosted": (C.c_void_p, [C.c_int64, C.c_int, C.c_int, C.c_int, C.c_int]),
    "aq_create_fp32": (C.c_void_p, [C.c_int64, C.c_int, C.c_int, C.c_int, C.c_int]),
    "aq_create_lowbit": (C.c_void_p, [C.c_int64, C.c_int, C.c_int, C.c_int, C.c_int, C.c_int]),
    "aq_create_hosted_lowbit": (C.c_void_p, [C.c_int64, C.c_int, C.c_int, C.c_int, C.c_int, C.c_int]),
    "aq_destroy": (None, [C.c_void_p]),
    "aq_configure": (C.c_int, [C.c_void_p, C.c_int, C.c_int64]),
    "aq_encode": (C.c_int, [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]),
    "aq_decode": (C.c_int, [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]),
    "aq_encode_list": (C.c_int, [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]),
    "aq_decode_list": (C.c_int, [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]),
    "aq_quant_grad": (C.c_int, [C.c_void_p, C.c_void_p, C.c_int64, C.c_int, C.c_void_p, C.c_void_p]),
    "aq_dequant_grad": (C.c_int, [C.c_void_p, C.c_void_p, C.c_void_p, C.c_int64, C.c_int, C.c_void_p]),
    "aq_state_checksum": (C.c_int, [C.c_void_p, C.POINTER(C.c_uint64)]),
    "aq_state_checksum_noalloc": (C.c_int, [C.c_void_p, C.POINTER(C.c_uint64)]),
    "aq_status": (C.c_int, [C.c_void_p, C.POINTER(C.c_uint32)]),
    "aq_last_error": (C.c_char_p, [C.c_void_p]),
    "aq_last_error_code": (C.c_int, [C.c_void_p]),
    "aq_packed_bytes_per_sample": (C.c_int64, [C.c_void_p]),
    "aq_scales_per_sample": (C.c_int64, [C.c_void_p]),
    "aq_m_bytes_per_sample": (C.c_int64, [C.c_void_p]),
    "aq_encode_host": (C.c_int, [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]),
    "aq_decode_host": (C.c_int, [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]),
    "aq_wire_copy": (C.c_int, [C.c_void_p, C.c_int, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p,
                               C.c_void_p]),
    "aq_wire_copy_grad": (C.c_int, [C.c_void_p, C.c_int, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_int64, C.c_int]),
    "aq_prefetch": (C.c_int, [C.c_void_p, C.c_void_p, C.c_int]),
    "aq_export_sample": (C.c_int, [C.c_void_p, C.c_int64, C.c_void_p, C.c_void_p]),
    "aq_import_sample": (C.c_int, [C.c_void_p, C.c_int64, C.c_void_p, C.c_uint8]),
    "aq_stage_create": (_P, []),
    "aq_stage_destroy": (None, [_P]),
    "aq_stage_configure": (_I, [_P, _I, _L]),
    "aq_stage_status": (_I, [_P, C.POINTER(C.c_uint32)]),
    "aq_stage_last_error": (C.c_char_p, [_P]),
    "aq_stage_last_error_code": (_I, [_P]),
    "aq_token_logprobs": (_I, [_P, _P, _L, _L, _L, _P, _F, _I, _P, _P, _P, _P, _P]),
    "aq_token_logprobs_grad": (_I, [_P, _P, _L, _L, _L, _P, _F, _P, _P, _P, _P, _P, _L]),
    "aq_gated_ffn": (_I, [_P, _P, _L, _P, _P, _L, _L, _I, _I, _I, _P, _L, _P, _P, _L]),
    "aq_gated_ffn_grad": (_I, [_P, _P, _L, _P, _L, _P, _P, _L, _P, _P, _L, _L, _I, _I, _I, _P, _L, _P, _P, _L]),
    "aq_qk_norm_rope": (_I, [_P, _P, _L, _P, _L, _P, _L, _P, _P, _P, _P, _P, _L, _P, _L]),
    "aq_qk_norm_rope_grad": (_I, [_P, _P, _L, _P, _L, _P, _L, _P, _L, _P, _L, _P, _P, _P, _P, _P, _L, _P, _L, _P, _P]),
    "aq_layer_norm": (_I, [_P, _P, _L, _P, _L, _P, _P, _F, _L, _I, _P, _L, _P, _L, _P, _P]),
    "aq_layer_norm_grad": (_I, [_P, _P, _L, _P, _L, _P, _L, _P, _P, _P, _L, _I, _P, _L, _P, _P]),
    "aq_grad_norm": (_I, [_P, _P, _L, _D, _D, _P, _P, _P]),
    "aq_adamw": (_I, [_P, _P, _P, _L, _P, _P, _P]),
}

_lib = None


def lib():
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(
                f"{LIB_PATH} is missing: build it with `python -m paper_2206_01299_b200.build` "
                "(nvcc, sm_100a).  There is no fallback implementation.")
        L = C.CDLL(LIB_PATH)
        for name, (res, args) in SIGNATURES.items():
            fn = getattr(L, name)
            fn.restype, fn.argtypes = res, args
        _lib = L
    return _lib


class AqError(RuntimeError):
    def __init__(self, code, msg):
        super().__init__(f"aq error {code}: {msg}")
        self.code = code


def _ptr(x):
    if x is None:
        return None
    if isinstance(x, int):
        return x
    if hasattr(x, "data_ptr"):
        assert x.is_contiguous(), "tensor must be contiguous"
        return x.data_ptr()
    if hasattr(x, "ctypes"):
        assert x.flags["C_CONTIGUOUS"], "array must be contiguous"
        return x.ctypes.data
    raise TypeError(type(x))


def _check(h, rc):
    if rc != AQ_OK:
        raise AqError(rc, aq_last_error(h))
    return rc


def _created(h):
    if not h:
        raise AqError(aq_last_error_code(None), aq_last_error(None))
    return h


def aq_create(n_samples, seq, hidden, bits, group):
    return _created(lib().aq_create(n_samples, seq, hidden, bits, group))


def aq_create_hosted(n_samples, seq, hidden, bits, group):
    return _created(lib().aq_create_hosted(n_samples, seq, hidden, bits, group))


def aq_create_fp32(n_samples, seq, hidden, bits, group):
    return _created(lib().aq_create_fp32(n_samples, seq, hidden, bits, group))


def aq_create_lowbit(n_samples, seq, hidden, bits, group, m_bits):
    return _created(lib().aq_create_lowbit(n_samples, seq, hidden, bits, group, m_bits))


def aq_create_hosted_lowbit(n_samples, seq, hidden, bits, group, m_bits):
    return _created(lib().aq_create_hosted_lowbit(n_samples, seq, hidden, bits, group, m_bits))


def aq_destroy(h):
    lib().aq_destroy(h)


def aq_configure(h, key, value):
    """value: an int, or a tensor / None for the pointer-valued keys (AQ_RAW, AQ_FIRST_FLAGS)."""
    val = value if isinstance(value, int) else (_ptr(value) or 0)
    return _check(h, lib().aq_configure(h, key, val))


def aq_encode(h, act, sample_ids, packed, scales):
    return _check(h, lib().aq_encode(h, _ptr(act), _ptr(sample_ids), _ptr(packed), _ptr(scales)))


def aq_decode(h, packed, scales, sample_ids, out):
    return _check(h, lib().aq_decode(h, _ptr(packed), _ptr(scales), _ptr(sample_ids), _ptr(out)))


def aq_encode_list(h, act_list, sample_ids, packed_list, scales_list):
    """The *_list arguments are int64 device tensors holding one device address per sample."""
    return _check(h, lib().aq_encode_list(h, _ptr(act_list), _ptr(sample_ids), _ptr(packed_list), _ptr(scales_list)))


def aq_decode_list(h, packed_list, scales_list, sample_ids, out_list):
    return _check(h, lib().aq_decode_list(h, _ptr(packed_list), _ptr(scales_list), _ptr(sample_ids), _ptr(out_list)))


def aq_quant_grad(h, grad, n_elems, bits, packed, scales):
    return _check(h, lib().aq_quant_grad(h, _ptr(grad), n_elems, bits, _ptr(packed), _ptr(scales)))


def aq_dequant_grad(h, packed, scales, n_elems, bits, out):
    return _check(h, lib().aq_dequant_grad(h, _ptr(packed), _ptr(scales), n_elems, bits, _ptr(out)))


def aq_state_checksum(h):
    v = C.c_uint64(0)
    _check(h, lib().aq_state_checksum(h, C.byref(v)))
    return v.value


def aq_state_checksum_noalloc(h):
    """aq_state_checksum through the library's fixed scratch array: no device allocation."""
    v = C.c_uint64(0)
    _check(h, lib().aq_state_checksum_noalloc(h, C.byref(v)))
    return v.value


def aq_status(h):
    v = C.c_uint32(0)
    _check(h, lib().aq_status(h, C.byref(v)))
    return v.value


def aq_last_error(h):
    return lib().aq_last_error(h).decode()


def aq_last_error_code(h):
    return lib().aq_last_error_code(h)


def aq_packed_bytes_per_sample(h):
    return lib().aq_packed_bytes_per_sample(h)


def aq_scales_per_sample(h):
    return lib().aq_scales_per_sample(h)


def aq_m_bytes_per_sample(h):
    return lib().aq_m_bytes_per_sample(h)


def aq_encode_host(h, act_host, sample_ids_host, packed_host, scales_host):
    return _check(h, lib().aq_encode_host(h, _ptr(act_host), _ptr(sample_ids_host), _ptr(packed_host),
                                          _ptr(scales_host)))


def aq_decode_host(h, packed_host, scales_host, raw_host, sample_ids_host, out_host):
    return _check(h, lib().aq_decode_host(h, _ptr(packed_host), _ptr(scales_host), _ptr(raw_host),
                                          _ptr(sample_ids_host), _ptr(out_host)))


def aq_wire_copy(h, dst_device, packed_dst, scales_dst, raw_dst, packed_src, scales_src, raw_src):
    return _check(h, lib().aq_wire_copy(h, dst_device, _ptr(packed_dst), _ptr(scales_dst), _ptr(raw_dst),
                                        _ptr(packed_src), _ptr(scales_src), _ptr(raw_src)))


def aq_wire_copy_grad(h, dst_device, packed_dst, scales_dst, packed_src, scales_src, n_elems, bits):
    return _check(h, lib().aq_wire_copy_grad(h, dst_device, _ptr(packed_dst), _ptr(scales_dst), _ptr(packed_src),
                                             _ptr(scales_src), n_elems, bits))


def aq_prefetch(h, sample_ids_host):
    """sample_ids_host: int32 CPU tensor / numpy array of AQ_BATCH ids."""
    return _check(h, lib().aq_prefetch(h, _ptr(sample_ids_host), int(sample_ids_host.numel()
                                       if hasattr(sample_ids_host, "numel") else sample_ids_host.size)))


def aq_export_sample(h, sample_id, m_host):
    """Returns the seen flag; fills m_host (numpy / CPU tensor of seq*hidden 16-bit values)."""
    seen = C.c_uint8(0)
    _check(h, lib().aq_export_sample(h, sample_id, _ptr(m_host), C.addressof(seen)))
    return seen.value


def aq_import_sample(h, sample_id, m_host, seen):
    return _check(h, lib().aq_import_sample(h, sample_id, _ptr(m_host), int(bool(seen))))


# ---- stage operators: buffers are named with their row strides, so a tensor may be a slice whose rows are contiguous.  A small
# call takes a few microseconds on the GPU, so these wrappers do as little as they can: a tensor's element type, place and
# layout are checked (an int address is taken as it is), sizes and alignments by the library.

_stage_types = {}        # handle: element type of its operands; none for one that was not made here, whose operands' types go unchecked
_i32 = _f32 = _i64 = None  # torch.int32, torch.float32, torch.int64 once there is a handle


def _row(x, t):
    """Address of a CUDA tensor of type t whose rows (last dimension) are contiguous, of an int address, or None."""
    if x is None or type(x) is int:
        return x
    if (x.dtype is t or t is None) and x.is_cuda and (x.is_contiguous() or x.stride(-1) == 1 or x.shape[-1] == 1):
        return x.data_ptr()
    _unfit(x, t, "contiguous rows")


def _whole(x, t):
    """Address of a contiguous CUDA tensor of type t, an int address, or None."""
    if x is None or type(x) is int:
        return x
    if (x.dtype is t or t is None) and x.is_cuda and x.is_contiguous():
        return x.data_ptr()
    _unfit(x, t, "contiguous elements")


def _unfit(x, t, layout):
    raise AssertionError(f"needs a CUDA tensor of {t} with {layout}, got {x.dtype} on {x.device} with strides {x.stride()}")


def _stage_type(st, value):
    global _i32, _f32, _i64
    try:
        import torch
    except ImportError:  # then every operand is an address
        return
    _i32, _f32, _i64 = torch.int32, torch.float32, torch.int64
    _stage_types[st] = {AQ_FP16: torch.float16, AQ_BF16: torch.bfloat16, AQ_FP32: torch.float32}[value]


def _stage_error(st, rc):
    raise AqError(rc, aq_stage_last_error(st))


def aq_stage_create():
    st = lib().aq_stage_create()
    if not st:
        raise AqError(aq_stage_last_error_code(None), aq_stage_last_error(None))
    _stage_type(st, AQ_FP16)
    return st


def aq_stage_destroy(st):
    _stage_types.pop(st, None)
    lib().aq_stage_destroy(st)


def aq_stage_configure(st, key, value):
    rc = lib().aq_stage_configure(st, key, value)
    if rc:
        _stage_error(st, rc)
    if key == AQ_DTYPE:
        _stage_type(st, value)
    return rc


def aq_stage_status(st):
    v = C.c_uint32(0)
    rc = lib().aq_stage_status(st, C.byref(v))
    return _stage_error(st, rc) if rc else v.value


def aq_stage_last_error(st):
    return lib().aq_stage_last_error(st).decode()


def aq_stage_last_error_code(st):
    return lib().aq_stage_last_error_code(st)


def aq_token_logprobs(st, logits, rows, vocab, ld, targets, scale, top_k, logprob, entropy, lse, top_ids, top_logprobs):
    rc = (_lib or lib()).aq_token_logprobs(st, _row(logits, _stage_types.get(st)), rows, vocab, ld, _whole(targets, _i32), scale, top_k,
                                           _whole(logprob, _f32), _whole(entropy, _f32), _whole(lse, _f32), _whole(top_ids, _i32),
                                           _whole(top_logprobs, _f32))
    return rc and _stage_error(st, rc)


def aq_token_logprobs_grad(st, logits, rows, vocab, ld, targets, scale, lse, entropy, d_logprob, d_entropy, d_logits, ld_d):
    t = _stage_types.get(st)
    rc = (_lib or lib()).aq_token_logprobs_grad(st, _row(logits, t), rows, vocab, ld, _whole(targets, _i32), scale, _whole(lse, _f32),
                                                _whole(entropy, _f32), _whole(d_logprob, _f32), _whole(d_entropy, _f32), _row(d_logits, t), ld_d)
    return rc and _stage_error(st, rc)


def aq_gated_ffn(st, x, ldx, wg, wu, ldw, rows, hidden, inner, act, h, ldh, g, u, ldgu):
    t = _stage_types.get(st)
    rc = (_lib or lib()).aq_gated_ffn(st, _row(x, t), ldx, _row(wg, t), _row(wu, t), ldw, rows, hidden, inner, act, _row(h, t), ldh,
                                      _row(g, t), _row(u, t), ldgu)
    return rc and _stage_error(st, rc)


def aq_gated_ffn_grad(st, dh, lddh, x, ldx, wg, wu, ldw, g, u, ldgu, rows, hidden, inner, act, dx, lddx, dwg, dwu, lddw):
    t = _stage_types.get(st)
    rc = (_lib or lib()).aq_gated_ffn_grad(st, _row(dh, t), lddh, _row(x, t), ldx, _row(wg, t), _row(wu, t), ldw, _row(g, t), _row(u, t),
                                           ldgu, rows, hidden, inner, act, _row(dx, t), lddx, _row(dwg, t), _row(dwu, t), lddw)
    return rc and _stage_error(st, rc)


def aq_qk_norm_rope(st, shape, rows, q, q_stride, k, k_stride, wq, wk, cos_sin, positions, q_out, q_out_stride, k_out, k_out_stride):
    """shape: a QkShape."""
    t = _stage_types.get(st)
    rc = (_lib or lib()).aq_qk_norm_rope(st, C.addressof(shape), rows, _row(q, t), q_stride, _row(k, t), k_stride, _whole(wq, t),
                                         _whole(wk, t), _whole(cos_sin, _f32), _whole(positions, _i32), _row(q_out, t), q_out_stride,
                                         _row(k_out, t), k_out_stride)
    return rc and _stage_error(st, rc)


def aq_qk_norm_rope_grad(st, shape, rows, dq_out, dq_out_stride, dk_out, dk_out_stride, q, q_stride, k, k_stride, wq, wk, cos_sin,
                         positions, dq, dq_stride, dk, dk_stride, dwq, dwk):
    t = _stage_types.get(st)
    rc = (_lib or lib()).aq_qk_norm_rope_grad(st, C.addressof(shape), rows, _row(dq_out, t), dq_out_stride, _row(dk_out, t), dk_out_stride,
                                              _row(q, t), q_stride, _row(k, t), k_stride, _whole(wq, t), _whole(wk, t),
                                              _whole(cos_sin, _f32), _whole(positions, _i32), _row(dq, t), dq_stride, _row(dk, t),
                                              dk_stride, _whole(dwq, _f32), _whole(dwk, _f32))
    return rc and _stage_error(st, rc)


def aq_layer_norm(st, x, ldx, residual, ldr, w, b, eps, rows, hidden, sum, lds, y, ldy, mean, rstd):
    t = _stage_types.get(st)
    rc = (_lib or lib()).aq_layer_norm(st, _row(x, t), ldx, _row(residual, t), ldr, _whole(w, t), _whole(b, t), eps, rows, hidden,
                                       _row(sum, t), lds, _row(y, t), ldy, _whole(mean, _f32), _whole(rstd, _f32))
    return rc and _stage_error(st, rc)


def aq_layer_norm_grad(st, dy, lddy, dsum, ldds, s, lds, w, mean, rstd, rows, hidden, dx, lddx, dw, db):
    t = _stage_types.get(st)
    rc = (_lib or lib()).aq_layer_norm_grad(st, _row(dy, t), lddy, _row(dsum, t), ldds, _row(s, t), lds, _whole(w, t), _whole(mean, _f32),
                                            _whole(rstd, _f32), rows, hidden, _row(dx, t), lddx, _whole(dw, _f32), _whole(db, _f32))
    return rc and _stage_error(st, rc)


def aq_adam_table(st, grads, params=None, masters=None, m=None, v=None, m_scale=None, v_scale=None, weight_decay=0.0):
    """Array of AdamTensor for aq_adamw, or for aq_grad_norm where nothing but the gradients is given.

    Every argument is a list with one contiguous CUDA tensor (or None, for a tensor without that part; every one has a
    gradient) for each of the tensors; weight_decay is a number for all of them or a list.  Moments in 8 bits are torch.float8_e4m3fn (m) and torch.float8_e5m2 (v) or
    their bytes as torch.uint8, with m_scale and v_scale.  The array holds addresses: it can be kept for as long as the
    tensors keep their places, and does not keep them alive.  Lay it out anew where gradients are allocated in every step.
    aq_adamw refuses it with a handle of another element type.
    """
    import torch
    t, n = _stage_types.get(st), len(grads)
    narrow = m_scale is not None
    kinds = {"m": (torch.float8_e4m3fn, torch.uint8) if narrow else (torch.float32,), "v": (torch.float8_e5m2, torch.uint8) if narrow else (torch.float32,),
             "param": (t,), "grad": (t, torch.float32), "master": (torch.float32,), "m_scale": (torch.float32,), "v_scale": (torch.float32,)}
    codes = {torch.float16: AQ_FP16, torch.bfloat16: AQ_BF16, torch.float32: AQ_FP32}
    columns = {"grad": grads, "param": params, "master": masters, "m": m, "v": v, "m_scale": m_scale, "v_scale": v_scale}
    decay = [weight_decay] * n if isinstance(weight_decay, (int, float)) else weight_decay
    assert len(decay) == n and all(c is None or len(c) == n for c in columns.values()), "lists of different lengths"
    table = (AdamTensor * n)()
    table.element_type = t                              # the parameters'; nothing in the structure tells it
    written = []
    for i, row in enumerate(table):
        assert grads[i] is not None, f"tensor {i} has no gradient: one that is left out of a step is left out of its table"
        row.numel, row.weight_decay, row.grad_dtype = grads[i].numel(), decay[i], codes[grads[i].dtype]
        for name, column in columns.items():
            x = None if column is None else column[i]
            if x is None:
                continue
            assert t is None or x.dtype in kinds[name], f"{name} of tensor {i} is {x.dtype}"
            size = -(-row.numel // 256) if name.endswith("scale") else row.numel
            assert x.numel() == size, f"{name} of tensor {i} has {x.numel()} elements, not {size}"
            setattr(row, name, _whole(x, x.dtype))
            if name != "grad" and size:
                written.append((x.data_ptr(), x.data_ptr() + x.numel() * x.element_size()))
        assert not narrow or not (row.m or row.v) or (row.m_scale and row.v_scale), f"tensor {i} has 8-bit moments without m_scale or v_scale"
    written.sort()
    assert all(a[1] <= b[0] for a, b in zip(written, written[1:])), "two tensors overlap: one that layers share is listed once"
    return table


def _table(tensors, n):
    """An array of at least n AdamTensor, or an int address."""
    if type(tensors) is not int and tensors is not None:
        assert n <= len(tensors) and tensors._type_ is AdamTensor, "needs an array of AdamTensor with n of them"
    return tensors


def aq_grad_norm(st, tensors, n, inv_scale, max_norm, norm, factor, step):
    """tensors: an array of AdamTensor, or its address."""
    rc = (_lib or lib()).aq_grad_norm(st, _table(tensors, n), n, inv_scale, max_norm, _whole(norm, _f32), _whole(factor, _f32), _whole(step, _i64))
    return rc and _stage_error(st, rc)


def aq_adamw(st, config, tensors, n, factor, d_lr, d_step):
    """config: an AdamwConfig; tensors: an array of AdamTensor, or its address."""
    t, laid_out = _stage_types.get(st), getattr(tensors, "element_type", None)
    if laid_out is not t and laid_out is not None and t is not None:
        raise AqError(AQ_EINVAL, f"aq_adamw: the table was laid out for parameters of {laid_out}, the handle's type is {t}")
    rc = (_lib or lib()).aq_adamw(st, C.addressof(config), _table(tensors, n), n, _whole(factor, _f32), _whole(d_lr, _f32), _whole(d_step, _i64))
    return rc and _stage_error(st, rc)
