"""ctypes binding with the same names as the C ABI in include/vc_attn.h.

Argument marshalling only: tensors become raw device (or host) pointers, the current
PyTorch CUDA stream becomes the `stream` argument, status codes other than VC_OK raise
VcError.  Buffers are allocated by the caller (helpers below size them).
"""
import ctypes
import os

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_HERE, "libvc.so")

VC_P_DEFAULT, VC_P_EXPCAST_E4M3, VC_P_EXP_E4M3, VC_P_NVFP4 = 0, 1, 2, 3
VC_P_EXP_POLY_E4M3, VC_P_EXP_MIX_E4M3 = 4, 5
VC_FLAG_ROPE, VC_FLAG_HADAMARD, VC_FLAG_K_SMOOTH, VC_FLAG_V_SMOOTH, VC_FLAG_ALL = 1, 2, 4, 8, 15
VC_FLAG_INT8_QK = 16
VC_FLAG_CHECK_PERM = 32
VC_GROUP_LABELS_OFFSET = 1024
VC_OK, VC_ERR_INVALID_ARG, VC_ERR_UNSUPPORTED, VC_ERR_WORKSPACE, VC_ERR_CUDA, VC_ERR_TIMEOUT, VC_ERR_SCRATCH_LIMIT = range(7)


class VcError(RuntimeError):
    def __init__(self, code, where):
        self.code = code
        super().__init__(f"{where}: {vc_status_string(code)} (status {code})")


class Params(ctypes.Structure):
    """Mirror of vc_params."""
    _fields_ = [("B", ctypes.c_int32), ("H", ctypes.c_int32), ("N", ctypes.c_int32), ("d", ctypes.c_int32),
                ("grid_t", ctypes.c_int32), ("grid_h", ctypes.c_int32), ("grid_w", ctypes.c_int32),
                ("bits", ctypes.c_int32), ("p_format", ctypes.c_int32), ("flags", ctypes.c_int32),
                ("softmax_scale", ctypes.c_float), ("beta", ctypes.c_float),
                ("rope_dim_t", ctypes.c_int32), ("rope_dim_h", ctypes.c_int32), ("rope_dim_w", ctypes.c_int32),
                ("rope_theta", ctypes.c_float),
                ("stride_b", ctypes.c_int64), ("stride_h", ctypes.c_int64), ("stride_n", ctypes.c_int64),
                ("heads_per_pass", ctypes.c_int32), ("kernel_variant", ctypes.c_int32),
                ("block_q", ctypes.c_int32), ("block_k", ctypes.c_int32), ("block_v", ctypes.c_int32)]

    @classmethod
    def make(cls, B, H, N, d, grid, bits=8, p_format=VC_P_DEFAULT, flags=VC_FLAG_ALL, **kw):
        p = cls(B=B, H=H, N=N, d=d, grid_t=grid[0], grid_h=grid[1], grid_w=grid[2], bits=bits,
                p_format=p_format, flags=flags)
        for k, v in kw.items():
            setattr(p, k, v)
        return p


class QuantView(ctypes.Structure):
    """Mirror of vc_quant_ptrs."""
    _fields_ = ([(n, ctypes.c_void_p) for n in ("q_codes", "k_codes", "v_codes", "q_scale", "k_scale", "v_scale",
                                                "v_means", "k_mean", "q_micro", "k_micro", "v_micro")] +
                [(n + "_bytes", ctypes.c_size_t) for n in ("q_codes", "k_codes", "v_codes", "q_scale", "k_scale",
                                                           "v_scale", "v_means", "k_mean", "q_micro", "k_micro",
                                                           "v_micro")])


class PrepStats(ctypes.Structure):
    """Mirror of vc_prep_stats (device pointers)."""
    _fields_ = [("k_mean", ctypes.c_void_p), ("v_block_mean", ctypes.c_void_p), ("v_amax", ctypes.c_void_p)]


VC_DTYPE_BF16, VC_DTYPE_FP16, VC_DTYPE_FP32 = 0, 1, 2
VC_NORM_NONE, VC_NORM_HEAD, VC_NORM_TOKEN = 0, 1, 2
VC_ROTARY_NONE, VC_ROTARY_INTERLEAVED, VC_ROTARY_HALF = 0, 1, 2
VC_ROPE_SCALING_NONE, VC_ROPE_SCALING_LINEAR, VC_ROPE_SCALING_NTK, VC_ROPE_SCALING_YARN = 0, 1, 2, 3
_DTYPES = {torch.bfloat16: VC_DTYPE_BF16, torch.float16: VC_DTYPE_FP16, torch.float32: VC_DTYPE_FP32}


def _dtype(t):
    if t.dtype not in _DTYPES:
        raise ValueError(f"element type {t.dtype}: bfloat16, float16 or float32 is wanted")
    return _DTYPES[t.dtype]


class Strides(ctypes.Structure):
    """Mirror of vc_strides."""
    _fields_ = [("b", ctypes.c_int64), ("h", ctypes.c_int64), ("n", ctypes.c_int64)]

    @classmethod
    def of(cls, t):
        """Of a [B, H, N, d] tensor in elements; its channels have to lie side by side."""
        if t.dim() != 4 or (t.stride(3) != 1 and t.shape[3] != 1):
            raise ValueError("a [B, H, N, d] tensor with d contiguous is wanted")
        if t.shape[2] > 1 and t.stride(2) == 0:
            raise ValueError("rows that share one address: a [B, H, N, d] tensor with tokens apart is wanted")
        return cls(t.stride(0), t.stride(1), t.stride(2) or t.shape[3])         # (all zero would mean packed)


class RopeValues(ctypes.Structure):
    """Mirror of vc_rope_values."""
    _fields_ = [(n, ctypes.c_double) for n in ("theta", "factor_t", "factor_h", "factor_w")]


class QkParams(ctypes.Structure):
    """Mirror of vc_qk_params.  `rope` is None, or a RopeValues to go with the block: `of` makes one where theta or a factor is no FP32 number."""
    rope = None
    _fields_ = ([(n, ctypes.c_int32) for n in ("B", "N", "d", "H_q", "H_k", "dtype", "weight_dtype", "norm", "rotary",
                                               "rope_dim_t", "rope_dim_h", "rope_dim_w", "grid_t", "grid_h", "grid_w",
                                               "start_t", "start_h", "start_w", "rope_scaling",
                                               "rope_original_t", "rope_original_h", "rope_original_w")] +
                [(n, ctypes.c_float) for n in ("eps", "rope_theta", "rope_factor_t", "rope_factor_h", "rope_factor_w",
                                               "yarn_beta_fast", "yarn_beta_slow", "rope_attention_factor")] +
                [(n, Strides) for n in ("q", "k", "q_out", "k_out")])

    @classmethod
    def of(cls, q, k, q_out, k_out, grid=(0, 0, 0), weight=None, rope_dims=(0, 0, 0), start=(0, 0, 0), rope_factor=(0.0, 0.0, 0.0),
           rope_original=(0, 0, 0), **kw):
        """For [B, H, N, d] tensors, either of q and k (with its output) None; the triples run over (t, h, w)."""
        x = q if q is not None else k
        B, _, N, d = x.shape
        p = cls(B=B, N=N, d=d, dtype=_dtype(x), weight_dtype=_dtype(x if weight is None else weight))
        for name, t, out in (("q", q, q_out), ("k", k, k_out)):
            if t is None:
                continue
            if t.shape != out.shape or t.shape[0] != B or t.shape[2:] != x.shape[2:] or t.dtype != x.dtype or out.dtype != x.dtype:
                raise ValueError("q, k and their outputs differ in batches, tokens, head dimension or type")
            setattr(p, "H_" + name, t.shape[1])
            setattr(p, name, Strides.of(t))
            setattr(p, name + "_out", Strides.of(out))
        for field, values in (("grid", grid), ("rope_dim", rope_dims), ("start", start), ("rope_factor", rope_factor), ("rope_original", rope_original)):
            for axis, v in zip("thw", values):
                setattr(p, f"{field}_{axis}", v)
        for name, v in kw.items():
            setattr(p, name, v)
        exact = (float(kw.get("rope_theta", 0.0)), *map(float, rope_factor[:3]))
        if exact != p.rope_fields():
            p.rope = RopeValues(*exact)
            p.rope_rounded = p.rope_fields()
        return p

    def rope_fields(self):
        return self.rope_theta, self.rope_factor_t, self.rope_factor_h, self.rope_factor_w

    def rope_values(self):
        """The address of what goes with the block, or None; a field changed since `of` stands."""
        if self.rope is None:
            return None
        fields, rounded = self.rope_fields(), getattr(self, "rope_rounded", None)
        if rounded is not None and fields != rounded:
            for (name, _), field, was in zip(RopeValues._fields_, fields, rounded):
                if field != was:
                    setattr(self.rope, name, 0.0)
            self.rope_rounded = fields
        return ctypes.addressof(self.rope)


class CrossParams(ctypes.Structure):
    """Mirror of vc_cross_params."""
    _fields_ = ([(n, ctypes.c_int32) for n in ("B", "H", "H_kv", "N_q", "N_kv", "d", "dtype", "key_splits")] +
                [("softmax_scale", ctypes.c_float)] + [(n, Strides) for n in ("q", "k", "v", "o")])

    @classmethod
    def of(cls, q, k, v, o, **kw):
        """For q, o [B, H, N_q, d] and k, v [B, H_kv, N_kv, d]."""
        B, H, Nq, d = q.shape
        if k.shape != v.shape or o.shape != q.shape or k.shape[0] != B or k.shape[3] != d or not q.dtype == k.dtype == v.dtype == o.dtype:
            raise ValueError("q, k, v and o differ in batches, head dimension or type")
        p = cls(B=B, H=H, H_kv=k.shape[1], N_q=Nq, N_kv=k.shape[2], d=d, dtype=_dtype(q), q=Strides.of(q), k=Strides.of(k), v=Strides.of(v), o=Strides.of(o))
        for name, val in kw.items():
            setattr(p, name, val)
        return p


class QuantParams(ctypes.Structure):
    """Mirror of vc_quant_params."""
    _fields_ = [(n, ctypes.c_int32) for n in ("B", "H", "N", "d", "dtype", "block_rows")] + [("x", Strides)]

    @classmethod
    def of(cls, x, block_rows=1):
        """For a [B, H, N, d] tensor (rows b N + n, columns h d + channel) or a matrix [rows, columns]."""
        x = x if x.dim() == 4 else x[None, None]
        B, H, N, d = x.shape
        return cls(B=B, H=H, N=N, d=d, dtype=_dtype(x), block_rows=block_rows, x=Strides.of(x))


class LinearParams(ctypes.Structure):
    """Mirror of vc_linear_params."""
    _fields_ = ([(n, ctypes.c_int32) for n in ("M", "N", "K", "out_dtype", "bias_dtype", "k_splits")] +
                [(n, ctypes.c_int64) for n in ("ldx", "ldw", "ldo")])

    @classmethod
    def of(cls, x_codes, w_codes, out, bias=None, **kw):
        """For x_codes [M, K], w_codes [N, K], out [M, N], rows contiguous."""
        (M, K), (N, K_w) = x_codes.shape, w_codes.shape
        if K != K_w or out.shape != (M, N) or any(t.stride(1) != 1 and t.shape[1] > 1 for t in (x_codes, w_codes, out)):
            raise ValueError("x [M, K], w [N, K] and out [M, N] with contiguous rows are wanted")
        ld = [t.stride(0) if t.shape[0] > 1 else 0 for t in (x_codes, w_codes, out)]
        p = cls(M=M, N=N, K=K, out_dtype=_dtype(out), bias_dtype=_dtype(out if bias is None else bias), ldx=ld[0], ldw=ld[1], ldo=ld[2])
        for name, val in kw.items():
            setattr(p, name, val)
        return p


_lib = None


def load_library():
    """Loads libvc.so (built in-tree); raises if it is missing -- there is no fallback."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(_LIB_PATH):
        raise ImportError(f"{_LIB_PATH} not found: build it with `python -m paper_2609_15810_b200.build`")
    lib = ctypes.CDLL(_LIB_PATH)
    P, vp, i32p = ctypes.POINTER(Params), ctypes.c_void_p, ctypes.c_void_p
    lib.vc_quant_bytes.restype = ctypes.c_size_t
    lib.vc_quant_bytes.argtypes = [P]
    lib.vc_workspace_bytes.restype = ctypes.c_size_t
    lib.vc_workspace_bytes.argtypes = [P]
    lib.vc_prep.restype = ctypes.c_int
    lib.vc_prep.argtypes = [P, vp, vp, vp, i32p, vp, vp, vp]
    lib.vc_prep_with_stats.restype = ctypes.c_int
    lib.vc_prep_with_stats.argtypes = [P, vp, vp, vp, i32p, ctypes.POINTER(PrepStats), vp, vp, vp]
    lib.vc_prep_stats_view.restype = ctypes.c_int
    lib.vc_prep_stats_view.argtypes = [P, vp, vp, ctypes.POINTER(PrepStats)]
    lib.vc_prep_noalloc.restype = ctypes.c_int
    lib.vc_prep_noalloc.argtypes = [P, vp, vp, vp, i32p, vp, vp]
    lib.vc_attn_fwd.restype = ctypes.c_int
    lib.vc_attn_fwd.argtypes = [P, vp, vp, vp, vp]
    lib.vc_attn.restype = ctypes.c_int
    lib.vc_attn.argtypes = [P, vp, vp, vp, i32p, vp, vp, vp, vp]
    lib.vc_attn_host.restype = ctypes.c_int
    lib.vc_attn_host.argtypes = [P] + [vp] * 13
    lib.vc_group_workspace_bytes.restype = ctypes.c_size_t
    lib.vc_group_workspace_bytes.argtypes = [P]
    lib.vc_group.restype = ctypes.c_int
    lib.vc_group.argtypes = [P, vp, ctypes.c_int32, ctypes.c_int32, ctypes.c_int32, vp, i32p, vp, vp]
    lib.vc_group_schedule.restype = ctypes.c_int32
    lib.vc_group_schedule.argtypes = [ctypes.c_int32, ctypes.c_int32, ctypes.c_int32]
    lib.vc_quant_view.restype = ctypes.c_int
    lib.vc_quant_view.argtypes = [P, vp, ctypes.POINTER(QuantView)]
    lib.vc_poll_status.restype = ctypes.c_int
    lib.vc_poll_status.argtypes = [vp, vp]
    lib.vc_test_set_wait_limit.restype = None
    lib.vc_test_set_wait_limit.argtypes = [ctypes.c_uint32]
    lib.vc_test_expcast_codes.restype = ctypes.c_int
    lib.vc_test_expcast_codes.argtypes = [vp, ctypes.c_int64, ctypes.c_float, ctypes.c_float, ctypes.c_float, vp, vp]
    lib.vc_test_nvfp4_codes.restype = ctypes.c_int
    lib.vc_test_nvfp4_codes.argtypes = [vp, vp, ctypes.c_int64, ctypes.c_int32, ctypes.c_int32, ctypes.c_float, vp, vp, vp]
    lib.vc_mma_peak.restype = ctypes.c_int
    lib.vc_mma_peak.argtypes = [ctypes.c_int32, ctypes.c_int32, vp, ctypes.POINTER(ctypes.c_double),
                                ctypes.POINTER(ctypes.c_double), vp]
    lib.vc_qk_norm_rope.restype = ctypes.c_int
    lib.vc_qk_norm_rope.argtypes = [ctypes.POINTER(QkParams)] + [vp] * 8
    lib.vc_qk_norm_rope_with_values.restype = ctypes.c_int
    lib.vc_qk_norm_rope_with_values.argtypes = [ctypes.POINTER(QkParams)] + [vp] * 9
    lib.vc_cross_workspace_bytes.restype = ctypes.c_size_t
    lib.vc_cross_workspace_bytes.argtypes = [ctypes.POINTER(CrossParams)]
    lib.vc_cross_attn.restype = ctypes.c_int
    lib.vc_cross_attn.argtypes = [ctypes.POINTER(CrossParams)] + [vp] * 9
    lib.vc_quant_fp8.restype = ctypes.c_int
    lib.vc_quant_fp8.argtypes = [ctypes.POINTER(QuantParams)] + [vp] * 4
    lib.vc_linear_workspace_bytes.restype = ctypes.c_size_t
    lib.vc_linear_workspace_bytes.argtypes = [ctypes.POINTER(LinearParams)]
    lib.vc_linear_fp8.restype = ctypes.c_int
    lib.vc_linear_fp8.argtypes = [ctypes.POINTER(LinearParams)] + [vp] * 8
    lib.vc_launch_count.restype = ctypes.c_uint64
    lib.vc_launch_count.argtypes = []
    lib.vc_status_string.restype = ctypes.c_char_p
    lib.vc_status_string.argtypes = [ctypes.c_int]
    _lib = lib
    return lib


def _ptr(t):
    if t is None:
        return None
    if isinstance(t, int):
        return t
    assert t.is_contiguous() or t.dim() == 4, "pass strides through Params for non-packed inputs"
    return t.data_ptr()


# The current stream's handle.  torch.cuda.current_stream() builds an object around it, 3 us of a small call's 10; PyTorch's own
# generated code asks for the number alone.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream():
    return _raw_stream(torch.cuda.current_device()) if _raw_stream is not None else torch.cuda.current_stream().cuda_stream


def _check(code, where):
    if code != 0:
        raise VcError(code, where)


def vc_status_string(code):
    return load_library().vc_status_string(int(code)).decode()


def vc_quant_bytes(p):
    return int(load_library().vc_quant_bytes(ctypes.byref(p)))


def vc_workspace_bytes(p):
    return int(load_library().vc_workspace_bytes(ctypes.byref(p)))


def vc_prep(p, q, k, v, perm, quant, workspace):
    _check(load_library().vc_prep(ctypes.byref(p), _ptr(q), _ptr(k), _ptr(v), _ptr(perm), _ptr(quant),
                                  _ptr(workspace), _stream()), "vc_prep")


def vc_prep_with_stats(p, q, k, v, perm, k_mean, v_block_mean, v_amax, quant, workspace):
    """vc_prep with the statistics supplied by the caller (fp32 device tensors): no statistics launches."""
    st = PrepStats(_ptr(k_mean), _ptr(v_block_mean), _ptr(v_amax))
    _check(load_library().vc_prep_with_stats(ctypes.byref(p), _ptr(q), _ptr(k), _ptr(v), _ptr(perm), ctypes.byref(st),
                                             _ptr(quant), _ptr(workspace), _stream()), "vc_prep_with_stats")


def vc_prep_stats_view(p, quant, workspace):
    """(k_mean [BH, d], v_block_mean [BH, nb, d], v_amax [BH, d]) fp32 tensors aliasing where vc_prep left them."""
    st = PrepStats()
    _check(load_library().vc_prep_stats_view(ctypes.byref(p), _ptr(quant), _ptr(workspace), ctypes.byref(st)), "vc_prep_stats_view")
    BH, d, nb = p.B * p.H, p.d, (p.N + 127) // 128
    def alias(ptr, base, n):
        off = ptr - base.data_ptr()
        return base[off:off + 4 * n].view(torch.float32)
    return (alias(st.k_mean, quant, BH * d).view(BH, d), alias(st.v_block_mean, workspace, BH * nb * d).view(BH, nb, d),
            alias(st.v_amax, workspace, BH * d).view(BH, d))


def vc_prep_noalloc(p, q, k, v, perm, quant):
    """vc_prep on the library's built-in scratch array: no workspace, no allocation (size-limited)."""
    _check(load_library().vc_prep_noalloc(ctypes.byref(p), _ptr(q), _ptr(k), _ptr(v), _ptr(perm), _ptr(quant),
                                          _stream()), "vc_prep_noalloc")


def vc_attn_fwd(p, quant, o, workspace):
    _check(load_library().vc_attn_fwd(ctypes.byref(p), _ptr(quant), _ptr(o), _ptr(workspace), _stream()),
           "vc_attn_fwd")


def vc_attn(p, q, k, v, perm, o, quant, workspace):
    _check(load_library().vc_attn(ctypes.byref(p), _ptr(q), _ptr(k), _ptr(v), _ptr(perm), _ptr(o), _ptr(quant),
                                  _ptr(workspace), _stream()), "vc_attn")


def vc_attn_host(p, q_host, k_host, v_host, perm_host, o_host, q_dev, k_dev, v_dev, perm_dev, o_dev, quant,
                 workspace):
    _check(load_library().vc_attn_host(ctypes.byref(p), _ptr(q_host), _ptr(k_host), _ptr(v_host), _ptr(perm_host),
                                       _ptr(o_host), _ptr(q_dev), _ptr(k_dev), _ptr(v_dev), _ptr(perm_dev),
                                       _ptr(o_dev), _ptr(quant), _ptr(workspace), _stream()), "vc_attn_host")


def vc_group_workspace_bytes(p):
    return int(load_library().vc_group_workspace_bytes(ctypes.byref(p)))


def vc_group(p, v, k, iters, warm_start, centroids, perm, workspace):
    """k-means on the value tokens -> perm = stable argsort of the labels (centroids in/out)."""
    _check(load_library().vc_group(ctypes.byref(p), _ptr(v), int(k), int(iters), int(bool(warm_start)), _ptr(centroids),
                                   _ptr(perm), _ptr(workspace), _stream()), "vc_group")


VC_GROUP_RECOMPUTE, VC_GROUP_REUSE, VC_GROUP_FROZEN = 0, 1, 2


def vc_group_schedule(step, n_steps, reuse=4):
    """What the step-indexed grouping schedule asks for at denoising step `step` of `n_steps`."""
    return int(load_library().vc_group_schedule(int(step), int(n_steps), int(reuse)))


def vc_quant_view(p, quant):
    out = QuantView()
    _check(load_library().vc_quant_view(ctypes.byref(p), _ptr(quant), ctypes.byref(out)), "vc_quant_view")
    return out


def vc_poll_status(workspace):
    _check(load_library().vc_poll_status(_ptr(workspace), _stream()), "vc_poll_status")


def vc_test_set_wait_limit(polls):
    """Test hook: polls after which a device-side wait gives up (0 = the default)."""
    load_library().vc_test_set_wait_limit(int(polls))


def vc_test_expcast_codes(s, cs, m, beta=0.0):
    """Test hook: the ExpCast-FP8 codes of the fp32 scores `s` (CUDA tensor, numel a multiple of 4)
    under the factor cs and the running maximum m, as the attention kernels form them (uint8 tensor)."""
    assert s.dtype == torch.float32 and s.is_cuda and s.is_contiguous()
    out = torch.empty(s.numel(), dtype=torch.uint8, device=s.device)
    _check(load_library().vc_test_expcast_codes(_ptr(s), s.numel(), float(cs), float(m), float(beta), _ptr(out), _stream()),
           "vc_test_expcast_codes")
    return out.view(s.shape)


def vc_test_nvfp4_codes(s, m, d, cs, polynomial=True):
    """Test hook: (E2M1 codes [rows, 64], two a byte, E4M3 factors [rows, 8]) of the fp32 scores `s` [rows, 128] under the
    factor cs and the running maxima `m` [rows], as the 4-bit attention kernel for head dimension d forms them, with some groups'
    codes by polynomial or with none."""
    assert s.dtype == m.dtype == torch.float32 and s.is_cuda and s.is_contiguous() and m.is_contiguous() and s.shape == (m.numel(), 128)
    codes = torch.empty(m.numel(), 64, dtype=torch.uint8, device=s.device)
    factors = torch.empty(m.numel(), 8, dtype=torch.uint8, device=s.device)
    _check(load_library().vc_test_nvfp4_codes(_ptr(s), _ptr(m), m.numel(), int(d), int(polynomial), float(cs), _ptr(codes), _ptr(factors), _stream()),
           "vc_test_nvfp4_codes")
    return codes, factors


def vc_mma_peak(kind, groups=4096):
    """(TFLOP/s over the whole GPU, MAC per clock per SM) of back-to-back MMAs of one kind (8 or 4)."""
    scratch = torch.zeros(1, dtype=torch.int64, device="cuda")
    tf, mac = ctypes.c_double(0.0), ctypes.c_double(0.0)
    _check(load_library().vc_mma_peak(int(kind), int(groups), _ptr(scratch), ctypes.byref(tf), ctypes.byref(mac), _stream()),
           "vc_mma_peak")
    return tf.value, mac.value


_TORCH = (torch.bfloat16, torch.float16, torch.float32)
_FP32, _INT32, _BYTES, _MASK, _CODES = (torch.float32,), (torch.int32,), (torch.uint8,), (torch.bool, torch.uint8), (torch.float8_e4m3fn, torch.uint8)


def _types(code):
    if not 0 <= code < len(_TORCH):
        raise ValueError(f"element type {code}: VC_DTYPE_BF16, VC_DTYPE_FP16 or VC_DTYPE_FP32 is wanted")
    return (_TORCH[code],)


# The operators around the attention take tensors of several types and layouts, and the C entry sees addresses alone, so the binding
# compares the tensors with what the parameter block says.  What a block asks of each argument, (name, types, shape, strides), is
# derived from its bytes once: reading it from the structure field by field cost 7 of a call's 20 us of host time.
_wants = {}


def _wanted(p, derive):
    key = (derive, bytes(p))
    got = _wants.get(key)
    if got is None:
        if len(_wants) >= 4096:
            _wants.clear()
        got = _wants[key] = derive(p)
    return got


def _packed(shape):
    out, n = [], 1
    for s in reversed(shape):
        out.append(n)
        n *= s
    return tuple(reversed(out))


def _head_want(name, code, shape, s):
    """A [B, H, N, d] tensor under the vc_strides of the parameter block."""
    return (name, _types(code), shape, (s.b, s.h, s.n, 1) if s.b or s.h or s.n else _packed(shape))


def _want(name, types, shape):
    return (name, types, shape, _packed(shape))


def _address(t, device, want):
    if t is None:
        return None
    name, types, shape, strides = want
    if t.get_device() != device:
        raise ValueError(f"{name}: on {t.device}, and the current device is cuda:{device}")
    if t.dtype not in types:
        raise ValueError(f"{name}: {t.dtype}, not {' or '.join(str(d) for d in types)}")
    if t.shape != shape:
        raise ValueError(f"{name}: shape {tuple(t.shape)}, not {shape}")
    if t.stride() != strides and 0 not in shape:          # (a dimension of one entry may have any, a tensor without entries too)
        for n, got, wanted in zip(shape, t.stride(), strides):
            if n > 1 and got != wanted:
                raise ValueError(f"{name}: strides {t.stride()}, not {strides}")
    return t.data_ptr()


def _workspace(t, device, need, where):
    if need == 0:
        raise VcError(VC_ERR_INVALID_ARG, where)
    if t is None:
        return None
    if t.get_device() != device or t.dtype != torch.uint8 or not t.is_contiguous():
        raise ValueError(f"workspace: contiguous uint8 on cuda:{device} is wanted")
    if t.numel() < need:
        raise ValueError(f"workspace: {t.numel()} bytes, not {need}")
    return t.data_ptr()


def _qk_wants(p):
    qs, ks = (p.B, p.H_q, p.N, p.d), (p.B, p.H_k, p.N, p.d)
    wt, heads = _types(p.weight_dtype), p.norm == VC_NORM_TOKEN
    return (_head_want("q", p.dtype, qs, p.q), _head_want("k", p.dtype, ks, p.k), _want("q_weight", wt, (p.d * (p.H_q if heads else 1),)),
            _want("k_weight", wt, (p.d * (p.H_k if heads else 1),)), _want("positions", _INT32, (p.B, p.N, 3)),
            _head_want("q_out", p.dtype, qs, p.q_out), _head_want("k_out", p.dtype, ks, p.k_out))


def vc_qk_norm_rope(p, q, k, q_weight, k_weight, positions, q_out, k_out):
    """RMS norm (p.norm) and rotation (p.rotary) of q and k into q_out and k_out; q, k, a weight [d] or [H d], or positions may be None."""
    dev, w = torch.cuda.current_device(), _wanted(p, _qk_wants)
    _check(load_library().vc_qk_norm_rope_with_values(ctypes.byref(p), p.rope_values(), _address(q, dev, w[0]), _address(k, dev, w[1]),
                                                      _address(q_weight, dev, w[2]), _address(k_weight, dev, w[3]), _address(positions, dev, w[4]),
                                                      _address(q_out, dev, w[5]), _address(k_out, dev, w[6]), _stream()), "vc_qk_norm_rope")


def vc_cross_workspace_bytes(p):
    return int(load_library().vc_cross_workspace_bytes(ctypes.byref(p)))


def _cross_wants(p):
    qs, ks = (p.B, p.H, p.N_q, p.d), (p.B, p.H_kv, p.N_kv, p.d)
    return (_head_want("q", p.dtype, qs, p.q), _head_want("k", p.dtype, ks, p.k), _head_want("v", p.dtype, ks, p.v), _want("kv_len", _INT32, (p.B,)),
            _want("key_mask", _MASK, (p.B, p.N_kv)), _head_want("o", p.dtype, qs, p.o), _want("lse", _FP32, (p.B, p.H, p.N_q)), vc_cross_workspace_bytes(p))


def vc_cross_attn(p, q, k, v, kv_len, key_mask, o, lse, workspace):
    """o = softmax(scale q k^T over the kept keys) v; kv_len int32 [B], key_mask bool or uint8 [B, N_kv] and lse fp32 [B, H, N_q] may be None."""
    dev, w = torch.cuda.current_device(), _wanted(p, _cross_wants)
    _check(load_library().vc_cross_attn(ctypes.byref(p), _address(q, dev, w[0]), _address(k, dev, w[1]), _address(v, dev, w[2]),
                                        _address(kv_len, dev, w[3]), _address(key_mask, dev, w[4]), _address(o, dev, w[5]), _address(lse, dev, w[6]),
                                        _workspace(workspace, dev, w[7], "vc_cross_attn"), _stream()), "vc_cross_attn")


def _quant_wants(p):
    rows, cols = p.B * p.N, p.H * p.d
    nb = (cols + 127) // 128
    x = _head_want("x", p.dtype, (p.B, p.H, p.N, p.d), p.x)
    return (x, (x[0], x[1], x[2][2:], x[3][2:]) if p.B == p.H == 1 else x, _want("codes", _CODES, (rows, cols)),
            _want("scale", _FP32, (nb, rows) if p.block_rows == 1 else ((rows + 127) // 128, nb)))


def vc_quant_fp8(p, x, codes, scale):
    """E4M3 codes [B N, H d] (float8_e4m3fn or uint8) and FP32 scales of x, [B, H, N, d] or a matrix [rows, columns]."""
    dev, w = torch.cuda.current_device(), _wanted(p, _quant_wants)
    _check(load_library().vc_quant_fp8(ctypes.byref(p), _address(x, dev, w[0] if x.dim() == 4 else w[1]), _address(codes, dev, w[2]),
                                       _address(scale, dev, w[3]), _stream()), "vc_quant_fp8")


def vc_linear_workspace_bytes(p):
    return int(load_library().vc_linear_workspace_bytes(ctypes.byref(p)))


def _linear_wants(p):
    nb = (p.K + 127) // 128
    return (("x_codes", _CODES, (p.M, p.K), (p.ldx or p.K, 1)), _want("x_scale", _FP32, (nb, p.M)), ("w_codes", _CODES, (p.N, p.K), (p.ldw or p.K, 1)),
            _want("w_scale", _FP32, ((p.N + 127) // 128, nb)), _want("bias", _types(p.bias_dtype), (p.N,)),
            ("out", _types(p.out_dtype), (p.M, p.N), (p.ldo or p.N, 1)), vc_linear_workspace_bytes(p))


def vc_linear_fp8(p, x_codes, x_scale, w_codes, w_scale, bias, out, workspace):
    """out = x w^T + bias from codes and scales as vc_quant_fp8 writes them (x with block_rows 1, w with 128); bias [N] or None."""
    dev, w = torch.cuda.current_device(), _wanted(p, _linear_wants)
    _check(load_library().vc_linear_fp8(ctypes.byref(p), _address(x_codes, dev, w[0]), _address(x_scale, dev, w[1]), _address(w_codes, dev, w[2]),
                                        _address(w_scale, dev, w[3]), _address(bias, dev, w[4]), _address(out, dev, w[5]),
                                        _workspace(workspace, dev, w[6], "vc_linear_fp8"), _stream()), "vc_linear_fp8")


def vc_launch_count():
    return int(load_library().vc_launch_count())


# ----------------------------------------------------------------------------- conveniences
def alloc_buffers(p, device="cuda"):
    """(quant, workspace) uint8 tensors of the sizes the library asks for."""
    qb, wb = vc_quant_bytes(p), vc_workspace_bytes(p)
    if qb == 0 or wb == 0:
        raise VcError(1, "alloc_buffers")
    return (torch.empty(qb, dtype=torch.uint8, device=device), torch.empty(wb, dtype=torch.uint8, device=device))


def section(view, name, quant, dtype=torch.uint8):
    """A tensor aliasing one section of the bundle (for tests)."""
    off = getattr(view, name) - quant.data_ptr()
    nbytes = getattr(view, name + "_bytes")
    return quant[off:off + nbytes].view(dtype)
