"""What the operators around the quantized attention refuse, on the host and before any launch (no GPU)."""
import ctypes

import pytest
import torch

import paper_2609_15810_b200 as vc
from paper_2609_15810_b200 import binding
from paper_2609_15810_b200.binding import CrossParams, LinearParams, QkParams, QuantParams, Strides

P = 4096          # stands for an aligned address: a refused call never looks at it


def _qk(lib=None, ptrs=(P, P, P, P, P, P, P), **kw):
    p = QkParams(B=1, N=24, d=64, H_q=2, H_k=2, grid_t=2, grid_h=3, grid_w=4, norm=vc.VC_NORM_HEAD, rotary=vc.VC_ROTARY_HALF)
    for k, v in kw.items():
        setattr(p, k, v)
    q, k, wq, wk, pos, qo, ko = ptrs
    return vc.load_library().vc_qk_norm_rope(ctypes.byref(p), q, k, wq, wk, pos, qo, ko, None)


NO_POS = (P, P, P, P, None, 2 * P, 2 * P)


@pytest.mark.parametrize("kw", [
    dict(B=0), dict(B=65536), dict(N=0), dict(N=(1 << 22) + 1), dict(d=0), dict(d=60), dict(d=264), dict(H_q=0, H_k=0), dict(H_q=-1), dict(H_k=65536),
    dict(dtype=3), dict(dtype=-1), dict(weight_dtype=3), dict(norm=3), dict(norm=-1), dict(rotary=3), dict(rotary=-1), dict(eps=-1.0), dict(eps=float("nan")),
    dict(grid_t=3), dict(grid_h=0), dict(grid_w=-4), dict(start_t=2 ** 31 - 2), dict(rope_dim_t=3, rope_dim_h=5), dict(rope_dim_t=-2, rope_dim_h=4),
    dict(rope_dim_t=60, rope_dim_h=8), dict(rope_theta=0.5), dict(rope_theta=float("inf")), dict(rope_theta=float("nan")), dict(rope_scaling=4),
    dict(rope_scaling=-1), dict(rope_factor_t=-1.0), dict(rope_factor_w=float("nan")), dict(rope_attention_factor=-1.0), dict(yarn_beta_fast=-2.0),
    dict(rope_scaling=vc.VC_ROPE_SCALING_YARN),
    dict(q=Strides(0, 0, 63)), dict(q=Strides(0, 0, 68)), dict(B=2, k=Strides(-64, 64, 64)), dict(q=Strides(0, 3, 64)), dict(q_out=Strides(0, 0, 64)),
    dict(q=Strides(0, 1 << 40, 64)), dict(k_out=Strides(1536, 1536, 32))])
def test_qk_norm_rope_parameters(kw):
    assert _qk(ptrs=NO_POS, **kw) == vc.VC_ERR_INVALID_ARG


@pytest.mark.parametrize("at", range(7))
def test_qk_norm_rope_pointers(at):
    ptrs = [P, 3 * P, P, P, P, 2 * P, 4 * P]
    ptrs[at] += 8
    assert _qk(ptrs=ptrs) == vc.VC_ERR_INVALID_ARG
    if at in (0, 1, 5, 6):
        ptrs[at] = None
        assert _qk(ptrs=ptrs) == vc.VC_ERR_INVALID_ARG


def test_qk_norm_rope_in_place_wants_the_same_strides():
    assert _qk(ptrs=(P, P, P, P, None, P, 2 * P), q_out=Strides(0, 64, 128)) == vc.VC_ERR_INVALID_ARG


@pytest.mark.parametrize("values", [(0.5, 0, 0, 0), (1.0, 0, 0, 0), (float("inf"), 0, 0, 0), (float("nan"), 0, 0, 0), (0, -1.5, 0, 0), (0, 0, float("nan"), 0),
                                    (0, 0, 0, float("inf"))])
def test_qk_norm_rope_values(values):
    p = QkParams(B=1, N=24, d=64, H_q=2, H_k=2, grid_t=2, grid_h=3, grid_w=4, norm=vc.VC_NORM_HEAD, rotary=vc.VC_ROTARY_HALF, rope_scaling=vc.VC_ROPE_SCALING_LINEAR)
    rope = vc.RopeValues(*values)
    assert vc.load_library().vc_qk_norm_rope_with_values(ctypes.byref(p), ctypes.byref(rope), *NO_POS, None) == vc.VC_ERR_INVALID_ARG
    assert vc.load_library().vc_qk_norm_rope_with_values(None, ctypes.byref(rope), *NO_POS, None) == vc.VC_ERR_INVALID_ARG
    p.rope_theta = 0.5                                            # (without values the fields are looked at)
    assert vc.load_library().vc_qk_norm_rope_with_values(ctypes.byref(p), None, *NO_POS, None) == vc.VC_ERR_INVALID_ARG


def test_theta_and_factors_keep_their_64_bits_on_the_way():
    x = torch.zeros(1, 2, 24, 64)
    of = lambda **kw: QkParams.of(x, None, x, None, grid=(2, 3, 4), **kw)
    for p in (of(), of(rope_theta=10000.0, rope_factor=(4.0, 1.5, 0.0))):
        assert p.rope is None and p.rope_values() is None
    p = of(rope_theta=12345.678, rope_factor=(3.3, 2.0, 0.1))
    at = p.rope_values()
    got = vc.RopeValues.from_address(at)
    assert (got.theta, got.factor_t, got.factor_h, got.factor_w) == (12345.678, 3.3, 2.0, 0.1) and abs(p.rope_factor_t - 3.3) < 1e-6
    p.rope_factor_t = 8.0                                         # a field that is changed stands, the others keep theirs
    p.rope_theta = 0.0
    got = vc.RopeValues.from_address(p.rope_values())
    assert (got.theta, got.factor_t, got.factor_h, got.factor_w) == (0.0, 0.0, 2.0, 0.1) and p.rope_factor_t == 8.0
    assert p.rope_values() == ctypes.addressof(p.rope)
    assert ctypes.sizeof(vc.RopeValues) == 32


OVERLAPPING = [Strides(0, 8, 64), Strides(0, 64, 64), Strides(0, 64, 72), Strides(0, 64 * 23, 64), Strides(0, 128, 64)]


@pytest.mark.parametrize("at", range(len(OVERLAPPING)))
@pytest.mark.parametrize("name", ["q_out", "k_out"])
def test_qk_norm_rope_outputs_whose_heads_overlap(name, at):
    assert _qk(ptrs=NO_POS, **{name: OVERLAPPING[at]}) == vc.VC_ERR_INVALID_ARG


def _quant(x=P, codes=P, scale=P, **kw):
    p = QuantParams(B=1, H=2, N=5, d=64, block_rows=1)
    for k, v in kw.items():
        setattr(p, k, v)
    return vc.load_library().vc_quant_fp8(ctypes.byref(p), x, codes, scale, None)


@pytest.mark.parametrize("kw", [
    dict(x=None), dict(codes=None), dict(scale=None), dict(x=P + 8), dict(codes=P + 1), dict(scale=P + 4), dict(B=0), dict(H=0), dict(N=0), dict(d=0),
    dict(d=12), dict(H=1, d=24), dict(H=1 << 15), dict(B=1 << 16, N=1 << 15), dict(dtype=5), dict(block_rows=0), dict(block_rows=64)])
def test_quant_fp8(kw):
    assert _quant(**kw) == vc.VC_ERR_INVALID_ARG


def _cross(q=P, k=P, v=P, kv_len=P, mask=P, o=P, lse=P, work=P, **kw):
    p = CrossParams(B=2, H=4, H_kv=2, N_q=5, N_kv=7, d=64)
    for n, val in kw.items():
        setattr(p, n, val)
    return vc.load_library().vc_cross_attn(ctypes.byref(p), q, k, v, kv_len, mask, o, lse, work, None), vc.vc_cross_workspace_bytes(p)


@pytest.mark.parametrize("kw", [
    dict(B=0), dict(H=0), dict(H_kv=0), dict(H_kv=3), dict(H_kv=8), dict(B=8192, H=8), dict(N_q=0), dict(N_q=(1 << 22) + 1), dict(N_kv=-1),
    dict(N_kv=(1 << 22) + 1), dict(d=32), dict(d=96), dict(d=256), dict(dtype=vc.VC_DTYPE_FP32), dict(dtype=-1), dict(key_splits=-1), dict(key_splits=65),
    dict(softmax_scale=-1.0), dict(softmax_scale=float("nan")), dict(softmax_scale=float("inf")), dict({"q": Strides(20 * 64, 5 * 64, 60)}),
    dict({"k": Strides(1, 7 * 64, 64)}), dict({"v": Strides(14 * 64, -64, 64)}), dict({"o": Strides(0, 5 * 64, 64)}), dict({"o": Strides(20 * 64, 0, 64)})])
def test_cross_attn_parameters(kw):
    p = CrossParams(B=2, H=4, H_kv=2, N_q=5, N_kv=7, d=64)
    for n, val in kw.items():
        setattr(p, n, val)
    assert vc.load_library().vc_cross_attn(ctypes.byref(p), P, P, P, P, P, P, P, P, None) == vc.VC_ERR_INVALID_ARG
    assert vc.vc_cross_workspace_bytes(p) == 0


@pytest.mark.parametrize("kw", [dict(q=None), dict(k=None), dict(v=None), dict(o=None), dict(work=None), dict(q=P + 8), dict(k=P + 2), dict(v=P + 8),
                                dict(o=P + 8), dict(work=P + 4), dict(lse=P + 2), dict(kv_len=P + 1)])
def test_cross_attn_pointers(kw):
    assert _cross(**kw)[0] == vc.VC_ERR_INVALID_ARG


def test_cross_attn_workspace():
    size = lambda **kw: _size(CrossParams(B=1, H=2, H_kv=2, N_q=1, N_kv=4096, d=128), **kw)
    def _size(p, **kw):
        for n, val in kw.items():
            setattr(p, n, val)
        return vc.vc_cross_workspace_bytes(p)
    assert size(key_splits=1) == 256
    assert size(key_splits=4) >= 256 + 4 * 2 * (128 + 1) * 4
    assert size(key_splits=64) == size(key_splits=32)            # no more than there are key tiles
    assert size(N_kv=0) == size(N_kv=128) == 256
    assert size() >= 256 and size(N_q=100000) == 256             # enough rows: nothing to split


@pytest.mark.parametrize("o", [
    Strides(20 * 64, 8, 64), Strides(20 * 64, 64, 64), Strides(20 * 64, 64, 128), Strides(20 * 64, 4 * 64, 64), Strides(19 * 64, 5 * 64, 64),
    Strides(64, 5 * 64, 64), Strides(8, 5 * 64, 64), Strides(20 * 64, 64, 4 * 64 - 8)])
def test_cross_attn_outputs_whose_heads_or_batches_overlap(o):
    p = CrossParams(B=2, H=4, H_kv=2, N_q=5, N_kv=7, d=64, o=o)
    assert vc.load_library().vc_cross_attn(ctypes.byref(p), P, P, P, P, P, P, P, P, None) == vc.VC_ERR_INVALID_ARG
    assert vc.vc_cross_workspace_bytes(p) == 0


@pytest.mark.parametrize("o", [
    Strides(20 * 64, 5 * 64, 64), Strides(20 * 64, 64, 4 * 64), Strides(64, 2 * 64, 8 * 64), Strides(64, 10 * 64, 2 * 64), Strides(4 * 64, 64, 8 * 64),
    Strides(2 ** 39 - 8, 72, 4 * 72)])
def test_cross_attn_outputs_in_any_order_of_dimensions(o):
    assert vc.vc_cross_workspace_bytes(CrossParams(B=2, H=4, H_kv=2, N_q=5, N_kv=7, d=64, o=o)) == 256


def test_cross_attn_inputs_whose_heads_overlap_are_read():
    p = CrossParams(B=2, H=4, H_kv=2, N_q=5, N_kv=7, d=64, q=Strides(0, 8, 64), k=Strides(64, 64, 64), v=Strides(0, 0, 64))
    assert vc.vc_cross_workspace_bytes(p) == 256


@pytest.mark.parametrize("kw", [dict(B=1), dict(H=1, H_kv=1), dict(N_q=1)])
def test_cross_attn_strides_of_dimensions_of_one_entry_are_not_looked_at(kw):
    """With one batch, head or query its stride overlaps nothing."""
    at = {"B": "b", "H": "h", "N_q": "n"}[next(iter(kw))]
    o = Strides(20 * 64, 5 * 64, 64)
    setattr(o, at, 8)
    p = CrossParams(B=2, H=4, H_kv=2, N_q=5, N_kv=7, d=64, o=o)
    for n, val in kw.items():
        setattr(p, n, val)
    assert vc.vc_cross_workspace_bytes(p) == 256


def _linear(ptrs=(P,) * 7, **kw):
    p = LinearParams(M=5, N=6, K=32)
    for n, val in kw.items():
        setattr(p, n, val)
    return vc.load_library().vc_linear_fp8(ctypes.byref(p), *ptrs, None), vc.vc_linear_workspace_bytes(p)


@pytest.mark.parametrize("kw", [dict(M=0), dict(N=0), dict(K=0), dict(K=24), dict(K=(1 << 20) + 16), dict(M=(1 << 30) + 1), dict(N=(1 << 30) + 1), dict(out_dtype=3),
                                dict(bias_dtype=-1), dict(k_splits=-1), dict(k_splits=65), dict(ldx=16), dict(ldx=40), dict(ldw=-32), dict(ldo=5),
                                dict(ldo=1 << 32)])
def test_linear_fp8_parameters(kw):
    assert _linear(**kw) == (vc.VC_ERR_INVALID_ARG, 0)


@pytest.mark.parametrize("at", range(7))
def test_linear_fp8_pointers(at):
    for bad in (P + 8, None):
        ptrs = [P] * 7
        ptrs[at] = bad
        if not (at == 4 and bad is None):                        # (no bias is no mistake)
            assert _linear(ptrs)[0] == vc.VC_ERR_INVALID_ARG


def test_linear_fp8_workspace():
    def size(M, N, K, splits=0):
        return vc.vc_linear_workspace_bytes(LinearParams(M=M, N=N, K=K, k_splits=splits))
    assert size(1, 5120, 5120, 1) == 256
    assert size(1, 5120, 5120, 3) == 256 + 3 * 5120 * 4
    assert size(2, 5, 512, 64) == 256 + 4 * 2 * 8 * 4            # no more splits than blocks; rows of a part padded to 16 bytes
    assert size(32760, 5120, 5120) == 256


def test_no_parameters():
    lib = vc.load_library()
    assert lib.vc_linear_fp8(None, P, P, P, P, P, P, P, None) == vc.VC_ERR_INVALID_ARG and lib.vc_linear_workspace_bytes(None) == 0
    assert lib.vc_cross_attn(None, P, P, P, P, P, P, P, P, None) == vc.VC_ERR_INVALID_ARG and lib.vc_cross_workspace_bytes(None) == 0
    assert lib.vc_qk_norm_rope(None, P, P, P, P, P, P, P, None) == vc.VC_ERR_INVALID_ARG
    assert lib.vc_quant_fp8(None, P, P, P, None) == vc.VC_ERR_INVALID_ARG


def test_parameter_blocks_from_tensors():
    x = torch.zeros(2, 6, 3, 64, dtype=torch.float16).transpose(1, 2)          # [B, H, N, d] of [B, N, H, d] memory
    p = QkParams.of(x, None, torch.zeros(2, 3, 6, 64, dtype=torch.float16), None, grid=(1, 2, 3))
    assert (p.B, p.N, p.d, p.H_q, p.H_k, p.dtype, p.grid_h, p.grid_w) == (2, 6, 64, 3, 0, vc.VC_DTYPE_FP16, 2, 3)
    assert (p.q.b, p.q.h, p.q.n) == (6 * 3 * 64, 64, 3 * 64) and (p.q_out.b, p.q_out.h, p.q_out.n) == (3 * 6 * 64, 6 * 64, 64)
    with pytest.raises(ValueError):
        QkParams.of(x, x[:, :, :5], x, x[:, :, :5])
    with pytest.raises(ValueError):
        QkParams.of(x, None, x.float(), None)
    with pytest.raises(ValueError):
        QuantParams.of(x.transpose(2, 3))
    with pytest.raises(ValueError):
        QuantParams.of(x.to(torch.float64))
    m = QuantParams.of(torch.zeros(7, 48), 128)
    assert (m.B, m.H, m.N, m.d, m.block_rows, m.dtype) == (1, 1, 7, 48, 128, vc.VC_DTYPE_FP32)


def test_sizes_of_the_parameter_blocks():
    """The C structs have no padding the mirrors lack: 8-byte members start on 8-byte boundaries."""
    assert ctypes.sizeof(Strides) == 24
    assert ctypes.sizeof(QkParams) == 22 * 4 + 8 * 4 + 4 * 24
    assert ctypes.sizeof(CrossParams) == 8 * 4 + 4 + 4 + 4 * 24          # 4 bytes of padding in front of the strides, as in C
    assert ctypes.sizeof(LinearParams) == 6 * 4 + 3 * 8
    assert ctypes.sizeof(QuantParams) == 6 * 4 + 24


def test_a_key_mask_of_no_keys_is_taken():
    """[B, 0] tensors have strides of their own; with nothing to address none is wrong."""
    p = CrossParams(B=3, H=4, H_kv=2, N_q=5, N_kv=0, d=64)
    want = binding._cross_wants(p)[4]
    for dt in (torch.bool, torch.uint8):
        binding._address(torch.zeros(3, 0, dtype=dt), -1, want)
    for wrong in (torch.zeros(2, 0, dtype=torch.bool), torch.zeros(3, 1, dtype=torch.bool), torch.zeros(3, 0)):
        with pytest.raises(ValueError):
            binding._address(wrong, -1, want)
