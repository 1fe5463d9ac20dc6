"""vc_qk_norm_rope against the formulas in 64 bits.

Tolerance: one rounding to the output's type, half a step of the value (eps / 2), and the FP32 arithmetic in front of it, bounded
by 64 * 2^-24 of what the channel is a sum of: the sum of squares is a chain of at most 8 additions a chunk, 8 or more chunks
a thread, 5 shuffles and 16 partial sums (relative error below 90 * 2^-24 at the sizes here, halved by the root), then rsqrt
(2 ulp), two multiplications, sincospi (its argument half an ulp of 1, which is pi * 2^-24, and 2 ulp), the factor, two products, one sum.
"""
import math
from decimal import Decimal, getcontext

import numpy as np
import pytest
import torch

import paper_2609_15810_b200 as vc
from oracle import layer as L

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
NORM = {"none": vc.VC_NORM_NONE, "head": vc.VC_NORM_HEAD, "token": vc.VC_NORM_TOKEN}
ROT = {None: vc.VC_ROTARY_NONE, L.INTERLEAVED: vc.VC_ROTARY_INTERLEAVED, L.HALF: vc.VC_ROTARY_HALF}
SCAL = {"none": vc.VC_ROPE_SCALING_NONE, "linear": vc.VC_ROPE_SCALING_LINEAR, "ntk": vc.VC_ROPE_SCALING_NTK, "yarn": vc.VC_ROPE_SCALING_YARN}


def _tensor(shape, dt, token_major, g, scale=1.5):
    B, H, N, d = shape
    x = torch.randn((B, N, H, d) if token_major else shape, generator=g) * scale
    x = x.to(DT[dt]).cuda()
    return x.transpose(1, 2) if token_major else x


def _close(got, want, size, dt):
    got, err = got.double().cpu().numpy(), None
    err = np.abs(got - want)
    tol = torch.finfo(DT[dt]).eps / 2 * np.abs(want) + 64 * 2.0 ** -24 * size
    if dt == "fp16":
        tol += 2.0 ** -25              # half a step of the subnormals
    bad = err > tol
    assert not bad.any(), f"{bad.sum()} of {bad.size} off, worst {np.max(err / tol):.2f} of the tolerance"


def _run(B, Hq, Hk, grid, d, dt="bf16", norm="head", layout=L.INTERLEAVED, dims=None, scaling="none", factor=(1.0, 1.0, 1.0), original=0,
         start=(0, 0, 0), positions=None, in_major=True, out_major=False, weights=True, weight_dt=None, in_place=False, seed=1, eps=0.0, **kw):
    g = torch.Generator().manual_seed(seed)
    N = grid[0] * grid[1] * grid[2]
    q = _tensor((B, Hq, N, d), dt, in_major, g) if Hq else None
    k = _tensor((B, Hk, N, d), dt, in_major, g) if Hk else None
    x64 = [None if t is None else t.double().cpu().numpy() for t in (q, k)]
    wdt = weight_dt or dt
    w = [None, None]
    if norm != "none" and weights:
        w = [(1.0 + 0.3 * torch.randn(d * (H if norm == "token" else 1), generator=g)).to(DT[wdt]).cuda() if H else None for H in (Hq, Hk)]
    pos = None if positions is None else torch.from_numpy(positions.astype(np.int32)).cuda()
    out = []
    for t, H in ((q, Hq), (k, Hk)):
        if t is None:
            out.append(None)
        elif in_place:
            out.append(t)
        else:
            o = torch.full((B, N, H, d) if out_major else (B, H, N, d), float("nan"), dtype=DT[dt], device="cuda")
            out.append(o.transpose(1, 2) if out_major else o)
    p = vc.QkParams.of(q, k, *out, grid=grid if positions is None else (0, 0, 0), weight=next((t for t in w if t is not None), None), norm=NORM[norm],
                       rotary=ROT[layout], rope_dims=dims or (0, 0, 0), start=start, rope_scaling=SCAL[scaling], rope_factor=factor,
                       rope_original=(original,) * 3, eps=eps, **kw)
    vc.vc_qk_norm_rope(p, q, k, *w, pos, *out)
    dims = dims or L.default_dims(d)
    theta = kw.get("rope_theta") or 10000.0
    freqs = [L.frequencies(n, theta, scaling, f, original) for n, f in zip(dims, factor)]
    big = max([f for n, f in zip(dims, factor) if n] + [1.0])
    mult = kw.get("rope_attention_factor") or (0.1 * np.log(big) + 1.0 if scaling == "yarn" else 1.0)
    at = L.positions_of(grid, start) if positions is None else positions
    for x, t, o in zip(x64, w, out):
        if x is not None:
            want, size = L.qk_norm_rope(x, None if t is None else t.double().cpu().numpy(), norm, eps or 1e-6, layout, dims, at, freqs, mult)
            _close(o, want, size, dt)


@pytest.mark.parametrize("dt", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("norm", ["none", "head", "token"])
@pytest.mark.parametrize("layout", [None, L.INTERLEAVED, L.HALF])
@pytest.mark.parametrize("d", [64, 128])
def test_types_norms_and_layouts(dt, norm, layout, d):
    _run(2, 5, 3, (3, 5, 7), d, dt, norm, layout)


@pytest.mark.parametrize("d,dims", [(8, (8, 0, 0)), (8, (2, 2, 2)), (16, (0, 6, 0)), (80, (0, 0, 0)), (80, (30, 26, 24)), (96, (64, 0, 32)),
                                    (192, (64, 64, 64)), (256, (256, 0, 0)), (256, (2, 128, 120)), (248, (10, 20, 30)), (128, (48, 0, 0))])
@pytest.mark.parametrize("layout", [L.INTERLEAVED, L.HALF])
def test_head_dimensions_and_parts_of_the_head(d, dims, layout):
    dims = dims if any(dims) else L.default_dims(d)
    _run(1, 3, 2, (2, 9, 5), d, "bf16", "head", layout, dims)
    _run(1, 3, 2, (2, 9, 5), d, "fp32", "token", layout, dims)


@pytest.mark.parametrize("N,H", [(1, 1), (1, 40), (2, 7), (15, 2), (16, 3), (17, 1), (129, 24), (1, 200), (33, 150), (2, 300)])
@pytest.mark.parametrize("norm", ["head", "token"])
def test_rows_and_heads_from_one_on(N, H, norm):
    _run(1, H, max(1, H // 2), (1, 1, N), 128, "bf16", norm)


@pytest.mark.parametrize("scaling", ["none", "linear", "ntk", "yarn"])
@pytest.mark.parametrize("layout", [L.INTERLEAVED, L.HALF])
def test_scaled_frequencies_at_far_positions(scaling, layout):
    _run(1, 2, 2, (61, 1, 3), 128, "fp32", "none", layout, (64, 32, 30), scaling, (4.0, 1.0, 2.5), 256, start=(1000000, 7, 100000))
    _run(1, 2, 2, (61, 1, 1), 64, "bf16", "head", layout, (64, 0, 0), scaling, (8.0, 1.0, 1.0), 4096, start=(32768, 0, 0))
    _run(1, 1, 1, (33, 1, 1), 64, "fp32", "none", layout, (2, 2, 8), scaling, (3.0, 2.0, 1.0), 16, rope_theta=500000.0)


def test_factor_of_the_rotated_channels():
    _run(1, 2, 2, (9, 2, 2), 64, "fp32", "head", L.HALF, (32, 0, 0), "yarn", (4.0, 1.0, 1.0), 64, rope_attention_factor=1.25)
    _run(1, 2, 2, (9, 2, 2), 64, "fp32", "head", L.INTERLEAVED, (32, 0, 0), "yarn", (0.5, 1.0, 1.0), 64)      # no factor above 1: m = 1


@pytest.mark.parametrize("layout,dims", [(L.INTERLEAVED, None), (L.HALF, None), (L.HALF, (64, 32, 32)), (None, None)])
@pytest.mark.parametrize("Hq,Hk,grid", [(12, 3, (7, 23, 61)), (2, 11, (7, 23, 61)), (40, 40, (3, 40, 41))])
def test_long_sequences_under_the_token_norm(layout, dims, Hq, Hk, grid):
    """So many tokens that a CTA takes its tokens' queries and then their keys."""
    _run(1, Hq, Hk, grid, 128, "bf16", "token", layout, dims)
    _run(1, Hq, Hk, grid, 128, "fp16", "token", layout, dims, in_place=True)


@pytest.mark.parametrize("layout", [L.INTERLEAVED, L.HALF])
def test_positions_over_the_whole_range_of_int32(layout):
    """The angle in FP64 is off by 2^31 2^-53 there: nothing beside a step of bf16."""
    rng = np.random.default_rng(12)
    pos = rng.integers(-2 ** 31, 2 ** 31, size=(2, 300, 3))
    pos[:, :4] = [[[-2 ** 31] * 3, [2 ** 31 - 1] * 3, [-1] * 3, [0] * 3]]
    _run(2, 2, 1, (300, 1, 1), 64, "bf16", "none", layout, (16, 32, 16), positions=pos)
    _run(1, 2, 1, (300, 1, 1), 64, "bf16", "head", layout, (16, 32, 16), start=(2 ** 31 - 400, 5, 2 ** 30))


def _turns(positions, n, theta, scaling, factor):
    """position * frequency of an axis's pairs in turns within [-1/2, 1/2], [positions, pairs], from 50 decimal digits."""
    getcontext().prec = 50
    two_pi, base, factor = 2 * Decimal("3.14159265358979323846264338327950288419716939937511"), Decimal(theta), Decimal(factor)
    if scaling == "ntk":
        base *= (factor.ln() * n / (n - 2)).exp()
    out = np.empty((len(positions), n // 2))
    for i in range(n // 2):
        f = (base.ln() * -2 * i / n).exp() / two_pi / (factor if scaling == "linear" else 1)
        if scaling == "yarn":
            lo, hi = (n * math.log(4096 / (2 * math.pi * b)) / (2 * math.log(theta)) for b in (32.0, 1.0))
            lo, hi = max(math.floor(lo), 0), min(math.ceil(hi), n - 1)
            r = min(max(Decimal(i - lo) / Decimal(hi - lo), Decimal(0)), Decimal(1))
            f = f * (1 - r) + f / factor * r
        out[:, i] = [float(int(p) * f - (int(p) * f).to_integral_value()) for p in positions]
    return out


@pytest.mark.parametrize("layout,dims", [(L.INTERLEAVED, (256, 0, 0)), (L.HALF, (256, 0, 0)), (L.HALF, (0, 0, 250))])
@pytest.mark.parametrize("theta,scaling,factor", [(10000.0, "none", 1.0), (1.0009765625, "none", 1.0), (1.0 + 2.0 ** -23, "none", 1.0), (10000.0, "linear", 1.5),
                                                  (1.0009765625, "ntk", 1.25), (12345.678, "none", 1.0), (10000.0, "linear", 3.3), (12345.678, "ntk", 2.7),
                                                  (10000.0, "yarn", 1.1)])
def test_angles_of_the_farthest_positions(layout, dims, theta, scaling, factor):
    """Frequencies that hardly fall from pair to pair, theta and factors that are no FP32 numbers, at positions up to 2^31, to the accuracy of FP32.

    In units of 2^-24: the turns are off by 2^31 ((2 i + 8) f_i + 1) 2^-64 <= 44 * 2^-33 (0.6 in the angle), cut to 32 bits (0.03) and rounded to a float of at
    most one half turn, 2^-25 of it (1.6); sincospi is off by 2 ulp of a value below 1 (2), a product by 1, the sum by 1: 6.2 of |a| + |b|, 8 with room."""
    d, axis = 256, int(np.argmax(dims))
    n = dims[axis]
    rng = np.random.default_rng(21)
    pos = np.zeros((1, 64, 3), np.int64)
    pos[0, :, axis] = rng.integers(-2 ** 31, 2 ** 31, 64)
    pos[0, :4, axis] = (-2 ** 31, 2 ** 31 - 1, -1, 10 ** 9)
    x = torch.randn(1, 2, 64, d, generator=torch.Generator().manual_seed(22))
    out = torch.empty(x.shape, device="cuda")
    p = vc.QkParams.of(out, None, out, None, rotary=ROT[layout], rope_dims=dims, rope_theta=theta, rope_scaling=SCAL[scaling], rope_factor=(factor,) * 3,
                       rope_original=(4096,) * 3, rope_attention_factor=1.0)
    vc.vc_qk_norm_rope(p, x.cuda(), None, None, None, torch.from_numpy(pos.astype(np.int32)).cuda(), out, None)
    x, got = x.double().numpy(), out.double().cpu().numpy()
    angle = 2.0 * math.pi * _turns(pos[0, :, axis], n, theta, scaling, factor)
    for i in range(n // 2):
        a, b = (2 * i, 2 * i + 1) if layout == L.INTERLEAVED else (i, i + n // 2)
        c, s = np.cos(angle[:, i]), np.sin(angle[:, i])
        tol = 8 * 2.0 ** -24 * (np.abs(x[..., a]) + np.abs(x[..., b]))
        assert (np.abs(got[..., a] - (x[..., a] * c - x[..., b] * s)) <= tol).all(), i
        assert (np.abs(got[..., b] - (x[..., a] * s + x[..., b] * c)) <= tol).all(), i
    assert np.array_equal(got[..., n:], x[..., n:])


@pytest.mark.parametrize("layout", [L.INTERLEAVED, L.HALF])
def test_positions_from_an_array(layout):
    rng = np.random.default_rng(3)
    pos = rng.integers(-5000, 2 ** 20, (2, 45, 3))
    pos[0, 0] = (2 ** 31 - 1, -2 ** 31, 0)
    _run(2, 3, 1, (45, 1, 1), 128, "bf16", "head", layout, positions=pos)


@pytest.mark.parametrize("in_major,out_major", [(False, False), (False, True), (True, True)])
@pytest.mark.parametrize("norm", ["head", "token"])
def test_layouts(in_major, out_major, norm):
    _run(2, 4, 4, (2, 3, 11), 64, "fp16", norm, in_major=in_major, out_major=out_major)


@pytest.mark.parametrize("norm", ["none", "head", "token"])
@pytest.mark.parametrize("layout", [L.INTERLEAVED, L.HALF])
def test_in_place(norm, layout):
    _run(1, 150, 20, (2, 3, 11), 128, "bf16", norm, layout, in_place=True)


def test_either_tensor_alone_no_weights_other_weight_types():
    _run(1, 3, 0, (2, 3, 4), 128)
    _run(1, 0, 3, (2, 3, 4), 128, norm="token")
    _run(1, 3, 2, (2, 3, 4), 128, weights=False)
    _run(1, 3, 2, (2, 3, 4), 128, norm="token", weights=False, eps=1e-2)
    for norm in ("head", "token"):
        _run(1, 3, 2, (2, 3, 4), 64, "bf16", norm, weight_dt="fp32")
        _run(1, 3, 2, (2, 3, 4), 64, "fp32", norm, weight_dt="fp16")
        _run(1, 3, 2, (2, 3, 4), 64, "fp16", norm, weight_dt="bf16")


def test_views_of_one_projection_and_rows_behind_them_untouched():
    """Q and K rotated in place inside the [B, N, 3, H, d] output of a fused projection; V and what lies around stay."""
    B, N, H, d = 2, 35, 3, 64
    g = torch.Generator().manual_seed(5)
    x = torch.randn(B, N + 2, 3, H, d, generator=g).to(torch.bfloat16).cuda()
    before = x.clone()
    q, k = (x[:, 1:N + 1, i].transpose(1, 2) for i in (0, 1))
    want = [L.qk_norm_rope(t.double().cpu().numpy(), None, "head", 1e-6, L.INTERLEAVED, L.default_dims(d), L.positions_of((5, 7, 1)),
                           [L.frequencies(n) for n in L.default_dims(d)]) for t in (q, k)]
    p = vc.QkParams.of(q, k, q, k, grid=(5, 7, 1), norm=vc.VC_NORM_HEAD, rotary=vc.VC_ROTARY_INTERLEAVED)
    vc.vc_qk_norm_rope(p, q, k, None, None, None, q, k)
    for t, (y, size) in zip((q, k), want):
        _close(t, y, size, "bf16")
    assert torch.equal(x[:, :, 2], before[:, :, 2])
    assert torch.equal(x[:, 0], before[:, 0]) and torch.equal(x[:, N + 1], before[:, N + 1])


def test_channels_that_are_not_rotated_pass_infinities_through():
    x = torch.zeros(1, 1, 4, 64, dtype=torch.float32, device="cuda")
    x[..., 40], x[..., 63], x[..., 50] = float("inf"), float("-inf"), float("nan")
    for layout in (vc.VC_ROTARY_INTERLEAVED, vc.VC_ROTARY_HALF):
        o = torch.empty_like(x)
        p = vc.QkParams.of(x, None, o, None, grid=(4, 1, 1), rotary=layout, rope_dims=(32, 0, 0))
        vc.vc_qk_norm_rope(p, x, None, None, None, None, o, None)
        assert torch.equal(torch.nan_to_num(o, nan=7.0), torch.nan_to_num(x, nan=7.0))


def test_other_stream_and_a_captured_call():
    g = torch.Generator().manual_seed(6)
    q = _tensor((1, 4, 100, 128), "bf16", False, g)
    want, got = torch.empty_like(q), torch.empty_like(q)
    p = vc.QkParams.of(q, None, want, None, grid=(4, 5, 5), norm=vc.VC_NORM_HEAD, rotary=vc.VC_ROTARY_HALF)
    vc.vc_qk_norm_rope(p, q, None, None, None, None, want, None)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        vc.vc_qk_norm_rope(p, q, None, None, None, None, got, None)
    s.synchronize()
    assert torch.equal(got, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        vc.vc_qk_norm_rope(p, q, None, None, None, None, got, None)
    q.mul_(-2.0)
    vc.vc_qk_norm_rope(p, q, None, None, None, None, want, None)
    got.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(got, want)


def test_same_rotation_as_the_preprocessing_pass():
    """Rotated in front, with the flag off, the bundle's mean of K is that of the pass's own rotation."""
    g = torch.Generator().manual_seed(7)
    q, k, v = (_tensor((1, 2, 256, 128), "bf16", False, g) for _ in range(3))
    from paper_2609_15810_b200.binding import Params, alloc_buffers, section
    out = []
    qo, ko = torch.empty_like(q), torch.empty_like(k)
    p = vc.QkParams.of(q, k, qo, ko, grid=(4, 8, 8), rotary=vc.VC_ROTARY_INTERLEAVED)
    vc.vc_qk_norm_rope(p, q, k, None, None, None, qo, ko)
    for qq, kk, flags in ((q, k, vc.VC_FLAG_ALL), (qo, ko, vc.VC_FLAG_ALL & ~vc.VC_FLAG_ROPE)):
        pp = Params.make(1, 2, 256, 128, (4, 8, 8), flags=flags)
        quant, work = alloc_buffers(pp)
        vc.vc_prep(pp, qq, kk, v, None, quant, work)
        out.append(section(vc.vc_quant_view(pp, quant), "k_mean", quant, torch.float32).clone())
    # a mean over 256 rotated values, each off by half a bf16 step of at most max |k_out|: independent of sign, at most that
    assert (out[0] - out[1]).abs().max().item() <= 2.0 ** -9 * ko.float().abs().max().item() + 1e-6
