"""vc_quant_fp8 against the oracle: codes and scales are single FP32 operations and one rounding, so they agree bit for bit."""
import numpy as np
import pytest
import torch

import paper_2609_15810_b200 as vc
from oracle import layer as L

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


def _quant(x, block_rows):
    p = vc.QuantParams.of(x, block_rows)
    rows, cols = p.B * p.N, p.H * p.d
    nb = (cols + 127) // 128
    codes = torch.full((rows, cols), 0x55, dtype=torch.uint8, device="cuda")
    scale = torch.full((nb, rows) if block_rows == 1 else ((rows + 127) // 128, nb), -1.0, device="cuda")
    vc.vc_quant_fp8(p, x, codes, scale)
    return codes, scale.t() if block_rows == 1 else scale


def _matrix(x):
    return x.float().cpu() if x.dim() == 2 else x.float().cpu().transpose(1, 2).reshape(x.shape[0] * x.shape[2], -1)


def _check(x, block_rows):
    codes, scale = _quant(x, block_rows)
    want_c, want_s = L.quant_fp8(_matrix(x).numpy(), block_rows)
    scale, codes = scale.cpu().numpy(), codes.cpu().numpy()
    assert np.array_equal(scale, want_s, equal_nan=True)
    whole = np.isfinite(np.repeat(np.repeat(scale, block_rows, 0)[:x.shape[0] if x.dim() == 2 else None], 128, 1))[:codes.shape[0], :codes.shape[1]]
    assert np.array_equal(codes[whole], want_c[whole])
    assert (codes[~whole] & 127 == 127).all()           # under a scale of NaN every code is NaN


@pytest.mark.parametrize("dt", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("block_rows", [1, 128])
@pytest.mark.parametrize("rows,cols", [(1, 16), (1, 128), (31, 144), (32, 256), (33, 1024), (130, 272), (257, 128), (5, 5120)])
def test_matrices(dt, block_rows, rows, cols):
    g = torch.Generator().manual_seed(rows * 7919 + cols)
    x = torch.randn(rows, cols, generator=g) * torch.exp(2.0 * torch.randn(rows, 1, generator=g))
    _check(x.to(DT[dt]).cuda(), block_rows)


@pytest.mark.parametrize("B,H,N,d", [(2, 3, 37, 64), (1, 2, 50, 128), (3, 2, 9, 8), (1, 5, 20, 80), (2, 1, 130, 144)])
@pytest.mark.parametrize("token_major", [False, True])
@pytest.mark.parametrize("block_rows", [1, 128])
def test_heads(B, H, N, d, token_major, block_rows):
    g = torch.Generator().manual_seed(B + 10 * H + N)
    x = torch.randn((B, N, H, d) if token_major else (B, H, N, d), generator=g).to(torch.bfloat16).cuda()
    _check(x.transpose(1, 2) if token_major else x, block_rows)


def test_rows_of_a_wider_matrix_and_its_neighbours():
    g = torch.Generator().manual_seed(3)
    full = torch.randn(40, 512, generator=g).to(torch.float16).cuda()
    _check(full[3:20, 128:400], 1)
    _check(full[3:20, 128:400], 128)


@pytest.mark.parametrize("block_rows", [1, 128])
def test_zeros_tiny_values_and_extremes(block_rows):
    x = torch.zeros(6, 256)
    x[1] = 1e-42                                   # subnormal: far below the least scale, codes 0
    x[2, :128] = torch.linspace(-3.0e38, 3.0e38, 128)      # (its step overflows: a block of infinities and NaN)
    x[3] = 448.0 * 2.0 ** -100                     # the least maximum there is a scale for
    x[4, 0] = 1.0
    x[5, 200] = -0.0
    _check(x.cuda(), block_rows)


@pytest.mark.parametrize("block_rows", [1, 128])
def test_values_up_to_the_type_s_largest(block_rows):
    x = 3.4e38 * torch.linspace(-1.0, 1.0, 256).repeat(3, 1)
    x[1] *= 1e-38
    _check(x.cuda(), block_rows)


@pytest.mark.parametrize("bad", [float("inf"), float("-inf"), float("nan")])
@pytest.mark.parametrize("block_rows", [1, 128])
def test_a_block_with_an_infinity_or_nan_stands_for_nan(bad, block_rows):
    x = torch.ones(130, 256)
    x[3, 70] = bad
    codes, scale = _quant(x.cuda(), block_rows)
    val = torch.from_numpy(L.e4m3_values())[codes.cpu().long()]
    s = scale.cpu().double().repeat_interleave(block_rows, 0)[:130].repeat_interleave(128, 1)
    y = val * s
    hit = torch.zeros(130, 256, dtype=torch.bool)
    hit[3 if block_rows == 1 else slice(0, 128), :128] = True
    assert torch.isnan(y[hit]).all() and torch.isfinite(y[~hit]).all()


def test_captured_call_and_other_stream():
    g = torch.Generator().manual_seed(4)
    x = torch.randn(100, 256, generator=g).cuda()
    p = vc.QuantParams.of(x)
    codes, scale = torch.empty(100, 256, dtype=torch.float8_e4m3fn, device="cuda"), torch.empty(2, 100, device="cuda")
    graph = torch.cuda.CUDAGraph()
    vc.vc_quant_fp8(p, x, codes, scale)
    with torch.cuda.graph(graph):
        vc.vc_quant_fp8(p, x, codes, scale)
    x.mul_(3.0)
    graph.replay()
    torch.cuda.synchronize()
    want_c, want_s = L.quant_fp8(x.cpu().numpy(), 1)
    assert np.array_equal(codes.view(torch.uint8).cpu().numpy(), want_c) and np.array_equal(scale.t().cpu().numpy(), want_s)
