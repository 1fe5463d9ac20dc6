"""The oracle of the operators around the quantized attention, pinned against independent forms (CPU)."""
import math

import numpy as np
import pytest
import torch

from oracle import layer as L


@pytest.mark.parametrize("layout", [L.INTERLEAVED, L.HALF])
@pytest.mark.parametrize("dims", [(16, 0, 0), (4, 6, 2), (0, 8, 8)])
def test_rotation_is_a_complex_product(layout, dims):
    rng = np.random.default_rng(1)
    x = rng.normal(size=(1, 2, 12, 16))
    pos = L.positions_of((2, 3, 2), (5, 7, 11))
    freqs = [L.frequencies(n) for n in dims]
    y, size = L.qk_norm_rope(x, None, "none", layout=layout, dims=dims, pos=pos, freqs=freqs, mult=1.5)
    for n, (t, h, w) in enumerate((t, h, w) for t in (5, 6) for h in (7, 8, 9) for w in (11, 12)):
        c0 = 0
        for p, d in zip((t, h, w), dims):
            for i in range(d // 2):
                a, b = (c0 + 2 * i, c0 + 2 * i + 1) if layout == L.INTERLEAVED else (c0 + i, c0 + d // 2 + i)
                z = (x[0, :, n, a] + 1j * x[0, :, n, b]) * 1.5 * np.exp(1j * p * 10000.0 ** (-2.0 * i / d))
                assert np.allclose(y[0, :, n, a], z.real, atol=1e-12) and np.allclose(y[0, :, n, b], z.imag, atol=1e-12)
            c0 += d
    assert np.array_equal(y[..., sum(dims):], x[..., sum(dims):])
    assert (np.abs(y) <= size + 1e-12).all()


@pytest.mark.parametrize("norm", ["head", "token"])
def test_norm(norm):
    g = torch.Generator().manual_seed(2)
    x = torch.randn(2, 3, 5, 8, generator=g, dtype=torch.float64)
    w = torch.rand(24 if norm == "token" else 8, generator=g, dtype=torch.float64)
    y, _ = L.qk_norm_rope(x.numpy(), w.numpy(), norm, eps=1e-3)
    if norm == "head":
        want = torch.nn.functional.rms_norm(x, (8,), w, 1e-3)
    else:
        flat = x.transpose(1, 2).reshape(2, 5, 24)
        want = torch.nn.functional.rms_norm(flat, (24,), w, 1e-3).view(2, 5, 3, 8).transpose(1, 2)
    assert np.allclose(y, want.numpy(), atol=1e-12)


def test_frequencies_under_scaling():
    f = L.frequencies(8)
    assert np.allclose(f, [1.0, 0.1, 0.01, 0.001])
    assert np.allclose(L.frequencies(8, scaling="linear", factor=4.0), f / 4)
    # NTK: the first pair stays, the last one is slowed by exactly the factor
    ntk = L.frequencies(8, scaling="ntk", factor=4.0)
    assert ntk[0] == 1.0 and math.isclose(ntk[-1], f[-1] / 4.0, rel_tol=1e-12)
    # YaRN: pairs that turn often keep their frequency, those that turn less than once over the trained length are slowed by the factor
    y = L.frequencies(64, scaling="yarn", factor=8.0, original=4096)
    g = L.frequencies(64)
    turns = 4096 * g / (2 * math.pi)
    assert np.allclose(y[turns > 64], g[turns > 64]) and np.allclose(y[turns < 0.5], g[turns < 0.5] / 8.0)
    assert ((y <= g) & (y >= g / 8.0 - 1e-18)).all() and (np.diff(y) < 0).all()


def test_cross_attention():
    g = torch.Generator().manual_seed(3)
    q, k, v = (torch.randn(2, h, n, 16, generator=g, dtype=torch.float64) for h, n in ((4, 7), (2, 11), (2, 11)))
    lens, mask = np.array([11, 6]), np.ones((2, 11), bool)
    mask[0, 3] = mask[1, 0] = False
    o, lse = L.cross_attention(q.numpy(), k.numpy(), v.numpy(), 0.3, lens, mask)
    keep = torch.from_numpy(mask & (np.arange(11) < lens[:, None]))[:, None, None]
    s = (0.3 * q @ k.repeat_interleave(2, 1).transpose(2, 3)).masked_fill(~keep, -math.inf)
    assert np.allclose(o, (s.softmax(-1) @ v.repeat_interleave(2, 1)).numpy(), atol=1e-12)
    assert np.allclose(lse, s.logsumexp(-1).numpy(), atol=1e-12)
    o, lse = L.cross_attention(q.numpy(), k.numpy(), v.numpy(), 0.3, np.array([0, 11]))
    assert (o[0] == 0).all() and np.isneginf(lse[0]).all() and np.isfinite(lse[1]).all()


def test_e4m3_values_and_rounding():
    t = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(L.e4m3_values(), t, equal_nan=True)
    grid = L.e4m3_values()[:127]
    x = np.concatenate([grid, (grid[1:] + grid[:-1]) / 2, np.random.default_rng(4).normal(size=20000) * 30.0])
    x = np.concatenate([x, -x]).astype(np.float32)
    x = x[np.abs(x) <= 448.0]
    assert np.array_equal(L.round_e4m3(x.astype(np.float64)), torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy())


@pytest.mark.parametrize("block_rows", [1, 128])
def test_quantizer_and_product(block_rows):
    g = torch.Generator().manual_seed(5)
    x = torch.randn(130, 272, generator=g) * torch.rand(130, 1, generator=g).exp()
    codes, scale = L.quant_fp8(x.numpy(), block_rows)
    full = np.repeat(np.repeat(scale, block_rows, 0)[:130], 128, 1)[:, :272].astype(np.float64)
    back = L.e4m3_values()[codes] * full
    # half a step: 2^-4 of the value, or half of the least step 2^-9 times the scale; each block's largest value is hit to FP32's accuracy
    assert (np.abs(back - x.numpy()) <= 2.0 ** -4 * np.abs(x.numpy()) + 2.0 ** -10 * full + 1e-7).all()
    for i in range(scale.shape[0]):
        for j in range(scale.shape[1]):
            b = x.numpy()[i * block_rows:(i + 1) * block_rows, 128 * j:128 * j + 128]
            assert scale[i, j] == np.float32(np.abs(b).max()) / np.float32(448.0)
    w, ws = L.quant_fp8(torch.randn(150, 272, generator=g).numpy(), 128)
    if block_rows == 1:
        y, size = L.linear_fp8(codes, scale.T.copy(), w, ws, np.arange(150.0))
        wback = L.e4m3_values()[w] * np.repeat(np.repeat(ws, 128, 0)[:150], 128, 1)[:, :272].astype(np.float64)
        assert np.allclose(y, back @ wback.T + np.arange(150.0), rtol=1e-12) and (np.abs(y) <= size * (1 + 1e-12)).all()
