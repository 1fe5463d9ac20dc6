"""vc_linear_fp8 against the product in 64 bits.

Tolerance per output: u |y| (its rounding, u = eps / 2 of the type) and, of the sum of the products' magnitudes, (132 + blocks + 8) 2^-24: an
instruction adds 32 exact products and its accumulator, each term cut at no less than 24 bits below the largest (33 of them, 4
instructions a block); each block's sum is scaled (2 roundings) and added (1 each; the parts of a split sum count among them), the bias last.
A half value below 2^-14 lies on a grid of 2^-24 and is off by up to half of that, whatever its size: fp16 adds 2^-25.
"""
import numpy as np
import pytest
import torch

import paper_2609_15810_b200 as vc
from oracle import layer as L

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


def _operands(M, N, K, seed, spread=1.0):
    rng = np.random.default_rng(seed)
    nb = -(-K // 128)
    codes = [rng.integers(0, 256, (n, K)).astype(np.uint8) for n in (M, N)]
    for c in codes:
        c[c & 127 == 127] = 0x30                                    # no NaN codes
        c[rng.random(c.shape) < 0.7] &= 0xbf                        # most of them moderate
    xs = np.exp(spread * rng.normal(size=(nb, M))).astype(np.float32)
    ws = np.exp(spread * rng.normal(size=(-(-N // 128), nb))).astype(np.float32)
    return codes[0], xs, codes[1], ws


def _dev(a):
    return torch.from_numpy(a).cuda()


def _run(x, xs, w, ws, dt, bias=None, out=None, **kw):
    M, N = x.shape[0], w.shape[0]
    out = torch.full((M, N), float("nan"), dtype=DT[dt], device="cuda") if out is None else out
    p = vc.LinearParams.of(x, w, out, bias, **kw)
    work = torch.full((vc.vc_linear_workspace_bytes(p),), 0xff, dtype=torch.uint8, device="cuda")
    vc.vc_linear_fp8(p, x, xs, w, ws, bias, out, work)
    vc.vc_poll_status(work)
    return out


def _close(got, x, xs, w, ws, dt, bias=None):
    want, size = L.linear_fp8(x, xs, w, ws, None if bias is None else bias.double().cpu().numpy())
    blocks = xs.shape[0]
    tol = torch.finfo(DT[dt]).eps / 2 * np.abs(want) + (132 + blocks + 8) * 2.0 ** -24 * size
    if dt == "fp16":
        tol = tol + 2.0 ** -25
    err = np.abs(got.double().cpu().numpy() - want)
    assert (err <= tol).all(), f"{(~(err <= tol)).sum()} of {err.size} off, worst {np.nanmax(err / tol):.2f}"


def _check(M, N, K, dt="bf16", bias=True, bias_dt=None, seed=1, **kw):
    x, xs, w, ws = _operands(M, N, K, seed + M + 3 * N + 7 * K)
    b = torch.randn(N, generator=torch.Generator().manual_seed(seed)).mul(100.0).to(DT[bias_dt or dt]).cuda() if bias else None
    if dt == "fp16":                                                # keep the outputs inside the type's range
        xs, ws = xs * np.float32(2.0 ** -8), ws * np.float32(2.0 ** -8)
    out = _run(_dev(x), _dev(xs), _dev(w), _dev(ws), dt, b, **kw)
    _close(out, x, xs, w, ws, dt, b)


@pytest.mark.parametrize("dt", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("M,N,K", [(1, 1, 16), (1, 129, 128), (16, 128, 256), (17, 64, 144), (64, 300, 1024), (65, 1, 16), (100, 130, 272), (128, 256, 128),
                                   (129, 257, 400), (300, 513, 640)])
def test_sizes_and_types(dt, M, N, K):
    _check(M, N, K, dt)
    _check(M, N, K, dt, bias=False)


@pytest.mark.parametrize("M,N,K", [(1, 640, 5120), (7, 200, 2048), (40, 384, 1536), (200, 136, 2176), (130, 260, 4096)])
@pytest.mark.parametrize("splits", [0, 1, 2, 5, 64])
def test_sums_split_between_ctas(M, N, K, splits):
    _check(M, N, K, "bf16", k_splits=splits)
    _check(M, N, K, "fp32", bias_dt="bf16", k_splits=splits)


@pytest.mark.parametrize("N", [2560, 2570, 2433])
def test_wide_tiles(N):
    """Enough tiles of 128 x 256 for every SM, several a CTA; widths whose rows of outputs are and are not on 16-byte boundaries."""
    _check(2500, N, 256, "bf16")
    _check(2500, N, 144, "fp32", bias_dt="fp16")


@pytest.mark.parametrize("M,N", [(2305, 2560), (2433, 2600), (256 * 75, 130), (100, 256 * 80)])
@pytest.mark.parametrize("splits", [1, 3])
def test_tiles_of_two_ctas(M, N, splits):
    """A CTA without rows, halves of weights that end inside or in front of a tile, one tile and more a pair, sums split between pairs."""
    _check(M, N, 640, "bf16", k_splits=splits)
    _check(M, N, 16, "fp16", bias=False, k_splits=splits)


@pytest.mark.parametrize("M,N", [(1300, 1800), (1409, 1665), (1500, 1630), (5000, 2000), (4609, 1665)])
@pytest.mark.parametrize("splits", [0, 3])
def test_fewer_rounds_by_pairs_of_ctas(M, N, splits):
    """Sizes at which a tile is two CTAs': the last one with a CTA without rows or with one, weights that end in either half, up to three tiles a pair."""
    _check(M, N, 400, "bf16", k_splits=splits)
    _check(M, N, 16, "fp16", bias=False, k_splits=splits)
    _check(M, N, 272, "fp32", bias_dt="bf16", k_splits=splits)


@pytest.mark.parametrize("M,N,K", [(1, 5120, 5120), (16, 1, 4096), (17, 640, 2064), (64, 1537, 1024), (33, 130, 5120)])
@pytest.mark.parametrize("splits", [0, 2, 3, 7, 8, 9])
def test_parts_joined_by_a_cluster_and_by_a_launch(M, N, K, splits):
    _check(M, N, K, "bf16", k_splits=splits)
    _check(M, N, K, "fp32", bias=False, k_splits=splits)


@pytest.mark.parametrize("N", [1800, 1801])
def test_pairs_of_ctas_leave_neighbours_alone(N):
    M, K = 1301, 144
    x, xs, w, ws = _operands(M, N, K, 6)
    wide_x, wide_w = np.full((M + 3, K + 32), 0x7f, np.uint8), np.full((N + 5, K + 48), 0x7f, np.uint8)      # NaN codes around
    wide_x[:M, :K], wide_w[:N, :K] = x, w
    around = torch.full((M + 4, N + 24), -7.0, dtype=DT["bf16"], device="cuda")
    out = _run(_dev(wide_x)[:M, :K], _dev(xs), _dev(wide_w)[:N, :K], _dev(ws), "bf16", out=around[:M, 8:N + 8])
    _close(out, x, xs, w, ws, "bf16")
    assert (around[M:] == -7).all() and (around[:, :8] == -7).all() and (around[:, N + 8:] == -7).all()


@pytest.mark.parametrize("K", [1024, 16384])
def test_wait_of_a_pair_of_ctas_that_runs_out(K):
    """As below, for both CTAs: they end together, and the next call is right."""
    g = torch.Generator().manual_seed(14)
    M, N = 2300, 1800
    x, w = (torch.randint(0, 120, (n, K), generator=g, dtype=torch.uint8).cuda() for n in (M, N))
    xs, ws = torch.rand(K // 128, M, generator=g).cuda(), torch.rand(-(-N // 128), K // 128, generator=g).cuda()
    want = _run(x, xs, w, ws, "bf16")
    out = torch.empty_like(want)
    p = vc.LinearParams.of(x, w, out)
    work = torch.empty(vc.vc_linear_workspace_bytes(p), dtype=torch.uint8, device="cuda")
    code = vc.VC_OK
    try:
        vc.vc_test_set_wait_limit(1)
        vc.vc_linear_fp8(p, x, xs, w, ws, None, out, work)
        vc.vc_poll_status(work)
    except vc.VcError as e:
        code = e.code
    finally:
        vc.vc_test_set_wait_limit(0)
    assert code == vc.VC_ERR_TIMEOUT or (K == 1024 and code == vc.VC_OK and torch.equal(out, want))
    for _ in range(3):
        vc.vc_linear_fp8(p, x, xs, w, ws, None, out, work)
        vc.vc_poll_status(work)
        assert torch.equal(out, want)


@pytest.mark.parametrize("M", [5, 50, 200, 2500])
def test_rows_of_wider_matrices_and_neighbours(M):
    N, K = 2500, 160
    x, xs, w, ws = _operands(M, N, K, 5)
    wide_x, wide_w = np.full((M, K + 32), 0x7f, np.uint8), np.full((N, K + 48), 0x7f, np.uint8)      # NaN codes around
    wide_x[:, 16:16 + K], wide_w[:, 16:16 + K] = x, w
    room = torch.full((M + 2, N + 11), 7.0, dtype=torch.float32, device="cuda")
    for pad in (4, 8):
        out = room[1:M + 1, pad:pad + N] if pad == 4 else torch.full((M + 2, N + 12), 7.0, device="cuda")[1:M + 1, 4:4 + N]
        if out.data_ptr() % 16:
            continue
        _run(_dev(wide_x)[:, 16:16 + K], _dev(xs), _dev(wide_w)[:, 16:16 + K], _dev(ws), "fp32", None, out)
        _close(out, x, xs, w, ws, "fp32")
    assert (room[0] == 7).all() and (room[M + 1] == 7).all()


@pytest.mark.parametrize("pitch", ["rows on 16 bytes", "odd rows"])
@pytest.mark.parametrize("dt", ["bf16", "fp32"])
@pytest.mark.parametrize("splits", [1, 3, 9])
@pytest.mark.parametrize("M,N", [(1, 2500), (5, 2500), (50, 2499), (64, 130), (65, 2500), (200, 2499), (1301, 1801), (2500, 2500), (5000, 2003)])
def test_what_lies_around_the_output_and_the_workspace_stays(M, N, splits, dt, pitch):
    """Rows in front and behind, columns on both sides and the bytes around the workspace, for every shape of tile and way of joining parts."""
    K, edge = 1168, 8 if dt == "bf16" else 4                        # ten blocks; elements of 16 bytes
    x, xs, w, ws = _operands(M, N, K, 15)
    wide = (N + 3 * edge) // edge * edge if pitch != "odd rows" else N + 2 * edge + 1 + N % 2
    room = torch.full((M + 2 * edge, wide), -7.0, dtype=DT[dt], device="cuda")
    out = room[edge:edge + M, edge:edge + N]
    assert out.data_ptr() % 16 == 0 and (wide % edge == 0) == (pitch != "odd rows")
    p = vc.LinearParams.of(_dev(x), _dev(w), out, None, k_splits=splits)
    need = vc.vc_linear_workspace_bytes(p)
    work = torch.full((need + 1024,), 0xa5, dtype=torch.uint8, device="cuda")
    vc.vc_linear_fp8(p, _dev(x), _dev(xs), _dev(w), _dev(ws), None, out, work[512:512 + need])
    vc.vc_poll_status(work[512:512 + need])
    _close(out, x, xs, w, ws, dt)
    out.fill_(-7.0)
    assert (room == -7.0).all()
    assert (work[:512] == 0xa5).all() and (work[512 + need:] == 0xa5).all()


def test_scales_far_apart_and_zero():
    x, xs, w, ws = _operands(90, 140, 1024, 8, spread=6.0)
    xs[3], ws[0, 5] = 0.0, 0.0
    _close(_run(_dev(x), _dev(xs), _dev(w), _dev(ws), "fp32"), x, xs, w, ws, "fp32")


@pytest.mark.parametrize("M", [4, 200])
def test_nan_and_infinite_scales_stay_in_their_rows(M):
    x, xs, w, ws = _operands(M, 150, 512, 9)
    xs[1, 2] = np.nan
    x[3, 200] = 0x7f
    out = _run(_dev(x), _dev(xs), _dev(w), _dev(ws), "fp32").cpu()
    bad = torch.zeros(M, dtype=torch.bool)
    bad[2] = bad[3] = True
    assert torch.isnan(out[bad]).all() and torch.isfinite(out[~bad]).all()


@pytest.mark.parametrize("M,N,splits", [(4, 150, 0), (50, 150, 3), (200, 300, 0), (200, 300, 4), (1301, 1801, 0)])
def test_infinite_scales_make_infinities_and_nan_where_the_formula_does(M, N, splits):
    """A sum over blocks with one that is infinite: the sign of that block's product, NaN where two of them disagree or the product is 0."""
    K = 512
    x, xs, w, ws = _operands(M, N, K, 16)
    xs[1, 2], ws[1, 3] = np.inf, np.inf
    x[3, 128:256] = 0                                               # (a product of 0 under a finite scale: nothing)
    x[2, 300:] = 0
    xs[0, 3] = np.inf
    x[3, :128] = 0                                                  # under an infinite one: NaN
    out = _run(_dev(x), _dev(xs), _dev(w), _dev(ws), "fp32", k_splits=splits).double().cpu().numpy()
    val, want, sure = L.e4m3_values(), np.zeros((M, N)), np.ones((M, N), bool)
    with np.errstate(invalid="ignore"):
        for kb in range(K // 128):
            part = slice(128 * kb, 128 * kb + 128)
            a, b = val[x[:, part]], val[w[:, part]]
            S, size = a @ b.T, np.abs(a) @ np.abs(b).T
            f = xs[kb][:, None].astype(np.float64) * np.repeat(ws[:, kb].astype(np.float64), 128)[None, :N]
            want += f * S
            sure &= np.isfinite(f) | (size == 0) | (np.abs(S) > 132 * 2.0 ** -24 * size)      # (else its sign is a matter of rounding)
    odd = ~np.isfinite(want)
    assert odd[2].all() and np.isnan(want[3]).all() and odd[:, 128:256].all() and odd.sum() == 2 * N + (M - 2) * min(N - 128, 128)
    assert sure.mean() > 0.99 and not np.isfinite(out[odd]).any() and np.isfinite(out[~odd]).all()
    assert np.array_equal(out[odd & sure], want[odd & sure], equal_nan=True)
    keep = ~odd.any(axis=1)
    assert not keep.any()
    few = [m for m in range(M) if m not in (2, 3)]
    _close(torch.from_numpy(out[few][:, :128]), x[few], xs[:, few], w[:128], ws[:1], "fp32")


@pytest.mark.parametrize("bad", [float("inf"), float("-inf"), float("nan")])
@pytest.mark.parametrize("M", [4, 300])
def test_quantised_infinities_and_nan_become_nan(M, bad):
    """The blocks that hold one stand for NaN throughout: their row of y, and the 128 columns of their weights."""
    g = torch.Generator().manual_seed(17)
    x, w = torch.randn(M, 400, generator=g).cuda(), torch.randn(300, 400, generator=g).cuda()
    x[1, 390], w[140, 5] = bad, bad
    args = []
    for t, rows in ((x, 1), (w, 128)):
        codes = torch.empty(t.shape, dtype=torch.float8_e4m3fn, device="cuda")
        scale = torch.empty((4, M) if rows == 1 else (3, 4), device="cuda")
        vc.vc_quant_fp8(vc.QuantParams.of(t, rows), t, codes, scale)
        args += [codes, scale]
    out = _run(*args, "fp32").cpu()
    bad = torch.zeros(M, 300, dtype=torch.bool)
    bad[1], bad[:, 128:256] = True, True
    assert torch.isnan(out[bad]).all() and torch.isfinite(out[~bad]).all()


@pytest.mark.parametrize("M,N,splits", [(1, 300, 0), (7, 300, 3), (50, 300, 9), (200, 300, 0), (1301, 1801, 0)])
@pytest.mark.parametrize("x_exp,w_exp,dim", [(-61, -61, False), (-22, -100, False), (-100, -22, False), (-120, -2, False), (61, 61, True), (118, 4, True)])
def test_products_of_scales_near_the_ends_of_the_range_of_fp32(M, N, splits, x_exp, w_exp, dim):
    """x_scale * w_scale from 2^-126 and up to 2^127, as far as they are to be used: no bits are lost on the way."""
    K = 1168
    x, xs, w, ws = _operands(M, N, K, 18, spread=0.3)
    if dim:
        x, w = (c & 0x83 for c in (x, w))                           # magnitudes below 2^-6: products below 2^-12, sums of ten blocks below 2^-2
        x[x & 127 == 0] |= 1
    xs, ws = np.ldexp(xs, x_exp).astype(np.float32), np.ldexp(ws, w_exp).astype(np.float32)
    f = [t.astype(np.float64) for t in (xs, ws)]
    assert all(2.0 ** -126 <= f[0][kb].min() * f[1][:, kb].min() and f[0][kb].max() * f[1][:, kb].max() < 2.0 ** 127 for kb in range(K // 128 + 1))
    out = _run(_dev(x), _dev(xs), _dev(w), _dev(ws), "fp32", k_splits=splits).cpu().double().numpy()
    want, size = L.linear_fp8(x, xs, w, ws)
    assert np.isfinite(want).all() and 2.0 ** -126 < np.median(np.abs(want)) and np.abs(want).max() < 2.0 ** 128
    # as above; and each block's term, and each of their sums, may lie on the grid of the subnormals: half a step of 2^-149 each
    tol = (132 + 10 + 8) * 2.0 ** -24 * size + 2.0 ** -24 * np.abs(want) + 20 * 2.0 ** -150
    assert (np.abs(out - want) <= tol).all(), np.nanmax(np.abs(out - want) / tol)


def test_codes_as_quantised_and_as_float8_tensors():
    """Quantised by the library and multiplied: the product of what the codes stand for."""
    g = torch.Generator().manual_seed(10)
    x, w = torch.randn(70, 400, generator=g).to(torch.bfloat16).cuda(), torch.randn(200, 400, generator=g).cuda()
    out = []
    for t, rows in ((x, 1), (w, 128)):
        codes = torch.empty(t.shape, dtype=torch.float8_e4m3fn, device="cuda")
        scale = torch.empty((4, 70) if rows == 1 else (2, 4), device="cuda")
        vc.vc_quant_fp8(vc.QuantParams.of(t, rows), t, codes, scale)
        out += [codes, scale]
    y = _run(*out, "fp32")
    c = [t.view(torch.uint8).cpu().numpy() if t.dtype == torch.float8_e4m3fn else t.cpu().numpy() for t in out]
    _close(y, *c, "fp32")
    # two roundings of at most 2^-4 relative (or half the least step of a block, 2^-10 of 448) each
    ref, size = x.double() @ w.double().t(), x.double().abs() @ w.double().abs().t()
    assert ((y.double() - ref).abs() <= 0.13 * size + 1.0).all()


@pytest.mark.parametrize("M", [3, 300])
def test_same_answer_other_stream_and_captured(M):
    x, xs, w, ws = (_dev(t) for t in _operands(M, 400, 4096, 11))
    want = _run(x, xs, w, ws, "bf16")
    assert torch.equal(_run(x, xs, w, ws, "bf16"), want)
    out = torch.empty_like(want)
    p = vc.LinearParams.of(x, w, out)
    work = torch.empty(vc.vc_linear_workspace_bytes(p), dtype=torch.uint8, device="cuda")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        vc.vc_linear_fp8(p, x, xs, w, ws, None, out, work)
        vc.vc_poll_status(work)
    assert torch.equal(out, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        vc.vc_linear_fp8(p, x, xs, w, ws, None, out, work)
    xs.mul_(2.0)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, _run(x, xs, w, ws, "bf16"))


@pytest.mark.parametrize("M,N", [(3, 400), (40, 400), (300, 400), (2500, 2560)])
@pytest.mark.parametrize("K", [1024, 16384])
def test_wait_that_runs_out_is_reported_and_leaves_the_library_usable(M, N, K):
    """With a limit of one poll a wait gives up unless what it waits for is there already.  At a few blocks of K, all copied in front of
    the first wait, that can be so for every wait: then the answer is the right one.  At 128 blocks some wait gives up."""
    x, xs, w, ws = (_dev(t) for t in _operands(M, N, K, 12))
    want = _run(x, xs, w, ws, "bf16")
    out = torch.empty_like(want)
    p = vc.LinearParams.of(x, w, out)
    work = torch.empty(vc.vc_linear_workspace_bytes(p), dtype=torch.uint8, device="cuda")
    code = vc.VC_OK
    try:
        vc.vc_test_set_wait_limit(1)
        vc.vc_linear_fp8(p, x, xs, w, ws, None, out, work)
        vc.vc_poll_status(work)
    except vc.VcError as e:
        code = e.code
    finally:
        vc.vc_test_set_wait_limit(0)
    assert code == vc.VC_ERR_TIMEOUT or (K == 1024 and code == vc.VC_OK and torch.equal(out, want))
    vc.vc_poll_status(work)
    vc.vc_linear_fp8(p, x, xs, w, ws, None, out, work)
    vc.vc_poll_status(work)
    assert torch.equal(out, want)
