"""vc_cross_attn against attention in 64 bits.

Tolerance per output, with u = eps / 2 of the type, w the row's weights and A = sum w |v|:
  u |o|                    the rounding of the output
  u A                      the rounding of each probability (the row sum takes them unrounded)
  2 D A                    the scores: a chain of d FP32 additions, D = (d + 8) 2^-24 scale max_j sum_c |q_c k_jc| as an error of the
                           exponent, in the weights above and in the sum below, plus its product with log2(e) and the reference (|x| 2^-23)
  2^-19 A                  ex2.approx (2^-22), 16 additions of 128 / 16 values, the division; rescales by the same
  fp16: 2^-24 sum |v|      probabilities below the type's normal numbers (the largest one is 1 or more)
"""
import numpy as np
import pytest
import torch

import paper_2609_15810_b200 as vc
from oracle import layer as L

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "fp16": torch.float16}


def _heads(B, H, N, d, dt, g, token_major=False, scale=1.0):
    x = (torch.randn((B, N, H, d) if token_major else (B, H, N, d), generator=g) * scale).to(DT[dt]).cuda()
    return x.transpose(1, 2) if token_major else x


def _call(q, k, v, kv_len=None, mask=None, lse=True, o=None, work=None, **kw):
    o = torch.full(q.shape, float("nan"), dtype=q.dtype, device="cuda") if o is None else o
    out_lse = torch.full(q.shape[:3], float("nan"), device="cuda") if lse else None
    p = vc.CrossParams.of(q, k, v, o, **kw)
    work = torch.full((vc.vc_cross_workspace_bytes(p),), 0xff, dtype=torch.uint8, device="cuda") if work is None else work
    vc.vc_cross_attn(p, q, k, v, kv_len, mask, o, out_lse, work)
    vc.vc_poll_status(work)
    return o, out_lse


def _check(q, k, v, o, lse, kv_len=None, mask=None, scale=0.0):
    d = q.shape[3]
    scale = scale or d ** -0.5
    lens = None if kv_len is None else np.clip(kv_len.cpu().numpy(), 0, k.shape[2])
    m = None if mask is None else mask.cpu().numpy()
    keep = np.ones((q.shape[0], k.shape[2]), bool)
    if lens is not None:
        keep &= np.arange(k.shape[2])[None] < lens[:, None]
    if m is not None:
        keep &= m != 0
    at = keep[:, None, :, None]
    q64, k64, v64 = (t.double().cpu().numpy() for t in (q, k, v))
    k64, v64 = np.where(at, k64, 0.0), np.where(at, v64, 0.0)       # what masked places hold is nothing to the oracle either
    want, want_lse = L.cross_attention(q64, k64, v64, scale, lens, m)
    A, _ = L.cross_attention(q64, k64, np.abs(v64), scale, lens, m)
    G = q.shape[1] // k.shape[1]
    rep = lambda t: np.repeat(t, G, axis=1)
    size = scale * np.einsum("bhnc,bhjc->bhnj", np.abs(q64), rep(np.abs(k64))).max(axis=3, initial=0.0)[..., None]
    D = (d + 8 + 4) * 2.0 ** -24 * size
    u = torch.finfo(q.dtype).eps / 2
    tol = u * np.abs(want) + (u + 2 * D + 2.0 ** -19) * A
    if q.dtype == torch.float16:
        tol = tol + 2.0 ** -24 * rep(np.abs(v64)).sum(axis=2, keepdims=True) + 2.0 ** -25
    err = np.abs(o.double().cpu().numpy() - want)
    assert np.isfinite(err).all() and (err <= tol).all(), f"{(~(err <= tol)).sum()} of {err.size} off, worst {np.nanmax(err / np.maximum(tol, 1e-300)):.2f}"
    if lse is not None:
        got = lse.double().cpu().numpy()
        none = np.isneginf(want_lse)
        assert np.array_equal(np.isneginf(got), none)
        got, want_lse, D = got[~none], want_lse[~none], np.broadcast_to(D[..., 0], none.shape)[~none]
        assert (np.abs(got - want_lse) <= D + 2.0 ** -19 + 2.0 ** -22 * np.abs(want_lse)).all()


@pytest.mark.parametrize("dt", ["bf16", "fp16"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("Nq,Nkv", [(1, 1), (1, 128), (128, 128), (129, 129), (127, 257), (300, 512), (257, 77), (5, 1000), (640, 640)])
def test_lengths(dt, d, Nq, Nkv):
    g = torch.Generator().manual_seed(Nq * 10007 + Nkv + d)
    q, k, v = _heads(2, 3, Nq, d, dt, g, scale=2.0), _heads(2, 3, Nkv, d, dt, g), _heads(2, 3, Nkv, d, dt, g)
    o, lse = _call(q, k, v)
    _check(q, k, v, o, lse)


@pytest.mark.parametrize("dt", ["bf16", "fp16"])
@pytest.mark.parametrize("B,H,Hkv,Nq,Nkv", [(3, 6, 2, 195, 257), (1, 40, 40, 700, 512), (2, 16, 1, 33, 300), (4, 60, 20, 513, 130)])
def test_pairs_of_tiles_and_shared_heads(dt, B, H, Hkv, Nq, Nkv):
    """Many heads: items are pairs of query tiles, some pairs without their second one."""
    g = torch.Generator().manual_seed(B + H + Nq)
    q, k, v = _heads(B, H, Nq, 64, dt, g, True, 2.0), _heads(B, Hkv, Nkv, 64, dt, g, True), _heads(B, Hkv, Nkv, 64, dt, g)
    o, lse = _call(q, k, v)
    _check(q, k, v, o, lse)


@pytest.mark.parametrize("splits", [0, 1, 2, 3, 7, 64])
@pytest.mark.parametrize("d", [64, 128])
def test_keys_split_between_ctas(splits, d):
    g = torch.Generator().manual_seed(splits + d)
    q, k, v = _heads(2, 2, 140, d, "bf16", g, scale=3.0), _heads(2, 1, 1500, d, "bf16", g), _heads(2, 1, 1500, d, "bf16", g)
    lens = torch.tensor([1500, 130], dtype=torch.int32, device="cuda")
    o, lse = _call(q, k, v, lens, key_splits=splits)
    _check(q, k, v, o, lse, lens)


@pytest.mark.parametrize("dt,d", [("bf16", 128), ("fp16", 64)])
@pytest.mark.parametrize("H,Nq", [(16, 1), (40, 100), (40, 128)])
def test_heads_of_one_query_tile(dt, d, H, Nq):
    """More heads than SMs, a query tile each: several items a CTA, of no, one, an odd and an even number of key tiles."""
    B, N = 16, 600
    g = torch.Generator().manual_seed(H + Nq)
    q, k, v = _heads(B, H, Nq, d, dt, g, True, 2.0), _heads(B, 8, N, d, dt, g, True), _heads(B, 8, N, d, dt, g, True)
    lens = torch.tensor([600, 0, 128, 1, 129, 300, 600, 257, 0, 0, 513, 384, 127, 130, 600, 256], dtype=torch.int32, device="cuda")
    mask = torch.rand(B, N, generator=g) < 0.7
    mask[3] = mask[6, :128] = mask[11, 128:256] = False
    o, lse = _call(q, k, v)
    _check(q, k, v, o, lse)
    o, lse = _call(q, k, v, lens)
    _check(q, k, v, o, lse, lens)
    o, lse = _call(q, k, v, lens, mask.cuda())
    _check(q, k, v, o, lse, lens, mask.cuda())


@pytest.mark.parametrize("dt,d", [("bf16", 128), ("fp16", 64)])
@pytest.mark.parametrize("splits", [2, 3, 7, 8, 9])
@pytest.mark.parametrize("Nq", [1, 64, 100, 129])
def test_parts_joined_by_a_cluster_and_by_a_launch(dt, d, splits, Nq):
    """Parts without a key, rows whose keys are all masked."""
    B, H, N = 2, 4, 1300
    g = torch.Generator().manual_seed(splits + Nq + d)
    q, k, v = _heads(B, H, Nq, d, dt, g, True, 2.0), _heads(B, 2, N, d, dt, g, True), _heads(B, 2, N, d, dt, g, True)
    lens = torch.tensor([1300, 400], dtype=torch.int32, device="cuda")
    mask = torch.rand(B, N, generator=g) < 0.6
    mask[1, :256] = False
    for a in ((), (lens,), (lens, mask.cuda()), (None, torch.zeros_like(mask).cuda())):
        o, lse = _call(q, k, v, *a, key_splits=splits)
        _check(q, k, v, o, lse, *a)


def test_nan_of_one_part_reaches_the_row():
    g = torch.Generator().manual_seed(31)
    q, k, v = _heads(1, 2, 3, 128, "bf16", g), _heads(1, 2, 1000, 128, "bf16", g), _heads(1, 2, 1000, 128, "bf16", g)
    q[0, 1, 2, 5] = float("nan")
    for splits in (1, 4):
        o, lse = _call(q, k, v, key_splits=splits)
        bad = torch.isnan(o).all(-1)
        assert bad[0, 1, 2] and bad.sum() == 1 and torch.isfinite(o[~bad]).all() and torch.isnan(lse).sum() == 1


@pytest.mark.parametrize("splits", [5, 6, 12])
@pytest.mark.parametrize("Nq", [1, 200])
def test_many_parts_of_keys(splits, Nq):
    """Few heads, and more parts of their keys than SMs: several a CTA, of no, one, two and three key tiles."""
    B, H, N = 4, 9, 1500
    g = torch.Generator().manual_seed(splits + Nq)
    q, k, v = _heads(B, H, Nq, 128, "bf16", g, scale=2.0), _heads(B, 3, N, 128, "bf16", g), _heads(B, 3, N, 128, "bf16", g)
    lens = torch.tensor([1500, 700, 0, 1290], dtype=torch.int32, device="cuda")
    o, lse = _call(q, k, v, key_splits=splits)
    _check(q, k, v, o, lse)
    o, lse = _call(q, k, v, lens, key_splits=splits)
    _check(q, k, v, o, lse, lens)


@pytest.mark.parametrize("lens", [[0, 1, 127, 128], [129, 0, 400, 256], [-5, 500, 399, 2], [0, 0, 0, 0]])
@pytest.mark.parametrize("splits", [1, 2])
def test_lengths_per_batch(lens, splits):
    """Lengths outside [0, N_kv] are clamped; a batch of length 0 gives rows of 0 and -infinity."""
    g = torch.Generator().manual_seed(sum(lens) + 11)
    q, k, v = _heads(4, 3, 200, 128, "bf16", g, scale=2.0), _heads(4, 3, 400, 128, "bf16", g), _heads(4, 3, 400, 128, "bf16", g)
    kv = torch.tensor(lens, dtype=torch.int32, device="cuda")
    o, lse = _call(q, k, v, kv, key_splits=splits)
    _check(q, k, v, o, lse, kv)
    empty = torch.tensor([n <= 0 for n in lens])
    assert (o.cpu()[empty] == 0).all() and torch.isneginf(lse.cpu()[empty]).all()


@pytest.mark.parametrize("dt", ["bf16", "fp16"])
@pytest.mark.parametrize("kind", ["random", "one", "first tiles", "last tiles", "none"])
def test_masks(dt, kind):
    g = torch.Generator().manual_seed(21)
    B, N = 2, 389
    q, k, v = _heads(B, 4, 150, 64, dt, g, scale=2.0), _heads(B, 2, N, 64, dt, g), _heads(B, 2, N, 64, dt, g)
    mask = torch.zeros(B, N, dtype=torch.bool)
    if kind == "random":
        mask = torch.rand(B, N, generator=g) < 0.3
    elif kind == "one":
        mask[0, 200] = mask[1, 388] = True
    elif kind == "first tiles":
        mask[:, :100] = True
    elif kind == "last tiles":
        mask[:, 300:] = True                                  # two whole tiles without a key before the first one kept
    lens = torch.tensor([N, 350], dtype=torch.int32, device="cuda")
    for kv in (None, lens):
        o, lse = _call(q, k, v, kv, mask.cuda())
        _check(q, k, v, o, lse, kv, mask)
    o8, _ = _call(q, k, v, lens, mask.to(torch.uint8).cuda() * 255)
    assert torch.equal(o, o8)


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
def test_what_masked_places_hold_is_not_used(bad):
    g = torch.Generator().manual_seed(22)
    q, k, v = _heads(2, 2, 130, 128, "bf16", g, scale=2.0), _heads(2, 2, 300, 128, "bf16", g), _heads(2, 2, 300, 128, "bf16", g)
    lens = torch.tensor([200, 300], dtype=torch.int32, device="cuda")
    mask = torch.ones(2, 300, dtype=torch.bool, device="cuda")
    mask[1, 17] = mask[1, 250:] = False
    clean, _ = _call(q, k, v, lens, mask)
    k[0, :, 200:], v[0, :, 200:], k[1, :, 17], v[1, :, 17], k[1, :, 250:], v[1, :, 250:] = (bad,) * 6
    for splits in (1, 2):
        o, lse = _call(q, k, v, lens, mask, key_splits=splits)
        assert torch.isfinite(lse).all()
        _check(q, k, v, o, lse, lens, mask)
    o, _ = _call(q, k, v, lens, mask, key_splits=1)
    assert torch.equal(o, clean)


def test_nan_in_a_kept_key_reaches_its_rows():
    g = torch.Generator().manual_seed(23)
    q, k, v = _heads(2, 1, 10, 64, "bf16", g), _heads(2, 1, 50, 64, "bf16", g), _heads(2, 1, 50, 64, "bf16", g)
    k[1, 0, 3, 5] = float("nan")
    for splits in (0, 1):
        o, lse = _call(q, k, v, key_splits=splits)
        assert torch.isfinite(o[0]).all() and torch.isnan(o[1]).all() and torch.isnan(lse[1]).all()


def test_reference_far_below_later_scores():
    """Scores that grow by hundreds from tile to tile: every tile rescales; and the other way round, none does."""
    g = torch.Generator().manual_seed(24)
    q, k, v = _heads(1, 2, 200, 64, "bf16", g), _heads(1, 2, 640, 64, "bf16", g), _heads(1, 2, 640, 64, "bf16", g)
    q[..., 0] = 8.0
    for ramp in (torch.arange(640.0) // 128 * 40.0, -(torch.arange(640.0) // 128) * 40.0, (torch.arange(640.0) % 7) * 6.0):
        k[..., 0] = ramp.to(torch.bfloat16).cuda()
        o, lse = _call(q, k, v)
        _check(q, k, v, o, lse)


def test_scale():
    g = torch.Generator().manual_seed(25)
    q, k, v = _heads(1, 2, 60, 128, "fp16", g), _heads(1, 2, 90, 128, "fp16", g), _heads(1, 2, 90, 128, "fp16", g)
    o, lse = _call(q, k, v, softmax_scale=0.31)
    _check(q, k, v, o, lse, scale=0.31)


def test_no_keys_at_all():
    q = torch.randn(1, 2, 150, 64, device="cuda").bfloat16()
    k = torch.empty(1, 2, 0, 64, device="cuda", dtype=torch.bfloat16)
    o, lse = _call(q, k, k)
    assert (o == 0).all() and torch.isneginf(lse).all()


@pytest.mark.parametrize("mask_type", [torch.bool, torch.uint8])
def test_no_keys_under_a_mask_and_lengths(mask_type):
    q = torch.randn(3, 4, 150, 64, device="cuda").bfloat16()
    k = torch.empty(3, 0, 2, 64, device="cuda", dtype=torch.bfloat16).transpose(1, 2)
    o, lse = _call(q, k, k, torch.tensor([0, 3, -1], dtype=torch.int32, device="cuda"), torch.empty(3, 0, dtype=mask_type, device="cuda"))
    assert (o == 0).all() and torch.isneginf(lse).all()


def test_layouts_views_and_neighbours():
    """Queries and outputs inside [B, N, H, d] memory, keys and values two halves of one projection; what lies around the output stays."""
    g = torch.Generator().manual_seed(26)
    B, H, N, M, d = 2, 3, 140, 90, 64
    kv = torch.randn(B, M, 2, H, d, generator=g).to(torch.float16).cuda()
    q = _heads(B, H, N, d, "fp16", g, True)
    room = torch.full((B, N + 2, H, d + 8), 7.0, dtype=torch.float16, device="cuda")
    o = room[:, 1:N + 1, :, :d].transpose(1, 2)
    k, v = kv[:, :, 0].transpose(1, 2), kv[:, :, 1].transpose(1, 2)
    for splits in (1, 2):
        _, lse = _call(q, k, v, o=o, key_splits=splits)
        _check(q, k, v, o, lse)
        assert (room[:, 0] == 7).all() and (room[:, N + 1] == 7).all() and (room[..., d:] == 7).all()


@pytest.mark.parametrize("dt,d", [("bf16", 128), ("fp16", 64)])
@pytest.mark.parametrize("B,H,Hkv,Nq,Nkv,splits", [(2, 45, 45, 300, 130, 1), (2, 45, 9, 300, 300, 2), (2, 3, 1, 129, 700, 1), (1, 4, 2, 5, 4096, 0), (1, 4, 2, 100, 2048, 4),
                                                   (1, 2, 2, 131, 1300, 9), (2, 2, 2, 1, 0, 0)])
def test_what_lies_around_the_outputs_and_the_workspace_stays(dt, d, B, H, Hkv, Nq, Nkv, splits):
    """One and two query tiles an item, parts joined by a cluster and by a launch, no keys; a batch without any."""
    g = torch.Generator().manual_seed(Nq + Nkv)
    q, k, v = _heads(B, H, Nq, d, dt, g), _heads(B, Hkv, Nkv, d, dt, g), _heads(B, Hkv, Nkv, d, dt, g)
    lens = torch.tensor([Nkv, 0][:B], dtype=torch.int32, device="cuda")
    room = torch.full((B + 2, Nq + 2, H + 2, d + 8), 7.0, dtype=DT[dt], device="cuda")
    o = room[1:B + 1, 1:Nq + 1, 1:H + 1, :d].transpose(1, 2)
    lse = torch.full((B * H * Nq + 8,), 7.0, device="cuda")
    p = vc.CrossParams.of(q, k, v, o, key_splits=splits)
    need = vc.vc_cross_workspace_bytes(p)
    work = torch.full((need + 1024,), 0xa5, dtype=torch.uint8, device="cuda")
    mine = lse[4:-4].view(B, H, Nq)
    vc.vc_cross_attn(p, q, k, v, lens, None, o, mine, work[512:512 + need])
    vc.vc_poll_status(work[512:512 + need])
    _check(q, k, v, o, mine, lens)
    o.fill_(7.0)
    assert (room == 7).all() and (lse[:4] == 7).all() and (lse[-4:] == 7).all()
    assert (work[:512] == 0xa5).all() and (work[512 + need:] == 0xa5).all()


def test_broadcast_keys_and_queries():
    g = torch.Generator().manual_seed(27)
    q1, k1, v1 = _heads(1, 1, 70, 64, "bf16", g), _heads(1, 2, 200, 64, "bf16", g), _heads(3, 1, 200, 64, "bf16", g)
    q, k, v = q1.expand(3, 4, 70, 64), k1.expand(3, 2, 200, 64), v1.expand(3, 2, 200, 64)
    o = torch.empty(3, 4, 70, 64, dtype=torch.bfloat16, device="cuda")
    o, lse = _call(q, k, v, o=o)
    _check(q, k, v, o, lse)


def test_offsets_beyond_32_bits():
    """Batches 2.4 billion elements apart in every tensor."""
    B, H, N, d, gap = 2, 1, 130, 64, 2400000000
    g = torch.Generator().manual_seed(28)
    room = torch.empty(gap + 4 * H * N * d, dtype=torch.bfloat16, device="cuda")
    at = lambda i: room.as_strided((B, H, N, d), (gap, N * d, d, 1), i * H * N * d)
    q, k, v, o = (at(i) for i in range(4))
    for t in (q, k, v):
        t.copy_(torch.randn(B, H, N, d, generator=g))
    _, lse = _call(q, k, v, o=o)
    _check(q, k, v, o, lse)


def test_same_answer_every_time_other_stream_and_captured():
    g = torch.Generator().manual_seed(29)
    q, k, v = _heads(2, 4, 300, 128, "bf16", g, scale=2.0), _heads(2, 4, 1100, 128, "bf16", g), _heads(2, 4, 1100, 128, "bf16", g)
    lens = torch.tensor([1100, 700], dtype=torch.int32, device="cuda")
    want, _ = _call(q, k, v, lens, key_splits=3)
    for _ in range(3):
        assert torch.equal(_call(q, k, v, lens, key_splits=3)[0], want)
    o = torch.empty_like(want)
    p = vc.CrossParams.of(q, k, v, o, key_splits=3)
    work = torch.empty(vc.vc_cross_workspace_bytes(p), dtype=torch.uint8, device="cuda")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        vc.vc_cross_attn(p, q, k, v, lens, None, o, None, work)
        vc.vc_poll_status(work)
    assert torch.equal(o, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        vc.vc_cross_attn(p, q, k, v, lens, None, o, None, work)
    lens.copy_(torch.tensor([1, 1099], dtype=torch.int32))
    q.mul_(0.5)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(o, _call(q, k, v, lens, key_splits=3)[0])


@pytest.mark.parametrize("splits", [1, 2])
def test_wait_that_runs_out_is_reported_and_leaves_the_library_usable(splits):
    g = torch.Generator().manual_seed(30)
    q, k, v = _heads(2, 4, 600, 128, "bf16", g), _heads(2, 4, 500, 128, "bf16", g), _heads(2, 4, 500, 128, "bf16", g)
    o = torch.empty_like(q)
    p = vc.CrossParams.of(q, k, v, o, key_splits=splits)
    work = torch.empty(vc.vc_cross_workspace_bytes(p), dtype=torch.uint8, device="cuda")
    lens = torch.tensor([500, 400], dtype=torch.int32, device="cuda")
    vc.vc_cross_attn(p, q, k, v, lens, None, o, None, work)
    vc.vc_poll_status(work)
    before = o.clone()
    try:
        vc.vc_test_set_wait_limit(1)
        vc.vc_cross_attn(p, q, k, v, lens, None, o, None, work)
        with pytest.raises(vc.VcError) as e:
            vc.vc_poll_status(work)
        assert e.value.code == vc.VC_ERR_TIMEOUT
    finally:
        vc.vc_test_set_wait_limit(0)
    vc.vc_poll_status(work)
    o.zero_()
    vc.vc_cross_attn(p, q, k, v, lens, None, o, None, work)
    vc.vc_poll_status(work)
    assert torch.equal(o, before)
