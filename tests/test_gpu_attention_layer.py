"""A video-DiT block's attention as a program runs it, every step through the library: E4M3 projection to Q, K and V, norm and rotation
inside the projection's output, quantized self-attention, E4M3 output projection; then the same with an encoder's states.

Every stage is compared with the oracle's form of it on what the stage in front of it really wrote, so each tolerance is the
stage's own.
"""
import numpy as np
import pytest
import torch

import paper_2609_15810_b200 as vc
from oracle import attention as OA
from oracle import compare as CMP
from oracle import layer as L
from oracle import prep as OP
from paper_2609_15810_b200.binding import Params, alloc_buffers

pytestmark = pytest.mark.gpu

B, H, d, GRID, TEXT = 2, 3, 128, (3, 7, 11), 77
N, DIM = GRID[0] * GRID[1] * GRID[2], H * d
BF = torch.bfloat16


def _np(t):
    return t.double().cpu().numpy()


class Weights:
    def __init__(self, n, k, g):
        w = (torch.randn(n, k, generator=g) / k ** 0.5).cuda()
        self.codes = torch.empty(n, k, dtype=torch.float8_e4m3fn, device="cuda")
        self.scale = torch.empty((n + 127) // 128, (k + 127) // 128, device="cuda")
        self.bias = (0.1 * torch.randn(n, generator=g)).to(BF).cuda()
        vc.vc_quant_fp8(vc.QuantParams.of(w, 128), w, self.codes, self.scale)


def _project(x, w):
    """x [B, H, N, d] or [rows, width] -> [rows, n] bf16, and the check of both steps."""
    p = vc.QuantParams.of(x)
    rows, k = p.B * p.N, p.H * p.d
    codes, scale = torch.empty(rows, k, dtype=torch.uint8, device="cuda"), torch.empty((k + 127) // 128, rows, device="cuda")
    vc.vc_quant_fp8(p, x, codes, scale)
    out = torch.empty(rows, w.codes.shape[0], dtype=BF, device="cuda")
    pl = vc.LinearParams.of(codes, w.codes, out, w.bias)
    work = torch.empty(vc.vc_linear_workspace_bytes(pl), dtype=torch.uint8, device="cuda")
    vc.vc_linear_fp8(pl, codes, scale, w.codes, w.scale, w.bias, out, work)
    vc.vc_poll_status(work)
    m = x.float().cpu().numpy() if x.dim() == 2 else x.float().cpu().transpose(1, 2).reshape(rows, k).numpy()
    want_c, want_s = L.quant_fp8(m, 1)
    assert np.array_equal(codes.cpu().numpy(), want_c) and np.array_equal(scale.t().cpu().numpy(), want_s)
    y, size = L.linear_fp8(want_c, want_s.T, w.codes.view(torch.uint8).cpu().numpy(), w.scale.cpu().numpy(), _np(w.bias))
    assert (np.abs(_np(out) - y) <= 2.0 ** -8 * np.abs(y) + (140 + want_s.shape[1]) * 2.0 ** -24 * size).all()
    return out


def _norm(q, k, q_out, k_out, wq, wk, layout, grid):
    want = [None if t is None else L.qk_norm_rope(_np(t), _np(w), "token", 1e-6, layout, L.default_dims(d), L.positions_of(grid),
                                                  [L.frequencies(n) for n in L.default_dims(d)]) for t, w in ((q, wq), (k, wk))]
    rot = {None: vc.VC_ROTARY_NONE, L.INTERLEAVED: vc.VC_ROTARY_INTERLEAVED}[layout]
    p = vc.QkParams.of(q, k, q_out, k_out, grid=grid, weight=wq if wq is not None else wk, norm=vc.VC_NORM_TOKEN, rotary=rot)
    vc.vc_qk_norm_rope(p, q, k, wq, wk, None, q_out, k_out)
    for t, w in zip((q_out, k_out), want):
        if t is not None:
            assert (np.abs(_np(t) - w[0]) <= 2.0 ** -8 * np.abs(w[0]) + 64 * 2.0 ** -24 * w[1]).all()


@pytest.mark.parametrize("bits", [8, 4])
def test_block(bits):
    g = torch.Generator().manual_seed(40)
    norm_w = [(1.0 + 0.1 * torch.randn(DIM, generator=g)).to(BF).cuda() for _ in range(4)]
    qkv_w, out_w, q_w, kv_w, out2_w = (Weights(n, DIM, g) for n in (3 * DIM, DIM, DIM, 2 * DIM, DIM))
    x = torch.randn(B * N, DIM, generator=g).to(BF).cuda()
    text = torch.randn(B * TEXT, DIM, generator=g).to(BF).cuda()

    # ---- self-attention: Q and K rotated where the projection left them, [B, N, 3, H, d]
    qkv = _project(x, qkv_w).view(B, N, 3, H, d)
    q, k, v = (qkv[:, :, i].transpose(1, 2) for i in range(3))
    _norm(q, k, q, k, norm_w[0], norm_w[1], L.INTERLEAVED, GRID)
    flags = vc.VC_FLAG_ALL & ~vc.VC_FLAG_ROPE
    p = Params.make(B, H, N, d, GRID, bits=bits, flags=flags, stride_b=q.stride(0), stride_h=q.stride(1), stride_n=q.stride(2))
    quant, work = alloc_buffers(p)
    o = torch.empty(B, H, N, d, dtype=BF, device="cuda")
    vc.vc_attn(p, q, k, v, None, o, quant, work)
    vc.vc_poll_status(work)
    cfg = OP.PrepConfig(N=N, d=d, grid=GRID, bits=bits, rope=False)
    for b in range(B):
        f = lambda t: t[b, 1].float().cpu().numpy()
        ref = OA.emulate_head(OP.prep_head(f(q), f(k), f(v), np.arange(N), cfg), cfg)
        m = CMP.output_metrics(f(o), ref, float(v.float().abs().max()))
        assert m["max_err_over_vmax"] <= 2e-2 and m["cos"] >= 0.999, m
    y = _project(o, out_w)
    x = (x.float() + y.float()).to(BF)

    # ---- cross attention: the same norm without a rotation, keys and values two halves of one projection of the encoder's states
    q = _project(x, q_w).view(B, N, H, d).transpose(1, 2)
    kv = _project(text, kv_w).view(B, TEXT, 2, H, d)
    k, v = (kv[:, :, i].transpose(1, 2) for i in range(2))
    qn = torch.empty(B, H, N, d, dtype=BF, device="cuda")
    _norm(q, None, qn, None, norm_w[2], None, None, GRID)
    _norm(None, k, None, k, None, norm_w[3], None, (1, 1, TEXT))
    lens = torch.tensor([TEXT, 19], dtype=torch.int32, device="cuda")
    pc = vc.CrossParams.of(qn, k, v, o)
    cwork = torch.empty(vc.vc_cross_workspace_bytes(pc), dtype=torch.uint8, device="cuda")
    vc.vc_cross_attn(pc, qn, k, v, lens, None, o, None, cwork)
    vc.vc_poll_status(cwork)
    want, _ = L.cross_attention(_np(qn), _np(k), _np(v), d ** -0.5, lens.cpu().numpy())
    size, _ = L.cross_attention(_np(qn), _np(k), np.abs(_np(v)), d ** -0.5, lens.cpu().numpy())
    # (normed queries and keys: scores of at most 1.5^2 sqrt(128) * d / sqrt(d), 2 D below 2^-8)
    assert (np.abs(_np(o) - want) <= 2.0 ** -8 * np.abs(want) + 2.0 ** -7 * size).all()
    _project(o, out2_w)


def test_block_captured_into_one_graph():
    """Projection, norm, attention and output projection in one graph, replayed on other inputs."""
    g = torch.Generator().manual_seed(41)
    qkv_w, out_w = Weights(3 * DIM, DIM, g), Weights(DIM, DIM, g)
    nw = [(1.0 + 0.1 * torch.randn(d, generator=g)).to(BF).cuda() for _ in range(2)]
    xs = [torch.randn(B * N, DIM, generator=g).to(BF).cuda() for _ in range(2)]
    x = xs[0].clone()
    codes, scale = torch.empty(B * N, DIM, dtype=torch.uint8, device="cuda"), torch.empty(H, B * N, device="cuda")
    qkv, o, y = (torch.empty(B * N, 3 * DIM, dtype=BF, device="cuda"), torch.empty(B, H, N, d, dtype=BF, device="cuda"),
                 torch.empty(B * N, DIM, dtype=BF, device="cuda"))
    q, k, v = (qkv.view(B, N, 3, H, d)[:, :, i].transpose(1, 2) for i in range(3))
    p0, p1 = vc.QuantParams.of(x), vc.LinearParams.of(codes, qkv_w.codes, qkv, qkv_w.bias)
    p2 = vc.QkParams.of(q, k, q, k, grid=GRID, weight=nw[0], norm=vc.VC_NORM_HEAD, rotary=vc.VC_ROTARY_HALF)
    p3 = Params.make(B, H, N, d, GRID, flags=vc.VC_FLAG_ALL & ~vc.VC_FLAG_ROPE, stride_b=q.stride(0), stride_h=q.stride(1), stride_n=q.stride(2))
    p4, p5 = vc.QuantParams.of(o), vc.LinearParams.of(codes, out_w.codes, y, out_w.bias)
    quant, work = alloc_buffers(p3)
    w1, w5 = (torch.empty(vc.vc_linear_workspace_bytes(t), dtype=torch.uint8, device="cuda") for t in (p1, p5))

    def layer():
        vc.vc_quant_fp8(p0, x, codes, scale)
        vc.vc_linear_fp8(p1, codes, scale, qkv_w.codes, qkv_w.scale, qkv_w.bias, qkv, w1)
        vc.vc_qk_norm_rope(p2, q, k, nw[0], nw[1], None, q, k)
        vc.vc_attn(p3, q, k, v, None, o, quant, work)
        vc.vc_quant_fp8(p4, o, codes, scale)
        vc.vc_linear_fp8(p5, codes, scale, out_w.codes, out_w.scale, out_w.bias, y, w5)

    want = []
    for t in xs:
        x.copy_(t)
        layer()
        for w in (w1, work, w5):
            vc.vc_poll_status(w)
        want.append(y.clone())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        layer()
    for t, ref in zip(xs, want):
        x.copy_(t)
        y.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, ref)
