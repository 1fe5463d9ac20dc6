"""The operators around the quantized attention called the ways a serving program may call them: on two streams at once, from two
captured graphs in flight together, with one tensor in several places, behind kernels of the library that let their successor start early."""
import pytest
import torch

import paper_2609_15810_b200 as vc
from paper_2609_15810_b200.binding import Params, alloc_buffers

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


def _cross_call(seed, Nq=500, Nkv=900, splits=0, H=6):
    g = torch.Generator().manual_seed(seed)
    q, k, v = (torch.randn(2, H, n, 128, generator=g).to(BF).cuda() for n in (Nq, Nkv, Nkv))
    lens = torch.tensor([Nkv, Nkv // 3], dtype=torch.int32, device="cuda")
    o, lse = torch.empty_like(q), torch.empty(2, H, Nq, device="cuda")
    p = vc.CrossParams.of(q, k, v, o, key_splits=splits)
    work = torch.empty(vc.vc_cross_workspace_bytes(p), dtype=torch.uint8, device="cuda")
    return (lambda: vc.vc_cross_attn(p, q, k, v, lens, None, o, lse, work)), (o, lse), work


def _linear_call(seed, M):
    g = torch.Generator().manual_seed(seed)
    x, w = torch.randn(M, 1536, generator=g).to(BF).cuda(), torch.randn(700, 1536, generator=g).to(BF).cuda()
    xc, wc = (torch.empty(t.shape, dtype=torch.float8_e4m3fn, device="cuda") for t in (x, w))
    xs, ws = torch.empty(12, M, device="cuda"), torch.empty(6, 12, device="cuda")
    px, pw = vc.QuantParams.of(x), vc.QuantParams.of(w, 128)
    vc.vc_quant_fp8(pw, w, wc, ws)
    out = torch.empty(M, 700, dtype=BF, device="cuda")
    p = vc.LinearParams.of(xc, wc, out)
    work = torch.empty(vc.vc_linear_workspace_bytes(p), dtype=torch.uint8, device="cuda")

    def call():
        vc.vc_quant_fp8(px, x, xc, xs)
        vc.vc_linear_fp8(p, xc, xs, wc, ws, None, out, work)
    return call, (out, xs), work


CALLS = [lambda s: _cross_call(s), lambda s: _cross_call(s, 1, 5000, 7), lambda s: _linear_call(s, 2), lambda s: _linear_call(s, 300)]


@pytest.mark.parametrize("which", range(len(CALLS)))
@pytest.mark.parametrize("graphs", [False, True])
def test_two_streams_at_once(which, graphs):
    a, b = CALLS[which](1), CALLS[which](2)
    for call, _, work in (a, b):
        call()
        vc.vc_poll_status(work)
    want = [[t.clone() for t in outs] for _, outs, _ in (a, b)]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    run = [a[0], b[0]]
    if graphs:
        run = []
        for call, _, _ in (a, b):
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                call()
            run.append(graph.replay)
    for _, outs, _ in (a, b):
        for t in outs:
            t.zero_()
    torch.cuda.synchronize()
    for _ in range(20):
        for s, r in zip(streams, run):
            with torch.cuda.stream(s):
                r()
    torch.cuda.synchronize()
    for (_, outs, work), ref in zip((a, b), want):
        vc.vc_poll_status(work)
        for t, r in zip(outs, ref):
            assert torch.equal(t, r)


def _attention_call(seed):
    g = torch.Generator().manual_seed(seed)
    q, k, v = (torch.randn(1, 4, 1280, 128, generator=g).to(BF).cuda() for _ in range(3))
    o = torch.empty_like(q)
    p = Params.make(1, 4, 1280, 128, (10, 8, 16), flags=vc.VC_FLAG_ALL & ~vc.VC_FLAG_ROPE)
    quant, work = alloc_buffers(p)
    return (lambda: vc.vc_attn(p, q, k, v, None, o, quant, work)), (o,), work


def _wide_linear_call(seed, M, N, K=1024):
    g = torch.Generator().manual_seed(seed)
    x, w = (torch.randint(0, 120, (n, K), generator=g, dtype=torch.uint8).cuda() for n in (M, N))
    xs, ws = torch.rand(K // 128, M, generator=g).cuda(), torch.rand((N + 127) // 128, K // 128, generator=g).cuda()
    out = torch.empty(M, N, dtype=BF, device="cuda")
    p = vc.LinearParams.of(x, w, out)
    work = torch.empty(vc.vc_linear_workspace_bytes(p), dtype=torch.uint8, device="cuda")
    return (lambda: vc.vc_linear_fp8(p, x, xs, w, ws, None, out, work)), (out,), work


def test_every_kind_at_once():
    """Products by pairs of CTAs and by single ones, both attentions, on five streams: they take turns on the SMs and their tensor memory."""
    calls = [_wide_linear_call(1, 5000, 2000), _wide_linear_call(2, 3000, 2560), _wide_linear_call(3, 700, 640), _cross_call(4, 2000, 700, H=12), _attention_call(5)]
    for call, _, work in calls:
        call()
        vc.vc_poll_status(work)
    want = [[t.clone() for t in outs] for _, outs, _ in calls]
    streams = [torch.cuda.Stream() for _ in calls]
    for _, outs, _ in calls:
        for t in outs:
            t.zero_()
    torch.cuda.synchronize()
    for _ in range(40):
        for s, (call, _, _) in zip(streams, calls):
            with torch.cuda.stream(s):
                call()
    torch.cuda.synchronize()
    for (_, outs, work), ref in zip(calls, want):
        vc.vc_poll_status(work)
        for t, r in zip(outs, ref):
            assert torch.equal(t, r)


def test_one_tensor_as_queries_keys_and_values():
    g = torch.Generator().manual_seed(3)
    x = torch.randn(1, 2, 333, 64, generator=g).to(BF).cuda()
    o, o2 = torch.empty_like(x), torch.empty_like(x)
    p = vc.CrossParams.of(x, x, x, o)
    work = torch.empty(vc.vc_cross_workspace_bytes(p), dtype=torch.uint8, device="cuda")
    vc.vc_cross_attn(p, x, x, x, None, None, o, None, work)
    y, z = x.clone(), x.clone()
    vc.vc_cross_attn(p, x, y, z, None, None, o2, None, work)
    vc.vc_poll_status(work)
    assert torch.equal(o, o2)


def test_one_tensor_as_queries_and_keys_of_the_norm():
    g = torch.Generator().manual_seed(4)
    x = torch.randn(1, 5, 70, 128, generator=g).to(BF).cuda()
    a, b = torch.empty_like(x), torch.empty_like(x)
    p = vc.QkParams.of(x, x, a, b, grid=(70, 1, 1), norm=vc.VC_NORM_TOKEN, rotary=vc.VC_ROTARY_HALF, rope_dims=(128, 0, 0))
    vc.vc_qk_norm_rope(p, x, x, None, None, None, a, b)
    assert torch.equal(a, b)


def test_back_to_back_with_kernels_that_let_their_successor_start_early():
    """Norm in place -> quantized attention -> E4M3 codes of its output -> cross attention on the same output, many times over: each
    call reads what the one in front of it wrote."""
    g = torch.Generator().manual_seed(5)
    B, H, N, d = 1, 2, 640, 128
    src = [torch.randn(B, H, N, d, generator=g).to(BF).cuda() for _ in range(3)]
    q, k, v = (t.clone() for t in src)
    o, o2 = torch.empty_like(q), torch.empty_like(q)
    pn = vc.QkParams.of(q, k, q, k, grid=(5, 8, 16), norm=vc.VC_NORM_HEAD, rotary=vc.VC_ROTARY_INTERLEAVED)
    pa = Params.make(B, H, N, d, (5, 8, 16), flags=vc.VC_FLAG_ALL & ~vc.VC_FLAG_ROPE)
    quant, work = alloc_buffers(pa)
    pq = vc.QuantParams.of(o)
    codes, scale = torch.empty(N, H * d, dtype=torch.uint8, device="cuda"), torch.empty(2, N, device="cuda")
    pc = vc.CrossParams.of(o, k, v, o2)
    cwork = torch.empty(vc.vc_cross_workspace_bytes(pc), dtype=torch.uint8, device="cuda")

    def chain(wait):
        for t, s in zip((q, k, v), src):
            t.copy_(s)
        for step in (lambda: vc.vc_qk_norm_rope(pn, q, k, None, None, None, q, k), lambda: vc.vc_attn(pa, q, k, v, None, o, quant, work),
                     lambda: vc.vc_quant_fp8(pq, o, codes, scale), lambda: vc.vc_cross_attn(pc, o, k, v, None, None, o2, None, cwork),
                     lambda: vc.vc_attn(pa, o2, k, v, None, o, quant, work)):
            if wait:
                torch.cuda.synchronize()
            step()
        return [t.clone() for t in (o, o2, codes, scale)]
    want = chain(True)
    for _ in range(30):
        for got, ref in zip(chain(False), want):
            assert torch.equal(got, ref)


def test_tensors_that_do_not_fit_the_parameters_are_refused_by_the_binding():
    x = torch.zeros(1, 2, 8, 64, dtype=BF, device="cuda")
    o = torch.empty_like(x)
    p = vc.CrossParams.of(x, x, x, o)
    work = torch.empty(vc.vc_cross_workspace_bytes(p), dtype=torch.uint8, device="cuda")
    ok = [p, x, x, x, None, None, o, None, work]
    vc.vc_cross_attn(*ok)
    wide = torch.zeros(1, 2, 8, 128, dtype=BF, device="cuda")
    for at, bad in ((1, x.cpu()), (2, x.half()), (3, x[:, :, :7]), (1, wide[..., ::2]), (4, torch.zeros(1, device="cuda")), (4, torch.zeros(2, dtype=torch.int32, device="cuda")),
                    (5, torch.ones(1, 9, dtype=torch.bool, device="cuda")), (6, x[:, :1]), (7, torch.empty(1, 2, 8, dtype=BF, device="cuda")), (8, work[:100]), (8, work.cpu())):
        args = list(ok)
        args[at] = bad
        with pytest.raises(ValueError):
            vc.vc_cross_attn(*args)
    with pytest.raises(vc.VcError):
        vc.vc_cross_attn(p, x, x, x, None, None, o, None, None)
    pq = vc.QuantParams.of(x)
    codes, scale = torch.empty(8, 128, dtype=torch.uint8, device="cuda"), torch.empty(1, 8, device="cuda")
    vc.vc_quant_fp8(pq, x, codes, scale)
    for args in ((x, codes.t(), scale), (x, codes, scale.t()), (x.float(), codes, scale), (x, codes.view(torch.int8), scale), (x[0, 0], codes, scale)):
        with pytest.raises(ValueError):
            vc.vc_quant_fp8(pq, *args)
    pn = vc.QkParams.of(x, None, o, None, grid=(8, 1, 1), norm=vc.VC_NORM_HEAD)
    for w in (torch.ones(128, dtype=BF, device="cuda"), torch.ones(64, device="cuda"), torch.ones(64, dtype=BF)):
        with pytest.raises(ValueError):
            vc.vc_qk_norm_rope(pn, x, None, w, None, None, o, None)
    torch.cuda.synchronize()
