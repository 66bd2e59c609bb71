"""Stand-alone operators one right behind the other, each on what the one in front has just written, on buffers that are used again."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def s2d2():
    import paper_2603_25702_b200 as m
    return m


# one CTA per tile and few logits; clusters that share k; pairs of CTAs; more rows than one wave of score CTAs
@pytest.mark.parametrize("M,N,K", [(3, 1000, 256), (64, 4097, 4096), (300, 20001, 512), (700, 6000, 64)])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_back_to_back_calls_see_what_the_one_in_front_wrote(s2d2, M, N, K, dtype):
    """Quantise, product, scores of the logits, quantise the logits (rows that are not aligned to 16 bytes), dequantise over the same
    logits, scores again, scores from hidden rows; twice with other hidden rows in the same buffers. Without pauses, in a graph as well, and
    with a synchronisation behind every call: the same bits."""
    dt = {"fp32": torch.float32, "bf16": torch.bfloat16}[dtype]
    g = torch.Generator(device="cuda").manual_seed(M)
    hidden = [torch.randn(M, K, generator=g, device="cuda") * s for s in (1.0, 0.5)]
    w = torch.randn(N, K, generator=g, device="cuda") * 0.1
    u8 = lambda n: torch.empty(n, dtype=torch.uint8, device="cuda")
    xc, xs = (u8(n) for n in s2d2.mxfp4_sizes(M, K))
    wc, ws = (u8(n) for n in s2d2.mxfp4_sizes(N, K))
    yc, ys = (u8(n) for n in s2d2.mxfp4_sizes(M, N))
    work = u8(s2d2.mxfp4_score_workspace(M, N, K))
    buf = torch.empty(M * (N + 1) + 1, dtype=dt, device="cuda")
    y = buf[1:].view(M, N + 1)[:, :N]                                # neither rows nor the first element aligned
    tok = torch.randint(0, N, (M,), generator=g, device="cuda", dtype=torch.int32)
    outs = [dict(f=torch.empty(3, M, device="cuda"), rank=torch.empty(M, dtype=torch.int32, device="cuda"),
                 ids=torch.empty(M, 7, dtype=torch.int32, device="cuda"), lp=torch.empty(M, 7, device="cuda")) for _ in range(4)]
    direct = [torch.empty(3, M, device="cuda") for _ in range(2)]

    def calls(st):
        def score(o):
            s2d2.score_logits(y.data_ptr(), dtype, M, N, N + 1, tok.data_ptr(), 7, d_logprob=o["f"][0].data_ptr(),
                              d_lse=o["f"][1].data_ptr(), d_entropy=o["f"][2].data_ptr(), d_rank=o["rank"].data_ptr(),
                              d_top_ids=o["ids"].data_ptr(), d_top_logprobs=o["lp"].data_ptr(), stream=st)
        yield lambda: s2d2.mxfp4_quantize(w.data_ptr(), "fp32", N, K, K, wc.data_ptr(), ws.data_ptr(), st)
        for i, h in enumerate(hidden):
            yield lambda: s2d2.mxfp4_quantize(h.data_ptr(), "fp32", M, K, K, xc.data_ptr(), xs.data_ptr(), st)
            yield lambda: s2d2.mxfp4_gemm(xc.data_ptr(), xs.data_ptr(), wc.data_ptr(), ws.data_ptr(), y.data_ptr(), dtype, M, N, K, N + 1,
                                          stream=st)
            yield lambda: score(outs[2 * i])
            yield lambda: s2d2.mxfp4_quantize(y.data_ptr(), dtype, M, N, N + 1, yc.data_ptr(), ys.data_ptr(), st)
            yield lambda: s2d2.mxfp4_dequantize(yc.data_ptr(), ys.data_ptr(), M, N, y.data_ptr(), dtype, N + 1, st)
            yield lambda: score(outs[2 * i + 1])
            yield lambda: s2d2.mxfp4_score(xc.data_ptr(), xs.data_ptr(), wc.data_ptr(), ws.data_ptr(), M, N, K, tok.data_ptr(), work.data_ptr(),
                                           work.numel(), d_logprob=direct[i][0].data_ptr(), d_lse=direct[i][1].data_ptr(),
                                           d_entropy=direct[i][2].data_ptr(), stream=st)

    results = [t for o in outs for t in o.values()] + direct + [y]

    def clear():
        for t in (xc, xs, wc, ws, yc, ys, work):
            t.fill_(0xFF)
        for t in results:
            t.fill_(-7)
        torch.cuda.synchronize()

    side = torch.cuda.Stream()
    clear()
    for call in calls(side.cuda_stream):
        call()
        torch.cuda.synchronize()
    want = [t.clone() for t in results]
    assert all((t != -7).any() for t in want)
    # the two hidden batches differ, and so does what stands in the logits' buffer before and after the rounding
    assert not torch.equal(want[0], want[8]) and not torch.equal(want[0], want[4])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        for call in calls(side.cuda_stream):
            call()
    for rep in range(12):
        clear()
        if rep % 2:
            graph.replay()
        else:
            for call in calls(side.cuda_stream):
                call()
        torch.cuda.synchronize()
        for a, b in zip(results, want):
            assert torch.equal(a.nan_to_num(nan=1e30), b.nan_to_num(nan=1e30)) if a.is_floating_point() else torch.equal(a, b)
    s2d2.ops_status(side.cuda_stream)
    assert np.isfinite(want[0].cpu().numpy()).all()
