"""Scores of device logits (log probability, rank, entropy, alternatives) against a 64-bit restatement on the CPU."""
import numpy as np
import pytest

from tests import ops_util as ou

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

DT = {"fp32": torch.float32, "bf16": torch.bfloat16}
LOWEST = {"fp32": float(torch.finfo(torch.float32).min), "bf16": float(torch.finfo(torch.bfloat16).min)}


@pytest.fixture(scope="module")
def s2d2():
    import paper_2603_25702_b200 as m
    return m


def stream():
    return torch.cuda.current_stream().cuda_stream


def run(s2d2, x, tokens, k):
    """All outputs for a 2-d device tensor of logits (any row stride, any first element)."""
    rows, V = x.shape
    name = "fp32" if x.dtype == torch.float32 else "bf16"
    o = {n: torch.full((rows + 1,), 7.0, device="cuda") for n in ("logprob", "lse", "entropy")}
    o["rank"] = torch.full((rows + 1,), 7, dtype=torch.int32, device="cuda")
    kw = {}
    if k:
        o["top_ids"] = torch.full((rows + 1, k), 7, dtype=torch.int32, device="cuda")
        o["top_logprobs"] = torch.full((rows + 1, k), 7.0, device="cuda")
        kw = dict(d_top_ids=o["top_ids"].data_ptr(), d_top_logprobs=o["top_logprobs"].data_ptr())
    tok = torch.as_tensor(np.asarray(tokens), dtype=torch.int32, device="cuda")
    s2d2.score_logits(x.data_ptr(), name, rows, V, x.stride(0), tok.data_ptr(), k, d_logprob=o["logprob"].data_ptr(),
                      d_rank=o["rank"].data_ptr(), d_lse=o["lse"].data_ptr(), d_entropy=o["entropy"].data_ptr(), stream=stream(), **kw)
    torch.cuda.synchronize()
    for v in o.values():
        assert (v[rows:] == 7).all()                                 # rows behind the last one stay as they were
    return {n: v[:rows].cpu().numpy() for n, v in o.items()}


def check(got, x64, tokens, k):
    want = ou.scores(x64, tokens, k)
    V = x64.shape[1]
    tol = ou.score_tolerance(V, want["log_s"])
    ulp = 2.0 ** -23                                                 # two roundings of the result itself
    for n, t in (("lse", tol), ("logprob", tol), ("entropy", 3 * tol * (1 + np.abs(want["entropy"])))):
        w, g = want[n], got[n].astype(np.float64)
        fine = np.isfinite(w)
        assert np.array_equal(np.isnan(w), np.isnan(g)) and np.array_equal(w[~fine & ~np.isnan(w)], g[~fine & ~np.isnan(w)]), n
        err = np.abs(g - w)[fine]
        assert (err <= (t + ulp * np.abs(np.where(fine, w, 0)))[fine]).all(), (n, err.max())
    assert np.array_equal(got["rank"], want["rank"])
    if k:
        assert np.array_equal(got["top_ids"], want["top_ids"])
        w, g = want["top_logprobs"], got["top_logprobs"].astype(np.float64)
        fine = np.isfinite(w)
        assert np.array_equal(np.isnan(w), np.isnan(g)) and (g[~fine & ~np.isnan(w)] == -np.inf).all()
        err = np.abs(np.where(fine, g, 0) - np.where(fine, w, 0))
        assert (err <= tol[:, None] + ulp * np.abs(np.where(fine, w, 0))).all()


def logits(rows, V, dtype, seed, pad=0, lead=0, spread=2.5):
    g = torch.Generator(device="cuda").manual_seed(seed)
    buf = (torch.randn(rows * (V + pad) + lead, generator=g, device="cuda") * spread).to(DT[dtype])
    return buf[lead:].view(rows, V + pad)[:, :V]


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("rows,V,pad,lead,k", [(1, 1, 0, 0, 1), (2, 2, 1, 1, 5), (3, 31, 0, 3, 32), (5, 50, 14, 0, 32), (4, 1000, 0, 0, 0),
                                               (7, 1001, 0, 0, 20), (3, 4096, 0, 0, 8), (2, 4097, 3, 5, 1), (1, 151936, 0, 0, 20),
                                               (9, 50001, 1, 1, 5), (40, 2000, 0, 7, 7), (1300, 600, 0, 0, 3), (2, 157184, 0, 2, 32)])
def test_scores(s2d2, dtype, rows, V, pad, lead, k):
    x = logits(rows, V, dtype, rows + V, pad, lead)
    rng = np.random.default_rng(V)
    tokens = rng.integers(0, V, rows)
    tokens[::2] = x.float().argmax(1).cpu().numpy()[::2]
    check(run(s2d2, x, tokens, k), x.double().cpu().numpy(), tokens, k)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("lowest", ["inf", "lowest"])
@pytest.mark.parametrize("V", [50, 5000, 60000])
def test_masked_rows(s2d2, dtype, lowest, V):
    """Masks that leave half of the row, a handful of tokens, one token, or nothing."""
    bar = -np.inf if lowest == "inf" else LOWEST[dtype]
    x = logits(6, V, dtype, V).clone()
    g = torch.Generator(device="cuda").manual_seed(V)
    x[0, torch.rand(V, generator=g, device="cuda") < 0.5] = bar
    keep = torch.randint(0, V, (6,), generator=g, device="cuda")
    for r, n in ((1, 6), (2, 3), (3, 1), (4, 0)):
        row = torch.full((V,), bar, dtype=x.dtype, device="cuda")
        row[keep[:n]] = x[r, keep[:n]]
        x[r] = row
    tokens = [0, int(keep[0]), (int(keep[0]) + 1) % V, int(keep[0]), V - 1, 3]
    check(run(s2d2, x, tokens, 8), x.double().cpu().numpy(), tokens, 8)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_undefined_rows_and_tokens_outside(s2d2, dtype):
    V = 9000
    x = logits(6, V, dtype, 3).clone()
    x[0, 8000] = float("nan")
    x[1, 5] = float("inf")
    x[2] = float("nan")
    x[3, 17] = float("-inf")
    tokens = [1, 5, 0, -1, V, 17]
    check(run(s2d2, x, tokens, 4), x.double().cpu().numpy(), tokens, 4)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("V,levels", [(300, 1), (20000, 1), (20000, 2), (151936, 5), (151936, 4000)])
def test_ties_go_to_the_lowest_id(s2d2, dtype, V, levels):
    g = torch.Generator(device="cuda").manual_seed(V + levels)
    x = (torch.randint(0, levels, (3, V), generator=g, device="cuda").float() / max(1, levels // 4)).to(DT[dtype])
    x[1] = -x[1]                                                     # -0 and +0 are equal
    x[1, ::3] = x[1, ::3] + 0.0
    tokens = [V - 1, V // 2, 1]
    check(run(s2d2, x, tokens, 32), x.double().cpu().numpy(), tokens, 32)


@pytest.mark.parametrize("rows", [1, 3])
@pytest.mark.parametrize("kind", ["rising", "falling", "few_threads", "few_threads_ties"])
def test_orders_that_defeat_the_threshold(s2d2, kind, rows):
    """Large logits that all fall to a few threads: more candidates than fit, found value by value."""
    V = 151936
    x = torch.linspace(-4, 4, V, device="cuda").repeat(rows, 1)
    if kind == "falling":
        x = x.flip(1).contiguous()
    if kind.startswith("few"):
        x = torch.randn(rows, V, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda")
        at = torch.arange(V, device="cuda") // 4 % 256 < 12          # vectors of 12 of 256 threads
        x[:, at] = 50 + x[:, at] if kind == "few_threads" else 50 + torch.round(x[:, at])
    tokens = [7] * rows
    check(run(s2d2, x.contiguous(), tokens, 20), x.double().cpu().numpy(), tokens, 20)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("V,left,k", [(151936, 700, 20), (151936, 300, 32), (60000, 1100, 8), (60000, 5000, 5), (670, 670, 8), (1081, 1081, 20),
                                      (257, 257, 32), (40, 40, 32), (5000, 513, 1)])
def test_masks_that_leave_a_stretch_and_short_rows(s2d2, dtype, V, left, k):
    """Only some warps see logits: rows shorter than a tile, masks that leave a stretch of ids (also of equal values)."""
    x = logits(4, V, dtype, V + k).clone()
    x[1] = torch.round(x[1])
    x[2] = torch.round(x[2] / 4)
    for r, at in enumerate((0, V // 3, V - left, (V - left) // 2)):
        keep = x[r, at:at + left].clone()
        x[r] = float("-inf")
        x[r, at:at + left][:keep.numel()] = keep[:x[r, at:at + left].numel()]
    tokens = [0, V // 3, V - 1, 7]
    check(run(s2d2, x, tokens, k), x.double().cpu().numpy(), tokens, k)
    x[torch.isneginf(x)] = LOWEST[dtype]                             # the same with the type's lowest value: hundreds of equal logits
    check(run(s2d2, x, tokens, k), x.double().cpu().numpy(), tokens, k)


def test_extreme_logits(s2d2):
    """Differences that underflow, a certain token, values near the type's ends."""
    x = torch.zeros(5, 5000, device="cuda")
    x[0, 77] = 200.0
    x[1] = -3e38
    x[1, 9] = 1.0
    x[2, :] = 3e38
    x[3] = torch.linspace(-100, 0, 5000, device="cuda")
    x[4] = 1e-40
    tokens = [77, 9, 4999, 4999, 0]
    check(run(s2d2, x, tokens, 3), x.double().cpu().numpy(), tokens, 3)


def test_outputs_are_optional_and_independent(s2d2):
    x = logits(4, 3000, "fp32", 0)
    tok = torch.tensor([1, 2, 3, 4], dtype=torch.int32, device="cuda")
    full = run(s2d2, x, tok.cpu().numpy(), 6)
    only = torch.empty(4, device="cuda")
    s2d2.score_logits(x.data_ptr(), "fp32", 4, 3000, 3000, d_entropy=only.data_ptr(), stream=stream())
    assert np.array_equal(only.cpu().numpy(), full["entropy"])
    ids = torch.empty(4, 6, dtype=torch.int32, device="cuda")
    s2d2.score_logits(x.data_ptr(), "fp32", 4, 3000, 3000, 0, 6, d_top_ids=ids.data_ptr(), stream=stream())
    assert np.array_equal(ids.cpu().numpy(), full["top_ids"])
    s2d2.score_logits(0, "fp32", 0, 3000, 3000, d_entropy=only.data_ptr(), stream=stream())        # no rows
    host = torch.zeros(4)
    for bad in (dict(d_entropy=host.data_ptr()), dict(d_entropy=only.data_ptr() + 2)):
        with pytest.raises(s2d2.S2D2Error) as e:
            s2d2.score_logits(x.data_ptr(), "fp32", 4, 3000, 3000, stream=stream(), **bad)
        assert e.value.code == -1


def test_captured_call_follows_its_inputs(s2d2):
    x = torch.zeros(3, 20000, device="cuda")
    lse, ids = torch.empty(3, device="cuda"), torch.empty(3, 4, dtype=torch.int32, device="cuda")

    def call():
        s2d2.score_logits(x.data_ptr(), "fp32", 3, 20000, 20000, 0, 4, d_lse=lse.data_ptr(), d_top_ids=ids.data_ptr(), stream=stream())

    call()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    for seed in range(3):
        x.copy_(logits(3, 20000, "fp32", seed))
        g.replay()
        torch.cuda.synchronize()
        want = ou.scores(x.double().cpu().numpy(), None, 4)
        assert np.array_equal(ids.cpu().numpy(), want["top_ids"])
        assert np.abs(lse.cpu().numpy() - want["lse"]).max() <= ou.score_tolerance(20000, want["log_s"]).max() + 2.0 ** -23 * 20


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("rows,V,k", [(2, 2000000, 32), (2, 1999999, 5), (6000, 60, 4), (700, 30000, 8)])
def test_largest_vocabulary_and_many_rows(s2d2, dtype, rows, V, k):
    x = logits(rows, V, dtype, V)
    tokens = np.arange(rows) % V
    check(run(s2d2, x, tokens, k), x.double().cpu().numpy(), tokens, k)


def test_rows_further_apart_than_32_bits(s2d2):
    """Three rows 2^31 + 5 elements apart: offsets of the last one pass 2^32."""
    stride, V = 2 ** 31 + 5, 3000
    buf = torch.empty(2 * stride + V, dtype=torch.bfloat16, device="cuda")
    x = torch.as_strided(buf, (3, V), (stride, 1))
    x.copy_(logits(3, V, "bf16", 5))
    check(run(s2d2, x, [5, 6, 7], 4), x.double().cpu().numpy(), [5, 6, 7], 4)


def test_concurrent_and_repeated_calls_agree_bit_for_bit(s2d2):
    jobs = [(logits(r, V, d, r), np.arange(r) % V, k) for r, V, d, k in ((1, 151936, "fp32", 20), (300, 20000, "bf16", 8), (7, 999, "fp32", 3))]
    alone = [run(s2d2, *j) for j in jobs]
    outs = []
    streams = [torch.cuda.Stream() for _ in jobs]
    torch.cuda.synchronize()
    for (x, tokens, k), st in zip(jobs, streams):
        with torch.cuda.stream(st):
            rows, V = x.shape
            tok = torch.as_tensor(tokens, dtype=torch.int32).cuda(non_blocking=False)
            reps = []
            for _ in range(4):
                f, i = torch.empty(3, rows, device="cuda"), torch.empty(rows, k + 1, dtype=torch.int32, device="cuda")
                lp = torch.empty(rows, k, device="cuda")
                ids = torch.empty(rows, k, dtype=torch.int32, device="cuda")
                s2d2.score_logits(x.data_ptr(), "fp32" if x.dtype == torch.float32 else "bf16", rows, V, x.stride(0), tok.data_ptr(), k,
                                  d_logprob=f[0].data_ptr(), d_lse=f[1].data_ptr(), d_entropy=f[2].data_ptr(), d_rank=i.data_ptr(),
                                  d_top_ids=ids.data_ptr(), d_top_logprobs=lp.data_ptr(), stream=stream())
                reps.append((f, i, ids, lp, tok))
            outs.append(reps)
    torch.cuda.synchronize()
    for want, reps, (x, _, k) in zip(alone, outs, jobs):
        rows = x.shape[0]
        for f, i, ids, lp, _ in reps:
            assert np.array_equal(f[0].cpu().numpy(), want["logprob"]) and np.array_equal(f[1].cpu().numpy(), want["lse"])
            assert np.array_equal(f[2].cpu().numpy(), want["entropy"]) and np.array_equal(i.view(-1)[:rows].cpu().numpy(), want["rank"])
            assert np.array_equal(ids.cpu().numpy(), want["top_ids"]) and np.array_equal(lp.cpu().numpy(), want["top_logprobs"])


def test_score_pass_of_an_engine(s2d2):
    """Scores of the draft and the verifier logits of a decode step against the logits themselves."""
    from s2d2_inputs import generate_prompts, generate_weights, get_config
    wl = get_config("t_bf16_128")
    eng = s2d2.Engine(wl.model, block_size=wl.block_size, max_batch=wl.batch, max_seq_len=256, kv_page_tokens=wl.kv_page_tokens,
                      seed=1, stream=stream())
    eng.load_weights(generate_weights(wl.model, seed=0, gain_jitter=0.1))
    ids = eng.prefill(generate_prompts(wl))
    with pytest.raises(s2d2.S2D2Error):
        eng.score_pass(0, 1)                                         # nothing drafted yet
    st = eng.draft_block(ids)
    n = sum(s.n_masked for s in st)
    proposals = [s.xhat[i] for s in st for i in range(s.n_masked)]
    x = eng.debug_copy_logits(0, n).astype(np.float64)
    got = eng.score_pass(0, n, proposals, 5)
    check({k: v for k, v in got.items()}, x, proposals, 5)
    assert (got["rank"] == 0).all()                                  # greedy proposals
    conf = np.array([s.conf[i] for s in st for i in range(s.n_masked)])
    assert np.allclose(np.exp(got["logprob"]), conf, rtol=1e-5)
    eng.verify_block(ids, [1] * len(ids))
    x = eng.debug_copy_logits(1, n).astype(np.float64)
    tokens = list(range(x.shape[0]))
    check(eng.score_pass(1, x.shape[0], tokens, 32), x, tokens, 32)
    assert set(eng.score_pass(1, 1)) == {"lse", "entropy"}
    for bad in (dict(which=2, n_rows=1), dict(which=0, n_rows=n + 1), dict(which=0, n_rows=1, top_k=33)):
        with pytest.raises(s2d2.S2D2Error):
            eng.score_pass(**bad)
    eng.close()


def test_four_bit_head_then_scores(s2d2):
    """Hidden rows -> MXFP4 -> head product -> scores, as a decode step with a 4-bit head uses them."""
    M, N, K = 12, 5000, 512
    g = torch.Generator(device="cuda").manual_seed(4)
    h = torch.randn(M, K, generator=g, device="cuda").to(torch.bfloat16)
    w = (torch.randn(N, K, generator=g, device="cuda") * 0.1).to(torch.bfloat16)

    def q(x):
        nc, ns = s2d2.mxfp4_sizes(*x.shape)
        c, s = torch.empty(nc, dtype=torch.uint8, device="cuda"), torch.empty(ns, dtype=torch.uint8, device="cuda")
        s2d2.mxfp4_quantize(x.data_ptr(), "bf16", x.shape[0], x.shape[1], x.stride(0), c.data_ptr(), s.data_ptr(), stream())
        return c, s

    (hc, hs), (wc, ws) = q(h), q(w)
    y = torch.empty(M, N, device="cuda")
    s2d2.mxfp4_gemm(hc.data_ptr(), hs.data_ptr(), wc.data_ptr(), ws.data_ptr(), y.data_ptr(), "fp32", M, N, K, stream=stream())
    tokens = np.arange(M) * 17
    got = run(s2d2, y, tokens, 10)
    check(got, y.double().cpu().numpy(), tokens, 10)
    hv = ou.mxfp4_values(*ou.mxfp4_encode(h.double().cpu().numpy()), K)
    wv = ou.mxfp4_values(*ou.mxfp4_encode(w.double().cpu().numpy()), K)
    want = ou.scores(hv @ wv.T, tokens, 1)
    # a logit is off by at most the product's bound; so is the log of a sum of their exponentials
    slack = ((np.abs(hv) @ np.abs(wv).T) * (K // 64 + 10) * 2.0 ** -23).max()
    assert np.abs(got["lse"] - want["lse"]).max() <= slack + ou.score_tolerance(N, want["log_s"]).max() + 2.0 ** -20
    s2d2.ops_status(stream())
