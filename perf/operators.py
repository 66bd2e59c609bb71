"""Cases of the 4-bit head and of token scoring: MXFP4 quantisation, the MXFP4 product, log probabilities of given tokens
with entropy, rank and top alternatives, and log probabilities straight from hidden rows.

MXFP4: blocks of 32 elements along a row share a scale 2^e, e = floor(log2(largest magnitude)) - 2 held as the byte e + 127;
elements are e2m1 codes (0, .5, 1, 1.5, 2, 3, 4, 6 and their negatives), two to a byte, the lower nibble first.  Code rows
are padded to whole blocks.  Scale bytes stand in tiles of 128 rows x 4 blocks (512 bytes): row r, block b at byte
(r % 32) * 16 + (r % 128) // 32 * 4 + b % 4 of tile (r // 128, b // 4); tiles of one row group are contiguous.
"""
import math

import torch

own = False

BLOCK = 32


# ---------------------------------------------------------------------------------------------------------------
# cases
# ---------------------------------------------------------------------------------------------------------------
def listed():
    return [
        # activations of a ragged batch, rows cut out of a wider buffer, a last block that is not full
        dict(name="quantize-ragged", op="quantize", rows=333, cols=2049, pad=31, dtype="float32"),
        # one projection matrix of the 8B-class model, quantised when weights are loaded
        dict(name="quantize-weight", op="quantize", rows=12288, cols=4096, pad=0, dtype="bfloat16"),
        # attention output projection of one token: the smallest product of a decode step
        dict(name="product-1", op="product", m=1, n=4096, k=4096, y="float32"),
        # odd sizes in every direction, as a small or a sharded model has them
        dict(name="product-ragged", op="product", m=77, n=1001, k=2050, y="bfloat16"),
        # gate and up projection of the verifier rows of a batch
        dict(name="product-64", op="product", m=64, n=24576, k=4096, y="bfloat16"),
        # language-model head over the eight masked rows of one block
        dict(name="product-head-8", op="product", m=8, n=151936, k=4096, y="float32"),
        # gate and up projection of a prefill pass
        dict(name="product-1024", op="product", m=1024, n=24576, k=4096, y="bfloat16"),
        # one committed token with the alternatives that a server reports
        dict(name="score-1", op="score", rows=1, vocab=151936, pad=0, dtype="float32", top=20, mask="none"),
        # draft rows of a batch under constrained decoding: most tokens masked, a few rows left with nothing
        dict(name="score-256-masked", op="score", rows=256, vocab=151936, pad=0, dtype="bfloat16", top=8, mask="inf"),
        # every token of a long prompt
        dict(name="score-1024", op="score", rows=1024, vocab=157184, pad=0, dtype="float32", top=5, mask="none"),
        # the eight masked rows of one block scored from their hidden rows
        dict(name="hidden-8", op="hidden", m=8, n=151936, k=4096),
        # every token of a long prompt scored from its hidden row: the logits would take 600 MB
        dict(name="hidden-1024", op="hidden", m=1024, n=151936, k=4096),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["quantize", "product", "product", "score", "score", "hidden"])
    if op == "quantize":
        cols = _log(rng, 16, 12288)
        rows = _log(rng, 1, max(1, min(16384, 12288 * 4096 // cols)))
        return dict(op=op, rows=rows, cols=cols, pad=rng.choice([0, 0, 1, 8, 37]), dtype=rng.choice(["float32", "bfloat16"]))
    if op == "product":
        n, k = _log(rng, 64, 151936), _log(rng, 32, 12288)
        while n * k > 151936 * 4096:
            n, k = _log(rng, 64, 151936), _log(rng, 32, 12288)
        m = _log(rng, 1, min(1024, 1024 * 24576 * 4096 // (n * k)))
        return dict(op=op, m=m, n=n, k=k, y=rng.choice(["float32", "bfloat16"]))
    if op == "score":
        return dict(op=op, rows=_log(rng, 1, 1024), vocab=_log(rng, 50, 157184), pad=rng.choice([0, 0, 1, 64]),
                    dtype=rng.choice(["float32", "bfloat16"]), top=rng.choice([0, 1, 5, 8, 20, 32]),
                    mask=rng.choice(["none", "none", "inf", "lowest"]))
    return dict(op=op, m=_log(rng, 1, 1024), n=_log(rng, 500, 151936), k=_log(rng, 64, 4096))


def work(case):
    """Inputs read once, outputs written once.  A block of 32 elements is 17 bytes."""
    if case["op"] == "quantize":
        n = case["rows"] * case["cols"]
        size = 4 if case["dtype"] == "float32" else 2
        # the values are asked for again: codes and scales are written and read once in between
        return {"bytes": 2 * n * size + 2 * n * 17 / 32, "flops": 4 * n}
    if case["op"] == "score":
        n = case["rows"] * case["vocab"]
        size = 4 if case["dtype"] == "float32" else 2
        return {"bytes": n * size + case["rows"] * (20 + 8 * case["top"]), "flops": 8 * n}
    m, n, k = case["m"], case["n"], case["k"]
    weights = n * k * 17 / 32 + m * k * 2
    if case["op"] == "product":
        return {"bytes": weights + m * n * (4 if case["y"] == "float32" else 2), "flops": 2 * m * n * k}
    return {"bytes": weights + 16 * m, "flops": 2 * m * n * k + 6 * m * n}


# ---------------------------------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------------------------------
def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def randn(*shape):
        return torch.randn(*shape, generator=gen, device="cuda")

    state = dict(case)
    if case["op"] == "quantize":
        # hidden rows and weights: near normal, rows of different size
        x = randn(case["rows"], case["cols"] + case["pad"]) * torch.exp(randn(case["rows"], 1))
        state["x"] = x.to(getattr(torch, case["dtype"]))[:, :case["cols"]]
        return state
    if case["op"] == "score":
        rows, vocab = case["rows"], case["vocab"]
        x = randn(rows, vocab + case["pad"]) * 2.5
        tokens = torch.randint(0, vocab, (rows,), generator=gen, device="cuda")
        tokens = torch.where(torch.rand(rows, generator=gen, device="cuda") < 0.5, x[:, :vocab].argmax(1), tokens)
        if case["mask"] != "none":
            # constrained decoding: one row in eight allows a handful of tokens, the others half of the vocabulary
            keep = torch.rand(rows, 1, generator=gen, device="cuda")
            keep = torch.where(keep < 0.125, min(0.5, 6.0 / vocab), 0.5)
            shut = torch.rand(rows, vocab + case["pad"], generator=gen, device="cuda") >= keep
            lowest = float("-inf") if case["mask"] == "inf" else torch.finfo(getattr(torch, case["dtype"])).min
            x = x.masked_fill(shut, lowest)
            # and some rows are left with nothing
            x = x.masked_fill(torch.rand(rows, 1, generator=gen, device="cuda") < 0.02, lowest)
        state["logits"] = x.to(getattr(torch, case["dtype"]))[:, :vocab]
        state["tokens"] = tokens.to(torch.int32)
        return state
    state["x"] = randn(case["m"], case["k"]).to(torch.bfloat16)
    codes, scales = _encode((randn(case["n"], case["k"]) * 0.02).to(torch.bfloat16))
    state["w_codes"], state["w_scales"] = codes, _tile(scales)
    if case["op"] == "hidden":
        state["tokens"] = torch.randint(0, case["n"], (case["m"],), generator=gen, device="cuda", dtype=torch.int32)
    return state


# ---------------------------------------------------------------------------------------------------------------
# plain forms
# ---------------------------------------------------------------------------------------------------------------
def _encode(x):
    """Codes [rows, 16 * blocks] and scale bytes [rows, blocks] of x [rows, cols]."""
    rows, cols = x.shape
    blocks = -(-cols // BLOCK)
    x = torch.nn.functional.pad(x.float(), (0, blocks * BLOCK - cols)).view(rows, blocks, BLOCK)
    largest = x.abs().amax(2)
    bad = ~torch.isfinite(largest)
    byte = (torch.frexp(largest).exponent - 1 - 2 + 127).clamp(0, 254)
    byte = torch.where(largest == 0, 0, byte)
    byte = torch.where(bad, 127, byte).to(torch.int32)
    inverse = ((254 - byte) << 23).view(torch.float32)
    y = x * inverse.unsqueeze(2)
    a = y.abs()
    code = ((a > 0.25).to(torch.uint8) + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5.0)
            + torch.signbit(y).to(torch.uint8) * 8)
    code = torch.where(bad.unsqueeze(2), 0, code).to(torch.uint8).view(rows, -1, 2)
    byte = torch.where(bad, 255, byte)
    return code[:, :, 0] + code[:, :, 1] * 16, byte.to(torch.uint8)


def _decode(codes, scales, cols):
    """Values [rows, cols] in 32 bits of codes [rows, 16 * blocks] and scale bytes [rows, blocks]."""
    rows, blocks = scales.shape
    table = torch.tensor([0, .5, 1, 1.5, 2, 3, 4, 6, -0., -.5, -1, -1.5, -2, -3, -4, -6], device=codes.device)
    byte = torch.arange(256, device=codes.device)
    pairs = torch.stack([table[byte % 16], table[byte // 16]], 1)
    scale = torch.where(scales == 255, float("nan"), torch.exp2(scales.double() - 127).float())
    values = pairs[codes.int()].view(rows, blocks, BLOCK) * scale.unsqueeze(2)
    return values.view(rows, blocks * BLOCK)[:, :cols]


def _tile(scales):
    """Scale bytes [rows, blocks] in tiles of 128 rows x 4 blocks, padded with zeros."""
    rows, blocks = scales.shape
    scales = torch.nn.functional.pad(scales, (0, -blocks % 4, 0, -rows % 128))
    tiles = scales.view(-(-rows // 128), 4, 32, -(-blocks // 4), 4)
    return tiles.permute(0, 3, 2, 1, 4).contiguous().view(-1)


def _untile(tiles, rows, cols):
    blocks = -(-cols // BLOCK)
    groups, quads = -(-rows // 128), -(-blocks // 4)
    scales = tiles.view(groups, quads, 32, 4, 4).permute(0, 3, 2, 1, 4).reshape(groups * 128, quads * 4)
    return scales[:rows, :blocks]


def _log_probs(x, tokens):
    """(log probability of the tokens, log-sum-exp, entropy) of logits x [rows, vocab] in 32 bits, and what turns a logit into
    its log probability: the row's largest value and the logarithm of its sum."""
    m = x.amax(1, keepdim=True)
    m = torch.where(torch.isneginf(m), 0.0, m)
    e = torch.exp(x - m)
    s = e.sum(1, keepdim=True)
    lse = m + torch.log(s)
    moment = torch.where(e > 0, (x - m) * e, 0.0).sum(1, keepdim=True)
    entropy = torch.where(s > 0, torch.log(s) - moment / s, 0.0)
    x_t = x.gather(1, tokens.long().unsqueeze(1))
    logprob = torch.where(s > 0, (x_t - m) - torch.log(s), float("-inf"))
    return logprob.squeeze(1), lse.squeeze(1), entropy.squeeze(1), m, torch.log(s)


def _plain(state):
    op = state["op"]
    if op == "quantize":
        x = state["x"]
        codes, scales = _encode(x)
        return _decode(codes, scales, x.shape[1]).to(x.dtype)
    if op == "score":
        x, tokens = state["logits"].float(), state["tokens"]
        logprob, lse, entropy, m, log_s = _log_probs(x, tokens)
        x_t = x.gather(1, tokens.long().unsqueeze(1))
        ids = torch.arange(x.shape[1], device=x.device)
        before = (x > x_t) | ((x == x_t) & (ids < tokens.unsqueeze(1)))
        out = dict(logprob=logprob, rank=before.sum(1).to(torch.int32), lse=lse, entropy=entropy)
        if state["top"]:
            # value and inverted id in one whole number: the largest value first, then the lowest id
            bits = (x + 0.0).view(torch.int32).long()
            key = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits) * 2 ** 32 + (x.shape[1] - 1 - ids)
            top = min(state["top"], x.shape[1])
            at = x.shape[1] - 1 - (key.topk(top, dim=1).values & 0xFFFFFFFF)
            value = x.gather(1, at)
            top_lp = torch.where(torch.isneginf(value), float("-inf"), (value - m) - log_s)
            at = torch.where(torch.isneginf(value), -1, at)
            more = (0, state["top"] - top)
            out["top_ids"] = torch.nn.functional.pad(at, more, value=-1).to(torch.int32)
            out["top_logprobs"] = torch.nn.functional.pad(top_lp, more, value=float("-inf"))
        return out
    m, n, k = state["m"], state["n"], state["k"]
    x = _decode(*_encode(state["x"]), k)
    w = _decode(state["w_codes"], _untile(state["w_scales"], n, k), k)
    y = x @ w.t()
    if op == "product":
        return y.to(getattr(torch, state["y"]))
    logprob, lse, entropy, _, _ = _log_probs(y, state["tokens"])
    return dict(logprob=logprob, lse=lse, entropy=entropy)


# ---------------------------------------------------------------------------------------------------------------
# the framework's calls
# ---------------------------------------------------------------------------------------------------------------
_DTYPE = {torch.float32: "fp32", torch.bfloat16: "bf16"}


def _own(state):
    import paper_2603_25702_b200 as s2d2
    stream = torch.cuda.current_stream().cuda_stream
    op = state["op"]

    def quantize(x):
        rows, cols = x.shape
        n_codes, n_scales = s2d2.mxfp4_sizes(rows, cols)
        codes = torch.empty(n_codes, dtype=torch.uint8, device=x.device)
        scales = torch.empty(n_scales, dtype=torch.uint8, device=x.device)
        s2d2.mxfp4_quantize(x.data_ptr(), _DTYPE[x.dtype], rows, cols, x.stride(0), codes.data_ptr(), scales.data_ptr(), stream)
        return codes, scales

    if op == "quantize":
        x = state["x"]
        codes, scales = quantize(x)
        y = torch.empty(x.shape, dtype=x.dtype, device=x.device)
        s2d2.mxfp4_dequantize(codes.data_ptr(), scales.data_ptr(), x.shape[0], x.shape[1], y.data_ptr(), _DTYPE[y.dtype],
                              y.stride(0), stream)
        return y
    if op == "score":
        x, tokens, top = state["logits"], state["tokens"], state["top"]
        rows, vocab = x.shape
        f = torch.empty(3, rows, device=x.device)
        rank = torch.empty(rows, dtype=torch.int32, device=x.device)
        out = dict(logprob=f[0], rank=rank, lse=f[1], entropy=f[2])
        if top:
            out["top_ids"] = torch.empty(rows, top, dtype=torch.int32, device=x.device)
            out["top_logprobs"] = torch.empty(rows, top, device=x.device)
        s2d2.score_logits(x.data_ptr(), _DTYPE[x.dtype], rows, vocab, x.stride(0), tokens.data_ptr(), top,
                          d_logprob=f[0].data_ptr(), d_rank=rank.data_ptr(), d_lse=f[1].data_ptr(), d_entropy=f[2].data_ptr(),
                          d_top_ids=out["top_ids"].data_ptr() if top else 0,
                          d_top_logprobs=out["top_logprobs"].data_ptr() if top else 0, stream=stream)
        return out
    m, n, k = state["m"], state["n"], state["k"]
    x = state["x"]
    codes, scales = quantize(x)
    if op == "product":
        y = torch.empty(m, n, dtype=getattr(torch, state["y"]), device=x.device)
        s2d2.mxfp4_gemm(codes.data_ptr(), scales.data_ptr(), state["w_codes"].data_ptr(), state["w_scales"].data_ptr(),
                        y.data_ptr(), _DTYPE[y.dtype], m, n, k, stream=stream)
        return y
    f = torch.empty(3, m, device=x.device)
    ws = torch.empty(s2d2.mxfp4_score_workspace(m, n, k), dtype=torch.uint8, device=x.device)
    s2d2.mxfp4_score(codes.data_ptr(), scales.data_ptr(), state["w_codes"].data_ptr(), state["w_scales"].data_ptr(), m, n, k,
                     state["tokens"].data_ptr(), ws.data_ptr(), ws.numel(), d_logprob=f[0].data_ptr(), d_lse=f[1].data_ptr(),
                     d_entropy=f[2].data_ptr(), stream=stream)
    return dict(logprob=f[0], lse=f[1], entropy=f[2])


def run(state):
    return _own(state) if own else _plain(state)


# ---------------------------------------------------------------------------------------------------------------
# from the definition, in 64 bits
# ---------------------------------------------------------------------------------------------------------------
def _nearest(x):
    """The MXFP4 value of every element of x [rows, cols], by search over the e2m1 grid."""
    x = x.double()
    rows, cols = x.shape
    width = -(-cols // BLOCK) * BLOCK
    b = torch.zeros(rows, width, dtype=torch.float64, device=x.device)
    b[:, :cols] = x
    b = b.view(-1, BLOCK)
    largest = b.abs().max(dim=1, keepdim=True).values
    # frexp has mantissas in [0.5, 1): the largest power of two not above x is 2^(exponent - 1)
    e = torch.frexp(largest.clamp_min(2.0 ** -149)).exponent - 3
    unit = torch.ldexp(torch.ones_like(largest), e.clamp(-127, 127))
    v = b / unit
    size = v.abs()
    # the spacing of the grid around a magnitude: 0.5 below 2, 1 below 4, 2 above; round() takes ties to even multiples
    step = torch.where(size < 2.0, 0.5, torch.where(size < 4.0, 1.0, 2.0))
    near = (torch.round(size / step) * step).clamp_max(6.0)
    return (near * torch.sign(v) * unit).view(rows, width)[:, :cols]


def _weights(state):
    n, k = state["n"], state["k"]
    blocks = -(-k // BLOCK)
    quads = -(-blocks // 4)
    r = torch.arange(n, device="cuda").unsqueeze(1)
    b = torch.arange(blocks, device="cuda").unsqueeze(0)
    at = ((r // 128) * quads + b // 4) * 512 + (r % 32) * 16 + (r % 128) // 32 * 4 + b % 4
    scale = torch.exp2(state["w_scales"][at].double() - 127)
    codes = state["w_codes"].view(n, blocks, 16)
    w = torch.empty(n, blocks, 16, 2, dtype=torch.float64, device="cuda")
    grid = torch.tensor([0, .5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64, device="cuda")
    w[..., 0] = grid[(codes & 7).int()] * (1.0 - 2.0 * (codes >> 3 & 1))
    w[..., 1] = grid[(codes >> 4 & 7).int()] * (1.0 - 2.0 * (codes >> 7))
    return (w.view(n, blocks, 32) * scale.unsqueeze(2)).view(n, -1)[:, :k]


def _scores(x, tokens):
    # shifted by the row's maximum first: next to the lowest values of a type the logarithm would be lost
    shift = x.max(dim=1).values
    shift = torch.where(torch.isneginf(shift), 0.0, shift)
    x = x - shift.unsqueeze(1)
    log_sum = torch.logsumexp(x, 1)
    some = ~torch.isneginf(log_sum)
    entropy = torch.where(some, torch.special.entr(torch.softmax(x, 1)).sum(1), 0.0)
    taken = x[torch.arange(x.shape[0], device=x.device), tokens.long()]
    return torch.where(some, taken - log_sum, float("-inf")), shift + log_sum, entropy, shift + 0.0, log_sum


def exact(case, seed):
    state = prepare(case, seed)
    if case["op"] == "quantize":
        return _nearest(state["x"])
    if case["op"] == "score":
        x, tokens = state["logits"].double(), state["tokens"]
        logprob, lse, entropy, shift, log_sum = _scores(x, tokens)
        out = dict(logprob=logprob, rank=None, lse=lse, entropy=entropy)
        if case["top"]:
            value = torch.full((x.shape[0], case["top"]), float("-inf"), dtype=torch.float64, device=x.device)
            some = min(case["top"], x.shape[1])
            value[:, :some] = torch.topk(x, some, dim=1).values
            out["top_ids"] = None
            out["top_logprobs"] = torch.where(torch.isneginf(value), value, value - shift.unsqueeze(1) - log_sum.unsqueeze(1))
        return out
    y = _nearest(state["x"]) @ _weights(state).t()
    if case["op"] == "product":
        return y
    logprob, lse, entropy, _, _ = _scores(y, state["tokens"])
    return dict(logprob=logprob, lse=lse, entropy=entropy)
