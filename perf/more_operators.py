"""Cases of the attention block of a layer on a host's own buffers: rotary positions, norms of queries and keys with the rotation,
appending keys and values to a paged cache, and attention of new tokens over that cache.

A batch is a list of sequences. Rows (new tokens) of sequence s are row0[s] .. row0[s + 1]; with them its cache holds kv_len[s]
tokens, so that its n rows stand at cache indices kv_len - n .. kv_len - 1; index j is token j % page of page table[s][j // page].
Rows behind row0[-1] pad the batch and are left as they are.
"""
import math
import random

import torch

own = False

BASE = 1.0e6
EPS = 1.0e-6


# ---------------------------------------------------------------------------------------------------------------
# cases
# ---------------------------------------------------------------------------------------------------------------
def listed():
    return [
        # queries and keys of one token of the 8B-class model
        _rotate("rotate-1", rows=1),
        # a part of every head rotated, pairs side by side, frequencies spread for a long context, rows of a fused projection
        _rotate("rotate-partial", rows=2049, rot=64, layout="interleaved", scaling="yarn", far=131072, dtype="float32", pad=1024),
        # a ragged batch with the heads of a small model, in 32 bits, rows not aligned to vectors
        _rotate("norm-rotate-ragged", rows=333, heads=4, kv_heads=2, dim=64, norm=True, dtype="float32", pad=3),
        # a whole prompt of the 8B-class model
        _rotate("norm-rotate-8192", rows=8192, norm=True),
        # the masked rows of one block, projected in 32 bits by a 4-bit product
        _append("append-block", rows=8, context=1031, dtype="float32"),
        # prompts of different lengths in one batch, tokens side by side in small pages, a padded end
        _append("append-ragged", seqs=24, rows=700, context=900, spread=True, page=16, order="token", heads=16, kv_heads=4, spare=37),
        # one new token of one sequence
        _attend("attend-1", context=1221),
        # one new token for each of 64 sequences of very different lengths, some slots idle
        _attend("attend-tokens", seqs=64, context=16384, spread=True, page=16, order="token", heads=16, kv_heads=4, spare=3),
        # verifier rows of 32 blocks of 8 drafted tokens: the drafted tokens, then one masked copy of each
        _attend("attend-verify", seqs=32, rows=16, context=1206, mask="rows"),
        # the masked rows of one block behind a very long document
        _attend("attend-long", rows=8, context=131072, mask="full", lse=True),
        # a prompt, token by token
        _attend("attend-prompt", rows=4096, context=0),
        # chunks of several prompts, whole blocks of 32 at a time, heads of 64 with an odd group
        _attend("attend-chunks", seqs=5, rows=2500, context=20000, spread=True, mask="block", heads=12, kv_heads=4, dim=64, lse=True, spare=11),
    ]


def _rotate(name, rows, heads=32, kv_heads=8, dim=128, rot=0, layout="half", scaling="none", far=32768, norm=False, dtype="bfloat16", pad=0):
    return dict(name=name, op="rotate", rows=rows, heads=heads, kv_heads=kv_heads, dim=dim, rot=rot or dim, layout=layout, scaling=scaling,
                far=far, norm=norm, dtype=dtype, pad=pad)


def _append(name, seqs=1, rows=1, context=0, spread=False, page=64, order="head", heads=32, kv_heads=8, dim=128, rot=0, layout="half",
            scaling="none", norm=True, dtype="bfloat16", spare=0):
    return dict(name=name, op="append", seqs=seqs, rows=rows, context=context, spread=spread, page=page, order=order, heads=heads,
                kv_heads=kv_heads, dim=dim, rot=rot or dim, layout=layout, scaling=scaling, norm=norm, dtype=dtype, spare=spare)


def _attend(name, seqs=1, rows=1, context=0, spread=False, page=64, order="head", heads=32, kv_heads=8, dim=128, mask="causal", lse=False, spare=0):
    return dict(name=name, op="attend", seqs=seqs, rows=rows, context=context, spread=spread, page=page, order=order, heads=heads,
                kv_heads=kv_heads, dim=dim, mask=mask, lse=lse, spare=spare)


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["rotate", "append", "attend", "attend", "attend"])
    kv_heads = rng.choice([1, 2, 4, 5, 8])
    heads = kv_heads * rng.choice([1, 2, 3, 4, 6, 8])
    dim = rng.choice([32, 64, 80, 96, 128, 128])
    page, order = rng.choice([8, 16, 32, 64, 128]), rng.choice(["head", "token"])
    rot, layout = rng.choice([dim, dim, dim // 2]), rng.choice(["half", "interleaved"])
    scaling, norm, dtype = rng.choice(["none", "linear", "ntk", "yarn", "bands"]), rng.random() < 0.5, rng.choice(["float32", "bfloat16"])
    if op == "rotate":
        case = _rotate("", _log(rng, 1, 8192), heads, kv_heads, dim, rot, layout, scaling, _log(rng, 1000, 1000000), norm, dtype,
                       rng.choice([0, 0, 3, 64]))
        while work(case)["bytes"] > 160e6:
            case["rows"] //= 2
    else:
        seqs, context = _log(rng, 1, 64), _log(rng, 1, 131072) - 1
        if op == "append":
            case = _append("", seqs, _log(rng, 1, 2048), min(context, 4096), rng.random() < 0.7, page, order, heads, kv_heads, dim, rot, layout,
                           scaling, norm, dtype, rng.choice([0, 0, 5]))
        else:
            mask = rng.choice(["causal", "causal", "full", "block", "rows"])
            case = _attend("", seqs, _log(rng, 1, 64 if mask == "rows" else rng.choice([1, 64, 4096])), context, rng.random() < 0.7, page, order,
                           heads, kv_heads, dim, mask, rng.random() < 0.3, rng.choice([0, 0, 5]))
        while work(case)["bytes"] > 400e6 or work(case)["flops"] > 120e9 or case["seqs"] * case["rows"] > 16384:
            if case["seqs"] > 1:
                case["seqs"] //= 2
            else:
                case["rows"], case["context"] = max(1, case["rows"] // 2), case["context"] // 2
    del case["name"]
    return case


def _lengths(case):
    """(new tokens, cached tokens with them) of every sequence: the same for every seed."""
    n, kv = [], []
    rng = random.Random(",".join("%s=%s" % i for i in sorted(case.items()) if i[0] != "name"))
    for s in range(case["seqs"]):
        rows, context = case["rows"], case["context"]
        if case["spread"]:
            rows, context = _log(rng, max(1, rows / 16), rows), _log(rng, 1, context + 1) - 1
            if s % 16 == 5:
                rows = 0          # a slot that has nothing to do in this step
        n.append(rows)
        kv.append(context + rows)
    return n, kv


def _block(case):
    return {"causal": 1, "full": 0, "block": 32, "rows": 0}[case["mask"]]


def _pairs(case):
    """Pairs of a query and a key that it sees, and keys that anything sees."""
    pairs, keys = 0, 0
    for n, kv in zip(*_lengths(case)):
        if not n:
            continue
        keys += kv
        if case["mask"] == "rows":
            pairs += n * (kv - n) + n * (n + 1) // 4
        elif case["mask"] == "full":
            pairs += n * kv
        else:
            block = _block(case)
            pairs += sum(min(kv, (p // block + 1) * block) for p in range(kv - n, kv))
    return pairs, keys


def work(case):
    heads, kv_heads, dim = case["heads"], case["kv_heads"], case["dim"]
    if case["op"] == "rotate":
        n = case["rows"] * (heads + kv_heads)
        size = 4 if case["dtype"] == "float32" else 2
        return {"bytes": 2 * n * dim * size + 4 * case["rows"], "flops": n * (3 * case["rot"] + (4 * dim if case["norm"] else 0))}
    if case["op"] == "append":
        rows = sum(_lengths(case)[0])
        size = 4 if case["dtype"] == "float32" else 2
        return {"bytes": rows * (heads + 2 * kv_heads) * dim * (size + 2),
                "flops": rows * (heads + kv_heads) * (3 * case["rot"] + (4 * dim if case["norm"] else 0))}
    pairs, keys = _pairs(case)
    rows = sum(_lengths(case)[0])
    return {"bytes": 4 * keys * kv_heads * dim + rows * heads * (4 * dim + (4 if case["lse"] else 0)), "flops": 4 * pairs * heads * dim}


# ---------------------------------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------------------------------
def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def randn(*shape):
        return torch.randn(*shape, generator=gen, device="cuda")

    state = dict(case)
    heads, kv_heads, dim = case["heads"], case["kv_heads"], case["dim"]
    if case["op"] != "attend":
        state["freqs"], state["scale"] = _frequencies(case["rot"], case["scaling"])
        state["freqs"] = torch.tensor(state["freqs"], dtype=torch.float64, device="cuda")
        state["q_gain"], state["k_gain"] = (1 + 0.2 * randn(dim), 1 + 0.2 * randn(dim)) if case["norm"] else (None, None)
    if case["op"] == "rotate":
        rows, wide = case["rows"], (heads + kv_heads) * dim
        # one projection holds queries and keys of a row side by side
        x = (randn(rows, wide + case["pad"]) * torch.exp(0.5 * randn(rows, 1))).to(getattr(torch, case["dtype"]))
        state["q"], state["k"] = x[:, :heads * dim].unflatten(1, (heads, dim)), x[:, heads * dim:wide].unflatten(1, (kv_heads, dim))
        state["pos"] = torch.randint(0, case["far"], (rows,), generator=gen, device="cuda", dtype=torch.int32)
        if own:
            state["rope"] = _own_rope(state)
        return state
    n, kv = _lengths(case)
    page = case["page"]
    need = [-(-k // page) for k in kv]
    pages, rows = sum(need) + 3, sum(n) + case["spare"]
    order = torch.randperm(pages, generator=gen, device="cuda").to(torch.int32)
    table = torch.full((case["seqs"], max(1, max(need))), -1, dtype=torch.int32, device="cuda")
    at = 0
    for s, k in enumerate(need):
        table[s, :k] = order[at:at + k]
        at += k
    first = [0]
    for k in n:
        first.append(first[-1] + k)
    state.update(n=n, kv=kv, first=first, pages=pages, table=table)
    state["row0"] = torch.tensor(first, dtype=torch.int32, device="cuda")
    state["kv_len"] = torch.tensor(kv, dtype=torch.int32, device="cuda")
    # keys and values of a page together; within them either the tokens of a head or the heads of a token are neighbours
    shape = (pages, 2, kv_heads, page, dim) if case["order"] == "head" else (pages, 2, page, kv_heads, dim)
    cache = torch.empty(shape, dtype=torch.bfloat16, device="cuda")
    for i in range(0, pages, 4096):
        cache[i:i + 4096] = randn(*cache[i:i + 4096].shape).to(torch.bfloat16)
    state["cache"] = cache
    both = cache if case["order"] == "head" else cache.transpose(2, 3)
    state["keys"], state["values"] = both[:, 0], both[:, 1]                   # [page, head, token, dim]
    if case["op"] == "append":
        x = randn(rows, (heads + 2 * kv_heads) * dim).to(getattr(torch, case["dtype"]))
        state["q"], state["k"], state["v"] = (t.unflatten(1, (-1, dim)) for t in x.split([heads * dim, kv_heads * dim, kv_heads * dim], 1))
        state["q_out"] = torch.zeros(rows, heads, dim, dtype=torch.bfloat16, device="cuda")
    else:
        # queries a little longer than unit normal: some rows look at few keys, most at many
        state["q"] = (randn(rows, heads, dim) * torch.exp(0.5 * randn(rows, heads, 1))).to(torch.bfloat16)
        state["out"] = torch.zeros_like(state["q"])
        state["lse_out"] = torch.zeros(rows, heads, device="cuda") if case["lse"] else None
        state["row_mask"] = None
        if case["mask"] == "rows":
            state["row_mask"] = torch.tensor([_verifier_mask(k, i) for k in n for i in range(k)] + [0] * case["spare"], dtype=torch.int64, device="cuda")
    if own:
        _own_batch(state)
    return state


def _verifier_mask(n, i):
    """Bits of the new rows that row i of n sees: the first half causally; a row of the second half itself and the first half up to
    the token in front of the one that it stands for."""
    half = n // 2
    bits = (1 << i + 1) - 1 if i < half else 1 << i | (1 << min(half, i - half)) - 1
    return bits - (1 << 64) if bits >> 63 else bits


def _frequencies(rot, scaling, factor=8.0, original=16384.0):
    """Radians per position of each pair, and what queries and keys are multiplied by."""
    plain = [BASE ** (-2.0 * i / rot) for i in range(rot // 2)]
    if scaling == "linear":
        return [f / factor for f in plain], 1.0
    if scaling == "ntk":
        base = BASE * factor ** (rot / (rot - 2.0))
        return [base ** (-2.0 * i / rot) for i in range(rot // 2)], 1.0
    if scaling == "yarn":
        # pairs that turn more than 32 times in the original length stay, those that turn less than once are slowed down
        low, high = (rot * math.log(original / (t * 2 * math.pi)) / (2 * math.log(BASE)) for t in (32.0, 1.0))
        low, high = max(math.floor(low), 0), min(math.ceil(high), rot - 1)
        high = high + 0.001 if high == low else high
        ramp = [min(max((i - low) / (high - low), 0.0), 1.0) for i in range(rot // 2)]
        return [f / factor * r + f * (1 - r) for f, r in zip(plain, ramp)], 0.1 * math.log(factor) + 1.0
    if scaling == "bands":
        # the same between 4 turns and 1 turn, the ramp linear in the turns
        keep = [min(max((original * f / (2 * math.pi) - 1.0) / 3.0, 0.0), 1.0) for f in plain]
        return [f / factor * (1 - r) + f * r for f, r in zip(plain, keep)], 1.0
    return plain, 1.0


# ---------------------------------------------------------------------------------------------------------------
# plain forms
# ---------------------------------------------------------------------------------------------------------------
def _turn(x, gain, pos, state):
    """x [rows, heads, dim] normed over each head and rotated, in 32 bits."""
    x = x.float()
    if gain is not None:
        x = x * torch.rsqrt((x * x).mean(2, keepdim=True) + EPS) * gain
    # far positions: the angle in 64 bits
    angle = pos.double().unsqueeze(1) * state["freqs"]
    cos, sin = (torch.cos(angle) * state["scale"]).float().unsqueeze(1), (torch.sin(angle) * state["scale"]).float().unsqueeze(1)
    rot = state["rot"]
    turned, rest = x[:, :, :rot], x[:, :, rot:]
    if state["layout"] == "half":
        a, b = turned[:, :, :rot // 2], turned[:, :, rot // 2:]
        return torch.cat([a * cos - b * sin, b * cos + a * sin, rest], 2)
    a, b = turned[:, :, 0::2], turned[:, :, 1::2]
    return torch.cat([torch.stack([a * cos - b * sin, b * cos + a * sin], 3).flatten(2), rest], 2)


def _places(state):
    """Of every row that belongs to a sequence: its cache index, page and token in the page."""
    rows = state["first"][-1]
    row = torch.arange(rows, device="cuda", dtype=torch.int32)
    seq = torch.searchsorted(state["row0"], row, right=True).long() - 1
    index = (state["kv_len"][seq] - state["row0"][seq + 1] + row).long()
    return index, state["table"][seq, index // state["page"]].long(), index % state["page"]


def _plain(state):
    if state["op"] == "rotate":
        dtype = state["q"].dtype
        return dict(q=_turn(state["q"], state["q_gain"], state["pos"], state).to(dtype), k=_turn(state["k"], state["k_gain"], state["pos"], state).to(dtype))
    if state["op"] == "append":
        index, page, token = _places(state)
        rows = state["first"][-1]
        state["q_out"][:rows] = _turn(state["q"][:rows], state["q_gain"], index, state).to(torch.bfloat16)
        state["keys"].transpose(1, 2)[page, token] = _turn(state["k"][:rows], state["k_gain"], index, state).to(torch.bfloat16)
        state["values"].transpose(1, 2)[page, token] = state["v"][:rows].to(torch.bfloat16)
        return dict(q=state["q_out"], cache=state["cache"])
    heads, kv_heads, dim, page = (state[k] for k in ("heads", "kv_heads", "dim", "page"))
    group, scale = heads // kv_heads, dim ** -0.5
    for s, (n, kv) in enumerate(zip(state["n"], state["kv"])):
        if not n:
            continue
        table = state["table"][s, :-(-kv // page)].long()
        keys, values = (state[t][table].transpose(1, 2).reshape(-1, kv_heads, dim)[:kv].float().permute(1, 2, 0) for t in ("keys", "values"))
        j = torch.arange(kv, device="cuda")
        step = max(1, 2 ** 28 // (heads * kv))
        for i in range(0, n, step):
            m = min(step, n - i)
            at = slice(state["first"][s] + i, state["first"][s] + i + m)
            q = state["q"][at].float().view(m, kv_heads, group, dim).permute(1, 2, 0, 3).reshape(kv_heads, group * m, dim)
            x = torch.bmm(q, keys).view(kv_heads, group, m, kv) * scale
            p = kv - n + i + torch.arange(m, device="cuda").unsqueeze(1)
            if state["mask"] == "rows":
                new = (j - (kv - n)).clamp(0, 63)
                seen = (j < kv - n) | ((state["row_mask"][at].unsqueeze(1) >> new & 1) == 1)
                x = torch.where(seen, x, float("-inf"))
            elif state["mask"] != "full":
                block = _block(state)
                x = torch.where(j < (p // block + 1) * block, x, float("-inf"))
            top = x.amax(3, keepdim=True)
            top = torch.where(torch.isneginf(top), 0.0, top)
            e = torch.exp(x - top)
            total = e.sum(3, keepdim=True)
            y = torch.bmm(e.view(kv_heads, group * m, kv), values.transpose(1, 2)).view(kv_heads, group, m, dim)
            y = torch.where(total > 0, y / total, 0.0)
            state["out"][at] = y.permute(2, 0, 1, 3).reshape(m, heads, dim).to(torch.bfloat16)
            if state["lse"]:
                state["lse_out"][at] = (top + torch.log(total)).squeeze(3).permute(2, 0, 1).reshape(m, heads)
    return dict(out=state["out"], lse=state["lse_out"]) if state["lse"] else state["out"]


# ---------------------------------------------------------------------------------------------------------------
# the framework's calls
# ---------------------------------------------------------------------------------------------------------------
_DTYPE = {torch.float32: "fp32", torch.bfloat16: "bf16"}


def _own_rope(state):
    import paper_2603_25702_b200 as s2d2
    freqs, scale = s2d2.rope_frequencies(state["rot"], BASE, state["scaling"], factor=8.0, original_len=16384,
                                         turns_fast=32.0 if state["scaling"] == "yarn" else 4.0, turns_slow=1.0)
    state["own_freqs"] = torch.from_numpy(freqs).cuda()
    gains = (state["q_gain"].data_ptr(), state["k_gain"].data_ptr()) if state["norm"] else (0, 0)
    return s2d2.Rope(state["own_freqs"].data_ptr(), state["rot"], state["layout"], scale, d_q_gain=gains[0], d_k_gain=gains[1], eps=EPS)


def _own_batch(state):
    import paper_2603_25702_b200 as s2d2
    keys, values, table = state["keys"], state["values"], state["table"]
    state["kv_cache"] = s2d2.PagedKV(keys.data_ptr(), values.data_ptr(), state["pages"], state["page"], state["kv_heads"], state["dim"],
                                     page_stride=keys.stride(0), head_stride=keys.stride(1), token_stride=keys.stride(2))
    state["batch"] = s2d2.Rows(state["q"].shape[0], state["seqs"], state["row0"].data_ptr(), state["kv_len"].data_ptr(), table.data_ptr(),
                               table.shape[1], max_rows=max(state["n"]))
    if state["op"] == "append":
        state["rope"] = _own_rope(state)
    else:
        size = s2d2.paged_attention_workspace(state["batch"], state["kv_cache"], state["heads"])
        state["workspace"] = torch.empty(size, dtype=torch.uint8, device="cuda")


def _own(state):
    import paper_2603_25702_b200 as s2d2
    stream = torch.cuda.current_stream().cuda_stream
    heads, kv_heads, dim = state["heads"], state["kv_heads"], state["dim"]
    q = state["q"]
    if state["op"] == "rotate":
        k = state["k"]
        q_out, k_out = (torch.empty(t.shape, dtype=t.dtype, device=t.device) for t in (q, k))
        s2d2.qk_rope(q.data_ptr(), q_out.data_ptr(), heads, k.data_ptr(), k_out.data_ptr(), kv_heads, _DTYPE[q.dtype], q.shape[0], dim,
                     state["pos"].data_ptr(), state["rope"], q_stride=q.stride(0), k_stride=k.stride(0), stream=stream)
        return dict(q=q_out, k=k_out)
    if state["op"] == "append":
        k, v = state["k"], state["v"]
        s2d2.kv_append(k.data_ptr(), v.data_ptr(), _DTYPE[q.dtype], state["batch"], state["kv_cache"], state["rope"], k_stride=k.stride(0),
                       v_stride=v.stride(0), d_q=q.data_ptr(), d_q_out=state["q_out"].data_ptr(), n_q_heads=heads, q_stride=q.stride(0), stream=stream)
        return dict(q=state["q_out"], cache=state["cache"])
    work = state["workspace"]
    s2d2.paged_attention(q.data_ptr(), state["out"].data_ptr(), heads, state["batch"], state["kv_cache"], work.data_ptr(), work.numel(),
                         mask_block=_block(state), d_row_mask=state["row_mask"].data_ptr() if state["mask"] == "rows" else 0,
                         d_lse=state["lse_out"].data_ptr() if state["lse"] else 0, stream=stream)
    return dict(out=state["out"], lse=state["lse_out"]) if state["lse"] else state["out"]


def run(state):
    return _own(state) if own else _plain(state)


# ---------------------------------------------------------------------------------------------------------------
# from the definition, in 64 bits
# ---------------------------------------------------------------------------------------------------------------
def _exact_turn(x, gain, pos, state):
    x = x.double()
    if gain is not None:
        x = x / torch.sqrt((x ** 2).sum(-1, keepdim=True) / x.shape[-1] + EPS) * gain.double()
    rot, pairs = state["rot"], state["rot"] // 2
    # a pair is a complex number, its rotation a product with one of length `scale`
    turn = torch.polar(torch.full((pos.numel(), 1, pairs), state["scale"], dtype=torch.float64, device=x.device), (pos.double()[:, None] * state["freqs"])[:, None])
    i = torch.arange(pairs, device=x.device)
    first, second = (i, i + pairs) if state["layout"] == "half" else (2 * i, 2 * i + 1)
    z = torch.complex(x[..., first], x[..., second]) * turn
    y = x.clone()
    y[..., first], y[..., second] = z.real, z.imag
    return y


def exact(case, seed):
    state = prepare(case, seed)
    if case["op"] == "rotate":
        return {name: _exact_turn(state[name], state[name + "_gain"], state["pos"], state) for name in ("q", "k")}
    first, page = state["first"], case["page"]
    if case["op"] == "append":
        q, cache = state["q_out"].double(), state["cache"].double()
        both = cache if case["order"] == "head" else cache.transpose(2, 3)
        for s, (n, kv) in enumerate(zip(state["n"], state["kv"])):
            if not n:
                continue
            rows = slice(first[s], first[s] + n)
            index = torch.arange(kv - n, kv, device="cuda")
            q[rows] = _exact_turn(state["q"][rows], state["q_gain"], index, state)
            k = _exact_turn(state["k"][rows], state["k_gain"], index, state)
            for b in range((kv - n) // page, (kv - 1) // page + 1):
                lo, hi = max(b * page, kv - n), min((b + 1) * page, kv)
                to, from_ = both[int(state["table"][s, b])], slice(lo - (kv - n), hi - (kv - n))
                to[0, :, lo - b * page:hi - b * page] = k[from_].transpose(0, 1)
                to[1, :, lo - b * page:hi - b * page] = state["v"][rows][from_].double().transpose(0, 1)
        return dict(q=q, cache=cache)
    heads, kv_heads, dim = case["heads"], case["kv_heads"], case["dim"]
    out = state["out"].double()
    lse = torch.zeros(out.shape[:2], dtype=torch.float64, device="cuda")
    for s, (n, kv) in enumerate(zip(state["n"], state["kv"])):
        if not n:
            continue
        table = state["table"][s, :(kv + page - 1) // page].long()
        for g in range(kv_heads):
            keys, values = (state[t][table, g].flatten(0, 1)[:kv].double() for t in ("keys", "values"))
            mine = slice(g * (heads // kv_heads), (g + 1) * (heads // kv_heads))
            step = max(1, 2 ** 26 // (kv * (heads // kv_heads)))
            for lo in range(0, n, step):
                hi = min(n, lo + step)
                score = torch.einsum("ihd,jd->ihj", state["q"][first[s] + lo:first[s] + hi, mine].double(), keys) / math.sqrt(dim)
                i, j = torch.arange(lo, hi, device="cuda")[:, None], torch.arange(kv, device="cuda")[None]
                old = kv - n
                if case["mask"] == "causal":
                    hidden = j > old + i
                elif case["mask"] == "block":
                    hidden = j // 32 > torch.div(old + i, 32, rounding_mode="floor")
                elif case["mask"] == "rows":
                    # drafted tokens see one another causally; a masked copy sees itself and the drafted tokens in front of its own
                    half, a = n // 2, j - old
                    drafted = torch.where(i < half, a <= i, a < torch.clamp(i - half, max=half))
                    hidden = (a >= 0) & ~(drafted | (a == i))
                else:
                    hidden = torch.zeros(hi - lo, kv, dtype=torch.bool, device="cuda")
                score.masked_fill_(hidden[:, None], float("-inf"))
                norm = torch.logsumexp(score, 2)
                lse[first[s] + lo:first[s] + hi, mine] = norm
                out[first[s] + lo:first[s] + hi, mine] = torch.einsum("ihj,jd->ihd", torch.exp(score - norm[..., None]), values)
    return dict(out=out, lse=lse) if case["lse"] else out
