"""Plain 64-bit restatements of the attention-block operators, and batches for their tests (torch, on any device)."""
import math

import torch


def frequencies(rot, base=1e6):
    return base ** (-2.0 * torch.arange(rot // 2, dtype=torch.float64) / rot)


def rope(x, pos, freqs, rot, layout="half", scale=1.0, gain=None, eps=1e-6):
    """x [rows, heads, dim] fp64: (result, size of the pair that an element belongs to, for tolerances)."""
    x = x.double()
    if gain is not None:
        x = x / torch.sqrt((x * x).mean(2, keepdim=True) + eps) * gain.double()
    a = pos.double()[:, None, None] * freqs.to(x.device)
    c, s = torch.cos(a) * scale, torch.sin(a) * scale
    i = torch.arange(rot // 2, device=x.device)
    lo, hi = (i, i + rot // 2) if layout == "half" else (2 * i, 2 * i + 1)
    y, size = x.clone(), x.abs()
    y[..., lo] = x[..., lo] * c - x[..., hi] * s
    y[..., hi] = x[..., hi] * c + x[..., lo] * s
    size[..., lo] = size[..., hi] = torch.hypot(x[..., lo], x[..., hi]) * abs(scale)
    return y, size


def rope_tolerance(want, size, dtype):
    """The angle is off by 2^-24 of half a turn at most (2^-22.3), cosine, sine and the two products by a few 2^-24; a norm adds a sum
    of up to 512 squares in a tree of at most 64 steps per thread (64 2^-24 / 2 of the size), a root and a quotient: 2^-18 of the pair in all.
    Then one rounding to the output's type."""
    return 2.0 ** -18 * size + want.abs() * torch.finfo(dtype).eps / 2


class Batch:
    """Sequences of (new rows, cached tokens with them) over a paged cache with poisoned spare room."""

    def __init__(self, lens, heads, kv_heads, dim, page=64, order="head", spare=0, seed=0, device="cuda", poison=float("nan"), q_pad=0, gap=0,
                 n_spare_pages=2):
        g = torch.Generator(device=device).manual_seed(seed)
        self.lens, self.heads, self.kv_heads, self.dim, self.page, self.order = lens, heads, kv_heads, dim, page, order
        self.first = [0]
        for n, _ in lens:
            self.first.append(self.first[-1] + n)
        self.n_rows = self.first[-1] + spare
        need = [-(-kv // page) for _, kv in lens]
        self.n_pages = sum(need) + n_spare_pages
        self.max_pages = max([1] + need) + 1
        self.table = torch.full((len(lens), self.max_pages), -7, dtype=torch.int32, device=device)
        perm = torch.randperm(self.n_pages, generator=g, device=device).int()
        at = 0
        for s, k in enumerate(need):
            self.table[s, :k] = perm[at:at + k]
            at += k
        shape = (self.n_pages, 2, kv_heads, page, dim + gap) if order == "head" else (self.n_pages, 2, page, kv_heads, dim + gap)
        self.cache = torch.full(shape, poison, dtype=torch.bfloat16, device=device)
        both = (self.cache if order == "head" else self.cache.transpose(2, 3))[..., :dim]
        self.k, self.v = both[:, 0], both[:, 1]                    # [page, head, token, dim]
        rnd = lambda *s: torch.randn(*s, generator=g, device=device)
        self.keys = [rnd(kv, kv_heads, dim).bfloat16() for _, kv in lens]
        self.values = [rnd(kv, kv_heads, dim).bfloat16() for _, kv in lens]
        self.write()
        self.q_buf = (rnd(self.n_rows, heads * dim + q_pad) * 1.5).bfloat16()
        self.q = self.q_buf[:, :heads * dim].unflatten(1, (heads, dim))
        self.row0 = torch.tensor(self.first, dtype=torch.int32, device=device)
        self.kv_len = torch.tensor([kv for _, kv in lens], dtype=torch.int32, device=device)

    def places(self, s):
        j = torch.arange(self.lens[s][1], device=self.cache.device)
        return self.table[s, j // self.page].long(), j % self.page

    def write(self):
        for s in range(len(self.lens)):
            page, tok = self.places(s)
            self.k.transpose(1, 2)[page, tok] = self.keys[s]
            self.v.transpose(1, 2)[page, tok] = self.values[s]

    def kv(self, m):
        return m.PagedKV(self.k.data_ptr(), self.v.data_ptr(), self.n_pages, self.page, self.kv_heads, self.dim, page_stride=self.k.stride(0),
                         head_stride=self.k.stride(1), token_stride=self.k.stride(2))

    def rows(self, m, max_rows=None):
        if max_rows is None:
            max_rows = max([1] + [n for n, _ in self.lens])
        return m.Rows(self.n_rows, len(self.lens), self.row0.data_ptr(), self.kv_len.data_ptr(), self.table.data_ptr(), self.max_pages, max_rows)

    def attend(self, m, mask_block=1, row_mask=None, scale=None, lse=True, max_rows=None, out_pad=0, stream=None, ws=None):
        """(out, lse) of the operator; rows that it must leave alone hold 7."""
        dev = self.cache.device
        out = torch.full((self.n_rows, self.heads * self.dim + out_pad), 7.0, dtype=torch.bfloat16, device=dev)
        lse_out = torch.full((self.n_rows, self.heads), 7.0, device=dev) if lse else None
        rows, kv = self.rows(m, max_rows), self.kv(m)
        if ws is None:
            ws = torch.full((m.paged_attention_workspace(rows, kv, self.heads) + 16,), 0xFF, dtype=torch.uint8, device=dev)
        m.paged_attention(self.q_buf.data_ptr(), out.data_ptr(), self.heads, rows, kv, ws.data_ptr(), ws.numel(), mask_block=mask_block,
                          d_row_mask=0 if row_mask is None else row_mask.data_ptr(), scale=scale, d_lse=lse_out.data_ptr() if lse else 0,
                          q_stride=self.q_buf.stride(0), out_stride=out.stride(0),
                          stream=torch.cuda.current_stream().cuda_stream if stream is None else stream)
        if out_pad:
            assert (out[:, self.heads * self.dim:] == 7).all()
        return out[:, :self.heads * self.dim].unflatten(1, (self.heads, self.dim)), lse_out

    def seen(self, s, mask_block=1, row_mask=None):
        """[n, kv] truth values: what each row of sequence s sees."""
        n, kv = self.lens[s]
        dev = self.cache.device
        j, i = torch.arange(kv, device=dev)[None], torch.arange(n, device=dev)[:, None]
        if row_mask is not None:
            b = j - (kv - n)
            bits = (row_mask[self.first[s]:self.first[s] + n, None] >> b.clamp(0, 63)) & 1
            return (b < 0) | ((b < 64) & (bits == 1))
        p = kv - n + i
        if mask_block == 0:
            return torch.ones(n, kv, dtype=torch.bool, device=dev)
        return (p >= 0) & (j < (torch.div(p, mask_block, rounding_mode="floor") + 1) * mask_block)

    def want(self, mask_block=1, row_mask=None, scale=None):
        """(out, lse, tolerance of out, tolerance of lse) in fp64; rows of no sequence hold 7 with tolerance 0.

        Tolerances.  A score is a sum of dim products in fp32, each addition off by at most 2^-23 of the sum of magnitudes (the tensor core
        may cut off): ds = dim 2^-23 scale |q| |k|, plus 2^-22 of the score for the change of base.  It and the exponential (2^-22)
        change a probability by that factor, in the numerator and in the sum.  Rounding probabilities to bf16 changes each by at
        most 2^-8 of itself, adding up to kv of them in fp32 by kv 2^-23.  With A = sum p |v| / sum p the output is off by that times A, and
        by one rounding to bf16."""
        dev, group = self.cache.device, self.heads // self.kv_heads
        scale = self.dim ** -0.5 if scale is None else scale
        out = torch.full((self.n_rows, self.heads, self.dim), 7.0, dtype=torch.float64, device=dev)
        lse = torch.full((self.n_rows, self.heads), 7.0, dtype=torch.float64, device=dev)
        tol, tol_lse = torch.zeros_like(out), torch.zeros_like(lse)
        for s, (n, kv) in enumerate(self.lens):
            if not n:
                continue
            at = slice(self.first[s], self.first[s] + n)
            seen = self.seen(s, mask_block, row_mask)
            for h in range(self.heads):
                q = self.q[at, h].double()
                k, v = self.keys[s][:, h // group].double(), self.values[s][:, h // group].double()
                x = torch.where(seen, q @ k.t() * scale, -math.inf)
                big = torch.where(seen, q.abs() @ k.abs().t() * scale, 0.0)
                top = x.amax(1, keepdim=True) if kv else torch.full((n, 1), -math.inf, dtype=torch.float64, device=dev)
                top0 = torch.where(torch.isneginf(top), 0.0, top)
                # keys that are not seen have no influence, whatever stands there
                e = torch.where(seen, torch.exp(x - top0), 0.0)
                total = e.sum(1, keepdim=True)
                if bool(torch.isfinite(v).all()):
                    num, mag = e @ v, e @ v.abs()
                else:
                    num = torch.stack([(e[r][seen[r], None] * v[seen[r]]).sum(0) for r in range(n)])
                    mag = torch.stack([(e[r][seen[r], None] * v[seen[r]].abs()).sum(0) for r in range(n)])
                out[at, h] = torch.where(total == 0, 0.0, num / total)
                lse[at, h] = (top0 + torch.log(total))[:, 0]
                ds = self.dim * 2.0 ** -23 * (big.amax(1, keepdim=True) if kv else 0.0) + 2.0 ** -21
                tol[at, h] = torch.where(total == 0, 0.0, mag / total) * (2.0 ** -8 + kv * 2.0 ** -23 + 2 * ds) + out[at, h].abs() * 2.0 ** -8
                tol_lse[at, h] = (ds + kv * 2.0 ** -24 + lse[at, h].abs()[:, None] * 2.0 ** -21 + 2.0 ** -20)[:, 0]
        return out, lse, tol, tol_lse

    def check(self, got, want):
        out, lse, tol, tol_lse = want
        for name, g, w, t in (("out", got[0], out, tol), ("lse", got[1], lse, tol_lse)):
            if g is None:
                continue
            g = g.double()
            same = (g == w) | (torch.isnan(g) & torch.isnan(w))
            err = torch.where(same, 0.0, (g - w).abs())
            bad = ~same & ~(err <= t)
            assert not bool(bad.any()), (name, int(bad.sum()), bad.nonzero()[:4].tolist(), g[bad][:4].tolist(), w[bad][:4].tolist(), t[bad][:4].tolist())


def verifier_masks(lens, spare=0, device="cuda"):
    """Row masks of a verifier pass: n / 2 drafted rows, causal, then a copy for each that sees the drafted rows in front of its own and itself."""
    out = []
    for n, _ in lens:
        half = n // 2
        for i in range(n):
            b = (1 << (i + 1)) - 1 if i < half else (1 << i) | ((1 << min(half, i - half)) - 1)
            out.append(b - (1 << 64) if b >> 63 else b)
    return torch.tensor(out + [0] * spare, dtype=torch.int64, device=device)
