"""The attention block as a host runs it: projection, append with norms and rotation, attention, output projection; and the ends of its waits."""
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

from tests import attention_util as au  # noqa: E402


@pytest.fixture(scope="module")
def s2d2():
    import paper_2603_25702_b200 as m
    return m


def near(got, want, size):
    bad = ~((got.double() - want).abs() <= au.rope_tolerance(want, size, torch.bfloat16))
    assert not bool(bad.any()), (int(bad.sum()), bad.nonzero()[:4].tolist(), got[bad][:4].tolist(), want[bad][:4].tolist())


class Layer:
    """A layer's attention on buffers of a host's own: 4-bit projections, a paged cache, one workspace."""

    def __init__(self, s2d2, batch, hidden, seed):
        b, self.m, self.b, self.hidden = batch, s2d2, batch, hidden
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.dim, self.hq, self.hk = b.dim, b.heads, b.kv_heads
        self.wide = (self.hq + 2 * self.hk) * self.dim
        self.freqs = au.frequencies(self.dim).cuda()
        self.gains = [torch.rand(self.dim, generator=g, device="cuda") + 0.5 for _ in range(2)]
        self.rope = s2d2.Rope(self.freqs.data_ptr(), self.dim, d_q_gain=self.gains[0].data_ptr(), d_k_gain=self.gains[1].data_ptr())
        u8 = lambda n: torch.empty(n, dtype=torch.uint8, device="cuda")
        f32 = lambda *s: torch.empty(*s, device="cuda")
        self.weights = []
        for n, k in ((self.wide, hidden), (hidden, self.hq * self.dim)):
            w, (codes, scales) = torch.randn(n, k, generator=g, device="cuda") / 8, (u8(x) for x in s2d2.mxfp4_sizes(n, k))
            s2d2.mxfp4_quantize(w.data_ptr(), "fp32", n, k, k, codes.data_ptr(), scales.data_ptr(), torch.cuda.current_stream().cuda_stream)
            self.weights.append((codes, scales))
        self.x, self.qkv, self.y = f32(b.n_rows, hidden), f32(b.n_rows, self.wide), f32(b.n_rows, hidden)
        self.codes = [[u8(x) for x in s2d2.mxfp4_sizes(b.n_rows, k)] for k in (hidden, self.hq * self.dim)]
        self.q = torch.zeros(b.n_rows, self.hq, self.dim, dtype=torch.bfloat16, device="cuda")
        self.o = torch.zeros_like(self.q)
        self.lse = f32(b.n_rows, self.hq)
        self.rows, self.kv = b.rows(s2d2), b.kv(s2d2)
        self.ws = u8(s2d2.paged_attention_workspace(self.rows, self.kv, self.hq))
        torch.cuda.synchronize()

    def step(self, mask_block, row_mask, pos, st):
        m, n = self.m, self.b.n_rows
        ptr = lambda t: 0 if t is None else t.data_ptr()

        def product(x, dtype, k, i, y, width):
            codes, scales = self.codes[i]
            m.mxfp4_quantize(x.data_ptr(), dtype, n, k, k, codes.data_ptr(), scales.data_ptr(), st)
            m.mxfp4_gemm(codes.data_ptr(), scales.data_ptr(), self.weights[i][0].data_ptr(), self.weights[i][1].data_ptr(), y.data_ptr(), "fp32",
                         n, width, k, width, stream=st)
        product(self.x, "fp32", self.hidden, 0, self.qkv, self.wide)
        at = lambda h: self.qkv.data_ptr() + 4 * h * self.dim
        m.kv_append(at(self.hq), at(self.hq + self.hk), "fp32", self.rows, self.kv, self.rope, k_stride=self.wide, v_stride=self.wide, d_pos=ptr(pos),
                    d_q=at(0), d_q_out=self.q.data_ptr(), n_q_heads=self.hq, q_stride=self.wide, stream=st)
        m.paged_attention(self.q.data_ptr(), self.o.data_ptr(), self.hq, self.rows, self.kv, self.ws.data_ptr(), self.ws.numel(), mask_block=mask_block,
                          d_row_mask=ptr(row_mask), d_lse=self.lse.data_ptr(), stream=st)
        product(self.o, "bf16", self.hq * self.dim, 1, self.y, self.hidden)

    def check(self, mask_block, row_mask, pos):
        """Each operator against the formula on what the one in front of it left."""
        b, hq, hk, dim = self.b, self.hq, self.hk, self.dim
        parts = self.qkv.unflatten(1, (hq + 2 * hk, dim))
        for s, (n, kv) in enumerate(b.lens):
            if not n:
                continue
            at = slice(b.first[s], b.first[s] + n)
            p = torch.arange(kv - n, kv, device="cuda") if pos is None else pos[at]
            near(self.q[at], *au.rope(parts[at, :hq], p, self.freqs, dim, gain=self.gains[0]))
            page, tok = b.places(s)
            new, kept = max(kv - n, 0), max(n - kv, 0)                    # (rows in front of the cache's first index have no place)
            near(b.k.transpose(1, 2)[page, tok][new:], *(t[kept:] for t in au.rope(parts[at, hq:hq + hk], p, self.freqs, dim, gain=self.gains[1])))
            assert torch.equal(b.v.transpose(1, 2)[page, tok][new:], parts[at, hq + hk:][kept:].bfloat16())
            b.keys[s], b.values[s] = b.k.transpose(1, 2)[page, tok], b.v.transpose(1, 2)[page, tok]
        b.q = self.q
        got = self.o.clone(), self.lse.clone()
        got[0][b.first[-1]:], got[1][b.first[-1]:] = 7, 7               # padding: a host's own
        b.check(got, b.want(mask_block, row_mask))


# masked blocks of the draft, a verifier pass with copies that share positions, single tokens, a ragged prompt with idle slots and padding
CASES = {"draft": ([(8, 1031), (8, 72), (8, 8)], 0, "head", 0), "verify": ([(16, 320), (16, 40), (8, 8)], "rows", "head", 0),
         "tokens": ([(1, 700), (0, 12), (1, 1), (1, 64), (1, 65)], 1, "token", 3), "prompt": ([(300, 300), (0, 0), (70, 500), (33, 1)], 1, "token", 2),
         "blocks": ([(64, 640), (40, 40)], 32, "head", 0)}


@pytest.mark.parametrize("name", list(CASES))
@pytest.mark.parametrize("heads,kv_heads,dim", [(8, 2, 128), (6, 2, 64)])
def test_layer(s2d2, name, heads, kv_heads, dim):
    """Eager, with a pause behind every call, and as a graph on a side stream with two other inputs in the same buffers."""
    lens, mask, order, spare = CASES[name]
    b = au.Batch(lens, heads, kv_heads, dim, order=order, spare=spare)
    layer = Layer(s2d2, b, 256, 1)
    row_mask = pos = None
    if mask == "rows":
        row_mask, mask = au.verifier_masks(lens, spare), 0
        pos = torch.cat([torch.arange(n) % (n // 2) + kv - n for n, kv in lens]).int().cuda()
    empty = b.cache.clone()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    layer.step(mask, row_mask, pos, side.cuda_stream)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        layer.step(mask, row_mask, pos, side.cuda_stream)
    for seed in (2, 3):
        results = []
        for how in ("eager", "graph", "eager again"):
            b.cache.copy_(empty)
            layer.x.normal_(generator=torch.Generator(device="cuda").manual_seed(seed))
            for t in (layer.q, layer.o, layer.lse, layer.y):
                t.zero_()
            layer.ws.fill_(0xFF)
            torch.cuda.synchronize()
            if how == "graph":
                graph.replay()
            else:
                layer.step(mask, row_mask, pos, side.cuda_stream)
            torch.cuda.synchronize()
            results.append([t.clone() for t in (b.cache.nan_to_num(nan=3.0), layer.q, layer.o, layer.lse, layer.y)])
        assert all(torch.equal(x, y) for r in results[1:] for x, y in zip(r, results[0]))
        layer.check(mask, row_mask, pos)
    s2d2.ops_status(side.cuda_stream)


def test_two_graphs_at_once_on_one_cache(s2d2):
    """Two heads' worth of queries over the same cache, captured with their own workspaces and replayed together."""
    b = au.Batch([(1, 3000), (40, 900)], 8, 2, 128)
    want = b.want()
    rows, kv = b.rows(s2d2), b.kv(s2d2)
    streams, graphs, outs = [torch.cuda.Stream() for _ in range(2)], [], []
    s2d2.ops_status()
    keep = []
    for st in streams:
        o, lse = torch.zeros(b.n_rows, 8, 128, dtype=torch.bfloat16, device="cuda"), torch.zeros(b.n_rows, 8, device="cuda")
        ws = torch.full((s2d2.paged_attention_workspace(rows, kv, 8),), 0xFF, dtype=torch.uint8, device="cuda")
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=st):
            for _ in range(3):
                s2d2.paged_attention(b.q_buf.data_ptr(), o.data_ptr(), 8, rows, kv, ws.data_ptr(), ws.numel(), d_lse=lse.data_ptr(), stream=st.cuda_stream)
        graphs.append(graph), outs.append((o, lse)), keep.append(ws)
    for _ in range(5):
        for o, lse in outs:
            o.zero_(), lse.zero_()
        torch.cuda.synchronize()
        for st, graph in zip(streams, graphs):
            with torch.cuda.stream(st):
                graph.replay()
        torch.cuda.synchronize()
        for got in outs:
            b.check(got, want)


# items of one and two tiles, whole ones and ones that CTAs share; both sizes of heads
@pytest.mark.parametrize("lens,heads,kv_heads,dim", [([(1, 60)], 4, 2, 64), ([(1, 3000), (3, 200)], 8, 2, 128), ([(300, 700), (1, 40)], 4, 2, 64),
                                                     ([(0, 3), (500, 500)], 8, 2, 128)])
def test_attention_that_runs_out_is_nan_and_reported(s2d2, lens, heads, kv_heads, dim):
    from paper_2603_25702_b200 import binding
    b = au.Batch(lens, heads, kv_heads, dim, spare=2)
    stream = torch.cuda.current_stream().cuda_stream
    want = b.attend(s2d2)
    s2d2.ops_status(stream)
    binding.debug_attention_wait(64, True)
    out, lse = b.attend(s2d2)
    with pytest.raises(s2d2.S2D2Error) as e:
        s2d2.ops_status(stream)
    assert e.value.code == -5
    n = b.first[-1]
    assert out[:n].isnan().all() and lse[:n].isnan().all() and (out[n:] == 7).all() and (lse[n:] == 7).all()
    s2d2.ops_status(stream)                                          # reported once
    again = b.attend(s2d2)
    s2d2.ops_status(stream)
    assert all(torch.equal(x, y) for x, y in zip(again, want))       # and nothing of it is left


def test_a_limit_that_is_not_reached_changes_nothing(s2d2):
    from paper_2603_25702_b200 import binding
    b = au.Batch([(1, 3000), (200, 700)], 8, 2, 128)
    want = b.attend(s2d2)
    binding.debug_attention_wait(4096)
    got = b.attend(s2d2)
    s2d2.ops_status(torch.cuda.current_stream().cuda_stream)
    assert all(torch.equal(x, y) for x, y in zip(got, want))


def test_a_list_that_gives_rows_to_several_sequences_is_not_followed(s2d2):
    b = au.Batch([(8, 100)] * 6, 4, 2, 64, spare=1)
    for row0 in ([0, 49, 0, 49, 0, 49, 49], [0, 30, 10, 40, 20, 49, 49], [8, 16, 0, 49, 49, 49, 49]):
        b.row0.copy_(torch.tensor(row0, dtype=torch.int32))
        out, lse = b.attend(s2d2)
        assert (out == 7).all() and (lse == 7).all(), row0
    b.row0.copy_(torch.tensor(b.first, dtype=torch.int32))
    b.check(b.attend(s2d2), b.want())


def test_references_that_rise_and_fall(s2d2):
    """Scores that rise from step to step by more than the range that a reference is kept for, fall, stay, and one step that is far above all."""
    b = au.Batch([(130, 1500), (1, 4000)], 4, 2, 64)
    for s, (_, kv) in enumerate(b.lens):
        j = torch.arange(kv, device="cuda").float()
        size = 1 + 6 * (torch.sin(j / 150) + 1) + 40 * (j == 1111)
        b.keys[s].copy_((b.keys[s].float().abs() * size[:, None, None]).bfloat16())
    b.write()
    for sign in (1, -1):
        b.q.copy_(b.q.abs() * sign)
        b.check(b.attend(s2d2, scale=0.25), b.want(scale=0.25))


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("lens", [[(64, 64)], [(64, 64), (40, 40), (64, 64)]])
def test_rows_that_see_a_single_key(s2d2, lens, dim):
    """Each at another place of the tile, with scores far from zero on either side."""
    bits = torch.cat([1 << torch.arange(n, dtype=torch.int64).roll(7) for n, _ in lens]).cuda()
    b = au.Batch(lens, 4, 2, dim)
    b.q.mul_(20)
    b.check(b.attend(s2d2, 0, bits), b.want(0, bits))
