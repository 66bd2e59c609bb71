"""Plain 64-bit restatements of the stand-alone operators (MXFP4 and token scores), numpy only, on the CPU."""
import numpy as np

GRID = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=np.float64)


def bf16_round(x: np.ndarray) -> np.ndarray:
    """fp32 values rounded to the nearest bfloat16 (finite inputs), as fp32."""
    b = np.ascontiguousarray(x, dtype=np.float32).view(np.uint32)
    b = (b + np.uint32(0x7FFF) + ((b >> np.uint32(16)) & np.uint32(1))) & np.uint32(0xFFFF0000)
    return b.view(np.float32)


def n_blocks(cols: int) -> int:
    return -(-cols // 32)


def mxfp4_encode(x: np.ndarray):
    """(codes [rows, 16 * blocks], scale bytes [rows, blocks]) of x [rows, cols], element by element from the definition."""
    rows, cols = x.shape
    nb = n_blocks(cols)
    b = np.zeros((rows, nb * 32))
    b[:, :cols] = x
    b = b.reshape(rows, nb, 32)
    big = np.abs(b).max(axis=2)
    bad = ~np.isfinite(big)
    _, e = np.frexp(np.where(bad | (big == 0), 1.0, big))            # big = f * 2^e, f in [0.5, 1)
    e = np.clip(e - 1 - 2, -127, 127)
    e = np.where(big == 0, -127, e)
    v = np.where(bad[:, :, None], 0.0, b) * np.exp2(-e.astype(np.float64))[:, :, None]
    mag = np.minimum(np.abs(v), 6.0)
    dist = np.abs(mag[..., None] - GRID)
    nearest = dist.min(axis=-1, keepdims=True)
    tie = dist == nearest                                            # one or two candidates; of two the even code
    code = np.where(tie & (np.arange(8) % 2 == 0), np.arange(8), -1).max(axis=-1)
    code = np.where(code < 0, tie.argmax(axis=-1), code)
    code = np.where(bad[:, :, None], 0, code | (np.signbit(np.where(bad[:, :, None], 0.0, b)) << 3)).astype(np.uint8)
    code = code.reshape(rows, nb * 16, 2)
    scale = np.where(bad, 255, e + 127).astype(np.uint8)
    return code[:, :, 0] | (code[:, :, 1] << 4), scale


def mxfp4_values(codes: np.ndarray, scales: np.ndarray, cols: int) -> np.ndarray:
    """The fp64 values of codes [rows, 16 * blocks] and scale bytes [rows, blocks]."""
    rows, nb = scales.shape
    nib = np.stack([codes & 15, codes >> 4], axis=-1).reshape(rows, nb, 32)
    v = GRID[nib & 7] * np.where(nib & 8, -1.0, 1.0)
    s = np.where(scales == 255, np.nan, np.exp2(scales.astype(np.float64) - 127))
    return (v * s[:, :, None]).reshape(rows, nb * 32)[:, :cols]


def tile_scales(scales: np.ndarray) -> np.ndarray:
    """Scale bytes [rows, blocks] in tiles of 128 rows x 4 blocks, byte by byte from the layout's definition."""
    rows, nb = scales.shape
    quads = -(-nb // 4)
    out = np.zeros((-(-rows // 128)) * quads * 512, dtype=np.uint8)
    r, b = np.meshgrid(np.arange(rows), np.arange(nb), indexing="ij")
    out[((r // 128) * quads + b // 4) * 512 + (r % 32) * 16 + (r % 128) // 32 * 4 + b % 4] = scales
    return out


def scores(x: np.ndarray, tokens=None, k: int = 0):
    """lse, entropy, logprob, rank, top ids and log probabilities of fp64 logits x [rows, vocab] (documented special rows)."""
    rows, V = x.shape
    out = {n: np.zeros(rows) for n in ("lse", "entropy", "logprob")}
    out["rank"] = np.zeros(rows, np.int64)
    out["log_s"] = np.zeros(rows)
    out["top_ids"], out["top_logprobs"] = np.full((rows, k), -1, np.int64), np.full((rows, k), -np.inf)
    for r in range(rows):
        z = x[r]
        undefined = bool(np.isnan(z).any() or (z == np.inf).any())
        tok = None if tokens is None else int(tokens[r])
        ok = tok is not None and 0 <= tok < V
        if undefined:
            for n in ("lse", "entropy", "logprob"):
                out[n][r] = np.nan
            out["rank"][r] = -1
            out["top_logprobs"][r] = np.nan
            continue
        m = z.max()
        if ok:
            out["rank"][r] = int((z > z[tok]).sum() + (z[:tok] == z[tok]).sum())
        else:
            out["rank"][r], out["logprob"][r] = -1, np.nan
        if m == -np.inf:
            out["lse"][r] = -np.inf
            if ok:
                out["logprob"][r] = -np.inf
            continue
        d = z - m
        e = np.exp(d)
        s = e.sum()
        out["log_s"][r] = np.log(s)
        out["lse"][r] = m + np.log(s)
        out["entropy"][r] = np.log(s) - (np.where(e > 0, d, 0.0) * e).sum() / s
        if ok:
            out["logprob"][r] = d[tok] - np.log(s)
        order = np.lexsort((np.arange(V), -z))[:k]
        order = order[z[order] > -np.inf]
        out["top_ids"][r, :order.size] = order
        out["top_logprobs"][r, :order.size] = d[order] - np.log(s)
    return out


def score_tolerance(V: int, log_s: np.ndarray):
    """Absolute error allowed to log s, from the arithmetic of an fp32 pass with 256 threads per 4096-element tile: every
    thread adds 16 terms per tile (one rounding each, relative 2^-24 of the running sum), about 64 more roundings merge threads
    and rescale; a term carries the error of a fast exp2 (2^-22) and of its argument (|u| 2^-24, weighted by 2^u: below 2^-23)."""
    return (16 * -(-V // 4096) + 64) * 2.0 ** -24 + 2.0 ** -21 + np.abs(log_s) * 2.0 ** -22
