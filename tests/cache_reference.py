"""The operators around the paged caches in numpy binary64, from their definitions (public header), for the tests."""
import numpy as np

from paper_2608_04074_b200 import cache_format

bf16_eps = 2.0 ** -8          # half a step of bfloat16, relative to the value
fp16_tiny = 2.0 ** -24


def to_bf16(x):
    """float32 -> nearest bfloat16 (ties to even) as float32; NaN stays NaN."""
    x = np.ascontiguousarray(x, np.float32)
    u = x.view(np.uint32)
    r = ((u.astype(np.uint64) + 0x7fff + (u >> 16 & 1)) >> 16 << 16).astype(np.uint32).view(np.float32)
    return np.where(np.isnan(x), x, r)


def transform(x, pos, inv_freq=None, weight=None, eps=1e-6, interleaved=False, amplitude=1.0):
    """x [n][heads][d] -> (y, size): y in binary64 and, of each element, |a| + |b| of the pair it comes from (times amplitude),
    which the rounding errors of a binary32 evaluation are measured by."""
    y = x.astype(np.float64)
    if weight is not None:
        y = y / np.sqrt((y * y).mean(-1, keepdims=True) + np.float64(np.float32(eps))) * weight.astype(np.float64)
    size = np.abs(y)
    if inv_freq is None:
        return y, size
    half = len(inv_freq)
    i = np.arange(half)
    a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
    t = np.asarray(pos, np.float64)[:, None, None] * inv_freq.astype(np.float64)
    amp = np.float64(np.float32(amplitude))
    xa, xb = y[..., a], y[..., b]
    out, size = y.copy(), size.copy()
    out[..., a], out[..., b] = amp * (xa * np.cos(t) - xb * np.sin(t)), amp * (xb * np.cos(t) + xa * np.sin(t))
    size[..., a] = size[..., b] = amp * (np.abs(xa) + np.abs(xb))
    return out, size


def quantise(x):
    """float32 [..., d] -> codes uint8 [..., d], scale, zero float32 [..., d / 64]."""
    x = np.asarray(x, np.float32)
    g = x.reshape(x.shape[:-1] + (x.shape[-1] // 64, 64))
    with np.errstate(all="ignore"):
        zero = to_bf16(g.min(-1, keepdims=True))
        scale = to_bf16((g.max(-1, keepdims=True) - zero) * (np.float32(1) / np.float32(15)))
        scale = np.where((scale > 0) & np.isfinite(scale), scale, np.float32(1))
        t = np.rint((g - zero) / scale)
        codes = np.where(np.isnan(t), 0, np.clip(t, 0, 15)).astype(np.uint8)
    return codes.reshape(x.shape), scale[..., 0], zero[..., 0]


def values(codes, scale, zero):
    c = codes.astype(np.float64).reshape(scale.shape + (64,))
    return (zero.astype(np.float64)[..., None] + scale.astype(np.float64)[..., None] * c).reshape(codes.shape)


def write_tokens(pool, table_row, pos, hkv, d, codes, scale, zero):
    """Codes [n][Hkv][d] and pairs [n][Hkv][d / 64] to positions `pos` of a sequence in a pool uint8 [n_pages][Hkv * chunk]."""
    chunk = pool.reshape(len(pool), hkv, cache_format.int4_chunk_bytes(d))
    page, slot = table_row[pos // 64], pos % 64
    heads = np.arange(hkv)[None, :, None]
    chunk[page[:, None, None], heads, cache_format.int4_code_offsets(d)[slot][:, None]] = codes[..., 0::2] | codes[..., 1::2] << 4
    at = cache_format.int4_pair_offsets(d)[slot][:, None]
    for i, half in enumerate((scale, zero)):
        bits = np.ascontiguousarray(half, np.float32).view(np.uint32) >> 16
        chunk[page[:, None, None], heads, at + 2 * i] = bits & 255
        chunk[page[:, None, None], heads, at + 2 * i + 1] = bits >> 8


def attention(q, k, v, scale, sink=None):
    """q [Hq][d], k, v [n][Hkv][d] binary64 -> (o [Hq][d], tol, coarse), [Hq][1] each: tol bounds the evaluation behind a binary32
    output, coarse what the one behind a bf16 output adds to it, its rounding apart.

    tol.  The products of a logit are exact (q and codes are short numbers), their sums are cut off below 2^-23 of the largest
    product at worst, at most 128 + 8 times, and a few binary32 roundings of scale code, zero q and their sum follow: less than
    2^-15 (136 2^-23 and 8 2^-24) of the largest single term scale |q| 2 max|k| - and the test takes 2^-19 of the sum of all d of
    them, of which the largest is at least a sixteenth for queries that are not spread evenly and which exceeds it otherwise.  A
    weight is off by as much, relatively, and by 2^-20 for the base-2 exponential and its 22 bits; numerator and normaliser both,
    hence twice.  The numerator is a sum of sums of 32 tokens, each cut off at 2^-24 of its largest product 68 times, added in
    binary32 by n / 32 additions over the warps, whose errors go with the root of their number.

    coarse.  Codes are taken as they lie, 2^-10 of a number's leading bit, so that a cut is 2^-15 of |q| max times one step of a
    code, at most 136 times in a logit; the weights have 12 bits."""
    hkv, hg = k.shape[1], q.shape[0] // k.shape[1]
    qh = q.astype(np.float64).reshape(hkv, hg, -1)
    z = scale * np.einsum("hgd,nhd->hgn", qh, k)
    m = z.max(-1, keepdims=True)
    s = None if sink is None else sink.astype(np.float64).reshape(hkv, hg, 1)
    if s is not None:
        m = np.maximum(m, s)
    p = np.exp(z - m)
    total = p.sum(-1, keepdims=True) + (0 if s is None else np.exp(s - m))
    o = np.einsum("hgn,nhd->hgd", p, v) / total
    vmax, kmax = np.abs(v).max(), np.abs(k).max()
    size = scale * np.abs(qh).sum(-1, keepdims=True) * 2 * kmax
    steps = np.sqrt(len(k)) + 8
    tol = vmax * (2 * (2.0 ** -19 * size + 2.0 ** -20) + steps * 2.0 ** -21)
    step = 2 * kmax / 15                                       # (a group's range is at most twice its largest value)
    coarse = vmax * 2 * (136 * 2.0 ** -15 * scale * np.abs(qh).max() * step + 2.0 ** -12)
    return o.reshape(q.shape), tol.reshape(-1, 1), np.full((q.shape[0], 1), coarse)
