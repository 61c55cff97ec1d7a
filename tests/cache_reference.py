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
    """q [Hq][d], k, v [n][Hkv][d] binary64 -> (o [Hq][d], tol): tol [Hq][1] bounds a binary32 evaluation on the codes.

    A logit is a sum of d products whose factors are exact, so it is off by at most 2^-19 (128 additions, each cut off below
    2^-23 of the running sum at worst, and a few roundings of binary32: < 2^-16 2^-3) of S = scale sum_i |q_i| vmax_i, vmax the
    largest |value| in the key's group.  A weight is then off by the same times ln 2 / ln 2, relatively, plus 2^-20 of the base-2
    exponential and the weight's 22 bits; numerator and normaliser both, hence the two.  The numerator's accumulation adds
    (n + 8) 2^-23 of the largest magnitude at most, in sums of 32 tokens at a time that are themselves cut off."""
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
    vmax = np.abs(v).max()
    size = scale * np.abs(qh).sum(-1, keepdims=True) * 2 * np.abs(k).max()
    steps = np.sqrt(len(k)) + 8
    tol = vmax * (2 * (2.0 ** -19 * size + 2.0 ** -20) + steps * 2.0 ** -21)
    return o.reshape(q.shape), tol.reshape(-1, 1)
