"""The bounds of int4_accuracy.py, shown to tell the evaluations apart that they are there to tell apart: weights of 22 and of 11 bits,
float32 and bf16 outputs, codes counted from their middle and from 0."""
import numpy as np
import pytest

import cache_reference as R
import int4_accuracy as A

torch = pytest.importorskip("torch")


def half(x):
    return x.to(torch.float16).double()


def model(q, codes, scale, zero, p, bits, middle):
    """The decode's value side with the weights as binary16 numbers (11 bits) or pairs of them (22), all else in binary64."""
    def groups(x):                                            # [n][Hkv][groups] -> [Hkv][1][n][groups]
        return x.permute(1, 0, 2)[:, None]
    w = p[..., None] * groups(scale)                          # [Hkv][Hg][n][groups]
    top = 2.0 ** 13 / w.max().item()                          # (as the kernel: the largest at 2^13, what is far below loses bits)
    hi = half(w * top)
    used = (hi + half(w * top - hi) if bits == 22 else hi) / top
    c = (codes.double() - middle).unflatten(-1, (-1, 64))      # [n][Hkv][groups][64]
    o = torch.einsum("hgnc,nhce->hgce", used, c) + (p[..., None] * groups(zero + middle * scale)).sum(2)[..., None]
    return o.flatten(0, 1).flatten(-2)


@pytest.mark.parametrize("n,std", [(40, 3.0), (777, 3.0), (777, 0.3), (4097, 1.0), (4097, 3e-4), (4097, 8.0)])
@pytest.mark.parametrize("shape", [(32, 4, 64), (16, 4, 128)])
def test_the_bounds_tell_evaluations_apart(shape, n, std):
    hq, hkv, d = shape
    gen = np.random.default_rng(n)
    q = torch.from_numpy(R.to_bf16(std * gen.normal(size=(hq, d))))
    k = torch.from_numpy(R.values(*R.quantise(R.to_bf16(gen.normal(size=(n, hkv, d))))))
    code = R.quantise(R.to_bf16(gen.normal(size=(n, hkv, d))))
    v = torch.from_numpy(R.values(*code))
    codes, scale, zero = (torch.from_numpy(x) if x.dtype == np.uint8 else torch.from_numpy(x).double() for x in code)
    o, p = A.attention(q, k, v, d ** -0.5)
    o32, _ = A.attention(q, k, v, d ** -0.5, torch.float32)
    fine, coarse = A.float32_bound(o, o32, p, v), A.bf16_bound(o, p, v)
    assert A.rms(model(q, codes, scale, zero, p, 22, 8.0) - o) <= fine
    assert A.rms(model(q, codes, scale, zero, p, 11, 8.0) - o) > 2 * fine
    assert A.rms(o.to(torch.bfloat16).double() - o) > 2 * fine
    short = model(q, codes, scale, zero, p, 11, 7.5)
    assert A.rms(short.to(torch.bfloat16).double() - o) <= coarse


def test_weights_that_agree_need_codes_from_the_middle():
    """One weight and one scale for all tokens, long and flat: an error of the weight is one of the result, or, with codes from 0,
    of a sum that is far larger."""
    hq, hkv, d, n = 8, 2, 64, 40000
    gen = np.random.default_rng(3)
    codes = torch.from_numpy(gen.integers(0, 16, (n, hkv, d)).astype(np.uint8))
    scale = torch.full((n, hkv, 1), 0.2734375, dtype=torch.float64)
    zero = -7.5 * scale
    v = zero + scale * codes.double()
    p = torch.full((hkv, hq // hkv, n), 0.7 / n, dtype=torch.float64)
    p[..., 0] *= 1.3                                          # (the largest weight is another's: the many are no power of two of it)
    o = torch.einsum("hgn,nhd->hgd", p, v).flatten(0, 1)
    coarse = A.bf16_bound(o, p, v)
    middle, bottom = (A.rms(model(None, codes, scale, zero, p, 11, m).to(torch.bfloat16).double() - o) for m in (7.5, 0.0))
    assert middle <= coarse < bottom / 5
