"""Decode over the 4-bit cache where attention is long and flat: the output is a small rest of a large sum."""
import pytest

import int4_accuracy as A

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def contexts():
    from paper_2608_04074_b200.binding import Context
    made = {}

    def get(shape):
        if shape not in made:
            made[shape] = Context(*shape)
        return made[shape]
    return get


def filled(ctx, n, seed, batch=1):
    """A cache of `batch` sequences of n near-Gaussian rows, and what its slots stand for (float32 [batch n][Hkv][d])."""
    from paper_2608_04074_b200.runtime import Int4Cache
    g = torch.Generator(device="cuda").manual_seed(seed)
    k, v = (torch.randn((batch * n, ctx.n_kv_heads, ctx.head_dim), generator=g, device="cuda").to(torch.bfloat16) for _ in range(2))
    seq = torch.arange(batch, dtype=torch.int32, device="cuda").repeat_interleave(n)
    pos = torch.arange(n, dtype=torch.int32, device="cuda").repeat(batch)
    cache = Int4Cache(ctx, batch, n, seed=seed)
    cache.append(None, k, v, seq, pos)
    return cache, *cache.gather(seq, pos, torch.float32), g


SHAPES = [(64, 8, 64), (32, 8, 64), (32, 16, 64), (32, 32, 64), (32, 8, 128), (16, 8, 128), (16, 16, 128)]


@pytest.mark.parametrize("std", [0.0, 3e-4, 0.3, 1.0])
@pytest.mark.parametrize("ctas", [1, 0])
@pytest.mark.parametrize("shape", SHAPES)
def test_long_flat_attention(contexts, shape, ctas, std):
    """Logits of a standard deviation of `std`, bf16 outputs; with one CTA a warp holds 16384 tokens of a pair and more."""
    ctx, n = contexts(shape), 32768
    cache, k, v, g = filled(ctx, n, 80)
    q = (std * torch.randn((1, shape[0], shape[2]), generator=g, device="cuda")).to(torch.bfloat16)
    out = torch.empty(q.shape, dtype=torch.bfloat16, device="cuda")
    try:
        ctx.novakv_debug_set_scan_ctas(ctas)
        cache.decode(q, out=out)
    finally:
        ctx.novakv_debug_set_scan_ctas(0)
    o, p = A.attention(q[0], k, v, shape[2] ** -0.5)
    error, bound = A.rms(out[0].double() - o), A.bf16_bound(o, p, v)
    assert error <= bound, (error, bound, A.rms(o))


@pytest.mark.parametrize("std", [0.0, 3e-4, 0.3, 1.0, 3.0, 8.0])
@pytest.mark.parametrize("n,ctas", [(40, 0), (777, 0), (4097, 0), (32768, 0), (32768, 1)])
@pytest.mark.parametrize("shape", SHAPES)
def test_float32_outputs(contexts, shape, n, ctas, std):
    """What a float32 output is worth on ordinary data: that of a binary32 evaluation."""
    ctx = contexts(shape)
    cache, k, v, g = filled(ctx, n, 81)
    q = (std * torch.randn((1, shape[0], shape[2]), generator=g, device="cuda")).to(torch.bfloat16)
    sink = torch.randn(shape[0], generator=g, device="cuda")
    try:
        ctx.novakv_debug_set_scan_ctas(ctas)
        out = cache.decode(q, sink_logits=sink)
    finally:
        ctx.novakv_debug_set_scan_ctas(0)
    o, p = A.attention(q[0], k, v, shape[2] ** -0.5, sink=sink)
    o32, _ = A.attention(q[0], k, v, shape[2] ** -0.5, torch.float32, sink=sink)
    error, bound = A.rms(out[0].double() - o), A.float32_bound(o, o32, p, v)
    assert error <= bound, (error, bound, A.rms(o))


@pytest.mark.parametrize("std", [3.0, 10.0, 30.0])
@pytest.mark.parametrize("n", [40, 777, 32768])
@pytest.mark.parametrize("shape", SHAPES)
def test_bf16_outputs(contexts, shape, n, std):
    """Logits that matter one by one.  Each is a sum of d products that are cut off at 2^-15 of a step of the key's code in the query's
    largest channel, 136 times with either sign: sqrt(136) 2^-15 in the mean at most, 2^-11 here, times half a group's range."""
    ctx = contexts(shape)
    cache, k, v, g = filled(ctx, n, 82)
    q = (std * torch.randn((1, shape[0], shape[2]), generator=g, device="cuda")).to(torch.bfloat16)
    out = torch.empty(q.shape, dtype=torch.bfloat16, device="cuda")
    cache.decode(q, out=out)
    scale = shape[2] ** -0.5
    o, p = A.attention(q[0], k, v, scale)
    half = lambda x: (lambda y: (y.amax(-1) - y.amin(-1)) / 2)(x.double().unflatten(-1, (-1, 64)))  # noqa: E731
    logit = 2.0 ** -11 * scale * q.abs().max().item() * (half(k) / 7.5).max().item()
    moved = logit * torch.einsum("hgn,nhc->hgc", p ** 2, half(v) ** 2).mean().sqrt().item()
    error, bound = A.rms(out[0].double() - o), (A.bf16_bound(o, p, v) ** 2 + moved ** 2) ** 0.5
    assert error <= bound, (error, bound, A.rms(o))
