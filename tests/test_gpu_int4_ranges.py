"""Decode over the 4-bit cache with queries far from 1, brought back by the logits' factor."""
import pytest

import int4_accuracy as A
from test_gpu_int4_accuracy import contexts, filled  # noqa: F401

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("shape", [(32, 8, 128), (64, 8, 64), (4, 2, 64)])
@pytest.mark.parametrize("exponent", [-118, -100, -30, 30, 100, 112, 114, 116, 119])
def test_queries_of_any_exponent(contexts, shape, exponent, dtype):  # noqa: F811
    """The sum of a head's coordinates stays below 2^128: what lies above is infinite in a binary32 evaluation, too."""
    ctx = contexts(shape)
    cache, k, v, g = filled(ctx, 500, 95)
    q = (torch.randn((1, shape[0], shape[2]), generator=g, device="cuda").clamp(-3.5, 3.5).double() * 2.0 ** exponent).to(torch.bfloat16)
    out, scale = torch.empty(q.shape, dtype=dtype, device="cuda"), 0.125 * 2.0 ** -exponent
    cache.decode(q, out=out, sm_scale=scale)
    o, p = A.attention(q[0], k, v, scale)
    unit = (q[0].double() * 2.0 ** -exponent).float()         # (the same numbers, for the binary32 evaluation)
    o32, _ = A.attention(unit, k, v, 0.125, torch.float32)
    bound = A.float32_bound(o, o32, p, v) if dtype == torch.float32 else A.bf16_bound(o, p, v)
    error = A.rms(out[0].double() - o)
    assert error <= bound, (error, bound, A.rms(o))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("small", [0, 1])
@pytest.mark.parametrize("shape", [(32, 8, 128), (16, 16, 128)])
def test_groups_of_channels_of_two_sizes(contexts, shape, small, dtype):  # noqa: F811
    """Values of 64 channels 2^10 times as large as those of the other 64: each group is as exact as if it were alone."""
    from paper_2608_04074_b200.runtime import Int4Cache
    ctx, n = contexts(shape), 3000
    g = torch.Generator(device="cuda").manual_seed(96)
    k, v = (torch.randn((n, shape[1], 128), generator=g, device="cuda") for _ in range(2))
    v[..., 64 * small:64 * small + 64] *= 2.0 ** -10
    pos = torch.arange(n, dtype=torch.int32, device="cuda")
    cache = Int4Cache(ctx, 1, n)
    cache.append(None, k.to(torch.bfloat16), v.to(torch.bfloat16), torch.zeros_like(pos), pos)
    k, v = cache.gather(torch.zeros_like(pos), pos, torch.float32)
    q = torch.randn((1, shape[0], 128), generator=g, device="cuda").to(torch.bfloat16)
    out = torch.empty(q.shape, dtype=dtype, device="cuda")
    cache.decode(q, out=out)
    o, p = A.attention(q[0], k, v, 128 ** -0.5)
    o32, _ = A.attention(q[0], k, v, 128 ** -0.5, torch.float32)
    for c in (slice(0, 64), slice(64, 128)):
        part = (o[:, c], o32[:, c], p, v[..., c]) if dtype == torch.float32 else (o[:, c], p, v[..., c])
        bound = (A.float32_bound if dtype == torch.float32 else A.bf16_bound)(*part)
        error = A.rms(out[0, :, c].double() - o[:, c])
        assert error <= bound, (c, error, bound, A.rms(o[:, c]))


def test_scales_are_products_not_quotients(contexts):  # noqa: F811
    """Keys of groups whose range times the binary32 number next to 1/15 and whose range divided by 15 round to different scales:
    the cache holds the product."""
    import numpy as np

    import cache_reference as R
    from paper_2608_04074_b200 import cache_format
    from paper_2608_04074_b200.binding import QKTransform
    ctx, gen = contexts((4, 1, 64)), np.random.default_rng(97)
    w = R.to_bf16(1 + 0.3 * gen.normal(size=64))
    rows = []
    for _ in range(40):
        k = R.to_bf16(gen.normal(size=(50000, 1, 64)))
        x = R.transform(k, np.zeros(len(k)), weight=w)[0].astype(np.float32)
        span = x.max(-1) - R.to_bf16(x.min(-1))
        apart = R.to_bf16(span * (np.float32(1) / np.float32(15))) != R.to_bf16(span / np.float32(15))
        rows.append(k[apart[:, 0]])
        if sum(map(len, rows)) >= 3:
            break
    k = np.concatenate(rows)
    n = len(k)
    assert 3 <= n <= 64
    x = R.transform(k, np.zeros(n), weight=w)[0].astype(np.float32)
    codes, scale, zero = R.quantise(x)
    dev = lambda a: torch.from_numpy(a).cuda()  # noqa: E731
    pools = [torch.zeros((1, ctx.novakv_int4_page_bytes()), dtype=torch.uint8, device="cuda") for _ in range(2)]
    kd = dev(k).to(torch.bfloat16)
    ctx.novakv_int4_append(QKTransform(k_weight=dev(w).to(torch.bfloat16)), kd, kd, dev(np.zeros(n, np.int32)), dev(np.arange(n, dtype=np.int32)), *pools,
                           dev(np.zeros((1, 1), np.int32)), torch.zeros(1, dtype=torch.int32, device="cuda"))
    c, s, z = cache_format.int4_read_tokens(pools[0].cpu().numpy(), np.zeros(1, np.int32), 1, 64, 0, n)
    assert np.array_equal(s, scale) and np.array_equal(z, zero) and np.array_equal(c, codes)
    span = x.max(-1) - zero[..., 0]
    assert np.array_equal(s[..., 0], R.to_bf16(span * (np.float32(1) / np.float32(15)))) and (s[..., 0] != R.to_bf16(span / np.float32(15))).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("ctas", [0, 1])
@pytest.mark.parametrize("run", ["rising", "falling", "mixed"])
@pytest.mark.parametrize("shape", [(32, 8, 128), (64, 8, 64), (4, 2, 64)])
def test_scales_over_a_sequence(contexts, shape, run, ctas, dtype):  # noqa: F811
    """Values that grow or shrink by 2^16 over a sequence, or differ by as much from token to token: sums are brought along."""
    from paper_2608_04074_b200.runtime import Int4Cache
    ctx, n = contexts(shape), 3000
    g = torch.Generator(device="cuda").manual_seed(98)
    k, v = (torch.randn((n, shape[1], shape[2]), generator=g, device="cuda") for _ in range(2))
    exponent = {"rising": torch.linspace(-8, 8, n, device="cuda"), "falling": torch.linspace(8, -8, n, device="cuda"),
                "mixed": torch.randint(-8, 9, (n,), generator=g, device="cuda").float()}[run]
    v = v * torch.exp2(exponent)[:, None, None]
    pos = torch.arange(n, dtype=torch.int32, device="cuda")
    cache = Int4Cache(ctx, 1, n)
    cache.append(None, k.to(torch.bfloat16), v.to(torch.bfloat16), torch.zeros_like(pos), pos)
    k, v = cache.gather(torch.zeros_like(pos), pos, torch.float32)
    q = torch.randn((1, shape[0], shape[2]), generator=g, device="cuda").to(torch.bfloat16)
    out = torch.empty(q.shape, dtype=dtype, device="cuda")
    try:
        ctx.novakv_debug_set_scan_ctas(ctas)
        cache.decode(q, out=out)
    finally:
        ctx.novakv_debug_set_scan_ctas(0)
    o, p = A.attention(q[0], k, v, shape[2] ** -0.5)
    o32, _ = A.attention(q[0], k, v, shape[2] ** -0.5, torch.float32)
    bound = A.float32_bound(o, o32, p, v) if dtype == torch.float32 else A.bf16_bound(o, p, v)
    error = A.rms(out[0].double() - o)
    assert error <= bound, (error, bound, A.rms(o))
