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
