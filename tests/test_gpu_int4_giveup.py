"""Waits of the 4-bit decode that give up: reported with certainty, in each form of the walk, and the next call is right."""
import pytest

from test_gpu_int4_accuracy import contexts, filled  # noqa: F401

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

WAIT_TIMEOUT = 4


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("shape", [(32, 8, 128), (64, 8, 64)])
@pytest.mark.parametrize("batch,n", [(1, 100), (2, 9000), (40, 700)])           # a CTA a pair, up to 32 sequences, more
def test_a_limit_of_zero(contexts, batch, n, shape, dtype):  # noqa: F811
    ctx = contexts(shape)
    cache, _, _, g = filled(ctx, n, 90, batch)
    q = torch.randn((batch, shape[0], shape[2]), generator=g, device="cuda").to(torch.bfloat16)
    first, out = (torch.empty(q.shape, dtype=dtype, device="cuda") for _ in range(2))
    cache.decode(q, out=first)
    assert ctx.novakv_last_device_status() == 0
    pools = cache.k_pages.clone(), cache.v_pages.clone()
    try:
        ctx.novakv_debug_set_wait_limit(0)
        cache.decode(q, out=out)
        assert ctx.novakv_last_device_status() == WAIT_TIMEOUT
    finally:
        ctx.novakv_debug_set_wait_limit(2000000000)
    cache.decode(q, out=out)
    assert ctx.novakv_last_device_status() == 0
    assert torch.equal(out, first)
    assert torch.equal(cache.k_pages, pools[0]) and torch.equal(cache.v_pages, pools[1])
