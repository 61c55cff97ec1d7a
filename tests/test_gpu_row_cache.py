"""The caches whose append takes the projection's rows, at the end of their capacity."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

BAD_PAGE, BAD_TOKEN = 1, 8


@pytest.mark.parametrize("cache", ["int4", "bf16"])
def test_a_sequence_ends_with_its_capacity(cache):
    """Sequences of different capacities share a table as wide as the largest: a token behind a smaller one's pages is skipped and
    reported, and touches no other sequence's page."""
    from paper_2608_04074_b200.binding import Context
    from paper_2608_04074_b200.runtime import BF16Cache, Int4Cache
    ctx = Context(32, 8, 128)
    made = (Int4Cache if cache == "int4" else BF16Cache)(ctx, 3, np.array([10, 400, 64]))
    g = torch.Generator(device="cuda").manual_seed(1)
    rows = lambda n: torch.randn((n, 8, 128), generator=g, device="cuda").to(torch.bfloat16)  # noqa: E731
    ints = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    q = torch.randn((3, 32, 128), generator=g, device="cuda").to(torch.bfloat16)
    pos = torch.arange(400, dtype=torch.int32, device="cuda")
    made.append(None, rows(400), rows(400), torch.ones_like(pos), pos)
    made.append(None, rows(2), rows(2), ints(0, 2), ints(5, 63))
    assert ctx.novakv_last_device_status() == 0 and made.seq_lens.tolist() == [6, 400, 64]
    before, out = (made.k_pages.clone(), made.v_pages.clone()), made.decode(q)
    assert ctx.novakv_last_device_status() == 0
    made.append(None, rows(3), rows(3), ints(0, 2, 0), ints(64, 64, 399))
    assert ctx.novakv_last_device_status() == BAD_PAGE
    assert made.seq_lens.tolist() == [6, 400, 64]
    assert torch.equal(made.k_pages, before[0]) and torch.equal(made.v_pages, before[1]) and torch.equal(made.decode(q), out)
    made.append(None, rows(1), rows(1), ints(1), ints(448))
    assert ctx.novakv_last_device_status() == BAD_TOKEN
    ctx.close()
