"""Queries that a call between the projection and the cache writes, and the decode attention directly behind it on the same stream:
the query transform, which starts beside the kernel in front, has to see them."""
import numpy as np
import pytest

from gpu_common import Case
from paper_2608_04074_b200 import workloads

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

TIMES, BATCH = 20, 3


@pytest.fixture(scope="module")
def cases():
    made = {}

    def get(scaled):
        if scaled not in made:
            made[scaled] = Case(workloads.qwen3_8b(batch=1, seq_len=1024, calib_tokens=2048, lloyd_iters=4), key_scale=scaled)
        return made[scaled]
    return get


def _decoder(cases, kind):
    """(context, q -> output) of a decode call over a cache of random indices."""
    from paper_2608_04074_b200.runtime import BandedCache, PagedCache
    case = cases(kind in ("scaled", "deployed", "banded"))
    ctx, lens = case.ctx, np.full(BATCH, 70, np.int32)
    gen = torch.Generator(device="cuda").manual_seed(7)
    if kind == "banded":
        banded = BandedCache(ctx, BATCH, 700, seed=1, key_scale=True)
        for b in range(BATCH):
            rows = torch.randn((2, 400, ctx.n_kv_heads, ctx.head_dim), generator=gen, device="cuda").to(torch.bfloat16)
            banded.prefill(0, b, rows[0], rows[1])
        return ctx, lambda q, out: banded.decode(0, q, out=out)
    cache = PagedCache(ctx, lens, seed=1, key_scale=kind == "scaled", int2_values=kind == "deployed")
    for pool in (cache.k_pages, cache.v_pages):
        pool.copy_(torch.randint(0, 256, pool.shape, generator=gen, dtype=torch.uint8, device="cuda"))
    if cache.v_meta is not None:
        cache.v_meta.copy_(torch.rand(cache.v_meta.shape, generator=gen, device="cuda"))
    if kind == "noalloc":
        return ctx, lambda q, out: ctx.novakv_decode_attention_noalloc(0, q, cache.k_pages, cache.v_pages, cache.page_table, cache.seq_lens, out)
    sink = torch.zeros(ctx.n_q_heads, device="cuda") if kind == "sink" else None
    return ctx, lambda q, out: cache.decode(0, q, out=out, sink_logits=sink)


def _writer(ctx, kind, n):
    """(rows of queries that the call writes, the call)."""
    from paper_2608_04074_b200.binding import QKTransform
    from paper_2608_04074_b200.runtime import BF16Cache, Int4Cache
    gen = torch.Generator(device="cuda").manual_seed(n)
    draw = lambda heads: torch.randn((n, heads, ctx.head_dim), generator=gen, device="cuda").to(torch.bfloat16)  # noqa: E731
    tr = QKTransform(torch.logspace(0, -5, ctx.head_dim // 2, device="cuda"), q_weight=torch.ones(ctx.head_dim, dtype=torch.bfloat16, device="cuda"))
    q, pos = draw(ctx.n_q_heads), torch.arange(n, dtype=torch.int32, device="cuda")
    q_out = torch.zeros_like(q)
    if kind == "qk":
        return q_out, lambda: ctx.novakv_qk_norm_rope(tr, q, None, pos, q_out, None)
    cache, k, v = (BF16Cache if kind == "bf16" else Int4Cache)(ctx, 1, n), draw(ctx.n_kv_heads), draw(ctx.n_kv_heads)
    return q_out, lambda: cache.append(tr, k, v, torch.zeros_like(pos), pos, q=q, q_out=q_out)


def _run(write, decode, q_out, wait):
    q_out.zero_()
    out = torch.empty((BATCH,) + q_out.shape[1:], device="cuda")
    torch.cuda.synchronize()
    write()
    if wait:
        torch.cuda.synchronize()
    decode(q_out[-BATCH:], out)
    return out


@pytest.mark.parametrize("n", [BATCH, 20000])
@pytest.mark.parametrize("writer", ["qk", "bf16", "int4"])
@pytest.mark.parametrize("kind", ["plain", "noalloc", "sink", "scaled", "deployed", "banded"])
def test_decode_directly_behind(cases, kind, writer, n):
    ctx, decode = _decoder(cases, kind)
    q_out, write = _writer(ctx, writer, n)
    expected = _run(write, decode, q_out, True)
    assert expected.any()
    for _ in range(TIMES):
        assert torch.equal(_run(write, decode, q_out, False), expected)
    # captured on a stream of its own, and replayed
    side, out = torch.cuda.Stream(), torch.empty_like(expected)
    with torch.cuda.stream(side):
        decode(q_out[-BATCH:], out)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            write()
            decode(q_out[-BATCH:], out)
    for _ in range(TIMES):
        q_out.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, expected)
    assert ctx.novakv_last_device_status() == 0


def test_the_queries_of_another_context(cases):
    from paper_2608_04074_b200.binding import Context
    ctx, decode = _decoder(cases, "plain")
    q_out, write = _writer(Context(ctx.n_q_heads, ctx.n_kv_heads, ctx.head_dim), "qk", 20000)
    expected = _run(write, decode, q_out, True)
    for _ in range(TIMES):
        assert torch.equal(_run(write, decode, q_out, False), expected)


def test_a_capture_between_the_calls(cases):
    """A decode that is captured between the two does not stand between them on the stream."""
    ctx, decode = _decoder(cases, "plain")
    q_out, write = _writer(ctx, "qk", 20000)
    expected = _run(write, decode, q_out, True)
    side, other, out = torch.cuda.Stream(), torch.zeros_like(q_out[:BATCH]), torch.empty_like(expected)
    unused = torch.empty_like(expected)
    with torch.cuda.stream(side):
        decode(other, unused)
        for _ in range(3):
            q_out.zero_()
            torch.cuda.synchronize()
            write()
            graph = torch.cuda.CUDAGraph()
            graph.capture_begin(capture_error_mode="relaxed")
            decode(other, unused)
            graph.capture_end()
            decode(q_out[-BATCH:], out)
            torch.cuda.synchronize()
            assert torch.equal(out, expected)


def test_the_record_is_emptied(cases):
    """Behind the decode no entry of the library's record is left: later calls overlap as before."""
    import ctypes

    ctx, decode = _decoder(cases, "plain")
    q_out, write = _writer(ctx, "qk", 300)
    expected = _run(write, decode, q_out, True)
    count = ctypes.c_int.in_dll(ctx.lib, "novakv_query_writers")
    before = count.value
    write()
    assert count.value == before + 1
    out = torch.empty_like(expected)
    decode(q_out[-BATCH:], out)
    assert count.value == before and torch.equal(out, expected)
