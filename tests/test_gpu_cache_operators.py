"""The calls around the BF16 and the 4-bit cache on the device, against binary64 references (cache_reference.py): norms and
rotation, appends (bytes compared exactly), read-back, decode attention, and runs of them together."""
import numpy as np
import pytest

import cache_reference as R
from paper_2608_04074_b200 import cache_format

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

SHAPES = [(4, 1, 64), (8, 8, 64), (4, 2, 64), (16, 2, 64), (32, 8, 128), (3, 3, 128), (4, 2, 128)]
EPS = 1e-6
BAD_PAGE, BAD_LENGTH, WAIT_TIMEOUT, BAD_TOKEN = 1, 2, 4, 8


@pytest.fixture(scope="module")
def contexts():
    from paper_2608_04074_b200.binding import Context
    made = {}

    def get(shape):
        if shape not in made:
            made[shape] = Context(*shape)
        return made[shape]
    return get


def dev(a, dtype=None):
    t = torch.from_numpy(np.ascontiguousarray(a)).cuda()
    return t if dtype is None else t.to(dtype)


def bf16(a):
    return dev(np.asarray(a, np.float32), torch.bfloat16)


def host(t):
    return t.float().cpu().numpy()


def draw(gen, *shape):
    return R.to_bf16(gen.normal(size=shape))


def frequencies(rot, base=1e6):
    return (base ** (-np.arange(rot // 2) / max(rot // 2, 1))).astype(np.float32)


def make_transform(gen, d, norm, rot, interleaved=False, amplitude=1.0):
    """(QKTransform, keyword arguments of the reference for q and for k)."""
    from paper_2608_04074_b200.binding import QKTransform
    f = frequencies(rot) if rot else None
    wq, wk = (R.to_bf16(1 + 0.3 * gen.normal(size=d)) if norm else None for _ in range(2))
    tr = QKTransform(None if f is None else dev(f), interleaved=interleaved, amplitude=amplitude, q_weight=None if wq is None else bf16(wq),
                     k_weight=None if wk is None else bf16(wk), eps=EPS)
    common = dict(inv_freq=f, eps=EPS, interleaved=interleaved, amplitude=amplitude)
    return tr, dict(weight=wq, **common), dict(weight=wk, **common)


def check_rows(got, ref, size):
    """A binary32 evaluation rounded to bf16: half a step of bf16, and 2^-19 of the pair's size (mean of d squares, root, two
    products and their sum, cos and sin: fewer than 32 roundings of 2^-24)."""
    err = np.abs(np.asarray(got, np.float64) - ref)
    bound = R.bf16_eps * np.abs(ref) + 2.0 ** -19 * size + 2.0 ** -130
    assert (err <= bound).all(), (err / bound).max()


# ------------------------------------------------------------------------------------------------ norms and rotation
@pytest.mark.parametrize("norm,rot,interleaved,amplitude", [(True, 1.0, False, 1.0), (False, 1.0, False, 1.3466), (True, 0.5, False, 1.0),
                                                            (True, 1.0, True, 0.7), (False, 0.25, True, 1.0), (True, 0.0, False, 1.0)])
@pytest.mark.parametrize("n", [1, 5, 1300])
@pytest.mark.parametrize("shape", SHAPES)
def test_qk_norm_rope(contexts, shape, n, norm, rot, interleaved, amplitude):
    hq, hkv, d = shape
    ctx, gen = contexts(shape), np.random.default_rng(n + d)
    tr, rq, rk = make_transform(gen, d, norm, int(rot * d), interleaved, amplitude)
    q, k = draw(gen, n, hq, d), draw(gen, n, hkv, d)
    pos = gen.integers(-5, 200000, n).astype(np.int32)
    pos[0] = 2 ** 31 - 1
    qo, ko = (torch.empty((n, h, d), dtype=torch.bfloat16, device="cuda") for h in (hq, hkv))
    ctx.novakv_qk_norm_rope(tr, bf16(q), bf16(k), dev(pos), qo, ko)
    check_rows(host(qo), *R.transform(q, pos, **rq))
    check_rows(host(ko), *R.transform(k, pos, **rk))


@pytest.mark.parametrize("shape", [(4, 2, 64), (32, 8, 128)])
@pytest.mark.parametrize("offset,pad", [(0, 0), (0, 8), (1, 0), (0, 3), (3, 5)])        # elements: start of the rows, and between tokens
def test_strided_and_misaligned_rows(contexts, shape, offset, pad):
    hq, hkv, d = shape
    ctx, gen, n = contexts(shape), np.random.default_rng(3), 21
    width = (hq + 2 * hkv) * d + pad
    buffer = torch.full((offset + n * width,), 9.0, dtype=torch.bfloat16, device="cuda")
    rows = draw(gen, n, hq + 2 * hkv, d)
    fused = buffer[offset:].view(n, width)[:, :(hq + 2 * hkv) * d].unflatten(1, (hq + 2 * hkv, d))
    fused.copy_(bf16(rows))
    tr, rq, rk = make_transform(gen, d, True, d)
    pos = np.arange(n, dtype=np.int32)
    expected = [torch.empty((n, h, d), dtype=torch.bfloat16, device="cuda") for h in (hq, hkv)]
    ctx.novakv_qk_norm_rope(tr, fused[:, :hq], fused[:, hq:hq + hkv], dev(pos), *expected)
    check_rows(host(expected[0]), *R.transform(rows[:, :hq], pos, **rq))
    check_rows(host(expected[1]), *R.transform(rows[:, hq:hq + hkv], pos, **rk))
    # in place, one side at a time, and nothing else of the buffer moves
    before = buffer.clone()
    ctx.novakv_qk_norm_rope(tr, fused[:, :hq], None, dev(pos), fused[:, :hq], None)
    ctx.novakv_qk_norm_rope(tr, None, fused[:, hq:hq + hkv], dev(pos), None, fused[:, hq:hq + hkv])
    assert torch.equal(fused[:, :hq], expected[0]) and torch.equal(fused[:, hq:hq + hkv], expected[1])
    fused[:, :hq + hkv] = bf16(rows[:, :hq + hkv])
    assert torch.equal(buffer, before)


def test_non_finite_rows_stay_in_their_head(contexts):
    ctx, gen = contexts((4, 2, 64)), np.random.default_rng(4)
    tr, rq, _ = make_transform(gen, 64, True, 64)
    q = draw(gen, 3, 4, 64)
    q[1, 2, 5] = np.nan
    q[2, 0, 7] = np.inf
    out = torch.empty((3, 4, 64), dtype=torch.bfloat16, device="cuda")
    ctx.novakv_qk_norm_rope(tr, bf16(q), None, dev(np.arange(3, dtype=np.int32)), out, None)
    got = host(out)
    assert np.isnan(got[1, 2]).all()
    for t, h in [(t, h) for t in range(3) for h in range(4) if (t, h) not in ((1, 2), (2, 0))]:
        ref, size = R.transform(q[t:t + 1, h:h + 1], [t], **rq)
        check_rows(got[t:t + 1, h:h + 1], ref, size)


@pytest.mark.parametrize("rot,interleaved", [(0, False), (32, False), (32, True)])
def test_channels_that_do_not_turn_are_left_alone(contexts, rot, interleaved):
    """Infinities and NaN in a channel behind the rotated ones reach no other channel."""
    shape = (4, 2, 64)
    ctx, gen = contexts(shape), np.random.default_rng(6)
    tr, rq, _ = make_transform(gen, 64, False, rot, interleaved)
    q = draw(gen, 4, 4, 64)
    q[:, :, rot], q[:, :, 50], q[:, :, 63] = np.inf, np.nan, -np.inf
    out = torch.empty((4, 4, 64), dtype=torch.bfloat16, device="cuda")
    ctx.novakv_qk_norm_rope(tr, bf16(q), None, dev(np.arange(4, dtype=np.int32)), out, None)
    got = host(out)
    assert np.array_equal(got[..., rot:], q[..., rot:], equal_nan=True)
    ref, size = R.transform(q[..., :max(rot, 1)], np.arange(4), **rq)
    if rot:
        check_rows(got[..., :rot], ref, size)
    pools = [torch.zeros((1, 2, 64, 64), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    seq, pos = dev(np.zeros(4, np.int32)), dev(np.arange(4, dtype=np.int32))
    ctx.novakv_bf16_append(None, bf16(q[:, :2]), bf16(q[:, 2:]), seq, pos, *pools, dev(np.zeros((1, 1), np.int32)), torch.zeros(1, dtype=torch.int32, device="cuda"))
    for pool, x in zip(pools, (q[:, :2], q[:, 2:])):
        assert np.array_equal(host(pool)[0, :, :4].transpose(1, 0, 2), x, equal_nan=True)


# ------------------------------------------------------------------------------------------------ appends
def lists(gen, kind, n):
    """tok_seq, tok_pos of n entries over three sequences of up to 320 tokens."""
    if kind == "step":
        return np.arange(3, dtype=np.int32)[:n], np.array([0, 63, 319], np.int32)[:n]
    if kind == "prompts":                                     # one after another, the second from inside a page
        seq = np.repeat(np.arange(3), [n - n // 2 - n // 3, n // 2, n // 3]).astype(np.int32)
        return seq, np.concatenate([np.arange((seq == s).sum()) + [0, 37, 128][s] for s in range(3)]).astype(np.int32)
    slots = gen.permutation(3 * 320)[:n]                      # any order, and some entries unused
    seq, pos = (slots // 320).astype(np.int32), (slots % 320).astype(np.int32)
    seq[::4] = -1
    return seq, pos


@pytest.mark.parametrize("kind,n", [("step", 1), ("step", 3), ("prompts", 199), ("mixed", 100), ("prompts", 310)])
@pytest.mark.parametrize("with_q,norm,rot,interleaved", [(True, True, 1.0, False), (False, False, 0.5, True), (True, True, 0.5, False), (False, False, 0.0, False)])
@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("cache", ["bf16", "int4"])
def test_append(contexts, cache, shape, with_q, norm, rot, interleaved, kind, n):
    hq, hkv, d = shape
    ctx, gen = contexts(shape), np.random.default_rng(n + d)
    tr, rq, rk = make_transform(gen, d, norm, int(rot * d), interleaved)
    seq, pos = lists(gen, kind, n)
    n = len(seq)
    table = gen.permutation(20)[:15].reshape(3, 5).astype(np.int32)
    q, k, v = draw(gen, n, hq, d), draw(gen, n, hkv, d), draw(gen, n, hkv, d)
    k[:, :, 3] *= 40
    k = R.to_bf16(k)                                          # (what the call is given)
    if cache == "bf16":
        pools = [draw(gen, 20, hkv, 64, d) for _ in range(2)]
        pools_dev = [bf16(p) for p in pools]
    else:
        pools = [gen.integers(0, 256, (20, hkv * cache_format.int4_chunk_bytes(d)), dtype=np.uint8) for _ in range(2)]
        pools_dev = [dev(p) for p in pools]
    lens = np.array([0, 400, 7], np.int32)
    lens_dev, q_out = dev(lens), torch.full((n, hq, d), 5.0, dtype=torch.bfloat16, device="cuda")
    call = ctx.novakv_bf16_append if cache == "bf16" else ctx.novakv_int4_append
    call(tr, bf16(k), bf16(v), dev(seq), dev(pos), *pools_dev, dev(table), lens_dev, bf16(q) if with_q else None, q_out if with_q else None)
    assert ctx.novakv_last_device_status() == 0

    used = seq >= 0
    kt, size = R.transform(k, pos, **rk)
    page, slot = table[seq[used], pos[used] // 64], pos[used] % 64
    if cache == "bf16":
        got = [host(p) for p in pools_dev]
        check_rows(got[0][page, :, slot], kt[used], size[used])
        assert np.array_equal(got[1][page, :, slot], v[used])
        for g, p in zip(got, pools):
            p[page, :, slot] = g[page, :, slot]
            assert np.array_equal(g, p)                       # nothing else has moved
    else:
        # (a binary64 key rounds to the same binary32 number here and there but for one in ~2^28)
        for x, p, g in ((kt.astype(np.float32), pools[0], pools_dev[0]), (v, pools[1], pools_dev[1])):
            for s in range(3):
                mine = used & (seq == s)
                R.write_tokens(p, table[s], pos[mine], hkv, d, *R.quantise(x[mine]))
            assert np.array_equal(g.cpu().numpy(), p)
    for s in range(3):
        if (used & (seq == s)).any():
            lens[s] = max(lens[s], pos[used & (seq == s)].max() + 1)
    assert np.array_equal(lens_dev.cpu().numpy(), lens)
    if with_q:
        ref, size = R.transform(q, pos, **rq)
        check_rows(host(q_out)[used], ref[used], size[used])
        assert (host(q_out)[~used] == 5.0).all()


@pytest.mark.parametrize("norm,rot,interleaved,amplitude", [(True, 128, False, 1.0), (False, 128, True, 1.5), (True, 48, False, 1.0), (True, 128, True, 1.0)])
def test_keys_of_a_long_prompt(contexts, norm, rot, interleaved, amplitude):
    """64000 groups a case: among them are minima, maxima and quotients next to a border, which binary32 alone would decide
    either way.  All bytes are those of the binary64 key."""
    ctx, gen, n, hkv, d = contexts((32, 8, 128)), np.random.default_rng(rot + norm), 4000, 8, 128
    tr, _, rk = make_transform(gen, d, norm, rot, interleaved, amplitude)
    k = draw(gen, n, hkv, d)
    k[:, :, [5, 77]] *= 8                                     # (a power of two: still bf16)
    pos = np.arange(n, dtype=np.int32) + 32
    pages = (n + 160) // 64 + 1
    pools = [torch.zeros((pages, ctx.novakv_int4_page_bytes()), dtype=torch.uint8, device="cuda") for _ in range(2)]
    table = gen.permutation(pages).astype(np.int32)[None]
    ctx.novakv_int4_append(tr, bf16(k), bf16(k), dev(np.zeros(n, np.int32)), dev(pos), *pools, dev(table), torch.zeros(1, dtype=torch.int32, device="cuda"))
    expected = np.zeros(tuple(pools[0].shape), np.uint8)
    R.write_tokens(expected, table[0], pos, hkv, d, *R.quantise(R.transform(k, pos, **rk)[0].astype(np.float32)))
    assert np.array_equal(pools[0].cpu().numpy(), expected)


@pytest.mark.parametrize("cache", ["bf16", "int4"])
def test_append_from_a_fused_projection(contexts, cache):
    """Rows with a token stride, aligned and not, give what contiguous ones give."""
    hq, hkv, d = shape = (32, 8, 128)
    ctx, gen, n = contexts(shape), np.random.default_rng(8), 70
    tr, _, _ = make_transform(gen, d, True, d)
    seq, pos, table = np.zeros(n, np.int32), np.arange(n, dtype=np.int32), np.array([[1, 0]], np.int32)
    rows = bf16(draw(gen, n, hq + 2 * hkv, d))
    results = []
    for pad in (None, 0, 1):
        if pad is None:
            q, k, v = (rows[:, a:b].contiguous() for a, b in ((0, hq), (hq, hq + hkv), (hq + hkv, hq + 2 * hkv)))
        else:
            wide = torch.zeros((n, (hq + 2 * hkv) * d + pad), dtype=torch.bfloat16, device="cuda")
            fused = wide[:, pad:].unflatten(1, (hq + 2 * hkv, d))
            fused.copy_(rows)
            q, k, v = fused[:, :hq], fused[:, hq:hq + hkv], fused[:, hq + hkv:]
        if cache == "bf16":
            pools = [torch.zeros((2, hkv, 64, d), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        else:
            pools = [torch.zeros((2, ctx.novakv_int4_page_bytes()), dtype=torch.uint8, device="cuda") for _ in range(2)]
        out, lens = torch.zeros((n, hq, d), dtype=torch.bfloat16, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
        (ctx.novakv_bf16_append if cache == "bf16" else ctx.novakv_int4_append)(tr, k, v, dev(seq), dev(pos), *pools, dev(table), lens, q, out)
        results.append([*pools, out, lens])
    for other in results[1:]:
        assert all(torch.equal(a, b) for a, b in zip(results[0], other))


@pytest.mark.parametrize("cache", ["bf16", "int4"])
def test_bad_entries_are_skipped_and_reported(contexts, cache):
    hq, hkv, d = shape = (4, 2, 64)
    ctx, gen = contexts(shape), np.random.default_rng(9)
    seq = np.array([0, 2, -2, 0, 0, 1, 0], np.int32)          # a sequence that is none, twice; positions out of range; a bad page
    pos = np.array([1, 0, 0, -1, 128, 64, 5], np.int32)
    table = np.array([[0, 1], [1, 7]], np.int32)
    n = len(seq)
    if cache == "bf16":
        pools = [torch.zeros((2, hkv, 64, d), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    else:
        pools = [torch.zeros((2, ctx.novakv_int4_page_bytes()), dtype=torch.uint8, device="cuda") for _ in range(2)]
    lens, out = torch.zeros(2, dtype=torch.int32, device="cuda"), torch.full((n, hq, d), 5.0, dtype=torch.bfloat16, device="cuda")
    k, v, q = draw(gen, n, hkv, d), draw(gen, n, hkv, d), draw(gen, n, hq, d)
    call = ctx.novakv_bf16_append if cache == "bf16" else ctx.novakv_int4_append
    call(None, bf16(k), bf16(v), dev(seq), dev(pos), *pools, dev(table), lens, bf16(q), out)
    assert ctx.novakv_last_device_status() == BAD_TOKEN | BAD_PAGE
    assert lens.tolist() == [6, 0]
    good = np.array([0, 6])
    assert np.array_equal(host(out)[good], q[good]) and (np.delete(host(out), good, 0) == 5.0).all()
    if cache == "bf16":
        slots = host(pools[0])[0].transpose(1, 0, 2)
        assert np.array_equal(slots[[1, 5]], k[good]) and not np.delete(slots, [1, 5], 0).any() and not host(pools[0])[1].any()
    else:
        expected = np.zeros(tuple(pools[0].shape), np.uint8)
        R.write_tokens(expected, table[0], pos[good], hkv, d, *R.quantise(k[good]))
        assert np.array_equal(pools[0].cpu().numpy(), expected)
        gk, gv = (torch.full((n, hkv, d), 5.0, device="cuda") for _ in range(2))
        ctx.novakv_int4_gather(dev(seq), dev(pos), *pools, dev(table), gk, gv)
        assert ctx.novakv_last_device_status() == BAD_TOKEN | BAD_PAGE
        assert np.array_equal(host(gv)[good], R.values(*R.quantise(v[good])).astype(np.float32)) and (np.delete(host(gk), good, 0) == 5.0).all()


@pytest.mark.parametrize("d", [64, 128])
def test_quantiser_corners(contexts, d):
    """Equal values, a NaN, infinities, tiny and huge ranges, halves between two codes."""
    ctx = contexts((4, 2, 64) if d == 64 else (4, 2, 128))
    gen, n = np.random.default_rng(10), 12
    v = draw(gen, n, 2, d)
    v[0] = 0
    v[1] = -2.5
    v[2, 0, 5] = np.nan
    v[3, 0, 5], v[3, 1, 9] = np.inf, -np.inf
    v[4] = R.to_bf16(v[4] * 1e-38)
    v[5] = R.to_bf16(v[5] * 3e37)
    v[6] = R.to_bf16(np.resize(np.arange(31) * 0.5, (2, d)))              # scale 1: every second one is a half
    v[7] = R.to_bf16(100 + 0.25 * v[7])
    v[8] = np.nan
    v[9, :, 0] = 1e30
    seq, pos = np.zeros(n, np.int32), np.arange(n, dtype=np.int32) + 25      # (over a tile's edge)
    pools = [torch.zeros((1, ctx.novakv_int4_page_bytes()), dtype=torch.uint8, device="cuda") for _ in range(2)]
    ctx.novakv_int4_append(None, bf16(v), bf16(v), dev(seq), dev(pos), *pools, dev(np.zeros((1, 1), np.int32)), torch.zeros(1, dtype=torch.int32, device="cuda"))
    c, s, z = cache_format.int4_read_tokens(pools[1].cpu().numpy(), np.zeros(1, np.int32), 2, d, 25, n)
    rc, rs, rz = R.quantise(v)
    assert np.array_equal(c, rc) and np.array_equal(s, rs) and np.array_equal(z, rz, equal_nan=True)
    assert torch.equal(pools[0], pools[1])
    assert (c[6][0, :31] == np.rint(np.arange(31) * 0.5)).all()               # (the second head starts elsewhere in the ramp)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("shape,n", [((4, 1, 64), 1), ((3, 3, 128), 37), ((32, 8, 128), 1500), ((16, 2, 64), 333)])
def test_gather(contexts, shape, n, dtype):
    hq, hkv, d = shape
    ctx, gen = contexts(shape), np.random.default_rng(n)
    table = gen.permutation(12).reshape(2, 6).astype(np.int32)
    pools = [np.zeros((12, hkv * cache_format.int4_chunk_bytes(d)), np.uint8) for _ in range(2)]
    x = [[draw(gen, 384, hkv, d) * s for s in (1, 3)] for _ in range(2)]
    for p, both in zip(pools, x):
        for s in range(2):
            R.write_tokens(p, table[s], np.arange(384), hkv, d, *R.quantise(both[s]))
    seq, pos = gen.integers(0, 2, n).astype(np.int32), gen.integers(0, 384, n).astype(np.int32)
    seq[::5] = -1
    out = [torch.full((n, hkv, d), 7.0, dtype=dtype, device="cuda") for _ in range(2)]
    ctx.novakv_int4_gather(dev(seq), dev(pos), *(dev(p) for p in pools), dev(table), *out)
    for o, both in zip(out, x):
        ref = np.full((n, hkv, d), 7.0, np.float32)
        for i in np.flatnonzero(seq >= 0):                    # zero + scale code: an exact product, one rounding
            ref[i] = R.values(*R.quantise(both[seq[i]][pos[i]]))
        assert np.array_equal(host(o), ref if dtype == torch.float32 else R.to_bf16(ref))
    ctx.novakv_int4_gather(dev(seq[:0]), dev(pos[:0]), *(dev(p) for p in pools), dev(table), out[0][:0], out[1][:0])


# ------------------------------------------------------------------------------------------------ decode attention
class Cache4:
    """A 4-bit cache filled from the reference; what was never written holds NaN pairs and ones as codes."""

    def __init__(self, shape, lens, seed, scale_k=1.0, scale_v=1.0, table=None):
        self.hq, self.hkv, self.d = shape
        gen = np.random.default_rng(seed)
        lens = np.asarray(lens, np.int32)
        pages = max(1, int(-(-lens.max() // 64)))
        self.table = gen.permutation(len(lens) * pages).reshape(len(lens), pages).astype(np.int32) if table is None else table
        self.lens = lens
        self.pools = [np.full((int(self.table.max()) + 1, self.hkv * cache_format.int4_chunk_bytes(self.d)), 255, np.uint8) for _ in range(2)]
        self.x = []
        for b, n in enumerate(lens):
            rows = []
            for p, s in zip(self.pools, (scale_k, scale_v)):
                c, sc, z = R.quantise(R.to_bf16(draw(gen, n, self.hkv, self.d) * (s(gen, n) if callable(s) else s)))
                R.write_tokens(p, self.table[b], np.arange(n), self.hkv, self.d, c, sc, z)
                rows.append(R.values(c, sc, z))
            self.x.append(rows)
        self.q = draw(gen, len(lens), self.hq, self.d) * 3
        self.q = R.to_bf16(self.q)
        self.dev = (bf16(self.q), dev(self.pools[0]), dev(self.pools[1]), dev(self.table), dev(lens))

    def run(self, ctx, dtype=torch.float32, **kw):
        out = torch.full((len(self.lens), self.hq, self.d), float("nan"), dtype=dtype, device="cuda")
        ws = torch.empty(ctx.novakv_int4_workspace_bytes(len(self.lens)), dtype=torch.uint8, device="cuda").fill_(255)
        ctx.novakv_int4_decode_attention(*self.dev, out, ws, **kw)
        return out

    def check(self, out, window=0, sink_logits=None, sm_scale=None, only=None):
        got, sink = host(out), None if sink_logits is None else sink_logits.cpu().numpy()
        for b in range(len(self.lens)) if only is None else only:
            n = int(self.lens[b])
            first = max(0, n - window) if window else 0
            if n == 0:
                assert not got[b].any()
                continue
            ref, tol, coarse = R.attention(self.q[b], *(x[first:] for x in self.x[b]), self.d ** -0.5 if sm_scale is None else sm_scale, sink)
            if out.dtype == torch.bfloat16:
                tol = tol + coarse + R.bf16_eps * np.abs(ref)
            err = np.abs(got[b] - ref)
            assert (err <= tol).all(), (b, n, (err / tol).max())


LENS = [[1], [0, 1, 2], [777], [31, 32, 33, 63, 64, 65, 127, 128, 129], [0, 0, 0], [5, 0, 4097, 0, 1, 1000, 64], [2500, 2501]]


@pytest.mark.parametrize("lens", LENS, ids=str)
@pytest.mark.parametrize("shape", SHAPES)
def test_decode(contexts, shape, lens):
    ctx, c = contexts(shape), Cache4(shape, lens, 20 + len(lens))
    c.check(c.run(ctx))
    c.check(c.run(ctx, torch.bfloat16))
    sink = dev(np.random.default_rng(5).normal(size=shape[0]).astype(np.float32) * 3)
    c.check(c.run(ctx, sink_logits=sink), sink_logits=sink)
    for window in (1, 33, 128, 2 ** 31 - 1):
        c.check(c.run(ctx, window=window, sink_logits=sink), window=window, sink_logits=sink)
    c.check(c.run(ctx, sm_scale=0.01), sm_scale=0.01)
    assert ctx.novakv_last_device_status() == 0


@pytest.mark.parametrize("shape", [(32, 8, 128), (16, 2, 64), (3, 3, 128)])
@pytest.mark.parametrize("ctas", [1, 2, 7, 40])
def test_the_split_moves_nothing(contexts, shape, ctas):
    """Few CTAs: several pairs and many tiles each, pieces that reach over CTAs, warps without a tile."""
    ctx, c = contexts(shape), Cache4(shape, [700, 0, 33, 1, 2050, 64, 96], 31)
    sink = dev(np.linspace(-4, 4, shape[0]).astype(np.float32))
    try:
        ctx.novakv_debug_set_scan_ctas(ctas)
        c.check(c.run(ctx))
        c.check(c.run(ctx, sink_logits=sink, window=640), sink_logits=sink, window=640)
    finally:
        ctx.novakv_debug_set_scan_ctas(0)


@pytest.mark.parametrize("batch", [511, 513, 1100])
def test_large_batches(contexts, batch):
    """More sequences than a CTA has threads: the prefix holds runs of them."""
    shape = (4, 1, 64)
    gen = np.random.default_rng(batch)
    lens = gen.integers(0, 70, batch)
    lens[gen.integers(0, batch, batch // 3)] = 0
    ctx, c = contexts(shape), Cache4(shape, lens, 40)
    c.check(c.run(ctx))
    c.check(c.run(ctx, window=20), window=20)


@pytest.mark.parametrize("shape", [(32, 8, 128), (16, 2, 64), (8, 8, 64), (4, 2, 64)])
def test_ranges(contexts, shape):
    """Values whose scales run over 2^20 within a sequence, tiny and huge rows, logits far apart."""
    ctx = contexts(shape)
    spread = lambda gen, n: 2.0 ** gen.integers(-10, 11, (n, 1, 1))  # noqa: E731
    rising = lambda gen, n: 2.0 ** np.linspace(-10, 10, n)[:, None, None]  # noqa: E731
    for kw in (dict(scale_v=spread), dict(scale_v=rising), dict(scale_v=1e-30), dict(scale_v=1e30), dict(scale_k=20.0), dict(scale_k=1e-3)):
        c = Cache4(shape, [600, 65], 50, **kw)
        c.check(c.run(ctx))


def test_queries_of_any_size(contexts):
    ctx = contexts((4, 2, 64))
    for size in (1e-30, 1e-6, 300.0):
        c = Cache4((4, 2, 64), [200, 3], 51)
        c.q = R.to_bf16(c.q * size)
        c.q[0, 1] = 0
        c.dev = (bf16(c.q),) + c.dev[1:]
        c.check(c.run(ctx, sm_scale=0.1 / size), sm_scale=0.1 / size)


def test_one_token_takes_all(contexts):
    """A key that meets the query far above the others, early, late and in the last tile."""
    shape = (32, 8, 128)
    ctx = contexts(shape)
    for at in (0, 1000, 1499):
        c = Cache4(shape, [1500], 52)
        gen = np.random.default_rng(at)
        c.q = R.to_bf16(gen.normal(size=(1, 32, 128)))
        rows = R.to_bf16(np.repeat(c.q[0].reshape(8, 4, 128).mean(1, keepdims=True), 1, 1)[:, 0] * 8)[None]
        code = R.quantise(rows)
        R.write_tokens(c.pools[0], c.table[0], np.array([at]), 8, 128, *code)
        c.x[0][0][at] = R.values(*code)[0]
        c.dev = (bf16(c.q), dev(c.pools[0])) + c.dev[2:]
        c.check(c.run(ctx))


def test_a_nan_stays_with_its_head(contexts):
    """A value row with a NaN reaches its KV head's queries and no other; a NaN query its own head."""
    shape = (4, 2, 64)
    ctx, c = contexts(shape), Cache4(shape, [100, 100], 53)
    pool = c.pools[1].reshape(-1, 2, cache_format.int4_chunk_bytes(64))
    at = cache_format.int4_pair_offsets(64)[10, 0]
    pool[c.table[0, 0], 1, at + 2:at + 4] = 255                # the zero of token 10, KV head 1
    c.dev = c.dev[:2] + (dev(c.pools[1]),) + c.dev[3:]
    got = host(c.run(ctx))
    assert np.isnan(got[0, 2:]).all() and np.isfinite(got[0, :2]).all() and np.isfinite(got[1]).all()
    c.q[1, 3, 9] = np.nan
    c.dev = (bf16(c.q),) + c.dev[1:]
    got = host(c.run(ctx))
    assert np.isnan(got[1, 3]).all() and np.isfinite(got[1, :3]).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("shape", [(4, 1, 64), (16, 2, 64), (32, 8, 128), (4, 2, 128)])
def test_heads_of_any_size_side_by_side(contexts, shape, dtype):
    """Heads of one KV head whose queries are far apart in size, or hold an infinity, do not touch one another."""
    ctx, c = contexts(shape), Cache4(shape, [300, 40], 57)
    hg = shape[0] // shape[1]
    c.q[:, 0::hg] = R.to_bf16(c.q[:, 0::hg] * 2.0 ** 12)
    c.q[0, 1::hg] = R.to_bf16(c.q[0, 1::hg] * 2.0 ** -30)
    c.dev = (bf16(c.q),) + c.dev[1:]
    c.check(c.run(ctx, dtype, sm_scale=0.02), sm_scale=0.02)
    c.q[1, 1, 5] = np.inf
    c.dev = (bf16(c.q),) + c.dev[1:]
    got = host(c.run(ctx, dtype, sm_scale=0.02))
    keep = [h for h in range(shape[0]) if h != 1]
    assert not np.isfinite(got[1, 1]).all()
    c.check(torch.from_numpy(np.where(np.isfinite(got), got, 0)).cuda().to(dtype), sm_scale=0.02, only=[0])
    ref, tol, coarse = R.attention(np.where(np.isinf(c.q[1]), 0, c.q[1]), *c.x[1], 0.02)
    err, bound = np.abs(got[1] - ref)[keep], (tol + (dtype == torch.bfloat16) * (coarse + R.bf16_eps * np.abs(ref)))[keep]
    assert (err <= bound).all()


def test_bad_pages_and_lengths(contexts):
    shape = (4, 2, 64)
    ctx, c = contexts(shape), Cache4(shape, [128, 100, 64], 54)
    table, lens = c.table.copy(), c.lens.copy()
    table[0, 1] = 10 ** 6
    table[1, 1] = -3
    table[2, 1] = 10 ** 6                                     # (not used: the sequence ends before)
    c.dev = c.dev[:3] + (dev(table), dev(lens))
    out = c.run(ctx)
    assert ctx.novakv_last_device_status() == BAD_PAGE
    c.check(out, only=[2])
    table[:] = c.table
    lens[:] = [129, 100, -4]                                  # clamped to 128, as it is, to 0
    c.dev = c.dev[:3] + (dev(table), dev(lens))
    out = c.run(ctx)
    assert ctx.novakv_last_device_status() == BAD_LENGTH
    c.lens[2] = 0
    c.check(out)


def test_library_refuses(contexts):
    from paper_2608_04074_b200.binding import NovaKVError, QKTransform
    shape = (4, 2, 64)
    ctx, c = contexts(shape), Cache4(shape, [128, 100], 55)
    out = torch.zeros((2, 4, 64), device="cuda")
    ws = torch.empty(ctx.novakv_int4_workspace_bytes(2) + 256, dtype=torch.uint8, device="cuda")
    before = ctx.novakv_launch_count()
    for bad in (ws[:ctx.novakv_int4_workspace_bytes(2) - 1], ws[16:]):
        with pytest.raises(NovaKVError, match="workspace"):
            ctx.novakv_int4_decode_attention(*c.dev, out, bad)
    for kw in (dict(window=-1), dict(sm_scale=float("nan"))):
        with pytest.raises(NovaKVError, match="invalid"):
            ctx.novakv_int4_decode_attention(*c.dev, out, ws, **kw)
    q = torch.zeros(2 * 4 * 64 + 1, dtype=torch.bfloat16, device="cuda")[1:].view(2, 4, 64)        # not on 16 bytes
    with pytest.raises(NovaKVError, match="invalid"):
        ctx.novakv_int4_decode_attention(q, *c.dev[1:], out, ws)
    pos, rows = dev(np.zeros(2, np.int32)), torch.zeros((2, 2, 64), dtype=torch.bfloat16, device="cuda")
    for tr, what in ((QKTransform(torch.ones(4, device="cuda")), "shape"), (QKTransform(torch.ones(40, device="cuda")), "shape"),
                     (QKTransform(eps=-1.0), "invalid"), (QKTransform(amplitude=float("nan")), "invalid")):
        with pytest.raises(NovaKVError, match=what):
            ctx.novakv_qk_norm_rope(tr, None, rows, pos, None, rows)
    tr = QKTransform()
    for args in ((None, None, pos, None, None), (None, rows, pos, None, None), (None, None, pos, None, rows)):
        with pytest.raises(NovaKVError, match="invalid"):
            ctx.novakv_qk_norm_rope(tr, *args)
    with pytest.raises(ValueError, match="device"):
        ctx.novakv_qk_norm_rope(tr, None, rows.cpu(), pos, None, rows)
    with pytest.raises(TypeError, match="QKTransform"):
        ctx.novakv_qk_norm_rope(object(), None, rows, pos, None, rows)
    with pytest.raises(ValueError, match="weight"):
        ctx.novakv_qk_norm_rope(QKTransform(k_weight=torch.ones(32, dtype=torch.bfloat16, device="cuda")), None, rows, pos, None, rows)
    assert ctx.novakv_launch_count() == before
    # nothing to do is done
    ctx.novakv_qk_norm_rope(tr, None, rows[:0], pos[:0], None, rows[:0])
    ctx.novakv_int4_decode_attention(c.dev[0][:0], *c.dev[1:3], c.dev[3][:0], c.dev[4][:0], out[:0], ws)
    assert ctx.novakv_launch_count() == before


def test_a_wait_that_gives_up_is_reported(contexts):
    shape = (4, 2, 64)
    ctx, c = contexts(shape), Cache4(shape, [5000, 3], 56)
    try:
        ctx.novakv_debug_set_wait_limit(0)
        c.run(ctx)
        assert ctx.novakv_last_device_status() in (0, WAIT_TIMEOUT)      # (a copy may have landed before its first look)
    finally:
        ctx.novakv_debug_set_wait_limit(2000000000)
    c.check(c.run(ctx))
    assert ctx.novakv_last_device_status() == 0


# ------------------------------------------------------------------------------------------------ together, as they are used
@pytest.mark.parametrize("window", [0, 48])
@pytest.mark.parametrize("shape", [(32, 8, 128), (16, 2, 64)])
@pytest.mark.parametrize("cache", ["int4", "bf16"])
def test_prompt_and_steps(contexts, cache, shape, window):
    """Prompts of three sequences in one call, then steps of one token each: rotation, append, attention, one behind another on
    the current stream without a look in between; then the same steps as one captured graph, replayed."""
    from paper_2608_04074_b200.runtime import BF16Cache, Int4Cache
    hq, hkv, d = shape
    ctx, gen = contexts(shape), np.random.default_rng(60)
    tr, rq, rk = make_transform(gen, d, True, d)
    lens, steps = np.array([70, 1, 200]), 5
    seq = np.repeat(np.arange(3), lens).astype(np.int32)
    pos = np.concatenate([np.arange(n) for n in lens]).astype(np.int32)
    kp, vp = draw(gen, len(seq), hkv, d), draw(gen, len(seq), hkv, d)
    rows = [draw(gen, 3, hq + 2 * hkv, d) for _ in range(steps)]
    rows_dev, pos_dev = [bf16(r) for r in rows], [dev((lens + i).astype(np.int32)) for i in range(steps)]
    each, prompt = dev(np.arange(3, dtype=np.int32)), (bf16(kp), bf16(vp), dev(seq), dev(pos))
    made = (Int4Cache if cache == "int4" else BF16Cache)(ctx, 3, 300, seed=2)
    outs, qs = ([torch.zeros((3, hq, d), dtype=t, device="cuda") for _ in range(steps)] for t in (torch.float32, torch.bfloat16))

    def run():
        made.seq_lens.zero_()
        made.append(tr, *prompt)
        for i in range(steps):
            r = rows_dev[i]
            made.append(tr, r[:, hq:hq + hkv], r[:, hq + hkv:], each, pos_dev[i], q=r[:, :hq], q_out=qs[i])
            made.decode(qs[i], out=outs[i], window=window)
    run()
    assert ctx.novakv_last_device_status() == 0
    assert made.seq_lens.tolist() == (lens + steps).tolist()
    first = [o.clone() for o in outs]
    # reference: the cached rows themselves (their bytes are tested above), exactly as the attention reads them
    back_seq = np.repeat(np.arange(3), lens + steps).astype(np.int32)
    back_pos = np.concatenate([np.arange(n + steps) for n in lens]).astype(np.int32)
    if cache == "int4":
        k, v = (host(x).astype(np.float64) for x in made.gather(dev(back_seq), dev(back_pos), torch.float32))
    else:
        table = made.page_table.cpu().numpy()
        k, v = (host(p)[table[back_seq, back_pos // 64], :, back_pos % 64].astype(np.float64) for p in (made.k_pages, made.v_pages))
    for s in range(3):                                        # a first look at the rows: half a step of the codec, or of bf16
        mine = (seq == s)
        ref = R.transform(kp[mine], pos[mine], **rk)[0]
        got = k[back_seq == s][:lens[s]]
        step = (ref.max(-1) - ref.min(-1)).max() / 15 if cache == "int4" else 0.02 * np.abs(ref).max()
        assert np.abs(got - ref).max() <= step
    for i in range(steps):
        q_ref, size = R.transform(rows[i][:, :hq], lens + i, **rq)
        check_rows(host(qs[i]), q_ref, size)
        for s in range(3):
            n = lens[s] + i + 1
            lo = max(0, n - window) if window else 0
            ref, tol, _ = R.attention(host(qs[i])[s], k[back_seq == s][lo:n], v[back_seq == s][lo:n], d ** -0.5)
            bound = tol if cache == "int4" else 2e-3 * np.abs(ref).max()       # (the BF16 decode's own stated tolerance)
            assert (np.abs(host(first[i])[s] - ref) <= bound).all()
    # captured and replayed: the same bits
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        run()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            run()
    torch.cuda.synchronize()
    for o in outs:
        o.fill_(float("nan"))
    made.k_pages.zero_()
    made.v_pages.zero_()
    for _ in range(2):
        graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(first, outs))


def test_in_front_of_the_index_cache(contexts):
    """The transform alone, then the 2-bit cache's own append and attention: what they give on rows rotated beforehand."""
    from gpu_common import Case
    from paper_2608_04074_b200 import workloads
    from paper_2608_04074_b200.runtime import PagedCache
    case = Case(workloads.tiny())
    ctx, gen, n = case.ctx, np.random.default_rng(61), 130
    tr, rq, rk = make_transform(gen, 64, True, 64)
    k, v, q = draw(gen, n, 1, 64), draw(gen, n, 1, 64), draw(gen, 1, 4, 64)
    pos, seq, at = dev(np.arange(n, dtype=np.int32)), dev(np.zeros(n, np.int32)), dev(np.array([n - 1], np.int32))
    outs = []
    for fused in (True, False):
        cache = PagedCache(ctx, np.array([n], np.int32), seed=1)
        cache.seq_lens.zero_()
        kr, qr = torch.empty((n, 1, 64), dtype=torch.bfloat16, device="cuda"), torch.empty((1, 4, 64), dtype=torch.bfloat16, device="cuda")
        ctx.novakv_qk_norm_rope(tr, bf16(q), None, at, qr, None)
        ctx.novakv_qk_norm_rope(tr, None, bf16(k), pos, None, kr)
        if not fused:
            torch.cuda.synchronize()
        cache.append(0, kr, bf16(v), seq, pos)
        outs.append(cache.decode(0, qr))
    check_rows(host(kr), *R.transform(k, np.arange(n), **rk))
    check_rows(host(qr), *R.transform(q, [n - 1], **rq))
    assert torch.equal(*outs) and torch.isfinite(outs[0]).all()


@pytest.mark.parametrize("shape", [(32, 8, 128), (64, 8, 64)])
@pytest.mark.parametrize("cache", ["int4", "bf16"])
def test_pools_beyond_32_bits(contexts, cache, shape):
    """Pages behind the first 4 GB of a pool: what a small pool of the same pages gives."""
    hq, hkv, d = shape
    ctx, gen, n = contexts(shape), np.random.default_rng(72), 200
    tr, _, _ = make_transform(gen, d, False, d)
    page = ctx.novakv_int4_page_bytes() if cache == "int4" else hkv * 64 * d * 2
    pages = (9 << 29) // page                                 # 4.5 GB
    assert pages * page > 1 << 32
    order = np.array([pages - 1, 0, pages - 3, pages // 2], np.int32)
    k, v, q = bf16(draw(gen, n, hkv, d)), bf16(draw(gen, n, hkv, d)), bf16(draw(gen, 1, hq, d) * 2)
    seq, pos, outs = dev(np.zeros(n, np.int32)), dev(np.arange(n, dtype=np.int32)), []
    for total, table in ((pages, order), (4, np.arange(4, dtype=np.int32))):
        if cache == "int4":
            pools = [torch.empty((total, page), dtype=torch.uint8, device="cuda") for _ in range(2)]
            ws = torch.empty(ctx.novakv_int4_workspace_bytes(1), dtype=torch.uint8, device="cuda")
        else:
            pools = [torch.empty((total, hkv, 64, d), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
            ws = torch.empty(ctx.novakv_bf16_workspace_bytes(1, 4), dtype=torch.uint8, device="cuda")
        table, lens, out = dev(table[None]), torch.zeros(1, dtype=torch.int32, device="cuda"), torch.zeros((1, hq, d), device="cuda")
        if cache == "int4":
            ctx.novakv_int4_append(tr, k, v, seq, pos, *pools, table, lens)
            rows = [torch.zeros((n, hkv, d), device="cuda") for _ in range(2)]
            ctx.novakv_int4_gather(seq, pos, *pools, table, *rows)
            ctx.novakv_int4_decode_attention(q, *pools, table, lens, out, ws)
        else:
            ctx.novakv_bf16_append(tr, k, v, seq, pos, *pools, table, lens)
            rows = [p[table[0].long()[pos.long() // 64], :, pos.long() % 64].float() for p in pools]
            ctx.novakv_bf16_decode_attention(q, *pools, table, lens, out, ws)
        assert ctx.novakv_last_device_status() == 0 and lens.item() == n
        outs.append([*rows, out])
        del pools
    assert all(torch.equal(a, b) for a, b in zip(*outs)) and torch.isfinite(outs[0][2]).all()


def test_first_call_inside_a_capture():
    """A context's first calls, captured: nothing of their set-up may need a stream that is not capturing."""
    from paper_2608_04074_b200.binding import Context
    shape = (4, 2, 64)
    ctx, c = Context(*shape), Cache4(shape, [100, 70], 73)
    out = torch.zeros((2, 4, 64), device="cuda")
    ws = torch.empty(ctx.novakv_int4_workspace_bytes(2), dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ctx.novakv_int4_decode_attention(*c.dev, out, ws)
    graph.replay()
    torch.cuda.synchronize()
    c.check(out)
    ctx.close()


def test_two_streams_with_workspaces_of_their_own(contexts):
    shape = (32, 8, 128)
    ctx = contexts(shape)
    caches = [Cache4(shape, [3000, 100], 70), Cache4(shape, [64, 2000, 500], 71)]
    expected = [c.run(ctx) for c in caches]
    streams = [torch.cuda.Stream() for _ in caches]
    torch.cuda.synchronize()
    outs = [[] for _ in caches]
    for _ in range(20):
        for c, s, o in zip(caches, streams, outs):
            with torch.cuda.stream(s):
                o.append(c.run(ctx))
    torch.cuda.synchronize()
    for e, o in zip(expected, outs):
        assert all(torch.equal(e, x) for x in o)
