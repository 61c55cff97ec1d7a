"""What the calls around the BF16 and the 4-bit cache refuse before anything reaches a device, the 4-bit page's layout, and the
reference of the GPU tests, pinned."""
import ctypes

import numpy as np
import pytest

import cache_reference as R
from paper_2608_04074_b200 import binding, build, cache_format

torch = pytest.importorskip("torch")

EINVAL = 1
HQ, HKV, D, N, PAGES = 8, 2, 64, 3, 5


@pytest.fixture(scope="module")
def calls():
    build.build_cuda()
    from paper_2608_04074_b200 import _novakv_calls
    _novakv_calls.setup(lambda device: 0, lambda: 0, torch.float32)
    # (device -1: what a CPU tensor's get_device() gives, so that the checks behind it are reached here)
    yield _novakv_calls.bind_operators(binding.load_library()._handle, -1, HQ, HKV, D, (torch.bfloat16, torch.int32, torch.uint8))
    if torch.cuda.is_available():
        _novakv_calls.setup(torch._C._cuda_getCurrentRawStream, torch._C._cuda_getDevice, torch.float32)


def _rows(heads, dtype=torch.bfloat16):
    return torch.zeros((N, heads, D), dtype=dtype)


def _ints(*shape):
    return torch.zeros(shape, dtype=torch.int32)


def _pool4():
    return torch.zeros((PAGES, HKV * cache_format.int4_chunk_bytes(D)), dtype=torch.uint8)


def _pool16():
    return torch.zeros((PAGES, HKV, 64, D), dtype=torch.bfloat16)


def _args(name):
    """(name of the argument, value) of a call that only its null context is wrong with."""
    tr = binding.QKTransform()
    if name == "novakv_qk_norm_rope":
        return dict(transform=tr, q=_rows(HQ), k=_rows(HKV), tok_pos=_ints(N), q_out=_rows(HQ), k_out=_rows(HKV))
    if name == "novakv_int4_gather":
        return dict(tok_seq=_ints(N), tok_pos=_ints(N), k_pages=_pool4(), v_pages=_pool4(), page_table=_ints(2, 4), k_out=_rows(HKV), v_out=_rows(HKV))
    if name == "novakv_int4_decode_attention":
        return dict(q=_rows(HQ), k_pages=_pool4(), v_pages=_pool4(), page_table=_ints(N, 4), seq_lens=_ints(N), out=_rows(HQ, torch.float32),
                    workspace=torch.zeros(256, dtype=torch.uint8), sm_scale=0.125, window=0, sink_logits=torch.zeros(HQ))
    pool = _pool4 if "int4" in name else _pool16
    return dict(transform=tr, k_new=_rows(HKV), v_new=_rows(HKV), tok_seq=_ints(N), tok_pos=_ints(N), k_pages=pool(), v_pages=pool(),
                page_table=_ints(2, 4), seq_lens=_ints(2), q=_rows(HQ), q_out=_rows(HQ))


NAMES = ["novakv_qk_norm_rope", "novakv_bf16_append", "novakv_int4_append", "novakv_int4_gather", "novakv_int4_decode_attention"]
# (an output goes with its input: the extension takes one without the other, the library refuses it)
MAY_BE_NONE = {"novakv_qk_norm_rope": {"q", "k", "q_out", "k_out"}, "novakv_bf16_append": {"transform", "q", "q_out"},
               "novakv_int4_append": {"transform", "q", "q_out"}, "novakv_int4_gather": set(), "novakv_int4_decode_attention": {"sink_logits"}}


def test_every_operator_is_bound(calls):
    assert set(calls) == set(NAMES)


@pytest.mark.parametrize("name", NAMES)
def test_null_context_and_argument_count(calls, name):
    args = list(_args(name).values())
    assert calls[name](0, *args) == EINVAL and calls[name](None, *args) == EINVAL
    for wrong in (args[:-1], args + [0]):
        with pytest.raises(TypeError, match="positional"):
            calls[name](0, *wrong)
    with pytest.raises(TypeError):
        calls[name](0, *args[:-1], last=args[-1])


@pytest.mark.parametrize("name,arg", [(n, a) for n in NAMES for a in _args(n)])
def test_wrong_arguments_are_refused(calls, name, arg):
    good = _args(name)
    wrong = [7, "x"]
    if arg not in MAY_BE_NONE[name]:
        wrong.append(None)
    x = good[arg]
    if arg in ("sm_scale", "window"):
        wrong = [None, "x", [1]]
    elif torch.is_tensor(x):
        other = torch.float16 if x.dtype != torch.float16 else torch.int64
        if arg != "workspace":
            wrong += [x.to(other), x[..., :-1], x[None], x.repeat_interleave(2, -1)[..., ::2]]     # type, sizes, inner stride
        else:
            wrong += [torch.zeros(512, dtype=torch.uint8)[::2]]
    for w in wrong:
        with pytest.raises((TypeError, ValueError, AttributeError)):
            calls[name](0, *{**good, arg: w}.values())


def test_none_where_it_is_allowed(calls):
    for name in NAMES:
        for arg in MAY_BE_NONE[name]:
            assert calls[name](0, *{**_args(name), arg: None}.values()) == EINVAL


def test_rows_with_a_token_stride_are_taken(calls):
    fused = torch.zeros((N, HQ + 2 * HKV, D), dtype=torch.bfloat16)
    q, k, v = fused[:, :HQ], fused[:, HQ:HQ + HKV], fused[:, HQ + HKV:]
    assert calls["novakv_qk_norm_rope"](0, *{**_args("novakv_qk_norm_rope"), "q": q, "k": k, "q_out": q, "k_out": k}.values()) == EINVAL
    assert calls["novakv_int4_append"](0, *{**_args("novakv_int4_append"), "q": q, "k_new": k, "v_new": v}.values()) == EINVAL
    with pytest.raises(ValueError, match="contiguous"):               # (heads not side by side; decode attention takes no stride)
        calls["novakv_int4_append"](0, *{**_args("novakv_int4_append"), "k_new": torch.zeros((N, 2 * HKV, D), dtype=torch.bfloat16)[:, ::2]}.values())
    with pytest.raises(ValueError, match="contiguous"):
        calls["novakv_int4_decode_attention"](0, *{**_args("novakv_int4_decode_attention"), "q": q}.values())


def test_outputs_of_two_types_and_too_few_lengths(calls):
    good = _args("novakv_int4_gather")
    with pytest.raises(ValueError, match="type"):
        calls["novakv_int4_gather"](0, *{**good, "k_out": _rows(HKV, torch.float32)}.values())
    good = _args("novakv_int4_decode_attention")
    for arg, w in (("page_table", _ints(2, 4)), ("seq_lens", _ints(2))):
        with pytest.raises(ValueError):
            calls["novakv_int4_decode_attention"](0, *{**good, arg: w}.values())


@pytest.mark.parametrize("kwargs", [dict(inv_freq=torch.zeros(32, dtype=torch.float64)), dict(q_weight=torch.zeros(64)),
                                    dict(inv_freq=torch.zeros(2, 16)), dict(inv_freq=torch.zeros(64)[::2])])
def test_transform_refuses(kwargs):
    with pytest.raises(ValueError):
        binding.QKTransform(**kwargs)


def test_transform_has_to_fit_the_context():
    tr = binding.QKTransform(q_weight=torch.zeros(64, dtype=torch.bfloat16))
    tr.check(64, -1)
    with pytest.raises(ValueError):
        tr.check(128, -1)
    with pytest.raises(ValueError):
        tr.check(64, 0)


def test_entry_points_refuse_a_null_context():
    lib = binding.load_library()
    assert lib.novakv_qk_norm_rope(None, None, None, 0, None, 0, None, 0, None, 0, None, 0, None) == EINVAL
    for f in (lib.novakv_bf16_append, lib.novakv_int4_append):
        assert f(None, None, None, 0, None, 0, None, None, 0, None, None, 0, None, 0, 0, None, None, 0, None, 0, None) == EINVAL
    assert lib.novakv_int4_gather(None, None, None, 0, None, None, 0, None, 0, 0, None, None, 0, None) == EINVAL
    assert lib.novakv_int4_decode_attention(None, None, None, None, 0, None, 0, None, 0, 1.0, 0, None, None, 0, None, 0, None) == EINVAL
    assert lib.novakv_int4_page_bytes(None) == 0 and lib.novakv_int4_workspace_bytes(None, 1) == 0


# ------------------------------------------------------------------------------------------------ layout and reference
@pytest.mark.parametrize("d", [64, 128])
def test_page_layout(d):
    codes, pairs = cache_format.int4_code_offsets(d), cache_format.int4_pair_offsets(d)
    used = np.concatenate([codes.ravel(), (pairs[..., None] + np.arange(4)).ravel()])
    assert np.array_equal(np.sort(used), np.arange(cache_format.int4_chunk_bytes(d)))          # every byte once
    # eight rows that a matrix load reads at a time, one 16-byte piece each, lie in eight different groups of banks
    for t in range(0, 64, 8):
        for p in range(d // 32):
            assert len(set(codes[t:t + 8, 16 * p] // 16 % 8)) == 8


@pytest.mark.parametrize("d", [64, 128])
def test_write_and_read_tokens(d):
    gen = np.random.default_rng(0)
    hkv, table = 3, np.array([4, 0, 2], np.int32)
    pool = gen.integers(0, 256, (5, hkv * cache_format.int4_chunk_bytes(d)), dtype=np.uint8)
    before = pool.copy()
    pos = np.arange(30, 161)
    x = R.to_bf16(gen.normal(size=(len(pos), hkv, d)))
    c, s, z = R.quantise(x)
    R.write_tokens(pool, table, pos, hkv, d, c, s, z)
    c2, s2, z2 = cache_format.int4_read_tokens(pool, table, hkv, d, 30, len(pos))
    assert np.array_equal(c, c2) and np.array_equal(s, s2) and np.array_equal(z, z2)
    # half a step, and what the roundings of zero (2^-9 of it) and of scale (15 steps of 2^-9 each) leave outside 0..15
    assert (np.abs(R.values(c, s, z) - x) <= (0.5 * s + R.bf16_eps * (np.abs(z) + 15 * s)).repeat(64, -1)).all()
    assert np.array_equal(pool[[1, 3]], before[[1, 3]])


def test_quantiser_corners():
    g = np.zeros((5, 64), np.float32)
    g[1] = 3.25
    g[2] = np.linspace(-1, 2, 64)
    g[3, 7] = np.nan
    g[4, 9] = np.inf
    c, s, z = R.quantise(g)
    assert s[0] == 1 and z[0] == 0 and not c[0].any()
    assert s[1] == 1 and z[1] == 3.25 and not c[1].any()
    assert c[2][0] == 0 and c[2][-1] == 15
    assert np.isnan(z[3]) and s[3] == 1 and not c[3].any()
    assert z[4] == 0 and s[4] == 1 and c[4][9] == 15 and c[4].sum() == 15


def test_rotation_identities():
    gen = np.random.default_rng(1)
    x, f = gen.normal(size=(4, 2, 64)), (10000.0 ** (-np.arange(32) / 32)).astype(np.float32)
    assert np.allclose(R.transform(x, np.zeros(4), f)[0], x)
    for il in (False, True):
        y, _ = R.transform(x, np.full(4, 77), f, interleaved=il)
        assert np.allclose(R.transform(y, np.full(4, -77), f, interleaved=il)[0], x)
        assert np.allclose((y ** 2).sum(-1), (x ** 2).sum(-1))
        # products of rotated rows depend on the distance alone
        a, b = (R.transform(x, np.full(4, p), f, interleaved=il)[0] for p in (105, 100))
        c, e = (R.transform(x, np.full(4, p), f, interleaved=il)[0] for p in (5, 0))
        assert np.allclose((a * b[::-1]).sum(-1), (c * e[::-1]).sum(-1))
    w = np.ones(64)
    assert np.allclose((R.transform(x, np.zeros(4), weight=w, eps=0.0)[0] ** 2).mean(-1), 1)


def test_attention_reference_against_torch():
    gen = np.random.default_rng(2)
    q, k, v = gen.normal(size=(4, 64)), gen.normal(size=(50, 2, 64)), gen.normal(size=(50, 2, 64))
    o, _, _ = R.attention(q, k, v, 0.125)
    z = torch.softmax(0.125 * torch.einsum("hgd,nhd->hgn", torch.tensor(q).view(2, 2, 64), torch.tensor(k)), -1)
    assert np.allclose(o, torch.einsum("hgn,nhd->hgd", z, torch.tensor(v)).reshape(4, 64).numpy())
    far, _, _ = R.attention(q, k, v, 0.125, sink=np.full(4, 1e4))
    none, _, _ = R.attention(q, k, v, 0.125, sink=np.full(4, -1e4))
    assert not far.any() and np.allclose(none, o)
