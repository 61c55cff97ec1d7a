"""What the operators around the paged caches are measured on: per-head norms and position rotation of queries and keys, the
append of a step's or a prompt's keys and values to the BF16 and to the 4-bit cache, the read-back of the 4-bit cache, and
decode attention over it.

    listed() -> cases    draw(rng) -> case    prepare(case, seed) -> state    run(state) -> outputs
    work(case) -> bytes, flops                exact(case, seed) -> outputs in 64 bits

``own`` selects the library's calls; otherwise the operators are computed in their plain form.
"""
from __future__ import annotations

import functools
import math

import numpy as np
import torch

own = False

DEV = "cuda:0"
PAGE, TILE, GROUP = 64, 32, 64             # tokens of a page, of a tile of the 4-bit page; channels that share (scale, zero)
MODELS = {"qwen3_8b": (32, 8, 128), "gpt_oss_20b": (64, 8, 64)}      # query heads, KV heads, head dimension
SHAPES = [(32, 8, 128), (64, 8, 64), (16, 8, 128), (8, 8, 128), (32, 8, 64), (8, 8, 64)]
EPS = 1e-6
YARN = 0.1 * math.log(32.0) + 1.0          # amplitude of a context extended 32 times


def _case(name, kind, heads, **more):
    hq, hkv, d = MODELS[heads] if isinstance(heads, str) else heads
    case = {"kind": kind, "hq": hq, "hkv": hkv, "d": d, **more}
    return {"name": name, **case} if name else case


def _rotation(name, kind, heads, tokens, *, norm=True, rot=None, interleaved=False, amplitude=1.0, seqs=0, first=0, with_q=True):
    """seqs = 0: one token of each of `tokens` sequences (a decode step); else prompts of `tokens` tokens in all."""
    d = (MODELS[heads] if isinstance(heads, str) else heads)[2]
    return _case(name, kind, heads, tokens=tokens, norm=norm, rot=rot or d, interleaved=interleaved, amplitude=amplitude, seqs=seqs,
                 first=first, with_q=with_q)


def _decode(name, heads, batch, length, *, ragged=False, window=0, sink=False, out="bf16"):
    return _case(name, "decode", heads, batch=batch, length=length, ragged=ragged, window=window, sink=sink, out=out)


def listed():
    return [
        # one user's decode step, before the 2-bit cache's append and attention: nothing but latency
        _rotation("qk_b1", "qk", "qwen3_8b", 1),
        # a long prompt of the model without norms, rows cut out of the fused projection
        _rotation("qk_prompt_16384", "qk", "gpt_oss_20b", 16384, norm=False, amplitude=YARN, seqs=1),
        # sliding-window layer of a decode step of 16 sequences
        _rotation("append_bf16_b16", "append_bf16", "gpt_oss_20b", 16, norm=False, amplitude=YARN),
        # one chunk of a chunked prefill, odd length, starting inside a page
        _rotation("append_bf16_8191", "append_bf16", "gpt_oss_20b", 8191, norm=False, amplitude=YARN, seqs=1, first=4133),
        # a decode step of 128 sequences: append, and the appended rows read back
        _rotation("append_int4_b128", "append_int4", "qwen3_8b", 128),
        # four prompts of together 16384 tokens
        _rotation("append_int4_16384", "append_int4", "qwen3_8b", 16384, seqs=4),
        # the cached prefix of a prompt, for the attention of its next chunk
        _case("gather_int4_24575", "gather", "qwen3_8b", tokens=24575, seqs=1, first=0, out="bf16"),
        # interactive single user, short context
        _decode("decode_int4_b1_s777", "qwen3_8b", 1, 777, out="fp32"),
        # small-batch serving step at medium context
        _decode("decode_int4_b8_s16384", "qwen3_8b", 8, 16384),
        # continuous batching, lengths over two orders of magnitude
        _decode("decode_int4_mix32", "qwen3_8b", 32, 32768, ragged=True),
        # the long-context batch of the d = 64 model, learned sink logits
        _decode("decode_int4_gptoss_b16_s65536", "gpt_oss_20b", 16, 65536, sink=True),
        # its sliding-window layer
        _decode("decode_int4_window128_b16", "gpt_oss_20b", 16, 8192, window=128, sink=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    heads = rng.choice(SHAPES)
    hq, hkv, d = heads
    kind = rng.choice(["qk", "append_bf16", "append_int4", "append_int4", "gather", "decode", "decode", "decode", "decode"])
    if kind == "decode":
        batch = _log_int(rng, 1, 64)
        length = min(_log_int(rng, 5, 65536), 2 ** 20 * 64 // (batch * d))
        window = rng.choice([0, 0, 0, 128, 1000])
        return _decode(None, heads, batch, length, ragged=rng.random() < 0.5, window=window, sink=rng.random() < 0.4,
                       out=rng.choice(["bf16", "bf16", "fp32"]))
    tokens = _log_int(rng, 1, 16384)
    seqs = min(rng.choice([0, 1, 1, 3]), tokens) if tokens <= 128 else rng.choice([1, 1, 3, 5])
    first = 0 if seqs == 0 else rng.choice([0, 0, 64, rng.randint(1, 5000)])
    if kind == "gather":
        return _case(None, kind, heads, tokens=tokens, seqs=max(seqs, 1), first=first, out=rng.choice(["bf16", "fp32"]))
    return _rotation(None, kind, heads, tokens, norm=rng.random() < 0.5, rot=rng.choice([d, d, d // 2]), interleaved=rng.random() < 0.3,
                     amplitude=rng.choice([1.0, YARN]), seqs=seqs, first=first, with_q=kind == "qk" or rng.random() < 0.7)


# ------------------------------------------------------------------------------------------------ geometry
def _lengths(case):
    """Lengths of a decode case's sequences: part of the case, not of the seed."""
    if not case["ragged"]:
        return np.full(case["batch"], case["length"], np.int64)
    gen = np.random.default_rng(case["batch"] * 100003 + case["length"])
    lens = np.exp(gen.uniform(np.log(max(1.0, case["length"] / 200)), np.log(case["length"]), case["batch"])).astype(np.int64)
    lens[gen.integers(case["batch"])] = case["length"]
    return np.maximum(lens, 1)


def _tokens(case):
    """(sequence, position) of the tokens that a call appends or reads, and the lengths afterwards: part of the case, too."""
    n, seqs = case["tokens"], case["seqs"]
    gen = np.random.default_rng(n * 8191 + seqs)
    if seqs == 0:                                              # a decode step: one token of each sequence, at its end
        pos = np.exp(gen.uniform(np.log(64), np.log(8192), n)).astype(np.int64)
        return np.arange(n), pos, pos + 1
    cuts = np.sort(gen.choice(np.arange(1, n), seqs - 1, replace=False)) if seqs > 1 else np.zeros(0, np.int64)
    counts = np.diff(np.concatenate([[0], cuts, [n]]))
    seq = np.repeat(np.arange(seqs), counts)
    pos = case["first"] + np.concatenate([np.arange(c) for c in counts])
    return seq, pos, case["first"] + counts


def _pages(lens, gen):
    """Shuffled page table [sequences][pages] and the number of pages; entries behind a sequence name page 0."""
    per = -(-np.maximum(lens, 1) // PAGE)
    ids = gen.permutation(int(per.sum()))
    table = np.zeros((len(lens), int(per.max())), np.int32)
    at = np.concatenate([[0], np.cumsum(per)])
    for b in range(len(lens)):
        table[b, :per[b]] = ids[at[b]:at[b + 1]]
    return table, len(ids)


def _row_bytes(d):
    return d // 2 + d // GROUP * 4                             # codes and (scale, zero) pairs of one token and head


def _i32(x):
    return torch.as_tensor(np.ascontiguousarray(x), dtype=torch.int32).to(DEV)


# ------------------------------------------------------------------------------------------------ state
def prepare(case, seed):
    gen = np.random.default_rng(seed)
    g = torch.Generator(device=DEV).manual_seed(seed)
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    randn = lambda *shape: torch.randn(shape, generator=g, device=DEV)  # noqa: E731
    s = {"case": case}
    if case["kind"] == "decode":
        lens = _lengths(case)
        table, n_pages = _pages(lens, gen)
        s |= {"lens": _i32(lens), "table": _i32(table), "k_pages": _cache4(n_pages, hkv, d, g), "v_pages": _cache4(n_pages, hkv, d, g)}
        # key rows have about unit variance (codes of 3 steps, steps of 1/3): logits of a standard deviation of 3
        s["q"] = (3.0 * randn(case["batch"], hq, d)).to(torch.bfloat16)
        s["sink"] = randn(hq) if case["sink"] else None
        return s
    seq, pos, lens = _tokens(case)
    s |= {"seq": _i32(seq), "pos": _i32(pos)}
    if case["kind"] != "qk":
        table, n_pages = _pages(lens, gen)
        s |= {"table": _i32(table), "n_pages": n_pages, "lens": torch.zeros(len(lens), dtype=torch.int32, device=DEV)}
    if case["kind"] == "gather":
        return s | {"k_pages": _cache4(n_pages, hkv, d, g), "v_pages": _cache4(n_pages, hkv, d, g)}
    # rows of the fused projection [tokens][(Hq + 2 Hkv) d]; a few key channels are outliers
    qkv = randn(case["tokens"], hq + 2 * hkv, d)
    qkv[:, hq:hq + hkv, torch.randperm(d, generator=g, device=DEV)[:4]] *= 10
    qkv = qkv.to(torch.bfloat16)
    s |= {"q": qkv[:, :hq] if case["with_q"] else None, "k": qkv[:, hq:hq + hkv], "v": qkv[:, hq + hkv:]}
    s["inv_freq"] = (1e6 if case["norm"] else 150000.0) ** (-torch.arange(0, case["rot"], 2, device=DEV, dtype=torch.float64) / case["rot"])
    s["inv_freq"] = s["inv_freq"].float()
    weight = lambda: (1 + 0.2 * randn(d)).to(torch.bfloat16) if case["norm"] else None  # noqa: E731
    s["q_weight"], s["k_weight"] = weight(), weight()
    if case["kind"] == "append_bf16":
        s["k_pages"], s["v_pages"] = (torch.zeros((n_pages, hkv, PAGE, d), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    if case["kind"] == "append_int4":
        s["k_pages"], s["v_pages"] = (torch.zeros((n_pages, hkv * PAGE * _row_bytes(d)), dtype=torch.uint8, device=DEV) for _ in range(2))
    return s


def _cache4(n_pages, hkv, d, g):
    """A pool of the 4-bit cache as quantised near-Gaussian rows leave it."""
    codes = (torch.randn((n_pages, hkv, 2, TILE, d), generator=g, device=DEV, dtype=torch.float16) * 3 + 7.5).round().clamp(0, 15).to(torch.uint8)
    scale = (torch.exp(0.25 * torch.randn((n_pages, hkv, 2, TILE, d // GROUP), generator=g, device=DEV)) / 3).to(torch.bfloat16)
    zero = (-7.5 * scale.float() + 0.1 * torch.randn(scale.shape, generator=g, device=DEV)).to(torch.bfloat16)
    return _pack(codes, scale, zero).reshape(n_pages, -1)


# ------------------------------------------------------------------------------------------------ the 4-bit page, in torch
@functools.cache
def _swizzle(d):
    """Where the 16-byte pieces of a token's codes are kept, [32][pieces]: its own inverse."""
    t, pieces = torch.arange(TILE, device=DEV)[:, None], d // 32
    return torch.arange(pieces, device=DEV)[None] ^ ((t * pieces // 8) & (pieces - 1))


def _pieces(rows, d):
    """Code bytes [..., 32][d / 2] in the page's order from the channels' order, or back."""
    pieces = rows.unflatten(-1, (d // 32, 16))
    return pieces.gather(-2, _swizzle(d)[..., None].expand(pieces.shape)).flatten(-2)


def _pack(codes, scale, zero):
    """[..., 32][d] codes and [..., 32][groups] scales and zeros -> the bytes of tiles [..., bytes]."""
    rows = _pieces(codes[..., 0::2] | codes[..., 1::2] << 4, codes.shape[-1])
    meta = torch.stack([scale, zero], -1).flatten(-3).view(torch.uint8)
    return torch.cat([rows.flatten(-2), meta], -1)


def _unpack(tiles, d, dtype):
    """The values [..., 32][d] that tiles stand for."""
    rows = _pieces(tiles[..., :TILE * d // 2].unflatten(-1, (TILE, d // 2)), d)
    codes = torch.stack([rows & 15, rows >> 4], -1).flatten(-2).to(dtype).unflatten(-1, (d // GROUP, GROUP))
    meta = tiles[..., TILE * d // 2:].contiguous().view(torch.bfloat16).to(dtype).unflatten(-1, (TILE, d // GROUP, 2))
    return (codes * meta[..., :1] + meta[..., 1:]).flatten(-2)


def _slots(s):
    """Page, tile of the page and row of the tile of every token."""
    pos = s["pos"].long()
    return s["table"][s["seq"].long(), pos // PAGE].long(), pos % PAGE // TILE, pos % TILE


def _byte_index(s, d):
    """Byte offsets in a (page, head) chunk [tokens][d / 2] of a token's codes and [tokens][4 groups] of its pairs."""
    _, tile, row = _slots(s)
    base = tile * (TILE * _row_bytes(d))
    at = torch.arange(d // 2, device=DEV)
    piece = _swizzle(d)[row][:, at // 16]
    codes = (base + row * (d // 2))[:, None] + piece * 16 + at % 16
    pairs = (base + TILE * d // 2 + row * (d // GROUP * 4))[:, None] + torch.arange(d // GROUP * 4, device=DEV)
    return codes, pairs


# ------------------------------------------------------------------------------------------------ one pass
def run(s):
    return (_run_own if own else _run_plain)(s)


def _run_plain(s):
    case = s["case"]
    kind = case["kind"]
    if kind == "decode":
        return _plain_decode(s)
    if kind == "gather":
        return tuple(_plain_gather(s, s[p], torch.float32 if case["out"] == "fp32" else torch.bfloat16) for p in ("k_pages", "v_pages"))
    # the 4-bit codes are decided in 64 bits: a key next to a border would fall to either side in 32
    dtype = torch.float64 if kind == "append_int4" else torch.float32
    q = None if s["q"] is None else _plain_transform(s, s["q"], s["q_weight"], torch.float32).to(torch.bfloat16)
    k = _plain_transform(s, s["k"], s["k_weight"], dtype)
    if kind == "qk":
        return q, k.to(torch.bfloat16)
    s["lens"].scatter_reduce_(0, s["seq"].long(), s["pos"] + 1, "amax")
    if kind == "append_bf16":
        page, tile, row = _slots(s)
        s["k_pages"][page, :, tile * TILE + row] = k.to(torch.bfloat16)
        s["v_pages"][page, :, tile * TILE + row] = s["v"]
        return q, s["k_pages"], s["v_pages"], s["lens"]
    _plain_append4(s, s["k_pages"], k.float())
    _plain_append4(s, s["v_pages"], s["v"].float())
    return q, _plain_gather(s, s["k_pages"], torch.bfloat16), _plain_gather(s, s["v_pages"], torch.bfloat16), s["lens"]


def _plain_transform(s, x, weight, dtype):
    case, x = s["case"], x.to(dtype)
    if weight is not None:
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * weight.to(dtype)
    angle = s["pos"].double()[:, None] * s["inv_freq"].double()
    cos, sin = ((f(angle) * case["amplitude"]).to(dtype)[:, None] for f in (torch.cos, torch.sin))
    turned, rest = x[..., :case["rot"]], x[..., case["rot"]:]
    if case["interleaved"]:
        a, b = turned[..., 0::2], turned[..., 1::2]
        turned = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    else:
        a, b = turned.chunk(2, -1)
        turned = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    return torch.cat([turned, rest], -1)


def _plain_append4(s, pool, x):
    case = s["case"]
    hkv, d = case["hkv"], case["d"]
    x = x.unflatten(-1, (d // GROUP, GROUP))
    zero = x.amin(-1, keepdim=True).to(torch.bfloat16).float()
    scale = ((x.amax(-1, keepdim=True) - zero) / 15).to(torch.bfloat16).float()
    scale = torch.where((scale > 0) & torch.isfinite(scale), scale, torch.ones_like(scale))
    code = ((x - zero) / scale).round().clamp(0, 15).to(torch.uint8).flatten(-2)
    pairs = torch.cat([scale, zero], -1).to(torch.bfloat16).flatten(-2).view(torch.uint8)
    at_codes, at_pairs = _byte_index(s, d)
    chunk, page = pool.view(-1, hkv, PAGE * _row_bytes(d)), _slots(s)[0]
    head = torch.arange(hkv, device=DEV)[None, :, None]
    chunk[page[:, None, None], head, at_codes[:, None]] = code[..., 0::2] | code[..., 1::2] << 4
    chunk[page[:, None, None], head, at_pairs[:, None]] = pairs


def _plain_gather(s, pool, dtype):
    case = s["case"]
    hkv, d = case["hkv"], case["d"]
    at_codes, at_pairs = _byte_index(s, d)
    chunk, page = pool.view(-1, hkv, PAGE * _row_bytes(d)), _slots(s)[0]
    head = torch.arange(hkv, device=DEV)[None, :, None]
    rows = chunk[page[:, None, None], head, at_codes[:, None]]
    pairs = chunk[page[:, None, None], head, at_pairs[:, None]].view(torch.bfloat16).float().unflatten(-1, (d // GROUP, 2))
    codes = torch.stack([rows & 15, rows >> 4], -1).flatten(-2).float().unflatten(-1, (d // GROUP, GROUP))
    return (codes * pairs[..., :1] + pairs[..., 1:]).flatten(-2).to(dtype)


def _plain_decode(s):
    case = s["case"]
    hq, hkv, d, batch = case["hq"], case["hkv"], case["d"], case["batch"]

    def rows(pool):                                            # [batch][Hkv][positions][d]
        tiles = pool.view(-1, hkv, 2, TILE * _row_bytes(d))[s["table"].long()]
        return _unpack(tiles, d, torch.float32).permute(0, 2, 1, 3, 4, 5).reshape(batch, hkv, -1, d)

    q = s["q"].float().view(batch, hkv, hq // hkv, d)
    z = q @ rows(s["k_pages"]).transpose(-1, -2) * d ** -0.5
    pos, lens = torch.arange(z.shape[-1], device=DEV), s["lens"][:, None]
    seen = pos < lens
    if case["window"]:
        seen = seen & (pos >= lens - case["window"])
    z = z.masked_fill(~seen[:, None, None], -math.inf)
    top = z.amax(-1, keepdim=True)
    sink = None
    if s["sink"] is not None:
        sink = s["sink"].view(hkv, hq // hkv, 1)
        top = torch.maximum(top, sink)
    p = torch.exp(z - top)
    total = p.sum(-1, keepdim=True)
    if sink is not None:
        total = total + torch.exp(sink - top)
    # rows behind a sequence may hold anything: their weight is zero, their value is taken out
    v = rows(s["v_pages"]).masked_fill(~seen[:, None, :, None], 0.0)
    out = (p @ v / total).view(batch, hq, d)
    return out if case["out"] == "fp32" else out.to(torch.bfloat16)


# ------------------------------------------------------------------------------------------------ the library's calls
@functools.cache
def _context(hq, hkv, d):
    from paper_2608_04074_b200.binding import Context
    return Context(hq, hkv, d)


@functools.cache
def _workspace(hq, hkv, d, batch):
    ctx = _context(hq, hkv, d)
    return torch.empty(ctx.novakv_int4_workspace_bytes(batch), dtype=torch.uint8, device=DEV)


def _transform(s):
    """Frequencies and weights of the layer: laid down once, as a program keeps them."""
    if "transform" not in s:
        from paper_2608_04074_b200.binding import QKTransform
        s["transform"] = QKTransform(s["inv_freq"], interleaved=s["case"]["interleaved"], amplitude=s["case"]["amplitude"],
                                     q_weight=s["q_weight"], k_weight=s["k_weight"], eps=EPS)
    return s["transform"]


def _run_own(s):
    case = s["case"]
    kind, hq, hkv, d = case["kind"], case["hq"], case["hkv"], case["d"]
    ctx = _context(hq, hkv, d)
    if kind == "decode":
        out = torch.empty((case["batch"], hq, d), dtype=torch.float32 if case["out"] == "fp32" else torch.bfloat16, device=DEV)
        ctx.novakv_int4_decode_attention(s["q"], s["k_pages"], s["v_pages"], s["table"], s["lens"], out,
                                         _workspace(hq, hkv, d, case["batch"]), window=case["window"], sink_logits=s["sink"])
        return out
    n = case["tokens"]
    rows = lambda heads, dtype=torch.bfloat16: torch.empty((n, heads, d), dtype=dtype, device=DEV)  # noqa: E731
    if kind == "gather":
        k, v = (rows(hkv, torch.float32 if case["out"] == "fp32" else torch.bfloat16) for _ in range(2))
        ctx.novakv_int4_gather(s["seq"], s["pos"], s["k_pages"], s["v_pages"], s["table"], k, v)
        return k, v
    q = None if s["q"] is None else rows(hq)
    if kind == "qk":
        k = rows(hkv)
        ctx.novakv_qk_norm_rope(_transform(s), s["q"], s["k"], s["pos"], q, k)
        return q, k
    append = ctx.novakv_bf16_append if kind == "append_bf16" else ctx.novakv_int4_append
    append(_transform(s), s["k"], s["v"], s["seq"], s["pos"], s["k_pages"], s["v_pages"], s["table"], s["lens"], q=s["q"], q_out=q)
    if kind == "append_bf16":
        return q, s["k_pages"], s["v_pages"], s["lens"]
    k, v = rows(hkv), rows(hkv)
    ctx.novakv_int4_gather(s["seq"], s["pos"], s["k_pages"], s["v_pages"], s["table"], k, v)
    return q, k, v, s["lens"]


# ------------------------------------------------------------------------------------------------ what a pass cannot do without
def work(case):
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    if case["kind"] == "decode":
        lens = _lengths(case)
        seen = int((np.minimum(lens, case["window"]) if case["window"] else lens).sum())
        out = 4 if case["out"] == "fp32" else 2
        return {"bytes": seen * hkv * 2 * _row_bytes(d) + case["batch"] * hq * d * (2 + out), "flops": 4 * seen * hq * d}
    n = case["tokens"]
    if case["kind"] == "gather":
        return {"bytes": n * hkv * 2 * (_row_bytes(d) + d * (4 if case["out"] == "fp32" else 2)), "flops": n * hkv * d * 4}
    rows = (hq if case["with_q"] else 0) + hkv
    per = rows * d * 2 * 2 + 4                                 # q and k, read and written; the position
    flops = rows * d * 7
    if case["kind"] == "append_bf16":
        per += hkv * d * 2 * 2 + 4                             # v read and written; the sequence
    if case["kind"] == "append_int4":                          # k and v: read in BF16, written in 4 bits, read back as BF16
        per += hkv * d * 2 * 2 + hkv * 2 * _row_bytes(d) + 4
        flops += hkv * d * 12
    return {"bytes": n * per, "flops": n * flops}


# ------------------------------------------------------------------------------------------------ from the definition, in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "decode":
        return _exact_decode(s)
    if case["kind"] == "gather":
        return tuple(_exact_rows(s, s[p]) for p in ("k_pages", "v_pages"))
    q = None if s["q"] is None else _exact_turn(s, s["q"], s["q_weight"])
    k = _exact_turn(s, s["k"], s["k_weight"])
    if case["kind"] == "qk":
        return q, k
    if case["kind"] == "append_int4":
        return q, _exact_quantised(k), _exact_quantised(s["v"].double()), None
    pools = []
    for x in (k, s["v"].double()):
        where = s["table"].long()[s["seq"].long(), s["pos"].long() // PAGE] * PAGE + s["pos"].long() % PAGE
        slots = torch.zeros((s["n_pages"] * PAGE, case["hkv"], case["d"]), dtype=torch.float64, device=DEV)
        slots[where] = x
        pools.append(slots.view(s["n_pages"], PAGE, case["hkv"], case["d"]).transpose(1, 2).contiguous())
    return q, pools[0], pools[1], None


def _exact_turn(s, x, weight):
    """As products of complex numbers."""
    case, x = s["case"], x.double()
    if weight is not None:
        x = x / ((x ** 2).sum(-1, keepdim=True) / case["d"] + EPS).sqrt() * weight.double()
    half = case["rot"] // 2
    i = torch.arange(half, device=DEV)
    a, b = (2 * i, 2 * i + 1) if case["interleaved"] else (i, i + half)
    turn = torch.polar(torch.full((case["tokens"], half), float(case["amplitude"]), dtype=torch.float64, device=DEV),
                       torch.outer(s["pos"].double(), s["inv_freq"].double()))
    z = torch.complex(x[..., a], x[..., b]) * turn[:, None]
    y = x.clone()
    y[..., a], y[..., b] = z.real, z.imag
    return y


def _exact_quantised(x):
    y = x.float().double()                                     # the definition quantises the binary32 number
    out = torch.empty_like(y)
    for c in range(0, y.shape[-1], GROUP):
        part = y[..., c:c + GROUP]
        zero = part.min(-1, keepdim=True).values.bfloat16().double()
        step = ((part.max(-1, keepdim=True).values - zero) / 15).float().bfloat16().double()
        step[~((step > 0) & (step < math.inf))] = 1.0
        out[..., c:c + GROUP] = zero + step * ((part - zero) / step).round().clamp(0, 15)
    return out


def _exact_rows(s, pool):
    """Token by token through the byte addresses, all heads at once."""
    case = s["case"]
    hkv, d = case["hkv"], case["d"]
    page = s["table"].long()[s["seq"].long(), s["pos"].long() // PAGE]
    return _exact_values(pool, page, s["pos"].long() % PAGE, hkv, d)


def _exact_values(pool, page, slot, hkv, d):
    """Values [tokens][Hkv][d] of slots of pages: byte c / 2 of a row of d / 2 bytes holds channel c in its low (even c) or high
    four bits; 16-byte pieces of a row are permuted; the rows of 32 tokens are followed by their bfloat16 (scale, zero) pairs."""
    tile_bytes = 32 * (d // 2 + d // 64 * 4)
    chunk = pool.view(pool.shape[0], hkv, 2 * tile_bytes)
    base = slot // 32 * tile_bytes
    t = slot % 32
    out = torch.empty((len(page), hkv, d), dtype=torch.float64, device=DEV)
    for c in range(0, d, 32):                                  # one 16-byte piece
        turn = t // 2 % 4 if d == 128 else t // 4 % 2
        start = base + t * (d // 2) + (c // 32 ^ turn) * 16
        pair = base + 32 * (d // 2) + (t * (d // 64) + c // 64) * 4
        h = torch.arange(hkv, device=DEV)[None, :, None]
        two = chunk[page[:, None, None], h, pair[:, None, None] + torch.arange(4, device=DEV)].to(torch.int32)
        scale, zero = ((two[..., 2 * i] | two[..., 2 * i + 1] << 8) << 16 for i in (0, 1))
        scale, zero = (x.view(torch.float32).double() for x in (scale.contiguous(), zero.contiguous()))
        byte = chunk[page[:, None, None], h, start[:, None, None] + torch.arange(16, device=DEV)]
        out[..., c:c + 32:2] = zero[..., None] + scale[..., None] * (byte % 16).double()
        out[..., c + 1:c + 32:2] = zero[..., None] + scale[..., None] * (byte // 16).double()
    return out


def _exact_decode(s):
    case = s["case"]
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    out = torch.empty((case["batch"], hq, d), dtype=torch.float64, device=DEV)
    for b, n in enumerate(_lengths(case)):
        pos = torch.arange(max(0, n - case["window"]) if case["window"] else 0, n, device=DEV)
        page = s["table"].long()[b, pos // PAGE]
        k = _exact_values(s["k_pages"], page, pos % PAGE, hkv, d)
        v = _exact_values(s["v_pages"], page, pos % PAGE, hkv, d)
        q = s["q"][b].double().view(hkv, hq // hkv, d)
        z = torch.einsum("hgd,nhd->hgn", q, k) / math.sqrt(d)
        if s["sink"] is not None:                              # one more logit, without a value
            z = torch.cat([z, s["sink"].double().view(hkv, hq // hkv, 1)], -1)
        p = torch.softmax(z, -1)[..., :len(pos)]
        out[b] = torch.einsum("hgn,nhd->hgd", p, v).reshape(hq, d)
    return out
