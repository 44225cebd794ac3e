"""Timing cases of a speculative serving step on a KV cache of 4 bits a value: append with rotary positions, reading rows back,
decode attention over the cache, verification of drafted tokens.

Every case is what a serving loop does with the public binding: ``xattn_rope_kvcache_mx`` on a step's fused QKV projection, with
``xattn_read_kvcache_mx`` behind it, whose rows are what ``xattn_prefill`` takes for a prompt; ``xattn_read_kvcache_mx`` of cached
rows; ``xattn_decode_mx``; ``xbeam_verify`` on a step's logits.  Beside the calls stand their plain forms, elementary operations in 32
bits (64 where a rounding decides a code or a token), and their definitions in 64 bits.

The cache: blocks of 32 values along a head of 128 share a scale 2^e (a byte, e + 127), a value is one of 0, 0.5, 1, 1.5, 2, 3, 4, 6 times
that, with a sign, in 4 bits.  64 tokens of a KV head are a tile of 4352 bytes, 4096 of codes and 256 of scales; a sequence's tiles lie one
behind the other, all heads of the same tokens together.
"""
import math
import random

import torch

own = False

HEAD_DIM, TILE, TILE_BYTES, CODE_BYTES = 128, 64, 4352, 4096
ROPE_BASE = 1e6
DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


# ------------------------------------------------------------------------------------------------ the cases
def _append(name, hq, hkv, groups, axes, pairs=False, far=0):
    """groups: text "count x q_lo..q_hi + prefix_lo..prefix_hi; ...": sequences, their new tokens, what the cache holds already."""
    return dict(name=name, op="append", n_q_heads=hq, n_kv_heads=hkv, groups=groups, axes=axes, pairs=pairs, far=far)


def _read(name, hkv, groups):
    return dict(name=name, op="read", n_q_heads=hkv, n_kv_heads=hkv, groups=groups)


def _decode(name, hq, hkv, q_len, groups):
    return dict(name=name, op="decode", n_q_heads=hq, n_kv_heads=hkv, q_len=q_len, groups=groups)


def _verify(name, batch, q_len, vocab, dtype, drafts="logits", ragged=False, greedy=False, pad=0, temperature=1.0, masked=0.0):
    return dict(name=name, op="verify", batch=batch, q_len=q_len, vocab=vocab, dtype=dtype, drafts=drafts, ragged=ragged, greedy=greedy, pad=pad,
                temperature=temperature, masked=masked)


def listed():
    return [
        # a decode step of four short requests of the smallest workload's head counts: latency
        _append("append_tiny_step", 8, 2, "4x1..1+16..255", axes=1),
        # a speculative step of many requests: three drafts and the token before them
        _append("append_verify_step", 40, 8, "256x4..4+16..4095", axes=1),
        # a video prompt: time, height and width, far into a long session
        _append("append_video_prompt", 32, 8, "2x4096..8191+0..64", axes=3, far=1000000),
        # what four short requests have cached, ahead of a second chunk of their prompts: latency
        _read("read_tiny", 2, "4x17..256+0..0"),
        # a long document's cached part, ahead of its next chunk
        _read("read_document", 8, "1x28672..28672+0..0"),
        # four short requests: latency
        _decode("decode_tiny", 8, 2, 1, "4x1..1+16..255"),
        # an ordinary step of an 8B-shaped model
        _decode("decode_chats", 32, 8, 1, "64x1..1+511..4095"),
        # long contexts, groups of eight
        _decode("decode_long", 64, 8, 1, "16x1..1+16383..32767"),
        # three drafts and the token before them are verified
        _decode("decode_verify", 32, 8, 4, "128x4..4+1024..8192"),
        # one request's four drafts, full vocabulary: latency
        _verify("verify_one", 1, 5, 131072, "bf16"),
        # the same of many requests
        _verify("verify_batch", 64, 5, 131072, "bf16", temperature=0.8),
        # drafts without probabilities (looked up in the prompt), not the same number everywhere; odd vocabulary in padded rows, part
        # of the tokens forbidden
        _verify("verify_lookup", 48, 4, 100003, "fp32", drafts="certain", ragged=True, pad=5, temperature=0.7, masked=0.3),
    ]


_HEADS = [(8, 2), (4, 4), (5, 1), (16, 2), (12, 2), (32, 8), (64, 8), (40, 8), (16, 8), (8, 1)]
_MOST_APPENDED, _MOST_READ, _MOST_KEYS, _MOST_LOGITS = 12000, 229000, 4.5e6, 7.5e7


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _draw_groups(rng, most_new, most_tokens):
    parts = []
    for _ in range(rng.choice([1, 1, 2])):
        if rng.random() < 0.3:
            q_hi, count = rng.randint(1, 5), _log_uniform(rng, 4, 256)
        else:
            q_hi = _log_uniform(rng, 5, most_new)
            count = _log_uniform(rng, 1, max(1, min(48, most_new // q_hi)))
        prefix = 0 if rng.random() < 0.4 else _log_uniform(rng, 16, max(17, most_tokens // count))
        parts.append("%dx%d..%d+%d..%d" % (count, max(1, q_hi // rng.choice([1, 2, 8])), q_hi, prefix // rng.choice([1, 4]), prefix))
    return ";".join(parts)


def draw(rng):
    """One more case: head counts of the workloads and tests; appends and reads of 1 to 16384 rows a sequence; decode steps of 1 to 256
    sequences of 1 to 40000 keys with 1 to 16 new tokens; verification of 0 to 7 drafts of 1 to 128 requests over 500 to 200000 tokens."""
    while True:
        op = rng.choice(["append", "read", "decode", "decode", "verify", "verify"])
        hq, hkv = rng.choice(_HEADS)
        if op == "append":
            case = _append("", hq, hkv, _draw_groups(rng, 12000, 60000), axes=rng.randint(1, 4), pairs=rng.random() < 0.4, far=rng.choice([0, 0, 70000, 4000000]))
            fits = sum(n for n, _ in _lengths(case)) * (hq + 2 * hkv) <= _MOST_APPENDED * 48 and sum(n for _, n in _lengths(case)) <= 250000
        elif op == "read":
            case = _read("", hkv, _draw_groups(rng, 16384, 60000))
            fits = sum(n for n, _ in _lengths(case)) * hkv <= _MOST_READ and sum(n for _, n in _lengths(case)) <= 250000
        elif op == "decode":
            q_len = rng.choice([1, 1, 1, 2, 3, 4, 5, 8, 16])
            count, hi = _log_uniform(rng, 1, 256), _log_uniform(rng, 16, 40000)
            lo = hi // rng.choice([1, 1, 2, 8])
            case = _decode("", hq, hkv, q_len, "%dx%d..%d+%d..%d" % (count, q_len, q_len, max(0, lo - q_len), max(0, hi - q_len)))
            fits = hq // hkv * q_len <= 64 and count * hi * hkv <= _MOST_KEYS
        else:
            batch, q_len, vocab = _log_uniform(rng, 1, 128), rng.randint(1, 8), _log_uniform(rng, 500, 200000)
            case = _verify("", batch, q_len, vocab, rng.choice(["bf16", "bf16", "fp16", "fp32"]), drafts=rng.choice(["logits", "logits", "certain"]),
                           ragged=rng.random() < 0.4, greedy=rng.random() < 0.2, pad=rng.choice([0, 0, rng.randint(1, 64)]),
                           temperature=rng.choice([1.0, round(rng.uniform(0.3, 2.0), 2)]), masked=rng.choice([0.0, 0.0, 0.25]))
            fits = batch * (2 * q_len - 1) * vocab <= _MOST_LOGITS
        if fits:
            del case["name"]
            return case


def _lengths(case, seed=None):
    """(new tokens, keys in all) of every sequence; the seed only decides which sequence has which."""
    rng = random.Random("%s %d" % (case["groups"], case["n_q_heads"]))
    lens = []
    for part in case["groups"].split(";"):
        count, rest = part.split("x")
        (q_lo, q_hi), (p_lo, p_hi) = (tuple(int(v) for v in r.split("..")) for r in rest.split("+"))
        for _ in range(int(count)):
            n = rng.randint(q_lo, q_hi)
            lens.append((n, n + rng.randint(p_lo, p_hi)))
    if seed is not None:
        random.Random(seed).shuffle(lens)
    return lens


def work(case):
    if case["op"] == "verify":
        rows = case["batch"] * (case["q_len"] + (case["q_len"] - 1 if case["drafts"] == "logits" and not case["greedy"] else 0))
        size = torch.empty(0, dtype=DTYPES[case["dtype"]]).element_size()
        return {"bytes": rows * case["vocab"] * size + case["batch"] * case["q_len"] * 16, "flops": 4 * rows * case["vocab"]}
    hq, hkv, lens = case["n_q_heads"], case["n_kv_heads"], _lengths(case)
    new, row = sum(n for n, _ in lens), 2 * TILE_BYTES // TILE
    if case["op"] == "append":
        return {"bytes": new * (4 * hq * HEAD_DIM + 4 * hkv * HEAD_DIM + 2 * hkv * row + 4 * hkv * HEAD_DIM + 4 * case["axes"]), "flops": 3 * new * (hq + hkv) * HEAD_DIM}
    if case["op"] == "read":
        return {"bytes": new * hkv * (row + 4 * HEAD_DIM), "flops": 2 * new * hkv * HEAD_DIM}
    seen = sum(n * (total - n) + n * (n + 1) // 2 for n, total in lens)
    return {"bytes": sum(total for _, total in lens) * hkv * row + new * hq * (4 * HEAD_DIM + 4), "flops": 4 * HEAD_DIM * hq * seen}


# ------------------------------------------------------------------------------------------------ the cache's format
def _codes(x):
    """(codes with signs, e + 127) of [rows, heads, 128]: e is the least with |x| <= 7 * 2^e in the block, a value goes to the nearest
    code, to the even one of two that are as near."""
    blocks = x.unflatten(-1, (4, 32))
    most = blocks.abs().amax(-1)
    fraction, power = torch.frexp(most)
    e = torch.where(most > 0, power - 3 + (fraction > 0.875), -125).clamp_(-125, 126)
    y = torch.ldexp(blocks, -e[..., None])
    a = y.abs()
    code = (a > 0.25).to(torch.uint8) + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5)
    return (code + 8 * torch.signbit(y).to(torch.uint8)).flatten(-2), (e + 127).to(torch.uint8)


def _values(codes, scales, dtype=torch.float32):
    """What codes and scales stand for, [rows, heads, 128]."""
    levels = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6, 0, -0.5, -1, -1.5, -2, -3, -4, -6], dtype=dtype, device=codes.device)
    return torch.ldexp(levels[codes.int()].unflatten(-1, (4, 32)), (scales.int() - 127)[..., None]).flatten(-2)


def _bytes_of(row, heads, is_v):
    """Where in a sequence's range the bytes of token `row` are, [rows, heads, 64] of codes and [rows, heads, 4] of scales."""
    d = row.device
    base = ((row // TILE)[:, None] * heads + torch.arange(heads, device=d))[..., None] * TILE_BYTES
    t = (row % TILE)[:, None, None]
    s, u = t // 16, t % 16
    byte, block = torch.arange(64, device=d), torch.arange(4, device=d)
    if is_v:      # 16 tokens: groups of four; 16 times 8 values (4 bytes), of which the four tokens' lie together
        g, r = u // 4, u % 4
        return base + s * 1024 + g * 256 + (byte // 4) * 16 + r * 4 + byte % 4, base + CODE_BYTES + (g * 4 + block) * 16 + s * 4 + r
    # 16 tokens: four blocks of 32 values (16 bytes), of which the 16 tokens' lie together
    return base + s * 1024 + (byte // 16) * 256 + u * 16 + byte % 16, base + CODE_BYTES + (block * 16 + u) * 4 + s


def _put(cache, start, row, heads, is_v, codes, scales):
    """Writes rows of tokens, of sequences whose ranges begin at the bytes `start` of the buffer."""
    at, at_scale = _bytes_of(row, heads, is_v)
    cache[at + start[:, None, None]] = codes[..., 0::2] | codes[..., 1::2] << 4
    cache[at_scale + start[:, None, None]] = scales


def _get(cache, start, row, heads, is_v):
    at, at_scale = _bytes_of(row, heads, is_v)
    both = cache[at + start[:, None, None]]
    return torch.stack((both & 15, both >> 4), -1).flatten(-2), cache[at_scale + start[:, None, None]]


# ------------------------------------------------------------------------------------------------ inputs
def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _sequences(case, seed):
    """Lengths, where the packed rows of a sequence begin, ranges, addresses, and the caches filled with rows from N(0, 1)."""
    lens, hkv = _lengths(case, seed), case["n_kv_heads"]
    starts, ends = [0], [0]
    for n, total in lens:
        starts.append(starts[-1] + n)
        ends.append(ends[-1] + -(-total // TILE) * hkv * TILE_BYTES)
    g = _generator(seed)
    s = dict(case=case, lens=lens, starts=starts, ends=ends, batch=len(lens), new=starts[-1], q_starts=_ints(starts), kv_lens=_ints([n for _, n in lens]))
    tiles = ends[-1] // TILE_BYTES // hkv
    for which in ("k", "v"):
        cache = torch.empty(ends[-1], dtype=torch.uint8, device="cuda")
        part = max(1, (1 << 25) // (hkv * HEAD_DIM * TILE))      # tiles at a time
        for at in range(0, tiles, part):
            row = torch.arange(at * TILE, min(tiles, at + part) * TILE, device="cuda")
            _put(cache, torch.zeros_like(row), row, hkv, which == "v", *_codes(torch.randn((row.shape[0], hkv, HEAD_DIM), generator=g, device="cuda")))
        s[which] = cache
        s[which + "_ptrs"] = torch.tensor([cache.data_ptr() + e for e in ends[:-1]], dtype=torch.int64, device="cuda")
    return s, g


def _rows(s):
    """(first byte of the range, row in the sequence) of each new token."""
    start = torch.cat([torch.full((n,), e) for e, (n, _) in zip(s["ends"], s["lens"])])
    return start.cuda(), torch.cat([torch.arange(total - n, total) for n, total in s["lens"]]).cuda()


def _positions(case, lens, axes):
    """Positions of the new tokens, [axes, new] int32: with one axis where a token stands in its sequence; with more, frames of
    24 x 24 patches, time counted on from the prefix (and from `far`)."""
    where = torch.cat([torch.arange(total - n, total) for n, total in lens])
    if axes == 1:
        return (where + case["far"]).to(torch.int32)[None]
    inside = torch.cat([torch.arange(n) for n, _ in lens])
    grid = [case["far"] + where - inside + inside // 576, inside // 24 % 24, inside % 24, inside % 7]
    return torch.stack(grid[:axes]).to(torch.int32)


def _sections(axes):
    """Frequencies of each axis, 64 in all."""
    return {1: [64], 2: [32, 32], 3: [16, 24, 24], 4: [10, 22, 22, 10]}[axes]


def _prepare_verify(case, seed):
    g = _generator(seed)
    batch, q_len, vocab, dtype = case["batch"], case["q_len"], case["vocab"], DTYPES[case["dtype"]]
    n = q_len - 1
    d = dict(device="cuda")
    wide = torch.empty((batch, q_len, vocab + case["pad"]), dtype=dtype, **d).normal_(0.0, 2.5, generator=g)
    target = wide[..., :vocab]
    # a model is sure of some tokens, and a draft of about the same
    likely = torch.randint(0, vocab, (batch, q_len, 1), generator=g, **d)
    target.scatter_add_(2, likely, (8 + 8 * torch.rand((batch, q_len, 1), generator=g, **d)).to(dtype))
    banned = torch.rand(vocab, generator=g, **d) < case["masked"]
    if case["masked"]:
        target[..., banned] = -math.inf
    scale = float(torch.tensor(1.0 / case["temperature"], dtype=torch.float32))      # as a call takes it
    s = dict(case=case, scale=scale, target=target, uniforms=torch.rand((batch, q_len), generator=g, **d), draft=None, n_drafts=None,
             tokens=torch.empty((batch, q_len), dtype=torch.int32, **d), accepted=torch.empty(batch, dtype=torch.int32, **d), lp=torch.empty((batch, q_len), **d))
    if n == 0:
        s["draft_tokens"] = torch.zeros((batch, 0), dtype=torch.int32, **d)
    elif case["drafts"] == "logits" and not case["greedy"]:
        draft = torch.empty((batch, n, vocab + case["pad"]), dtype=dtype, **d).normal_(0.0, 0.7, generator=g)
        draft += wide[:, :n]
        s["draft"] = draft[..., :vocab]
        p = torch.softmax(s["draft"].float() * scale, -1).view(batch * n, vocab)
        s["draft_tokens"] = torch.multinomial(p, 1, generator=g).view(batch, n).to(torch.int32)
    else:
        other = torch.randint(0, vocab, (batch, n), generator=g, **d)
        right = torch.rand((batch, n), generator=g, **d) < 0.8
        s["draft_tokens"] = torch.where(right, target[:, :n].argmax(-1), other).to(torch.int32)
    if case["ragged"]:
        s["n_drafts"] = torch.randint(0, n + 1, (batch,), generator=g, dtype=torch.int32, **d)
    return s


def prepare(case, seed):
    if case["op"] == "verify":
        return _prepare_verify(case, seed)
    s, g = _sequences(case, seed)
    hq, hkv, new = case["n_q_heads"], case["n_kv_heads"], s["new"]
    bf16 = dict(device="cuda", dtype=torch.bfloat16)
    if case["op"] == "decode":
        s["q"] = torch.randn((s["batch"], case["q_len"], hq, HEAD_DIM), generator=g, **bf16)
        s["out"] = torch.empty_like(s["q"])
        s["lse"] = torch.empty((s["batch"], case["q_len"], hq), device="cuda")
        return s
    s["k_rows"], s["v_rows"] = (torch.empty((new, hkv, HEAD_DIM), **bf16) for _ in range(2))
    if case["op"] == "append":
        axes = case["axes"]
        s["q_out"] = torch.empty((new, hq, HEAD_DIM), **bf16)
        s["qkv"] = torch.randn((new, (hq + 2 * hkv) * HEAD_DIM), generator=g, **bf16)
        s["pos"] = _positions(case, s["lens"], axes).to("cuda").contiguous()
        s["inv_freq"] = (ROPE_BASE ** (-torch.arange(64, dtype=torch.float64) / 64)).to(torch.float32).cuda()
        s["sections"] = _sections(axes)
        s["axis_of"] = torch.repeat_interleave(torch.arange(axes), torch.tensor(s["sections"])).cuda()
    s["range_start"], s["row"] = _rows(s)
    return s


# ------------------------------------------------------------------------------------------------ the calls and their plain forms
def run(state):
    return {"append": _run_append, "read": _run_read, "decode": _run_decode, "verify": _run_verify}[state["case"]["op"]](state)


def _split_pairs(x, pairs):
    return (x[..., 0::2], x[..., 1::2]) if pairs else (x[..., :64], x[..., 64:])


def _join_pairs(x, y, pairs):
    return torch.stack((x, y), -1).flatten(-2) if pairs else torch.cat((x, y), -1)


def _read_back(s):
    import paper_2510_14686_amd as xa
    xa.xattn_read_kvcache_mx(s["k_ptrs"], s["v_ptrs"], s["q_starts"], s["kv_lens"], s["batch"], s["new"], s["case"]["n_kv_heads"], HEAD_DIM, s["k_rows"],
                             s["v_rows"], torch.cuda.current_stream())
    return s["k_rows"], s["v_rows"]


def _run_append(s):
    case = s["case"]
    hq, hkv, new = case["n_q_heads"], case["n_kv_heads"], s["new"]
    q, k, v = s["qkv"].split([hq * HEAD_DIM, hkv * HEAD_DIM, hkv * HEAD_DIM], 1)
    if own:
        import paper_2510_14686_amd as xa
        xa.xattn_rope_kvcache_mx(q, k, v, q.stride(0), k.stride(0), v.stride(0), s["pos"], s["inv_freq"], s["sections"],
                                 xa.XATTN_ROPE_PAIRS if case["pairs"] else 0, s["k_ptrs"], s["v_ptrs"], s["q_starts"], s["kv_lens"], s["batch"], new,
                                 hq, hkv, HEAD_DIM, s["q_out"], torch.cuda.current_stream())
        return (s["q_out"],) + _read_back(s)
    angle = s["pos"].double()[s["axis_of"]].t() * s["inv_freq"].double()          # [new, 64]; 32 bits lose far positions
    cos, sin = angle.cos()[:, None], angle.sin()[:, None]
    x, y = _split_pairs(q.float().view(new, hq, HEAD_DIM), case["pairs"])
    c, n = cos.float(), sin.float()
    q_out = _join_pairs(x * c - y * n, y * c + x * n, case["pairs"]).to(torch.bfloat16)
    # K in 64 bits: a rounding decides between two codes
    x, y = _split_pairs(k.double().view(new, hkv, HEAD_DIM), case["pairs"])
    both = []
    for which, rows in (("k", _join_pairs(x * cos - y * sin, y * cos + x * sin, case["pairs"])), ("v", v.float().view(new, hkv, HEAD_DIM))):
        codes, scales = _codes(rows)
        _put(s[which], s["range_start"], s["row"], hkv, which == "v", codes, scales)
        both.append(_values(codes, scales).to(torch.bfloat16))
    return q_out, both[0], both[1]


def _run_read(s):
    if own:
        return _read_back(s)
    return tuple(_values(*_get(s[w], s["range_start"], s["row"], s["case"]["n_kv_heads"], w == "v")).to(torch.bfloat16) for w in ("k", "v"))


def _run_decode(s):
    case, scale = s["case"], 1.0 / math.sqrt(HEAD_DIM)
    hq, hkv, q_len = case["n_q_heads"], case["n_kv_heads"], case["q_len"]
    group = hq // hkv
    if own:
        import paper_2510_14686_amd as xa
        xa.xattn_decode_mx(s["q"], s["k_ptrs"], s["v_ptrs"], s["kv_lens"], s["batch"], q_len, hq, hkv, HEAD_DIM, scale, s["out"], s["lse"],
                           torch.cuda.current_stream())
        return s["out"], s["lse"]
    # a sequence at a time, as the caches lie; rows behind a sequence's last are in its last tile
    out, lse = torch.empty_like(s["out"]), torch.empty_like(s["lse"])
    for b, (n, total) in enumerate(s["lens"]):
        tiles = slice(s["ends"][b], s["ends"][b + 1])
        k, v = (_whole_tiles(s[w][tiles], hkv, w == "v", torch.float32)[:, :total] for w in ("k", "v"))      # [heads, keys, 128]
        q = s["q"][b].float().view(q_len, hkv, group, HEAD_DIM).permute(1, 2, 0, 3).reshape(hkv, group * q_len, HEAD_DIM)
        x = torch.matmul(q, k.transpose(1, 2).contiguous()).view(hkv, group, q_len, total).mul_(scale)
        if q_len > 1:
            x.masked_fill_(torch.ones((q_len, total), dtype=torch.bool, device="cuda").triu_(total - q_len + 1), -math.inf)
        m = x.amax(-1, keepdim=True)
        x = x.sub_(m).exp_()
        z = x.sum(-1, keepdim=True)
        o = torch.matmul(x.view(hkv, -1, total), v.contiguous()).view(hkv, group, q_len, HEAD_DIM) / z
        out[b] = o.permute(2, 0, 1, 3).reshape(q_len, hq, HEAD_DIM).to(out.dtype)
        lse[b] = (m + z.log()).squeeze(-1).permute(2, 0, 1).reshape(q_len, hq)
    return out, lse


def _whole_tiles(cache, heads, is_v, dtype):
    """The rows that a range's tiles stand for, [heads, rows, 128]."""
    tiles = cache.view(-1, heads, TILE_BYTES)
    raw, scales = tiles[..., :CODE_BYTES], tiles[..., CODE_BYTES:]
    codes = torch.stack((raw & 15, raw >> 4), -1).flatten(-2)
    if is_v:      # 4 x 16 tokens, 4 groups, 16 times 8 values, 4 tokens
        codes = codes.unflatten(-1, (4, 4, 16, 4, 8)).permute(1, 0, 2, 3, 5, 4, 6)
        scales = scales.unflatten(-1, (4, 4, 4, 4)).permute(1, 0, 4, 2, 5, 3)
    else:         # 4 x 16 tokens, 4 blocks, 16 tokens, 32 values
        codes = codes.unflatten(-1, (4, 4, 16, 32)).permute(1, 0, 2, 4, 3, 5)
        scales = scales.unflatten(-1, (4, 16, 4)).permute(1, 0, 4, 3, 2)
    return _values(codes.reshape(heads, -1, HEAD_DIM), scales.reshape(heads, -1, 4), dtype)


def _run_verify(s):
    case, scale = s["case"], s["scale"]
    batch, q_len, vocab = case["batch"], case["q_len"], case["vocab"]
    target, draft = s["target"], s["draft"]
    if own:
        import paper_2510_14686_amd as xa
        kind = {"bf16": xa.XBEAM_BF16, "fp16": xa.XBEAM_FP16, "fp32": xa.XBEAM_FP32}[case["dtype"]]
        xa.xbeam_verify(target, target.stride(1), draft, 0 if draft is None else draft.stride(1), kind, vocab, scale, scale, s["draft_tokens"] if q_len > 1 else None,
                        s["n_drafts"], None if case["greedy"] else s["uniforms"], batch, q_len, xa.XBEAM_GREEDY if case["greedy"] else 0, s["tokens"],
                        s["accepted"], s["lp"], torch.cuda.current_stream())
        return s["tokens"], s["accepted"], s["lp"]
    n = q_len - 1
    drafted = s["draft_tokens"].long()
    here = torch.arange(n, device="cuda")[None] < (n if s["n_drafts"] is None else s["n_drafts"][:, None])
    each = torch.arange(batch, device="cuda")
    # 64 bits: borders between tokens lie closer together than 32 bits tell
    lp = _log_softmax(target.double() * scale)
    if case["greedy"]:
        best = (target == target.amax(-1, keepdim=True)).to(torch.uint8).argmax(-1)      # the first of equal ones
        stands = drafted == best[:, :n]
    else:
        p = lp[:, :n].gather(2, drafted[..., None])[..., 0].exp()
        lq = None if draft is None else _log_softmax(draft.double() * scale)
        q = 1.0 if draft is None else lq.gather(2, drafted[..., None])[..., 0].exp()
        stands = s["uniforms"][:, :n].double() * q < p
    accepted = (stands & here).to(torch.int64).cumprod(1).sum(1)
    row = lp[each, accepted]
    if case["greedy"]:
        new = best[each, accepted]
    else:
        w = row.exp()
        if n:
            fell = accepted < here.sum(1)
            at = accepted.clamp(max=n - 1)
            if draft is None:
                less = w.scatter(1, drafted[each, at][:, None], 0.0)
            else:
                less = (w - lq[each, at].exp()).clamp_(min=0.0)
            w = torch.where((fell & (less.sum(1) > 0))[:, None], less, w)
        sums = w.cumsum(1)
        new = (sums <= s["uniforms"][:, -1:].double() * sums[:, -1:]).sum(1).clamp_(max=vocab - 1)
    places = torch.arange(q_len, device="cuda")[None]
    tokens = torch.cat((drafted, new[:, None]), 1)
    tokens = torch.where(places == accepted[:, None], new[:, None], torch.where(places < accepted[:, None], tokens, -1))
    token_lp = torch.where(tokens >= 0, lp.gather(2, tokens.clamp(min=0)[..., None])[..., 0], 0.0)
    return tokens.to(torch.int32), accepted.to(torch.int32), token_lp.float()


def _log_softmax(x):
    m = x.amax(-1, keepdim=True)
    return x - (m + (x - m).exp().sum(-1, keepdim=True).log())


# ------------------------------------------------------------------------------------------------ the definitions in 64 bits
def exact(case, seed):
    return {"append": _exact_append, "read": _exact_read, "decode": _exact_decode, "verify": _exact_verify}[case["op"]](case, prepare(case, seed))


def _nearest(x):
    """Every value of [..., 128] as the nearest one that 4 bits and its block's scale hold, by trying all of them."""
    levels = torch.tensor([0.0, 1.0, 2.0, 3.0, 4.0, 6.0, 8.0, 12.0], dtype=torch.float64, device="cuda") / 2
    order = torch.tensor([0, 2, 4, 6, 1, 3, 5, 7], device="cuda")      # of two as near, an even code comes first
    blocks = x.reshape(*x.shape[:-1], 4, 32)
    most = blocks.abs().amax(-1, keepdim=True)
    e = torch.ceil(torch.log2(torch.where(most > 0, most, 1.0) / 7.0))
    e = torch.where(most > 7.0 * 2.0 ** e, e + 1, torch.where(most <= 7.0 * 2.0 ** (e - 1), e - 1, e)).clamp(-125, 126)
    y = blocks / 2.0 ** e
    best, far = torch.zeros_like(y), torch.full_like(y, math.inf)
    for i in order.tolist():
        off = (y.abs() - levels[i]).abs()
        best, far = torch.where(off < far, levels[i], best), torch.minimum(off, far)
    return (torch.copysign(best, y) * 2.0 ** e).reshape(x.shape)


def _exact_append(case, s):
    hq, hkv, new = case["n_q_heads"], case["n_kv_heads"], s["new"]
    angle = torch.zeros((new, 64), dtype=torch.float64, device="cuda")
    first = 0
    for a, n in enumerate(s["sections"]):
        angle[:, first:first + n] = s["pos"][a].double()[:, None] * s["inv_freq"][first:first + n].double()
        first += n
    turn = torch.polar(torch.ones_like(angle), angle)[:, None]
    x = s["qkv"].double().view(new, hq + 2 * hkv, HEAD_DIM)
    head = x[:, :hq + hkv]
    z = torch.view_as_complex(head.reshape(new, hq + hkv, 64, 2) if case["pairs"] else torch.stack((head[..., :64], head[..., 64:]), -1)) * turn
    turned = torch.view_as_real(z).reshape(new, hq + hkv, HEAD_DIM) if case["pairs"] else torch.cat((z.real, z.imag), -1)
    return turned[:, :hq].contiguous(), _nearest(turned[:, hq:]), _nearest(x[:, hq + hkv:])


def _one_sequence(s, case, b, which):
    """K or V of sequence b in 64 bits, [keys, heads, 128], byte by byte of the definition of a tile."""
    hkv, total = case["n_kv_heads"], s["lens"][b][1]
    cache = s[which][s["ends"][b]:s["ends"][b + 1]]
    j, h, d = torch.arange(total, device="cuda")[:, None, None], torch.arange(hkv, device="cuda")[None, :, None], torch.arange(HEAD_DIM, device="cuda")
    tile = ((j // 64) * hkv + h) * TILE_BYTES
    t = j % 64
    if which == "k":
        byte = (t // 16) * 1024 + (d // 32) * 256 + (t % 16) * 16 + d % 32 // 2
        scale = CODE_BYTES + ((d // 32) * 16 + t % 16) * 4 + t // 16
    else:
        byte = (t // 4) * 256 + (d // 8) * 16 + (t % 4) * 4 + d % 8 // 2
        scale = CODE_BYTES + ((t % 16 // 4) * 4 + d // 32) * 16 + (t // 16) * 4 + t % 4
    code = cache[tile + byte].int() >> 4 * (d % 2) & 15
    size = code & 7
    value = torch.where(size < 2, 0.5 * size, (1 + 0.5 * (size % 2)) * 2.0 ** (size // 2 - 1).double())
    return torch.where(code > 7, -value, value).double() * 2.0 ** (cache[tile + scale].double() - 127)


def _exact_read(case, s):
    return tuple(torch.cat([_one_sequence(s, case, b, w)[total - n:] for b, (n, total) in enumerate(s["lens"])]) for w in ("k", "v"))


def _exact_decode(case, s):
    out, lse = torch.empty(s["out"].shape, dtype=torch.float64, device="cuda"), torch.empty(s["lse"].shape, dtype=torch.float64, device="cuda")
    group = case["n_q_heads"] // case["n_kv_heads"]
    for b, (n, total) in enumerate(s["lens"]):
        k, v = _one_sequence(s, case, b, "k"), _one_sequence(s, case, b, "v")
        hidden = torch.arange(total, device="cuda")[None] > torch.arange(total - n, total, device="cuda")[:, None]
        for g in range(case["n_kv_heads"]):
            heads = slice(g * group, (g + 1) * group)
            q = s["q"][b, :, heads].double().reshape(n * group, HEAD_DIM)
            x = (q @ k[:, g].t().contiguous()).view(n, group, total) / math.sqrt(HEAD_DIM)
            x.masked_fill_(hidden[:, None], -math.inf)
            lse[b, :, heads] = torch.logsumexp(x, -1)
            out[b, :, heads] = (torch.exp(x - lse[b, :, heads, None]).view(n * group, total) @ v[:, g].contiguous()).view(n, group, HEAD_DIM)
    return out, lse


def _exact_verify(case, s):
    """Whole numbers have no value of their own here; the log-probabilities of what a request is given do."""
    batch, q_len, scale = case["batch"], case["q_len"], s["scale"]
    lp = torch.zeros((batch, q_len), dtype=torch.float64, device="cuda")
    drafted, numbers = s["draft_tokens"].tolist(), s["uniforms"].double()
    counts = [q_len - 1] * batch if s["n_drafts"] is None else s["n_drafts"].tolist()
    for b in range(batch):
        t = 0
        while True:
            p = torch.softmax(s["target"][b, t].double() * scale, 0)
            best = None
            if case["greedy"]:
                best = int((s["target"][b, t] == s["target"][b, t].max()).nonzero()[0])
            if t == counts[b]:
                w = p
                break
            x = drafted[b][t]
            if case["greedy"]:
                fine = x == best
            else:
                q = None if s["draft"] is None else torch.softmax(s["draft"][b, t].double() * scale, 0)
                fine = bool(numbers[b, t] * (1.0 if q is None else q[x]) < p[x])
            if not fine:
                if not case["greedy"]:
                    w = p.clone()
                    if q is None:
                        w[x] = 0
                    else:
                        w = torch.relu(p - q)
                    w = w if float(w.sum()) > 0 else p
                break
            lp[b, t] = torch.log(p[x])
            t += 1
        if case["greedy"]:
            new = best
        else:
            sums = torch.cumsum(w, 0)
            new = int(torch.searchsorted(sums, (numbers[b, -1] * sums[-1])[None], right=True)[0])
        lp[b, t] = torch.log(p[new])
    return None, None, lp
