"""Timing cases of what a serving step does around decode attention: rotary positions and append, prompt attention, log
probabilities.

Every case is one call of the public binding as a serving loop makes it: ``xattn_rope_kvcache`` on a step's fused QKV
projection, ``xattn_prefill`` on the packed new tokens of a batch, ``xbeam_logprobs`` on a step's logits.  Beside the calls
stand their plain forms, elementary operations in 32 bits, and their definitions in 64 bits.
"""
import math
import random

import torch

own = False

HEAD_DIM = 128
ROPE_BASE = 1e6
DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


# ------------------------------------------------------------------------------------------------ the cases
def _prefill(name, hq, hkv, groups):
    """groups: text "count x q_lo..q_hi + prefix_lo..prefix_hi; ...": sequences, their new tokens, what the cache holds already."""
    return dict(name=name, op="prefill", n_q_heads=hq, n_kv_heads=hkv, groups=groups)


def _rope(name, hq, hkv, groups, axes, pairs=False, far=0):
    return dict(name=name, op="rope", n_q_heads=hq, n_kv_heads=hkv, groups=groups, axes=axes, pairs=pairs, far=far)


def _logprobs(name, rows, vocab, top_k, dtype, pad=0, temperature=1.0, masked=0.0):
    return dict(name=name, op="logprobs", rows=rows, vocab=vocab, top_k=top_k, dtype=dtype, pad=pad, temperature=temperature, masked=masked)


def listed():
    return [
        # four short requests of the smallest workload's head counts, some behind a cached prefix: latency
        _prefill("prefill_tiny", 8, 2, "4x3..20+0..236"),
        # a batch of chat prompts of an 8B-shaped model, nothing cached
        _prefill("prefill_chats", 32, 8, "16x512..4096+0..0"),
        # one long document
        _prefill("prefill_document", 32, 8, "1x16001..16001+0..0"),
        # a chunk of a long document behind what earlier chunks have left in the cache, groups of eight
        _prefill("prefill_chunk", 64, 8, "1x2048..2048+28672..28672"),
        # a mixed serving step: one prompt chunk, requests that verify a draft, and decoding requests
        _prefill("prefill_mixed_step", 40, 8, "1x1000..1000+500..500;8x5..5+1024..8192;48x1..1+512..4096"),
        # a decode step of four short requests: latency
        _rope("rope_tiny_step", 8, 2, "4x1..1+16..255", axes=1),
        # a decode step of many requests
        _rope("rope_decode_step", 40, 8, "256x1..1+16..4095", axes=1),
        # a video prompt: time, height and width, far into a long session
        _rope("rope_video_prompt", 32, 8, "2x4096..8191+0..64", axes=3, far=1000000),
        # one request's next token, full vocabulary, 20 alternatives: latency
        _logprobs("logprobs_one_row", 1, 131072, 20, "bf16"),
        # candidates of the widest beam-search workload, 8 requests x 128 sequences
        _logprobs("logprobs_beams", 1024, 8192, 512, "fp32"),
        # a sampling step of a batch: odd vocabulary in padded rows, a temperature, part of the tokens forbidden
        _logprobs("logprobs_batch", 192, 100003, 50, "fp32", pad=5, temperature=0.7, masked=0.3),
        # scoring a prompt: every position's token and five alternatives
        _logprobs("logprobs_prompt", 4096, 131072, 5, "bf16"),
    ]


_HEADS = [(8, 2), (4, 4), (5, 1), (16, 2), (12, 2), (32, 8), (64, 8), (40, 8), (16, 8), (8, 1)]
_MOST_FLOPS, _MOST_ROPE_BYTES, _MOST_LOGITS = 2.0e12, 1.3e9, 5.0e8


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _draw_groups(rng, most_tokens):
    parts = []
    for _ in range(rng.choice([1, 1, 2])):
        if rng.random() < 0.25:
            q_hi, count = rng.randint(1, 4), _log_uniform(rng, 4, 128)
        else:
            q_hi = _log_uniform(rng, 5, most_tokens)
            count = _log_uniform(rng, 1, max(1, min(48, most_tokens // q_hi)))
        prefix = 0 if rng.random() < 0.4 else _log_uniform(rng, 16, 16384)
        parts.append("%dx%d..%d+%d..%d" % (count, max(1, q_hi // rng.choice([1, 2, 8])), q_hi, prefix // rng.choice([1, 4]), prefix))
    return ";".join(parts)


def draw(rng):
    """One more case: head counts of the workloads and tests, prompts of 1 to 16384 new tokens behind up to 16384 cached ones;
    1 to 4096 rows of 500 to 200000 logits with 0 to 512 alternatives."""
    while True:
        op = rng.choice(["prefill", "prefill", "rope", "logprobs"])
        hq, hkv = rng.choice(_HEADS)
        if op == "prefill":
            case = dict(_prefill("", hq, hkv, _draw_groups(rng, 16384)))
            fits = work(case)["flops"] <= _MOST_FLOPS and sum(n for _, n in _lengths(case)) <= 400000
        elif op == "rope":
            case = _rope("", hq, hkv, _draw_groups(rng, 16384), axes=rng.randint(1, 4), pairs=rng.random() < 0.4, far=rng.choice([0, 0, 70000, 4000000]))
            fits = work(case)["bytes"] <= _MOST_ROPE_BYTES and sum(n for _, n in _lengths(case)) <= 400000
        else:
            vocab = _log_uniform(rng, 500, 200000)
            case = _logprobs("", _log_uniform(rng, 1, 4096), vocab, rng.choice([0, 1, rng.randint(2, 20), _log_uniform(rng, 21, min(512, vocab // 2))]),
                             rng.choice(["bf16", "bf16", "fp16", "fp32"]), pad=rng.choice([0, 0, rng.randint(1, 64)]),
                             temperature=rng.choice([1.0, round(rng.uniform(0.3, 2.0), 2)]), masked=rng.choice([0.0, 0.0, 0.25]))
            fits = case["rows"] * vocab * (2 if case["dtype"] != "fp32" else 4) <= 2 * _MOST_LOGITS
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
    if case["op"] == "logprobs":
        n = case["rows"] * case["vocab"]
        size = torch.empty(0, dtype=DTYPES[case["dtype"]]).element_size()
        return {"bytes": n * size + case["rows"] * (16 + 8 * case["top_k"]), "flops": 6 * n}
    hq, hkv, lens = case["n_q_heads"], case["n_kv_heads"], _lengths(case)
    new = sum(n for n, _ in lens)
    if case["op"] == "rope":
        return {"bytes": new * (4 * (hq + 2 * hkv) * HEAD_DIM + 4 * case["axes"]), "flops": 3 * new * (hq + hkv) * HEAD_DIM}
    seen = sum(n * (total - n) + n * (n + 1) // 2 for n, total in lens)
    return {"bytes": 4 * new * hq * HEAD_DIM + 4 * new * hq + 4 * sum(total for _, total in lens) * hkv * HEAD_DIM, "flops": 4 * HEAD_DIM * hq * seen}


# ------------------------------------------------------------------------------------------------ inputs
def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _sequences(case, seed):
    """What both cache operators take: lengths, where the packed rows of a sequence begin, ranges, addresses."""
    lens = _lengths(case, seed)
    starts, ends = [0], [0]
    for n, total in lens:
        starts.append(starts[-1] + n)
        ends.append(ends[-1] + total)
    g = _generator(seed)
    shape = (ends[-1], case["n_kv_heads"], HEAD_DIM)
    s = dict(case=case, lens=lens, starts=starts, ends=ends, batch=len(lens), new=starts[-1], q_starts=_ints(starts), kv_lens=_ints([n for _, n in lens]),
             k=torch.randn(shape, generator=g, device="cuda", dtype=torch.bfloat16), v=torch.randn(shape, generator=g, device="cuda", dtype=torch.bfloat16))
    row = case["n_kv_heads"] * HEAD_DIM * 2
    for which in ("k", "v"):
        s[which + "_ptrs"] = torch.tensor([s[which].data_ptr() + row * e for e in ends[:-1]], dtype=torch.int64, device="cuda")
    return s, g


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


def prepare(case, seed):
    if case["op"] == "logprobs":
        g = _generator(seed)
        rows, vocab = case["rows"], case["vocab"]
        wide = torch.empty((rows, vocab + case["pad"]), device="cuda", dtype=DTYPES[case["dtype"]])
        wide.normal_(0.0, 2.5, generator=g)
        logits = wide[:, :vocab]
        if case["masked"]:
            logits[:, torch.rand(vocab, generator=g, device="cuda") < case["masked"]] = -math.inf
        tokens = torch.randint(0, vocab, (rows,), generator=g, device="cuda", dtype=torch.int32)
        f = lambda *shape: torch.empty(shape, device="cuda", dtype=torch.float32)  # noqa: E731
        return dict(case=case, logits=logits, tokens=tokens, token_lp=f(rows), lse=f(rows), entropy=f(rows), top_lp=f(rows, case["top_k"]),
                    top_tok=torch.empty((rows, case["top_k"]), device="cuda", dtype=torch.int32))
    s, g = _sequences(case, seed)
    hq, hkv, new = case["n_q_heads"], case["n_kv_heads"], s["new"]
    s["out"] = torch.empty((new, hq, HEAD_DIM), device="cuda", dtype=torch.bfloat16)
    if case["op"] == "rope":
        axes = case["axes"]
        s["qkv"] = torch.randn((new, (hq + 2 * hkv) * HEAD_DIM), generator=g, device="cuda", dtype=torch.bfloat16)
        s["pos"] = _positions(case, s["lens"], axes).to("cuda").contiguous()
        s["inv_freq"] = (ROPE_BASE ** (-torch.arange(64, dtype=torch.float64) / 64)).to(torch.float32).cuda()
        s["sections"] = _sections(axes)
        s["axis_of"] = torch.repeat_interleave(torch.arange(axes), torch.tensor(s["sections"])).cuda()
        # the row of the caches that each new token gets
        s["rows"] = torch.cat([torch.arange(e + total - n, e + total) for e, (n, total) in zip(s["ends"], s["lens"])]).cuda()
        return s
    s["q"] = torch.randn((new, hq, HEAD_DIM), generator=g, device="cuda", dtype=torch.bfloat16)
    s["lse"] = torch.empty((new, hq), device="cuda", dtype=torch.float32)
    return s


# ------------------------------------------------------------------------------------------------ the calls and their plain forms
def run(state):
    return {"prefill": _run_prefill, "rope": _run_rope, "logprobs": _run_logprobs}[state["case"]["op"]](state)


def _run_prefill(s):
    case, scale = s["case"], 1.0 / math.sqrt(HEAD_DIM)
    hq, hkv = case["n_q_heads"], case["n_kv_heads"]
    if own:
        import paper_2510_14686_amd as xa
        xa.xattn_prefill(s["q"], s["k_ptrs"], s["v_ptrs"], s["q_starts"], s["kv_lens"], s["batch"], s["new"], hq, hkv, HEAD_DIM, scale, s["out"], s["lse"],
                         torch.cuda.current_stream())
        return s["out"], s["lse"]
    # a sequence at a time, as the caches lie
    out, lse = torch.empty_like(s["out"]), torch.empty_like(s["lse"])
    for b, (n, total) in enumerate(s["lens"]):
        rows, keys = slice(s["starts"][b], s["starts"][b + 1]), slice(s["ends"][b], s["ends"][b + 1])
        q = s["q"][rows].float().view(n, hkv, hq // hkv, HEAD_DIM).permute(1, 2, 0, 3).reshape(hkv, -1, HEAD_DIM)
        k, v = (s[w][keys].float().permute(1, 0, 2).contiguous() for w in ("k", "v"))
        x = torch.matmul(q, k.transpose(1, 2).contiguous()).view(hkv, hq // hkv, n, total).mul_(scale)
        if n > 1:
            x.masked_fill_(torch.ones((n, total), dtype=torch.bool, device="cuda").triu_(total - n + 1), -math.inf)
        m = x.amax(-1, keepdim=True)
        x = x.sub_(m).exp_()
        z = x.sum(-1, keepdim=True)
        o = torch.matmul(x.view(hkv, -1, total), v).view(hkv, hq // hkv, n, HEAD_DIM) / z
        out[rows] = o.permute(2, 0, 1, 3).reshape(n, hq, HEAD_DIM).to(out.dtype)
        lse[rows] = (m + z.log()).squeeze(-1).permute(2, 0, 1).reshape(n, hq)
    return out, lse


def _split_pairs(x, pairs):
    return (x[..., 0::2], x[..., 1::2]) if pairs else (x[..., :64], x[..., 64:])


def _join_pairs(x, y, pairs):
    return torch.stack((x, y), -1).flatten(-2) if pairs else torch.cat((x, y), -1)


def _run_rope(s):
    case = s["case"]
    hq, hkv, new = case["n_q_heads"], case["n_kv_heads"], s["new"]
    q, k, v = s["qkv"].split([hq * HEAD_DIM, hkv * HEAD_DIM, hkv * HEAD_DIM], 1)
    if own:
        import paper_2510_14686_amd as xa
        xa.xattn_rope_kvcache(q, k, v, q.stride(0), k.stride(0), v.stride(0), s["pos"], s["inv_freq"], s["sections"],
                              xa.XATTN_ROPE_PAIRS if case["pairs"] else 0, s["k_ptrs"], s["v_ptrs"], s["q_starts"], s["kv_lens"], s["batch"], new,
                              hq, hkv, HEAD_DIM, s["out"], torch.cuda.current_stream())
        return s["out"], s["k"], s["v"]
    angle = s["pos"].double()[s["axis_of"]].t() * s["inv_freq"].double()          # [new, 64]; 32 bits lose far positions
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
    x, y = _split_pairs(torch.cat((q, k), 1).float().view(new, hq + hkv, HEAD_DIM), case["pairs"])
    turned = _join_pairs(x * cos - y * sin, y * cos + x * sin, case["pairs"]).to(torch.bfloat16)
    s["k"][s["rows"]] = turned[:, hq:]
    s["v"][s["rows"]] = v.view(new, hkv, HEAD_DIM)
    return turned[:, :hq].contiguous(), s["k"], s["v"]


def _run_logprobs(s):
    case, logits, scale = s["case"], s["logits"], 1.0 / s["case"]["temperature"]
    rows, vocab, k = case["rows"], case["vocab"], case["top_k"]
    if own:
        import paper_2510_14686_amd as xa
        kind = {"bf16": xa.XBEAM_BF16, "fp16": xa.XBEAM_FP16, "fp32": xa.XBEAM_FP32}[case["dtype"]]
        xa.xbeam_logprobs(logits, kind, logits.stride(0), rows, vocab, scale, s["tokens"], k, s["token_lp"], s["top_lp"] if k else None,
                          s["top_tok"] if k else None, s["lse"], s["entropy"], torch.cuda.current_stream())
        return {n: s[n] for n in ("token_lp", "lse", "entropy") + (("top_lp", "top_tok") if k else ())}
    raw = logits.float()
    x = raw * scale
    m = x.amax(1, keepdim=True)
    e = (x - m).exp()
    z = e.sum(1, keepdim=True)
    lse = m + z.log()
    lp = x - lse
    out = dict(token_lp=lp.gather(1, s["tokens"].long()[:, None])[:, 0], lse=lse[:, 0], entropy=-(e * lp).nan_to_num_(nan=0.0).sum(1) / z[:, 0])
    if k:
        # value, then the lowest index, as one whole number
        bits = (raw + 0.0).view(torch.int32)
        order = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits).long() * (1 << 32) + (vocab - 1 - torch.arange(vocab, device="cuda"))
        best = vocab - 1 - (order.topk(k, 1, sorted=True).values & 0xFFFFFFFF)
        out.update(top_lp=lp.gather(1, best), top_tok=best.to(torch.int32))
    return out


# ------------------------------------------------------------------------------------------------ the definitions in 64 bits
def exact(case, seed):
    return {"prefill": _exact_prefill, "rope": _exact_rope, "logprobs": _exact_logprobs}[case["op"]](case, prepare(case, seed))


def _exact_prefill(case, s):
    out, lse = torch.empty(s["out"].shape, dtype=torch.float64, device="cuda"), torch.empty(s["lse"].shape, dtype=torch.float64, device="cuda")
    group = case["n_q_heads"] // case["n_kv_heads"]
    for b, (n, total) in enumerate(s["lens"]):
        r0, k0 = s["starts"][b], s["ends"][b]
        last = torch.arange(total - n, total, device="cuda")[:, None]
        hidden = torch.arange(total, device="cuda")[None] > last
        for h in range(case["n_q_heads"]):
            k, v = (s[w][k0:k0 + total, h // group].double() for w in ("k", "v"))
            x = (s["q"][r0:r0 + n, h].double() @ k.t().contiguous()) / math.sqrt(HEAD_DIM)
            x[hidden] = -math.inf
            lse[r0:r0 + n, h] = torch.logsumexp(x, 1)
            out[r0:r0 + n, h] = torch.exp(x - lse[r0:r0 + n, h, None]) @ v
    return out, lse


def _exact_rope(case, s):
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
    k, v = s["k"].double(), s["v"].double()
    k[s["rows"]], v[s["rows"]] = turned[:, hq:], x[:, hq + hkv:]
    return turned[:, :hq].contiguous(), k, v


def _exact_logprobs(case, s):
    rows, vocab, k = case["rows"], case["vocab"], case["top_k"]
    f = lambda *shape: torch.empty(shape, dtype=torch.float64, device="cuda")  # noqa: E731
    out = dict(token_lp=f(rows), lse=f(rows), entropy=f(rows))
    if k:
        out.update(top_lp=f(rows, k), top_tok=None)
    for r in range(0, rows, 256):
        x = s["logits"][r:r + 256].double() / case["temperature"]
        lp = torch.log_softmax(x, 1)
        out["lse"][r:r + 256] = torch.logsumexp(x, 1)
        out["token_lp"][r:r + 256] = lp.gather(1, s["tokens"][r:r + 256].long()[:, None])[:, 0]
        out["entropy"][r:r + 256] = torch.special.entr(lp.exp()).sum(1)
        if k:
            out["top_lp"][r:r + 256] = lp.sort(1, descending=True).values[:, :k]
    return out
