"""Log-probabilities, entropy and alternatives (xbeam_logprobs) against the definition in 64 bits.

The alternatives' indices have to be equal.  What the values may be off by, in fp32 (u = 2^-24): x = scale * logit and a difference
of two, 4 u (|x| + |max x|); a term of the sum, its exponent's rounding times its exponent, at most 2 u times 150, and 2 u for exp2; a sum of n terms of one
sign in lanes, waves and parts, (n / 512 + 30) u; the logarithm and the products, 4 u of what they give.  Entropy is a mean of
ln s - (x - m), whose terms p |x - m| sum up to the entropy and ln s; a lane's weights share an error of 2 u |max x|, against other lanes' twice
that, which moves the entropy by the weights' mean distance from it, less than 2 (1 + entropy), times that.
"""
import math

import numpy as np
import pytest
import torch

import oracle
import paper_2510_14686_amd as xa

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
KINDS = {torch.bfloat16: 0, torch.float16: 1, torch.float32: 2}


def run(logits, k, scale=1.0, tokens=True, stream=None, out=None):
    rows, vocab = logits.shape
    f = lambda *s: torch.full(s, 5.0, device="cuda")  # noqa: E731
    r = out or dict(lse=f(rows), entropy=f(rows), token_lp=f(rows) if tokens else None, top_lp=f(rows, k) if k else None,
                    top_tok=torch.full((rows, k), -7, dtype=torch.int32, device="cuda") if k else None)
    if tokens and "tokens" not in r:
        r["tokens"] = (torch.arange(rows, device="cuda") * 7919 % vocab).int()
    xa.xbeam_logprobs(logits, KINDS[logits.dtype], logits.stride(0), rows, vocab, scale, r.get("tokens"), k, r["token_lp"], r["top_lp"], r["top_tok"],
                      r["lse"], r["entropy"], stream or torch.cuda.current_stream())
    return r


def check(logits, k, r, scale=1.0):
    torch.cuda.synchronize()
    rows, vocab = logits.shape
    for first in range(0, rows, 64):
        part = slice(first, min(rows, first + 64))
        x = logits[part].double() * float(np.float32(scale))
        lse = torch.logsumexp(x, 1)
        lp = x - lse[:, None]
        m = x.amax(1)
        s = torch.exp(x - m[:, None]).sum(1).log()
        base = (vocab / 512 + 30 + 300 + 8) * U
        near = lambda got, want, tol: bool(((got.double() - want).abs() <= tol).logical_or(got.double() == want).all())  # noqa: E731
        assert near(r["lse"][part], lse, base + 4 * U * (m.abs() + s))
        entropy = torch.special.entr(lp.exp()).sum(1)
        assert near(r["entropy"][part], entropy, (base + 8 * U) * (1 + entropy + s) + 8 * U * m.abs() * (1 + entropy))
        if r["token_lp"] is not None:
            at = r["tokens"][part].long()
            want, xt = lp.gather(1, at[:, None])[:, 0], x.gather(1, at[:, None])[:, 0]
            assert near(r["token_lp"][part], want, base + 4 * U * (xt.abs() + m.abs() + s))
        if k:
            raw = logits[part].float() + 0.0
            bits = raw.view(torch.int32)
            order = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits).long() * (1 << 32) + (vocab - 1 - torch.arange(vocab, device="cuda"))
            best = vocab - 1 - (order.sort(1, descending=True).values[:, :k] & 0xFFFFFFFF)
            assert torch.equal(r["top_tok"][part].long(), best)
            want, xt = lp.gather(1, best), x.gather(1, best)
            assert near(r["top_lp"][part], want, base + 4 * U * (xt.abs() + m.abs()[:, None] + s[:, None]))


def normal(rows, vocab, dtype=torch.float32, seed=0, std=2.5, pad=0, offset=0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    wide = torch.empty((rows * (vocab + pad) + offset,), device="cuda", dtype=dtype)
    wide.normal_(0, std, generator=g)
    return wide[offset:].view(rows, vocab + pad)[:, :vocab]


@pytest.mark.parametrize("dtype", list(KINDS), ids=str)
@pytest.mark.parametrize("vocab", [1, 2, 7, 511, 512, 513, 1500, 8192, 8193, 50001, 131072])
def test_sizes(vocab, dtype):
    for rows in (1, 3, 70):
        for k in sorted({0, 1, min(5, vocab), min(64, vocab), min(65, vocab), min(512, vocab)}):
            logits = normal(rows, vocab, dtype, seed=vocab + rows)
            check(logits, k, run(logits, k))


@pytest.mark.parametrize("rows", [2, 100, 511, 513, 2000])
def test_rows(rows):
    for vocab, k in ((9000, 3), (5000, 300), (33, 33)):
        logits = normal(rows, vocab, torch.bfloat16, seed=rows)
        check(logits, k, run(logits, k))


@pytest.mark.parametrize("dtype", list(KINDS), ids=str)
def test_strides_and_places(dtype):
    for pad, offset in ((1, 0), (3, 1), (0, 5), (64, 7)):
        logits = normal(5, 10007, dtype, seed=pad, pad=pad, offset=offset)
        check(logits, 20, run(logits, 20))


@pytest.mark.parametrize("scale", [0.5, 1.4285714, 2.0 ** -20, 100.0])
def test_temperatures(scale):
    logits = normal(4, 20001, seed=1)
    check(logits, 30, run(logits, 30, scale), scale)


@pytest.mark.parametrize("k", [1, 20, 64, 65, 512])
@pytest.mark.parametrize("rows,vocab", [(2, 40000), (3, 60001), (300, 20000), (600, 6000), (530, 1999)])
def test_orders_that_fill_the_lists(rows, vocab, k):
    """Rows that ascend, descend, are all equal, hold few different values, or have their best at the end."""
    up = torch.linspace(-3, 3, vocab, device="cuda").repeat(rows, 1)
    few = normal(rows, vocab, seed=2).round()
    late = normal(rows, vocab, seed=3)
    late[:, -700:] += 40
    for logits in (up, up.flip(1), torch.zeros_like(up), few, late, few.bfloat16()):
        logits = logits.contiguous()
        check(logits, k, run(logits, k))


@pytest.mark.parametrize("dtype", list(KINDS), ids=str)
def test_forbidden_tokens(dtype):
    for mask in (-math.inf, torch.finfo(dtype).min):
        for rows, vocab in ((3, 30000), (2, 70000), (520, 700)):
            logits = normal(rows, vocab, dtype, seed=4).contiguous()
            logits[:, torch.rand(vocab, device="cuda") < 0.9] = mask
            logits[1] = mask
            logits[1, vocab - 3] = 2.0
            for k in (5, 200):
                r = run(logits, k)
                r["tokens"][:] = vocab - 3
                r = run(logits, k, out=r)
                check(logits, k, r)
                assert not torch.isnan(r["lse"]).any() and not torch.isnan(r["entropy"]).any()


@pytest.mark.parametrize("rows,vocab", [(2, 30000), (2, 70000), (9, 8000), (520, 700)])
def test_rows_of_nothing_but_forbidden_tokens(rows, vocab):
    logits = normal(rows, vocab, seed=5).contiguous()
    logits[1] = -math.inf
    r = run(logits, 6)
    torch.cuda.synchronize()
    assert r["lse"][1].item() == -math.inf and math.isnan(r["entropy"][1].item()) and math.isnan(r["token_lp"][1].item())
    assert r["top_tok"][1].tolist() == list(range(6)) and bool(r["top_lp"][1].isnan().all())
    logits[1] = torch.finfo(torch.float32).min      # all alike: ln s is lost beside such a value, the entropy is not
    r = run(logits, 6)
    torch.cuda.synchronize()
    assert r["lse"][1].item() == torch.finfo(torch.float32).min
    assert abs(r["entropy"][1].item() - math.log(vocab)) <= (vocab / 512 + 400) * U * (1 + math.log(vocab))
    assert r["top_tok"][1].tolist() == list(range(6))
    assert bool(((r["top_lp"][1] + math.log(vocab)).abs() <= (vocab / 512 + 400) * U).all())


@pytest.mark.parametrize("rows,vocab", [(2, 30000), (2, 70000), (9, 8000), (520, 700)])
def test_values_that_are_no_numbers(rows, vocab):
    logits = normal(rows, vocab, seed=6).contiguous()
    clean = run(logits, 4)
    logits[1, 17] = math.nan
    logits[1, 19] = -math.nan
    r = run(logits, 4)
    torch.cuda.synchronize()
    for n in ("lse", "entropy", "token_lp", "top_lp", "top_tok"):
        assert torch.equal(r[n][0], clean[n][0])
    assert math.isnan(r["lse"][1].item()) and math.isnan(r["entropy"][1].item()) and bool(r["top_lp"][1].isnan().all())
    assert 17 not in r["top_tok"][1].tolist() and 19 not in r["top_tok"][1].tolist() and min(r["top_tok"][1].tolist()) >= 0
    logits[1] = math.nan
    logits[1, 5], logits[1, 4] = 1.0, 2.0
    r = run(logits, 4)
    torch.cuda.synchronize()
    assert r["top_tok"][1].tolist() == [4, 5, -1, -1]
    logits[1] = 0.0
    logits[1, 8] = math.inf
    r = run(logits, 4)
    torch.cuda.synchronize()
    assert r["top_tok"][1].tolist() == [8, 0, 1, 2] and math.isnan(r["lse"][1].item()) and bool(r["top_lp"][1].isnan().all())


@pytest.mark.parametrize("k", [0, 1, 50, 64, 65, 300, 512])
@pytest.mark.parametrize("rows,vocab,dtype", [(129, 82000, torch.bfloat16), (131, 100003, torch.float32), (256, 90001, torch.float16), (257, 82000, torch.bfloat16)])
def test_long_rows_of_a_batch(rows, vocab, dtype, k):
    """Of any order, with forbidden tokens, values that are no numbers, and rows of nothing but forbidden tokens."""
    logits = normal(rows, vocab + 3, dtype, seed=k)[:, :vocab]
    logits[3] = torch.linspace(-3, 3, vocab, device="cuda").to(dtype)
    logits[4] = logits[3].flip(0)
    logits[5] = 1.0
    logits[6] = logits[6].round()
    logits[7, -700:] += 40
    logits[8, torch.rand(vocab, device="cuda") < 0.99] = -math.inf
    logits[9] = -math.inf
    logits[9, 5], logits[9, vocab - 1] = 1.0, 1.0
    logits[10] = torch.finfo(dtype).min
    logits[10, vocab - 2] = 0.0
    r = run(logits, k)
    if k:
        r["tokens"][:] = r["top_tok"][:, 0]
    r = run(logits, k, out=r)
    keep = [i for i in range(rows) if k or i not in (8, 9)]      # (a token of probability 0 has no finite log-probability)
    if not k:
        r["token_lp"][8:10] = 0
        r = {n: v if v is None else v[keep] for n, v in r.items()}
    check(logits[keep], k, r)
    logits[2] = -math.inf
    logits[1, 11] = math.nan
    again = run(logits, k)
    torch.cuda.synchronize()
    assert again["lse"][2].item() == -math.inf and math.isnan(again["lse"][1].item()) and math.isnan(again["entropy"][1].item())
    if k:
        assert again["top_tok"][2].tolist() == list(range(k)) and 11 not in again["top_tok"][1].tolist()


def test_the_most_rows():
    logits = normal(2 ** 22, 3, torch.float32, seed=11)
    r = run(logits, 2)
    torch.cuda.synchronize()
    x = logits.double()
    lse = torch.logsumexp(x, 1)
    lp = x - lse[:, None]
    tol = (400 * U) * (4 + x.abs().amax(1))
    assert bool(((r["lse"].double() - lse).abs() <= tol).all())
    assert bool(((r["token_lp"].double() - lp.gather(1, r["tokens"].long()[:, None])[:, 0]).abs() <= tol).all())
    best = x.sort(dim=1, descending=True, stable=True).indices[:, :2]
    assert torch.equal(r["top_tok"].long(), best)
    assert bool(((r["top_lp"].double() - lp.gather(1, best)).abs() <= tol[:, None]).all())


@pytest.mark.parametrize("dtype", list(KINDS), ids=str)
def test_the_longest_row(dtype):
    logits = normal(1, 2 ** 24, dtype, seed=12)
    logits[0, -1] = 14.0
    r = run(logits, 30)
    check(logits, 30, r)
    assert r["top_tok"][0, 0].item() == 2 ** 24 - 1


def test_zeros_of_both_signs_are_equal():
    logits = torch.full((1, 5000), -1.0, device="cuda")
    logits[0, 100:200:2], logits[0, 101:200:2] = -0.0, 0.0
    r = run(logits, 50)
    torch.cuda.synchronize()
    assert r["top_tok"][0].tolist() == list(range(100, 150))


@pytest.mark.parametrize("vocab", [5000, 9000, 60000])
def test_large_values(vocab):
    for big in (1e31, 3e38, -1e31):
        logits = normal(2, vocab, seed=7).contiguous()
        logits[1] = -3e38
        logits[1, 4000:4002] = big
        r = run(logits, 3)
        torch.cuda.synchronize()
        assert r["top_tok"][1].tolist() == [4000, 4001, 0]
        assert abs(r["entropy"][1].item() - math.log(2)) < 1e-5 and r["lse"][1].item() == np.float32(big)
        assert bool(((r["top_lp"][1, :2] + math.log(2)).abs() < 1e-5).all())


@pytest.mark.parametrize("k", [1, 7, 100, 512])
def test_last_part_of_a_few_values(k):
    """122883 logits are cut into 16 parts, the last of three values, fewer than a load takes."""
    logits = normal(1, 122883, torch.bfloat16, seed=16).contiguous()
    check(logits, k, run(logits, k))
    logits[0, -3:] = 30.0
    check(logits, k, run(logits, k))
    logits[0, -3:] = -math.inf
    check(logits, k, run(logits, k))


def test_short_rows_of_few_values():
    """Fewer logits than a load takes, also where most are forbidden."""
    for vocab in range(1, 9):
        for dtype in KINDS:
            logits = normal(40, vocab, dtype, seed=vocab).contiguous()
            logits[::3, 0] = -math.inf if vocab > 1 else 0.0
            check(logits, vocab, run(logits, vocab))


def test_tokens_outside():
    logits = normal(4, 1000, seed=8)
    r = run(logits, 0)
    r["tokens"][:] = torch.tensor([-1, 1000, 5, -2 ** 31], dtype=torch.int32)
    r = run(logits, 0, out=r)
    torch.cuda.synchronize()
    lp = r["token_lp"].tolist()
    assert lp[0] == 0 and math.isnan(lp[1]) and lp[3] == 0
    assert abs(lp[2] - torch.log_softmax(logits[2].double(), 0)[5].item()) < 1e-5


def test_each_output_alone():
    logits = normal(3, 20000, seed=9)
    whole = run(logits, 10)
    for asked in (("lse",), ("entropy",), ("token_lp",), ("top_lp", "top_tok")):
        r = run(logits, 10)
        keep = {n: (v if n in asked else None) for n, v in r.items() if n != "tokens"}
        if "token_lp" in asked:
            keep["tokens"] = r["tokens"]
        for n in asked:
            keep[n].zero_()
        run(logits, 10 if "top_lp" in asked else 0, tokens="token_lp" in asked, out=keep)
        torch.cuda.synchronize()
        for n in asked:
            assert torch.equal(keep[n], whole[n])


def test_graph_replays_and_streams():
    stream = torch.cuda.Stream()
    logits = normal(3, 60000, torch.bfloat16, seed=10).contiguous()
    torch.cuda.synchronize()
    r = run(logits, 40, stream=stream)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        run(logits, 40, stream=torch.cuda.current_stream(), out=r)
    for seed in (11, 12, 13):
        logits.copy_(normal(3, 60000, torch.bfloat16, seed=seed))
        for n in ("lse", "top_lp", "top_tok"):
            r[n].zero_()
        torch.cuda.synchronize()
        graph.replay()
        check(logits, 40, r)
        other = normal(2, 70000, seed=seed)
        check(other, 7, run(other, 7))


def test_caller_workspace():
    logits = normal(3, 60000, seed=14)
    need = xa.xbeam_logprobs_workspace_bytes(3, 60000, 40)
    ws = torch.full((need + 256,), 0xFF, dtype=torch.uint8, device="cuda")
    at = -(-ws.data_ptr() // 256) * 256
    try:
        xa.xattn_set_workspace(at, need)
        check(logits, 40, run(logits, 40))
        xa.xattn_set_workspace(at, need - 1)
        with pytest.raises(xa.XattnError) as e:
            run(logits, 40)
        assert e.value.status == -3
    finally:
        torch.cuda.synchronize()
        xa.xattn_set_workspace(0, 0)


def test_alternatives_are_what_beam_selection_takes():
    n_req, width, top_k, vocab = 2, 4, 8, 512
    logits = normal(n_req * width, vocab, seed=15)
    r = run(logits, top_k)
    torch.cuda.synchronize()
    cand = r["top_lp"].cpu().numpy().reshape(n_req, width, top_k)
    tok = r["top_tok"].cpu().numpy().reshape(n_req, width, top_k)
    beam = -np.sort(np.random.RandomState(0).rand(n_req, width).astype(np.float32) * 6, axis=1)
    got = xa.xbeam_select(beam, cand, tok, flags=xa.XBEAM_CHECK_INPUT)
    want = oracle.beam_select(beam, cand, tok)
    assert all(np.array_equal(a, b) for a, b in zip(got[:3], want))
