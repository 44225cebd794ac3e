"""xbeam_logprobs on rows that lie far from zero: log-probabilities and entropy depend on the differences of logits alone.

The logits are multiples of a power of two that stay exact behind the offset, so the rows hold the very differences that they are checked
for.  What the values may be off by, in fp32 (u = 2^-24), with m the row's largest x = scale * logit: a weight by the rounding of its exponent and of the
factor in it, at most 2 u times 150, and 2 u for exp2; a sum of n terms of one sign in lanes, waves and parts, (n / 512 + 30) u; 8 u for the
products on the way: `base` in all.  The logarithm and the difference x - m add 4 u of what they give.  Nothing of it grows with |m|, but for lse, which
is as large itself.
"""
import math

import numpy as np
import pytest
import torch

import paper_2510_14686_amd as xa

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
KINDS = {torch.bfloat16: 0, torch.float16: 1, torch.float32: 2}


def run(logits, k, scale, tokens):
    rows, vocab = logits.shape
    f = lambda *s: torch.full(s, 5.0, device="cuda")  # noqa: E731
    r = dict(lse=f(rows), entropy=f(rows), token_lp=f(rows), top_lp=f(rows, k), top_tok=torch.full((rows, k), -7, dtype=torch.int32, device="cuda"))
    xa.xbeam_logprobs(logits, KINDS[logits.dtype], logits.stride(0), rows, vocab, scale, tokens, k, r["token_lp"], r["top_lp"], r["top_tok"], r["lse"],
                      r["entropy"], torch.cuda.current_stream())
    torch.cuda.synchronize()
    return r


def check(logits, k, scale=1.0):
    rows, vocab = logits.shape
    tokens = (torch.arange(rows, device="cuda") * 7919 % vocab).int()
    r = run(logits, k, scale, tokens)
    x = logits.double() * float(np.float32(scale))
    m = x.amax(1, keepdim=True)
    d = x - m
    s = d.exp().sum(1).log()
    lp = d - s[:, None]
    base = (vocab / 512 + 30 + 300 + 8) * U

    def near(name, want, tol):
        over = ((r[name].double() - want).abs() - tol).max().item()
        assert over <= 0, "%s is %.3g further off than it may be" % (name, over)

    near("lse", (m[:, 0] + s), base + 4 * U * (m[:, 0].abs() + s))
    entropy = torch.special.entr(lp.exp()).sum(1)
    near("entropy", entropy, (base + 8 * U) * (1 + entropy + s))
    at = tokens.long()[:, None]
    near("token_lp", lp.gather(1, at)[:, 0], base + 4 * U * (d.gather(1, at)[:, 0].abs() + s))
    best = lp.sort(dim=1, descending=True, stable=True).indices[:, :k]
    assert torch.equal(r["top_tok"].long(), best)
    near("top_lp", lp.gather(1, best), base + 4 * U * (d.gather(1, best).abs() + s[:, None]))
    assert bool((r["top_lp"] <= 0).all()) and bool((r["token_lp"] <= 0).all())


def multiples(rows, vocab, offset, quantum, std, dtype=torch.float32, seed=0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    x = torch.empty((rows, vocab), device="cuda").normal_(0.0, std / quantum, generator=g).round_().mul_(quantum)
    logits = (x + offset).to(dtype)
    assert torch.equal(logits.double(), x.double() + offset)
    return logits


# one round of two and of eight waves, lists of both lengths, rows in parts, sixteen waves
SHAPES = [(3, 500, 5), (600, 1999, 20), (9, 8000, 300), (300, 20000, 20), (270, 9000, 100), (5, 60000, 20), (150, 100003, 100)]


@pytest.mark.parametrize("rows,vocab,k", SHAPES)
@pytest.mark.parametrize("offset,quantum", [(0.0, 2.0 ** -18), (20.0, 2.0 ** -18), (1024.0, 2.0 ** -12), (-8192.0, 2.0 ** -10), (30000.0, 2.0 ** -8),
                                            (2.0 ** 17, 2.0 ** -6), (-2.0 ** 22, 1.0), (2.0 ** 26, 8.0), (2.0 ** 40, 2.0 ** 17)])
def test_offsets(rows, vocab, k, offset, quantum):
    check(multiples(rows, vocab, offset, quantum, max(2.5, quantum), seed=vocab), k)


@pytest.mark.parametrize("rows,vocab,k", SHAPES)
@pytest.mark.parametrize("scale", [0.7, 100.0, 2.0 ** 20, 2.0 ** -20])
def test_scales(rows, vocab, k, scale):
    """A scale enlarges what lies far from zero as an offset does."""
    std = 2.5 / scale
    top = 2.0 ** math.ceil(math.log2(512 * std))
    check(multiples(rows, vocab, top, top * 2.0 ** -22, std, seed=vocab + 1), k, scale)


@pytest.mark.parametrize("dtype,offset,quantum", [(torch.float16, 1536.0, 1.0), (torch.float16, 32768.0, 32.0), (torch.bfloat16, 192.0, 1.0), (torch.bfloat16, -12288.0, 64.0)],
                         ids=str)
@pytest.mark.parametrize("rows,vocab,k", [SHAPES[0], SHAPES[2], SHAPES[5], SHAPES[6]])
def test_types(dtype, offset, quantum, rows, vocab, k):
    """Values nine quanta and less from the offset, which the type's 8 (or 11) bits hold, at a scale that spreads them over some nats."""
    x = multiples(rows, vocab, 0.0, quantum, 2 * quantum, seed=vocab + 2).clamp_(-9 * quantum, 9 * quantum) + offset
    logits = x.to(dtype)
    assert torch.equal(logits.float(), x)
    check(logits, k, 1.0 / quantum)


@pytest.mark.parametrize("rows,vocab,k", SHAPES)
def test_one_token_that_is_not_forbidden(rows, vocab, k):
    """It has all of the probability: its log-probability is 0, wherever the row lies."""
    for at in (12345.678, -7.77, 1234567.8, 3e37):
        logits = torch.full((rows, vocab), -math.inf, device="cuda")
        logits[:, vocab - 3] = at
        tokens = torch.full((rows,), vocab - 3, dtype=torch.int32, device="cuda")
        r = run(logits, k, 1.0, tokens)
        assert bool((r["token_lp"] == 0).all()) and bool((r["top_lp"][:, 0] == 0).all()) and bool((r["top_lp"][:, 1:] == -math.inf).all())
        assert bool((r["entropy"].abs() <= 8 * U).all()) and bool((r["lse"] == np.float32(at)).all())
