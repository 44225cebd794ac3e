"""Verification of drafted tokens (xbeam_verify) against the definition in 64 bits.

Tokens and counts are equal: a draft's fate turns on probabilities that are off by 2^-20 of themselves, a new token's on sums off by 2^-45, and
no random number of these inputs lies that near to a border.  token_lp: 2^-20 for the sum of exponentials, 2^-23 of itself for its roundings.
"""
import math

import numpy as np
import pytest
import torch

import paper_2510_14686_amd as xa

pytestmark = pytest.mark.gpu
TYPES = {"bf16": (torch.bfloat16, xa.XBEAM_BF16), "fp16": (torch.float16, xa.XBEAM_FP16), "fp32": (torch.float32, xa.XBEAM_FP32)}


def reference(target, draft, scale, draft_scale, draft_tokens, counts, uniforms, greedy):
    """(tokens, accepted, token_lp) of lists; logits [batch, rows, vocab], in double."""
    batch, q_len, vocab = target.shape
    tokens, accepted, lps = [], [], []

    def probabilities(x, s):      # step by step: torch.softmax of doubles on the GPU is off by 2e-6 of them
        x = x.double() * s
        if not bool((x < math.inf).all()) or not bool((x > -math.inf).any()):
            return None
        e = torch.exp(x - x.max())
        return e / e.sum()

    for b in range(batch):
        n = min(max(counts[b], 0), q_len - 1)
        given, lp, t, new = [], [], 0, None
        while True:
            p = probabilities(target[b, t], scale)
            best = int(torch.nonzero(target[b, t] == target[b, t].max())[0]) if greedy and p is not None else None
            w = p
            if t == n:
                break
            x = int(draft_tokens[b][t])
            fine = 0 <= x < vocab and p is not None
            q = None
            if greedy:
                fine = fine and x == best
            elif draft is not None:
                q = probabilities(draft[b, t], draft_scale)
                fine = fine and q is not None and float(uniforms[b, t]) * float(q[x]) < float(p[x])
            else:
                fine = fine and float(uniforms[b, t]) < float(p[x])
            if not fine:
                if p is not None and not greedy:
                    if draft is not None:
                        w = torch.relu(p - q) if q is not None else p
                    elif 0 <= x < vocab:
                        w = p.clone()
                        w[x] = 0
                    w = w if float(w.sum()) > 0 else p
                break
            given.append(x)
            lp.append(float(torch.log(p[x])))
            t += 1
        if p is None:
            new, new_lp = -1, math.nan
        else:
            if greedy:
                new = best
            else:
                sums = torch.cumsum(w, 0)
                over = torch.nonzero((sums > float(uniforms[b, -1]) * float(sums[-1])) & (w > 0))
                new = int(over[0]) if len(over) else int(torch.nonzero(w > 0)[-1])
            new_lp = float(torch.log(p[new]))
        tokens.append(given + [new] + [-1] * (q_len - t - 1))
        accepted.append(t)
        lps.append(lp + [new_lp] + [0.0] * (q_len - t - 1))
    return tokens, accepted, lps


class Case:
    def __init__(self, batch, q_len, vocab, dtype="fp32", drafts="logits", seed=0, pad=0, scale=1.0, draft_scale=None, greedy=False, near=0.7, counts=None, sd=2.5):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        t, self.kind = TYPES[dtype]
        n = q_len - 1
        self.batch, self.q_len, self.vocab, self.greedy, self.scale = batch, q_len, vocab, greedy, scale
        self.draft_scale = scale if draft_scale is None else draft_scale
        wide = torch.empty((batch, q_len, vocab + pad), device="cuda", dtype=t).normal_(0.0, sd, generator=g)
        self.target = wide[..., :vocab]
        likely = torch.randint(0, vocab, (batch, q_len, 1), generator=g, device="cuda")
        self.target.scatter_add_(2, likely, torch.full(likely.shape, 9.0, device="cuda", dtype=t))
        self.draft = None
        if drafts == "logits" and n:
            d = torch.empty((batch, n, vocab + pad), device="cuda", dtype=t).normal_(0.0, near, generator=g)
            d += wide[:, :n]
            self.draft = d[..., :vocab]
            p = torch.softmax(self.draft.float() * self.draft_scale, -1).view(batch * n, vocab)
            self.draft_tokens = torch.multinomial(p, 1, generator=g).view(batch, n).int()
        else:
            other = torch.randint(0, vocab, (batch, n), generator=g, device="cuda")
            right = torch.rand((batch, n), generator=g, device="cuda") < 0.8
            self.draft_tokens = torch.where(right, self.target[:, :n].argmax(-1) if n else other, other).int()
        self.uniforms = torch.rand((batch, q_len), generator=g, device="cuda")
        self.counts = counts
        self.n_drafts = None if counts is None else torch.tensor(counts, dtype=torch.int32, device="cuda")
        self.tokens = torch.full((batch, q_len), -7, dtype=torch.int32, device="cuda")
        self.accepted = torch.full((batch,), -7, dtype=torch.int32, device="cuda")
        self.lp = torch.full((batch, q_len), 7.0, device="cuda")

    def call(self, stream=None, lp=True):
        xa.xbeam_verify(self.target, self.target.stride(1), self.draft, self.draft.stride(1) if self.draft is not None else 0, self.kind, self.vocab, self.scale,
                        self.draft_scale, self.draft_tokens if self.q_len > 1 else None, self.n_drafts, None if self.greedy else self.uniforms, self.batch,
                        self.q_len, xa.XBEAM_GREEDY if self.greedy else 0, self.tokens, self.accepted, self.lp if lp else None, stream or torch.cuda.current_stream())

    def check(self):
        torch.cuda.synchronize()
        f32 = lambda v: float(torch.tensor(v, dtype=torch.float32))  # noqa: E731
        tokens, accepted, lps = reference(self.target, self.draft, f32(self.scale), f32(self.draft_scale), self.draft_tokens.tolist(),
                                          self.counts or [self.q_len - 1] * self.batch, self.uniforms, self.greedy)
        assert self.accepted.tolist() == accepted
        assert self.tokens.tolist() == tokens
        for got, want in zip(self.lp.tolist(), lps):
            for x, y in zip(got, want):
                assert (math.isnan(x) and math.isnan(y)) or abs(x - y) <= 2.0 ** -20 + 2.0 ** -23 * abs(y), (x, y)
        return accepted


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("drafts", ["logits", "certain"])
@pytest.mark.parametrize("vocab,pad", [(7, 0), (500, 3), (5000, 0), (100003, 5)])
def test_types_and_sizes(vocab, pad, drafts, dtype):
    c = Case(12, 5, vocab, dtype, drafts, seed=vocab, pad=pad)
    c.call()
    c.check()


@pytest.mark.parametrize("q_len", [1, 2, 3, 9, 16])
@pytest.mark.parametrize("greedy", [False, True])
def test_rows(q_len, greedy):
    c = Case(7, q_len, 3001, "bf16", seed=q_len, greedy=greedy)
    c.call()
    c.check()


@pytest.mark.parametrize("vocab", [1, 2, 8, 2047, 2048, 2049, 131072, 200001])
def test_vocabularies(vocab):
    for drafts in ("logits", "certain"):
        c = Case(3, 3, vocab, "fp16", drafts, seed=vocab)
        c.call()
        c.check()


@pytest.mark.parametrize("batch,vocab", [(1, 131072), (300, 1000), (1500, 600)])
def test_batches(batch, vocab):
    c = Case(batch, 4, vocab, "bf16", seed=batch)
    c.call()
    accepted = c.check()
    if batch > 100:
        assert set(accepted) == {0, 1, 2, 3}


@pytest.mark.parametrize("drafts", ["logits", "certain"])
def test_the_largest_vocabulary(drafts):
    c = Case(2, 2, 1 << 24, "bf16", drafts, seed=8, sd=1.5)
    c.call()
    c.check()


def test_most_rows():
    """A batch of 4096 with 16 rows each: their number passes 65535."""
    c = Case(4096, 16, 40, "bf16", seed=1, near=0.1)
    c.call()
    c.check()


@pytest.mark.parametrize("scale,draft_scale", [(0.5, 0.5), (1 / 0.7, 1 / 0.7), (1.3, 0.6), (8.0, 8.0), (0.01, 1.0)])
def test_temperatures(scale, draft_scale):
    c = Case(40, 4, 2000, "fp32", seed=3, scale=scale, draft_scale=draft_scale)
    c.call()
    c.check()


def test_numbers_of_drafts():
    for greedy in (False, True):
        for drafts in ("logits", "certain"):
            c = Case(9, 5, 700, "fp32", drafts, seed=4, counts=[0, 1, 2, 3, 4, -3, 99, 4, 0], greedy=greedy)
            c.target[1, 2:] = math.nan      # rows behind the last draft's are not looked at
            c.call()
            c.check()


def test_forbidden_tokens():
    for drafts in ("logits", "certain"):
        c = Case(30, 4, 5000, "fp32", drafts, seed=5)
        c.target[:, :, ::3] = -math.inf
        if c.draft is not None:
            c.draft[:10, :, ::3] = -math.inf
            c.draft[10:20, :, 1::3] = -math.inf
        c.target[20:24] = -math.inf
        c.target[20:24, :, 4] = 1.0         # one token is left
        c.draft_tokens[21:23] = 4
        c.call()
        c.check()


def test_tokens_that_do_not_exist():
    for drafts in ("logits", "certain"):
        for greedy in (False, True):
            c = Case(6, 3, 900, "bf16", drafts, seed=6, greedy=greedy)
            c.draft_tokens[0, 0] = -1
            c.draft_tokens[1, 1] = 900
            c.draft_tokens[2, 0] = 2 ** 31 - 1
            c.draft_tokens[3, 0] = -2 ** 31
            c.call()
            c.check()


@pytest.mark.parametrize("greedy", [False, True])
def test_rows_without_probabilities(greedy):
    c = Case(10, 3, 3000, "fp32", seed=7, greedy=greedy, near=0.0)
    c.target[0, 0, 5] = math.nan
    c.target[1, 1, 2999] = math.inf
    c.target[2, 2] = -math.inf
    c.target[3, 0] = math.nan
    c.target[4, 0, ::2] = -math.inf
    if c.draft is not None:
        c.draft[5, 0, 17] = math.nan
        c.draft[6, 1] = -math.inf
        c.draft[7, 0, 0] = math.inf
    c.call()
    c.check()


def test_greedy_takes_the_first_of_equal_ones():
    c = Case(8, 3, 5000, "bf16", seed=8, greedy=True)
    c.target[:, :, 4000] = 30.0
    c.target[:4, :, 1234] = 30.0
    c.target[2, 0, 0] = 30.0
    c.draft_tokens[:, 0] = torch.tensor([1234, 4000, 0, 1234, 4000, 1234, 4000, 4000])
    c.call()
    c.check()


def test_numbers_at_their_ends():
    for drafts in ("logits", "certain"):
        for u in (0.0, 1.0 - 2.0 ** -24):
            c = Case(20, 3, 4000, "fp32", drafts, seed=9)
            c.uniforms.fill_(u)
            c.target[:, :, :7] = -math.inf
            c.target[:, :, -9:] = -math.inf
            c.call()
            c.check()


def test_a_draft_of_the_targets_own_probabilities_stands():
    c = Case(50, 6, 1000, "fp32", seed=10, near=0.0)
    c.uniforms.fill_(1.0 - 2.0 ** -10)
    c.call()
    assert c.check() == [5] * 50


def check_what_is_left(c):
    """The first draft falls; the new token, by the definition with 64 bits of significand."""
    assert c.accepted.tolist() == [0] * c.batch
    target, draft, u = (x.cpu().numpy().astype(np.longdouble) for x in (c.target[:, 0], c.draft[:, 0], c.uniforms[:, -1]))
    for b in range(c.batch):
        p, q = (np.exp(x[b] - x[b].max()) for x in (target, draft))
        w = np.maximum(p / p.sum() - q / q.sum(), 0)
        sums = np.cumsum(w if w.sum() > 0 else p)
        assert int(c.tokens[b, 0]) == int(np.argmax(sums > u[b] * sums[-1])), b


@pytest.mark.parametrize("by", [0.0, 1e-6, 1e-5, 1e-4, 1e-3, 1e-2])
@pytest.mark.parametrize("tokens", [8, 400, 20000])
def test_probabilities_that_are_nearly_equal(tokens, by):
    """A draft row off the target's by `by` at so many tokens: what is left over is as small, below 2^-30 of p where doubles would leave open which
    of 20000 tokens it is, so the definition is computed with 64 bits of significand.  The drafts, which are no tokens, fall."""
    c = Case(48, 3, 20000, "fp32", seed=tokens + int(1 / by if by else 0))
    g = torch.Generator(device="cuda")
    g.manual_seed(tokens)
    at = torch.randperm(20000, generator=g, device="cuda")[:tokens]
    c.draft.copy_(c.target[:, :-1])
    c.draft[..., at] += by * torch.randn((48, 2, tokens), generator=g, device="cuda")
    c.draft_tokens.fill_(-1)
    c.call()
    check_what_is_left(c)


@pytest.mark.parametrize("tokens", [2, 40, 5000])
@pytest.mark.parametrize("vocab", [12000, 131072])
def test_probabilities_that_are_nearly_equal_but_for_some_tokens(vocab, tokens):
    """Pairs of tokens one of which a draft row gives what the other has in the target's: the ratio of the sums is that of all other tokens."""
    c = Case(48, 3, vocab, "fp32", seed=tokens)
    g = torch.Generator(device="cuda")
    g.manual_seed(tokens)
    at = torch.randperm(vocab, generator=g, device="cuda")[:2 * tokens]
    c.draft.copy_(c.target[:, :-1])
    x = c.target[:, :-1][..., at]
    more = torch.log(x.exp().unflatten(-1, (2, tokens)).sum(2))
    c.draft[..., at[:tokens]] = more + math.log(0.9)
    c.draft[..., at[tokens:]] = more + math.log(0.1)
    c.draft_tokens.fill_(-1)
    c.call()
    check_what_is_left(c)


@pytest.mark.parametrize("far", [3e4, -3e4])
def test_logits_far_from_zero(far):
    c = Case(20, 3, 3000, "fp32", seed=11)
    c.target += far
    c.draft -= far
    c.call()
    c.check()


def test_tokens_come_as_often_as_they_are_likely():
    """4096 numbers spread over [0, 1) on one row: every token as often as its probability says, to one."""
    c = Case(4096, 1, 300, "fp32", seed=12)
    c.target.copy_(c.target[:1].expand_as(c.target).clone())
    c.uniforms.copy_(((torch.arange(4096, device="cuda") + 0.5) / 4096)[:, None])
    c.call()
    torch.cuda.synchronize()
    counts = torch.bincount(c.tokens[:, 0].long(), minlength=300).double()
    assert ((counts - 4096 * torch.softmax(c.target[0, 0].double(), 0)).abs() <= 1.0).all()


def test_what_is_given_follows_the_target():
    """Drafts drawn from q, judged with numbers of their own: the first tokens' frequencies are p's (4 standard deviations)."""
    n, vocab = 4096, 6
    g = torch.Generator(device="cuda")
    g.manual_seed(13)
    c = Case(n, 2, vocab, "fp32", seed=13)
    c.target.copy_(torch.tensor([0.0, 1.0, -1.0, 0.5, 2.0, -math.inf], device="cuda").expand_as(c.target))
    c.draft.copy_(torch.tensor([1.0, 1.0, 0.0, -1.0, 0.5, 0.5], device="cuda").expand_as(c.draft))
    c.draft_tokens.copy_(torch.multinomial(torch.softmax(c.draft[:, 0], -1), 1, generator=g))
    c.call()
    torch.cuda.synchronize()
    p = torch.softmax(c.target[0, 0].double(), 0)
    counts = torch.bincount(c.tokens[:, 0].long(), minlength=vocab).double()
    assert ((counts - n * p).abs() <= 4 * torch.sqrt(n * p * (1 - p)) + 1e-9).all()


def test_without_token_lp_and_twice_the_same_bits():
    c = Case(64, 5, 20000, "bf16", seed=14)
    c.call()
    torch.cuda.synchronize()
    was = c.tokens.clone(), c.accepted.clone(), c.lp.clone()
    c.lp.fill_(7)
    c.call(lp=False)
    torch.cuda.synchronize()
    assert (c.lp == 7).all() and torch.equal(c.tokens, was[0]) and torch.equal(c.accepted, was[1])
    for _ in range(3):
        c.call()
        torch.cuda.synchronize()
        assert torch.equal(c.lp, was[2]) and torch.equal(c.tokens, was[0])


def test_captured_and_replayed():
    c = Case(16, 4, 30000, "bf16", seed=15, counts=[3] * 16)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    c.call(s)
    s.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        c.call(s)
    for i in range(5):
        c.counts = [(i + j) % 4 for j in range(16)]
        c.n_drafts.copy_(torch.tensor(c.counts, dtype=torch.int32))
        c.uniforms.uniform_()
        c.target += 0.25 * i
        c.tokens.fill_(-7)
        torch.cuda.synchronize()
        graph.replay()
        c.check()


def test_two_streams_at_once():
    cases = [Case(20, 3, 50000, "bf16", seed=16 + i) for i in range(2)]
    streams = [torch.cuda.Stream() for _ in cases]
    torch.cuda.synchronize()
    for _ in range(10):
        for c, s in zip(cases, streams):
            c.call(s)
    for c in cases:
        c.check()


def test_a_workspace_of_the_callers():
    c = Case(5, 4, 30000, "bf16", seed=18)
    need = xa.xbeam_verify_workspace_bytes(5, 4, 30000)
    ws = torch.full((need + 256,), 255, dtype=torch.uint8, device="cuda")
    try:
        xa.xattn_set_workspace((ws.data_ptr() + 255) // 256 * 256, need)
        c.call()
        c.check()
    finally:
        torch.cuda.synchronize()
        xa.xattn_set_workspace(None, 0)


def test_a_first_part_with_no_weight_and_a_number_of_zero():
    """The first 2048 of 6144 tokens have the same logits in both rows, e^-40 of the others', and the draft row has the target's others in another order: p's sum is
    q's, and the weights begin behind the first 2048.  The weights' sum may be off by 2^-30 of it, so a token up to there may come."""
    c = Case(512, 2, 6144, "fp32", seed=19, sd=1.0)
    g = torch.Generator(device="cuda")
    g.manual_seed(19)
    c.target.normal_(0.0, 1.0, generator=g)
    c.target[..., :2048] -= 40.0
    c.draft.copy_(c.target[:, :1])
    c.draft[..., 2048:] = torch.gather(c.draft[..., 2048:], 2, torch.rand((512, 1, 4096), generator=g, device="cuda").argsort(-1))
    c.draft_tokens.fill_(-1)
    c.uniforms.zero_()
    c.call()
    torch.cuda.synchronize()
    assert c.accepted.tolist() == [0] * 512
    target, draft = (x[:, 0].cpu().numpy().astype(np.longdouble) for x in (c.target, c.draft))
    tokens, lps = c.tokens[:, 0].tolist(), c.lp[:, 0].tolist()
    for b in range(512):
        p, q = (np.exp(x[b] - x[b].max()) for x in (target, draft))
        p, q = p / p.sum(), q / q.sum()
        sums = np.cumsum(np.maximum(p - q, 0))
        last = int(np.argmax(sums > 2.0 ** -30 * sums[-1]))
        assert 0 <= tokens[b] <= last and last >= 2048, (b, tokens[b], last)
        assert abs(lps[b] - float(np.log(p[tokens[b]]))) <= 2.0 ** -20 + 2.0 ** -23 * 60, b


@pytest.mark.parametrize("far", [5e10, -5e10, 1e11, -1e11, -1e30, 3e38, -3.4028234663852886e38])
@pytest.mark.parametrize("drafts", ["logits", "certain", "greedy"])
def test_finite_logits_of_any_size_have_probabilities(drafts, far):
    """So far from 0 a row's logits are all one value, and those of its tokens that lie a step of fp32 above it share p."""
    c = Case(24, 3, 3000, "fp32", "logits" if drafts == "greedy" else drafts, seed=20, greedy=drafts == "greedy")
    c.target.fill_(far)
    c.target[8:, :, 100:103] = float(np.nextafter(np.float32(far), np.float32(0)))
    c.target[16:, :, 2900:] = -math.inf
    c.target[16:20, :, 7] = 1.0                # has p alone where far is below it, none of it where above
    c.draft_tokens[:, 1] = 101
    if c.draft is not None:
        c.draft[:12] = -far
        c.draft[:6, :, 102] = float(np.nextafter(np.float32(-far), np.float32(0)))
    c.call()
    c.check()


@pytest.mark.parametrize("scale", [2.0 ** 20, 1.0, 2.0 ** -20])
@pytest.mark.parametrize("dtype,big", [("fp16", 64000.0), ("fp16", -65504.0), ("bf16", 3e38), ("bf16", -3e38), ("fp32", 1e34)])
def test_scales_and_logits_at_their_ends(dtype, big, scale):
    for drafts in ("logits", "certain"):
        c = Case(16, 3, 2500, dtype, drafts, seed=21, scale=scale, draft_scale=1.0)
        c.target[:8] = big
        c.target[8:, :, ::5] = big
        c.draft_tokens[:, 0] = 5
        c.call()
        c.check()


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
def test_tokens_forbidden_by_the_lowest_value(dtype):
    for drafts in ("logits", "certain"):
        c = Case(24, 4, 5000, dtype, drafts, seed=22)
        low = torch.finfo(c.target.dtype).min
        c.target[:, :, ::3] = low
        if c.draft is not None:
            c.draft[:12, :, ::3] = low
            c.draft[12:, :, 1::3] = low
        c.target[20:] = low                    # nothing else: all tokens are as likely
        c.call()
        c.check()


def test_no_row_takes_the_long_way_for_where_its_logits_lie():
    """Rows of logits moved by a constant, with temperatures of their own, take as long as others: the ratio of the sums of p and q that the first pass gives does not
    depend on that.  (A row whose sums are made anew takes 60 us more, four times a call's time.  Least of several runs, all calls in turn.)"""
    cases = [Case(4, 2, 131072, "fp32", seed=23)]
    for scale, draft_scale, far in ((0.5, 0.5, 300.0), (1.3, 0.6, 100.0), (1 / 0.65, 1 / 0.65, 100.0), (0.2, 1.0, 1000.0)):
        cases.append(Case(4, 2, 131072, "fp32", seed=23, scale=scale, draft_scale=draft_scale))
        cases[-1].target += far
    least = [math.inf] * len(cases)
    for c in cases:
        c.draft_tokens.fill_(-1)
        c.call()
    for _ in range(8):
        for i, c in enumerate(cases):
            begin, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
            torch.cuda.synchronize()
            begin.record()
            for _ in range(20):
                c.call()
            end.record()
            torch.cuda.synchronize()
            least[i] = min(least[i], begin.elapsed_time(end) / 20)
    assert max(least[1:]) < 2 * least[0], least
    for c in cases:
        c.check()
