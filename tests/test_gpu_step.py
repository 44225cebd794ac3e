"""A serving step's operators together, as a loop uses them: rotary positions and append, prompt attention, a head projection,
log-probabilities, beam selection; then decode steps on the same ranges, eager and from a captured graph."""
import math

import numpy as np
import pytest
import torch

import oracle
import paper_2510_14686_amd as xa

pytestmark = pytest.mark.gpu
HQ, HKV, D, VOCAB, TOP = 8, 2, 128, 5000, 8
MAX = 512


class Model:
    """One attention layer and a head projection on random weights; the ranges of up to `batch` sequences on an xTensor pool."""

    def __init__(self, batch, seed=0):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        self.batch = batch
        self.w_qkv = (torch.randn((256, (HQ + 2 * HKV) * D), generator=g, device="cuda") / 16).bfloat16()
        self.w_out = (torch.randn((HQ * D, VOCAB), generator=g, device="cuda") / 32).bfloat16()
        self.embed = torch.randn((VOCAB, 256), generator=g, device="cuda").bfloat16()
        self.inv_freq = (1e4 ** (-torch.arange(64, dtype=torch.float64) / 64)).float().cuda()
        self.pool = xa.xtensor_pool_create(0, 2 * batch, seed)
        row = HKV * D * 2
        opened = [[xa.xtensor_open(self.pool, b, MAX * row, MAX * row) for b in range(batch)] for _ in range(2)]
        self.ranges = [r for side in opened for (_, r, _) in side]
        self.ptrs = [torch.tensor([base for base, _, _ in side], dtype=torch.int64, device="cuda") for side in opened]
        self.kv_lens = torch.zeros(batch, dtype=torch.int32, device="cuda")

    def close(self):
        torch.cuda.synchronize()
        for r in self.ranges:
            xa.xtensor_close(r, False)
        xa.xtensor_pool_destroy(self.pool)

    def step(self, tokens, pos, q_starts, out, prefill=True):
        """Adds the packed tokens to the sequences (kv_lens holds the lengths after it) and gives their logits' log-probabilities."""
        n, stream = tokens.shape[0], torch.cuda.current_stream()
        qkv = self.embed[tokens.long()] @ self.w_qkv
        q, k, v = qkv.split([HQ * D, HKV * D, HKV * D], 1)
        xa.xattn_rope_kvcache(q, k, v, qkv.stride(0), qkv.stride(0), qkv.stride(0), pos, self.inv_freq, [16, 24, 24], 0, self.ptrs[0], self.ptrs[1],
                              q_starts, self.kv_lens, self.batch, n, HQ, HKV, D, out["q"], stream)
        if prefill:
            xa.xattn_prefill(out["q"], self.ptrs[0], self.ptrs[1], q_starts, self.kv_lens, self.batch, n, HQ, HKV, D, 1 / math.sqrt(D), out["att"], out["lse"], stream)
        else:
            xa.xattn_decode(out["q"], self.ptrs[0], self.ptrs[1], self.kv_lens, self.batch, n // self.batch, HQ, HKV, D, 1 / math.sqrt(D), out["att"], out["lse"], stream)
        out["logits"] = out["att"].view(n, HQ * D) @ self.w_out
        xa.xbeam_logprobs(out["logits"], xa.XBEAM_BF16, VOCAB, n, VOCAB, 1.0, out["given"], TOP, out["token_lp"], out["top_lp"], out["top_tok"],
                          out["row_lse"], out["entropy"], stream)
        return out, qkv


def buffers(n):
    f = lambda *s: torch.zeros(s, device="cuda")  # noqa: E731
    return dict(q=torch.zeros((n, HQ, D), dtype=torch.bfloat16, device="cuda"), att=torch.zeros((n, HQ, D), dtype=torch.bfloat16, device="cuda"), lse=f(n, HQ),
                given=torch.arange(n, dtype=torch.int32, device="cuda") * 37 % VOCAB, token_lp=f(n), top_lp=f(n, TOP),
                top_tok=torch.zeros((n, TOP), dtype=torch.int32, device="cuda"), row_lse=f(n), entropy=f(n))


class Reference:
    """The same layer in 64 bits, on what the step rounds to bf16: projections as they come, turned heads rounded."""

    def __init__(self, model):
        self.m, self.k, self.v = model, [[] for _ in range(model.batch)], [[] for _ in range(model.batch)]

    def turn(self, x, pos):
        axes = torch.repeat_interleave(torch.arange(3), torch.tensor([16, 24, 24])).cuda()
        a = (pos.double()[axes].t() * self.m.inv_freq.double())[:, None]
        u, v = x[..., :64].double(), x[..., 64:].double()
        return torch.cat((u * a.cos() - v * a.sin(), v * a.cos() + u * a.sin()), -1).bfloat16()

    def check(self, out, qkv, pos, starts):
        n = qkv.shape[0]
        q, k, v = qkv.split([HQ * D, HKV * D, HKV * D], 1)
        q, k, v = self.turn(q.reshape(n, HQ, D), pos), self.turn(k.reshape(n, HKV, D), pos), v.reshape(n, HKV, D)
        # turned heads: the same but for roundings that fall the other way, of one step; 2^-21 of two values of up to 5 each
        assert ((out["q"].double() - q.double()).abs() <= 2.0 ** -7 * q.double().abs() + 5e-6).all()
        for b in range(self.m.batch):
            rows = slice(starts[b], starts[b + 1])
            if starts[b] == starts[b + 1]:
                continue
            self.k[b].append(k[rows])
            self.v[b].append(v[rows])
            keys, values = torch.cat(self.k[b]), torch.cat(self.v[b])
            total, new = keys.shape[0], starts[b + 1] - starts[b]
            seen = torch.arange(total, device="cuda")[None] < (total - new + 1 + torch.arange(new, device="cuda"))[:, None]
            for h in range(HQ):
                kk, vv = keys[:, h // 4].double(), values[:, h // 4].double()
                x = (out["q"][rows, h].double() @ kk.t().contiguous() / math.sqrt(D)).masked_fill(~seen, -math.inf)
                p = torch.softmax(x, 1)
                ref, size = p @ vv, p @ vv.abs()
                # roundings of result and weights (2^-8 each), and a key that fell the other way: 2^-8 of a product of the score
                off = 2.0 ** -8 * (out["q"][rows, h].double().abs() @ kk.abs().t().contiguous() / math.sqrt(D)).masked_fill(~seen, 0).amax(1)[:, None] * 2 / 8
                assert ((out["att"][rows, h].double() - ref).abs() <= 2.0 ** -8 * ref.abs() + size * (2.0 ** -8 + off) + 1e-6).all(), (b, h)
        lp = torch.log_softmax(out["logits"].double(), 1)
        assert (out["token_lp"].double() - lp.gather(1, out["given"].long()[:, None])[:, 0]).abs().max() < 2e-5
        assert (out["entropy"].double() - torch.special.entr(lp.exp()).sum(1)).abs().max() < 2e-5
        best = lp.sort(dim=1, descending=True, stable=True)
        assert torch.equal(out["top_tok"].long(), best.indices[:, :TOP])
        assert (out["top_lp"].double() - best.values[:, :TOP]).abs().max() < 2e-5


def test_prompts_then_decode_steps():
    m = Model(4)
    try:
        ref, rng = Reference(m), np.random.RandomState(1)
        lens = np.zeros(4, np.int64)
        # prompts, a second chunk for some of them beside single tokens for the others, then decode steps of one and of two tokens
        for new, prefill in (([100, 37, 1, 64], True), ([1, 150, 1, 0], True), ([1, 1, 1, 1], True), ([1, 1, 1, 1], False), ([2, 2, 2, 2], False)):
            starts = [0] + list(np.cumsum(new))
            lens += new
            m.kv_lens.copy_(torch.tensor(lens, dtype=torch.int32))
            n = starts[-1]
            tokens = torch.tensor(rng.randint(0, VOCAB, n), device="cuda")
            pos = torch.tensor(rng.randint(0, 400, (3, n)), dtype=torch.int32, device="cuda")
            out, qkv = m.step(tokens, pos, torch.tensor(starts, dtype=torch.int32, device="cuda"), buffers(n), prefill)
            torch.cuda.synchronize()
            ref.check(out, qkv, pos, starts)
        # the last step's alternatives through beam selection: a request of four beams
        cand, tok = out["top_lp"][1::2].cpu().numpy()[None], out["top_tok"][1::2].cpu().numpy()[None]
        beam = np.array([[-1.0, -1.5, -2.0, -2.5]], np.float32)
        got, want = xa.xbeam_select(beam, cand, tok, flags=xa.XBEAM_CHECK_INPUT), oracle.beam_select(beam, cand, tok)
        assert all(np.array_equal(a, b) for a, b in zip(got[:3], want))
    finally:
        m.close()


def test_captured_steps():
    """A decode step of all operators as a graph: every replay the bits of the eager step."""
    m, other = Model(4, seed=2), Model(4, seed=2)
    try:
        starts = torch.arange(5, dtype=torch.int32, device="cuda")
        tokens, pos = torch.zeros(4, dtype=torch.int64, device="cuda"), torch.zeros((3, 4), dtype=torch.int32, device="cuda")
        out, eager = buffers(4), buffers(4)
        stream = torch.cuda.Stream()
        with torch.cuda.stream(stream):
            m.kv_lens.fill_(1)
            other.kv_lens.fill_(1)
            for _ in range(2):
                m.step(tokens, pos, starts, out)
                other.step(tokens, pos, starts, eager)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            m.step(tokens, pos, starts, out)
        for i in range(2, 12):
            for x in (m, other):
                x.kv_lens.fill_(i)
            tokens.copy_(torch.arange(4, device="cuda") * 997 * i % VOCAB)
            pos.fill_(i)
            torch.cuda.synchronize()
            graph.replay()
            with torch.cuda.stream(stream):
                other.step(tokens, pos, starts, eager)
            torch.cuda.synchronize()
            for name in ("q", "att", "lse", "logits", "token_lp", "top_lp", "top_tok", "row_lse", "entropy"):
                assert torch.equal(out[name], eager[name]), (i, name)
    finally:
        m.close()
        other.close()
