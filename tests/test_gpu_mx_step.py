"""A speculative serving loop on a cache of 4 bits a value, all its operators together: prompts (append, read back, prompt attention), then steps of a
token and its drafts (append, decode attention, a head projection, verification), after which the sequences keep the rows of what stands."""
import math

import numpy as np
import pytest
import torch

import mx_util
import paper_2510_14686_amd as xa

pytestmark = pytest.mark.gpu
HQ, HKV, D, VOCAB = 8, 2, 128, 3000
SCALE = 1 / math.sqrt(D)


class Model:
    """One attention layer and a head projection on random weights; the ranges of `batch` sequences on an xTensor pool."""

    def __init__(self, batch, seed=0, most=512):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        self.batch = batch
        self.w_qkv = (torch.randn((256, (HQ + 2 * HKV) * D), generator=g, device="cuda") / 16).bfloat16()
        self.w_out = (torch.randn((HQ * D, VOCAB), generator=g, device="cuda") / 16).bfloat16()
        self.embed = torch.randn((VOCAB, 256), generator=g, device="cuda").bfloat16()
        self.inv_freq = (1e4 ** (-torch.arange(64, dtype=torch.float64) / 64)).float().cuda()
        size = xa.xattn_mx_range_bytes(most, HKV)
        self.pool = xa.xtensor_pool_create(0, 2 * batch, seed)
        opened = [[xa.xtensor_open(self.pool, b, size, size) for b in range(batch)] for _ in range(2)]
        self.ranges = [r for side in opened for (_, r, _) in side]
        self.ptrs = [torch.tensor([base for base, _, _ in side], dtype=torch.int64, device="cuda") for side in opened]
        self.kv_lens = torch.zeros(batch, dtype=torch.int32, device="cuda")

    def close(self):
        torch.cuda.synchronize()
        for r in self.ranges:
            xa.xtensor_close(r, False)
        xa.xtensor_pool_destroy(self.pool)

    def project(self, tokens):
        qkv = self.embed[tokens.long()] @ self.w_qkv
        return qkv, qkv.split([HQ * D, HKV * D, HKV * D], 1)

    def append(self, tokens, pos, q_starts, q_out):
        qkv, (q, k, v) = self.project(tokens)
        xa.xattn_rope_kvcache_mx(q, k, v, qkv.stride(0), qkv.stride(0), qkv.stride(0), pos, self.inv_freq, [64], 0, *self.ptrs, q_starts, self.kv_lens, self.batch,
                                 tokens.shape[0], HQ, HKV, D, q_out, torch.cuda.current_stream())

    def prompt(self, tokens, pos, q_starts, lens):
        """Attention of the packed new tokens: all rows are read back, and attended by xattn_prefill."""
        stream, n = torch.cuda.current_stream(), tokens.shape[0]
        q = torch.empty((n, HQ, D), dtype=torch.bfloat16, device="cuda")
        self.append(tokens, pos, q_starts, q)
        starts = torch.tensor(np.concatenate([[0], np.cumsum(lens)]), dtype=torch.int32, device="cuda")
        rows = [torch.empty((int(sum(lens)), HKV, D), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        xa.xattn_read_kvcache_mx(*self.ptrs, starts, self.kv_lens, self.batch, int(sum(lens)), HKV, D, *rows, stream)
        ptrs = [r.data_ptr() + starts[:-1].long() * HKV * D * 2 for r in rows]
        out = torch.empty((n, HQ, D), dtype=torch.bfloat16, device="cuda")
        xa.xattn_prefill(q, *ptrs, q_starts, self.kv_lens, self.batch, n, HQ, HKV, D, SCALE, out, None, stream)
        return q, out

    def buffers(self, q_len):
        n = self.batch
        f = lambda *s: torch.zeros(s, device="cuda")  # noqa: E731
        i = lambda *s: torch.zeros(s, device="cuda", dtype=torch.int32)  # noqa: E731
        bf = lambda *s: torch.zeros(s, device="cuda", dtype=torch.bfloat16)  # noqa: E731
        return dict(q=bf(n * q_len, HQ, D), out=bf(n, q_len, HQ, D), lse=f(n, q_len, HQ), tokens=i(n, q_len), accepted=i(n), lp=f(n, q_len), uniforms=f(n, q_len),
                    starts=torch.arange(0, n * q_len + 1, q_len, dtype=torch.int32, device="cuda"), pos=i(1, n * q_len), last=i(n), drafted=i(n, q_len - 1))

    def step(self, b, q_len, draft=None):
        """A speculative step: the last token and its drafts go in, what stands and one more token come out; kv_lens is what is kept before and after."""
        stream, n = torch.cuda.current_stream(), self.batch
        self.kv_lens.add_(q_len)
        b["pos"].copy_((self.kv_lens[:, None] - q_len + torch.arange(q_len, dtype=torch.int32, device="cuda")).view(1, -1))
        self.append(torch.cat((b["last"][:, None], b["drafted"]), 1).view(-1), b["pos"], b["starts"], b["q"])
        xa.xattn_decode_mx(b["q"], *self.ptrs, self.kv_lens, n, q_len, HQ, HKV, D, SCALE, b["out"], b["lse"], stream)
        b["logits"] = b["out"].view(n * q_len, HQ * D) @ self.w_out
        xa.xbeam_verify(b["logits"], VOCAB, draft, VOCAB if draft is not None else 0, xa.XBEAM_BF16, VOCAB, 1.0, 1.0, b["drafted"], None, b["uniforms"], n, q_len, 0,
                        b["tokens"], b["accepted"], b["lp"], stream)
        self.kv_lens.sub_(q_len - 1 - b["accepted"])
        b["last"].copy_(b["tokens"].gather(1, b["accepted"][:, None].long())[:, 0])
        return b


class Reference:
    """The layer in 64 bits on the rows that the definition stores."""

    def __init__(self, model):
        self.m, self.k, self.v = model, [torch.zeros((0, HKV, D), dtype=torch.float64, device="cuda") for _ in range(model.batch)], \
            [torch.zeros((0, HKV, D), dtype=torch.float64, device="cuda") for _ in range(model.batch)]

    def rows(self, tokens, pos):
        _, (q, k, v) = self.m.project(tokens)
        a = (pos.double()[0][:, None] * self.m.inv_freq.double())[:, None]

        def turn(x):
            x, y = x.double().unflatten(1, (-1, D))[..., :64], x.double().unflatten(1, (-1, D))[..., 64:]
            return torch.cat((x * a.cos() - y * a.sin(), y * a.cos() + x * a.sin()), -1)

        stored = [mx_util.decode(*mx_util.encode(x)) for x in (turn(k), v.double().unflatten(1, (-1, D)))]
        return turn(q), stored[0], stored[1]

    def add(self, tokens, pos, starts):
        q, k, v = self.rows(tokens, pos)
        for b in range(self.m.batch):
            self.k[b], self.v[b] = torch.cat((self.k[b], k[starts[b]:starts[b + 1]])), torch.cat((self.v[b], v[starts[b]:starts[b + 1]]))
        return q

    def keep(self, b, n):
        self.k[b], self.v[b] = self.k[b][:n], self.v[b][:n]

    def check(self, q_got, q, out, starts, weights_off):
        # turned heads: one rounding of 2^-8, 2^-21 of two values of up to 5 each
        assert ((q_got.double() - q).abs() <= 2.0 ** -8 * q.abs() + 5e-6).all()
        for b in range(self.m.batch):
            rows = slice(starts[b], starts[b + 1])
            total, new = self.k[b].shape[0], starts[b + 1] - starts[b]
            seen = torch.arange(total, device="cuda")[None] < (total - new + 1 + torch.arange(new, device="cuda"))[:, None]
            for h in range(HQ):
                k, v = self.k[b][:, h // 4], self.v[b][:, h // 4]
                x = (SCALE * (q_got[rows, h].double() @ k.t().contiguous())).masked_fill(~seen, -math.inf)
                p = torch.softmax(x, 1)
                a = 2.0 ** -17 * SCALE * (q_got[rows, h].double().abs() @ k.abs().t().contiguous()).masked_fill(~seen, 0).amax(1)[:, None]
                # the result's rounding 2^-8, a weight's as given, scores as in test_gpu_mx_decode.py
                assert ((out[rows, h].double() - p @ v).abs() <= 2.0 ** -8 * (p @ v).abs() + (weights_off + 2 * a) * (p @ v.abs()) + 1e-9).all(), (b, h)


def verified(logits, drafted, uniforms):
    """(tokens, accepted) of certain drafts."""
    tokens, accepted = [], []
    for b in range(logits.shape[0]):
        p = torch.softmax(logits[b].double(), 1)
        t = 0
        while t < len(drafted[b]) and float(uniforms[b, t]) < float(p[t, drafted[b][t]]):
            t += 1
        w = p[t].clone()
        if t < len(drafted[b]):
            w[drafted[b][t]] = 0
        c = torch.cumsum(w, 0)
        tokens.append(list(drafted[b][:t]) + [int((c <= float(uniforms[b, -1]) * float(c[-1])).sum())] + [-1] * (len(drafted[b]) - t))
        accepted.append(t)
    return tokens, accepted


def test_prompts_and_speculative_steps():
    m = Model(4)
    try:
        ref, rng = Reference(m), np.random.RandomState(1)
        lens = np.zeros(4, np.int64)
        for new in ([100, 37, 1, 64], [30, 150, 70, 1]):      # two chunks of every prompt
            starts = [0] + [int(x) for x in np.cumsum(new)]
            pos = torch.tensor(np.concatenate([np.arange(a, a + n) for a, n in zip(lens, new)])[None], dtype=torch.int32, device="cuda")
            lens += new
            m.kv_lens.copy_(torch.tensor(lens, dtype=torch.int32))
            tokens = torch.tensor(rng.randint(0, VOCAB, starts[-1]), device="cuda")
            q, out = m.prompt(tokens, pos, torch.tensor(starts, dtype=torch.int32, device="cuda"), lens)
            torch.cuda.synchronize()
            ref.check(q, ref.add(tokens, pos, starts), out, starts, 2.0 ** -7)      # xattn_prefill's weights: 2^-8, and their sum's
        for q_len in (4, 4, 2, 1, 5):
            b = m.buffers(q_len)
            b["last"].copy_(torch.tensor(rng.randint(0, VOCAB, 4)))
            b["uniforms"].copy_(torch.tensor(rng.rand(4, q_len), dtype=torch.float32))
            before = [x.shape[0] for x in ref.k]
            # drafts that the model is likely to agree with: its own best ones, found by running the step with others
            b["drafted"].copy_(torch.tensor(rng.randint(0, VOCAB, (4, q_len - 1))))
            for _ in range(q_len - 1):
                m.kv_lens.copy_(torch.tensor(before, dtype=torch.int32))
                last = b["last"].clone()
                m.step(b, q_len)
                b["last"].copy_(last)
                b["drafted"].copy_(b["logits"].view(4, q_len, VOCAB)[:, :-1].argmax(-1))
            m.kv_lens.copy_(torch.tensor(before, dtype=torch.int32))
            tokens = torch.cat((b["last"][:, None], b["drafted"]), 1).view(-1)
            m.step(b, q_len)
            torch.cuda.synchronize()
            starts = list(range(0, 4 * q_len + 1, q_len))
            ref.check(b["q"], ref.add(tokens, b["pos"], starts), b["out"].view(4 * q_len, HQ, D), starts, 2.0 ** -14)
            want = verified(b["logits"].view(4, q_len, VOCAB), b["drafted"].tolist(), b["uniforms"])
            assert (b["tokens"].tolist(), b["accepted"].tolist()) == want
            for i in range(4):
                ref.keep(i, before[i] + 1 + want[1][i])      # the last token and the drafts that stand; the next step writes over the others
            assert m.kv_lens.tolist() == [x.shape[0] for x in ref.k]
    finally:
        m.close()


def test_captured_steps():
    """A speculative step of all operators as a graph: every replay the tokens and bits of the eager step."""
    m, other = Model(3, seed=2, most=2048), Model(3, seed=2, most=2048)
    try:
        b, eager = m.buffers(3), other.buffers(3)
        draft = torch.randn((6, VOCAB), device="cuda").bfloat16()
        stream = torch.cuda.Stream()
        stream.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(stream):
            for _ in range(2):
                m.step(b, 3, draft)
                other.step(eager, 3, draft)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            m.step(b, 3, draft)
        g = torch.Generator(device="cuda")
        g.manual_seed(3)
        for i in range(30):
            draft.normal_(generator=g)
            for x in (b, eager):
                x["uniforms"].copy_(torch.rand((3, 3), generator=torch.Generator("cuda").manual_seed(i), device="cuda"))
                x["drafted"].copy_(torch.arange(6, device="cuda").view(3, 2) * 37 * (i + 1) % VOCAB)
            torch.cuda.synchronize()
            graph.replay()
            with torch.cuda.stream(stream):
                other.step(eager, 3, draft)
            torch.cuda.synchronize()
            assert torch.equal(m.kv_lens, other.kv_lens)
            for name in ("q", "out", "lse", "logits", "tokens", "accepted", "lp", "last"):
                assert torch.equal(b[name], eager[name]), (i, name)
    finally:
        m.close()
        other.close()
