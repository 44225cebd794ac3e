"""Decode attention over a cache of 4 bits a value (xattn_decode_mx) against the definition in 64 bits on the same codes.

What may be off: the result's rounding to bf16, 2^-8 of it; a score, 128 products added in fp32 and scaled, by 2^-17 of its products' sizes
added up (A), which moves a weight by as much of itself, and a result by twice that of sum p |v|; a weight as two bf16, 2^-16 of it, its
exponential 2^-21, sums over lanes and parts in fp32 2^-18: together 2^-14 of sum p |v|.
"""
import math

import numpy as np
import pytest
import torch

import mx_util
import paper_2510_14686_amd as xa

pytestmark = pytest.mark.gpu
D = 128


class Case:
    def __init__(self, lens, hq, hkv, q_len=1, scale=None, seed=0, size=1.0, grow=0):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        self.lens, self.hq, self.hkv, self.q_len, self.batch = lens, hq, hkv, q_len, len(lens)
        self.scale = 1 / math.sqrt(D) if scale is None else scale
        rows = [[size * torch.randn((max(n, 0) + grow, hkv, D), generator=g, device="cuda") for n in lens] for _ in range(2)]
        self.ranges = mx_util.Ranges([max(n, 0) + grow for n in lens], hkv, fill=255, rows=rows)
        self.q = torch.randn((self.batch, q_len, hq, D), generator=g, device="cuda").bfloat16()
        self.kv_lens = torch.tensor(lens, dtype=torch.int32, device="cuda")
        self.out = torch.full_like(self.q, 7.0)
        self.lse = torch.full((self.batch, q_len, hq), 7.0, device="cuda")

    def call(self, stream=None, lse=True):
        xa.xattn_decode_mx(self.q, *self.ranges.ptrs, self.kv_lens, self.batch, self.q_len, self.hq, self.hkv, D, self.scale, self.out,
                           self.lse if lse else None, stream or torch.cuda.current_stream())

    def check(self, sequences=None, lens=None):
        torch.cuda.synchronize()
        group = self.hq // self.hkv
        for b in range(self.batch) if sequences is None else sequences:
            n = max((lens or self.lens)[b], 0)
            out, lse = self.out[b].double(), self.lse[b].double()
            k, v = (self.ranges.values(w, b, n) for w in range(2))
            seen = torch.arange(n, device="cuda")[None] < (n - self.q_len + 1 + torch.arange(self.q_len, device="cuda"))[:, None]
            for h in range(self.hq):
                kk, vv, q = k[:, h // group], v[:, h // group], self.q[b, :, h].double()
                x = (self.scale * (q @ kk.t().contiguous())).masked_fill(~seen, -math.inf)
                a = 2.0 ** -17 * abs(self.scale) * (q.abs() @ kk.abs().t().contiguous()).masked_fill(~seen, 0.0).amax(1) if n else torch.zeros(self.q_len, device="cuda")
                some = seen.any(1)
                assert (out[~some, h] == 0).all() and (lse[~some, h] == -math.inf).all(), (b, h)
                if not some.any():
                    continue
                p = torch.softmax(x[some], 1)
                ref, size = p @ vv, p @ vv.abs()
                assert ((out[some, h] - ref).abs() <= 2.0 ** -8 * ref.abs() + size * (2.0 ** -14 + 2 * a[some, None]) + 1e-30).all(), (b, h, n)
                want = torch.logsumexp(x[some], 1)
                assert ((lse[some, h] - want).abs() <= a[some] + 2.0 ** -18 * (1 + want.abs())).all(), (b, h, n)


@pytest.mark.parametrize("hq,hkv", [(8, 2), (4, 4), (5, 1), (16, 2), (64, 8), (40, 8), (8, 1), (64, 1), (1, 1), (9, 3)])
def test_heads(hq, hkv):
    c = Case([17, 64, 100, 256, 1, 65, 1000], hq, hkv, seed=hq)
    c.call()
    c.check()


@pytest.mark.parametrize("q_len", [2, 3, 4, 8, 16])
@pytest.mark.parametrize("hq,hkv", [(4, 4), (8, 2), (3, 1)])
def test_new_tokens_see_what_is_before_them(hq, hkv, q_len):
    c = Case([q_len, 64, 100, 63 + q_len, 1000, 129, q_len + 1], hq, hkv, q_len, seed=q_len)
    c.call()
    c.check()


@pytest.mark.parametrize("q_len", [1, 4])
def test_lengths_of_nothing_and_below_the_new_tokens(q_len):
    c = Case([0, 3, 1, 0, -5, 70, 2, 0], 8, 2, q_len, seed=1)
    c.call()
    c.check()
    c = Case([0, -2 ** 31, 0], 8, 2, q_len)
    c.call()
    c.check()


@pytest.mark.parametrize("length", [1, 2, 15, 16, 17, 63, 64, 65, 127, 128, 129, 511, 512, 513, 3000])
def test_one_sequence(length):
    c = Case([length], 8, 2, seed=length)
    c.call()
    c.check()


@pytest.mark.parametrize("hq,hkv,q_len,lens", [
    (32, 8, 1, [40000]), (8, 1, 1, [70001]), (32, 8, 4, [9000, 10, 20000, 1]), (16, 1, 4, [5000, 64, 12345]), (8, 8, 1, [30, 20000] + [100] * 30),
    (64, 2, 2, [700, 1300, 64]), (40, 8, 3, [1 + 37 * i for i in range(70)])], ids=str)
def test_long_and_uneven(hq, hkv, q_len, lens):
    c = Case(lens, hq, hkv, q_len, seed=len(lens))
    c.call()
    c.check(range(0, len(lens), 1 if len(lens) < 20 else 9))


@pytest.mark.parametrize("batch", [63, 64, 65, 500, 4096])
def test_batches(batch):
    c = Case([(i * 31) % 150 for i in range(batch)], 4, 2, 1, seed=batch)
    c.call()
    c.check(range(0, batch, max(1, batch // 60)))


@pytest.mark.parametrize("scale", [0.0, -0.1, 1.0, 20.0, 1e-30])
def test_scales(scale):
    c = Case([5, 200, 700], 8, 2, 2, scale=scale, seed=2)
    c.call()
    c.check()


@pytest.mark.parametrize("size", [2.0 ** -100, 2.0 ** -30, 2.0 ** 30])
def test_rows_far_from_one(size):
    c = Case([5, 200], 8, 2, 1, scale=0.1 / size, seed=3, size=size)
    c.call()
    c.check()


def test_scales_of_single_blocks_differ_widely():
    """Blocks 2^40 apart in one row, and rows 2^40 apart in one tile."""
    c = Case([130, 64], 4, 2, 1, seed=4)
    g = torch.Generator(device="cuda")
    g.manual_seed(4)
    for which in range(2):
        for b, n in enumerate(c.lens):
            x = torch.randn((n, 2, D), generator=g, device="cuda").double()
            if which == 1:
                x *= torch.exp2(torch.randint(-20, 21, (n, 2, 4), generator=g, device="cuda").double()).repeat_interleave(32, -1)
            else:
                x[:, :, 32:64] *= 2.0 ** -40
                x[:, :, 96:] *= 2.0 ** -20
            mx_util.put(c.ranges.caches[which][b], torch.arange(n, device="cuda"), 2, which == 1, *mx_util.encode(x))
    c.call()
    c.check()


def test_a_key_that_has_all_the_weight():
    c = Case([3, 64, 200, 1000], 4, 2, 1, seed=5)
    for b, n in enumerate(c.lens):
        x = torch.zeros((1, 2, D), device="cuda")
        x[0, :] = 6 * torch.sign(c.q[b, 0, ::2].float())
        mx_util.put(c.ranges.caches[0][b], torch.tensor([n // 2], device="cuda"), 2, False, *mx_util.encode(x))
    c.call()
    c.check()


def test_another_sequence_with_nan_changes_nothing():
    c = Case([100, 300, 64], 8, 2, 1, seed=6)
    c.call()
    torch.cuda.synchronize()
    was = c.out.clone(), c.lse.clone()
    for which in range(2):
        mx_util.put(c.ranges.caches[which][1], torch.tensor([0, 299], device="cuda"), 2, which == 1, torch.zeros((2, 2, D), device="cuda", dtype=torch.int32),
                    torch.full((2, 2, 4), 255, device="cuda"))
    c.call()
    torch.cuda.synchronize()
    for b in (0, 2):
        assert torch.equal(c.out[b], was[0][b]) and torch.equal(c.lse[b], was[1][b])


def test_without_lse_and_twice_the_same_bits():
    c = Case([1000, 17, 3000, 64, 5], 32, 8, 2, seed=7)
    c.call(lse=False)
    torch.cuda.synchronize()
    was = c.out.clone()
    assert (c.lse == 7).all()
    for _ in range(3):
        c.out.fill_(7)
        c.call()
        torch.cuda.synchronize()
        assert torch.equal(c.out, was)
    c.check()


def test_captured_and_replayed_with_other_lengths():
    c = Case([500, 17, 900, 64, 130], 8, 2, 2, seed=8)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    c.call(s)
    s.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        c.call(s)
    for lens in ([500, 17, 900, 64, 130], [1, 2, 3, 0, 130], [2, 17, 64, 63, 65], [400, 1, 899, 10, 128]):
        c.kv_lens.copy_(torch.tensor(lens, dtype=torch.int32))
        c.out.fill_(7)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        c.check(lens=lens)
        got = c.out.clone()
        c.call()
        torch.cuda.synchronize()
        assert torch.equal(got, c.out)


def test_two_streams_at_once():
    cases = [Case([700 + 100 * i, 64, 3000], 32, 8, 1, seed=20 + i) for i in range(2)]
    streams = [torch.cuda.Stream() for _ in cases]
    torch.cuda.synchronize()
    for _ in range(20):
        for c, s in zip(cases, streams):
            c.call(s)
    for c in cases:
        c.check()


def test_a_workspace_of_the_callers():
    c = Case([1000, 17, 3000], 16, 4, 2, seed=9)
    need = xa.xattn_decode_mx_workspace_bytes(3, 2, 16, 4)
    ws = torch.full((need + 256,), 255, dtype=torch.uint8, device="cuda")
    base = (ws.data_ptr() + 255) // 256 * 256
    try:
        xa.xattn_set_workspace(base, need)
        c.call()
        c.check()
        xa.xattn_set_workspace(base, need - 1)
        with pytest.raises(xa.XattnError):
            c.call()
    finally:
        torch.cuda.synchronize()
        xa.xattn_set_workspace(None, 0)


def test_on_an_xtensor_range():
    """The tiles of a sequence on 2 MiB pages that lie anywhere; the sequence ends inside the last page's last tile."""
    c = Case([20000], 32, 8, 1, seed=10)
    handles, ptrs = [], []
    try:
        for side in c.ranges.caches:
            base, handle = xa.xtensor_map(64 << 20, side[0].numel(), 3, 0)
            handles.append(handle)
            xa.xtensor_upload(base, side[0].cpu().numpy())
            ptrs.append(torch.tensor([base], dtype=torch.int64, device="cuda"))
        xa.xattn_decode_mx(c.q, *ptrs, c.kv_lens, 1, 1, 32, 8, D, c.scale, c.out, c.lse, torch.cuda.current_stream())
        c.check()
    finally:
        torch.cuda.synchronize()
        for h in handles:
            xa.xtensor_unmap(h)


def test_a_range_of_more_than_four_gigabytes():
    """64 heads, a million tokens of zeros but for one behind 4 GiB, which has nearly all the weight."""
    n, heads = 1000001, 64
    size = xa.xattn_mx_range_bytes(n, heads)
    caches = [torch.zeros(size, dtype=torch.uint8, device="cuda") for _ in range(2)]
    ptrs = [torch.tensor([x.data_ptr()], dtype=torch.int64, device="cuda") for x in caches]
    q = torch.randn((1, 1, heads, D), device="cuda").bfloat16()
    at = torch.tensor([n - 2], device="cuda")
    k, v = 3 * q[0].double(), torch.randn((1, heads, D), device="cuda").double()
    kc, vc = mx_util.encode(k), mx_util.encode(v)
    mx_util.put(caches[0], at, heads, False, *kc)
    mx_util.put(caches[1], at, heads, True, *vc)
    out = torch.empty_like(q)
    lse = torch.empty((1, 1, heads), device="cuda")
    xa.xattn_decode_mx(q, *ptrs, torch.tensor([n], dtype=torch.int32, device="cuda"), 1, 1, heads, heads, D, 1 / math.sqrt(D), out, lse, torch.cuda.current_stream())
    torch.cuda.synchronize()
    s = (mx_util.decode(*kc)[0] * q[0, 0].double()).sum(-1) / math.sqrt(D)
    p = 1 / (1 + (n - 1) * torch.exp(-s))
    ref = p[:, None] * mx_util.decode(*vc)[0]
    size = p[:, None] * mx_util.decode(*vc)[0].abs()
    a = 2.0 ** -17 * (mx_util.decode(*kc)[0].abs() * q[0, 0].double().abs()).sum(-1)[:, None] / math.sqrt(D)
    # the zeros' weights are added up a million times in 32 bits, by lanes of at most 2000: 2^-13
    assert ((out[0, 0].double() - ref).abs() <= 2.0 ** -8 * ref.abs() + size * (2.0 ** -13 + 2 * a)).all()
    want = torch.logsumexp(torch.stack((s, math.log(n - 1) + torch.zeros_like(s))), 0)
    assert ((lse[0, 0].double() - want).abs() <= a[:, 0] + 2.0 ** -13).all()
