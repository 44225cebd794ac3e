"""Rotary positions with append (xattn_rope_kvcache) against the definition in 64 bits.

A turned value x cos a - y sin a is rounded to bf16 once (2^-8 of it); sine and cosine are off by 2^-22, and the two products and
their sum in fp32 by 2^-23 of |x| + |y|: 2^-21 (|x| + |y|) in all; an angle a of a far position, of which both sides round products in
double, by 2^-51 a besides.  Everything that is only moved stays as it is, bit for bit.
"""
import math

import numpy as np
import pytest
import torch

import paper_2510_14686_amd as xa

pytestmark = pytest.mark.gpu


def axis_list(sections, dealt):
    if not dealt:
        return [a for a, n in enumerate(sections) for _ in range(n)]
    left, out, a = list(sections), [], 0
    while sum(left):
        if left[a]:
            out.append(a)
            left[a] -= 1
        a = (a + 1) % len(left)
    return out


class Batch:
    def __init__(self, lens, hq, hkv, d, sections, flags=0, far=0, extra=0, pad=0, seed=0, inplace=False):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        self.lens, self.hq, self.hkv, self.d, self.sections, self.flags = lens, hq, hkv, d, sections, flags
        self.starts = np.concatenate([[0], np.cumsum([n for n, _ in lens])])
        self.total = int(self.starts[-1]) + extra
        width = (hq + 2 * hkv) * d + pad
        self.qkv = torch.randn((self.total, width), generator=g, device="cuda").bfloat16()
        if inplace:
            self.q, self.k_new, self.v_new = (torch.randn((self.total, h * d), generator=g, device="cuda").bfloat16() for h in (hq, hkv, hkv))
        else:
            self.q, self.k_new, self.v_new = self.qkv[:, :hq * d], self.qkv[:, hq * d:(hq + hkv) * d], self.qkv[:, (hq + hkv) * d:(hq + 2 * hkv) * d]
        f = sum(sections)
        self.pos = torch.randint(-50, 5000, (len(sections), self.total), generator=g, device="cuda", dtype=torch.int32) + far
        self.inv_freq = (1e4 ** (-torch.arange(f, dtype=torch.float64) / max(f, 1))).float().cuda()
        self.caches = [torch.randn((sum(max(kv, 1) for _, kv in lens), hkv, d), generator=g, device="cuda").bfloat16() for _ in range(2)]
        self.bounds = np.concatenate([[0], np.cumsum([max(kv, 1) for _, kv in lens])])
        self.ptrs = [torch.tensor([c.data_ptr() + int(b) * hkv * d * 2 for b in self.bounds[:-1]], dtype=torch.int64, device="cuda") for c in self.caches]
        self.q_starts = torch.tensor(self.starts, dtype=torch.int32, device="cuda")
        self.kv_lens = torch.tensor([kv for _, kv in lens], dtype=torch.int32, device="cuda")
        self.inplace = inplace
        self.out = self.q if inplace else torch.full((self.total, hq, d), 7.0, dtype=torch.bfloat16, device="cuda")
        self.before = [c.clone() for c in self.caches]
        self.was = [x.clone() for x in (self.q, self.k_new, self.v_new)]

    def call(self, stream=None):
        xa.xattn_rope_kvcache(self.q, self.k_new, self.v_new, self.q.stride(0), self.k_new.stride(0), self.v_new.stride(0), self.pos, self.inv_freq,
                              self.sections, self.flags, self.ptrs[0], self.ptrs[1], self.q_starts, self.kv_lens, len(self.lens), self.total,
                              self.hq, self.hkv, self.d, self.out, stream or torch.cuda.current_stream())

    def turned(self, x):
        """(rotated heads in 64 bits, how far off they may be) of [rows, heads, d]."""
        x, f = x.double(), sum(self.sections)
        axes = torch.tensor(axis_list(self.sections, self.flags & xa.XATTN_ROPE_DEALT), device="cuda")
        a = (self.pos.double()[axes].t() * self.inv_freq.double())[:, None] if f else torch.zeros((x.shape[0], 1, 0), device="cuda", dtype=torch.float64)
        at = (slice(0, 2 * f, 2), slice(1, 2 * f, 2)) if self.flags & xa.XATTN_ROPE_PAIRS else (slice(0, f), slice(f, 2 * f))
        u, v = x[..., at[0]], x[..., at[1]]
        out, tol = x.clone(), torch.zeros_like(x)
        out[..., at[0]], out[..., at[1]] = u * a.cos() - v * a.sin(), v * a.cos() + u * a.sin()
        for i in at:
            tol[..., i] = 2.0 ** -8 * out[..., i].abs() + (2.0 ** -21 + 2.0 ** -51 * a.abs()) * (u.abs() + v.abs())
        return out, tol

    def check(self):
        torch.cuda.synchronize()
        new = int(self.starts[-1])
        q, k, v = (x.view(self.total, -1, self.d) if self.inplace else x.unflatten(1, (-1, self.d)) for x in self.was)
        ref, tol = self.turned(q)
        got = self.out.view(self.total, self.hq, self.d)
        assert bool(((got.double() - ref).abs() <= tol)[:new].all())
        assert torch.equal(got[new:], (self.was[0].view_as(got) if self.inplace else torch.full_like(got, 7.0))[new:])
        ref, tol = self.turned(k)
        moved = torch.zeros(self.caches[0].shape[0], dtype=torch.bool, device="cuda")
        for b, (n, kv) in enumerate(self.lens):
            skip = max(0, n - kv)
            if n == skip:
                continue
            rows, to = slice(int(self.starts[b]) + skip, int(self.starts[b]) + n), slice(int(self.bounds[b]) + kv - n + skip, int(self.bounds[b]) + kv)
            moved[to] = True
            assert bool(((self.caches[0][to].double() - ref[rows]).abs() <= tol[rows]).all()), (b, n, kv)
            assert torch.equal(self.caches[1][to], v[rows].contiguous()), (b, n, kv)
        for c, was in zip(self.caches, self.before):
            assert torch.equal(c[~moved], was[~moved])


LENS = [(3, 17), (0, 4), (20, 20), (1, 300), (5, 3), (2, 0), (1, 1), (70, 90)]
FLAGS = [0, xa.XATTN_ROPE_PAIRS, xa.XATTN_ROPE_DEALT, xa.XATTN_ROPE_PAIRS | xa.XATTN_ROPE_DEALT]


@pytest.mark.parametrize("flags", FLAGS)
@pytest.mark.parametrize("sections", [[64], [16, 24, 24], [0, 40, 24], [10, 22, 22, 10], [20, 12], [8], [24, 0, 0]], ids=str)
def test_axes(sections, flags):
    b = Batch(LENS, 8, 2, 128, sections, flags, extra=3, seed=len(sections))
    b.call()
    b.check()


@pytest.mark.parametrize("flags", FLAGS[:2])
@pytest.mark.parametrize("d,sections", [(16, [8]), (64, [32]), (64, [8, 4, 4]), (80, [20, 20]), (96, [48]), (256, [128]), (256, [32, 64, 24]), (128, [0])], ids=str)
def test_head_sizes(d, sections, flags):
    b = Batch(LENS, 5, 1, d, sections, flags, extra=1, pad=8, seed=d)
    b.call()
    b.check()


@pytest.mark.parametrize("far", [-2 ** 31 + 60, 1000000, 2 ** 31 - 6000])
def test_far_positions(far):
    b = Batch(LENS, 4, 4, 128, [16, 24, 24], far=far, seed=3)
    b.call()
    b.check()


@pytest.mark.parametrize("hq,hkv", [(1, 1), (40, 8), (64, 8), (7, 1)])
def test_heads_and_many_rows(hq, hkv):
    b = Batch([(1, 1 + i % 50) for i in range(200)] + [(1500, 1600), (3, 3)], hq, hkv, 128, [64], seed=hq)
    b.call()
    b.check()


@pytest.mark.parametrize("d,hq,hkv", [(16, 40, 4), (80, 6, 3), (80, 24, 4), (96, 64, 16), (256, 6, 2), (256, 30, 10)])
def test_rows_of_many_sizes(d, hq, hkv):
    """Rows with little and with much to move, enough of them that several may share a workgroup, the last ones alone in theirs."""
    b = Batch([(1, 1 + i % 9) for i in range(100)] + [(1001, 1300), (2, 2)], hq, hkv, d, [8 * (d // 32), 8 * (d // 16 - d // 32)], seed=d + hq)
    b.call()
    b.check()


def test_batches():
    for batch in (64, 65, 1000, 4096):
        b = Batch([((i * 7) % 4, (i * 7) % 4 + i % 5) for i in range(batch)], 2, 1, 128, [64], extra=5, seed=batch)
        b.call()
        b.check()


def test_in_place():
    b = Batch(LENS, 8, 2, 128, [16, 24, 24], extra=2, seed=4, inplace=True)
    b.call()
    b.check()


def test_bounds_that_do_not_ascend():
    b = Batch([(3, 17), (20, 40), (9, 9)], 4, 2, 128, [64], seed=5)
    for starts in ([5, 1, 0, 32], [-9, -5, -1, -1], [40, 50, 60, 70]):
        b.q_starts.copy_(torch.tensor(starts, dtype=torch.int32))
        b.kv_lens.fill_(0)                      # nothing is written to the ranges
        b.call()
    b.q_starts.copy_(torch.tensor(b.starts, dtype=torch.int32))
    b.kv_lens.copy_(torch.tensor([17, 40, 9], dtype=torch.int32))
    b.call()
    b.check()


def test_lengths_below_the_new_rows():
    """Down to the least there is: the rows are turned, and not written to the ranges."""
    b = Batch([(3, 17), (20, 40), (9, 9)], 4, 2, 128, [64], seed=8)
    for lens in ([-1, 0, 8], [-2 ** 31, -2 ** 31 + 5, -7]):
        b.kv_lens.copy_(torch.tensor(lens, dtype=torch.int32))
        b.call()
        torch.cuda.synchronize()
        moved = int((b.caches[0] != b.before[0]).any(-1).any(-1).sum())
        assert moved == (8 if lens[2] == 8 else 0)
        for c, was in zip(b.caches, b.before):
            c.copy_(was)
        b.out.fill_(7)
    b.kv_lens.copy_(torch.tensor([17, 40, 9], dtype=torch.int32))
    b.call()
    b.check()


def test_no_rotation_is_write_kvcache():
    """Positions of 0: the same as the plain append, on another batch shape."""
    b = Batch([(2, 9), (2, 30), (2, 2)], 4, 2, 128, [64], seed=6)
    b.pos.zero_()
    b.call()
    b.check()
    k, v = b.k_new.contiguous(), b.v_new.contiguous()
    appended = [c.clone() for c in b.before]
    ptrs = [torch.tensor([c.data_ptr() + int(x) * 2 * 128 * 2 for x in b.bounds[:-1]], dtype=torch.int64, device="cuda") for c in appended]
    xa.xattn_write_kvcache(k, v, ptrs[0], ptrs[1], b.kv_lens, 3, 2, 2, 128, torch.cuda.current_stream())
    torch.cuda.synchronize()
    assert torch.equal(b.caches[0], appended[0]) and torch.equal(b.caches[1], appended[1])


def test_graph_replays():
    b = Batch(LENS, 8, 2, 128, [16, 24, 24], seed=7)
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        b.call(torch.cuda.current_stream())
    for add in (0, 11, 100000):
        b.pos += add
        for c, was in zip(b.caches, b.before):
            c.copy_(was)
        b.out.fill_(7)
        torch.cuda.synchronize()
        graph.replay()
        b.check()
