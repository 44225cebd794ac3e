"""Rows into and out of a cache of 4 bits a value (xattn_rope_kvcache_mx, xattn_read_kvcache_mx) against the definition in 64 bits.

Codes and scales are compared bit for bit: both sides rotate K in double (off by 2^-50 of a value, an angle's rounded product and all), and a
value that lies that near to a border between two codes does not come up in 10^6 random ones.  q as in test_gpu_rope.py: one rounding to
bf16 (2^-8 of it), 2^-21 of its two values for sine, cosine and products.
"""
import numpy as np
import pytest
import torch

import mx_util
import paper_2510_14686_amd as xa

pytestmark = pytest.mark.gpu
D = 128


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
    def __init__(self, lens, hq, hkv, sections, flags=0, far=0, extra=0, pad=0, seed=0, inplace=False):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        self.lens, self.hq, self.hkv, self.sections, self.flags = lens, hq, hkv, sections, flags
        self.starts = np.concatenate([[0], np.cumsum([n for n, _ in lens])])
        self.total = int(self.starts[-1]) + extra
        width = (hq + 2 * hkv) * D + pad
        self.qkv = torch.randn((self.total, width), generator=g, device="cuda").bfloat16()
        if inplace:
            self.q, self.k_new, self.v_new = (torch.randn((self.total, h * D), generator=g, device="cuda").bfloat16() for h in (hq, hkv, hkv))
        else:
            self.q, self.k_new, self.v_new = self.qkv[:, :hq * D], self.qkv[:, hq * D:(hq + hkv) * D], self.qkv[:, (hq + hkv) * D:(hq + 2 * hkv) * D]
        f = sum(sections)
        self.pos = torch.randint(-50, 5000, (len(sections), self.total), generator=g, device="cuda", dtype=torch.int32) + far
        self.inv_freq = (1e4 ** (-torch.arange(f, dtype=torch.float64) / max(f, 1))).float().cuda()
        self.ranges = mx_util.Ranges([max(kv, 0) for _, kv in lens], hkv, g=g)
        self.before = [[c.clone() for c in side] for side in self.ranges.caches]
        self.q_starts = torch.tensor(self.starts, dtype=torch.int32, device="cuda")
        self.kv_lens = torch.tensor([kv for _, kv in lens], dtype=torch.int32, device="cuda")
        self.inplace = inplace
        self.out = self.q if inplace else torch.full((self.total, hq, D), 7.0, dtype=torch.bfloat16, device="cuda")
        self.was = [x.clone() for x in (self.q, self.k_new, self.v_new)]

    def call(self, stream=None):
        xa.xattn_rope_kvcache_mx(self.q, self.k_new, self.v_new, self.q.stride(0), self.k_new.stride(0), self.v_new.stride(0), self.pos,
                                 self.inv_freq if sum(self.sections) else None, self.sections, self.flags, *self.ranges.ptrs, self.q_starts, self.kv_lens,
                                 len(self.lens), self.total, self.hq, self.hkv, D, self.out, stream or torch.cuda.current_stream())

    def turned(self, x):
        """(rotated heads in 64 bits, how far off they may be in bf16) of [rows, heads, 128]."""
        x, f = x.double(), sum(self.sections)
        axes = torch.tensor(axis_list(self.sections, self.flags & xa.XATTN_ROPE_DEALT), device="cuda", dtype=torch.long)
        a = (self.pos.double()[axes].t() * self.inv_freq.double())[:, None] if f else torch.zeros((x.shape[0], 1, 0), device="cuda", dtype=torch.float64)
        at = (slice(0, 2 * f, 2), slice(1, 2 * f, 2)) if self.flags & xa.XATTN_ROPE_PAIRS else (slice(0, f), slice(f, 2 * f))
        u, v = x[..., at[0]], x[..., at[1]]
        out, tol = x.clone(), torch.zeros_like(x)
        out[..., at[0]], out[..., at[1]] = u * a.cos() - v * a.sin(), v * a.cos() + u * a.sin()
        for i in at:
            tol[..., i] = 2.0 ** -8 * out[..., i].abs() + 2.0 ** -21 * (u.abs() + v.abs())
        return out, tol

    def check(self):
        torch.cuda.synchronize()
        new = int(self.starts[-1])
        q, k, v = (x.view(self.total, -1, D) if self.inplace else x.unflatten(1, (-1, D)) for x in self.was)
        ref, tol = self.turned(q)
        got = self.out.view(self.total, self.hq, D)
        assert bool(((got.double() - ref).abs() <= tol)[:new].all())
        assert torch.equal(got[new:], (self.was[0].view_as(got) if self.inplace else torch.full_like(got, 7.0))[new:])
        for which, x in enumerate((self.turned(k)[0], v.double())):
            codes, scales = mx_util.encode(x)
            for b, (n, kv) in enumerate(self.lens):
                want, skip = self.before[which][b].clone(), max(0, n - kv)
                rows = slice(int(self.starts[b]) + skip, int(self.starts[b]) + n)
                if n > skip:
                    mx_util.put(want, torch.arange(kv - n + skip, kv, device="cuda"), self.hkv, which == 1, codes[rows], scales[rows])
                assert torch.equal(self.ranges.caches[which][b], want), (which, b, n, kv)


LENS = [(3, 17), (0, 4), (20, 20), (1, 300), (5, 3), (2, 0), (1, 1), (70, 90), (64, 128), (65, 65)]
FLAGS = [0, xa.XATTN_ROPE_PAIRS, xa.XATTN_ROPE_DEALT, xa.XATTN_ROPE_PAIRS | xa.XATTN_ROPE_DEALT]


@pytest.mark.parametrize("flags", FLAGS)
@pytest.mark.parametrize("sections", [[64], [16, 24, 24], [0, 40, 24], [10, 22, 22, 10], [20, 12], [8], [24, 0, 0], [0], [40]], ids=str)
def test_append(sections, flags):
    b = Batch(LENS, 8, 2, sections, flags, extra=3, seed=len(sections))
    b.call()
    b.check()


@pytest.mark.parametrize("far", [-2 ** 31 + 60, 1000000, 2 ** 31 - 6000])
def test_far_positions(far):
    b = Batch(LENS, 4, 4, [16, 24, 24], far=far, seed=3)
    b.call()
    b.check()


@pytest.mark.parametrize("hq,hkv", [(1, 1), (40, 8), (64, 8), (7, 1), (6, 3)])
def test_heads_and_many_rows(hq, hkv):
    b = Batch([(1, 1 + i % 50) for i in range(200)] + [(1500, 1600), (3, 3)], hq, hkv, [64], seed=hq, pad=8)
    b.call()
    b.check()


@pytest.mark.parametrize("batch", [64, 65, 1000, 4096])
def test_batches(batch):
    b = Batch([((i * 7) % 4, (i * 7) % 4 + i % 5) for i in range(batch)], 2, 1, [64], extra=5, seed=batch)
    b.call()
    b.check()


def test_in_place():
    b = Batch(LENS, 8, 2, [16, 24, 24], extra=2, seed=4, inplace=True)
    b.call()
    b.check()


def test_bounds_that_do_not_ascend_and_lengths_below_the_new_rows():
    b = Batch([(3, 17), (20, 40), (9, 9)], 4, 2, [64], seed=5)
    for starts in ([5, 1, 0, 32], [-9, -5, -1, -1], [40, 50, 60, 70]):
        b.q_starts.copy_(torch.tensor(starts, dtype=torch.int32))
        b.kv_lens.fill_(0)                      # nothing is written to the ranges
        b.call()
    b.q_starts.copy_(torch.tensor(b.starts, dtype=torch.int32))
    for lens in ([-1, 0, -2], [-2 ** 31, -2 ** 31 + 5, -7]):
        b.kv_lens.copy_(torch.tensor(lens, dtype=torch.int32))
        b.call()
        torch.cuda.synchronize()
        for side, was in zip(b.ranges.caches, b.before):
            for c, w in zip(side, was):
                assert torch.equal(c, w)
    b.kv_lens.copy_(torch.tensor([17, 40, 9], dtype=torch.int32))
    b.call()
    b.check()


def test_values_of_every_size():
    """Zeros, the least and the largest values, infinities and NaN, values on the borders between codes; positions of 0."""
    b = Batch([(40, 50)], 2, 2, [64], seed=6)
    b.pos.zero_()
    k, v = (x.unflatten(1, (-1, D)) for x in (b.k_new, b.v_new))
    for x in (k, v):
        x[0] = 0.0
        x[1] = -0.0
        x[2] *= 2.0 ** -126
        x[3] *= 2.0 ** -130
        x[4] *= 2.0 ** 124
        x[5] = 3.3895e38
        x[6, :, 7] = float("inf")
        x[7, :, 40] = float("nan")
        x[8, :, 99] = -float("inf")
        borders = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 7.0, 6.0, 0.0, 4.0, -0.25, -0.75, -1.25, -2.5, -5.0], device="cuda").bfloat16()
        for i in range(9, 25):
            x[i] = borders.repeat(8) * 2.0 ** (i - 15)
        x[25, :, ::2] *= 1e-3
    b.was = [x.clone() for x in (b.q, b.k_new, b.v_new)]
    b.call()
    torch.cuda.synchronize()
    for which, x in enumerate((b.turned(k)[0], v)):      # an infinity that is turned by 0 makes NaN of its pair's other value, too
        got_c, got_s = mx_util.get(b.ranges.caches[which][0], torch.arange(10, 50, device="cuda"), 2, which == 1)
        code, scale = mx_util.encode(x.double())
        assert torch.equal(got_s, scale.int())
        fine = (scale != 255).repeat_interleave(32, -1)
        assert torch.equal(got_c[fine], code[fine])


def test_strides_and_another_stream():
    b = Batch(LENS, 8, 2, [64], seed=8, pad=72)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    b.call(s)
    s.synchronize()
    b.check()


# ---------------------------------------------------------------------------------- reading rows back
def read(ranges, q_lens, kv_lens, heads, extra=0, stream=None):
    starts = np.concatenate([[0], np.cumsum(q_lens)])
    total = int(starts[-1]) + extra
    out = [torch.full((total, heads, D), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    xa.xattn_read_kvcache_mx(*ranges.ptrs, torch.tensor(starts, dtype=torch.int32, device="cuda"), torch.tensor(kv_lens, dtype=torch.int32, device="cuda"),
                             len(q_lens), total, heads, D, *out, stream or torch.cuda.current_stream())
    torch.cuda.synchronize()
    return starts, out


@pytest.mark.parametrize("heads", [1, 2, 8, 5])
def test_read(heads):
    g = torch.Generator(device="cuda")
    g.manual_seed(heads)
    kv = [17, 4, 20, 300, 3, 0, 1, 1000, 64, 65, 128]
    q = [3, 0, 20, 300, 5, 2, 1, 77, 64, 1, 128]
    ranges = mx_util.Ranges(kv, heads, g=g)
    for side in ranges.caches:      # any codes; scales that bf16 holds, a NaN here and there
        for c in side:
            scale = c.view(-1, mx_util.TILE_BYTES)[:, mx_util.CODES:]
            scale.copy_(torch.where(scale == 255, scale, 2 + scale % 250))
    starts, out = read(ranges, q, kv, heads, extra=9)
    for which in range(2):
        for b, (n, total) in enumerate(zip(q, kv)):
            got = out[which][int(starts[b]):int(starts[b + 1])].double()
            want = torch.zeros((n, heads, D), dtype=torch.float64, device="cuda")
            if min(n, total):
                want[n - min(n, total):] = ranges.values(which, b)[total - min(n, total):]
            assert torch.equal(got.isnan(), want.isnan()) and torch.equal(got.nan_to_num(0.0), want.nan_to_num(0.0)), (which, b)
        assert (out[which][int(starts[-1]):] == 7).all()


@pytest.mark.parametrize("batch", [64, 65, 1000, 4096])
def test_read_batches(batch):
    g = torch.Generator(device="cuda")
    g.manual_seed(batch)
    kv = [(i * 5) % 7 for i in range(batch)]
    q = [min(k, i % 4) for i, k in enumerate(kv)]
    rows = [[torch.randn((k, 2, D), generator=g, device="cuda") for k in kv] for _ in range(2)]
    ranges = mx_util.Ranges(kv, 2, fill=255, rows=rows)
    starts, out = read(ranges, q, kv, 2, extra=1)
    for which in range(2):
        want = torch.cat([mx_util.decode(*mx_util.encode(rows[which][b][kv[b] - n:])) for b, n in enumerate(q) if n])
        assert torch.equal(out[which][:int(starts[-1])].double(), want)
        assert (out[which][int(starts[-1]):] == 7).all()


@pytest.mark.parametrize("heads,lens", [(8, [2040]), (8, [2041]), (8, [1500, 0, 9, 3001, 70]), (1, [16375, 1]), (1, [16376, 1]), (5, [3268, 1, 1])], ids=str)
def test_read_of_eight_megabytes_and_around(heads, lens):
    g = torch.Generator(device="cuda")
    g.manual_seed(sum(lens))
    ranges = mx_util.Ranges(lens, heads, rows=[[torch.randn((n, heads, D), generator=g, device="cuda") for n in lens] for _ in range(2)])
    starts, out = read(ranges, lens, lens, heads, extra=7)
    for which in range(2):
        for b, n in enumerate(lens):
            assert torch.equal(out[which][int(starts[b]):int(starts[b + 1])].double(), ranges.values(which, b)[:n]), (which, b)
        assert (out[which][int(starts[-1]):] == 7).all()


def test_what_was_appended_is_read():
    """A prompt in two chunks and a single token, through both operators; the rows are those that the definition stores."""
    chunks = [70, 130, 1]
    g = torch.Generator(device="cuda")
    g.manual_seed(9)
    ranges = mx_util.Ranges([sum(chunks)], 2, fill=255)
    have, every = 0, []
    freq = torch.ones(64, device="cuda")
    for n in chunks:
        have += n
        x = torch.randn((n, 8 * D), generator=g, device="cuda").bfloat16()
        starts, lens = torch.tensor([0, n], dtype=torch.int32, device="cuda"), torch.tensor([have], dtype=torch.int32, device="cuda")
        pos = torch.zeros((1, n), dtype=torch.int32, device="cuda")
        xa.xattn_rope_kvcache_mx(x, x[:, 4 * D:], x[:, 6 * D:], 8 * D, 8 * D, 8 * D, pos, freq, [64], 0, *ranges.ptrs, starts, lens, 1, n, 4, 2, D,
                                 torch.empty((n, 4, D), dtype=torch.bfloat16, device="cuda"), torch.cuda.current_stream())
        every.append(x)
    _, out = read(ranges, [have], [have], 2)
    x = torch.cat(every)
    for which, first in ((0, 4), (1, 6)):
        assert torch.equal(out[which].double(), mx_util.decode(*mx_util.encode(x[:, first * D:(first + 2) * D].reshape(-1, 2, D).double())))


def test_ranges_of_more_than_four_gigabytes():
    """The last token of a million, 64 heads: its tile lies behind 4 GiB of the range."""
    n, heads = 1000001, 64
    size = xa.xattn_mx_range_bytes(n, heads)
    assert size > 2 ** 32
    caches = [torch.zeros(size, dtype=torch.uint8, device="cuda") for _ in range(2)]
    ptrs = [torch.tensor([c.data_ptr()], dtype=torch.int64, device="cuda") for c in caches]
    x = torch.randn((3, 3 * heads * D), device="cuda").bfloat16()
    starts, lens = torch.tensor([0, 3], dtype=torch.int32, device="cuda"), torch.tensor([n], dtype=torch.int32, device="cuda")
    xa.xattn_rope_kvcache_mx(x, x[:, heads * D:], x[:, 2 * heads * D:], *[3 * heads * D] * 3, torch.zeros((1, 3), dtype=torch.int32, device="cuda"),
                             torch.ones(64, device="cuda"), [64], 0, *ptrs, starts, lens, 1, 3, heads, heads, D,
                             torch.empty((3, heads, D), dtype=torch.bfloat16, device="cuda"), torch.cuda.current_stream())
    out = [torch.empty((3, heads, D), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    xa.xattn_read_kvcache_mx(*ptrs, starts, lens, 1, 3, heads, D, *out, torch.cuda.current_stream())
    torch.cuda.synchronize()
    for which in range(2):
        want = mx_util.encode(x[:, (1 + which) * heads * D:(2 + which) * heads * D].reshape(3, heads, D).double())
        row = torch.arange(n - 3, n, device="cuda")
        got = mx_util.get(caches[which], row, heads, which == 1)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1].int())
        assert torch.equal(out[which].double(), mx_util.decode(*want))
        nonzero = int((caches[which].view(-1, heads * mx_util.TILE_BYTES).amax(1) > 0).sum())
        assert nonzero == len(set((row // 64).tolist()))


def test_the_largest_scales():
    """Scale bytes 252 and 253 with every code: 4 and 6 times 2^126 are past the largest bf16, all others exact."""
    lens = [130, 64]
    g = torch.Generator(device="cuda")
    g.manual_seed(10)
    ranges = mx_util.Ranges(lens, 2, g=g)
    for side in ranges.caches:
        for c in side:
            scale = c.view(-1, mx_util.TILE_BYTES)[:, mx_util.CODES:]
            scale.copy_(252 + scale % 2)
    starts, out = read(ranges, lens, lens, 2)
    for which in range(2):
        for b, n in enumerate(lens):
            want = ranges.values(which, b)
            assert int((want.abs() >= 2.0 ** 128).sum()) > 1000 and int((want.abs() == 1.5 * 2.0 ** 127).sum()) > 1000
            assert torch.equal(out[which][int(starts[b]):int(starts[b + 1])].double(), torch.where(want.abs() < 2.0 ** 128, want, want.sign() * torch.inf))


def test_the_largest_values_of_bf16():
    """Appended and read: from 1.75 * 2^127 on a value comes back infinite, below it is off by a quarter of 2^127 at most, half a step of its code."""
    b = Batch([(32, 32)], 2, 2, [0], seed=11)
    edge = torch.tensor([1.734375 * 2.0 ** 127, 1.75 * 2.0 ** 127, 1.7578125 * 2.0 ** 127, 3.3895e38, 2.0 ** 127, 1.5 * 2.0 ** 127, 0.0, 1.0], device="cuda", dtype=torch.float64)
    for x in (b.k_new, b.v_new):
        v = x.unflatten(1, (2, 4, 32))
        v[:4] = edge[:4].bfloat16()[:, None, None, None]
        v[4:8] = edge[4:8].bfloat16()[:, None, None, None]
        v[8:] = edge.bfloat16().repeat(4)
        v[16:] *= -1
    b.was = [x.clone() for x in (b.q, b.k_new, b.v_new)]
    b.call()
    b.check()
    _, out = read(b.ranges, [32], [32], 2)
    for which, x in enumerate((b.k_new, b.v_new)):
        x, got = x.unflatten(1, (2, D)).double(), out[which].double()
        beyond = x.abs().unflatten(-1, (4, 32)).amax(-1, keepdim=True) > 1.75 * 2.0 ** 127      # blocks of e = 126
        infinite = (beyond & (x.abs().unflatten(-1, (4, 32)) >= 1.75 * 2.0 ** 127)).flatten(-2)
        assert int(infinite.sum()) and torch.equal(got.isinf(), infinite) and torch.equal(got.sign()[infinite], x.sign()[infinite])
        assert ((got - x).abs()[~infinite] <= 2.0 ** 127 / 4).all()
