"""Every key counts in xattn_prefill: rows whose softmax rests on a key of their own, at places where a key could get lost.

A row's key is a multiple of its query, so that its score exceeds what all the other keys have together, and its value is like no other's: a
row that misses it, or reads it from another place, has an output that is off by the order of 1.  What a result may be off by, with A = sum_j
p_j |v_j| and u = 2^-24: 2^-8 |out| for its rounding, 2^-8 A for the weights', twice what the scores are off by (128 products summed in fp32,
and 2^-22 of a score in the exponent) relative to A, and u of A per addition that a sum passes through: the keys of a part, at most
max(512, 1.002 kv tiles / 512) + 64 of them, and 1024 parts.
"""
import math

import pytest
import torch

import paper_2510_14686_amd as xa
from test_gpu_prefill import D, call, make

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
SCALE = 1 / math.sqrt(D)
SCORE = 26.0


def mark(s, b, rows, keys, h):
    """Row rows[i] (of sequence b, query head h) rests on key keys[i]."""
    q = s["q"][int(s["starts"][b]) + rows, h].float()
    group = s["hq"] // s["hkv"]
    s["k"][b][keys, h // group] = (q * (SCORE / SCALE / q.square().sum(1, keepdim=True))).bfloat16()
    g = torch.Generator(device="cuda")
    g.manual_seed(h + 1)
    s["v"][b][keys, h // group] = torch.randn((len(keys), D), generator=g, device="cuda").mul_(2).bfloat16()


def check(s, b, heads, keys_of):
    """keys_of[h]: the key that each row of head h rests on."""
    torch.cuda.synchronize()
    (n, kv), group = s["lens"][b], s["hq"] // s["hkv"]
    rows = slice(int(s["starts"][b]), int(s["starts"][b]) + n)
    tiles = sum((m * group + 127) // 128 for m, _ in s["lens"]) * s["hkv"]
    n_adds = max(512, 1.002 * kv * tiles / 512) + 64 + 1024
    seen = torch.arange(kv, device="cuda")[None] < (kv - n + 1 + torch.arange(n, device="cuda"))[:, None]
    for h in heads:
        q, k, v = s["q"][rows, h].double(), s["k"][b][:, h // group].double(), s["v"][b][:, h // group].double()
        x = ((q @ k.t().contiguous()) * SCALE).masked_fill(~seen, -math.inf)
        off = (q.abs() @ k.abs().t().contiguous() * SCALE).masked_fill(~seen, 0.0).amax(1) * (D * U + 2.0 ** -22)
        lse = torch.logsumexp(x, 1)
        p = torch.exp(x - lse[:, None])
        rest = p.gather(1, keys_of[h][:, None])[:, 0]
        assert bool((rest > 0.5).all()), "a row does not rest on its key"
        ref, a = p @ v, p @ v.abs()
        tol = 2.0 ** -8 * ref.abs() + a * (2.0 ** -8 + 2 * off[:, None] + n_adds * U) * (1 + 2.0 ** -7)
        wrong = ((s["out"][rows, h].double() - ref).abs() > tol).any(1).nonzero()[:, 0]
        assert len(wrong) == 0, "head %d: rows %s, which rest on keys %s" % (h, wrong[:8].tolist(), keys_of[h][wrong[:8]].tolist())
        far = (s["lse"][rows, h].double() - lse).abs() - off - n_adds * U - 2.0 ** -22 * (1 + lse.abs())
        assert far.max().item() <= 0, "head %d: lse" % h
        # What would be seen: without a row's key the output is far outside.
        lost = (p * (torch.arange(kv, device="cuda")[None] != keys_of[h][:, None])) @ v
        assert bool(((lost - ref).abs() > 8 * tol).any(1).all()), "a key that got lost would not show"


def spread(n, kv, count, seed):
    """`count` different keys that every row sees: of each stretch of kv / count keys one, in an order that rows and keys do not share."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    last = kv - n + 1
    at = torch.arange(count, device="cuda") * last // count
    width = (torch.arange(1, count + 1, device="cuda") * last // count - at).clamp_(min=1)
    keys = at + (torch.rand(count, generator=g, device="cuda") * width).long().clamp_(max=width - 1)
    return keys[torch.randperm(count, generator=g, device="cuda")]


@pytest.mark.parametrize("n,kv,hq,hkv", [(130, 16384, 8, 1), (700, 12345, 2, 1), (40, 20000, 8, 2), (16, 9001, 8, 8), (1000, 3001, 1, 1), (300, 1024, 6, 3)])
def test_a_key_of_its_own_for_every_row(n, kv, hq, hkv):
    """Long sequences in parts, one half block of keys after the other; a group's heads share their keys' places."""
    s = make([(3, 30), (n, kv), (1, 5)], hq, hkv, seed=kv)
    group, keys_of = hq // hkv, {}
    for g in range(hkv):
        keys = spread(n, kv, n * group, seed=g)
        for j in range(group):
            h = g * group + j
            keys_of[h] = keys[j::group].contiguous()
            mark(s, 1, torch.arange(n, device="cuda"), keys_of[h], h)
    call(s)
    check(s, 1, range(hq), keys_of)


@pytest.mark.parametrize("kv", [1, 31, 32, 33, 63, 64, 65, 96, 127, 128, 129, 511, 512, 513, 1000, 4097, 33000])
@pytest.mark.parametrize("last", [0, 1, 2])
def test_the_first_and_the_last_key_of_a_token(kv, last):
    """One new token per sequence, whose heads rest on the first key, on the last one, and on those around the middle."""
    s = make([(1, kv)] * 3, 8, 8, seed=kv)
    keys_of = {}
    for h in range(8):
        keys_of[h] = torch.tensor([[0, kv - 1, kv // 2, kv // 2 - 1, kv - 2, 1, (kv - 1) // 32 * 32, (kv - 1) // 64 * 64][h] % kv], device="cuda")
        mark(s, last, torch.zeros(1, dtype=torch.long, device="cuda"), keys_of[h], h)
    call(s)
    check(s, last, range(8), keys_of)


def test_keys_behind_4_gib_of_a_sequence():
    """K and V of 16 heads and 1200000 tokens, 4.9 GB each: what lies 4 GiB further on, and where it would wrap to."""
    hq, hkv, kv = 16, 16, 1200000
    wrap = (4 << 30) // (hkv * D * 2)
    s = make([(1, 1)], hq, hkv, seed=19)
    k = torch.empty((kv, hkv, D), dtype=torch.bfloat16, device="cuda").normal_()
    v = torch.empty_like(k).normal_()
    s["lens"], s["k"], s["v"] = [(1, kv)], [k], [v]
    s["k_ptrs"][0], s["v_ptrs"][0], s["kv_lens"][0] = k.data_ptr(), v.data_ptr(), kv
    keys_of = {}
    at = [wrap, wrap + 1, wrap - 1, kv - 1, wrap + 31, wrap + 32, wrap + 63, wrap + 64, wrap // 2, wrap // 2 - 1, wrap + 70001, kv - 64, kv - 65, 0, 17, wrap + 17]
    for h in range(hq):
        keys_of[h] = torch.tensor([at[h]], device="cuda")
        mark(s, 0, torch.zeros(1, dtype=torch.long, device="cuda"), keys_of[h], h)
    call(s)
    check(s, 0, range(hq), keys_of)
