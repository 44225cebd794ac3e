"""How many bits xattn_prefill's softmax weights keep on their way into the product with V (XATTN_CFG_PV_MODE).

With weights of 24 bits a result may be off by, per element, with A = sum_j p_j |v_j| and u = 2^-24:
  2^-8 |out| for its rounding to bf16;
  what the scores are off by, `off`: 128 products summed in fp32, each step by u of the sum of magnitudes, and 2^-22 of a score in the exponent;
  twice that much relative to A, for the weight and its part of the sum; 8 u for the exponential, the division and the parts' joining;
  u of A for every addition: three products per key, and one to the sum.
One bf16 per weight adds 2^-8 A.
"""
import math

import pytest
import torch

import paper_2510_14686_amd as xa
from test_gpu_prefill import D, LENS, call, make

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
SCALE = 1 / math.sqrt(D)


@pytest.fixture(autouse=True)
def default_mode():
    yield
    torch.cuda.synchronize()
    xa.xattn_configure(xa.XATTN_CFG_PV_MODE, 0)


def worst(s, weight=0.0, scale=SCALE):
    """The largest excess of an error over what it may be, over the rows that see a key; a weight may be off by `weight` of it besides."""
    torch.cuda.synchronize()
    group, most = s["hq"] // s["hkv"], -math.inf
    for b, (n, kv) in enumerate(s["lens"]):
        if n == 0 or kv == 0:
            continue
        rows = slice(int(s["starts"][b]), int(s["starts"][b]) + n)
        seen = torch.arange(kv, device="cuda")[None] < (kv - n + 1 + torch.arange(n, device="cuda"))[:, None]
        ok = seen.any(1)
        for h in range(s["hq"]):
            q, k, v = s["q"][rows, h].double()[ok], s["k"][b][:, h // group].double(), s["v"][b][:, h // group].double()
            x = ((q @ k.t().contiguous()) * scale).masked_fill(~seen[ok], -math.inf)
            off = (q.abs() @ k.abs().t().contiguous() * abs(scale)).masked_fill(~seen[ok], 0.0).amax(1) * (D * U + 2.0 ** -22)
            p = torch.softmax(x, 1)
            ref, a = p @ v, p @ v.abs()
            tol = 2.0 ** -8 * ref.abs() + a * (weight + 2 * off[:, None] + 8 * U + 4 * kv * U) * (1 + 2.0 ** -7)
            most = max(most, ((s["out"][rows, h].double()[ok] - ref).abs() - tol).max().item())
    return most


# a tile each: up to 128 rows of a KV head
SHORT = [(1, 1), (1, 2), (3, 17), (1, 100), (20, 256), (1, 300), (7, 7), (5, 2), (16, 130), (1, 3000)]


@pytest.mark.parametrize("heads", [(8, 2), (4, 4), (5, 1), (40, 8), (16, 16)], ids=lambda h: "%dof%d" % h)
def test_sequences_of_one_tile(heads):
    s = make(SHORT, *heads, seed=40)
    xa.xattn_configure(xa.XATTN_CFG_PV_MODE, 1)
    call(s)
    assert worst(s) <= 0


@pytest.mark.parametrize("spread", [0.0, 4.0, 16.0])
def test_flat_and_peaked_rows_of_one_tile(spread):
    s = make([(20, 256), (1, 700), (9, 41)], 8, 2, seed=41, spread=spread)
    xa.xattn_configure(xa.XATTN_CFG_PV_MODE, 1)
    call(s)
    assert worst(s) <= 0


def test_one_tile_in_parts():
    """Long sequences of few rows, whose parts are put together by the merge."""
    s = make([(1, 9000), (3, 5001), (20, 4000)], 8, 2, seed=42)
    xa.xattn_configure(xa.XATTN_CFG_PV_MODE, 1)
    call(s)
    assert worst(s) <= 0


@pytest.mark.parametrize("lens", ["small", "edges", "odd", "long"])
@pytest.mark.parametrize("heads", [(8, 2), (5, 1), (16, 1)], ids=lambda h: "%dof%d" % h)
def test_prompts(lens, heads):
    s = make(LENS[lens], *heads, seed=43)
    xa.xattn_configure(xa.XATTN_CFG_PV_MODE, 1)
    call(s)
    assert worst(s) <= 0


@pytest.mark.parametrize("mode", [0, 2])
def test_one_bf16_per_weight(mode):
    s = make(LENS["long"] + LENS["edges"] + SHORT, 8, 2, seed=44)
    xa.xattn_configure(xa.XATTN_CFG_PV_MODE, mode)
    call(s)
    assert worst(s, 2.0 ** -8) <= 0
    assert worst(s) > 0      # (or nothing here tells the forms apart)


def test_the_mode_of_a_recorded_call_stays():
    """Also the sums, which do not depend on it, stay the same."""
    s = make(SHORT, 8, 2, seed=45)
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    call(s, stream=stream)
    torch.cuda.synchronize()
    lse = s["lse"].clone()
    xa.xattn_configure(xa.XATTN_CFG_PV_MODE, 1)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        call(s, stream=torch.cuda.current_stream())
    xa.xattn_configure(xa.XATTN_CFG_PV_MODE, 0)
    for _ in range(3):
        s["out"].fill_(3)
        s["lse"].fill_(3)
        torch.cuda.synchronize()
        graph.replay()
        assert worst(s) <= 0 and torch.equal(s["lse"], lse)
        call(s, stream=stream)
        assert worst(s) > 0


@pytest.mark.parametrize("q_len,hq,hkv", [(1, 32, 8), (4, 8, 2), (16, 4, 1)])
def test_as_near_as_decode(q_len, hq, hkv):
    """The same call through both operators: within the same bound."""
    s = make([(q_len, q_len + n) for n in (0, 1, 60, 500, 2000)], hq, hkv, seed=46)
    xa.xattn_configure(xa.XATTN_CFG_PV_MODE, 1)
    call(s)
    assert worst(s) <= 0
    xa.xattn_configure(xa.XATTN_CFG_PV_MODE, 0)
    xa.xattn_decode(s["q"], s["k_ptrs"], s["v_ptrs"], s["kv_lens"], s["batch"], q_len, hq, hkv, D, SCALE, s["out"], s["lse"], torch.cuda.current_stream())
    assert worst(s) <= 0
