"""Calls of xattn_prefill, xattn_rope_kvcache and xbeam_logprobs that are refused before any GPU work (host code only)."""
import pytest

import paper_2510_14686_amd as xa
from paper_2510_14686_amd import binding

EINVAL, EUNSUPPORTED = binding.XATTN_EINVAL, binding.XATTN_EUNSUPPORTED
A = 4096                                # an address that is never looked at


def refused(status, fn, *args, **kw):
    with pytest.raises(xa.XattnError) as e:
        fn(*args, **kw)
    assert e.value.status == status and xa.xattn_last_error(), (args, kw, str(e.value))


def prefill(q=A, k=A, v=A, starts=A, lens=A, batch=2, total=9, hq=8, hkv=2, d=128, scale=0.1, out=A, lse=None):
    xa.xattn_prefill(q, k, v, starts, lens, batch, total, hq, hkv, d, scale, out, lse)


@pytest.mark.parametrize("status,change", [
    (EINVAL, dict(q=None)), (EINVAL, dict(k=None)), (EINVAL, dict(v=None)), (EINVAL, dict(starts=None)), (EINVAL, dict(lens=None)), (EINVAL, dict(out=None)),
    (EINVAL, dict(batch=0)), (EINVAL, dict(total=0)), (EINVAL, dict(total=-1)), (EINVAL, dict(hq=0)), (EINVAL, dict(hkv=-2)), (EINVAL, dict(d=0)),
    (EINVAL, dict(scale=float("nan"))), (EINVAL, dict(scale=float("inf"))), (EINVAL, dict(q=A + 8)), (EINVAL, dict(out=A + 2)),
    (EUNSUPPORTED, dict(batch=4097)), (EUNSUPPORTED, dict(total=2 ** 24 + 1)), (EUNSUPPORTED, dict(hq=9)), (EUNSUPPORTED, dict(d=64)),
    (EUNSUPPORTED, dict(hq=2048)), (EUNSUPPORTED, dict(total=2 ** 24, hq=128))], ids=str)
def test_prefill(status, change):
    refused(status, prefill, **change)


def rope(q=A, k=A, v=A, qs=1024, ks=256, vs=256, pos=A, freq=A, sections=(64,), flags=0, kp=A, vp=A, starts=A, lens=A, batch=2, total=9, hq=8, hkv=2, d=128,
         out=A):
    xa.xattn_rope_kvcache(q, k, v, qs, ks, vs, pos, freq, sections, flags, kp, vp, starts, lens, batch, total, hq, hkv, d, out)


@pytest.mark.parametrize("status,change", [
    *[(EINVAL, {n: None}) for n in ("q", "k", "v", "pos", "freq", "kp", "vp", "starts", "lens", "out")],
    (EINVAL, dict(batch=0)), (EINVAL, dict(total=0)), (EINVAL, dict(hq=0)), (EINVAL, dict(flags=4)), (EINVAL, dict(flags=-1)), (EINVAL, dict(sections=(65,))),
    (EINVAL, dict(sections=(40, 32))), (EINVAL, dict(sections=(-8, 16))), (EINVAL, dict(qs=1016)), (EINVAL, dict(ks=248)), (EINVAL, dict(vs=-256)),
    (EINVAL, dict(qs=1028)), (EINVAL, dict(q=A + 8)), (EINVAL, dict(k=A + 2)), (EINVAL, dict(v=A + 4)), (EINVAL, dict(out=A + 8)),
    (EUNSUPPORTED, dict(sections=())), (EUNSUPPORTED, dict(sections=(8,) * 5)), (EUNSUPPORTED, dict(sections=(63,))), (EUNSUPPORTED, dict(d=120)),
    (EUNSUPPORTED, dict(d=512)), (EUNSUPPORTED, dict(batch=5000)), (EUNSUPPORTED, dict(total=2 ** 25)), (EUNSUPPORTED, dict(hkv=1025)),
    (EUNSUPPORTED, dict(qs=2 ** 33))], ids=str)
def test_rope(status, change):
    refused(status, rope, **change)


def test_rope_in_place_on_rows_with_gaps():
    refused(EINVAL, rope, q=A, out=A, qs=1536)


def test_prefill_scale_that_overflows():
    refused(EINVAL, prefill, scale=3e38)
    refused(EINVAL, prefill, scale=-3e38)


def logprobs(logits=A, dtype=0, stride=1000, rows=3, vocab=1000, scale=1.0, tokens=A, k=4, lp=A, top=A, tok=A, lse=A, entropy=A):
    xa.xbeam_logprobs(logits, dtype, stride, rows, vocab, scale, tokens, k, lp, top, tok, lse, entropy)


@pytest.mark.parametrize("status,change", [
    (EINVAL, dict(logits=None)), (EINVAL, dict(dtype=3)), (EINVAL, dict(dtype=-1)), (EINVAL, dict(rows=0)), (EINVAL, dict(vocab=0)), (EINVAL, dict(stride=999)),
    (EINVAL, dict(scale=0.0)), (EINVAL, dict(scale=-1.0)), (EINVAL, dict(scale=float("nan"))), (EINVAL, dict(scale=float("inf"))), (EINVAL, dict(tokens=None)),
    (EINVAL, dict(lp=None)), (EINVAL, dict(k=-1)), (EINVAL, dict(k=1001)), (EINVAL, dict(k=0)), (EINVAL, dict(top=None)), (EINVAL, dict(tok=None)),
    (EINVAL, dict(logits=A + 1)), (EINVAL, dict(logits=A + 2, dtype=2)), (EINVAL, dict(tokens=None, lp=None, k=0, top=None, tok=None, lse=None, entropy=None)),
    (EUNSUPPORTED, dict(k=513)), (EUNSUPPORTED, dict(scale=2.0 ** 21)), (EUNSUPPORTED, dict(scale=2.0 ** -21)),
    (EUNSUPPORTED, dict(rows=2 ** 24 + 1)), (EUNSUPPORTED, dict(vocab=2 ** 24 + 1, stride=2 ** 25))], ids=str)
def test_logprobs(status, change):
    refused(status, logprobs, **change)


def test_logprobs_of_more_rows_than_a_launch_has_threads_for():
    refused(EUNSUPPORTED, logprobs, rows=2 ** 22 + 1)
    with pytest.raises(xa.XattnError):
        xa.xbeam_logprobs_workspace_bytes(2 ** 22 + 1, 1000, 0)


def test_arguments_that_are_no_numbers_or_tensors():
    for fn, bad in ((prefill, dict(q="x")), (prefill, dict(scale="x")), (rope, dict(pos=1.5)), (rope, dict(sections=(6.5,))), (logprobs, dict(scale=None))):
        with pytest.raises(TypeError):
            fn(**bad)


def test_workspace_sizes():
    for batch, total, hq, hkv in ((1, 1, 8, 8), (4, 55, 8, 2), (16, 40000, 32, 8)):
        rows = min(128, total * hq // hkv)
        ml = (1024 * rows * 8 + 255) // 256 * 256
        assert xa.xattn_prefill_workspace_bytes(batch, total, hq, hkv) == 16640 + ml + 1024 * rows * 512
    assert xa.xbeam_logprobs_workspace_bytes(4096, 131072, 5) == 256      # a workgroup per row
    for rows, vocab, k in ((1, 131072, 20), (3, 100003, 512), (200, 100003, 0)):
        n = xa.xbeam_logprobs_workspace_bytes(rows, vocab, k)
        assert 256 <= n <= 513 * (16 + 8 * k)
    for fn, args in ((xa.xattn_prefill_workspace_bytes, (0, 1, 8, 8)), (xa.xattn_prefill_workspace_bytes, (1, 1, 8, 3)),
                     (xa.xbeam_logprobs_workspace_bytes, (0, 1, 0)), (xa.xbeam_logprobs_workspace_bytes, (1, 10, 11))):
        with pytest.raises(xa.XattnError):
            fn(*args)
