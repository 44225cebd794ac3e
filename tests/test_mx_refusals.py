"""Calls of the 4-bit cache's operators and of xbeam_verify that are refused before any GPU work (host code only)."""
import pytest

import paper_2510_14686_amd as xa
from paper_2510_14686_amd import binding

EINVAL, EUNSUPPORTED = binding.XATTN_EINVAL, binding.XATTN_EUNSUPPORTED
A = 4096                                # an address that is never looked at


def refused(status, fn, *args, **kw):
    with pytest.raises(xa.XattnError) as e:
        fn(*args, **kw)
    assert e.value.status == status and xa.xattn_last_error(), (args, kw, str(e.value))


def decode(q=A, k=A, v=A, lens=A, batch=2, q_len=1, hq=8, hkv=2, d=128, scale=0.1, out=A, lse=None):
    xa.xattn_decode_mx(q, k, v, lens, batch, q_len, hq, hkv, d, scale, out, lse)


@pytest.mark.parametrize("status,change", [
    *[(EINVAL, {n: None}) for n in ("q", "k", "v", "lens", "out")],
    (EINVAL, dict(batch=0)), (EINVAL, dict(q_len=0)), (EINVAL, dict(hq=0)), (EINVAL, dict(hkv=-2)), (EINVAL, dict(d=0)), (EINVAL, dict(scale=float("nan"))),
    (EINVAL, dict(scale=float("inf"))), (EINVAL, dict(scale=3e38)), (EINVAL, dict(scale=-3e38)), (EINVAL, dict(q=A + 8)), (EINVAL, dict(out=A + 2)),
    (EUNSUPPORTED, dict(batch=4097)), (EUNSUPPORTED, dict(q_len=17)), (EUNSUPPORTED, dict(hq=9)), (EUNSUPPORTED, dict(d=64)),
    (EUNSUPPORTED, dict(q_len=16, hq=40, hkv=8)), (EUNSUPPORTED, dict(hq=2048, hkv=1025)), (EUNSUPPORTED, dict(hq=1025, hkv=1025))], ids=str)
def test_decode(status, change):
    refused(status, decode, **change)


def rope(q=A, k=A, v=A, qs=1024, ks=256, vs=256, pos=A, freq=A, sections=(64,), flags=0, kp=A, vp=A, starts=A, lens=A, batch=2, total=9, hq=8, hkv=2, d=128,
         out=A):
    xa.xattn_rope_kvcache_mx(q, k, v, qs, ks, vs, pos, freq, sections, flags, kp, vp, starts, lens, batch, total, hq, hkv, d, out)


@pytest.mark.parametrize("status,change", [
    *[(EINVAL, {n: None}) for n in ("q", "k", "v", "pos", "freq", "kp", "vp", "starts", "lens", "out")],
    (EINVAL, dict(batch=0)), (EINVAL, dict(total=0)), (EINVAL, dict(hq=0)), (EINVAL, dict(d=0)), (EINVAL, dict(flags=4)), (EINVAL, dict(sections=(65,))),
    (EINVAL, dict(sections=(-8, 16))), (EINVAL, dict(qs=1016)), (EINVAL, dict(qs=1028)), (EINVAL, dict(q=A + 8)), (EINVAL, dict(k=A + 2)), (EINVAL, dict(v=A + 4)),
    (EINVAL, dict(out=A + 8)), (EINVAL, dict(q=A, out=A, qs=1536)), (EUNSUPPORTED, dict(sections=())), (EUNSUPPORTED, dict(sections=(63,))),
    (EUNSUPPORTED, dict(d=64, sections=(32,))), (EUNSUPPORTED, dict(d=256, qs=2048, ks=512, vs=512)), (EUNSUPPORTED, dict(batch=5000)),
    (EUNSUPPORTED, dict(total=2 ** 25)), (EUNSUPPORTED, dict(hkv=1025)), (EUNSUPPORTED, dict(qs=2 ** 33))], ids=str)
def test_rope(status, change):
    refused(status, rope, **change)


def read(kp=A, vp=A, starts=A, lens=A, batch=2, total=9, hkv=2, d=128, k=A, v=A):
    xa.xattn_read_kvcache_mx(kp, vp, starts, lens, batch, total, hkv, d, k, v)


@pytest.mark.parametrize("status,change", [
    *[(EINVAL, {n: None}) for n in ("kp", "vp", "starts", "lens", "k", "v")], (EINVAL, dict(batch=0)), (EINVAL, dict(total=0)), (EINVAL, dict(hkv=0)),
    (EINVAL, dict(d=-1)), (EINVAL, dict(k=A + 8)), (EINVAL, dict(v=A + 2)), (EUNSUPPORTED, dict(d=64)), (EUNSUPPORTED, dict(batch=4097)),
    (EUNSUPPORTED, dict(total=2 ** 24 + 1)), (EUNSUPPORTED, dict(hkv=1025)), (EUNSUPPORTED, dict(total=2 ** 24, hkv=128))], ids=str)
def test_read(status, change):
    refused(status, read, **change)


def verify(target=A, ts=1000, draft=A, ds=1000, dtype=0, vocab=1000, scale=1.0, dscale=1.0, drafted=A, counts=None, uniforms=A, batch=2, q_len=3, flags=0, tokens=A,
           accepted=A, lp=None):
    xa.xbeam_verify(target, ts, draft, ds, dtype, vocab, scale, dscale, drafted, counts, uniforms, batch, q_len, flags, tokens, accepted, lp)


@pytest.mark.parametrize("status,change", [
    *[(EINVAL, {n: None}) for n in ("target", "drafted", "uniforms", "tokens", "accepted")], (EINVAL, dict(batch=0)), (EINVAL, dict(q_len=0)), (EINVAL, dict(vocab=0)),
    (EINVAL, dict(dtype=3)), (EINVAL, dict(dtype=-1)), (EINVAL, dict(flags=2)), (EINVAL, dict(ts=999)), (EINVAL, dict(ds=999)), (EINVAL, dict(scale=0.0)),
    (EINVAL, dict(scale=-1.0)), (EINVAL, dict(scale=float("nan"))), (EINVAL, dict(dscale=0.0)), (EINVAL, dict(dscale=float("inf"))), (EINVAL, dict(target=A + 1)),
    (EINVAL, dict(draft=A + 1)), (EINVAL, dict(target=A + 2, dtype=2)), (EUNSUPPORTED, dict(batch=4097)), (EUNSUPPORTED, dict(q_len=17)),
    (EUNSUPPORTED, dict(vocab=2 ** 24 + 1, ts=2 ** 25, ds=2 ** 25)), (EUNSUPPORTED, dict(scale=2.0 ** 21)), (EUNSUPPORTED, dict(dscale=2.0 ** -21))], ids=str)
def test_verify(status, change):
    refused(status, verify, **change)


def test_arguments_that_are_no_numbers_or_tensors():
    for fn, bad in ((decode, dict(q="x")), (decode, dict(scale="x")), (rope, dict(pos=1.5)), (read, dict(k=0.5)), (verify, dict(scale=None)), (verify, dict(target="x"))):
        with pytest.raises(TypeError):
            fn(**bad)


def test_workspace_sizes():
    def up(x):
        return (x + 255) // 256 * 256

    for batch, q_len, hq, hkv, pieces in ((64, 1, 32, 8, 32), (1, 4, 8, 2, 128), (3, 16, 4, 1, 128), (3, 1, 64, 64, 8), (5, 1, 5, 5, 48)):
        slots, rows = pieces + batch, q_len * hq
        assert xa.xattn_decode_mx_workspace_bytes(batch, q_len, hq, hkv) == up(batch * 8) + up(slots * rows * 8) + up(slots * rows * 512)
    for args in ((0, 1, 8, 8), (1, 1, 8, 3), (1, 17, 8, 8), (4097, 1, 8, 8), (1, 1, 1025, 1025)):
        with pytest.raises(xa.XattnError):
            xa.xattn_decode_mx_workspace_bytes(*args)
    for batch, q_len, vocab in ((1, 1, 1), (1, 5, 131072), (64, 5, 131072), (4096, 16, 40), (4096, 16, 2 ** 24)):
        assert 256 <= xa.xbeam_verify_workspace_bytes(batch, q_len, vocab) <= 32 << 20
    for args in ((0, 1, 5), (1, 0, 5), (1, 1, 0), (4097, 1, 5), (1, 17, 5), (1, 1, 2 ** 24 + 1)):
        with pytest.raises(xa.XattnError):
            xa.xbeam_verify_workspace_bytes(*args)
