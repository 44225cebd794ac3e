"""The plain form of the 4-bit cache that the GPU tests compare with, against the format's own statements (no GPU)."""
import itertools

import pytest
import torch

import mx_util
import paper_2510_14686_amd as xa


def rows(values):
    x = torch.zeros((1, 1, 128), dtype=torch.float64)
    x.view(-1)[:len(values)] = torch.tensor(values, dtype=torch.float64)
    return x


def test_codes_are_nearest_and_ties_even():
    x = [7.0] + [v + d for v in (0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0) for d in (-1e-9, 0.0, 1e-9)]
    code, scale = mx_util.encode(rows(x))
    assert scale[0, 0, 0] == 127 and scale[0, 0, 1] == 2
    assert code[0, 0, :len(x)].tolist() == [7] + list(itertools.chain(*((i, i if i % 2 == 0 else i + 1, i + 1) for i in range(7))))


@pytest.mark.parametrize("most,e", [(7.0, 0), (7.0000001, 1), (3.5, -1), (3.6, 0), (1.0, -2), (0.876, -2), (0.875, -3), (7 * 2.0 ** 126, 126), (2.0 ** -125, -125), (0, -125)])
def test_scales(most, e):
    assert int(mx_util.encode(rows([0.0, -most]))[1][0, 0, 0]) == e + 127


def test_every_value_is_within_half_a_step():
    g = torch.Generator().manual_seed(0)
    x = torch.randn((200, 2, 128), generator=g, dtype=torch.float64) * torch.exp2(torch.randint(-20, 20, (200, 2, 1), generator=g).double())
    code, scale = mx_util.encode(x)
    back = mx_util.decode(code, scale)
    s = torch.exp2(scale.double() - 127)[..., None]
    a = (x.unflatten(-1, (4, 32)) / s).abs()
    step = torch.where(a <= 2, 0.5, torch.where(a <= 4, 1.0, 2.0))
    assert ((x - back).abs().unflatten(-1, (4, 32)) <= step / 2 * s).all()
    assert torch.equal(mx_util.encode(back)[0] % 8, code % 8) or ((mx_util.decode(*mx_util.encode(back)) - back) == 0).all()


@pytest.mark.parametrize("is_v", [False, True])
@pytest.mark.parametrize("heads", [1, 3])
def test_places_cover_a_tile_once(heads, is_v):
    at, scale = mx_util.places(torch.arange(128), heads, is_v)
    every = torch.cat((at[..., 0::2].flatten(), scale.flatten())).sort().values
    assert torch.equal(every, torch.arange(2 * heads * xa.XATTN_MX_TILE_BYTES))
    assert torch.equal(at[..., 0::2], at[..., 1::2])


def test_put_and_get():
    g = torch.Generator().manual_seed(1)
    x = torch.randn((70, 2, 128), generator=g)
    cache = torch.zeros(2 * 2 * xa.XATTN_MX_TILE_BYTES, dtype=torch.uint8)
    code, scale = mx_util.encode(x)
    for is_v in (False, True):
        mx_util.put(cache, torch.arange(70), 2, is_v, code, scale)
        c, s = mx_util.get(cache, torch.arange(70), 2, is_v)
        assert torch.equal(c, code) and torch.equal(s, scale)


def test_range_bytes():
    for tokens, heads, size in ((0, 8, 0), (1, 1, 4352), (64, 2, 8704), (65, 2, 17408), (2 ** 31 - 1, 1024, 2 ** 25 * 1024 * 4352)):
        assert xa.xattn_mx_range_bytes(tokens, heads) == size
    for args in ((-1, 8, 128), (5, 0, 128), (5, 8, 64), (5, 1025, 128), (2 ** 31, 8, 128)):
        with pytest.raises(xa.XattnError):
            xa.xattn_mx_range_bytes(*args)
