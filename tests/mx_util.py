"""A cache of 4 bits a value in plain torch, 64 bits: from values to codes and tiles, and back."""
import torch

TILE, TILE_BYTES, CODES = 64, 4352, 4096
LEVELS = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


def encode(x):
    """(codes 0..15, scale bytes) of float64 [rows, heads, 128], by the definition: the least scale with all values within 7 times
    it; the nearest code, of two as near the even one."""
    blocks = x.double().unflatten(-1, (4, 32))
    most = blocks.abs().amax(-1)
    bad = ~torch.isfinite(blocks).all(-1)
    e = torch.full(most.shape, -125, dtype=torch.int32, device=x.device)
    for up in (64, 32, 16, 8, 4, 2, 1):      # the largest e whose 7 * 2^(e - 1) is still too small
        for _ in range(2):
            more = (e + up - 1).double()
            e = torch.where((most > 7.0 * torch.exp2(more)) & (e + up <= 126), e + up, e)
    y = blocks / torch.exp2(e.double())[..., None]
    a = y.abs()
    levels = torch.tensor(LEVELS, dtype=torch.float64, device=x.device)
    middle = (levels[1:] + levels[:-1]) / 2
    code = torch.zeros(a.shape, dtype=torch.int32, device=x.device)
    for i, m in enumerate(middle.tolist()):      # between codes i and i + 1
        code += (a > m) if i % 2 == 0 else (a >= m)
    code += 8 * torch.signbit(y).int()
    return code.flatten(-2), torch.where(bad, 255, e + 127)


def decode(codes, scales):
    """float64 values of codes [rows, heads, 128] and scale bytes [rows, heads, 4]."""
    levels = torch.tensor(LEVELS + [-v for v in LEVELS], dtype=torch.float64, device=codes.device)
    s = torch.exp2(scales.double() - 127)
    return (levels[codes.long()].unflatten(-1, (4, 32)) * torch.where(scales == 255, torch.nan, s)[..., None]).flatten(-2)


def places(row, heads, is_v):
    """(byte of each value [rows, heads, 128], byte of each scale [rows, heads, 4]) of tokens `row` in a range; a value is in the lower half of
    its byte if its index is even."""
    device = row.device
    t = (row % TILE)[:, None, None]
    base = ((row // TILE)[:, None] * heads + torch.arange(heads, device=device))[..., None] * TILE_BYTES
    s, u = t // 16, t % 16
    d, c = torch.arange(128, device=device), torch.arange(4, device=device)
    if is_v:
        return base + 1024 * s + 256 * (u // 4) + 16 * (d // 8) + 4 * (u % 4) + d % 8 // 2, base + CODES + 16 * (4 * (u // 4) + c) + 4 * s + u % 4
    return base + 1024 * s + 256 * (d // 32) + 16 * u + d % 32 // 2, base + CODES + 4 * (16 * c + u) + s


def put(cache, row, heads, is_v, codes, scales):
    """Writes tokens `row` into the range, a uint8 tensor."""
    at, at_scale = places(row, heads, is_v)
    cache[at[..., 0::2].flatten()] = (codes[..., 0::2] + 16 * codes[..., 1::2]).flatten().to(torch.uint8)
    cache[at_scale.flatten()] = scales.flatten().to(torch.uint8)


def get(cache, row, heads, is_v):
    at, at_scale = places(row, heads, is_v)
    byte = cache[at].int()
    return torch.where(torch.arange(128, device=cache.device) % 2 == 0, byte & 15, byte >> 4), cache[at_scale].int()


def tiles(length):
    return -(-length // TILE)


class Ranges:
    """K and V of a batch of sequences, each range in a buffer of its own with room for `room` tokens: what no row was written to is `fill`."""

    def __init__(self, lens, heads, fill=None, g=None, rows=None, device="cuda"):
        self.lens, self.heads = lens, heads
        self.caches = []
        for which in range(2):
            side = []
            for b, n in enumerate(lens):
                size = max(1, tiles(n)) * heads * TILE_BYTES
                c = torch.full((size,), fill, dtype=torch.uint8, device=device) if fill is not None else \
                    torch.randint(0, 256, (size,), generator=g, device=device, dtype=torch.int32).to(torch.uint8)
                if rows is not None and n:
                    put(c, torch.arange(n, device=device), heads, which == 1, *encode(rows[which][b].to(device)))
                side.append(c)
            self.caches.append(side)
        self.ptrs = [torch.tensor([c.data_ptr() for c in side], dtype=torch.int64, device=device) for side in self.caches]

    def values(self, which, b, upto=None):
        n = self.lens[b] if upto is None else upto
        return decode(*get(self.caches[which][b], torch.arange(n, device=self.caches[which][b].device), self.heads, which == 1))
