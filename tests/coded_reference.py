"""What rows in 8 bits hold, from the definition: a table of the e4m3 values and exact searches, one row after the other."""
import torch


def e4m3_values():
    """The 127 finite values of e4m3 without a sign, ascending; entry c is the value of code c."""
    v = [m / 8.0 * 2.0 ** -6 for m in range(8)] + [(1 + m / 8.0) * 2.0 ** (e - 7) for e in range(1, 16) for m in range(8)]
    return torch.tensor(v[:127], dtype=torch.float64)


def byte_of(top):
    """Scale bytes of largest magnitudes: the first power of two of which 448 times is no less."""
    powers = torch.tensor([2.0 ** k for k in range(-127, 129)], dtype=torch.float64, device=top.device)
    return torch.searchsorted(448.0 * powers, top.double().contiguous())


def unit_of(byte):
    return torch.tensor([2.0 ** k for k in range(-127, 129)], dtype=torch.float64, device=byte.device)[byte.long()]


def codes_of(x, unit):
    """Codes of x / unit, to the nearest, ties to the even code; what is not finite becomes NaN."""
    x = x.double()
    table = e4m3_values().to(x.device)
    y = (x / unit).abs()
    bad = ~torch.isfinite(y)
    y = torch.where(bad, torch.zeros_like(y), y)
    hi = torch.searchsorted(table, y.contiguous()).clamp(max=126)
    lo = (hi - 1).clamp(min=0)
    dl, dh = y - table[lo], table[hi] - y
    c = torch.where((dl < dh) | ((dl == dh) & (lo % 2 == 0)), lo, hi)
    c = torch.where(bad, torch.full_like(c, 127), c) | torch.where(torch.signbit(x) & ~bad, 128, 0)
    return c.to(torch.uint8)


def values_of(codes, unit):
    table = torch.cat([e4m3_values(), torch.full((1,), float("nan"), dtype=torch.float64)]).to(codes.device)
    v = table[(codes & 127).long()]
    return torch.where(codes >= 128, -v, v) * unit


def finite_top(x):
    """Largest finite magnitude over the last dimension."""
    x = x.double().abs()
    return torch.where(torch.isfinite(x), x, torch.zeros_like(x)).amax(-1)


class Store:
    """Codes [rows, heads, dim] and scale bytes [blocks, heads], as a write leaves them."""

    def __init__(self, rows, heads, dim, block, device="cuda"):
        self.rows, self.block, self.dim = rows, block, dim
        self.codes = torch.zeros(rows, heads, dim, dtype=torch.uint8, device=device)
        self.scales = torch.zeros((rows + block - 1) // block, heads, dtype=torch.uint8, device=device)

    def write(self, x, ids):
        last = {}
        for p, r in enumerate(ids):
            if 0 <= r < self.rows:
                last[r] = p
        blocks = {}
        for r, p in last.items():
            blocks.setdefault(r // self.block, []).append((r, p))
        for b, rows in blocks.items():
            first, end = b * self.block, min((b + 1) * self.block, self.rows)
            new = x[[p for _, p in rows]]
            need = byte_of(finite_top(new).amax(0)).to(torch.uint8)
            stays = [r for r in range(first, end) if r not in last]
            if stays:
                before = self.scales[b].clone()
                need = torch.maximum(need, before)
                old = values_of(self.codes[stays], unit_of(before)[None, :, None])
                kept = self.codes[stays]
                again = codes_of(old, unit_of(need)[None, :, None])
                again = torch.where((kept & 127) == 127, kept | 127, again)
                # a NaN keeps its code where nothing is requantised
                changed = (need != before)[None, :, None]
                again = torch.where((again & 127) == 127, torch.full_like(again, 127), again)
                self.codes[stays] = torch.where(changed, again, kept)
            self.scales[b] = need
            self.codes[[r for r, _ in rows]] = codes_of(new, unit_of(need)[None, :, None])

    def read(self, ids):
        out = torch.zeros(len(ids), self.codes.shape[1], self.dim, dtype=torch.float64, device=self.codes.device)
        for p, r in enumerate(ids):
            if 0 <= r < self.rows:
                out[p] = values_of(self.codes[r], unit_of(self.scales[r // self.block])[:, None])
        return out
