"""Plain 64-bit reference of the 8-bit paged cache: planning by a loop, codes
from their bits, attention by dense products.  Test infrastructure only."""

import math

import torch

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}
FLOOR = 2.0 ** -60


def plan(lengths, added, table, ring, state, page):
    """(table, lengths, state, slots per unit) after the units, in order, took
    their pages; lengths [R, L, H] and added [R, L, H] on the CPU."""
    R, L, H = lengths.shape
    table = table.clone()
    head, count = state.tolist()
    used, slots = 0, []
    for r in range(R):
        for l in range(L):
            for h in range(H):
                n, a = int(lengths[r, l, h]), int(added[r, l, h])
                mine = []
                for x in range(n, n + a):
                    b = x // page
                    if x % page == 0:
                        table[r, l, h, b] = ring[(head + used) % len(ring)]
                        used += 1
                    mine.append(int(table[r, l, h, b]) * page + x % page)
                slots.append(mine)
    assert used <= count
    return (table, lengths + added,
            torch.tensor([(head + used) % len(ring), count - used], dtype=torch.int32), slots)


def value(codes, format):
    """What the codes stand for, in 64 bits."""
    b = codes.to(torch.int64)
    if format == "int8":
        return torch.where(b > 127, b - 256, b).double()
    e, m = b >> 3 & 15, (b & 7).double()
    power = (torch.where(e > 0, e - 10, e - 9) + 1023 << 52).view(torch.float64)
    x = torch.where(e > 0, 8 + m, m) * power
    x = torch.where((b & 127) == 127, float("nan"), x)
    return torch.where(b > 127, -x, x)


def scale_of(amax, format):
    """The scale of a page whose largest finite magnitude is amax (a number)."""
    if amax == 0:
        return FLOOR
    if format == "e4m3":
        e = -60
        while amax > 448 * 2.0 ** e:
            e += 1
        return 2.0 ** e
    m, e = math.frexp(amax / 127)  # m in [1/2, 1): eight bits are m 2^8
    return max(FLOOR, math.ldexp(math.ceil(m * 256), e - 8))


def rounded(y, format):
    """The value of the code nearest to y (ties to even), saturated."""
    if format == "int8":
        return torch.nan_to_num(y, nan=0.0, posinf=127, neginf=-127).round().clamp(-127, 127)
    e = torch.frexp(y.abs().clamp(2.0 ** -6, 448)).exponent.to(torch.int64)
    step = (e - 4 + 1023 << 52).view(torch.float64)
    return ((y.clamp(-448, 448) / step).round() * step).clamp(-448, 448)


class Pages:
    """Pages held as (scale, the values of their codes in units of it)."""

    def __init__(self, format, page, d):
        self.format, self.page, self.d, self.pages = format, page, d, {}

    def store(self, rows, slots):
        """One call's rows [n, d] of one page after the other, slots a list."""
        i = 0
        while i < len(slots):
            n = 1
            while (i + n < len(slots) and slots[i + n] == slots[i] + n
                   and slots[i + n] % self.page):
                n += 1
            self._run(rows[i:i + n].double(), *divmod(slots[i], self.page))
            i += n

    def _run(self, x, page, off):
        finite = x[torch.isfinite(x)]
        s = scale_of(float(finite.abs().max()) if finite.numel() else 0.0, self.format)
        old, code = self.pages.get(page, (0.0, None)) if off else (0.0, None)
        code = torch.full((self.page, self.d), float("nan"), dtype=torch.float64) \
            if code is None else code.clone()
        if off and s > old:
            code[:off] = rounded(code[:off] * old / s, self.format)
        s = max(s, old)
        code[off:off + len(x)] = rounded(x / s, self.format)
        self.pages[page] = (s, code)

    def load(self, slots):
        out = [self.pages[s // self.page][1][s % self.page] * self.pages[s // self.page][0]
               if s >= 0 else torch.zeros(self.d, dtype=torch.float64) for s in slots]
        return torch.stack(out)


def attend(q, k, v, seen, scale, v_scale):
    """One unit: q [G, a, d], k, v [n, d], v_scale [n] that of each token's
    page, seen [a] (how many positions each query sees), all in 64 bits.
    Returns out [G, a, d], lse [G, a], and what bounds errors: sum p |v| / sum
    p, the largest sum of |q k| scale, and the largest p v_scale / sum p."""
    x = torch.matmul(q, k.T) * scale
    hidden = torch.arange(k.shape[0], device=k.device) >= seen[:, None]
    x = x.masked_fill(hidden, float("-inf"))
    lse = torch.logsumexp(x, dim=-1) if k.shape[0] else x.new_full(x.shape[:2], float("-inf"))
    empty = (seen <= 0)[None, :, None]
    p = torch.where(empty, 0, torch.exp(x - lse[..., None]))
    size = torch.matmul(q.abs(), k.abs().T).masked_fill(hidden, 0) * scale
    most = size.amax(-1) if k.shape[0] else size.new_zeros(size.shape[:2])
    weight = (p * v_scale).amax(-1) if k.shape[0] else most
    return torch.matmul(p, v), lse, torch.matmul(p, v.abs()), most, weight
