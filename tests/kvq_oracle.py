"""Plain 64-bit statements of the 8-bit cache and of rotary positions, on the CPU, one block or token at a time."""
import math

import numpy as np
import torch

TOP = {"e4m3": 8, "e5m2": 15}
MANTISSA = {"e4m3": 3, "e5m2": 2}
LOWEST = {"e4m3": -6, "e5m2": -14}
CODES = {"e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}
DT = {"bf16": torch.bfloat16, "f16": torch.float16}


def most(dtype, code):
    """The largest element that both types have."""
    return (2.0 - 2.0 ** -MANTISSA[code]) * 2.0 ** (127 if dtype == torch.bfloat16 else 15)


def code_of(x, e, code):
    """x 2^-e rounded to the code's values, ties to even; what is not finite as the code holds it."""
    with np.errstate(invalid="ignore"):
        y = np.ldexp(x, -e)
        at = np.maximum(np.frexp(np.where(np.isfinite(y) & (y != 0), y, 1.0))[1] - 1, LOWEST[code]) - MANTISSA[code]
        r = np.ldexp(np.rint(np.ldexp(np.where(np.isfinite(y), y, 0.0), -at)), at)
        return np.where(np.isfinite(y), r, y if code == "e5m2" else np.nan)


def exponent_for(top, code):
    """Smallest e >= -126 with top <= 1.75 * 2^TOP * 2^e."""
    e = -126
    while top > 1.75 * 2.0 ** TOP[code] * 2.0 ** e:
        e += 1
    return e


class Cache:
    """One layer's codes [pages, tokens, heads, dim] (as the values of the codes) and exponents [pages, heads, blocks]
    of keys and values."""

    def __init__(self, pool, layer=0):
        self.code = next(n for n, t in CODES.items() if t == pool.k.dtype)
        self.dtype, self.block, self.pt = pool.dtype, pool.block_tokens, pool.page_tokens
        get = lambda t: (t[layer] if pool.order == "token" else t[layer].transpose(1, 2)).float().cpu().double().numpy()  # noqa: E731
        self.codes = [get(pool.k), get(pool.v)]
        self.exps = [pool.scale[layer, ..., i].cpu().numpy().astype(np.int64) - 127 for i in range(2)]

    def append(self, new, off, length, table):
        """new: k and v rows [total, heads, dim] in 64 bits."""
        lim = most(self.dtype, self.code)
        for j, x in enumerate(new):
            x = np.where(np.isfinite(x), np.clip(x, -lim, lim), x)
            for i, n in enumerate(length):
                pos = n - (off[i + 1] - off[i])
                while pos < n:
                    end = min(n, (pos // self.block + 1) * self.block)
                    g, s = table[i][pos // self.pt], pos % self.pt
                    b, old = s // self.block, s % self.block
                    rows = x[off[i + 1] - (n - pos):off[i + 1] - (n - end)]
                    for h in range(x.shape[1]):
                        part = np.abs(rows[:, h])
                        e = exponent_for(np.max(part[np.isfinite(part)], initial=0.0), self.code)
                        if old:
                            e_old = self.exps[j][g, h, b]
                            e = max(e, e_old)
                            self.codes[j][g, s - old:s, h] = code_of(self.codes[j][g, s - old:s, h], e - e_old, self.code)
                        self.codes[j][g, s:s + end - pos, h] = code_of(rows[:, h], e, self.code)
                        self.exps[j][g, h, b] = e
                    pos = end

    def tokens(self, j, row, n):
        """The first n tokens of a row of pages [n, heads, dim]: what the codes stand for."""
        out = np.zeros((n,) + self.codes[j].shape[2:])
        for t in range(n):
            g, s = row[t // self.pt], t % self.pt
            out[t] = np.ldexp(self.codes[j][g, s], self.exps[j][g, :, s // self.block][:, None])
        return out


def turn(x, positions, freq, rotated, layout, magnitude):
    """x [tokens, heads, dim] turned, in 64 bits."""
    y = x.copy()
    for t, p in enumerate(positions):
        for i, f in enumerate(freq):
            a, b = (i, i + rotated // 2) if layout == "half" else (2 * i, 2 * i + 1)
            c, s = math.cos(p * f) * magnitude, math.sin(p * f) * magnitude
            y[t, :, a], y[t, :, b] = x[t, :, a] * c - x[t, :, b] * s, x[t, :, b] * c + x[t, :, a] * s
    return y
