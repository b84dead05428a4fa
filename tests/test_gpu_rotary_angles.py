"""Cosines and sines of rotary positions within 2^-22: pairs of whole numbers that nearly cancel, so that what the cosine and the
sine are off by is most of what comes out, and not lost behind its rounding to 16 bits."""
import math

import numpy as np
import pytest
import torch

from paper_2608_19677_amd import serve

import serve_oracle as so
from cr_check import say

pytestmark = pytest.mark.gpu

MOST = 2047  # whole numbers that float16 has


def _angles(freq, positions):
    """cos and sin of positions * freq / 2^64 turns, [positions, pairs], in 64 bits."""
    f, p = np.asarray(freq, dtype=np.uint64), np.asarray(positions, dtype=np.int64).astype(np.uint64)
    with np.errstate(over="ignore"):
        turn = (p[:, None] * f[None]).astype(np.int64).astype(np.float64) * 2.0 ** -64  # of the signed fraction: within 2^-54
    t = turn * (2 * math.pi)
    return np.cos(t), np.sin(t)


def _nearly_cancelling(c, s):
    """Whole a, b up to MOST with a c - b s the smallest there is with b (or a) the larger: [positions, pairs] each."""
    a, b = np.zeros(c.shape), np.zeros(c.shape)
    for i in np.ndindex(*c.shape):
        big, small = (c[i], s[i]) if abs(c[i]) >= abs(s[i]) else (s[i], c[i])
        y = np.arange(MOST // 2, MOST + 1)  # of the smaller one's factor's partner: |x| <= y
        x = np.rint(y * (small / big))
        j = int(np.argmin(np.abs(x * big - y * small)))
        a[i], b[i] = (x[j], y[j]) if abs(c[i]) >= abs(s[i]) else (y[j], x[j])
    return a, b


@pytest.mark.parametrize("layout", ["half", "pairs"])
@pytest.mark.parametrize("span", [20, 1 << 12, (1 << 31) - 1])
def test_cosines_and_sines(layout, span):
    """x1' = a cos - b sin with a, b nearly cancelling, x2' = b cos + a sin. Cosine and sine are off by 2^-22 at most, times |a| + |b|; the
    product b sin is rounded once (2^-24 of it) and their difference once (2^-24 of it); then comes one rounding to float16
    (2^-11 of it, or half of 2^-24)."""
    say(f"[case] rotary angles, positions to {span}, {layout}")
    r = np.random.default_rng(span)
    rot = serve.Rotary(64, 16, layout=layout, frequencies=[0.9 * 1.7 ** -i if span < 1 << 20 else 0.37 + 0.3 * i for i in range(8)])
    turns = [int(x) & ((1 << 64) - 1) for x in rot.freq.cpu().tolist()]
    pos = np.unique(r.integers(-span, span + 1, 2000))
    c, s = _angles(turns, pos)
    a, b = _nearly_cancelling(c, s)
    x = torch.zeros(len(pos), 1, 64, dtype=torch.float16)
    first, second = (slice(0, 8), slice(8, 16)) if layout == "half" else (slice(0, 16, 2), slice(1, 16, 2))
    x[:, 0, first], x[:, 0, second] = torch.from_numpy(a).half(), torch.from_numpy(b).half()
    assert np.array_equal(x[:, 0, first].double().numpy(), a) and np.array_equal(x[:, 0, second].double().numpy(), b)
    got = so.f64(rot.apply(x.cuda(), None, torch.from_numpy(pos).to(torch.int32).cuda())[0])[:, 0]
    for g, want, product in ((got[:, first], a * c - b * s, b * s), (got[:, second], b * c + a * s, a * s)):
        off = (np.abs(a) + np.abs(b)) * 2.0 ** -22
        wide = off + 2.0 ** -24 * np.abs(product) * (1 + 2.0 ** -20)
        total = wide + 2.0 ** -24 * (np.abs(want) + wide)
        tol = total + np.maximum(2.0 ** -11 * (np.abs(want) + total), 2.0 ** -25)
        worst = np.max(np.abs(g - want) / tol)
        assert worst <= 1, f"{worst:.3f} of what is allowed"
    # what the bound is measured with: rounding to 16 bits is a small part of it where the pair cancels
    small = np.abs(a * c - b * s)
    assert np.median(small * 2.0 ** -11 / ((np.abs(a) + np.abs(b)) * 2.0 ** -22)) < 0.1
