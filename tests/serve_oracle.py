"""Plain 64-bit statements of the serving operators, on the CPU, one row or page at a time."""
import math

import numpy as np
import torch

UNIT = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}  # unit roundoff


def rows(q, parts, scale):
    """q [n, D]; parts: (k [m, D], v [m, D], limit [n]) per stretch of keys; row i sees the keys of a
    part below its limit. Returns out [n, D], lse [n], the weighed sum of |v| (bounds the error of
    rounded weights) and the largest scale * sum |q k| (bounds the scores' error)."""
    out, lse = np.zeros(q.shape), np.full(len(q), -math.inf)
    mag, reach = np.zeros(q.shape), np.zeros(len(q))
    for i in range(len(q)):
        k = np.concatenate([p[0][:max(0, int(p[2][i]))] for p in parts])
        v = np.concatenate([p[1][:max(0, int(p[2][i]))] for p in parts])
        if not len(k):
            continue
        s = k @ q[i] * scale
        w = np.exp(s - s.max())
        total = w.sum()
        out[i], lse[i] = w @ v / total, s.max() + math.log(total)
        mag[i], reach[i] = w @ np.abs(v) / total, (np.abs(k) @ np.abs(q[i])).max() * scale
    return out, lse, mag, reach


def f64(t):
    return t.detach().to("cpu", torch.float64).numpy()


def check(out, lse, ref, dtype, where=""):
    """Weights and outputs are rounded to the type once each (u (sum w |v| + |o|)); scores and sums
    are fp32 sums of up to some thousands of terms (2^-14 of sum w |v| and 2^-18 of the scores'
    reach are ample); float16 weights below 2^-14 of the largest carry 2^-24 of it."""
    o, l, mag, reach = ref
    u = UNIT[dtype]
    tol = u * (mag + np.abs(o)) * 1.02 + 2.0 ** -14 * mag + 2.0 ** -18 * reach[:, None] * mag + 1e-30
    if dtype == torch.float16:
        tol = tol + 2.0 ** -24 * 256  # subnormal outputs and weights
    got = f64(out)
    assert np.isfinite(got).all(), where
    worst = np.max((np.abs(got - o) - tol), initial=-1.0)
    assert worst <= 0, f"{where}: off by {worst:.3g} more than {tol.max():.3g}"
    if lse is not None:
        gl = f64(lse)
        empty = np.isneginf(l)
        assert np.array_equal(np.isneginf(gl), empty), where
        assert np.all(np.abs(gl - l)[~empty] <= (2.0 ** -18 * (1.0 + reach))[~empty]), where


def prompt(q, k, v, q_off, k_off, scale, causal):
    """All rows [tokens, heads]: out, lse, mag, reach as `rows` gives them."""
    q, k, v = f64(q), f64(k), f64(v)
    g = q.shape[1] // k.shape[1]
    res = [np.zeros(q.shape), np.zeros(q.shape[:2]), np.zeros(q.shape), np.zeros(q.shape[:2])]
    for b in range(len(q_off) - 1):
        a, e, c, f = q_off[b], q_off[b + 1], k_off[b], k_off[b + 1]
        nq, nk = e - a, f - c
        lim = np.arange(nq) + nk - nq + 1 if causal else np.full(nq, nk)
        for h in range(q.shape[1]):
            for x, y in zip(res, rows(q[a:e, h], [(k[c:f, h // g], v[c:f, h // g], lim)], scale)):
                x[a:e, h] = y
    return res


def flat(res):
    return [x.reshape(-1, x.shape[-1]) if x.ndim == 3 else x.reshape(-1) for x in res]


def shared(q, prefix, own, q_off, group_off, scale):
    """prefix[g], own[r]: (k [n, Hkv, D], v) float64."""
    q = f64(q)
    hkv = own[0][0].shape[1]
    g = q.shape[1] // hkv
    res = [np.zeros(q.shape), np.zeros(q.shape[:2]), np.zeros(q.shape), np.zeros(q.shape[:2])]
    for x in range(len(group_off) - 1):
        pk, pv = prefix[x]
        for r in range(group_off[x], group_off[x + 1]):
            a, e = q_off[r], q_off[r + 1]
            ok, ov = own[r]
            lim = np.arange(e - a) + len(ok) - (e - a) + 1
            every = np.full(e - a, len(pk))
            for h in range(q.shape[1]):
                got = rows(q[a:e, h], [(pk[:, h // g], pv[:, h // g], every), (ok[:, h // g], ov[:, h // g], lim)], scale)
                for y, z in zip(res, got):
                    y[a:e, h] = z
    return res


class Pages:
    """The page calls, one page at a time."""

    def __init__(self, refs, page_tokens):
        self.refs, self.pt = [int(x) for x in refs], page_tokens

    def pages(self, n):
        return -(-n // self.pt)

    def take(self, n):
        free = [p for p, r in enumerate(self.refs) if r == 0]
        if len(free) < n:
            return None
        for p in free[:n]:
            self.refs[p] = 1
        return free[:n]

    def extend(self, table, old, new):
        table = [list(r) for r in table]
        got = self.take(sum(self.pages(b) - self.pages(a) for a, b in zip(old, new)))
        if got is None:
            return table, False
        at = 0
        for row, a, b in zip(table, old, new):
            for j in range(self.pages(a), self.pages(b)):
                row[j] = got[at]
                at += 1
        return table, True

    def fork(self, table, parent, length, width):
        """Child rows and the copies (source, destination, tokens)."""
        need = [i for i, n in enumerate(length) if n % self.pt]
        got = self.take(len(need))
        if got is None:
            return [[-1] * width for _ in parent], [], False
        own, rows_, copies = dict(zip(need, got)), [], []
        for i, (p, n) in enumerate(zip(parent, length)):
            full = n // self.pt
            row = list(table[p][:full])
            for g in row:
                self.refs[g] += 1
            if i in own:
                copies.append((table[p][full], own[i], n % self.pt))
                row.append(own[i])
            rows_.append(row + [-1] * (width - len(row)))
        return rows_, copies, True

    def free(self, table, length):
        for row, n in zip(table, length):
            for g in row[:self.pages(n)]:
                assert self.refs[g] > 0
                self.refs[g] -= 1

    def compact(self, table, length):
        live = sum(r > 0 for r in self.refs)
        src = [p for p, r in enumerate(self.refs) if r and p >= live]
        dst = [p for p, r in enumerate(self.refs) if not r and p < live]
        name = dict(zip(src, dst))
        for s, d in name.items():
            self.refs[d], self.refs[s] = self.refs[s], 0
        table = [[name.get(g, g) if j < self.pages(n) else g for j, g in enumerate(row)] for row, n in zip(table, length)]
        return table, list(name.items())


def head_on_gpu(q, parts, scale):
    """`rows` for one head's many rows, float64 on the GPU: q [n, D]; parts (k, v, limit [n])."""
    dev = q.device
    s, ab = [], []
    for k, _, lim in parts:
        seen = torch.arange(k.shape[0], device=dev) < lim[:, None]
        s.append(torch.where(seen, (q @ k.t().contiguous()) * scale, -math.inf))
        ab.append(torch.where(seen, (q.abs() @ k.abs().t().contiguous()) * scale, 0.0).amax(1) if k.shape[0] else torch.zeros(len(q), dtype=q.dtype, device=dev))
    s, v = torch.cat(s, 1), torch.cat([p[1] for p in parts])
    lse = torch.logsumexp(s, 1)
    w = torch.exp(s - torch.where(lse == -math.inf, torch.zeros_like(lse), lse)[:, None])
    return w @ v, lse, w @ v.abs(), torch.stack(ab).amax(0)


def many(q, seqs, hkv, scale):
    """Sequences of (first row, rows, parts) with parts (k [m, Hkv, D], v, limit): the four results of `rows`
    for all rows and heads, flat."""
    n, hq, d = q.shape
    g = hq // hkv
    res = [torch.zeros(n, hq, d, dtype=torch.float64, device=q.device), torch.full((n, hq), -math.inf, dtype=torch.float64, device=q.device),
           torch.zeros(n, hq, d, dtype=torch.float64, device=q.device), torch.zeros(n, hq, dtype=torch.float64, device=q.device)]
    for a, m, parts in seqs:
        for h in range(hkv):
            rows_ = q[a:a + m, h * g:(h + 1) * g].double().transpose(0, 1).reshape(-1, d)
            got = head_on_gpu(rows_, [(k[:, h].double(), v[:, h].double(), lim.repeat(g)) for k, v, lim in parts], scale)
            for x, y in zip(res, got):
                x[a:a + m, h * g:(h + 1) * g] = y.reshape(g, m, *y.shape[1:]).transpose(0, 1)
    return flat([x.cpu().numpy() for x in res])
