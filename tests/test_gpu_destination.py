"""A destination run with the serving operators: what it counts is the replay's statistics of that
destination, and what it computes is attention over the cached prefixes and the requests' tokens."""
import numpy as np
import pytest
import torch

from paper_2608_19677_amd import workload as wl_mod
from paper_2608_19677_amd.destination import Destination
from paper_2608_19677_amd.pipeline import Pipeline

import serve_oracle as so
from cr_check import say

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("W,batch,samples", [(3, 16, 0), (8, 5, 2)])
def test_counts_are_the_replays(W, batch, samples):
    wl = wl_mod.small_random(81, num_keys=60, n=500, R=4, Ws=[W], hot=2, hot_share=0.2)
    wl.prefix_len[:] = 1 + wl.prefix_len % 90
    wl.suffix[:] = 1 + wl.suffix % 23
    pipe = Pipeline(wl)
    pipe.step()
    h = pipe.host()
    dest, stats = h["dest"][0], h["stats"].sum(axis=0)[0]
    for r in (0, 3):
        mine = np.flatnonzero(dest == r)
        say(f"[case] destination {r}: {len(mine)} requests, W {W}, batches of {batch}")
        keys, suffix = wl.keys[mine], wl.suffix[mine].astype(np.int64)
        plen = wl.prefix_len[keys].astype(np.int64)
        d = Destination(W, int(plen.max()), int(suffix.max()), batch, layers=2, heads_q=4, heads_kv=2, dim=64, page_tokens=8, samples=samples)
        for b in range(0, len(mine), batch):
            e = min(len(mine), b + batch)
            d.serve(keys[b:e], plen[b:e], suffix[b:e], first_id=b)
            if b % 3 == 0:
                d.compact()
        c = d.counts
        assert [c.requests, c.hits, c.prefill, c.hit_prefix] == stats[r].tolist()
        assert int(d.pool.err.item()) == 0
        # the cache holds the replay's final prefixes, most recent first, and nothing else
        lru = h["lru"][0, r]
        assert list(reversed(d.slots)) == lru[lru != 0xFFFFFFFF].tolist()
        assert int(d.pool.refs.sum().item()) == sum(d.pool.pages_of(int(d.length[x])) for x in d.slots.values())


def test_outputs_of_hits_misses_and_samples():
    d = Destination(2, 50, 12, 6, layers=2, heads_q=4, heads_kv=1, dim=64, page_tokens=8, samples=2)
    d.serve([7, 9], [33, 50], [3, 4])
    d.compact()
    keys, plen, suffix = [9, 5, 9, 7, 5], [50, 16, 50, 33, 16], [12, 1, 5, 2, 7]
    say("[case] outputs of a batch of hits and misses")
    hit, order, (out, off, decoded) = d.serve(keys, plen, suffix, first_id=100)
    # two slots: 5 drops 7, 7 drops 5, and 5 has to come again
    assert hit == [True, False, True, False, False]
    x = lambda i, n: [so.f64(t) for t in d.project(1, [i], [n])]  # noqa: E731
    q_all, prefix, own = [], [], []
    for i in order:
        _, pk, pv = x(keys[i], plen[i])
        q, k, v = x(1 << 40 | 100 + int(i), suffix[i])
        for s in [None, 0, 1]:  # the suffix itself, then its two continuations
            if s is None:
                q_all.append(q), own.append((k, v))
            else:
                dq, dk, dv = x(2 << 40 | (100 + int(i)) * 2 + s, 1)
                q_all.append(dq), own.append((np.concatenate([k, dk]), np.concatenate([v, dv])))
            prefix.append((pk, pv))
    q_off = np.concatenate([[0], np.cumsum([len(q) for q in q_all])])
    ref = so.shared(torch.from_numpy(np.concatenate(q_all)), prefix, own, q_off, list(range(len(own) + 1)), d.scale)
    at = np.concatenate([np.arange(q_off[j], q_off[j + 1]) for j in range(0, len(own), 3)])
    so.check(out.reshape(-1, 64), None, so.flat([y[at] for y in ref]), torch.bfloat16, "suffixes")
    at = np.concatenate([np.arange(q_off[j], q_off[j + 1]) for j in range(len(own)) if j % 3])
    so.check(decoded.reshape(-1, 64), None, so.flat([y[at] for y in ref]), torch.bfloat16, "samples")
    assert off.tolist() == [0] + np.cumsum([suffix[i] for i in order]).tolist()
