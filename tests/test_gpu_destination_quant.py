"""A destination whose cache holds 8-bit floats and whose queries and keys are turned by their positions: the replay's counts,
and outputs that are attention over what the codes stand for, in 64 bits."""
import numpy as np
import pytest
import torch

from paper_2608_19677_amd import serve
from paper_2608_19677_amd import workload as wl_mod
from paper_2608_19677_amd.destination import Destination, Projection, main
from paper_2608_19677_amd.pipeline import Pipeline

import kvq_oracle as ko
import serve_oracle as so
from cr_check import say

pytestmark = pytest.mark.gpu

HQ, HKV, D, BLOCK = 8, 2, 128, 16


def _turned(x, first, rot):
    return ko.turn(so.f64(x), np.arange(len(x)) + first, rot.frequencies, rot.rotated, rot.layout, rot.magnitude) if len(x) else so.f64(x)


def _held(x, code, dtype):
    """What the cache holds of tokens written at once, from the start of a page on."""
    out = np.zeros(x.shape)
    lim = ko.most(dtype, code)
    for t in range(0, len(x), BLOCK):
        for h in range(x.shape[1]):
            part = np.clip(x[t:t + BLOCK, h], -lim, lim)
            e = ko.exponent_for(np.abs(part).max(), code)
            out[t:t + BLOCK, h] = np.ldexp(ko.code_of(part, e, code), e)
    return out


@pytest.mark.parametrize("code", ["e4m3", "e5m2"])
def test_destination_in_8_bits(code):
    wl = wl_mod.small_random(9, num_keys=40, n=600, R=4, Ws=[4], J=1)
    pipe = Pipeline(wl)
    pipe.step()
    h = pipe.host()
    assert h["err"] == 0
    mine = np.flatnonzero(h["dest"][0] == 0)[:60]
    keys, suffix = wl.keys[mine], np.minimum(wl.suffix[mine].astype(np.int64), 30)
    plen = np.minimum(wl.prefix_len[keys].astype(np.int64), 200)
    say(f"[case] destination in {code}: {len(mine)} requests")
    dt, project = torch.bfloat16, Projection(HQ, HKV, D, torch.bfloat16, "cuda")
    rot = serve.Rotary(D, 64, layout="pairs", scaling="linear", factor=2.0)
    both = []
    for kw in (dict(), dict(codes=ko.CODES[code], rotary=rot)):
        d = Destination(4, 200, 30, 20, layers=2, heads_q=HQ, heads_kv=HKV, dim=D, samples=2, project=project, **kw)
        hits = []
        for b in range(0, len(mine), 20):
            e = min(len(mine), b + 20)
            hit, order, (out, off, decoded) = d.serve(keys[b:e], plen[b:e], suffix[b:e], first_id=b)
            hits += hit
        d.compact()
        both.append((d, hits))
    (plain, plain_hits), (d, hits) = both
    assert hits == plain_hits and d.counts == plain.counts
    assert type(d.pool) is serve.QuantPagePool and torch.equal(d.pool.refs, plain.pool.refs)

    # the last batch's outputs, a request in three: the last layer's attention over the cached prefix and the suffix
    b = len(mine) - (len(mine) - 1) % 20 - 1
    off = off.tolist()
    for x in range(0, len(order), 3):
        i = b + order[x]
        n, m = int(plen[i]), int(suffix[i])
        pq, pk, pv = project(1, [int(keys[i])], [n])
        q, k, v = project(1, [1 << 40 | int(i)], [m])
        # turned values are rounded to bfloat16 before they are held: what the library's rotation gives, itself within its
        # bounds of the definition
        pk, k = (rot.apply(t, None, torch.arange(len(t), dtype=torch.int32, device="cuda") + a)[0] for t, a in ((pk, 0), (k, n)))
        q = rot.apply(q, None, torch.arange(m, dtype=torch.int32, device="cuda") + n)[0]
        parts = [_held(so.f64(t), code, dt) for t in (pk, pv, k, v)]
        ref = so.shared(q, [(parts[0], parts[1])], [(parts[2], parts[3])], [0, m], [0, 1], d.scale)
        so.check(out[off[x]:off[x + 1]].reshape(-1, D), None, so.flat(ref), dt, f"request {i}")
        assert np.abs(so.f64(k) - _turned(project(1, [1 << 40 | int(i)], [m])[1], n, rot)).max() <= 2.0 ** -8 * np.abs(so.f64(k)).max() * 1.01


def test_command(monkeypatch, capsys):
    say("[case] the destination's command, in 8 bits and turned")
    monkeypatch.setattr("sys.argv", ["destination", "--requests", "40", "--batch", "16", "--codes", "e4m3", "--rotary"])
    main()
    assert "40 requests" in capsys.readouterr().out
