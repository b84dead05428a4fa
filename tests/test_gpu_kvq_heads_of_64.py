"""Few rows over codes of heads of 64 elements, where a wavefront keeps two tiles of codes on their way: stretches of six tiles and
more, odd and even ones, with whole and with partial last tiles."""
import math

import pytest
import torch

from paper_2608_19677_amd import binding as B
from paper_2608_19677_amd import serve

import kvq_oracle as ko
import serve_oracle as so
from cr_check import say

pytestmark = pytest.mark.gpu

TILE = 32
LEAST = 6  # tiles of a stretch from which two are on their way


def _i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _randn(g, *shape, dtype, scale=1.0):
    return (torch.randn(shape, generator=g, device="cuda") * scale).to(dtype)


def _cum(t):
    return torch.cat([torch.zeros(1, dtype=torch.int32, device="cuda"), t.cumsum(0).to(torch.int32)])


def _most_shares(hkv):
    """No launch cuts a key head's line of work into more: two blocks of four wavefronts for each compute unit."""
    return 4 * -(-2 * torch.cuda.get_device_properties(0).multi_processor_count // hkv)


def _lengths(hkv):
    """Own lengths: of every kind of 6 to 9 tiles (odd or even, the last tile whole or partial) more than a line has cuts, so
    that whichever sequences are cut, one of each kind is a stretch of its own; and short and long ones between them."""
    cuts, own = _most_shares(hkv) - 1, []
    kinds = {}
    for i in range(4 * cuts + 8):
        tiles, partial = LEAST + i % 4, i // 4 % 2
        n = TILE * tiles - partial * (1 + 7 * i % (TILE - 1))
        own.append(n)
        kinds[(-(-n // TILE) % 2, n % TILE != 0)] = kinds.get((-(-n // TILE) % 2, n % TILE != 0), 0) + 1
        if i % 5 == 0:
            own.append(1 + 37 * i % 700)
    assert len(kinds) == 4 and min(kinds.values()) > cuts
    return own


@pytest.mark.parametrize("case", [("bf16", "e4m3", 16, 8, "head"), ("bf16", "e5m2", 4, 4, "token"), ("f16", "e4m3", 128, 64, "token"),
                                  ("f16", "e5m2", 32, 32, "head")], ids=lambda c: "-".join(map(str, c)))
def test_stretches_of_many_tiles(case):
    name, code, pg, block, order = case
    say(f"[case] 8-bit attention, stretches of many tiles {case}")
    dt, g, hq, hkv, d = ko.DT[name], _gen(pg), 48, 16, 64
    own = _i32(_lengths(hkv))
    n = len(own)
    ql = torch.minimum(own, _i32([(1, 2, 5, 1)[i % 4] for i in range(n)]))
    groups = n * 15 // 64 + 1  # so that the prefixes' rows are few, too
    prefix = torch.randint(0, 330, (groups,), generator=g, device="cuda").to(torch.int32)
    cuts = torch.randint(0, n + 1, (groups - 1,), generator=g, device="cuda").sort().values
    go = torch.cat([_i32([0]), cuts.to(torch.int32), _i32([n])])
    lens = torch.cat([prefix, own])
    need = (lens + pg - 1) // pg
    pages = int(need.sum()) + 1
    pool = serve.QuantPagePool.empty(1, pages, hkv, pg, d, dt, order=order, codes=ko.CODES[code], block_tokens=block)
    pool.k.view(torch.uint8).fill_(0x7F), pool.v.view(torch.uint8).fill_(0xFF), pool.scale.fill_(255)
    table = torch.full((groups + n, int(need.max())), -1, dtype=torch.int32, device="cuda")
    ids, col = torch.randperm(pages, generator=g, device="cuda").to(torch.int32), torch.arange(table.shape[1], device="cuda")
    table[col < need[:, None]] = ids[:int(need.sum())]
    off, total = _cum(lens), int(lens.sum())
    k, v = _randn(g, total, hkv, d, dtype=dt), _randn(g, total, hkv, d, dtype=dt)
    pool.append(0, k, v, off, lens, table)
    pool.read(0, k, v, off, lens, table)  # what the codes stand for
    qo, scale, nq = _cum(ql), 1 / math.sqrt(d), int(ql.sum())
    q = _randn(g, nq, hq, d, dtype=dt, scale=1.5)
    args = (q, pool, 0, qo, go, table[:groups].contiguous(), prefix, table[groups:].contiguous(), own, scale)
    lse = torch.full((nq, hq), math.nan, device="cuda")
    out = serve.attend_shared(*args, out=torch.full_like(q, math.nan), lse=lse)
    assert int(pool.err.item()) == 0
    assert torch.equal(serve.attend_shared(*args), out)  # the same every time
    # padded, in 64 bits: query t of a request sees its group's prefix and own tokens below own - ql + t + 1
    group = torch.searchsorted(go[1:].long(), torch.arange(n, device="cuda"), right=True)
    i, j, t = (torch.arange(int(x), device="cuda") for x in (prefix.max(), own.max(), ql.max()))
    per = hq // hkv
    for a in range(0, n, 150):
        r = torch.arange(a, min(n, a + 150), device="cuda")
        x = group[r]
        at = torch.cat([(off[x].long()[:, None] + i), (off[groups + r].long()[:, None] + j)], 1).clamp(max=total - 1)
        rows = (qo[r].long()[:, None] + t).clamp(max=nq - 1)
        lim = (own[r] - ql[r] + 1)[:, None] + t  # [requests, queries]
        seen = torch.cat([(i < prefix[x][:, None])[:, None].expand(-1, len(t), -1), j < lim[..., None]], 2).repeat_interleave(per, 1)
        real = (t < ql[r][:, None])
        for h in range(hkv):
            kk, vv = k[at, h].double(), v[at, h].double()
            qq = q[rows, h * per:(h + 1) * per].double().flatten(1, 2)
            s = torch.where(seen, torch.bmm(qq, kk.transpose(1, 2).contiguous()) * scale, -math.inf)
            reach = torch.where(seen, torch.bmm(qq.abs(), kk.abs().transpose(1, 2).contiguous()) * scale, 0.0).amax(2)
            l = torch.logsumexp(s, 2)
            w = torch.exp(s - l[..., None])
            pick = lambda y: y.unflatten(1, (len(t), per))[real].flatten(0, 1).cpu().numpy()  # noqa: E731
            ref = [pick(y) for y in (torch.bmm(w, vv), l, torch.bmm(w, vv.abs()), reach)]
            got = slice(h * per, (h + 1) * per)
            so.check(out[rows[real], got].reshape(-1, d), lse[rows[real], got].reshape(-1), ref, dt, f"{case} head {h}")


@pytest.mark.parametrize("code,n", [("e4m3", 70001), ("e5m2", 40007), ("e4m3", 33312)])
def test_a_long_sequence_cut(code, n):
    """One request on many tokens: the slots are so few that every wavefront has more than six tiles of it."""
    say(f"[case] 8-bit attention, {n} tokens of heads of 64")
    hq, hkv, d, pg, g = 4, 2, 64, 64, _gen(n)
    pool = serve.QuantPagePool.empty(1, -(-n // pg) + 2, hkv, pg, d, codes=ko.CODES[code], block_tokens=32)
    table = torch.randperm(pool.num_pages, generator=g, device="cuda")[:-(-n // pg)].to(torch.int32)[None].contiguous()
    k, v = _randn(g, n, hkv, d, dtype=torch.bfloat16), _randn(g, n, hkv, d, dtype=torch.bfloat16)
    off, length = _i32([0, n]), _i32([n])
    pool.append(0, k, v, off, length, table)
    pool.read(0, k, v, off, length, table)
    one = table[:, :1].contiguous()
    for ql in (1, 9):
        q = _randn(g, ql, hq, d, dtype=torch.bfloat16, scale=1.5)
        a = B.CrAttnSharedArgs(hq, 0, 1, 1, ql, 1, table.shape[1], 1.0)
        slots = B.cr_kvq_attn_workspace_bytes(pool.c, a) // (ql * hq * (d + 1) * 4) - 1  # but the prefix's
        assert 1 < slots and n > slots * TILE * LEAST
        lse = torch.empty(ql, hq, device="cuda")
        out = serve.attend_shared(q, pool, 0, _i32([0, ql]), _i32([0, 1]), one, _i32([0]), table, length, 0.12, lse=lse)
        lim = torch.arange(ql, device="cuda") + n - ql + 1
        so.check(out.reshape(-1, d), lse.reshape(-1), so.many(q, [(0, ql, [(k, v, lim)])], hkv, 0.12), torch.bfloat16, f"own, {ql}")
        # behind a group of one, the prefix's way: every row sees all
        two = serve.attend_shared(q, pool, 0, _i32([0, ql]), _i32([0, 1]), table, length, one, _i32([0]), 0.12, lse=lse)
        ref = so.many(q, [(0, ql, [(k, v, torch.full((ql,), n, device="cuda"))])], hkv, 0.12)
        so.check(two.reshape(-1, d), lse.reshape(-1), ref, torch.bfloat16, f"prefix, {ql}")
