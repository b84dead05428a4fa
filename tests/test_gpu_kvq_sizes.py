"""The 8-bit calls at the sizes that take other ways: more sequences than a block looks at at once, and than it has sums for; empty
sequences in long runs; sequences cut over many wavefronts; refusals that need tensors on the GPU."""
import math

import pytest
import torch

from paper_2608_19677_amd import binding as B
from paper_2608_19677_amd import serve

import kvq_oracle as ko
import serve_oracle as so
from cr_check import say

pytestmark = pytest.mark.gpu


def _i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _randn(g, *shape, dtype, scale=1.0):
    return (torch.randn(shape, generator=g, device="cuda") * scale).to(dtype)


def _cum(t):
    return torch.cat([torch.zeros(1, dtype=torch.int32, device="cuda"), t.cumsum(0).to(torch.int32)])


CASES = {
    # type, code, heads, key heads, dim, page, requests, groups, longest own, longest prefix, share of empty requests
    "windows": ("bf16", "e4m3", 8, 2, 64, 8, 700, 40, 70, 90, 0.0),
    "windows-empty": ("f16", "e4m3", 16, 2, 128, 16, 900, 300, 40, 0, 0.8),
    "entries": ("bf16", "e5m2", 4, 1, 64, 4, 40000, 7, 3, 20, 0.3),
    "runs": ("bf16", "e4m3", 4, 4, 64, 8, 500, 12, 64, 33, 0.97),
}


@pytest.mark.parametrize("name", CASES)
def test_many_sequences(name):
    kind, code, hq, hkv, d, pg, n, groups, longest, longest_prefix, empty = CASES[name]
    say(f"[case] 8-bit attention of many sequences, {name}")
    dt, g = ko.DT[kind], _gen(n)
    own = torch.randint(1, longest + 1, (n,), generator=g, device="cuda").to(torch.int32)
    own *= torch.rand(n, generator=g, device="cuda") >= empty
    prefix = torch.randint(0, longest_prefix + 1, (groups,), generator=g, device="cuda").to(torch.int32)
    prefix[0] = longest_prefix
    cuts = torch.randint(0, n + 1, (groups - 1,), generator=g, device="cuda").sort().values  # some groups without requests
    go = torch.cat([_i32([0]), cuts.to(torch.int32), _i32([n])])
    lens = torch.cat([prefix, own])
    need = (lens + pg - 1) // pg
    pages = int(need.sum()) + 1
    pool = serve.QuantPagePool.empty(1, pages, hkv, pg, d, dt, codes=ko.CODES[code], block_tokens=min(pg, 8))
    table = torch.full((groups + n, int(need.max())), -1, dtype=torch.int32, device="cuda")
    ids, col = torch.randperm(pages, generator=g, device="cuda").to(torch.int32), torch.arange(table.shape[1], device="cuda")
    table[col < need[:, None]] = ids[:int(need.sum())]
    off, total = _cum(lens), int(lens.sum())
    k, v = _randn(g, total, hkv, d, dtype=dt), _randn(g, total, hkv, d, dtype=dt)
    pool.append(0, k, v, off, lens, table)
    pool.read(0, k, v, off, lens, table)  # what the codes stand for
    q = _randn(g, n, hq, d, dtype=dt, scale=1.5)  # one query a request, also of those without tokens
    scale, qo = 1 / math.sqrt(d), torch.arange(n + 1, dtype=torch.int32, device="cuda")
    lse = torch.empty(n, hq, device="cuda")
    out = serve.attend_shared(q, pool, 0, qo, go, table[:groups].contiguous(), prefix, table[groups:].contiguous(), own, scale, lse=lse)
    assert int(pool.err.item()) == 0
    # padded, in 64 bits: keys of the group's prefix, then the request's own; the one query sees them all
    group = torch.searchsorted(go[1:].long(), torch.arange(n, device="cuda"), right=True)
    for a in range(0, n, 4000):
        r = torch.arange(a, min(n, a + 4000), device="cuda")
        x = group[r]
        i, j = torch.arange(longest_prefix, device="cuda"), torch.arange(longest, device="cuda")
        at = torch.cat([(off[x].long()[:, None] + i), (off[groups + r].long()[:, None] + j)], 1).clamp(max=total - 1)
        seen = torch.cat([i < prefix[x][:, None], j < own[r][:, None]], 1)[:, None]
        for h in range(hkv):
            kk, vv = k[at, h].double(), v[at, h].double()
            qq = q[r, h * (hq // hkv):(h + 1) * (hq // hkv)].double()
            s = torch.where(seen, torch.bmm(qq, kk.transpose(1, 2).contiguous()) * scale, -math.inf)
            reach = torch.where(seen, torch.bmm(qq.abs(), kk.abs().transpose(1, 2).contiguous()) * scale, 0.0).amax(2)
            l = torch.logsumexp(s, 2)
            w = torch.exp(s - torch.where(l == -math.inf, 0.0, l)[..., None])
            res = [torch.bmm(w, vv), l, torch.bmm(w, vv.abs()), reach]
            res = [t.reshape(-1, *t.shape[2:]).cpu().numpy() for t in res]
            so.check(out[r, h * (hq // hkv):(h + 1) * (hq // hkv)].reshape(-1, d), lse[r, h * (hq // hkv):(h + 1) * (hq // hkv)].reshape(-1), res, dt, name)


def test_long_sequence_over_many_wavefronts():
    """One request on 70,001 tokens of its own: shares of every wavefront, all slots."""
    say("[case] 8-bit attention, one long sequence")
    n, hq, hkv, d, pg = 70001, 4, 2, 128, 64
    g = _gen(7)
    for code, ql in (("e4m3", 1), ("e5m2", 9)):
        pool = serve.QuantPagePool.empty(1, -(-n // pg) + 2, hkv, pg, d, codes=ko.CODES[code], block_tokens=32)
        table = torch.randperm(pool.num_pages, generator=g, device="cuda")[:-(-n // pg)].to(torch.int32)[None].contiguous()
        k, v = _randn(g, n, hkv, d, dtype=torch.bfloat16), _randn(g, n, hkv, d, dtype=torch.bfloat16)
        off, length = _i32([0, n]), _i32([n])
        pool.append(0, k, v, off, length, table)
        pool.read(0, k, v, off, length, table)
        q = _randn(g, ql, hq, d, dtype=torch.bfloat16, scale=1.5)
        lse = torch.empty(ql, hq, device="cuda")
        out = serve.attend_shared(q, pool, 0, _i32([0, ql]), _i32([0, 1]), table[:, :1].contiguous(), _i32([0]), table, length, 0.09, lse=lse)
        lim = torch.arange(ql, device="cuda") + n - ql + 1
        ref = so.many(q, [(0, ql, [(k, v, lim)])], hkv, 0.09)
        so.check(out.reshape(-1, d), lse.reshape(-1), ref, torch.bfloat16, code)
        # the prefix's way: the same keys behind a group of one
        two = serve.attend_shared(q[:1], pool, 0, _i32([0, 1]), _i32([0, 1]), table, _i32([n]), table[:, :1].contiguous(), _i32([0]), 0.09)
        ref = so.many(q[:1], [(0, 1, [(k, v, torch.full((1,), n, device="cuda"))])], hkv, 0.09)
        so.check(two.reshape(-1, d), None, ref, torch.bfloat16, code + " prefix")


def test_refusals_of_tensors():
    say("[case] 8-bit wrappers, tensors that do not fit")
    pool = serve.QuantPagePool.empty(1, 4, 2, 16, 64)
    k = torch.zeros(3, 2, 64, dtype=torch.bfloat16, device="cuda")
    off, length, table = _i32([0, 3]), _i32([3]), _i32([[0]])
    for call in (pool.append, pool.read):
        for bad in (k.half(), k[:, :1], k[..., :32], k.transpose(0, 2), k.float()):
            with pytest.raises(B.CrError, match="heads, dim and type"):
                call(0, bad, bad, off, length, table)
        with pytest.raises(B.CrError, match="heads, dim and type"):
            call(0, k, k[:2], off, length, table)
        with pytest.raises(B.CrError, match="int32"):
            call(0, k, k, off.long(), length, table)
        with pytest.raises(B.CrError, match="entries"):
            call(0, k, k, off[:1], length, table)
        with pytest.raises(B.CrError, match="a table is"):
            call(0, k, k, off, length, table[0])
        with pytest.raises(B.CrError, match="no gradient"):
            call(0, k.clone().requires_grad_(), k, off, length, table)
        with pytest.raises(B.CrError, match="out of range"):
            call(-1, k, k, off, length, table)
        with pytest.raises(B.CrError, match="-1"):
            call(1, k, k, off, length, table)
    with pytest.raises(B.CrError, match="wanted"):
        pool.read(0, None, None, off, length, table)
    with pytest.raises(B.CrError, match="type and dim"):
        serve.attend_shared(k.half(), pool, 0, off, _i32([0, 1]), table, _i32([0]), table, length, 1.0)
    codes = torch.zeros(1, 4, 2, 16, 64, dtype=torch.uint8, device="cuda")
    refs = torch.zeros(4, dtype=torch.int32, device="cuda")
    scale = torch.zeros(1, 4, 2, 2, 2, dtype=torch.uint8, device="cuda")
    e4 = codes.view(torch.float8_e4m3fn)
    with pytest.raises(B.CrError, match="float8"):
        serve.QuantPagePool(codes, codes, scale, refs)
    with pytest.raises(B.CrError, match="bfloat16 or float16"):
        serve.QuantPagePool(e4, e4, scale, refs, dtype=torch.float32)
    for bad in (scale[0], scale[..., :1], scale.float(), scale[:, :, :, :0], scale.transpose(3, 4), torch.zeros(1, 4, 2, 3, 2, dtype=torch.uint8, device="cuda")):
        with pytest.raises(B.CrError, match="scale is uint8"):
            serve.QuantPagePool(e4, e4, bad, refs)
    rot = serve.Rotary(64, 32)
    pos = _i32([0, 1, 2])
    with pytest.raises(B.CrError, match="dim of this handle"):
        rot.apply(torch.zeros(3, 2, 128, dtype=torch.bfloat16, device="cuda"), None, pos)
    with pytest.raises(B.CrError, match="q's tokens"):
        rot.apply(k, k[:2], pos)
    with pytest.raises(B.CrError, match="q's tokens"):
        rot.apply(k, k.half(), pos)
    with pytest.raises(B.CrError, match="bfloat16 or float16"):
        rot.apply(k.float(), None, pos)
    with pytest.raises(B.CrError, match="entries"):
        rot.apply(k, None, pos[:2])
    with pytest.raises(B.CrError, match="int32"):
        rot.apply(k, None, pos.long())
    with pytest.raises(B.CrError, match="q_out has"):
        rot.apply(k, None, pos, q_out=k[:2])
    with pytest.raises(B.CrError, match="k_out has"):
        rot.apply(k, k, pos, k_out=k.half())
    with pytest.raises(B.CrError, match="no keys"):
        rot.apply(k, None, pos, k_out=k)
    with pytest.raises(B.CrError, match="no gradient"):
        rot.apply(k.clone().requires_grad_(), None, pos)
    with pytest.raises(B.CrError, match="-1"):  # over itself, shifted strides
        x = torch.zeros(3, 4, 64, dtype=torch.bfloat16, device="cuda")
        rot.apply(x[:, :2], None, pos, q_out=x.view(3, 4, 64)[:, ::2])
    assert int(pool.err.item()) == 0
