"""The binding's functions of the serving calls, which take structures, against the handles that wrap the same
library calls."""
import torch
import pytest

from paper_2608_19677_amd import binding as B
from paper_2608_19677_amd import serve

from cr_check import say

pytestmark = pytest.mark.gpu


def _i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _rows(t):
    return B.CrRows(t.data_ptr(), t.stride(0), t.stride(1))


def _pools():
    a, b = (serve.PagePool.empty(2, 40, 2, 8, 64) for _ in range(2))
    for x, y in ((a.k, b.k), (a.v, b.v)):
        x.normal_(generator=torch.Generator(device="cuda").manual_seed(1))
        y.copy_(x)
    return a, b


def _same(a, b):
    assert int(a.err.item()) == 0 and int(b.err.item()) == 0
    return all(torch.equal(getattr(a, n), getattr(b, n)) for n in ("k", "v", "refs"))


def test_page_calls():
    a, b = _pools()
    ws, err = torch.empty(B.cr_pages_workspace_bytes(40, 4), dtype=torch.uint8, device="cuda"), b.err
    ta, tb = (torch.full((3, 6), -1, dtype=torch.int32, device="cuda") for _ in range(2))
    ca, cb = (torch.full((4, 6), -1, dtype=torch.int32, device="cuda") for _ in range(2))
    old, new = _i32([0, 3, 8]), _i32([20, 9, 48])
    say("[case] page calls by structures")
    for first, last in ((None, old), (old, new)):
        a.extend(ta, first, last)
        B.cr_pages_extend(b.c, first, last, tb, ws, err)
        assert torch.equal(ta, tb) and _same(a, b)
    parent, length = _i32([0, 1, 2, 0]), _i32([20, 5, 41, 0])
    a.fork(ta, parent, length, ca)
    B.cr_pages_fork(b.c, tb, parent, length, cb, ws, err)
    assert torch.equal(ca, cb) and _same(a, b)
    a.free(ta, new)
    B.cr_pages_free(b.c, tb, new, err)
    assert _same(a, b)
    a.compact(ca, length)
    B.cr_pages_compact(b.c, cb, length, cb, b.refs, ws, err)
    assert torch.equal(ca, cb) and _same(a, b)
    a.copy(_i32([0, 1]), _i32([30, 31]))
    B.cr_pages_copy(b.c, _i32([0, 1]), _i32([30, 31]), err)
    assert _same(a, b)
    B.cr_pages_compact(b.c, None, None, None, b.refs, ws, err)  # the pages are at the front already
    assert _same(a, b)
    x = torch.randn(3, 2, 64, device="cuda").to(torch.bfloat16)
    off, held = _i32([0, 1, 1, 3, 3]), _i32([20, 5, 41, 0])
    a.append(1, x, x, off, held, ca)
    B.cr_kv_append(b.c, 1, _rows(x), _rows(x), 3, off, held, cb, err)
    assert _same(a, b)


def test_attention():
    a, _ = _pools()
    a.refs[:6] = 1
    g = torch.Generator(device="cuda").manual_seed(2)
    q = torch.randn(9, 4, 64, generator=g, device="cuda").to(torch.bfloat16)
    k, v = (torch.randn(900, 2, 64, generator=g, device="cuda").to(torch.bfloat16) for _ in range(2))
    qo, ko, err = _i32([0, 4, 9]), _i32([0, 400, 900]), _i32([0])
    want = serve.attend_prompt(q, k, v, qo, ko, 0.125)
    out, lse = torch.empty_like(q), torch.empty(9, 4, device="cuda")
    args = B.CrAttnPromptArgs(B.CR_BF16, 4, 2, 64, 2, 1, 9, 900, 0.125, _rows(q), _rows(k), _rows(v), _rows(out), lse.data_ptr(),
                              qo.data_ptr(), ko.data_ptr())
    ws = torch.empty(max(16, B.cr_attn_prompt_workspace_bytes(args)), dtype=torch.uint8, device="cuda")
    say("[case] prompt attention by structures")
    B.cr_attn_prompt(args, ws, err)
    assert torch.equal(out, want) and bool(torch.isfinite(lse).all())
    go, ptab, plen, otab, olen = _i32([0, 2]), _i32([[0, 1, 2]]), _i32([20]), _i32([[3], [4]]), _i32([8, 7])
    want = serve.attend_shared(q, a, 1, qo, go, ptab, plen, otab, olen, 0.125)
    args = B.CrAttnSharedArgs(4, 1, 2, 1, 9, 3, 1, 0.125, _rows(q), _rows(out), None, qo.data_ptr(), go.data_ptr(), ptab.data_ptr(),
                              plen.data_ptr(), otab.data_ptr(), olen.data_ptr())
    ws = torch.empty(max(16, B.cr_attn_shared_workspace_bytes(a.c, args)), dtype=torch.uint8, device="cuda")
    say("[case] shared attention by structures")
    B.cr_attn_shared(a.c, args, ws, err)
    assert torch.equal(out, want) and int(err.item()) == 0 and int(a.err.item()) == 0
