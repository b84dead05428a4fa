"""Page calls of caches too large for one block: free pages in several chunks of 4,096, sequences in several
rounds of 256, and every error that the calls of small caches report."""
import pytest
import torch

from paper_2608_19677_amd import binding as B
from paper_2608_19677_amd import serve

from cr_check import say

pytestmark = pytest.mark.gpu

PAGES = 20_000  # from 16,385 on the calls take many blocks


def _i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _pool(pages, pt=4, layers=1, heads=1, dim=64):
    pool = serve.PagePool.empty(layers, pages, heads, pt, dim)
    # page p of layer l holds 1 + (p + l) % 251 in k and its negative in v: exact in 16 bits
    mark = 1 + (torch.arange(pages, device="cuda")[None] + torch.arange(layers, device="cuda")[:, None]) % 251
    pool.k.copy_(mark[:, :, None, None, None].expand(pool.k.shape))
    pool.v.copy_(-pool.k)
    return pool


def _err(pool):
    v = int(pool.err.item())
    pool.err.zero_()
    return v


@pytest.mark.parametrize("pages", [10, PAGES])
def test_fork_of_a_tail_in_a_free_page(pages):
    """A tail's entry that names a free page, one out of range or CR_NO_PAGE is copied from nowhere, whatever the size
    of the cache and whether that page is handed out meanwhile; the other children are served."""
    pool = _pool(pages)
    pool.refs[2] = 1
    # the free pages are taken by id: 0, 1, 3, 4. Rows 0 and 1 have their tails in pages 0 and 3, which are free.
    table = _i32([[2, 0], [2, 3], [2, pages], [2, -1], [2, 2]])
    child = torch.full((5, 2), -7, dtype=torch.int32, device="cuda")
    k, v, refs = pool.k.clone(), pool.v.clone(), pool.refs.clone()
    say(f"[case] fork of free tails, {pages} pages")
    pool.fork(table, _i32([0, 1, 2, 3, 4]), _i32([6, 7, 5, 6, 7]), child)
    assert _err(pool) == B.CR_ERR_PAGE
    assert child.tolist() == [[2, 0], [2, 1], [2, 3], [2, 4], [2, 5]]
    refs[2] += 5
    refs[[0, 1, 3, 4, 5]] = 1
    assert torch.equal(pool.refs, refs)
    k[:, 5, :, :3], v[:, 5, :, :3] = k[:, 2, :, :3], v[:, 2, :, :3]
    assert torch.equal(pool.k, k) and torch.equal(pool.v, v)


@pytest.mark.parametrize("later", [40, 31_000], ids=["same", "grown"])
def test_a_graph_keeps_its_workspace(later):
    """A captured call's workspace stays the pool's when later calls have more sequences, whether they fit it or
    not: a replay writes into nobody else's memory."""
    pool = _pool(PAGES)
    live = torch.randperm(PAGES, generator=torch.Generator().manual_seed(5))[:9000].sort().values.cuda()
    table, length = live[::300].to(torch.int32).reshape(1, -1).contiguous(), _i32([4 * 30])
    out, counts = torch.empty_like(table), torch.empty_like(pool.refs)
    pool.refs[live] = 1
    pool.compact(table, length, table_out=out, refs_out=counts)
    want, want_counts = out.clone(), counts.clone()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        pool.compact(table, length, table_out=out, refs_out=counts)
    size = pool._ws.numel()
    say(f"[case] compaction in a graph, then {later} sequences")
    free = torch.full((later, 1), -1, dtype=torch.int32, device="cuda")
    pool.extend(free, None, torch.zeros(later, dtype=torch.int32, device="cuda"))
    torch.cuda.synchronize()
    others = [torch.full((size,), 0x5A, dtype=torch.uint8, device="cuda") for _ in range(6)]
    for _ in range(3):
        out.zero_(), counts.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(counts, want_counts)
        assert all(bool((x == 0x5A).all()) for x in others)
    assert _err(pool) == 0
