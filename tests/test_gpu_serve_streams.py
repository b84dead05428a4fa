"""Memory that the serving calls take, on streams other than the one it was taken on: it stays its owner's until the
work enqueued with it is done."""
import math

import pytest
import torch

from paper_2608_19677_amd import serve

from cr_check import say

pytestmark = pytest.mark.gpu


def _i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _busy(stream):
    """Some milliseconds of work in front of what comes next on the stream."""
    with torch.cuda.stream(stream):
        torch.cuda._sleep(10_000_000)


def _handed_out(size, at, n=8):
    """Whether one of n pieces of `size` bytes taken now on the current stream lies at the address."""
    return at in [t.data_ptr() for t in [torch.empty(size, dtype=torch.uint8, device="cuda") for _ in range(n)]]


@pytest.mark.parametrize("named", [False, True], ids=["current", "stream"])
def test_a_dropped_pool_is_kept_until_its_work_is_done(named):
    pool = serve.PagePool.empty(1, 20_000, 1, 4, 64)
    pool.refs[::3] = 1
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    torch.cuda.synchronize()
    _busy(side)
    say(f"[case] compaction on another stream, pool dropped, stream named: {named}")
    if named:
        pool.compact(None, None, stream=side)
    else:
        with torch.cuda.stream(side):
            pool.compact(None, None)
    held = [(t.data_ptr(), t.numel() * t.element_size()) for t in (pool.k, pool.refs, pool._ws, pool.err)]
    del pool
    taken = [_handed_out(n, p) for p, n in held]
    assert not side.query() and not any(taken)
    side.synchronize()


@pytest.mark.parametrize("named", [False, True], ids=["current", "stream"])
def test_a_dropped_workspace_is_kept_until_its_work_is_done(named):
    q = torch.randn(1, 8, 128, device="cuda").to(torch.bfloat16)
    k = torch.randn(100_000, 1, 128, device="cuda").to(torch.bfloat16)
    qo, ko, out = _i32([0, 1]), _i32([0, 100_000]), torch.empty_like(q)
    want = serve.attend_prompt(q, k, k, qo, ko, 1 / math.sqrt(128))
    ws = serve.prompt_workspace(q, k, qo)
    assert ws.buf.numel() > 16
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    _busy(side)
    say(f"[case] attention on another stream, workspace dropped, stream named: {named}")
    if named:
        serve.attend_prompt(q, k, k, qo, ko, 1 / math.sqrt(128), out=out, ws=ws, stream=side)
    else:
        with torch.cuda.stream(side):
            serve.attend_prompt(q, k, k, qo, ko, 1 / math.sqrt(128), out=out, ws=ws)
    p, n = ws.buf.data_ptr(), ws.buf.numel()
    del ws
    taken = _handed_out(n, p)
    assert not side.query() and not taken
    side.synchronize()
    assert torch.equal(out, want)


def _pool_of(t):
    """Handle of the stream from whose memory a tensor was taken."""
    for s in torch.cuda.memory_snapshot():
        if s["address"] <= t.data_ptr() < s["address"] + s["total_size"]:
            return s["stream"]
    raise AssertionError("not in any segment")


def test_what_a_call_takes_is_its_streams():
    """Outputs and workspaces made for a call on a named stream come from that stream's memory: the current
    stream's may still be written to by work enqueued there. The output also stays whole for the current stream."""
    q = torch.randn(3, 8, 64, device="cuda").to(torch.float16)
    k = torch.randn(3, 4, 64, device="cuda").to(torch.float16)
    off = _i32([0, 3])
    side = torch.cuda.Stream()
    say("[case] prompt attention on a named stream")
    want = serve.attend_prompt(q, k, k, off, off, 0.1)
    torch.cuda.synchronize()
    out = serve.attend_prompt(q, k, k, off, off, 0.1, stream=side)
    assert _pool_of(want) != side.cuda_stream and _pool_of(out) == side.cuda_stream
    side.synchronize()
    assert torch.equal(out, want)
    say("[case] shared attention and a growing workspace on a named stream")
    pool = serve.PagePool.empty(1, 300, 4, 16, 64, torch.float16)
    table, n = torch.zeros(2000, 1, dtype=torch.int32, device="cuda"), torch.zeros(2000, dtype=torch.int32, device="cuda")
    torch.cuda.synchronize()
    pool.extend(table, None, n, stream=side)
    assert _pool_of(pool._ws) == side.cuda_stream
    pool.append(0, k, k, off, _i32([3]), table[:1])
    torch.cuda.synchronize()
    args = (q, pool, 0, off, _i32([0, 1]), table[:1], _i32([0]), table[:1], _i32([3]), 0.1)
    torch.cuda.synchronize()
    out = serve.attend_shared(*args, stream=side)
    assert _pool_of(out) == side.cuda_stream
    _busy(torch.cuda.current_stream())  # the caller goes on with it
    at, size = out.data_ptr(), out.numel() * 2
    del out
    with torch.cuda.stream(side):
        assert not _handed_out(size, at)
    assert int(pool.err.item()) == 0
