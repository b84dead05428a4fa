"""Tables without columns: every length but 0 is beyond them, and is reported."""
import pytest
import torch

from paper_2608_19677_amd import binding as B
from paper_2608_19677_amd import serve

from cr_check import say

pytestmark = pytest.mark.gpu


def _i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _none(rows):
    return torch.empty((rows, 0), dtype=torch.int32, device="cuda")


def _pool():
    pool = serve.PagePool.empty(1, 10, 1, 4, 64)
    pool.refs[:3] = 1
    return pool


@pytest.mark.parametrize("length,bits", [([0, 0], 0), ([0, 5], B.CR_ERR_SEQ), ([1], B.CR_ERR_SEQ), ([0] * 300 + [2 ** 31 - 1], B.CR_ERR_SEQ)])
def test_free(length, bits):
    pool = _pool()
    say(f"[case] free, no columns, {len(length)} rows")
    pool.free(_none(len(length)), _i32(length))
    assert int(pool.err.item()) == bits and pool.refs.tolist() == [1] * 3 + [0] * 7


@pytest.mark.parametrize("length,bits", [([0, 0], 0), ([0, 5], B.CR_ERR_SEQ), ([1], B.CR_ERR_SEQ), ([0] * 300 + [2 ** 31 - 1], B.CR_ERR_SEQ)])
def test_compact(length, bits):
    pool = _pool()
    pool.refs[8] = 2
    say(f"[case] compact, no columns, {len(length)} rows")
    pool.compact(_none(len(length)), _i32(length))
    assert int(pool.err.item()) == bits and pool.refs.tolist() == [1, 1, 1, 2] + [0] * 6
