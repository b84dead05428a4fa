"""Rotary positions whose outputs would lie over each other or over the other's input are refused: the rows would be turned twice, or
not at all, as blocks come and go. On the host: nothing is enqueued."""
import ctypes

import pytest
import torch

from paper_2608_19677_amd import binding as B

from test_kvq_validation import BAD_ROTARY, _rotary
from test_serve_validation import FAKE, L, _rows  # noqa: F401

# As in test_serve_validation.py: a regression would launch a kernel on a fake address where a GPU is.
pytestmark = pytest.mark.skipif(torch.cuda.is_available(), reason="host-side validation tests run without a GPU")


def _apart(**kw):
    f = dict(q=_rows(FAKE), k=_rows(FAKE + (1 << 20)), q_out=_rows(FAKE + (2 << 20)), k_out=_rows(FAKE + (3 << 20)))
    f.update(kw)
    return _rotary(**f)


@pytest.mark.parametrize("kw", BAD_ROTARY, ids=[next(iter(k)) + str(i) for i, k in enumerate(BAD_ROTARY)])
def test_rotary_of_tensors_apart_refuses(L, kw):  # noqa: F811
    assert L.cr_rotary(ctypes.byref(_apart(**kw)), None) == B.CR_EINVAL


@pytest.mark.parametrize("kw", [
    dict(q=_rows(FAKE), k=_rows(FAKE), q_out=_rows(FAKE), k_out=_rows(FAKE)),  # the same rows as queries and as keys, in place
    dict(k_out=_rows(FAKE + (2 << 20))),                                        # one place for both
    dict(q_out=_rows(FAKE + (1 << 20))), dict(k_out=_rows(FAKE)),               # the other's input
    dict(q_out=_rows(FAKE + (1 << 20)), k_out=_rows(FAKE)),
], ids=["both in place", "one place", "keys", "queries", "crossed"])
def test_rotary_over_the_other_refuses(L, kw):  # noqa: F811
    assert L.cr_rotary(ctypes.byref(_apart(**kw)), None) == B.CR_EINVAL
