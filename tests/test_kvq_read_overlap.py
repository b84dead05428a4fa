"""Reading the 8-bit cache back into one place for keys and for values is refused: what lay there then would be either, as the lanes'
stores come. On the host: nothing is enqueued."""
import ctypes

import pytest
import torch

from paper_2608_19677_amd import binding as B

from test_kvq_validation import BAD_TOKENS, _cache, _tokens
from test_serve_validation import FAKE, L, _rows  # noqa: F401

# As in test_serve_validation.py: a regression would launch a kernel on a fake address where a GPU is.
pytestmark = pytest.mark.skipif(torch.cuda.is_available(), reason="host-side validation tests run without a GPU")


def _apart(**kw):
    f = dict(k=_rows(FAKE), v=_rows(FAKE + (1 << 20)))
    f.update(kw)
    return _tokens(**f)


def test_one_place_refuses(L):  # noqa: F811
    c = ctypes.byref(_cache())
    assert L.cr_kvq_read(c, ctypes.byref(_apart(v=_rows(FAKE))), FAKE, None) == B.CR_EINVAL
    # other strides from the same place on lie over each other, too
    assert L.cr_kvq_read(c, ctypes.byref(_apart(v=_rows(FAKE, token=2048))), FAKE, None) == B.CR_EINVAL
    # nothing to read: nothing is looked at
    assert L.cr_kvq_read(c, ctypes.byref(_apart(v=_rows(FAKE), total=0)), FAKE, None) == B.CR_OK


@pytest.mark.parametrize("call", ["cr_kvq_append", "cr_kvq_read"])
@pytest.mark.parametrize("kw", BAD_TOKENS, ids=[next(iter(k)) + str(i) for i, k in enumerate(BAD_TOKENS)])
def test_tokens_apart_refuse(L, call, kw):  # noqa: F811
    assert getattr(L, call)(ctypes.byref(_cache()), ctypes.byref(_apart(**kw)), FAKE, None) == B.CR_EINVAL
