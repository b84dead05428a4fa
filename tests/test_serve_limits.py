"""Sizes that pass what a launch takes are refused on the host, before any kernel of the call is enqueued
(no GPU, no pointer is dereferenced)."""
import ctypes

import pytest
import torch

from paper_2608_19677_amd import binding as B

from test_serve_validation import FAKE, L, _cache, _prompt, _shared  # noqa: F401

# As in test_serve_validation.py: a regression would launch a kernel on a fake address where a GPU is.
pytestmark = pytest.mark.skipif(torch.cuda.is_available(), reason="host-side validation tests run without a GPU")


@pytest.mark.parametrize("pages", [40, 4097, 1 << 26])
def test_fork_of_more_children_than_a_launch_takes(L, pages):  # noqa: F811
    """A block of 256 threads a child, one for the prefix of needs and one per 4,096 pages: 2^32 threads are too many."""
    c = ctypes.byref(_cache(num_pages=pages))
    chunks = -(-pages // 4096)
    fork = lambda n: L.cr_pages_fork(c, FAKE, 1, 4, FAKE, FAKE, n, FAKE + 64, 4, FAKE, 0, FAKE, None)  # noqa: E731
    assert fork((1 << 24) - chunks - 1) == B.CR_EINVAL and fork(1 << 24) == B.CR_EINVAL
    assert fork((1 << 24) - chunks - 2) == B.CR_ESIZE  # the sizes are taken, the workspace is too small


def _attend_shared(L, ws_bytes=1 << 50, **kw):  # noqa: F811
    return L.cr_attn_shared(ctypes.byref(_cache(heads=1)), ctypes.byref(_shared(**kw)), FAKE, ws_bytes, FAKE, None)


def test_join_of_more_rows_than_a_launch_takes(L):  # noqa: F811
    """A block of 256 threads per query token joins prefix and own tokens: 2^24 tokens are too many."""
    few = dict(heads_q=1, prefix_width=4, own_width=2)
    for batch, n in ((1 << 24, 1 << 24), ((1 << 24) - 8, (1 << 24) + 5)):
        assert _attend_shared(L, **few, batch=batch, groups=batch, total_q=n) == B.CR_EINVAL
    n = (1 << 24) - 1
    assert _attend_shared(L, 64, **few, batch=n, groups=n, total_q=n) == B.CR_ESIZE


def test_prompt_attention_has_no_gradient():
    from paper_2608_19677_amd import serve
    q, off = torch.zeros(3, 4, 64, dtype=torch.bfloat16), torch.tensor([0, 3], dtype=torch.int32)
    for i in range(3):
        x = [q, q, q]
        x[i] = q.clone().requires_grad_()
        with pytest.raises(B.CrError, match="no gradient"):
            serve.attend_prompt(*x, off, off, 1.0)
        with torch.no_grad(), pytest.raises(B.CrError, match="device tensors"):
            serve.attend_prompt(*x, off, off, 1.0)
