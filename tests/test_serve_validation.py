"""Refusals of the serving calls: every malformed call returns its code on the host before anything is
enqueued (no GPU, no pointer is dereferenced), the sizes are checked, and the wrappers refuse
tensors that do not fit."""
import ctypes

import pytest
import torch

from paper_2608_19677_amd import binding as B
from paper_2608_19677_amd import serve

FAKE = 0x10000  # never dereferenced: every call below fails validation first

# Host-only checks: with a GPU visible a validation regression would launch a kernel on a
# fake address, so these run only where no GPU is present.
pytestmark = pytest.mark.skipif(torch.cuda.is_available(), reason="host-side validation tests run without a GPU")


@pytest.fixture(scope="module")
def L():
    import os

    from paper_2608_19677_amd import build
    if not os.path.exists(build.LIB):
        build.build()
    return B.load()


def _cache(**kw):
    f = dict(dtype=B.CR_BF16, heads=2, dim=128, page_tokens=16, num_pages=40, layers=2, k=FAKE, v=FAKE,
             layer_stride=40 * 4096, page_stride=4096, head_stride=2048, token_stride=128, refs=FAKE)
    f.update(kw)
    return B.CrKvCache(**f)


def _rows(p=FAKE, token=1024, head=128):
    return B.CrRows(p, token, head)


BAD_CACHES = [dict(dtype=2), dict(heads=0), dict(heads=1025), dict(dim=32), dict(dim=96), dict(page_tokens=0), dict(page_tokens=24),
              dict(page_tokens=2048), dict(num_pages=0), dict(num_pages=(1 << 26) + 1), dict(layers=0), dict(layers=1025), dict(k=None),
              dict(v=FAKE + 2), dict(page_stride=4095), dict(head_stride=-8), dict(token_stride=1 << 31), dict(layer_stride=12)]


@pytest.mark.parametrize("kw", BAD_CACHES, ids=[str(k) for k in BAD_CACHES])
def test_every_call_refuses_a_bad_cache(L, kw):
    c = ctypes.byref(_cache(**kw))
    r = ctypes.byref(_rows())
    assert L.cr_pages_extend(c, None, FAKE, 1, FAKE, 4, FAKE, 1 << 20, FAKE, None) == B.CR_EINVAL
    assert L.cr_pages_fork(c, FAKE, 1, 4, FAKE, FAKE, 1, FAKE + 64, 4, FAKE, 1 << 20, FAKE, None) == B.CR_EINVAL
    assert L.cr_pages_free(c, FAKE, 4, FAKE, 1, FAKE, None) == B.CR_EINVAL
    assert L.cr_pages_compact(c, FAKE, FAKE, 1, 4, FAKE, FAKE, FAKE, 1 << 20, FAKE, None) == B.CR_EINVAL
    assert L.cr_pages_copy(c, FAKE, FAKE, 1, FAKE, None) == B.CR_EINVAL
    assert L.cr_kv_append(c, 0, r, r, 1, FAKE, FAKE, 1, FAKE, 4, FAKE, None) == B.CR_EINVAL
    assert L.cr_attn_shared(c, ctypes.byref(_shared()), FAKE, 1 << 40, FAKE, None) == B.CR_EINVAL


def test_page_calls_refuse(L):
    c = ctypes.byref(_cache())
    need = B.cr_pages_workspace_bytes(40, 1)
    assert L.cr_pages_extend(c, None, FAKE, 1, FAKE, 4, FAKE, need - 1, FAKE, None) == B.CR_ESIZE
    assert L.cr_pages_extend(c, None, None, 1, FAKE, 4, FAKE, need, FAKE, None) == B.CR_EINVAL
    assert L.cr_pages_extend(c, None, FAKE, 1, None, 4, FAKE, need, FAKE, None) == B.CR_EINVAL
    assert L.cr_pages_extend(c, None, FAKE, 1, FAKE, 4, FAKE + 2, need, FAKE, None) == B.CR_EINVAL
    assert L.cr_pages_extend(c, None, FAKE, 1, FAKE, 4, FAKE, need, None, None) == B.CR_EINVAL
    assert L.cr_pages_extend(c, None, None, 0, None, 4, FAKE, need, FAKE, None) == B.CR_OK
    assert L.cr_pages_fork(c, FAKE, 1, 4, FAKE, FAKE, 1, FAKE, 4, FAKE, need, FAKE, None) == B.CR_EINVAL  # child is table
    assert L.cr_pages_fork(c, FAKE, 1, 4, FAKE, FAKE, 1, FAKE + 64, 4, FAKE, need - 4, FAKE, None) == B.CR_ESIZE
    assert L.cr_pages_fork(c, FAKE, 1, 4, None, FAKE, 1, FAKE + 64, 4, FAKE, need, FAKE, None) == B.CR_EINVAL
    assert L.cr_pages_free(c, None, 4, FAKE, 1, FAKE, None) == B.CR_EINVAL
    assert L.cr_pages_free(c, None, 0, None, 0, FAKE, None) == B.CR_OK
    big = B.cr_pages_workspace_bytes(40, 0)
    assert L.cr_pages_compact(c, FAKE, FAKE, 1, 4, FAKE, None, FAKE, big, FAKE, None) == B.CR_EINVAL
    assert L.cr_pages_compact(c, FAKE, FAKE, 1, 4, FAKE, FAKE, FAKE, big - 4, FAKE, None) == B.CR_ESIZE
    assert L.cr_pages_compact(ctypes.byref(_cache(refs=None)), None, None, 0, 0, None, FAKE, FAKE, big, FAKE, None) == B.CR_EINVAL
    assert L.cr_pages_copy(c, FAKE, None, 1, FAKE, None) == B.CR_EINVAL
    assert L.cr_pages_copy(c, None, None, 0, FAKE, None) == B.CR_OK
    r, off = ctypes.byref(_rows()), ctypes.byref(_rows(token=100))
    assert L.cr_kv_append(c, 2, r, r, 1, FAKE, FAKE, 1, FAKE, 4, FAKE, None) == B.CR_EINVAL
    assert L.cr_kv_append(c, 0, off, r, 1, FAKE, FAKE, 1, FAKE, 4, FAKE, None) == B.CR_EINVAL
    assert L.cr_kv_append(c, 0, r, r, 1, FAKE, FAKE, 0, FAKE, 4, FAKE, None) == B.CR_EINVAL
    assert L.cr_kv_append(c, 0, r, r, 0, None, None, 0, None, 0, FAKE, None) == B.CR_OK


def _prompt(**kw):
    f = dict(dtype=B.CR_BF16, heads_q=8, heads_kv=2, dim=128, batch=1, causal=1, total_q=200, total_k=200, scale=0.1, q=_rows(),
             k=_rows(), v=_rows(), out=_rows(), lse=FAKE, q_off=FAKE, k_off=FAKE)
    f.update(kw)
    return B.CrAttnPromptArgs(**f)


BAD_PROMPTS = [dict(dtype=3), dict(heads_q=7), dict(heads_q=1), dict(heads_kv=0), dict(heads_q=2048), dict(dim=80), dict(batch=0),
               dict(batch=(1 << 24) + 1), dict(causal=2), dict(total_q=1 << 28), dict(total_k=1 << 31), dict(scale=0.0), dict(scale=-1.0),
               dict(scale=float("nan")), dict(scale=float("inf")), dict(q=_rows(None)), dict(k=_rows(FAKE + 4)), dict(v=_rows(token=9)),
               dict(out=_rows(head=-8)), dict(lse=FAKE + 1), dict(q_off=None), dict(k_off=None)]


@pytest.mark.parametrize("kw", BAD_PROMPTS, ids=[next(iter(k)) + str(i) for i, k in enumerate(BAD_PROMPTS)])
def test_prompt_refuses(L, kw):
    assert L.cr_attn_prompt(ctypes.byref(_prompt(**kw)), FAKE, 1 << 50, FAKE, None) == B.CR_EINVAL


def test_prompt_sizes(L):
    assert L.cr_attn_prompt(ctypes.byref(_prompt(total_q=0)), None, 0, FAKE, None) == B.CR_OK
    assert L.cr_attn_prompt(None, None, 0, FAKE, None) == B.CR_EINVAL
    assert L.cr_attn_prompt(ctypes.byref(_prompt()), FAKE, 1 << 50, None, None) == B.CR_EINVAL
    few = _prompt(total_q=1, total_k=100_000)  # its keys are split: partial results in the workspace
    need = B.cr_attn_prompt_workspace_bytes(few)
    assert need >= 2 * 8 * (128 + 1) * 4
    assert L.cr_attn_prompt(ctypes.byref(few), FAKE, need - 1, FAKE, None) == B.CR_ESIZE
    assert L.cr_attn_prompt(ctypes.byref(few), None, need, FAKE, None) == B.CR_EINVAL
    assert L.cr_attn_prompt(ctypes.byref(few), FAKE + 4, need, FAKE, None) == B.CR_EINVAL
    assert B.cr_attn_prompt_workspace_bytes(_prompt(heads_q=64, total_q=16384, total_k=16384)) == 0  # rows fill the GPU


def _shared(**kw):
    f = dict(heads_q=8, layer=0, batch=3, groups=2, total_q=3, prefix_width=9, own_width=4, scale=0.1, q=_rows(), out=_rows(), lse=None,
             q_off=FAKE, group_off=FAKE, prefix_table=FAKE, prefix_len=FAKE, own_table=FAKE, own_len=FAKE)
    f.update(kw)
    return B.CrAttnSharedArgs(**f)


BAD_SHARED = [dict(heads_q=3), dict(layer=2), dict(groups=4), dict(groups=0), dict(total_q=1 << 29), dict(scale=0.0), dict(q=_rows(FAKE + 8)),
              dict(out=_rows(token=4)), dict(q_off=None), dict(group_off=None), dict(prefix_table=None), dict(prefix_len=None),
              dict(own_table=None), dict(own_len=None), dict(lse=FAKE + 2), dict(prefix_width=1 << 27)]


@pytest.mark.parametrize("kw", BAD_SHARED, ids=[next(iter(k)) + str(i) for i, k in enumerate(BAD_SHARED)])
def test_shared_refuses(L, kw):
    assert L.cr_attn_shared(ctypes.byref(_cache()), ctypes.byref(_shared(**kw)), FAKE, 1 << 50, FAKE, None) == B.CR_EINVAL


def test_shared_sizes(L):
    c, a = _cache(), _shared()
    need = B.cr_attn_shared_workspace_bytes(c, a)
    assert need >= 2 * 3 * 8 * (128 + 1) * 4
    assert L.cr_attn_shared(ctypes.byref(c), ctypes.byref(a), FAKE, need - 1, FAKE, None) == B.CR_ESIZE
    assert L.cr_attn_shared(ctypes.byref(c), ctypes.byref(_shared(total_q=0)), None, 0, FAKE, None) == B.CR_OK
    # a table without columns needs no pointer, and its sequences no keys
    assert B.cr_attn_shared_workspace_bytes(c, _shared(prefix_width=0, prefix_table=None)) > 0


def test_struct_layouts_match_header(L):
    assert ctypes.sizeof(B.CrRows) == 24
    assert ctypes.sizeof(B.CrKvCache) == 6 * 4 + 2 * 8 + 4 * 8 + 8
    assert ctypes.sizeof(B.CrAttnPromptArgs) == 40 + 4 * 24 + 3 * 8
    assert ctypes.sizeof(B.CrAttnSharedArgs) == 8 * 4 + 2 * 24 + 7 * 8


def test_wrappers_refuse_tensors_that_do_not_fit():
    k = torch.zeros(1, 4, 2, 16, 64, dtype=torch.bfloat16)
    refs = torch.zeros(4, dtype=torch.int32)
    with pytest.raises(B.CrError, match="device tensors"):
        serve.PagePool(k, k, refs)
    with pytest.raises(B.CrError, match="alike"):
        serve.PagePool(k, k[..., :32], refs)
    with pytest.raises(ValueError, match="order"):
        serve.PagePool(k, k, refs, order="page")
    q = torch.zeros(3, 4, 64, dtype=torch.bfloat16)
    off = torch.tensor([0, 3], dtype=torch.int32)
    with pytest.raises(B.CrError, match="one type"):
        serve.attend_prompt(q, q, q.float(), off, off, 1.0)
    with pytest.raises(B.CrError, match="bfloat16 or float16"):
        serve.attend_prompt(q.float(), q.float(), q.float(), off, off, 1.0)
    with pytest.raises(B.CrError, match="out has"):
        serve.attend_prompt(q, q, q, off, off, 1.0, out=q[:2])
    with pytest.raises(B.CrError, match="lse"):
        serve.attend_prompt(q, q, q, off, off, 1.0, out=q, lse=torch.zeros(3, 4, dtype=torch.float16))
    with pytest.raises(B.CrError, match="dim contiguous"):
        serve.attend_prompt(q.transpose(1, 2), q.transpose(1, 2), q.transpose(1, 2), off, off, 1.0)
    with pytest.raises(B.CrError, match="device tensors"):
        serve.attend_prompt(q, q, q, off, off, 1.0)


def test_counts_that_pass_32_bits_are_refused(L):
    c = ctypes.byref(_cache())
    assert L.cr_pages_extend(c, None, FAKE, 1 << 16, FAKE, 1 << 16, FAKE, 1 << 40, FAKE, None) == B.CR_EINVAL
    assert L.cr_pages_free(c, FAKE, 1 << 16, FAKE, 1 << 16, FAKE, None) == B.CR_EINVAL
    assert L.cr_attn_prompt(ctypes.byref(_prompt(total_k=0x7FFFFC00)), FAKE, 1 << 50, FAKE, None) == B.CR_EINVAL
    wide = _shared(prefix_width=(1 << 27) - 64, own_width=0)  # 2^31 - 1,024 tokens
    assert L.cr_attn_shared(c, ctypes.byref(wide), FAKE, 1 << 50, FAKE, None) == B.CR_EINVAL
    many = _prompt(heads_q=1024, heads_kv=1024, batch=1 << 15, total_q=1 << 20, total_k=1 << 30)  # 2^25 workgroups
    assert L.cr_attn_prompt(ctypes.byref(many), FAKE, 1 << 50, FAKE, None) == B.CR_EINVAL


def test_packed_arguments_are_the_structures():
    v = [(1, 8, 2, 128, 5, 1, 70, 90, 0.25), [(11 * i, 8 * i, 16 * i) for i in range(1, 5)], (3, 4, 5)]
    a = B.CrAttnPromptArgs(*v[0], *v[1], *v[2])
    assert B.PROMPT_ARGS.pack(*v[0], *(x for r in v[1] for x in r), *v[2]) == bytes(a)
    s = (8, 1, 5, 2, 70, 9, 4, 0.5)
    b = B.CrAttnSharedArgs(*s, *v[1][:2], *range(3, 10))
    assert B.SHARED_ARGS.pack(*s, *(x for r in v[1][:2] for x in r), *range(3, 10)) == bytes(b)
    assert B.ROWS.pack(*v[1][0]) == bytes(B.CrRows(*v[1][0]))
