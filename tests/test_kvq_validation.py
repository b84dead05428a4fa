"""Refusals of the 8-bit cache's calls and of rotary positions: every malformed call returns its code on the host before
anything is enqueued (no GPU, no pointer is dereferenced), and the wrappers refuse what does not fit. Frequencies against
their formulas."""
import ctypes
import math

import pytest
import torch

from paper_2608_19677_amd import binding as B
from paper_2608_19677_amd import serve

from test_serve_validation import BAD_SHARED, FAKE, L, _rows, _shared  # noqa: F401

# As in test_serve_validation.py: a regression would launch a kernel on a fake address where a GPU is.
pytestmark = pytest.mark.skipif(torch.cuda.is_available(), reason="host-side validation tests run without a GPU")


def _cache(**kw):
    f = dict(dtype=B.CR_BF16, code=B.CR_E4M3, heads=2, dim=128, page_tokens=16, block_tokens=8, num_pages=40, layers=2, k=FAKE, v=FAKE,
             layer_stride=40 * 4096, page_stride=4096, head_stride=2048, token_stride=128, scale=FAKE, refs=FAKE)
    f.update(kw)
    return B.CrKvqCache(**f)


BAD_CACHES = [dict(dtype=2), dict(code=2), dict(heads=0), dict(heads=1025), dict(dim=32), dict(dim=96), dict(page_tokens=0), dict(page_tokens=24),
              dict(page_tokens=2048), dict(block_tokens=0), dict(block_tokens=32), dict(block_tokens=3), dict(page_tokens=512, block_tokens=256),
              dict(num_pages=0), dict(num_pages=(1 << 26) + 1), dict(layers=0), dict(layers=1025), dict(k=None), dict(v=FAKE + 8),
              dict(page_stride=4088), dict(head_stride=-16), dict(token_stride=1 << 31), dict(layer_stride=24), dict(scale=None), dict(scale=FAKE + 1)]


@pytest.mark.parametrize("kw", BAD_CACHES, ids=[str(k) for k in BAD_CACHES])
def test_every_call_refuses_a_bad_cache(L, kw):  # noqa: F811
    c = ctypes.byref(_cache(**kw))
    assert L.cr_kvq_extend(c, None, FAKE, 1, FAKE, 4, FAKE, 1 << 20, FAKE, None) == B.CR_EINVAL
    assert L.cr_kvq_fork(c, FAKE, 1, 4, FAKE, FAKE, 1, FAKE + 64, 4, FAKE, 1 << 20, FAKE, None) == B.CR_EINVAL
    assert L.cr_kvq_free(c, FAKE, 4, FAKE, 1, FAKE, None) == B.CR_EINVAL
    assert L.cr_kvq_compact(c, FAKE, FAKE, 1, 4, FAKE, FAKE, FAKE, 1 << 20, FAKE, None) == B.CR_EINVAL
    assert L.cr_kvq_copy(c, FAKE, FAKE, 1, FAKE, None) == B.CR_EINVAL
    assert L.cr_kvq_append(c, ctypes.byref(_tokens()), FAKE, None) == B.CR_EINVAL
    assert L.cr_kvq_read(c, ctypes.byref(_tokens()), FAKE, None) == B.CR_EINVAL
    assert L.cr_kvq_attn(c, ctypes.byref(_shared()), FAKE, 1 << 40, FAKE, None) == B.CR_EINVAL


def test_page_calls_refuse(L):  # noqa: F811
    c = ctypes.byref(_cache())
    need = B.cr_pages_workspace_bytes(40, 1)
    assert L.cr_kvq_extend(c, None, FAKE, 1, FAKE, 4, FAKE, need - 1, FAKE, None) == B.CR_ESIZE
    assert L.cr_kvq_extend(c, None, FAKE, 1 << 16, FAKE, 1 << 16, FAKE, 1 << 40, FAKE, None) == B.CR_EINVAL
    assert L.cr_kvq_extend(c, None, None, 0, None, 4, FAKE, need, FAKE, None) == B.CR_OK
    assert L.cr_kvq_fork(c, FAKE, 1, 4, FAKE, FAKE, 1, FAKE, 4, FAKE, need, FAKE, None) == B.CR_EINVAL  # child is table
    assert L.cr_kvq_fork(c, FAKE, 1, 4, FAKE, FAKE, 1 << 24, FAKE + 64, 4, FAKE, 0, FAKE, None) == B.CR_EINVAL
    assert L.cr_kvq_free(c, None, 4, FAKE, 1, FAKE, None) == B.CR_EINVAL
    assert L.cr_kvq_compact(c, FAKE, FAKE, 1, 4, FAKE, FAKE, FAKE, B.cr_pages_workspace_bytes(40, 0) - 4, FAKE, None) == B.CR_ESIZE
    assert L.cr_kvq_copy(c, FAKE, None, 1, FAKE, None) == B.CR_EINVAL
    assert L.cr_kvq_copy(c, None, None, 0, FAKE, None) == B.CR_OK


def _tokens(**kw):
    f = dict(layer=0, total=1, n=1, width=4, k=_rows(), v=_rows(), off=FAKE, length=FAKE, table=FAKE)
    f.update(kw)
    return B.CrKvqTokens(**f)


BAD_TOKENS = [dict(layer=2), dict(k=_rows(token=100)), dict(v=_rows(FAKE + 2)), dict(v=_rows(head=-8)), dict(off=None), dict(length=None), dict(n=0),
              dict(table=None), dict(total=1 << 31), dict(n=(1 << 24) + 1), dict(width=(1 << 28) + 1)]


@pytest.mark.parametrize("call", ["cr_kvq_append", "cr_kvq_read"])
@pytest.mark.parametrize("kw", BAD_TOKENS, ids=[next(iter(k)) + str(i) for i, k in enumerate(BAD_TOKENS)])
def test_tokens_refuse(L, call, kw):  # noqa: F811
    assert getattr(L, call)(ctypes.byref(_cache()), ctypes.byref(_tokens(**kw)), FAKE, None) == B.CR_EINVAL


def test_more_spans_than_are_counted(L):  # noqa: F811
    """Spans of 8 tokens (blocks of 8, rows of 128 elements) times 2 heads: 2^32 of them and more are refused."""
    c = _cache(heads=1024)
    assert L.cr_kvq_append(ctypes.byref(c), ctypes.byref(_tokens(total=(1 << 31) - 1)), FAKE, None) == B.CR_EINVAL


def test_tokens_of_nothing(L):  # noqa: F811
    c, none = ctypes.byref(_cache()), ctypes.byref(_tokens(total=0, n=0, width=0, k=_rows(None), v=_rows(None), off=None, length=None, table=None))
    for f in (L.cr_kvq_append, L.cr_kvq_read):
        assert f(c, none, FAKE, None) == B.CR_OK
        assert f(c, none, None, None) == B.CR_EINVAL and f(c, None, FAKE, None) == B.CR_EINVAL
    # rows to read into may be left out, rows to write may not
    assert L.cr_kvq_append(c, ctypes.byref(_tokens(v=_rows(None))), FAKE, None) == B.CR_EINVAL
    assert L.cr_kvq_append(c, ctypes.byref(_tokens(k=_rows(None))), FAKE, None) == B.CR_EINVAL


@pytest.mark.parametrize("kw", BAD_SHARED, ids=[next(iter(k)) + str(i) for i, k in enumerate(BAD_SHARED)])
def test_attention_refuses(L, kw):  # noqa: F811
    assert L.cr_kvq_attn(ctypes.byref(_cache()), ctypes.byref(_shared(**kw)), FAKE, 1 << 50, FAKE, None) == B.CR_EINVAL


def test_attention_sizes(L):  # noqa: F811
    c, a = _cache(), _shared()
    need = B.cr_kvq_attn_workspace_bytes(c, a)
    assert need >= 2 * 3 * 8 * (128 + 1) * 4
    assert L.cr_kvq_attn(ctypes.byref(c), ctypes.byref(a), FAKE, need - 1, FAKE, None) == B.CR_ESIZE
    assert L.cr_kvq_attn(ctypes.byref(c), ctypes.byref(a), FAKE + 4, need, FAKE, None) == B.CR_EINVAL
    assert L.cr_kvq_attn(ctypes.byref(c), ctypes.byref(a), FAKE, need, None, None) == B.CR_EINVAL
    assert L.cr_kvq_attn(ctypes.byref(c), ctypes.byref(_shared(total_q=0)), None, 0, FAKE, None) == B.CR_OK
    assert B.cr_kvq_attn_workspace_bytes(_cache(code=7), a) == 0


def _rotary(**kw):
    f = dict(dtype=B.CR_F16, heads_q=8, heads_k=2, dim=128, rotated=64, layout=B.CR_ROTARY_PAIRS, total=5, magnitude=1.0, q=_rows(), k=_rows(),
             q_out=_rows(), k_out=_rows(), positions=FAKE, freq=FAKE)
    f.update(kw)
    return B.CrRotaryArgs(**f)


BAD_ROTARY = [dict(dtype=2), dict(heads_q=0), dict(heads_q=1025), dict(heads_k=1025), dict(dim=96), dict(rotated=0), dict(rotated=8), dict(rotated=40),
              dict(rotated=144), dict(layout=2), dict(total=1 << 28), dict(magnitude=math.inf), dict(magnitude=math.nan), dict(q=_rows(None)),
              dict(k=_rows(FAKE + 4)), dict(q_out=_rows(token=9)), dict(k_out=_rows(head=-8)), dict(positions=None), dict(positions=FAKE + 2),
              dict(freq=None), dict(freq=FAKE + 4)]


@pytest.mark.parametrize("kw", BAD_ROTARY, ids=[next(iter(k)) + str(i) for i, k in enumerate(BAD_ROTARY)])
def test_rotary_refuses(L, kw):  # noqa: F811
    assert L.cr_rotary(ctypes.byref(_rotary(**kw)), None) == B.CR_EINVAL


def test_rotary_over_itself_with_other_strides(L):  # noqa: F811
    other = _rows(FAKE + 4096)
    for kw in (dict(q_out=_rows(head=256), k_out=other), dict(q_out=other, k_out=_rows(token=2048))):
        assert L.cr_rotary(ctypes.byref(_rotary(**kw)), None) == B.CR_EINVAL


def test_rotary_of_nothing(L):  # noqa: F811
    assert L.cr_rotary(ctypes.byref(_rotary(total=0, q=_rows(None), positions=None)), None) == B.CR_OK
    assert L.cr_rotary(None, None) == B.CR_EINVAL


def test_struct_layouts_match_header(L):  # noqa: F811
    assert ctypes.sizeof(B.CrKvqCache) == 8 * 4 + 2 * 8 + 4 * 8 + 2 * 8
    assert ctypes.sizeof(B.CrRotaryArgs) == 8 * 4 + 4 * 24 + 2 * 8
    t = (1, 70, 5, 9, (11, 8, 16), (22, 24, 32), 3, 4, 5)
    assert B.TOKENS_ARGS.pack(*t[:4], *t[4], *t[5], *t[6:]) == bytes(B.CrKvqTokens(*t))
    v = [(1, 8, 2, 128, 64, 1, 70, 0.25), [(11 * i, 8 * i, 16 * i) for i in range(1, 5)], (3, 4)]
    assert B.ROTARY_ARGS.pack(*v[0], *(x for r in v[1] for x in r), *v[2]) == bytes(B.CrRotaryArgs(*v[0], *v[1], *v[2]))


def test_wrappers_refuse_tensors_that_do_not_fit():
    k = torch.zeros(1, 4, 2, 16, 64, dtype=torch.uint8).view(torch.float8_e4m3fn)
    scale, refs = torch.zeros(1, 4, 2, 2, 2, dtype=torch.uint8), torch.zeros(4, dtype=torch.int32)
    with pytest.raises(B.CrError, match="device tensors"):
        serve.QuantPagePool(k, k, scale, refs)
    with pytest.raises(ValueError, match="order"):
        serve.QuantPagePool(k, k, scale, refs, order="page")
    with pytest.raises(B.CrError, match="alike"):
        serve.QuantPagePool(k, k[..., :32], scale, refs)
    with pytest.raises(B.CrError, match="whole blocks"):
        serve.QuantPagePool.empty(1, 4, 2, 16, 64, block_tokens=32, device="cpu")
    with pytest.raises(B.CrError, match="device tensors"):
        serve.Rotary(64, device="cpu")
    with pytest.raises(ValueError, match="layout"):
        serve.Rotary(64, layout="thirds")
    with pytest.raises(ValueError, match="scaling"):
        serve.Rotary(64, scaling="squared")
    for dim, rotated in ((96, None), (64, 8), (64, 80), (128, 40), (64, 0)):
        with pytest.raises(B.CrError, match="multiple of 16"):
            serve.Rotary(dim, rotated)
    for kw in (dict(base=1.0), dict(factor=0.0), dict(base=math.inf), dict(scaling="turns"), dict(scaling="index", length=100, low=4.0, high=4.0)):
        with pytest.raises(B.CrError):
            serve.Rotary(64, **kw)
    with pytest.raises(B.CrError, match="32 finite frequencies"):
        serve.Rotary(64, frequencies=[1.0] * 31)
    with pytest.raises(B.CrError, match="magnitude"):
        serve.Rotary(64, magnitude=math.nan)


def test_frequencies():
    r, base = 64, 10000.0
    plain = serve.rotary_frequencies(r, base)
    assert plain == [base ** (-2 * i / r) for i in range(32)] and plain[0] == 1.0
    assert serve.rotary_frequencies(r, base, "linear", 4.0) == [f / 4 for f in plain]
    scaled = serve.rotary_frequencies(r, base, "base", 8.0)
    assert scaled[0] == 1.0 and math.isclose(scaled[-1], plain[-1] / 8, rel_tol=1e-12)
    assert all(a > b for a, b in zip(scaled, scaled[1:]))
    # by turns: kept from `high` on, divided up to `low`, the formula between
    n, low, high, factor = 8192, 1.0, 4.0, 8.0
    for f, g in zip(plain, serve.rotary_frequencies(r, base, "turns", factor, n, low, high)):
        t = n * f / (2 * math.pi)
        if t >= high:
            assert g == f
        elif t <= low:
            assert math.isclose(g, f / factor, rel_tol=1e-15)
        else:
            w = (t - low) / (high - low)
            assert math.isclose(g, (1 - w) * f / factor + w * f, rel_tol=1e-12)
    # by index: the pair that makes `high` turns, rounded down, is the last that stays, that of `low`, rounded up, the first divided
    got = serve.rotary_frequencies(r, base, "index", 16.0, 4096, 1.0, 32.0)
    turns = [4096 * f / (2 * math.pi) for f in plain]
    a = max(i for i, t in enumerate(turns) if t >= 32.0)
    b = min(i for i, t in enumerate(turns) if t <= 1.0)
    for i, (f, g) in enumerate(zip(plain, got)):
        w = min(1.0, max(0.0, (i - a) / (b - a)))
        assert math.isclose(g, f * (1 - w) + f / 16 * w, rel_tol=1e-12)
    for factor in (1.0, 1):
        for s in ("linear", "base", "turns", "index"):
            assert all(math.isclose(x, y, rel_tol=1e-12) for x, y in zip(serve.rotary_frequencies(r, base, s, factor, 4096), plain))


@pytest.mark.parametrize("kw", [dict(frequencies=[1e300] * 32), dict(base=1e300, scaling="base", factor=1e300)])
def test_frequencies_beyond_floats(kw):
    """Finite arguments whose turns or base pass a float's range are refused as any other argument."""
    with pytest.raises(B.CrError):
        serve.Rotary(64, **kw, device="cpu")
