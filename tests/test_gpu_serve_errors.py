"""What only the device sees reaches its caller, with and without a workspace."""
import pytest
import torch

from paper_2608_19677_amd import binding as B
from paper_2608_19677_amd import serve
from paper_2608_19677_amd.destination import Destination

import serve_oracle as so
from cr_check import say

pytestmark = pytest.mark.gpu


def _i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def test_prompt_without_a_workspace():
    q = torch.randn(20, 4, 64, device="cuda").to(torch.bfloat16)
    err, good, bad = _i32([0]), _i32([0, 20]), _i32([0, 21])
    say("[case] prompt attention with an error word")
    serve.attend_prompt(q, q, q, good, good, 0.1, err=err)
    assert int(err.item()) == 0
    serve.attend_prompt(q, q, q, good, bad, 0.1, err=err)
    assert int(err.item()) == B.CR_ERR_SEQ
    with pytest.raises(B.CrError, match="word of its own"):
        serve.attend_prompt(q, q, q, good, good, 0.1, err=err, ws=serve.prompt_workspace(q, q, good))


def _destination(project=None):
    return Destination(2, 50, 12, 6, layers=2, heads_q=4, heads_kv=1, dim=64, page_tokens=8, project=project)


def test_a_destination_raises_what_its_calls_report():
    d = _destination()
    d.serve([7], [33], [3])
    real = d.project

    class Short:
        """A query too few for the prompts' offsets: their attention reports it, nothing else does."""

        def __call__(self, layer, ids, lengths):
            q, k, v = real(layer, ids, lengths)
            return (q[:-1] if 9 in list(ids) else q), k, v

    d.project = Short()
    d.serve([7], [33], [4])
    say("[case] a destination's prompt attention with a row too few")
    with pytest.raises(B.CrError, match="0x10"):
        d.serve([7, 9], [33, 20], [4, 4])


def test_a_destinations_prompts():
    d = _destination()
    d.serve([7], [33], [3])
    d.serve([7], [33], [5])
    assert d.prefilled is None
    say("[case] a destination's prompt attention")
    d.serve([9, 7, 5], [50, 33, 17], [3, 4, 2])
    keys, off, out = d.prefilled
    assert keys == [9, 5] and off.tolist() == [0, 50, 67]
    q, k, v = d.project(1, keys, [50, 17])
    ref = so.flat(so.prompt(q, k, v, [0, 50, 67], [0, 50, 67], d.scale, True))
    so.check(out.reshape(-1, 64), None, ref, torch.bfloat16)


def test_a_destination_raises_what_compaction_reports():
    d = _destination()
    d.serve([7, 9], [33, 20], [3, 4])
    d.table[d.slots[9], 1] = -1  # an entry that names no page
    say("[case] a destination's compaction with an entry that names no page")
    with pytest.raises(B.CrError, match="0x20"):
        d.compact()


def test_tensors_that_require_a_gradient_are_refused():
    """Where gradients are recorded; under no_grad, or detached, the same tensors are taken."""
    q, k, v = (torch.randn(20, 4, 64, device="cuda").to(torch.bfloat16) for _ in range(3))
    off, n = _i32([0, 20]), _i32([20])
    want = serve.attend_prompt(q, k, v, off, off, 0.1)
    say("[case] gradients refused")
    for name in "qkv":
        x = dict(q=q, k=k, v=v)
        x[name] = x[name].clone().requires_grad_()
        with pytest.raises(B.CrError, match="no gradient"):
            serve.attend_prompt(x["q"], x["k"], x["v"], off, off, 0.1)
        with torch.no_grad():
            assert torch.equal(serve.attend_prompt(x["q"], x["k"], x["v"], off, off, 0.1), want)
    pool = serve.PagePool.empty(1, 4, 4, 8, 64)
    table = _i32([[2, 0, 1]])
    for x in ((k.clone().requires_grad_(), v), (k, v.clone().requires_grad_())):
        with pytest.raises(B.CrError, match="no gradient"):
            pool.append(0, *x, off, n, table)
    pool.append(0, k, v, off, n, table)
    args = (pool, 0, off, _i32([0, 1]), torch.empty((1, 0), dtype=torch.int32, device="cuda"), _i32([0]), table, n, 0.1)
    with pytest.raises(B.CrError, match="no gradient"):
        serve.attend_shared(q.clone().requires_grad_(), *args)
    with torch.inference_mode():
        assert (serve.attend_shared(q, *args).float() - want.float()).abs().max() <= 2 * so.UNIT[q.dtype] * want.float().abs().max()
    pool.k.requires_grad_()
    with pytest.raises(B.CrError, match="no gradient"):
        serve.attend_shared(q, *args)
