"""What only the device sees reaches its caller, with and without a workspace."""
import pytest
import torch

from paper_2608_19677_amd import binding as B
from paper_2608_19677_amd import serve

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
