"""Calls around the step at the edges of what they take."""
import pytest
import torch

from gpu_helpers import say

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2609_20186_amd import binding  # noqa: F401


def test_packed_outputs_of_two_axes_are_refused():
    from paper_2609_20186_amd import binding as sd
    say("[spans] outputs of two axes")
    B, n = 4, 20
    i32 = dict(dtype=torch.int32, device="cuda")
    begin, end = torch.zeros(B, **i32), torch.full((B,), n, **i32)
    tokens, cu = torch.zeros((B, 64), **i32), torch.full((B + 1,), -7, **i32)
    pos = torch.full((B, n), -7, **i32)
    with pytest.raises(ValueError, match="capacity"):
        sd.switchsd_span_slots(begin, end, tokens, None, None, 16, cu, None, pos, None, None)
    assert bool((pos == -7).all()) and bool((cu == -7).all())
    sd.switchsd_span_slots(begin, end, tokens, None, None, 16, cu, None, pos.view(-1), None, None)
    assert torch.equal(pos, torch.arange(n, **i32).expand(B, n))
