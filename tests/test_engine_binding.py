"""What the binding of the calls around the step refuses before it looks at a
device (no GPU needed)."""
import pytest
import torch

from paper_2609_20186_amd import binding as sd


def i32(*shape):
    return torch.zeros(shape, dtype=torch.int32)


def spans(tokens, outs, **kw):
    """Two sequences; outs = slots, positions, packed, seq."""
    sd.switchsd_span_slots(i32(2), i32(2), tokens, i32(2, 4), i32(2), 16, i32(3), *outs, **kw)


@pytest.mark.parametrize("at", range(4))
@pytest.mark.parametrize("shape", [(2, 5), (1, 1, 5), ()])
def test_packed_outputs_have_one_axis(at, shape):
    """Of outputs [B, m] only the first B entries would be written."""
    outs = [None] * 4
    outs[at] = torch.zeros(shape, dtype=torch.int64 if at == 0 else torch.int32)
    with pytest.raises(ValueError, match=r"\[capacity\]"):
        spans(i32(2, 9), outs)
