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


def test_spans_without_tokens():
    """Without packed, tokens are not needed, as in the C call; Lmax then is."""
    outs = [None, i32(5), None, i32(5)]
    with pytest.raises(ValueError, match="Lmax"):
        spans(None, outs)
    with pytest.raises(ValueError, match="tokens is required"):
        spans(None, [None, None, i32(5), None], Lmax=9)
    with pytest.raises(ValueError, match="Lmax is 8"):
        spans(i32(2, 9), outs, Lmax=8)
    # complete: what is refused is that these are host tensors
    with pytest.raises(ValueError, match="begin must be a device tensor"):
        spans(None, outs, Lmax=9)
