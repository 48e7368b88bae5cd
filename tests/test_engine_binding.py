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


def test_missing_workspace():
    """None is refused as every other missing tensor is."""
    a = sd.LogitsArgs()
    a.shape, a.device = (2, 3, 8), sd._current_device()
    with pytest.raises(ValueError, match="workspace is required"):
        sd.switchsd_verify_processed(a, i32(2), i32(2), i32(2), i32(2, 3), i32(2, 3), None)
    a = sd.PageArgs()
    a.device = sd._current_device()
    with pytest.raises(ValueError, match="workspace is required"):
        sd.switchsd_page_plan(a, None)
    with pytest.raises(ValueError, match="workspace must be a device tensor"):
        sd.switchsd_page_plan(a, torch.zeros(1024, dtype=torch.uint8))


def test_spans_ranks():
    outs = [torch.zeros(5, dtype=torch.int64), None, None, None]
    with pytest.raises(ValueError, match="tokens must be"):
        spans(i32(9), outs)
    for table, held in ((None, i32(2)), (i32(8), i32(2)), (i32(2, 4), None)):
        with pytest.raises(ValueError, match="slots need table"):
            sd.switchsd_span_slots(i32(2), i32(2), i32(2, 9), table, held, 16, i32(3), *outs)


HUGE = 2 ** 32 + 16                     # 16 in its low 32 bits


def huge(*shape, dtype=torch.int32):
    """A tensor of that shape over one element."""
    return torch.zeros(1, dtype=dtype).expand(shape)


@pytest.mark.parametrize("call", [
    lambda: sd.build_logits_args(huge(1, 1, HUGE, dtype=torch.bfloat16), i32(1, 1), None, i32(1)),
    lambda: sd.build_logits_args(huge(HUGE, 1, 8, dtype=torch.float32), i32(1, 1), None, i32(1)),
    lambda: sd.build_page_args(i32(2), None, i32(2), HUGE, 4, i32(2, 3), i32(2), i32(9), i32(2),
                               None, None, i32(2), R=2),
    lambda: sd.build_page_args(i32(2), None, i32(2), 9, HUGE, i32(2, 3), i32(2), i32(9), i32(2),
                               None, None, i32(2), R=2),
    lambda: sd.build_page_args(i32(2), None, i32(2), 9, 4, huge(2, HUGE), i32(2), i32(9), i32(2),
                               None, None, i32(2), R=2),
    lambda: sd.build_page_args(i32(2), None, i32(2), 9, 4, i32(2, 3), i32(2), i32(9), i32(2),
                               None, None, i32(2), R=HUGE),
    lambda: sd.switchsd_span_slots(i32(2), i32(2), huge(2, HUGE), None, None, 16, i32(3), None,
                                   i32(5), None, None),
    lambda: sd.switchsd_span_slots(i32(2), i32(2), i32(2, 9), None, None, HUGE, i32(3), None,
                                   i32(5), None, None),
    lambda: sd.switchsd_span_slots(i32(2), i32(2), i32(2, 9), None, None, 16 - 2 ** 32, i32(3),
                                   None, i32(5), None, None),
    lambda: sd.switchsd_span_slots(i32(2), i32(2), None, None, None, 16, i32(3), None,
                                   i32(5), None, None, Lmax=HUGE),
])
def test_sizes_beyond_32_bits(call):
    """ctypes passes the low 32 bits on: 2^32 + 16 would be taken for 16."""
    assert sd.ctypes.c_int32(HUGE).value == 16
    with pytest.raises(ValueError, match="does not fit 32 bits"):
        call()


def test_sizes_that_fit_reach_the_library():
    """A negative size is not the binding's to refuse."""
    sd._sizes(B=-2 ** 31, R=-3, V=2 ** 31 - 1)
    for n in (2 ** 31, -2 ** 31 - 1, HUGE):
        with pytest.raises(ValueError, match="does not fit 32 bits"):
            sd._sizes(V=n)
