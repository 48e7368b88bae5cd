"""Sizes and temperatures at the ends of what the log probabilities take (no GPU)."""
import ctypes

import pytest

from paper_2609_20186_amd import binding as sd
from test_attention_abi import P, logprob_args


def size(**kw):
    return sd.logprob_workspace_bytes(logprob_args(logits=None, tokens=None, **kw))


@pytest.mark.parametrize("kw", [
    dict(B=0), dict(B=-1), dict(R=0), dict(R=1025), dict(R=1025, accept_node=P), dict(V=0), dict(V=(1 << 26) + 1),
    dict(B=1 << 14, R=1024), dict(logits_type=3), dict(logits_type=-1)])
def test_no_workspace_for_what_is_refused(kw):
    """One row of the largest vocabularies is cut; the same with a size or a type that the
    calls refuse is not."""
    assert size(**{**dict(B=1, R=1, V=1 << 26), **kw}) == 0


def test_workspace_at_the_largest_sizes():
    for type in range(3):
        assert size(B=1, R=1, V=1 << 26, logits_type=type) > 0
    assert size(B=1, R=1024, V=1 << 26) == 0        # as many rows as are held at once
    assert size(B=1, R=512, V=1 << 26) > 0
    assert sd.lib.switchsd_logprob_workspace_bytes(None) == 0


@pytest.mark.parametrize("T", [3.0e-39, 3.5e-39, 4.2e-39])
def test_temperatures_whose_factor_has_no_32_bits(T):
    """1 / T is a finite number here, log2(e) / T, which the kernels multiply with, is not."""
    a = logprob_args(temperature=T)
    assert 1 / a.temperature < 3.4e38 < 1.4426 / a.temperature
    assert sd.lib.switchsd_token_logprobs(ctypes.byref(a), P, None, None, None, 0, None, None,
                                          None) == -1
    assert sd.lib.switchsd_token_logprobs_grad(ctypes.byref(a), P, None, P, None, P + 4096,
                                               None) == -1
