"""Calls around the step at the edges of what they take."""
import numpy as np
import pytest
import torch

import engine_ref as ref
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


def test_spans_without_tokens():
    """Positions, slots and sequences of ranges whose tokens are not given."""
    from paper_2609_20186_amd import binding as sd
    say("[spans] without tokens")
    B, Lmax, page, most = 7, 90, 16, 6
    rng = np.random.default_rng(5)
    table = rng.integers(0, 1000, (B, most)).astype(np.int32)
    held = rng.integers(0, most + 1, B).astype(np.int32)
    begin = rng.integers(-2, 60, B).astype(np.int32)
    end = rng.integers(0, Lmax + 20, B).astype(np.int32)
    cu, rec = ref.spans(begin, end, np.zeros((B, Lmax), np.int32), table, held, page, 1 << 40)
    dev = [torch.from_numpy(x).cuda() for x in (begin, end, table, held)]
    n = len(rec) + 3
    i32 = dict(dtype=torch.int32, device="cuda")
    c = torch.full((B + 1,), -7, **i32)
    slots = torch.full((n,), -7, dtype=torch.int64, device="cuda")
    pos, seq = torch.full((n,), -7, **i32), torch.full((n,), -7, **i32)
    sd.switchsd_span_slots(dev[0], dev[1], None, dev[2], dev[3], page, c, slots, pos, None, seq,
                           Lmax=Lmax)
    np.testing.assert_array_equal(c.cpu().numpy(), cu)
    want = np.array(rec, np.int64).reshape(-1, 4)
    for j, t in ((0, slots), (1, pos), (3, seq)):
        np.testing.assert_array_equal(t[:len(rec)].cpu().numpy(), want[:, j])
        assert bool((t[len(rec):] == -7).all())


def test_compact_without_slots():
    """Slots that are missing or of another rank are refused by name."""
    from paper_2609_20186_amd import binding as sd
    say("[compact] without slots")
    cache = torch.zeros((2, 8, 4), device="cuda")
    i32 = dict(dtype=torch.int32, device="cuda")
    par, one = torch.full((1, 3), -1, **i32), torch.ones(1, **i32)
    for slots in (None, torch.zeros(3, dtype=torch.int64, device="cuda")):
        with pytest.raises(ValueError, match="slots must be"):
            sd.switchsd_compact_cache(cache, slots, par, one, one)


def test_sizes_beyond_32_bits():
    """A vocabulary and rows of bytes whose low 32 bits are a valid size are
    refused; packed outputs of more than 2^32 entries are filled."""
    from paper_2609_20186_amd import binding as sd
    say("[binding] sizes beyond 32 bits")
    i32 = dict(dtype=torch.int32, device="cuda")
    one = torch.ones(1, **i32)
    x = torch.empty((1, 1, 2 ** 32 + 64), dtype=torch.bfloat16, device="cuda")
    with pytest.raises(ValueError, match="V = 4294967360 does not fit"):
        sd.build_logits_args(x, one.view(1, 1), None, one)
    del x
    cache = torch.empty((1, 2, 2 ** 32 + 64), dtype=torch.uint8, device="cuda")
    with pytest.raises(ValueError, match="row_bytes = 4294967360 does not fit"):
        sd.switchsd_compact_cache(cache, torch.zeros((1, 2), dtype=torch.int64, device="cuda"),
                                  torch.zeros((1, 2), **i32), one, one)
    del cache
    B, n = 4, 20
    big = torch.empty(2 ** 32 + 5, **i32)
    big[:B * n + 9] = -7
    cu = torch.full((B + 1,), -7, **i32)
    sd.switchsd_span_slots(torch.zeros(B, **i32), torch.full((B,), n, **i32),
                           torch.zeros((B, 64), **i32), None, None, 16, cu, None, big, None, None)
    assert cu.tolist() == [0, 20, 40, 60, 80]
    assert torch.equal(big[:B * n].view(B, n), torch.arange(n, **i32).expand(B, n))
    assert bool((big[B * n:B * n + 9] == -7).all())
