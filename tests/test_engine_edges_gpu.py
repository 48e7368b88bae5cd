"""Calls around the step at the edges of what they take."""
import numpy as np
import pytest
import torch

import engine_ref as ref
from gpu_helpers import say
from test_processed_gpu import check_rows, device_args, gpu_verify, make

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


@pytest.mark.parametrize("src", ["bf16", "f32"])
@pytest.mark.parametrize("R", [2, 17])
def test_largest_vocabulary(src, R):
    """V = 2^26: tokens at either end are penalised, biased, forbidden and
    chosen; all others pass as they are."""
    from paper_2609_20186_amd import binding as sd
    say(f"[process] V = 2^26 {src} {R}")
    V, words = 1 << 26, 1 << 21
    i32 = dict(dtype=torch.int32, device="cuda")
    f32 = dict(dtype=torch.float32, device="cuda")
    x = torch.zeros((1, R, V), dtype=ref.TYPES[src], device="cuda")
    x[0, :, V - 1], x[0, :, V - 2], x[0, :, 3] = 8.0, 7.0, 7.5
    x[0, R - 1, V - 3] = 7.25
    allowed = torch.full((1, R, words), -1, **i32)
    allowed[0, R - 1, words - 1] = 0x3FFFFFFF                 # not the last two tokens
    tokens = torch.tensor([[V - 1, 3, 5, V - 1]], **i32)
    args = sd.build_logits_args(
        x, torch.full((1, R), -1, **i32), None, torch.full((1,), R, **i32), tokens,
        torch.tensor([4], **i32), None, None, torch.tensor([0.5], **f32), None,
        torch.tensor([[V - 2, V, 7]], **i32), torch.tensor([[0.75, 9.0, -1.0]], **f32), allowed)
    want = x.clone()
    want[0, :, V - 1], want[0, :, 3], want[0, :, 5] = 7.0, 7.0, -0.5    # 8 - 2 / 2, 7.5 - 1 / 2
    want[0, :, V - 2], want[0, :, 7] = 7.75, -1.0
    want[0, R - 1, V - 2:] = -float("inf")
    out = torch.full_like(x, 77.0)
    sd.switchsd_process_logits(args, out)
    assert torch.equal(out, want)
    del want, out
    o = [torch.full(s, -9, **i32) for s in ((1,), (1,), (1,), (1, R), (1, R))]
    ws = sd.alloc_workspace(1, R)
    sd.switchsd_verify_processed(args, *o, ws)
    assert o[4].tolist() == [[V - 2] * (R - 1) + [V - 3]]
    assert o[0].tolist() == [0] and o[2].tolist() == [V - 2]
    assert int(ws.count_nonzero()) == 0


@pytest.mark.parametrize("rho", [0.0, -0.0, float("inf"), -1.5, float("nan"), 1e-45])
def test_penalties_that_are_not_ordinary(rho):
    """A repetition penalty of zero, infinity, NaN or below zero, and infinite
    frequencies and presences, follow the arithmetic."""
    from paper_2609_20186_amd import binding as sd
    say(f"[process] repetition {rho}")
    for src in ("bf16", "f16", "f32"):
        d = make(4, 5, 1201, 60, seed=21, src=src, draft="tree")
        d["repetition"][:] = rho
        d["frequency"][2], d["presence"][3] = np.inf, -np.inf
        d["lengths"][1] = 60
        o = torch.full(d["logits"].shape, 77.0, dtype=ref.TYPES[src], device="cuda")
        sd.switchsd_process_logits(device_args(d), o)
        check_rows(d, o, ref.TYPES[src], 77.0)
        want = ref.greedy(d, ref.processed(d, np.float32))
        got, _ = gpu_verify(device_args(d))
        for name, t in got.items():
            np.testing.assert_array_equal(t.cpu().numpy(), want[name], err_msg=name)


def test_in_place_beyond_32_bits_leaves_other_rows():
    """In place on the last sequence of more than 2^31 logits: where a 32-bit
    offset would wrap to, nothing changes."""
    from paper_2609_20186_amd import binding as sd
    say("[process] in place, large offsets")
    B, R, V = 35, 32, 2000000
    i32 = dict(dtype=torch.int32, device="cuda")
    x = torch.full((B, R, V), 1.0, dtype=torch.bfloat16, device="cuda")
    assert x.numel() > 2 ** 31
    dn = torch.ones(B, **i32)
    dn[B - 1] = R
    lengths = torch.zeros(B, **i32)
    lengths[B - 1] = 3
    tokens = torch.tensor([[0, V - 1, 77]], **i32).repeat(B, 1)
    args = sd.build_logits_args(x, torch.full((B, R), -1, **i32), None, dn, tokens, lengths,
                                presence=torch.full((B,), 0.5, device="cuda"))
    sd.switchsd_process_logits(args, x)
    assert bool((x[:B - 1] == 1.0).all())
    want = torch.ones(V, device="cuda")
    want[tokens[0].long()] = 0.5
    assert bool((x[B - 1].float() == want).all())
