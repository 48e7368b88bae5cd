"""Every compiled form of the attention where its work is cut: both types, 16- and 8-bit
caches, three widths, both forms, the join of one row and of four at once; and item counts
on both sides of those from which each work-group takes a whole item, in long tables, so that
the device decides."""
import math

import numpy as np
import pytest
import torch

import attention_ref as ref
from test_attention_gpu import check, make, run

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2609_20186_amd import binding  # noqa: F401


def host(a):
    """By the host's rules: rows of a work-group, items there can be, whether the context is
    so short that nothing is cut, rows that the join takes at once."""
    G = a["Hq"] // a["Hkv"]
    tile = 32 if a["R"] * G <= 32 else 128
    items = a["B"] * -(-a["R"] * G // tile)
    if "cu" in a:
        items = min(items, a["rows"] * G // tile + a["B"])
    items *= a["Hkv"]
    short = min(a["Lmax"] + a["R"], a["table"].shape[1] * a["page"]) <= 1024
    sets, rows = 256 // (a["D"] // 4), min(a["R"] * G, tile)
    few = min(items, 4096 if tile == 32 else 1024)
    limit, parts = 256 if a["D"] == 256 else 512, 1
    while parts < sets and parts * few < limit and few * -(-rows * parts // sets) < 1024:
        parts *= 2
    return tile, items, short, 4 if few * -(-rows * parts // sets) >= 8192 else 1


def live_items(a):
    """Items that there are."""
    tile, _, _, _ = host(a)
    G = a["Hq"] // a["Hkv"]
    return a["Hkv"] * sum(-(-ref.rows_of(a, b)[1] * G // tile) for b in range(a["B"]))


TYPES = [("bf16", "bf16"), ("f16", "f16"), ("bf16", "e4m3"), ("f16", "e4m3")]


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("type,cache", TYPES)
@pytest.mark.parametrize("R,Hq,mask", [(1, 2, None), (5, 4, None), (5, 4, "tree"), (30, 8, None),
                                       (30, 8, "tree")])
def test_cut(D, type, cache, R, Hq, mask):
    """Odd numbers of blocks, so that a work-group ends one item and begins another; a second
    call gives the same bits."""
    a = make([1300, 700, 1501, 65], [R, R, max(1, R - 2), 1], Hq=Hq, Hkv=2, D=D, page=16,
             type=type, cache=cache, mask=mask, seed=R)
    tile, _, short, rows = host(a)
    assert not short and tile == (32 if R < 30 else 128) and rows == 1
    out, lse, args, ws = run(a)
    check(a, out, lse, f"{R} rows, {Hq} heads of {D}, {type} {cache}, mask {mask}")
    again = run(a, ws=ws, args=args)
    assert torch.equal(out.view(torch.int16), again[0].view(torch.int16))
    assert torch.equal(lse.view(torch.int32), again[1].view(torch.int32))


def shared(lengths, new, Hq, Hkv, D, R, type="bf16", mask=None, seed=0, pages=120, page=16,
           long=1600):
    """Many sequences over a few pages, which they share, with tables for `long` positions."""
    rng = np.random.default_rng(seed)
    g = torch.Generator().manual_seed(seed)
    lengths, new = np.asarray(lengths, np.int32), np.asarray(new, np.int32)
    B = len(lengths)
    a = dict(B=B, R=R, Hq=Hq, Hkv=Hkv, D=D, page=page, type=type, cache=type, Lmax=long,
             n_slots=pages * page, scale=D ** -0.5, lengths=lengths, dn=new, rows=B * R,
             k_scale=None, v_scale=None)
    a["table"] = rng.integers(0, pages, (B, -(-(long + R) // page))).astype(np.int32)
    a["held"] = np.where(lengths > 0, -(-(lengths - 1 + new) // page), 0).astype(np.int32)
    kind = ref.HALF[type]
    q = torch.randn(B * R, Hq, D, generator=g) * 1.5
    for b in range(B):
        n = int(new[b]) if lengths[b] > 0 else 0
        q[b * R + n:(b + 1) * R] = math.nan
    a["q"] = q.to(kind).cuda()
    for name in ("k_cache", "v_cache"):
        a[name] = torch.randn(a["n_slots"], Hkv, D, generator=g).to(kind).cuda()
    if mask is not None:
        a["mask"] = rng.integers(0, 2 ** 32, (B * R, (R + 31) // 32), dtype=np.uint64).astype(
            np.uint32)
    return a


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("type", ["bf16", "f16"])
@pytest.mark.parametrize("mask", [None, "random"])
def test_join_of_four_rows(D, type, mask):
    """As many items as there can be without all of them being whole; most are short, some
    cut, of tiles that are full and of such that end within the four rows."""
    # up to 32 rows of 128 heads of the cache, one sequence without rows
    B = 32
    L, n = np.full(B, 40), np.full(B, 1)
    L[[0, 3, 9]], n[[0, 3, 9]] = [1550, 1200, 900], [32, 3, 6]
    L[5] = 0
    a = shared(L, n, 128, 128, D, 32, type=type, mask=mask, seed=D)
    assert host(a) == (32, 4096, False, 4) and live_items(a) < 4096
    check(a, *run(a)[:2], f"32 rows, 128 heads of {D}, {type}, mask {mask}")
    # up to 512 rows of 16 heads of the cache; without a mask the second sequence's tiles see
    # more and more
    B = 16
    L, n = np.full(B, 90), np.full(B, 20)
    L[[0, 1, 7]], n[[0, 1, 7]] = [1500, 500, 1100], [70, 256, 31]
    a = shared(L, n, 32, 16, D, 256, type=type, mask=mask, seed=D + 1)
    assert host(a) == (128, 1024, False, 4) and live_items(a) < 1024
    check(a, *run(a)[:2], f"256 rows, 32 heads of {D}, {type}, mask {mask}")


@pytest.mark.parametrize("cache", ["bf16", "f16"])
@pytest.mark.parametrize("finished", [False, True])
@pytest.mark.parametrize("R,Hq,Hkv,B,whole", [(3, 128, 128, 32, 4096), (20, 32, 16, 64, 1024)])
def test_whole_items_by_the_device(cache, finished, R, Hq, Hkv, B, whole):
    """Exactly as many items as are taken whole, and one sequence fewer, which is cut."""
    rng = np.random.default_rng(R)
    L, n = rng.integers(1, 90, B), rng.integers(1, R + 1, B)
    L[[0, 4]], n[[0, 4]] = [1590, 1100], R
    if finished:
        L[B // 2] = 0
    a = shared(L, n, Hq, Hkv, 64, R, type=cache, seed=R)
    tile, items, short, _ = host(a)
    assert items == whole and not short
    assert live_items(a) == whole - (Hkv if finished else 0)
    check(a, *run(a)[:2], f"{live_items(a)} items of {tile} rows")
