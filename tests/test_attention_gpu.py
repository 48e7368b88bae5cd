"""The cache store and the attention over a paged cache against the references in
64 bits, on the sizes, masks and values where they can go wrong."""
import math

import numpy as np
import pytest
import torch

import attention_ref as ref
from gpu_helpers import say

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2609_20186_amd import binding  # noqa: F401


def i32(x):
    x = np.ascontiguousarray(x)
    return torch.from_numpy(x.view(np.int32) if x.dtype == np.uint32 else x.astype(np.int32)).to(DEV)


# ------------------------------------------------------------------ inputs

def make(lengths, new, Hq=4, Hkv=2, D=128, page=16, type="bf16", cache=None, R=None, seed=0,
         packed=False, mask=None, spare=3, scale=None, qpad=0, amp=1.5, Lmax=None):
    """A state: lengths are contexts with the anchor for drafted rows (new rows
    from position length - 1 on), first positions for packed ones.  Slots that hold
    no key of a sequence are NaN, and so are rows of q that belong to none."""
    rng = np.random.default_rng(seed)
    B, new = len(lengths), np.asarray(new)
    R = int(R or max(1, new.max()))
    first = np.asarray(lengths) if packed else np.asarray(lengths) - 1
    end = np.where(np.asarray(lengths) > 0, first + new, 0) if not packed else first + new
    most = max(1, -(-int(end.max()) // page)) + 1
    n_pages = B * most + spare
    ids = rng.permutation(n_pages)[:B * most].reshape(B, most)
    held = -(-end // page)
    table = np.where(np.arange(most) < held[:, None], ids, -1).astype(np.int32)
    a = dict(B=B, R=R, Hq=Hq, Hkv=Hkv, D=D, page=page, type=type, cache=cache or type,
             Lmax=Lmax or int(max(1, max(lengths))) + 5, n_slots=n_pages * page, table=table,
             held=held.astype(np.int32), scale=D ** -0.5 if scale is None else scale)
    if packed:
        a["cu"] = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
        a["begin"], a["rows"] = first.astype(np.int32), int(new.sum()) + 3
    else:
        a["lengths"], a["dn"] = np.asarray(lengths, np.int32), new.astype(np.int32)
        a["rows"] = B * R
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(a["rows"], Hq * D + qpad, generator=g) * amp
    live = torch.zeros(a["rows"], dtype=torch.bool)
    for b in range(B):
        lo, n, _ = ref.rows_of(a, b)
        live[lo:lo + n] = True
    x[~live] = math.nan
    a["qbuf"] = x.to(ref.HALF[type]).to(DEV)
    a["q"] = a["qbuf"][:, :Hq * D].view(a["rows"], Hq, D)
    used = torch.zeros(a["n_slots"], dtype=torch.bool)
    for b in range(B):
        s = ref.slots_of(a, b, int(end[b]))
        used[s[s >= 0]] = True
    a["k_scale"] = a["v_scale"] = None
    kind = ref.HALF[type]
    if a["cache"] == "e4m3":
        kind = torch.float8_e4m3fn
        a["k_scale"] = torch.rand(Hkv, generator=g) * 0.02 + 0.01
        a["v_scale"] = torch.rand(Hkv, generator=g) * 0.02 + 0.01
    for name in ("k", "v"):
        x = torch.randn(a["n_slots"], Hkv, D, generator=g)
        if a["cache"] == "e4m3":
            x = x / a[name + "_scale"][:, None]
        x[~used] = math.nan
        a[name + "_cache"] = x.to(kind).to(DEV)
    if mask is not None:
        words = (R + 31) // 32
        if mask == "tree":
            bits = np.zeros((B, R, words * 32), bool)
            for b in range(B):
                for i in range(R):
                    if i:
                        bits[b, i] = bits[b, rng.integers(0, i)]
                    bits[b, i, i] = True
        elif mask == "none":
            bits = np.zeros((B, R, words * 32), bool)
        else:
            bits = rng.random((B, R, words * 32)) < mask
        m = (bits.reshape(B, R, words, 32).astype(np.uint64) << np.arange(32, dtype=np.uint64))
        m = m.sum(3).astype(np.uint32)
        if packed:
            rows = np.zeros((a["rows"], words), np.uint32)
            for b in range(B):
                rows[a["cu"][b]:a["cu"][b + 1]] = m[b, :new[b]]
            m = rows
        a["mask"] = m.reshape(a["rows"], words)
    return a


def run(a, out=None, lse=None, ws=None, stream=None, args=None):
    from paper_2609_20186_amd import binding as sd
    if args is None:
        where = {n: i32(a[n]) for n in (("begin", "cu") if "cu" in a else ("lengths", "dn"))}
        args = sd.build_attention_args(
            a["rows"], a["R"], a["Hq"], a["Hkv"], a["D"], a["page"], i32(a["table"]),
            i32(a["held"]), a["Lmax"], mask=None if a.get("mask") is None else i32(a["mask"]),
            scale=a["scale"], **where)
    if out is None:
        out = torch.full((a["rows"], a["Hq"], a["D"]), 77.0, dtype=ref.HALF[a["type"]], device=DEV)
        lse = torch.full((a["rows"], a["Hq"]), 77.0, device=DEV)
    if ws is None:
        ws = sd.alloc_attention_workspace(args)
        ws.fill_(0xFF)                       # NaN: whatever it holds is not used
    sc = {n: None if a[n] is None else a[n].to(DEV) for n in ("k_scale", "v_scale")}
    sd.switchsd_paged_attention(args, a["q"], a["k_cache"], a["v_cache"], out, ws, lse=lse,
                                stream=stream, **sc)
    return out, lse, args, ws


def check(a, out, lse, what=""):
    sc = {n: None if a[n] is None else a[n].numpy() for n in ("k_scale", "v_scale")}
    want = ref.attention(a, ref.f64(a["q"]), ref.f64(a["k_cache"]), ref.f64(a["v_cache"]), **sc)
    out, lse = ref.f64(out), ref.f64(lse)
    worst = 0.0
    for row in range(a["rows"]):
        if row not in want:
            assert (out[row] == 77).all() and (lse[row] == 77).all(), (what, row)
            continue
        o, low, tol, ltol = want[row]
        fine = np.isfinite(o)
        np.testing.assert_array_equal(np.isfinite(out[row]), fine, err_msg=f"{what} row {row}")
        assert (np.isnan(out[row]) == np.isnan(o))[~fine].all(), (what, row)
        d = np.abs(out[row] - o)[fine] - tol[fine]
        assert (d <= 0).all(), (what, row, float(d.max()))
        if fine.any() and tol[fine].max() > 0:
            worst = max(worst, float((np.abs(out[row] - o)[fine] / np.maximum(tol[fine], 1e-300)).max()))
        ok = np.isfinite(low)
        np.testing.assert_array_equal(np.isfinite(lse[row]), ok, err_msg=f"{what} lse {row}")
        assert (np.abs(lse[row] - low)[ok] <= ltol[ok]).all(), (what, row)
        assert (lse[row][~ok & ~np.isnan(low)] == low[~ok & ~np.isnan(low)]).all()
    say(f"{what}: largest error {worst:.2f} of its bound")


# ------------------------------------------------------------------ attention

HEADS = [(1, 1), (4, 1), (5, 5), (8, 2), (14, 2), (16, 1)]


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("type,cache", [("bf16", "bf16"), ("f16", "f16"), ("bf16", "e4m3"),
                                        ("f16", "e4m3")])
@pytest.mark.parametrize("form", ["single", "chain", "tree", "packed"])
def test_types_and_forms(D, type, cache, form):
    """Every kernel: one tile of 32 rows, several of 128, by the heads."""
    for n, (Hq, Hkv) in enumerate([(4, 2), (16, 2), (8, 1)]):
        new = {"single": [1, 1, 1], "chain": [6, 1, 5], "tree": [13, 12, 7],
               "packed": [19, 1, 33]}[form]
        a = make([70, 1, 133], new, Hq=Hq, Hkv=Hkv, D=D, page=[16, 24, 1][n], type=type,
                 cache=cache, packed=form == "packed", mask="tree" if form == "tree" else None,
                 seed=n)
        out, lse, _, _ = run(a)
        check(a, out, lse, f"{form} {Hq}/{Hkv} x {D} {type} {cache}")


@pytest.mark.parametrize("Hq,Hkv", HEADS)
@pytest.mark.parametrize("R", [1, 3, 8, 17, 40])
def test_heads(Hq, Hkv, R):
    a = make([40, 129], [R, max(1, R - 1)], Hq=Hq, Hkv=Hkv, D=64, page=64, seed=R)
    check(a, *run(a)[:2], f"{R} rows, {Hq}/{Hkv}")


@pytest.mark.parametrize("R", [1, 20, 50])
@pytest.mark.parametrize("page", [1, 16, 24])
def test_lengths_around_the_blocks(R, page):
    """Contexts that end inside, at and behind a block of 32, 64 and 128 keys."""
    L = [1, 2, 31, 32, 33, 63, 64, 65, 96, 127, 128, 129, 160, 191, 193, 255, 256, 257, 300]
    a = make(L, np.minimum(R, np.arange(1, len(L) + 1) * 7), R=R, Hq=2, Hkv=1, D=64, page=page)
    check(a, *run(a)[:2], f"{R} rows, pages of {page}")


@pytest.mark.parametrize("Hq,R,L", [(4, 1, 9000), (4, 8, 5000), (8, 8, 3001), (8, 30, 4000),
                                    (2, 300, 2500)])
def test_keys_cut_over_work_groups(Hq, R, L):
    """Long contexts and few heads: work-groups share an item's keys, and their
    partial results are joined; a second call gives the same bits."""
    for B in (1, 3):
        lengths = [L, 2, L // 3][:B]
        a = make(lengths, [R, 1, max(1, R // 2)][:B], Hq=Hq, Hkv=1, D=128, page=16, seed=B)
        out, lse, args, ws = run(a)
        check(a, out, lse, f"{B} x {R} rows over {L}")
        again = run(a, ws=ws, args=args)
        assert torch.equal(out.view(torch.int16), again[0].view(torch.int16))
        assert torch.equal(lse.view(torch.int32), again[1].view(torch.int32))


@pytest.mark.parametrize("R", [1, 5, 40])
def test_many_items(R):
    """From 2048 tiles and heads on every work-group takes a whole one."""
    B = 300
    rng = np.random.default_rng(R)
    L = rng.integers(0, 90, B)
    a = make(L, rng.integers(1, R + 1, B), R=R, Hq=16, Hkv=8, D=64, page=16, Lmax=2000)
    check(a, *run(a)[:2], f"{B} sequences of {R} rows")


@pytest.mark.parametrize("hq", [2, 8, 64])
def test_packed_chunks(hq):
    """Prompts, continued chunks, single tokens and empty sequences side by side."""
    a = make([0, 50, 0, 777, 300, 12], [65, 1, 0, 130, 1, 33], Hq=hq, Hkv=2, D=64, page=24,
             packed=True, Lmax=2000)
    check(a, *run(a)[:2], f"packed {hq}")
    # rows beyond R are left as they are; a broken cu gives no rows
    a["R"] = 60
    check(a, *run(a)[:2], "packed, at most 60 rows")
    a["R"] = 130
    a["cu"] = np.array([0, 65, -3, 65, 190, a["rows"] + 1, 5], np.int32)
    check(a, *run(a)[:2], "packed, broken")


@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (5, 1), (6, 2)])
@pytest.mark.parametrize("held", [True, False])
def test_chunks_that_are_most_of_their_context(Hq, Hkv, held):
    """Few items whose tiles see more and more keys, cut by what they see, beside a
    single token and a short chunk of a long context; pages that end early; values that
    are not finite."""
    a = make([0, 1700, 390, 5, 1203], [700, 1, 517, 385, 90], Hq=Hq, Hkv=Hkv, D=64, page=16,
             packed=True, Lmax=2000, seed=Hq)
    if not held:
        a["held"] = np.minimum(a["held"], np.array([21, 107, 33, 2, 0], np.int32))
    v = a["v_cache"]
    v[int(a["table"][0, 20]) * 16 + 3, 0, 7] = math.inf
    v[int(a["table"][2, 30]) * 16 + 5, 0, 40] = math.nan
    check(a, *run(a)[:2], f"{Hq}/{Hkv} held {held}")


@pytest.mark.parametrize("R,Hq", [(1, 4), (12, 4), (40, 8)])
@pytest.mark.parametrize("mask", [None, "tree"])
def test_holes_in_the_table(R, Hq, mask):
    """Entries that name no page in the middle of long and short contexts, whole tiles and
    parts of them, where no row's own positions are near."""
    a = make([1500, 900, 1300, 40], [R, R, max(1, R - 1), 1], Hq=Hq, Hkv=2, D=64, page=16, mask=mask,
             seed=7)
    rng = np.random.default_rng(8)
    a["table"] = np.where(rng.random(a["table"].shape) < 0.25, -1, a["table"]).astype(np.int32)
    a["table"][0, 8:24] = a["n_slots"] // 16 + 5
    check(a, *run(a)[:2], f"{R} rows, {Hq} heads, mask {mask}")


@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (6, 2)])
def test_positions_far_behind_the_pages(Hq, Hkv):
    """Chunks at positions of up to 2^30 of which the table holds the first 2000 or so:
    only those have keys, and the work is theirs."""
    a = make([1500, 0, 700, 3], [500, 400, 300, 1], Hq=Hq, Hkv=Hkv, D=64, page=16, packed=True,
             seed=2)
    far, cap = 2 ** 30, a["table"].shape[1] * a["page"]
    a["held"] = np.full(4, a["table"].shape[1], np.int32)
    for begin in ([far, far - 1, 700, far], [far - 7] * 4):
        a["begin"], a["Lmax"] = np.array(begin, np.int32), far
        out, lse, _, _ = run(a)
        # the same as right behind the last page
        near = dict(a, begin=np.minimum(a["begin"], cap))
        check(near, out, lse, f"{Hq}/{Hkv} from {begin[0]}")


@pytest.mark.parametrize("R,Hq", [(5, 4), (40, 4), (70, 8), (33, 2)])
def test_masks(R, Hq):
    """Random masks, masks that leave rows empty, masks of several words."""
    for mask in (0.5, 0.03, "none"):
        a = make([1, 40, 64, 100], [R, R, R - 1, R // 2], Hq=Hq, Hkv=2, D=64, mask=mask, R=R)
        check(a, *run(a)[:2], f"mask {mask}")
    a = make([0, 40, 64], [R, R - 2, 1], Hq=Hq, Hkv=2, D=64, mask="none", packed=True)
    out, lse, _, _ = run(a)
    check(a, out, lse, "empty rows")
    assert (lse[:R] == -math.inf).all() and (out[:R] == 0).all()


@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
@pytest.mark.parametrize("R,Hq,L", [(6, 2, 40), (20, 8, 70), (50, 8, 3000)])
def test_not_finite_where_not_seen(R, Hq, L, cache):
    """NaN and infinities in keys and values of drafted rows reach only the rows
    that see them (what lies behind the last row is NaN in every test)."""
    for mask in (None, "tree", 0.4):
        a = make([L, L + 31], [R, R], Hq=Hq, Hkv=2, D=64, mask=mask, cache=cache, page=16, seed=4)
        rng = np.random.default_rng(3)
        for b in range(2):
            s = ref.slots_of(a, b, int(a["lengths"][b]) - 1 + R)[-R:]
            for name in ("k_cache", "v_cache"):
                x = a[name].float()
                for j in rng.integers(R // 2, R, 3):
                    x[s[j], rng.integers(0, 2), rng.integers(0, 64, 2)] = torch.tensor(
                        [math.nan, math.inf if name == "v_cache" and cache != "e4m3" else math.nan],
                        device=DEV)
                a[name] = x.to(a[name].dtype)
        out, lse, _, _ = run(a)
        check(a, out, lse, f"not finite, mask {mask}")
        if mask != 0.4:                      # no row sees later ones
            assert torch.isfinite(out[:R // 2]).all()


def test_missing_pages():
    """Pages that are not held, entries outside the cache, no page at all."""
    for R, Hq in ((4, 4), (20, 4), (60, 4)):
        a = make([100, 200, 60, 300], [R] * 4, Hq=Hq, Hkv=2, D=64, page=16, seed=R)
        a["held"] = np.array([3, 99, 0, 12], np.int32)
        a["table"][1, 5] = -7
        a["table"][1, 2] = a["n_slots"]
        a["table"][3, 1] = 2 ** 31 - 1
        out, lse, _, _ = run(a)
        check(a, out, lse, f"missing pages, {R} rows")
        assert (lse[2 * R:3 * R] == -math.inf).all()
    for name in ("k_cache", "v_cache"):
        a[name] = a[name][:0]
    a["n_slots"] = 0
    out, lse, _, _ = run(a)
    check(a, out, lse, "no cache")


@pytest.mark.parametrize("scale", [-0.1, 0.0, 3.0])
def test_scales(scale):
    for R in (3, 40):
        for cache in ("f16", "e4m3"):
            a = make([50, 90], [R, R], Hq=4, Hkv=2, D=64, type="f16", cache=cache, scale=scale)
            if cache == "e4m3":
                a["k_scale"][0] *= -1
                a["v_scale"] = None
            check(a, *run(a)[:2], f"scale {scale} {cache}")


def test_query_rows_apart():
    """q as a part of a wider projection; the rest of it is NaN."""
    a = make([50, 90], [7, 3], Hq=4, Hkv=2, D=128, qpad=512)
    a["qbuf"][:, 512:] = math.nan
    assert a["q"].stride(0) == 1024
    check(a, *run(a)[:2], "rows apart")


def test_clamped_device_data():
    """Lengths, node counts and positions out of range."""
    a = make([50, 90, 30], [7, 3, 5], Hq=4, Hkv=2, D=64, R=7)
    a["dn"] = np.array([100, -3, 0], np.int32)
    a["lengths"] = np.array([50, 10 ** 9, -5], np.int32)
    a["qbuf"].nan_to_num_(0.5)
    a["k_cache"], a["v_cache"] = (a[n].nan_to_num(0.25) for n in ("k_cache", "v_cache"))
    check(a, *run(a)[:2], "clamped")


def test_offsets_beyond_32_bits():
    """A cache of over 4 GiB a plane, its pages at both ends."""
    Hkv, D, page = 8, 128, 64
    a = make([500, 300], [5, 1], Hq=16, Hkv=Hkv, D=D, page=page)
    n = (2 ** 32 + 2 ** 28) // (Hkv * D * 2 * page) + 5    # pages
    old = a["table"].copy()
    held = old >= 0
    ids = np.arange(held.sum())
    a["table"][held] = np.where(ids % 2 == 0, n - 1 - ids, ids)
    big = {}
    for name in ("k_cache", "v_cache"):
        big[name] = torch.empty(n * page, Hkv, D, dtype=torch.bfloat16, device=DEV)
        for x, y in zip(old[held], a["table"][held]):
            big[name][y * page:(y + 1) * page] = a[name][x * page:(x + 1) * page]
    small = {"table": old, "k_cache": a["k_cache"], "v_cache": a["v_cache"],
             "n_slots": a["n_slots"]}
    a.update(big, n_slots=n * page)
    out, lse, _, _ = run(a)
    a.update(small)
    check(a, out, lse, "long cache")


def test_streams_and_graphs():
    """Two calls at once with workspaces of their own; a captured call, replayed
    with other inputs between eager ones."""
    a = make([3000, 200], [8, 8], Hq=8, Hkv=2, D=128, seed=1)
    c = make([1500, 900], [40, 40], Hq=8, Hkv=2, D=128, seed=2)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    got = [run(x, stream=s) for x, s in zip((a, c), streams)]
    torch.cuda.synchronize()
    check(a, *got[0][:2], "stream 1")
    check(c, *got[1][:2], "stream 2")
    out, lse, args, ws = got[0]
    sc = dict(lse=lse)
    from paper_2609_20186_amd import binding as sd
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        sd.switchsd_paged_attention(args, a["q"], a["k_cache"], a["v_cache"], out, ws, **sc)
    for seed in range(3):
        a["qbuf"].copy_(torch.randn(a["qbuf"].shape, generator=torch.Generator().manual_seed(seed)))
        out.fill_(77.0)
        graph.replay()
        torch.cuda.synchronize()
        once = out.clone(), lse.clone()
        eager = run(a)
        torch.cuda.synchronize()
        assert torch.equal(once[0], eager[0]) and torch.equal(once[1], eager[1])
    check(a, *once, "replayed")


# ------------------------------------------------------------------ store

@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("type,cache", [("bf16", "bf16"), ("f16", "f16"), ("bf16", "e4m3"),
                                        ("f16", "e4m3")])
def test_store(D, type, cache):
    from paper_2609_20186_amd import binding as sd
    Hkv, n, n_slots = 3, 37, 64
    g = torch.Generator().manual_seed(D)
    wide = torch.randn(n, Hkv * D * 2 + 64, generator=g) * 30
    wide[3, :40] = torch.tensor([math.nan, math.inf, -math.inf, 0.0] * 10)
    wide = wide.to(ref.HALF[type]).to(DEV)
    k, v = (wide[:, o:o + Hkv * D].view(n, Hkv, D) for o in (0, Hkv * D + 64))
    slots = torch.randperm(n_slots, generator=g)[:n]
    slots[[2, 5, 9]] = torch.tensor([-1, n_slots, 2 ** 40])
    kind = torch.float8_e4m3fn if cache == "e4m3" else ref.HALF[type]
    scales = dict(k_scale=torch.tensor([0.5, 0.07, 1.0]), v_scale=None) if cache == "e4m3" else {}
    for count in (None, 0, 20, 99):
        kc, vc = (torch.full((n_slots, Hkv, D), 7.0).to(kind).to(DEV) for _ in range(2))
        sd.switchsd_store_cache(
            k, v, slots.to(DEV), kc, vc,
            count=None if count is None else torch.tensor([count], dtype=torch.int32, device=DEV),
            **{m: None if t is None else t.to(DEV) for m, t in scales.items()})
        for x, got, scale in ((k, kc, scales.get("k_scale")), (v, vc, None)):
            want = torch.full((n_slots, Hkv, D), 7.0).to(kind).view(
                torch.uint8 if cache == "e4m3" else torch.int16)
            for j in range(n if count is None else min(count, n)):
                s = int(slots[j])
                if not 0 <= s < n_slots:
                    continue
                row = x[j].cpu()
                if cache != "e4m3":
                    want[s] = row.view(torch.int16)
                    continue
                f = row.float().numpy()
                if scale is not None:
                    f = f / scale.numpy()[:, None]
                want[s] = torch.from_numpy(ref.to_e4m3(f.astype(np.float32)))
            got = got.cpu().view(want.dtype)
            if cache == "e4m3":              # a NaN is a NaN, of either sign
                got, want = (torch.where(t & 0x7F == 0x7F, torch.full_like(t, 0x7F), t)
                             for t in (got, want))
            assert torch.equal(got, want), (count, cache)


def test_store_every_e4m3_step():
    """All 16-bit values: each code's neighbourhood, ties, the denormal range."""
    from paper_2609_20186_amd import binding as sd
    for type in ("bf16", "f16"):
        x = torch.arange(-2 ** 15, 2 ** 15, dtype=torch.int32).to(torch.int16)
        x = x.view(ref.HALF[type]).view(-1, 1, 64)
        n = x.shape[0]
        kc, vc = (torch.zeros(n, 1, 64, dtype=torch.float8_e4m3fn, device=DEV) for _ in range(2))
        sd.switchsd_store_cache(x.to(DEV), x.to(DEV), torch.arange(n, device=DEV), kc, vc)
        f = x.float().numpy()
        vals = ref.e4m3_values()
        a = np.minimum(np.abs(f.astype(np.float64)), 448.0)
        mid = (vals[1:] + vals[:-1]) / 2
        code = np.searchsorted(mid, np.nan_to_num(a), side="left")
        tie = np.isin(a, mid)
        code = np.where(tie & (code % 2 == 1), code + 1, code)
        got = kc.cpu().view(torch.uint8).numpy()
        ok = ~np.isnan(f)
        np.testing.assert_array_equal((got & 0x7F)[ok], code[ok])
        np.testing.assert_array_equal((got >> 7)[ok], np.signbit(f)[ok])
        assert ((got & 0x7F)[~ok] == 0x7F).all()
        assert torch.equal(kc.view(torch.uint8), vc.view(torch.uint8))
