"""Penalties, biases and grammar masks on the logits (switchsd_process_logits)
and the greedy verification over them (switchsd_verify_processed) against the
definitions: bit for bit in float, and in 64 bits within the roundings."""
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


def make(B, R, V, L, seed, src="bf16", draft="chain", penal="rfp", n_bias=9, mask=True, k=3,
         special=True):
    """Inputs full of edges: ragged, clamped and empty lengths, repeated tokens,
    ids outside the vocabulary, broken parents, rows that allow nothing."""
    rng = np.random.default_rng(seed)
    hot = rng.integers(0, V, 12)                        # tokens that repeat
    pick = np.where(rng.random((B, L)) < 0.7, hot[rng.integers(0, 12, (B, L))],
                    rng.integers(-2, V + 3, (B, L)))
    d = {"tokens": pick.astype(np.int32)}
    d["lengths"] = rng.integers(0, L + 1, B).astype(np.int32)
    d["lengths"][0] = L + 7                             # clamped
    if B > 1:
        d["lengths"][1] = 0
    if B > 2:
        d["lengths"][2] = 1
    d["prompt_lens"] = rng.integers(-1, L + 2, B).astype(np.int32)
    d["dtok"] = np.where(rng.random((B, R)) < 0.6, hot[rng.integers(0, 12, (B, R))],
                         rng.integers(-1, V + 1, (B, R))).astype(np.int32)
    d["dn"] = rng.integers(0, R + 2, B).astype(np.int32)
    d["dn"][0] = R
    i = np.arange(R)
    if draft == "chain":
        d["dpar"] = None
    elif draft == "candidates":
        d["dpar"] = np.tile(np.where((i - 1) % k == 0, 0, i - 1), (B, 1)).astype(np.int32)
    else:
        d["dpar"] = (rng.random((B, R)) * i).astype(np.int32)
        bad = rng.random((B, R)) < 0.1
        d["dpar"][bad] = rng.integers(-3, R + 3, int(bad.sum()))
    if d["dpar"] is not None:
        d["dpar"][:, 0] = -1
    for key, name, lo, hi in (("r", "repetition", 0.5, 2.0), ("f", "frequency", -1.0, 2.0),
                              ("p", "presence", -1.0, 2.0)):
        d[name] = rng.uniform(lo, hi, B).astype(np.float32) if key in penal else None
    d["bias_ids"] = d["bias_vals"] = None
    if n_bias:
        # repeated ids, ids outside the vocabulary, ids the history holds too
        d["bias_ids"] = np.where(rng.random((B, n_bias)) < 0.5, hot[rng.integers(0, 12, (B, n_bias))],
                                 rng.integers(-1, V + 2, (B, n_bias))).astype(np.int32)
        d["bias_vals"] = rng.normal(0, 4, (B, n_bias)).astype(np.float32)
        d["bias_vals"][:, ::5] = -np.inf
    d["allowed"] = d["allowed_on"] = None
    if mask:
        words = (V + 31) // 32
        m = rng.integers(0, 2 ** 32, (B, R, words), dtype=np.uint32)
        kind = rng.integers(0, 4, (B, R))
        m[kind == 0] = 0                                # nothing is allowed
        m[kind == 1] = 0xFFFFFFFF
        d["allowed"] = m
        d["allowed_on"] = rng.integers(0, 2, B).astype(np.int32)
        d["allowed_on"][0] = -3
    x = rng.normal(0, 3, (B, R, V)).astype(np.float32)
    if special and V > 4:
        at = rng.integers(0, V, (B, R))
        for s, val in enumerate((np.nan, np.inf, -np.inf, -0.0, 0.0)):
            np.put_along_axis(x, ((at + 7 * s) % V)[:, :, None], val, 2)
        x[B - 1, 0] = np.nan if V % 2 else x[B - 1, 0]
        lots = hot[None, None, :3] + np.zeros((B, R, 1), np.int64)
        np.put_along_axis(x, lots, np.float32(9.0), 2)  # ties, mended by the penalties
    d["logits"] = torch.from_numpy(x).to(ref.TYPES[src])
    return d


def device_args(d, logits=None):
    from paper_2609_20186_amd import binding as sd
    dev = {}
    for name, t in d.items():
        if t is None or name == "logits":
            dev[name] = None
        elif t.dtype == np.uint32:
            dev[name] = torch.from_numpy(t.view(np.int32)).cuda()
        else:
            dev[name] = torch.from_numpy(t).cuda()
    dev["logits"] = d["logits"].cuda() if logits is None else logits
    return sd.build_logits_args(**dev)


def check_rows(d, out, dtype, sentinel):
    """out against the float definition bit for bit, and against the 64-bit one
    within the roundings: 2^-24 of every intermediate value, then half a step
    of the output's type."""
    B, R, V = d["logits"].shape
    r32, r64 = ref.processed(d, np.float32), ref.processed(d, np.float64)
    half = torch.finfo(dtype).eps / 2
    tiny = float(torch.finfo(dtype).smallest_normal) * half
    out = out.cpu()
    for b in range(B):
        n = ref.nodes(d, b)
        assert bool((out[b, n:] == sentinel).all()), f"rows behind the draft of {b}"
        for r in range(n):
            y, _, touched = r32[b, r]
            want = ref.rounded(y, dtype)
            got = out[b, r]
            same = (got == want) | (got.isnan() & want.isnan())
            assert bool(same.all()), (b, r, int((~same).nonzero()[0]), got[~same][:3],
                                      want[~same][:3])
            if dtype == d["logits"].dtype:              # untouched values keep their bits
                word = torch.int32 if dtype == torch.float32 else torch.int16
                t = torch.from_numpy(~touched)
                assert torch.equal(got.view(word)[t], d["logits"][b, r].view(word)[t])
            y, size, _ = r64[b, r]
            with np.errstate(all="ignore"):
                big = float(torch.finfo(dtype).max)
                fin = np.isfinite(y) & (np.abs(y) < big / 2)
                err = np.abs(got.double().numpy() - y)[fin]
                tol = (1.01 * 2.0 ** -24 * size + half * (np.abs(y) + 2.0 ** -23 * size) + tiny)[fin]
            assert (err <= tol).all(), (b, r, err.max())


SHAPES = [(1, 1, 1, 1), (2, 1, 7, 5), (3, 8, 1000, 40), (2, 8, 2048, 300), (3, 5, 2049, 100),
          (1, 70, 4097, 64), (4, 11, 16387, 2000)]


@pytest.mark.parametrize("src,out", [("bf16", "bf16"), ("f16", "f16"), ("f16", "bf16"),
                                     ("f32", "f32"), ("f32", "bf16")])
@pytest.mark.parametrize("shape", SHAPES)
def test_process(src, out, shape):
    from paper_2609_20186_amd import binding as sd
    say(f"[process] {src}->{out} {shape}")
    for draft in ("chain", "tree"):
        d = make(*shape, seed=sum(shape), src=src, draft=draft)
        o = torch.full(d["logits"].shape, 77.0, dtype=ref.TYPES[out], device="cuda")
        sd.switchsd_process_logits(device_args(d), o)
        check_rows(d, o, ref.TYPES[out], 77.0)


@pytest.mark.parametrize("opts", [
    dict(penal="r"), dict(penal="f"), dict(penal="p"), dict(penal=""), dict(n_bias=0),
    dict(mask=False), dict(penal="", n_bias=0), dict(penal="", n_bias=0, mask=False),
    dict(penal="", mask=False), dict(n_bias=511), dict(draft="candidates"),
])
def test_process_options(opts):
    from paper_2609_20186_amd import binding as sd
    say(f"[process] {opts}")
    for src in ("bf16", "f32"):
        d = make(3, 13, 5003, 200, seed=5, src=src, **opts)
        o = torch.full(d["logits"].shape, 77.0, dtype=ref.TYPES[src], device="cuda")
        sd.switchsd_process_logits(device_args(d), o)
        check_rows(d, o, ref.TYPES[src], 77.0)


@pytest.mark.parametrize("src", ["bf16", "f32"])
@pytest.mark.parametrize("B,R,V", [(64, 2, 70001), (64, 3, 36000), (2, 201, 9001)])
def test_process_grids(src, B, R, V):
    """Sizes that take the larger chunks, and several groups of rows."""
    from paper_2609_20186_amd import binding as sd
    say(f"[process] grids {src} {B}x{R}x{V}")
    d = make(B, R, V, 50, seed=V, src=src, draft="candidates", k=20)
    o = torch.full(d["logits"].shape, 77.0, dtype=ref.TYPES[src], device="cuda")
    sd.switchsd_process_logits(device_args(d), o)
    check_rows(d, o, ref.TYPES[src], 77.0)


@pytest.mark.parametrize("src", ["bf16", "f16", "f32"])
def test_process_in_place_and_unaligned(src):
    """In place, and tensors that start at an odd element."""
    from paper_2609_20186_amd import binding as sd
    say(f"[process] in place {src}")
    d = make(3, 7, 4099, 90, seed=11, src=src, draft="tree")
    x = d["logits"].cuda().clone()
    sd.switchsd_process_logits(device_args(d, x), x)
    for b in range(3):                                  # rows behind the draft keep their logits
        n = ref.nodes(d, b)
        word = torch.int32 if src == "f32" else torch.int16
        assert torch.equal(x[b, n:].cpu().view(word), d["logits"][b, n:].view(word))
        x[b, n:] = 77.0
    check_rows(d, x, ref.TYPES[src], 77.0)
    for shift in (1, 3):
        n = d["logits"].numel()
        raw = torch.zeros(n + 8, dtype=ref.TYPES[src], device="cuda")
        view = raw[shift:shift + n].view(d["logits"].shape)
        view.copy_(d["logits"])
        o = torch.full((n + 8,), 77.0, dtype=ref.TYPES[src], device="cuda")
        ov = o[shift + 1:shift + 1 + n].view(d["logits"].shape)
        sd.switchsd_process_logits(device_args(d, view), ov)
        check_rows(d, ov, ref.TYPES[src], 77.0)
        assert bool((o[:shift + 1] == 77).all()) and bool((o[shift + 1 + n:] == 77).all())


def gpu_verify(args, ws=None, stream=None):
    from paper_2609_20186_amd import binding as sd
    B, R, _ = args.shape
    o = {n: torch.full((B,), -9, dtype=torch.int32, device="cuda")
         for n in ("accept_len", "accept_node", "bonus")}
    for n in ("out_tokens", "amax"):
        o[n] = torch.full((B, R), -9, dtype=torch.int32, device="cuda")
    if ws is None:
        ws = sd.alloc_workspace(B, R)
    sd.switchsd_verify_processed(args, o["accept_len"], o["accept_node"], o["bonus"],
                                 o["out_tokens"], o["amax"], ws, stream)
    return o, ws


def plant(d, seed):
    """Raise the drafted children of a random path, so that drafts are accepted."""
    rng = np.random.default_rng(seed)
    for b in range(d["dtok"].shape[0]):
        node = int(rng.integers(0, ref.nodes(d, b)))
        par = ref.parents(d, b)
        for q in ref.path_of(par, node)[0]:
            v, r = int(d["dtok"][b, q]), int(par[q])
            if 0 <= v < d["logits"].shape[2] and 0 <= r < q:
                d["logits"][b, r, v] = 60.0
                if d["allowed"] is not None:
                    d["allowed"][b, r, v // 32] |= np.uint32(1 << (v % 32))
    return d


@pytest.mark.parametrize("src", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("shape", SHAPES + [(2, 201, 3001, 64), (1, 1024, 257, 30),
                                            (64, 2, 70001, 50)])
def test_verify(src, shape):
    say(f"[verify] {src} {shape}")
    for draft in ("chain", "tree", "candidates"):
        d = make(*shape, seed=sum(shape) + 1, src=src, draft=draft, k=20)
        if draft != "tree":
            d["dn"][-1] = shape[1]
        plant(d, shape[2])
        if d["bias_vals"] is not None:
            d["bias_vals"] = np.maximum(d["bias_vals"], np.float32(-9))
        want = ref.greedy(d, ref.processed(d, np.float32))
        got, ws = gpu_verify(device_args(d))
        for name, t in got.items():
            np.testing.assert_array_equal(t.cpu().numpy(), want[name],
                                          err_msg=f"{draft} {name}")
        assert int(ws.count_nonzero()) == 0


@pytest.mark.parametrize("src,B,R,V,L,spread", [
    ("bf16", 64, 17, 70001, 50, False), ("bf16", 64, 20, 70001, 6000, True),
    ("bf16", 64, 16, 70000, 60000, True), ("f16", 64, 19, 66000, 6000, True),
    ("f16", 64, 17, 70001, 60000, True), ("f32", 40, 18, 70001, 300, False),
    ("f32", 40, 21, 70002, 9000, True), ("f32", 40, 16, 66000, 60000, True),
    ("bf16", 9, 201, 70001, 3000, True),
])
def test_verify_large_batches(src, B, R, V, L, spread):
    """Sizes at which a wave takes whole rows: few listed tokens, more vectors
    with one than the wave keeps, more tokens than the list holds."""
    say(f"[verify] large {src} {B}x{R}x{V} L={L}")
    d = make(B, R, V, L, seed=V + L, src=src, draft="candidates", k=5)
    if spread:                                          # a history over the whole vocabulary
        d["tokens"] = np.random.default_rng(L).integers(0, V, (B, L)).astype(np.int32)
        d["lengths"][::2] = L
    d["dn"][::3] = R
    plant(d, L)
    d["bias_vals"] = np.maximum(d["bias_vals"], np.float32(-9))
    # rows where nothing but -inf is left, with and without a mask's help
    d["logits"][4, 3] = -np.inf
    d["logits"][5, 2] = float("nan")
    d["allowed_on"][5] = 0
    d["allowed"][6, 1, :] = 0
    want = ref.greedy(d, ref.processed(d, np.float32))
    got, ws = gpu_verify(device_args(d))
    for name, t in got.items():
        np.testing.assert_array_equal(t.cpu().numpy(), want[name], err_msg=name)
    assert int(ws.count_nonzero()) == 0


def test_verify_is_process_then_accept():
    """The two routes agree, on a workspace that calls of other shapes used."""
    from paper_2609_20186_amd import binding as sd
    say("[verify] two routes")
    ws = sd.alloc_workspace(9, 60)
    for seed, (B, R, V) in enumerate([(9, 60, 20000), (3, 8, 32000), (7, 21, 1001)]):
        d = plant(make(B, R, V, 400, seed=seed, src="f32", draft="tree", special=False), seed)
        args = device_args(d)
        out = torch.zeros((B, R, V), dtype=torch.bfloat16, device="cuda")
        sd.switchsd_process_logits(args, out)
        got, _ = gpu_verify(args, ws)
        o = {n: torch.full_like(t, -9) for n, t in got.items()}
        dpar = torch.from_numpy(d["dpar"]).cuda()
        sd.switchsd_verify_accept(out, torch.from_numpy(d["dtok"]).cuda(), dpar,
                                  torch.from_numpy(d["dn"]).cuda(), o["accept_len"],
                                  o["accept_node"], o["bonus"], o["out_tokens"], o["amax"], ws)
        for name in got:
            assert torch.equal(got[name], o[name]), name
        assert int(ws.count_nonzero()) == 0


def test_captured_and_on_another_stream():
    """Captured once, replayed on changing inputs between eager calls; and the
    same calls on a side stream."""
    from paper_2609_20186_amd import binding as sd
    say("[process] graph")
    d = [plant(make(4, 9, 9001, 300, seed=s, draft="tree"), s) for s in range(3)]
    for e in d:
        e["dpar"], e["dn"] = d[0]["dpar"], d[0]["dn"]
    x = d[0]["logits"].cuda()
    args = device_args(d[0], x)
    out = torch.full(x.shape, 77.0, dtype=torch.bfloat16, device="cuda")
    got, ws = gpu_verify(args)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        sd.switchsd_process_logits(args, out, side)
        sd.switchsd_verify_processed(args, got["accept_len"], got["accept_node"], got["bonus"],
                                     got["out_tokens"], got["amax"], ws, side)
    for k in (1, 2, 0, 2):
        x.copy_(d[k]["logits"])
        graph.replay()
        torch.cuda.synchronize()
        now = dict(d[0], logits=d[k]["logits"])
        check_rows(now, out, torch.bfloat16, 77.0)
        want = ref.greedy(now, ref.processed(now, np.float32))
        for name, t in got.items():
            np.testing.assert_array_equal(t.cpu().numpy(), want[name], err_msg=name)
        eager, _ = gpu_verify(args)
        assert all(torch.equal(eager[n], got[n]) for n in got)
    side.wait_stream(torch.cuda.current_stream())
    o2 = torch.full_like(out, 77.0)
    side.wait_stream(torch.cuda.current_stream())
    sd.switchsd_process_logits(args, o2, side)
    side.synchronize()
    word = torch.int16
    assert torch.equal(o2.view(word), out.view(word))


def test_two_streams_at_once():
    """Verifications that may overlap, each with a workspace of its own."""
    from paper_2609_20186_amd import binding as sd
    say("[verify] two streams")
    runs = []
    for seed, (B, R, V) in enumerate([(9, 20, 30000), (5, 66, 20001)]):
        d = plant(make(B, R, V, 400, seed=70 + seed, draft="tree"), seed)
        out, ws = gpu_verify(device_args(d))
        runs.append((d, device_args(d), out, ws, torch.cuda.Stream(),
                     ref.greedy(d, ref.processed(d, np.float32))))
    for d, args, out, ws, stream, want in runs:
        for t in out.values():
            t.fill_(-9)
        stream.wait_stream(torch.cuda.current_stream())
    for turn in range(20):
        for d, args, out, ws, stream, want in runs:
            sd.switchsd_verify_processed(args, out["accept_len"], out["accept_node"],
                                         out["bonus"], out["out_tokens"], out["amax"], ws,
                                         stream)
    torch.cuda.synchronize()
    for d, args, out, ws, stream, want in runs:
        for name, t in out.items():
            np.testing.assert_array_equal(t.cpu().numpy(), want[name], err_msg=name)
        assert int(ws.count_nonzero()) == 0


def test_two_graphs_share_a_workspace():
    """Two captured verifications of different shapes on one workspace, replayed
    in turn."""
    from paper_2609_20186_amd import binding as sd
    say("[verify] two graphs")
    ws = sd.alloc_workspace(6, 70)
    side = torch.cuda.Stream()
    runs = []
    for seed, (B, R, V) in enumerate([(6, 70, 3001), (4, 5, 40000)]):
        d = plant(make(B, R, V, 100, seed=40 + seed, draft="tree"), seed)
        args = device_args(d)
        out, _ = gpu_verify(args, ws)
        graph = torch.cuda.CUDAGraph()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.graph(graph, stream=side):
            sd.switchsd_verify_processed(args, out["accept_len"], out["accept_node"],
                                         out["bonus"], out["out_tokens"], out["amax"], ws, side)
        runs.append((d, args, out, graph, ref.greedy(d, ref.processed(d, np.float32))))
    for turn in range(3):
        for d, args, out, graph, want in runs:
            for t in out.values():
                t.fill_(-9)
            graph.replay()
            for name, t in out.items():
                np.testing.assert_array_equal(t.cpu().numpy(), want[name], err_msg=name)
    assert int(ws.count_nonzero()) == 0


def test_longest_history():
    """A token repeated through the longest history and drafted again: its count
    fills the whole field."""
    from paper_2609_20186_amd import binding as sd
    say("[process] longest history")
    L = sd.MAX_HISTORY
    d = make(2, 3, 50, 8, seed=1, n_bias=3, mask=False, special=False)
    d["tokens"] = np.full((2, L), 7, np.int32)
    d["tokens"][1, :5] = 9
    d["lengths"], d["prompt_lens"] = np.array([L, L], np.int32), np.array([0, 5], np.int32)
    d["dtok"] = np.array([[-1, 7, 7], [-1, 9, 7]], np.int32)
    d["dn"][:] = 3
    d["frequency"] = np.array([1e-5, 2e-5], np.float32)
    o = torch.full(d["logits"].shape, 77.0, dtype=torch.float32, device="cuda")
    d["logits"] = d["logits"].float()
    sd.switchsd_process_logits(device_args(d), o)
    check_rows(d, o, torch.float32, 77.0)


def test_more_than_two_to_the_31_logits():
    """Offsets beyond 32 bits: the last sequences of a 2.2e9-element tensor."""
    from paper_2609_20186_amd import binding as sd
    say("[process] large offsets")
    B, R, V = 35, 32, 2000000
    x = torch.zeros((B, R, V), dtype=torch.bfloat16, device="cuda")
    small = plant(make(3, R, V, 60, seed=3, n_bias=5, mask=False, special=False), 3)
    x[B - 3:] = small["logits"].cuda()
    i32 = dict(dtype=torch.int32, device="cuda")
    full = {}
    for name in ("tokens", "lengths", "prompt_lens", "dtok", "dn", "repetition", "frequency",
                 "presence", "bias_ids", "bias_vals"):
        t = torch.from_numpy(small[name]).cuda()
        full[name] = torch.zeros((B,) + tuple(t.shape[1:]), dtype=t.dtype, device="cuda")
        full[name][B - 3:] = t
    full["dn"][:B - 3] = 1
    args = sd.build_logits_args(x, full["dtok"], None, full["dn"], full["tokens"],
                                full["lengths"], full["prompt_lens"], full["repetition"],
                                full["frequency"], full["presence"], full["bias_ids"],
                                full["bias_vals"])
    assert x.numel() > 2 ** 31
    got, _ = gpu_verify(args)
    rows = ref.processed(small, np.float32)
    want = ref.greedy(small, rows)
    for name, t in got.items():
        np.testing.assert_array_equal(t[B - 3:].cpu().numpy(), want[name], err_msg=name)
    sd.switchsd_process_logits(args, x)                 # in place
    for b in range(3):
        for r in range(ref.nodes(small, b)):
            y = ref.rounded(rows[b, r][0], torch.bfloat16)
            assert torch.equal(x[B - 3 + b, r].cpu(), y), (b, r)
    assert torch.empty(0, **i32).numel() == 0
