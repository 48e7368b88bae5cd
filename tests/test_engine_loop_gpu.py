"""The calls around the step as an engine uses them together: pages and slots
for the drafted rows, verification over processed logits, the accepted nodes'
cache rows moved into place, the commit, and the slots of the draft model's
lag -- eagerly against plain loops, and captured in a HIP graph."""
import numpy as np
import pytest
import torch

import engine_ref as ref
from gpu_helpers import say
from test_processed_gpu import check_rows, device_args, make, plant

pytestmark = pytest.mark.gpu

PAGE, ROW = 8, 16


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2609_20186_amd import binding  # noqa: F401


class Engine:
    """Device state of a small engine: contexts, drafts, pages, one cache plane
    per two tokens' worth of bytes (a row holds its sequence position)."""

    def __init__(self, B, R, V, cap, draft, seed):
        from paper_2609_20186_amd import binding as sd
        self.d = make(B, R, V, cap, seed, draft=draft, k=3, special=False)
        d = self.d
        rng = np.random.default_rng(seed)
        d["lengths"] = rng.integers(1, cap // 3, B).astype(np.int32)
        d["lengths"][0] = 0                                # a finished sequence
        d["dn"] = np.full(B, R, np.int32)
        if d["dpar"] is None:
            d["dpar"] = np.tile(np.arange(-1, R - 1, dtype=np.int32), (B, 1))
        self.use_copy = rng.integers(0, 2, B).astype(np.int32)
        self.B, self.R, self.cap = B, R, cap
        most = (cap + R + PAGE - 1) // PAGE
        P = B * most
        self.plan = {"B": B, "R": R, "Lmax": cap, "page": PAGE, "dpar": d["dpar"],
                     "lengths": d["lengths"], "dn": d["dn"],
                     "table": np.full((B, most), -1, np.int32), "held": np.zeros(B, np.int32),
                     "ring": rng.permutation(P).astype(np.int32),
                     "ring_state": np.array([P // 2, P], np.int32)}
        self.dev = {k: torch.from_numpy(v.copy()).cuda() for k, v in self.plan.items()
                    if not isinstance(v, int)}
        dev = self.dev
        i32 = dict(dtype=torch.int32, device="cuda")
        dev["slots"] = torch.empty((B, R), dtype=torch.int64, device="cuda")
        dev["positions"], dev["missing"] = torch.empty((B, R), **i32), torch.empty(B, **i32)
        self.pargs = sd.build_page_args(
            dev["lengths"], dev["dpar"], dev["dn"], cap, PAGE, dev["table"], dev["held"],
            dev["ring"], dev["ring_state"], dev["slots"], dev["positions"], dev["missing"])
        self.logits = d["logits"].cuda()
        self.tokens = torch.from_numpy(d["tokens"]).cuda()
        opt = {n: None if d[n] is None else
               torch.from_numpy(d[n].view(np.int32) if d[n].dtype == np.uint32 else d[n]).cuda()
               for n in ("prompt_lens", "repetition", "frequency", "presence", "bias_ids",
                         "bias_vals", "allowed", "allowed_on")}
        self.dtok = torch.from_numpy(d["dtok"]).cuda()
        self.largs = sd.build_logits_args(self.logits, self.dtok, dev["dpar"], dev["dn"],
                                          self.tokens, dev["lengths"], **opt)
        self.out = {n: torch.empty(B, **i32) for n in ("accept_len", "accept_node", "bonus")}
        self.out.update({n: torch.empty((B, R), **i32) for n in ("out_tokens", "amax")})
        self.ws = sd.alloc_workspace(B, R)
        self.draft_pos = dev["lengths"].clone()
        self.lag = torch.empty(B, **i32)
        self.copy_dev = torch.from_numpy(self.use_copy).cuda()
        self.cache = torch.zeros((2, P * PAGE, ROW), device="cuda")
        n = B * cap
        self.span = [torch.empty(B + 1, **i32), torch.empty(n, dtype=torch.int64, device="cuda")]
        self.span += [torch.empty(n, **i32) for _ in range(3)]

    def step(self, stream=None):
        from paper_2609_20186_amd import binding as sd
        dev, o = self.dev, self.out
        sd.switchsd_page_plan(self.pargs, self.ws, stream)
        sd.switchsd_verify_processed(self.largs, o["accept_len"], o["accept_node"], o["bonus"],
                                     o["out_tokens"], o["amax"], self.ws, stream)
        sd.switchsd_compact_cache(self.cache, dev["slots"], dev["dpar"], dev["dn"],
                                  o["accept_node"], stream)
        sd.switchsd_commit(self.tokens, dev["lengths"], o["out_tokens"], o["accept_len"],
                           self.copy_dev, self.draft_pos, self.lag, stream)
        sd.switchsd_span_slots(self.draft_pos, dev["lengths"], self.tokens, dev["table"],
                               dev["held"], PAGE, *self.span, stream)

    def expected(self, state):
        """The same step in plain loops; returns its results, advances `state`
        (tokens, lengths, draft_pos, cache, plan)."""
        d = dict(self.d, tokens=state["tokens"], lengths=state["lengths"])
        state["plan"]["lengths"] = state["lengths"]
        slots, positions, missing = ref.page_plan(state["plan"])
        res = ref.greedy(d, ref.processed(d, np.float32))
        ref.compact(state["cache"], slots, d["dpar"], d["dn"], res["accept_node"])
        cap = self.cap
        for b in range(self.B):
            L, a = int(state["lengths"][b]), int(res["accept_len"][b])
            new = res["out_tokens"][b, :a + 1]
            n = max(0, min(cap - L, a + 1))
            state["tokens"][b, L:L + n] = new[:n]
            state["lengths"][b] = min(L + a + 1, cap)
            if not self.use_copy[b]:
                state["draft_pos"][b] = L + a
            state["draft_pos"][b] = np.clip(state["draft_pos"][b], 0, state["lengths"][b])
        cu, rec = ref.spans(state["draft_pos"], state["lengths"], state["tokens"],
                            state["plan"]["table"], state["plan"]["held"], PAGE, 1 << 40)
        return dict(res, slots=slots, positions=positions, missing=missing, cu=cu, rec=rec)

    def host_state(self):
        return {"tokens": self.d["tokens"].copy(), "lengths": self.d["lengths"].copy(),
                "draft_pos": self.d["lengths"].copy(), "cache": self.cache.cpu().numpy(),
                "plan": {k: v.copy() if hasattr(v, "copy") else v for k, v in self.plan.items()}}

    def check(self, want, state, what):
        got = dict(self.out, slots=self.dev["slots"], positions=self.dev["positions"],
                   missing=self.dev["missing"], cu=self.span[0])
        for name, t in got.items():
            np.testing.assert_array_equal(t.cpu().numpy(), want[name], err_msg=f"{what} {name}")
        for name, t in (("tokens", self.tokens), ("lengths", self.dev["lengths"]),
                        ("draft_pos", self.draft_pos)):
            np.testing.assert_array_equal(t.cpu().numpy(), state[name], err_msg=f"{what} {name}")
        rec = np.array(want["rec"], np.int64).reshape(-1, 4)
        for j, t in enumerate(self.span[1:]):
            np.testing.assert_array_equal(t.cpu().numpy()[:len(rec)], rec[:, j],
                                          err_msg=f"{what} span {j}")
        assert torch.equal(self.cache.cpu(), torch.from_numpy(state["cache"])), what
        assert int(self.ws.count_nonzero()) == 0


@pytest.mark.parametrize("draft,R,captured", [("tree", 9, False), ("candidates", 13, True),
                                              ("chain", 5, True)])
def test_engine_steps(draft, R, captured):
    """Several steps on one state; the logits and the draft change between them
    (the cache's drafted rows are written anew, as a target's pass would)."""
    say(f"[engine] {draft} captured={captured}")
    B, V = 5, 700
    e = Engine(B, R, V, 90, draft, seed=R)
    state = e.host_state()
    graph = None
    if captured:
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            e.step(side)
    rng = np.random.default_rng(99)
    for it in range(5):
        new = plant(make(B, R, V, 8, 100 + it, draft=draft, k=3, special=False), it)
        e.d["logits"], e.d["dtok"] = new["logits"], new["dtok"]
        e.logits.copy_(new["logits"])
        e.dtok.copy_(torch.from_numpy(new["dtok"]))
        fill = rng.normal(0, 1, e.cache.shape).astype(np.float32)
        e.cache.copy_(torch.from_numpy(fill))
        state["cache"] = fill.copy()
        want = e.expected(state)
        if captured:
            graph.replay()
        else:
            e.step()
        torch.cuda.synchronize()
        e.check(want, state, f"step {it}")


def test_processed_logits_feed_the_draw():
    """At T > 0 the processed logits are written and then drawn from: the same
    tokens as the oracle's draw over the reference's processed rows."""
    import oracle
    from paper_2609_20186_amd import binding as sd
    say("[engine] draw")
    B, R, V, T = 3, 6, 1024, 0.8
    d = make(B, R, V, 60, 7, draft="chain", special=False)
    d["dn"][:] = R
    d["allowed"][:, :, 0] |= 1
    out = torch.zeros((B, R, V), dtype=torch.bfloat16, device="cuda")
    sd.switchsd_process_logits(device_args(d), out)
    check_rows(d, out, torch.bfloat16, 0.0)
    rng = np.random.default_rng(3)
    u = rng.integers(0, 2 ** 64, (B, R), dtype=np.uint64)
    o = {n: torch.empty(B, dtype=torch.int32, device="cuda")
         for n in ("accept_len", "accept_node", "bonus")}
    o.update({n: torch.empty((B, R), dtype=torch.int32, device="cuda")
              for n in ("out_tokens", "amax")})
    ws = sd.alloc_workspace(B, R)
    sd.switchsd_verify_sample(out, T, torch.from_numpy(u.view(np.int64)).cuda(),
                              torch.from_numpy(d["dtok"]).cuda(), None,
                              torch.from_numpy(d["dn"]).cuda(), o["accept_len"],
                              o["accept_node"], o["bonus"], o["out_tokens"], o["amax"], ws,
                              sd.alloc_sample_workspace(B, R, V))
    bits = out.view(torch.int16).cpu().numpy().view(np.uint16)
    rows = ref.processed(d, np.float32)
    for b in range(B):
        for r in range(R):
            want = oracle.sample_row(bits[b, r], T, int(u[b, r]))
            assert int(o["amax"][b, r]) == int(want), (b, r)
            # only what the mask allows is drawn
            assert np.isfinite(rows[b, r][0][int(want)]) or np.isneginf(rows[b, r][0]).all()
