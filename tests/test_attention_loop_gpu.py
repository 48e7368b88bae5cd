"""The cache store, the attention and the log probabilities as an engine uses them
together with the calls that were there: prompts stored and attended packed, then
steps of page plan, store, tree mask, attention, verification, log probabilities of
what was emitted, compaction and commit -- eagerly against plain references, and
captured in a HIP graph."""
import numpy as np
import pytest
import torch

import attention_ref as ref
from gpu_helpers import say

pytestmark = pytest.mark.gpu

V, HQ, HKV, D, PAGE, CAP = 8, 4, 2, 64, 8, 160


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2609_20186_amd import binding  # noqa: F401


class Model:
    """One attention layer over token embeddings: a token's queries, keys and values
    side by side, and an output head of V rows."""

    def __init__(self, seed):
        g = torch.Generator().manual_seed(seed)
        self.table = torch.randn(V, (HQ + 2 * HKV) * D, generator=g).bfloat16()
        self.head = torch.randn(V, HQ * D, generator=g).bfloat16()
        self.dev_table, self.dev_head = self.table.cuda(), self.head.cuda()
        t = ref.f64(self.table).reshape(V, HQ + 2 * HKV, D)
        self.q, self.k, self.v = t[:, :HQ], t[:, HQ:HQ + HKV], t[:, HQ + HKV:]

    def attend(self, tokens):
        """Output and its magnitude of the last of the tokens in 64 bits."""
        out, big = np.zeros((HQ, D)), np.zeros((HQ, D))
        for h in range(HQ):
            k, v = self.k[tokens, h // 2], self.v[tokens, h // 2]
            s = k @ self.q[tokens[-1], h] / D ** 0.5
            p = np.exp(s - s.max())
            p /= p.sum()
            out[h], big[h] = p @ v, p @ np.abs(v)
        return out, big


class Engine:
    def __init__(self, B, R, seed):
        from paper_2609_20186_amd import binding as sd
        self.sd, self.B, self.R, self.rng = sd, B, R, np.random.default_rng(seed)
        self.model = Model(seed)
        i32 = dict(dtype=torch.int32, device="cuda")
        most = (CAP + R + PAGE - 1) // PAGE
        P = B * most
        self.tokens = torch.zeros((B, CAP), **i32)
        self.lengths = torch.zeros(B, **i32)
        L = self.rng.integers(3, 40, B)
        for b in range(B):
            self.tokens[b, :L[b]] = torch.from_numpy(self.rng.integers(0, V, L[b])).int()
        self.lengths.copy_(torch.from_numpy(L))
        self.table = torch.full((B, most), -1, **i32)
        self.held = torch.zeros(B, **i32)
        self.ring = torch.from_numpy(self.rng.permutation(P).astype(np.int32)).cuda()
        self.ring_state = torch.tensor([0, P], **i32)
        self.slots = torch.empty((B, R), dtype=torch.int64, device="cuda")
        self.positions, self.missing = torch.empty((B, R), **i32), torch.empty(B, **i32)
        self.dtok, self.dpar = torch.full((B, R), -1, **i32), torch.full((B, R), -1, **i32)
        self.dn = torch.ones(B, **i32)
        self.cache = torch.full((2, P * PAGE, HKV, D), float("nan"), dtype=torch.bfloat16,
                                device="cuda")
        self.mask = torch.empty((B, R, (R + 31) // 32), **i32)
        self.plan = sd.build_page_args(self.lengths, self.dpar, self.dn, CAP, PAGE, self.table,
                                       self.held, self.ring, self.ring_state, self.slots,
                                       self.positions, self.missing)
        self.args = sd.build_attention_args(B * R, R, HQ, HKV, D, PAGE, self.table, self.held, CAP,
                                            lengths=self.lengths, dn=self.dn, mask=self.mask)
        self.ws, self.aws = sd.alloc_workspace(B, R), sd.alloc_attention_workspace(self.args)
        self.out = torch.zeros((B * R, HQ, D), dtype=torch.bfloat16, device="cuda")
        self.logits = torch.zeros((B, R, V), dtype=torch.bfloat16, device="cuda")
        self.res = {n: torch.zeros(B, **i32) for n in ("accept_len", "accept_node", "bonus")}
        self.res.update({n: torch.zeros((B, R), **i32) for n in ("out_tokens", "amax")})
        self.largs = sd.build_logprob_args(self.logits, self.res["out_tokens"], self.dn, self.dpar,
                                           self.res["accept_node"])
        f32 = dict(dtype=torch.float32, device="cuda")
        self.lp = {n: torch.zeros((B, R), **f32) for n in ("logprob", "entropy", "lse")}
        self.lp["top_ids"] = torch.zeros((B, R, 3), **i32)
        self.draft_pos, self.lag = self.lengths.clone(), torch.empty(B, **i32)
        self.use_copy = torch.zeros(B, **i32)

    def prompts(self):
        """All but the last token of each context: pages by a plan of one node (a
        chain of R nodes later), slots packed, keys and values stored, attended."""
        sd, B = self.sd, self.B
        sd.switchsd_page_plan(self.plan, self.ws)
        room = B * 64
        i32 = dict(dtype=torch.int32, device="cuda")
        cu = torch.empty(B + 1, **i32)
        slots = torch.full((room,), 5, dtype=torch.int64, device="cuda")  # left over ones
        packed = torch.zeros(room, **i32)
        begin, end = torch.zeros(B, **i32), self.lengths - 1
        sd.switchsd_span_slots(begin, end, self.tokens, self.table, self.held, PAGE, cu, slots,
                               None, packed, None)
        qkv = self.model.dev_table[packed.long()]
        q, k, v = (x.view(room, -1, D) for x in qkv.split([HQ * D, HKV * D, HKV * D], 1))
        sd.switchsd_store_cache(k, v, slots, self.cache[0], self.cache[1], count=cu[-1:])
        out = torch.full((room, HQ, D), 77.0, dtype=torch.bfloat16, device="cuda")
        args = sd.build_attention_args(room, 64, HQ, HKV, D, PAGE, self.table, self.held, CAP,
                                       begin=begin, cu=cu)
        sd.switchsd_paged_attention(args, q, self.cache[0], self.cache[1], out,
                                    sd.alloc_attention_workspace(args))
        o, at = ref.f64(out), cu.tolist()
        for b in range(B):
            x = self.tokens[b].tolist()
            for i in range(at[b + 1] - at[b]):
                self.close(o[at[b] + i], x[:i + 1])
        assert (o[at[B]:] == 77).all()

    def close(self, got, tokens):
        want, big = self.model.attend(tokens)
        # half a step of the result and of the weights, and what 32 bits leave
        tol = 2.0 ** -8 * (np.abs(want) + big) * 1.01 + big * 2.0 ** -17
        assert (np.abs(got - want) <= tol).all()

    def draft(self):
        """Random trees, two and more children to a node."""
        for b in range(self.B):
            n = int(self.rng.integers(1, self.R + 1))
            par = [-1] + [int(self.rng.integers(0, (i + 1) // 2)) for i in range(1, n)]
            self.dn[b] = n
            self.dpar[b] = torch.tensor(par + [-1] * (self.R - n), dtype=torch.int32)
            tok = self.rng.integers(0, V, self.R)
            tok[0] = -1
            tok[n:] = -1
            self.dtok[b] = torch.from_numpy(tok).int()

    def step(self, stream=None):
        sd, B, R = self.sd, self.B, self.R
        sd.switchsd_page_plan(self.plan, self.ws, stream)
        last = self.tokens.gather(1, (self.lengths[:, None] - 1).long())
        rows = torch.cat([last, self.dtok[:, 1:].clamp(min=0)], 1).long()
        qkv = self.model.dev_table[rows].view(B * R, -1)
        q, k, v = (x.view(B * R, -1, D) for x in qkv.split([HQ * D, HKV * D, HKV * D], 1))
        sd.switchsd_store_cache(k, v, self.slots, self.cache[0], self.cache[1], stream=stream)
        sd.switchsd_tree_mask(self.dpar, self.dn, self.mask, stream)
        sd.switchsd_paged_attention(self.args, q, self.cache[0], self.cache[1], self.out, self.aws,
                                    stream=stream)
        x = self.out.view(B * R, HQ * D) @ self.model.dev_head.t().contiguous()
        self.logits.copy_(x.view(B, R, V))
        r = self.res
        sd.switchsd_verify_accept(self.logits, self.dtok, self.dpar, self.dn, r["accept_len"],
                                  r["accept_node"], r["bonus"], r["out_tokens"], r["amax"],
                                  self.ws, stream)
        sd.switchsd_token_logprobs(self.largs, stream=stream, **self.lp)
        sd.switchsd_compact_cache(self.cache, self.slots, self.dpar, self.dn, r["accept_node"],
                                  stream)
        sd.switchsd_commit(self.tokens, self.lengths, r["out_tokens"], r["accept_len"],
                           self.use_copy, self.draft_pos, self.lag, stream)

    def check_rows(self, context, L):
        """The attention's rows, against the tokens on each node's path, and the log
        probabilities of what was emitted."""
        out, par = ref.f64(self.out).reshape(self.B, self.R, HQ, D), self.dpar.tolist()
        tok, moved = self.dtok.tolist(), 0
        for b in range(self.B):
            paths = []
            for i in range(int(self.dn[b])):
                paths.append([] if i == 0 else paths[par[b][i]] + [tok[b][i]])
                self.close(out[b, i], context[b][:L[b]] + paths[i])
            a, node = int(self.res["accept_len"][b]), int(self.res["accept_node"][b])
            rows = [node]
            while rows[-1] > 0:
                rows.append(par[b][rows[-1]])
            rows = rows[::-1]
            assert len(rows) == a + 1
            moved += rows != list(range(a + 1))
            for i, r in enumerate(rows):
                x = ref.f64(self.logits[b, r])
                lse, lp, h = ref.row_logprobs(x, 1.0)
                t = int(self.res["out_tokens"][b, i])
                assert float(self.lp["logprob"][b, i]) == pytest.approx(lp[t], abs=1e-5)
                assert float(self.lp["entropy"][b, i]) == pytest.approx(h, abs=1e-5)
                assert self.lp["top_ids"][b, i].tolist() == ref.order(x)[:3]
                if i < a:
                    assert t == tok[b][rows[i + 1]]
        return moved

    def check_cache(self):
        """Every position of the context but the last holds its token's keys and values."""
        kv = self.model.table.view(V, HQ + 2 * HKV, D)
        cache = self.cache.cpu()
        for b in range(self.B):
            L = int(self.lengths[b])
            for pos in range(L - 1):
                s = int(self.table[b, pos // PAGE]) * PAGE + pos % PAGE
                t = int(self.tokens[b, pos])
                assert torch.equal(cache[0, s], kv[t, HQ:HQ + HKV]), (b, pos)
                assert torch.equal(cache[1, s], kv[t, HQ + HKV:]), (b, pos)


def test_steps_against_references():
    e = Engine(5, 13, seed=3)
    e.prompts()
    moved = 0
    for _ in range(8):
        e.draft()
        L, context = e.lengths.tolist(), e.tokens.tolist()
        e.step()
        moved += e.check_rows(context, L)
        e.check_cache()
    assert moved > 0                       # some accepted path had to be moved
    say("lengths", e.lengths.tolist())


def test_captured_steps():
    """The same steps replayed from one graph leave the same contexts and caches."""
    runs = []
    for captured in (False, True):
        e = Engine(4, 9, seed=11)
        e.prompts()
        e.draft()
        graph = None
        if captured:
            keep = {n: getattr(e, n).clone() for n in ("tokens", "lengths", "table", "held", "ring",
                                                       "ring_state", "cache", "draft_pos")}
            side = torch.cuda.Stream()
            side.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(side):  # the product's first call is not captured
                e.step()
            torch.cuda.current_stream().wait_stream(side)
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                e.step()
            for n, t in keep.items():
                getattr(e, n).copy_(t)
        got = []
        for _ in range(6):
            if captured:
                graph.replay()
            else:
                e.step()
            torch.cuda.synchronize()
            got.append([e.tokens.clone(), e.lengths.clone(), e.out.clone(), e.lp["logprob"].clone()])
            e.draft()
        e.check_cache()
        runs.append(got)
    for i, (x, y) in enumerate(zip(*runs)):
        for a, b in zip(x, y):
            assert torch.equal(a, b), i
