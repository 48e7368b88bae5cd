"""The operators around a verification step whose speed matters, as cases: what
a decoding engine calls next to the step itself.

  own                False: run() computes the plain form (elementary torch
                     operations); True: it makes the library's calls
  listed()           the cases by name
  draw(rng)          one more case from the same ranges
  prepare(case, s)   what the engine holds before the call, from the seed alone
  run(state)         one pass through one operator, and its outputs
  work(case)         bytes and operations a pass cannot do without
  exact(case, s)     the computed outputs in 64 bits, from the definitions

Kinds of case:
  process  penalties for repeated tokens, biases and grammar masks on the logits
           of every drafted row (switchsd_process_logits)
  verify   the greedy accept over logits processed on the fly
           (switchsd_verify_processed)
  plan     pages for the drafted rows, their slots and positions
           (switchsd_page_plan)
  spans    packed slots, positions and tokens of ragged ranges of the contexts:
           prompts, or what a lagging draft model has yet to read
           (switchsd_span_slots)
  compact  the accepted nodes' cache rows moved to their final slots
           (switchsd_compact_cache)
"""
import math

import torch

own = False

DEV = "cuda"
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
SIZE = {"bf16": 2, "f16": 2, "f32": 4}


# ------------------------------------------------------------------ cases

def listed():
    logits = dict(W=1, tree=False, penalties=True, n_bias=0, grammar=False, src="bf16",
                  out="bf16")
    return [
        # one user without a draft: one row, launch latency is everything
        dict(logits, name="process_one_token", kind="process", B=1, R=1, k=0, V=32000, L=512),
        # the ordinary serving batch: chains, repetition penalties and a few biases
        dict(logits, name="process_chat", kind="process", B=32, R=8, k=7, V=128256, L=4096,
             n_bias=300),
        # trees over constrained output, float logits straight from the head: the largest call
        dict(logits, name="process_grammar_tree", kind="process", B=32, R=60, k=7, V=128256,
             L=2048, tree=True, grammar=True, src="f32"),
        # the ordinary serving batch, greedy, nothing written but the result
        dict(logits, name="verify_chat", kind="verify", B=32, R=8, k=7, V=128256, L=4096,
             n_bias=300),
        # ten copy candidates of twenty tokens under a grammar, half of the batch copying
        dict(logits, name="verify_candidates", kind="verify", B=32, R=201, k=20, W=10, V=128256,
             L=4096, grammar=True),
        # few users with long documents: the history counts; an odd vocabulary, half precision
        dict(logits, name="verify_long_odd", kind="verify", B=7, R=11, k=10, V=50257, L=32768,
             n_bias=41, src="f16"),
        # pages and slots of the ordinary batch
        dict(name="plan_chat", kind="plan", B=32, R=8, k=7, W=1, tree=False, L=4096, page=16,
             finished=2, scarce=False),
        # a large batch of trees
        dict(name="plan_trees", kind="plan", B=1024, R=60, k=7, W=1, tree=True, L=8192, page=64,
             finished=9, scarce=False),
        # what the draft model of the ordinary batch has yet to read
        dict(name="spans_lag", kind="spans", B=32, L=4096, page=16, span=21),
        # whole prompts of a large batch
        dict(name="spans_prompts", kind="spans", B=256, L=8192, page=16, span=8192),
        # one user's accepted candidate: a few rows of every layer
        dict(name="compact_one_user", kind="compact", B=1, R=61, k=20, W=3, L=200, page=16,
             planes=32, row=512),
        # ten candidates of twenty tokens, half of the batch copying
        dict(name="compact_candidates", kind="compact", B=32, R=201, k=20, W=10, L=128, page=16,
             planes=32, row=512),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


MOST_LOGITS = 32 * 60 * 128256  # elements of one logits tensor of a drawn case
MOST_TOKENS = 256 * 8192


def draw(rng):
    kind = rng.choice(["process", "process", "verify", "verify", "plan", "spans", "compact"])
    B, k, W = _log(rng, 1, 96), rng.randint(2, 12), 1
    shape = rng.choice(["chain", "chain", "tree", "candidates", "single"])
    if kind == "compact" or shape == "candidates":
        W = rng.randint(2, 10)
    if kind == "compact":
        R = 1 + W * k
        B = min(B, 48)
        row = rng.choice([128, 512, 1000, 2048])
        planes = max(1, min(_log(rng, 2, 128), 150000000 // (B * (R + 232) * row * 2)))
        return dict(kind="compact", B=B, R=R, k=k, W=W, L=_log(rng, 16, 200),
                    page=rng.choice([1, 16, 16, 24, 64]), planes=planes, row=row)
    if kind == "spans":
        B = _log(rng, 1, 512)
        L = max(16, min(_log(rng, 64, 32768), MOST_TOKENS // B))
        return dict(kind="spans", B=B, L=L, page=rng.choice([1, 16, 16, 24, 64, 256]),
                    span=rng.choice([min(L, rng.randint(2, 40)), L]))
    tree = shape == "tree"
    R = 1 if shape == "single" else rng.randint(max(12, k + 1), 64) if tree else 1 + W * k
    if shape == "single":
        k = 0
    if kind == "plan":
        B = _log(rng, 1, 1024)
        L = max(16, min(_log(rng, 64, 32768), 4 * MOST_TOKENS // B))
        scarce = rng.random() < 0.3
        return dict(kind="plan", B=B, R=R, k=k, W=W, tree=tree, L=L,
                    page=rng.choice([1, 16, 16, 24, 64]),
                    finished=0 if scarce else rng.randint(0, max(1, B // 8)), scarce=scarce)
    c = dict(kind=kind, B=B, R=R, k=k, W=W, tree=tree,
             V=rng.choice([32000, 50257, 128256, 151936, _log(rng, 1000, 200000)]),
             L=max(8, min(_log(rng, 8, 40000), 1048576 // B)),
             penalties=rng.random() < 0.8, n_bias=rng.choice([0, 0, rng.randint(1, 300)]),
             grammar=rng.random() < 0.4, src=rng.choice(["bf16", "bf16", "f16", "f32"]))
    c["out"] = rng.choice(["bf16", c["src"]]) if kind == "process" else "bf16"
    c["penalties"] |= not c["n_bias"] and not c["grammar"]
    while c["B"] * c["R"] * c["V"] > MOST_LOGITS and c["B"] > 1:
        c["B"] //= 2
    return c


# ------------------------------------------------------------------ inputs

def _zipf(g, shape, V, s=1.1):
    """Truncated Zipf token ids (the continuous inverse CDF, rounded down)."""
    u = torch.rand(shape, generator=g, device=DEV, dtype=torch.float64)
    a = 1.0 - s
    x = ((float(V + 1) ** a - 1.0) * u + 1.0) ** (1.0 / a)
    return (x.long() - 1).clamp_(0, V - 1).to(torch.int32)


def _rand(g, *shape):
    return torch.rand(shape, generator=g, device=DEV)


def _nodes(case):
    """Drafted nodes per sequence, anchor included: with several candidates
    every second sequence copies, the others draft a chain of k tokens."""
    B, R = case["B"], case["R"]
    return [R if case["W"] == 1 or b % 2 == 0 else 1 + case["k"] for b in range(B)]


def _draft(case, g):
    """dpar [B, R], dn [B]: a chain, a random tree, or W chains behind the anchor."""
    B, R, k = case["B"], case["R"], case["k"]
    i = torch.arange(R, device=DEV, dtype=torch.int32)
    if case.get("tree"):
        # parents spread over the earlier nodes: paths of several times ln R
        dpar = (_rand(g, B, R) * i).to(torch.int32)
    elif case["W"] > 1:
        dpar = torch.where((i - 1) % k == 0, torch.zeros_like(i), i - 1).expand(B, R).clone()
        one = torch.arange(B, device=DEV) % 2 == 1
        dpar[one] = i - 1
    else:
        dpar = (i - 1).expand(B, R).clone()
    dpar[:, 0] = -1
    dn = torch.tensor(_nodes(case), dtype=torch.int32, device=DEV)
    dpar[i[None, :] >= dn[:, None]] = -1
    return dpar.contiguous(), dn


def _ancestors(dpar, dn):
    """[B, R, R] float: 1 where node j is node i or an ancestor of it."""
    B, R = dpar.shape
    i = torch.arange(R, device=DEV)
    ok = (dpar >= 0) & (dpar < i) & (i < dn[:, None])
    up = torch.zeros(B, R, R, device=DEV)
    up.scatter_(2, dpar.clamp(min=0).long()[:, :, None], ok.float()[:, :, None])
    anc = (up + torch.eye(R, device=DEV)).clamp_(max=1.0)
    n = 1
    while n < R:  # paths of up to n edges, doubled
        anc = torch.bmm(anc, anc).clamp_(max=1.0)
        n *= 2
    return anc * (i < dn[:, None]).float()[:, :, None]


def _logits_state(case, g):
    B, R, V, L = case["B"], case["R"], case["V"], case["L"]
    st = {"case": case}
    st["tokens"] = _zipf(g, (B, L), V)
    st["lengths"] = (L - (_rand(g, B) * (L // 16)).long()).to(torch.int32)
    st["prompt_lens"] = (st["lengths"] * _rand(g, B)).to(torch.int32)
    st["dpar"], st["dn"] = _draft(case, g)
    dtok = _zipf(g, (B, R), V)
    # drafts repeat what the context holds about half of the time
    at = (_rand(g, B, R) * L).long().clamp_(max=L - 1)
    dtok = torch.where(_rand(g, B, R) < 0.5, st["tokens"].gather(1, at), dtok)
    i = torch.arange(R, device=DEV)
    st["dtok"] = torch.where((i >= 1) & (i < st["dn"][:, None]), dtok,
                             torch.full_like(dtok, -1)).contiguous()
    x = torch.randn((B, R, V), generator=g, device=DEV).mul_(2.0)
    # an accepted path: the drafted children along it are the likely tokens
    leaf = (_rand(g, B) * st["dn"]).long()
    path = _ancestors(st["dpar"], st["dn"])[torch.arange(B, device=DEV), leaf] > 0
    b, n = torch.nonzero(path & (i >= 1), as_tuple=True)
    x[b, st["dpar"][b, n].long(), st["dtok"][b, n].long()] = 24.0
    st["logits"] = x.to(TYPES[case["src"]])
    del x
    for name in ("repetition", "frequency", "presence"):
        st[name] = None
    if case["penalties"]:
        st["repetition"] = 1.0 + 0.5 * _rand(g, B)
        st["frequency"] = 0.8 * _rand(g, B)
        st["presence"] = 1.5 * _rand(g, B) - 0.5
    st["bias_ids"] = st["bias_vals"] = None
    if case["n_bias"]:
        n = case["n_bias"]
        ids = (_rand(g, B, n) * V).to(torch.int32)
        ids[:, 1::2] = _zipf(g, (B, n), V)[:, 1::2]
        used = (torch.arange(B, device=DEV) * 7 + n) % (n + 1)  # some lists are shorter
        ids[torch.arange(n, device=DEV)[None, :] >= used[:, None].clamp(min=1)] = -1
        st["bias_ids"] = ids
        st["bias_vals"] = 10.0 * _rand(g, B, n) - 5.0
        st["bias_vals"][:, ::17] = -100.0
    st["allowed"] = st["allowed_on"] = None
    if case["grammar"]:
        words = (V + 31) // 32
        bits = torch.randint(-2 ** 31, 2 ** 31, (B, R, words), generator=g, device=DEV,
                             dtype=torch.int64).to(torch.int32)
        # inside a string nearly everything is allowed, between fields nearly nothing
        some = _rand(g, B, R, words) < 0.02
        few = (_rand(g, B, R) < 0.5)[:, :, None]
        st["allowed"] = torch.where(few, torch.where(some, bits, torch.zeros_like(bits)),
                                    torch.where(some, bits, torch.full_like(bits, -1)))
        st["allowed_on"] = (torch.arange(B, device=DEV) % 4 != 3).to(torch.int32)
    return st


def _pages(case, g, count):
    """Distinct page numbers in a random order."""
    return torch.randperm(count, generator=g, device=DEV).to(torch.int32)


def _plan_state(case, g):
    B, R, L, page = case["B"], case["R"], case["L"], case["page"]
    st = {"case": case}
    st["dpar"], st["dn"] = _draft(case, g)
    lengths = (L - (_rand(g, B) * (L // 2)).long()).to(torch.int32)
    held = (lengths - 1 - (_rand(g, B) * 8).to(torch.int32)).clamp(min=0)  # pages of the last step
    held = (held + page - 1) // page
    if case["finished"]:
        at = torch.randperm(B, generator=g, device=DEV)[:case["finished"]]
        lengths[at] = 0
    most = (L + R + page - 1) // page
    st["lengths"], st["held"] = lengths, held.clamp(max=most).to(torch.int32)
    total = B * most + 3
    ids = _pages(case, g, total)
    st["table"] = torch.full((B, most), -1, dtype=torch.int32, device=DEV)
    have = torch.arange(most, device=DEV)[None, :] < st["held"][:, None]
    n = int(have.sum())
    st["table"][have] = ids[:n]
    free = total - n
    head = total - total // 3  # the ring's free part wraps around
    ring = torch.full((total,), -1, dtype=torch.int32, device=DEV)
    ring[(head + torch.arange(free, device=DEV)) % total] = ids[n:]
    count = min(free, B // 2) if case["scarce"] else free
    st["ring"] = ring
    st["ring_state"] = torch.tensor([head, count], dtype=torch.int32, device=DEV)
    st["slots"] = torch.full((B, R), -1, dtype=torch.int64, device=DEV)
    st["positions"] = torch.full((B, R), -1, dtype=torch.int32, device=DEV)
    st["missing"] = torch.zeros(B, dtype=torch.int32, device=DEV)
    return st


def _spans_state(case, g):
    B, L, page = case["B"], case["L"], case["page"]
    st = {"case": case}
    st["tokens"] = _zipf(g, (B, L), 128256)
    end = (L - (_rand(g, B) * (L // 4)).long()).to(torch.int32)
    if case["span"] < L:
        length = torch.minimum((_rand(g, B) * (case["span"] + 1)).to(torch.int32), end)
    else:
        length = end.clone()
    st["end"], st["begin"] = end, end - length
    most = (L + page - 1) // page
    st["held"] = (end + page - 1) // page
    st["table"] = _pages(case, g, B * most).view(B, most)
    total = B * case["span"]
    st["cu"] = torch.zeros(B + 1, dtype=torch.int32, device=DEV)
    st["slots"] = torch.full((total,), -1, dtype=torch.int64, device=DEV)
    for name in ("positions", "packed", "seq"):
        st[name] = torch.full((total,), -1, dtype=torch.int32, device=DEV)
    return st


def _compact_state(case, g):
    B, R, k, W, page = case["B"], case["R"], case["k"], case["W"], case["page"]
    st = {"case": case}
    st["dpar"], st["dn"] = _draft(case, g)
    most = (case["L"] + R + page - 1) // page
    table = _pages(case, g, B * most).view(B, most).long()
    pos = (case["L"] - (_rand(g, B) * (case["L"] // 2)).long() - 1)[:, None]
    pos = pos + torch.arange(R, device=DEV)[None, :]
    slots = table.gather(1, pos // page) * page + pos % page
    i = torch.arange(R, device=DEV)
    st["slots"] = torch.where(i < st["dn"][:, None], slots, torch.full_like(slots, -1))
    # copying sequences accept one of the later candidates in full, the others
    # a part of their chain (already in place)
    b = torch.arange(B, device=DEV)
    cand = 1 + (b // 2) % (W - 1)
    part = (_rand(g, B) * (k + 1)).long()
    st["accept_node"] = torch.where(b % 2 == 0, (cand + 1) * k, part).to(torch.int32)
    st["cache"] = torch.randn((case["planes"], B * most * page, case["row"]), generator=g,
                              device=DEV, dtype=torch.bfloat16)
    return st


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    kind = case["kind"]
    if kind in ("process", "verify"):
        st = _logits_state(case, g)
    else:
        st = {"plan": _plan_state, "spans": _spans_state, "compact": _compact_state}[kind](case, g)
    B, R = case["B"], case.get("R")
    if kind == "process":
        st["out"] = torch.zeros(st["logits"].shape, dtype=TYPES[case["out"]], device=DEV)
    if kind == "verify":
        for name in ("accept_len", "accept_node", "bonus"):
            st[name] = torch.zeros(B, dtype=torch.int32, device=DEV)
        for name in ("out_tokens", "amax"):
            st[name] = torch.zeros((B, R), dtype=torch.int32, device=DEV)
    if own:
        from paper_2609_20186_amd import binding as sd
        st["sd"] = sd
        if kind in ("process", "verify"):
            opt = {n: st[n] for n in ("repetition", "frequency", "presence", "bias_ids",
                                      "bias_vals", "allowed", "allowed_on")}
            ctx = {n: st[n] for n in ("tokens", "lengths", "prompt_lens")}
            st["args"] = sd.build_logits_args(st["logits"], st["dtok"], st["dpar"], st["dn"],
                                              **ctx, **opt)
        if kind == "verify":
            st["workspace"] = sd.alloc_workspace(B, R)
        if kind == "plan":
            st["args"] = sd.build_page_args(
                st["lengths"], st["dpar"], st["dn"], case["L"], case["page"], st["table"],
                st["held"], st["ring"], st["ring_state"], st["slots"], st["positions"],
                st["missing"])
            st["workspace"] = sd.alloc_workspace(B, 0)
    return st


# ------------------------------------------------------------------ plain forms

def _processed(st):
    """The processed logits [B, R, V] in 32 bits."""
    case = st["case"]
    B, R, V, L = case["B"], case["R"], case["V"], case["L"]
    y = st["logits"].float()
    if case["penalties"]:
        at = torch.arange(L, device=DEV)
        ids = st["tokens"].long()
        live = at < st["lengths"][:, None]
        prompt = live & (at < st["prompt_lens"][:, None])
        seen = torch.zeros(B, V, device=DEV).scatter_add_(1, ids, prompt.float())
        count = torch.zeros(B, V, device=DEV).scatter_add_(1, ids, (live & ~prompt).float())
        # the drafted tokens on each row's path (not the anchor: it is the
        # last token of the context)
        anc = _ancestors(st["dpar"], st["dn"])
        anc[:, :, 0] = 0.0
        nodes = st["dtok"].clamp(min=0).long()[:, None, :].expand(B, R, R)
        count = count[:, None, :].repeat(1, R, 1).scatter_add_(2, nodes, anc)
        rho = st["repetition"][:, None, None]
        y = torch.where((seen[:, None, :] > 0) | (count > 0), torch.where(y > 0, y / rho, y * rho),
                        y)
        y = y - st["frequency"][:, None, None] * count
        y = y - st["presence"][:, None, None] * (count > 0).float()
        del count, anc, nodes
    if case["n_bias"]:
        n = case["n_bias"]
        ids = st["bias_ids"].long()
        rank = torch.where(ids >= 0, torch.arange(1, n + 1, device=DEV), torch.zeros_like(ids))
        # of several entries for one token the last one holds
        last = torch.zeros(B, V, dtype=torch.int64, device=DEV)
        last.scatter_reduce_(1, ids.clamp(min=0), rank, "amax")
        val = torch.cat([torch.zeros(B, 1, device=DEV), st["bias_vals"]], 1).gather(1, last)
        y = y + val[:, None, :]
    if case["grammar"]:
        bits = (st["allowed"][:, :, :, None] >> torch.arange(32, device=DEV)) & 1
        bits = bits.view(B, R, -1)[:, :, :V] != 0
        bits = bits | (st["allowed_on"] == 0)[:, None, None]
        y = torch.where(bits, y, torch.full((), -math.inf, device=DEV))
    return y


def _plain_process(st):
    i = torch.arange(st["case"]["R"], device=DEV)
    live = (i < st["dn"][:, None])[:, :, None]
    return {"out": torch.where(live, _processed(st).to(st["out"].dtype), st["out"])}


def _plain_verify(st):
    case = st["case"]
    B, R, V = case["B"], case["R"], case["V"]
    y = _processed(st).to(torch.bfloat16).float()
    top = y.amax(2, keepdim=True)
    vocab = torch.arange(V, device=DEV)
    amax = torch.where(y == top, vocab, torch.full((), V, device=DEV)).amin(2)
    i = torch.arange(R, device=DEV)
    live = i < st["dn"][:, None]
    par = st["dpar"].clamp(min=0).long()
    good = (st["dtok"] == amax.gather(1, par)) & (i >= 1) & live
    good[:, 0] = True
    anc = _ancestors(st["dpar"], st["dn"])
    depth = anc.sum(2) - 1.0
    fails = torch.bmm(anc, (~good).float()[:, :, None])[:, :, 0]
    reach = torch.where((fails == 0) & live, depth.long() * R + (R - 1 - i), -1)
    best = reach.amax(1)
    node = R - 1 - best % R
    alen = best // R
    rows = torch.arange(B, device=DEV)
    bonus = amax[rows, node]
    path = anc[rows, node] > 0
    rank = path.long().cumsum(1) - 1           # nodes ascend along a path
    out = torch.full((B, R + 1), -1, dtype=torch.int64, device=DEV)
    to = torch.where(path & (i >= 1), rank - 1, torch.full_like(rank, R))
    out.scatter_(1, to, st["dtok"].long())
    out.scatter_(1, alen[:, None], bonus[:, None])
    i32 = torch.int32
    return {"accept_len": alen.to(i32), "accept_node": node.to(i32), "bonus": bonus.to(i32),
            "out_tokens": out[:, :R].to(i32),
            "amax": torch.where(live, amax, torch.full_like(amax, -1)).to(i32)}


def _plain_plan(st):
    case = st["case"]
    B, R, page = case["B"], case["R"], case["page"]
    most, total = st["table"].shape[1], st["ring"].numel()
    L, n, held = st["lengths"].long(), st["dn"].long(), st["held"].long()
    need = torch.where(L > 0, (L - 1 + n + page - 1) // page, torch.zeros_like(L))
    need = need.clamp(max=most)
    grow = torch.where(L > 0, (need - held).clamp(min=0), torch.zeros_like(L))
    back = torch.where(L > 0, torch.zeros_like(L), held)
    upto, backto = grow.cumsum(0), back.cumsum(0)
    head, count = st["ring_state"][0].long(), st["ring_state"][1].long()
    served = upto <= count
    took = torch.where(served, grow, torch.zeros_like(grow))
    col = torch.arange(most, device=DEV)[None, :]
    k = col - held[:, None]
    new = (k >= 0) & (k < took[:, None])
    page_of = st["ring"][((head + (upto - grow)[:, None] + k) % total).long()]
    gone = col < back[:, None]
    to = torch.where(gone, (head + count + (backto - back)[:, None] + col) % total,
                     torch.full_like(k, total))
    ring = torch.cat([st["ring"], st["ring"][:1]])
    ring.scatter_(0, to.flatten(), st["table"].flatten())
    st["ring"].copy_(ring[:total])
    st["table"].copy_(torch.where(new, page_of, torch.where(gone, torch.full_like(page_of, -1),
                                                            st["table"])))
    st["held"].copy_(torch.where(L > 0, held + took, torch.zeros_like(held)))
    st["missing"].copy_(grow - took)
    popped = took.sum()
    st["ring_state"].copy_(torch.stack([(head + popped) % total, count - popped + back.sum()]))
    i = torch.arange(R, device=DEV)[None, :]
    live = (i < n[:, None]) & (L > 0)[:, None]
    pos = L[:, None] - 1 + i
    at = pos // page
    have = live & (at < st["held"].long()[:, None])
    slot = st["table"].gather(1, at.clamp(0, most - 1)).long() * page + pos % page
    depth = _ancestors(st["dpar"], st["dn"]).sum(2).long() - 1
    st["slots"].copy_(torch.where(have, slot, torch.full_like(slot, -1)))
    st["positions"].copy_(torch.where(live, L[:, None] - 1 + depth, torch.full_like(depth, -1)))
    return {n: st[n] for n in ("table", "held", "ring", "ring_state", "slots", "positions",
                               "missing")}


def _plain_spans(st):
    case = st["case"]
    B, page = case["B"], case["page"]
    most, total = st["table"].shape[1], st["slots"].numel()
    size = (st["end"] - st["begin"]).long()
    st["cu"][1:].copy_(size.cumsum(0))
    j = torch.arange(total, device=DEV)
    seq = torch.searchsorted(st["cu"][1:].long(), j, right=True)
    live = seq < B
    b = seq.clamp(max=B - 1)
    pos = st["begin"].long()[b] + j - st["cu"].long()[b]
    at = (pos // page).clamp(0, most - 1)
    slot = torch.where(at < st["held"][b], st["table"][b, at].long() * page + pos % page,
                       torch.full_like(pos, -1))
    tok = st["tokens"][b, pos.clamp(0, case["L"] - 1)]
    for name, val in (("slots", slot), ("positions", pos), ("packed", tok), ("seq", b)):
        st[name].copy_(torch.where(live, val.to(st[name].dtype), st[name]))
    return {n: st[n] for n in ("cu", "slots", "positions", "packed", "seq")}


def _plain_compact(st):
    B, R, k = (st["case"][n] for n in ("B", "R", "k"))
    node = st["accept_node"].long()
    path = _ancestors(st["dpar"], st["dn"])[torch.arange(B, device=DEV), node] > 0
    rank = torch.where(path, path.long().cumsum(1) - 1, torch.full((), R, device=DEV))
    src = torch.cat([st["slots"], st["slots"][:, :1]], 1).scatter_(1, rank, st["slots"])
    # no path is longer than k nodes behind the anchor; places beyond its own
    # path a sequence copies onto themselves
    to, fro = st["slots"][:, :k + 1].flatten(), src[:, :k + 1].flatten()
    st["cache"][:, to] = st["cache"][:, fro]
    return {"cache": st["cache"]}


# ------------------------------------------------------------------ one pass

def run(st):
    kind = st["case"]["kind"]
    if not own:
        return {"process": _plain_process, "verify": _plain_verify, "plan": _plain_plan,
                "spans": _plain_spans, "compact": _plain_compact}[kind](st)
    sd = st["sd"]
    if kind == "process":
        sd.switchsd_process_logits(st["args"], st["out"])
        return {"out": st["out"]}
    if kind == "verify":
        sd.switchsd_verify_processed(st["args"], st["accept_len"], st["accept_node"], st["bonus"],
                                     st["out_tokens"], st["amax"], st["workspace"])
        return {n: st[n] for n in ("accept_len", "accept_node", "bonus", "out_tokens", "amax")}
    if kind == "plan":
        sd.switchsd_page_plan(st["args"], st["workspace"])
        return {n: st[n] for n in ("table", "held", "ring", "ring_state", "slots", "positions",
                                   "missing")}
    if kind == "spans":
        sd.switchsd_span_slots(st["begin"], st["end"], st["tokens"], st["table"], st["held"],
                               st["case"]["page"], st["cu"], st["slots"], st["positions"],
                               st["packed"], st["seq"])
        return {n: st[n] for n in ("cu", "slots", "positions", "packed", "seq")}
    sd.switchsd_compact_cache(st["cache"], st["slots"], st["dpar"], st["dn"], st["accept_node"])
    return {"cache": st["cache"]}


def work(case):
    kind, B, R = case["kind"], case["B"], case.get("R")
    if kind in ("process", "verify"):
        V, rows = case["V"], sum(_nodes(case))
        by = rows * V * SIZE[case["src"]] + 12 * B * R
        fl = 0
        if case["penalties"]:
            by += B * (int(case["L"] * 31 / 32) * 4 + 20)
            fl += 5 * rows * V
        by += B * case["n_bias"] * 8
        fl += rows * V if case["n_bias"] else 0
        if case["grammar"]:
            by += rows * ((V + 31) // 32) * 4 * 3 // 4
        by += rows * V * SIZE[case["out"]] if kind == "process" else 4 * (3 * B + 2 * B * R)
        return {"bytes": by, "flops": fl + (rows * V if kind == "verify" else 0)}
    if kind == "plan":
        return {"bytes": B * (4 * 6 + 4 * (1 + R // case["page"])) + 16 * B * R,
                "flops": 4 * B * R}
    if kind == "spans":
        n = B * (case["L"] * 7 // 8 if case["span"] == case["L"] else case["span"] // 2)
        return {"bytes": 24 * n + 4 * n // case["page"] + 16 * B, "flops": 4 * n}
    moved = (B + 1) // 2 * case["k"]
    return {"bytes": moved * case["planes"] * case["row"] * 4 + 20 * B * R, "flops": 0}


# ------------------------------------------------------------------ definitions in 64 bits

def exact(case, seed):
    kind = case["kind"]
    if kind in ("verify", "plan", "spans"):
        return None  # whole numbers only
    st = prepare(case, seed)
    dpar, dn = st["dpar"].tolist(), st["dn"].tolist()

    def path(b, node):
        """The nodes from `node` up to the child of the anchor."""
        up = []
        while node > 0:
            up.append(node)
            q = dpar[b][node]
            if not 0 <= q < node:
                break
            node = q
        return up

    if kind == "compact":
        cache, slots = st["cache"].double(), st["slots"].tolist()
        before = st["cache"]
        for b, node in enumerate(st["accept_node"].tolist()):
            for j, q in enumerate(reversed(path(b, node)), 1):
                cache[:, slots[b][j]] = before[:, slots[b][q]].double()
        return {"cache": cache}
    V = case["V"]
    out = st["out"].double()
    dtok = st["dtok"].tolist()
    for b in range(case["B"]):
        x = st["tokens"][b, :int(st["lengths"][b])].long()
        P = int(st["prompt_lens"][b])
        given = torch.bincount(x[:P], minlength=V)
        made = torch.bincount(x[P:], minlength=V)
        bias = torch.zeros(V, dtype=torch.float64, device=DEV)
        if case["n_bias"]:
            table = {}
            for v, val in zip(st["bias_ids"][b].tolist(), st["bias_vals"][b].double().tolist()):
                if v >= 0:
                    table[v] = val
            if table:
                bias[torch.tensor(list(table), device=DEV)] = torch.tensor(
                    list(table.values()), dtype=torch.float64, device=DEV)
        for r in range(dn[b]):
            y = st["logits"][b, r].double()
            if case["penalties"]:
                c = made.clone()
                for q in path(b, r):
                    c[dtok[b][q]] += 1
                rho, f, p = (st[n][b].double() for n in ("repetition", "frequency", "presence"))
                hit = (given + c) > 0
                y = torch.where(hit & (y > 0), y / rho, torch.where(hit, y * rho, y))
                y = y - f * c - p * (c > 0)
            y = y + bias
            if case["grammar"] and int(st["allowed_on"][b]):
                w = st["allowed"][b, r].long() & 0xFFFFFFFF
                bit = (w[torch.arange(V, device=DEV) // 32] >> (torch.arange(V, device=DEV) % 32))
                y[(bit & 1) == 0] = -math.inf
            out[b, r] = y
    return {"out": out}
