"""The operators between the page plan and the verified tokens, as cases: a paged
cache that is written and read, and the probabilities of what a step emitted.

  own                False: run() computes the plain form (elementary torch
                     operations); True: it makes the library's calls
  listed()           the cases by name
  draw(rng)          one more case from the same ranges
  prepare(case, s)   what the engine holds before the call, from the seed alone
  run(state)         one pass through one operator, and its outputs
  work(case)         bytes and operations a pass cannot do without
  exact(case, s)     the computed outputs in 64 bits, from the definitions

Kinds of case:
  store   keys and values of new tokens written to their cache slots
          (switchsd_store_cache)
  attend  attention of new tokens -- drafted rows, single tokens, chunks of
          prompts -- over the paged cache (switchsd_paged_attention)
  score   log probabilities of given tokens, entropies, ranks and the most
          likely alternatives (switchsd_token_logprobs)
  grad    the gradient of log probabilities and entropies with respect to the
          logits (switchsd_token_logprobs_grad)
"""
import math

import torch

own = False

DEV = "cuda"
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32,
         "e4m3": torch.float8_e4m3fn}
SIZE = {"bf16": 2, "f16": 2, "f32": 4, "e4m3": 1}


# ------------------------------------------------------------------ cases

def listed():
    heads = dict(Hq=32, Hkv=8, D=128, page=16, type="bf16", cache="bf16")
    draft = dict(heads, kind="attend", packed=False, W=1, tree=False, k=0, decoding=0)
    score = dict(path=False, tree=False, k=0, rank=True, entropy=True, type="bf16", T=1.0)
    return [
        # the drafted rows of the ordinary serving batch, one layer
        dict(heads, name="store_step", kind="store", packed=False, B=32, R=8, L=4096),
        # whole prompts of a batch, half precision, a small model's heads
        dict(heads, name="store_prompts", kind="store", packed=True, B=16, R=2048, L=4096,
             type="f16", cache="f16", D=64, page=24),
        # one user without a draft: launch latency is everything
        dict(draft, name="attend_one_token", B=1, R=1, L=512),
        # the ordinary serving batch: chains of seven drafted tokens
        dict(draft, name="attend_chat", B=32, R=8, k=7, L=4096),
        # a large batch of drafted trees
        dict(draft, name="attend_trees", B=256, R=60, k=7, L=2048, tree=True),
        # ten copy candidates of twenty tokens for half of the batch, keys and values in 8 bits
        dict(draft, name="attend_candidates", B=32, R=201, k=20, W=10, L=4096, cache="e4m3"),
        # few users with long documents, wide heads, half precision, odd pages
        dict(draft, name="attend_long_odd", B=7, R=11, k=10, L=32768, Hq=64, page=24, type="f16",
             cache="f16"),
        # prompts taken in chunks, beside sequences that decode one token
        dict(draft, name="attend_prompts", packed=True, B=8, R=2048, L=8192, decoding=2),
        # what a step emitted, for a request that asks for the twenty likeliest alternatives
        dict(score, name="score_chat", kind="score", path=True, tree=True, B=32, R=60, k=7,
             V=128256, n_top=20),
        # prompts scored token by token, each with its likeliest alternative
        dict(score, name="score_prompts", kind="score", B=8, R=512, V=151936, n_top=1),
        # a short sequence with an odd vocabulary and float logits
        dict(score, name="grad_short_odd", kind="grad", B=1, R=23, V=50257, type="f32", T=0.7),
        # a training batch: policy loss and entropy bonus
        dict(score, name="grad_batch", kind="grad", B=4, R=1024, V=128256),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


MOST_ELEMENTS = 256 * 2200 * 8 * 128  # keys of one drawn case
MOST_PAIRS = 256 * 60 * 32 * 2048     # rows x query heads x context of one drawn case
MOST_QUERIES = 8 * 2048 * 48 * 128    # queries, keys and values of one drawn case's new rows
MOST_LOGITS = 4 * 1024 * 128256       # elements of one logits tensor of a drawn case


def draw(rng):
    kind = rng.choice(["store", "attend", "attend", "attend", "attend", "score", "score", "grad"])
    if kind in ("store", "attend"):
        Hkv = rng.choice([1, 2, 4, 8, 8, 8, 16])
        D = rng.choice([64, 128, 128, 128, 256])
        kt = rng.choice(["bf16", "bf16", "f16"])
        c = dict(kind=kind, Hq=Hkv * rng.choice([1, 2, 4, 4, 5, 7, 8, 16]), Hkv=Hkv, D=D,
                 page=rng.choice([1, 16, 16, 24, 64, 256]), type=kt, cache=kt)
        c["packed"] = rng.random() < 0.4
        c["B"] = _log(rng, 1, 64 if c["packed"] else 256)
        c["L"] = max(16, min(_log(rng, 64, 65536), MOST_ELEMENTS // (c["B"] * Hkv * D)))
        width = (c["Hq"] + 2 * Hkv) * D
        if kind == "store":
            c["R"] = min(c["L"], _log(rng, 16, 4096)) if c["packed"] else rng.randint(1, 64)
            c["R"] = min(c["R"], MOST_QUERIES // (c["B"] * width) + 1)
            return c
        c["cache"] = rng.choice([kt, kt, "e4m3"])
        c["W"], c["tree"], c["k"], c["decoding"] = 1, False, 0, 0
        if c["packed"]:
            c["R"] = min(c["L"], _log(rng, 16, 4096))
            c["decoding"] = rng.randint(0, c["B"] // 2)
        else:
            shape = rng.choice(["single", "chain", "chain", "tree", "candidates"])
            c["k"] = 0 if shape == "single" else rng.randint(2, 20)
            c["tree"] = shape == "tree"
            c["W"] = rng.randint(2, 10) if shape == "candidates" else 1
            c["R"] = rng.randint(12, 64) if c["tree"] else 1 + c["W"] * c["k"]
        while c["B"] > 1 and c["B"] * c["R"] > min(MOST_PAIRS // (c["Hq"] * c["L"]),
                                                   MOST_QUERIES // width):
            c["B"] //= 2
        if c["packed"]:
            c["R"] = max(1, min(c["R"], MOST_PAIRS // (c["Hq"] * c["L"])))
        c["decoding"] = min(c["decoding"], c["B"] // 2)
        return c
    c = dict(kind=kind, path=False, tree=False, k=0, rank=rng.random() < 0.7,
             entropy=rng.random() < 0.7, type=rng.choice(["bf16", "bf16", "f16", "f32"]),
             T=rng.choice([1.0, 1.0, 0.7, 1.3]),
             V=rng.choice([32000, 50257, 128256, 151936, _log(rng, 1000, 200000)]))
    if kind == "score":
        c["path"] = rng.random() < 0.5
        c["n_top"] = rng.choice([0, 1, 5, 20, rng.randint(1, 32)])
    if c["path"]:
        c["B"], c["k"], c["tree"] = _log(rng, 1, 128), rng.randint(2, 12), rng.random() < 0.5
        c["R"] = rng.randint(13, 64) if c["tree"] else 1 + c["k"]
    else:
        c["B"], c["R"] = _log(rng, 1, 64), _log(rng, 1, 512)
    most = MOST_LOGITS // (2 if c["type"] == "f32" else 1)
    while c["B"] * c["R"] * c["V"] > most and c["B"] > 1:
        c["B"] //= 2
    return c


# ------------------------------------------------------------------ inputs

def _rand(g, *shape):
    return torch.rand(shape, generator=g, device=DEV)


def _draft(case, g):
    """dpar [B, R], dn [B]: a chain, a random tree, or W chains of k tokens behind
    the anchor for every second sequence and one for the others."""
    B, R, k = case["B"], case["R"], case["k"]
    i = torch.arange(R, device=DEV, dtype=torch.int32)
    dn = torch.full((B,), R, dtype=torch.int32, device=DEV)
    if case["tree"]:
        dpar = (_rand(g, B, R) * i).to(torch.int32)
        dn -= (_rand(g, B) * (R // 4)).to(torch.int32)
    else:
        dpar = (i - 1).expand(B, R).clone()
        if case.get("W", 1) > 1:
            dpar[::2] = torch.where((i - 1) % k == 0, torch.zeros_like(i), i - 1)
            dn[1::2] = 1 + k
    dpar[:, 0] = -1
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


def _cache_state(case, g):
    """Contexts, pages, slots of the new rows, and the new rows' projection:
    queries, keys and values side by side, as one matrix product leaves them."""
    B, R, L, page = case["B"], case["R"], case["L"], case["page"]
    Hq, Hkv, D = case["Hq"], case["Hkv"], case["D"]
    st = {"case": case}
    if case["packed"]:
        n = (R - (_rand(g, B) * (R // 2)).long()).clamp(max=L)
        n[:case.get("decoding", 0)] = 1
        end = torch.maximum(n, L - (_rand(g, B) * (L // 2)).long())
        st["cu"] = torch.cat([n.new_zeros(1), n.cumsum(0)]).to(torch.int32)
        first = end - n
        st["begin"] = first.to(torch.int32)
        st["rows"] = B * R
        row = torch.arange(B * R, device=DEV)
        seq = torch.searchsorted(st["cu"][1:].long(), row, right=True)
        live = seq < B
        seq = seq.clamp(max=B - 1)
        pos = first[seq] + row - st["cu"].long()[seq]
    else:
        if case["kind"] == "attend":
            st["dpar"], st["dn"] = _draft(case, g)
        else:
            st["dn"] = (R - (_rand(g, B) * (R // 4)).long()).to(torch.int32)
        st["lengths"] = (L - (_rand(g, B) * (L // 2)).long()).to(torch.int32)
        if B >= 8:
            st["lengths"][B // 3] = 0  # a finished sequence
        st["rows"] = B * R
        row = torch.arange(B * R, device=DEV)
        seq = row // R
        live = (row % R < st["dn"][seq]) & (st["lengths"][seq] > 0)
        pos = st["lengths"].long()[seq] - 1 + row % R
        first, n = st["lengths"].long() - 1, st["dn"].long()
        end = torch.where(st["lengths"] > 0, first + n, torch.zeros_like(first))
    most = (L + R + page - 1) // page
    st["held"] = ((end + page - 1) // page).to(torch.int32)
    pages = B * most + 3
    ids = torch.randperm(pages, generator=g, device=DEV)[:B * most].to(torch.int32).view(B, most)
    held = torch.arange(most, device=DEV) < st["held"][:, None]
    st["table"] = torch.where(held, ids, torch.full_like(ids, -1))
    slot = ids.long()[seq, (pos // page).clamp(0, most - 1)] * page + pos % page
    st["slots"] = torch.where(live, slot, torch.full_like(slot, -1))
    st["qkv"] = torch.randn((st["rows"], (Hq + 2 * Hkv) * D), generator=g, device=DEV).mul_(1.25) \
        .to(TYPES[case["type"]])
    st["q"], st["k"], st["v"] = (
        x.view(st["rows"], -1, D) for x in st["qkv"].split([Hq * D, Hkv * D, Hkv * D], 1))
    st["k_scale"] = st["v_scale"] = None
    if case["cache"] == "e4m3":
        st["k_scale"] = 0.02 + 0.01 * _rand(g, Hkv)
        st["v_scale"] = 0.02 + 0.01 * _rand(g, Hkv)
    for name in ("k", "v"):
        x = torch.randn((pages * page, Hkv, D), generator=g, device=DEV)
        if case["cache"] == "e4m3":
            x.div_(st[name + "_scale"][:, None])
        st[name + "_cache"] = x.to(TYPES[case["cache"]])
        del x
    return st


def _score_state(case, g):
    B, R, V = case["B"], case["R"], case["V"]
    st = {"case": case}
    x = torch.randn((B, R, V), generator=g, device=DEV).mul_(2.0)
    # a few likely tokens in each row, and in every fourth one a grammar that
    # leaves a part of the vocabulary
    hot = (_rand(g, B, R, 12) * V).long()
    x.scatter_(2, hot, 6.0 + 8.0 * _rand(g, B, R, 12))
    x[:, ::4, ::3] = -math.inf
    st["logits"] = x.to(TYPES[case["type"]])
    del x
    pick = (_rand(g, B, R) * 12).long()[:, :, None]
    st["tokens"] = torch.where(_rand(g, B, R) < 0.8, hot.gather(2, pick)[:, :, 0],
                               (_rand(g, B, R) * V).long()).to(torch.int32)
    if case["path"]:
        st["dpar"], st["dn"] = _draft(case, g)
        st["accept_node"] = (_rand(g, B) * st["dn"]).to(torch.int32)
    else:
        st["dn"] = (R - (_rand(g, B) * (R // 4)).long()).to(torch.int32)
    return st


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    kind = case["kind"]
    B, R = case["B"], case["R"]
    if kind in ("store", "attend"):
        st = _cache_state(case, g)
        if kind == "attend":
            st["out"] = torch.zeros((st["rows"], case["Hq"], case["D"]),
                                    dtype=TYPES[case["type"]], device=DEV)
            st["lse"] = torch.zeros((st["rows"], case["Hq"]), device=DEV)
            st["mask"] = None
            if not case["packed"] and (case["tree"] or case["W"] > 1):
                words = (R + 31) // 32
                bits = torch.zeros((B, R, words * 32), dtype=torch.int64, device=DEV)
                bits[:, :, :R] = _ancestors(st["dpar"], st["dn"]).long()
                bits = (bits.view(B, R, words, 32) << torch.arange(32, device=DEV)).sum(3)
                st["mask"] = torch.where(bits >= 2 ** 31, bits - 2 ** 32, bits).to(torch.int32)
    else:
        st = _score_state(case, g)
        names = [("logprob", True), ("lse", True), ("entropy", case["entropy"])]
        for name, on in names if kind == "score" else []:
            st[name] = torch.zeros((B, R), device=DEV) if on else None
        if kind == "score":
            st["rank"] = torch.zeros((B, R), dtype=torch.int32, device=DEV) if case["rank"] \
                else None
            st["top_ids"] = st["top_logprobs"] = None
            if case["n_top"]:
                st["top_ids"] = torch.zeros((B, R, case["n_top"]), dtype=torch.int32, device=DEV)
                st["top_logprobs"] = torch.zeros((B, R, case["n_top"]), device=DEV)
        else:
            # what the forward pass left behind, and the loss's gradients
            st["lse"] = torch.empty((B, R), device=DEV)
            st["entropy"] = torch.empty((B, R), device=DEV)
            for b in range(B):
                z = st["logits"][b].double() / case["T"]
                lse = z.logsumexp(1)
                z.sub_(lse[:, None])
                st["lse"][b] = lse
                st["entropy"][b] = -(z.exp() * z.clamp(min=-1e30)).sum(1)
            st["g_logprob"] = torch.randn((B, R), generator=g, device=DEV)
            st["g_entropy"] = 0.1 * _rand(g, B, R) if case["entropy"] else None
            st["g_logits"] = torch.zeros_like(st["logits"])
    if own:
        from paper_2609_20186_amd import binding as sd
        st["sd"] = sd
        if kind == "attend":
            where = {n: st[n] for n in (("begin", "cu") if case["packed"] else ("lengths", "dn"))}
            st["args"] = sd.build_attention_args(
                st["rows"], R, case["Hq"], case["Hkv"], case["D"], case["page"], st["table"],
                st["held"], case["L"] + R, mask=st["mask"], **where)
            st["workspace"] = sd.alloc_attention_workspace(st["args"])
        if kind in ("score", "grad"):
            where = {n: st[n] for n in (("dpar", "accept_node") if case["path"] else ())}
            st["args"] = sd.build_logprob_args(st["logits"], st["tokens"], st["dn"],
                                               temperature=case["T"], **where)
    return st


# ------------------------------------------------------------------ plain forms

def _plain_store(st):
    row = torch.arange(st["rows"], device=DEV)
    live = st["slots"] >= 0
    if st["case"]["packed"]:
        live = live & (row < st["cu"][-1])
    # a row without a slot repeats the first one, which has one
    row = torch.where(live, row, torch.zeros_like(row))
    at = st["slots"][row]
    st["k_cache"][at] = st["k"][row].to(st["k_cache"].dtype)
    st["v_cache"][at] = st["v"][row].to(st["v_cache"].dtype)
    return {"k_cache": st["k_cache"], "v_cache": st["v_cache"]}


def _plain_attend(st):
    case = st["case"]
    B, R, page = case["B"], case["R"], case["page"]
    Hq, Hkv, D = case["Hq"], case["Hkv"], case["D"]
    G, S = Hq // Hkv, case["L"] + R
    i = torch.arange(R, device=DEV)
    if case["packed"]:
        first, n = st["begin"].long(), (st["cu"][1:] - st["cu"][:-1]).long()
        row = st["cu"][:-1].long()[:, None] + i
    else:
        first = st["lengths"].long() - 1
        n = torch.where(st["lengths"] > 0, st["dn"].long(), torch.zeros_like(first))
        row = torch.arange(B, device=DEV)[:, None] * R + i
    live = i < n[:, None]                                              # [B, R]
    row = torch.where(live, row, torch.zeros_like(row))
    pos = torch.arange(S, device=DEV)
    held = (pos[None, :] // page < st["held"][:, None]) & (pos < (first + n)[:, None])
    slot = st["table"].long()[:, (pos // page).clamp(max=st["table"].shape[1] - 1)] * page \
        + pos % page
    slot = torch.where(held, slot, torch.zeros_like(slot))
    after = pos[None, :] - first[:, None]                              # [B, S] place among the new
    if st["mask"] is None:
        seen = after[:, None, :] <= i[None, :, None]
    else:
        at = after.clamp(0, R - 1)
        word = st["mask"].long().gather(2, (at // 32)[:, None, :].expand(B, R, S))
        seen = (after < 0)[:, None, :] | ((word >> (at % 32)[:, None, :]) & 1 != 0)
    seen = seen & held[:, None, :] & live[:, :, None]                  # [B, R, S]
    k = st["k_cache"][slot].float().permute(0, 2, 3, 1).contiguous()   # [B, Hkv, D, S]
    if st["k_scale"] is not None:
        k = k * st["k_scale"][:, None, None]
    q = st["q"][row].float().view(B, R, Hkv, G, D).permute(0, 2, 1, 3, 4).reshape(B, Hkv, R * G, D)
    s = torch.matmul(q, k).view(B, Hkv, R, G, S) * (1.0 / math.sqrt(D))
    del k, q
    s = torch.where(seen[:, None, :, None, :], s, torch.full((), -math.inf, device=DEV))
    m = s.amax(4, keepdim=True)
    m = torch.where(m > -math.inf, m, torch.zeros_like(m))
    p = (s - m).exp()
    del s
    total = p.sum(4, keepdim=True)
    p = (p / torch.where(total > 0, total, torch.ones_like(total))).view(B, Hkv, R * G, S)
    v = st["v_cache"][slot].float().permute(0, 2, 1, 3).contiguous()   # [B, Hkv, S, D]
    v = torch.where(held[:, None, :, None], v, torch.zeros((), device=DEV))
    if st["v_scale"] is not None:
        v = v * st["v_scale"][:, None, None]
    o = torch.matmul(p, v).view(B, Hkv, R, G, D).permute(0, 2, 1, 3, 4).reshape(B, R, Hq, D)
    lse = (m + total.log())[..., 0].permute(0, 2, 1, 3).reshape(B, R, Hq)
    out, low = st["out"].clone(), st["lse"].clone()
    # what is no row repeats the first one
    src = torch.where(live, torch.arange(B * R, device=DEV).view(B, R), torch.zeros_like(row))
    src, to = src.flatten(), row.flatten()
    out[to] = o.reshape(B * R, Hq, D)[src].to(out.dtype)
    low[to] = lse.reshape(B * R, Hq)[src]
    return {"out": out, "lse": low}


def _plain_rows(st):
    """[B, R]: the logits row of each entry, and which entries there are."""
    B, R = st["tokens"].shape
    i = torch.arange(R, device=DEV)
    if not st["case"]["path"]:
        return i.expand(B, R), i < st["dn"][:, None]
    path = _ancestors(st["dpar"], st["dn"])[torch.arange(B, device=DEV),
                                            st["accept_node"].long()] > 0
    rank = torch.where(path, path.long().cumsum(1) - 1, torch.full((), R, device=DEV))
    node = torch.zeros((B, R + 1), dtype=torch.int64, device=DEV)
    node.scatter_(1, rank, i.expand(B, R))
    return node[:, :R], i < path.sum(1)[:, None]


def _plain_score(st):
    case = st["case"]
    row, live = _plain_rows(st)
    b, e = torch.nonzero(live, as_tuple=True)
    x = st["logits"][b, row[b, e]]                                     # [N, V]
    tok = st["tokens"][b, e].long()[:, None]
    z = x.float() / case["T"]
    m = z.amax(1, keepdim=True)
    w = (z - m).exp()
    total = w.sum(1, keepdim=True)
    lse = m + total.log()
    got = {"lse": lse[:, 0], "logprob": (z.gather(1, tok) - lse)[:, 0]}
    if case["entropy"]:
        gap = torch.where(w > 0, z - m, torch.zeros((), device=DEV))
        got["entropy"] = (total.log() - (w * gap).sum(1, keepdim=True) / total)[:, 0]
        del gap
    del w
    vocab = torch.arange(case["V"], device=DEV)
    if case["rank"]:
        mine = x.gather(1, tok)
        ahead = (x > mine) | ((x == mine) & (vocab < tok))
        got["rank"] = ahead.sum(1).to(torch.int32)
    if case["n_top"]:
        # keys that order by value, then by the lower index
        bits = x.float().view(torch.int32).long()
        key = torch.where(bits >= 0, bits, -(bits & 0x7FFFFFFF)) * (1 << 24) - vocab
        best = key.topk(case["n_top"], 1).values
        ids = -best % (1 << 24)
        got["top_ids"] = ids.to(torch.int32)
        got["top_logprobs"] = z.gather(1, ids) - lse
    res = {}
    for name in got:
        res[name] = st[name].clone()
        res[name][b, e] = got[name]
    return res


def _plain_grad(st):
    case = st["case"]
    T = case["T"]
    live = torch.arange(case["R"], device=DEV) < st["dn"][:, None]
    lp = st["logits"].float() / T - st["lse"][:, :, None]
    p = lp.exp()
    g = st["g_logprob"][:, :, None]
    d = -g * p
    if case["entropy"]:
        lp = torch.where(p > 0, lp, torch.zeros((), device=DEV))
        d = d - st["g_entropy"][:, :, None] * p * (lp + st["entropy"][:, :, None])
    d.scatter_add_(2, st["tokens"].long()[:, :, None], g)
    return {"g_logits": torch.where(live[:, :, None], (d / T).to(st["g_logits"].dtype),
                                    st["g_logits"])}


# ------------------------------------------------------------------ one pass

OUT = ("logprob", "lse", "entropy", "rank", "top_ids", "top_logprobs")


def run(st):
    kind = st["case"]["kind"]
    if not own:
        return {"store": _plain_store, "attend": _plain_attend, "score": _plain_score,
                "grad": _plain_grad}[kind](st)
    sd = st["sd"]
    if kind == "store":
        sd.switchsd_store_cache(st["k"], st["v"], st["slots"], st["k_cache"], st["v_cache"],
                                count=st["cu"][-1:] if st["case"]["packed"] else None)
        return {"k_cache": st["k_cache"], "v_cache": st["v_cache"]}
    if kind == "attend":
        sd.switchsd_paged_attention(st["args"], st["q"], st["k_cache"], st["v_cache"], st["out"],
                                    st["workspace"], lse=st["lse"], k_scale=st["k_scale"],
                                    v_scale=st["v_scale"])
        return {"out": st["out"], "lse": st["lse"]}
    if kind == "score":
        sd.switchsd_token_logprobs(st["args"], **{n: st[n] for n in OUT})
        return {n: st[n] for n in OUT if st[n] is not None}
    sd.switchsd_token_logprobs_grad(st["args"], st["lse"], st["entropy"], st["g_logprob"],
                                    st["g_entropy"], st["g_logits"])
    return {"g_logits": st["g_logits"]}


def work(case):
    kind, B, R = case["kind"], case["B"], case["R"]
    size = SIZE[case["type"]]
    if kind in ("store", "attend"):
        L, Hq, Hkv, D = case["L"], case["Hq"], case["Hkv"], case["D"]
        done = 1 if B >= 8 and not case["packed"] else 0
        if case["packed"]:
            one = case.get("decoding", 0)
            n = [1] * one + [min(R * 3 / 4, L)] * (B - one)
        elif kind == "store" or case["tree"]:
            n = [R * 7 / 8] * (B - done)
        else:
            n = [R if case["W"] == 1 or b % 2 == 0 else 1 + case["k"] for b in range(B - done)]
        if kind == "store":
            return {"bytes": sum(n) * (4 * Hkv * D * size + 8), "flops": 0}
        end = [max(x, 3 * L / 4) for x in n]
        pairs = sum(x * (e - x / 2) for x, e in zip(n, end))
        return {"bytes": sum(n) * Hq * (2 * D * size + 4) + sum(end) * 2 * Hkv * D
                * SIZE[case["cache"]], "flops": 4 * D * Hq * pairs}
    V = case["V"]
    if case["path"]:
        # the mean depth of a random tree's nodes, and the anchor
        rows = B * (math.log(7 * R / 8) + 0.58 if case["tree"] else 1 + case["k"] / 2)
    else:
        rows = B * (R - (R // 4) / 2)
    if kind == "score":
        return {"bytes": rows * (V * size + 12 + 8 * case["n_top"]), "flops": 6 * rows * V}
    return {"bytes": rows * (2 * V * size + 16), "flops": 6 * rows * V}


# ------------------------------------------------------------------ definitions in 64 bits

def exact(case, seed):
    kind = case["kind"]
    st = prepare(case, seed)

    def attend():
        B, R, page, D = case["B"], case["R"], case["page"], case["D"]
        Hq, Hkv = case["Hq"], case["Hkv"]
        G = Hq // Hkv
        out, lse = st["out"].double(), st["lse"].double()
        for b in range(B):
            if case["packed"]:
                lo, hi = st["cu"][b:b + 2].tolist()
                first, n = int(st["begin"][b]), hi - lo
            else:
                lo, first, n = b * R, int(st["lengths"][b]) - 1, int(st["dn"][b])
                if first < 0:
                    continue
            pos = torch.arange(min(first + n, int(st["held"][b]) * page), device=DEV)
            slot = st["table"][b, pos // page].long() * page + pos % page
            new = pos >= first
            if st["mask"] is None:
                seen = pos[None, :] <= first + torch.arange(n, device=DEV)[:, None]
            else:
                seen = torch.ones(n, pos.numel(), dtype=torch.bool, device=DEV)
                j = pos[new] - first
                seen[:, new] = (st["mask"][b, :n][:, j // 32].long() >> (j % 32)) % 2 == 1
            for h in range(Hkv):
                key, val = st["k_cache"][slot, h].double(), st["v_cache"][slot, h].double()
                if st["k_scale"] is not None:
                    key, val = key * st["k_scale"][h].double(), val * st["v_scale"][h].double()
                for x in range(h * G, h * G + G):
                    s = st["q"][lo:lo + n, x].double() @ key.T.contiguous() / D ** 0.5
                    s = s.masked_fill(~seen, -math.inf)
                    low = s.logsumexp(1, keepdim=True)
                    lse[lo:lo + n, x] = low[:, 0]
                    low = low.masked_fill(low == -math.inf, 0.0)
                    out[lo:lo + n, x] = (s - low).exp() @ val
        return {"out": out, "lse": lse}

    def rows_of(b):
        """The logits rows of sequence b's entries."""
        if not case["path"]:
            return list(range(int(st["dn"][b])))
        node, up = int(st["accept_node"][b]), []
        while node >= 0:
            up.append(node)
            node = int(st["dpar"][b, node])
        return up[::-1]

    if kind == "store":
        res = {}
        n = int(st["cu"][-1]) if case["packed"] else st["rows"]
        slots = st["slots"][:n]
        for name in ("k", "v"):
            res[name + "_cache"] = st[name + "_cache"].double()
            res[name + "_cache"][slots[slots >= 0]] = st[name][:n][slots >= 0].double()
        return res
    if kind == "attend":
        # about a millisecond for each query head of a sequence
        return attend() if case["B"] * case["Hq"] <= 16384 else None
    T = case["T"]
    if kind == "score":
        res = {n: st[n].double() if st[n] is not None else None
               for n in ("logprob", "lse", "entropy", "top_logprobs")}
        res = {n: t for n, t in res.items() if t is not None}
        res.update({n: None for n in ("rank", "top_ids") if st[n] is not None})
    else:
        res = {"g_logits": st["g_logits"].double()}
    for b in range(case["B"]):
        rows = rows_of(b)
        n = len(rows)
        z = st["logits"][b, rows].double() / T
        tok = st["tokens"][b, :n].long()
        if kind == "score":
            lse = z.logsumexp(1)
            lp = z - lse[:, None]
            res["lse"][b, :n] = lse
            res["logprob"][b, :n] = lp[torch.arange(n), tok]
            if case["entropy"]:
                res["entropy"][b, :n] = -(lp.exp() * lp.clamp(min=-1e30)).sum(1)
            if case["n_top"]:
                res["top_logprobs"][b, :n] = lp.sort(1, descending=True).values[:, :case["n_top"]]
            continue
        # d(sum of g log p_t + h H) with the forward pass's own lse and entropy
        lp = z - st["lse"][b, :n].double()[:, None]
        p = lp.exp()
        d = p * -st["g_logprob"][b, :n].double()[:, None]
        if case["entropy"]:
            d -= p * (lp.clamp(min=-1e30) + st["entropy"][b, :n].double()[:, None]) \
                * st["g_entropy"][b, :n].double()[:, None]
        d[torch.arange(n), tok] += st["g_logprob"][b, :n].double()
        res["g_logits"][b, :n] = d / T
    return res
