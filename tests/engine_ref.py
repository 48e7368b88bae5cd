"""Plain CPU formulations of the calls around the step, written from their
definitions: loops over sequences, rows and nodes (numpy)."""
import numpy as np
import torch

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
NAN = float("nan")


def path_of(par, node):
    """Nodes from `node` up to the anchor's child (ends at an invalid parent)."""
    up = []
    while node > 0:
        up.append(node)
        q = int(par[node])
        if not 0 <= q < node:
            return up, False
        node = q
    return up, True


def parents(d, b):
    R = d["dtok"].shape[1]
    return np.arange(-1, R - 1) if d["dpar"] is None else d["dpar"][b]


def nodes(d, b):
    return int(np.clip(d["dn"][b], 1, d["dtok"].shape[1]))


def processed(d, real):
    """Rows (b, r) -> (values in `real`, a bound on the float error before the
    last rounding, which values are touched), from the formulas: every
    operation rounded to `real`."""
    B, R, V = d["logits"].shape
    words = (V + 31) // 32
    rows = {}
    for b in range(B):
        par = parents(d, b)
        made, given = np.zeros(V, np.int64), np.zeros(V, np.int64)
        penal = any(d[k] is not None for k in ("repetition", "frequency", "presence"))
        if penal:
            L = int(np.clip(d["lengths"][b], 0, d["tokens"].shape[1]))
            P = 0 if d["prompt_lens"] is None else int(np.clip(d["prompt_lens"][b], 0, L))
            for counts, x in ((given, d["tokens"][b, :P]), (made, d["tokens"][b, P:L])):
                counts += np.bincount(x[(x >= 0) & (x < V)], minlength=V)
        rho = real(1 if d["repetition"] is None else d["repetition"][b])
        freq = real(0 if d["frequency"] is None else d["frequency"][b])
        pres = real(0 if d["presence"] is None else d["presence"][b])
        bias, biased = np.zeros(V, real), np.zeros(V, bool)
        if d["bias_ids"] is not None:
            for v, val in zip(d["bias_ids"][b], d["bias_vals"][b]):
                if 0 <= v < V:
                    bias[v], biased[v] = real(val), True
        for r in range(nodes(d, b)):
            c = made.copy()
            if penal:
                for q in path_of(par, r)[0]:
                    v = int(d["dtok"][b, q])
                    if 0 <= v < V:
                        c[v] += 1
            y = d["logits"][b, r].to(torch.float64).numpy().astype(real)
            with np.errstate(all="ignore"):
                seen = (c > 0) | (given > 0)
                y = np.where(seen, np.where(y > 0, y / rho, y * rho), y)
                size = np.where(seen, np.abs(y), 0)
                fc = freq * c.astype(real)
                size = np.where(c > 0, size + np.abs(fc) + np.abs(y - fc), size)
                y = np.where(c > 0, y - fc, y)
                size = np.where(c > 0, size + np.abs(y - pres), size)
                y = np.where(c > 0, y - pres, y)
                size = np.where(biased, size + np.abs(y + bias), size)
                y = np.where(biased, y + bias, y)
            touched = seen | biased
            if d["allowed"] is not None and (d["allowed_on"] is None or d["allowed_on"][b] != 0):
                w = d["allowed"][b, r].view(np.uint8)
                ok = np.unpackbits(w, bitorder="little")[:V].astype(bool)
                assert d["allowed"].shape[2] == words
                y = np.where(ok, y, real(-np.inf))
                size = np.where(ok, size, 0)
                touched |= ~ok
            assert y.dtype == real
            rows[b, r] = y, size, touched
    return rows


def rounded(y, dtype):
    """float32 values in `dtype` (a torch CPU tensor)."""
    return torch.from_numpy(np.ascontiguousarray(y, np.float32)).to(dtype)


def greedy(d, rows):
    """The greedy accept over rows of float32 values rounded to bf16: loops
    over nodes in order."""
    B, R = d["dtok"].shape
    V = d["logits"].shape[2]
    res = {k: np.zeros(B, np.int32) for k in ("accept_len", "accept_node", "bonus")}
    res["amax"] = np.full((B, R), -1, np.int32)
    res["out_tokens"] = np.full((B, R), -1, np.int32)
    for b in range(B):
        n, par = nodes(d, b), parents(d, b)
        for r in range(n):
            y = rounded(rows[b, r][0], torch.bfloat16).float().numpy()
            best = 0
            if not np.isnan(y).all():
                best = int(np.flatnonzero(y == np.nanmax(y))[0])
            res["amax"][b, r] = best
        depth = {0: 0}
        for i in range(1, n):
            q = int(par[i])
            if 0 <= q < i and q in depth and int(d["dtok"][b, i]) == res["amax"][b, q]:
                depth[i] = depth[q] + 1
        deepest = max(depth.values())
        node = min(i for i, v in depth.items() if v == deepest)
        path = [int(d["dtok"][b, q]) for q in reversed(path_of(par, node)[0])] if node else []
        bonus = res["amax"][b, node]
        res["accept_len"][b], res["accept_node"][b], res["bonus"][b] = deepest, node, bonus
        res["out_tokens"][b, :deepest + 1] = path + [bonus]
    assert V > 0
    return res


def page_plan(s):
    """One call of the page plan on the numpy state `s` (changed in place)."""
    B, R = s["B"], s["R"]
    most, P, page = s["table"].shape[1], len(s["ring"]), s["page"]
    head = int(np.clip(s["ring_state"][0], 0, P - 1))
    count = int(np.clip(s["ring_state"][1], 0, P))
    slots = np.full((B, R), -1, np.int64)
    positions = np.full((B, R), -1, np.int32)
    missing = np.zeros(B, np.int32)
    free = [int(s["ring"][(head + i) % P]) for i in range(count)]
    back, asked, popped = [], 0, 0
    for b in range(B):
        L = int(np.clip(s["lengths"][b], 0, s["Lmax"]))
        n = int(np.clip(s["dn"][b], 1, R))
        held = int(np.clip(s["held"][b], 0, most))
        if L == 0:
            back += [int(x) for x in s["table"][b, :held]]
            s["table"][b, :held] = -1
            if held:
                s["held"][b] = 0
            continue
        lack = max(0, min(most, -(-(L - 1 + n) // page)) - held)
        asked += lack
        if lack and asked <= count:
            s["table"][b, held:held + lack] = free[popped:popped + lack]
            popped += lack
            held += lack
            s["held"][b] = held
        elif lack:
            missing[b] = lack
        par = np.arange(-1, R - 1) if s["dpar"] is None else s["dpar"][b]
        for r in range(n):
            p = L - 1 + r
            if p // page < held:
                slots[b, r] = int(s["table"][b, p // page]) * page + p % page
            up, whole = path_of(par, r)
            positions[b, r] = L - 1 + len(up) - (0 if whole else 1)
    back = back[:P - count]
    for i, x in enumerate(back):
        s["ring"][(head + count + i) % P] = x
    s["ring_state"][0] = (head + popped) % P
    s["ring_state"][1] = count - popped + len(back)
    return slots, positions, missing


def spans(begin, end, tokens, table, held, page, cap):
    B, Lmax = tokens.shape
    cu, rec = [0], []
    for b in range(B):
        hi = int(np.clip(end[b], 0, Lmax))
        lo = int(np.clip(begin[b], 0, hi))
        h = int(np.clip(held[b], 0, table.shape[1]))
        for i in range(lo, hi):
            slot = int(table[b, i // page]) * page + i % page if i // page < h else -1
            rec.append((slot, i, int(tokens[b, i]), b))
        cu.append(len(rec))
    return np.array(cu, np.int32), rec[:cap]


def compact(cache, slots, dpar, dn, accept_node):
    """cache [planes, n_slots, row] (numpy), moved in place."""
    B, R = slots.shape
    before = cache.copy()
    for b in range(B):
        n, a = int(np.clip(dn[b], 1, R)), int(accept_node[b])
        if not 0 <= a < n:
            continue
        up, whole = path_of(dpar[b], a)
        if not whole:
            continue
        for j, q in enumerate(reversed(up), 1):
            fro, to = int(slots[b, q]), int(slots[b, j])
            if 0 <= fro < cache.shape[1] and 0 <= to < cache.shape[1]:
                cache[:, to] = before[:, fro]
