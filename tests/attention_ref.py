"""Plain references in 64 bits of the cache store, the attention over a paged
cache and the log probabilities, written from their definitions with loops, and
the bounds that the kernels' roundings leave them."""
import math

import numpy as np
import torch

HALF = {"bf16": torch.bfloat16, "f16": torch.float16}
U = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11, "f32": 2.0 ** -24}  # half a step, relative


def f64(t):
    return t.detach().cpu().to(torch.float64).numpy()


# ------------------------------------------------------------------ 8-bit floats

def e4m3_values():
    """The 127 finite magnitudes, by code: 4 exponent bits of bias 7, 3 of fraction,
    code 127 being NaN."""
    out = []
    for code in range(127):
        e, f = code >> 3, code & 7
        out.append((1 + f / 8) * 2.0 ** (e - 7) if e else f / 8 * 2.0 ** -6)
    return np.array(out)


def to_e4m3(x):
    """Codes of float32 values: nearest, ties to the even code, saturating."""
    vals = e4m3_values()
    out = np.zeros(x.shape, np.uint8)
    for at, v in np.ndenumerate(x):
        s = 0x80 if np.signbit(v) else 0
        if np.isnan(v):
            out[at] = 0x7F | s
            continue
        a = min(abs(float(v)), 448.0)
        d = np.abs(vals - a)
        best = np.flatnonzero(d == d.min())
        out[at] = s | (best[0] if len(best) == 1 or best[0] % 2 == 0 else best[1])
    return out


# ------------------------------------------------------------------ attention

def rows_of(a, b):
    """(first row, rows, first position) of sequence b; a: dict of numpy arrays and
    sizes."""
    if a.get("cu") is not None:
        lo, hi = int(a["cu"][b]), int(a["cu"][b + 1])
        if lo < 0 or hi < lo or hi > a["rows"]:
            return 0, 0, 0
        return lo, min(hi - lo, a["R"]), min(max(int(a["begin"][b]), 0), a["Lmax"])
    L = min(max(int(a["lengths"][b]), 0), a["Lmax"])
    n = min(max(int(a["dn"][b]), 1), a["R"]) if L > 0 else 0
    return b * a["R"], n, L - 1


def slots_of(a, b, end):
    """Slot of each position, -1 where there is no key."""
    out = np.full(max(end, 0), -1, np.int64)
    held = min(max(int(a["held"][b]), 0), a["table"].shape[1])
    for pos in range(end):
        page = pos // a["page"]
        if page < held:
            s = int(a["table"][b, page]) * a["page"] + pos % a["page"]
            if 0 <= s < a["n_slots"]:
                out[pos] = s
    return out


def seen_of(a, b, row, i, n, pos, slots):
    seen = slots >= 0
    j = np.arange(len(slots)) - pos
    new = j >= 0
    if a.get("mask") is None:
        seen &= ~new | (j <= i)
    else:
        w = a["mask"].reshape(a["rows"], -1).view(np.uint32)[row]
        jj = j[new]
        seen[new] &= (w[jj // 32] >> (jj % 32).astype(np.uint32)) & 1 == 1
    return seen


def attention(a, q, k, v, k_scale=None, v_scale=None):
    """{row: (out [Hq, D], lse [Hq], bound of out, bound of lse)} of all rows, from q
    [rows, Hq, D], k, v [n_slots, Hkv, D] in float64."""
    Hq, Hkv, D = a["Hq"], a["Hkv"], a["D"]
    G, u = Hq // Hkv, U[a["type"]]
    res = {}
    for b in range(a["table"].shape[0]):
        first, n, pos = rows_of(a, b)
        slots = slots_of(a, b, pos + n)
        for i in range(n):
            row = first + i
            seen = seen_of(a, b, row, i, n, pos, slots)
            at = slots[seen]
            out, lse = np.zeros((Hq, D)), np.full(Hq, -math.inf)
            tol, ltol = np.zeros((Hq, D)), np.zeros(Hq)
            if len(at):
                for h in range(Hq):
                    ks = 1.0 if k_scale is None else float(k_scale[h // G])
                    vs = 1.0 if v_scale is None else float(v_scale[h // G])
                    with np.errstate(invalid="ignore", over="ignore"):
                        kk, vv = k[at, h // G], v[at, h // G] * vs
                        s = a["scale"] * ks * (kk @ q[row, h])
                        m = s.max()
                        p = np.exp(s - m) if np.isfinite(m) else s * np.nan
                        lse[h] = m + math.log(p.sum()) if np.isfinite(m) else m
                        p = p / p.sum()
                        out[h] = p @ vv
                        # the products of 16-bit numbers are exact in 32 bits, a
                        # sum of D of them is off by at most D roundings of the
                        # sum of their magnitudes (MFMA's own order and the two
                        # factors behind it: a few more); a weight is off by that,
                        # the rounding of its exponent (|s| of them) and of exp2
                        # (an error of a few units), and one rounding to q's type
                        big = abs(a["scale"] * ks) * (np.abs(kk) @ np.abs(q[row, h])).max()
                        es = (D + 8) * 2.0 ** -24 * big + 2.0 ** -21
                        N = len(at)
                        A = p @ np.abs(vv)
                        tol[h] = u * (np.abs(out[h]) + A) * 1.01 + A * (2 * es + N * 2.0 ** -23)
                        if a["type"] == "f16":
                            # weights (the largest at least 1) and results below the
                            # normal range: half a step of 2^-24
                            tol[h] += 2.0 ** -25 * (np.abs(vv).sum(0) + 1)
                        ltol[h] = 2 * es + (N + 16) * 2.0 ** -24 + 2.0 ** -22 * abs(lse[h])
            res[row] = (out, lse, tol, ltol)
    return res


# ------------------------------------------------------------------ log probabilities

def entries(a, b):
    """The logits rows of sequence b's entries."""
    R = a["R"]
    n = R if a.get("dn") is None else min(max(int(a["dn"][b]), 1), R)
    if a.get("accept_node") is None:
        return list(range(n))
    node = int(a["accept_node"][b])
    if not 0 <= node < n:
        return []
    if a.get("dpar") is None:
        return list(range(node + 1))
    up = [node]
    while up[-1] > 0:
        q = int(a["dpar"][b, up[-1]])
        if not 0 <= q < up[-1]:
            return []
        up.append(q)
    return up[::-1]


def order(x):
    """Tokens by falling logit, ties by index, NaN last."""
    key = np.where(np.isnan(x), -math.inf, x)
    return sorted(range(len(x)), key=lambda v: (bool(np.isnan(x[v])), -key[v], v))


def row_logprobs(x, T):
    """lse, the log probabilities of all tokens, entropy of one row of float64 logits."""
    num = x[~np.isnan(x)]
    m = num.max() if len(num) else -math.inf
    if not np.isfinite(m):
        lp = np.full(len(x), -math.inf)
        hit = np.flatnonzero(x == m) if len(num) else [0]
        lp[hit[0]] = 0.0
        return m, lp, 0.0
    z = np.where(np.isnan(x), -math.inf, x) / T
    top = m / T
    w = np.exp(z - top)
    lse = top + math.log(w.sum())
    lp = z - lse
    p = np.exp(lp)
    return lse, lp, float(-(p[p > 0] * lp[p > 0]).sum())


def grad_row(x, T, tok, lse, entropy, g, ge):
    """The gradient of one row, from the formula in 64 bits, with the given lse and
    entropy."""
    V = len(x)
    if not np.isfinite(lse):
        return np.zeros(V)
    z = np.where(np.isnan(x), -math.inf, x) / T - lse
    p = np.exp(z)
    d = -g * p
    on = p > 0
    d[on] -= ge * p[on] * (z[on] + entropy)
    if 0 <= tok < V:
        d[tok] += g
    return d / T
