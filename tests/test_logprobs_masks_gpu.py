"""Logits masked with large finite values, the types' lowest among them: log
probabilities, entropies and gradients are those of what is left."""
import math

import numpy as np
import pytest
import torch

import attention_ref as ref
from gpu_helpers import say
from test_logprobs_gpu import DEV, TYPES, args_of, make, run

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2609_20186_amd import binding  # noqa: F401


LOWEST = {t: torch.finfo(TYPES[t]).min for t in TYPES}


def masked(V, type, where, rng):
    """Which of the tokens are masked; a lane takes one vector of 16 bytes in 256, a wave
    64 of them."""
    vec = np.arange(V) // (4 if type == "f32" else 8)
    if where == "first":                      # whole vectors in front
        return np.arange(V) < V * 3 // 4
    if where == "last":
        return np.arange(V) >= V // 3
    if where == "lanes":
        return vec % 256 % 3 == 0
    if where == "waves":
        return vec % 256 // 64 % 2 == 0
    if where == "vectors":
        return rng.random(vec[-1] + 1)[vec] < 0.6
    if where == "but one":
        return np.arange(V) != V // 2 + 1
    return rng.random(V) < 0.5                # anywhere


WHERE = ["first", "last", "lanes", "waves", "vectors", "but one", "anywhere"]


def tolerance(V, T, big, value):
    """As for logits without a mask (two roundings of |z - max|, of exp2 and its argument a
    few, the sum's); what is masked weighs exactly nothing."""
    return 2.0 ** -24 * (math.sqrt(V) + 16 + 8 * big * max(1.0, abs(value)) / T + 4 * abs(value))


def order(row):
    """Tokens by falling logit, ties by index (no NaN here)."""
    return np.argsort(-row, kind="stable")


def reference(row, T):
    """lse, log probabilities and entropy of a row of finite logits in 64 bits, against the
    maximum, beside which the logarithm of the sum can be too small for 64 bits."""
    z = (row - row.max()) / T
    total = math.log(np.exp(z).sum())
    p = np.exp(z - total)
    return row.max() / T + total, z - total, -(p[p > 0] * (z - total)[p > 0]).sum()


def references(x, T):
    return [[reference(row, T) for row in rows] for rows in x]


def check(a, T, x, first, want, out, what):
    B, R, V = x.shape
    o = {n: t.cpu().numpy() for n, t in out.items()}
    for b in range(B):
        for i in range(R):
            row, (lse, lp, h) = x[b, i], want[b][i]
            big = np.abs(row[row > -1e4]).max() if (row > -1e4).any() else 1.0
            tok = int(a["tokens"][b, i])
            at = f"{what} {b} {i}"
            assert abs(o["entropy"][b, i] - h) <= tolerance(V, T, big, h), (at, o["entropy"][b, i], h)
            near = np.float32(np.clip(lse, LOWEST["f32"], -LOWEST["f32"]))
            assert o["lse"][b, i] == near or \
                abs(o["lse"][b, i] - lse) <= tolerance(V, T, big, lse), (at, o["lse"][b, i], lse)
            if 0 <= tok < V:
                far = lp[tok] < -1e4          # a masked token
                with np.errstate(over="ignore"):
                    near = np.float32(lp[tok])
                tol = 2.0 ** -22 * abs(lp[tok]) if far else tolerance(V, T, big, lp[tok])
                assert o["logprob"][b, i] == near or abs(o["logprob"][b, i] - lp[tok]) <= tol, at
                assert first[b][i][o["rank"][b, i]] == tok, at
            np.testing.assert_array_equal(o["top_ids"][b, i], first[b][i][:o["top_ids"].shape[2]],
                                          err_msg=at)


@pytest.mark.parametrize("type,low", [("bf16", LOWEST["bf16"]), ("bf16", -1e37), ("bf16", -1e30),
                                      ("f16", LOWEST["f16"]), ("f32", LOWEST["f32"]),
                                      ("f32", -1e38), ("f32", -1e36), ("f32", -1e9)])
@pytest.mark.parametrize("where", WHERE)
def test_masks(type, low, where):
    from paper_2609_20186_amd import binding as sd
    rng = np.random.default_rng(1)
    for V in (300, 5003, 50257):
        a = make(2, 2, V, type, seed=V, dn=False)
        hide = torch.from_numpy(masked(V, type, where, rng))
        a["logits"][..., hide] = torch.tensor(low).to(TYPES[type])
        x = ref.f64(a["logits"])
        first = [[order(row) for row in rows] for rows in x]
        logits = a["logits"].to(DEV)
        for T in (0.7, 1.0, 1.6):
            refs = references(x, T)
            for cut in (True, False):
                args = args_of(a, T, logits)
                if not cut:
                    args.workspace, args.workspace_bytes = None, 0
                out, _ = run(a, T, 5, args=args)
                what = f"{type} {low:.2g} {where} V={V} T={T} cut={cut}"
                check(a, T, x, first, refs, out, what)
            # the gradient takes this lse and entropy
            g = torch.tensor([[0.7, -1.0], [0.0, 0.3]])
            ge = torch.tensor([[0.2, 0.5], [1.0, 0.0]])
            grad = torch.full_like(logits, 5.0)
            sd.switchsd_token_logprobs_grad(args, out["lse"], out["entropy"], g.to(DEV),
                                            ge.to(DEV), grad)
            got = ref.f64(grad)
            for b in range(2):
                for i in range(2):
                    if (x[b, i] < -1e4).all():
                        continue              # p is not exp(z - lse) in 32 bits (below)
                    lse, h = float(out["lse"][b, i]), float(out["entropy"][b, i])
                    want = ref.grad_row(x[b, i], T, int(a["tokens"][b, i]), lse, h,
                                        float(g[b, i]), float(ge[b, i]))
                    z = np.clip(x[b, i] / T - lse, -1e3, None)
                    p = np.exp(z)
                    err = 2.0 ** -24 * (16 * (np.abs(z) + abs(lse)) + 16)
                    part = p * (abs(g[b, i].item()) + abs(ge[b, i].item()) * (np.abs(z) + abs(h) + 1))
                    tol = 1.01 * ref.U[type] * np.abs(want) + \
                        (part * err + 2.0 ** -22 * (part + abs(g[b, i].item()))) / T
                    tol += {"bf16": 1e-38, "f16": 2.0 ** -25, "f32": 1e-38}[type]
                    assert (np.abs(got[b, i] - want) <= tol).all(), (what, b, i)
        say(f"{type} {low:.2g} {where} V={V}")


@pytest.mark.parametrize("type", ["bf16", "f32"])
@pytest.mark.parametrize("low", [-1.0, 1.0])
def test_logits_far_apart(type, low):
    """Steps of many sizes between the smallest and the largest numbers, falling and
    rising: the largest one takes it all, whatever lay before it."""
    for V in (300, 5003, 50257):
        a = make(1, 2, V, type, seed=V, dn=False)
        x = torch.logspace(-3, 38, V)
        a["logits"][0, 0] = (x * low).to(TYPES[type])
        a["logits"][0, 1] = (x.flip(0) * low).to(TYPES[type])
        a["tokens"][:] = 3
        rows = ref.f64(a["logits"])
        for cut in (True, False):
            args = args_of(a, 1.0, a["logits"].to(DEV))
            if not cut:
                args.workspace, args.workspace_bytes = None, 0
            out, _ = run(a, 1.0, 5, args=args)
            for i in range(2):
                lse, lp, h = reference(rows[0, i], 1.0)
                # |z - max| of the logits that weigh something is below 100
                near = rows[0, i][rows[0, i] >= rows[0, i].max() - 100]
                big = np.abs(near - near.max()).max()
                got = {n: float(out[n][0, i]) for n in ("lse", "entropy", "logprob")}
                assert abs(got["entropy"] - h) <= tolerance(V, 1.0, big, h), (V, i, got, h)
                assert abs(got["lse"] - lse) <= tolerance(V, 1.0, big, lse), (V, i, got, lse)
                np.testing.assert_array_equal(out["top_ids"][0, i].cpu(), order(rows[0, i])[:5])


def gradient(a, T, logits, g, ge):
    """The forward pass's entropy and the gradient."""
    from paper_2609_20186_amd import binding as sd
    out, args = run(a, T, 0, args=args_of(a, T, logits))
    grad = torch.full_like(logits, 5.0)
    call = (out["lse"], out["entropy"], g.to(DEV), ge.to(DEV))
    sd.switchsd_token_logprobs_grad(args, *call, grad)
    sd.switchsd_token_logprobs_grad(args, *call, logits)   # in the logits' place
    bits = torch.int32 if logits.dtype == torch.float32 else torch.int16
    assert torch.equal(grad.view(bits), logits.view(bits))
    return out, ref.f64(grad)


def check_gradient(a, T, x, got, g, ge, what):
    """Against the formula with the row's own probabilities, whatever lse has of them in 32
    bits.  log p is off by 8 roundings of |z - max| and the sum's, sqrt V and 32 of them; the
    products by a few of their own."""
    B, R, V = x.shape
    u = ref.U[a["type"]]
    for b in range(B):
        for i in range(R):
            _, lp, h = reference(x[b, i], T)
            lp = np.clip(lp, -1e3, None)
            p = np.exp(lp)
            gl, gh = float(g[b, i]), float(ge[b, i])
            hit = np.arange(V) == int(a["tokens"][b, i])
            want = (gl * (hit - p) - gh * p * (lp + h)) / T
            err = 2.0 ** -24 * (8 * np.abs(lp) + math.sqrt(V) + 32)
            part = p * (abs(gl) + abs(gh) * (np.abs(lp) + abs(h)))
            tol = 1.01 * u * np.abs(want) + (part * err + p * abs(gh) * (err + 2.0 ** -23 * math.sqrt(V))
                                             + 2.0 ** -22 * (part + abs(gl) * hit)) / T
            tol += {"bf16": 1e-38, "f16": 2.0 ** -25, "f32": 1e-38}[a["type"]]
            d = np.abs(got[b, i] - want)
            assert (d <= tol).all(), (what, b, i, float(d.max()), float(want[d.argmax()]))


@pytest.mark.parametrize("type,low", [("bf16", LOWEST["bf16"]), ("bf16", -1e30), ("bf16", 1e37),
                                      ("f16", LOWEST["f16"]), ("f32", LOWEST["f32"]),
                                      ("f32", -1e9), ("f32", 3e38)])
def test_gradient_of_rows_of_one_value(type, low):
    """All masked, with a value beside which the logarithm of the sum has no place in 32
    bits: every token is as likely, and with T below 1 z itself is beyond the largest number."""
    g, ge = torch.tensor([[0.7, -1.0, 0.0]]), torch.tensor([[0.2, 0.5, 1.0]])
    for V in (1, 9, 300, 5003, 50257):
        a = make(1, 3, V, type, seed=V, dn=False)
        a["logits"][:] = torch.tensor(low).to(TYPES[type])
        if V > 4:                             # a likelier one beside the others
            a["logits"][0, 1, V // 2] = torch.tensor(low * 0.5 if low < 0 else low * 1.1).to(
                TYPES[type])
        x = ref.f64(a["logits"])
        for T in (0.7, 1.0, 1.6):
            out, got = gradient(a, T, a["logits"].to(DEV), g, ge)
            assert torch.isfinite(out["lse"]).all()
            check_gradient(a, T, x, got, g, ge, f"{type} {low:.2g} V={V} T={T}")


@pytest.mark.parametrize("type", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("T", [2.0 ** -6, 1e-3, 1e-5])
def test_gradient_at_low_temperatures(type, T):
    """Rows of which a few tokens are nearly as likely, with |z| of 10^3 to 10^6."""
    g, ge = torch.tensor([[0.7, -1.0, 0.4]]) * T, torch.tensor([[0.2, 0.5, 0.0]]) * T
    for V in (9, 5003, 50257):
        a = make(1, 3, V, type, seed=V, dn=False)
        at = V // 3
        step = 2.0 ** -3 if type != "f32" else T    # apart by what the type has at 20
        for i in range(3):
            a["logits"][0, i, at:at + 3] = (20.0 + i + step * torch.arange(3)).to(TYPES[type])
        x = ref.f64(a["logits"])
        _, got = gradient(a, T, a["logits"].to(DEV), g, ge)
        check_gradient(a, T, x, got, g, ge, f"{type} V={V} T={T}")
