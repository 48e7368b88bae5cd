"""Keys far below the largest one: what they add together."""
import math

import numpy as np
import pytest
import torch

import attention_ref as ref
from gpu_helpers import say
from test_attention_gpu import make, run

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2609_20186_amd import binding  # noqa: F401


@pytest.mark.parametrize("type", ["f16", "bf16"])
@pytest.mark.parametrize("cache", ["half", "e4m3"])
@pytest.mark.parametrize("R,Hq,L", [(1, 1, 900), (1, 1, 6000), (40, 2, 900), (40, 2, 6000)])
@pytest.mark.parametrize("gap", [10, 16, 18])
def test_many_keys_far_below_the_largest(type, cache, R, Hq, L, gap):
    """One key's product is 0 and its value 0, all others' `gap` below and 1 (448 with the
    products of a whole 8-bit cache): the result is what the others weigh together, L e^-gap.
    A weight's rounding is half a step, U of it, or where it lies below fp16's normal numbers
    half a step of 2^-24 with the largest weight at least 2^7: 2^-32 of the largest, for each
    key.  The result's own is U of it, or half a step of 2^-24 below fp16's normal numbers."""
    a = make([L], [R], R=R, Hq=Hq, Hkv=1, D=64, page=16, type=type, scale=1.0, seed=gap,
             cache="e4m3" if cache == "e4m3" else type)
    for name in ("k_scale", "v_scale"):
        a[name] = None if a[name] is None else torch.ones(1)
    q, k, v = (torch.zeros_like(a[n].float()) for n in ("q", "k_cache", "v_cache"))
    slots = ref.slots_of(a, 0, L - 1 + R)
    big = 1.0 if cache == "half" else 448.0
    q[:, :, 0] = 1.0
    k[:, :, 0] = -float(gap)
    v[:] = big
    k[slots[L // 3]] = 0.0
    v[slots[L // 3]] = 0.0
    a["q"] = q.to(a["q"].dtype)
    a["k_cache"], a["v_cache"] = k.to(a["k_cache"].dtype), v.to(a["v_cache"].dtype)
    out, lse, _, _ = run(a)
    out, lse = ref.f64(out), ref.f64(lse)
    u = ref.U[type]
    worst = 0.0
    for i in range(R):
        n = L - 1 + i                         # keys that are not the largest
        w = math.exp(-gap)
        total = 1 + n * w
        want = n * w / total * big
        tol = want * (2 * u + (n + 64) * 2.0 ** -23)
        if type == "f16":
            tol += n * 2.0 ** -32 * big + 2.0 ** -25
        worst = max(worst, np.abs(out[i] - want).max() / tol)
        assert (np.abs(out[i] - want) <= tol).all(), (i, out[i, 0, 0], want, tol)
        assert np.abs(lse[i] - math.log(total)).max() <= (n + 64) * 2.0 ** -23
    say(f"{R} rows over {L}, gap {gap}: {worst:.2f} of the bound")
