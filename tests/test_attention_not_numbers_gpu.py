"""NaN that a row of the attention sees, in queries, keys and scales: it reaches the
result and the log of the sum in both forms, whole and cut over work-groups, and no
other row."""
import math

import numpy as np
import pytest
import torch

import attention_ref as ref
from gpu_helpers import say
from test_attention_gpu import DEV, make, run

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2609_20186_amd import binding  # noqa: F401


def check(a, what):
    """As the references, NaN in lse where they have it; how many heads of rows are NaN."""
    out, lse, _, _ = run(a)
    sc = {n: None if a[n] is None else a[n].numpy() for n in ("k_scale", "v_scale")}
    want = ref.attention(a, ref.f64(a["q"]), ref.f64(a["k_cache"]), ref.f64(a["v_cache"]), **sc)
    out, lse = ref.f64(out), ref.f64(lse)
    heads = 0
    for row in range(a["rows"]):
        if row not in want:
            assert (out[row] == 77).all() and (lse[row] == 77).all(), (what, row)
            continue
        o, low, tol, ltol = want[row]
        np.testing.assert_array_equal(np.isnan(out[row]), np.isnan(o), err_msg=f"{what} row {row}")
        np.testing.assert_array_equal(np.isnan(lse[row]), np.isnan(low), err_msg=f"{what} lse {row}")
        bad = np.isnan(low)
        heads += int(bad.sum())
        for h in np.flatnonzero(~bad):
            assert (np.abs(out[row, h] - o[h]) <= tol[h]).all(), (what, row, h)
            assert lse[row, h] == low[h] or abs(lse[row, h] - low[h]) <= ltol[h], (what, row, h)
    say(f"{what}: {heads} heads of rows are NaN")
    return heads


# rows, query heads (2 heads of the cache), contexts: the form for up to 32 rows and the one
# for more, whole and cut
FORMS = [(1, 4, 40), (6, 4, 300), (6, 4, 3000), (1, 2, 5000), (50, 8, 70), (50, 8, 3000)]


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("R,Hq,L", FORMS)
def test_query_rows(R, Hq, L, D):
    for type in ("bf16", "f16"):
        a = make([L, L - 3], [R, max(1, R - 1)], Hq=Hq, Hkv=2, D=D, page=16, type=type, seed=R)
        a["q"][0, 1, 5] = math.nan
        a["q"][R, 0, D - 1] = math.nan
        assert check(a, f"{R} rows over {L}, {type}") == 2


@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
@pytest.mark.parametrize("R,Hq", [(1, 4), (5, 4), (40, 8)])
def test_the_only_keys(R, Hq, cache):
    """A context whose first key is NaN: the only one that its first row sees, and one that
    all rows see."""
    a = make([1, 1], [R, 1], Hq=Hq, Hkv=2, D=64, page=16, cache=cache)
    at = ref.slots_of(a, 0, 1)[0]
    x = a["k_cache"].float()
    x[at, 1] = math.nan
    a["k_cache"] = x.to(a["k_cache"].dtype)
    assert check(a, f"{R} rows, {cache}") == R * Hq // 2


@pytest.mark.parametrize("R,Hq", [(1, 4), (5, 4), (40, 8)])
@pytest.mark.parametrize("at", [32, 64, 96, 128])
def test_a_key_alone_in_its_block(R, Hq, at):
    """The first drafted row's own key is NaN and the first of a block of 32."""
    a = make([at + 1, at], [R, R], Hq=Hq, Hkv=2, D=64, page=16)
    a["k_cache"][ref.slots_of(a, 0, at + 1)[at], 0, 3] = math.nan
    assert check(a, f"{R} rows, key {at}") == R * Hq // 2


@pytest.mark.parametrize("R,Hq", [(1, 4), (5, 4), (40, 8)])
@pytest.mark.parametrize("page", [0, 2, 8, 100, 180])
def test_a_key_alone_in_its_share(R, Hq, page):
    """Long contexts of which one page is held, its keys all but one behind the cache and
    that one NaN: one work-group of those that share the keys sees it, the others nothing, and
    the rows' own keys are missing as well."""
    a = make([3000, 2900], [R, R], Hq=Hq, Hkv=2, D=64, page=16)
    # the cache's first slot, behind which the page's other 15 are cut off
    own = a["table"][0, page]
    a["table"][0] = -1
    a["table"][0, page] = 0
    a["table"][1][a["table"][1] == 0] = own
    for name in ("q", "k_cache", "v_cache"):
        a[name] = torch.nan_to_num(a[name], nan=0.25)
    a["k_cache"][0, 1, 9] = math.nan
    a["held"][1] = 0
    a["k_cache"], a["v_cache"], a["n_slots"] = a["k_cache"][:1], a["v_cache"][:1], 1
    assert check(a, f"{R} rows, page {page}") == R * Hq // 2
    a["held"][0] = page                       # not even that one
    assert check(a, f"{R} rows, no page") == 0


@pytest.mark.parametrize("R,Hq,L", FORMS)
def test_scales_of_keys(R, Hq, L):
    """A head of the cache whose scale is NaN: NaN for all its rows but those that see
    nothing, which are 0 with -inf."""
    for mask in (None, "none"):
        a = make([L, 1], [R, R], Hq=Hq, Hkv=2, D=64, page=16, cache="e4m3", mask=mask, seed=3)
        a["k_scale"][1] = math.nan
        want = R * Hq // 2 * (2 if mask is None else 1)
        assert check(a, f"{R} rows over {L}, mask {mask}") == want


@pytest.mark.parametrize("R,Hq,L", FORMS)
def test_rows_that_see_nothing_under_broken_scales(R, Hq, L):
    """They are 0 with -inf whatever their head's scales are."""
    a = make([L, 1], [R, R], Hq=Hq, Hkv=2, D=64, page=16, cache="e4m3", mask="none", seed=3)
    for bad in (math.nan, math.inf, -math.inf):
        a["k_scale"][1] = bad
        a["v_scale"][1] = bad
        out, lse, _, _ = run(a)
        out, lse = ref.f64(out), ref.f64(lse)
        assert (out[R:] == 0).all() and (lse[R:] == -math.inf).all(), bad
        assert np.isfinite(out[:R, :Hq // 2]).all() and np.isfinite(lse[:R, :Hq // 2]).all()


@pytest.mark.parametrize("R,Hq,L", FORMS)
def test_scales_of_values(R, Hq, L):
    """NaN there is the result's alone."""
    a = make([L, 1], [R, R], Hq=Hq, Hkv=2, D=64, page=16, cache="e4m3", mask="none", seed=3)
    a["v_scale"][0] = math.nan
    out, lse, _, _ = run(a)
    out, lse = ref.f64(out), ref.f64(lse)
    assert np.isnan(out[:R, :Hq // 2]).all() and np.isfinite(out[:R, Hq // 2:]).all()
    assert np.isfinite(lse[:R]).all()
    assert (out[R:] == 0).all() and (lse[R:] == -math.inf).all()


@pytest.mark.parametrize("R,Hq,L", FORMS)
@pytest.mark.parametrize("scale", [0.2, -0.2])
def test_infinite_products(R, Hq, L, scale):
    """+inf is NaN for the rows that see it; -inf weighs nothing, and a row that sees nothing
    else is as one that sees nothing."""
    inf = math.inf if scale > 0 else -math.inf
    for L0 in (L, 1):
        a = make([L0, L], [R, 1], R=R, Hq=Hq, Hkv=2, D=64, page=16, scale=scale, seed=5)
        a["q"][:, :, 5] = 1.0
        slots = ref.slots_of(a, 0, L0 - 1 + R)
        at = slots[L0 // 2]
        a["k_cache"][at, 0, 5] = inf
        out, lse, _, _ = run(a)
        out, lse = ref.f64(out[:R]), ref.f64(lse[:R])
        assert np.isnan(out[:, :Hq // 2]).all() and np.isnan(lse[:, :Hq // 2]).all()
        assert np.isfinite(out[:, Hq // 2:]).all() and np.isfinite(lse[:, Hq // 2:]).all()
        a["k_cache"][at, 0, 5] = -inf
        out, lse, _, _ = run(a)
        if L0 == 1:
            assert (out[0, :Hq // 2] == 0).all() and (lse[0, :Hq // 2] == -math.inf).all()
        a["table"][0, L0 // 2 // 16] = -1      # the page of the key with it
        a["k_cache"][slots[L0 // 2 // 16 * 16:][:16], 0, 5] = -inf
        few = run(a)
        a["table"][0, L0 // 2 // 16] = at // 16
        full = run(a)
        assert torch.equal(full[0][:R, :Hq // 2].isfinite(), few[0][:R, :Hq // 2].isfinite())
        d = (full[1][:R, :Hq // 2] - few[1][:R, :Hq // 2]).abs()
        same = full[1][:R, :Hq // 2] == few[1][:R, :Hq // 2]      # -inf both
        assert (same | (d <= (L + 64) * 2.0 ** -23)).all()   # the order of the sums
