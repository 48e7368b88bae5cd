"""NaN that a row of the attention sees, in queries, keys and scales: it reaches the
result and the log of the sum in both forms, whole and cut over work-groups, and no
other row."""
import math

import numpy as np
import pytest
import torch

import attention_ref as ref
from test_attention_gpu import DEV, make, run

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2609_20186_amd import binding  # noqa: F401


# rows, query heads (2 heads of the cache), contexts: the form for up to 32 rows and the one
# for more, whole and cut
FORMS = [(1, 4, 40), (6, 4, 300), (6, 4, 3000), (1, 2, 5000), (50, 8, 70), (50, 8, 3000)]


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
