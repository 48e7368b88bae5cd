"""The most sequences of an attention and the largest vocabulary."""
import math

import numpy as np
import pytest
import torch

from test_attention_gpu import check, run
from test_attention_instances_gpu import shared

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2609_20186_amd import binding  # noqa: F401


def test_most_sequences():
    """65536 of them, many finished: 256 for each lane that sums up the work."""
    B = 65536
    rng = np.random.default_rng(1)
    a = shared(np.maximum(rng.integers(-20, 12, B), 0), np.ones(B), 2, 1, 64, 1, long=31)
    check(a, *run(a)[:2], f"{B} sequences")


@pytest.mark.parametrize("type", [torch.bfloat16, torch.float32])
def test_largest_vocabulary(type):
    """2^26 logits: a row that is cut, two that are not, and their gradient."""
    from paper_2609_20186_amd import binding as sd
    V, u = 2 ** 26, 2.0 ** -8 if type == torch.bfloat16 else 2.0 ** -24
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn((1, 2, V), generator=g, device="cuda").to(type)
    x[0, 0, V - 1], x[0, 1, 12345] = 9.0, 8.5
    tokens = torch.tensor([[V - 1, V - 2]], dtype=torch.int32, device="cuda")
    z = x.double()
    lse = z.logsumexp(2)
    lp = z - lse[:, :, None]
    entropy = -(lp.exp() * lp).sum(2)
    own = x.gather(2, tokens.long()[:, :, None])
    at = torch.arange(V, device="cuda")
    rank = ((x > own) | ((x == own) & (at < tokens[:, :, None]))).sum(2)
    tol = 2.0 ** -24 * (math.sqrt(V) + 16 + 8 * 9 * 20 + 4 * 20)
    for cut in (True, False):
        args = sd.build_logprob_args(x, tokens)
        assert args.workspace
        if not cut:
            args.workspace, args.workspace_bytes = None, 0
        out = {n: torch.zeros((1, 2), device="cuda") for n in ("logprob", "lse", "entropy")}
        out["rank"] = torch.zeros((1, 2), dtype=torch.int32, device="cuda")
        out["top_ids"] = torch.zeros((1, 2, 1), dtype=torch.int32, device="cuda")
        sd.switchsd_token_logprobs(args, **out)
        for n, want in (("lse", lse), ("entropy", entropy),
                        ("logprob", lp.gather(2, tokens.long()[:, :, None])[:, :, 0])):
            assert (out[n].double() - want).abs().max() <= tol, (cut, n)
        assert torch.equal(out["rank"].long(), rank)
        assert out["top_ids"].flatten().tolist() == [V - 1, 12345]
    gl, ge = torch.tensor([[0.7, -1.0]], device="cuda"), torch.tensor([[0.5, 0.25]], device="cuda")
    sd.switchsd_token_logprobs_grad(args, out["lse"], out["entropy"], gl, ge, x)
    p = lp.exp()
    want = -p * (gl[:, :, None] + ge[:, :, None] * (lp + entropy[:, :, None]))
    want.scatter_add_(2, tokens.long()[:, :, None], gl.double()[:, :, None])
    # p by the given lse and entropy, and a few roundings of each term
    part = p * (1 + lp.abs() + entropy[:, :, None])
    bound = 1.01 * u * want.abs() + part * 2 * (tol + 2.0 ** -20)
    bound.scatter_add_(2, tokens.long()[:, :, None], 2.0 ** -22 * gl.double().abs()[:, :, None])
    assert ((x.double() - want).abs() <= bound + 1e-38).all()
