"""The workspace that the arguments of the log probabilities bring: zeroed on the stream
that is current where they are built, used on any."""
import numpy as np
import pytest
import torch

from gpu_helpers import say
from test_logprobs_gpu import DEV, check, dev, make, run

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2609_20186_amd import binding  # noqa: F401


def busy(x):
    """Some tens of milliseconds of work on the current stream."""
    for _ in range(40):
        torch.mm(x, x)


class Handle:
    """A stream of another library: its handle alone."""

    def __init__(self, stream):
        self.cuda_stream = stream.cuda_stream


@pytest.mark.parametrize("first", ["other", "handle", "same"])
def test_first_call_waits_for_the_zeroing(first):
    """The memory held something else before and the building stream is busy; a call on
    another stream, or one there behind a call on the building stream."""
    from paper_2609_20186_amd import binding as sd
    a = make(2, 3, 50257, "bf16", seed=3, dn=False)
    logits, tokens = a["logits"].to(DEV), dev(a["tokens"])
    x = torch.zeros(8192, 8192, dtype=torch.bfloat16, device=DEV)
    out = {n: torch.full((2, 3), 77.0, device=DEV) for n in ("logprob", "lse", "entropy")}
    out["rank"] = torch.full((2, 3), 77, dtype=torch.int32, device=DEV)
    out["top_ids"] = torch.full((2, 3, 5), 77, dtype=torch.int32, device=DEV)
    out["top_logprobs"] = torch.full((2, 3, 5), 77.0, device=DEV)
    other = torch.cuda.Stream()
    busy(x)
    torch.cuda.synchronize()
    for _ in range(3):
        need = sd.logprob_workspace_bytes(sd.build_logprob_args(logits, tokens))
        assert need > 0
        torch.full((need,), 0xFF, dtype=torch.uint8, device=DEV)  # given back at once
        busy(x)
        args = sd.build_logprob_args(logits, tokens)
        if first == "same":
            run(a, 1.0, 5, args=args, out=out)
            other.wait_stream(torch.cuda.current_stream())
        run(a, 1.0, 5, args=args, out=out, stream=Handle(other) if first == "handle" else other)
        other.synchronize()
        got = {n: t.clone() for n, t in out.items()}
        check(a, 1.0, 5, got, f"{first} stream first")
        assert int(args.keep[-1].count_nonzero()) == 0   # left zeroed
        for t in out.values():
            t.fill_(77)
        torch.cuda.synchronize()
    say("waited")


def test_calls_on_two_streams_at_once():
    """Each with arguments of its own, built while the current stream is busy."""
    from paper_2609_20186_amd import binding as sd
    made = [make(4, 8, 32000, "bf16", seed=1), make(4, 8, 50257, "f32", seed=2)]
    on = [a["logits"].to(DEV) for a in made]
    where = [[dev(a[n]) for n in ("tokens", "dn")] for a in made]
    outs = [{n: torch.full((4, 8), 77.0, device=DEV) for n in ("logprob", "lse", "entropy")}
            for _ in made]
    for o in outs:
        o["rank"] = torch.full((4, 8), 77, dtype=torch.int32, device=DEV)
        o["top_ids"] = torch.full((4, 8, 5), 77, dtype=torch.int32, device=DEV)
        o["top_logprobs"] = torch.full((4, 8, 5), 77.0, device=DEV)
    x = torch.zeros(8192, 8192, dtype=torch.bfloat16, device=DEV)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    busy(x)
    args = [sd.build_logprob_args(t, *w, temperature=T)
            for t, w, T in zip(on, where, (1.0, 0.7))]
    for a, g, o, s in zip(made, args, outs, streams):
        run(a, None, 5, args=g, out=o, stream=s)
    torch.cuda.synchronize()
    for a, o, T in zip(made, outs, (1.0, 0.7)):
        check(a, T, 5, o, f"T={T}")
    assert all(int(np.count_nonzero(g.keep[-1].cpu())) == 0 for g in args)
