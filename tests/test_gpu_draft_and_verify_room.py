"""The example in which pruned blocks draft: a round that the cache has no room for is refused, and leaves everything as it was."""
import pytest
import torch

from test_gpu_draft_and_verify import example

pytestmark = pytest.mark.gpu


def test_rounds_beyond_the_room_are_refused():
    ex = example()
    w = ex.weights(1, 64, 128, 2, 1, 64, 32, torch.float32, seed=2)
    run = ex.Speculation(w, 2, 1, 64, 3, 20, 9, 2, keep=1.0)
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    tokens = torch.randint(32, (20,), generator=g, device="cuda")
    for _ in range(2):                                    # ... and another prompt begins anew
        last = run.prompt(tokens)
        rounds = 0
        while int(run.lens.max()) + 3 <= 9 + 2 + 1:
            _, _, last = run.round(last)
            rounds += 1
        assert rounds >= 3
        held = run.lens.clone()
        pools = [t.clone() for C in run.caches for t in C._keep]
        with pytest.raises(ValueError, match="12 tokens a row"):
            run.round(last)
        assert torch.equal(run.lens, held) and all(torch.equal(a, b) for a, b in zip(pools, (t for C in run.caches for t in C._keep)))
