"""One object of the example, used for more than one prompt."""
import pytest
import torch

from test_gpu_continue_prompt import example

pytestmark = pytest.mark.gpu


def fresh(ex, w, steps=3):
    return ex.Continuations(w, 4, 2, 64, 3, 70, steps)


def tokens(seed, n):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return torch.randint(128, (n,), generator=g, device="cuda")


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_a_second_prompt_is_continued_as_by_a_new_object(dtype):
    """Its own blocks and no tokens of the first prompt's continuations: the same kernels on the same numbers, so the same bits."""
    ex = example()
    w = ex.weights(2, 256, 512, 4, 2, 64, 128, dtype, seed=3)
    run, other = fresh(ex, w), fresh(ex, w)
    run.prompt(tokens(1, 70))
    for i in range(2):
        run.generate(tokens(10 + i, 3))
    assert torch.equal(run.prompt(tokens(2, 70)), other.prompt(tokens(2, 70)))
    assert len(run.kept) == 2 and all(torch.equal(a, b) for a, b in zip(run.kept, other.kept))
    for i in range(3):
        assert torch.equal(run.generate(tokens(20 + i, 3)), other.generate(tokens(20 + i, 3))), i
    assert run.lens.tolist() == [3, 3, 3]


def test_more_steps_than_there_is_room_for_are_refused():
    """The pages and tables hold `steps` tokens of a row; one more would be seen by nobody."""
    ex = example()
    run = fresh(ex, ex.weights(2, 256, 512, 4, 2, 64, 128, torch.float32, seed=3), steps=2)
    for _ in range(2):
        run.prompt(tokens(1, 70))
        for i in range(2):
            run.generate(tokens(i, 3))
        with pytest.raises(ValueError):
            run.generate(tokens(2, 3))
        assert run.lens.tolist() == [2, 2, 2]
