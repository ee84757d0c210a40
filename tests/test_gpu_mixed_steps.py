"""Steps in which some sequences bring a token and others many, behind a prefix, against the definition in 64 bits."""
import pytest

import synth
from test_gpu_layer import check_attention

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("prefix", [70, 900, 4100])
def test_single_tokens_beside_a_prompt(dim, prefix):
    """More than 128 tiles of rows, nearly all of them a few rows: a short prefix ahead of own keys, a long one in chunks of its own."""
    new = [1] * 12 + [40] + [1] * 6 + [0, 66]
    check_attention(3 + dim, heads=24, kv_heads=8, dim=dim, page=32, prefix=prefix, held=[(37 * i) % 150 for i in range(len(new))], new=new, dtype=synth.DT_BF16)


@pytest.mark.parametrize("prefix", [300, 5000])
def test_drafts_of_several_tokens(prefix):
    check_attention(9, "thd", heads=64, kv_heads=8, dim=64, page=64, prefix=prefix, held=list(range(0, 170, 10)), new=[9] * 17, dtype=synth.DT_BF16)
