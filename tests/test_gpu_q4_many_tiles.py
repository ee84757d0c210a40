"""Attention over a cache in 4 bits of prompts of more than 512 tiles of all heads, cut and whole, against one token a call (straight from memory)."""
import pytest

from test_gpu_q4 import test_attention_of_prompts_in_several_rounds_and_row_by_row as rounds

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("heads,kv_heads,dim,prefix,held,new", [
    (32, 8, 128, 0, 30000, 2100),           # 528 tiles in three parts
    (32, 8, 128, 0, 4000, 2500),            # 632, whole
    (64, 64, 64, 0, 30000, 1100),           # 576 of one query head each
    (32, 8, 256, 0, 30000, 1300),           # 656 of 64 rows
    (32, 8, 128, 5000, 0, 2500)])           # ... that take a prefix ahead of their own keys
def test_prompts_of_more_tiles_than_a_round(heads, kv_heads, dim, prefix, held, new):
    rounds(heads, kv_heads, dim, prefix, held, new)
