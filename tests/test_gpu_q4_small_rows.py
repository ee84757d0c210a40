"""Attention over a cache in 4 bits of rows whose scores are next to nothing: queries below fp32's normal numbers, scales that take the product there."""
import numpy as np
import pytest

import layer_plain as plain
import q4_plain
import synth
from test_gpu_q4 import attention_close, reference, run_attention

pytestmark = pytest.mark.gpu

F32, BF16 = synth.DT_F32, synth.DT_BF16


# A score below 2^-60 changes no weight in fp32: the rows weigh their keys alike to the tolerance that other rows have, and their neighbours are as ever.
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("new", [[1, 3], [70, 40]])           # a few rows from memory; many, which bf16 caches take through LDS
@pytest.mark.parametrize("power,scale", [(-135, None), (-141, None), (-142, None), (-148, None), (-133, 1e-4), (-100, 1e-20)])
def test_rows_next_to_zero_weigh_their_keys_alike(dtype, dim, new, power, scale):
    c = plain.Case(31, heads=8, kv_heads=4, dim=dim, page=16, prefix=20, held=[300, 5], new=new, dtype=dtype)
    for row in ((0, 0), (1, 2), (-1, 7)):
        c.q[row] = plain.stored(c.q[row] * 2.0 ** power, dtype)
    K, V = q4_plain.pool_of(c.K, 32), q4_plain.pool_of(c.V, 32)
    ref, most = reference(c, K, V, 32, scale)
    attention_close(run_attention(c, K, V, 32, scale=scale), ref, most, dtype)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("new", [[1, 3], [70, 40]])
@pytest.mark.parametrize("scale", [2.0 ** -126, 1e-42, 2.0 ** -149])
def test_scales_next_to_zero_weigh_all_keys_alike(dtype, new, scale):
    c = plain.Case(32, heads=8, kv_heads=4, dim=64, page=16, prefix=20, held=[300, 5], new=new, dtype=dtype)
    K, V = q4_plain.pool_of(c.K, 32), q4_plain.pool_of(c.V, 32)
    ref, most = reference(c, K, V, 32, scale)
    attention_close(run_attention(c, K, V, 32, scale=scale), ref, most, dtype)
