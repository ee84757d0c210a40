"""The sums of an attention: its weights add up to one, and what is infinite is counted where it is and nowhere else."""
import numpy as np
import pytest

import layer_plain as plain
import synth
from test_gpu_layer import attention_close, run_attention

pytestmark = pytest.mark.gpu

BF16, F32 = synth.DT_BF16, synth.DT_F32


def set_scores(c, key_of):
    """q k of every row and key: key_of(slots of a page) where something is stored"""
    c.q[:], c.q[..., 0] = 0.0, 1.0
    held = ~np.isnan(c.K)
    c.K[held] = 0.0
    first = np.broadcast_to(key_of(np.arange(c.page)), c.K.shape[:3])
    c.K[..., 0] = np.where(held[..., 0], first, np.nan)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("heads,kv_heads,dim,prefix,held,new", [
    (4, 4, 128, 0, [100], [1]),                              # one launch
    (4, 2, 64, 0, [512, 40], [1, 2]),                        # chunks
    (8, 2, 256, 333, [90], [1]),
    (8, 8, 128, 64, [60] * 160, [1] * 160),                  # a wavefront each
    (4, 2, 128, 0, [0, 33], [300, 70]),                      # prompts in chunks of keys
    (32, 32, 64, 70, [0, 17], [260, 300]),                   # ... that take the prefix ahead of their own keys
    (4, 2, 256, 40, [10], [140]),
    (64, 2, 128, 43700, [700, 0, 250], [1, 1, 2]),           # a prefix in tiles
])
def test_the_mean_of_equal_values_is_that_value(dtype, heads, kv_heads, dim, prefix, held, new):
    """Every sixteenth key has the weight 1, the others 0.5 (1 + 0.98 x 2^-8), which bf16 rounds to 0.5.  As numerator and sum are made of the same weights, a mean
    of equal values is their value whatever the weights were rounded to: products of 8 bits by 8 are exact, sums of up to 44000 terms in fp32 are off by less than
    the half last place (2^-9) of an output."""
    c = plain.Case(5, heads=heads, kv_heads=kv_heads, dim=dim, page=64, prefix=prefix, held=held, new=new, dtype=dtype)
    set_scores(c, lambda slot: (slot % 16 == 0).astype(float))
    value = 1.9921875
    c.V[~np.isnan(c.V)] = value
    got = run_attention(c, scale=-np.log(0.5 * (1 + 0.98 * 2.0 ** -8)))
    assert np.all(got == value) if dtype == BF16 else np.abs(got - value).max() <= 2e-5
