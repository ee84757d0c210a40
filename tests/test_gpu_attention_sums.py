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


@pytest.mark.parametrize("dim,early", [(64, 100), (128, 100), (256, 170)])
def test_an_infinite_value_is_added_by_its_own_chunk(dim, early):
    """A prompt in chunks of 64 keys (32 of wide heads), nearly all of whose weight lies on one key with an infinite feature.  A chunk behind that key's, which has an infinite
    value of its own, has sums that the join scales by 2^-288: it must not add the early key's once more (0 x Inf)."""
    c = plain.Case(6, heads=1, kv_heads=1, dim=dim, page=256, prefix=0, held=[0], new=[256], dtype=BF16)
    set_scores(c, lambda slot: np.where(slot == early, 200.0, 0.0))
    ref, size = c.attention(1.0)
    page = c.pages[0, 0]
    c.V[page, 0, early, 7], c.V[page, 0, 200, 9] = np.inf, np.inf
    got = run_attention(c, scale=1.0)
    assert np.all(got[early:, :, 7] == np.inf) and np.isfinite(got[:early]).all()
    assert not np.isfinite(got[200:, :, 9]).any()
    got[early:, :, 7], got[200:, :, 9] = ref[early:, :, 7], ref[200:, :, 9]
    attention_close(got, ref, size, BF16)
