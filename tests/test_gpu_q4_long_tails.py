"""Attention over a cache in 4 bits, fp32: keys of little weight beside one of much."""
import numpy as np
import pytest

import layer_plain as plain
import q4_plain
import synth
from test_gpu_q4 import run_attention

pytestmark = pytest.mark.gpu


# Of 32 keys one has a score that is 2^gap times the others' weight above theirs, at places that every wavefront meets first.  The heavy keys' values are 0 and the others' 1, so that the output is
# the others' share of the sum.  Weights are held to 2^-22 of themselves and 2^-32 of the row's largest, that is 2^(gap - 32) of a light one.  A score of up to 22 (base 2) is off by its
# roundings: scale and its product with log2(e), 2^-24 each, the queries' pairs of fp16, 2^-23, the exponent's own, 2^-24 of 22: 22 ln 2 x 5 x 2^-24 of a weight; exp2 and the sums as much as 2^-20.
@pytest.mark.parametrize("new", [1, 40])
@pytest.mark.parametrize("gap", [14.3, 17.31, 19.7])
def test_light_keys_keep_their_share(new, gap):
    heads, page, n = 8, 16, 1024
    c = plain.Case(3, heads=heads, kv_heads=1, dim=64, page=page, prefix=0, held=[n - new], new=[new], dtype=synth.DT_F32)
    light = np.ones(n, bool)
    light[::32] = False
    for i in range(n):
        at = c.pages[0, i // page], 0, i % page
        c.K[at] = 0
        c.K[at][:3] = -8 if light[i] else 7, -8, 7           # the first group's scale is 1 and its middle 0, whatever the first feature is
        c.V[at] = 1.0 if light[i] else 0.0
    # queries that put a light key's weight at every sixteenth of a step of fp16 below its normal numbers
    gaps = gap + np.arange(new * heads).reshape(new, heads) / 16 * 2.0 ** -10 / np.log(2)
    c.q[:] = 0
    c.q[..., 0] = plain.stored(gaps * np.log(2) / 15, synth.DT_F32)
    K, V = q4_plain.pool_of(c.K, 32), q4_plain.pool_of(c.V, 32)
    got = run_attention(c, K, V, 32, scale=1.0)
    for t in range(new):
        seen = n - new + t + 1
        heavy, few = int((~light[:seen]).sum()), int(light[:seen].sum())
        w = np.exp(-15 * c.q[t, :, 0])
        share = few * w / (heavy + few * w)
        tol = 2.0 ** -22 + 2.0 ** -32 / w + 22 * np.log(2) * 5 * 2.0 ** -24 + 2.0 ** -20
        off = np.abs(got[t] / share[:, None] - 1).max(axis=1)
        assert np.all(off <= tol), (t, (off / tol).max(), off.max())
