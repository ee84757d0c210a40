"""The example in which pruned blocks draft and full blocks verify: the calls of a run, each checked against its definition on the very inputs that it got."""
import importlib.util
import os

import numpy as np
import pytest
import torch

import layer_plain as plain
import q4_plain
import synth
from test_gpu_q4 import attention_close

pytestmark = pytest.mark.gpu

PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "draft_and_verify.py")


def example():
    spec = importlib.util.spec_from_file_location("draft_and_verify", PATH)
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


def host(t):
    return t.detach().double().cpu().numpy()


class Checked:
    """The binding, whose calls of the cache in 4 bits and of the verification are followed by their definitions"""

    def __init__(self, G, shape, dtype):
        self.G, self.shape, self.dtype, self.count = G, shape, dtype, dict(append=0, attend=0, verify=0)

    def __getattr__(self, name):
        return getattr(self.G, name)

    def pools(self, C):
        return [t.cpu().numpy() for t in C._keep]

    def batch(self, B):
        arr, lens, pages, prefix = B._keep
        return list(arr), lens.tolist(), pages.cpu().numpy(), np.zeros(0, np.int32) if prefix is None else prefix.cpu().numpy(), B.max_len, B.n_prefix

    def griffin_kv_append_q4(self, C, B, k, v, *, q, q_out, cos, sin):
        kv_heads, dim, page, group = self.shape
        before = self.pools(C)
        self.G.griffin_kv_append_q4(C, B, k, v, q=q, q_out=q_out, cos=cos, sin=sin)
        c = plain.Case.__new__(plain.Case)
        c.cu, c.lens, c.pages, _, c.max_len, c.prefix = self.batch(B)
        c.page, c.k, c.v = page, host(k), host(v)
        views = [np.array(x) for pool in before for x in q4_plain.parts(pool, kv_heads, dim, page, group)]
        q4_plain.append(*views, c, cos.cpu().numpy(), sin.cpu().numpy(), "half", group)
        for pool, codes, pairs in zip(self.pools(C), views[::2], views[1::2]):
            got = q4_plain.parts(pool, kv_heads, dim, page, group)
            assert np.array_equal(got[0], codes) and np.array_equal(np.ascontiguousarray(got[1]).view(np.uint16), np.ascontiguousarray(pairs).view(np.uint16))
        self.count["append"] += 1

    def griffin_attention_q4(self, C, B, q, out, *, workspace):
        kv_heads, dim, page, group = self.shape
        self.G.griffin_attention_q4(C, B, q, out, workspace=workspace)
        K, V = (q4_plain.values(*q4_plain.parts(pool, kv_heads, dim, page, group), dim, group) for pool in self.pools(C))
        cu, lens, pages, prefix, max_len, n_prefix = self.batch(B)
        ref, size = plain.attention(host(q), K, V, cu, lens, pages, prefix, page, n_prefix, max_len, dim ** -0.5)
        attention_close(host(out), ref, size, self.dtype)
        self.count["attend"] += 1

    def griffin_verify_drafts(self, cu, p, drafted, u, r, tokens, kept, *, draft_p=None, lens=None, lens_out=None, workspace):
        before = None if lens is None else lens.cpu().numpy()
        self.G.griffin_verify_drafts(cu, p, drafted, u, r, tokens, kept, draft_p=draft_p, lens=lens, lens_out=lens_out, workspace=workspace)
        on = lambda t: None if t is None else t.cpu().numpy()  # noqa: E731
        want = q4_plain.verify(on(p), on(draft_p), on(drafted), list(cu), on(u), on(r))
        assert np.array_equal(on(tokens), want[0]) and np.array_equal(on(kept), want[1])
        if lens is not None:
            assert np.array_equal(on(lens_out), before + want[1] + 1)
        self.count["verify"] += 1


@pytest.mark.parametrize("dtype", [synth.DT_F32, synth.DT_BF16])
@pytest.mark.parametrize("rows,drafts,keep,group", [(3, 4, 0.5, 32), (5, 1, 0.75, 64), (1, 6, 0.25, 32)])
def test_rounds_of_drafts(dtype, rows, drafts, keep, group):
    ex = example()
    real = ex.G
    ex.G = checked = Checked(real, (2, 64, ex.PAGE, group), dtype)
    w = ex.weights(2, 128, 256, 4, 2, 64, 96, torch.float32 if dtype == synth.DT_F32 else torch.bfloat16, seed=rows)
    run = ex.Speculation(w, 4, 2, 64, rows, 70, 12, drafts, keep=keep, group=group)
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    last = run.prompt(torch.randint(96, (70,), generator=g, device="cuda"))
    out = run.generate(last)
    assert all(0 <= t < 96 for row in out for t in row)
    assert [len(row) - 1 for row in out] == run.lens.tolist() and max(run.lens.tolist()) >= 12
    rounds = (checked.count["verify"] - 1) // (drafts + 1)
    assert rounds >= 2 and checked.count["append"] == checked.count["attend"] == 2 * (1 + rounds * (drafts + 1))


def test_drafts_of_blocks_that_keep_everything_are_kept():
    """A draft that is the target up to the order of fp32 sums: u q(d) < p(d) fails for a u within some 1e-5 of one at most"""
    ex = example()
    w = ex.weights(2, 128, 256, 4, 2, 64, 96, torch.float32, seed=9)
    run = ex.Speculation(w, 4, 2, 64, 8, 40, 30, 3, keep=1.0)
    g = torch.Generator(device="cuda")
    g.manual_seed(5)
    last = run.prompt(torch.randint(96, (40,), generator=g, device="cuda"))
    all_kept = []
    while int(run.lens.max()) < run.steps:
        _, kept, last = run.round(last)
        all_kept += kept.tolist()
    assert np.mean(all_kept) > 2.9


def test_more_rows_than_a_block_takes_are_refused():
    ex = example()
    w = ex.weights(1, 64, 64, 2, 1, 64, 32, torch.float32)
    with pytest.raises(ValueError, match="more than a block takes"):
        ex.Speculation(w, 2, 1, 64, 13, 8, 8, 4)
