"""Verification of drafted tokens against its definition, sums in 64 bits."""
import numpy as np
import pytest
import torch

import paper_2404_01365_amd as G
import q4_plain
from test_gpu_layer import ints

pytestmark = pytest.mark.gpu


def softmax(x):
    e = np.exp(x - x.max(axis=-1, keepdims=True))
    return (e / e.sum(axis=-1, keepdims=True)).astype(np.float32)


class Drafts:
    def __init__(self, seed, rows, vocab, *, agree=0.3, sharp=2.0, greedy=False):
        rng = np.random.default_rng(seed)
        self.cu = [0] + [int(x) for x in np.cumsum(rows)]
        T = self.cu[-1]
        logits = rng.standard_normal((T, vocab)) * sharp
        self.p = softmax(logits)
        self.q = None if greedy else softmax(logits + agree * rng.standard_normal((T, vocab)))
        draw = self.p if greedy else self.q
        self.drafted = (draw / rng.exponential(size=(T, vocab))).argmax(axis=1).astype(np.int32)
        self.u, self.r = rng.random(T).astype(np.float32), rng.random(len(rows)).astype(np.float32)
        self.vocab, self.lens = vocab, rng.integers(0, 1000, len(rows)).astype(np.int32)

    def run(self, pad=0, lens="in place", stream=None):
        f = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()  # noqa: E731

        def rows(a):
            if a is None:
                return None
            buf = torch.full((a.shape[0], self.vocab + pad), float("nan"), device="cuda")
            buf[:, :self.vocab] = f(a)
            return buf[:, :self.vocab]

        tokens, accepted = (torch.full((n,), 77, dtype=torch.int32, device="cuda") for n in (self.cu[-1], len(self.cu) - 1))
        held = ints(self.lens)
        out = held if lens == "in place" else torch.zeros_like(held)
        size = G.griffin_verify_workspace_bytes(len(self.cu) - 1, self.vocab)
        ws = torch.full((size + 256,), 0xFF, dtype=torch.uint8, device="cuda")
        G.griffin_verify_drafts(self.cu, rows(self.p), ints(self.drafted), f(self.u), f(self.r), tokens, accepted, draft_p=rows(self.q),
                                lens=None if lens is None else held, lens_out=None if lens is None else out, workspace=ws, stream=stream)
        torch.cuda.synchronize()
        return tokens.cpu().numpy(), accepted.cpu().numpy(), out.cpu().numpy()

    def check(self, **kw):
        tokens, accepted, lens = self.run(**kw)
        want = q4_plain.verify(self.p, self.q, self.drafted, self.cu, self.u, self.r)
        assert np.array_equal(accepted, want[1])
        assert np.array_equal(tokens, want[0]), np.argwhere(tokens != want[0])[:5].tolist()
        if kw.get("lens", "") is not None:
            assert np.array_equal(lens, self.lens + accepted + (np.diff(self.cu) > 0))


@pytest.mark.parametrize("greedy", [False, True])
@pytest.mark.parametrize("rows,vocab,pad", [
    ([1], 1, 0), ([3], 2, 0), ([5], 1000, 0), ([2, 1, 4, 9], 255, 1), ([5] * 16, 4096, 0), ([3, 3], 4097, 3), ([9, 1], 8191, 0), ([4, 2, 7], 32000, 0),
    ([2] * 64, 5000, 8), ([1] * 256, 300, 0), ([70, 130], 600, 0), ([4], 128001, 0), ([0, 3, 0], 777, 0)])
def test_drafts(rows, vocab, pad, greedy):
    for seed in range(3):
        Drafts(seed + vocab, rows, vocab, greedy=greedy).check(pad=pad)


@pytest.mark.parametrize("agree,sharp", [(0.0, 2.0), (3.0, 2.0), (0.5, 0.01), (0.5, 12.0)])
def test_drafts_that_agree_more_or_less(agree, sharp):
    """The same probabilities (everything is kept), others altogether, flat ones and ones with next to all on one token"""
    d = Drafts(5, [6] * 40, 3000, agree=agree, sharp=sharp)
    if agree == 0.0:
        d.q = d.p.copy()
        assert np.array_equal(d.run()[1], np.full(40, 5))
    d.check()


def test_lengths_are_as_asked_for():
    d = Drafts(6, [3, 1, 4], 500)
    d.check(lens="apart")
    d.check(lens=None)


def test_drafts_that_are_none():
    """Tokens outside the vocabulary end their sequence, with the target's own probabilities; a last row's entry is not looked at."""
    for greedy in (False, True):
        d = Drafts(7, [5, 5, 5, 2], 900, greedy=greedy)
        d.u[:] = 0.0
        d.drafted[1], d.drafted[7], d.drafted[14], d.drafted[16] = -1, 900, 2 ** 31 - 1, -(2 ** 31)
        d.check()
        assert d.run()[1][:2].tolist() == [1, 2]


@pytest.mark.parametrize("r", [0.0, 0.5, np.float32(1 - 2.0 ** -24)])
def test_draws_at_the_ends(r):
    d = Drafts(8, [3] * 20, 4500)
    d.u[:] = np.float32(1 - 2.0 ** -24)
    d.r[:] = r
    d.p[:, :7] = 0
    d.p[:, -5:] = 0                          # no weight at either end
    d.check()
    tokens, accepted, _ = d.run()
    drawn = tokens.reshape(20, 3)[np.arange(20), accepted]
    assert drawn.min() >= 7 and drawn.max() < 4495


def test_ties_of_the_goal_go_to_the_token_behind():
    """Sums that are exact: the goal is one of them, and the token that the sum passes it at comes out"""
    d = Drafts(9, [1] * 8, 4096 + 512)
    d.p[:] = 2.0 ** -13
    d.r = (np.arange(8) / 8).astype(np.float32)
    tokens, _, _ = d.run()
    assert tokens.tolist() == [i * (4096 + 512) // 8 for i in range(8)]
    d.check()


def test_weights_that_are_all_zero():
    d = Drafts(10, [2, 2, 2], 700)
    d.q = d.p.copy()
    d.q[:, :] = d.p * np.float32(2)          # refused, and nothing is left over: drawn from p
    d.u[:] = np.float32(0.9)
    d.check()
    d = Drafts(10, [2, 2], 700, greedy=True)
    d.p[:] = 0                               # nothing at all: the last token
    d.check()
    assert d.run()[0].tolist() == [699, -1, 699, -1]
    d = Drafts(11, [2], 4097, greedy=True)
    d.p[0] = 0
    d.p[0, 5], d.drafted[0], d.u[0] = 1e-30, 5, 0.5       # kept: 0.5 < 1e-30 is not; refused, and p is what is drawn from
    d.check()


def test_the_distribution_is_the_target_s():
    """What a verified step says first, over many random numbers, is distributed as the target's first row: a chi-square statistic of 15 degrees of freedom beyond
    50 has a probability of 1e-5."""
    vocab, n = 16, 256
    rng = np.random.default_rng(0)
    logits, near = rng.standard_normal(vocab), rng.standard_normal(vocab)
    count = np.zeros(vocab)
    for i in range(40):
        d = Drafts(100 + i, [2] * n, vocab)
        d.p[:], d.q[:] = softmax(logits), softmax(logits + near)
        d.drafted = rng.choice(vocab, size=2 * n, p=d.q[0].astype(np.float64) / d.q[0].astype(np.float64).sum()).astype(np.int32)
        count += np.bincount(d.run()[0].reshape(n, 2)[:, 0], minlength=vocab)
    want = softmax(logits) * count.sum()
    assert ((count - want) ** 2 / want).sum() < 50


def test_verification_on_another_stream_and_in_a_graph():
    d = Drafts(12, [5] * 6, 20000)
    f = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()  # noqa: E731
    p, q, drafted, u, r = f(d.p), f(d.q), ints(d.drafted), f(d.u), f(d.r)
    lens = ints(d.lens)
    ws = torch.empty(G.griffin_verify_workspace_bytes(6, d.vocab) + 256, dtype=torch.uint8, device="cuda")
    tokens, accepted = torch.zeros(30, dtype=torch.int32, device="cuda"), torch.zeros(6, dtype=torch.int32, device="cuda")
    cu = G.cu_seqlens(d.cu)
    call = lambda: G.griffin_verify_drafts(cu, p, drafted, u, r, tokens, accepted, draft_p=q, lens=lens, lens_out=lens, workspace=ws)  # noqa: E731
    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        call()
    stream.synchronize()
    held = lens.cpu().numpy()
    assert np.array_equal(held, d.lens + q4_plain.verify(d.p, d.q, d.drafted, d.cu, d.u, d.r)[1] + 1)
    with torch.cuda.graph(graph, stream=stream):
        call()
    for i in range(4):
        d.u, d.r = np.roll(d.u, 3), np.roll(d.r, 1)
        u.copy_(f(d.u)), r.copy_(f(d.r)), tokens.fill_(5)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        want = q4_plain.verify(d.p, d.q, d.drafted, d.cu, d.u, d.r)
        assert np.array_equal(tokens.cpu().numpy(), want[0]) and np.array_equal(accepted.cpu().numpy(), want[1])
        held = held + want[1] + 1
        assert np.array_equal(lens.cpu().numpy(), held)
