"""Verification of drafted tokens where a goal lies within a rounding of a running sum: sums of one order pass it and sums of another do not.  Any token with weight may come
out there, and none without."""
import numpy as np
import pytest
import torch

import paper_2404_01365_amd as G
from test_gpu_layer import ints

pytestmark = pytest.mark.gpu

PIECE = 1024


def draw(p, r, q=None, drafted=None):
    """the token drawn at a first row of every sequence: two rows each, the first one's draft refused, or (drafted None) one row"""
    n, vocab = p.shape
    rows = 1 if drafted is None else 2
    f = lambda a: torch.from_numpy(np.ascontiguousarray(a, np.float32)).cuda()  # noqa: E731
    full = lambda a: f(np.repeat(a, rows, axis=0))  # noqa: E731
    d = np.zeros(n * rows, np.int32)
    if drafted is not None:
        d[::2] = drafted
    u = f(np.full(n * rows, 1 - 2.0 ** -24))
    out, kept = ints(np.zeros(n * rows)), ints(np.zeros(n))
    ws = torch.zeros(G.griffin_verify_workspace_bytes(n, vocab) + 256, dtype=torch.uint8, device="cuda")
    G.griffin_verify_drafts(range(0, n * rows + 1, rows), full(p), ints(d), u, f(r), out, kept, draft_p=None if q is None else full(q), workspace=ws)
    assert kept.tolist() == [0] * n
    return out.cpu().numpy()[::rows]


def cases(vocab):
    """weights and what is known of them: 1, light ones that are lost or not by the order in which they are added to it, none up to the piece's end, and 1 in the next piece"""
    w = np.zeros((6, vocab), np.float32)
    w[:, 0] = w[:, PIECE] = 1
    w[0, 1:1000] = 3 * 2.0 ** -63
    w[1, 4:8] = 0.3 * 2.0 ** -52
    w[2, 4:8] = 0.45 * 2.0 ** -52
    w[3, 1:512] = 3 * 2.0 ** -62
    w[4, 64:1020] = 3 * 2.0 ** -63
    w[5, 1:PIECE:2] = 3 * 2.0 ** -62
    return w


@pytest.mark.parametrize("vocab", [2048, 2047, 32768, 33000, 40001])
@pytest.mark.parametrize("form", ["p", "p - q", "looked up"])
def test_no_token_without_weight_is_drawn(vocab, form):
    w = cases(vocab)
    r = np.full(len(w), 0.5)
    if form == "p":
        got = draw(w, r)
    elif form == "p - q":
        drafted = np.full(len(w), 1020)
        q = np.where(w > 0, np.float32(0), np.float32(0.25))           # nothing of the draft's is left where w is zero
        got = draw(w, r, q, drafted)
    else:
        drafted = np.full(len(w), 1020)
        p = w.copy()
        p[:, 1020] = 0.5                                               # refused (u is next to one), and left out
        got = draw(p, r, None, drafted)
        w = np.where(np.arange(vocab) == 1020, np.float32(0), w)
    assert np.all(w[np.arange(len(w)), got] > 0), got.tolist()


def test_pieces_without_weight_are_passed_over():
    """sums of pieces, added up in two orders: a thread's pieces one behind the other, the threads' together"""
    vocab = 300 * PIECE                                                # two pieces a thread
    w = np.zeros((3, vocab), np.float32)
    w[:, 0] = w[:, 200 * PIECE] = 1
    w[0, 2 * PIECE], w[0, 3 * PIECE] = 0.4 * 2.0 ** -52, 0.4 * 2.0 ** -52
    w[1, 2 * PIECE:4 * PIECE] = 3 * 2.0 ** -64
    w[2, 2 * PIECE:90 * PIECE:PIECE] = 3 * 2.0 ** -58
    got = draw(w, np.full(3, 0.5))
    assert np.all(w[np.arange(3), got] > 0), got.tolist()


@pytest.mark.parametrize("vocab", [700, 50000])
def test_goals_beyond_the_sum_give_the_last_token(vocab):
    w = np.zeros((2, vocab), np.float32)
    w[0, :100] = 0.01
    got = draw(w, np.array([1.0, 0.5]))                                # a random number that is not below one; no weight at all
    assert got.tolist() == [vocab - 1, vocab - 1]
