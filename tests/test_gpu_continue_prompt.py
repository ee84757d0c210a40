"""The example that runs the blocks, norms, cache and attention together, against the same stack in 64 bits on the host."""
import importlib.util
import os

import numpy as np
import pytest
import torch

import layer_plain as plain

pytestmark = pytest.mark.gpu

PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "continue_prompt.py")


def example():
    spec = importlib.util.spec_from_file_location("continue_prompt", PATH)
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


def host(t):
    return t.detach().double().cpu().numpy()


def silu(a):
    return a / (1 + np.exp(-a))


def reference(w, kept, prompt, rows, heads, kv_heads, dim, eps):
    """Logits of the prompt's tokens, then a function that takes one token of every row and gives the logits of the next."""
    layers = [{k: host(v) for k, v in x.items()} for x in w["layers"]]
    embed, last = host(w["embed"]), host(w["last"])
    norm = lambda v, g: plain.unit(v, g, None, layer=False, eps=eps, offset=0.0)  # noqa: E731
    keys = [[np.zeros((0, kv_heads, dim)) for _ in range(rows)] for _ in layers]
    vals = [[np.zeros((0, kv_heads, dim)) for _ in range(rows)] for _ in layers]
    rate = 10000.0 ** (-np.arange(0, dim, 2) / dim)

    def attend(q, k, v, seen):
        out = np.zeros_like(q)
        for i in range(q.shape[0]):
            for h in range(heads):
                kh = k[:seen + i + 1, h // (heads // kv_heads)]
                s = kh @ q[i, h] * dim ** -0.5
                p = np.exp(s - s.max())
                out[i, h] = (p / p.sum()) @ v[:seen + i + 1, h // (heads // kv_heads)]
        return out

    def run(tokens, per_row, neurons):
        """tokens [rows][n] of sequences (one for the prompt); per_row: which of their caches they go on with"""
        n, count = tokens.shape[1], tokens.shape[0]
        h = embed[tokens]                                          # [row][n][d]
        for i, x in enumerate(layers):
            y = np.zeros_like(h)
            for b in range(count):
                qkv = (norm(h[b], x["norm1"]) @ x["qkv"].T).reshape(n, -1, dim)
                pos = per_row[i][b].shape[0] + np.arange(n)
                c, s = np.cos(pos[:, None] * rate)[:, None], np.sin(pos[:, None] * rate)[:, None]
                q, k, v = plain.rotate(qkv[:, :heads], c, s, "half"), plain.rotate(qkv[:, heads:heads + kv_heads], c, s, "half"), qkv[:, heads + kv_heads:]
                seen = per_row[i][b].shape[0]
                per_row[i][b] = np.concatenate([per_row[i][b], k])
                vals[i][b] = np.concatenate([vals[i][b], v])
                y[b] = attend(q, per_row[i][b], vals[i][b], seen).reshape(n, -1) @ x["out"].T
            h = h + y
            u = norm(h, x["norm2"])
            Wg, W1, W2 = (x[m] if neurons is None else x[m][neurons[i]] for m in ("Wg", "W1", "W2"))
            h = h + (silu(u @ Wg.T) * (u @ W1.T)) @ W2
        return norm(h, last) @ embed.T

    first = run(prompt[None], keys, None)[0]
    for i in range(len(layers)):
        for b in range(1, rows):
            keys[i][b], vals[i][b] = keys[i][0], vals[i][0]
    return first, lambda tokens: run(tokens[:, None], keys, kept)[:, 0]


@pytest.mark.parametrize("dtype,rel", [(torch.float32, 2e-5), (torch.bfloat16, 4e-2)])
def test_continuations_of_a_prompt(dtype, rel):
    """fp32: products of up to 256 terms and a dozen operators on the way, 1e-6 each.  bf16: every operator rounds what it passes on (2^-8 of itself), some ten
    of them a layer in a random walk, two layers: 4e-2 of the largest logit is four times that."""
    ex = example()
    rows, steps, heads, kv_heads, dim, vocab = 3, 4, 4, 2, 64, 128
    w = ex.weights(2, 256, 512, heads, kv_heads, dim, vocab, dtype, seed=3)
    run = ex.Continuations(w, heads, kv_heads, dim, rows, 70, steps)
    rng = np.random.default_rng(5)
    prompt = rng.integers(0, vocab, 70)
    got = host(run.prompt(torch.from_numpy(prompt).cuda()))
    kept = [host(k).astype(int) for k in run.kept]
    assert all(len(k) == 256 and np.all(np.diff(k) > 0) for k in kept)
    first, more = reference(w, kept, prompt, rows, heads, kv_heads, dim, ex.EPS)
    assert np.abs(got - first).max() <= rel * np.abs(first).max()
    for i in range(steps):
        tokens = rng.integers(0, vocab, rows)
        got, ref = host(run.generate(torch.from_numpy(tokens).cuda())), more(tokens)
        assert np.abs(got - ref).max() <= rel * np.abs(ref).max(), i
    assert run.lens.tolist() == [steps] * rows
