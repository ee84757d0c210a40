"""Several continuations of one prompt through a stack of decoder layers whose feed-forward blocks are pruned by it.

The prompt goes through the full blocks once and leaves its keys and values in the cache; what its activations select is copied
into compact blocks.  Then all continuations generate together: they share the prompt's pages and the compact blocks, and have pages of their own for
what they add.  Norms and residual sums, the cache, the attention and the blocks are the library's; the projections are plain
products of PyTorch.  Weights are random, of the shape asked for.

    python examples/continue_prompt.py --layers 4 --prompt 512 --rows 16 --steps 64
"""
import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2404_01365_amd as G  # noqa: E402

EPS, PAGE = 1e-5, 64


def weights(layers, d, d_ff, heads, kv_heads, dim, vocab, dtype, seed=0):
    """Random weights: per layer norms, projections and the block's three matrices (neuron-major; W2p is W2 once more, by features)."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    normal = lambda *s, scale: (torch.randn(*s, generator=g, device="cuda") * scale).to(dtype)  # noqa: E731
    stack = []
    for _ in range(layers):
        w = dict(norm1=1 + normal(d, scale=0.1), norm2=1 + normal(d, scale=0.1), qkv=normal((heads + 2 * kv_heads) * dim, d, scale=d ** -0.5),
                 out=normal(d, heads * dim, scale=(heads * dim) ** -0.5), Wg=normal(d_ff, d, scale=d ** -0.5), W1=normal(d_ff, d, scale=d ** -0.5),
                 W2=normal(d_ff, d, scale=d_ff ** -0.5))
        w["W2p"] = w["W2"].t().contiguous()
        stack.append(w)
    return dict(layers=stack, embed=normal(vocab, d, scale=1.0), last=1 + normal(d, scale=0.1))


class Continuations:
    def __init__(self, w, heads, kv_heads, dim, rows, prompt_len, steps, keep=0.5):
        self.w, self.heads, self.kv_heads, self.dim, self.rows, self.prompt_len = w, heads, kv_heads, dim, rows, prompt_len
        self.steps, self.done = steps, 0                      # that there is room for; since the prompt
        dtype, dev = w["embed"].dtype, "cuda"
        self.d, d_ff = w["embed"].shape[1], w["layers"][0]["W1"].shape[0]
        self.k = G.griffin_k_from_fraction(d_ff, keep)
        self.blocks = [G.layer(x["W1"], x["W2"], x["Wg"], act=G.ACT_SILU) for x in w["layers"]]
        self.compact, self.kept = [], []
        # one table of pages for all layers, each with pools of its own: the prompt's pages first, then every row's
        up = lambda n: -(-n // PAGE)  # noqa: E731
        shared, own = up(prompt_len), up(steps)
        self.prefix_pages = torch.arange(shared, dtype=torch.int32, device=dev)
        self.pages = shared + torch.arange(rows * own, dtype=torch.int32, device=dev).view(rows, own)
        pools = lambda: torch.zeros(shared + rows * own, kv_heads, PAGE, dim, dtype=dtype, device=dev)  # noqa: E731
        self.caches = [G.kv_cache(pools(), pools()) for _ in w["layers"]]
        self.lens = torch.zeros(rows, dtype=torch.int32, device=dev)
        self.step = G.kv_batch(range(rows + 1), self.lens, self.pages, steps, prefix_pages=self.prefix_pages, n_prefix=prompt_len)
        rate = 10000.0 ** (-torch.arange(0, dim, 2, dtype=torch.float64, device=dev) / dim)
        angle = torch.arange(prompt_len + steps, dtype=torch.float64, device=dev)[:, None] * rate
        self.cos, self.sin = angle.cos().float(), angle.sin().float()
        # what follows a residual sum: the norm in front of the block, or of the next layer, or of the output
        nexts = [x["norm1"] for x in w["layers"][1:]] + [w["last"]]
        self.norm_in = G.norm(w["layers"][0]["norm1"], eps=EPS)
        self.norm_ff = [G.norm(x["norm2"], eps=EPS) for x in w["layers"]]
        self.norm_next = [G.norm(n, eps=EPS) for n in nexts]
        need = G.griffin_attention_workspace_bytes(self.caches[0], self.step, heads)
        self.ws_attention = torch.empty(max(need, 256), dtype=torch.uint8, device=dev)
        self.ws_block = torch.empty(G.griffin_decode_workspace_bytes(self.d, self.k, rows), dtype=torch.uint8, device=dev)

    def _attend(self, i, x, batch, workspace):
        """The attention of layer i: projections, cache, attention; returns what is added to the residual stream."""
        w, H, KV, D = self.w["layers"][i], self.heads, self.kv_heads, self.dim
        qkv = (x @ w["qkv"].t()).view(-1, H + 2 * KV, D)
        q, out = torch.empty_like(qkv[:, :H]), torch.empty(qkv.shape[0], H, D, dtype=x.dtype, device=x.device)
        G.griffin_kv_append(self.caches[i], batch, qkv[:, H:H + KV], qkv[:, H + KV:], q=qkv[:, :H], q_out=q, cos=self.cos, sin=self.sin)
        G.griffin_attention(self.caches[i], batch, q, out, workspace=workspace)
        return out.flatten(1) @ w["out"].t()

    def _stack(self, tokens, batch, workspace, block):
        h = self.w["embed"][tokens].float()                   # the residual stream stays in fp32
        x = torch.empty(h.shape, dtype=self.w["embed"].dtype, device=h.device)
        G.griffin_norm_residual(self.norm_in, h, None, None, x)
        for i in range(len(self.blocks)):
            y = self._attend(i, x, batch, workspace)
            G.griffin_norm_residual(self.norm_ff[i], h, y, h, x)
            G.griffin_norm_residual(self.norm_next[i], h, block(i, x), h, x)
        return x @ self.w["embed"].t()

    def prompt(self, tokens):
        """The prompt through the full blocks; fills the shared pages and selects and copies the neurons that generation keeps.  What an earlier prompt
        left, its blocks and its continuations' tokens, is dropped."""
        n = self.prompt_len
        self.compact, self.kept = [], []
        self.lens.zero_()
        self.done = 0
        batch = G.kv_batch([0, n], torch.zeros(1, dtype=torch.int32, device="cuda"), self.prefix_pages[None], n)
        need = G.griffin_attention_workspace_bytes(self.caches[0], batch, self.heads)
        ws_attention = torch.empty(max(need, 256), dtype=torch.uint8, device="cuda")
        ws = torch.empty(G.griffin_prompt_phase_workspace_bytes(self.blocks[0], n, 1), dtype=torch.uint8, device="cuda")

        def block(i, x):
            w, L, y = self.w["layers"][i], self.blocks[i], torch.empty_like(x)
            idx = torch.empty(1, self.k, dtype=torch.int32, device="cuda")
            G.griffin_prompt_phase(L, w["W2p"], x, [0, n], self.k, idx, y, workspace=ws)
            held = torch.empty(self.k, 3, self.d, dtype=x.dtype, device="cuda")
            C = G.layer(held[:, 1], held[:, 2], held[:, 0], act=G.ACT_SILU)
            G.griffin_compact(L, idx, self.k, C)
            self.compact.append(C)
            self.kept.append(idx[0])
            return y

        return self._stack(tokens, batch, ws_attention, block)

    def generate(self, tokens):
        """One token of every row in, the logits of the next out."""
        if self.done >= self.steps:
            raise ValueError("generate: the cache holds %d tokens a row" % self.steps)
        def block(i, x):
            y = torch.empty_like(x)
            G.griffin_ff_decode(self.compact[i], x, y, self.rows, workspace=self.ws_block)
            return y

        logits = self._stack(tokens, self.step, self.ws_attention, block)
        self.lens.add_(1)
        self.done += 1
        return logits


def main():
    a = argparse.ArgumentParser()
    for name, value in (("layers", 4), ("d", 4096), ("d-ff", 14336), ("heads", 32), ("kv-heads", 8), ("dim", 128), ("vocab", 2048),
                        ("prompt", 512), ("rows", 16), ("steps", 64)):
        a.add_argument("--" + name, type=int, default=value)
    a.add_argument("--dtype", choices=("bf16", "f32"), default="bf16")
    a = a.parse_args()
    w = weights(a.layers, a.d, a.d_ff, a.heads, a.kv_heads, a.dim, a.vocab, torch.bfloat16 if a.dtype == "bf16" else torch.float32)
    run = Continuations(w, a.heads, a.kv_heads, a.dim, a.rows, a.prompt, a.steps)
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    first = run.prompt(torch.randint(a.vocab, (a.prompt,), generator=g, device="cuda"))[-1].float()
    # every row draws its own first token from the prompt's last logits, then goes on with its likeliest
    tokens = torch.multinomial(torch.softmax(first, 0), a.rows, replacement=True, generator=g)
    torch.cuda.synchronize()
    t = time.perf_counter()
    for _ in range(a.steps):
        tokens = run.generate(tokens).argmax(dim=1)
    torch.cuda.synchronize()
    t = time.perf_counter() - t
    print("%d layers, prompt %d, %d rows: %.2f ms a step, %.0f tokens/s; last tokens %s"
          % (a.layers, a.prompt, a.rows, t / a.steps * 1e3, a.rows * a.steps / t, tokens[:8].tolist()))


if __name__ == "__main__":
    main()
