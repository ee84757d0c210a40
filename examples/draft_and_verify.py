"""Several continuations of one prompt in which pruned blocks draft tokens and full blocks verify them, over a cache of keys and values in 4 bits.

The prompt goes through the full blocks once, and what its activations select is copied into compact blocks, as in continue_prompt.py.  Then, round by round, every row
drafts a few tokens with the compact blocks, one step each; one step of the full blocks over all of a row's drafted tokens gives the target's probabilities behind each, and
griffin_verify_drafts keeps as many as leave the target's distribution as it is and draws the token behind them.  Draft and target share the cache: the target's step
writes its own keys and values over the draft's, and the places of dropped tokens are written again in the next round.  Weights are random, of the shape asked for.

    python examples/draft_and_verify.py --layers 4 --prompt 512 --rows 12 --drafts 4 --steps 64
"""
import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))

import paper_2404_01365_amd as G  # noqa: E402
from continue_prompt import EPS, PAGE, weights  # noqa: E402


class Speculation:
    def __init__(self, w, heads, kv_heads, dim, rows, prompt_len, steps, drafts, keep=0.5, group=32, seed=0):
        """steps: tokens that a row has room for; drafts: tokens drafted a round"""
        if rows * (drafts + 1) > G.MAX_BATCH:
            raise ValueError("%d rows of %d tokens are more than a block takes at a time" % (rows, drafts + 1))
        self.w, self.heads, self.kv_heads, self.dim, self.rows, self.prompt_len, self.drafts = w, heads, kv_heads, dim, rows, prompt_len, drafts
        dtype, dev = w["embed"].dtype, "cuda"
        self.vocab, self.d = w["embed"].shape
        d_ff = w["layers"][0]["W1"].shape[0]
        self.k = G.griffin_k_from_fraction(d_ff, keep)
        self.full = [G.layer(x["W1"], x["W2"], x["Wg"], act=G.ACT_SILU) for x in w["layers"]]
        self.compact = []
        up = lambda n: -(-n // PAGE)  # noqa: E731
        # a round may go past the last step that is asked for
        self.steps = steps
        self.room = room = steps + drafts + 1
        shared, own = up(prompt_len), up(room)
        self.prefix_pages = torch.arange(shared, dtype=torch.int32, device=dev)
        self.pages = shared + torch.arange(rows * own, dtype=torch.int32, device=dev).view(rows, own)
        size = G.griffin_kv_q4_page_bytes(kv_heads, dim, PAGE, group)
        pool = lambda: torch.zeros(shared + rows * own, size, dtype=torch.uint8, device=dev)  # noqa: E731
        self.caches = [G.kv_cache_q4(pool(), pool(), kv_heads=kv_heads, dim=dim, page_size=PAGE, group=group, dtype=dtype) for _ in w["layers"]]
        self.lens, self.ahead = (torch.zeros(rows, dtype=torch.int32, device=dev) for _ in range(2))
        batch = lambda n, lens: G.kv_batch(range(0, rows * n + 1, n), lens, self.pages, room, prefix_pages=self.prefix_pages, n_prefix=prompt_len)  # noqa: E731
        # a drafted token's lengths are the row's own and what was drafted before it
        self.one, self.several = batch(1, self.ahead), batch(drafts + 1, self.lens)
        self.ends_one, self.ends_several = (G.cu_seqlens(range(0, rows * n + 1, n)) for n in (1, drafts + 1))
        rate = 10000.0 ** (-torch.arange(0, dim, 2, dtype=torch.float64, device=dev) / dim)
        angle = torch.arange(prompt_len + room, dtype=torch.float64, device=dev)[:, None] * rate
        self.cos, self.sin = angle.cos().float(), angle.sin().float()
        nexts = [x["norm1"] for x in w["layers"][1:]] + [w["last"]]
        self.norm_in = G.norm(w["layers"][0]["norm1"], eps=EPS)
        self.norm_ff = [G.norm(x["norm2"], eps=EPS) for x in w["layers"]]
        self.norm_next = [G.norm(n, eps=EPS) for n in nexts]
        space = lambda n: torch.empty(max(n, 256), dtype=torch.uint8, device=dev)  # noqa: E731
        self.ws_attention = space(max(G.griffin_attention_q4_workspace_bytes(self.caches[0], b, heads) for b in (self.one, self.several)))
        self.ws_block = space(max(G.griffin_decode_workspace_bytes(self.d, n, r) for n, r in ((self.k, rows), (d_ff, rows * (drafts + 1)))))
        self.ws_verify = space(G.griffin_verify_workspace_bytes(rows, self.vocab))
        self.random = torch.Generator(device=dev)
        self.random.manual_seed(seed)

    def _attend(self, i, x, batch, workspace):
        w, H, KV, D = self.w["layers"][i], self.heads, self.kv_heads, self.dim
        qkv = (x @ w["qkv"].t()).view(-1, H + 2 * KV, D)
        q, out = torch.empty_like(qkv[:, :H]), torch.empty(qkv.shape[0], H, D, dtype=x.dtype, device=x.device)
        G.griffin_kv_append_q4(self.caches[i], batch, qkv[:, H:H + KV], qkv[:, H + KV:], q=qkv[:, :H], q_out=q, cos=self.cos, sin=self.sin)
        G.griffin_attention_q4(self.caches[i], batch, q, out, workspace=workspace)
        return out.flatten(1) @ w["out"].t()

    def _stack(self, tokens, batch, workspace, block):
        """Probabilities behind each of the tokens"""
        h = self.w["embed"][tokens].float()                   # the residual stream stays in fp32
        x = torch.empty(h.shape, dtype=self.w["embed"].dtype, device=h.device)
        G.griffin_norm_residual(self.norm_in, h, None, None, x)
        for i in range(len(self.full)):
            y = self._attend(i, x, batch, workspace)
            G.griffin_norm_residual(self.norm_ff[i], h, y, h, x)
            G.griffin_norm_residual(self.norm_next[i], h, block(i, x), h, x)
        return torch.softmax((x @ self.w["embed"].t()).float(), dim=1)

    def _decode(self, blocks):
        def block(i, x):
            y = torch.empty_like(x)
            G.griffin_ff_decode(blocks[i], x, y, x.shape[0], workspace=self.ws_block)
            return y
        return block

    def _uniform(self, n):
        return torch.rand(n, generator=self.random, device="cuda")

    def _draw(self, p):
        """One token of every row of probabilities: what verification draws where there is no draft"""
        tokens, kept = (torch.empty(self.rows, dtype=torch.int32, device="cuda") for _ in range(2))
        G.griffin_verify_drafts(self.ends_one, p, torch.zeros_like(tokens), self._uniform(self.rows), self._uniform(self.rows), tokens, kept, workspace=self.ws_verify)
        return tokens

    def prompt(self, tokens):
        """The prompt through the full blocks: fills the shared pages, copies the neurons that drafting keeps, and gives every row its first token"""
        n = self.prompt_len
        self.compact = []
        self.lens.zero_()
        batch = G.kv_batch([0, n], torch.zeros(1, dtype=torch.int32, device="cuda"), self.prefix_pages[None], n)
        need = G.griffin_attention_q4_workspace_bytes(self.caches[0], batch, self.heads)
        ws_attention = torch.empty(max(need, 256), dtype=torch.uint8, device="cuda")
        ws = torch.empty(G.griffin_prompt_phase_workspace_bytes(self.full[0], n, 1), dtype=torch.uint8, device="cuda")

        def block(i, x):
            w, L, y = self.w["layers"][i], self.full[i], torch.empty_like(x)
            idx = torch.empty(1, self.k, dtype=torch.int32, device="cuda")
            G.griffin_prompt_phase(L, w["W2p"], x, [0, n], self.k, idx, y, workspace=ws)
            held = torch.empty(self.k, 3, self.d, dtype=x.dtype, device="cuda")
            C = G.layer(held[:, 1], held[:, 2], held[:, 0], act=G.ACT_SILU)
            G.griffin_compact(L, idx, self.k, C)
            self.compact.append(C)
            return y

        p = self._stack(tokens, batch, ws_attention, block)
        return self._draw(p[-1:].expand(self.rows, -1).contiguous())

    def round(self, last):
        """From every row's last token: its new tokens [rows][drafts + 1] (-1 behind them), how many drafted ones were kept, and the last again"""
        R, K = self.rows, self.drafts
        if int(self.lens.max()) + K + 1 > self.room:
            raise ValueError("round: the cache holds %d tokens a row" % self.room)
        tokens = torch.zeros(R, K + 1, dtype=torch.int32, device="cuda")
        tokens[:, 0] = last
        draft_p = torch.empty(R, K + 1, self.vocab, device="cuda")          # a row's last probabilities are never read
        for i in range(K):
            torch.add(self.lens, i, out=self.ahead)
            draft_p[:, i] = self._stack(tokens[:, i].contiguous(), self.one, self.ws_attention, self._decode(self.compact))
            tokens[:, i + 1] = self._draw(draft_p[:, i].contiguous())
        p = self._stack(tokens.flatten(), self.several, self.ws_attention, self._decode(self.full))
        drafted = torch.cat([tokens[:, 1:], torch.full_like(tokens[:, :1], -1)], dim=1).flatten()
        out, kept = torch.empty_like(drafted), torch.empty(R, dtype=torch.int32, device="cuda")
        G.griffin_verify_drafts(self.ends_several, p, drafted, self._uniform(R * (K + 1)), self._uniform(R), out, kept, draft_p=draft_p.view(-1, self.vocab),
                                lens=self.lens, lens_out=self.lens, workspace=self.ws_verify)
        out = out.view(R, K + 1)
        return out, kept, out.gather(1, kept.long()[:, None])[:, 0]

    def generate(self, last):
        """Rounds until a row may have no room for another; the rows' tokens"""
        rows = [[int(t)] for t in last]
        while int(self.lens.max()) < self.steps:
            out, kept, last = self.round(last)
            for row, new, n in zip(rows, out.tolist(), kept.tolist()):
                row += new[:n + 1]
        return rows


def main():
    a = argparse.ArgumentParser()
    for name, value in (("layers", 4), ("d", 4096), ("d-ff", 14336), ("heads", 32), ("kv-heads", 8), ("dim", 128), ("vocab", 2048),
                        ("prompt", 512), ("rows", 12), ("drafts", 4), ("steps", 64)):
        a.add_argument("--" + name, type=int, default=value)
    a.add_argument("--keep", type=float, default=0.5)
    a.add_argument("--dtype", choices=("bf16", "f32"), default="bf16")
    a = a.parse_args()
    w = weights(a.layers, a.d, a.d_ff, a.heads, a.kv_heads, a.dim, a.vocab, torch.bfloat16 if a.dtype == "bf16" else torch.float32)
    run = Speculation(w, a.heads, a.kv_heads, a.dim, a.rows, a.prompt, a.steps, a.drafts, keep=a.keep)
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    last = run.prompt(torch.randint(a.vocab, (a.prompt,), generator=g, device="cuda"))
    torch.cuda.synchronize()
    t = time.perf_counter()
    rows = run.generate(last)
    t = time.perf_counter() - t
    n = sum(len(r) - 1 for r in rows)
    print("%d layers, prompt %d, %d rows, %d drafts a round: %d tokens in %.1f ms; first row %s"
          % (a.layers, a.prompt, a.rows, a.drafts, n, t * 1e3, rows[0][:10]))


if __name__ == "__main__":
    main()
