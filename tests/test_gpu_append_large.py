"""A step so large that its rotation goes out in more than one launch."""
import pytest
import torch

import paper_2404_01365_amd as G

pytestmark = pytest.mark.gpu


def test_append_in_two_launches():
    """2^20 tokens (256 sequences) of 590 query heads, of which one pair is rotated: 17 workgroups a token, 2^24 / 17 = 986895 tokens the first launch.  What is
    not rotated is copied bit by bit, on either side of the seam and at the ends; the pair is off by an fp32 product and sum and by its rounding (2^-8)."""
    tokens, heads, seqs, dim = 1 << 20, 590, 256, 8
    each, g = tokens // seqs, torch.Generator(device="cuda").manual_seed(3)
    qkv = torch.randn(tokens, heads + 2, dim, generator=g, device="cuda", dtype=torch.bfloat16)
    q, k, v = qkv[:, :heads], qkv[:, heads:heads + 1], qkv[:, heads + 1:]
    out = torch.zeros(tokens, heads, dim, device="cuda", dtype=torch.bfloat16)
    pool = [torch.zeros(tokens // 256, 1, 256, dim, device="cuda", dtype=torch.bfloat16) for _ in range(2)]
    pages = torch.arange(tokens // 256, device="cuda", dtype=torch.int32).view(seqs, -1)
    angle = torch.arange(each, device="cuda")[:, None] * 0.37
    G.griffin_kv_append(G.kv_cache(*pool), G.kv_batch(range(0, tokens + 1, each), torch.zeros(seqs, device="cuda", dtype=torch.int32), pages, each), k, v, q=q, q_out=out,
                        cos=angle.cos(), sin=angle.sin())
    assert torch.equal(out[..., 2:], q[..., 2:])
    assert torch.equal(pool[1].view(tokens, 1, dim), v) and torch.equal(pool[0].view(tokens, 1, dim)[..., 2:], k[..., 2:])
    c, s = (f(angle).repeat(seqs, 1) for f in (torch.cos, torch.sin))
    for at in (slice(0, 3), slice(986890, 986900), slice(tokens - 3, tokens)):
        for got, x in ((out[at], q[at]), (pool[0].view(tokens, 1, dim)[at], k[at])):
            a, b = x[..., 0].float(), x[..., 1].float()
            want = torch.stack([a * c[at] - b * s[at], b * c[at] + a * s[at]], -1)
            assert bool(((got[..., :2].float() - want).abs() <= 2.0 ** -8 * want.abs() + 1e-5).all())
