"""A cache of keys and values held in 4 bits and what goes with it where the pruned block drafts tokens and the full block verifies them, as timed cases: a
step's keys and values quantised on their way into the pages, reading them back, the attention over such a cache, and the verification of drafted tokens.

A case is a dict of plain values:
  op       append  griffin_kv_append_q4      rotated keys and values into 4-bit pages, rotated queries; the step's tokens are read back behind it
           read    griffin_kv_read_q4        keys and values of a run of tokens out of the pages
           attend  griffin_attention_q4      softmax(scale q k) v over a shared prefix and own tokens, all held in 4 bits
           verify  griffin_verify_drafts     the drafted tokens that the target's probabilities keep, and the token behind them
  append, read, attend:
           heads, kv_heads, dim, page, group (features that share a scale), prefix (tokens that all sequences share), own ("a+b+c": a sequence's
           tokens in the cache before the call), new ("a+b+c": its tokens in this call), dtype
  append:  rot (rotated dims), style ("half" or "pairs"), fused (q, k, v are slices of one product's output)
  verify:  vocab, rows ("a+b+c": a sequence's rows of probabilities, drafted tokens and one more), greedy (the draft has no probabilities)

What a page holds, for every kv head a block [page] rows of codes, 16 bytes for 32 features, then [page][groups] pairs (scale, middle) of fp16.  With lo and hi the
least and greatest of a group's values (cut to +-32768), scale = (hi - lo) / 15 and middle = lo + 8 scale, both in fp16, a value x has the code
c = round((x - middle) / scale) in -8 .. 7, kept as c + 8, of even features in the low half of a byte; it stands for middle + scale c in fp16.  A group with a value that is
not finite has a scale of NaN.
"""
import math

import torch

own = False


def _cached(op, name, heads, kv_heads, dim, *, page, group=32, prefix=0, held, new, dtype="bf16", **more):
    return dict(name=name, op=op, heads=heads, kv_heads=kv_heads, dim=dim, page=page, group=group, prefix=prefix, own=held, new=new, dtype=dtype, **more)


def _append(name, *shape, rot, style="half", fused=True, **kw):
    return _cached("append", name, *shape, rot=rot, style=style, fused=fused, **kw)


def _verify(name, vocab, rows, greedy=False):
    return dict(name=name, op="verify", vocab=vocab, rows=rows, greedy=greedy)


def _ramp(count, lo, hi):
    """count lengths from lo to hi in no particular order"""
    return "+".join(str(lo + (hi - lo) * ((7 * i + 3) % count) // max(1, count - 1)) for i in range(count))


def _each(count, value):
    return "+".join([str(value)] * count)


def listed():
    return [
        # one token of each of sixteen sequences of the Mistral-shaped layer: the smallest call, latency counts
        _append("append_mistral_16", 32, 8, 128, page=64, prefix=2048, held=_ramp(16, 0, 200), new=_each(16, 1), rot=128),
        # the prompts of a packed batch going into the cache, ragged, small pages, half of the dims rotated in pairs, wide groups
        _append("append_packed_7b", 32, 32, 128, page=16, group=64, held="0+0+33+0", new="2048+1117+604+381", rot=64, style="pairs"),
        # one conversation of the 7B-shaped layer read back, to go on in 16 bits
        _cached("read", "read_7b_chat", 32, 32, 128, page=16, held="0", new="777"),
        # a long document of the Mistral-shaped layer, read back whole
        _cached("read", "read_long", 32, 8, 128, page=128, group=64, held="0", new="32768"),
        # a single sequence on the 7B-shaped layer, no prefix: the commonest call of a chat
        _cached("attend", "attend_7b_row1", 32, 32, 128, page=16, held="2048", new="1"),
        # thirty-two conversations of 500 to 8000 tokens each, a token a sequence: what a cache in 4 bits is held for
        _cached("attend", "attend_mistral_own32", 32, 8, 128, page=64, held=_ramp(32, 500, 8000), new=_each(32, 1)),
        # four drafted tokens and one more of sixteen questions that a long document is asked
        _cached("attend", "attend_drafts_shared16", 32, 8, 128, page=128, group=64, prefix=32768, held=_ramp(16, 5, 700), new=_each(16, 5)),
        # packed prompts attending to themselves, ragged: the largest
        _cached("attend", "attend_prompt_packed", 32, 8, 128, page=64, held="0+0+0+0", new="2048+1117+604+381"),
        # a small fp32 layer whose prompts come in behind a shared instruction
        _cached("attend", "attend_small_f32", 8, 4, 64, page=16, prefix=301, held="0+17+64", new="64+5+33", dtype="f32"),
        # one sequence's four drafted tokens
        _verify("verify_one", 32000, "5"),
        # sixty-four sequences' drafts of one to eight tokens, some rejected at once
        _verify("verify_64", 128001, "+".join(str(2 + (5 * i) % 8) for i in range(64))),
        # sixteen drafts that were looked up in the prompt, so without probabilities of their own
        _verify("verify_lookup_16", 50257, _each(16, 9), greedy=True),
    ]


def draw(rng):
    """One more case of the same ranges: 1 to 64 sequences of 1 to 32 kv heads of 64 to 256 dims with prefixes of 0 to 32768 tokens and own parts up to
    8000, or prompts of up to 4096 tokens, one in six in fp32; vocabularies of 1000 to 150000 tokens with 1 to 9 rows a sequence."""
    log = lambda lo, hi: lo * (hi / lo) ** rng.random()  # noqa: E731
    op = rng.choice(["append", "read", "attend", "attend", "attend", "verify"])
    text = lambda v: "+".join(str(x) for x in v)  # noqa: E731
    seqs = int(log(1, 64.99))
    if op == "verify":
        rows = [rng.randint(1, 9) for _ in range(seqs)]
        c = _verify("", int(log(1000, 150000.99)), text(rows), rng.random() < 0.3)
        return {k: v for k, v in c.items() if k != "name"}
    dtype = "f32" if rng.random() < 1 / 6 else "bf16"
    kv_heads = rng.choice([1, 2, 4, 5, 8, 16, 32])
    members = rng.choice([g for g in (1, 1, 2, 4, 5, 7, 8) if g * kv_heads <= 40])
    dim = rng.choice([64, 80, 96, 128, 128, 128, 256])
    page = rng.choice([16, 16, 32, 64, 128, 256])
    width = members * kv_heads * dim
    if op == "read" or (op == "append" and rng.random() < 0.5) or (op == "attend" and rng.random() < 0.35):       # prompts
        seqs = min(seqs, 8)
        most = {"read": 3.3e7 / (kv_heads * dim), "append": 5e7 / ((members + 2) * kv_heads * dim), "attend": 4096.99}[op]
        total = int(log(seqs, max(seqs + 0.5, min(32768.99 if op == "read" else 4096.99, most) / (2 if dtype == "f32" else 1))))
        cuts = sorted(rng.randint(0, total) for _ in range(seqs - 1))
        new = [b - a for a, b in zip([0] + cuts, cuts + [total])]        # a sequence without new tokens among them
        held = [rng.choice([0, 0, rng.randint(1, 100)]) for _ in range(seqs)]
        prefix = 0 if rng.random() < 0.6 else int(log(1, 512.99))
    else:                                # generation: one token a sequence, at times a few (a draft to be verified)
        few = rng.random() < 0.35
        new = [rng.randint(1, 8) if few else 1 for _ in range(seqs)]
        longest = int(log(1, 8000.99))
        held = [rng.randint(0, longest) for _ in range(seqs)]
        prefix = 0 if rng.random() < 0.4 else int(log(1, min(32768.99, 4e9 / (sum(new) * width))))
    # what the largest listed cases compute and move is not passed
    while op == "attend" and 4 * width * sum(n * (prefix + h) + n * (n + 1) // 2 for n, h in zip(new, held)) > 4.6e10:
        new, prefix = [(n + 1) // 2 for n in new], prefix // 2
    while op != "read" and sum(held) * kv_heads * dim > 2.6e8:
        held = [h // 2 for h in held]
    kw = dict(page=page, group=rng.choice([32, 32, 64]), prefix=prefix, held=text(held), new=text(new), dtype=dtype)
    if op == "append":
        c = _append("", members * kv_heads, kv_heads, dim, rot=rng.choice([dim, dim, dim // 2, 0]), style=rng.choice(["half", "pairs"]),
                    fused=rng.random() < 0.7, **kw)
    else:
        c = _cached(op, "", members * kv_heads, kv_heads, dim, **kw)
    return {k: v for k, v in c.items() if k != "name"}


# ----------------------------------------------------------------------------------------------- inputs
def _type(text):
    return torch.bfloat16 if text == "bf16" else torch.float32


def _numbers(text):
    return [int(v) for v in text.split("+")]


def _generator(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 1000003 + 31)
    return g


def _row_bytes(case):
    return 16 * -(-case["dim"] // 32)


def _groups(case):
    return -(-case["dim"] // case["group"])


def _block_bytes(case):
    return case["page"] * (_row_bytes(case) + 4 * _groups(case))


def _parts(case, pool):
    """Codes [page][head][token][bytes] and (scale, middle) [page][head][token][group][2] of pages [page][bytes], as views"""
    x = pool.view(pool.shape[0], case["kv_heads"], -1)
    cut = case["page"] * _row_bytes(case)
    codes = x[:, :, :cut].unflatten(2, (case["page"], -1))
    return codes, x[:, :, cut:].view(torch.float16).unflatten(2, (case["page"], -1, 2))


def _plain_quantise(case, x):
    """Codes in bytes [..][row bytes] and (scale, middle) [..][group][2] of [..][dim] in 64 bits, as a value may lie next to the border of two codes"""
    dim, size, n = case["dim"], case["group"], _groups(case)
    fine = x.isfinite()
    x = x.clamp(-32768, 32768)
    if n * size > dim:                   # a last group of fewer features: one of them fills it up
        x, fine = (torch.cat([v, v[..., -1:].expand(*v.shape[:-1], n * size - dim)], dim=-1) for v in (x, fine))
    x, fine = x.unflatten(-1, (n, size)), fine.unflatten(-1, (n, size)).all(dim=-1)
    lo, hi = x.amin(dim=-1), x.amax(dim=-1)
    scale = torch.div(hi - lo, torch.full_like(hi, 15.0)).half()
    middle = (lo + 8 * scale.double()).half()
    step = scale.double()[..., None]
    code = ((x - middle.double()[..., None]) / torch.where(step > 0, step, 1.0)).round().clamp(-8, 7)
    code = torch.where(fine[..., None] & (step > 0), code, 0.0).to(torch.int16) + 8
    code = code.flatten(-2)[..., :dim]
    pad = 2 * _row_bytes(case) - dim
    if pad:
        code = torch.cat([code, code.new_zeros(*code.shape[:-1], pad)], dim=-1)
    code = (code[..., 0::2] + 16 * code[..., 1::2]).to(torch.uint8)
    pair = torch.stack([torch.where(fine, scale, math.nan), torch.where(fine, middle, 0.0)], dim=-1)
    return code, pair


def _plain_values(case, codes, pairs):
    """What they stand for, in 32 bits"""
    c = torch.stack([codes & 15, codes >> 4], dim=-1).flatten(-2)[..., :case["dim"]].float() - 8
    scale, middle = (pairs[..., i].float().repeat_interleave(case["group"], dim=-1)[..., :case["dim"]] for i in (0, 1))
    return (middle + scale * c).half().float()


def _cache_inputs(case, seed):
    """Pools with some more pages than are used, handed out in random order, of keys with a few channels that stand out; q such that some scores do."""
    g, t = _generator(case, seed), _type(case["dtype"])
    kvh, dim, page, prefix = case["kv_heads"], case["dim"], case["page"], case["prefix"]
    held, new = _numbers(case["own"]), _numbers(case["new"])
    total = sum(new)
    up = lambda v: -(-v // page)  # noqa: E731
    width = max(1, max(up(h + n) for h, n in zip(held, new)))
    need = up(prefix) + sum(up(h + n) for h, n in zip(held, new))
    n_pages = need + need // 8 + 1

    def normal(*shape, scale=1.0):
        return torch.randn(*shape, generator=g, device="cuda") * scale

    channel = 1 + 3 * (torch.rand(kvh, 1, dim, generator=g, device="cuda") < 0.04).float()
    pools = []
    for k in (channel, 1.0):
        pool = torch.empty(n_pages, kvh * _block_bytes(case), dtype=torch.uint8, device="cuda")
        codes, pairs = _parts(case, pool)
        some = max(1, (1 << 25) // (kvh * page * dim))
        for at in range(0, n_pages, some):
            c, pr = _plain_quantise(case, (normal(min(some, n_pages - at), kvh, page, dim) * k).double())
            codes[at:at + some], pairs[at:at + some] = c, pr
        pools.append(pool)
    order = torch.randperm(n_pages, generator=g, device="cuda").to(torch.int32)
    at = up(prefix)
    pages = torch.zeros(len(new), width, dtype=torch.int32, device="cuda")
    for b, (h, n) in enumerate(zip(held, new)):
        c = up(h + n)
        pages[b, :c] = order[at:at + c]
        at += c
    cu = [0]
    for n in new:
        cu.append(cu[-1] + n)
    st = dict(K=pools[0], V=pools[1], prefix_pages=order[:up(prefix)].clone(), pages=pages, held=held, new=new, cu=cu,
              lens=torch.tensor(held, dtype=torch.int32, device="cuda"), max_len=max(1, max(h + n for h, n in zip(held, new))))
    heads = case["heads"]
    if case["op"] == "attend":
        st["q"] = normal(total, heads, dim, scale=1.2).to(t)
        st["out"] = torch.zeros(total, heads, dim, dtype=t, device="cuda")
        return st
    st["k_out"], st["v_out"] = (torch.zeros(total, kvh, dim, dtype=t, device="cuda") for _ in range(2))
    if case["op"] == "read":
        return st
    if case["fused"]:                    # one product's output: a token's queries, keys and values side by side
        qkv = normal(total, heads + 2 * kvh, dim).to(t)
        st["q"], st["k"], st["v"] = qkv[:, :heads], qkv[:, heads:heads + kvh], qkv[:, heads + kvh:]
    else:
        st["q"], st["k"], st["v"] = normal(total, heads, dim).to(t), normal(total, kvh, dim).to(t), normal(total, kvh, dim).to(t)
    st["q_out"] = torch.zeros(total, heads, dim, dtype=t, device="cuda")
    st["cos"] = st["sin"] = None
    if case["rot"]:
        rate = 10000.0 ** (-torch.arange(0, case["rot"], 2, dtype=torch.float64, device="cuda") / case["rot"])
        angle = torch.arange(prefix + st["max_len"], dtype=torch.float64, device="cuda")[:, None] * rate
        st["cos"], st["sin"] = angle.cos().float(), angle.sin().float()
    return st


def _verify_inputs(case, seed):
    """A target's probabilities and a draft's that mostly agree with them, tokens drawn from the draft's, and the random numbers."""
    g = _generator(case, seed)
    rows, vocab = _numbers(case["rows"]), case["vocab"]
    total = sum(rows)
    logits = torch.randn(total, vocab, generator=g, device="cuda") * 2.5
    st = dict(p=torch.softmax(logits * 1.2, dim=1))
    near = torch.softmax(logits + 0.3 * torch.randn(total, vocab, generator=g, device="cuda"), dim=1)
    clock = torch.empty(total, vocab, device="cuda").exponential_(generator=g)
    st["drafted"] = (near / clock).argmax(dim=1).to(torch.int32)
    st["draft_p"] = None if case["greedy"] else near
    if case["greedy"]:                   # what was looked up is mostly what the target finds likeliest
        hit = torch.rand(total, generator=g, device="cuda") < 0.7
        st["drafted"] = torch.where(hit, st["p"].argmax(dim=1).to(torch.int32), st["drafted"])
    st["u"] = torch.rand(total, generator=g, device="cuda")
    st["r"] = torch.rand(len(rows), generator=g, device="cuda")
    cu = [0]
    for n in rows:
        cu.append(cu[-1] + n)
    st["cu"] = cu
    st["first"] = torch.tensor(cu[:-1], device="cuda")
    st["rows"] = torch.tensor(rows, device="cuda")
    st["most"] = max(rows)
    st["lens"] = torch.randint(0, 4000, (len(rows),), generator=g, device="cuda").to(torch.int32)
    st["tokens"] = torch.zeros(total, dtype=torch.int32, device="cuda")
    st["accepted"], st["lens_out"] = torch.zeros_like(st["lens"]), torch.zeros_like(st["lens"])
    return st


def prepare(case, seed):
    st = (_verify_inputs if case["op"] == "verify" else _cache_inputs)(case, seed)
    st["case"] = case
    if not own:
        return st
    import paper_2404_01365_amd as G
    if case["op"] == "verify":
        st["ws"] = torch.empty(max(256, G.griffin_verify_workspace_bytes(len(st["cu"]) - 1, case["vocab"])), dtype=torch.uint8, device="cuda")
        st["cu"] = G.cu_seqlens(st["cu"])
        return st
    st["C"] = G.kv_cache_q4(st["K"], st["V"], kv_heads=case["kv_heads"], dim=case["dim"], page_size=case["page"], group=case["group"],
                            dtype=_type(case["dtype"]))
    st["B"] = G.kv_batch(st["cu"], st["lens"], st["pages"], st["max_len"], prefix_pages=st["prefix_pages"], n_prefix=case["prefix"])
    if case["op"] == "attend":
        size = G.griffin_attention_q4_workspace_bytes(st["C"], st["B"], case["heads"])
        st["ws"] = torch.empty(max(int(size), 256), dtype=torch.uint8, device="cuda")
    return st


# ----------------------------------------------------------------------------------------------- the passes
def _plain_rotate(case, x, cos, sin):
    r = case["rot"]
    if r == 0:
        return x
    a, b = (x[..., :r // 2], x[..., r // 2:r]) if case["style"] == "half" else (x[..., 0:r:2], x[..., 1:r:2])
    cos, sin = cos.to(x.dtype), sin.to(x.dtype)
    a, b = a * cos - b * sin, b * cos + a * sin
    turned = torch.cat([a, b], dim=-1) if case["style"] == "half" else torch.stack([a, b], dim=-1).flatten(-2)
    return torch.cat([turned, x[..., r:]], dim=-1)


def _places(case, st):
    """Page and slot of each of the step's tokens, and its place among its sequence's own"""
    dev, page = st["lens"].device, case["page"]
    seq = torch.repeat_interleave(torch.arange(len(st["new"]), device=dev), torch.tensor(st["new"], device=dev), output_size=st["cu"][-1])
    slot = st["lens"].long()[seq] + torch.arange(st["cu"][-1], device=dev) - torch.tensor(st["cu"][:-1], device=dev)[seq]
    return st["pages"].long()[seq, slot // page], slot % page, slot


def _plain_read(case, st, where, at):
    for pool, out in ((st["K"], st["k_out"]), (st["V"], st["v_out"])):
        codes, pairs = _parts(case, pool)
        out.copy_(_plain_values(case, codes[where, :, at], pairs[where, :, at]))
    return {"k": st["k_out"], "v": st["v_out"]}


def _plain_append(case, st):
    where, at, slot = _places(case, st)
    cos = sin = None
    if case["rot"]:
        cos, sin = (v[case["prefix"] + slot][:, None] for v in (st["cos"], st["sin"]))
    for pool, x in ((st["K"], _plain_rotate(case, st["k"].double(), cos, sin)), (st["V"], st["v"].double())):
        codes, pairs = _parts(case, pool)
        codes[where, :, at], pairs[where, :, at] = _plain_quantise(case, x)
    st["q_out"].copy_(_plain_rotate(case, st["q"].float(), cos, sin))
    return {"q": st["q_out"], **_plain_read(case, st, where, at)}


def _rows_of(case, pool, pages):
    """Pages [..] of a pool: [..][head][token][dim] in 32 bits"""
    codes, pairs = _parts(case, pool)
    return _plain_values(case, codes[pages.long()], pairs[pages.long()])


def _plain_attend(case, st):
    kvh, dim, prefix = case["kv_heads"], case["dim"], case["prefix"]
    group, scale = case["heads"] // kvh, dim ** -0.5
    q = st["q"].float().view(-1, kvh, group, dim).permute(1, 0, 2, 3)       # [kv head][token][member of the group][dim]
    out = st["out"]
    if prefix:
        pk, pv = (_rows_of(case, st[x], st["prefix_pages"]).transpose(0, 1).flatten(1, 2)[:, :prefix] for x in "KV")
        # the prefix's part of every row's scores in one product, then joined with the row's own part
        shared = torch.matmul(q.reshape(kvh, -1, dim), pk.transpose(1, 2)).mul_(scale).view(kvh, -1, group, prefix)
    if min(st["new"]) == max(st["new"]):
        # as many new tokens each: all own parts at once, padded to the longest
        seqs, n = len(st["new"]), st["new"][0]
        k, v = (_rows_of(case, st[x], st["pages"]).transpose(1, 2).flatten(2, 3) for x in "KV")            # [sequence][kv head][slot][dim]
        rows = q.reshape(kvh, seqs, n * group, dim).transpose(0, 1)
        s = torch.matmul(rows, k.transpose(2, 3).contiguous()).mul_(scale).view(seqs, kvh, n, group, -1)
        last = st["lens"][:, None] + torch.arange(n, device=q.device)
        s.masked_fill_((torch.arange(k.shape[2], device=q.device) > last[..., None])[:, None, :, None], -math.inf)
        if prefix:
            shared = shared.view(kvh, seqs, n, group, prefix).transpose(0, 1)
            s = torch.cat([shared, s], dim=-1)
        p = (s - s.amax(dim=-1, keepdim=True)).exp_()
        o = torch.matmul(p[..., prefix:].reshape(seqs, kvh, n * group, -1), v)
        if prefix:
            o += torch.matmul(p[..., :prefix].transpose(0, 1).reshape(kvh, -1, prefix), pv).view(kvh, seqs, n * group, dim).transpose(0, 1)
        o = o.view(seqs, kvh, n, group, dim) / p.sum(dim=-1, keepdim=True)
        out.copy_(o.permute(0, 2, 1, 3, 4).reshape(out.shape))
        return {"out": out}
    for b, (held, n) in enumerate(zip(st["held"], st["new"])):
        if n == 0:
            continue
        rows = slice(st["cu"][b], st["cu"][b + 1])
        used = st["pages"][b, :-(-(held + n) // case["page"])]
        k, v = (_rows_of(case, st[x], used).transpose(0, 1).flatten(1, 2)[:, :held + n] for x in "KV")
        s = torch.matmul(q[:, rows].reshape(kvh, -1, dim), k.transpose(1, 2)).mul_(scale).view(kvh, n, group, held + n)
        if n > 1:
            later = torch.arange(held + n, device=q.device)[None] > held + torch.arange(n, device=q.device)[:, None]
            s.masked_fill_(later[None, :, None], -math.inf)
        if prefix:
            s = torch.cat([shared[:, rows], s], dim=-1)
            v = torch.cat([pv, v], dim=1)
        p = (s - s.amax(dim=-1, keepdim=True)).exp_()
        o = torch.matmul(p.view(kvh, n * group, -1), v).view(kvh, n, group, dim) / p.sum(dim=-1, keepdim=True)
        out[rows] = o.permute(1, 0, 2, 3).reshape(n, -1, dim).to(out.dtype)
    return {"out": out}


def _plain_verify(case, st):
    p, q, first, rows, vocab = st["p"], st["draft_p"], st["first"], st["rows"], case["vocab"]
    i = torch.arange(st["most"], device=p.device)
    at = (first[:, None] + i).clamp(max=p.shape[0] - 1)
    token = st["drafted"].long()[at]
    by = 1.0 if q is None else q[at, token]
    kept = (i < rows[:, None] - 1) & (st["u"][at] * by < p[at, token])
    accepted = kept.long().cumprod(dim=1).sum(dim=1)
    row = first + accepted
    weight = p[row]
    refused = (accepted < rows - 1)[:, None]
    if q is None:                        # the draft had all its weight on one token
        rest = weight.scatter(1, token.gather(1, accepted[:, None]), 0.0)
    else:
        rest = (weight - q[row]).clamp(min=0)
    rest = torch.where(refused, rest, weight)
    rest = torch.where(rest.amax(dim=1, keepdim=True) > 0, rest, weight)
    total = rest.double().cumsum(dim=1)
    drawn = (total <= st["r"].double()[:, None] * total[:, -1:]).sum(dim=1).clamp(max=vocab - 1)
    out = torch.where(i < accepted[:, None], token, torch.where(i == accepted[:, None], drawn[:, None], -1))
    inside = i < rows[:, None]
    st["tokens"].copy_(out[inside])
    st["accepted"].copy_(accepted)
    st["lens_out"].copy_(st["lens"] + accepted + 1)
    return {"tokens": st["tokens"], "accepted": st["accepted"], "lens": st["lens_out"]}


def run(st):
    case = st["case"]
    op = case["op"]
    if not own:
        if op == "read":
            return _plain_read(case, st, *_places(case, st)[:2])
        return (_plain_append if op == "append" else _plain_attend if op == "attend" else _plain_verify)(case, st)
    import paper_2404_01365_amd as G
    if op == "append":
        G.griffin_kv_append_q4(st["C"], st["B"], st["k"], st["v"], q=st["q"], q_out=st["q_out"], cos=st["cos"], sin=st["sin"],
                               style=G.ROT_HALF if case["style"] == "half" else G.ROT_PAIRS)
        G.griffin_kv_read_q4(st["C"], st["B"], st["k_out"], st["v_out"])
        return {"q": st["q_out"], "k": st["k_out"], "v": st["v_out"]}
    if op == "read":
        G.griffin_kv_read_q4(st["C"], st["B"], st["k_out"], st["v_out"])
        return {"k": st["k_out"], "v": st["v_out"]}
    if op == "attend":
        G.griffin_attention_q4(st["C"], st["B"], st["q"], st["out"], scale=case["dim"] ** -0.5, workspace=st["ws"])
        return {"out": st["out"]}
    G.griffin_verify_drafts(st["cu"], st["p"], st["drafted"], st["u"], st["r"], st["tokens"], st["accepted"], draft_p=st["draft_p"], lens=st["lens"],
                            lens_out=st["lens_out"], workspace=st["ws"])
    return {"tokens": st["tokens"], "accepted": st["accepted"], "lens": st["lens_out"]}


def work(case):
    if case["op"] == "verify":
        rows, vocab = _numbers(case["rows"]), case["vocab"]
        # a drafted token is one number a row of each; whole rows are read where a token is drawn
        whole = len(rows) * vocab * (1 if case["greedy"] else 2)
        return {"bytes": 4 * (whole + 5 * sum(rows) + 4 * len(rows)), "flops": 2.0 * whole}
    es = 2 if case["dtype"] == "bf16" else 4
    held, new = _numbers(case["own"]), _numbers(case["new"])
    total, heads, kvh, dim, prefix = sum(new), case["heads"], case["kv_heads"], case["dim"], case["prefix"]
    key = kvh * (dim / 2 + 4 * _groups(case))                    # bytes of a token's keys, or values
    tables = sum(-(-(h + n) // case["page"]) for h, n in zip(held, new)) + -(-prefix // case["page"])
    if case["op"] == "read":
        return {"bytes": total * (2 * key + 2 * es * kvh * dim) + 4 * (tables + len(new)), "flops": 4.0 * total * kvh * dim}
    if case["op"] == "append":
        # queries, keys and values in, queries and codes out; codes in, keys and values out
        return {"bytes": es * total * (2 * heads + 2 * kvh) * dim + 4 * total * case["rot"] + total * (4 * key + 2 * es * kvh * dim) + 4 * (tables + len(new)),
                "flops": total * (3.0 * (heads + kvh) * case["rot"] + 14.0 * kvh * dim)}
    keys = prefix + sum(h + n for h, n in zip(held, new) if n)
    seen = sum(n * (prefix + h) + n * (n + 1) // 2 for h, n in zip(held, new))
    return {"bytes": 2 * es * total * heads * dim + 2 * key * keys + 4 * (tables + len(new)), "flops": 4.0 * dim * heads * seen}


# ----------------------------------------------------------------------------------------------- in 64 bits
def _exact_rows(case, pool, head, pages, slots):
    """Values [place][dim] of a kv head at pages and slots, from the pool's bytes"""
    size = _block_bytes(case)
    blocks = pool.view(pool.shape[0], case["kv_heads"], size)[:, head]
    out = torch.empty(len(slots), case["dim"], dtype=torch.float64, device=pool.device)
    rb, n = _row_bytes(case), _groups(case)
    f = torch.arange(case["dim"], device=pool.device)
    if len(slots) == 0:
        return out
    byte = blocks[pages[:, None], slots[:, None] * rb + f // 2].long()
    code = torch.where(f % 2 == 0, byte % 16, byte // 16).double() - 8
    at = case["page"] * rb + 4 * (slots[:, None] * n + f // case["group"])
    half = lambda o: torch.stack([blocks[pages[:, None], at + o], blocks[pages[:, None], at + o + 1]], dim=-1).view(torch.float16)[..., 0].double()  # noqa: E731
    return (half(2) + half(0) * code).to(torch.float16).double()


def _exact_quantised(case, x):
    """What values in 64 bits come back as: group by group, from the definition"""
    out = torch.empty_like(x)
    for a in range(0, case["dim"], case["group"]):
        y = x[..., a:a + case["group"]]
        lo, hi = torch.aminmax(y.clip(-32768, 32768), dim=-1, keepdim=True)
        scale = ((hi - lo) / 15).to(torch.float16).double()
        middle = (lo + scale * 8).to(torch.float16).double()
        code = torch.where(scale > 0, torch.round((y - middle) / scale), 0.0).clip(-8, 7)
        out[..., a:a + case["group"]] = (middle + code * scale).to(torch.float16).double()
    return out


def exact(case, seed):
    if case["op"] == "verify":
        st = {k: v.cpu() if torch.is_tensor(v) else v for k, v in _verify_inputs(case, seed).items()}
        tokens, accepted = [], []
        for b, (lo, hi) in enumerate(zip(st["cu"], st["cu"][1:])):
            row = lo
            while row < hi - 1:
                d = int(st["drafted"][row])
                share = 1.0 if st["draft_p"] is None else float(st["draft_p"][row, d])
                if not float(st["u"][row]) * share < float(st["p"][row, d]):
                    break
                tokens.append(d)
                row += 1
            weight = st["p"][row].double()
            if row < hi - 1:
                if st["draft_p"] is None:
                    weight[int(st["drafted"][row])] = 0
                else:
                    weight = torch.relu(weight - st["draft_p"][row].double())
            goal = float(st["r"][b]) * float(weight.sum())
            tokens.append(int(torch.searchsorted(weight.cumsum(0), goal, right=True)))
            tokens += [-1] * (hi - 1 - row)
            accepted.append(row - lo)
        a = torch.tensor(accepted, dtype=torch.int32)
        return {"tokens": torch.tensor(tokens, dtype=torch.int32).cuda(), "accepted": a.cuda(), "lens": (st["lens"] + a + 1).cuda()}
    st = _cache_inputs(case, seed)
    page, prefix, kvh, dim = case["page"], case["prefix"], case["kv_heads"], case["dim"]
    dev = st["K"].device
    if case["op"] == "read":
        out = {x: torch.empty(st["cu"][-1], kvh, dim, dtype=torch.float64, device=dev) for x in "kv"}
        for b, (held, n) in enumerate(zip(st["held"], st["new"])):
            slot = torch.arange(held, held + n, device=dev)
            where = st["pages"][b][slot // page].long()
            for hk in range(kvh):
                for x, pool in (("k", st["K"]), ("v", st["V"])):
                    out[x][st["cu"][b]:st["cu"][b + 1], hk] = _exact_rows(case, pool, hk, where, slot % page)
        return out
    if case["op"] == "append":
        k, q = st["k"].double().clone(), st["q"].double().clone()
        r = case["rot"]
        if r:
            slot = torch.cat([torch.arange(h, h + n, device=dev) for h, n in zip(st["held"], st["new"])])
            # as a complex number times e^(i angle), pair by pair
            turn = torch.complex(st["cos"].double(), st["sin"].double())[prefix + slot][:, None]
            lo = torch.arange(r // 2, device=dev) if case["style"] == "half" else torch.arange(0, r, 2, device=dev)
            hi = lo + (r // 2 if case["style"] == "half" else 1)
            for x in (k, q):
                z = torch.complex(x[:, :, lo], x[:, :, hi]) * turn
                x[:, :, lo], x[:, :, hi] = z.real, z.imag
        return {"q": q, "k": _exact_quantised(case, k), "v": _exact_quantised(case, st["v"].double())}
    heads = case["heads"]
    group = heads // kvh
    out = torch.zeros(st["q"].shape, dtype=torch.float64, device=dev)
    at = torch.arange(prefix, device=dev)
    for hk in range(kvh):
        before = [_exact_rows(case, pool, hk, st["prefix_pages"][at // page].long(), at % page) for pool in (st["K"], st["V"])]
        for b, (held, n) in enumerate(zip(st["held"], st["new"])):
            if n == 0:
                continue
            own_at = torch.arange(held + n, device=dev)
            where = st["pages"][b][own_at // page].long()
            k, v = (torch.cat([x, _exact_rows(case, pool, hk, where, own_at % page)]) for x, pool in zip(before, (st["K"], st["V"])))
            position = torch.cat([torch.full((prefix,), -1, device=dev), own_at])
            for g in range(group) if n > 64 else [slice(0, group)]:
                # many rows go head by head, a few all members of the group at once
                qs = st["q"][st["cu"][b]:st["cu"][b + 1], hk * group:(hk + 1) * group].double()
                qs = qs[:, g] if n > 64 else qs.reshape(-1, dim)
                logits = qs @ k.t() / math.sqrt(dim)
                i = torch.arange(n, device=dev) if n > 64 else torch.arange(n, device=dev).repeat_interleave(group)
                logits = torch.where(position[None] <= held + i[:, None], logits, -math.inf)
                o = torch.softmax(logits, dim=1) @ v
                if n > 64:
                    out[st["cu"][b]:st["cu"][b + 1], hk * group + g] = o
                else:
                    out[st["cu"][b]:st["cu"][b + 1], hk * group:(hk + 1) * group] = o.view(n, group, dim)
    return {"out": out}
