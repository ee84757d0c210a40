"""What the binding of the entry points around the block looks at before it hands addresses over (no GPU: nothing here is launched)."""
import pytest
import torch

import paper_2404_01365_amd as G


def t(*s, dtype=torch.float32):
    return torch.zeros(*s, dtype=dtype)


def i(*s):
    return torch.zeros(*s, dtype=torch.int32)


class OnCard:
    """A tensor that says it lies on a card: what the binding looks at, and no memory that could be read."""

    def __init__(self, like, device=0):
        self.like, self.device = like, device

    def __getattr__(self, name):
        return getattr(self.like, name)

    def get_device(self):
        return self.device


@pytest.fixture
def calls(monkeypatch):
    """The library's functions, replaced: a call that gets as far as that is noted and not made."""
    made = []

    class Lib:
        def __getattr__(self, name):
            return lambda *a: made.append(name) or G.OK

    monkeypatch.setattr(G, "lib", Lib())
    return made


def norm_call(w=0, h=0, y=0, h_out=0, x=0, gate=0):
    N = G.norm(OnCard(t(64), w), eps=1e-5)
    G.griffin_norm_residual(N, OnCard(t(2, 64), h), OnCard(t(2, 64), y), OnCard(t(2, 64), h_out), OnCard(t(2, 64), x), gate=OnCard(t(64), gate), stream=1)


def cache(K=0, V=0):
    return G.kv_cache(OnCard(t(9, 2, 16, 64), K), OnCard(t(9, 2, 16, 64), V))


def batch(lens=0, pages=0, prefix=0):
    return G.kv_batch([0, 1], OnCard(i(1), lens), OnCard(i(1, 2), pages), 20, prefix_pages=OnCard(i(1), prefix), n_prefix=16)


def append_call(k=0, v=0, q=0, q_out=0, cos=0, sin=0, pool=0, **kw):
    G.griffin_kv_append(cache(pool, pool), batch(**kw), OnCard(t(1, 2, 64), k), OnCard(t(1, 2, 64), v), q=OnCard(t(1, 4, 64), q), q_out=OnCard(t(1, 4, 64), q_out),
                        cos=OnCard(t(40, 32), cos), sin=OnCard(t(40, 32), sin), stream=1)


def attention_call(q=0, out=0, workspace=0, pool=0, **kw):
    G.griffin_attention(cache(pool, pool), batch(**kw), OnCard(t(1, 4, 64), q), OnCard(t(1, 4, 64), out), workspace=OnCard(t(4096, dtype=torch.uint8), workspace), stream=1)


@pytest.mark.parametrize("call,names", [
    (norm_call, ["w", "h", "y", "h_out", "x", "gate"]),
    (append_call, ["k", "v", "q", "q_out", "cos", "sin", "pool", "lens", "pages", "prefix"]),
    (attention_call, ["q", "out", "workspace", "pool", "lens", "pages", "prefix"]),
])
def test_tensors_that_are_not_on_the_card_are_refused(calls, call, names):
    call()
    assert len(calls) == 1
    for name in names:
        for device in (-1, 1):                                   # the host's memory, another card's
            with pytest.raises(ValueError, match="is on|lie on"):
                call(**{name: device})
    with pytest.raises(ValueError):                              # all of them on the host
        call(**dict.fromkeys(names, -1))
    call(**dict.fromkeys(names, 1))
    assert len(calls) == 2


def test_pools_of_one_cache_lie_on_one_card():
    with pytest.raises(ValueError):
        cache(V=-1)
    with pytest.raises(ValueError):
        cache(V=1)


def test_a_residual_sum_without_norms(calls):
    """No weights, so the card is the stream's."""
    N = G.norm(d=64, dtype=G.F32, eps=1e-5)
    for y, ok in ((1, True), (0, False), (-1, False)):
        if ok:
            G.griffin_norm_residual(N, OnCard(t(2, 64), 1), OnCard(t(2, 64), y), OnCard(t(2, 64), 1), stream=1)
        else:
            with pytest.raises(ValueError):
                G.griffin_norm_residual(N, OnCard(t(2, 64), 1), OnCard(t(2, 64), y), OnCard(t(2, 64), 1), stream=1)
    with pytest.raises(ValueError):
        G.griffin_norm_residual(N, t(2, 64), t(2, 64), t(2, 64), stream=1)
    assert len(calls) == 1


def test_a_workspace_has_no_gaps(calls):
    """Its size is what its elements take, so one element that is repeated is not a workspace."""
    C, B, q = cache(), batch(), OnCard(t(1, 4, 64))
    with pytest.raises(ValueError):
        G.griffin_attention(C, B, q, OnCard(t(1, 4, 64)), workspace=OnCard(t(1, dtype=torch.uint8).expand(4096)), stream=1)
    with pytest.raises(ValueError):
        G.griffin_attention(C, B, q, OnCard(t(1, 4, 64)), workspace=OnCard(t(4096, dtype=torch.uint8)[::2]), stream=1)
    assert not calls


def test_a_step_whose_bounds_were_raised_is_looked_at_as_it_is(calls):
    """max_len and n_prefix belong to the descriptor and may change from step to step: calls compare what is in it with the tables of pages."""
    q, ws = OnCard(t(1, 4, 64)), OnCard(t(4096, dtype=torch.uint8))
    C, B = cache(), batch()                                      # two pages of 16 tokens, one of the prefix
    run = (lambda: G.griffin_attention(C, B, q, OnCard(t(1, 4, 64)), workspace=ws, stream=1),
           lambda: G.griffin_kv_append(C, B, OnCard(t(1, 2, 64)), OnCard(t(1, 2, 64)), stream=1))
    for field, fits, too_many in (("max_len", (1, 32), 33), ("n_prefix", (0, 16), 17)):
        for call in run:
            for value in fits:
                setattr(B, field, value)
                call()
            setattr(B, field, too_many)
            with pytest.raises(ValueError, match="fewer pages"):
                call()
            setattr(B, field, fits[-1])
    assert len(calls) == 8
    C.dtype = G.BF16
    for call in run:
        with pytest.raises(TypeError):
            call()


def test_descriptors_that_are_filled_in_by_hand(calls):
    """Structures as the C header has them; tensors are then held against their fields."""
    N = G.griffin_norm()
    N.d, N.dtype, N.kind, N.eps, N.h_scale, N.y_scale, N.w_pre = 64, G.F32, G.NORM_RMS, 1e-5, 1.0, 1.0, 0x7F0000001000
    h = OnCard(t(2, 64))
    G.griffin_norm_residual(N, h, OnCard(t(2, 64)), h, OnCard(t(2, 64)), stream=1)
    with pytest.raises(ValueError):
        G.griffin_norm_residual(N, h, OnCard(t(2, 32)), h, OnCard(t(2, 64)), stream=1)
    with pytest.raises(TypeError):
        G.griffin_norm_residual(N, h, OnCard(t(2, 64).bfloat16()), h, OnCard(t(2, 64)), stream=1)
    C, B, made, step = G.griffin_kv_cache(), G.griffin_kv_batch(), cache(), batch()
    for mine, theirs in ((C, made), (B, step)):
        for name, _ in mine._fields_:
            setattr(mine, name, getattr(theirs, name))
    for c, b in ((C, B), (made, B), (C, step)):
        G.griffin_attention(c, b, OnCard(t(1, 4, 64)), OnCard(t(1, 4, 64)), workspace=OnCard(t(4096, dtype=torch.uint8)), stream=1)
        G.griffin_kv_append(c, b, OnCard(t(1, 2, 64)), OnCard(t(1, 2, 64)), stream=1)
        with pytest.raises(ValueError):
            G.griffin_attention(c, b, OnCard(t(2, 4, 64)), OnCard(t(2, 4, 64)), stream=1)
        with pytest.raises(ValueError):
            G.griffin_attention(c, b, OnCard(t(1, 4, 64), -1), OnCard(t(1, 4, 64), -1), stream=1)
    assert len(calls) == 7
