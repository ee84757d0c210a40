"""How long prompts over a cache in 4 bits are cut, as the workspace that they ask for tells (no GPU).  A launch takes 512 workgroups of tiles a round; rounds that hold fewer than one for
every tile there cannot be, and are not what others are compared with."""
import pytest

import paper_2404_01365_amd as G
from test_q4_abi_cpu import mk_batch, mk_cache


def parts(cu, held, heads=32, kv_heads=8, dim=128, prefix=0):
    B = mk_batch(cu, max_len=held + max(b - a for a, b in zip(cu, cu[1:])), n_prefix=prefix)
    need = G.griffin_attention_q4_workspace_bytes(mk_cache(kv_heads=kv_heads, dim=dim), B, heads)
    return max(1, need // (cu[-1] * heads * (dim + 2) * 4))


# a full round and a little more of another, each for all of the keys, would be twice the full one's time or next to it
@pytest.mark.parametrize("new,held,kw", [(2049, 30000, {}), (2100, 30000, {}), (2500, 30000, {}), (2100, 16000, {}), (2049, 60000, {}), (3500, 120000, {}), (4300, 30000, dict(heads=16, dim=64)),
                                         (1300, 30000, dict(dim=256)), (1100, 30000, dict(heads=64, kv_heads=64, dim=64))])
def test_prompts_of_more_tiles_than_a_round_are_cut_on_long_caches(new, held, kw):
    assert 2 <= parts((0, new), held, **kw) <= 8


@pytest.mark.parametrize("new,held,kw", [
    (2048, 30000, {}),                                # 512 tiles: a round that is full
    (2100, 4000, {}), (3000, 4000, {}), (3000, 8000, {}), (2500, 0, {}), (4096, 0, {}), (16000, 30000, {}), (2100, 8000, dict(kv_heads=32, dim=64))])
def test_prompts_that_are_quicker_whole_stay_whole(new, held, kw):
    assert parts((0, new), held, **kw) == 1


def test_tiles_of_a_shared_prefix_are_cut_alike():
    """256 sequences of nine tokens: 144 tiles of a prefix's rows, of 8 kv heads each; own parts beside them are few rows, which the device cuts"""
    cu = tuple(range(0, 256 * 9 + 1, 9))
    few = parts(cu, 100, prefix=3000)
    assert parts(cu, 100, prefix=30000) >= few + 2
