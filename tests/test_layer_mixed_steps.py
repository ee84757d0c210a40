"""Which steps read a shared prefix once for all rows, and which once a tile of a sequence's own rows (no GPU)."""
import pytest

from test_layer_routes import record, step  # noqa: F401  (record: a fixture)


def kinds(got):
    return ["join" if "join" in name else "tile" if "attend_tile_kernel" in name else "rows" for name, _ in got]


@pytest.mark.parametrize("call", [
    step(32, 8, 128, [1] * 47 + [17], 717, 32768), step(32, 8, 128, [1] * 47 + [17], 717, 2048),     # tiles of 4 rows of 256
    step(64, 8, 128, [9] * 17, 109, 8192), step(32, 8, 128, [20] * 20, 70, 8192),                     # a third full
    step(32, 32, 128, [70] * 8, 90, 8192), step(32, 8, 256, [1] * 30 + [40], 200, 4096),
])
def test_a_long_prefix_is_not_read_by_tiles_of_a_few_rows(record, call):  # noqa: F811
    (got,) = record([call])
    assert kinds(got) == ["tile", "join"], got
    # the prefix in chunks for as many workgroups as fill the chip, and not one workgroup a sequence
    per = 256 if call["dim"] <= 128 else 128
    group = call["heads"] // call["kv_heads"]
    own = call["kv_heads"] * sum(-(-n * group // per) for n in call["new"])
    rows = -(-sum(call["new"]) * group // per) * call["kv_heads"]
    assert got[0][1] >= own + 2 * rows, (got, own, rows)


@pytest.mark.parametrize("call", [
    step(32, 8, 128, [2048, 1117, 604, 381], 2048, 300), step(32, 8, 128, [2048, 1117, 604, 381], 2048, 32768),     # nearly full: whatever its length
    step(32, 8, 128, [3400], 3400, 8192), step(32, 8, 128, [300] * 4, 300, 32768),
    step(64, 8, 128, [9] * 17, 109, 300), step(32, 8, 128, [20] * 20, 70, 1024), step(32, 32, 128, [70] * 8, 90, 2048),     # short: a few more keys a tile
])
def test_full_tiles_and_short_prefixes_go_in_one_launch(record, call):  # noqa: F811
    (got,) = record([call])
    assert kinds(got) == ["tile"], got


def test_a_token_more_does_not_cost_a_prefix_more(record):  # noqa: F811
    """16 sequences of 9 tokens take tiles cut into chunks; so do 17, with work for about as many workgroups."""
    few, more = record([step(64, 8, 128, [9] * n, 109, 32768) for n in (16, 17)])
    assert kinds(few) == kinds(more) == ["tile", "join"]
    assert 0.5 * few[0][1] <= more[0][1] <= 2 * few[0][1]
