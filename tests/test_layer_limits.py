"""Sizes at the ends of what an attention takes, without a GPU: every call either launches work for all its rows and keys or is refused."""
import json
import os
import subprocess
import sys

import pytest

import launches
import paper_2404_01365_amd as G

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

CHILD = """
import ctypes, json, sys
shim = ctypes.CDLL(sys.argv[1])
sys.path.insert(0, sys.argv[2])
import launches
import paper_2404_01365_amd as G
import test_layer_abi_cpu as T
notes = (launches._Note * 64)()
for c in json.load(sys.stdin):
    seqs, new, dim, kvh, heads = c['seqs'], c['new'], c['dim'], c['kv_heads'], c['heads']
    C = T.mk_cache(dtype=c['dtype'], kv_heads=kvh, dim=dim, page_size=65536, page_stride=kvh * 65536 * dim, head_stride=65536 * dim, token_stride=dim)
    B = T.mk_batch(cu=[new * b for b in range(seqs + 1)], n_prefix=c['prefix'], max_len=c['max_len'], ld_pages=1 << 20)
    print(json.dumps(c), file=sys.stderr, flush=True)
    need = G.griffin_attention_workspace_bytes(C, B, heads)
    shim.shim_take(notes)
    rc = T.attend(C, B, heads=heads, ldq=dim, hsq=dim, ldo=dim, hso=dim, ws_bytes=need)
    print(json.dumps([rc, need, [(notes[i].name.decode(), notes[i].grid[0]) for i in range(shim.shim_take(notes))]]), flush=True)
"""


@pytest.fixture(scope="module")
def record(tmp_path_factory):
    tmp = tmp_path_factory.mktemp("shim")
    src, so = str(tmp / "shim.c"), str(tmp / "shim.so")
    open(src, "w").write(launches._SHIM)
    subprocess.check_call(["gcc", "-shared", "-fPIC", "-O1", src, "-o", so, "-ldl"])

    def run(calls, child=CHILD):
        env = dict(os.environ, LD_PRELOAD=":".join(filter(None, [so, os.environ.get("LD_PRELOAD")])), PYTHONPATH=ROOT)
        r = subprocess.run([sys.executable, "-c", child, so, os.path.join(ROOT, "tests")], input=json.dumps(calls), env=env, capture_output=True,
                           text=True, timeout=120)
        assert r.returncode == 0, (r.returncode, r.stderr.strip().splitlines()[-1])
        return [json.loads(line) for line in r.stdout.splitlines()]
    return run


def step(seqs, new, max_len, *, prefix=0, heads=32, kv_heads=8, dim=128, dtype=G.BF16):
    return dict(seqs=seqs, new=new, max_len=max_len, prefix=prefix, heads=heads, kv_heads=kv_heads, dim=dim, dtype=dtype)


def check(c, rc, need, got):
    """What a call that is taken launches: workgroups for every row, and a join of as many parts as the workspace holds."""
    assert rc == G.OK and got, (c, rc, got)
    rows = c["seqs"] * c["new"] * c["heads"]
    parts = need // (4 * rows * (c["dim"] + 2))
    assert need == parts * 4 * rows * (c["dim"] + 2) and parts != 1, (c, need)
    assert ("attend_join_kernel" in got[-1][0]) == (parts > 1), (c, got)
    work = [g for n, g in got if "join" not in n]
    # a workgroup takes no more than 256 rows, or eight items of 16
    assert work and min(work) > 0 and sum(work) * 256 >= rows * max(parts - 1, 1) and sum(work) < 1 << 23, (c, got)


EXTREME = [
    step(1, 2 ** 17, 2 ** 23, dtype=G.F32), step(1, 2 ** 18, 2 ** 22, dtype=G.F32), step(1, 2 ** 18, 2 ** 23, dtype=G.F32),
    step(1, 2 ** 18, 2 ** 18, prefix=2 ** 22, dtype=G.F32), step(1, 2 ** 18, 2 ** 30),
    step(32, 1, 2 ** 30, kv_heads=32), step(64, 1, 2 ** 30, kv_heads=32), step(256, 1, 2 ** 29), step(256, 1, 2 ** 30, kv_heads=32, dtype=G.F32),
    step(256, 20, 2 ** 30, kv_heads=32), step(256, 1, 2 ** 29, prefix=2 ** 29, kv_heads=32), step(1, 1, 1, prefix=2 ** 30 - 1),
    step(1, 1, 2 ** 30, heads=1, kv_heads=1, dim=8), step(256, 1, 16, prefix=2 ** 30 - 16, heads=1024, kv_heads=1024, dim=64),
    step(1, 2 ** 20 - 1, 2 ** 30, heads=8, kv_heads=8, dim=256), step(8, 2 ** 17, 2 ** 30, heads=1, kv_heads=1, dtype=G.F32),
    step(256, 8, 2 ** 30, heads=1024, kv_heads=1024, dim=8, dtype=G.F32),
]


def test_long_parts_of_many_rows_are_planned_in_64_bits(record):
    for c, (rc, need, got) in zip(EXTREME, record(EXTREME)):
        check(c, rc, need, got)


def test_a_query_of_sizes_that_are_not_taken_ends(record):
    calls = [step(1, 2 ** 20, 2 ** 21, dtype=G.F32), step(1, 2 ** 20, 2 ** 30, heads=1024, kv_heads=1024), step(256, 4096, 2 ** 30, heads=64, kv_heads=64)]
    for c, (rc, need, got) in zip(calls, record(calls)):
        assert rc == G.EUNSUPPORTED and not got, c


def test_a_longer_prefix_takes_no_more_workspace(record):
    """... nor more workgroups, up to the longest there is; every step launches something."""
    calls = [step(16, 1, 201, prefix=p) for p in (4096, 65536, 1 << 20, 1 << 25, (1 << 30) - 201)]
    found = record(calls)
    for c, one in zip(calls, found):
        check(c, *one)
    assert max(need for _, need, _ in found) <= 2 * min(need for _, need, _ in found)
    grids = [sum(g for n, g in got if "join" not in n) for _, _, got in found]
    assert max(grids) <= 2 * min(grids)


@pytest.mark.parametrize("dtype", [G.F32, G.BF16])
def test_rows_at_the_limits_of_an_attention(record, dtype):
    """tokens * n_heads < 2^24 and tokens * n_heads^2 < 2^32, as the header says; a query of more gives 0."""
    inside = [step(1, 2 ** 19 - 1, 2 ** 20, dtype=dtype), step(1, 2 ** 20, 2 ** 20, heads=15, kv_heads=15, dtype=dtype), step(256, 2047, 4096, dtype=dtype),
              step(5, 819, 1000, heads=1024, kv_heads=1024, dim=64, dtype=dtype), step(1, 4095, 2 ** 14, heads=1024, kv_heads=8, prefix=99, dtype=dtype)]
    outside = [step(1, 2 ** 19, 2 ** 20, dtype=dtype), step(1, 2 ** 20, 2 ** 20, heads=16, kv_heads=16, dtype=dtype), step(256, 2048, 4096, dtype=dtype),
               step(4, 1024, 1024, heads=1024, kv_heads=1024, dim=64, dtype=dtype), step(1, 4096, 2 ** 14, heads=1024, kv_heads=8, prefix=99, dtype=dtype)]
    found = record(inside + outside)
    for c, one in zip(inside, found):
        check(c, *one)
    for c, one in zip(outside, found[len(inside):]):
        assert one == [G.EUNSUPPORTED, 0, []], c


def test_the_header_names_these_limits():
    text = open(os.path.join(ROOT, "include", "griffin.h")).read()
    assert "tokens * n_heads < 2^24 and tokens * n_heads^2 < 2^32" in text


APPEND = """
import ctypes, json, sys
shim = ctypes.CDLL(sys.argv[1])
sys.path.insert(0, sys.argv[2])
import launches
import paper_2404_01365_amd as G
import test_layer_abi_cpu as T
notes = (launches._Note * 64)()
for c in json.load(sys.stdin):
    C = T.mk_cache(dtype=c['dtype'], kv_heads=c['kv_heads'], dim=c['dim'], page_stride=c['kv_heads'] * 16 * c['dim'], head_stride=16 * c['dim'], token_stride=c['dim'])
    B = T.mk_batch(cu=c['cu'], max_len=1 << 20, ld_pages=1 << 16)
    shim.shim_take(notes)
    d = c['dim']
    rc = T.append(C, B, ldk=d, hsk=d, ldv=d, hsv=d, ldq=d, hsq=d, ldo=d, hso=d, heads=c['heads'], rot=c['rot'], style=c['style'])
    print(json.dumps([rc, 0, [(notes[i].name.decode(), notes[i].grid[0]) for i in range(shim.shim_take(notes))]]), flush=True)
"""


def test_an_append_of_any_step_is_taken(record):
    """2^20 tokens and 1024 heads are all that limits a step: one that would need 2^24 workgroups or more is launched in parts."""
    form = lambda cu, heads, kv_heads, dim, rot, style, dtype=G.BF16: dict(cu=cu, heads=heads, kv_heads=kv_heads, dim=dim, rot=rot, style=style, dtype=dtype)  # noqa: E731
    calls = [form([0, 2 ** 19], 128, 128, 256, 256, 0), form([0, 2 ** 19], 1024, 1024, 256, 254, 0), form([0, 2 ** 18, 2 ** 19], 1024, 1024, 256, 2, 1, G.F32),
             form([0, 5, 2 ** 20], 32, 8, 128, 128, 0), form([0, 1], 1024, 1024, 256, 256, 0)]
    # items of a token: pieces of rotated heads (8, 1 and 2 features, both halves of a pair together) and of values, 256 a workgroup
    items = [256 * 16 + 128 * 32, 2048 * (127 + 2) + 1024 * 32, 2048 * 128 + 1024 * 32, 40 * 8 + 8 * 16, 2048 * 16 + 1024 * 32]
    for c, n, (rc, _, got) in zip(calls, items, record(calls, APPEND)):
        assert rc == G.OK and sum(g for _, g in got) == c["cu"][-1] * -(-n // 256), (c, rc, got)
        assert all("kv_append_kernel" in name and 0 < g < 1 << 24 for name, g in got) and len(got) < 60, got
