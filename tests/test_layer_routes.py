"""Which kernels an attention launches, and that none of the kernels around the block keeps registers in scratch (no GPU)."""
import json
import os
import re
import subprocess
import sys

import pytest

import launches
import test_kernel_resources as resources

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

CHILD = """
import ctypes, json, sys
shim = ctypes.CDLL(sys.argv[1])
sys.path.insert(0, sys.argv[2])
import launches
import paper_2404_01365_amd as G
import test_layer_abi_cpu as T
notes = (launches._Note * 64)()
out = []
for c in json.load(sys.stdin):
    cu = [0]
    for n in c['new']:
        cu.append(cu[-1] + n)
    dim, kvh = c['dim'], c['kv_heads']
    C = T.mk_cache(dtype=G.BF16 if c['bf16'] else G.F32, kv_heads=kvh, dim=dim, page_stride=kvh * 16 * dim, head_stride=16 * dim, token_stride=dim)
    B = T.mk_batch(cu=cu, n_prefix=c['prefix'], max_len=c['max_len'], ld_pages=1 << 20)
    need = G.griffin_attention_workspace_bytes(C, B, c['heads'])
    shim.shim_take(notes)
    assert T.attend(C, B, heads=c['heads'], ldq=dim, hsq=dim, ldo=dim, hso=dim, ws_bytes=need) == G.OK, c
    out.append([(notes[i].name.decode(), notes[i].grid[0]) for i in range(shim.shim_take(notes))])
json.dump(out, sys.stdout)
"""


@pytest.fixture(scope="module")
def record(tmp_path_factory):
    tmp = tmp_path_factory.mktemp("shim")
    src, so = str(tmp / "shim.c"), str(tmp / "shim.so")
    open(src, "w").write(launches._SHIM)
    subprocess.check_call(["gcc", "-shared", "-fPIC", "-O1", src, "-o", so, "-ldl"])

    def run(calls):
        env = dict(os.environ, LD_PRELOAD=":".join(filter(None, [so, os.environ.get("LD_PRELOAD")])), PYTHONPATH=ROOT)
        r = subprocess.run([sys.executable, "-c", CHILD, so, os.path.join(ROOT, "tests")], input=json.dumps(calls), env=env, capture_output=True,
                           text=True, timeout=120)
        assert r.returncode == 0, r.stderr[-2000:]
        return json.loads(r.stdout)
    return run


def step(heads, kv_heads, dim, new, max_len, prefix=0, bf16=True):
    return dict(heads=heads, kv_heads=kv_heads, dim=dim, new=new, max_len=max_len, prefix=prefix, bf16=bf16)


# a step and its launches: rows<rows of the prefix / 16, of own parts / 16, own parts a wavefront each>, tiles of many rows, the join
ROUTES = [
    (step(32, 32, 128, [1], 100), ["few"]),                                                  # a few steps are cheaper than a second launch
    (step(32, 32, 128, [1], 257), ["rows 1 1", "join"]),
    (step(8, 4, 64, [1, 1], 100, 150), ["few"]),                                        # ... the prefix ahead of own keys
    (step(32, 8, 128, [2048, 1117, 604, 381], 2048, 300), ["tile"]),
    (step(32, 8, 128, [1] * 16, 201, 2048), ["rows 2 1", "join"]),
    (step(40, 40, 128, [1] * 64, 121, 1024), ["rows 2 1 alone", "join"]),
    (step(32, 8, 128, [1] * 48, 701, 32768), ["tile and rows", "join"]),                  # 192 rows share the prefix
    (step(16, 16, 256, [1] * 5, 91, 1999), ["rows 1 1", "join"]),                            # wide heads go sixteen rows at a time
    (step(32, 8, 128, [2048, 1117, 604, 381], 2048), ["tile"]),
    (step(32, 8, 128, [20, 10], 40, 64), ["tile", "join"]),                                  # 80 rows: own parts and prefix in one launch
    (step(32, 8, 128, [8, 8], 40, 640), ["rows 2 1", "join"]),                               # 32 rows a sequence, 64 in all
    (step(4, 2, 64, [20, 10], 40, 640, bf16=False), ["rows 2 2", "join"]),
    (step(8, 4, 64, [500, 9], 600, 0, bf16=False), ["rows 2 2", "join"]),
    (step(32, 32, 64, [1500, 9], 1600, 0, bf16=False), ["rows 2 2"]),                        # long ones wait for each other: a workgroup each
    (step(32, 32, 64, [40] * 16, 250, 0, bf16=False), ["rows 2 2 alone"]),
    (step(32, 8, 128, [1] * 20, 60, 8000), ["rows 2 1", "join"]),                            # 80 rows: a prefix with too little for tiles ...
    (step(32, 8, 128, [1] * 20, 60, 30000), ["tile and rows", "join"]),                      # ... and one with enough
    (step(40, 20, 128, [1] * 64, 121, 8192), ["tile and rows alone", "join"]),
    (step(80, 10, 256, [1] * 9, 60, 30000), ["tile", "rows 1 1", "join"]),                   # heads whose rows need more registers than tiles leave
]


def test_routes_of_an_attention(record):
    for (call, want), got in zip(ROUTES, record([c for c, _ in ROUTES])):
        names = []
        for name, _ in got:
            m = re.search(r"attend_rows_kernelILb(\d)ELi(\d+)ELb(\d)ELi(\d)ELi(\d)ELb(\d)E", name)
            if m:
                assert m[1] == str(int(call["bf16"])) and m[3] == "1"
                names.append("rows %s %s%s" % (m[4], m[5], " alone" if m[6] == "1" else ""))
            elif "attend_tile_kernel" in name:
                names.append(("tile", "tile and rows", "tile and rows alone")[int(re.search(r"TileOwnE(\d)E", name)[1])])
            else:
                names.append(next((k for k in ("join", "few") if "attend_%s_kernel" % k in name), name))
        assert names == want, (call, names)


def test_launches_stay_in_proportion(record):
    """A longer prefix takes longer chunks, not more workgroups; a workspace does not grow with it."""
    grids = [sum(g for n, g in got if "join" not in n) for got in record([step(32, 8, 128, [1] * 16, 201, p) for p in (4096, 65536, 1 << 20)])]
    assert max(grids) <= 1.5 * 1024 and max(grids) <= 2 * min(grids)


def test_kernels_around_the_block_stay_out_of_scratch():
    """... but for a norm of rows wider than 16384; rows of the attention go two workgroups a CU up to 128 features (fp32: sixteen rows at a time)."""
    found = {n: k for n, k in resources.kernels().items() if re.search("attend_|kv_append_kernel|norm_residual_kernel", n)}
    assert len(found) >= 60
    for n, k in found.items():
        wide = re.search(r"norm_residual_kernelI\w*Li16ELi4E", n)
        assert k[".private_segment_fixed_size"] <= (128 if wide else 0), n
        m = re.search(r"attend_rows_kernelILb(\d)ELi(\d+)ELb\dELi(\d)E", n)
        if m and int(m[2]) <= 128 and (m[1] == "1" or m[2] == "64" or m[3] == "1"):
            assert k[".vgpr_count"] <= 256 and k[".group_segment_fixed_size"] <= 80 * 1024, n
        if "attend_tile_kernel" in n:
            assert k[".vgpr_count"] <= 256, n
