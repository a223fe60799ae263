"""Which kernels the 8-bit calls launch, on which grids, read off the library's host code without a GPU (see
test_launch_routes_host.py): both sides of every rule, and that no launch is larger than a grid may be."""
import json
import os
import shutil
import subprocess
import sys

import pytest

from tests import test_launch_routes_host as host


@pytest.fixture(scope="module")
def run(tmp_path_factory):
    if shutil.which("gcc") is None:
        pytest.skip("no gcc")
    so = str(tmp_path_factory.mktemp("rec") / "recorder.so")
    subprocess.run(["gcc", "-O1", "-shared", "-fPIC", os.path.join(host.HERE, "launch_recorder.c"), "-o", so], check=True)

    def calls(list_of_calls):
        r = subprocess.run([sys.executable, "-c", host.CHILD, so, host.LIB], input=json.dumps(list_of_calls), capture_output=True, text=True, timeout=120)
        assert r.returncode == 0, r.stderr
        out = []
        for line in r.stdout.splitlines():
            rc, launches = json.loads(line)
            out.append((rc, [(host.short(l.split()[0]), [int(v) for v in l.split()[1:]]) for l in launches]))
        return out
    return calls


def experts(P, H, E, I, lo=0, hi=None, K=1):
    at = lambda n: ["p", n << 40]
    i = lambda *vs: [["i", v] for v in vs]
    return ["moe_expert_group_forward_mx",
            i(lo, E if hi is None else hi) + [at(1), at(2), ["p", None]] + i(K) + [at(n) for n in range(3, 10)] + i(P, H, E, I) +
            [at(10), at(11), ["z", 2 * P * I + 256], ["p", None]]]


def rows(call, n, H, extra):
    at = lambda k: ["p", k << 42]
    if call == "moe_quantize_mx":
        return [call, [at(1), ["i", n], ["i", H], at(2), at(3), ["p", None]]]
    if call == "moe_residual_norm_mx":
        return [call, [at(1), at(2), at(3), ["i", n], ["i", H], ["f", 1e-6], at(4), at(5), at(6), at(7), ["p", None]]]
    E, K = extra
    return [call, [at(1), at(2), ["p", None], ["i", n], ["i", H], ["i", E], ["i", K], ["i", 0], ["i", 1], ["i", 1], ["i", 1], ["i", 0], ["f", 1.0],
                   at(3), at(4), ["p", None]]]


def in_bounds(launches):
    for name, (x, y, z, threads, lds) in launches:
        assert 0 < x and x * threads < 1 << 32 and y == z == 1 and lds <= 160 * 1024, (name, x, y, z, threads, lds)


STREAM = "expert_stream_mx_kernel"
TILES = {"gate/up": "expert_tile_mx_kernel<1,0>", "half": "expert_tile_mx_kernel<1,1>", "down": "expert_tile_mx_kernel<0,0>"}


@pytest.mark.parametrize("P,H,E,I,want", [
    (4, 2048, 60, 1408, [STREAM + "<1,4,1,2>", STREAM + "<1,2,0,2>"]),                # few workgroups: two stages, narrower blocks for down
    (8, 2048, 60, 1408, [STREAM + "<1,4,1,1>", STREAM + "<1,2,0,2>"]),
    (9, 2048, 60, 1408, [STREAM + "<1,4,1,1>", STREAM + "<1,4,0,1>"]),
    (720, 2048, 60, 1408, [STREAM + "<1,4,1,1>", STREAM + "<1,4,0,1>"]),              # 12 rows per expert
    (721, 2048, 60, 1408, [STREAM + "<2,4,1,1>", STREAM + "<2,4,0,1>"]),
    (1440, 2048, 60, 1408, [STREAM + "<2,4,1,1>", STREAM + "<2,4,0,1>"]),             # 24
    (1441, 2048, 60, 1408, [TILES["gate/up"], TILES["down"]]),
    (1441, 2112, 60, 1408, [TILES["half"], TILES["down"]]),                           # a contraction of half steps
    (9000, 448, 60, 1408, [STREAM + "<2,4,1,1>", TILES["down"]]),                       # contractions too short for tiles
    (9000, 512, 60, 448, [TILES["gate/up"], STREAM + "<2,4,0,1>"]),
    (65536, 2048, 60, 1408, [TILES["gate/up"], TILES["down"]]),
])
def test_kernels_of_the_expert_blocks(run, P, H, E, I, want):
    (rc, launches), = run([experts(P, H, E, I)])
    assert rc == 0 and [n for n, _ in launches] == want
    in_bounds(launches)
    # the block cut changes no kernel that changes bits: only the stages, and the width of down's blocks of columns, go by the block
    (rc, launches), = run([experts(P, H, E, I, 7, 11)])
    same = lambda names: [n.replace("<1,2,0,2>", "<1,4,0,1>").replace("<1,4,1,2>", "<1,4,1,1>") for n in names]
    assert rc == 0 and same([n for n, _ in launches]) == same(want)


def test_no_launch_is_larger_than_a_grid(run):
    limits = [experts((1 << 31) // 64 - 64, 64, 1, 64), experts((1 << 31) // 64 - 64, 64, 256, 64), experts((1 << 31) // 16384 - 64, 448, 1, 16384),
              experts((1 << 31) // 16384 - 64, 16384, 256, 512), experts((1 << 31) // 512 - 64, 512, 256, 512)]
    for rc, launches in run(limits):
        assert rc == 0 and len(launches) == 2
        in_bounds(launches)
    top = (1 << 31) - 1
    big = [rows("moe_quantize_mx", top, 64, None), rows("moe_quantize_mx", 5_000_000, 16384, None), rows("moe_residual_norm_mx", top, 64, None),
           rows("moe_route_scored", top, 64, (60, 4)), rows("moe_route_scored", top, 64, (256, 8))]
    for (rc, launches), n in zip(run(big), (8, 5, 256, 128, 128)):
        assert rc == 0 and len(launches) == n, len(launches)
        in_bounds(launches)


@pytest.mark.parametrize("T,E,want", [(1, 8, "<4,1>"), (4096, 64, "<4,1>"), (4097, 64, "<4,2>"), (13, 65, "<8,1>"), (13, 129, "<12,1>"), (5000, 256, "<16,2>")])
def test_kernels_of_the_gating(run, T, E, want):
    (rc, launches), = run([rows("moe_route_scored", T, 2048, (E, 4))])
    assert rc == 0 and [n for n, _ in launches] == ["route_scored_kernel" + want]
    in_bounds(launches)
