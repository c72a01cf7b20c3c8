"""Sums over a token's heads go through shared memory with a place for each warp of the thread block.  Where its warps are no multiple of a team's, those behind the last
team have no sums to read: the places that they would take lie past the array.  The plan compiled from its source, the reads counted: no device."""
import ctypes as C
import os
import re
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2604_10103_b200", "csrc")
KERNELS = open(os.path.join(CSRC, "k_heads.cuh")).read()


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    text = open(os.path.join(CSRC, "hf_heads.cu")).read()
    struct = text[text.index("struct HeadsPlan {"):text.index("hf_status heads_check")]
    body = text[text.index("HeadsPlan heads_plan("):text.index("// Backward: thread blocks for q, k, v")]
    d = tmp_path_factory.mktemp("plan")
    (d / "p.cpp").write_text(f'#include "{CSRC}/../../include/hf.h"\n' + struct + body + '''
extern "C" void plan(int type, int heads, int kv_heads, int head_dim, int wide, int* out) {
    hf_heads_shape g = {};
    g.type = type; g.heads = heads; g.kv_heads = kv_heads; g.head_dim = head_dim;
    const HeadsPlan n = heads_plan(&g, wide != 0);
    out[0] = n.threads / 32; out[1] = n.big;
    for (int i = 0; i < 3; ++i) { out[2 + i] = n.warps[i]; out[5 + i] = n.teams[i]; }
}
''')
    subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", str(d / "p.cpp"), "-o", str(d / "p.so")], check=True)
    lib = C.CDLL(str(d / "p.so"))

    def made(*args):
        out = (C.c_int * 8)()
        lib.plan(*args, out)
        return out[0], bool(out[1]), out[2:5], out[5:8]
    return made


def test_every_read_is_of_a_place_that_was_written(plan):
    function = KERNELS[KERNELS.index("void heads_team_sum("):]
    function = function[:function.index("\n}\n")]
    skips = re.search(r"__syncthreads\(\);\s*if \(team >= teams\) return;\s*", function) is not None
    assert skips and len(re.findall(r"heads_team_sum\(all, team, (?:p\.teams\[part\]|teams), team_warp, warps, s_sum", KERNELS)) == KERNELS.count("heads_team_sum(") - 1 == 3
    idle = 0
    for head_dim in (2, 8, 24, 64, 96, 128, 256):
        lanes = 1
        while 8 * lanes < head_dim:
            lanes *= 2
        most = min(2048, 2048 // lanes)
        for heads in {h for h in list(range(1, 140)) + [192, 255, 256, 500, 1000, 2047, 2048] if h <= most}:
            for kv_heads in range(1, heads + 1) if heads <= 140 else (1, heads // 3, heads):
                for type_, wide in ((0, 1), (2, 1), (0, 0)):
                    block, big, warps, teams = plan(type_, heads, kv_heads, head_dim, wide)
                    assert block <= (16 if big else 4)
                    for w, t in zip(warps, teams):
                        assert t >= 1 and w * t <= block < w * (t + 1)
                        written = set(range(block))                     # (team * warps + warp of the team: the warp's own place)
                        for team in range(-(-block // w)):
                            if skips and team >= t:
                                idle += 1
                                continue
                            assert {team * w + i for i in range(w)} <= written
    assert idle                                                         # (there are such warps)
