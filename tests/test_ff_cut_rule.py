"""The feed-forward's tiling rule, compiled from its source: numbers alone, no device."""
import ctypes as C
import os
import re
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2604_10103_b200", "csrc")
GATED, Y, DH, DX, DW = range(5)


@pytest.fixture(scope="module")
def rule(tmp_path_factory):
    text = open(os.path.join(CSRC, "hf_ff.cu")).read()
    body = text[text.index("struct Tiling {"):text.index("// One launch being put together")]
    d = tmp_path_factory.mktemp("rule")
    (d / "r.cpp").write_text("struct Device { int sm_count, pairs; };\n" + body + '''
extern "C" void cut(int sms, int pairs, const long long* sizes, int n, int segments, int which, int* out) {
    Size s[3];
    for (int i = 0; i < n; ++i) s[i] = {sizes[3 * i], sizes[3 * i + 1], sizes[3 * i + 2]};
    const Device d = {sms, pairs};
    const Tiling t = ff_tiling(&d, s, n, segments, (FfCut)which);
    out[0] = t.cg; out[1] = t.bn; out[2] = t.splits;
}
''')
    subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", str(d / "r.cpp"), "-o", str(d / "r.so")], check=True)
    lib = C.CDLL(str(d / "r.so"))

    def cut(which, sizes, segments=1, sms=148, pairs=74):
        flat = (C.c_longlong * (3 * len(sizes)))(*[v for s in sizes for v in s])
        out = (C.c_int * 3)()
        lib.cut(sms, pairs, flat, len(sizes), segments, which, out)
        return tuple(out)
    return cut


def sizes_of(which, M, K, N, O):
    return {GATED: [(M, N, K)], Y: [(M, O, N)], DH: [(M, N, O)], DX: [(M, K, N)], DW: [(N, K, M), (N, K, M), (O, N, M)]}[which]


@pytest.mark.parametrize("which", [GATED, Y, DH, DX, DW])
@pytest.mark.parametrize("pairs", [60, 74])
def test_every_cut_is_one_that_the_kernel_has(rule, which, pairs):
    for M in (1, 17, 77, 129, 300, 1000, 1560, 4680, 32760, 1 << 24):
        for K, N, O in ((8, 8, 8), (64, 1000, 64), (1536, 4096, 1536), (2048, 8192, 2048), (1 << 17, 8, 1 << 17)):
            cg, bn, splits = rule(which, sizes_of(which, M, K, N, O), 2 if which == DX else 1, pairs=pairs)
            assert cg in (1, 2) and bn % 32 == 0 and bn >= 64
            assert bn <= 256 or (which == DW and cg == 2 and bn == 512 and splits == 1)
            if which >= DH:
                assert bn % (64 * cg) == 0                          # boxes of 64 columns a thread block
            if which == GATED:
                assert bn % 64 == 0 and splits == 1
            if which == DH:
                assert splits == 1 and (cg == 2 or bn <= 128)       # four stages beside the staging
            # a part of the contraction is never empty
            blocks = min((s[2] + 63) // 64 for s in sizes_of(which, M, K, N, O)) * (2 if which == DX else 1)
            assert 1 <= splits <= 16 and (splits == 1 or blocks >= 4 * splits)


def test_what_was_measured_best_is_chosen(rule):
    """Width 1536, hidden 4096."""
    def best(which, M):
        return rule(which, sizes_of(which, M, 1536, 4096, 1536), 2 if which == DX else 1)
    assert best(GATED, 4680) == (2, 256, 1) and best(Y, 4680) == (2, 224, 1) and best(DX, 4680) == (2, 256, 1)
    assert best(DW, 4680) == (2, 512, 1) and best(DW, 32760) == (2, 512, 1) and best(DX, 1000) == (2, 256, 3)
    assert best(Y, 77)[2] > 1 and best(DX, 77)[2] > 1
