"""How layer norm's backward pass is cut, compiled from its source: the plan and the kernel that the dispatch launches for it agree, at every
width, type and alignment.  Numbers alone, no device."""
import ctypes as C
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2604_10103_b200", "csrc")
SMEM, SMS = 232448, 148


def between(text, first, last):
    return text[text.index(first):text.index(last)]


@pytest.fixture(scope="module")
def rules(tmp_path_factory):
    host, kernel = (open(os.path.join(CSRC, f)).read() for f in ("hf_layers.cu", "k_norm.cuh"))
    d = tmp_path_factory.mktemp("plan")
    # the launches are recorded instead of made; types of the same sizes stand for the device's
    (d / "p.cpp").write_text('#include "%s/include/hf.h"\n#include <stdint.h>\n#define __host__\n#define __device__\n' % ROOT + '''
typedef void* cudaStream_t;
struct bf16 { uint16_t v; };
struct __half { uint16_t v; };
struct Device { int sm_count; };
struct NormParams { int width; };
inline int element_bytes(int type) { return type == HF_F32 ? 4 : 2; }
inline bool aligned(const void* p, size_t bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0; }
bool stride_ok(long long s, int bytes) { return s * bytes % 16 == 0; }
hf_status fail(hf_status s, const char*, ...) { return s; }
#define HFL_TRY(expr) do { hf_status s_ = (expr); if (s_ != HF_OK) return s_; } while (0)
''' + between(kernel, "constexpr int NORM_TEAM_BYTES", "struct NormParams") + between(host, "struct NormPlan {", "template <typename T, int V, int NV, int TPR, bool WIDE = true>") + '''
static int launched[5];
template <typename T, int V, int NV, bool RING, bool WIDE = true>
hf_status launch_norm_bwd(const Device*, const NormParams&, const NormPlan&, cudaStream_t) {
    launched[0] = sizeof(T); launched[1] = V; launched[2] = NV; launched[3] = RING; launched[4] = WIDE;
    return HF_OK;
}
''' + between(host, "template <typename T>\nhf_status launch_norm_bwd_of(", "template <typename T, int V, bool HALVES, bool WIDE>\nhf_status launch_rope(") + '''
extern "C" void bwd(int type, int wide, int width, long long rows, long long per_group, int sms, long long* out) {
    const hf_norm_shape g = {type, type, width, rows, width, width, width, per_group, width, 0.f, 0.f};
    const NormPlan n = norm_bwd_plan(&g, wide != 0, sms);
    const Device d = {sms};
    const NormParams p = {width};
    if (type == HF_BF16) launch_norm_bwd_of<bf16>(&d, p, n, nullptr);
    else if (type == HF_F16) launch_norm_bwd_of<__half>(&d, p, n, nullptr);
    else launch_norm_bwd_of<float>(&d, p, n, nullptr);
    const long long o[] = {n.wide, n.groups, n.nv, n.tpr, n.teams, n.group_blocks, n.stages, n.smem, launched[0], launched[1], launched[2], launched[3], launched[4],
                           norm_bwd_warps(launched[1] * launched[2]), NORM_TEAM_BYTES};
    for (int i = 0; i < 15; ++i) out[i] = o[i];
}
''')
    subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", str(d / "p.cpp"), "-o", str(d / "p.so")], check=True)
    lib = C.CDLL(str(d / "p.so"))
    out = (C.c_longlong * 15)()

    def bwd(type, wide, width, rows, per_group=0, sms=SMS):
        lib.bwd(type, int(wide), width, C.c_longlong(rows), C.c_longlong(per_group), sms, out)
        return list(out)
    return bwd


@pytest.mark.parametrize("type", [0, 1, 2])
@pytest.mark.parametrize("wide", [True, False])
def test_the_plan_is_that_of_the_kernel_launched(rules, type, wide):
    e = 4 if type == 2 else 2
    for width in range(1, 16385):
        if wide and width * e % 16:
            continue
        for rows in (1, 500, 33000):
            p_wide, groups, nv, tpr, teams, blocks, stages, smem, size, V, NV, ring, k_wide, warps, team_bytes = rules(type, wide, width, rows)
            at = (type, wide, width, rows)
            assert size == e and bool(p_wide) == wide == bool(k_wide), at
            assert 1 <= teams and teams * tpr <= 32 * warps and blocks >= 1 and groups == 1, at         # the launch bounds
            assert nv == NV and V * NV * tpr >= width, at                       # every column has a thread
            assert bool(ring) == (stages > 0) and stages in (0, 2, 3, 4), at
            # shared memory: the factors, the barriers and sums, the rings; at the end the teams' sums
            row = width * e if wide else (width * e + 30) // 16 * 16
            assert smem <= SMEM and smem >= (width * 4 + 4 + 15) // 16 * 16 + teams * (team_bytes + stages * 2 * row), at
            assert smem >= teams * 2 * V * NV * tpr * 4, at


@pytest.mark.parametrize("per_group", [0, 1, 4])
def test_no_rows_need_no_workspace(per_group):
    """The empty batch of a modulated norm has no groups to share the multiprocessors among."""
    from paper_2604_10103_b200 import binding as hf, build
    build.build()
    s = hf.hf_norm_shape(type=0, param_type=0, width=64, rows=0, x_stride=64, y_stride=64, dx_stride=64, rows_per_group=per_group, param_stride=64,
                         weight_offset=1.0, eps=1e-6)
    n = C.c_size_t(1)
    assert hf.lib().hf_layer_norm_workspace(C.byref(s), C.byref(n)) == 0 and n.value == 0


@pytest.mark.gpu
def test_gradients_of_no_rows_in_groups():
    import torch
    from paper_2604_10103_b200 import layers
    for dtype in (torch.bfloat16, torch.float32):
        e, w = torch.empty(0, 64, device="cuda", dtype=dtype), torch.empty(0, 64, device="cuda", dtype=dtype)
        y, mean, rstd = layers.layer_norm(e, w, w, weight_offset=1.0, rows_per_group=4)
        dx, dw, db = layers.layer_norm_backward(e, e, mean, rstd, w, weight_offset=1.0, rows_per_group=4)
        assert y.shape == dx.shape == (0, 64) and dw.shape == db.shape == (0, 64)


def test_groups_longer_than_any_number_of_rows(rules):
    """One group, however many rows it might hold."""
    for per_group in (1, 4, 2 ** 31, 2 ** 63 - 2, 2 ** 63 - 1):
        for rows in (1, 2, 500, 2 ** 31 - 1):
            if per_group == 1 and rows > 500:
                continue
            _, groups, _, _, teams, blocks, _, smem, *_ = rules(0, True, 64, rows, per_group)
            assert groups == -(-rows // per_group) and teams >= 1 and blocks >= 1 and 0 < smem <= SMEM, (per_group, rows)


@pytest.mark.gpu
def test_one_group_of_any_number_of_rows():
    import torch
    from paper_2604_10103_b200 import layers
    for rows, width in ((5, 64), (4000, 1455)):          # (a few rows, and many that walk through rings)
        x, w, dy = (torch.randn(n, width, device="cuda").bfloat16() for n in (rows, 1, rows))
        ref = layers.layer_norm(x, w, w)
        refb = layers.layer_norm_backward(dy, x, ref[1], ref[2], w)
        got = layers.layer_norm(x, w, w, rows_per_group=2 ** 63 - 1)
        gotb = layers.layer_norm_backward(dy, x, ref[1], ref[2], w, rows_per_group=2 ** 63 - 1)
        assert all(torch.equal(p, q) for p, q in zip(ref + refb, got + gotb))
