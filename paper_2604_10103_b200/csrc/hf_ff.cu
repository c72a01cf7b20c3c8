// Gated feed-forward: host side and the kernels' instantiations.
#include "hf_layers.h"
#include <type_traits>
#include "k_ff_gemm.cuh"
#include "k_ff_rows.cuh"

#include <cstring>

using namespace hf_layers;

namespace {

typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                                  const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                  CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

// Map of a matrix [rows, cols] of 16-bit elements with `stride` between rows; box of box_cols (64: 128-byte swizzle; 32: 64-byte) x box_rows.
// planes: that many such matrices `plane_bytes` apart, and as many boxes at a time.
hf_status matrix_map(const Device* d, CUtensorMap* m, int type, const void* base, long long rows, long long cols, long long stride,
                     int box_cols, int box_rows, int planes = 1, size_t plane_bytes = 0) {
    const cuuint64_t dims[3] = {(cuuint64_t)cols, (cuuint64_t)rows, (cuuint64_t)planes};
    const cuuint64_t strides[2] = {(cuuint64_t)(rows > 1 ? stride : (cols + 7) / 8 * 8) * 2, plane_bytes};
    const cuuint32_t box[3] = {(cuuint32_t)box_cols, (cuuint32_t)box_rows, (cuuint32_t)planes};
    const cuuint32_t es[3] = {1, 1, 1};
    const CUresult r = reinterpret_cast<EncodeTiledFn>(d->encode_tiled)(
        m, type == HF_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, planes > 1 ? 3 : 2, const_cast<void*>(base), dims, strides, box, es,
        CU_TENSOR_MAP_INTERLEAVE_NONE, box_cols == 64 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B,
        CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    if (r != CUDA_SUCCESS) return fail(HF_ERR_CUDA, "cuTensorMapEncodeTiled failed with %d", (int)r);
    return HF_OK;
}

struct Matrix { const void* p; long long rows, cols, stride; };

// How a launch's products are cut: thread blocks a tile (cg), accumulator columns a tile (bn), parts of a tile's contraction (splits).
struct Tiling { int cg, bn, splits; };
struct Size { long long rows, cols, contraction; };

// The tiling of least estimated time, in cycles: rounds of tiles over the device, each of the tile's blocks of 64 of the contraction (2 bn cycles
// of MMAs, or what bringing 128 + bn / cg columns of both operands into shared memory and out of it was seen to take, which depends on how
// they lie) and some cycles between tiles.  Tiles of 512 columns (dW) have their epilogue between the MMAs.  STORE may split the contraction:
// another launch, the parts' sums (8 bytes an element and part) on their way through L2, and something for each part.
// What the numbers come from, us a call with the other products of the call unchanged, width 1536, hidden 4096, [thread blocks] x columns
// (/ splits).  4680 rows: g, u 2x256 125.7, 1x256 130.6, 2x192 132; y 2x224 135, 2x256 137, 1x192 139, 1x256 140, 2x192 141, 2x128 151;
// dx 2x256 321, 1x192 330, 1x256 335, 2x192 345; dW 2x512 278, 2x256 292, (2x256 317, 2x224 334, 1x256 335 before other parts were faster).
// 1000 rows: dx 2x256/3 82, /2 87, /1 96, 2x128 92, 1x128 96.  300 rows: dx 1x128/4 56.5, 2x128/3 57, 1x64 67.5; y 1x64 30.5, 2x128 31; g, u 1x256
// 31.9, 2x256 32, 1x128 35, 1x64 41.  77 rows: y 1x64/3 22.4, /4 23, /6 25.6, /1 26.8; dx 1x128/6 38.9, /4 40.9, /12 43.4, 1x64 57.9.
enum FfCut { FF_CUT_GATED, FF_CUT_Y, FF_CUT_DH, FF_CUT_DX, FF_CUT_DW };
Tiling ff_tiling(const Device* d, const Size* s, int n, int segments, FfCut cut) {
    const bool gated = cut == FF_CUT_GATED, b_mn = cut >= FF_CUT_DH, a_mn = cut == FF_CUT_DW, may_split = cut != FF_CUT_GATED && cut != FF_CUT_DH;
    Tiling best = {1, 64, 1};
    double least = 1e300;
    for (int cg = 1; cg <= 2; ++cg)
        for (int bn = b_mn ? 64 * cg : 64; bn <= (a_mn && cg == 2 ? 512 : 256); bn += gated ? 64 : (b_mn ? 64 * cg : 32)) {
            if (bn > 256 && bn != 512) continue;
            if (cut == FF_CUT_DH && cg == 1 && bn > 128) break;         // (its staging leaves two stages)
            const int out = gated ? bn / 2 : bn, slots = cg == 1 ? d->sm_count : d->pairs;
            long long tiles = 0;
            double blocks = 0;
            for (int i = 0; i < n; ++i) {
                tiles += (s[i].rows + 128 * cg - 1) / (128 * cg) * ((s[i].cols + out - 1) / out);
                if (blocks < (double)((s[i].contraction + 63) / 64)) blocks = (double)((s[i].contraction + 63) / 64);
            }
            const double columns = 128 + bn / cg, mma = 2.0 * bn;
            const double memory = a_mn ? 430 + 0.78 * columns : (b_mn ? 260 + 0.95 * columns : 150 + 1.15 * columns), block = mma > memory ? mma : memory;
            const double between = bn == 512 ? 6500.0 : 1500.0;
            blocks *= segments;
            for (int k = 1; k <= (may_split && bn <= 256 && tiles < slots ? 16 : 1); ++k) {
                if (k > 1 && blocks < 4 * k) break;
                double cost = (double)((tiles * k + slots - 1) / slots) * (blocks / k * block + between);
                if (k > 1) cost += 4000.0 + 1200.0 * k + tiles * k * 128.0 * cg * bn * 8.0 / 2300.0;
                if (cost < least) { least = cost; best = {cg, bn, k}; }
            }
        }
    return best;
}

// One launch being put together: operands, outputs, tiles.
struct Launch {
    const Device* d;
    int type;
    Tiling tiling;
    FfGemmParams p;
    FfJoinOut join = {};
    Launch(const Device* dev, int t, int act, Tiling cut) : d(dev), type(t), tiling(cut) {
        memset(&p, 0, sizeof(p));
        p.segments = 1; p.act = act; p.dev_status = dev->status; p.bn = cut.bn; p.splits = cut.splits;
    }
    // Contraction-contiguous (K-major) operand of `tile` rows; row-contiguous (MN-major) operand.
    hf_status k_major(CUtensorMap* m, const Matrix& x, int tile) { return matrix_map(d, m, type, x.p, x.rows, x.cols, x.stride, 64, tile); }
    hf_status mn_major(CUtensorMap* m, const Matrix& x) { return matrix_map(d, m, type, x.p, x.rows, x.cols, x.stride, 64, 64); }
    // What an epilogue reads or writes: boxes of 32 x 32.
    hf_status box(CUtensorMap* m, const Matrix& x) { return matrix_map(d, m, type, x.p, x.rows, x.cols, x.stride, 32, 32); }
    hf_status output(int i, const Matrix& x) {
        join.out[i] = const_cast<void*>(x.p); join.stride[i] = x.stride;
        return box(&p.out[i], x);
    }
    void product(long long rows, int cols, long long contraction, int bn_out) {
        const int i = p.products++, bm = 128 * tiling.cg;
        p.rows[i] = (int)rows; p.cols[i] = cols; p.kb[i] = (int)((contraction + 63) / 64);
        const long long tiles = (rows + bm - 1) / bm * ((cols + bn_out - 1) / bn_out);
        p.tile0[i + 1] = p.tile0[i] + (int)tiles;
    }
    template <typename T, int EPI, bool A_MN, bool B_MN, int CG, int NB = 1>
    hf_status run_t(cudaStream_t st) {
        typedef FfGemm<EPI, CG, NB> C;
        p.stages = C::stages_for(p.bn);
        auto kernel = k_ff_gemm<T, EPI, A_MN, B_MN, CG, NB>;
        struct Key {};
        HFL_TRY(allow_shared<Key>(d, kernel, C::SMEM_MAX));
        const int tiles = p.tile0[p.products] * p.splits, slots = CG == 1 ? d->sm_count : d->pairs;
        cudaLaunchConfig_t cfg = {};
        cudaLaunchAttribute attr[2];
        attr[0].id = cudaLaunchAttributeClusterDimension;
        attr[0].val.clusterDim.x = CG; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
        attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[1].val.programmaticStreamSerializationAllowed = 1;
        cfg.gridDim = dim3(CG * (tiles < slots ? tiles : slots)); cfg.blockDim = dim3(C::THREADS);
        cfg.dynamicSmemBytes = C::smem_bytes(p.bn, p.stages); cfg.stream = st; cfg.attrs = attr; cfg.numAttrs = 2;
        HFL_CUDA(cudaLaunchKernelEx(&cfg, kernel, p));
        if (p.splits == 1) return HF_OK;
        const long long warps = (long long)p.tile0[p.products] * 4 * CG * (p.bn / 8);
        join.cg = CG;
        return launch_after(k_ff_join<T>, dim3((unsigned)((warps + 3) / 4)), dim3(128), 0, st, p, join);
    }
    template <int EPI, bool A_MN, bool B_MN>
    hf_status run(cudaStream_t st) {
        if constexpr (A_MN)
            if (tiling.bn == 512) {
                p.bn = 256;
                return type == HF_BF16 ? run_t<bf16, EPI, A_MN, B_MN, 2, 2>(st) : run_t<__half, EPI, A_MN, B_MN, 2, 2>(st);
            }
        if (tiling.cg == 1) return type == HF_BF16 ? run_t<bf16, EPI, A_MN, B_MN, 1>(st) : run_t<__half, EPI, A_MN, B_MN, 1>(st);
        return type == HF_BF16 ? run_t<bf16, EPI, A_MN, B_MN, 2>(st) : run_t<__half, EPI, A_MN, B_MN, 2>(st);
    }
};

hf_status ff_check(const hf_ff_shape* g) {
    if (g == nullptr) return fail(HF_ERR_INVALID_ARG, "shape is null");
    if (g->type != HF_BF16 && g->type != HF_F16) return fail(HF_ERR_UNSUPPORTED, "type %d: bf16 and f16 are taken", g->type);
    if (g->act != HF_ACT_SILU && g->act != HF_ACT_GELU_TANH) return fail(HF_ERR_UNSUPPORTED, "act %d unknown", g->act);
    if (g->rows < 0 || g->rows > (1 << 24)) return fail(HF_ERR_SHAPE, "rows %lld outside [0, 2^24]", (long long)g->rows);
    const int w[3] = {g->width, g->hidden, g->out_width};
    for (int v : w)
        if (v < 8 || v % 8 || v > (1 << 17)) return fail(HF_ERR_SHAPE, "width, hidden and out_width are multiples of 8 up to 2^17: got %d", v);
    if (g->rows > 1) {
        if (g->x_stride < g->width || g->y_stride < g->out_width) return fail(HF_ERR_SHAPE, "row strides must be at least the width");
        if (g->x_stride % 8 || g->y_stride % 8) return fail(HF_ERR_SHAPE, "row strides must be multiples of 8");
        if (g->x_stride > (1LL << 36) || g->y_stride > (1LL << 36)) return fail(HF_ERR_SHAPE, "row strides too large");
    }
    return HF_OK;
}
hf_status ff_pointer(const void* p, const char* name) {
    if (p == nullptr) return fail(HF_ERR_INVALID_ARG, "%s is null", name);
    if (!aligned(p, 16)) return fail(HF_ERR_INVALID_ARG, "%s is not 16-byte aligned", name);
    return HF_OK;
}
size_t round_up(size_t n) { return (n + 255) / 256 * 256; }

// The products' sizes and cuts.
struct Sizes { Size data[3]; };
Sizes y_sizes(const hf_ff_shape* g) { return {{{g->rows, g->out_width, g->hidden}}}; }
Sizes dx_sizes(const hf_ff_shape* g) { return {{{g->rows, g->width, g->hidden}}}; }
Sizes dw_sizes(const hf_ff_shape* g) {
    return {{{g->hidden, g->width, g->rows}, {g->hidden, g->width, g->rows}, {g->out_width, g->hidden, g->rows}}};
}
Tiling cut_gated(const Device* d, const hf_ff_shape* g) {
    const Size s = {g->rows, g->hidden, g->width};
    return ff_tiling(d, &s, 1, 1, FF_CUT_GATED);
}
Tiling cut_y(const Device* d, const hf_ff_shape* g) { return ff_tiling(d, y_sizes(g).data, 1, 1, FF_CUT_Y); }
Tiling cut_dh(const Device* d, const hf_ff_shape* g) {
    const Size s = {g->rows, g->hidden, g->out_width};
    return ff_tiling(d, &s, 1, 1, FF_CUT_DH);
}
Tiling cut_dx(const Device* d, const hf_ff_shape* g) { return ff_tiling(d, dx_sizes(g).data, 1, 2, FF_CUT_DX); }
Tiling cut_dw(const Device* d, const hf_ff_shape* g) { return ff_tiling(d, dw_sizes(g).data, 3, 1, FF_CUT_DW); }
size_t ff_partial_bytes(const Tiling& t, const Size* s, int n) {
    if (t.splits == 1) return 0;
    size_t tiles = 0;
    for (int i = 0; i < n; ++i)
        tiles += (size_t)((s[i].rows + 128 * t.cg - 1) / (128 * t.cg)) * ((s[i].cols + t.bn - 1) / t.bn);
    return tiles * t.splits * 128 * t.cg * t.bn * sizeof(float);
}

// Up to 16 rows: both products by k_ff_rows (width 1536, hidden 4096: 1 row 10.5 us, 16 rows 13.7; with tiles 23.5; its form for 32 rows took 26).
constexpr int FF_ROWS_MOST = 16;
template <typename T, int NT, int ACT>
hf_status launch_rows(const hf_ff_shape* g, const FfRowsParams& first, const FfRowsParams& second, cudaStream_t st) {
    HFL_TRY(launch_after(k_ff_rows<T, NT, true, ACT>, dim3((g->hidden + 7) / 8), dim3(256), 0, st, first));
    return launch_after(k_ff_rows<T, NT, false, 0>, dim3((g->out_width + 7) / 8), dim3(512), 0, st, second);
}
template <typename T, int NT>
hf_status launch_rows(const hf_ff_shape* g, const FfRowsParams& first, const FfRowsParams& second, cudaStream_t st) {
    return g->act == HF_ACT_SILU ? launch_rows<T, NT, HF_ACT_SILU>(g, first, second, st) : launch_rows<T, NT, HF_ACT_GELU_TANH>(g, first, second, st);
}
template <typename T>
hf_status launch_rows(const hf_ff_shape* g, const FfRowsParams& first, const FfRowsParams& second, cudaStream_t st) {
    if (g->rows <= 8) return launch_rows<T, 1>(g, first, second, st);
    return launch_rows<T, 2>(g, first, second, st);
}

}  // namespace

namespace {
// The current device, with the pairs of multiprocessors that can hold a cluster of two thread blocks at a time (a persistent grid of more
// would run in two rounds): asked on the first call of this module, which is loaded by it.
hf_status ff_device(const Device** out) {
    HFL_TRY(current_device(out));
    if ((*out)->pairs) return HF_OK;
    typedef FfGemm<FF_STORE, 2> C;
    auto kernel = k_ff_gemm<bf16, FF_STORE, false, false, 2>;
    HFL_CUDA(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, C::SMEM_MAX));
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr;
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim.x = 2; attr.val.clusterDim.y = 1; attr.val.clusterDim.z = 1;
    cfg.gridDim = dim3(256); cfg.blockDim = dim3(C::THREADS); cfg.dynamicSmemBytes = C::SMEM_MAX; cfg.attrs = &attr; cfg.numAttrs = 1;
    int pairs = 0;
    HFL_CUDA(cudaOccupancyMaxActiveClusters(&pairs, kernel, &cfg));
    if (pairs < 1) return fail(HF_ERR_UNSUPPORTED, "the device holds no cluster of two thread blocks");
    (*out)->pairs = pairs;
    return HF_OK;
}
}  // namespace

extern "C" {

hf_status hf_gated_ff_workspace(const hf_ff_shape* g, int backward, size_t* bytes) {
    HFL_TRY(ff_check(g));
    if (!bytes) return fail(HF_ERR_INVALID_ARG, "bytes is null");
    const Device* d;
    HFL_TRY(ff_device(&d));
    const size_t h = round_up((size_t)g->rows * g->hidden * 2);
    if (backward) {             // dg, du, h; the parts' sums of dx, then of dW
        const size_t x = ff_partial_bytes(cut_dx(d, g), dx_sizes(g).data, 1), w = ff_partial_bytes(cut_dw(d, g), dw_sizes(g).data, 3);
        *bytes = 3 * h + (x > w ? x : w);
    } else
        *bytes = h + ff_partial_bytes(cut_y(d, g), y_sizes(g).data, 1);
    return HF_OK;
}

hf_status hf_gated_ff(const hf_ff_shape* g, const void* x, const void* w_gate, const void* w_up, const void* w_down, void* y, void* gate,
                      void* up, void* workspace, void* stream) {
    HFL_TRY(ff_check(g));
    if (g->rows == 0) return HF_OK;
    HFL_TRY(ff_pointer(x, "x")); HFL_TRY(ff_pointer(w_gate, "w_gate")); HFL_TRY(ff_pointer(w_up, "w_up")); HFL_TRY(ff_pointer(w_down, "w_down"));
    HFL_TRY(ff_pointer(y, "y")); HFL_TRY(ff_pointer(workspace, "workspace"));
    if ((gate == nullptr) != (up == nullptr)) return fail(HF_ERR_INVALID_ARG, "gate and up are saved together or not at all");
    if (gate) { HFL_TRY(ff_pointer(gate, "gate")); HFL_TRY(ff_pointer(up, "up")); }
    const Device* d;
    HFL_TRY(ff_device(&d));
    const cudaStream_t st = (cudaStream_t)stream;
    const long long M = g->rows, K = g->width, N = g->hidden, O = g->out_width;
    if (M <= FF_ROWS_MOST) {
        const FfRowsParams first = {x, w_gate, w_up, workspace, gate, up, g->x_stride, N, (int)M, (int)K, (int)N};
        const FfRowsParams second = {workspace, w_down, w_down, y, nullptr, nullptr, N, g->y_stride, (int)M, (int)N, (int)O};
        return g->type == HF_BF16 ? launch_rows<bf16>(g, first, second, st) : launch_rows<__half>(g, first, second, st);
    }
    const Matrix h = {workspace, M, N, N};
    {
        Launch l(d, g->type, g->act, cut_gated(d, g));
        const int hn = l.p.bn / 2;
        HFL_TRY(l.k_major(&l.p.a[0], {x, M, K, g->x_stride}, 128));
        HFL_TRY(l.k_major(&l.p.b[0], {w_gate, N, K, K}, hn));
        HFL_TRY(l.k_major(&l.p.b[1], {w_up, N, K, K}, hn));
        HFL_TRY(l.output(0, h));
        if (gate) {
            HFL_TRY(l.output(1, {gate, M, N, N}));
            HFL_TRY(l.output(2, {up, M, N, N}));
            l.p.save = 1;
        }
        l.product(M, N, K, hn);
        HFL_TRY((l.run<FF_GATED, false, false>(st)));
    }
    Launch l(d, g->type, g->act, cut_y(d, g));
    l.p.partials = reinterpret_cast<float*>(static_cast<uint8_t*>(workspace) + round_up((size_t)M * N * 2));
    HFL_TRY(l.k_major(&l.p.a[0], h, 128));
    HFL_TRY(l.k_major(&l.p.b[0], {w_down, O, N, N}, l.p.bn / l.tiling.cg));
    HFL_TRY(l.output(0, {y, M, O, g->y_stride}));
    l.product(M, O, N, l.p.bn);
    l.p.early_b = 1;
    return l.run<FF_STORE, false, false>(st);
}

hf_status hf_gated_ff_backward(const hf_ff_shape* g, const void* dy, const void* x, const void* w_gate, const void* w_up, const void* w_down,
                               const void* gate, const void* up, void* dx, void* dw_gate, void* dw_up, void* dw_down, void* workspace,
                               void* stream) {
    HFL_TRY(ff_check(g));
    const int n_dw = (dw_gate != nullptr) + (dw_up != nullptr) + (dw_down != nullptr);
    if (n_dw != 0 && n_dw != 3) return fail(HF_ERR_INVALID_ARG, "the weights' gradients are formed together or not at all");
    const cudaStream_t st = (cudaStream_t)stream;
    const long long M = g->rows, K = g->width, N = g->hidden, O = g->out_width;
    if (n_dw) { HFL_TRY(ff_pointer(dw_gate, "dw_gate")); HFL_TRY(ff_pointer(dw_up, "dw_up")); HFL_TRY(ff_pointer(dw_down, "dw_down")); }
    if (M == 0) {
        if (n_dw) {
            HFL_CUDA(cudaMemsetAsync(dw_gate, 0, (size_t)N * K * 2, st));
            HFL_CUDA(cudaMemsetAsync(dw_up, 0, (size_t)N * K * 2, st));
            HFL_CUDA(cudaMemsetAsync(dw_down, 0, (size_t)O * N * 2, st));
        }
        return HF_OK;
    }
    if (!dx && !n_dw) return HF_OK;
    HFL_TRY(ff_pointer(dy, "dy")); HFL_TRY(ff_pointer(x, "x")); HFL_TRY(ff_pointer(w_gate, "w_gate")); HFL_TRY(ff_pointer(w_up, "w_up"));
    HFL_TRY(ff_pointer(w_down, "w_down")); HFL_TRY(ff_pointer(gate, "gate")); HFL_TRY(ff_pointer(up, "up")); HFL_TRY(ff_pointer(workspace, "workspace"));
    if (dx) HFL_TRY(ff_pointer(dx, "dx"));
    const Device* d;
    HFL_TRY(ff_device(&d));
    const size_t part = round_up((size_t)M * N * 2);
    uint8_t* ws = static_cast<uint8_t*>(workspace);
    const Matrix mdy = {dy, M, O, g->y_stride}, mx = {x, M, K, g->x_stride}, dg = {ws, M, N, N}, du = {ws + part, M, N, N}, h = {ws + 2 * part, M, N, N};
    {
        Launch l(d, g->type, g->act, cut_dh(d, g));
        HFL_TRY(l.box(&l.p.in[0], {gate, M, N, N})); HFL_TRY(l.box(&l.p.in[1], {up, M, N, N}));
        HFL_TRY(l.k_major(&l.p.a[0], mdy, 128));
        HFL_TRY(l.mn_major(&l.p.b[0], {w_down, O, N, N}));
        HFL_TRY(matrix_map(d, &l.p.out[0], g->type, ws, M, N, N, 32, 32, 3, part));
        l.product(M, (int)N, O, l.p.bn);
        HFL_TRY((l.run<FF_DHIDDEN, false, true>(st)));
    }
    if (dx) {
        Launch l(d, g->type, g->act, cut_dx(d, g));
        l.p.partials = reinterpret_cast<float*>(ws + 3 * part);
        HFL_TRY(l.k_major(&l.p.a[0], dg, 128)); HFL_TRY(l.k_major(&l.p.a[1], du, 128));
        HFL_TRY(l.mn_major(&l.p.b[0], {w_gate, N, K, K})); HFL_TRY(l.mn_major(&l.p.b[1], {w_up, N, K, K}));
        HFL_TRY(l.output(0, {dx, M, K, K}));
        l.product(M, (int)K, N, l.p.bn);
        l.p.segments = 2; l.p.kb[1] = l.p.kb[0];
        l.p.early_b = 1;
        HFL_TRY((l.run<FF_STORE, false, true>(st)));
    }
    if (n_dw) {
        Launch l(d, g->type, g->act, cut_dw(d, g));
        l.p.partials = reinterpret_cast<float*>(ws + 3 * part);
        HFL_TRY(l.mn_major(&l.p.a[0], dg)); HFL_TRY(l.mn_major(&l.p.a[1], du)); HFL_TRY(l.mn_major(&l.p.a[2], mdy));
        HFL_TRY(l.mn_major(&l.p.b[0], mx)); l.p.b[1] = l.p.b[0]; HFL_TRY(l.mn_major(&l.p.b[2], h));
        HFL_TRY(l.output(0, {dw_gate, N, K, K})); HFL_TRY(l.output(1, {dw_up, N, K, K})); HFL_TRY(l.output(2, {dw_down, O, N, N}));
        l.product(N, (int)K, M, l.tiling.bn); l.product(N, (int)K, M, l.tiling.bn); l.product(O, (int)N, M, l.tiling.bn);
        HFL_TRY((l.run<FF_STORE, true, true>(st)));
    }
    return HF_OK;
}

}  // extern "C"
