// Host side of the calls that need no context: layer norm and rotary positions with several axes, and what they share with the gated
// feed-forward (the device's status word, errors).
#include "hf_layers.h"
#include "k_norm.cuh"
#include "k_rope_axes.cuh"

#include <cstdarg>
#include <cstdio>
#include <mutex>

extern "C" void hf_internal_set_error(const char* text);

namespace hf_layers {

namespace {
constexpr int MAX_DEVICES = 64;
__device__ int g_status[4];             // status word of the calls without a context, one per device
std::mutex g_mutex;
Device g_devices[MAX_DEVICES];
volatile bool g_known[MAX_DEVICES];
}  // namespace

hf_status fail(hf_status s, const char* fmt, ...) {
    char buf[384];
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(buf, sizeof(buf), fmt, ap);
    va_end(ap);
    hf_internal_set_error(buf);
    return s;
}

hf_status current_device(const Device** out) {
    int dev = -1;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) { cudaGetLastError(); return fail(HF_ERR_CUDA, "cudaGetDevice: %s", cudaGetErrorString(e)); }
    if (dev < 0 || dev >= MAX_DEVICES) return fail(HF_ERR_UNSUPPORTED, "device index %d not supported", dev);
    if (!g_known[dev]) {
        std::lock_guard<std::mutex> lock(g_mutex);
        if (!g_known[dev]) {
            Device d = {dev, 0, nullptr, nullptr, 0};
            int major = 0;
            HFL_CUDA(cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, dev));
            if (major != 10) return fail(HF_ERR_UNSUPPORTED, "device of compute capability %d.x; this library is built for sm_100a only", major);
            HFL_CUDA(cudaDeviceGetAttribute(&d.sm_count, cudaDevAttrMultiProcessorCount, dev));
            void* p = nullptr;
            HFL_CUDA(cudaGetSymbolAddress(&p, g_status));
            d.status = static_cast<int*>(p);
            cudaDriverEntryPointQueryResult q;
            e = cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &d.encode_tiled, cudaEnableDefault, &q);
            if (e != cudaSuccess || q != cudaDriverEntryPointSuccess || d.encode_tiled == nullptr)
                return fail(HF_ERR_CUDA, "cuTensorMapEncodeTiled is not available from the driver");
            g_devices[dev].index = d.index; g_devices[dev].sm_count = d.sm_count;
            g_devices[dev].status = d.status; g_devices[dev].encode_tiled = d.encode_tiled;
            g_known[dev] = true;
        }
    }
    *out = &g_devices[dev];
    return HF_OK;
}

namespace {

bool stride_ok(long long s, int bytes) { return s * bytes % 16 == 0; }

// ------------------------------------------------------------------------------------------------ layer norm
struct NormPlan {
    bool wide;                  // 16-byte accesses
    int groups, nv, tpr, teams, group_blocks, stages, smem;
};
constexpr int NORM_SMEM = 232448;       // shared memory of a multiprocessor's one thread block

hf_status norm_check(const hf_norm_shape* g) {
    if (g == nullptr) return fail(HF_ERR_INVALID_ARG, "shape is null");
    if (g->type != HF_BF16 && g->type != HF_F16 && g->type != HF_F32) return fail(HF_ERR_UNSUPPORTED, "type %d unknown", g->type);
    if (g->param_type != g->type && g->param_type != HF_F32) return fail(HF_ERR_UNSUPPORTED, "param_type %d is neither the type nor HF_F32", g->param_type);
    if (g->width < 1 || g->width > 16384) return fail(HF_ERR_SHAPE, "width %d outside [1, 16384]", g->width);
    if (g->rows < 0 || g->rows > 0x7fffffffLL) return fail(HF_ERR_SHAPE, "rows %lld outside [0, 2^31)", (long long)g->rows);
    if (g->rows_per_group < 0) return fail(HF_ERR_SHAPE, "rows_per_group must be >= 0");
    if (!(g->eps >= 0.f)) return fail(HF_ERR_SHAPE, "eps must be >= 0");
    if (g->rows > 1 && (g->x_stride < g->width || g->y_stride < g->width)) return fail(HF_ERR_SHAPE, "row strides must be at least the width");
    if (g->rows_per_group > 0 && g->rows > g->rows_per_group && g->param_stride < g->width)
        return fail(HF_ERR_SHAPE, "param_stride must be at least the width");
    return HF_OK;
}
int norm_groups(const hf_norm_shape* g) {
    if (g->rows_per_group == 0) return 1;
    return g->rows == 0 ? 0 : (int)((g->rows - 1) / g->rows_per_group + 1);       // (rows_per_group may be any 64-bit number)
}
// Whether every row of a tensor and every group of the parameters starts on 16 bytes.
bool norm_wide(const hf_norm_shape* g, const void* const* rows, const long long* strides, int n, const void* w, const void* b) {
    const int e = element_bytes(g->type), pe = element_bytes(g->param_type);
    if (g->width * e % 16 != 0) return false;
    for (int i = 0; i < n; ++i)
        if (rows[i] && (!aligned(rows[i], 16) || (g->rows > 1 && !stride_ok(strides[i], e)))) return false;
    if ((w && !aligned(w, 16)) || (b && !aligned(b, 16))) return false;
    return !((w || b) && norm_groups(g) > 1 && !stride_ok(g->param_stride, pe));
}

// Backward: threads a row, teams of them, thread blocks.  A team has as few warps as its columns' sums fit in (48 columns a thread; 32760 rows
// of 1536 bf16, when that was measured: 59 us, with 24 columns and two warps a team 64, with 16 and three 69).  A thread block has up to twelve warps, fewer where
// there are not two rows a team for every multiprocessor or two rows of each team do not fit in shared memory.  The number of thread
// blocks depends on the shape and its alignment alone, as the workspace does.
NormPlan norm_bwd_plan(const hf_norm_shape* g, bool wide, int sms) {
    NormPlan p;
    const int e = element_bytes(g->type), V = wide ? 16 / e : 4 / e;
    p.wide = wide;
    p.groups = norm_groups(g);
    const int factors = (g->width * 4 + 4 + 15) / 16 * 16, row = 2 * (wide ? g->width * e : (g->width * e + 30) / 16 * 16);
    // (floats one by one want a few registers more: 32 columns a thread where twelve warps are enough then and two rows fit; rows too long
    // for a ring, of over 11604 floats, or 11608 that start on 16 bytes, are read from global memory by one form, of 48)
    const bool rings = factors + NORM_TEAM_BYTES + 2 * row <= NORM_SMEM;
    const int most_cols = V == 1 && rings && g->width <= 12 * 32 * 32 ? 32 : 48, warps = (g->width + 32 * most_cols - 1) / (32 * most_cols);
    p.tpr = 32 * warps;
    p.nv = (g->width + V * p.tpr - 1) / (V * p.tpr);
    // (the instantiations)
    if (V == 8) p.nv = p.nv <= 1 ? 1 : (p.nv <= 2 ? 2 : (p.nv <= 4 ? 4 : 6));
    else if (V == 4) p.nv = p.nv <= 2 ? 2 : (p.nv <= 4 ? 4 : (p.nv <= 8 ? 8 : 12));
    else if (V == 2) p.nv = p.nv <= 4 ? 4 : (p.nv <= 12 ? 12 : 24);
    else p.nv = p.nv <= 8 ? 8 : (p.nv <= 24 ? 24 : (p.nv <= 32 ? 32 : 48));
    const long long rows = g->rows_per_group ? (g->rows < g->rows_per_group ? g->rows : g->rows_per_group) : g->rows;
    long long n = sms > p.groups ? sms / p.groups : 1;         // one round of thread blocks
    p.teams = norm_bwd_warps(V * p.nv) / warps;
    const long long most = (rows + 2 * n - 1) / (2 * n);
    if (p.teams > most) p.teams = most < 1 ? 1 : (int)most;
    auto fit = [&] { return (NORM_SMEM - factors - p.teams * NORM_TEAM_BYTES) / (p.teams * row); };
    while (p.teams > 1 && fit() < 2) --p.teams;
    p.stages = fit();
    if (p.stages > 4) p.stages = 4;
    if (!rings) p.stages = 0;
    p.smem = factors + p.teams * (NORM_TEAM_BYTES + p.stages * row);
    const int join = p.teams * 2 * V * p.nv * p.tpr * 4;
    if (join > p.smem) p.smem = join;
    if (n > (rows + p.teams - 1) / p.teams) n = (rows + p.teams - 1) / p.teams;
    p.group_blocks = n < 1 ? 1 : (int)n;
    return p;
}

template <typename T, int V, int NV, int TPR, bool WIDE = true>
hf_status launch_norm(const NormParams& p, cudaStream_t st) {
    k_norm<T, V, NV, TPR, WIDE><<<TPR == 32 ? (unsigned)((p.rows + 7) / 8) : (unsigned)p.rows, TPR == 32 ? 256 : TPR, 0, st>>>(p);
    HFL_CUDA(cudaGetLastError());
    return HF_OK;
}
// A warp a row up to 64 elements a lane, else a thread block a row.
template <typename T>
hf_status launch_norm_of(const NormParams& p, bool wide, cudaStream_t st) {
    constexpr int V = 16 / sizeof(T);
    const int w = p.width;
    if (wide) {
        const int n = (w + 32 * V - 1) / (32 * V);
        if (n <= 1) return launch_norm<T, V, 1, 32>(p, st);
        if (n <= 2) return launch_norm<T, V, 2, 32>(p, st);
        if (n <= 4) return launch_norm<T, V, 4, 32>(p, st);
        if (n <= 6) return launch_norm<T, V, 6, 32>(p, st);
        if (n <= 8) return launch_norm<T, V, 8, 32>(p, st);
        if (n <= 16) return launch_norm<T, V, 4, 128>(p, st);
        if (n <= 32) return launch_norm<T, V, 8, 128>(p, st);
        if (n <= 64) return launch_norm<T, V, 4, 512>(p, st);
        return launch_norm<T, V, 8, 512>(p, st);
    }
    constexpr int P = 4 / sizeof(T);            // 16-bit elements in pairs
    if (w <= 256) return launch_norm<T, P, 8 / P, 32, false>(p, st);
    if (w <= 512) return launch_norm<T, P, 4 / P, 128, false>(p, st);
    if (w <= 1024) return launch_norm<T, P, 8 / P, 128, false>(p, st);
    if (w <= 2048) return launch_norm<T, P, 16 / P, 128, false>(p, st);
    if (w <= 4096) return launch_norm<T, P, 8 / P, 512, false>(p, st);
    if (w <= 8192) return launch_norm<T, P, 16 / P, 512, false>(p, st);
    return launch_norm<T, P, 32 / P, 512, false>(p, st);
}

// Many rows (k_norm_rows): as norm_bwd_plan, with 24 warps a thread block, and no sums over rows to hold.  us, this / a thread block's rows at
// once (k_norm): 28213 x 1456 bf16 34 / 40, 8000 rows 16.6 / 17.6, 4680 x 1536 10.3 / 9 (so from two rows a team on); rows that do not
// start on 16 bytes, where the copies also align them: 28213 x 1455 61 / 125, 4000 rows 17 / 19, 600 rows 7.5 / 7.2, 300 rows 7.5 / 6.8,
// 600 x 6001 10 / 16 (so from four rows a multiprocessor on).  Floats on 16 bytes: 28213 x 1536 69 / 56 (never).
template <typename T, int V, int NV, bool WIDE>
hf_status launch_norm_rows(const Device* d, const NormParams& p, const NormPlan& n, cudaStream_t st) {
    struct Key {};
    HFL_TRY(allow_shared<Key>(d, k_norm_rows<T, V, NV, WIDE>, NORM_SMEM));
    k_norm_rows<T, V, NV, WIDE><<<(unsigned)(n.groups * n.group_blocks), dim3(n.tpr, n.teams), n.smem, st>>>(p);
    HFL_CUDA(cudaGetLastError());
    return HF_OK;
}
bool norm_rows_plan(const hf_norm_shape* g, bool wide, int sms, NormPlan* p) {
    const int e = element_bytes(g->type), V = wide ? 16 / e : 4 / e;
    p->groups = norm_groups(g);
    const long long rows = g->rows_per_group ? (g->rows < g->rows_per_group ? g->rows : g->rows_per_group) : g->rows;
    const int most_cols = V == 1 ? 24 : 48, warps = (g->width + 32 * most_cols - 1) / (32 * most_cols);
    p->tpr = 32 * warps;
    p->nv = (g->width + V * p->tpr - 1) / (V * p->tpr);
    p->group_blocks = sms / p->groups;
    if (p->group_blocks < 1 || (wide && e == 4)) return false;
    p->teams = NORM_ROWS_WARPS / warps;
    const long long each = (rows + p->group_blocks - 1) / p->group_blocks;
    if (p->teams > each) p->teams = each < 1 ? 1 : (int)each;
    const int factors = 2 * ((g->width * 4 + 4 + 15) / 16 * 16), row = wide ? g->width * e : (g->width * e + 30) / 16 * 16;
    auto fit = [&] { return (NORM_SMEM - factors - p->teams * NORM_ROWS_TEAM_BYTES) / (p->teams * row); };
    while (p->teams > 1 && fit() < 2) --p->teams;
    p->stages = fit() > 4 ? 4 : fit();
    p->smem = factors + p->teams * (NORM_ROWS_TEAM_BYTES + p->stages * row);
    return p->stages >= 2 && (wide ? rows >= 2LL * p->group_blocks * p->teams : each >= 4);
}
template <typename T>
hf_status launch_norm_rows_of(const Device* d, const NormParams& p, const NormPlan& n, bool wide, cudaStream_t st) {
    constexpr int P = 4 / sizeof(T);
    if constexpr (sizeof(T) == 2) {
        if (wide) {
            if (n.nv <= 1) return launch_norm_rows<T, 8, 1, true>(d, p, n, st);
            if (n.nv <= 3) return launch_norm_rows<T, 8, 3, true>(d, p, n, st);
            return launch_norm_rows<T, 8, 6, true>(d, p, n, st);
        }
        if (n.nv > 12) return launch_norm_rows<T, 2, 24, false>(d, p, n, st);
    }
    if (n.nv <= 8 / P) return launch_norm_rows<T, P, 8 / P, false>(d, p, n, st);
    return launch_norm_rows<T, P, 24 / P, false>(d, p, n, st);
}

template <typename T, int V, int NV, bool RING, bool WIDE = true>
hf_status launch_norm_bwd(const Device* d, const NormParams& p, const NormPlan& n, cudaStream_t st) {
    struct Key {};
    HFL_TRY(allow_shared<Key>(d, k_norm_bwd<T, V, NV, RING, WIDE>, NORM_SMEM));
    k_norm_bwd<T, V, NV, RING, WIDE><<<(unsigned)((long long)n.groups * n.group_blocks), dim3(n.tpr, n.teams), n.smem, st>>>(p);
    HFL_CUDA(cudaGetLastError());
    if (n.group_blocks > 1 && (p.dw || p.db))
        HFL_TRY(launch_after(k_norm_bwd_sum, dim3((p.width + 31) / 32, 2 * n.groups), dim3(32, 32), 0, st, (const float*)p.partials, n.group_blocks,
                             p.width, p.dw, p.db));
    return HF_OK;
}
template <typename T>
hf_status launch_norm_bwd_of(const Device* d, const NormParams& p, const NormPlan& n, cudaStream_t st) {
    if constexpr (sizeof(T) == 4)
        if (!n.stages) return n.wide ? launch_norm_bwd<T, 4, 12, false>(d, p, n, st) : launch_norm_bwd<T, 1, 48, false, false>(d, p, n, st);
    if (!n.wide) {
        constexpr int P = 4 / sizeof(T);
        if (n.nv == 8 / P) return launch_norm_bwd<T, P, 8 / P, true, false>(d, p, n, st);
        if (n.nv == 24 / P) return launch_norm_bwd<T, P, 24 / P, true, false>(d, p, n, st);
        if constexpr (P == 1)
            if (n.nv == 32) return launch_norm_bwd<T, 1, 32, true, false>(d, p, n, st);
        return launch_norm_bwd<T, P, 48 / P, true, false>(d, p, n, st);
    }
    if constexpr (sizeof(T) == 2) {
        if (n.nv == 1) return launch_norm_bwd<T, 8, 1, true>(d, p, n, st);
        if (n.nv == 2) return launch_norm_bwd<T, 8, 2, true>(d, p, n, st);
        if (n.nv == 4) return launch_norm_bwd<T, 8, 4, true>(d, p, n, st);
        return launch_norm_bwd<T, 8, 6, true>(d, p, n, st);
    } else {
        if (n.nv == 2) return launch_norm_bwd<T, 4, 2, true>(d, p, n, st);
        if (n.nv == 4) return launch_norm_bwd<T, 4, 4, true>(d, p, n, st);
        if (n.nv == 8) return launch_norm_bwd<T, 4, 8, true>(d, p, n, st);
        return launch_norm_bwd<T, 4, 12, true>(d, p, n, st);
    }
}

// ------------------------------------------------------------------------------------------------ rotary positions
template <typename T, int V, bool HALVES, bool WIDE>
hf_status launch_rope(RopeParams& p, int sms, cudaStream_t st) {
    p.units = p.head_dim / (2 * V);
    const long long threads = (long long)p.batch * p.tokens * p.units, blocks = (threads + 255) / 256;
    // Heads are cut into slices while all thread blocks still run at once, a batch of heads each at least: the angles are
    // looked up once a slice.
    int slices = (int)((long long)ROPE_BLOCKS * sms / blocks);
    const int batch = rope_batch<T, V, WIDE>(), most = (p.total_heads + batch - 1) / batch;
    p.slices = slices < 1 ? 1 : (slices > most ? most : slices);
    k_rope_axes<T, V, HALVES, WIDE><<<dim3((unsigned)blocks, p.slices), 256, 0, st>>>(p);
    HFL_CUDA(cudaGetLastError());
    return HF_OK;
}
template <typename T>
hf_status launch_rope_of(RopeParams& p, bool halves, bool wide, int sms, cudaStream_t st) {
    constexpr int V = 16 / sizeof(T);
    if (halves) return wide ? launch_rope<T, V, true, true>(p, sms, st) : launch_rope<T, 1, true, false>(p, sms, st);
    return wide ? launch_rope<T, V / 2, false, true>(p, sms, st) : launch_rope<T, 1, false, false>(p, sms, st);
}

}  // namespace
}  // namespace hf_layers

using namespace hf_layers;

extern "C" {

hf_status hf_layer_norm(const hf_norm_shape* g, const void* x, const void* weight, const void* bias, void* y, float* mean, float* rstd,
                        void* stream) {
    HFL_TRY(norm_check(g));
    if (g->rows == 0) return HF_OK;
    if (!x || !y) return fail(HF_ERR_INVALID_ARG, "x or y is null");
    const int e = element_bytes(g->type), pe = element_bytes(g->param_type);
    if (!aligned(x, e) || !aligned(y, e) || !aligned(weight, pe) || !aligned(bias, pe) || !aligned(mean, 4) || !aligned(rstd, 4))
        return fail(HF_ERR_INVALID_ARG, "a pointer is not aligned to its element");
    const Device* d;
    HFL_TRY(current_device(&d));
    NormParams p = {};
    p.x = x; p.y = y; p.w = weight; p.b = bias; p.mean = mean; p.rstd = rstd;
    p.rows = g->rows; p.x_stride = g->x_stride; p.y_stride = g->y_stride; p.param_stride = g->param_stride;
    p.rows_per_group = g->rows_per_group < g->rows ? g->rows_per_group : g->rows;
    p.width = g->width; p.params_f32 = g->param_type == HF_F32; p.weight_offset = g->weight_offset; p.eps = g->eps;
    const void* rows[2] = {x, y};
    const long long strides[2] = {g->x_stride, g->y_stride};
    const bool wide = norm_wide(g, rows, strides, 2, weight, bias);
    const cudaStream_t st = (cudaStream_t)stream;
    NormPlan n;
    if (norm_rows_plan(g, wide, d->sm_count, &n)) {
        p.group_blocks = n.group_blocks; p.stages = n.stages; p.dev_status = d->status;
        if (g->type == HF_BF16) return launch_norm_rows_of<bf16>(d, p, n, wide, st);
        if (g->type == HF_F16) return launch_norm_rows_of<__half>(d, p, n, wide, st);
        return launch_norm_rows_of<float>(d, p, n, wide, st);
    }
    if (g->type == HF_BF16) return launch_norm_of<bf16>(p, wide, st);
    if (g->type == HF_F16) return launch_norm_of<__half>(p, wide, st);
    return launch_norm_of<float>(p, wide, st);
}

hf_status hf_layer_norm_workspace(const hf_norm_shape* g, size_t* bytes) {
    HFL_TRY(norm_check(g));
    if (!bytes) return fail(HF_ERR_INVALID_ARG, "bytes is null");
    *bytes = 0;
    if (g->rows == 0) return HF_OK;             // (and there may be no groups to share the multiprocessors among)
    const Device* d;
    HFL_TRY(current_device(&d));
    // (the alignment of the tensors, which the shape does not say, changes the number of thread blocks)
    size_t most = 0;
    for (int wide = 0; wide < 2; ++wide) {
        const NormPlan n = norm_bwd_plan(g, wide != 0, d->sm_count);
        const size_t need = n.group_blocks > 1 ? (size_t)n.groups * n.group_blocks * 2 * g->width * sizeof(float) : 0;
        if (need > most) most = need;
    }
    *bytes = most;
    return HF_OK;
}

hf_status hf_layer_norm_backward(const hf_norm_shape* g, const void* dy, const void* x, const float* mean, const float* rstd, const void* weight,
                                 void* dx, float* dweight, float* dbias, void* workspace, void* stream) {
    HFL_TRY(norm_check(g));
    if (dx && g->rows > 1 && g->dx_stride < g->width) return fail(HF_ERR_SHAPE, "dx_stride must be at least the width");
    const int e = element_bytes(g->type), pe = element_bytes(g->param_type);
    if (!aligned(x, e) || !aligned(dy, e) || !aligned(dx, e) || !aligned(weight, pe) || !aligned(mean, 4) || !aligned(rstd, 4) ||
        !aligned(dweight, 4) || !aligned(dbias, 4) || !aligned(workspace, 16))
        return fail(HF_ERR_INVALID_ARG, "a pointer is not aligned");
    const cudaStream_t st = (cudaStream_t)stream;
    if (g->rows == 0) {
        const size_t n = (size_t)norm_groups(g) * g->width * sizeof(float);
        if (dweight) HFL_CUDA(cudaMemsetAsync(dweight, 0, n, st));
        if (dbias) HFL_CUDA(cudaMemsetAsync(dbias, 0, n, st));
        return HF_OK;
    }
    if (!dx && !dweight && !dbias) return HF_OK;
    if (!x || !dy || !mean || !rstd) return fail(HF_ERR_INVALID_ARG, "dy, x, mean or rstd is null");
    const Device* d;
    HFL_TRY(current_device(&d));
    const void* rows[3] = {x, dy, dx};
    const long long strides[3] = {g->x_stride, g->y_stride, g->dx_stride};
    const NormPlan n = norm_bwd_plan(g, norm_wide(g, rows, strides, 3, weight, nullptr), d->sm_count);
    if (n.group_blocks > 1 && (dweight || dbias) && !workspace) return fail(HF_ERR_INVALID_ARG, "workspace is null");
    NormParams p = {};
    p.x = x; p.dy = dy; p.y = dx; p.w = weight; p.mean = const_cast<float*>(mean); p.rstd = const_cast<float*>(rstd);
    p.partials = static_cast<float*>(workspace); p.dw = dweight; p.db = dbias;
    p.rows = g->rows; p.x_stride = g->x_stride; p.y_stride = g->y_stride; p.dx_stride = g->dx_stride;
    p.rows_per_group = g->rows_per_group; p.param_stride = g->param_stride;
    p.width = g->width; p.params_f32 = g->param_type == HF_F32; p.weight_offset = g->weight_offset; p.eps = g->eps; p.group_blocks = n.group_blocks;
    p.stages = n.stages; p.dev_status = d->status;
    if (g->type == HF_BF16) return launch_norm_bwd_of<bf16>(d, p, n, st);
    if (g->type == HF_F16) return launch_norm_bwd_of<__half>(d, p, n, st);
    return launch_norm_bwd_of<float>(d, p, n, st);
}

hf_status hf_rope_axes(const hf_rope_shape* g, const hf_rope_tensor* tensors, int n_tensors, const float* cos_tab, const float* sin_tab,
                       const int32_t* pos, void* stream) {
    if (!g || !tensors) return fail(HF_ERR_INVALID_ARG, "shape or tensors is null");
    if (g->type != HF_BF16 && g->type != HF_F16 && g->type != HF_F32) return fail(HF_ERR_UNSUPPORTED, "type %d unknown", g->type);
    if (g->pairing != HF_PAIRS_ADJACENT && g->pairing != HF_PAIRS_HALVES) return fail(HF_ERR_UNSUPPORTED, "pairing %d unknown", g->pairing);
    if (n_tensors < 1 || n_tensors > 3) return fail(HF_ERR_SHAPE, "%d tensors: one to three are taken", n_tensors);
    if (g->batch < 0 || g->tokens < 0) return fail(HF_ERR_SHAPE, "batch and tokens must be >= 0");
    if (g->head_dim < 2 || g->head_dim > 1024 || g->head_dim % 2) return fail(HF_ERR_SHAPE, "head_dim %d is not an even number in [2, 1024]", g->head_dim);
    if (g->axes < 1 || g->axes > 4) return fail(HF_ERR_SHAPE, "axes %d outside [1, 4]", g->axes);
    RopeParams p = {};
    long long entries = 0;
    for (int a = 0; a < g->axes; ++a) {
        if (g->pairs[a] < 0 || g->extent[a] < 1) return fail(HF_ERR_SHAPE, "axis %d: %d pairs, extent %d", a, g->pairs[a], g->extent[a]);
        p.first[a] = p.n_pairs; p.pairs[a] = g->pairs[a]; p.extent[a] = g->extent[a]; p.tab[a] = (int)entries;
        if (g->pairs[a] > g->head_dim / 2 - p.n_pairs) return fail(HF_ERR_SHAPE, "more than head_dim / 2 = %d pairs", g->head_dim / 2);
        p.n_pairs += g->pairs[a];
        entries += (long long)g->pairs[a] * g->extent[a];
        if (entries > 0x7fffffffLL) return fail(HF_ERR_SHAPE, "the tables have more than 2^31 entries");
    }
    if ((long long)g->batch * g->tokens == 0) return HF_OK;
    if (p.n_pairs && (!cos_tab || !sin_tab || !pos)) return fail(HF_ERR_INVALID_ARG, "cos_tab, sin_tab or pos is null");
    if (!aligned(cos_tab, 4) || !aligned(sin_tab, 4) || !aligned(pos, 4)) return fail(HF_ERR_INVALID_ARG, "a pointer is not aligned to its element");
    const int e = element_bytes(g->type);
    bool wide = g->head_dim * e % 32 == 0 || (g->pairing == HF_PAIRS_ADJACENT && g->head_dim * e % 16 == 0);
    if (g->pairing == HF_PAIRS_HALVES && p.n_pairs * e % 16 != 0) wide = false;
    for (int i = 0; i < n_tensors; ++i) {
        const hf_rope_tensor& t = tensors[i];
        if (t.heads < 0) return fail(HF_ERR_SHAPE, "tensor %d: heads must be >= 0", i);
        if (t.heads == 0) continue;
        if (!t.x || !t.y) return fail(HF_ERR_INVALID_ARG, "tensor %d is null", i);
        if (!aligned(t.x, e) || !aligned(t.y, e)) return fail(HF_ERR_INVALID_ARG, "tensor %d is not aligned to its element", i);
        const long long s[6] = {g->batch > 1 ? t.x_batch : 0, g->tokens > 1 ? t.x_token : 0, t.heads > 1 ? t.x_head : 0,
                                g->batch > 1 ? t.y_batch : 0, g->tokens > 1 ? t.y_token : 0, t.heads > 1 ? t.y_head : 0};
        for (long long v : s)
            if (!stride_ok(v, e)) wide = false;
        if (!aligned(t.x, 16) || !aligned(t.y, 16)) wide = false;
        p.t[p.n_tensors++] = {t.x, t.y, s[0], s[1], s[2], s[3], s[4], s[5], t.heads, t.rotate};
        if (t.heads > 0x7ffffff0 - p.total_heads) return fail(HF_ERR_SHAPE, "the tensors have more than 2^31 heads together");
        p.total_heads += t.heads;
    }
    if (p.total_heads == 0) return HF_OK;
    // (thread blocks of 256 threads; a thread takes at least two features)
    if ((long long)g->batch * g->tokens > 0x7ffffff0LL * 256 / (g->head_dim / 2)) return fail(HF_ERR_SHAPE, "too many tokens");
    const Device* d;
    HFL_TRY(current_device(&d));
    p.cos_tab = cos_tab; p.sin_tab = sin_tab; p.pos = pos; p.pos_batch = g->batch > 1 ? g->pos_batch : 0;
    p.axes = g->axes; p.batch = g->batch; p.tokens = g->tokens; p.head_dim = g->head_dim; p.inverse = g->inverse; p.dev_status = d->status;
    const cudaStream_t st = (cudaStream_t)stream;
    const bool halves = g->pairing == HF_PAIRS_HALVES;
    if (g->type == HF_BF16) return launch_rope_of<bf16>(p, halves, wide, d->sm_count, st);
    if (g->type == HF_F16) return launch_rope_of<__half>(p, halves, wide, d->sm_count, st);
    return launch_rope_of<float>(p, halves, wide, d->sm_count, st);
}

hf_status hf_layers_status(int* flags, int* detail) {
    const Device* d;
    HFL_TRY(current_device(&d));
    int h[2] = {0, 0};
    HFL_CUDA(cudaDeviceSynchronize());
    HFL_CUDA(cudaMemcpy(h, d->status, 8, cudaMemcpyDeviceToHost));
    if (flags) *flags = h[0];
    if (detail) *detail = h[1];
    if (h[0] == 0) return HF_OK;
    HFL_CUDA(cudaMemset(d->status, 0, 8));
    if (h[0] & HF_DEV_TIMEOUT_FLAG) return fail(HF_ERR_DEVICE_TIMEOUT, "a device-side wait ran out (flags %d, detail %d)", h[0], h[1]);
    return fail(HF_ERR_INVALID_ARG, "a position lay outside its table (token %d); position 0 was taken in its place", h[1]);
}

}  // extern "C"
