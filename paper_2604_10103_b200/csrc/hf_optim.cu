// The optimizer's step and the norm of many gradients: host side and the kernels' instantiations.
#include "hf_layers.h"
#include "k_optim.cuh"

#include <cmath>

using namespace hf_layers;

namespace {

// Tensors of a launch: as many as 32,764 bytes of parameters hold, or of two shorter tables, which are sent faster, where there are fewer (132 gradients: 52 us a call instead of 56).
constexpr int FEW = 32, SOME_ADAM = 100, MOST_ADAM = 300, SOME_NORM = 160, MOST_NORM = 1200;
constexpr long long MOST_CHUNKS = 0x7fffffff;

// Thread blocks of a launch: chunks, up to what the multiprocessors hold at a time (KERNEL: a type that stands for the instantiation).
template <typename KERNEL, typename F>
hf_status grid_for(const Device* d, F kernel, int threads, unsigned chunks, unsigned* grid) {
    static volatile int known[64];
    int per = known[d->index];
    if (!per) {
        HFL_CUDA(cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per, kernel, threads, 0));
        if (per < 1) per = 1;
        known[d->index] = per;
    }
    const unsigned most = (unsigned)(d->sm_count * per);
    *grid = chunks < most ? (chunks ? chunks : 1) : most;
    return HF_OK;
}

// Elements of a chunk: 2048 (a block of 256 for each warp) where that gives every multiprocessor few of them, up to `most` (what a chunk takes to look up is
// then spread over many blocks, and in 8 bits there is a next block to ask for; in 32 bits long chunks are no faster).
int adamw_chunk(const Device* d, const hf_adamw_tensor* t, int n, int most) {
    long long all = 0;
    for (int i = 0; i < n; ++i) all += t[i].n;
    int chunk = 2048;
    while (chunk < most && all / chunk > 16LL * d->sm_count) chunk *= 2;
    return chunk;
}

template <typename P, typename G, bool MASTER, bool BITS8, int CAP>
hf_status launch_adamw(const Device* d, const hf_adamw_step* g, const hf_adamw_tensor* t, int n, cudaStream_t st) {
    AdamParams<CAP> a;
    a.beta1 = (float)g->beta1; a.beta2 = (float)g->beta2; a.rest1 = (float)(1. - g->beta1); a.rest2 = (float)(1. - g->beta2);
    a.ln1 = std::log(g->beta1); a.ln2 = std::log(g->beta2); a.eps = (float)g->eps; a.seed = g->seed; a.factor = g->factor; a.counter = g->counter;
    a.n_tensors = 0; a.chunks = 0;
    a.chunk = adamw_chunk(d, t, n, BITS8 ? 65536 : 8192);
    for (int i = 0; i < n; ++i) {
        if (t[i].n == 0 && !t[i].step) continue;                        // (a tensor of no elements has its step counted)
        OptimTensor& o = a.t[a.n_tensors++];
        o.p = t[i].p; o.g = t[i].g; o.master = t[i].master; o.m = t[i].m; o.v = t[i].v; o.scales = reinterpret_cast<float2*>(t[i].scales);
        o.step = t[i].step; o.lr_at = t[i].lr_at; o.n = t[i].n; o.first_block = t[i].first_block; o.chunk0 = a.chunks;
        o.lr = (float)t[i].lr; o.decay = (float)t[i].weight_decay;
        o.wide = aligned(o.p, 8 * sizeof(P)) && aligned(o.g, 8 * sizeof(G)) && aligned(o.master, 32) && aligned(o.m, BITS8 ? 8 : 32) && aligned(o.v, BITS8 ? 8 : 32);
        a.chunks += (unsigned)((t[i].n + a.chunk - 1) / a.chunk);
    }
    if (a.n_tensors == 0) return HF_OK;
    auto kernel = k_adamw<P, G, MASTER, BITS8, CAP>;
    unsigned grid;
    struct Key {};
    HFL_TRY(grid_for<Key>(d, kernel, 32 * OPTIM_WARPS, a.chunks, &grid));
    kernel<<<grid, 32 * OPTIM_WARPS, 0, st>>>(a);
    HFL_CUDA(cudaGetLastError());
    return HF_OK;
}
template <typename P, typename G, bool MASTER, bool BITS8>
hf_status run_adamw(const Device* d, const hf_adamw_step* g, const hf_adamw_tensor* t, int n, cudaStream_t st) {
    if (n <= FEW) return launch_adamw<P, G, MASTER, BITS8, FEW>(d, g, t, n, st);
    if (n <= SOME_ADAM) return launch_adamw<P, G, MASTER, BITS8, SOME_ADAM>(d, g, t, n, st);
    for (int i = 0; i < n; i += MOST_ADAM)
        HFL_TRY((launch_adamw<P, G, MASTER, BITS8, MOST_ADAM>(d, g, t + i, n - i < MOST_ADAM ? n - i : MOST_ADAM, st)));
    return HF_OK;
}
template <bool BITS8>
hf_status run_adamw(const Device* d, const hf_adamw_step* g, const hf_adamw_tensor* t, int n, bool master, cudaStream_t st) {
    if (g->param_type == HF_F32) return run_adamw<float, float, false, BITS8>(d, g, t, n, st);
    if (g->grad_type == HF_F32) return master ? run_adamw<bf16, float, true, BITS8>(d, g, t, n, st) : run_adamw<bf16, float, false, BITS8>(d, g, t, n, st);
    return master ? run_adamw<bf16, bf16, true, BITS8>(d, g, t, n, st) : run_adamw<bf16, bf16, false, BITS8>(d, g, t, n, st);
}

hf_status adamw_check(const hf_adamw_step* g, const hf_adamw_tensor* t, int n) {
    if (g == nullptr || (t == nullptr && n > 0)) return fail(HF_ERR_INVALID_ARG, "step or tensors is null");
    if (n < 0) return fail(HF_ERR_SHAPE, "%d tensors", n);
    if (g->param_type != HF_BF16 && g->param_type != HF_F32) return fail(HF_ERR_UNSUPPORTED, "param_type %d: bf16 and f32 are taken", g->param_type);
    if (g->grad_type != g->param_type && g->grad_type != HF_F32) return fail(HF_ERR_UNSUPPORTED, "grad_type %d is neither the parameters' nor HF_F32", g->grad_type);
    if (g->state_bits != 32 && g->state_bits != 8) return fail(HF_ERR_UNSUPPORTED, "state_bits %d: 32 and 8 are taken", g->state_bits);
    if (!(g->beta1 >= 0. && g->beta1 < 1.) || !(g->beta2 >= 0. && g->beta2 < 1.)) return fail(HF_ERR_SHAPE, "betas lie in [0, 1)");
    if (!(g->eps >= 0. && g->eps <= 3e38)) return fail(HF_ERR_SHAPE, "eps must be >= 0 and finite");
    if (!aligned(g->factor, 4)) return fail(HF_ERR_INVALID_ARG, "factor is not aligned");
    const int pe = element_bytes(g->param_type), ge = element_bytes(g->grad_type), se = g->state_bits == 8 ? 1 : 4;
    bool first = true, master = false, counted = false;
    long long elements = 0;
    for (int i = 0; i < n; ++i) {
        const hf_adamw_tensor& o = t[i];
        if (o.n < 0) return fail(HF_ERR_SHAPE, "tensor %d: %lld elements", i, (long long)o.n);
        if (!aligned(o.step, 4)) return fail(HF_ERR_INVALID_ARG, "tensor %d: step is not aligned", i);
        if (o.step) counted = true;
        if (o.n == 0) continue;
        if (!o.p || !o.g || !o.m || !o.v || !o.step || (se == 1 && !o.scales)) return fail(HF_ERR_INVALID_ARG, "tensor %d: a pointer is null", i);
        if (!aligned(o.p, pe) || !aligned(o.g, ge) || !aligned(o.master, 4) || !aligned(o.m, se) || !aligned(o.v, se) || !aligned(o.scales, 8) ||
            !aligned(o.lr_at, 4))
            return fail(HF_ERR_INVALID_ARG, "tensor %d: a pointer is not aligned", i);
        if (o.master && g->param_type == HF_F32) return fail(HF_ERR_INVALID_ARG, "tensor %d: a float32 parameter has no master", i);
        if (first) { first = false; master = o.master != nullptr; }
        else if (master != (o.master != nullptr)) return fail(HF_ERR_INVALID_ARG, "the tensors of a call have masters together or not at all");
        elements += o.n;
        if (o.n > (1LL << 43) || elements > (1LL << 43)) return fail(HF_ERR_SHAPE, "more than 2^43 elements");
    }
    if (counted && (!g->counter || !aligned(g->counter, 4))) return fail(HF_ERR_INVALID_ARG, "counter is null or not aligned");
    return HF_OK;
}

template <int CAP>
hf_status launch_grad_norm(const Device* d, const hf_gradient* t, int n, double* partials, int* blocks, cudaStream_t st) {
    GradNormParams<CAP> a;
    a.n_tensors = 0; a.chunks = 0; a.partials = partials;
    for (int i = 0; i < n; ++i) {
        if (t[i].n == 0) continue;
        a.t[a.n_tensors++] = {t[i].p, t[i].n, a.chunks, t[i].type | (aligned(t[i].p, 16) ? 4 : 0)};
        a.chunks += (unsigned)((t[i].n + GNORM_CHUNK - 1) / GNORM_CHUNK);
    }
    *blocks = 0;
    if (a.n_tensors == 0) return HF_OK;
    const unsigned most = (unsigned)(8 * d->sm_count), grid = a.chunks < most ? a.chunks : most;
    k_grad_norm<CAP><<<grid, 256, 0, st>>>(a);
    HFL_CUDA(cudaGetLastError());
    *blocks = (int)grid;
    return HF_OK;
}

hf_status grad_norm_check(const hf_gradient* t, int n) {
    if (n < 0) return fail(HF_ERR_SHAPE, "%d tensors", n);
    if (t == nullptr && n > 0) return fail(HF_ERR_INVALID_ARG, "tensors is null");
    long long chunks = 0;
    for (int i = 0; i < n; ++i) {
        if (t[i].type != HF_BF16 && t[i].type != HF_F16 && t[i].type != HF_F32) return fail(HF_ERR_UNSUPPORTED, "tensor %d: type %d unknown", i, t[i].type);
        if (t[i].n < 0) return fail(HF_ERR_SHAPE, "tensor %d: %lld elements", i, (long long)t[i].n);
        if (t[i].n == 0) continue;
        if (!t[i].p || !aligned(t[i].p, element_bytes(t[i].type))) return fail(HF_ERR_INVALID_ARG, "tensor %d is null or not aligned to its element", i);
        chunks += (t[i].n - 1) / GNORM_CHUNK + 1;
        if (t[i].n > (1LL << 44) || chunks > MOST_CHUNKS) return fail(HF_ERR_SHAPE, "more than 2^44 elements");
    }
    return HF_OK;
}

}  // namespace

extern "C" {

hf_status hf_adamw(const hf_adamw_step* g, const hf_adamw_tensor* tensors, int n_tensors, void* stream) {
    HFL_TRY(adamw_check(g, tensors, n_tensors));
    bool master = false, any = false;
    for (int i = 0; i < n_tensors; ++i)
        if (tensors[i].n || tensors[i].step) { any = true; if (tensors[i].n) master = tensors[i].master != nullptr; }
    if (!any) return HF_OK;
    const Device* d;
    HFL_TRY(current_device(&d));
    const cudaStream_t st = (cudaStream_t)stream;
    return g->state_bits == 8 ? run_adamw<true>(d, g, tensors, n_tensors, master, st) : run_adamw<false>(d, g, tensors, n_tensors, master, st);
}

hf_status hf_gradient_norm_workspace(int n_tensors, size_t* bytes) {
    if (n_tensors < 0) return fail(HF_ERR_SHAPE, "%d tensors", n_tensors);
    if (!bytes) return fail(HF_ERR_INVALID_ARG, "bytes is null");
    const Device* d;
    HFL_TRY(current_device(&d));
    *bytes = (size_t)((n_tensors + MOST_NORM - 1) / MOST_NORM) * 8 * d->sm_count * sizeof(double);
    return HF_OK;
}

hf_status hf_gradient_norm(const hf_gradient* tensors, int n_tensors, float max_norm, float* out, void* workspace, void* stream) {
    HFL_TRY(grad_norm_check(tensors, n_tensors));
    if (!(max_norm >= 0.f)) return fail(HF_ERR_SHAPE, "max_norm must be >= 0");
    if (!out || !aligned(out, 4)) return fail(HF_ERR_INVALID_ARG, "out is null or not aligned");
    if (n_tensors && (!workspace || !aligned(workspace, 16))) return fail(HF_ERR_INVALID_ARG, "workspace is null or not 16-byte aligned");
    const Device* d;
    HFL_TRY(current_device(&d));
    const cudaStream_t st = (cudaStream_t)stream;
    double* partials = static_cast<double*>(workspace);
    int all = 0, blocks;
    if (n_tensors <= FEW) {
        HFL_TRY(launch_grad_norm<FEW>(d, tensors, n_tensors, partials, &blocks, st));
        all = blocks;
    } else if (n_tensors <= SOME_NORM) {
        HFL_TRY(launch_grad_norm<SOME_NORM>(d, tensors, n_tensors, partials, &blocks, st));
        all = blocks;
    } else
        for (int i = 0; i < n_tensors; i += MOST_NORM) {
            HFL_TRY(launch_grad_norm<MOST_NORM>(d, tensors + i, n_tensors - i < MOST_NORM ? n_tensors - i : MOST_NORM, partials + all, &blocks, st));
            all += blocks;
        }
    return launch_after(k_grad_norm_sum, dim3(1), dim3(256), 0, st, (const double*)partials, all, max_norm, out);
}

}  // extern "C"
