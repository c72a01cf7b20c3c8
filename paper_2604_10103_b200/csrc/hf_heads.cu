// Norms of q and k with the rotation and the split into heads: host side and the kernels' instantiations.
#include "hf_layers.h"
#include "k_heads.cuh"

using namespace hf_layers;

namespace {

// How a token's part is laid out over lanes: see k_heads.cuh.
struct HeadsPlan { int lanes, warps[3], teams[3], per_lane, threads; bool big; };

hf_status heads_check(const hf_heads_shape* g) {
    if (g == nullptr) return fail(HF_ERR_INVALID_ARG, "shape is null");
    if (g->type != HF_BF16 && g->type != HF_F16 && g->type != HF_F32) return fail(HF_ERR_UNSUPPORTED, "type %d unknown", g->type);
    if (g->param_type != g->type && g->param_type != HF_F32) return fail(HF_ERR_UNSUPPORTED, "param_type %d is neither the type nor HF_F32", g->param_type);
    if (g->pairing != HF_PAIRS_ADJACENT && g->pairing != HF_PAIRS_HALVES) return fail(HF_ERR_UNSUPPORTED, "pairing %d unknown", g->pairing);
    if (g->over != HF_NORM_OVER_HEAD && g->over != HF_NORM_OVER_WIDTH) return fail(HF_ERR_UNSUPPORTED, "over %d unknown", g->over);
    if (g->batch < 0 || g->tokens < 0 || (long long)g->batch * g->tokens > 0x7fffffffLL) return fail(HF_ERR_SHAPE, "batch x tokens outside [0, 2^31)");
    if (g->head_dim < 2 || g->head_dim > 256 || g->head_dim % 2) return fail(HF_ERR_SHAPE, "head_dim %d is not an even number in [2, 256]", g->head_dim);
    if (g->heads < 1 || g->kv_heads < 1 || g->kv_heads > g->heads) return fail(HF_ERR_SHAPE, "%d heads, %d kv_heads: 1 <= kv_heads <= heads", g->heads, g->kv_heads);
    // (as lanes hold them: head_dim in eights, up to a power of two of them)
    if (g->heads > 2048) return fail(HF_ERR_SHAPE, "%d heads: up to 2048", g->heads);
    int lanes = 1;
    while (8 * lanes < g->head_dim) lanes *= 2;
    if (g->heads * lanes * 8 > 16384) return fail(HF_ERR_SHAPE, "%d heads of %d: up to 16384 features (heads of a power of two from 8 on)", g->heads, g->head_dim);
    if (!(g->eps >= 0.f)) return fail(HF_ERR_SHAPE, "eps must be >= 0");
    if (g->axes < 1 || g->axes > 4) return fail(HF_ERR_SHAPE, "axes %d outside [1, 4]", g->axes);
    return HF_OK;
}
// The axes' part of the parameters.
hf_status heads_axes(const hf_heads_shape* g, HeadsParams* p) {
    long long entries = 0;
    for (int a = 0; a < g->axes; ++a) {
        if (g->pairs[a] < 0 || g->extent[a] < 1) return fail(HF_ERR_SHAPE, "axis %d: %d pairs, extent %d", a, g->pairs[a], g->extent[a]);
        p->first[a] = p->n_pairs; p->pairs[a] = g->pairs[a]; p->extent[a] = g->extent[a]; p->tab[a] = (int)entries;
        if (g->pairs[a] > g->head_dim / 2 - p->n_pairs) return fail(HF_ERR_SHAPE, "more than head_dim / 2 = %d pairs", g->head_dim / 2);
        p->n_pairs += g->pairs[a];
        entries += (long long)g->pairs[a] * g->extent[a];
        if (entries > 0x7fffffffLL) return fail(HF_ERR_SHAPE, "the tables have more than 2^31 entries");
    }
    return HF_OK;
}

// A warp a token's part where its heads fit in a lane's registers (`most` heads a lane), otherwise as many warps as that takes.
HeadsPlan heads_plan(const hf_heads_shape* g, bool wide) {
    HeadsPlan p;
    p.lanes = 1;
    while (8 * p.lanes < g->head_dim) p.lanes *= 2;
    const int per_warp = 32 / p.lanes, full = g->type == HF_F32 ? 4 : 6;
    auto warps = [&](int heads, int most) { return (heads + per_warp * most - 1) / (per_warp * most); };
    p.big = !wide || warps(g->heads, full) > 4;
    p.per_lane = p.big ? 4 : (warps(g->heads, 2) == 1 ? 2 : full);
    const int all = warps(g->heads, p.per_lane), block = all >= 4 ? all : 4 / all * all;       // warps of a thread block
    for (int i = 0; i < 3; ++i) {               // (shared key heads take fewer, so a thread block takes more tokens of theirs)
        p.warps[i] = warps(i ? g->kv_heads : g->heads, p.per_lane);
        p.teams[i] = block / p.warps[i];
    }
    p.threads = 32 * block;
    return p;
}
// Backward: thread blocks for q, k, v, by the time that they take (a head of v, which is copied, a quarter of one of q; by what they move it would be two
// thirds: 161 us instead of 144 for 32760 tokens of 12 + 24 heads of 128).
void heads_blocks(const hf_heads_shape* g, const HeadsPlan& n, int sms, int (&blocks)[3]) {
    const long long rows = (long long)g->batch * g->tokens, total = (long long)sms * ((n.big ? 512 : 256) / n.threads);
    const long long part[3] = {4LL * g->heads, 4LL * g->kv_heads, 1LL * g->kv_heads}, sum = part[0] + part[1] + part[2];
    for (int i = 0; i < 3; ++i) {           // (rounded down: one thread block too many would wait for the others' end)
        const long long all = (rows + n.teams[i] - 1) / n.teams[i];
        long long b = total * part[i] / sum;
        if (b > all) b = all;
        blocks[i] = b < 1 ? 1 : (int)b;
    }
}
int weight_width(const hf_heads_shape* g, int heads) { return g->over == HF_NORM_OVER_WIDTH ? heads * g->head_dim : g->head_dim; }

template <typename T, bool HALVES, bool WIDE, int HB, bool BIG>
hf_status launch_heads(const Device* d, const HeadsParams& p, const HeadsPlan& n, bool backward, int smem, cudaStream_t st) {
    if (!backward) {
        const long long rows = (long long)p.batch * p.tokens;
        k_heads<T, HALVES, WIDE, HB, BIG><<<dim3((unsigned)((rows + n.teams[0] - 1) / n.teams[0]), 3), n.threads, 0, st>>>(p);
    } else {
        struct Key {};
        const unsigned grid = p.blocks[0] + p.blocks[1] + p.blocks[2];
        if constexpr (WIDE && !BIG) {
            constexpr int MOST = 6144 * 4 + 4 * HEADS_SETS * (1024 + 2 * HB * 256 * sizeof(T));  // a row of the weight; four warps' angles and slots
            smem += n.threads / 32 * HEADS_SETS * (32 * n.lanes + 2 * HB * 256 * (int)sizeof(T));
            if (p.over_width) {
                HFL_TRY(allow_shared<Key>(d, k_heads_bwd_ring<T, HALVES, HB, true>, MOST));
                k_heads_bwd_ring<T, HALVES, HB, true><<<grid, n.threads, smem, st>>>(p);
            } else {
                struct HeadKey {};
                HFL_TRY(allow_shared<HeadKey>(d, k_heads_bwd_ring<T, HALVES, HB, false>, MOST));
                k_heads_bwd_ring<T, HALVES, HB, false><<<grid, n.threads, smem, st>>>(p);
            }
        } else {
            // (asked for whatever the row: beside the kernel's own shared memory one of 12225 features no longer fits in what a launch has unasked)
            HFL_TRY(allow_shared<Key>(d, k_heads_bwd<T, HALVES, WIDE, HB, BIG>, 16384 * 4));
            k_heads_bwd<T, HALVES, WIDE, HB, BIG><<<grid, n.threads, smem, st>>>(p);
        }
    }
    HFL_CUDA(cudaGetLastError());
    return HF_OK;
}
template <typename T, bool HALVES>
hf_status launch_heads(const Device* d, const HeadsParams& p, const HeadsPlan& n, bool wide, bool backward, int smem, cudaStream_t st) {
    constexpr int FULL = sizeof(T) == 4 ? 4 : 6;
    if (!wide) return launch_heads<T, HALVES, false, 4, true>(d, p, n, backward, smem, st);
    if (n.big) return launch_heads<T, HALVES, true, 4, true>(d, p, n, backward, smem, st);
    if (n.per_lane == 2) return launch_heads<T, HALVES, true, 2, false>(d, p, n, backward, smem, st);
    return launch_heads<T, HALVES, true, FULL, false>(d, p, n, backward, smem, st);
}
hf_status launch_heads(const Device* d, const hf_heads_shape* g, const HeadsParams& p, const HeadsPlan& n, bool wide, bool backward, int smem, cudaStream_t st) {
    const bool halves = g->pairing == HF_PAIRS_HALVES;
    if (g->type == HF_BF16) return halves ? launch_heads<bf16, true>(d, p, n, wide, backward, smem, st) : launch_heads<bf16, false>(d, p, n, wide, backward, smem, st);
    if (g->type == HF_F16) return halves ? launch_heads<__half, true>(d, p, n, wide, backward, smem, st) : launch_heads<__half, false>(d, p, n, wide, backward, smem, st);
    return halves ? launch_heads<float, true>(d, p, n, wide, backward, smem, st) : launch_heads<float, false>(d, p, n, wide, backward, smem, st);
}

void heads_layout(HeadsParams* p, const HeadsPlan& n) {
    p->lanes = n.lanes;
    for (int i = 0; i < 3; ++i) { p->warps[i] = n.warps[i]; p->teams[i] = n.teams[i]; }
}
// Parameters of both directions, and whether 16-byte accesses fit everywhere.
hf_status heads_params(const hf_heads_shape* g, const hf_heads_tensor* t, const void* rows, void* drows, const void* qw, const void* kw,
                       const float* cos_tab, const float* sin_tab, const int32_t* pos, HeadsParams* p, bool* wide) {
    HFL_TRY(heads_axes(g, p));
    if ((long long)g->batch * g->tokens == 0) return HF_OK;
    if (!rows) return fail(HF_ERR_INVALID_ARG, "rows is null");
    if (p->n_pairs && (!cos_tab || !sin_tab || !pos)) return fail(HF_ERR_INVALID_ARG, "cos_tab, sin_tab or pos is null");
    const int e = element_bytes(g->type), pe = element_bytes(g->param_type);
    if (!aligned(cos_tab, 4) || !aligned(sin_tab, 4) || !aligned(pos, 4) || !aligned(rows, e) || !aligned(drows, e) || !aligned(qw, pe) || !aligned(kw, pe))
        return fail(HF_ERR_INVALID_ARG, "a pointer is not aligned to its element");
    *wide = g->head_dim % 8 == 0 && (g->pairing == HF_PAIRS_ADJACENT || p->n_pairs % 4 == 0) && aligned(rows, 16) && aligned(drows, 16) && aligned(qw, 16) && aligned(kw, 16);
    const bool batches = g->batch > 1, tokens = g->tokens > 1;
    p->rows = rows; p->drows = drows;
    p->rows_b = batches ? g->rows_batch : 0; p->rows_t = tokens ? g->rows_token : 0;
    p->drows_b = batches ? g->grad_batch : 0; p->drows_t = tokens ? g->grad_token : 0;
    long long strides[13] = {p->rows_b, p->rows_t, drows ? p->drows_b : 0, drows ? p->drows_t : 0};
    for (int i = 0; i < 3; ++i) {
        if (!t[i].p || !aligned(t[i].p, e)) return fail(HF_ERR_INVALID_ARG, "tensor %d is null or not aligned to its element", i);
        p->heads[i] = i == 0 ? g->heads : g->kv_heads;
        p->t[i] = {t[i].p, batches ? t[i].batch : 0, tokens ? t[i].token : 0, p->heads[i] > 1 ? t[i].head : 0};
        strides[4 + 3 * i] = p->t[i].b; strides[5 + 3 * i] = p->t[i].t; strides[6 + 3 * i] = p->t[i].h;
        if (!aligned(t[i].p, 16)) *wide = false;
    }
    for (long long s : strides)
        if (s * e % 16 != 0) *wide = false;
    p->w[0] = qw; p->w[1] = kw; p->params_f32 = g->param_type == HF_F32; p->over_width = g->over == HF_NORM_OVER_WIDTH; p->eps = g->eps;
    p->cos_tab = cos_tab; p->sin_tab = sin_tab; p->pos = pos; p->pos_batch = batches ? g->pos_batch : 0;
    p->axes = g->axes; p->batch = g->batch; p->tokens = g->tokens; p->head_dim = g->head_dim;
    return HF_OK;
}

}  // namespace

extern "C" {

hf_status hf_split_heads_norm_rope(const hf_heads_shape* g, const void* rows, const void* q_weight, const void* k_weight, const float* cos_tab,
                                   const float* sin_tab, const int32_t* pos, const hf_heads_tensor* heads, void* stream) {
    HFL_TRY(heads_check(g));
    if (!heads) return fail(HF_ERR_INVALID_ARG, "heads is null");
    HeadsParams p = {};
    bool wide = false;
    HFL_TRY(heads_params(g, heads, rows, nullptr, q_weight, k_weight, cos_tab, sin_tab, pos, &p, &wide));
    if ((long long)g->batch * g->tokens == 0) return HF_OK;
    const Device* d;
    HFL_TRY(current_device(&d));
    const HeadsPlan n = heads_plan(g, wide);
    heads_layout(&p, n);
    p.dev_status = d->status;
    return launch_heads(d, g, p, n, wide, false, 0, (cudaStream_t)stream);
}

hf_status hf_split_heads_norm_rope_workspace(const hf_heads_shape* g, size_t* bytes) {
    HFL_TRY(heads_check(g));
    if (!bytes) return fail(HF_ERR_INVALID_ARG, "bytes is null");
    const Device* d;
    HFL_TRY(current_device(&d));
    *bytes = 0;
    for (int wide = 0; wide < 2; ++wide) {      // (the alignment of the tensors, which the shape does not say, changes the number of thread blocks)
        int blocks[3];
        heads_blocks(g, heads_plan(g, wide != 0), d->sm_count, blocks);
        const size_t need = ((size_t)blocks[0] * weight_width(g, g->heads) + (size_t)blocks[1] * weight_width(g, g->kv_heads)) * sizeof(float);
        if (need > *bytes) *bytes = need;
    }
    return HF_OK;
}

hf_status hf_split_heads_norm_rope_backward(const hf_heads_shape* g, const hf_heads_tensor* heads, const void* rows, const void* q_weight,
                                            const void* k_weight, const float* cos_tab, const float* sin_tab, const int32_t* pos, void* drows,
                                            float* dq_weight, float* dk_weight, void* workspace, void* stream) {
    HFL_TRY(heads_check(g));
    if (!heads) return fail(HF_ERR_INVALID_ARG, "heads is null");
    if (!aligned(dq_weight, 4) || !aligned(dk_weight, 4)) return fail(HF_ERR_INVALID_ARG, "dq_weight or dk_weight is not aligned");
    HeadsParams p = {};
    bool wide = false;
    HFL_TRY(heads_params(g, heads, rows, drows, q_weight, k_weight, cos_tab, sin_tab, pos, &p, &wide));
    const cudaStream_t st = (cudaStream_t)stream;
    const int wq = weight_width(g, g->heads), wk = weight_width(g, g->kv_heads);
    if ((long long)g->batch * g->tokens == 0) {
        if (dq_weight) HFL_CUDA(cudaMemsetAsync(dq_weight, 0, wq * sizeof(float), st));
        if (dk_weight) HFL_CUDA(cudaMemsetAsync(dk_weight, 0, wk * sizeof(float), st));
        return HF_OK;
    }
    if (!drows) return fail(HF_ERR_INVALID_ARG, "drows is null");
    if (!workspace || !aligned(workspace, 16)) return fail(HF_ERR_INVALID_ARG, "workspace is null or not 16-byte aligned");
    const Device* d;
    HFL_TRY(current_device(&d));
    const HeadsPlan n = heads_plan(g, wide);
    heads_layout(&p, n);
    p.dev_status = d->status; p.partials = static_cast<float*>(workspace);
    heads_blocks(g, n, d->sm_count, p.blocks);
    HFL_TRY(launch_heads(d, g, p, n, wide, true, wq * (int)sizeof(float), st));
    if (!dq_weight && !dk_weight) return HF_OK;
    return launch_after(k_heads_sum, dim3((wq + 31) / 32, 2), dim3(32, 32), 0, st, (const float*)p.partials, p.blocks[0], p.blocks[1], wq, wk, dq_weight, dk_weight);
}

}  // extern "C"
