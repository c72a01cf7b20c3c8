// The feed-forward's products for few rows of x (single tokens, short prompts): the weights are read once and bound the time, so they go
// straight from global memory to the registers that feed the (warp-level) tensor cores, all of a warp's loads in flight together.
//   GATED  h = act(x Wg^T) (x Wu^T): a thread block owns 8 hidden features; the 16 rows of an MMA are their 8 rows of Wg and 8 of Wu
//   PAIR   a linear layer with its epilogue: the 16 rows are 16 features, 8 of them w1's
//   else   y = h Wd^T: 8 rows of Wd, the MMA's other 8 rows stay zero (finer units keep more multiprocessors reading)
// The 8 columns of an MMA are 8 rows of x.  The warps of a thread block split the contraction, and their sums meet in shared memory, in
// order.  Sums are float32; h is rounded once between the products, as the tiled kernels round it.  A contraction index may be permuted if both operands are: lane (g, t) holds the 16 bytes at 32 j + 8 t of row g, and its four words
// serve as the two k-steps' fragments, so every load is 16 bytes.  The second product's weights are on their way before the first
// kernel has finished.  Width 1536, hidden 4096 (37.7 MB of weights, 5.8 us at the measured copy rate), weights from memory (in L2): one row
// 10.0 us (7.5) for both kernels (3.8 TB/s: two launches, and latency at their ends), 8 rows 10.8 (8.2), 16 rows 13.4 (11.1).  PAIR, one row of 1536 to 9216
// (28 MB, 4.3 us): 8.6 us (6.7).
#pragma once
#include "k_vec.cuh"

struct FfRowsParams {
    const void* x; const void* w0; const void* w1;      // w0: Wg or Wd, w1: Wu
    void* out; void* gate; void* up;                    // h or y; g, u (nullptr: not kept)
    long long x_stride, out_stride;
    int rows, contraction, features;
};
struct LinearRowsParams : FfRowsParams {                // (apart: as part of the feed-forward's they cost its two launches 1.4 us)
    LinearEpilogue linear;
    int act;
};

template <typename T> __device__ __forceinline__ void ff_mma_sync(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1);
template <> __device__ __forceinline__ void ff_mma_sync<bf16>(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    mma_bf16(c, a0, a1, a2, a3, b0, b1);
}
template <> __device__ __forceinline__ void ff_mma_sync<__half>(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};\n"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

template <typename T> __device__ __forceinline__ float linear_param(const void* base, bool f32, long long at) {
    return f32 ? static_cast<const float*>(base)[at] : to_float(static_cast<const T*>(base)[at]);
}
// The epilogue of one sum of a linear layer.
template <typename T> __device__ __forceinline__ void linear_one(const LinearEpilogue& e, int act, int row, int col, float v) {
    if (e.bias) v += linear_param<T>(e.bias, e.params_f32, col);
    if (e.pre) static_cast<T*>(e.pre)[row * e.pre_stride + col] = from_float<T>(v);
    v = act == HF_ACT_NONE ? v : (act == HF_ACT_SILU ? ff_act<HF_ACT_SILU>(v) : ff_act<HF_ACT_GELU_TANH>(v));
    const float gate = e.gate ? linear_param<T>(e.gate, e.params_f32, (long long)((uint32_t)row / (uint32_t)e.group) * e.gate_stride + col) : 1.f;
    const float residual = e.residual ? to_float(static_cast<const T*>(e.residual)[row * e.residual_stride + col]) : 0.f;
    static_cast<T*>(e.y)[row * e.y_stride + col] = from_float<T>(fmaf(v, gate, residual));
}

// NT: groups of 8 rows of x.  GATED: two products side by side, of two matrices or (LINEAR) of 16 features of one.  ACT: of GATED.
template <typename T, int NT, bool GATED, int ACT, bool LINEAR = false>
__global__ void __launch_bounds__(GATED ? 256 : 512, GATED ? 4 : 2)
k_ff_rows(const std::conditional_t<LINEAR, LinearRowsParams, FfRowsParams> p) {
    constexpr int WARPS = GATED ? 8 : 16, JB = GATED ? 6 : 8, MATS = GATED ? 2 : 1, OWN = LINEAR ? 8 * MATS : 8;
    __shared__ float s_sum[WARPS][MATS][8][8 * NT + 1];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const int feature = blockIdx.x * OWN + g, blocks = (p.contraction + 31) / 32;
    const bool on = feature < p.features, on1 = feature + 8 < p.features;
    const T* w0 = static_cast<const T*>(p.w0) + (size_t)feature * p.contraction + 8 * t;
    const T* w1 = static_cast<const T*>(p.w1) + (size_t)(feature + (LINEAR ? 8 : 0)) * p.contraction + 8 * t;
    const T* x = static_cast<const T*>(p.x) + 8 * t;
    float c[NT][4];
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i) c[n][i] = 0.f;
    constexpr bool FIRST = GATED || LINEAR;
    if (FIRST) { pdl_wait(); pdl_trigger(); }           // (what the first product reads may be the previous kernel's)
    bool waited = FIRST;
    for (int j0 = warp * JB; j0 < blocks || !waited; j0 += WARPS * JB) {
        uint4 a0[JB], a1[JB];
#pragma unroll
        for (int i = 0; i < JB; ++i) {
            a0[i] = make_uint4(0, 0, 0, 0); a1[i] = a0[i];
            if (on && 32 * (j0 + i) + 8 * t < p.contraction) {
                a0[i] = *reinterpret_cast<const uint4*>(w0 + 32 * (j0 + i));
                if (GATED && (!LINEAR || on1)) a1[i] = *reinterpret_cast<const uint4*>(w1 + 32 * (j0 + i));
            }
        }
        if constexpr (LINEAR) linear_touch(p.linear);
        if (!waited) { pdl_wait(); waited = true; }     // h is there; the weights above are no kernel's of this call
#pragma unroll
        for (int i = 0; i < JB; ++i) {
            if (j0 + i >= blocks) break;
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                uint4 b = make_uint4(0, 0, 0, 0);
                if (8 * n + g < p.rows && 32 * (j0 + i) + 8 * t < p.contraction)
                    b = *reinterpret_cast<const uint4*>(x + (size_t)(8 * n + g) * p.x_stride + 32 * (j0 + i));
                ff_mma_sync<T>(c[n], a0[i].x, a1[i].x, a0[i].y, a1[i].y, b.x, b.y);
                ff_mma_sync<T>(c[n], a0[i].z, a1[i].z, a0[i].w, a1[i].w, b.z, b.w);
            }
        }
    }
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            s_sum[warp][0][g][8 * n + 2 * t + i] = c[n][i];
            if (GATED) s_sum[warp][MATS - 1][g][8 * n + 2 * t + i] = c[n][2 + i];
        }
    __syncthreads();
    if constexpr (LINEAR) {
        for (int e = threadIdx.x; e < MATS * 64 * NT; e += 32 * WARPS) {
            const int f = e % OWN, row = e / OWN, col = blockIdx.x * OWN + f;
            if (row >= p.rows || col >= p.features) continue;
            float v = 0.f;
#pragma unroll
            for (int w = 0; w < WARPS; ++w) v += s_sum[w][f >> 3][f & 7][row];
            linear_one<T>(p.linear, p.act, row, col, v);
        }
    } else
    for (int e = threadIdx.x; e < 64 * NT; e += 32 * WARPS) {
        const int row = e >> 3, f = e & 7, col = blockIdx.x * 8 + f;
        if (row >= p.rows || col >= p.features) continue;
        float v0 = 0.f, v1 = 0.f;
#pragma unroll
        for (int w = 0; w < WARPS; ++w) {
            v0 += s_sum[w][0][f][row];
            if (GATED) v1 += s_sum[w][MATS - 1][f][row];
        }
        const size_t at = (size_t)row * p.features + col;
        if (GATED) {
            if (p.gate) {
                static_cast<T*>(p.gate)[at] = from_float<T>(v0);
                static_cast<T*>(p.up)[at] = from_float<T>(v1);
            }
            static_cast<T*>(p.out)[at] = from_float<T>(ff_act<ACT>(v0) * v1);
        } else
            static_cast<T*>(p.out)[(size_t)row * p.out_stride + col] = from_float<T>(v0);
    }
}
