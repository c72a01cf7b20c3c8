// The element-wise part of a linear layer's backward pass and its sums over rows.  From dy and pre = x W^T + b:
//   dp = dy gate act'(pre),  db = sum over the rows of dp,  dgate_g = sum over the group's rows of dy act(pre)
// dp is rounded to the type for the two products (dx = dp W, dW = dp^T x); the sums take it before.  Memory bounds it: dy and pre are read once, a lane
// takes eight neighbouring columns of every eighth row of its thread block's, and its sums stay in registers; the warps' meet in shared memory, the thread
// blocks' in a second kernel, in order.  Without activation and gate dp is dy, and only db is formed.
#pragma once
#include "k_ff_gemm.cuh"

struct LinearBwdParams {
    const void* dy; const void* pre; void* dp;          // dp [rows, cols] contiguous, pre too; nullptr: dp is dy
    const void* gate;
    long long dy_stride, gate_stride;
    float* db_part;                                     // [groups x parts][cols]; nullptr: not formed
    float* dgate_part;                                  // the same of dgate (parts == 1: dgate itself); nullptr: not formed
    int rows, cols, group, parts;                       // rows of a group; thread blocks that share a group's rows
    int params_f32;
};
constexpr int LINEAR_BWD_WARPS = 8, LINEAR_BWD_BLOCKS = 3;          // (thread blocks of a multiprocessor)

// grid: (groups x parts) x strips of 256 columns.  GATE: there is one (and its gradient may be asked for).  The arithmetic goes two columns an instruction: one by
// one, and with the gate's part always formed, it took the issue slots whole (311 us instead of 196, 6.2 TB/s, for 32760 rows of 6144 bf16, gelu).
template <typename T, int ACT, bool GATE>
__global__ void __launch_bounds__(32 * LINEAR_BWD_WARPS, LINEAR_BWD_BLOCKS)
k_linear_bwd(const LinearBwdParams p) {
    __shared__ float s_sum[LINEAR_BWD_WARPS][GATE ? 2 : 1][256];
    constexpr bool PRE = ACT != HF_ACT_NONE || GATE;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int col = blockIdx.y * 256 + 8 * lane;
    const int g = blockIdx.x / p.parts, part = blockIdx.x - g * p.parts;
    const int g0 = g * p.group, n = min(p.group, p.rows - g0);
    const int r0 = g0 + (int)((long long)n * part / p.parts), r1 = g0 + (int)((long long)n * (part + 1) / p.parts);
    float db[8], dgate[8], gate[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) { db[j] = 0.f; dgate[j] = 0.f; gate[j] = 1.f; }
    pdl_wait();
    pdl_trigger();
    if (col < p.cols) {
        if constexpr (GATE) linear_params<T>(p.gate, p.params_f32, g * p.gate_stride + col, gate);
        constexpr int U = 4;                            // rows in flight
        for (int r = r0 + warp; r < r1; r += U * LINEAR_BWD_WARPS) {
            Vec<T, 8> vd[U], vp[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const long long row = r + u * LINEAR_BWD_WARPS;
                if (row < r1) {
                    vd[u] = load_vec<T, 8>(static_cast<const T*>(p.dy) + row * p.dy_stride + col);
                    if constexpr (PRE) vp[u] = load_vec<T, 8>(static_cast<const T*>(p.pre) + row * p.cols + col);
                }
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const long long row = r + u * LINEAR_BWD_WARPS;
                if (row >= r1) break;
                float d[8], x[8];
                to_floats(vd[u], d);
                if constexpr (PRE) {
                    to_floats(vp[u], x);
#pragma unroll
                    for (int j = 0; j < 8; j += 2) {
                        float2 slope, dj = make_float2(d[j], d[j + 1]);
                        const float2 a = ff_act2<ACT, true>(make_float2(x[j], x[j + 1]), &slope);
                        if constexpr (GATE) {
                            const float2 s = ffma2(dj, a, make_float2(dgate[j], dgate[j + 1]));
                            dgate[j] = s.x; dgate[j + 1] = s.y;
                            dj = fmul2(dj, make_float2(gate[j], gate[j + 1]));
                        }
                        if constexpr (ACT != HF_ACT_NONE) dj = fmul2(dj, slope);
                        d[j] = dj.x; d[j + 1] = dj.y;
                    }
                }
                vadd(db, d);
                if (p.dp) {
                    Vec<T, 8> o;
                    from_floats(o, d);
                    store_vec(static_cast<T*>(p.dp) + row * p.cols + col, o);
                }
            }
        }
    }
    if (!p.db_part && !p.dgate_part) return;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        s_sum[warp][0][8 * lane + j] = db[j];
        if constexpr (GATE) s_sum[warp][1][8 * lane + j] = dgate[j];
    }
    __syncthreads();
    const int c = blockIdx.y * 256 + threadIdx.x;
    if (c >= p.cols) return;
#pragma unroll
    for (int which = 0; which < (GATE ? 2 : 1); ++which) {
        float* out = which ? p.dgate_part : p.db_part;
        if (!out) continue;
        float v = 0.f;
#pragma unroll
        for (int w = 0; w < LINEAR_BWD_WARPS; ++w) v += s_sum[w][which][threadIdx.x];
        out[(size_t)blockIdx.x * p.cols + c] = v;
    }
}

// db (blockIdx.x 0) and, where a group has several parts, dgate's rows: sums of `n` rows of a partial, 32 threads a column, in order.
__global__ void __launch_bounds__(1024)
k_linear_sum(const float* db_part, int n_db, float* db, const float* dgate_part, int parts, float* dgate, int cols) {
    __shared__ float s[32][33];
    pdl_wait();
    pdl_trigger();
    const bool of_gate = db == nullptr || blockIdx.x > 0;
    const int g = (int)blockIdx.x - (db != nullptr), n = of_gate ? parts : n_db, col = blockIdx.y * 32 + threadIdx.x;
    const float* src = of_gate ? dgate_part + (size_t)g * parts * cols : db_part;
    float* out = of_gate ? dgate + (size_t)g * cols : db;
    float a = 0.f;
    if (col < cols) {
#pragma unroll 4
        for (int i = threadIdx.y; i < n; i += 32) a += src[(size_t)i * cols + col];
    }
    s[threadIdx.y][threadIdx.x] = a;
    __syncthreads();
    float v = s[threadIdx.x][threadIdx.y];
#pragma unroll
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    if (threadIdx.x == 0 && blockIdx.y * 32 + threadIdx.y < cols) out[blockIdx.y * 32 + threadIdx.y] = v;
}
