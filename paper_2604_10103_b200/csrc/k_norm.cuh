// Layer norm over the rows of x [rows, width] and its gradients.
//   mean = sum x / D,  var = sum (x - mean)^2 / D,  rstd = 1 / sqrt(var + eps),  xhat = (x - mean) rstd
//   y = xhat a + b_g,  a = weight_offset + w_g,  g = the row's group
//   gh = dy a,  dx = rstd (gh - mean(gh) - xhat mean(gh xhat)),  dw_g = sum over the group's rows of dy xhat,  db_g = sum of dy
// All sums are float32.  A row stays in registers between its sums, so x (and dy) are read once; the variance is the mean of the squared
// differences from the mean, not a difference of two large sums.  Memory bounds all of it.
#pragma once
#include "k_vec.cuh"

struct NormParams {
    const void* x; void* y;                 // forward; backward: y = dx
    const void* dy;
    const void* w; const void* b;           // nullptr: factor 1, no bias
    float* mean; float* rstd;
    float* partials;                        // backward: [groups, group_blocks, 2, width]; with one thread block per group dw, db are written directly
    float* dw; float* db;                   // [groups, width]
    long long rows, x_stride, y_stride, dx_stride, rows_per_group, param_stride;
    int width;
    int params_f32;                         // w, b are float32, not of x's type
    float weight_offset, eps;
    int group_blocks;                       // backward: thread blocks per group
};

// V parameters from column col of row g on.
template <typename T, int V>
__device__ __forceinline__ void norm_params(const void* base, bool f32, long long row_at, int col, float (&out)[V]) {
    if (f32) {
        const Vec<float, V> p = *reinterpret_cast<const Vec<float, V>*>(static_cast<const float*>(base) + row_at + col);
#pragma unroll
        for (int j = 0; j < V; ++j) out[j] = p.v[j];
    } else {
        const Vec<T, V> p = *reinterpret_cast<const Vec<T, V>*>(static_cast<const T*>(base) + row_at + col);
#pragma unroll
        for (int j = 0; j < V; ++j) out[j] = to_float(p.v[j]);
    }
}

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}
// Sum over the TPR threads that share a row (a warp, or the whole thread block).
template <int TPR>
__device__ __forceinline__ float row_sum(float v, float* shared) {
    v = warp_sum(v);
    if constexpr (TPR > 32) {
        if ((threadIdx.x & 31) == 0) shared[threadIdx.x >> 5] = v;
        __syncthreads();
        v = 0.f;
#pragma unroll
        for (int w = 0; w < TPR / 32; ++w) v += shared[w];
    }
    return v;
}

// TPR threads share a row and hold V NV elements of it each.  TPR 32: eight rows a thread block of eight warps; otherwise one row.
template <typename T, int V, int NV, int TPR>
__global__ void __launch_bounds__(TPR == 32 ? 256 : TPR)
k_norm(const NormParams p) {
    __shared__ float s_sum[2][TPR / 32];
    const int t = TPR == 32 ? threadIdx.x & 31 : threadIdx.x;
    const long long row = TPR == 32 ? (long long)blockIdx.x * 8 + (threadIdx.x >> 5) : blockIdx.x;
    if (row >= p.rows) return;                  // (a whole warp; with TPR > 32 the grid is the rows)
    const T* x = static_cast<const T*>(p.x) + row * p.x_stride;
    Vec<T, V> xv[NV];
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int col = (i * TPR + t) * V;
        if (col < p.width) xv[i] = *reinterpret_cast<const Vec<T, V>*>(x + col);
    }
#pragma unroll
    for (int i = 0; i < NV; ++i)
        if ((i * TPR + t) * V < p.width)
#pragma unroll
            for (int j = 0; j < V; ++j) s += to_float(xv[i].v[j]);
    const float mean = row_sum<TPR>(s, s_sum[0]) / (float)p.width;
    s = 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i)
        if ((i * TPR + t) * V < p.width)
#pragma unroll
            for (int j = 0; j < V; ++j) { const float c = to_float(xv[i].v[j]) - mean; s = fmaf(c, c, s); }
    const float rstd = 1.f / sqrtf(row_sum<TPR>(s, s_sum[1]) / (float)p.width + p.eps);
    if (t == 0) {
        if (p.mean) p.mean[row] = mean;
        if (p.rstd) p.rstd[row] = rstd;
    }
    const long long at = p.rows_per_group ? row / p.rows_per_group * p.param_stride : 0;
    T* y = static_cast<T*>(p.y) + row * p.y_stride;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int col = (i * TPR + t) * V;
        if (col >= p.width) continue;
        float a[V], b[V];
#pragma unroll
        for (int j = 0; j < V; ++j) { a[j] = 1.f; b[j] = 0.f; }
        if (p.w) {
            norm_params<T, V>(p.w, p.params_f32, at, col, a);
#pragma unroll
            for (int j = 0; j < V; ++j) a[j] += p.weight_offset;
        }
        if (p.b) norm_params<T, V>(p.b, p.params_f32, at, col, b);
        Vec<T, V> o;
#pragma unroll
        for (int j = 0; j < V; ++j) o.v[j] = from_float<T>(fmaf((to_float(xv[i].v[j]) - mean) * rstd, a[j], b[j]));
        *reinterpret_cast<Vec<T, V>*>(y + col) = o;
    }
}

// Rows that a thread holds at a time: their loads are in flight together, and they share one barrier.
template <int NV, int V> __host__ __device__ constexpr int norm_bwd_rows() { return NV * V <= 8 ? 4 : (NV * V <= 16 ? 2 : 1); }

// grid groups x thread blocks per group, block (tpr, teams): a team of tpr threads shares a row, each thread V NV columns of it, the same
// ones in every row, so that the sums over rows stay in its registers; at the end the teams' sums are added in shared memory, in order,
// and a thread block writes one partial of the group's dw and db (the only one: dw and db themselves).  The teams walk in step.
template <typename T, int V, int NV>
__global__ void __launch_bounds__(512)
k_norm_bwd(const NormParams p) {
    constexpr int RB = norm_bwd_rows<NV, V>();
    extern __shared__ float s_dyn[];            // [2][teams][RB][warps of a team] float2, then (the same memory) [teams - 1][2][V NV tpr]
    const int t = threadIdx.x, tpr = blockDim.x, team = threadIdx.y, teams = blockDim.y, warps = tpr >> 5;
    const int nb = p.group_blocks, slot = blockIdx.x % nb;
    const long long g = blockIdx.x / nb, g0 = p.rows_per_group ? g * p.rows_per_group : 0;
    const long long g1 = p.rows_per_group ? min(p.rows, g0 + p.rows_per_group) : p.rows;
    const long long at = g * p.param_stride;
    const float inv = 1.f / (float)p.width;
    float accw[NV][V], accb[NV][V], a[NV][V];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
#pragma unroll
        for (int j = 0; j < V; ++j) { accw[i][j] = 0.f; accb[i][j] = 0.f; a[i][j] = 1.f; }
        const int col = (i * tpr + t) * V;
        if (p.w && col < p.width) {
            norm_params<T, V>(p.w, p.params_f32, at, col, a[i]);
#pragma unroll
            for (int j = 0; j < V; ++j) a[i][j] += p.weight_offset;
        }
    }
    float2* s_sum = reinterpret_cast<float2*>(s_dyn);
    int buf = 0;
    for (long long r0 = g0 + (long long)slot * teams * RB; r0 < g1; r0 += (long long)nb * teams * RB, buf ^= 1) {
        Vec<T, V> xv[RB][NV], dv[RB][NV];
        float mean[RB], rstd[RB];
        float2 s[RB];
#pragma unroll
        for (int k = 0; k < RB; ++k) {
            const long long row = r0 + k * teams + team;
            const bool on = row < g1;
            mean[k] = on ? p.mean[row] : 0.f;
            rstd[k] = on ? p.rstd[row] : 0.f;
            const T* x = static_cast<const T*>(p.x) + row * p.x_stride;
            const T* dy = static_cast<const T*>(p.dy) + row * p.y_stride;
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int col = (i * tpr + t) * V;
                if (on && col < p.width) {
                    xv[k][i] = *reinterpret_cast<const Vec<T, V>*>(x + col);
                    dv[k][i] = *reinterpret_cast<const Vec<T, V>*>(dy + col);
                } else {
#pragma unroll
                    for (int j = 0; j < V; ++j) { xv[k][i].v[j] = from_float<T>(0.f); dv[k][i].v[j] = from_float<T>(0.f); }
                }
            }
        }
#pragma unroll
        for (int k = 0; k < RB; ++k) {
            s[k] = make_float2(0.f, 0.f);
#pragma unroll
            for (int i = 0; i < NV; ++i)
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    const float xh = (to_float(xv[k][i].v[j]) - mean[k]) * rstd[k], d = to_float(dv[k][i].v[j]), gh = d * a[i][j];
                    accw[i][j] = fmaf(d, xh, accw[i][j]);
                    accb[i][j] += d;
                    s[k].x += gh;
                    s[k].y = fmaf(gh, xh, s[k].y);
                }
            s[k].x = warp_sum(s[k].x);
            s[k].y = warp_sum(s[k].y);
        }
        if (tpr > 32) {
            // (two buffers in turn: a warp that writes one has passed the barrier behind which the others read the other)
            float2* own = s_sum + (size_t)((buf * teams + team) * RB) * warps;
            if ((t & 31) == 0)
#pragma unroll
                for (int k = 0; k < RB; ++k) own[k * warps + (t >> 5)] = s[k];
            __syncthreads();
#pragma unroll
            for (int k = 0; k < RB; ++k) {
                s[k] = make_float2(0.f, 0.f);
                for (int w = 0; w < warps; ++w) { const float2 o = own[k * warps + w]; s[k].x += o.x; s[k].y += o.y; }
            }
        }
        if (p.y == nullptr) continue;
#pragma unroll
        for (int k = 0; k < RB; ++k) {
            const long long row = r0 + k * teams + team;
            T* dx = static_cast<T*>(p.y) + row * p.dx_stride;
            const float m1 = s[k].x * inv, m2 = s[k].y * inv;
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int col = (i * tpr + t) * V;
                if (row >= g1 || col >= p.width) continue;
                Vec<T, V> o;
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    const float xh = (to_float(xv[k][i].v[j]) - mean[k]) * rstd[k], gh = to_float(dv[k][i].v[j]) * a[i][j];
                    o.v[j] = from_float<T>(rstd[k] * (gh - m1 - xh * m2));
                }
                *reinterpret_cast<Vec<T, V>*>(dx + col) = o;
            }
        }
    }
    if (p.dw == nullptr && p.db == nullptr) return;
    // the teams' sums, one after the other
    const int cols = V * NV * tpr;
    if (teams > 1) {
        __syncthreads();
        if (team > 0)
#pragma unroll
            for (int i = 0; i < NV; ++i)
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    float* o = s_dyn + (size_t)(team - 1) * 2 * cols + (i * V + j) * tpr + t;
                    o[0] = accw[i][j];
                    o[cols] = accb[i][j];
                }
        __syncthreads();
        if (team > 0) return;
        for (int q = 0; q < teams - 1; ++q)
#pragma unroll
            for (int i = 0; i < NV; ++i)
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    const float* o = s_dyn + (size_t)q * 2 * cols + (i * V + j) * tpr + t;
                    accw[i][j] += o[0];
                    accb[i][j] += o[cols];
                }
    }
    const bool direct = nb == 1;
    float* ow = direct ? p.dw + g * p.width : p.partials + (long long)blockIdx.x * 2 * p.width;
    float* ob = direct ? p.db + g * p.width : ow + p.width;
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const int col = (i * tpr + t) * V + j;
            if (col >= p.width) continue;
            if (p.dw || !direct) ow[col] = accw[i][j];
            if (p.db || !direct) ob[col] = accb[i][j];
        }
}

// dw, db [groups, width] from the partials [groups, n, 2, width], always in the same order: 16 threads a column, then their sums.
__global__ void __launch_bounds__(512)
k_norm_bwd_sum(const float* partials, int n, int width, float* dw, float* db) {
    __shared__ float s[2][16][33];
    const int col = blockIdx.x * 32 + threadIdx.x;
    const float* src = partials + (size_t)blockIdx.y * n * 2 * width;
    float a = 0.f, b = 0.f;
    if (col < width)
        for (int i = threadIdx.y; i < n; i += 16) {
            a += src[(size_t)i * 2 * width + col];
            b += src[(size_t)i * 2 * width + width + col];
        }
    s[0][threadIdx.y][threadIdx.x] = a;
    s[1][threadIdx.y][threadIdx.x] = b;
    __syncthreads();
    if (threadIdx.y < 2 && col < width) {
        float v = 0.f;
#pragma unroll
        for (int q = 0; q < 16; ++q) v += s[threadIdx.y][q][threadIdx.x];
        float* out = threadIdx.y ? db : dw;
        if (out) out[(size_t)blockIdx.y * width + col] = v;
    }
}
