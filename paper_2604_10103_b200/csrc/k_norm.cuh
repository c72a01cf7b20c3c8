// Layer norm over the rows of x [rows, width] and its gradients.
//   mean = sum x / D,  var = sum (x - mean)^2 / D,  rstd = 1 / sqrt(var + eps),  xhat = (x - mean) rstd
//   y = xhat a + b_g,  a = weight_offset + w_g,  g = the row's group
//   gh = dy a,  dx = rstd (gh - mean(gh) - xhat mean(gh xhat)),  dw_g = sum over the group's rows of dy xhat,  db_g = sum of dy
// All sums are float32.  A row stays in registers between its sums, so x (and dy) are read once; the variance is the mean of the squared
// differences from the mean, not a difference of two large sums, and the backward pass forms x - mean before it scales it, so a row's offset
// costs neither pass its accuracy.  Memory bounds the long calls (backward of 32760 x 1536 bf16 60.7 us, 5.0 TB/s: the main kernel 57, the partials'
// sums 3; forward of 28213 x 1456 34.5 us, 4.8 TB/s), the loads' latency the short ones (4680 x 1536 forward 9.5 us, one round of thread blocks).
// 16-bit rows that do not start on 16 bytes (28213 x 1455 bf16: 61 us forward, 130 backward) come out of shared memory a word and a shift a pair
// on every pass, and leave as words or, where a row starts in the middle of one, element by element.
#pragma once
#include "k_vec.cuh"
#include "tc5_common.cuh"

constexpr int NORM_TEAM_BYTES = 64 + 2 * 12 * 8;          // backward, per team: up to 8 barriers, two buffers of sums of up to 12 warps
constexpr int NORM_ROWS_TEAM_BYTES = 64 + 4 * 24 * 4;     // forward, many rows: up to 8 barriers, four sums of up to 24 warps
// Warps of a thread block of the backward kernel, by the columns of a thread (registers): short rows are bound by their latency, and want more.
__host__ __device__ constexpr int norm_bwd_warps(int columns) { return columns <= 16 ? 24 : 12; }

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
    int stages;                             // ... sets of rows in the ring
    int* dev_status;
};

// V parameters from column col of row g on; `two`: of a pair, whether there is a second.
template <typename T, int V, bool WIDE>
__device__ __forceinline__ void norm_params(const void* base, bool f32, long long row_at, int col, float (&out)[V], bool two) {
    if (f32) {
        const float* p = static_cast<const float*>(base) + row_at + col;
        if constexpr (WIDE) to_floats(load_vec<float, V>(p), out);
        else {
            out[0] = p[0];
            if constexpr (V == 2) out[1] = two ? p[1] : 0.f;
        }
    } else
        Row<T, V, WIDE>(static_cast<const T*>(base) + row_at).get(col, out, two);
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
// The row stays packed (at most 64 registers a thread for the row lengths of models, so that 4736 rows are at work at a time).
// WIDE: 16-byte pieces; otherwise 16-bit elements in pairs, whatever the rows' alignment, and floats one by one.
template <typename T, int V, int NV, int TPR, bool WIDE>
__global__ void __launch_bounds__(TPR == 32 ? 256 : TPR, TPR == 32 ? 4 : (TPR == 128 && NV * V <= 32 ? 8 : 1))
k_norm(const NormParams p) {
    __shared__ float s_sum[2][TPR / 32];
    const int t = TPR == 32 ? threadIdx.x & 31 : threadIdx.x;
    const long long row = TPR == 32 ? (long long)blockIdx.x * 8 + (threadIdx.x >> 5) : blockIdx.x;
    if (row >= p.rows) return;                  // (a whole warp; with TPR > 32 the grid is the rows)
    // (rows and rows_per_group fit 31 bits; a division of 64 costs a microsecond here)
    const long long at = p.rows_per_group ? (uint32_t)row / (uint32_t)p.rows_per_group * p.param_stride : 0;
    Vec<T, V> xv[NV];
    const Row<T, V, WIDE> x(static_cast<const T*>(p.x) + row * p.x_stride);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int col = (i * TPR + t) * V;
        if constexpr (WIDE) {
            if (col < p.width) xv[i] = load_vec<T, V>(x.p + col);
        } else {                                // (many short steps: no branch among them, so that their loads overlap)
            float f[V];
            x.get(col < p.width ? col : 0, f, col + 1 < p.width);
            if (col >= p.width) f[0] = 0.f;
            from_floats(xv[i], f);              // (exact: they were of this type)
        }
    }
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i)
        if (!WIDE || (i * TPR + t) * V < p.width) {
            float f[V];
            to_floats(xv[i], f);
#pragma unroll
            for (int j = 0; j < V; ++j) s += f[j];
        }
    const float mean = row_sum<TPR>(s, s_sum[0]) / (float)p.width;
    s = 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i) stay_packed(xv[i]);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int col = (i * TPR + t) * V;
        if (!WIDE || col < p.width) {
            float f[V];
            to_floats(xv[i], f);
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const float c = WIDE || col + j < p.width ? f[j] - mean : 0.f;
                s = fmaf(c, c, s);
            }
        }
    }
    const float rstd = 1.f / sqrtf(row_sum<TPR>(s, s_sum[1]) / (float)p.width + p.eps);
    if (t == 0) {
        if (p.mean) p.mean[row] = mean;
        if (p.rstd) p.rstd[row] = rstd;
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) stay_packed(xv[i]);
    T* y = static_cast<T*>(p.y) + row * p.y_stride;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        int col = (i * TPR + t) * V;
        if constexpr (WIDE) { if (col >= p.width) continue; }
        const bool in = col < p.width, two = col + 1 < p.width;
        if constexpr (!WIDE) col = in ? col : 0;
        float a[V], b[V], f[V];
#pragma unroll
        for (int j = 0; j < V; ++j) { a[j] = 1.f; b[j] = 0.f; }
        if (p.w) {
            norm_params<T, V, WIDE>(p.w, p.params_f32, at, col, a, two);
#pragma unroll
            for (int j = 0; j < V; ++j) a[j] += p.weight_offset;
        }
        if (p.b) norm_params<T, V, WIDE>(p.b, p.params_f32, at, col, b, two);
        to_floats(xv[i], f);
#pragma unroll
        for (int j = 0; j < V; ++j) f[j] = fmaf((f[j] - mean) * rstd, a[j], b[j]);
        if (in) put_floats<T, V, WIDE>(y + col, f, two);
    }
}

// A row that a bulk copy brings has not come yet.  The wait is bounded like every wait: a row that never comes leaves garbage, and the flag.  lost: a word
// of the team's, set by then; the team waits for no other row and asks for no more copies.  In the kernel or out of it (norm_wait), us with both: backward
// of 32760 x 1536 bf16 60.7 / 62.5, of 28213 x 1455 134.3 / 129.6, of 28213 x 1535 floats 100.7 / 94.9, forward 81.9 / 78.9.
__device__ __forceinline__ void norm_wait_slow(uint32_t bar, uint32_t phase, volatile int* lost, int* dev_status, int where) {
    if (*lost) return;
    const long long t0 = clock64();
    while (clock64() - t0 < tc5::WAIT_LIMIT_CYCLES)
        if (tc5::mbar_try_wait(bar, phase)) return;
    *lost = 1;
    atomicOr(dev_status, HF_DEV_TIMEOUT_FLAG);
    atomicExch(dev_status + 1, where);
}
__device__ __noinline__ void norm_wait_out(uint32_t bar, uint32_t phase, volatile int* lost, int* dev_status, int where) {
    norm_wait_slow(bar, phase, lost, dev_status, where);
}
template <bool WIDE>
__device__ __forceinline__ void norm_wait(uint32_t bar, uint32_t phase, volatile int* lost, int* dev_status, int where) {
    if (tc5::mbar_try_wait(bar, phase)) return;
    if constexpr (WIDE) { norm_wait_slow(bar, phase, lost, dev_status, where); }
    else { norm_wait_out(bar, phase, lost, dev_status, where); }
}
// Copies in flight land before their memory is used for something else, or the thread block leaves.
__device__ __forceinline__ void norm_drain(const volatile int* lost) {
    if (!*lost) return;
    const long long t0 = clock64();
    while (clock64() - t0 < 400000) {}
}

// The same for many rows: thread blocks stay, one a multiprocessor, and their teams of tpr threads walk the rows of a group (the factors and
// shifts of the group in shared memory), each with a ring of `stages` rows in shared memory that bulk copies fill: as k_norm_bwd does,
// which see.  A row's stage is free as soon as its elements are in the team's registers.
constexpr int NORM_ROWS_WARPS = 24;
template <typename T, int V, int NV, bool WIDE>
__global__ void __launch_bounds__(32 * NORM_ROWS_WARPS, 1)
k_norm_rows(const NormParams p) {
    extern __shared__ __align__(16) uint8_t s_raw[];    // factors [width], shifts [width] | per team: barriers, sums | rings
    const int t = threadIdx.x, tpr = blockDim.x, team = threadIdx.y, teams = blockDim.y, warps = tpr >> 5;
    const int nb = p.group_blocks, slot = blockIdx.x % nb;
    const long long g = blockIdx.x / nb, g0 = p.rows_per_group ? g * p.rows_per_group : 0;
    const long long g1 = p.rows_per_group ? min(p.rows, g0 + p.rows_per_group) : p.rows;
    const float inv = 1.f / (float)p.width;
    const int factor_bytes = (p.width * 4 + 4 + 15) / 16 * 16;
    float* s_a = reinterpret_cast<float*>(s_raw);
    float* s_b = reinterpret_cast<float*>(s_raw + factor_bytes);
    uint8_t* s_team = s_raw + 2 * factor_bytes + team * NORM_ROWS_TEAM_BYTES;
    float* s_sum = reinterpret_cast<float*>(s_team + 64);               // [2 rows in turn][sum, squares][warps of the team]
    const uint32_t row_bytes = p.width * sizeof(T), slot_bytes = WIDE ? row_bytes : (row_bytes + 30) / 16 * 16;
    uint8_t* s_ring = s_raw + 2 * factor_bytes + teams * NORM_ROWS_TEAM_BYTES + (size_t)team * p.stages * slot_bytes;
    const uint32_t bar = smem_u32(s_team), ring = smem_u32(s_ring);
    volatile int* lost = reinterpret_cast<volatile int*>(s_team + 60);         // (behind the barriers)
    const long long first = g0 + (long long)slot * teams, step = (long long)nb * teams;
    auto load = [&](long long row, int s) {
        const T* from = static_cast<const T*>(p.x) + row * p.x_stride;
        const uint32_t lead = WIDE ? 0 : (uint32_t)(reinterpret_cast<uintptr_t>(from) & 15), bytes = WIDE ? row_bytes : (lead + row_bytes + 15) / 16 * 16;
        tc5::mbar_expect_tx(bar + 8 * s, bytes);
        tc5::bulk_load(ring + s * slot_bytes, reinterpret_cast<const uint8_t*>(from) - lead, bytes, bar + 8 * s);
    };
    if (t == 0) {
        *lost = 0;
        for (int s = 0; s < p.stages; ++s) tc5::mbar_init(bar + 8 * s, 1);
        asm volatile("fence.mbarrier_init.release.cluster;\n" ::: "memory");
        for (int s = 0; s < p.stages && first + team + s * step < g1; ++s) load(first + team + s * step, s);
    }
    // (V 8: the first and the second four of a thread's eight columns apart, so that neighbouring threads read neighbouring 16 bytes)
    for (int c = team * tpr + t; c < p.width; c += teams * tpr) {
        float a[1] = {1.f}, b[1] = {0.f};
        if (p.w) { norm_params<T, 1, false>(p.w, p.params_f32, g * p.param_stride, c, a, false); a[0] += p.weight_offset; }
        if (p.b) norm_params<T, 1, false>(p.b, p.params_f32, g * p.param_stride, c, b, false);
        const int at = V == 8 ? (c >> 2 & 1) * (p.width / 2) + (c >> 3) * 4 + (c & 3) : c;
        s_a[at] = a[0]; s_b[at] = b[0];
    }
    __syncthreads();
    auto factors = [&](const float* from, int col, float (&a)[V]) {
        if constexpr (V == 8) {
            const float4 lo = *reinterpret_cast<const float4*>(from + col / 2), hi = *reinterpret_cast<const float4*>(from + p.width / 2 + col / 2);
            a[0] = lo.x; a[1] = lo.y; a[2] = lo.z; a[3] = lo.w; a[4] = hi.x; a[5] = hi.y; a[6] = hi.z; a[7] = hi.w;
        } else if constexpr (V == 2) {
            const float2 v = *reinterpret_cast<const float2*>(from + col);
            a[0] = v.x; a[1] = v.y;
        } else
            to_floats(load_vec<float, V>(from + col), a);
    };
    int stage = 0, buf = 0;
    uint32_t phase = 0;
    for (long long r0 = first; r0 < g1; r0 += step, buf ^= 1) {         // (the teams walk in step)
        const long long row = r0 + team;
        const bool on = row < g1;
        const T* gx = static_cast<const T*>(p.x) + row * p.x_stride;
        const Row<T, V, WIDE> x(s_ring + stage * slot_bytes, WIDE ? 0 : (uint32_t)(reinterpret_cast<uintptr_t>(gx) & 15));
        if (on) norm_wait<WIDE>(bar + 8 * stage, phase, lost, p.dev_status, 92);
        Vec<T, V> xv[NV];
        float s[V];
#pragma unroll
        for (int j = 0; j < V; ++j) s[j] = 0.f;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int col = (i * tpr + t) * V;
            float f[V];
            x.get(col < p.width ? col : 0, f, col + 1 < p.width);
            if (col >= p.width) {
#pragma unroll
                for (int j = 0; j < V; ++j) f[j] = 0.f;
            }
            from_floats(xv[i], f);              // (exact: they were of this type)
            vadd(s, f);
        }
        float* own = s_sum + buf * 2 * warps;
        float sum = warp_sum(vsum(s));
        if (tpr > 32) {
            if ((t & 31) == 0) own[t >> 5] = sum;
            __syncthreads();
            sum = 0.f;
            for (int w = 0; w < warps; ++w) sum += own[w];
        }
        // (every thread of the team has its elements)
        if (t == 0 && on && row + p.stages * step < g1 && !*lost) load(row + p.stages * step, stage);
        if (++stage == p.stages) { stage = 0; phase ^= 1; }
        // (a quotient that float32 holds comes out exactly, so that the mean of a row of one value is that value: the product with the
        // rounded reciprocal, refined once by its residual, which the fused multiply-add forms exactly)
        float mean = sum * inv;
        if (fabsf(mean) < INFINITY) mean = fmaf(fmaf(-mean, (float)p.width, sum), inv, mean);
#pragma unroll
        for (int j = 0; j < V; ++j) s[j] = 0.f;
#pragma unroll
        for (int i = 0; i < NV; ++i) stay_packed(xv[i]);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int col = (i * tpr + t) * V;
            float f[V];
            to_floats(xv[i], f);
#pragma unroll
            for (int j = 0; j < V; ++j) f[j] = (WIDE ? col : col + j) < p.width ? f[j] - mean : 0.f;
            vfma(s, f, f, s);
        }
        sum = warp_sum(vsum(s));
        if (tpr > 32) {
            if ((t & 31) == 0) own[warps + (t >> 5)] = sum;
            __syncthreads();
            sum = 0.f;
            for (int w = 0; w < warps; ++w) sum += own[warps + w];
        }
        const float rstd = 1.f / sqrtf(sum * inv + p.eps);
        if (!on) continue;
        if (t == 0) {
            if (p.mean) p.mean[row] = mean;
            if (p.rstd) p.rstd[row] = rstd;
        }
#pragma unroll
        for (int i = 0; i < NV; ++i) stay_packed(xv[i]);
        T* y = static_cast<T*>(p.y) + row * p.y_stride;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int col = (i * tpr + t) * V;
            const bool in = col < p.width;
            float f[V], a[V], b[V];
            to_floats(xv[i], f);
            factors(s_a, in ? col : 0, a);
            factors(s_b, in ? col : 0, b);
#pragma unroll
            for (int j = 0; j < V; ++j) f[j] = (f[j] - mean) * rstd;
            vfma(f, f, a, b);
            if (in) put_floats<T, V, WIDE>(y + col, f, col + 1 < p.width);
        }
    }
    norm_drain(lost);
}

// grid groups x thread blocks per group, block (tpr, teams): a team of tpr threads shares a row, each thread V NV columns of it, the same
// ones in every row, so that the sums over rows stay in its registers (2 V NV of them, at most 96); at the end the teams' sums are added in
// shared memory, in order, and a thread block writes one partial of the group's dw and db (the only one: dw and db themselves).  A row is
// read twice, for its sums and for dx, from where it lies: RING: each team has a ring of `stages` rows of x and dy in shared memory, filled by
// bulk copies, so memory's latency is hidden whatever the registers allow; otherwise (rows too long for that) from global memory, the second
// time out of the caches.  A team of one warp (rows of up to 1536 elements) needs no barrier.  WIDE: rows start on 16 bytes and are taken
// in such pieces; otherwise a copy takes the 16-byte units that hold the row, and threads take 16-bit elements in pairs, floats one by one.
template <typename T, int V, int NV, bool RING, bool WIDE>
__global__ void __launch_bounds__(32 * norm_bwd_warps(V * NV), 1)
k_norm_bwd(const NormParams p) {
    extern __shared__ __align__(16) uint8_t s_raw[];    // factors [width] | per team: barriers, sums | rings; at the end the teams' sums
    const int t = threadIdx.x, tpr = blockDim.x, team = threadIdx.y, teams = blockDim.y, warps = tpr >> 5;
    const int nb = p.group_blocks, slot = blockIdx.x % nb;
    const long long g = blockIdx.x / nb, g0 = p.rows_per_group ? g * p.rows_per_group : 0;
    const long long g1 = p.rows_per_group ? min(p.rows, g0 + p.rows_per_group) : p.rows;
    const float inv = 1.f / (float)p.width;
    const int factor_bytes = (p.width * 4 + 4 + 15) / 16 * 16;
    float* s_a = reinterpret_cast<float*>(s_raw);
    uint8_t* s_team = s_raw + factor_bytes + team * NORM_TEAM_BYTES;
    float2* s_sum = reinterpret_cast<float2*>(s_team + 64);             // [2][warps of the team]
    const uint32_t row_bytes = p.width * sizeof(T), slot_bytes = WIDE ? row_bytes : (row_bytes + 30) / 16 * 16;
    uint8_t* s_ring = s_raw + factor_bytes + teams * NORM_TEAM_BYTES + (size_t)team * p.stages * 2 * slot_bytes;
    const uint32_t bar = smem_u32(s_team), ring = smem_u32(s_ring);
    volatile int* lost = reinterpret_cast<volatile int*>(s_team + 60);         // (behind the barriers)
    const long long first = g0 + (long long)slot * teams, step = (long long)nb * teams;     // the thread block's rows, one for each team
    // one thread of the team: the copies of a row into stage s
    auto load = [&](long long row, int s) {
        const T* from[2] = {static_cast<const T*>(p.x) + row * p.x_stride, static_cast<const T*>(p.dy) + row * p.y_stride};
        uint32_t lead[2] = {0, 0}, bytes[2] = {row_bytes, row_bytes};
        if constexpr (!WIDE) {
            lead[0] = (uint32_t)(reinterpret_cast<uintptr_t>(from[0]) & 15); lead[1] = (uint32_t)(reinterpret_cast<uintptr_t>(from[1]) & 15);
            bytes[0] = (lead[0] + row_bytes + 15) / 16 * 16; bytes[1] = (lead[1] + row_bytes + 15) / 16 * 16;
        }
        tc5::mbar_expect_tx(bar + 8 * s, bytes[0] + bytes[1]);
#pragma unroll
        for (int i = 0; i < 2; ++i)
            tc5::bulk_load(ring + (2 * s + i) * slot_bytes, reinterpret_cast<const uint8_t*>(from[i]) - lead[i], bytes[i], bar + 8 * s);
    };
    if (RING && t == 0) {
        *lost = 0;
        for (int s = 0; s < p.stages; ++s) tc5::mbar_init(bar + 8 * s, 1);
        asm volatile("fence.mbarrier_init.release.cluster;\n" ::: "memory");
        for (int s = 0; s < p.stages && first + team + s * step < g1; ++s) load(first + team + s * step, s);
    }
    // (V 8: the first and the second four of a thread's eight columns apart, so that neighbouring threads read neighbouring 16 bytes)
    for (int c = team * tpr + t; c < p.width; c += teams * tpr) {
        float a[1] = {1.f};
        if (p.w) { norm_params<T, 1, false>(p.w, p.params_f32, g * p.param_stride, c, a, false); a[0] += p.weight_offset; }
        s_a[V == 8 ? (c >> 2 & 1) * (p.width / 2) + (c >> 3) * 4 + (c & 3) : c] = a[0];
    }
    if (V == 2 && t == 0 && team == 0) s_a[p.width] = 0.f;              // (the other half of an odd row's last pair: it meets a zero of dy)
    __syncthreads();
    auto load_factors = [&](int col, float (&a)[V]) {
        if constexpr (V == 8) {
            const float4 lo = *reinterpret_cast<const float4*>(s_a + col / 2), hi = *reinterpret_cast<const float4*>(s_a + p.width / 2 + col / 2);
            a[0] = lo.x; a[1] = lo.y; a[2] = lo.z; a[3] = lo.w; a[4] = hi.x; a[5] = hi.y; a[6] = hi.z; a[7] = hi.w;
        } else if constexpr (V == 2) {
            const float2 v = *reinterpret_cast<const float2*>(s_a + col);
            a[0] = v.x; a[1] = v.y;
        } else
            to_floats(load_vec<float, V>(s_a + col), a);
    };
    float accw[NV][V], accb[NV][V];
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int j = 0; j < V; ++j) { accw[i][j] = 0.f; accb[i][j] = 0.f; }
    float mean_next = 0.f, rstd_next = 0.f;             // one row ahead
    if (first + team < g1) { mean_next = p.mean[first + team]; rstd_next = p.rstd[first + team]; }
    int stage = 0, buf = 0;
    uint32_t phase = 0;
    long long before = g1;                              // the row before (at first none), whose stage is read no more once the team has met
    int before_stage = 0;
    for (long long r0 = first; r0 < g1; r0 += step, buf ^= 1) {         // (the teams walk in step)
        const long long row = r0 + team;
        const bool on = row < g1;
        const float rstd = rstd_next, neg = -mean_next;                 // xhat = (x + neg) rstd: an offset of the row costs its gradients nothing
        if (row + step < g1) { mean_next = p.mean[row + step]; rstd_next = p.rstd[row + step]; }
        const T* gx = static_cast<const T*>(p.x) + row * p.x_stride;
        const T* gd = static_cast<const T*>(p.dy) + row * p.y_stride;
        const uint8_t* slot_x = s_ring + 2 * stage * slot_bytes;
        const Row<T, V, WIDE> x = RING ? Row<T, V, WIDE>(slot_x, WIDE ? 0 : (uint32_t)(reinterpret_cast<uintptr_t>(gx) & 15)) : Row<T, V, WIDE>(gx);
        const Row<T, V, WIDE> dy = RING ? Row<T, V, WIDE>(slot_x + slot_bytes, WIDE ? 0 : (uint32_t)(reinterpret_cast<uintptr_t>(gd) & 15)) : Row<T, V, WIDE>(gd);
        if (RING && on) norm_wait<WIDE>(bar + 8 * stage, phase, lost, p.dev_status, 91);
        float s1[V], s2[V];
#pragma unroll
        for (int j = 0; j < V; ++j) { s1[j] = 0.f; s2[j] = 0.f; }
        if (on) {
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                int col = (i * tpr + t) * V;
                if constexpr (WIDE) { if (col >= p.width) continue; }
                float xf[V], d[V], gh[V], a[V];
                const bool in = col < p.width, two = col + 1 < p.width;
                if constexpr (!WIDE) col = in ? col : 0;        // (many short steps: no branch among them, so that their loads overlap)
                x.get(col, xf, two);
                dy.get(col, d, two);
                load_factors(col, a);
                if constexpr (!WIDE) { if (!in) d[0] = 0.f; }
                vadd(xf, neg);
                vmul(xf, rstd);
                vmul(gh, d, a);
                vfma(accw[i], d, xf, accw[i]);
                vadd(accb[i], d);
                vadd(s1, gh);
                vfma(s2, gh, xf, s2);
            }
        }
        float m1 = warp_sum(vsum(s1)), m2 = warp_sum(vsum(s2));
        if (tpr > 32) {
            // (two buffers in turn: a warp that writes one has passed the barrier behind which the others read the other)
            float2* own = s_sum + buf * warps;
            if ((t & 31) == 0) own[t >> 5] = make_float2(m1, m2);
            __syncthreads();
            m1 = 0.f; m2 = 0.f;
            for (int w = 0; w < warps; ++w) { const float2 o = own[w]; m1 += o.x; m2 += o.y; }
        }
        if constexpr (RING) {                           // (behind the sums every thread of the team has left the row before)
            if (t == 0 && before + p.stages * step < g1 && !*lost) load(before + p.stages * step, before_stage);
            before = row; before_stage = stage;
            if (++stage == p.stages) { stage = 0; phase ^= 1; }
        }
        if (!on || p.y == nullptr) continue;
        // dx = rstd gh - rstd m1 - xhat rstd m2
        const float c1 = -m1 * inv * rstd, c2 = -m2 * inv * rstd * rstd;
        T* dx = static_cast<T*>(p.y) + row * p.dx_stride;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            int col = (i * tpr + t) * V;
            if constexpr (WIDE) { if (col >= p.width) continue; }
            float xf[V], d[V], a[V];
            const bool in = col < p.width, two = col + 1 < p.width;
            if constexpr (!WIDE) col = in ? col : 0;
            x.get(col, xf, two);
            dy.get(col, d, two);
            load_factors(col, a);
            vadd(xf, neg);
            vmul(d, d, a);
            vfma(xf, xf, c2, c1);
            vfma(xf, d, rstd, xf);
            if (in) put_floats<T, V, WIDE>(dx + col, xf, two);
        }
    }
    if constexpr (RING) norm_drain(lost);
    if (p.dw == nullptr && p.db == nullptr) return;
    // the teams' sums: all to shared memory, then added column by column
    const int cols = V * NV * tpr;
    float* s_join = reinterpret_cast<float*>(s_raw);
    __syncthreads();
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int j = 0; j < V; ++j) {
            float* o = s_join + (size_t)team * 2 * cols + (i * V + j) * tpr + t;
            o[0] = accw[i][j];
            o[cols] = accb[i][j];
        }
    __syncthreads();
    const bool direct = nb == 1;
    for (int e = team * tpr + t; e < 2 * cols; e += teams * tpr) {
        const int which = e >= cols, at = e - which * cols, ij = at / tpr, tt = at - ij * tpr;
        const int col = (ij / V * tpr + tt) * V + ij % V;
        if (col >= p.width) continue;
        float v = 0.f;
        for (int q = 0; q < teams; ++q) v += s_join[(size_t)q * 2 * cols + e];
        float* out = direct ? (which ? p.db : p.dw) : p.partials;
        if (out) out[direct ? g * p.width + col : ((long long)blockIdx.x * 2 + which) * p.width + col] = v;
    }
}

// dw, db [groups, width] from the partials [groups, n, 2, width], always in the same order: 32 threads a column, then their sums.  blockIdx.y:
// group x (dw or db).
__global__ void __launch_bounds__(1024)
k_norm_bwd_sum(const float* partials, int n, int width, float* dw, float* db) {
    __shared__ float s[32][33];
    pdl_wait();
    const int col = blockIdx.x * 32 + threadIdx.x, g = blockIdx.y >> 1, which = blockIdx.y & 1;
    float* out = which ? db : dw;
    if (out == nullptr) return;
    const float* src = partials + ((size_t)g * n * 2 + which) * width + col;
    float a = 0.f;
    if (col < width) {
#pragma unroll 4
        for (int i = threadIdx.y; i < n; i += 32) a += src[(size_t)i * 2 * width];
    }
    s[threadIdx.y][threadIdx.x] = a;
    __syncthreads();
    // warp y adds column y's 32 sums
    const float v = warp_sum(s[threadIdx.x][threadIdx.y]);
    if (threadIdx.x == 0 && blockIdx.x * 32 + threadIdx.y < width) out[(size_t)g * width + blockIdx.x * 32 + threadIdx.y] = v;
}
