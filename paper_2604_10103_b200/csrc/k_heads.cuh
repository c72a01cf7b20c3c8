// From the rows of a fused projection [batch, tokens, (heads + 2 kv_heads) head_dim] to q, k, v: q and k scaled by 1 / rms and a weight, then
// rotated, v copied, in one pass; and back.
//   r = 1 / sqrt(mean x^2 + eps) over a head, or over all heads of the token;  q = R (x r w)   (R: the rotation by the token's position)
//   g = R^T dq,  dx = r (g w - x r mean(g w x r)),  dw = sum over tokens (and heads, where they share it) of g x r
// Sums are float32, each output is rounded once.  Memory bounds it: a token's part of q (or k) stays in its team's registers, packed, between
// its sums and its output, so everything is read once; r costs less to form again in the backward pass than to keep.
// A lane holds eight features (a unit) of a head, and the same ones of other heads: the angles, and the sums over a head, are in lanes of one warp (L of them, the
// power of two from head_dim / 8 on), the token's sum in the team's W warps.  Pairs (2p, 2p + 1): features 8 u ..; pairs (p, P + p): 4 u .. and
// P + 4 u ..; so a pair's two features are the same lane's.
// Backward: thread blocks stay and walk tokens, since the weight's gradient is a sum over them: in registers, then the thread block's in
// shared memory, its warps one after the other, then the thread blocks' in a second kernel, always in the same order.
#pragma once
#include "k_vec.cuh"

struct HeadsTensor { void* p; long long b, t, h; };         // q, k, v or their gradients: elements between batches, tokens, heads
struct HeadsParams {
    const void* rows; void* drows;
    long long rows_b, rows_t, drows_b, drows_t;
    HeadsTensor t[3];
    const void* w[2];                       // of q and k (nullptr: 1)
    int params_f32, over_width;
    float eps;
    const float* cos_tab; const float* sin_tab;
    const int* pos;
    long long pos_batch;
    int first[4], pairs[4], extent[4], tab[4];
    int axes, n_pairs;
    int batch, tokens, head_dim, heads[3];
    int lanes, warps, teams;                // of a unit's heads: L; of a team: W; teams of a thread block
    int blocks[3];                          // backward: thread blocks for each of the three
    float* partials;                        // backward: [thread blocks of q and k][row of the weight]
    int* dev_status;
};

// What a lane holds: which features, which heads.
template <typename T, bool HALVES, bool WIDE>
struct HeadsLane {
    int unit, f0, f1;
    bool on;
    __device__ __forceinline__ HeadsLane(const HeadsParams& p, int u) : unit(u) {
        on = 8 * u < p.head_dim;
        const bool turned = HALVES && 4 * u < p.n_pairs;        // (WIDE: a unit's pairs are all rotated or none of them)
        f0 = turned ? 4 * u : 8 * u;
        f1 = turned ? p.n_pairs + 4 * u : 8 * u + 4;
    }
    // Place of value i of the unit (not WIDE), -1 past the head's end.
    __device__ __forceinline__ int at(const HeadsParams& p, int i) const {
        int f;
        if constexpr (HALVES) {
            const int pair = 4 * unit + (i & 3);
            f = pair < p.n_pairs ? pair + (i >> 2) * p.n_pairs : 2 * pair + (i >> 2);
        } else
            f = 8 * unit + i;
        return f < p.head_dim ? f : -1;
    }
    __device__ __forceinline__ Vec<T, 8> load(const HeadsParams& p, const T* head) const {
        Vec<T, 8> r;
        if constexpr (!WIDE) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int f = at(p, i);
                r.v[i] = f >= 0 ? head[f] : from_float<T>(0.f);
            }
        } else if constexpr (HALVES) {
            const Vec<T, 4> a = load_vec<T, 4>(head + f0), b = load_vec<T, 4>(head + f1);
            memcpy(&r, &a, sizeof(a));
            memcpy(reinterpret_cast<char*>(&r) + sizeof(a), &b, sizeof(b));
        } else
            r = load_vec<T, 8>(head + f0);
        return r;
    }
    __device__ __forceinline__ void store(const HeadsParams& p, T* head, const float (&f)[8]) const {
        Vec<T, 8> r;
        from_floats(r, f);
        if constexpr (!WIDE) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int a = at(p, i);
                if (a >= 0) head[a] = r.v[i];
            }
        } else if constexpr (HALVES) {
            Vec<T, 4> a, b;
            memcpy(&a, &r, sizeof(a));
            memcpy(&b, reinterpret_cast<char*>(&r) + sizeof(a), sizeof(b));
            store_vec(head + f0, a);
            store_vec(head + f1, b);
        } else
            store_vec(head + f0, r);
    }
    // The weight's values for head h.
    __device__ __forceinline__ void weight(const HeadsParams& p, const void* w, int h, float (&f)[8]) const {
        if (w == nullptr) {
#pragma unroll
            for (int i = 0; i < 8; ++i) f[i] = 1.f;
            return;
        }
        const size_t row = p.over_width ? (size_t)h * p.head_dim : 0;
        if (p.params_f32) {
            HeadsLane<float, HALVES, WIDE> as_floats(p, unit);
            to_floats(as_floats.load(p, static_cast<const float*>(w) + row), f);
        } else
            to_floats(load(p, static_cast<const T*>(w) + row), f);
    }
    // Values i and j of pair k.
    static constexpr int first(int k) { return HALVES ? k : 2 * k; }
    static constexpr int second(int k) { return HALVES ? 4 + k : 2 * k + 1; }
};

struct HeadsAngles {
    float c[4], s[4];
    __device__ __forceinline__ HeadsAngles(const HeadsParams& p, int unit, int b, int tok) {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int pr = 4 * unit + k;
            c[k] = 1.f; s[k] = 0.f;
            if (pr < p.n_pairs) {
                int a = 0;
                while (a + 1 < p.axes && pr >= p.first[a + 1]) ++a;
                int at = p.pos[b * p.pos_batch + (long long)tok * p.axes + a];
                if ((unsigned)at >= (unsigned)p.extent[a]) {            // outside the table: no address is formed from it
                    atomicOr(p.dev_status, HF_DEV_BAD_INDEX_FLAG);
                    atomicExch(p.dev_status + 1, tok);
                    at = 0;
                }
                const int e = p.tab[a] + at * p.pairs[a] + pr - p.first[a];
                c[k] = p.cos_tab[e];
                s[k] = p.sin_tab[e];
            }
        }
    }
};
// x by the angles (INVERSE: back).  Pairs that are not rotated are left as they are (an infinity is not multiplied by a zero sine).
template <bool HALVES, bool INVERSE>
__device__ __forceinline__ void heads_turn(const HeadsParams& p, const HeadsAngles& a, int unit, float (&x)[8]) {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const int i = HALVES ? k : 2 * k, j = HALVES ? 4 + k : 2 * k + 1;
        const float s = INVERSE ? -a.s[k] : a.s[k], x0 = x[i], x1 = x[j];
        if (4 * unit + k < p.n_pairs) {
            x[i] = x0 * a.c[k] - x1 * s;
            x[j] = x0 * s + x1 * a.c[k];
        }
    }
}

// Sum over the n lanes that differ in the low bits.
__device__ __forceinline__ float heads_lanes_sum(float v, int n) {
    for (int o = 1; o < n; o <<= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}
// Sums over a team's lanes; every thread of the thread block calls it.  s: [2][teams W], one half for each call in turn.
template <int N>
__device__ __forceinline__ void heads_team_sum(float (&v)[N], int team, int warp, int warps, float* s) {
#pragma unroll
    for (int n = 0; n < N; ++n) v[n] = heads_lanes_sum(v[n], 32);
    if (warps == 1) return;
    if ((threadIdx.x & 31) == 0)
#pragma unroll
        for (int n = 0; n < N; ++n) s[(team * warps + warp) * N + n] = v[n];
    __syncthreads();
#pragma unroll
    for (int n = 0; n < N; ++n) v[n] = 0.f;
    for (int w = 0; w < warps; ++w)
#pragma unroll
        for (int n = 0; n < N; ++n) v[n] += s[(team * warps + w) * N + n];
}

// HB: heads of a lane.  Threads of a thread block: at most 128, or 512 (BIG).
template <typename T, bool HALVES, bool WIDE, int HB, bool BIG>
__global__ void __launch_bounds__(BIG ? 512 : 128)
k_heads(const __grid_constant__ HeadsParams p) {
    __shared__ float s_sum[16];
    const int part = blockIdx.y, heads = p.heads[part];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, team = warp / p.warps, team_warp = warp - team * p.warps;
    const long long row = (long long)blockIdx.x * p.teams + team, rows = (long long)p.batch * p.tokens;
    const bool live = row < rows;
    const int b = live ? (int)((uint32_t)row / (uint32_t)p.tokens) : 0, tok = live ? (int)row - b * p.tokens : 0;      // (rows fit 31 bits)
    const HeadsLane<T, HALVES, WIDE> l(p, lane & (p.lanes - 1));
    const bool on = live && l.on;
    const int per_warp = 32 / p.lanes, slices = p.warps * per_warp, slice = team_warp * per_warp + lane / p.lanes;
    const int before = part == 0 ? 0 : (part == 1 ? p.heads[0] : p.heads[0] + p.heads[1]);
    const T* x = static_cast<const T*>(p.rows) + b * p.rows_b + tok * p.rows_t + (size_t)before * p.head_dim;
    T* y = static_cast<T*>(p.t[part].p) + b * p.t[part].b + tok * p.t[part].t;
    Vec<T, 8> v[HB];
#pragma unroll
    for (int k = 0; k < HB; ++k) {
        const int h = k * slices + slice;
        if (on && h < heads) v[k] = l.load(p, x + (size_t)h * p.head_dim);
        else {
            const float zero[8] = {};
            from_floats(v[k], zero);
        }
    }
    if (part == 2) {
#pragma unroll
        for (int k = 0; k < HB; ++k) {
            const int h = k * slices + slice;
            float f[8];
            to_floats(v[k], f);
            if (on && h < heads) l.store(p, y + h * p.t[2].h, f);
        }
        return;
    }
    const HeadsAngles angles(p, on ? l.unit : 1 << 20, b, tok);
    const void* w = p.w[part];
    float all[1] = {0.f}, own[HB];
#pragma unroll
    for (int k = 0; k < HB; ++k) {
        float f[8];
        to_floats(v[k], f);
        own[k] = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) own[k] = fmaf(f[i], f[i], own[k]);
        all[0] += own[k];
    }
    if (p.over_width) {
        heads_team_sum(all, team, team_warp, p.warps, s_sum);
        all[0] = 1.f / sqrtf(all[0] / (float)(heads * p.head_dim) + p.eps);
    }
    float f_w[8];
    if (on && !p.over_width) l.weight(p, w, 0, f_w);
#pragma unroll
    for (int k = 0; k < HB; ++k) {
        const int h = k * slices + slice;
        const float r = p.over_width ? all[0] : 1.f / sqrtf(heads_lanes_sum(own[k], p.lanes) / (float)p.head_dim + p.eps);
        if (!on || h >= heads) continue;
        stay_packed(v[k]);
        if (p.over_width) l.weight(p, w, h, f_w);
        float f[8];
        to_floats(v[k], f);
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = f[i] * r * f_w[i];
        heads_turn<HALVES, false>(p, angles, l.unit, f);
        l.store(p, y + h * p.t[part].h, f);
    }
}

template <typename T, bool HALVES, bool WIDE, int HB, bool BIG>
__global__ void __launch_bounds__(BIG ? 512 : 128)
k_heads_bwd(const __grid_constant__ HeadsParams p) {
    extern __shared__ float s_dw[];             // a row of the weight
    __shared__ float s_sum[2][32];
    int part = 0, block = blockIdx.x;
    while (part < 2 && block >= p.blocks[part]) block -= p.blocks[part++];
    const int heads = p.heads[part];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, team = warp / p.warps, team_warp = warp - team * p.warps;
    const HeadsLane<T, HALVES, WIDE> l(p, lane & (p.lanes - 1));
    const int per_warp = 32 / p.lanes, slices = p.warps * per_warp, slice = team_warp * per_warp + lane / p.lanes;
    const int before = part == 0 ? 0 : (part == 1 ? p.heads[0] : p.heads[0] + p.heads[1]);
    const long long rows = (long long)p.batch * p.tokens, step = (long long)p.blocks[part] * p.teams;
    const void* w = part < 2 ? p.w[part] : nullptr;
    float acc[HB][8];
#pragma unroll
    for (int k = 0; k < HB; ++k)
#pragma unroll
        for (int i = 0; i < 8; ++i) acc[k][i] = 0.f;
    float f_w[8];
    if (l.on && !p.over_width) l.weight(p, w, 0, f_w);
    int turn = 0;
    for (long long row0 = (long long)block * p.teams; row0 < rows; row0 += step, turn ^= 1) {       // (the teams walk in step)
        const long long row = row0 + team;
        const bool on = row < rows && l.on;
        const int b = row < rows ? (int)((uint32_t)row / (uint32_t)p.tokens) : 0, tok = row < rows ? (int)row - b * p.tokens : 0;
        const T* x = static_cast<const T*>(p.rows) + b * p.rows_b + tok * p.rows_t + (size_t)before * p.head_dim;
        T* dx = static_cast<T*>(p.drows) + b * p.drows_b + tok * p.drows_t + (size_t)before * p.head_dim;
        const T* dy = static_cast<const T*>(p.t[part].p) + b * p.t[part].b + tok * p.t[part].t;
        Vec<T, 8> vg[HB], vx[HB];
        const float zero[8] = {};
#pragma unroll
        for (int k = 0; k < HB; ++k) {
            const int h = k * slices + slice;
            from_floats(vg[k], zero);
            from_floats(vx[k], zero);
            if (on && h < heads) {
                vg[k] = l.load(p, dy + h * p.t[part].h);
                if (part < 2) vx[k] = l.load(p, x + (size_t)h * p.head_dim);
            }
        }
        if (part == 2) {
#pragma unroll
            for (int k = 0; k < HB; ++k) {
                const int h = k * slices + slice;
                float f[8];
                to_floats(vg[k], f);
                if (on && h < heads) l.store(p, dx + (size_t)h * p.head_dim, f);
            }
            continue;
        }
        const HeadsAngles angles(p, on ? l.unit : 1 << 20, b, tok);
        float all[2] = {0.f, 0.f}, own[HB][2];
#pragma unroll
        for (int k = 0; k < HB; ++k) {
            const int h = k * slices + slice;
            float g[8], f[8];
            to_floats(vg[k], g);
            to_floats(vx[k], f);
            heads_turn<HALVES, true>(p, angles, l.unit, g);
            if (p.over_width && on && h < heads) l.weight(p, w, h, f_w);
            own[k][0] = 0.f; own[k][1] = 0.f;
            if (on && h < heads) {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    own[k][0] = fmaf(f[i], f[i], own[k][0]);
                    own[k][1] = fmaf(g[i] * f_w[i], f[i], own[k][1]);
                }
            }
            all[0] += own[k][0];
            all[1] += own[k][1];
        }
        float r = 0.f, c = 0.f;
        if (p.over_width) {
            heads_team_sum(all, team, team_warp, p.warps, s_sum[turn]);
            const float n = (float)(heads * p.head_dim);
            r = 1.f / sqrtf(all[0] / n + p.eps);
            c = all[1] * r / n;                 // mean(g w x r)
        }
#pragma unroll
        for (int k = 0; k < HB; ++k) {
            stay_packed(vg[k]);
            stay_packed(vx[k]);
        }
#pragma unroll
        for (int k = 0; k < HB; ++k) {
            const int h = k * slices + slice;
            if (!p.over_width) {
                const float n = (float)p.head_dim, square = heads_lanes_sum(own[k][0], p.lanes), product = heads_lanes_sum(own[k][1], p.lanes);
                r = 1.f / sqrtf(square / n + p.eps);
                c = product * r / n;
            }
            if (!on || h >= heads) continue;
            if (p.over_width) l.weight(p, w, h, f_w);
            float g[8], f[8];
            to_floats(vg[k], g);
            to_floats(vx[k], f);
            heads_turn<HALVES, true>(p, angles, l.unit, g);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float xh = f[i] * r;
                acc[k][i] = fmaf(g[i], xh, acc[k][i]);
                f[i] = r * (g[i] * f_w[i] - xh * c);
            }
            l.store(p, dx + (size_t)h * p.head_dim, f);
        }
    }
    if (part == 2) return;
    const int width = p.over_width ? heads * p.head_dim : p.head_dim;
    for (int i = threadIdx.x; i < width; i += blockDim.x) s_dw[i] = 0.f;
    if (!p.over_width) {                        // the heads share the weight: the lane's, then the slices of the warp
#pragma unroll
        for (int k = 1; k < HB; ++k)
#pragma unroll
            for (int i = 0; i < 8; ++i) acc[0][i] += acc[k][i];
#pragma unroll
        for (int i = 0; i < 8; ++i)
            for (int o = p.lanes; o < 32; o <<= 1) acc[0][i] += __shfl_xor_sync(0xffffffffu, acc[0][i], o);
    }
    for (int turn_of = 0; turn_of < (p.over_width ? p.teams : (int)blockDim.x / 32); ++turn_of) {
        __syncthreads();
        if (turn_of != (p.over_width ? team : warp) || !l.on || (!p.over_width && lane >= p.lanes)) continue;
#pragma unroll
        for (int k = 0; k < HB; ++k) {
            const int h = p.over_width ? k * slices + slice : 0;
            if (h >= heads || (!p.over_width && k > 0)) continue;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int at = WIDE ? (i < 4 ? l.f0 + i : l.f1 + i - 4) : l.at(p, i);
                if (at >= 0) s_dw[(size_t)h * p.head_dim + at] += acc[k][i];
            }
        }
    }
    __syncthreads();
    float* out = p.partials + (part == 0 ? (size_t)block * width : (size_t)p.blocks[0] * (p.over_width ? p.heads[0] * p.head_dim : p.head_dim) + (size_t)block * width);
    for (int i = threadIdx.x; i < width; i += blockDim.x) out[i] = s_dw[i];
}

// dw of q (blockIdx.y 0) and k: the thread blocks' sums, 32 threads a column, always in the same order.
__global__ void __launch_bounds__(1024)
k_heads_sum(const float* partials, int n_q, int n_k, int width_q, int width_k, float* dq, float* dk) {
    __shared__ float s[32][33];
    pdl_wait();
    const int n = blockIdx.y ? n_k : n_q, width = blockIdx.y ? width_k : width_q, col = blockIdx.x * 32 + threadIdx.x;
    float* out = blockIdx.y ? dk : dq;
    if (out == nullptr) return;
    const float* src = partials + (blockIdx.y ? (size_t)n_q * width_q : 0) + col;
    float a = 0.f;
    if (col < width) {
#pragma unroll 4
        for (int i = threadIdx.y; i < n; i += 32) a += src[(size_t)i * width];
    }
    s[threadIdx.y][threadIdx.x] = a;
    __syncthreads();
    const float v = heads_lanes_sum(s[threadIdx.x][threadIdx.y], 32);
    if (threadIdx.x == 0 && blockIdx.x * 32 + threadIdx.y < width) out[blockIdx.x * 32 + threadIdx.y] = v;
}
