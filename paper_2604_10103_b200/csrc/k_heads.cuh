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
    int lanes, warps[3], teams[3];          // of a unit's heads: L; for each of the three, warps of a team W and teams of a thread block (warps behind them idle)
    int blocks[3];                          // backward: thread blocks for each of the three
    float* partials;                        // backward: [thread blocks of q and k][row of the weight]
    int* dev_status;
};

// A unit's eight values as floats in the order of the arithmetic, the first of each pair, then the second (two pairs an instruction), and back.
template <bool HALVES, typename T> __device__ __forceinline__ void heads_floats(const Vec<T, 8>& v, float (&f)[8]) {
    float raw[8];
    to_floats(v, raw);
#pragma unroll
    for (int j = 0; j < 4; ++j) { f[j] = raw[HALVES ? j : 2 * j]; f[4 + j] = raw[HALVES ? 4 + j : 2 * j + 1]; }
}
template <bool HALVES, typename T> __device__ __forceinline__ void heads_values(Vec<T, 8>& v, const float (&f)[8]) {
    float raw[8];
#pragma unroll
    for (int j = 0; j < 4; ++j) { raw[HALVES ? j : 2 * j] = f[j]; raw[HALVES ? 4 + j : 2 * j + 1] = f[4 + j]; }
    from_floats(v, raw);
}

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
        heads_values<HALVES>(r, f);
        store(p, head, r);
    }
    __device__ __forceinline__ void store(const HeadsParams& p, T* head, const Vec<T, 8>& r) const {
        if constexpr (!WIDE) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int a = at(p, i);
                if (a >= 0) head[a] = r.v[i];
            }
        } else if constexpr (HALVES) {
            Vec<T, 4> a, b;
            memcpy(&a, &r, sizeof(a));
            memcpy(&b, reinterpret_cast<const char*>(&r) + sizeof(a), sizeof(b));
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
            heads_floats<HALVES>(as_floats.load(p, static_cast<const float*>(w) + row), f);
        } else
            heads_floats<HALVES>(load(p, static_cast<const T*>(w) + row), f);
    }
    // Place of value i in the order of the arithmetic, -1 past the head's end.
    __device__ __forceinline__ int place(const HeadsParams& p, int i) const {
        const int raw = HALVES ? i : (i < 4 ? 2 * i : 2 * i - 7);
        if constexpr (WIDE) return raw < 4 ? f0 + raw : f1 + raw - 4;
        else return at(p, raw);
    }
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
// x by the angles (INVERSE: back).  Pairs that are not rotated are left as they are (an infinity is not multiplied by a zero sine): `turned`, one bit a
// pair.
template <bool INVERSE>
__device__ __forceinline__ void heads_turn(const float (&c)[4], const float (&s)[4], float (&x)[8]) {
#pragma unroll
    for (int k = 0; k < 4; k += 2) {
        const float2 x0 = make_float2(x[k], x[k + 1]), x1 = make_float2(x[4 + k], x[5 + k]), cc = make_float2(c[k], c[k + 1]);
        const float2 ss = make_float2(s[k], s[k + 1]), ns = make_float2(-s[k], -s[k + 1]);
        const float2 y0 = ffma2(x1, INVERSE ? ss : ns, fmul2(x0, cc)), y1 = ffma2(x0, INVERSE ? ns : ss, fmul2(x1, cc));
        x[k] = y0.x; x[k + 1] = y0.y; x[4 + k] = y1.x; x[5 + k] = y1.y;
    }
}
template <bool INVERSE>
__device__ __forceinline__ void heads_turn(const float (&c)[4], const float (&s)[4], int turned, float (&x)[8]) {
    float y[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = x[i];
    heads_turn<INVERSE>(c, s, y);
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = turned >> (i & 3) & 1 ? y[i] : x[i];
}
__device__ __forceinline__ int heads_turned(const HeadsParams& p, int unit) {
    const int n = p.n_pairs - 4 * unit;
    return n >= 4 ? 15 : (n <= 0 ? 0 : (1 << n) - 1);
}

// Sum over the n lanes that differ in the low bits.
__device__ __forceinline__ float heads_lanes_sum(float v, int n) {
    for (int o = 1; o < n; o <<= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}
// Sums over a team's lanes; every thread of the thread block calls it.  s: [2][warps of the thread block], one half for each call in turn.  The warps behind
// the last team come to the barrier and have no sums to read (there are fewer of them than a team has).
template <int N>
__device__ __forceinline__ void heads_team_sum(float (&v)[N], int team, int teams, int warp, int warps, float* s) {
#pragma unroll
    for (int n = 0; n < N; ++n) v[n] = heads_lanes_sum(v[n], 32);
    if (warps == 1) return;
    if ((threadIdx.x & 31) == 0)
#pragma unroll
        for (int n = 0; n < N; ++n) s[(team * warps + warp) * N + n] = v[n];
    __syncthreads();
    if (team >= teams) return;
#pragma unroll
    for (int n = 0; n < N; ++n) v[n] = 0.f;
    for (int w = 0; w < warps; ++w)
#pragma unroll
        for (int n = 0; n < N; ++n) v[n] += s[(team * warps + w) * N + n];
}

// A token's angles, looked up by the warp's lanes together (pairs lane, lane + 32, ...) into shared memory, cosines and then sines, from where each lane takes its
// unit's.  One lookup a pair: each lane's own four would be as many again in every slice of heads.
__device__ __forceinline__ void heads_look_up(const HeadsParams& p, int pairs, int b, int tok, float* s_angles) {
    const int lane = threadIdx.x & 31;
    const int* from = p.pos + b * p.pos_batch + (long long)tok * p.axes;
    for (int pr = lane; pr < pairs; pr += 32) {
        float c = 1.f, s = 0.f;
        if (pr < p.n_pairs) {
            int a = 0;
            while (a + 1 < p.axes && pr >= p.first[a + 1]) ++a;
            int at = from[a];
            if ((unsigned)at >= (unsigned)p.extent[a]) {                // outside the table: no address is formed from it
                atomicOr(p.dev_status, HF_DEV_BAD_INDEX_FLAG);
                atomicExch(p.dev_status + 1, tok);
                at = 0;
            }
            const int e = p.tab[a] + at * p.pairs[a] + pr - p.first[a];
            c = p.cos_tab[e];
            s = p.sin_tab[e];
        }
        s_angles[pr] = c;
        s_angles[pairs + pr] = s;
    }
}

// HB: heads of a lane.  Threads of a thread block: at most 128, or 512 (BIG).  4680 tokens of 12 + 24 heads of 128: 18.9 us with the inputs in L2, 23 from memory, where the loads'
// latency bounds it: a warp loads once, waits, computes and stores, a third of the warps are held, and half of the issue slots are used (13.6 M warp instructions:
// 12 us of the 592 schedulers).  With angles looked up by each lane, addresses formed anew for each head and selections for pairs that are not rotated 21.3 in L2.
template <typename T, bool HALVES, bool WIDE, int HB, bool BIG>
__global__ void __launch_bounds__(BIG ? 512 : 128)
k_heads(const __grid_constant__ HeadsParams p) {
    __shared__ float s_sum[16];
    __shared__ __align__(16) float s_angles[BIG ? 16 : 4][256];
    const int part = blockIdx.y, heads = p.heads[part];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = p.warps[part], team = warp / warps, team_warp = warp - team * warps;
    const uint32_t row = blockIdx.x * (uint32_t)p.teams[part] + team, rows = (uint32_t)p.batch * (uint32_t)p.tokens;
    if (blockIdx.x * (uint32_t)p.teams[part] >= rows) return;           // (the grid is for the part of fewest teams)
    const bool live = row < rows && team < p.teams[part];
    const int b = live ? (int)(row / (uint32_t)p.tokens) : 0, tok = live ? (int)(row - b * p.tokens) : 0;
    const HeadsLane<T, HALVES, WIDE> l(p, lane & (p.lanes - 1));
    const int per_warp = 32 / p.lanes, slices = warps * per_warp, slice = team_warp * per_warp + lane / p.lanes;
    const int before = part == 0 ? 0 : (part == 1 ? p.heads[0] : p.heads[0] + p.heads[1]);
    const T* x = static_cast<const T*>(p.rows) + b * p.rows_b + tok * p.rows_t + (before + slice) * p.head_dim;
    T* y = static_cast<T*>(p.t[part].p) + b * p.t[part].b + tok * p.t[part].t + slice * p.t[part].h;
    const int x_step = slices * p.head_dim;
    const long long y_step = slices * p.t[part].h;
    uint32_t mine = 0;                          // the lane's heads
#pragma unroll
    for (int k = 0; k < HB; ++k)
        if (live && l.on && k * slices + slice < heads) mine |= 1u << k;
    Vec<T, 8> v[HB];
#pragma unroll
    for (int k = 0; k < HB; ++k, x += x_step) {
        const float zero[8] = {};
        from_floats(v[k], zero);
        if (mine >> k & 1) v[k] = l.load(p, x);
    }
    if (part == 2) {
#pragma unroll
        for (int k = 0; k < HB; ++k, y += y_step)
            if (mine >> k & 1) l.store(p, y, v[k]);
        return;
    }
    const int pairs = 4 * p.lanes;
    if (live) heads_look_up(p, pairs, b, tok, s_angles[warp]);
    const void* w = p.w[part];
    const int turned = heads_turned(p, l.unit);
    const bool all_turned = 2 * p.n_pairs == p.head_dim && p.head_dim % 8 == 0;
    float all[1] = {0.f}, own[HB];
#pragma unroll
    for (int k = 0; k < HB; ++k) {
        float f[8];
        heads_floats<HALVES>(v[k], f);
        vmul(f, f, f);
        own[k] = vsum(f);
        all[0] += own[k];
    }
    if (p.over_width) {
        heads_team_sum(all, team, p.teams[part], team_warp, warps, s_sum);
        all[0] = 1.f / sqrtf(all[0] / (float)(heads * p.head_dim) + p.eps);
    }
    __syncwarp();
    float c[4], s[4], f_w[8];
    to_floats(load_vec<float, 4>(s_angles[warp] + 4 * l.unit), c);
    to_floats(load_vec<float, 4>(s_angles[warp] + pairs + 4 * l.unit), s);
    if (mine && !p.over_width) l.weight(p, w, 0, f_w);
#pragma unroll
    for (int k = 0; k < HB; ++k, y += y_step) {
        const float r = p.over_width ? all[0] : 1.f / sqrtf(heads_lanes_sum(own[k], p.lanes) / (float)p.head_dim + p.eps);
        if (!(mine >> k & 1)) continue;
        stay_packed(v[k]);
        if (p.over_width) l.weight(p, w, k * slices + slice, f_w);
        float f[8];
        heads_floats<HALVES>(v[k], f);
        vmul(f, r);
        vmul(f, f, f_w);
        if (all_turned) heads_turn<false>(c, s, f);
        else heads_turn<false>(c, s, turned, f);
        l.store(p, y, f);
    }
}

// The weight's gradient: the lanes' sums to the thread block's partial, its warps one after the other.  s_dw: a row of the weight, free for it.
template <typename T, bool HALVES, bool WIDE, int HB>
__device__ __forceinline__ void heads_weight_sum(const HeadsParams& p, const HeadsLane<T, HALVES, WIDE>& l, float (&acc)[HB][8], float* s_dw, int part, int block,
                                                 int team, int slices, int slice) {
    const int heads = p.heads[part], warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    __syncthreads();
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
    for (int turn_of = 0; turn_of < (p.over_width ? p.teams[part] : (int)blockDim.x / 32); ++turn_of) {
        __syncthreads();
        if (turn_of != (p.over_width ? team : warp) || !l.on || (!p.over_width && lane >= p.lanes)) continue;
#pragma unroll
        for (int k = 0; k < HB; ++k) {
            const int h = p.over_width ? k * slices + slice : 0;
            if (h >= heads || (!p.over_width && k > 0)) continue;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int at = l.place(p, i);
                if (at >= 0) s_dw[(size_t)h * p.head_dim + at] += acc[k][i];
            }
        }
    }
    __syncthreads();
    float* out = p.partials + (part == 0 ? (size_t)block * width : (size_t)p.blocks[0] * (p.over_width ? p.heads[0] * p.head_dim : p.head_dim) + (size_t)block * width);
    for (int i = threadIdx.x; i < width; i += blockDim.x) out[i] = s_dw[i];
}

template <typename T, bool HALVES, bool WIDE, int HB, bool BIG>
__global__ void __launch_bounds__(BIG ? 512 : 128)
k_heads_bwd(const __grid_constant__ HeadsParams p) {
    extern __shared__ float s_dw[];             // a row of the weight
    __shared__ float s_sum[2][32];
    int part = 0, block = blockIdx.x;
    while (part < 2 && block >= p.blocks[part]) block -= p.blocks[part++];
    const int heads = p.heads[part];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = p.warps[part], teams = p.teams[part], team = warp / warps, team_warp = warp - team * warps;
    const HeadsLane<T, HALVES, WIDE> l(p, lane & (p.lanes - 1));
    const int per_warp = 32 / p.lanes, slices = warps * per_warp, slice = team_warp * per_warp + lane / p.lanes;
    const int before = part == 0 ? 0 : (part == 1 ? p.heads[0] : p.heads[0] + p.heads[1]);
    const long long rows = (long long)p.batch * p.tokens, step = (long long)p.blocks[part] * teams;
    const void* w = part < 2 ? p.w[part] : nullptr;
    float acc[HB][8];
#pragma unroll
    for (int k = 0; k < HB; ++k)
#pragma unroll
        for (int i = 0; i < 8; ++i) acc[k][i] = 0.f;
    float f_w[8];
    if (l.on && !p.over_width) l.weight(p, w, 0, f_w);
    const int turned = heads_turned(p, l.unit);
    int turn = 0;
    for (long long row0 = (long long)block * teams; row0 < rows; row0 += step, turn ^= 1) {         // (the teams walk in step)
        const long long row = team < teams ? row0 + team : rows;
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
                if (on && h < heads) l.store(p, dx + (size_t)h * p.head_dim, vg[k]);
            }
            continue;
        }
        const HeadsAngles angles(p, on ? l.unit : 1 << 20, b, tok);
        float all[2] = {0.f, 0.f}, own[HB][2];
#pragma unroll
        for (int k = 0; k < HB; ++k) {
            const int h = k * slices + slice;
            float g[8], f[8];
            heads_floats<HALVES>(vg[k], g);
            heads_floats<HALVES>(vx[k], f);
            heads_turn<true>(angles.c, angles.s, turned, g);
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
            heads_team_sum(all, team, teams, team_warp, warps, s_sum[turn]);
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
            heads_floats<HALVES>(vg[k], g);
            heads_floats<HALVES>(vx[k], f);
            heads_turn<true>(angles.c, angles.s, turned, g);
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
    heads_weight_sum<T, HALVES, WIDE, HB>(p, l, acc, s_dw, part, block, team, slices, slice);
}

// The backward pass where 16-byte accesses fit and the heads of a token fit in four warps.  Each lane's pieces of the next token's dy and x, and its
// angles, are on their way into slots of shared memory (HEADS_SETS in turn) while it works on this one's, so nothing waits for memory; the pieces past the
// heads' end are zeros.  32760 tokens of 12 + 24 heads of 128, bf16: 144 us (5.6 TB/s); straight to registers with the weights from global memory 620.  A third
// set 147; three thread blocks a multiprocessor spill registers (218), or turn dy a second time instead of holding it (154).
__device__ __forceinline__ void heads_copy8(uint32_t dst, const void* src, bool valid) {
    const int sz = valid ? 8 : 0;
    asm volatile("cp.async.ca.shared.global [%0], [%1], 8, %2;\n" ::"r"(dst), "l"(src), "r"(sz));
}
__device__ __forceinline__ void heads_copy4(uint32_t dst, const void* src) {
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4;\n" ::"r"(dst), "l"(src));
}
constexpr int HEADS_SETS = 2;
template <typename T, bool HALVES, int HB, bool WIDTH>
__global__ void __launch_bounds__(128, 2)
k_heads_bwd_ring(const __grid_constant__ HeadsParams p) {
    extern __shared__ __align__(16) uint8_t s_raw[];            // weights [heads][first four, last four of each unit] | per warp: two sets of slots
    __shared__ float s_sum[2][32];
    __shared__ int4 s_axes[128];                // of each pair: axis, entries in a row of its table, its first entry
    constexpr int SETS = HEADS_SETS, SLOT = 32 * 8 * sizeof(T), SET = 2 * HB * SLOT;        // a warp's slot of a head: of each lane 8 values
    int part = 0, block = blockIdx.x;
    while (part < 2 && block >= p.blocks[part]) block -= p.blocks[part++];
    const int heads = p.heads[part], units = p.head_dim / 8;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = p.warps[part], teams = p.teams[part], team = warp / warps, team_warp = warp - team * warps;
    const HeadsLane<T, HALVES, true> l(p, lane & (p.lanes - 1));
    const int per_warp = 32 / p.lanes, slices = warps * per_warp, slice = team_warp * per_warp + lane / p.lanes;
    const int before = part == 0 ? 0 : (part == 1 ? p.heads[0] : p.heads[0] + p.heads[1]);
    const uint32_t rows = (uint32_t)p.batch * (uint32_t)p.tokens, step = (uint32_t)p.blocks[part] * (uint32_t)teams;
    const HeadsTensor dy_of = p.t[part];
    const T* dy = static_cast<const T*>(dy_of.p);
    const T* x = static_cast<const T*>(p.rows) + (size_t)before * p.head_dim;
    T* dx = static_cast<T*>(p.drows) + (size_t)before * p.head_dim;
    const uint32_t row0 = team < teams ? (uint32_t)block * teams + team : rows;
    // a lane's heads, and where the token of a row is: rows come in steps, so without a division
    uint32_t mine = 0;
#pragma unroll
    for (int k = 0; k < HB; ++k)
        if (l.on && k * slices + slice < heads) mine |= 1u << k;
    struct Place { uint32_t row; int b, tok; } at0;
    at0.row = row0; at0.b = row0 < rows ? row0 / (uint32_t)p.tokens : 0; at0.tok = row0 < rows ? row0 - at0.b * p.tokens : 0;
    const int step_b = (int)(step / (uint32_t)p.tokens), step_tok = (int)(step - step_b * (uint32_t)p.tokens);
    auto after = [&](const Place& a) {          // (past the end: it stays, for nothing)
        Place n = {a.row + step, a.b, a.tok};
        if (n.row < rows) {
            n.b += step_b; n.tok += step_tok;
            if (n.tok >= p.tokens) { n.tok -= p.tokens; ++n.b; }
        }
        return n;
    };
    if (part == 2) {
        // (several tokens' loads in flight: 110 rounds of one were what the call waited for)
        constexpr int U = sizeof(T) == 4 ? 2 : 4;
        Place a = at0;
        while (a.row < rows) {
            Vec<T, 8> v[U][HB];
            T* to[U];
            uint32_t on[U];
#pragma unroll
            for (int u = 0; u < U; ++u, a = after(a)) {
                const T* from = dy + a.b * dy_of.b + a.tok * dy_of.t + slice * dy_of.h;
                to[u] = dx + a.b * p.drows_b + a.tok * p.drows_t + slice * p.head_dim;
                on[u] = a.row < rows ? mine : 0u;
#pragma unroll
                for (int k = 0; k < HB; ++k)
                    if (on[u] >> k & 1) v[u][k] = l.load(p, from + k * (slices * dy_of.h));
            }
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int k = 0; k < HB; ++k)
                    if (on[u] >> k & 1) l.store(p, to[u] + k * (slices * p.head_dim), v[u][k]);
        }
        return;
    }
    const int w_rows = WIDTH ? heads : 1, width = w_rows * p.head_dim;
    float* s_w = reinterpret_cast<float*>(s_raw);
    const int pairs = 4 * p.lanes;              // (those past the rotated ones keep an angle of 0)
    float* s_angles = s_w + width + warp * SETS * 2 * pairs;            // sets of cosines and sines
    uint8_t* slots_gen = s_raw + ((size_t)width + blockDim.x / 32 * SETS * 2 * pairs) * 4 + warp * SETS * SET + lane * 8 * sizeof(T);
    const uint32_t slots = smem_u32(slots_gen);
    for (int i = warp; i < w_rows; i += blockDim.x / 32)
        if (lane < units) {
            const HeadsLane<T, HALVES, true> own(p, lane);
            float f[8];
            own.weight(p, p.w[part], i, f);
            float4* to = reinterpret_cast<float4*>(s_w + (size_t)i * p.head_dim) + lane;
            to[0] = make_float4(f[0], f[1], f[2], f[3]);
            to[units] = make_float4(f[4], f[5], f[6], f[7]);
        }
    for (int pr = threadIdx.x; pr < p.n_pairs; pr += blockDim.x) {
        int a = 0;
        while (a + 1 < p.axes && pr >= p.first[a + 1]) ++a;
        s_axes[pr] = make_int4(a, p.pairs[a], p.tab[a] + pr - p.first[a], 0);
    }
    for (int i = lane; i < SETS * 2 * pairs; i += 32) s_angles[i] = i / pairs & 1 ? 0.f : 1.f;
    // (slots that no copy fills are zeros from here on)
    for (int i = 0; i < SETS * 2 * HB; ++i)
#pragma unroll
        for (int q = 0; q < (int)sizeof(T) / 2; ++q) *reinterpret_cast<uint4*>(slots_gen + i * SLOT + 16 * q) = make_uint4(0, 0, 0, 0);
    __syncthreads();
    const float4* w_at = reinterpret_cast<const float4*>(s_w) + min(l.unit, units - 1);
    auto weight = [&](int k, float (&f)[8]) {
        const float4* from = w_at + (WIDTH ? (mine >> k & 1 ? k * slices + slice : 0) * 2 * units : 0);
        const float4 lo = from[0], hi = from[units];
        f[0] = lo.x; f[1] = lo.y; f[2] = lo.z; f[3] = lo.w; f[4] = hi.x; f[5] = hi.y; f[6] = hi.z; f[7] = hi.w;
    };
    const long long dy_step = (long long)slices * dy_of.h;
    const int x_step = slices * p.head_dim;
    // the token's angles: a lane asks for those of pairs lane, lane + 32, ..., whose positions it has asked for a round before
    int pos[4];
    auto ask_pos = [&](const Place& a) {
        const int* from = p.pos + a.b * p.pos_batch + (long long)a.tok * p.axes;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (lane + 32 * i < p.n_pairs) pos[i] = from[s_axes[lane + 32 * i].x];
    };
    auto ask_angles = [&](const Place& a, int set) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (lane + 32 * i < p.n_pairs) {
                const int4 axis = s_axes[lane + 32 * i];
                int row = pos[i];
                if ((unsigned)row >= (unsigned)p.extent[axis.x]) {      // outside the table: no address is formed from it
                    atomicOr(p.dev_status, HF_DEV_BAD_INDEX_FLAG);
                    atomicExch(p.dev_status + 1, a.tok);
                    row = 0;
                }
                const int e = axis.z + row * axis.y;
                const uint32_t to = smem_u32(s_angles + set * 2 * pairs + lane + 32 * i);
                heads_copy4(to, p.cos_tab + e);
                heads_copy4(to + 4 * pairs, p.sin_tab + e);
            }
    };
    auto ask = [&](const Place& a, int set) {
        ask_angles(a, set);
        const T* d = dy + a.b * dy_of.b + a.tok * dy_of.t + slice * dy_of.h;
        const T* f = x + a.b * p.rows_b + a.tok * p.rows_t + slice * p.head_dim;
        const bool live = a.row < rows;
        uint32_t to = slots + set * SET;
#pragma unroll
        for (int k = 0; k < HB; ++k, to += 2 * SLOT, d += dy_step, f += x_step) {
            if (!(mine >> k & 1)) continue;
            if constexpr (sizeof(T) == 4) {
                cp_async16(to, d + l.f0, live); cp_async16(to + 16, d + l.f1, live);
                cp_async16(to + SLOT, f + l.f0, live); cp_async16(to + SLOT + 16, f + l.f1, live);
            } else if constexpr (HALVES) {
                heads_copy8(to, d + l.f0, live); heads_copy8(to + 8, d + l.f1, live);
                heads_copy8(to + SLOT, f + l.f0, live); heads_copy8(to + SLOT + 8, f + l.f1, live);
            } else {
                cp_async16(to, d + l.f0, live);
                cp_async16(to + SLOT, f + l.f0, live);
            }
        }
        cp_async_commit();
    };
    auto get = [&](int set, int k, int i, float (&f)[8]) {
        heads_floats<HALVES>(load_vec<T, 8>(reinterpret_cast<const T*>(slots_gen + set * SET + (2 * k + i) * SLOT)), f);
    };
    const int turned = heads_turned(p, l.unit);
    const bool all_turned = 2 * p.n_pairs == p.head_dim;
    // SETS - 1 tokens ahead; of the one after those the positions
    Place here = at0, ahead = at0;
    ask_pos(ahead);
#pragma unroll
    for (int i = 0; i + 1 < SETS; ++i) {
        ask(ahead, i);
        ahead = after(ahead);
        ask_pos(ahead);
    }
    constexpr int KEPT = WIDTH ? HB : 1;        // (heads that share a weight share its sums)
    float acc[KEPT][8];
#pragma unroll
    for (int k = 0; k < KEPT; ++k)
#pragma unroll
        for (int i = 0; i < 8; ++i) acc[k][i] = 0.f;
    int set = 0, set_ahead = SETS - 1, turn = 0;
    const float inv = 1.f / (float)(WIDTH ? heads * p.head_dim : p.head_dim);
    // (the teams walk in step: as many rounds for each)
    for (uint32_t first = (uint32_t)block * teams; first < rows; first += step, turn ^= 1) {
        __syncwarp();                           // (the angles of the round before have been read)
        ask(ahead, set_ahead);
        ahead = after(ahead);
        ask_pos(ahead);
        cp_async_wait<SETS - 1>();
        __syncwarp();
        float c4[4], s4[4];
        to_floats(load_vec<float, 4>(s_angles + set * 2 * pairs + 4 * l.unit), c4);
        to_floats(load_vec<float, 4>(s_angles + set * 2 * pairs + pairs + 4 * l.unit), s4);
        auto turn_back = [&](float (&g)[8]) {   // R^T dy
            if (all_turned) heads_turn<true>(c4, s4, g);
            else heads_turn<true>(c4, s4, turned, g);
        };
        const bool live = here.row < rows;
        T* to = dx + here.b * p.drows_b + here.tok * p.drows_t + slice * p.head_dim;
        // f = x, w, r, c = mean(g w x r): the head's part of the weight's gradient, and its dx
        auto finish = [&](float (&f)[8], float (&w)[8], const float (&g)[8], float r, float c, float (&sum)[8], T* at) {
            vmul(f, r);
            vfma(sum, g, f, sum);
            vmul(w, w, g);
            vfma(f, f, -c, w);                  // g w - x r mean
            vmul(f, r);
            l.store(p, at, f);
        };
        if constexpr (WIDTH) {
            float g[HB][8], s1[8], s2[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) { s1[i] = 0.f; s2[i] = 0.f; }
#pragma unroll
            for (int k = 0; k < HB; ++k) {
                float f[8], w[8];
                get(set, k, 0, g[k]);
                get(set, k, 1, f);
                weight(k, w);
                turn_back(g[k]);
                vmul(w, g[k], w);
                vfma(s1, f, f, s1);
                vfma(s2, w, f, s2);
            }
            float all[2] = {vsum(s1), vsum(s2)};
            heads_team_sum(all, team, teams, team_warp, warps, s_sum[turn]);
            const float r = 1.f / sqrtf(all[0] * inv + p.eps), c = all[1] * r * inv;
#pragma unroll
            for (int k = 0; k < HB; ++k, to += x_step) {
                if (!live || !(mine >> k & 1)) continue;
                float f[8], w[8];
                get(set, k, 1, f);
                weight(k, w);
                finish(f, w, g[k], r, c, acc[k], to);
            }
        } else {
            float w0[8];
            weight(0, w0);
#pragma unroll
            for (int k = 0; k < HB; ++k, to += x_step) {
                float g[8], f[8], w[8], s1[8], s2[8];
                get(set, k, 0, g);
                get(set, k, 1, f);
                turn_back(g);
                vmul(w, g, w0);
                vmul(s1, f, f);
                vmul(s2, w, f);
                const float square = heads_lanes_sum(vsum(s1), p.lanes), product = heads_lanes_sum(vsum(s2), p.lanes);
                const float r = 1.f / sqrtf(square * inv + p.eps), c = product * r * inv;
                if (!live || !(mine >> k & 1)) continue;
#pragma unroll
                for (int i = 0; i < 8; ++i) w[i] = w0[i];
                finish(f, w, g, r, c, acc[0], to);
            }
        }
        here = after(here);
        if (++set == SETS) set = 0;
        if (++set_ahead == SETS) set_ahead = 0;
    }
    cp_async_wait<0>();
    heads_weight_sum<T, HALVES, true, KEPT>(p, l, acc, reinterpret_cast<float*>(s_raw), part, block, team, slices, slice);
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
