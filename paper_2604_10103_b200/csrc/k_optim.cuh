// The optimizer's step over many tensors and the norm of many gradients, each over all tensors in one launch: a table of tensors travels as
// the kernel's parameter, so nothing is copied to the device before, and thread blocks walk chunks of all tensors one after the other.
//   AdamW, step t of a tensor:  g = factor grad,  m = b1 m + (1 - b1) g,  v = b2 v + (1 - b2) g^2,
//     p = p - lr ((m / (1 - b1^t)) / (sqrt(v / (1 - b2^t)) + eps) + wd p)
// Everything is float32; a bf16 parameter is rounded once, and may have a float32 master that is not.  Memory bounds it: each element is read and
// written once, a warp a block of 256 elements, eight neighbours a lane.
// States in 8 bits: m in e4m3, v in e5m2, each block of 256 with a float32 scale of its own (its largest value is the type's largest).  They are
// rounded up or down at random, up with the probability of what is cut off: their mean is right.  Rounded to the nearest, v would stand still:
// a step changes it by a factor of 1 - b2, far less than half the distance of two neighbours.  The random bits are a hash of seed, step and place, so a repeated run gives the same bits.  v is rounded, not its
// root, since the root's rounding would add its variance to v step after step.  A v > 0 becomes at least the smallest code (its step would be m / eps at 0).
#pragma once
#include "k_vec.cuh"

struct OptimTensor {
    void* p; const void* g; float* master; void* m; void* v;
    float2* scales;                         // 8 bits: of m and v, for each block of 256
    int* step;                              // steps taken before this one
    const float* lr_at;                     // nullptr: lr
    long long n;
    long long first_block;                  // the first block's place in the hash
    unsigned chunk0;                        // chunks of the tensors before
    float lr, decay;
    int wide;                               // p and g (and the states) take 16-byte accesses
};
constexpr int OPTIM_BLOCK = 256, OPTIM_CHUNK = 8192, OPTIM_WARPS = 8;
template <int CAP> struct AdamParams {
    int n_tensors;
    unsigned chunks;
    float beta1, beta2, rest1, rest2;       // rest: 1 - beta
    double ln1, ln2;                        // logarithms of the betas
    float eps;
    unsigned seed;
    const float* factor;                    // nullptr: 1
    int* counter;                           // thread blocks that are done; 0 between launches
    OptimTensor t[CAP];
};

// Eight neighbours as floats; beyond `left` elements 0.
template <typename T> __device__ __forceinline__ void optim_load(const T* p, bool wide, int left, float (&f)[8]) {
    if (wide && left >= 8) to_floats(load_vec<T, 8>(p), f);
    else {
#pragma unroll
        for (int j = 0; j < 8; ++j) f[j] = j < left ? to_float(p[j]) : 0.f;
    }
}
template <typename T> __device__ __forceinline__ void optim_store(T* p, bool wide, int left, const float (&f)[8]) {
    if (wide && left >= 8) { Vec<T, 8> o; from_floats(o, f); store_vec(p, o); }
    else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j < left) p[j] = from_float<T>(f[j]);
    }
}
__device__ __forceinline__ uint2 optim_load_codes(const uint8_t* p, bool wide, int left) {
    if (wide && left >= 8) return *reinterpret_cast<const uint2*>(p);
    uint32_t w[2] = {0, 0};
#pragma unroll
    for (int j = 0; j < 8; ++j)
        if (j < left) w[j >> 2] |= (uint32_t)p[j] << 8 * (j & 3);
    return make_uint2(w[0], w[1]);
}
__device__ __forceinline__ void optim_store_codes(uint8_t* p, bool wide, int left, uint2 c) {
    if (wide && left >= 8) { *reinterpret_cast<uint2*>(p) = c; return; }
    const uint32_t w[2] = {c.x, c.y};
#pragma unroll
    for (int j = 0; j < 8; ++j)
        if (j < left) p[j] = (uint8_t)(w[j >> 2] >> 8 * (j & 3));
}

// Codes of 8 bits in pairs, to floats (exactly) and back (what is given here has a code of its own, or is NaN).
template <bool E5> __device__ __forceinline__ float2 optim_decode(uint32_t two) {
    uint32_t h;
    if constexpr (E5) asm("cvt.rn.f16x2.e5m2x2 %0, %1;\n" : "=r"(h) : "h"((uint16_t)two));
    else asm("cvt.rn.f16x2.e4m3x2 %0, %1;\n" : "=r"(h) : "h"((uint16_t)two));
    return __half22float2(*reinterpret_cast<const __half2*>(&h));
}
template <bool E5> __device__ __forceinline__ uint32_t optim_encode(float lo, float hi) {
    uint16_t c;
    if constexpr (E5) asm("cvt.rn.satfinite.e5m2x2.f32 %0, %1, %2;\n" : "=h"(c) : "f"(hi), "f"(lo));
    else asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;\n" : "=h"(c) : "f"(hi), "f"(lo));
    return c;
}
template <bool E5> __device__ __forceinline__ void optim_decode(uint2 c, float scale, float (&f)[8]) {
    const uint32_t w[4] = {c.x & 0xffffu, c.x >> 16, c.y & 0xffffu, c.y >> 16};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const float2 v = optim_decode<E5>(w[j]);
        f[2 * j] = v.x * scale; f[2 * j + 1] = v.y * scale;
    }
}
// An invertible mix of 32 bits.
__device__ __forceinline__ uint32_t optim_mix(uint32_t x) {
    x = (x ^ (x >> 16)) * 0x7feb352du;
    x = (x ^ (x >> 15)) * 0x846ca68bu;
    return x ^ (x >> 16);
}
// y >= 0 without the last DROP bits of its mantissa, or of numbers below `least`, the type's smallest normal one, as many as there: they are next to it.  Up
// where what is cut off and 16 random bits of the same weight carry.
template <int DROP> __device__ __forceinline__ float optim_up_or_down(float y, uint32_t bits16, float least) {
    const float off = y < least ? least : 0.f;
    return __uint_as_float((__float_as_uint(y + off) + (bits16 << (DROP - 16))) & ~((1u << DROP) - 1u)) - off;
}
// A block's largest value (>= 0, as its bits) to its scale: largest value / the type's, at least the smallest normal float; NaN and infinity stay.
__device__ __forceinline__ float optim_scale(float largest, float of_type) {
    const float s = largest * (1.f / of_type);
    return s < 1.17549435e-38f ? 1.17549435e-38f : s;
}

template <typename P, typename G, bool MASTER, bool BITS8, int CAP>
__global__ void __launch_bounds__(32 * OPTIM_WARPS)
k_adamw(const __grid_constant__ AdamParams<CAP> a) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    float factor = 1.f;
    if (a.factor) {
        factor = *a.factor;
        if (!(fabsf(factor) < INFINITY)) return;        // nothing is changed, the number of steps neither
    }
    for (unsigned chunk = blockIdx.x; chunk < a.chunks; chunk += gridDim.x) {
        int lo = 0, hi = a.n_tensors - 1;               // the last tensor that starts at this chunk or before
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (a.t[mid].chunk0 <= chunk) lo = mid; else hi = mid - 1;
        }
        const OptimTensor& t = a.t[lo];
        const bool wide = t.wide;
        const int step = *t.step + 1;
        // 1 - b^t without cancellation (a product of 53 bits, then float32)
        const float c1 = -expm1f((float)(a.ln1 * step)), c2 = -expm1f((float)(a.ln2 * step));
        const float inv1 = 1.f / c1, root2 = 1.f / sqrtf(c2);
        const float lr = t.lr_at ? *t.lr_at : t.lr, decay = t.decay;
        const long long start = (long long)(chunk - t.chunk0) * OPTIM_CHUNK, end = min(t.n, start + OPTIM_CHUNK);
        for (long long at = start + warp * OPTIM_BLOCK; at < end; at += OPTIM_WARPS * OPTIM_BLOCK) {
            const long long i = at + 8 * lane;
            const int left = (int)min(t.n - i, 8LL);    // (may be negative)
            float p[8], g[8], m[8], v[8];
            if constexpr (MASTER) optim_load(t.master + i, wide, left, p);
            else optim_load(static_cast<const P*>(t.p) + i, wide, left, p);
            optim_load(static_cast<const G*>(t.g) + i, wide, left, g);
            const long long block = at / OPTIM_BLOCK;
            if constexpr (BITS8) {
                const float2 s = t.scales[block];
                optim_decode<false>(optim_load_codes(static_cast<const uint8_t*>(t.m) + i, wide, left), s.x, m);
                optim_decode<true>(optim_load_codes(static_cast<const uint8_t*>(t.v) + i, wide, left), s.y, v);
            } else {
                optim_load(static_cast<const float*>(t.m) + i, wide, left, m);
                optim_load(static_cast<const float*>(t.v) + i, wide, left, v);
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float gj = g[j] * factor;
                // (each product and sum rounded by itself: the states have the bits of the formula in elementary steps)
                m[j] = __fadd_rn(__fmul_rn(a.beta1, m[j]), __fmul_rn(a.rest1, gj));
                v[j] = __fadd_rn(__fmul_rn(a.beta2, v[j]), __fmul_rn(__fmul_rn(a.rest2, gj), gj));
                const float s = (m[j] * inv1) / fmaf(sqrtf(v[j]), root2, a.eps);
                p[j] = fmaf(-lr, fmaf(decay, p[j], s), p[j]);
            }
            if constexpr (MASTER) optim_store(t.master + i, wide, left, p);
            optim_store(static_cast<P*>(t.p) + i, wide, left, p);
            if constexpr (BITS8) {
                // (the bits of numbers >= 0 are in their order, infinities and NaN above all)
                uint32_t bm = 0, bv = 0;
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const bool on = j < left;
                    bm = max(bm, on ? __float_as_uint(fabsf(m[j])) : 0u);
                    bv = max(bv, on ? __float_as_uint(v[j]) & 0x7fffffffu : 0u);
                }
                const float sm = optim_scale(__uint_as_float(__reduce_max_sync(0xffffffffu, bm)), 448.f);
                const float sv = optim_scale(__uint_as_float(__reduce_max_sync(0xffffffffu, bv)), 57344.f);
                if (lane == 0) t.scales[block] = make_float2(sm, sv);
                const uint32_t h = optim_mix((uint32_t)(t.first_block + block) ^ optim_mix(a.seed + 0x9e3779b9u * (uint32_t)step));
                uint32_t cm[4], cv[4];
#pragma unroll
                for (int j = 0; j < 8; j += 2) {
                    float y[2], z[2];
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        const uint32_t r = optim_mix(h + 8 * lane + j + k);
                        float q = fabsf(m[j + k]) / sm;
                        q = q > 448.f ? 448.f : q;
                        y[k] = copysignf(optim_up_or_down<20>(q, r & 0xffffu, 0x1p-6f), m[j + k]);
                        q = v[j + k] / sv;
                        q = q > 57344.f ? 57344.f : q;
                        z[k] = optim_up_or_down<21>(q, r >> 16, 0x1p-14f);
                        if (v[j + k] > 0.f && z[k] < 0x1p-16f) z[k] = 0x1p-16f;
                    }
                    cm[j / 2] = optim_encode<false>(y[0], y[1]);
                    cv[j / 2] = optim_encode<true>(z[0], z[1]);
                }
                optim_store_codes(static_cast<uint8_t*>(t.m) + i, wide, left, make_uint2(cm[0] | cm[1] << 16, cm[2] | cm[3] << 16));
                optim_store_codes(static_cast<uint8_t*>(t.v) + i, wide, left, make_uint2(cv[0] | cv[1] << 16, cv[2] | cv[3] << 16));
            } else {
                optim_store(static_cast<float*>(t.m) + i, wide, left, m);
                optim_store(static_cast<float*>(t.v) + i, wide, left, v);
            }
        }
    }
    // the last thread block to come here, when all have read the numbers of steps, counts the step
    __shared__ bool last;
    __syncthreads();
    if (threadIdx.x == 0) {
        __threadfence();
        last = atomicAdd(a.counter, 1) == (int)gridDim.x - 1;
        if (last) *a.counter = 0;
    }
    __syncthreads();
    if (last)
        for (int i = threadIdx.x; i < a.n_tensors; i += blockDim.x) ++*a.t[i].step;
}

// ------------------------------------------------------------------------------------------------ norm of many gradients
// The sum of the squares of all tensors: a thread's in float32 within a chunk, in double beyond, the thread block's sum (in order) to `partials`; the
// second kernel adds those in order, so a call repeated gives the same bits.
struct NormTensor { const void* p; long long n; unsigned chunk0; int type_wide; };        // type, and 4 where 16-byte accesses fit
constexpr int GNORM_CHUNK = 16384;
template <int CAP> struct GradNormParams {
    int n_tensors;
    unsigned chunks;
    double* partials;
    NormTensor t[CAP];
};

__device__ __forceinline__ double block_sum(double v, double* s) {          // thread 0's is the sum
#pragma unroll
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    if ((threadIdx.x & 31) == 0) s[threadIdx.x >> 5] = v;
    __syncthreads();
    v = 0.;
    if (threadIdx.x == 0)
        for (int w = 0; w < (int)blockDim.x >> 5; ++w) v += s[w];
    return v;
}
template <typename T> __device__ __forceinline__ float square_sum(const T* p, bool wide, int n) {
    constexpr int V = 16 / sizeof(T), STEP = 256 * V;
    float s[V];
#pragma unroll
    for (int j = 0; j < V; ++j) s[j] = 0.f;
    int at = 0;
    if (wide) {
#pragma unroll 4
        for (; at + STEP <= n; at += STEP) {
            float f[V];
            to_floats(load_vec<T, V>(p + at + threadIdx.x * V), f);
            vfma(s, f, f, s);
        }
    }
    for (int i = at + threadIdx.x; i < n; i += 256) {
        const float f = to_float(p[i]);
        s[0] = fmaf(f, f, s[0]);
    }
    return vsum(s);
}
template <int CAP>
__global__ void __launch_bounds__(256)
k_grad_norm(const __grid_constant__ GradNormParams<CAP> a) {
    __shared__ double s[8];
    double sum = 0.;
    for (unsigned chunk = blockIdx.x; chunk < a.chunks; chunk += gridDim.x) {
        int lo = 0, hi = a.n_tensors - 1;
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (a.t[mid].chunk0 <= chunk) lo = mid; else hi = mid - 1;
        }
        const NormTensor& t = a.t[lo];
        const long long start = (long long)(chunk - t.chunk0) * GNORM_CHUNK;
        const int n = (int)min(t.n - start, (long long)GNORM_CHUNK), type = t.type_wide & 3;
        const bool wide = t.type_wide & 4;
        if (type == HF_BF16) sum += square_sum(static_cast<const bf16*>(t.p) + start, wide, n);
        else if (type == HF_F16) sum += square_sum(static_cast<const __half*>(t.p) + start, wide, n);
        else sum += square_sum(static_cast<const float*>(t.p) + start, wide, n);
    }
    pdl_trigger();
    sum = block_sum(sum, s);
    if (threadIdx.x == 0) a.partials[blockIdx.x] = sum;
}
// out: the norm, and the factor min(1, most / norm) (NaN where the norm is not finite).
__global__ void __launch_bounds__(256)
k_grad_norm_sum(const double* partials, int n, float most, float* out) {
    __shared__ double s[8];
    pdl_wait();
    double sum = 0.;
    for (int i = threadIdx.x; i < n; i += 256) sum += partials[i];
    sum = block_sum(sum, s);
    if (threadIdx.x) return;
    const float norm = (float)sqrt(sum);
    out[0] = norm;
    out[1] = norm < INFINITY ? (norm <= most ? 1.f : (float)(most / sqrt(sum))) : __int_as_float(0x7fffffff);
}
