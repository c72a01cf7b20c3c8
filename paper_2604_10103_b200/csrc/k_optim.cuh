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
// 113 M elements, bf16 with masters: 529 us (6.0 TB/s, 92 % of the copy rate); 57 M elements in 8 bits: 173 us (5.3 TB/s: 72 instructions an element, and the loads'
// latency); the norm of 28 M bf16 elements 8.4 us.
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
    int wide;                               // eight elements of each tensor take one access
};
constexpr int OPTIM_BLOCK = 256, OPTIM_WARPS = 8, OPTIM_BLOCKS = 4;
template <int CAP> struct AdamParams {
    int n_tensors;
    unsigned chunks;
    int chunk;                              // elements of a chunk: a multiple of a thread block's 2048
    float beta1, beta2, rest1, rest2;       // rest: 1 - beta
    double ln1, ln2;                        // logarithms of the betas
    float eps;
    unsigned seed;
    const float* factor;                    // nullptr: 1
    int* counter;                           // thread blocks that are done; 0 between launches
    OptimTensor t[CAP];
};

// Eight neighbours as floats; FULL: in one access of 16 or 32 bytes (two of 16 would each touch half of every 32 bytes: 575 us instead of 529 for
// the four layers' step), otherwise one by one, beyond `left` elements 0.
template <bool FULL, typename T> __device__ __forceinline__ void optim_load(const T* p, int left, float (&f)[8]) {
    if constexpr (FULL && sizeof(T) == 4)
        asm volatile("ld.global.v8.f32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];\n" : "=f"(f[0]), "=f"(f[1]), "=f"(f[2]), "=f"(f[3]), "=f"(f[4]), "=f"(f[5]),
                     "=f"(f[6]), "=f"(f[7]) : "l"(p) : "memory");
    else if constexpr (FULL) to_floats(load_vec<T, 8>(p), f);
    else {
#pragma unroll
        for (int j = 0; j < 8; ++j) f[j] = j < left ? to_float(p[j]) : 0.f;
    }
}
template <bool FULL, typename T> __device__ __forceinline__ void optim_store(T* p, int left, const float (&f)[8]) {
    if constexpr (FULL && sizeof(T) == 4)
        asm volatile("st.global.v8.f32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};\n" ::"l"(p), "f"(f[0]), "f"(f[1]), "f"(f[2]), "f"(f[3]), "f"(f[4]), "f"(f[5]),
                     "f"(f[6]), "f"(f[7]) : "memory");
    else if constexpr (FULL) { Vec<T, 8> o; from_floats(o, f); store_vec(p, o); }
    else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j < left) p[j] = from_float<T>(f[j]);
    }
}
template <bool FULL> __device__ __forceinline__ uint2 optim_load_codes(const uint8_t* p, int left) {
    if constexpr (FULL) return *reinterpret_cast<const uint2*>(p);
    uint32_t w[2] = {0, 0};
#pragma unroll
    for (int j = 0; j < 8; ++j)
        if (j < left) w[j >> 2] |= (uint32_t)p[j] << 8 * (j & 3);
    return make_uint2(w[0], w[1]);
}
template <bool FULL> __device__ __forceinline__ void optim_store_codes(uint8_t* p, int left, uint2 c) {
    if constexpr (FULL) { *reinterpret_cast<uint2*>(p) = c; return; }
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
        const float2 v = fmul2(optim_decode<E5>(w[j]), make_float2(scale, scale));
        f[2 * j] = v.x; f[2 * j + 1] = v.y;
    }
}
// An invertible mix of 32 bits: two multiplications between shifts, with the published constants of lowbias32 (C. Wellons, 2018).
__device__ __forceinline__ uint32_t optim_mix(uint32_t x) {
    x = (x ^ (x >> 16)) * 0x7feb352du;
    x = (x ^ (x >> 15)) * 0x846ca68bu;
    return x ^ (x >> 16);
}
// y >= 0, two at a time, without the last DROP bits of its mantissa, or of numbers below `least`, the type's smallest normal one, as many as there: they
// are next to it.  Up where what is cut off and 16 random bits of the same weight carry.
template <int DROP> __device__ __forceinline__ float2 optim_up_or_down(float2 y, uint32_t bits0, uint32_t bits1, float least) {
    const float2 off = make_float2(y.x < least ? least : 0.f, y.y < least ? least : 0.f), z = fadd2(y, off);
    constexpr uint32_t KEEP = ~((1u << DROP) - 1u);
    return fadd2(make_float2(__uint_as_float((__float_as_uint(z.x) + (bits0 << (DROP - 16))) & KEEP), __uint_as_float((__float_as_uint(z.y) + (bits1 << (DROP - 16))) & KEEP)),
                 make_float2(-off.x, -off.y));
}
// Two quotients by a block's scale, no more than the type's largest value: products with its reciprocal, corrected by the residual, which the fused
// multiply-add forms exactly (P. Markstein, IBM Journal of Research and Development 34, 1990).
__device__ __forceinline__ float2 optim_quotient(float2 v, float scale, float inv, float most) {
    const float2 i2 = make_float2(inv, inv), q = fmul2(v, i2), r = ffma2(make_float2(-q.x, -q.y), make_float2(scale, scale), v), o = ffma2(r, i2, q);
    return make_float2(fminf(o.x, most), fminf(o.y, most));
}
// A block's largest value (>= 0, as its bits) to its scale: largest value / the type's, at least the smallest normal float; NaN and infinity stay.
__device__ __forceinline__ float optim_scale(float largest, float of_type) {
    const float s = largest * (1.f / of_type);
    return s < 1.17549435e-38f ? 1.17549435e-38f : s;
}
// The largest of eight, as unsigned numbers.
__device__ __forceinline__ uint32_t optim_max(const uint32_t (&v)[8]) {
    return __vimax3_u32(__vimax3_u32(v[0], v[1], v[2]), __vimax3_u32(v[3], v[4], v[5]), max(v[6], v[7]));
}
__device__ __forceinline__ float optim_sqrt(float v) {          // (2 ulp; nothing is flushed)
    float r;
    asm("sqrt.approx.f32 %0, %1;\n" : "=f"(r) : "f"(v));
    return r;
}
__device__ __forceinline__ float optim_rcp(float v) {           // (1 ulp)
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;\n" : "=f"(r) : "f"(v));
    return r;
}

// The warp's next block on its way into L2.  (8 bits, whose arithmetic takes longer than the loads in flight cover: 183 us instead of 173 for 57 M elements without;
// 32 bits: 529 without, 547 with.)
template <typename P, typename G, bool MASTER>
__device__ __forceinline__ void optim_ahead(const OptimTensor& t, long long at) {
    const long long i = at + 8 * (threadIdx.x & 31);
    const void* from[4] = {MASTER ? static_cast<const void*>(t.master + i) : static_cast<const P*>(t.p) + i, static_cast<const G*>(t.g) + i,
                           static_cast<const uint8_t*>(t.m) + i, static_cast<const uint8_t*>(t.v) + i};
#pragma unroll
    for (int k = 0; k < 4; ++k) asm volatile("prefetch.global.L2 [%0];\n" ::"l"(from[k]));
}

// What a tensor's step takes, the same for all its elements.
struct OptimStep { float factor, inv1, root2, lr, decay; uint32_t hash; };

// A warp's block of 256 elements from `at` on.
template <typename P, typename G, bool MASTER, bool BITS8, bool FULL, typename A>
__device__ __forceinline__ void optim_block(const A& a, const OptimTensor& t, long long at, const OptimStep& s) {
    const int lane = threadIdx.x & 31;
    const long long i = at + 8 * lane, block = at / OPTIM_BLOCK;
    const int left = FULL ? 8 : (int)min(t.n - i, 8LL);         // (may be negative)
    float p[8], g[8], m[8], v[8];
    if constexpr (MASTER) optim_load<FULL>(t.master + i, left, p);
    else optim_load<FULL>(static_cast<const P*>(t.p) + i, left, p);
    optim_load<FULL>(static_cast<const G*>(t.g) + i, left, g);
    if constexpr (BITS8) {
        const uint2 cm = optim_load_codes<FULL>(static_cast<const uint8_t*>(t.m) + i, left), cv = optim_load_codes<FULL>(static_cast<const uint8_t*>(t.v) + i, left);
        const float2 scale = t.scales[block];
        optim_decode<false>(cm, scale.x, m);
        optim_decode<true>(cv, scale.y, v);
    } else {
        optim_load<FULL>(static_cast<const float*>(t.m) + i, left, m);
        optim_load<FULL>(static_cast<const float*>(t.v) + i, left, v);
    }
    const float2 factor = make_float2(s.factor, s.factor), beta1 = make_float2(a.beta1, a.beta1), beta2 = make_float2(a.beta2, a.beta2);
    const float2 rest1 = make_float2(a.rest1, a.rest1), rest2 = make_float2(a.rest2, a.rest2), inv1 = make_float2(s.inv1, s.inv1);
    const float2 root2 = make_float2(s.root2, s.root2), eps = make_float2(a.eps, a.eps), lr = make_float2(-s.lr, -s.lr), decay = make_float2(s.decay, s.decay);
#pragma unroll
    for (int j = 0; j < 8; j += 2) {
        // (each product and sum of the moments rounded by itself: they have the bits of the formula in elementary steps.  The sums are taken one by one:
        // a packed sum of packed products would become a fused multiply-add.)
        const float2 gj = fmul2(make_float2(g[j], g[j + 1]), factor);
        const float2 m0 = fmul2(beta1, make_float2(m[j], m[j + 1])), m1 = fmul2(rest1, gj);
        const float2 v0 = fmul2(beta2, make_float2(v[j], v[j + 1])), v1 = fmul2(fmul2(rest2, gj), gj);
        const float2 mj = make_float2(__fadd_rn(m0.x, m1.x), __fadd_rn(m0.y, m1.y)), vj = make_float2(__fadd_rn(v0.x, v1.x), __fadd_rn(v0.y, v1.y));
        const float2 den = ffma2(make_float2(optim_sqrt(vj.x), optim_sqrt(vj.y)), root2, eps);
        const float2 q = fmul2(fmul2(mj, inv1), make_float2(optim_rcp(den.x), optim_rcp(den.y)));
        const float2 pj = make_float2(p[j], p[j + 1]), o = ffma2(lr, ffma2(decay, pj, q), pj);
        m[j] = mj.x; m[j + 1] = mj.y; v[j] = vj.x; v[j + 1] = vj.y; p[j] = o.x; p[j + 1] = o.y;
    }
    if constexpr (MASTER) optim_store<FULL>(t.master + i, left, p);
    optim_store<FULL>(static_cast<P*>(t.p) + i, left, p);
    if constexpr (BITS8) {
        // (the bits of numbers >= 0 are in their order, infinities and NaN above all: such a scale spoils the block, whatever its codes)
        uint32_t bm[8], bv[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) { bm[j] = __float_as_uint(m[j]) & 0x7fffffffu; bv[j] = __float_as_uint(v[j]); }
        const float sm = optim_scale(__uint_as_float(__reduce_max_sync(0xffffffffu, optim_max(bm))), 448.f);
        const float sv = optim_scale(__uint_as_float(__reduce_max_sync(0xffffffffu, optim_max(bv))), 57344.f);
        if (lane == 0) t.scales[block] = make_float2(sm, sv);
        const float im = 1.f / sm, iv = 1.f / sv;
        const uint32_t h = optim_mix((uint32_t)(t.first_block + block) ^ s.hash) + 8 * lane;
        uint32_t cm[4], cv[4];
#pragma unroll
        for (int j = 0; j < 8; j += 2) {
            const uint32_t r0 = optim_mix(h + j), r1 = optim_mix(h + j + 1);
            const float2 ym = optim_quotient(make_float2(__uint_as_float(bm[j]), __uint_as_float(bm[j + 1])), sm, im, 448.f);
            const float2 yv = optim_quotient(make_float2(v[j], v[j + 1]), sv, iv, 57344.f);
            const float2 y = optim_up_or_down<20>(ym, r0 & 0xffffu, r1 & 0xffffu, 0x1p-6f), z = optim_up_or_down<21>(yv, r0 >> 16, r1 >> 16, 0x1p-14f);
            cm[j / 2] = optim_encode<false>(copysignf(y.x, m[j]), copysignf(y.y, m[j + 1]));
            cv[j / 2] = optim_encode<true>(fmaxf(z.x, v[j] > 0.f ? 0x1p-16f : 0.f), fmaxf(z.y, v[j + 1] > 0.f ? 0x1p-16f : 0.f));
        }
        optim_store_codes<FULL>(static_cast<uint8_t*>(t.m) + i, left, make_uint2(cm[0] | cm[1] << 16, cm[2] | cm[3] << 16));
        optim_store_codes<FULL>(static_cast<uint8_t*>(t.v) + i, left, make_uint2(cv[0] | cv[1] << 16, cv[2] | cv[3] << 16));
    } else {
        optim_store<FULL>(static_cast<float*>(t.m) + i, left, m);
        optim_store<FULL>(static_cast<float*>(t.v) + i, left, v);
    }
}

template <typename P, typename G, bool MASTER, bool BITS8, int CAP>
__global__ void __launch_bounds__(32 * OPTIM_WARPS, OPTIM_BLOCKS)
k_adamw(const __grid_constant__ AdamParams<CAP> a) {
    const int warp = threadIdx.x >> 5;
    OptimStep s;
    s.factor = 1.f;
    if (a.factor) {
        s.factor = *a.factor;
        if (!(fabsf(s.factor) < INFINITY)) return;      // nothing is changed, the number of steps neither
    }
    for (unsigned chunk = blockIdx.x; chunk < a.chunks; chunk += gridDim.x) {
        int lo = 0, hi = a.n_tensors - 1;               // the last tensor that starts at this chunk or before
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (a.t[mid].chunk0 <= chunk) lo = mid; else hi = mid - 1;
        }
        const OptimTensor& t = a.t[lo];
        const int step = *t.step + 1;
        // 1 - b^t without cancellation (a product of 53 bits, then float32)
        s.inv1 = -1.f / expm1f((float)(a.ln1 * step));
        s.root2 = 1.f / sqrtf(-expm1f((float)(a.ln2 * step)));
        s.lr = t.lr_at ? *t.lr_at : t.lr;
        s.decay = t.decay;
        s.hash = optim_mix(a.seed + 0x9e3779b9u * (uint32_t)step);
        const long long start = (long long)(chunk - t.chunk0) * a.chunk, end = min(t.n, start + a.chunk);
        for (long long at = start + warp * OPTIM_BLOCK; at < end; at += OPTIM_WARPS * OPTIM_BLOCK) {
            if constexpr (BITS8) {
                const long long next = at + OPTIM_WARPS * OPTIM_BLOCK;
                if (next < end && next + OPTIM_BLOCK <= t.n) optim_ahead<P, G, MASTER>(t, next);
            }
            if (t.wide && at + OPTIM_BLOCK <= t.n) optim_block<P, G, MASTER, BITS8, true>(a, t, at, s);
            else optim_block<P, G, MASTER, BITS8, false>(a, t, at, s);
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
