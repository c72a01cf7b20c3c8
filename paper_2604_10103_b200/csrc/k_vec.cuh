// Elements of three types as float: V of them with one access.
#pragma once
#include "hf_common.cuh"
#include <cuda_fp16.h>

// (WIDE false: aligned as one element only)
template <typename T, int V, bool WIDE = true> struct alignas(!WIDE ? sizeof(T) : (sizeof(T) * V < 16 ? sizeof(T) * V : 16)) Vec { T v[V]; };

// One access of the whole (WIDE; at most 16 bytes each), or one for each element.  Written out: a copy of the structure is left to the compiler,
// which takes words.
template <typename T, int V, bool WIDE = true>
__device__ __forceinline__ Vec<T, V, WIDE> load_vec(const T* p) {
    Vec<T, V, WIDE> r;
    constexpr int B = sizeof(T) * V;
    if constexpr (WIDE && B % 16 == 0) {
#pragma unroll
        for (int i = 0; i < B / 16; ++i) {
            const uint4 w = reinterpret_cast<const uint4*>(p)[i];
            memcpy(reinterpret_cast<char*>(&r) + 16 * i, &w, 16);
        }
    } else if constexpr (WIDE && B == 8) {
        const uint2 w = *reinterpret_cast<const uint2*>(p);
        memcpy(&r, &w, 8);
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) r.v[i] = p[i];
    }
    return r;
}
template <typename T, int V, bool WIDE>
__device__ __forceinline__ void store_vec(T* p, const Vec<T, V, WIDE>& x) {
    constexpr int B = sizeof(T) * V;
    if constexpr (WIDE && B % 16 == 0) {
#pragma unroll
        for (int i = 0; i < B / 16; ++i) {
            uint4 w;
            memcpy(&w, reinterpret_cast<const char*>(&x) + 16 * i, 16);
            reinterpret_cast<uint4*>(p)[i] = w;
        }
    } else if constexpr (WIDE && B == 8) {
        uint2 w;
        memcpy(&w, &x, 8);
        *reinterpret_cast<uint2*>(p) = w;
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) p[i] = x.v[i];
    }
}

__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(bf16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float to_float(__half x) { return __half2float(x); }
template <typename T> __device__ __forceinline__ T from_float(float x);
template <> __device__ __forceinline__ float from_float<float>(float x) { return x; }
template <> __device__ __forceinline__ bf16 from_float<bf16>(float x) { return __float2bfloat16_rn(x); }
template <> __device__ __forceinline__ __half from_float<__half>(float x) { return __float2half_rn(x); }
// Two 16-bit elements in a word.
template <typename T> __device__ __forceinline__ uint32_t pack2(float lo, float hi);
template <> __device__ __forceinline__ uint32_t pack2<bf16>(float lo, float hi) { return pack_bf16(lo, hi); }
template <> __device__ __forceinline__ uint32_t pack2<__half>(float lo, float hi) {
    const __half2 t = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&t);
}
template <typename T> __device__ __forceinline__ float2 unpack2(uint32_t u);
template <> __device__ __forceinline__ float2 unpack2<bf16>(uint32_t u) { return unpack_bf16(u); }
template <> __device__ __forceinline__ float2 unpack2<__half>(uint32_t u) { return __half22float2(*reinterpret_cast<const __half2*>(&u)); }

// All elements as float and back.  16-bit elements go by the word: taken one by one each would occupy a register of its own.
template <typename T, int V, bool WIDE>
__device__ __forceinline__ void to_floats(const Vec<T, V, WIDE>& x, float (&f)[V]) {
    if constexpr (sizeof(T) == 2 && V % 2 == 0) {
        uint32_t w[V / 2];
        memcpy(w, &x, sizeof(x));
#pragma unroll
        for (int i = 0; i < V / 2; ++i) {
            const float2 p = unpack2<T>(w[i]);
            f[2 * i] = p.x; f[2 * i + 1] = p.y;
        }
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) f[i] = to_float(x.v[i]);
    }
}
template <typename T, int V, bool WIDE>
__device__ __forceinline__ void from_floats(Vec<T, V, WIDE>& x, const float (&f)[V]) {
    if constexpr (sizeof(T) == 2 && V % 2 == 0) {
        uint32_t w[V / 2];
#pragma unroll
        for (int i = 0; i < V / 2; ++i) w[i] = pack2<T>(f[2 * i], f[2 * i + 1]);
        memcpy(&x, w, sizeof(x));
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) x.v[i] = from_float<T>(f[i]);
    }
}

// A row of elements at p, aligned to an element: V of them from column col (a multiple of V) on.  WIDE: one access.  V 2, 16-bit elements:
// pairs out of the 4-byte words that hold them: whether the row starts in the middle of a word is looked at once, for the row.
// `two`: whether a pair has a second element; nothing is read beyond the words of the row's own elements.
template <typename T, int V, bool WIDE>
struct Row {
    const T* p;
    uint32_t shift;
    __device__ __forceinline__ explicit Row(const T* at) : p(at), shift(0) {
        if constexpr (!WIDE && V == 2) {
            shift = (uint32_t)(reinterpret_cast<uintptr_t>(at) & 2) * 8;
            p = at - (shift ? 1 : 0);
        }
    }
    // The same with the start given: `base` aligned to a word, `lead` bytes in front of the row (a shared-memory address stays one).
    __device__ __forceinline__ Row(const uint8_t* base, uint32_t lead) : p(reinterpret_cast<const T*>(base + (lead & ~3u))), shift((lead & 2) * 8) {
        if constexpr (WIDE || V != 2) p = reinterpret_cast<const T*>(base + lead);
    }
    __device__ __forceinline__ void get(int col, float (&f)[V], bool two) const {
        if constexpr (WIDE) to_floats(load_vec<T, V>(p + col), f);
        else if constexpr (V == 1) f[0] = to_float(p[col]);
        else {
            static_assert(V != 2 || sizeof(T) == 2, "pairs of 16-bit elements");
            const uint32_t* w = reinterpret_cast<const uint32_t*>(p + col);
            uint32_t v = w[0];
            if (shift) v = __funnelshift_r(v, two ? w[1] : 0u, 16);
            const float2 r = unpack2<T>(v);
            f[0] = r.x; f[1] = two ? r.y : 0.f;
        }
    }
};
template <typename T, int V, bool WIDE>
__device__ __forceinline__ void put_floats(T* p, const float (&f)[V], bool two) {
    if constexpr (WIDE) { Vec<T, V> o; from_floats(o, f); store_vec(p, o); }
    else if constexpr (V == 1) p[0] = from_float<T>(f[0]);
    else if (two && (reinterpret_cast<uintptr_t>(p) & 2) == 0) *reinterpret_cast<uint32_t*>(p) = pack2<T>(f[0], f[1]);
    else {
        p[0] = from_float<T>(f[0]);
        if (two) p[1] = from_float<T>(f[1]);
    }
}

// Packed elements that the compiler may not keep unpacked beside them: what is computed from v behind this is computed anew, which costs an
// instruction or two an element and saves the registers.
template <typename T, int V>
__device__ __forceinline__ void stay_packed(Vec<T, V>& v) {
    if constexpr (sizeof(T) == 2 && V % 2 == 0) {
        uint32_t w[V / 2];
        memcpy(w, &v, sizeof(v));
#pragma unroll
        for (int i = 0; i < V / 2; ++i) asm volatile("" : "+r"(w[i]));
        memcpy(&v, w, sizeof(v));
    }
}

// Element-wise arithmetic on V floats, two an instruction where V is even: r = a b + c, r = a b, r *= b, r += b.
template <int V> __device__ __forceinline__ void vfma(float (&r)[V], const float (&a)[V], const float (&b)[V], const float (&c)[V]) {
    if constexpr (V % 2 == 0) {
#pragma unroll
        for (int i = 0; i < V; i += 2) {
            const float2 o = ffma2(make_float2(a[i], a[i + 1]), make_float2(b[i], b[i + 1]), make_float2(c[i], c[i + 1]));
            r[i] = o.x; r[i + 1] = o.y;
        }
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) r[i] = fmaf(a[i], b[i], c[i]);
    }
}
template <int V> __device__ __forceinline__ void vfma(float (&r)[V], const float (&a)[V], float b, float c) {
    if constexpr (V % 2 == 0) {
#pragma unroll
        for (int i = 0; i < V; i += 2) {
            const float2 o = ffma2(make_float2(a[i], a[i + 1]), make_float2(b, b), make_float2(c, c));
            r[i] = o.x; r[i + 1] = o.y;
        }
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) r[i] = fmaf(a[i], b, c);
    }
}
template <int V> __device__ __forceinline__ void vfma(float (&r)[V], const float (&a)[V], float b, const float (&c)[V]) {
    if constexpr (V % 2 == 0) {
#pragma unroll
        for (int i = 0; i < V; i += 2) {
            const float2 o = ffma2(make_float2(a[i], a[i + 1]), make_float2(b, b), make_float2(c[i], c[i + 1]));
            r[i] = o.x; r[i + 1] = o.y;
        }
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) r[i] = fmaf(a[i], b, c[i]);
    }
}
template <int V> __device__ __forceinline__ void vmul(float (&r)[V], const float (&a)[V], const float (&b)[V]) {
    if constexpr (V % 2 == 0) {
#pragma unroll
        for (int i = 0; i < V; i += 2) {
            const float2 o = fmul2(make_float2(a[i], a[i + 1]), make_float2(b[i], b[i + 1]));
            r[i] = o.x; r[i + 1] = o.y;
        }
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) r[i] = a[i] * b[i];
    }
}
template <int V> __device__ __forceinline__ void vadd(float (&r)[V], const float (&b)[V]) {
    if constexpr (V % 2 == 0) {
#pragma unroll
        for (int i = 0; i < V; i += 2) {
            const float2 o = fadd2(make_float2(r[i], r[i + 1]), make_float2(b[i], b[i + 1]));
            r[i] = o.x; r[i + 1] = o.y;
        }
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) r[i] += b[i];
    }
}
template <int V> __device__ __forceinline__ void vadd(float (&r)[V], float b) {
    float v[V];
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = b;
    vadd(r, v);
}
template <int V> __device__ __forceinline__ void vmul(float (&r)[V], float b) {
    float v[V];
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = b;
    vmul(r, r, v);
}
template <int V> __device__ __forceinline__ float vsum(const float (&a)[V]) {
    float s = a[0];
#pragma unroll
    for (int i = 1; i < V; ++i) s += a[i];
    return s;
}
