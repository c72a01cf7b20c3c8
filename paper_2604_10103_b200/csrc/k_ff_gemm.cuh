// Products of the gated feed-forward on the Blackwell tensor path, one kernel for all of them: D = A B^T over tiles of 128 rows and up to
// 256 columns, accumulators in tensor memory, operands brought by TMA, with an epilogue of its own for each use:
//   GATED    g = x Wg^T and u = x Wu^T side by side in one accumulator; h = act(g) u (and g, u)       A, B: contraction contiguous
//   STORE    the product itself                                                                       (y, dx, dW)
//   DHIDDEN  dh = dy Wd; dg = dh u act'(g), du = dh act(g), h = act(g) u                               B: columns contiguous
// An operand whose contraction index is contiguous ("K-major") is a box of 64 contraction elements by its rows; one whose row index is
// contiguous ("MN-major": Wd in dh, Wg and Wu in dx, everything in dW) is read as it lies too, in boxes of 64 rows by 64 contraction
// elements: the tensor cores take both, so nothing is transposed in memory.  Elements past an operand's end read as zero.
// A thread block is persistent: a loader thread, an MMA thread, and eight epilogue warps that empty one accumulator while the MMAs fill the
// other.  Every wait is bounded (~1 s) and reports through the status word.
#pragma once
#include "tc5_common.cuh"
#include "k_vec.cuh"

enum { FF_GATED = 0, FF_STORE = 1, FF_DHIDDEN = 2 };

struct FfGemmParams {
    CUtensorMap a[3], b[3], out[3];     // operands of each product, or of each segment of the contraction; GATED: b = Wg, Wu
    const void* gate; const void* up;   // DHIDDEN: [rows, cols]
    int products;                       // products of this launch, each with tiles of its own ...
    int tile0[4];                       // ... from tile0[i] to tile0[i + 1]
    int rows[3], cols[3];               // of the output
    int kb[3];                          // blocks of 64 of each product's (or segment's) contraction
    int segments;                       // contraction in this many segments (dx = dg Wg + du Wu: two)
    int bn;                             // accumulator columns of a tile: a multiple of 32 (GATED: of 64, half of them g, half u)
    int stages;
    int act, save;
    int* dev_status;
};

struct FfGemm {
    static constexpr int BM = 128, BK = 64;
    static constexpr int A_BYTES = BM * BK * 2;
    static constexpr int EPI_WARPS = 8, WARP_TMA = 8, WARP_MMA = 9;
    static constexpr int THREADS = 32 * (EPI_WARPS + 2);
    static constexpr int MAX_STAGES = 8;
    static constexpr int STAGING = 2 * 2048;            // per epilogue warp: two boxes of 32 rows x 32 columns
    static constexpr int BAR_BYTES = 256;
    static constexpr int SMEM_MAX = 232448;
    __host__ __device__ static constexpr int stage_bytes(int bn) { return A_BYTES + (bn + 63) / 64 * 64 * BK * 2; }
    static constexpr int smem_bytes(int bn, int stages) { return stages * stage_bytes(bn) + EPI_WARPS * STAGING + BAR_BYTES + 1024; }
    static constexpr int stages_for(int bn) {
        const int n = (SMEM_MAX - EPI_WARPS * STAGING - BAR_BYTES - 1024) / stage_bytes(bn);
        return n < MAX_STAGES ? n : MAX_STAGES;
    }
};

// silu: a = g p, a' = p (1 + g (1 - p)), p = 1 / (1 + e^-g).   gelu (tanh form): with v = A (g + B g^3) the factor (1 + tanh v) / 2 is
// 1 / (1 + e^-2v), so it is g p with another exponent: a' = p + g p (1 - p) 2 A (1 + 3 B g^2).
// (An exponential that overflows gives p = 0, the right limit; __fdividef returns 0 there too.)
__device__ __forceinline__ float ff_sigmoid(float v) { return __fdividef(1.f, 1.f + __expf(-v)); }
constexpr float FF_GELU_2A = 1.5957691216057308f, FF_GELU_B = 0.044715f;
__device__ __forceinline__ float ff_act(float g, int act) {
    return g * ff_sigmoid(act == HF_ACT_SILU ? g : FF_GELU_2A * fmaf(FF_GELU_B * g * g, g, g));
}
__device__ __forceinline__ float ff_act(float g, int act, float* slope) {
    if (act == HF_ACT_SILU) {
        const float p = ff_sigmoid(g);
        *slope = p * fmaf(g, 1.f - p, 1.f);
        return g * p;
    }
    const float p = ff_sigmoid(FF_GELU_2A * fmaf(FF_GELU_B * g * g, g, g));
    *slope = fmaf(g * p * (1.f - p), FF_GELU_2A * fmaf(3.f * FF_GELU_B * g, g, 1.f), p);
    return g * p;
}

template <typename T> __device__ __forceinline__ uint32_t ff_pack(float lo, float hi);
template <> __device__ __forceinline__ uint32_t ff_pack<bf16>(float lo, float hi) { return pack_bf16(lo, hi); }
template <> __device__ __forceinline__ uint32_t ff_pack<__half>(float lo, float hi) {
    const __half2 t = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&t);
}
template <typename T> __device__ __forceinline__ float2 ff_unpack(uint32_t u);
template <> __device__ __forceinline__ float2 ff_unpack<bf16>(uint32_t u) { return unpack_bf16(u); }
template <> __device__ __forceinline__ float2 ff_unpack<__half>(uint32_t u) { return __half22float2(*reinterpret_cast<const __half2*>(&u)); }

struct FfTile { int product, m0, n0; };
// Tiles of a product in groups of 16 row tiles, all columns of a group before the next: the thread blocks at work at a time share rows
// and columns of both operands in L2.
__device__ __forceinline__ FfTile ff_tile(const FfGemmParams& p, int t, int bn_out) {
    FfTile r;
    r.product = 0;
    while (r.product + 1 < p.products && t >= p.tile0[r.product + 1]) ++r.product;
    t -= p.tile0[r.product];
    const int tm = (p.rows[r.product] + FfGemm::BM - 1) / FfGemm::BM, tn = (p.cols[r.product] + bn_out - 1) / bn_out;
    const int group = t / (16 * tn), first = group * 16, size = min(16, tm - first), in = t - group * 16 * tn;
    r.m0 = (first + in % size) * FfGemm::BM;
    r.n0 = in / size * bn_out;
    return r;
}

// One box of 32 rows x 32 columns on its way out: packed pairs of the lane's row -> the warp's staging buffer (64-byte rows, 16-byte pieces
// swizzled as the map says) -> TMA, which leaves out what lies past the tensor's end.
struct FfOut {
    uint32_t base;
    int next;
    __device__ __forceinline__ void put(const CUtensorMap* map, const uint32_t (&v)[16], int col, int row, int lane) {
        const uint32_t buf = base + next * 2048;
        next ^= 1;
        if (lane == 0) tc5::bulk_wait_read_but<1>();        // the store before the last has read this buffer
        __syncwarp();
#pragma unroll
        for (int c = 0; c < 4; ++c)
            asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};\n" ::"r"(buf + lane * 64 + ((c ^ ((lane >> 1) & 3)) << 4)),
                         "r"(v[4 * c]), "r"(v[4 * c + 1]), "r"(v[4 * c + 2]), "r"(v[4 * c + 3]) : "memory");
        tc5::fence_proxy_async();
        __syncwarp();
        if (lane == 0) {
            tc5::tma_store_2d(map, buf, col, row);
            tc5::bulk_commit();
        }
    }
};

template <typename T, int EPI, bool A_MN, bool B_MN>
__global__ void __launch_bounds__(FfGemm::THREADS, 1)
k_ff_gemm(const __grid_constant__ FfGemmParams p) {
    using namespace tc5;
    typedef FfGemm C;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t s_base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    uint8_t* s_gen = smem_raw + (s_base - smem_u32(smem_raw));
    const int stage_bytes = C::stage_bytes(p.bn), stages = p.stages;
    const uint32_t s_staging = s_base + stages * stage_bytes, bar0 = s_staging + C::EPI_WARPS * C::STAGING;
    const uint32_t bar_full = bar0, bar_free = bar0 + 64, bar_acc = bar0 + 128, bar_acc_free = bar0 + 144;
    uint8_t* bar_gen = s_gen + (bar0 - s_base);
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bar_gen + 160);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(bar_gen + 164);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int bn_out = EPI == FF_GATED ? p.bn / 2 : p.bn;
    const int n_tiles = p.tile0[p.products];

    if (threadIdx.x == 0) {
        for (int s = 0; s < stages; ++s) { mbar_init(bar_full + 8 * s, 1); mbar_init(bar_free + 8 * s, 1); }
        for (int s = 0; s < 2; ++s) { mbar_init(bar_acc + 8 * s, 1); mbar_init(bar_acc_free + 8 * s, C::EPI_WARPS); }
        *abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;\n" ::: "memory");
    }
    if (warp == C::WARP_MMA) {
        tmem_alloc(smem_u32(tmem_slot), 512);
        tmem_relinquish();
    }
    fence_before_sync();
    __syncthreads();
    fence_after_sync();
    const uint32_t tmem = *tmem_slot;

    if (warp == C::WARP_TMA) {
        // ================================================================= loader
        if (lane == 0) {
            bool ok = true;
            int s = 0;
            uint32_t phase = 1;                 // (the stages are free at first)
            const int b_boxes = B_MN ? (p.bn + 63) / 64 : 1;
            const uint32_t bytes = C::A_BYTES + (B_MN ? b_boxes * 8192 : p.bn * C::BK * 2);
            for (int t = blockIdx.x; ok && t < n_tiles; t += gridDim.x) {
                const FfTile tile = ff_tile(p, t, bn_out);
                for (int seg = 0; ok && seg < p.segments; ++seg) {
                    const int i = tile.product + seg;           // (one of the two is always 0)
                    for (int kb = 0; kb < p.kb[i]; ++kb) {
                        if (!(ok = mbar_wait<true>(bar_free + 8 * s, phase, abort_flag, p.dev_status, 81))) break;
                        const uint32_t sA = s_base + s * stage_bytes, sB = sA + C::A_BYTES, full = bar_full + 8 * s;
                        mbar_expect_tx(full, bytes);
                        if (A_MN) {
                            tma_load_2d(sA, &p.a[i], tile.m0, kb * C::BK, full);
                            tma_load_2d(sA + 8192, &p.a[i], tile.m0 + 64, kb * C::BK, full);
                        } else
                            tma_load_2d(sA, &p.a[i], kb * C::BK, tile.m0, full);
                        if (EPI == FF_GATED) {
                            tma_load_2d(sB, &p.b[0], kb * C::BK, tile.n0, full);
                            tma_load_2d(sB + bn_out * C::BK * 2, &p.b[1], kb * C::BK, tile.n0, full);
                        } else if (B_MN) {
                            for (int x = 0; x < b_boxes; ++x) tma_load_2d(sB + x * 8192, &p.b[i], tile.n0 + 64 * x, kb * C::BK, full);
                        } else
                            tma_load_2d(sB, &p.b[i], kb * C::BK, tile.n0, full);
                        if (++s == stages) { s = 0; phase ^= 1; }
                    }
                }
            }
            if (!ok) {                          // copies in flight land before the thread block leaves
                const long long t0 = clock64();
                while (clock64() - t0 < 400000) {}
            }
        }
    } else if (warp == C::WARP_MMA) {
        // ================================================================= MMA issuer (warp-uniform, one elected lane issues)
        constexpr uint32_t TYPE = sizeof(T) == 2 && std::is_same<T, bf16>::value ? 1u : 0u;
        const uint32_t idesc = (1u << 4) | (TYPE << 7) | (TYPE << 10) | ((A_MN ? 1u : 0u) << 15) | ((B_MN ? 1u : 0u) << 16) |
                               ((uint32_t)(p.bn >> 3) << 17) | ((uint32_t)(C::BM >> 4) << 24);
        const uint64_t da0 = smem_desc_sw128(s_base, A_MN ? 8192 : 16, 1024);
        const uint64_t db0 = smem_desc_sw128(s_base + C::A_BYTES, B_MN ? 8192 : 16, 1024);
        constexpr int A_STEP = (A_MN ? 2048 : 32) >> 4, B_STEP = (B_MN ? 2048 : 32) >> 4;
        bool ok = true;
        int s = 0, acc = 0;
        uint32_t phase = 0, acc_phase = 1;
        for (int t = blockIdx.x; ok && t < n_tiles; t += gridDim.x) {
            const FfTile tile = ff_tile(p, t, bn_out);
            int n_kb = p.kb[tile.product];
            for (int seg = 1; seg < p.segments; ++seg) n_kb += p.kb[seg];
            if (!(ok = mbar_wait_warp<true>(bar_acc_free + 8 * acc, acc_phase, abort_flag, p.dev_status, 82))) break;
            fence_after_sync();
            for (int kb = 0; kb < n_kb; ++kb) {
                if (!(ok = mbar_wait_warp<true>(bar_full + 8 * s, phase, abort_flag, p.dev_status, 83))) break;
                fence_after_sync();
                if (elect_one()) {
                    const uint64_t off = (uint64_t)((s * stage_bytes) >> 4);
#pragma unroll
                    for (int ks = 0; ks < C::BK / 16; ++ks)
                        mma_ss(tmem + acc * 256, da0 + off + ks * A_STEP, db0 + off + ks * B_STEP, idesc, kb > 0 || ks > 0);
                    mma_commit(bar_free + 8 * s);
                    if (kb == n_kb - 1) mma_commit(bar_acc + 8 * acc);
                }
                __syncwarp();
                if (++s == stages) { s = 0; phase ^= 1; }
            }
            if (acc) acc_phase ^= 1;
            acc ^= 1;
        }
    } else {
        // ================================================================= epilogue: warps w and w + 4 share the accumulator rows 32 (w & 3) ...
        const int quad = warp & 3, half = warp >> 2;
        const uint32_t lane_base = tmem + ((uint32_t)(quad * 32) << 16);
        FfOut out = {s_staging + warp * C::STAGING, 0};
        bool ok = true;
        int acc = 0;
        uint32_t acc_phase = 0;
        for (int t = blockIdx.x; t < n_tiles; t += gridDim.x) {
            const FfTile tile = ff_tile(p, t, bn_out);
            if (!(ok = mbar_wait_warp(bar_acc + 8 * acc, acc_phase, abort_flag, p.dev_status, 84))) break;
            fence_after_sync();
            const int row = tile.m0 + quad * 32, cols = p.cols[tile.product];
            const bool rows_on = row < p.rows[tile.product];
            for (int c = half; c < bn_out / 32; c += 2) {           // 32 columns at a time
                const int col = tile.n0 + 32 * c;
                if (!rows_on || col >= cols) break;
                const uint32_t at = lane_base + acc * 256 + 32 * c;
                uint32_t r[32], o[16];
                if constexpr (EPI == FF_STORE) {
                    tmem_ld32(at, r);
                    tmem_wait_ld();
#pragma unroll
                    for (int j = 0; j < 16; ++j) o[j] = ff_pack<T>(__uint_as_float(r[2 * j]), __uint_as_float(r[2 * j + 1]));
                    out.put(&p.out[tile.product], o, col, row, lane);
                } else if constexpr (EPI == FF_GATED) {
                    uint32_t u[32];
                    tmem_ld32(at, r);
                    tmem_ld32(at + bn_out, u);
                    tmem_wait_ld();
                    if (p.save) {
#pragma unroll
                        for (int j = 0; j < 16; ++j) o[j] = ff_pack<T>(__uint_as_float(r[2 * j]), __uint_as_float(r[2 * j + 1]));
                        out.put(&p.out[1], o, col, row, lane);
#pragma unroll
                        for (int j = 0; j < 16; ++j) o[j] = ff_pack<T>(__uint_as_float(u[2 * j]), __uint_as_float(u[2 * j + 1]));
                        out.put(&p.out[2], o, col, row, lane);
                    }
#pragma unroll
                    for (int j = 0; j < 16; ++j)
                        o[j] = ff_pack<T>(ff_act(__uint_as_float(r[2 * j]), p.act) * __uint_as_float(u[2 * j]),
                                          ff_act(__uint_as_float(r[2 * j + 1]), p.act) * __uint_as_float(u[2 * j + 1]));
                    out.put(&p.out[0], o, col, row, lane);
                } else {
                    // the lane's row of gate and up: 32 columns of each, in 16-byte pieces (cols is a multiple of 8)
                    uint32_t g[16], u[16], h[16];
                    const size_t e = (size_t)(row + lane) * cols + col;
                    const bool row_on = row + lane < p.rows[tile.product];
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        uint4 gv = make_uint4(0, 0, 0, 0), uv = gv;
                        if (row_on && col + 8 * q < cols) {
                            gv = *reinterpret_cast<const uint4*>(static_cast<const T*>(p.gate) + e + 8 * q);
                            uv = *reinterpret_cast<const uint4*>(static_cast<const T*>(p.up) + e + 8 * q);
                        }
                        g[4 * q] = gv.x; g[4 * q + 1] = gv.y; g[4 * q + 2] = gv.z; g[4 * q + 3] = gv.w;
                        u[4 * q] = uv.x; u[4 * q + 1] = uv.y; u[4 * q + 2] = uv.z; u[4 * q + 3] = uv.w;
                    }
                    tmem_ld32(at, r);
                    tmem_wait_ld();
#pragma unroll
                    for (int j = 0; j < 16; ++j) {
                        const float2 gf = ff_unpack<T>(g[j]), uf = ff_unpack<T>(u[j]);
                        const float d0 = __uint_as_float(r[2 * j]), d1 = __uint_as_float(r[2 * j + 1]);
                        float s0, s1;
                        const float a0 = ff_act(gf.x, p.act, &s0), a1 = ff_act(gf.y, p.act, &s1);
                        o[j] = ff_pack<T>(d0 * uf.x * s0, d1 * uf.y * s1);
                        u[j] = ff_pack<T>(d0 * a0, d1 * a1);
                        h[j] = ff_pack<T>(a0 * uf.x, a1 * uf.y);
                    }
                    out.put(&p.out[0], o, col, row, lane);
                    out.put(&p.out[1], u, col, row, lane);
                    out.put(&p.out[2], h, col, row, lane);
                }
            }
            fence_before_sync();
            __syncwarp();
            if (lane == 0) mbar_arrive(bar_acc_free + 8 * acc);
            if (acc) acc_phase ^= 1;
            acc ^= 1;
        }
        if (lane == 0) bulk_wait_all();
    }
    fence_before_sync();
    __syncthreads();
    if (warp == C::WARP_MMA) {
        fence_after_sync();
        tmem_dealloc(tmem, 512);
    }
}
