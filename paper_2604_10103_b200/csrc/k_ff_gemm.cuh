// Products of the gated feed-forward on the Blackwell tensor path, one kernel for all of them: D = A B^T over tiles of 128 rows and up to
// 256 columns, accumulators in tensor memory, operands brought by TMA, with an epilogue of its own for each use:
//   GATED    g = x Wg^T and u = x Wu^T side by side in one accumulator; h = act(g) u (and g, u)       A, B: contraction contiguous
//   STORE    the product itself                                                                       (y, dx, dW)
//   DHIDDEN  dh = dy Wd; dg = dh u act'(g), du = dh act(g), h = act(g) u                               B: columns contiguous
// An operand whose contraction index is contiguous ("K-major") is a box of 64 contraction elements by its rows; one whose row index is
// contiguous ("MN-major": Wd in dh, Wg and Wu in dx, everything in dW) is read as it lies too, in boxes of 64 rows by 64 contraction
// elements: the tensor cores take both, so nothing is transposed in memory.  Elements past an operand's end read as zero.
// A thread block is persistent: a loader thread, an MMA thread, and eight epilogue warps that empty one accumulator while the MMAs fill the
// other.  CG 2: two thread blocks on neighbouring SMs share a tile of 256 rows (cta_group::2): each holds its 128 rows of A and of the
// accumulator and half of B, which the tensor cores of both read, so a tile costs a third less operand traffic; the first of the pair
// issues the MMAs of both.  Every wait is bounded (~1 s) and reports through the status word; the two cluster barriers are reached by every
// thread whatever became of its waits: one before the roles part, one behind all of them.
// Roundings: accumulators and everything an epilogue computes are float32; what goes on to another product (h; dg, du, h) is rounded to the
// operands' 16-bit type there, once, as is each result.  Two roundings an output, 1.41 times one's error (bf16 0.00235 in the 2-norm of y, of one
// 0.00166).  Kept wider, as a high and a low half, it would take the products that read it twice over: a third more MMAs forward, five
// sixths backward, and twice the bytes between the launches.
// What bounds it: the MMAs, shared memory's bandwidth and the power limit, all near their ends at once.  Tiles of 256 x 256 a pair take 512
// cycles of MMAs for each 64 of the contraction, in which 32 KB are written into and 32 KB read out of each thread block's shared memory:
// its 128 bytes a cycle.  So tiles of one thread block (96 KB in the same cycles) are slower the longer they run, what an epilogue moves
// through shared memory stops the MMAs, and dW, whose contraction is long, has tiles of 256 x 512 (a quarter less).  us (TFLOP/s) alone: 4680
// rows, width 1536, hidden 4096: g, u, h 80 (1470), y 50 (1180: 114 tiles of 256 x 256, 133 of 224, on 74 pairs), dh and its epilogue 73
// (810: 304 tiles, four rounds and eight tiles; see FF_DHIDDEN below), dx 96 (1230), dW 118 (1500); 32760 rows: dh 410 (1005), dx 560 (1470), dW 751
// (1650).  In a loop the power limit takes a tenth off.
#pragma once
#include <cooperative_groups.h>
#include "tc5_common.cuh"
#include "k_vec.cuh"

enum { FF_GATED = 0, FF_STORE = 1, FF_DHIDDEN = 2 };

struct FfGemmParams {
    CUtensorMap a[3], b[3], out[3];     // operands of each product, or of each segment of the contraction; GATED: b = Wg, Wu
                                        // (DHIDDEN: out[0] is a map of dg, du, h as [3, rows, cols])
    CUtensorMap in[2];                  // DHIDDEN: gate and up [rows, cols]
    int products;                       // products of this launch, each with tiles of its own ...
    int tile0[4];                       // ... from tile0[i] to tile0[i + 1]
    int rows[3], cols[3];               // of the output
    int kb[3];                          // blocks of 64 of each product's (or segment's) contraction
    int segments;                       // contraction in this many segments (dx = dg Wg + du Wu: two)
    int splits;                         // STORE: the contraction of a tile is split over this many, whose sums go to `partials` (k_ff_join adds them)
    float* partials;
    int bn;                             // accumulator columns of a tile: a multiple of 32 (GATED: half of them g, half u)
    int stages;
    int act, save;
    int early_b;                        // B may be read before the kernel before this one is done
    int* dev_status;
};

// NB: accumulators of 256 columns a tile.  1: a tile's epilogue runs under the next tile's MMAs; 2 (STORE, long contractions): tiles of 512
// columns, a quarter less operand traffic, with the epilogue in between.
template <int EPI, int CG, int NB = 1>
struct FfGemm {
    static constexpr int BM = 128, BK = 64;             // rows of a thread block, contraction of a stage
    static constexpr int A_BYTES = BM * BK * 2;
    static constexpr int EPI_WARPS = 8, CW = 32;        // CW: columns that an epilogue warp takes at a time
    static constexpr int WARP_TMA = EPI_WARPS, WARP_MMA = EPI_WARPS + 1;
    static constexpr int THREADS = 32 * (EPI_WARPS + 2);
    static constexpr int MAX_STAGES = 8;
    // per epilogue warp: two boxes of 32 rows x CW columns on their way out; DHIDDEN: two sets of three, two of them in and out
    static constexpr int BOX = 64 * CW, STAGING = (EPI == FF_DHIDDEN ? 6 : 2) * BOX;
    static constexpr int BAR_BYTES = 384;
    static constexpr int SMEM_MAX = 232448;
    // bn: columns of an accumulator; NB bn / CG columns of B in each thread block (in boxes of 64 where the operand is MN-major)
    __host__ __device__ static constexpr int stage_bytes(int bn) { return A_BYTES + (NB * bn / CG + 63) / 64 * 64 * BK * 2; }
    static constexpr int smem_bytes(int bn, int stages) { return stages * stage_bytes(bn) + EPI_WARPS * STAGING + BAR_BYTES + 1024; }
    static constexpr int stages_for(int bn) {
        const int n = (SMEM_MAX - EPI_WARPS * STAGING - BAR_BYTES - 1024) / stage_bytes(bn);
        return n < MAX_STAGES ? n : MAX_STAGES;
    }
};

namespace tc5 {
template <int CG> __device__ __forceinline__ void ff_tmem_alloc(uint32_t smem_dst, uint32_t columns) {
    if constexpr (CG == 1) { tmem_alloc(smem_dst, columns); tmem_relinquish(); }
    else {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;\n" ::"r"(smem_dst), "r"(columns) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;\n" ::: "memory");
    }
}
template <int CG> __device__ __forceinline__ void ff_tmem_dealloc(uint32_t taddr, uint32_t columns) {
    if constexpr (CG == 1) tmem_dealloc(taddr, columns);
    else asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;\n" ::"r"(taddr), "r"(columns) : "memory");
}
template <int CG> __device__ __forceinline__ void ff_mma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, bool accumulate) {
    if constexpr (CG == 1) mma_ss(d, a, b, idesc, accumulate);
    else asm volatile("{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n}\n"
                      ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"((uint32_t)accumulate) : "memory");
}
// Arrival on the barrier at this place of shared memory (of both thread blocks of the pair) when the MMAs issued so far are done.
template <int CG> __device__ __forceinline__ void ff_commit(uint32_t bar) {
    if constexpr (CG == 1) mma_commit(bar);
    else asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;\n"
                      ::"r"(bar), "h"((uint16_t)3) : "memory");
}
// Load of this thread block's own tile; the bytes count on `bar`, which may be the pair's first thread block's.
template <int CG> __device__ __forceinline__ void ff_load(uint32_t dst, const CUtensorMap* map, int c0, int c1, uint32_t bar) {
    if constexpr (CG == 1) tma_load_2d(dst, map, c0, c1, bar);
    else asm volatile("cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];\n"
                      ::"r"(dst), "l"(reinterpret_cast<uint64_t>(map)), "r"(c0), "r"(c1), "r"(bar) : "memory");
}
// The same place of shared memory in the pair's first thread block.
template <int CG> __device__ __forceinline__ uint32_t ff_first(uint32_t addr) {
    if constexpr (CG == 1) return addr;
    uint32_t r;
    asm("mapa.shared::cluster.u32 %0, %1, 0;\n" : "=r"(r) : "r"(addr));
    return r;
}
template <int CG> __device__ __forceinline__ void ff_arrive_first(uint32_t bar) {
    if constexpr (CG == 1) mbar_arrive(bar);
    else asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];\n" ::"r"(bar) : "memory");
}
// All threads of the thread block, or of the pair.
template <int CG> __device__ __forceinline__ void ff_meet() {
    if constexpr (CG == 1) __syncthreads();
    else cooperative_groups::this_cluster().sync();
}
}  // namespace tc5

// silu: a = g p, a' = p (1 + g (1 - p)), p = 1 / (1 + e^-g).   gelu (tanh form): with v = A (g + B g^3) the factor (1 + tanh v) / 2 is
// 1 / (1 + e^-2v), so it is g p with another exponent: a' = p + g p (1 - p) 2 A (1 + 3 B g^2).
// ex2.approx and rcp.approx (2 and 1 ulp; an exponential that overflows gives p = 0, the right limit).
__device__ __forceinline__ float ff_rcp(float v) {
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;\n" : "=f"(r) : "f"(v));
    return r;
}
constexpr float FF_GELU_2A = 1.5957691216057308f, FF_GELU_B = 0.044715f, FF_LOG2E = 1.4426950408889634f;
// Two elements at a time (packed float32 arithmetic): a and, where asked for, a'.
template <int ACT, bool SLOPE> __device__ __forceinline__ float2 ff_act2(float2 g, float2* slope) {
    const float2 one = make_float2(1.f, 1.f);
    // - log2(e) times the exponent
    float2 x;
    if constexpr (ACT == HF_ACT_SILU) x = fmul2(g, make_float2(-FF_LOG2E, -FF_LOG2E));
    else x = fmul2(fmul2(g, make_float2(-FF_LOG2E * FF_GELU_2A, -FF_LOG2E * FF_GELU_2A)), ffma2(fmul2(g, g), make_float2(FF_GELU_B, FF_GELU_B), one));
    const float2 d = fadd2(make_float2(fast_exp2(x.x), fast_exp2(x.y)), one);
    const float2 p = make_float2(ff_rcp(d.x), ff_rcp(d.y)), a = fmul2(g, p);
    if constexpr (SLOPE) {
        const float2 q = ffma2(p, make_float2(-1.f, -1.f), one);
        if constexpr (ACT == HF_ACT_SILU) *slope = ffma2(a, q, p);
        else {
            // (a q is 0 long before the square of the gate overflows, which it may not make a NaN of)
            const float2 gg = fmul2(g, g), s = make_float2(fminf(gg.x, 1e30f), fminf(gg.y, 1e30f));
            *slope = ffma2(fmul2(a, q), ffma2(s, make_float2(3.f * FF_GELU_B * FF_GELU_2A, 3.f * FF_GELU_B * FF_GELU_2A), make_float2(FF_GELU_2A, FF_GELU_2A)), p);
        }
    }
    return a;
}
template <int ACT> __device__ __forceinline__ float ff_act(float g) { return ff_act2<ACT, false>(make_float2(g, g), nullptr).x; }
// The lane's 32 elements at a time, the activation known to the compiler: their latencies overlap, which a branch an element would prevent.
// h = act(g) u from the accumulators:
template <typename T, int ACT> __device__ __forceinline__ void ff_gated_row(const uint32_t (&g)[32], const uint32_t (&u)[32], uint32_t (&h)[16]) {
#pragma unroll
    for (int j = 0; j < 16; ++j) {
        const float2 a = ff_act2<ACT, false>(make_float2(__uint_as_float(g[2 * j]), __uint_as_float(g[2 * j + 1])), nullptr);
        const float2 o = fmul2(a, make_float2(__uint_as_float(u[2 * j]), __uint_as_float(u[2 * j + 1])));
        h[j] = pack2<T>(o.x, o.y);
    }
}
// g, u -> dg, du; h; from dh:
template <typename T, int ACT> __device__ __forceinline__ void ff_hidden_row(const uint32_t (&dh)[32], uint32_t (&g)[16], uint32_t (&u)[16], uint32_t (&h)[16]) {
#pragma unroll
    for (int j = 0; j < 16; ++j) {
        const float2 gf = unpack2<T>(g[j]), uf = unpack2<T>(u[j]), d = make_float2(__uint_as_float(dh[2 * j]), __uint_as_float(dh[2 * j + 1]));
        float2 s;
        const float2 a = ff_act2<ACT, true>(gf, &s), dg = fmul2(fmul2(d, uf), s), du = fmul2(d, a), o = fmul2(a, uf);
        g[j] = pack2<T>(dg.x, dg.y);
        u[j] = pack2<T>(du.x, du.y);
        h[j] = pack2<T>(o.x, o.y);
    }
}

struct FfTile { int product, m0, n0, split, index; };
// Tiles of a product in groups of 16 row tiles (bm rows each), all columns of a group before the next: the thread blocks at work at a time
// share rows and columns of both operands in L2.
__device__ __forceinline__ FfTile ff_tile(const FfGemmParams& p, int t, int bm, int bn_out) {
    FfTile r;
    r.split = 0;
    if (p.splits > 1) { r.split = t % p.splits; t /= p.splits; }
    r.index = t;
    r.product = 0;
    while (r.product + 1 < p.products && t >= p.tile0[r.product + 1]) ++r.product;
    t -= p.tile0[r.product];
    const int tm = (p.rows[r.product] + bm - 1) / bm, tn = (p.cols[r.product] + bn_out - 1) / bn_out;
    const int group = t / (16 * tn), first = group * 16, size = min(16, tm - first), in = t - group * 16 * tn;
    r.m0 = (first + in % size) * bm;
    r.n0 = in / size * bn_out;
    return r;
}

// A box of 32 rows x 32 columns in shared memory: 64-byte rows, 16-byte pieces swizzled as the maps say.
__device__ __forceinline__ uint32_t ff_piece(uint32_t box, int row, int piece) { return box + row * 64 + ((piece ^ ((row >> 1) & 3)) << 4); }
__device__ __forceinline__ void ff_put_row(uint32_t box, const uint32_t (&v)[16], int lane) {
#pragma unroll
    for (int c = 0; c < 4; ++c)
        asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};\n" ::"r"(ff_piece(box, lane, c)),
                     "r"(v[4 * c]), "r"(v[4 * c + 1]), "r"(v[4 * c + 2]), "r"(v[4 * c + 3]) : "memory");
}
__device__ __forceinline__ void ff_get_row(uint32_t box, uint32_t (&v)[16], int lane) {
#pragma unroll
    for (int c = 0; c < 4; ++c)
        asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];\n" : "=r"(v[4 * c]), "=r"(v[4 * c + 1]), "=r"(v[4 * c + 2]), "=r"(v[4 * c + 3])
                     : "r"(ff_piece(box, lane, c)) : "memory");
}
// One box on its way out: packed pairs of the lane's row -> one of the warp's two boxes -> TMA, which leaves out what lies past the
// tensor's end.
struct FfOut {
    uint32_t base;
    int next;
    __device__ __forceinline__ void put(const CUtensorMap* map, const uint32_t (&v)[16], int col, int row, int lane) {
        const uint32_t buf = base + next * 2048;
        next ^= 1;
        if (lane == 0) tc5::bulk_wait_read_but<1>();        // the store before the last has read this buffer
        __syncwarp();
        ff_put_row(buf, v, lane);
        tc5::fence_proxy_async();
        __syncwarp();
        if (lane == 0) {
            tc5::tma_store_2d(map, buf, col, row);
            tc5::bulk_commit();
        }
    }
};

template <typename T, int EPI, bool A_MN, bool B_MN, int CG, int NB = 1>
__global__ void __launch_bounds__(FfGemm<EPI, CG, NB>::THREADS, 1)
k_ff_gemm(const __grid_constant__ FfGemmParams p) {
    using namespace tc5;
    typedef FfGemm<EPI, CG, NB> C;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t s_base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    uint8_t* s_gen = smem_raw + (s_base - smem_u32(smem_raw));
    const int stage_bytes = C::stage_bytes(p.bn), stages = p.stages;
    const uint32_t s_staging = s_base + stages * stage_bytes, bar0 = s_staging + C::EPI_WARPS * C::STAGING;
    const uint32_t bar_full = bar0, bar_free = bar0 + 64, bar_acc = bar0 + 128, bar_acc_free = bar0 + 144, bar_in = bar0 + 192;
    uint8_t* bar_gen = s_gen + (bar0 - s_base);
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bar_gen + 160);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(bar_gen + 164);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int rank = CG == 1 ? 0 : (int)(blockIdx.x & 1);                   // (clusters are two neighbouring thread blocks)
    const int bn_out = EPI == FF_GATED ? p.bn / 2 : NB * p.bn, bn_own = NB * p.bn / CG;
    constexpr int ACCS = 2 / NB;                        // accumulators (sets of them) in turn
    const uint32_t acc_stride = p.bn > 128 ? 256 : (p.bn > 64 ? 128 : 64);         // columns of tensor memory from one to the next
    const int n_tiles = p.tile0[p.products] * p.splits, tile_first = blockIdx.x / CG, tile_step = gridDim.x / CG;

    if (threadIdx.x == 0) {
        for (int s = 0; s < stages; ++s) { mbar_init(bar_full + 8 * s, 1); mbar_init(bar_free + 8 * s, 1); }
        for (int s = 0; s < 2; ++s) { mbar_init(bar_acc + 8 * s, 1); mbar_init(bar_acc_free + 8 * s, C::EPI_WARPS * CG); }
        if (EPI == FF_DHIDDEN)
            for (int s = 0; s < 2 * C::EPI_WARPS; ++s) mbar_init(bar_in + 8 * s, 1);
        *abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;\n" ::: "memory");
    }
    if (warp == C::WARP_MMA) ff_tmem_alloc<CG>(smem_u32(tmem_slot), 2 * acc_stride);
    fence_before_sync();
    ff_meet<CG>();
    fence_after_sync();
    const uint32_t tmem = *tmem_slot;
    // The kernel may have been launched while the one before it still runs: only the threads that read global memory themselves wait for
    // that, everything else follows from what they read.  The next kernel may be launched once this one has waited, so that what was
    // written before this one is there for it from the start (early_b).
    if (warp == C::WARP_TMA) {
        // ================================================================= loader
        if (lane == 0) {
            bool ok = true;
            int s = 0;
            uint32_t phase = 1;                 // (the stages are free at first)
            const int b_boxes = B_MN ? (bn_own + 63) / 64 : 1;
            const uint32_t bytes = CG * (C::A_BYTES + (B_MN ? b_boxes * 8192 : bn_own * C::BK * 2));        // of the whole tile
            auto load_a = [&](const FfTile& tile, int k, uint32_t sA, uint32_t full) {
                const int seg = p.segments > 1 && k >= p.kb[0], i = tile.product + seg;       // (one of the two is always 0)
                const int kc = (k - seg * p.kb[0]) * C::BK, m0 = tile.m0 + rank * C::BM;
                if (A_MN) {
                    ff_load<CG>(sA, &p.a[i], m0, kc, full);
                    ff_load<CG>(sA + 8192, &p.a[i], m0 + 64, kc, full);
                } else
                    ff_load<CG>(sA, &p.a[i], kc, m0, full);
            };
            auto load_b = [&](const FfTile& tile, int k, uint32_t sB, uint32_t full) {
                const int seg = p.segments > 1 && k >= p.kb[0], i = tile.product + seg;
                const int kc = (k - seg * p.kb[0]) * C::BK, n0 = tile.n0 + (EPI == FF_GATED ? 0 : rank * bn_own);
                if (EPI == FF_GATED) {
                    // g's columns in front of u's: the pair's first thread block holds Wg's rows, the second Wu's
                    ff_load<CG>(sB, &p.b[rank], kc, n0, full);
                    if (CG == 1) ff_load<CG>(sB + bn_out * C::BK * 2, &p.b[1], kc, n0, full);
                } else if (B_MN) {
                    for (int x = 0; x < b_boxes; ++x) ff_load<CG>(sB + x * 8192, &p.b[i], n0 + 64 * x, kc, full);
                } else
                    ff_load<CG>(sB, &p.b[i], kc, n0, full);
            };
            bool first = true;
            for (int t = tile_first; ok && t < n_tiles; t += tile_step) {
                const FfTile tile = ff_tile(p, t, CG * C::BM, bn_out);
                const int k_all = p.kb[tile.product] * p.segments;      // (segments: of the same length)
                const int k_end = (int)((long long)k_all * (tile.split + 1) / p.splits);
                int k = (int)((long long)k_all * tile.split / p.splits);
                if (first) {
                    first = false;
                    // weights on their way before the rows of the other operand are there
                    const int ahead = p.early_b ? min(stages, k_end - k) : 0;
                    for (int j = 0; j < ahead; ++j) {
                        if (rank == 0) mbar_expect_tx(bar_full + 8 * j, bytes);
                        load_b(tile, k + j, s_base + j * stage_bytes + C::A_BYTES, ff_first<CG>(bar_full + 8 * j));
                    }
                    pdl_wait();
                    pdl_trigger();
                    for (int j = 0; j < ahead; ++j, ++k) {
                        load_a(tile, k, s_base + j * stage_bytes, ff_first<CG>(bar_full + 8 * j));
                        if (++s == stages) { s = 0; phase ^= 1; }
                    }
                }
                for (; k < k_end; ++k) {
                    if (!(ok = mbar_wait<true>(bar_free + 8 * s, phase, abort_flag, p.dev_status, 81))) break;
                    const uint32_t sA = s_base + s * stage_bytes, full = ff_first<CG>(bar_full + 8 * s);
                    if (rank == 0) mbar_expect_tx(bar_full + 8 * s, bytes);
                    load_a(tile, k, sA, full);
                    load_b(tile, k, sA + C::A_BYTES, full);
                    if (++s == stages) { s = 0; phase ^= 1; }
                }
            }
            // every stage's MMAs are done before this thread block (whose memory the pair's MMAs read and signal) may leave
            for (int i = 0; ok && i < stages; ++i) {
                ok = mbar_wait<true>(bar_free + 8 * s, phase, abort_flag, p.dev_status, 86);
                if (++s == stages) { s = 0; phase ^= 1; }
            }
            if (!ok) {                          // copies in flight land before the thread block leaves
                const long long t0 = clock64();
                while (clock64() - t0 < 400000) {}
            }
        }
    } else if (warp == C::WARP_MMA) {
        // ================================================================= MMA issuer (warp-uniform, one elected lane issues)
        constexpr uint32_t TYPE = std::is_same<T, bf16>::value ? 1u : 0u;
        const uint32_t idesc = (1u << 4) | (TYPE << 7) | (TYPE << 10) | ((A_MN ? 1u : 0u) << 15) | ((B_MN ? 1u : 0u) << 16) |
                               ((uint32_t)(p.bn >> 3) << 17) | ((uint32_t)(CG * C::BM >> 4) << 24);
        const uint64_t da0 = smem_desc_sw128(s_base, A_MN ? 8192 : 16, 1024);
        const uint64_t db0 = smem_desc_sw128(s_base + C::A_BYTES, B_MN ? 8192 : 16, 1024);
        constexpr int A_STEP = (A_MN ? 2048 : 32) >> 4, B_STEP = (B_MN ? 2048 : 32) >> 4;
        const int b_half = (p.bn / CG * C::BK * 2) >> 4;            // (NB 2: bn / CG is a multiple of 64)
        bool ok = rank == 0;
        int s = 0, acc = 0;
        uint32_t phase = 0, acc_phase = 1;
        for (int t = tile_first; ok && t < n_tiles; t += tile_step) {
            const FfTile tile = ff_tile(p, t, CG * C::BM, bn_out);
            const int k_all = p.kb[tile.product] * p.segments;
            const int n_kb = (int)((long long)k_all * (tile.split + 1) / p.splits) - (int)((long long)k_all * tile.split / p.splits);
            if (!(ok = mbar_wait_warp<true>(bar_acc_free + 8 * acc, acc_phase, abort_flag, p.dev_status, 82))) break;
            fence_after_sync();
            for (int kb = 0; kb < n_kb; ++kb) {
                if (!(ok = mbar_wait_warp<true>(bar_full + 8 * s, phase, abort_flag, p.dev_status, 83))) break;
                fence_after_sync();
                if (elect_one()) {
                    const uint64_t off = (uint64_t)((s * stage_bytes) >> 4);
#pragma unroll
                    for (int ks = 0; ks < C::BK / 16; ++ks)
#pragma unroll
                        for (int h = 0; h < NB; ++h)
                            ff_mma<CG>(tmem + (acc + h) * acc_stride, da0 + off + ks * A_STEP, db0 + off + ks * B_STEP + h * b_half, idesc, kb > 0 || ks > 0);
                    ff_commit<CG>(bar_free + 8 * s);
                    if (kb == n_kb - 1) ff_commit<CG>(bar_acc + 8 * acc);
                }
                __syncwarp();
                if (++s == stages) { s = 0; phase ^= 1; }
            }
            if (++acc == ACCS) { acc = 0; acc_phase ^= 1; }
        }
    } else {
        // ================================================================= epilogue: warps w and w + 4 share the accumulator rows 32 (w & 3) ...
        constexpr int CW = C::CW;
        const int quad = warp & 3, half = warp >> 2;
        const uint32_t lane_base = tmem + ((uint32_t)(quad * 32) << 16);
        const uint32_t staging = s_staging + warp * C::STAGING;
        FfOut out = {staging, 0};
        int acc = 0;
        uint32_t acc_phase = 0;
        // DHIDDEN moves five elements for each of dh (in: gate, up; out: dg, du, h).  us of 4680 rows under a profiler: this form 73; gate and up through
        // registers 76.5; sixteen warps with boxes of 16 columns 74.5; straight between registers and global memory, 32 bytes a lane, 87; without
        // an epilogue at all 50.
        // Boxes of gate and up come in by TMA one step ahead of their use and leave as dg and du, in place, with h in a third box; two
        // sets of the three in turn.  in_*: the next step to ask for.
        const uint32_t in_bar = bar_in + warp * 16;
        int in_t = tile_first, in_c = half, in_set = 0, use_n = 0;
        FfTile in_tile = ff_tile(p, min(tile_first, n_tiles - 1), CG * C::BM, bn_out);
        auto ask = [&]() {
            while (in_t < n_tiles) {
                const int row = in_tile.m0 + rank * C::BM + quad * 32, col = in_tile.n0 + CW * in_c;
                if (row >= p.rows[0] || in_c >= bn_out / CW || col >= p.cols[0]) {
                    in_t += tile_step; in_c = half;
                    if (in_t < n_tiles) in_tile = ff_tile(p, in_t, CG * C::BM, bn_out);
                    continue;
                }
                const uint32_t b = in_bar + 8 * in_set, to = staging + in_set * 3 * C::BOX;
                mbar_expect_tx(b, 2 * C::BOX);
                tma_load_2d(to, &p.in[0], col, row, b);
                tma_load_2d(to + C::BOX, &p.in[1], col, row, b);
                in_set ^= 1;
                in_c += 2;
                return;
            }
        };
        if (EPI == FF_DHIDDEN && lane == 0) { pdl_wait(); ask(); }
        for (int t = tile_first; t < n_tiles; t += tile_step) {
            const FfTile tile = ff_tile(p, t, CG * C::BM, bn_out);
            if (!mbar_wait_warp<true>(bar_acc + 8 * acc, acc_phase, abort_flag, p.dev_status, 84)) break;
            fence_after_sync();
            const int row = tile.m0 + rank * C::BM + quad * 32, cols = p.cols[tile.product];
            const bool rows_on = row < p.rows[tile.product];
            bool ok = true;
            for (int c = half; c < bn_out / CW; c += 2) {
                // NB 2: columns h bn + ... of the accumulators are, of each thread block's half of the tile's columns, the h-th half
                const int h2 = NB == 1 ? 0 : c / (p.bn / CW), in = CW * c - h2 * p.bn, owner = NB == 1 ? 0 : in / (p.bn / CG);
                const int col = tile.n0 + (NB == 1 ? in : owner * bn_own + h2 * (p.bn / CG) + in - owner * (p.bn / CG));
                if (!rows_on || (NB == 1 && col >= cols)) break;
                if (NB == 2 && col >= cols) continue;
                const uint32_t at = lane_base + (acc + h2) * acc_stride + in;
                uint32_t r[32], o[16];
                tmem_ld32(at, r);
                if constexpr (EPI == FF_STORE) {
                    tmem_wait_ld();
                    if (p.splits > 1) {             // [tile][split][32 rows][32 columns]: column by column, so that a warp's stores are whole lines
                        float* to = p.partials + ((((size_t)tile.index * p.splits + tile.split) * CG + rank) * 4 + quad) * 32 * p.bn + c * 1024 + lane;
#pragma unroll
                        for (int j = 0; j < 32; ++j) to[32 * j] = __uint_as_float(r[j]);
                        continue;
                    }
#pragma unroll
                    for (int j = 0; j < 16; ++j) o[j] = pack2<T>(__uint_as_float(r[2 * j]), __uint_as_float(r[2 * j + 1]));
                    out.put(&p.out[tile.product], o, col, row, lane);
                } else if constexpr (EPI == FF_GATED) {
                    uint32_t u[32];
                    tmem_ld32(at + bn_out, u);
                    tmem_wait_ld();
                    if (p.save) {
#pragma unroll
                        for (int j = 0; j < 16; ++j) o[j] = pack2<T>(__uint_as_float(r[2 * j]), __uint_as_float(r[2 * j + 1]));
                        out.put(&p.out[1], o, col, row, lane);
#pragma unroll
                        for (int j = 0; j < 16; ++j) o[j] = pack2<T>(__uint_as_float(u[2 * j]), __uint_as_float(u[2 * j + 1]));
                        out.put(&p.out[2], o, col, row, lane);
                    }
                    if (p.act == HF_ACT_SILU) ff_gated_row<T, HF_ACT_SILU>(r, u, o);
                    else ff_gated_row<T, HF_ACT_GELU_TANH>(r, u, o);
                    out.put(&p.out[0], o, col, row, lane);
                } else {
                    uint32_t u[16], h[16];
                    const int set = use_n & 1;
                    const uint32_t boxes = staging + set * 3 * C::BOX;
                    ok = mbar_wait_warp<true>(in_bar + 8 * set, (use_n >> 1) & 1, abort_flag, p.dev_status, 85);
                    ++use_n;
                    if (!ok) { tmem_wait_ld(); break; }
                    ff_get_row(boxes, o, lane);
                    ff_get_row(boxes + C::BOX, u, lane);
                    if (lane == 0) {
                        bulk_wait_read();           // the stores of the step before have read the other set
                        ask();
                    }
                    __syncwarp();
                    tmem_wait_ld();
                    if (p.act == HF_ACT_SILU) ff_hidden_row<T, HF_ACT_SILU>(r, o, u, h);
                    else ff_hidden_row<T, HF_ACT_GELU_TANH>(r, o, u, h);
                    // (each lane's row of dg and du takes the place of its own row of gate and up)
                    ff_put_row(boxes, o, lane);
                    ff_put_row(boxes + C::BOX, u, lane);
                    ff_put_row(boxes + 2 * C::BOX, h, lane);
                    fence_proxy_async();
                    __syncwarp();
                    if (lane == 0) {
                        tma_store_3d(&p.out[0], boxes, col, row, 0);        // all three boxes
                        bulk_commit();
                    }
                }
            }
            if (!ok) break;
            fence_before_sync();
            __syncwarp();
            if (lane == 0) ff_arrive_first<CG>(ff_first<CG>(bar_acc_free + 8 * acc));
            if (++acc == ACCS) { acc = 0; acc_phase ^= 1; }
        }
        if (lane == 0) bulk_wait_all();
        if (EPI == FF_DHIDDEN && *abort_flag) {         // boxes in flight land before the thread block leaves
            const long long t0 = clock64();
            while (clock64() - t0 < 400000) {}
        }
    }
    __syncwarp();
    fence_before_sync();
    ff_meet<CG>();
    if (warp == C::WARP_MMA) {
        fence_after_sync();
        ff_tmem_dealloc<CG>(tmem, 2 * acc_stride);
    }
}

// out = the sum over the splits of the partials of k_ff_gemm, in order, rounded once.  A warp takes 32 rows x 8 columns.
struct FfJoinOut { void* out[3]; long long stride[3]; int cg; };
template <typename T>
__global__ void __launch_bounds__(128)
k_ff_join(const __grid_constant__ FfGemmParams p, const FfJoinOut o) {
    const int lane = threadIdx.x & 31, eights = p.bn / 8, units = 4 * o.cg * eights;
    const int id = blockIdx.x * 4 + (threadIdx.x >> 5), index = id / units, unit = id - index * units;
    pdl_wait();
    if (index >= p.tile0[p.products]) return;
    const FfTile tile = ff_tile(p, index * p.splits, 128 * o.cg, p.bn);
    const int rows32 = unit / eights, c = unit - rows32 * eights, row = tile.m0 + rows32 * 32 + lane, col = tile.n0 + 8 * c;
    if (row >= p.rows[tile.product] || col >= p.cols[tile.product]) return;
    const size_t step = (size_t)o.cg * 128 * p.bn;
    const float* from = p.partials + (size_t)index * p.splits * step + (size_t)rows32 * 32 * p.bn + c * 256 + lane;
    float v[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = 0.f;
#pragma unroll 4
    for (int s = 0; s < p.splits; ++s, from += step)
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] += from[32 * j];
    T* to = static_cast<T*>(o.out[tile.product]) + (size_t)row * o.stride[tile.product] + col;
    *reinterpret_cast<uint4*>(to) = make_uint4(pack2<T>(v[0], v[1]), pack2<T>(v[2], v[3]), pack2<T>(v[4], v[5]), pack2<T>(v[6], v[7]));
}
