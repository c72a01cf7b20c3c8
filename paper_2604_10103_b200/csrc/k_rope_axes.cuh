// Rotary positions with several axes.  Feature pair p of a token turns by the angle of its axis a(p) at the token's position on that
// axis, read from tables: (x0, x1) -> (x0 c - x1 s, x0 s + x1 c) (inverse: s -> -s, the transposed rotation, which is the backward pass).
// Products and sums in float32, one rounding at the end.  Up to three tensors of [batch, tokens, heads, head_dim] with strides of their
// own go through one launch (q, k, v between a projection's rows and head-major tensors); one that is not rotated is copied.
// Memory bounds it: a thread keeps the angles of its features of a token in registers and walks heads with them.  (Floors at the measured
// copy rate: 13.2 and 92.3 us for the two sizes below; the rest is the launch and the first loads' latency, and in the long call reads and
// writes of 256 bytes at a time on one of the two sides.)
#pragma once
#include "k_vec.cuh"

struct RopeTensor {
    const void* x; void* y;
    long long xb, xt, xh, yb, yt, yh;       // elements between batches, tokens, heads
    int heads, rotate;
};
struct RopeParams {
    RopeTensor t[3];
    const float* cos_tab; const float* sin_tab;
    const int* pos;
    long long pos_batch;                    // ints between batches (0: shared)
    int first[4], pairs[4], extent[4], tab[4];      // per axis: first pair, pairs, rows of the table, first entry of the table
    int axes, n_pairs;                      // n_pairs: rotated pairs; features behind them are copied
    int batch, tokens, units;               // units: threads of a token
    int n_tensors, head_dim, slices, total_heads;
    int inverse;
    int* dev_status;
};

// HALVES: pair p = features (p, n_pairs + p), otherwise (2p, 2p + 1).  A thread owns 2 V features of a token: V pairs, or 2 V features
// behind the rotated ones, in two pieces of V (neighbours unless HALVES).  WIDE: every piece of every tensor starts on a boundary of its
// own size (at most 16 bytes); otherwise V is 1 and elements are accessed one by one.
// Heads of a batch, whose loads are in flight together, and thread blocks a multiprocessor (registers): four 16-byte pieces and four thread
// blocks.  Rows of 12 + 24 heads of 128, us for 4680 and (backward) 32760 tokens: 19.3, 111.5 (5.4 TB/s); batches of twelve and two thread
// blocks 24.0, 146; of six and four 19.3, 112.3; of three and five 20.6, 109.5; of two and six 20.6, 125.
template <typename T, int V, bool WIDE> __host__ __device__ constexpr int rope_batch() { return WIDE && V * sizeof(T) == 16 ? 2 : 4; }
constexpr int ROPE_BLOCKS = 4;

template <typename T, int V, bool HALVES, bool WIDE>
__global__ void __launch_bounds__(256, ROPE_BLOCKS)
k_rope_axes(const RopeParams p) {
    constexpr int HB = rope_batch<T, V, WIDE>();
    const long long id = (long long)blockIdx.x * 256 + threadIdx.x;
    const long long bt = id / p.units;
    if (bt >= (long long)p.batch * p.tokens) return;
    const int u = (int)(id - bt * p.units), b = (int)(bt / p.tokens), tok = (int)(bt - (long long)b * p.tokens);
    // features f0 .. f0 + V - 1 and f1 .. f1 + V - 1
    const int pair0 = u * V;
    const bool turned = pair0 < p.n_pairs;                          // (HALVES: n_pairs is a multiple of V)
    const int f0 = HALVES && turned ? pair0 : 2 * pair0;
    const int f1 = HALVES && turned ? p.n_pairs + pair0 : f0 + V;
    // this slice's part of all tensors' heads, one after the other; a batch stays inside a tensor
    int h = (int)((long long)p.total_heads * blockIdx.y / p.slices), n = 0, base = 0;
    const int h_end = (int)((long long)p.total_heads * (blockIdx.y + 1) / p.slices);
    Vec<T, V, WIDE> lo[HB], hi[HB];
    const T* x; T* y;
    int stop;
    auto seek = [&]() {             // the tensor of head h
        while (h >= base + p.t[n].heads) { base += p.t[n].heads; ++n; }
        const RopeTensor& t = p.t[n];
        stop = min(h_end, base + t.heads);
        x = static_cast<const T*>(t.x) + b * t.xb + tok * t.xt + (h - base) * t.xh;
        y = static_cast<T*>(t.y) + b * t.yb + tok * t.yt + (h - base) * t.yh;
    };
    auto load = [&]() {
        const long long xh = p.t[n].xh;
#pragma unroll
        for (int k = 0; k < HB; ++k)
            if (h + k < stop) {
                if constexpr (HALVES || !WIDE) {
                    lo[k] = load_vec<T, V, WIDE>(x + k * xh + f0);
                    hi[k] = load_vec<T, V, WIDE>(x + k * xh + f1);
                } else {
                    const Vec<T, 2 * V> v = load_vec<T, 2 * V>(x + k * xh + f0);
                    memcpy(&lo[k], &v, sizeof(lo[k]));
                    memcpy(&hi[k], reinterpret_cast<const char*>(&v) + sizeof(lo[k]), sizeof(hi[k]));
                }
            }
    };
    seek();
    load();                         // (on its way while the angles are looked up)
    float c[V], s[V];
    bool on[V];
#pragma unroll
    for (int j = 0; j < V; ++j) {
        const int pr = pair0 + j;
        on[j] = pr < p.n_pairs;
        c[j] = 1.f; s[j] = 0.f;
        if (on[j]) {
            int a = 0;
            while (a + 1 < p.axes && pr >= p.first[a + 1]) ++a;
            int at = p.pos[b * p.pos_batch + (long long)tok * p.axes + a];
            if ((unsigned)at >= (unsigned)p.extent[a]) {            // outside the table: no address is formed from it
                atomicOr(p.dev_status, HF_DEV_BAD_INDEX_FLAG);
                atomicExch(p.dev_status + 1, tok);
                at = 0;
            }
            const int e = p.tab[a] + at * p.pairs[a] + pr - p.first[a];
            c[j] = p.cos_tab[e];
            s[j] = p.inverse ? -p.sin_tab[e] : p.sin_tab[e];
        }
    }
    // (x and y may be the same tensor: a thread writes only what it alone reads, and has read)
    for (;;) {
        const RopeTensor& t = p.t[n];
#pragma unroll
        for (int k = 0; k < HB; ++k)
            if (h + k < stop) {
                if (t.rotate) {
                    float e[2 * V], l[V], u2[V];
                    to_floats(lo[k], l);
                    to_floats(hi[k], u2);
#pragma unroll
                    for (int j = 0; j < V; ++j) { e[j] = l[j]; e[V + j] = u2[j]; }
#pragma unroll
                    for (int j = 0; j < V; ++j)
                        if (on[j]) {            // (an infinity behind the rotated pairs is copied, not multiplied by a zero sine)
                            const int i0 = HALVES ? j : 2 * j, i1 = HALVES ? V + j : 2 * j + 1;     // neighbours: pair j is elements (2j, 2j + 1)
                            const float x0 = e[i0], x1 = e[i1];
                            e[i0] = x0 * c[j] - x1 * s[j];
                            e[i1] = x0 * s[j] + x1 * c[j];
                        }
#pragma unroll
                    for (int j = 0; j < V; ++j) { l[j] = e[j]; u2[j] = e[V + j]; }
                    from_floats(lo[k], l);
                    from_floats(hi[k], u2);
                }
                if constexpr (HALVES || !WIDE) {
                    store_vec(y + k * t.yh + f0, lo[k]);
                    store_vec(y + k * t.yh + f1, hi[k]);
                } else {
                    Vec<T, 2 * V> v;
                    memcpy(&v, &lo[k], sizeof(lo[k]));
                    memcpy(reinterpret_cast<char*>(&v) + sizeof(lo[k]), &hi[k], sizeof(hi[k]));
                    store_vec(y + k * t.yh + f0, v);
                }
            }
        h += HB; x += HB * t.xh; y += HB * t.yh;
        if (h >= stop) {
            h = stop;
            if (h >= h_end) break;
            seek();
        }
        load();
    }
}
