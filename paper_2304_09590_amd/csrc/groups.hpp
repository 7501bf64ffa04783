// groups.hpp -- rows that name their network: grouping them, and the products of one layer of
// every network with the rows that name it (forward, input gradient, weight gradient).
//
// Row r of n has per_row pairs p = r per_row + j, each naming one of K networks (or none: an id
// outside [0, K), the pair is dropped).  The grouping is a stable counting sort of the pairs by
// network; network e's pairs are then the positions off[e] .. off[e + 1) of `pairs`, the dropped
// ones the positions from off[K].  The products read rows and write results through `pairs`, so
// nothing is ever moved into sorted order: x is read at row pair / per_row, y, dy at row pair.
//
//   forward          y[p]  = phi(W_e x[p / per_row] + b_e), e = id[p]
//   input gradient   dx[r] = sum_j W_e^T dy[r per_row + j] (.) phi'(a[r])
//   weight gradient  dW_e  = sum_p dy[p] x[p / per_row]^T,  db_e = sum_p dy[p]
#pragma once
#include "kernels.hpp"

namespace pnn {

constexpr int GR_MAX_NETS = 1024;   // most networks of a grouping (its counters live in LDS)
constexpr int GR_THREADS = 512, GR_WAVES = GR_THREADS / 64;
constexpr int GR_MAX_BLOCKS = 256;  // most workgroups that count (each reads all their counts)
constexpr int GR_CHUNK = 4096;      // pairs of a workgroup, eight a thread, in registers
constexpr int GR_ALONE = 8192;      // pairs of one that is alone: one launch for two
constexpr int GR_HEIGHTS = 4;       // pairs per tile: 16, and 64, 128 or 256 for the matrix-tile kernels

// Layout of a plan (int32 words): off[K + 1] | pairs[P] | numbers of tiles | tiles of 16, 64, 128 and
// 256 pairs | counts of the workgroups | with several pairs a row, a byte for each pair: 1 unless it is dropped.  A tile
// is (network, first position); network K stands for the dropped pairs.  The host knows only the most tiles there can
// be (extra workgroups end at once).  What lies before the bytes depends on the number of pairs alone, so a plan also
// serves the same pairs as rows of one pair each.
struct GroupPlan {
    int64_t P;
    int K;
    int64_t o_pairs, o_count, o_tiles[GR_HEIGHTS], o_hist, o_kept, words;
    int64_t most[GR_HEIGHTS];
    int blocks;
    int64_t chunk;  // pairs per counting workgroup
};

__host__ __device__ inline int group_height(int h) { return h == 0 ? 16 : 32 << h; }

__host__ inline GroupPlan group_plan(int64_t n, int per_row, int K) {
    GroupPlan g;
    g.P = n * per_row;
    g.K = K;
    const int64_t extra = g.P < K + 1 ? g.P : K + 1;
    auto up = [](int64_t v) { return (v + 3) / 4 * 4; };
    g.o_pairs = up(K + 1);
    g.o_count = g.o_pairs + up(g.P);
    int64_t at = g.o_count + up(GR_HEIGHTS);
    for (int h = 0; h < GR_HEIGHTS; ++h) {
        g.most[h] = g.P / group_height(h) + extra;
        g.o_tiles[h] = at;
        at += up(2 * g.most[h]);
    }
    g.o_hist = at;
    g.chunk = (g.P + GR_MAX_BLOCKS - 1) / GR_MAX_BLOCKS;
    if (g.chunk < GR_CHUNK) g.chunk = g.P <= GR_ALONE ? GR_ALONE : GR_CHUNK;
    g.blocks = (int)((g.P + g.chunk - 1) / g.chunk);
    g.o_kept = g.o_hist + (g.blocks > 1 ? up((int64_t)g.blocks * (K + 1)) : 0);
    g.words = g.o_kept + (per_row > 1 ? up((g.P + 3) / 4) : 0);
    return g;
}

struct GroupArgs {
    const int32_t* ids;
    int32_t *off, *pairs, *count, *hist;
    int2* tiles[GR_HEIGHTS];
    uint8_t* kept;  // (nullable) of each pair: 1 unless it is dropped
    int64_t P, chunk;
    int K, blocks;
};

__device__ inline int group_key(const GroupArgs& g, int64_t i) {
    const int id = g.ids[i];
    return (unsigned)id < (unsigned)g.K ? id : g.K;
}

// the keys of pairs i, i + STEP, ... below `end` (-1 from there on), all loads in flight together
template <int N, int STEP>
__device__ inline void group_keys(const GroupArgs& g, int64_t i, int64_t end, int* keys) {
    int id[N];
#pragma unroll
    for (int t = 0; t < N; ++t) id[t] = g.ids[i + t * STEP < g.P ? i + t * STEP : g.P - 1];
#pragma unroll
    for (int t = 0; t < N; ++t) keys[t] = i + t * STEP >= end ? -1 : (unsigned)id[t] < (unsigned)g.K ? id[t] : g.K;
}

// pairs of network e within this workgroup's chunk, into hist
__global__ __launch_bounds__(GR_THREADS) void group_count_kernel(GroupArgs g) {
    __shared__ int cnt[GR_MAX_NETS + 1];
    for (int e = threadIdx.x; e <= g.K; e += GR_THREADS) cnt[e] = 0;
    __syncthreads();
    const int64_t lo = blockIdx.x * g.chunk, hi = lo + g.chunk < g.P ? lo + g.chunk : g.P;
    for (int64_t b = lo + threadIdx.x; b < hi; b += GR_THREADS * 8) {  // (eight loads in flight)
        int keys[8];
        group_keys<8, GR_THREADS>(g, b, hi, keys);
#pragma unroll
        for (int t = 0; t < 8; ++t)
            if (keys[t] >= 0) atomicAdd(&cnt[keys[t]], 1);
    }
    __syncthreads();
    for (int e = threadIdx.x; e <= g.K; e += GR_THREADS) g.hist[(int64_t)blockIdx.x * (g.K + 1) + e] = cnt[e];
}

// exclusive scan of f(0 .. n - 1) into out[0 .. n], by one wave; a lane's values are neighbours
template <typename F>
__device__ inline void wave_scan(int* out, int n, int lane, F f) {
    const int per = (n + 63) / 64, lo = lane * per, hi = lo + per < n ? lo + per : n;
    int own = 0;
    for (int e = lo; e < hi; ++e) own += f(e);
    int s = own;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int u = __shfl_up(s, d);
        if (lane >= d) s += u;
    }
    int at = s - own;
    for (int e = lo; e < hi; ++e) {
        out[e] = at;
        at += f(e);
    }
    if (lane == 63) out[n] = s;
}

// Stable placement.  Every workgroup counts its chunk by wave (a wave owns a contiguous part), adds what the
// chunks and waves before it hold, and places its pairs.  The lanes of a wave that hold the same key find each
// other in LDS: each sets its bit in the key's word, and the bits below its own are its order.  (One ballot
// per key bit instead is 130 instructions a step: 120,000 pairs, 256 networks 12.9 us, this way 11.4.)  Bound by
// latencies one after another: of 12.6 us for both launches over the same pairs the other workgroups' counts take
// 3.5, the placing 3.6 and the tile lists 0.7.  Integer sums only: the same bits every run.  With one workgroup its own counts are all there is
// (no earlier launch).  All workgroups share the tiles.
template <int KEYS>
__global__ __launch_bounds__(GR_THREADS) void group_place_kernel(GroupArgs g) {
    constexpr int THREADS = GR_THREADS, WAVES = GR_WAVES;
    extern __shared__ int gsm[];
    const int K1 = g.K + 1, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    unsigned long long* bits = (unsigned long long*)gsm;  // [WAVES][K1 + 1], the last for lanes without a pair
    int* cur = (int*)(bits + WAVES * (K1 + 1));           // [WAVES][K1]
    int* tot = cur + WAVES * K1;                          // [K1]
    int* off = tot + K1;                                  // [K1 + 1]
    int* first = off + K1 + 1;                            // [GR_HEIGHTS][K1 + 1] first tile of each network
    for (int e = tid; e < WAVES * K1; e += THREADS) cur[e] = 0;
    for (int e = tid; e < WAVES * (K1 + 1); e += THREADS) bits[e] = 0;
    __syncthreads();
    const int64_t lo = blockIdx.x * g.chunk, hi = lo + g.chunk < g.P ? lo + g.chunk : g.P;
    const int64_t part = (g.chunk + WAVES * 64 - 1) / (WAVES * 64) * 64;
    const int64_t w0 = lo + wave * part, w1 = w0 + part < hi ? w0 + part : hi;
    // (a chunk of at most KEYS pairs a thread is read once, all loads in flight together)
    int keys[KEYS];
    const bool kept = part <= 64 * KEYS;
    if (g.P == 0) {
#pragma unroll
        for (int t = 0; t < KEYS; ++t) keys[t] = -1;
    } else if (kept) {
        group_keys<KEYS, 64>(g, w0 + lane, w1, keys);
#pragma unroll
        for (int t = 0; t < KEYS; ++t)
            if (keys[t] >= 0) atomicAdd(&cur[wave * K1 + keys[t]], 1);
    } else {
        for (int64_t i = w0 + lane; i < w1; i += 64) atomicAdd(&cur[wave * K1 + group_key(g, i)], 1);
    }
    __syncthreads();
    for (int e = tid; e < K1; e += THREADS) {
        int before = 0, all = 0;
        if (g.blocks > 1)
            for (int b0 = 0; b0 < g.blocks; b0 += 16) {
                int h[16];
#pragma unroll
                for (int b = 0; b < 16; ++b) h[b] = g.hist[(int64_t)(b0 + b < g.blocks ? b0 + b : g.blocks - 1) * K1 + e];
#pragma unroll
                for (int b = 0; b < 16; ++b) {
                    all += b0 + b < g.blocks ? h[b] : 0;
                    before += b0 + b < (int)blockIdx.x ? h[b] : 0;
                }
            }
        for (int w = 0; w < WAVES; ++w) {
            const int c = cur[w * K1 + e];
            cur[w * K1 + e] = before;
            before += c;
        }
        tot[e] = g.blocks > 1 ? all : before;
    }
    __syncthreads();
    if (wave == 0) wave_scan(off, K1, lane, [&](int e) { return tot[e]; });
    if (wave >= 1 && wave <= GR_HEIGHTS) {
        const int h = group_height(wave - 1);
        wave_scan(first + (wave - 1) * (K1 + 1), K1, lane, [&](int e) { return (tot[e] + h - 1) / h; });
    }
    __syncthreads();
    const uint64_t below = (1ull << lane) - 1;
    volatile unsigned long long* word = bits + wave * (K1 + 1);
    // N steps at a time: their words (a wave's LDS accesses keep their order), their counters, their places
    auto place = [&](auto steps, int64_t b, const int* key) {
        constexpr int N = decltype(steps)::value;
        uint64_t same[N];
        int base[N];
#pragma unroll
        for (int t = 0; t < N; ++t) {
            const int at = key[t] < 0 ? K1 : key[t];
            atomicOr((unsigned long long*)&word[at], 1ull << lane);
            same[t] = word[at];
            word[at] = 0;
        }
#pragma unroll
        for (int t = 0; t < N; ++t) {
            base[t] = 0;
            if (key[t] >= 0 && (same[t] & below) == 0) base[t] = atomicAdd(&cur[wave * K1 + key[t]], __popcll(same[t]));
        }
#pragma unroll
        for (int t = 0; t < N; ++t) base[t] = __shfl(base[t], __ffsll((unsigned long long)same[t]) - 1);
#pragma unroll
        for (int t = 0; t < N; ++t)
            if (key[t] >= 0) {
                g.pairs[off[key[t]] + base[t] + __popcll(same[t] & below)] = (int)(b + 64 * t + lane);
                if (g.kept) g.kept[b + 64 * t + lane] = key[t] < g.K;
            }
    };
    if (kept) {
#pragma unroll
        for (int t = 0; t < KEYS; t += 8)
            if (w0 + 64 * t < w1) place(std::integral_constant<int, 8>{}, w0 + 64 * t, keys + t);
    } else {
        for (int64_t b = w0; b < w1; b += 64 * 4) {
            int key[4];
            group_keys<4, 64>(g, b + lane, w1, key);
            place(std::integral_constant<int, 4>{}, b, key);
        }
    }
    if (blockIdx.x == 0)
        for (int e = tid; e < K1; e += THREADS) g.off[e] = off[e];
    if (blockIdx.x == 0 && tid < GR_HEIGHTS) g.count[tid] = first[tid * (K1 + 1) + K1];
    int64_t n[GR_HEIGHTS];  // tiles of this height and the ones before it
    for (int h = 0; h < GR_HEIGHTS; ++h) n[h] = (h ? n[h - 1] : 0) + first[h * (K1 + 1) + K1];
    const int64_t step = (int64_t)gridDim.x * GR_THREADS;
    for (int64_t v = blockIdx.x * (int64_t)GR_THREADS + tid; v < n[GR_HEIGHTS - 1]; v += step) {
        int h = 0, u = (int)v;
#pragma unroll
        for (int q = 1; q < GR_HEIGHTS; ++q)
            if (v >= n[q - 1]) {
                h = q;
                u = (int)(v - n[q - 1]);
            }
        const int* f = first + h * (K1 + 1);
        int a = 0, b = K1;  // the last network whose first tile is at most u
        while (b - a > 1) {
            const int m = (a + b) >> 1;
            if (f[m] <= u) a = m;
            else b = m;
        }
        g.tiles[h][u] = make_int2(a, off[a] + (u - f[a]) * group_height(h));
    }
}

__host__ inline size_t group_lds(int K) {
    return (size_t)GR_WAVES * (K + 2) * 8 + sizeof(int) * ((size_t)GR_WAVES * (K + 1) + (2 + GR_HEIGHTS) * (K + 2));
}

// ------------------------------------------------------------------------------------
// products

// pair / per_row by a product: exact for pairs below 2^30 (l = ceil(log2 d), m = ceil(2^(30 + l) / d))
struct Div {
    uint32_t m;
    int s;
    __device__ inline uint32_t of(int pair) const { return (uint32_t)(((uint64_t)(uint32_t)pair * m) >> s); }
};
__host__ inline Div div_by(int d) {
    int l = 0;
    while ((1ll << l) < d) ++l;
    return {(uint32_t)(((1ull << (30 + l)) + (uint64_t)d - 1) / (uint64_t)d), 30 + l};
}

enum { GR_FWD = 0, GR_DX = 1, GR_DW = 2 };

// m is the result's contiguous extent (outputs of a forward product, inputs of both gradients), n
// the other one (pairs; outputs of a weight gradient), k the contraction.
struct GroupGemm {
    const int32_t *off, *pairs;
    const int2* tiles;
    const int32_t* n_tiles;
    int K;
    int M, N, Kx;              // extents; N of the pairs' products is the number of pairs, dropped ones among them,
                               // and k of a weight gradient the group's pairs
    const void* p;             // rows of pairs: x (forward), dy (gradients); row (pair / pdiv)
    int64_t ldp;
    Div pdiv;
    const void* w;             // weights; x of a weight gradient, row (pair / wdiv)
    int64_t wnet, ldw;
    Div wdiv;
    const float* b;            // bias (nullable)
    int64_t bnet;
    int act;                   // activation (forward), or the one whose slope at a scales the result; -1 none
    const void* a;             // stored activations of the slope, row (pair)
    int64_t lda;
    void* y;                   // result; fp32 gradients of a weight gradient
    int64_t ldy, ynet;
    bool stream = false;       // the result's rows pass the caches by
    float* db;                 // (weight gradient) bias gradient, nullable
    int64_t dbnet;
    int splits;                // (weight gradient) parts of a group, summed by group_join_kernel
    float lr;                  // (weight gradient) != 0: y -= lr / pairs * sum instead of y = sum
    bf16_t* shadow;            // (with lr) bf16 copy of y, same strides
};

// The activations of act_fn; a NaN stays one (the rectifiers' comparison is z < 0).
__device__ inline float group_act(int act, float z) {
    switch (act) {
    case ACT_SIGMOID: return 1.0f / (1.0f + expf(-z));
    case ACT_TANH: return tanhf(z);
    case ACT_RELU: return z < 0.0f ? -0.0f : z + 0.0f;
    case ACT_LEAKY: return z < 0.0f ? 0.01f * z : z + 0.0f;
    default: return z;
    }
}

// Eight neighbouring values as loaded.  Rows may start at any multiple of the value's size: the
// global loads of gfx950 take any alignment, so odd widths and strides cost lines, not instructions.
typedef uint32_t u4v __attribute__((ext_vector_type(4)));
typedef u4v u4v_a2 __attribute__((aligned(2)));
typedef f4 f4_a4 __attribute__((aligned(4)));
template <typename T> struct Raw8;
template <> struct Raw8<bf16_t> { u4v v; };
template <> struct Raw8<float> { f4 v[2]; };

// the first nv of eight values at p (the others 0); nv <= 0 reads nothing
__device__ inline void load8(Raw8<bf16_t>& r, const bf16_t* p, int nv) {
    if (nv >= 8) {
        r.v = *(const u4v_a2*)p;
    } else {
        uint32_t q[4] = {0, 0, 0, 0};
#pragma unroll
        for (int j = 0; j < 7; ++j)
            if (j < nv) q[j >> 1] |= (uint32_t)p[j] << (16 * (j & 1));
        r.v = u4v{q[0], q[1], q[2], q[3]};
    }
}
__device__ inline void load8(Raw8<float>& r, const float* p, int nv) {
    if (nv >= 8) {
        r.v[0] = *(const f4_a4*)p;
        r.v[1] = *(const f4_a4*)(p + 4);
    } else {
        r.v[0] = r.v[1] = f4{0, 0, 0, 0};
#pragma unroll
        for (int j = 0; j < 7; ++j)
            if (j < nv) r.v[j >> 2][j & 3] = p[j];
    }
}

template <typename T>
__device__ inline void raw8_f(float (&v)[8], const Raw8<T>& r) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        if constexpr (sizeof(T) == 4) v[i] = r.v[i >> 2][i & 3];
        else v[i] = i & 1 ? bf_hi(r.v[i >> 1]) : bf_lo(r.v[i >> 1]);
    }
}
template <typename T>
__device__ inline void load8_f(float (&v)[8], const T* p, int nv) {
    Raw8<T> r;
    load8(r, p, nv);
    raw8_f(v, r);
}

// the first nv of eight values; streamed past the caches where a result is too large to be found there again
template <bool STREAM = false>
__device__ inline void store8(float* p, const float (&v)[8], int nv) {
    if (nv >= 8) {
        const f4 lo = {v[0], v[1], v[2], v[3]}, hi = {v[4], v[5], v[6], v[7]};
        if (STREAM) {
            __builtin_nontemporal_store(lo, (f4_a4*)p);
            __builtin_nontemporal_store(hi, (f4_a4*)(p + 4));
        } else {
            *(f4_a4*)p = lo;
            *(f4_a4*)(p + 4) = hi;
        }
    } else {
#pragma unroll
        for (int i = 0; i < 7; ++i)
            if (i < nv) p[i] = v[i];
    }
}
template <bool STREAM = false>
__device__ inline void store8(bf16_t* p, const float (&v)[8], int nv) {
    if (nv >= 8) {
        const u4v q = {cvt_pk_bf16(v[0], v[1]), cvt_pk_bf16(v[2], v[3]), cvt_pk_bf16(v[4], v[5]), cvt_pk_bf16(v[6], v[7])};
        if (STREAM) __builtin_nontemporal_store(q, (u4v_a2*)p);
        else *(u4v_a2*)p = q;
    } else {
#pragma unroll
        for (int i = 0; i < 7; ++i)
            if (i < nv) p[i] = f2bf(v[i]);
    }
}

// workgroup number -> place in an order in which each XCD (its numbers are those equal mod 8) gets
// one contiguous stretch, so that neighbours in it share an L2
__device__ inline uint32_t group_xcd(uint32_t id, uint32_t total) {
    const uint32_t q = total >> 3, r = total & 7, x = id & 7;
    return x * q + (x < r ? x : r) + (id >> 3);
}

// A workgroup's tile: network, place in the result, its columns there, k from position p0 (weight gradient)
struct GroupPlace { int e, m0, n0, nv, split, p0, Kx; };

// Workgroups of a weight gradient: of every network's tiles each XCD takes one stretch, another one for the
// next network, so that unequal groups weigh on all XCDs alike.
__host__ __device__ inline int64_t group_dw_blocks(int64_t tiles, int64_t groups) {
    return tiles < 8 ? tiles * groups : 8 * ((tiles + 7) / 8) * groups;
}

template <int DIR, int BM, int BN, int STEP>
__device__ inline bool group_place_of(const GroupGemm& g, int mt, GroupPlace& o) {
    o.n0 = o.split = 0;
    if (DIR == GR_DW) {
        const int tiles = mt * ((g.N + BN - 1) / BN);
        const int id = (int)blockIdx.x;
        int t, grp;
        if (tiles < 8) {
            t = id % tiles;
            grp = id / tiles;
        } else {
            const int share = (tiles + 7) / 8, local = id >> 3;
            grp = local / share;
            t = ((id + grp) & 7) * share + local % share;
            if (t >= tiles) return false;
        }
        o.e = grp % g.K;
        o.split = grp / g.K;
        // a stretch of the order is about square (bands of four tiles along m), so an XCD's L2 holds what it shares:
        // row by row each XCD read all of x (32,768 pairs 2048 x 2048, 16 networks: 1,447 -> 1,060 MB of
        // memory traffic)
        const int nt = tiles / mt, band = t / (4 * nt), in = t - band * 4 * nt, wide = mt - band * 4 < 4 ? mt - band * 4 : 4;
        o.m0 = (band * 4 + in % wide) * BM;
        o.n0 = in / wide * BN;
        o.nv = g.N - o.n0 < BN ? g.N - o.n0 : BN;
        const int first = g.off[o.e], all = g.off[o.e + 1] - first;
        const int part = (all + g.splits * STEP - 1) / (g.splits * STEP) * STEP;
        o.p0 = first + (o.split * part < all ? o.split * part : all);
        o.Kx = first + all - o.p0 < part ? first + all - o.p0 : part;
        return true;
    }
    // WIDE tiles of pairs next to each other, then along m: the workgroups that an XCD runs at a time (32 of 256
    // x 256, 64 and more of smaller ones) are about as many tiles wide as high and share their operands in L2
    // (65,536 pairs 4096 -> 4096, 16 networks, bf16: 2,183 us with eight tiles of 256, 2,025 us with four)
    constexpr int WIDE = 4;
    // (a launch has fewer than 2^24 workgroups: 32 bits do, and 64-bit divisions are long)
    const uint32_t n_tiles = *g.n_tiles;
    if (blockIdx.x >= (uint64_t)n_tiles * mt) return false;
    const uint32_t id = group_xcd(blockIdx.x, n_tiles * mt);
    const uint32_t grp = id / (WIDE * mt), in = id - grp * WIDE * mt;
    const uint32_t left = n_tiles - grp * WIDE, wide = left < WIDE ? left : WIDE, row = wide == WIDE ? in / WIDE : in / wide;
    const int2 t = g.tiles[grp * WIDE + in - row * wide];
    o.m0 = (int)row * BM;
    o.e = t.x;
    o.p0 = t.y;
    const int end = o.e < g.K ? g.off[o.e + 1] : g.N;
    o.nv = end - o.p0 < BN ? end - o.p0 : BN;
    o.Kx = o.e < g.K ? g.Kx : 0;  // (dropped pairs: nothing to sum)
    return true;
}

typedef short s4v __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s4v lds_s4v;

// An operand tile in LDS, W wide and BK deep, in bf16 (fp32 operands as three such planes).
//  KC (memory runs along k): rows of BK values in 16-byte chunks; a row's chunks are permuted by
//     XOR so that eight neighbouring rows' reads of one chunk fall on different banks.
//  NC (memory runs across k): rows of W values, one per k, in 32-byte blocks, permuted by XOR so
//     that the rows which one transposing read touches fall on different banks.
template <bool KC, int BK, int W>
struct GTile {
    static constexpr int ELEMS = W * BK, CPR = KC ? BK / 8 : W / 8, BLOCKS = W / 16;
    static __device__ inline int row(int s) { return s / CPR; }
    static __device__ inline int chunk(int s) { return s % CPR; }
    static __device__ inline int key(int r) {
        if (KC) return CPR == 8 ? r & 7 : (r >> 1) & 3;
        return ((r & 3) | ((r >> 1) & 4)) & (BLOCKS - 1);
    }
    static __device__ inline int offset(int r, int c) {
        if (KC) return r * BK + (c ^ key(r)) * 8;
        return r * W + (((c >> 1) ^ key(r)) << 4) + (c & 1) * 8;
    }
    // operand fragment of the 16 x 16 x 32 instruction: index t0 + (lane & 15), k kb + 8 (lane >> 4) ..
    static __device__ inline bf8v frag(const bf16_t* lds, int t0, int kb, int lane) {
        const int l15 = lane & 15, kg = lane >> 4;
        if (KC) return *(const bf8v*)(lds + offset(t0 + l15, kb / 8 + kg));
        const int r = kb + 8 * kg + (l15 >> 2);
        const bf16_t* q = lds + r * W + (((t0 >> 4) ^ key(r)) << 4) + (l15 & 3) * 4;
        const s4v lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4v*)q);
        const s4v hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4v*)(q + 4 * W));
        const s4v both[2] = {lo, hi};
        return __builtin_bit_cast(bf8v, both);
    }
};

__device__ inline void gt_store(bf16_t* lds, int plane, const Raw8<bf16_t>& r) { *(u4v*)lds = r.v; }
__device__ inline void gt_store(bf16_t* lds, int plane, const Raw8<float>& r) {
    uint32_t h[4], m[4], l[4];
#pragma unroll
    for (int d = 0; d < 4; ++d) split3_pk(r.v[d >> 1][2 * (d & 1)], r.v[d >> 1][2 * (d & 1) + 1], h[d], m[d], l[d]);
    *(u4v*)lds = u4v{h[0], h[1], h[2], h[3]};
    *(u4v*)(lds + plane) = u4v{m[0], m[1], m[2], m[3]};
    *(u4v*)(lds + 2 * plane) = u4v{l[0], l[1], l[2], l[3]};
}

// activations / slopes of eight neighbouring values (the choice outside the loops: one copy of each)
__device__ inline void group_rectify8(int act, float (&v)[8]) {
    if (act != ACT_RELU && act != ACT_LEAKY) return;
    const float low = act == ACT_RELU ? 0.0f : 0.01f;
#pragma unroll
    for (int r = 0; r < 8; ++r) v[r] = v[r] < 0.0f ? (act == ACT_RELU ? -0.0f : low * v[r]) : v[r] + 0.0f;
}
__device__ inline void group_act8(int act, float (&v)[8]) {
    if (act == ACT_SIGMOID) {
#pragma unroll
        for (int r = 0; r < 8; ++r) v[r] = group_act(ACT_SIGMOID, v[r]);
    } else {
#pragma unroll
        for (int r = 0; r < 8; ++r) v[r] = group_act(ACT_TANH, v[r]);
    }
}
__device__ inline void group_slope8(int act, float (&v)[8], const float (&a)[8]) {
    if (act == ACT_SIGMOID || act == ACT_TANH) {
#pragma unroll
        for (int r = 0; r < 8; ++r) v[r] *= act == ACT_TANH ? 1.0f - a[r] * a[r] : a[r] * (1.0f - a[r]);
    } else if (act == ACT_RELU || act == ACT_LEAKY) {
        const float low = act == ACT_RELU ? 0.0f : 0.01f;
#pragma unroll
        for (int r = 0; r < 8; ++r) v[r] *= signbit(a[r]) ? low : 1.0f;
    }
}

// The results of a wave: a lane holds m0 + wm + 16 i + 4 kg + r of column n = wn + 16 j + l15.  Sixteen
// columns at a time go through the wave's own part of LDS (`turn`, no longer used by anyone), from where
// a lane takes eight neighbouring results of one column: rows leave in stores of 16 or 32 bytes a lane.
template <int MI> constexpr int group_turn() { return 16 * (16 * MI + 4); }  // floats of a wave
template <int DIR, typename T, typename TO, int MI, int NJ>
__device__ inline void group_store(const GroupGemm& g, const f4 (&acc)[MI][NJ], const f4 (&accb)[NJ], int e, int split, int p0, int m0,
                                   int n0, int nv, int wm, int wn, int lane, bool bias_rows, float* turn) {
    constexpr int LD = 16 * MI + 4, PER = 2 * MI, COLS = MI == 1 ? 16 : 64 / PER;  // lanes of a column, columns at a time
    const int l15 = lane & 15, kg = lane >> 4, part = lane % PER * 8, m = m0 + wm + part;
    const int left = lane < PER * COLS ? g.M - m : 0;
    const int pairs = DIR == GR_DW ? g.off[e + 1] - g.off[e] : 0;
    const float scale = DIR == GR_DW && g.lr != 0.0f && pairs > 0 ? g.lr / (float)pairs : 0.0f;
    if (DIR == GR_DW && g.lr != 0.0f && pairs == 0) return;  // no update
    // (the pair of column `lane` of the wave: asked of its lane in the loop, not of memory)
    constexpr int OWN = (16 * NJ + 63) / 64;
    int own[OWN];
#pragma unroll
    for (int h = 0; h < OWN; ++h) own[h] = DIR != GR_DW && wn + 64 * h + lane < nv ? g.pairs[p0 + wn + 64 * h + lane] : 0;
    float bias[8];
    if (DIR == GR_FWD) {
#pragma unroll
        for (int r = 0; r < 8; ++r) bias[r] = g.b && r < left && e < g.K ? g.b[e * g.bnet + m + r] : 0.0f;
    }
    // what a result is combined with (slopes' activations, weights to update) is loaded sixteen columns ahead:
    // behind a store it would wait for it
    typedef typename std::conditional<DIR == GR_DW, float, T>::type E;
    constexpr int TURNS = 16 / COLS;
    Raw8<E> with[2][TURNS];
    const bool has_with = DIR == GR_DX ? g.a && e < g.K : DIR == GR_DW && g.lr != 0.0f;
    auto column = [&](int j, int c) { return wn + 16 * j + c * COLS + lane / PER; };
    auto pair_of = [&](int j, int c) -> int64_t { return __shfl(own[j / 4], 16 * (j & 3) + c * COLS + lane / PER); };
    auto fetch = [&](int j) {
#pragma unroll
        for (int c = 0; c < TURNS; ++c) {
            const int64_t pair = DIR == GR_DX ? pair_of(j, c) : 0;
            const int n = column(j, c), nr = n < nv ? left : 0;
            if constexpr (DIR == GR_DX) load8(with[j & 1][c], (const T*)g.a + pair * g.lda + m, nr);
            if constexpr (DIR == GR_DW) load8(with[j & 1][c], (const float*)g.y + e * g.ynet + (int64_t)(n0 + n) * g.ldy + m, nr);
        }
    };
    if (has_with) fetch(0);
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
        if (has_with && j + 1 < NJ) fetch(j + 1);
#pragma unroll
        for (int i = 0; i < MI; ++i) *(f4*)(turn + l15 * LD + 16 * i + 4 * kg) = acc[i][j];
        __builtin_amdgcn_wave_barrier();
        auto leave = [&](int c, bool smooth) {
            const int col = c * COLS + lane / PER, n = column(j, c);
            const int64_t pair = DIR != GR_DW ? pair_of(j, c) : 0;
            if (n >= nv || left <= 0) return;
            const f4 lo = *(const f4*)(turn + col * LD + part), hi = *(const f4*)(turn + col * LD + part + 4);
            float v[8] = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
            float w[8];
            if (DIR != GR_FWD && has_with) raw8_f(w, with[j & 1][c]);
            if (DIR == GR_DW) {
                const int64_t at = (int64_t)(n0 + n) * g.ldy + m;
                if (g.lr != 0.0f) {
#pragma unroll
                    for (int r = 0; r < 8; ++r) v[r] = w[r] - scale * v[r];
                    if (g.shadow) store8(g.shadow + e * g.ynet + at, v, left);
                }
                store8((float*)g.y + ((int64_t)split * g.K + e) * g.ynet + at, v, left);
                return;
            }
            if (e == g.K) {  // dropped
#pragma unroll
                for (int r = 0; r < 8; ++r) v[r] = 0.0f;
            } else if (DIR == GR_FWD) {
#pragma unroll
                for (int r = 0; r < 8; ++r) v[r] += bias[r];
                if (smooth) group_act8(g.act, v);
                else group_rectify8(g.act, v);
            } else if (has_with) {
                group_slope8(g.act, v, w);
            }
            TO* y = (TO*)g.y + pair * g.ldy + m;
            if (g.stream) store8<true>(y, v, left);
            else store8(y, v, left);
        };
        if (DIR == GR_FWD && (g.act == ACT_SIGMOID || g.act == ACT_TANH)) {  // (one copy of their code)
#pragma unroll 1
            for (int c = 0; c < TURNS; ++c) leave(c, true);
        } else {
#pragma unroll
            for (int c = 0; c < TURNS; ++c) leave(c, false);
        }
        __builtin_amdgcn_wave_barrier();
        if (bias_rows && kg == 0 && wn + 16 * j + l15 < nv) {
            float* db = g.db + ((int64_t)split * g.K + e) * g.dbnet + n0 + wn + 16 * j + l15;
            *db = g.lr != 0.0f ? *db - scale * accb[j][0] : accb[j][0];
        }
    }
}

// Rows at any alignment, and fp32: S x S tiles (128, or 64 where those are too few) of one network's product.
// Bound by the matrix units for full tiles: 32,768 rows 784 -> 1024 over 64 networks in fp32 take 267 us, 197
// TFLOP/s or 1,180 of the six bf16 products.  Over pairs, four waves of 32 x 128: all waves share the tile's
// columns, so a tile that a group does not fill costs its share of the products only (the same over 256 networks
// of unequal groups 467 -> 401 us); a weight gradient's tiles are full, and 64 x 64 a wave reads less of LDS
// (32,768 rows, 64 networks, 2048 x 1024: 909 -> 867 us).
template <int DIR, typename T, typename TO, int S>
__global__ __launch_bounds__(256, 2) void group_tile_kernel(GroupGemm g) {
    constexpr bool F32 = sizeof(T) == 4;
    constexpr int BK = F32 ? 32 : 64, PL = F32 ? 3 : 1;
    typedef GTile<DIR == GR_FWD, BK, S> TA;
    typedef GTile<DIR != GR_DW, BK, S> TB;
    constexpr int U = TA::ELEMS / 8 / 256;
    __shared__ __align__(16) bf16_t lds[2 * PL * TA::ELEMS];
    bf16_t *la = lds, *lb = lds + PL * TA::ELEMS;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int mt = (g.M + S - 1) / S;
    GroupPlace at;
    if (!group_place_of<DIR, S, S, BK>(g, mt, at)) return;
    const int e = at.e, m0 = at.m0, n0 = at.n0, nv = at.nv, split = at.split, p0 = at.p0, Kx = at.Kx;
    const int mv = g.M - m0 < S ? g.M - m0 : S;
    constexpr int WN = DIR == GR_DW ? 2 : 1;  // waves across n
    constexpr int MI = S / 64 * WN, NJ = S / 16 / WN;
    f4 acc[MI][NJ], accb[NJ];
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
        accb[j] = f4{0, 0, 0, 0};
#pragma unroll
        for (int i = 0; i < MI; ++i) acc[i][j] = f4{0, 0, 0, 0};
    }
    const int wm = wave / WN * 16 * MI, wn = wave % WN * 16 * NJ;
    const bool bias_rows = DIR == GR_DW && g.db && m0 == 0 && wm == 0;

    // this thread's chunks of a tile
    const T *pa[U], *pb[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int s = u * 256 + tid;
        if (DIR == GR_FWD) {
            const int r = TA::row(s);
            pa[u] = r < mv ? (const T*)g.w + e * g.wnet + (int64_t)(m0 + r) * g.ldw + TA::chunk(s) * 8 : nullptr;
        }
        if (DIR != GR_DW) {
            const int r = TB::row(s);
            pb[u] = r < nv && Kx > 0 ? (const T*)g.p + (int64_t)(g.pdiv.of(g.pairs[p0 + r])) * g.ldp + TB::chunk(s) * 8 : nullptr;
        }
    }
    Raw8<T> ra[U], rb[U];  // the next step's operands, in flight
    int number[U];  // (weight gradient) the pairs of the step that is loaded next
    auto numbers = [&](int k0) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int k = k0 + TA::row(u * 256 + tid);
            number[u] = g.pairs[p0 + (k < Kx ? k : Kx - 1)];
        }
    };
    auto load = [&](int k0) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int s = u * 256 + tid;
            if (DIR == GR_FWD) {
                load8(ra[u], pa[u] + k0, pa[u] ? Kx - k0 - TA::chunk(s) * 8 : 0);
            } else if (DIR == GR_DX) {
                const int r = TA::row(s), c = TA::chunk(s) * 8;
                load8(ra[u], (const T*)g.w + e * g.wnet + (int64_t)(k0 + r) * g.ldw + m0 + c, k0 + r < Kx ? mv - c : 0);
            }
            if (DIR != GR_DW) {
                load8(rb[u], pb[u] + k0, pb[u] ? Kx - k0 - TB::chunk(s) * 8 : 0);
            } else {
                const int r = TA::row(s), c = TA::chunk(s) * 8;
                load8(ra[u], (const T*)g.w + (int64_t)g.wdiv.of(number[u]) * g.ldw + m0 + c, k0 + r < Kx ? mv - c : 0);
                load8(rb[u], (const T*)g.p + (int64_t)number[u] * g.ldp + n0 + c, k0 + r < Kx ? nv - c : 0);
            }
        }
        if (DIR == GR_DW) numbers(k0 + BK);
    };
    if (DIR == GR_DW && Kx > 0) numbers(0);
    if (Kx > 0) load(0);
    for (int k0 = 0; k0 < Kx; k0 += BK) {
        lds_barrier();  // (waits for no load)
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int s = u * 256 + tid;
            gt_store(la + TA::offset(TA::row(s), TA::chunk(s)), TA::ELEMS, ra[u]);
            gt_store(lb + TB::offset(TB::row(s), TB::chunk(s)), TB::ELEMS, rb[u]);
        }
        lds_barrier();
        if (k0 + BK < Kx) load(k0 + BK);
#pragma unroll
        for (int kb = 0; kb < BK; kb += 32) {
            bf8v fa[PL][MI];
#pragma unroll
            for (int q = 0; q < PL; ++q)
#pragma unroll
                for (int i = 0; i < MI; ++i) fa[q][i] = TA::frag(la + q * TA::ELEMS, wm + 16 * i, kb, lane);
#pragma unroll
            for (int j = 0; j < NJ; ++j) {
                if (wn + 16 * j >= nv) break;  // (the same for all lanes)
                bf8v fb[PL];
#pragma unroll
                for (int q = 0; q < PL; ++q) fb[q] = TB::frag(lb + q * TB::ELEMS, wn + 16 * j, kb, lane);
                // fp32: the six products of parts above 2^-24 of the whole, the smallest first
                constexpr int PA[6] = {1, 2, 0, 1, 0, 0}, PB[6] = {1, 0, 2, 0, 1, 0};
#pragma unroll
                for (int p = F32 ? 0 : 5; p < 6; ++p)
#pragma unroll
                    for (int i = 0; i < MI; ++i)
                        acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fa[PA[p]][i], fb[PB[p]], acc[i][j], 0, 0, 0);
                if (bias_rows) {  // sums over k: a product with ones
                    const u4v ones = {0x3f803f80, 0x3f803f80, 0x3f803f80, 0x3f803f80};
#pragma unroll
                    for (int q = PL - 1; q >= 0; --q)
                        accb[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf8v, ones), fb[q], accb[j], 0, 0, 0);
                }
            }
        }
    }
    __syncthreads();
    group_store<DIR, T, TO, MI, NJ>(g, acc, accb, e, split, p0, m0, n0, nv, wm, wn, lane, bias_rows,
                                    (float*)lds + wave * group_turn<MI>());
}

// ------------------------------------------------------------------------------------
// bf16 products whose rows start at multiples of 16 bytes: tiles of BM x BN, WM x WN waves, a ring of stages of
// 32 k in LDS that global memory fills directly.  A long contraction (65,536 pairs 4096 -> 4096, 16 networks) takes
// 2,025 to 2,060 us, 1,067 to 1,086 TFLOP/s of the 1,327 that a large library product reaches on the card: the matrix
// cores are busy in 0.50 to 0.54 of the cycles, at a clock of 2.1 to 1.9 GHz under this load (0.60 at 1.4 GHz in the
// first passes after an idle spell).  At a contraction of 1024 they are busy in 0.48 (16 even networks, one a row: 524 to
// 560 us) and in 0.35 (32,768 rows to two each of 32 networks: 660): the results' stores, which a round of workgroups
// makes at one time, add a quarter (without them 551 us of 671).

static __device__ __align__(64) uint32_t group_zeros[16];  // what lies outside an operand

// BYTES a lane from global memory to lds + BYTES lane.  In asm: the compiler, which cannot tell the ring's
// stages apart, waits for all copies in flight before a transposing read of LDS.  No register is written
// but m0, which nothing else in these kernels uses (and the compiler never allocates).
template <int BYTES>
__device__ inline void copy_to_lds(const void* src, uint32_t lds) {
    if (BYTES == 16)
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(__builtin_amdgcn_readfirstlane(lds)), "v"(src) : "memory");
    else
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off" ::"s"(__builtin_amdgcn_readfirstlane(lds)), "v"(src) : "memory");
}
// waits until at most N of the wave's copies are in flight, and for all other waves to have done so
template <int N>
__device__ inline void ring_wait() {
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
}

// An operand's stage: T values wide, 32 k deep; KC and NC as in GTile.
template <bool KC, int T>
struct RTile {
    static constexpr int ELEMS = T * 32, CHUNKS = ELEMS / 8;
    static __device__ inline int row(int s) { return KC ? s >> 2 : s / (T / 8); }  // (NC: the k)
    static __device__ inline int key(int r) { return KC ? (r >> 1) & 3 : ((r & 3) | ((r >> 1) & 4)) & (T / 16 - 1); }
    // the chunk of the row that belongs at place s
    static __device__ inline int chunk(int s) {
        const int r = row(s), c = KC ? s & 3 : s % (T / 8);
        return KC ? c ^ key(r) : ((c >> 1) ^ key(r)) << 1 | (c & 1);
    }
    static __device__ inline bf8v frag(const bf16_t* lds, int t0, int lane) {
        const int l15 = lane & 15, kg = lane >> 4;
        if (KC) {
            const int r = t0 + l15;
            return *(const bf8v*)(lds + r * 32 + ((kg ^ key(r)) << 3));
        }
        const int r = 8 * kg + (l15 >> 2);
        const bf16_t* q = lds + r * T + (((t0 >> 4) ^ key(r)) << 4) + (l15 & 3) * 4;
        const s4v both[2] = {__builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4v*)q),
                             __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4v*)(q + 4 * T))};
        return __builtin_bit_cast(bf8v, both);
    }
};

// AHEAD: a stage is waited for one step before it is multiplied, so that a step's first operands are read
// during the step before it.
template <int DIR, typename TO, int BM, int BN, int WM, int WN, int NST, bool AHEAD>
__global__ __launch_bounds__(64 * WM * WN, 2) void group_ring_kernel(GroupGemm g) {
    typedef RTile<DIR == GR_FWD, BM> TA;
    typedef RTile<DIR != GR_DW, BN> TB;
    constexpr int THREADS = 64 * WM * WN;
    constexpr int UA = TA::CHUNKS / THREADS, UB = TB::CHUNKS / THREADS, STAGE = TA::ELEMS + TB::ELEMS;
    constexpr int MI = BM / WM / 16, NJ = BN / WN / 16;  // 16 x 16 blocks of a wave
    extern __shared__ __align__(16) bf16_t ring[];
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int mt = (g.M + BM - 1) / BM;
    GroupPlace place;
    if (!group_place_of<DIR, BM, BN, 32>(g, mt, place)) return;
    const int e = place.e, m0 = place.m0, n0 = place.n0, nv = place.nv, split = place.split, p0 = place.p0, Kx = place.Kx;
    const int mv = g.M - m0 < BM ? g.M - m0 : BM;
    const bf16_t* zeros = (const bf16_t*)group_zeros;
    f4 acc[MI][NJ], accb[NJ];
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
        accb[j] = f4{0, 0, 0, 0};
#pragma unroll
        for (int i = 0; i < MI; ++i) acc[i][j] = f4{0, 0, 0, 0};
    }
    const int wm = wave % WM * (BM / WM), wn = wave / WM * (BN / WN);
    const bool bias_rows = DIR == GR_DW && g.db && m0 == 0 && wm == 0;

    // Addresses of this thread's chunks (of the weight gradient's rows: what does not depend on k).  Rows and
    // columns outside the tile repeat the last one inside: they reach only results that are not stored.
    const bf16_t *pa[UA], *pb[UB];
    int ka[UA], kb[UB];  // KC: k of the chunk in its stage; NC: the row's k
#pragma unroll
    for (int u = 0; u < UA; ++u) {
        const int s = u * THREADS + tid, r = TA::row(s), c = TA::chunk(s) * 8;
        ka[u] = DIR == GR_FWD ? c : r;
        const int rm = r < mv ? r : mv - 1, cm = c < mv ? c : mv - 8;
        pa[u] = (const bf16_t*)g.w + (DIR == GR_DW ? 0 : e * g.wnet) +
                (DIR == GR_FWD ? (int64_t)(m0 + rm) * g.ldw + c : DIR == GR_DX ? (int64_t)r * g.ldw + m0 + cm : (int64_t)(m0 + cm));
    }
#pragma unroll
    for (int u = 0; u < UB; ++u) {
        const int s = u * THREADS + tid, r = TB::row(s), c = TB::chunk(s) * 8;
        kb[u] = DIR != GR_DW ? c : r;
        pb[u] = (const bf16_t*)g.p;
        if (DIR == GR_DW) pb[u] += n0 + (c < nv ? c : nv - 8);
        else if (Kx > 0) pb[u] += (int64_t)g.pdiv.of(g.pairs[p0 + (r < nv ? r : nv - 1)]) * g.ldp + c;
    }
    const uint32_t base = __builtin_amdgcn_readfirstlane((uint32_t)(size_t)(lds_void*)ring);
    constexpr int IST = 2 * (NST - 1);  // stages of a wave's own ring of pair numbers (weight gradient)
    const int* numbers = (const int*)(ring + NST * STAGE) + wave * IST * 64;
    const uint32_t numbers_at = base + NST * STAGE * 2 + wave * IST * 256;
    // copies the numbers of the pairs k0 .. k0 + 31 (and more, not used)
    auto number = [&](int stage, int k0) {
        const int k = k0 + lane < Kx ? k0 + lane : Kx - 1;
        copy_to_lds<4>(g.pairs + p0 + k, numbers_at + stage * 256);
    };
    const int64_t step_a = DIR == GR_FWD ? 32 : 32 * g.ldw;
    // fills a stage with k0 .. k0 + 31 (zeros behind the last k); stages are filled in their order
    auto fill_as = [&](auto whole, int stage, int k0, int istage) {
        const uint32_t to = base + stage * (STAGE * 2) + wave * 1024;
        int na[UA], nb[UB];
        if (DIR == GR_DW) {  // (the numbers of pairs behind the last are the last one's)
#pragma unroll
            for (int u = 0; u < UA; ++u) na[u] = numbers[istage * 64 + ka[u]];
#pragma unroll
            for (int u = 0; u < UB; ++u) nb[u] = numbers[istage * 64 + kb[u]];
        }
#pragma unroll
        for (int u = 0; u < UA; ++u) {
            const bf16_t* q = pa[u];
            if (DIR == GR_DW) q += (uint64_t)g.wdiv.of(na[u]) * (uint32_t)g.ldw;
            else pa[u] += step_a;
            if (!whole && k0 + ka[u] >= Kx) q = zeros;
            copy_to_lds<16>(q, to + u * THREADS * 16);
        }
#pragma unroll
        for (int u = 0; u < UB; ++u) {
            const bf16_t* q = pb[u];
            if (DIR == GR_DW) q += (uint64_t)(uint32_t)nb[u] * (uint32_t)g.ldp;
            else pb[u] += 32;
            if (!whole && k0 + kb[u] >= Kx) q = zeros;
            copy_to_lds<16>(q, to + TA::ELEMS * 2 + u * THREADS * 16);
        }
    };
    auto fill = [&](int stage, int k0, int istage) {
        if (k0 + 32 <= Kx) fill_as(std::true_type{}, stage, k0, istage);
        else fill_as(std::false_type{}, stage, k0, istage);
    };
    constexpr int COPIES = UA + UB + (DIR == GR_DW ? 1 : 0);  // of a wave and stage
    const int steps = (Kx + 31) / 32;
    int at = 0, nat = NST - 1;  // the stage that is read, that of the numbers of the stage that is filled
    if (Kx > 0) {
        if (DIR == GR_DW) {
#pragma unroll
            for (int t = 0; t < IST; ++t) number(t, t * 32);
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        }
#pragma unroll
        for (int t = 0; t < NST - 1; ++t) fill(t, t * 32, t);  // (what lies behind the last k is filled with zeros)
        if (DIR == GR_DW) {  // (as many copies in flight as in the loop)
#pragma unroll
            for (int t = 0; t < NST - 1; ++t) number(t, (IST + t) * 32);
        }
    }
    constexpr int RA = DIR == GR_FWD ? 1 : 2, RB = DIR == GR_DW ? 2 : 1;  // reads of an operand
    auto load_b = [&](bf8v (&fb)[NJ], int stage) {
#pragma unroll
        for (int j = 0; j < NJ; ++j) fb[j] = TB::frag(ring + stage * STAGE + TA::ELEMS, wn + 16 * j, lane);
    };
    auto load_a = [&](int stage, int i) { return TA::frag(ring + stage * STAGE, wm + 16 * i, lane); };
    auto refill = [&](int t) {
        fill(at == 0 ? NST - 1 : at - 1, (t + NST - 1) * 32, nat);
        if (DIR == GR_DW) {
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // (the numbers are read: their place is free)
            number(nat, (t + NST - 1 + IST) * 32);
            nat = nat == IST - 1 ? 0 : nat + 1;
        }
    };
    auto add_bias = [&](const bf8v (&fb)[NJ]) {  // sums over k: a product with ones
        if (!bias_rows) return;
        const u4v ones = {0x3f803f80, 0x3f803f80, 0x3f803f80, 0x3f803f80};
#pragma unroll
        for (int j = 0; j < NJ; ++j)
            accb[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf8v, ones), fb[j], accb[j], 0, 0, 0);
    };
    if constexpr (AHEAD) {
        // the operands of step t from registers (fb, fa: its first two blocks) and LDS, the next step's into fbn, fan
        auto step = [&](int t, const bf8v (&fb)[NJ], const bf8v (&fa)[2], bf8v (&fbn)[NJ], bf8v (&fan)[2]) {
            ring_wait<(NST - 3) * COPIES>();
            if (DIR != GR_DW) refill(t);
            const int next = at == NST - 1 ? 0 : at + 1;
            bf8v f[MI];
            f[0] = fa[0];
            f[1] = fa[1];
#pragma unroll
            for (int i = 2; i < MI; ++i) f[i] = load_a(at, i);
            load_b(fbn, next);
            fan[0] = load_a(next, 0);
            fan[1] = load_a(next, 1);
#pragma unroll
            for (int i = 0; i < MI; ++i)
#pragma unroll
                for (int j = 0; j < NJ; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f[i], fb[j], acc[i][j], 0, 0, 0);
            if (DIR == GR_DW) refill(t);  // (behind the operands' reads, which then do not wait for the
            // numbers': 131,072 pairs 2048 x 2048 1,132 -> 1,103 us)
            // reads two operands ahead of the products that take them, the next step's with the last ones
            __builtin_amdgcn_sched_group_barrier(0x100, 2 * RA, 0);
#pragma unroll
            for (int i = 0; i < MI - 4; ++i) {
                __builtin_amdgcn_sched_group_barrier(0x008, NJ, 0);
                __builtin_amdgcn_sched_group_barrier(0x100, RA, 0);
            }
#pragma unroll
            for (int i = 0; i < 3; ++i) {
                __builtin_amdgcn_sched_group_barrier(0x008, NJ, 0);
                __builtin_amdgcn_sched_group_barrier(0x100, (RB * NJ + 2 * RA + 2) / 3, 0);
            }
            __builtin_amdgcn_sched_group_barrier(0x008, NJ, 0);
            add_bias(fb);
            at = next;
        };
        bf8v fb[2][NJ], fa[2][2];
        if (steps > 0) {
            ring_wait<(NST - 2) * COPIES>();
            load_b(fb[0], 0);
            fa[0][0] = load_a(0, 0);
            fa[0][1] = load_a(0, 1);
        }
        int t = 0;
        for (; t + 1 < steps; t += 2) {
            step(t, fb[0], fa[0], fb[1], fa[1]);
            step(t + 1, fb[1], fa[1], fb[0], fa[0]);
        }
        if (t < steps) step(t, fb[0], fa[0], fb[1], fa[1]);
    } else {
        for (int t = 0; t < steps; ++t) {
            ring_wait<(NST - 2) * COPIES>();
            refill(t);
            bf8v fa[MI], fb[NJ];
            load_b(fb, at);
#pragma unroll
            for (int i = 0; i < MI; ++i) fa[i] = load_a(at, i);
#pragma unroll
            for (int i = 0; i < MI; ++i)
#pragma unroll
                for (int j = 0; j < NJ; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fa[i], fb[j], acc[i][j], 0, 0, 0);
            // reads two operands ahead of the products that take them
            __builtin_amdgcn_sched_group_barrier(0x100, RB * NJ + 2 * RA, 0);
#pragma unroll
            for (int i = 0; i < MI - 2; ++i) {
                __builtin_amdgcn_sched_group_barrier(0x008, NJ, 0);
                __builtin_amdgcn_sched_group_barrier(0x100, RA, 0);
            }
            __builtin_amdgcn_sched_group_barrier(0x008, 2 * NJ, 0);
            add_bias(fb);
            at = at == NST - 1 ? 0 : at + 1;
        }
    }
    ring_wait<0>();  // (no copy outlives its workgroup)
    group_store<DIR, bf16_t, TO, MI, NJ>(g, acc, accb, e, split, p0, m0, n0, nv, wm, wn, lane, bias_rows,
                                         (float*)ring + wave * group_turn<MI>());
}

// Rows of `values` for workgroups of 256 threads: the power of two of threads that takes a row
__host__ __device__ inline int row_threads(int values) {
    int t = 1;
    while (t < values && t < 256) t *= 2;
    return t;
}

// the sum of a weight gradient's parts, in their order; with lr the update.  A row is an output's weights of a
// network and its bias, eight values a thread.
struct GroupJoin {
    const int32_t* off;
    const float *part, *dbpart;   // [splits][K][N][M], [splits][K][N]
    int K, M, N, splits;
    float* y;
    int64_t ldy, ynet;
    float* db;
    int64_t dbnet;
    float lr;
    bf16_t* shadow;
    int threads;                  // of a row
};

__global__ __launch_bounds__(256) void group_join_kernel(GroupJoin g) {
    const int rows = 256 / g.threads, tx = threadIdx.x % g.threads, ty = threadIdx.x / g.threads;
    const int64_t all = (int64_t)g.K * g.N * g.M;
    for (int64_t r = (int64_t)blockIdx.x * rows + ty; r < (int64_t)g.K * g.N; r += (int64_t)gridDim.x * rows) {
        const int e = (int)((uint32_t)r / (uint32_t)g.N), n = (int)r - e * g.N;
        const int pairs = g.off[e + 1] - g.off[e];
        if (g.lr != 0.0f && pairs == 0) continue;  // no update
        const float scale = g.lr != 0.0f ? g.lr / (float)pairs : 0.0f;
        const int64_t at = (int64_t)n * g.ldy + e * g.ynet;
        for (int m = tx * 8; m < g.M; m += g.threads * 8) {
            const float* p = g.part + r * g.M + m;
            float s[8];
            load8_f<float>(s, p, g.M - m);
            for (int k = 1; k < g.splits; ++k) {
                float v[8];
                load8_f<float>(v, p + k * all, g.M - m);
#pragma unroll
                for (int q = 0; q < 8; ++q) s[q] += v[q];
            }
            if (g.lr != 0.0f) {
                float w[8];
                load8_f<float>(w, g.y + at + m, g.M - m);
#pragma unroll
                for (int q = 0; q < 8; ++q) s[q] = w[q] - scale * s[q];
                if (g.shadow) store8(g.shadow + at + m, s, g.M - m);
            }
            store8(g.y + at + m, s, g.M - m);
        }
        if (g.db && tx == 0) {
            float s = g.dbpart[r];
            for (int k = 1; k < g.splits; ++k) s += g.dbpart[k * (int64_t)g.K * g.N + r];
            float* db = g.db + e * g.dbnet + n;
            *db = g.lr != 0.0f ? *db - scale * s : s;
        }
    }
}

// dx[r] = (sum over j of the pairs' shares, ascending) (.) phi'(a[r]), eight neighbouring values a thread.  A row
// without a pair that is kept gets 0 and not 0 times its slope, which a NaN in a[r] would show in.
// Bound by the shares' bytes: two of each of 16,384 rows of 2048 in fp32 to bf16, 336 MB in 58 us.
template <typename T, typename TO>
__global__ __launch_bounds__(256) void group_sum_pairs_kernel(const float* part, int64_t n, int per_row, int M, const uint8_t* kept,
                                                              const T* a, int64_t lda, int act, TO* dx, int64_t ldx, int threads) {
    const int rows = 256 / threads, tx = threadIdx.x % threads, ty = threadIdx.x / threads;
    for (int64_t r = (int64_t)blockIdx.x * rows + ty; r < n; r += (int64_t)gridDim.x * rows) {
        int some = 0;
        if (a)
            for (int j = 0; j < per_row; ++j) some |= kept[r * per_row + j];
        for (int m = tx * 8; m < M; m += threads * 8) {
            const int left = M - m;
            const float* p = part + r * per_row * M + m;
            float s[8], x[8];
            if (a) load8_f<T>(x, a + r * lda + m, left);
            load8_f<float>(s, p, left);
            for (int j = 1; j < per_row; ++j) {
                float v[8];
                load8_f<float>(v, p + (int64_t)j * M, left);
#pragma unroll
                for (int q = 0; q < 8; ++q) s[q] += v[q];
            }
            if (some) group_slope8(act, s, x);
            store8(dx + r * ldx + m, s, left);
        }
    }
}

// Few pairs a network: 16 pairs and a band of the weights per workgroup, whose four waves split the
// contraction and add their sums in order through LDS.  The weights go straight from memory into the
// matrix instructions' operands, whole 128-byte lines at a time (k is permuted the same way in both
// operands), and are read once: bound by the weights' bytes.  Eight rows to two each of 32 networks 2048 -> 4096 in
// bf16: 28.9 us where a part of the weights is cached, 173 MB of memory traffic.
constexpr int GS_OUT = 32;  // outputs of a workgroup (forward)
template <typename T, typename TO>
__global__ __launch_bounds__(256) void group_few_fwd_kernel(GroupGemm g) {
    constexpr bool F32 = sizeof(T) == 4;
    constexpr int STEP = F32 ? 32 : 64, W = STEP / 4;  // values of a lane per step
    __shared__ float part[4][GS_OUT / 16][16][20];
    const int tid = threadIdx.x, lane = tid & 63, l15 = lane & 15, kg = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int mt = (g.M + GS_OUT - 1) / GS_OUT;
    const uint32_t id = blockIdx.x;
    if (id >= (uint64_t)*g.n_tiles * mt) return;
    const uint32_t tile = id / mt, band = id - tile * mt;
    const int2 t = g.tiles[tile];
    const int e = t.x, m0 = (int)band * GS_OUT, p0 = t.y;
    const int end = e < g.K ? g.off[e + 1] : g.N;
    const int nv = end - p0 < 16 ? end - p0 : 16;
    f4 acc[GS_OUT / 16];
#pragma unroll
    for (int i = 0; i < GS_OUT / 16; ++i) acc[i] = f4{0, 0, 0, 0};
    if (e < g.K) {
        const int share = (g.Kx + 4 * STEP - 1) / (4 * STEP) * STEP;
        const int k1 = (wave + 1) * share < g.Kx ? (wave + 1) * share : g.Kx;
        const T* x = l15 < nv ? (const T*)g.p + (int64_t)(g.pdiv.of(g.pairs[p0 + l15])) * g.ldp : nullptr;
        const T* w[GS_OUT / 16];
#pragma unroll
        for (int i = 0; i < GS_OUT / 16; ++i)
            w[i] = m0 + 16 * i + l15 < g.M ? (const T*)g.w + e * g.wnet + (int64_t)(m0 + 16 * i + l15) * g.ldw : nullptr;
        for (int kk = wave * share; kk < k1; kk += STEP) {
            const int k = kk + kg * W;
            Raw8<T> rx[W / 8], rw[GS_OUT / 16][W / 8];
#pragma unroll
            for (int h = 0; h < W / 8; ++h) {
                load8(rx[h], x + k + 8 * h, x ? k1 - k - 8 * h : 0);
#pragma unroll
                for (int i = 0; i < GS_OUT / 16; ++i) load8(rw[i][h], w[i] + k + 8 * h, w[i] ? k1 - k - 8 * h : 0);
            }
#pragma unroll
            for (int i = 0; i < GS_OUT / 16; ++i)
#pragma unroll
                for (int h = 0; h < W / 8; ++h) {
                    if constexpr (F32) {
#pragma unroll
                        for (int c = 0; c < 8; ++c)
                            acc[i] = __builtin_amdgcn_mfma_f32_16x16x4f32(rw[i][h].v[c >> 2][c & 3], rx[h].v[c >> 2][c & 3], acc[i], 0, 0, 0);
                    } else {
                        acc[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf8v, rw[i][h].v),
                                                                         __builtin_bit_cast(bf8v, rx[h].v), acc[i], 0, 0, 0);
                    }
                }
        }
    }
#pragma unroll
    for (int i = 0; i < GS_OUT / 16; ++i) *(f4*)&part[wave][i][l15][4 * kg] = acc[i];
    __syncthreads();
    const int n = tid >> 4, i = (tid >> 3) & 1, o = (tid & 7) * 2;
    if (n >= nv) return;
    const int64_t pair = g.pairs[p0 + n];
#pragma unroll
    for (int r = 0; r < 2; ++r) {
        const int m = m0 + 16 * i + o + r;
        if (m >= g.M) continue;
        float v = 0.0f;
        if (e < g.K) {
#pragma unroll
            for (int q = 0; q < 4; ++q) v += part[q][i][n][o + r];
            if (g.b) v += g.b[e * g.bnet + m];
            v = group_act(g.act, v);
        }
        ((TO*)g.y)[pair * g.ldy + m] = from_f<TO>(v);
    }
}

// The input gradient of few pairs: lanes hold C neighbouring columns of eight (bf16) or four (fp32)
// rows of W; column c of all of them is one operand, so the columns of an instruction are C apart.
template <typename T, typename TO>
__global__ __launch_bounds__(256) void group_few_dx_kernel(GroupGemm g) {
    constexpr bool F32 = sizeof(T) == 4;
    constexpr int C = F32 ? 4 : 8, BAND = 16 * C, STEP = F32 ? 16 : 32;
    __shared__ float part[4][16][BAND + 4];
    const int tid = threadIdx.x, lane = tid & 63, l15 = lane & 15, kg = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int mt = (g.M + BAND - 1) / BAND;
    const uint32_t id = blockIdx.x;
    if (id >= (uint64_t)*g.n_tiles * mt) return;
    const uint32_t tile = id / mt, band = id - tile * mt;
    const int2 t = g.tiles[tile];
    const int e = t.x, m0 = (int)band * BAND, p0 = t.y;
    const int end = e < g.K ? g.off[e + 1] : g.N;
    const int nv = end - p0 < 16 ? end - p0 : 16;
    f4 acc[C];
#pragma unroll
    for (int c = 0; c < C; ++c) acc[c] = f4{0, 0, 0, 0};
    if (e < g.K) {
        const int share = (g.Kx + 4 * STEP - 1) / (4 * STEP) * STEP;
        const int k1 = (wave + 1) * share < g.Kx ? (wave + 1) * share : g.Kx;
        const T* d = l15 < nv ? (const T*)g.p + (int64_t)(g.pdiv.of(g.pairs[p0 + l15])) * g.ldp : nullptr;
        const int cols = g.M - m0 - C * l15;
        const T* w = (const T*)g.w + e * g.wnet + m0 + C * l15;
        for (int kk = wave * share; kk < k1; kk += STEP) {
            const int k = kk + kg * (STEP / 4);
            if constexpr (F32) {
                float dv[4], wv[4][4];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    dv[j] = d && k + j < k1 ? d[k + j] : 0.0f;
                    const int c4 = k + j < k1 ? cols : 0;
                    if (c4 >= 4) {
                        const f4 q = *(const f4_a4*)(w + (int64_t)(k + j) * g.ldw);
                        wv[j][0] = q[0]; wv[j][1] = q[1]; wv[j][2] = q[2]; wv[j][3] = q[3];
                    } else {
#pragma unroll
                        for (int c = 0; c < 4; ++c) wv[j][c] = c < c4 ? w[(int64_t)(k + j) * g.ldw + c] : 0.0f;
                    }
                }
#pragma unroll
                for (int j = 0; j < 4; ++j)
#pragma unroll
                    for (int c = 0; c < 4; ++c) acc[c] = __builtin_amdgcn_mfma_f32_16x16x4f32(wv[j][c], dv[j], acc[c], 0, 0, 0);
            } else {
                Raw8<T> rd, rw[8];
                load8(rd, d + k, d ? k1 - k : 0);
#pragma unroll
                for (int j = 0; j < 8; ++j) load8(rw[j], w + (int64_t)(k + j) * g.ldw, k + j < k1 ? cols : 0);
#pragma unroll
                for (int c = 0; c < 8; ++c) {
                    const uint32_t sel = c & 1 ? 0x07060302u : 0x05040100u;
                    u4v q;
#pragma unroll
                    for (int h = 0; h < 4; ++h) q[h] = __builtin_amdgcn_perm(rw[2 * h + 1].v[c >> 1], rw[2 * h].v[c >> 1], sel);
                    acc[c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf8v, q), __builtin_bit_cast(bf8v, rd.v),
                                                                     acc[c], 0, 0, 0);
                }
            }
        }
    }
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
        for (int r = 0; r < 4; ++r) part[wave][l15][C * (4 * kg + r) + c] = acc[c][r];
    __syncthreads();
    const int n = tid >> 4;
    if (n >= nv) return;
    const int64_t pair = g.pairs[p0 + n];
#pragma unroll
    for (int c = 0; c < C; ++c) {
        const int q = (tid & 15) + 16 * c, m = m0 + q;
        if (m >= g.M) continue;
        float v = 0.0f;
        if (e < g.K) {
#pragma unroll
            for (int s = 0; s < 4; ++s) v += part[s][n][q];
            if (g.a) v *= act_deriv(g.act, to_f<T>(((const T*)g.a)[pair * g.lda + m]));
        }
        ((TO*)g.y)[pair * g.ldy + m] = from_f<TO>(v);
    }
}

__global__ __launch_bounds__(256) void rows_to_bf16_kernel(const float* src, bf16_t* dst, int64_t n) {
    for (int64_t i = (blockIdx.x * 256ll + threadIdx.x) * 8; i < n; i += gridDim.x * 2048ll) {
        float v[8];
        const int left = n - i < 8 ? (int)(n - i) : 8;
        load8_f<float>(v, src + i, left);
        store8(dst + i, v, left);
    }
}

// A row's answer: the outputs x^L of its pairs, weighted (without weights each counts the same), and
// the class of the largest (lowest index on ties).  A row without a network: outputs 0, class -1.
__global__ __launch_bounds__(256) void routed_answer_kernel(const float* z, const int32_t* ids, const float* weights, int64_t n,
                                                            int per_row, int K, int O, int act, int32_t* pred, float* out) {
    const int64_t r = blockIdx.x * 256ll + threadIdx.x;
    if (r >= n) return;
    float sum[MAX_OUT], total = 0.0f;
#pragma unroll
    for (int o = 0; o < MAX_OUT; ++o) sum[o] = 0.0f;
    int kept = 0;
    for (int j = 0; j < per_row; ++j) {
        const int64_t p = r * per_row + j;
        if ((unsigned)ids[p] >= (unsigned)K) continue;
        ++kept;
        const float w = weights ? weights[p] : 1.0f;
        float v[MAX_OUT], m = -__builtin_huge_valf(), s = 0.0f;
#pragma unroll
        for (int o = 0; o < MAX_OUT; ++o)
            if (o < O) {
                v[o] = z[p * O + o];
                m = fmaxf(m, v[o]);
            }
#pragma unroll
        for (int o = 0; o < MAX_OUT; ++o)
            if (o < O) {
                v[o] = act == ACT_SOFTMAX ? expf(v[o] - m) : group_act(act, v[o]);
                s += v[o];
            }
        const float by = act == ACT_SOFTMAX ? w / s : w;
#pragma unroll
        for (int o = 0; o < MAX_OUT; ++o)
            if (o < O) sum[o] += v[o] * by;
    }
    total = weights || kept == 0 ? 1.0f : 1.0f / (float)kept;
    int best = kept ? 0 : -1;
    float top = 0.0f;
#pragma unroll
    for (int o = 0; o < MAX_OUT; ++o)
        if (o < O) {
            const float v = sum[o] * total;
            if (out) out[r * O + o] = v;
            if (kept && (o == 0 || v > top)) {
                top = v;
                best = o;
            }
        }
    pred[r] = best;
}

}  // namespace pnn
