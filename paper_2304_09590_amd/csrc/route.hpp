// route.hpp -- rows choose their networks, and the results of a row's pairs are weighed into one.
//
// Row r has a score s_e for each of K networks.  With p = softmax(s) it goes through the k networks of the largest
// scores (descending, the lowest index on ties; -inf is never chosen), its gates are p at these, or p divided by the
// chosen ones' sum.  With counts_e pairs of network e, C = sum counts and n' rows that have a pair,
//   loss = K sum_e (counts_e / C) (sum_r p_re) / n'          (1 where rows and choices are spread evenly)
//   ds_e = p_e (a_e - sum p a) + the gates' share, a_e = dloss K counts_e / (C n')
// with the share p_e ([e chosen] dgate_e - sum gate dgate), or with normalised gates gate_e (dgate_e - sum gate dgate)
// at the chosen ones alone.
//
//   combined         y[r]  = sum_j w_rj y[p],  p = r k + j, over the pairs that are not dropped
//   its gradients    dy[p] = w_rj g[r],  dw_rj = <g[r], y[p]>
#pragma once
#include "groups.hpp"

namespace pnn {

constexpr int RT_MAX_TOP = 64;       // most networks of a row
constexpr int RT_THREADS = 1024;     // threads of a workgroup that routes
constexpr int RT_MAX_BLOCKS = 256;   // most workgroups whose sums are joined
constexpr int RT_JOIN = 16;          // networks that a workgroup joins

struct RouteArgs {
    const void* s;
    int64_t lds, n;
    int K, k;
    bool normalize;
    int32_t* ids;
    float* gates;
    int32_t* counts;          // [K + 1]: pairs of each network, rows that have a pair (nullable: no balance)
    float* loss;
    float* part;              // [blocks][K] sums of p
    int32_t* part_counts;     // [blocks][K + 1]
    float* dots;              // [workgroups that join] sums of counts times sums of p, then their pairs
    int32_t* arrived;         // workgroups that have joined
    int blocks;
    // gradient
    const float *dgates, *dloss;
    void* ds;
    int64_t ldds;
};

// what lanes of a wave have written to LDS before is what others of it read after (its accesses keep their order)
__device__ inline void route_order() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_wave_barrier();
}

constexpr float RT_INF = __builtin_huge_valf();
constexpr float RT_LOG2E = 1.44269504f, RT_LOG2E_REST = 1.92596299e-8f;

// exp(d) for d <= 0, -inf among them: 2^t for the rounded t = d log2 e, times what the rounding leaves, 1 + (d - t ln 2).  The
// remainder is below 2^-15 where 2^t is not 0, and no number for -inf, where the median is its bound and 2^t is 0.
// Without it (in a row's sums, where the shares that are far off are small) the error grows by 2 |d| half steps; with it there too
// 60,000 rows of 256 networks take 50.0 us for 48.3, 16,384 of 1,000 in bf16 54.4 for 52.2.
__device__ inline float route_exp(float d) {
    const float t = d * RT_LOG2E, e = __builtin_amdgcn_exp2f(t);
    return __builtin_fmaf(e, __builtin_amdgcn_fmed3f(__builtin_fmaf(-t, 0.693147181f, d), -0x1p-12f, 0x1p-12f), e);
}

// A row lies on L lanes, V scores each: chunks of CH neighbouring ones, the lanes' chunks side by side.
template <int L, int V>
struct RouteLane {
    static constexpr int CH = V < 4 ? V : 4;
    static __device__ inline int column(int l, int v) { return (v / CH * L + l) * CH + v % CH; }
};

// the scores of a row as loaded (-inf outside it), and as fp32
template <typename T, int L, int V>
struct RouteRaw {
    typedef RouteLane<L, V> At;
    typedef typename std::conditional<sizeof(T) == 4, f4, u2v>::type Four;
    typedef typename std::conditional<sizeof(T) == 4, f4_a4, u2v_a2>::type Loose;
    Four four[V == 1 ? 1 : V / 4];
    T one;
    __device__ inline void load(const T* s, int K, int l) {
        const T none = from_f<T>(-RT_INF);
        if constexpr (V == 1) {
            one = l < K ? s[l] : none;
        } else {
#pragma unroll
            for (int h = 0; h < V / 4; ++h) {
                const int c = At::column(l, 4 * h);
                if (c + 4 <= K) {
                    four[h] = *(const Loose*)(s + c);
                } else {
                    T t[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) t[i] = c + i < K ? s[c + i] : none;
                    if constexpr (sizeof(T) == 4) four[h] = f4{t[0], t[1], t[2], t[3]};
                    else four[h] = u2v{(uint32_t)t[0] | (uint32_t)t[1] << 16, (uint32_t)t[2] | (uint32_t)t[3] << 16};
                }
            }
        }
    }
    __device__ inline void get(float (&x)[V]) const {
        if constexpr (V == 1) {
            x[0] = to_f<T>(one);
        } else {
#pragma unroll
            for (int v = 0; v < V; ++v) {
                if constexpr (sizeof(T) == 4) x[v] = four[v / 4][v % 4];
                else x[v] = v & 1 ? bf_hi(four[v / 4][v % 4 >> 1]) : bf_lo(four[v / 4][v % 4 >> 1]);
            }
        }
    }
};

template <int L> __device__ inline float route_max(float v) {
    return lanes_reduce<L>(v, [](float a, float b) { return fmaxf(a, b); });
}
template <int L> __device__ inline float route_sum(float v) {
    return lanes_reduce<L>(v, [](float a, float b) { return a + b; });
}
template <int L> __device__ inline int route_min(int v) {
    return lanes_reduce<L>(v, [](int a, int b) { return a < b ? a : b; });
}

// e = exp(x - max) of a row; 1 / sum: 0 for a row of -inf, NaN for one with a NaN or an infinity.  Of fp32 scores without
// the rounding of log2 e, which puts all of a row's sum off one way: gates among 256 networks 5.9 -> 5.4e-8 off, the gradient
// 6.7 -> 6.3e-8, for 0.3 us of 49 (bf16 scores gain nothing).
template <typename T, int L, int V>
__device__ inline void route_softmax(const float (&x)[V], float (&e)[V], float& top, float& inv) {
    float m = x[0];
#pragma unroll
    for (int v = 1; v < V; ++v) m = fmaxf(m, x[v]);
    m = route_max<L>(m);
    top = m == -RT_INF ? 0.0f : m;
    float s = 0.0f;
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const float d = x[v] - top;
        e[v] = __builtin_amdgcn_exp2f(sizeof(T) == 4 ? __builtin_fmaf(d, RT_LOG2E, d * RT_LOG2E_REST) : d * RT_LOG2E);
        s += e[v];
    }
    s = route_sum<L>(s);
    inv = s == 0.0f ? 0.0f : 1.0f / s;
}

// the counts and the loss of all networks: a workgroup's share of dot = sum counts_e sum p_e
__device__ inline float route_loss(float dot, int pairs, int rows, int K) {
    // (without a row to count the loss is 0, or NaN where a row held one)
    return dot * ((float)K / ((float)(pairs > 0 ? pairs : 1) * (float)(rows > 0 ? rows : 1)));
}

// Scores as integers that are ordered alike (-0 as 0): of bf16 ones the low half is free, and holds the column so that
// of equal scores the lowest index is the largest key.
constexpr int RT_GONE = INT32_MIN;               // a score that was chosen
constexpr int RT_NONE = (int)0x807fffffu;        // -inf, or anything below the smallest number
template <typename T>
__device__ inline int route_key(float x, int column) {
    constexpr int MASK = sizeof(T) == 4 ? 0x7fffffff : 0x7fff0000;
    const int b = __float_as_int(x + 0.0f), k = b ^ (b >> 31 & MASK);
    return sizeof(T) == 4 ? k : k | (0xffff - column);
}
template <typename T>
__device__ inline float route_value(int key) {
    constexpr int MASK = sizeof(T) == 4 ? 0x7fffffff : 0x7fff0000;
    const int k = sizeof(T) == 4 ? key : key & (int)0xffff0000;
    return __int_as_float(k ^ (k >> 31 & MASK));
}
template <int L> __device__ inline int route_top(int v) {
    return lanes_reduce<L>(v, [](int a, int b) { return a > b ? a : b; });
}

// Choosing is k times the largest of the row's lanes' largest (the lowest index on ties).  The lane that held it then
// needs its next: its V keys lie in LDS, where 16 lanes look at one each, so a choice costs the same whatever V is.
// 16,384 rows of 1,000 scores in bf16, eight each: 59 us with all lanes' scores looked through again for each choice, 35
// this way, 21 to 24 with keys that hold their columns and the next row's scores on their way (33 MB: 7 us; the rest is the
// choices' instructions, a third of them exchanges between lanes).  60,000 rows of 256 in fp32, two each: 17 us, 61 MB.
template <typename T, int L, int V>
__global__ __launch_bounds__(RT_THREADS) void route_kernel(RouteArgs a) {
    typedef RouteLane<L, V> At;
    constexpr bool APART = sizeof(T) == 4;  // columns apart from the keys
    constexpr int WAVES = RT_THREADS / 64, ROWS = 64 / L, KEEP = RT_MAX_TOP / L, LD = V == 1 ? 1 : V + 4;
    __shared__ int cnt[GR_MAX_NETS + 1];
    __shared__ __align__(16) int lds[RT_THREADS * LD];  // (LD of each lane; afterwards the waves' sums)
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, l = lane % L, sub = lane / L;
    int *mine = lds + tid * LD, *row0 = lds + (tid - l) * LD;  // this lane's keys, and the row's first lane's
    if (a.counts) {
        for (int e = tid; e <= a.K; e += RT_THREADS) cnt[e] = 0;
        __syncthreads();
    }
    float acc[V];
#pragma unroll
    for (int v = 0; v < V; ++v) acc[v] = 0.0f;
    const int64_t step = (int64_t)gridDim.x * WAVES * ROWS;
    int64_t r0 = ((int64_t)blockIdx.x * WAVES + wave) * ROWS;
    RouteRaw<T, L, V> raw;
    auto load = [&](int64_t at) { raw.load((const T*)a.s + (at + sub < a.n ? at + sub : a.n - 1) * a.lds, a.K, l); };
    if (r0 < a.n) load(r0);
    // (all lanes of a wave run every step: what they exchange needs all of them)
    for (; r0 < a.n; r0 += step) {
        const bool in = r0 + sub < a.n;
        const int64_t r = in ? r0 + sub : a.n - 1;
        float x[V], e[V], top, inv;
        raw.get(x);
        int best = RT_GONE, at = 0;  // the lane's largest key, and its column
        if (APART || V == 1) {
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const int k = route_key<T>(x[v], At::column(l, v));
                if (V > 1) mine[v] = k;
                if (APART && k > best) at = At::column(l, v);
                best = k > best ? k : best;
            }
        } else {
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const int k = route_key<T>(x[v], At::column(l, v));
                mine[v] = k;
                best = k > best ? k : best;
            }
        }
        route_order();
        route_softmax<T, L, V>(x, e, top, inv);
        if (r0 + step < a.n) load(r0 + step);
        const bool bad = inv != inv, has = inv > 0.0f;
        if (a.counts && in) {
#pragma unroll
            for (int v = 0; v < V; ++v) acc[v] += e[v] * inv;
            if (l == 0 && has) atomicAdd(&cnt[a.K], 1);
        }
        int id[KEEP], key[KEEP];
#pragma unroll
        for (int q = 0; q < KEEP; ++q) {
            id[q] = -1;
            key[q] = RT_NONE;
            for (int j = 0; j < L && q * L + j < a.k; ++j) {
                const int m = route_top<L>(best);
                const int c = APART ? route_min<L>(best == m ? at : INT32_MAX) : 0xffff - (m & 0xffff);
                if (l == j) {
                    id[q] = has && m > RT_NONE ? c : -1;
                    key[q] = m;
                }
                if (q * L + j + 1 == a.k) break;
                if (V == 1) {
                    if (l == c) best = RT_GONE;
                    continue;
                }
                // the lane that held it looks for its next (where nothing is left, any lane will do)
                const int o = c / At::CH % L, i = lane & 15, col = At::column(o, i < V ? i : 0);
                int w = i < V ? row0[o * LD + i] : RT_GONE;
                if (APART ? col == c : w == m) {
                    w = RT_GONE;
                    if (l < 16 && i < V) row0[o * LD + i] = RT_GONE;
                }
                route_order();  // (all lanes of the row read it in the next round)
                const int next = route_top<16>(w);
                if (APART) {
                    const int next_at = route_min<16>(i < V && w == next ? col : INT32_MAX);
                    if (l == o) at = next_at;
                }
                if (l == o) best = next;
            }
        }
        float ge[KEEP], chosen = 0.0f;
#pragma unroll
        for (int q = 0; q < KEEP; ++q) {
            ge[q] = id[q] >= 0 ? route_exp(route_value<T>(key[q]) - top) : 0.0f;
            chosen += ge[q];
        }
        if (a.normalize) chosen = route_sum<L>(chosen);
        if (in) {
            const float by = bad ? inv : a.normalize ? (chosen > 0.0f ? 1.0f / chosen : 0.0f) : inv;
#pragma unroll
            for (int q = 0; q < KEEP; ++q)
                if (q * L + l < a.k) {
                    a.ids[r * a.k + q * L + l] = id[q];
                    a.gates[r * a.k + q * L + l] = bad ? by : ge[q] * by;
                    if (a.counts && id[q] >= 0) atomicAdd(&cnt[id[q]], 1);
                }
        }
        route_order();  // (the next row's keys go where this one's were looked through)
    }
    if (!a.counts) return;
    // the workgroup's sums: of the rows within a wave, then of the waves, in their order
#pragma unroll
    for (int v = 0; v < V; ++v) {
#pragma unroll
        for (int d = L; d < 64; d <<= 1) acc[v] += __shfl_xor(acc[v], d);
    }
    __syncthreads();
    float* sums = (float*)lds;  // [waves][L * V]
    if (sub == 0) {
#pragma unroll
        for (int v = 0; v < V; ++v) sums[wave * L * V + At::column(l, v)] = acc[v];
    }
    __syncthreads();
    const bool alone = gridDim.x == 1;
    float dot = 0.0f;
    int pairs = 0;
    for (int e = tid; e <= a.K; e += RT_THREADS) {
        float s = e < a.K ? sums[e] : 0.0f;
        if (e < a.K) {
#pragma unroll
            for (int w = 1; w < WAVES; ++w) s += sums[w * L * V + e];
        }
        if (alone) {
            a.counts[e] = cnt[e];
            if (e < a.K) {
                dot += (float)cnt[e] * s;
                pairs += cnt[e];
            }
        } else {
            a.part_counts[(int64_t)blockIdx.x * (a.K + 1) + e] = cnt[e];
            if (e < a.K) a.part[(int64_t)blockIdx.x * a.K + e] = s;
        }
    }
    if (!alone) {
        if (blockIdx.x == 0 && tid == 0) *a.arrived = 0;
        return;
    }
    __syncthreads();
    dot = route_sum<64>(dot);
    pairs = lanes_reduce<64>(pairs, [](int x, int y) { return x + y; });
    if (lane == 0) {
        sums[wave] = dot;
        lds[WAVES + wave] = pairs;
    }
    __syncthreads();
    if (tid == 0) {
        for (int w = 1; w < WAVES; ++w) {
            dot += sums[w];
            pairs += lds[WAVES + w];
        }
        a.loss[0] = route_loss(dot, pairs, cnt[a.K], a.K);
    }
}

// Counts and loss from the workgroups' sums, in their order: 16 networks a workgroup, 16 threads each; the last
// workgroup to come adds up what all have written.  Latencies one after another: 5 to 7 us (one workgroup for all networks: 77).
__global__ __launch_bounds__(256) void route_join_kernel(RouteArgs a) {
    __shared__ float sums[16][RT_JOIN];
    __shared__ int counts[16][RT_JOIN];
    __shared__ bool last;
    const int tid = threadIdx.x, x = tid % RT_JOIN, y = tid / RT_JOIN, e = (int)blockIdx.x * RT_JOIN + x;
    int c[RT_MAX_BLOCKS / 16];
    float s[RT_MAX_BLOCKS / 16];
#pragma unroll
    for (int i = 0; i < RT_MAX_BLOCKS / 16; ++i) {
        const int b = y * (RT_MAX_BLOCKS / 16) + i;
        c[i] = e <= a.K && b < a.blocks ? a.part_counts[(int64_t)b * (a.K + 1) + e] : 0;
        s[i] = e < a.K && b < a.blocks ? a.part[(int64_t)b * a.K + e] : 0.0f;
    }
#pragma unroll
    for (int i = 1; i < RT_MAX_BLOCKS / 16; ++i) {
        c[0] += c[i];
        s[0] += s[i];
    }
    sums[y][x] = s[0];
    counts[y][x] = c[0];
    __syncthreads();
    if (tid < 64) {  // (lanes from RT_JOIN on add nothing)
        int all = 0;
        float p = 0.0f;
        if (tid < RT_JOIN) {
            for (int i = 0; i < 16; ++i) {
                all += counts[i][tid];
                p += sums[i][tid];
            }
            if (e <= a.K) a.counts[e] = all;
        }
        const bool network = tid < RT_JOIN && e < a.K;
        const float dot = route_sum<16>(network ? (float)all * p : 0.0f);
        const int pairs = lanes_reduce<16>(network ? all : 0, [](int x, int y) { return x + y; });
        if (tid == 0) {
            a.dots[2 * blockIdx.x] = dot;
            a.dots[2 * blockIdx.x + 1] = __int_as_float(pairs);
        }
        // (counts[K], the number of rows, is one of the networks' places of the last workgroup)
        __threadfence();
        if (tid == 0) last = atomicAdd(a.arrived, 1) == (int)gridDim.x - 1;
    }
    __syncthreads();
    if (!last || tid >= 64) return;
    __threadfence();
    float dot = 0.0f;
    int pairs = 0;
    for (int w = tid; w < (int)gridDim.x; w += 64) {
        dot += __hip_atomic_load(a.dots + 2 * w, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        pairs += __float_as_int(__hip_atomic_load(a.dots + 2 * w + 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT));
    }
    dot = route_sum<64>(dot);
    pairs = lanes_reduce<64>(pairs, [](int x, int y) { return x + y; });
    if (tid == 0) a.loss[0] = route_loss(dot, pairs, __hip_atomic_load(a.counts + a.K, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT), a.K);
}

// four neighbouring values, the first nv of them
__device__ inline void route_store4(float* p, const float* v, int nv) {
    if (nv >= 4) {
        *(f4_a4*)p = f4{v[0], v[1], v[2], v[3]};
    } else {
#pragma unroll
        for (int i = 0; i < 3; ++i)
            if (i < nv) p[i] = v[i];
    }
}
__device__ inline void route_store4(bf16_t* p, const float* v, int nv) {
    if (nv >= 4) {
        *(u2v_a2*)p = u2v{cvt_pk_bf16(v[0], v[1]), cvt_pk_bf16(v[2], v[3])};
    } else {
#pragma unroll
        for (int i = 0; i < 3; ++i)
            if (i < nv) p[i] = f2bf(v[i]);
    }
}

// What the gates add lies in LDS, a place for each score of the row, where the lanes that hold the choices write theirs (a
// network that stands twice gets a sum in the order of the choices).  Bound by bytes where rows are many: 60,000 rows of 256
// scores in fp32 26 to 27 us, 4.7 to 4.6 TB/s; 16,384 of 1,000 in bf16 20 to 24 us, 2.7 to 3.3 TB/s, instructions and the counts at its beginning.
template <typename T, int L, int V>
__global__ __launch_bounds__(256) void route_grad_kernel(RouteArgs a) {
    typedef RouteLane<L, V> At;
    constexpr int WAVES = 4, ROWS = 64 / L, KEEP = RT_MAX_TOP / L, LD = V == 1 ? 1 : V + 4;
    __shared__ __align__(16) float lds[256 * LD];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, l = lane % L, sub = lane / L;
    float *mine = lds + tid * LD, *row0 = lds + (tid - l) * LD;
    auto place = [&](int c) { return row0 + c / At::CH % L * LD + c / (At::CH * L) * At::CH + c % At::CH; };
#pragma unroll
    for (int v = 0; v < V; ++v) mine[v] = 0.0f;
    route_order();
    float w[V];  // a_e
#pragma unroll
    for (int v = 0; v < V; ++v) w[v] = 0.0f;
    const int64_t step = (int64_t)gridDim.x * WAVES * ROWS;
    int64_t r0 = ((int64_t)blockIdx.x * WAVES + wave) * ROWS;
    RouteRaw<T, L, V> raw;
    auto load = [&](int64_t at) { raw.load((const T*)a.s + (at + sub < a.n ? at + sub : a.n - 1) * a.lds, a.K, l); };
    if (r0 < a.n) load(r0);
    if (a.dloss) {
        int c[V], all = 0;
        const int rows = a.counts[a.K];
#pragma unroll
        for (int v = 0; v < V; ++v) c[v] = At::column(l, v) < a.K ? a.counts[At::column(l, v)] : 0;
#pragma unroll
        for (int v = 0; v < V; ++v) all += c[v];
        all = lanes_reduce<L>(all, [](int x, int y) { return x + y; });
        const float by = a.dloss[0] * route_loss(1.0f, all, rows, a.K);
#pragma unroll
        for (int v = 0; v < V; ++v) w[v] = by * (float)c[v];
    }
    for (; r0 < a.n; r0 += step) {
        const bool in = r0 + sub < a.n;
        const int64_t r = in ? r0 + sub : a.n - 1;
        int id[KEEP];
        float gate[KEEP], dg[KEEP], chosen = 0.0f, mix = 0.0f;
#pragma unroll
        for (int q = 0; q < KEEP; ++q) {
            id[q] = -1;
            gate[q] = -RT_INF;
            dg[q] = 0.0f;
            if (a.dgates && q * L + l < a.k) {
                const int i = a.ids[r * a.k + q * L + l];
                if ((unsigned)i < (unsigned)a.K) {
                    id[q] = i;
                    gate[q] = to_f<T>(((const T*)a.s)[r * a.lds + i]);
                    dg[q] = a.dgates[r * a.k + q * L + l];
                }
            }
        }
        float x[V], p[V], top, inv;
        raw.get(x);
        route_softmax<T, L, V>(x, p, top, inv);
        if (r0 + step < a.n) load(r0 + step);
        float dot = 0.0f;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            p[v] *= inv;
            dot += p[v] * w[v];
        }
        dot = route_sum<L>(dot);
        if (a.dgates) {
            // (gates among the chosen ones count from their own largest score: ids may be any, and all far below the row's)
            float peak = top;
            if (a.normalize) {
                peak = gate[0];
#pragma unroll
                for (int q = 1; q < KEEP; ++q) peak = fmaxf(peak, gate[q]);
                peak = route_max<L>(peak);
                if (peak == -RT_INF) peak = 0.0f;
            }
#pragma unroll
            for (int q = 0; q < KEEP; ++q) {
                gate[q] = route_exp(gate[q] - peak);
                if (id[q] >= 0) chosen += gate[q];
            }
            if (a.normalize) chosen = route_sum<L>(chosen);
            const float by = a.normalize ? (chosen != 0.0f ? 1.0f / chosen : 0.0f) : inv;
#pragma unroll
            for (int q = 0; q < KEEP; ++q) {
                gate[q] *= by;
                if (id[q] >= 0) mix += gate[q] * dg[q];
            }
            mix = route_sum<L>(mix);
            // each choice writes its number, and finds another's where the same network stands twice
            bool twice = false;
#pragma unroll
            for (int q = 0; q < KEEP; ++q)
                if (id[q] >= 0) *place(id[q]) = __int_as_float(q * L + l);
            route_order();
#pragma unroll
            for (int q = 0; q < KEEP; ++q)
                if (id[q] >= 0) twice |= __float_as_int(*place(id[q])) != q * L + l;
            route_order();
            const bool any = __ballot(twice) != 0;
#pragma unroll
            for (int q = 0; q < KEEP; ++q) {
                gate[q] *= a.normalize ? dg[q] - mix : dg[q];
                if (id[q] >= 0) *place(id[q]) = any ? 0.0f : gate[q];
            }
            route_order();
            if (any) {  // one after another
#pragma unroll
                for (int q = 0; q < KEEP; ++q)
                    for (int j = 0; j < L && q * L + j < a.k; ++j) {
                        if (l == j && id[q] >= 0) *place(id[q]) += gate[q];
                        route_order();
                    }
            }
        }
        const float off = a.normalize ? dot : dot + mix;
        float d[V];
#pragma unroll
        for (int v = 0; v < V; ++v) {
            d[v] = p[v] * (w[v] - off);
            if (a.dgates) d[v] += mine[v];
        }
        if (a.dgates) {
            route_order();
#pragma unroll
            for (int q = 0; q < KEEP; ++q)
                if (id[q] >= 0) *place(id[q]) = 0.0f;
            route_order();  // (other lanes' choices of the next row go there)
        }
        if (!in) continue;
        T* out = (T*)a.ds + r * a.ldds;
        if constexpr (V == 1) {
            if (l < a.K) out[l] = from_f<T>(d[0]);
        } else {
#pragma unroll
            for (int v = 0; v < V; v += 4) route_store4(out + At::column(l, v), d + v, a.K - At::column(l, v));
        }
    }
}

// ------------------------------------------------------------------------------------
// combining

struct CombineArgs {
    const void* y;            // [n per_row][M] results of the pairs
    int64_t ldy, n;
    int per_row, M, K;
    const int32_t* ids;
    const float* w;
    void* out;                // [n][M]
    int64_t ldo;
    // gradient
    const void* g;            // [n][M]
    int64_t ldg;
    void* dy;
    int64_t lddy;
    float* dw;
    int threads;              // of a row
};

// Eight neighbouring values a thread; a dropped pair's rows are not read.  Bound by bytes: 32,768 rows of two pairs of 4,096
// values in bf16, 805 MB in 143 us (5.6 TB/s).
template <typename T, typename TO>
__global__ __launch_bounds__(256) void combine_kernel(CombineArgs a) {
    const int rows = 256 / a.threads, tx = threadIdx.x % a.threads, ty = threadIdx.x / a.threads;
    for (int64_t r = (int64_t)blockIdx.x * rows + ty; r < a.n; r += (int64_t)gridDim.x * rows) {
        for (int m = tx * 8; m < a.M; m += a.threads * 8) {
            const int left = a.M - m;
            float s[8] = {0, 0, 0, 0, 0, 0, 0, 0};
            for (int j = 0; j < a.per_row; ++j) {
                const int64_t p = r * a.per_row + j;
                if ((unsigned)a.ids[p] >= (unsigned)a.K) continue;
                const float w = a.w[p];
                float v[8];
                load8_f<T>(v, (const T*)a.y + p * a.ldy + m, left);
#pragma unroll
                for (int q = 0; q < 8; ++q) s[q] = __builtin_fmaf(w, v[q], s[q]);
            }
            store8((TO*)a.out + r * a.ldo + m, s, left);
        }
    }
}

// A row's pairs four at a time, which share what is loaded of g's row.  The same rows as above: 1,342 MB in 238 us (5.6
// TB/s; a pair after the other reads a part of g twice, 1,549 MB in 247 us).
constexpr int CB_PAIRS = 4;
template <typename T, typename TG>
__global__ __launch_bounds__(256) void combine_grad_kernel(CombineArgs a) {
    __shared__ float red[CB_PAIRS][4];
    const int rows = 256 / a.threads, tx = threadIdx.x % a.threads, ty = threadIdx.x / a.threads;
    for (int64_t r0 = (int64_t)blockIdx.x * rows; r0 < a.n; r0 += (int64_t)gridDim.x * rows) {
        const bool in = r0 + ty < a.n;
        const int64_t r = in ? r0 + ty : a.n - 1;
        for (int j0 = 0; j0 < a.per_row; j0 += CB_PAIRS) {
            const int64_t p0 = r * a.per_row + j0;
            const int pairs = a.per_row - j0 < CB_PAIRS ? a.per_row - j0 : CB_PAIRS;
            bool kept[CB_PAIRS];
            float w[CB_PAIRS], dot[CB_PAIRS];
#pragma unroll
            for (int j = 0; j < CB_PAIRS; ++j) {
                kept[j] = j < pairs && (unsigned)a.ids[p0 + (j < pairs ? j : 0)] < (unsigned)a.K;
                w[j] = kept[j] ? a.w[p0 + j] : 0.0f;
                dot[j] = 0.0f;
            }
            for (int m = tx * 8; m < a.M && in; m += a.threads * 8) {
                const int left = a.M - m;
                Raw8<TG> gr;
                Raw8<T> yr[CB_PAIRS];
                load8(gr, (const TG*)a.g + r * a.ldg + m, left);
#pragma unroll
                for (int j = 0; j < CB_PAIRS; ++j)
                    if (kept[j]) load8(yr[j], (const T*)a.y + (p0 + j) * a.ldy + m, left);
                float g[8];
                raw8_f(g, gr);
#pragma unroll
                for (int j = 0; j < CB_PAIRS; ++j) {
                    if (j >= pairs) break;
                    float v[8] = {0, 0, 0, 0, 0, 0, 0, 0};
                    if (kept[j]) {
                        raw8_f(v, yr[j]);
#pragma unroll
                        for (int q = 0; q < 8; ++q) {
                            dot[j] = __builtin_fmaf(g[q], v[q], dot[j]);
                            v[q] = w[j] * g[q];
                        }
                    }
                    store8((T*)a.dy + (p0 + j) * a.lddy + m, v, left);
                }
            }
#pragma unroll
            for (int j = 0; j < CB_PAIRS; ++j)
                for (int d = 1; d < a.threads && d < 64; d <<= 1) dot[j] += __shfl_xor(dot[j], d);
            if (a.threads > 64) {
                __syncthreads();
                if ((threadIdx.x & 63) == 0) {
#pragma unroll
                    for (int j = 0; j < CB_PAIRS; ++j) red[j][threadIdx.x >> 6] = dot[j];
                }
                __syncthreads();
#pragma unroll
                for (int j = 0; j < CB_PAIRS; ++j) {
                    dot[j] = red[j][ty * (a.threads / 64)];
                    for (int q = 1; q < a.threads / 64; ++q) dot[j] += red[j][ty * (a.threads / 64) + q];
                }
            }
            if (in && tx == 0) {
#pragma unroll
                for (int j = 0; j < CB_PAIRS; ++j)
                    if (j < pairs) a.dw[p0 + j] = dot[j];
            }
        }
    }
}

}  // namespace pnn
