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
constexpr int RT_THREADS = 512;      // threads of a workgroup that routes
constexpr int RT_MAX_BLOCKS = 256;   // most workgroups whose sums are joined

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
    int blocks;
    // gradient
    const float *dgates, *dloss;
    void* ds;
    int64_t ldds;
};

constexpr float RT_INF = __builtin_huge_valf();
constexpr float RT_LOG2E = 1.44269504f;

// A row lies on L lanes, V scores each: chunks of CH neighbouring ones, the lanes' chunks side by side.
template <int L, int V>
struct RouteLane {
    static constexpr int CH = V < 4 ? V : 4;
    static __device__ inline int column(int l, int v) { return (v / CH * L + l) * CH + v % CH; }
};

// the scores of a row (-inf outside it)
template <typename T, int L, int V>
__device__ inline void route_load(float (&x)[V], const T* s, int K, int l) {
    typedef RouteLane<L, V> At;
    typedef uint32_t u2v __attribute__((ext_vector_type(2)));
    typedef u2v u2v_a2 __attribute__((aligned(2)));
#pragma unroll
    for (int v = 0; v < V; v += At::CH) {
        const int c = At::column(l, v);
        if (At::CH == 4 && c + 4 <= K) {
            if constexpr (sizeof(T) == 4) {
                const f4 q = *(const f4_a4*)(s + c);
#pragma unroll
                for (int i = 0; i < 4; ++i) x[(v + i) % V] = q[i];
            } else {
                const u2v q = *(const u2v_a2*)(s + c);
#pragma unroll
                for (int i = 0; i < 4; ++i) x[(v + i) % V] = i & 1 ? bf_hi(q[i >> 1]) : bf_lo(q[i >> 1]);
            }
        } else {
#pragma unroll
            for (int i = 0; i < At::CH; ++i) x[v + i] = c + i < K ? to_f<T>(s[c + i]) : -RT_INF;
        }
    }
}

template <int L> __device__ inline float route_max(float v) {
    v = row_allmax16(v);
    if (L == 64) {
        v = fmaxf(v, __shfl_xor(v, 16));
        v = fmaxf(v, __shfl_xor(v, 32));
    }
    return v;
}
template <int L> __device__ inline float route_sum(float v) {
    v = row_allsum16(v);
    if (L == 64) {
        v += __shfl_xor(v, 16);
        v += __shfl_xor(v, 32);
    }
    return v;
}
template <int L> __device__ inline int route_min(int v) {
#pragma unroll
    for (int d = 1; d < L; d <<= 1) {
        const int u = __shfl_xor(v, d);
        v = u < v ? u : v;
    }
    return v;
}

// e = exp(x - max) of a row; 1 / sum: 0 for a row of -inf, NaN for one with a NaN or an infinity
template <int L, int V>
__device__ inline void route_softmax(const float (&x)[V], float (&e)[V], float& top, float& inv) {
    float m = x[0];
#pragma unroll
    for (int v = 1; v < V; ++v) m = fmaxf(m, x[v]);
    m = route_max<L>(m);
    top = m == -RT_INF ? 0.0f : m;
    float s = 0.0f;
#pragma unroll
    for (int v = 0; v < V; ++v) {
        e[v] = __builtin_amdgcn_exp2f((x[v] - top) * RT_LOG2E);
        s += e[v];
    }
    s = route_sum<L>(s);
    inv = s == 0.0f ? 0.0f : 1.0f / s;
}

template <typename T, int L, int V>
__global__ __launch_bounds__(RT_THREADS) void route_kernel(RouteArgs a) {
    typedef RouteLane<L, V> At;
    constexpr int WAVES = RT_THREADS / 64, ROWS = 64 / L, KEEP = RT_MAX_TOP / L;
    __shared__ int cnt[GR_MAX_NETS + 1];
    __shared__ float sums[WAVES][L * V];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, l = lane % L, sub = lane / L;
    if (a.counts) {
        for (int e = tid; e <= a.K; e += RT_THREADS) cnt[e] = 0;
        __syncthreads();
    }
    float acc[V];
#pragma unroll
    for (int v = 0; v < V; ++v) acc[v] = 0.0f;
    const int64_t step = (int64_t)gridDim.x * WAVES * ROWS;
    // (all lanes of a wave run every step: what they exchange needs all of them)
    for (int64_t r0 = ((int64_t)blockIdx.x * WAVES + wave) * ROWS; r0 < a.n; r0 += step) {
        const bool in = r0 + sub < a.n;
        const int64_t r = in ? r0 + sub : a.n - 1;
        float x[V], e[V], top, inv;
        route_load<T, L, V>(x, (const T*)a.s + r * a.lds, a.K, l);
        route_softmax<L, V>(x, e, top, inv);
        const bool bad = inv != inv, has = inv > 0.0f;
        if (a.counts && in) {
#pragma unroll
            for (int v = 0; v < V; ++v) acc[v] += e[v] * inv;
            if (l == 0 && has) atomicAdd(&cnt[a.K], 1);
        }
        int id[KEEP];
        float ge[KEEP], chosen = 0.0f;
#pragma unroll
        for (int q = 0; q < KEEP; ++q) {
            id[q] = -1;
            ge[q] = 0.0f;
            for (int j = 0; j < L && q * L + j < a.k; ++j) {
                float best = x[0];
                int at = At::column(l, 0);
#pragma unroll
                for (int v = 1; v < V; ++v)
                    if (x[v] > best) {
                        best = x[v];
                        at = At::column(l, v);
                    }
                const float m = route_max<L>(best);
                const int c = route_min<L>(best == m ? at : INT32_MAX);
                if (m == -RT_INF || !has) continue;
#pragma unroll
                for (int v = 0; v < V; ++v)
                    if (At::column(l, v) == c) x[v] = -RT_INF;
                const float g = __builtin_amdgcn_exp2f((m - top) * RT_LOG2E);
                chosen += g;
                if (l == j) {
                    id[q] = c;
                    ge[q] = g;
                }
            }
        }
        if (in) {
            const float by = bad ? inv : a.normalize ? (chosen > 0.0f ? 1.0f / chosen : 0.0f) : inv;
#pragma unroll
            for (int q = 0; q < KEEP; ++q)
                if (q * L + l < a.k) {
                    a.ids[r * a.k + q * L + l] = id[q];
                    a.gates[r * a.k + q * L + l] = id[q] < 0 && !bad ? 0.0f : bad ? by : ge[q] * by;
                    if (a.counts && id[q] >= 0) atomicAdd(&cnt[id[q]], 1);
                }
        }
    }
    if (!a.counts) return;
    // the workgroup's sums: of the rows within a wave, then of the waves, in their order
#pragma unroll
    for (int v = 0; v < V; ++v) {
#pragma unroll
        for (int d = L; d < 64; d <<= 1) acc[v] += __shfl_xor(acc[v], d);
        if (sub == 0) sums[wave][At::column(l, v)] = acc[v];
    }
    __syncthreads();
    for (int e = tid; e < a.K; e += RT_THREADS) {
        float s = sums[0][e];
#pragma unroll
        for (int w = 1; w < WAVES; ++w) s += sums[w][e];
        a.part[(int64_t)blockIdx.x * a.K + e] = s;
    }
    for (int e = tid; e <= a.K; e += RT_THREADS) a.part_counts[(int64_t)blockIdx.x * (a.K + 1) + e] = cnt[e];
}

// counts and loss from the workgroups' sums, in their order
__global__ __launch_bounds__(1024) void route_join_kernel(RouteArgs a) {
    __shared__ float red[16];
    __shared__ int total[16], rows_of[1];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    float dot = 0.0f;
    int all = 0;
    for (int e = tid; e <= a.K; e += 1024) {
        int c = 0;
        float s = 0.0f;
        for (int b = 0; b < a.blocks; ++b) {
            c += a.part_counts[(int64_t)b * (a.K + 1) + e];
            if (e < a.K) s += a.part[(int64_t)b * a.K + e];
        }
        a.counts[e] = c;
        if (e == a.K) {
            rows_of[0] = c;
        } else {
            all += c;
            dot += (float)c * s;
        }
    }
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        dot += __shfl_xor(dot, d);
        all += __shfl_xor(all, d);
    }
    if (lane == 0) {
        red[wave] = dot;
        total[wave] = all;
    }
    __syncthreads();
    if (tid == 0) {
        for (int w = 1; w < 16; ++w) {
            dot += red[w];
            all += total[w];
        }
        const int rows = rows_of[0];
        // (without a row to count the loss is 0, or NaN where a row held one)
        a.loss[0] = dot * ((float)a.K / ((float)(all > 0 ? all : 1) * (float)(rows > 0 ? rows : 1)));
    }
}

template <typename T, int L, int V>
__global__ __launch_bounds__(256) void route_grad_kernel(RouteArgs a) {
    typedef RouteLane<L, V> At;
    constexpr int WAVES = 4, ROWS = 64 / L, KEEP = RT_MAX_TOP / L;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, l = lane % L, sub = lane / L;
    float w[V];  // a_e
#pragma unroll
    for (int v = 0; v < V; ++v) w[v] = 0.0f;
    if (a.dloss) {
        int all = 0;
        for (int e = lane; e < a.K; e += 64) all += a.counts[e];
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) all += __shfl_xor(all, d);
        const int rows = a.counts[a.K];
        const float by = a.dloss[0] * ((float)a.K / ((float)(all > 0 ? all : 1) * (float)(rows > 0 ? rows : 1)));
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int c = At::column(l, v);
            w[v] = c < a.K ? by * (float)a.counts[c] : 0.0f;
        }
    }
    const int64_t step = (int64_t)gridDim.x * WAVES * ROWS;
    for (int64_t r0 = ((int64_t)blockIdx.x * WAVES + wave) * ROWS; r0 < a.n; r0 += step) {
        const bool in = r0 + sub < a.n;
        const int64_t r = in ? r0 + sub : a.n - 1;
        float x[V], p[V], top, inv;
        route_load<T, L, V>(x, (const T*)a.s + r * a.lds, a.K, l);
        route_softmax<L, V>(x, p, top, inv);
        float dot = 0.0f;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            p[v] *= inv;
            dot += p[v] * w[v];
        }
        dot = route_sum<L>(dot);
        int id[KEEP];
        float gate[KEEP], dg[KEEP], chosen = 0.0f, mix = 0.0f;
        if (a.dgates) {
#pragma unroll
            for (int q = 0; q < KEEP; ++q) {
                id[q] = -1;
                gate[q] = dg[q] = 0.0f;
                if (q * L + l < a.k) {
                    const int i = a.ids[r * a.k + q * L + l];
                    if ((unsigned)i < (unsigned)a.K) {
                        id[q] = i;
                        gate[q] = __builtin_amdgcn_exp2f((to_f<T>(((const T*)a.s)[r * a.lds + i]) - top) * RT_LOG2E);
                        dg[q] = a.dgates[r * a.k + q * L + l];
                        chosen += gate[q];
                    }
                }
            }
            chosen = a.normalize ? route_sum<L>(chosen) : 0.0f;
            const float by = a.normalize ? (chosen != 0.0f ? 1.0f / chosen : 0.0f) : inv;
#pragma unroll
            for (int q = 0; q < KEEP; ++q) {
                gate[q] *= by;
                if (id[q] >= 0) mix += gate[q] * dg[q];
            }
            mix = route_sum<L>(mix);
        }
        const float off = a.normalize ? dot : dot + mix;
        float d[V];
#pragma unroll
        for (int v = 0; v < V; ++v) d[v] = p[v] * (w[v] - off);
        if (a.dgates) {
#pragma unroll
            for (int q = 0; q < KEEP; ++q) {
                const float mine = gate[q] * (a.normalize ? dg[q] - mix : dg[q]);
                for (int j = 0; j < L && q * L + j < a.k; ++j) {
                    const int at = __shfl(id[q], sub * L + j);
                    const float more = __shfl(mine, sub * L + j);
#pragma unroll
                    for (int v = 0; v < V; ++v)
                        if (At::column(l, v) == at) d[v] += more;
                }
            }
        }
        if (!in) continue;
        T* out = (T*)a.ds + r * a.ldds;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int c = At::column(l, v);
            if (c < a.K) out[c] = from_f<T>(d[v]);
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

// eight neighbouring values a thread; a dropped pair's rows are not read
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

template <typename T, typename TG>
__global__ __launch_bounds__(256) void combine_grad_kernel(CombineArgs a) {
    __shared__ float red[4];
    const int rows = 256 / a.threads, tx = threadIdx.x % a.threads, ty = threadIdx.x / a.threads;
    for (int64_t r0 = (int64_t)blockIdx.x * rows; r0 < a.n; r0 += (int64_t)gridDim.x * rows) {
        const bool in = r0 + ty < a.n;
        const int64_t r = in ? r0 + ty : a.n - 1;
        for (int j = 0; j < a.per_row; ++j) {
            const int64_t p = r * a.per_row + j;
            const bool kept = (unsigned)a.ids[p] < (unsigned)a.K;
            const float w = kept ? a.w[p] : 0.0f;
            float dot = 0.0f;
            for (int m = tx * 8; m < a.M && in; m += a.threads * 8) {
                const int left = a.M - m;
                float g[8], v[8];
                if (kept) {
                    load8_f<TG>(g, (const TG*)a.g + r * a.ldg + m, left);
                    load8_f<T>(v, (const T*)a.y + p * a.ldy + m, left);
                }
#pragma unroll
                for (int q = 0; q < 8; ++q) {
                    if (kept) dot = __builtin_fmaf(g[q], v[q], dot);
                    v[q] = kept ? w * g[q] : 0.0f;
                }
                store8((T*)a.dy + p * a.lddy + m, v, left);
            }
            for (int d = 1; d < a.threads && d < 64; d <<= 1) dot += __shfl_xor(dot, d);
            if (a.threads > 64) {
                __syncthreads();
                if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = dot;
                __syncthreads();
                dot = red[ty * (a.threads / 64)];
                for (int q = 1; q < a.threads / 64; ++q) dot += red[ty * (a.threads / 64) + q];
            }
            if (in && tx == 0) a.dw[p] = dot;
        }
    }
}

}  // namespace pnn
