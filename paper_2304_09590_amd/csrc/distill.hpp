// distill.hpp -- the loss of a network's logits against a teacher's top logits, and its gradient.
//
// Row r of the student has V logits z; its teacher gives k entries (class i_j, logit t_j), entries
// whose class lies outside [0, V) are padding.  With p = softmax(t / T) over the row's entries,
// q = softmax(z / T) and s = softmax(z) over all classes, and a label y (none if outside [0, V)):
//   loss = (1 - alpha) T^2 sum_j p_j (log p_j - log q_{i_j}) - alpha log s_y
//   dz_v = g [ (1 - alpha) T (q_v - sum_{j: i_j = v} p_j) + alpha (s_v - [v = y]) ]
// Both passes stream z: one running maximum and one or two running sums of exponentials forward,
// which the gradient then only has to divide by.  The maximum is subtracted before anything is
// scaled, and log q is formed as (z - m) / T - log sum, so logits near the type's ends lose nothing.
// Bound by the bytes of z (read twice) and dz; statistics and sums are fp32.  4,096 rows of 32,000 classes in bf16
// with 64 entries: the loss 287 MB of memory traffic in 49 us, the gradient 555 MB in 113.  60,000 rows of 10
// classes: 7.2 and 6.3 us, latency.  5 rows of 131,071 classes in fp32: parts 4.4 us, their join 3.7.
#pragma once
#include "groups.hpp"

namespace pnn {

constexpr int DL_MAX_TOP = 1024;  // most entries of a row (they are staged in LDS)
constexpr int DL_WAVE_TOP = 64;   // most entries of a row that one wave takes
constexpr int DL_TINY_TOP = 16, DL_TINY = 128;  // most entries and classes of a row that 16 lanes take

struct DistillArgs {
    const void* z;
    int64_t ldz, n;
    int64_t row0;             // first row of the launch
    int V, k;
    const int32_t* idx;
    const void* t;
    const int32_t* y;         // nullable
    float ct, cs;             // log2(e) / T, and of the one sum or of the second: log2(e)
    float inv_t, wt, ws;      // 1 / T; weights of the two losses
    float gt, gs;             // weights of the two gradients: (1 - alpha) T, alpha
    int rows_per;             // rows that share entries and a label: those of row / rows_per
    const int32_t* ids;       // (nullable) a row whose id lies outside [0, K) has neither
    int K;
    int S, part;              // parts of a row and classes of a part
    float4* stats;            // [n] maximum, reciprocals of the sums at T and at 1, what the row has
    float4* parts;            // [n][S] maximum, sums
    float* loss;
    const float* g;
    void* dz;
    int64_t lddz;
    bool stream = false;      // dz passes the caches by
};

// the row whose entries and label row r has (most calls: its own; a 64-bit division is long)
__device__ inline int64_t dl_shared(const DistillArgs& d, int64_t row) { return d.rows_per == 1 ? row : (int64_t)((uint32_t)row / (uint32_t)d.rows_per); }

constexpr float DL_INF = __builtin_huge_valf();

// Running maximum m and sums of exp2(z c - m c), at the scales c = ct and cs.  MODE 1: one sum; 2: two; 3: two
// whose second scale is twice the first (T = 2), so that its terms are the first's squares.  m c is rounded once
// and the same wherever it is used (Ref), so its rounding shifts all terms alike and cancels, as long as the shift
// is small: below 2^20 it is at most 2^-5.  From there on (`huge`) differences are taken before they are scaled,
// and nothing is shifted: the shift grows with m c, and at 2^31 the exponentials would leave fp32's range.
struct Sums { float m, a, b; };
constexpr float DL_FAR = 1048576.0f;
struct Ref {
    float t, s;
    bool huge;
};

__device__ inline Ref dl_ref(float m, const DistillArgs& d) {
    const float r = m == -DL_INF ? 0.0f : m;  // (no value yet, or only ones of -inf: their terms are 0)
    Ref f = {r * d.ct, r * d.cs, false};
    f.huge = !(__builtin_fabsf(f.t) < DL_FAR && __builtin_fabsf(f.s) < DL_FAR);
    if (f.huge) f.t = f.s = r;
    return f;
}
// what the terms' exponents at maximum m and scale c exceed (z - m) c by (exact: the rounding of m c)
__device__ inline float dl_shift(float m, float c, float ref, bool huge) { return huge ? 0.0f : __builtin_fmaf(m, c, -ref); }
// exponents (to base 2) of a logit
__device__ inline float dl_t(float z, const Ref& f, const DistillArgs& d) {
    return f.huge ? (z - f.t) * d.ct : __builtin_fmaf(z, d.ct, -f.t);
}
__device__ inline float dl_s(float z, const Ref& f, const DistillArgs& d) {
    return f.huge ? (z - f.s) * d.cs : __builtin_fmaf(z, d.cs, -f.s);
}

// moves the sums to a larger maximum
template <int MODE>
__device__ inline void dl_move(Sums& s, float m, const DistillArgs& d) {
    const Ref f = dl_ref(m, d), old = dl_ref(s.m, d);
    const bool none = s.m == -DL_INF;  // (the sums are 0, or NaN, and stay so)
    float by = old.t - f.t, bs = old.s - f.s;
    if (f.huge || old.huge) {  // (a maximum on either side of the switch: the shifts do not cancel)
        by = (s.m - m) * d.ct + (dl_shift(m, d.ct, f.t, f.huge) - dl_shift(s.m, d.ct, old.t, old.huge));
        bs = (s.m - m) * d.cs + (dl_shift(m, d.cs, f.s, f.huge) - dl_shift(s.m, d.cs, old.s, old.huge));
    }
    s.a *= none ? 0.0f : __builtin_amdgcn_exp2f(by);
    if (MODE != 1) s.b *= none ? 0.0f : __builtin_amdgcn_exp2f(bs);
    s.m = m;
}

template <int MODE, int N>
__device__ inline void dl_add(Sums& s, const float (&z)[N], const DistillArgs& d) {
    float m = z[0];
#pragma unroll
    for (int i = 1; i < N; ++i) m = fmaxf(m, z[i]);
    if (m > s.m) dl_move<MODE>(s, m, d);
    const Ref f = dl_ref(s.m, d);
    if (f.huge) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            s.a += __builtin_amdgcn_exp2f((z[i] - f.t) * d.ct);
            if (MODE != 1) s.b += __builtin_amdgcn_exp2f((z[i] - f.s) * d.cs);
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const float e = __builtin_amdgcn_exp2f(__builtin_fmaf(z[i], d.ct, -f.t));
        s.a += e;
        if (MODE == 2) s.b += __builtin_amdgcn_exp2f(__builtin_fmaf(z[i], d.cs, -f.s));
        if (MODE == 3) s.b = __builtin_fmaf(e, e, s.b);
    }
}

template <int MODE>
__device__ inline void dl_join(Sums& s, float m, float a, float b, const DistillArgs& d) {
    Sums o = {m, a, b};
    const float top = fmaxf(s.m, m);
    if (top > s.m) dl_move<MODE>(s, top, d);
    if (top > o.m) dl_move<MODE>(o, top, d);
    s.a += o.a;
    if (MODE != 1) s.b += o.b;
}

// over G = 16 or 64 lanes: by DPP within the rows of 16, the four rows by two exchanges
template <int G> __device__ inline float dl_max(float v) {
    v = row_allmax16(v);
    if (G == 64) {
        v = fmaxf(v, __shfl_xor(v, 16));
        v = fmaxf(v, __shfl_xor(v, 32));
    }
    return v;
}
template <int G> __device__ inline float dl_sum(float v) {
    v = row_allsum16(v);
    if (G == 64) {
        v += __shfl_xor(v, 16);
        v += __shfl_xor(v, 32);
    }
    return v;
}

template <int MODE, int G>
__device__ inline void dl_join_lanes(Sums& s, const DistillArgs& d) {
    const float m = dl_max<G>(s.m);
    if (m > s.m) dl_move<MODE>(s, m, d);
    s.a = dl_sum<G>(s.a);
    if (MODE != 1) s.b = dl_sum<G>(s.b);
}

// The teacher's distribution of a row, as a wave sees it: maximum and sum of the entries' exponentials, and
// the lane's first entry with the student's logit there.  A sum of 0: no entries, or only ones of -inf.
template <typename T>
struct Teacher {
    float ref = 0.0f, mass = 0.0f, t, z;
    int i = -1;
    const int32_t* idx;
    const T *ts, *zs;

    __device__ inline void load(const DistillArgs& d, int64_t row, int lane, bool logits) {
        idx = d.idx + dl_shared(d, row) * d.k;
        ts = (const T*)d.t + dl_shared(d, row) * d.k;
        zs = (const T*)d.z + row * d.ldz;
        if (d.wt == 0.0f) return;
        if (lane < d.k) {
            i = idx[lane];
            t = to_f<T>(ts[lane]);
            if ((unsigned)i >= (unsigned)d.V) i = -1;
            if (logits && i >= 0) z = to_f<T>(zs[i]);
        }
    }
    __device__ inline bool entry(const DistillArgs& d, int j, int& at, float& value) const {
        at = idx[j];
        value = to_f<T>(ts[j]);
        return (unsigned)at < (unsigned)d.V;
    }
    __device__ inline void sum(const DistillArgs& d, int lane) {
        if (d.wt == 0.0f) return;
        float m = i >= 0 ? t : -DL_INF, v;
        int at;
        for (int j = lane + 64; j < d.k; j += 64)
            if (entry(d, j, at, v)) m = fmaxf(m, v);
        m = dl_max<64>(m);
        ref = m == -DL_INF ? 0.0f : m;
        float s = i >= 0 ? exp2f((t - ref) * d.ct) : 0.0f;
        for (int j = lane + 64; j < d.k; j += 64)
            if (entry(d, j, at, v)) s += exp2f((v - ref) * d.ct);
        mass = dl_sum<64>(s);
    }
};

constexpr float DL_LN2 = 0.6931471806f;

// loss and statistics of a row from its sums, by a wave
template <typename T>
__device__ inline void dl_finish(const DistillArgs& d, int64_t row, int lane, const Teacher<T>& te, int has, const Sums& s, bool two) {
    const float la = logf(s.a), lb = two ? logf(s.b) : la;
    const Ref f = dl_ref(s.m, d);
    float kl = 0.0f;
    if (has & 1) {
        const float lm = logf(te.mass), im = 1.0f / te.mass;
        auto term = [&](float t, float z) {
            const float e = t - te.ref, p = exp2f(e * d.ct) * im;
            // (an entry without weight counts nothing, whatever the student gives it)
            return p == 0.0f ? 0.0f : p * ((e * d.inv_t - lm) - (dl_t(z, f, d) * DL_LN2 - la));
        };
        if (te.i >= 0) kl = term(te.t, te.z);
        float t;
        int at;
        for (int j = lane + 64; j < d.k; j += 64)
            if (te.entry(d, j, at, t)) kl += term(t, to_f<T>(te.zs[at]));
    }
    kl = dl_sum<64>(kl);
    if (lane != 0) return;
    float loss = 0.0f;
    if (s.a == 0.0f) has = 0;  // every logit is -inf: nothing to learn from
    if (has & 1) loss += d.wt * kl;
    if (has & 2) loss += d.ws * (lb - dl_s(to_f<T>(te.zs[d.y[dl_shared(d, row)]]), f, d) * DL_LN2);
    d.loss[row] = loss;
    d.stats[row] = make_float4(s.m, 1.0f / s.a, 1.0f / (two ? s.b : s.a), (float)has);
}

__device__ inline int dl_label(const DistillArgs& d, int64_t row) {
    if (!d.y) return -1;
    const int y = d.y[dl_shared(d, row)];
    return (unsigned)y < (unsigned)d.V ? y : -1;
}

// what a row learns from (bit 0 entries, bit 1 a label)
__device__ inline int dl_has(const DistillArgs& d, int64_t row, float mass) {
    if (d.ids && (unsigned)d.ids[row] >= (unsigned)d.K) return 0;
    return (mass == 0.0f ? 0 : 1) | (dl_label(d, row) >= 0 ? 2 : 0);
}

// dz of one value
__device__ inline float dl_grad(const DistillArgs& d, float z, const Ref& f, float ea, float eb, float gt, float gs, float g,
                                float psum, bool label) {
    const float q = __builtin_amdgcn_exp2f(dl_t(z, f, d)) * ea;
    const float s = __builtin_amdgcn_exp2f(dl_s(z, f, d)) * eb;
    return g * (gt * (q - psum) + gs * (s - (label ? 1.0f : 0.0f)));
}

// dz of values that are neither an entry's nor the label: ka, kb = g gt ea, g gs eb
template <int MODE>
__device__ inline void dl_grad8(const DistillArgs& d, float (&x)[8], const Ref& f, float ka, float kb) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float e = __builtin_amdgcn_exp2f(f.huge ? (x[i] - f.t) * d.ct : __builtin_fmaf(x[i], d.ct, -f.t));
        if (MODE == 1) x[i] = e * (ka + kb);
        if (MODE == 2) x[i] = __builtin_fmaf(kb, __builtin_amdgcn_exp2f(dl_s(x[i], f, d)), ka * e);
        if (MODE == 3) x[i] = e * __builtin_fmaf(kb, e, ka);
    }
}

// Loss, W waves a row (256 / (64 W) rows a workgroup), or one part of a row per workgroup (S > 1).
template <typename T, int MODE, int W>
__global__ __launch_bounds__(256) void distill_loss_kernel(DistillArgs d) {
    __shared__ Sums across[4];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int64_t row = d.row0 + (W == 4 ? blockIdx.x / (uint32_t)d.S : (int64_t)blockIdx.x * 4 + wave);
    const int part = W == 4 ? (int)(blockIdx.x % (uint32_t)d.S) : 0;
    if (row >= d.n) return;
    const int in = W == 4 ? tid : lane;
    const T* z = (const T*)d.z + row * d.ldz;
    const int64_t lo = (int64_t)part * d.part;
    const int len = (int)(d.V - lo < d.part ? d.V - lo : d.part);
    Teacher<T> te;
    int has = 3;
    if (W != 4 || d.S == 1) {  // (the parts of a row are summed whatever it has)
        te.load(d, row, lane, true);
        te.sum(d, lane);
        has = dl_has(d, row, te.mass);
        if (has == 0) {  // a padding row: its logits do not matter
            if (in == 0) {
                d.loss[row] = 0.0f;
                d.stats[row] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
            }
            return;
        }
    }
    Sums s = {-DL_INF, 0.0f, 0.0f};
    // sixteen values at a time, the next ones in flight; then what is left, eight at a time
    constexpr int LEAP = W * 512;
    int v = in * 8;
    const int pairs = len - v - 8 - LEAP >= 0 ? (len - v - 8 - LEAP) / (2 * LEAP) + 1 : 0;
    Raw8<T> r0, r1;
    if (pairs > 0) {
        load8(r0, z + lo + v, 8);
        load8(r1, z + lo + v + LEAP, 8);
    }
    for (int it = 0; it < pairs; ++it, v += 2 * LEAP) {
        float x[16];
        raw8_f(*(float(*)[8])x, r0);
        raw8_f(*(float(*)[8])(x + 8), r1);
        if (it + 1 < pairs) {
            load8(r0, z + lo + v + 2 * LEAP, 8);
            load8(r1, z + lo + v + 3 * LEAP, 8);
        }
        dl_add<MODE>(s, x, d);
    }
    for (; v < len; v += LEAP) {
        float x[8];
        load8_f<T>(x, z + lo + v, len - v);
        if (len - v < 8) {
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = i < len - v ? x[i] : -DL_INF;
        }
        dl_add<MODE>(s, x, d);
    }
    dl_join_lanes<MODE, 64>(s, d);
    if (W == 4) {
        if (lane == 0) across[wave] = s;
        __syncthreads();
        if (wave != 0) return;
#pragma unroll
        for (int w = 1; w < 4; ++w) dl_join<MODE>(s, across[w].m, across[w].a, across[w].b, d);
        if (d.S > 1) {
            if (lane == 0) d.parts[row * d.S + part] = make_float4(s.m, s.a, s.b, 0.0f);
            return;
        }
    }
    dl_finish<T>(d, row, lane, te, has, s, MODE != 1);
}

// joins the parts of a row, one wave a row
template <typename T, int MODE>
__global__ __launch_bounds__(64) void distill_join_kernel(DistillArgs d) {
    const int64_t row = d.row0 + blockIdx.x;
    const int lane = threadIdx.x;
    Teacher<T> te;
    te.load(d, row, lane, true);
    Sums s = {-DL_INF, 0.0f, 0.0f};
    for (int p = lane; p < d.S; p += 64) {
        const float4 v = d.parts[row * d.S + p];
        dl_join<MODE>(s, v.x, v.y, v.z, d);
    }
    te.sum(d, lane);
    const int has = dl_has(d, row, te.mass);
    if (has == 0) {  // a padding row, whatever its logits
        if (lane == 0) {
            d.loss[row] = 0.0f;
            d.stats[row] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        }
        return;
    }
    dl_join_lanes<MODE, 64>(s, d);
    dl_finish<T>(d, row, lane, te, has, s, MODE != 1);
}

// Gradient, W waves a row or one part of a row per workgroup.  The entries' classes (and the label)
// are written again after the stream has passed, from logits read before it: so dz may be z.  Each entry is
// compared with all others of its row for repeated classes, which is quadratic in the entries: 4,096 rows of
// 32,000 classes in bf16 with 64, 128, 256, 512 and 1,024 entries 113, 122, 151, 267 and 703 us.
template <typename T, int MODE, int W>
__global__ __launch_bounds__(256) void distill_grad_kernel(DistillArgs d) {
    constexpr int TOP = W == 4 ? DL_MAX_TOP : DL_WAVE_TOP;
    __shared__ int sidx[4 / W][TOP];
    __shared__ float sp[4 / W][TOP], sz[4 / W][TOP + 1];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int64_t row = d.row0 + (W == 4 ? blockIdx.x / (uint32_t)d.S : (int64_t)blockIdx.x * 4 + wave);
    const int part = W == 4 ? (int)(blockIdx.x % (uint32_t)d.S) : 0, slot = W == 4 ? 0 : wave;
    if (row >= d.n) return;
    const int in = W == 4 ? tid : lane;
    const T* z = (const T*)d.z + row * d.ldz;
    T* dz = (T*)d.dz + row * d.lddz;
    const int lo = part * d.part, hi = d.V - lo < d.part ? d.V : lo + d.part;
    const float4 st = d.stats[row];
    const float g = d.g ? d.g[row] : 1.0f;
    const int has = g == 0.0f ? 0 : (int)st.w;
    if (has == 0) {
        const float none[8] = {0, 0, 0, 0, 0, 0, 0, 0};
        for (int v = lo + in * 8; v < hi; v += W * 512) store8(dz + v, none, hi - v);
        return;
    }
    auto meet = [] {
        if (W == 4) __syncthreads();
        else __threadfence_block();
    };
    const float gt = has & 1 ? d.gt : 0.0f, gs = has & 2 ? d.gs : 0.0f;
    const float ea = has & 1 ? st.y : 0.0f, eb = has & 2 ? st.z : 0.0f;
    const int label = has & 2 ? dl_label(d, row) : -1;
    const int k = has & 1 ? d.k : 0;
    if (has & 1) {
        Teacher<T> te;
        te.load(d, row, lane, false);
        te.sum(d, lane);
        const float im = 1.0f / te.mass;
        for (int j = in; j < k; j += 64 * W) {
            float t;
            int i;
            te.entry(d, j, i, t);
            const bool mine = i >= lo && i < hi;
            sidx[slot][j] = mine ? i : -1;
            sp[slot][j] = mine ? exp2f((t - te.ref) * d.ct) * im : 0.0f;
            sz[slot][j] = mine ? to_f<T>(z[i]) : 0.0f;
        }
    }
    const bool own_label = label >= lo && label < hi;
    if (in == 0) sz[slot][TOP] = own_label ? to_f<T>(z[label]) : 0.0f;
    const Ref f = dl_ref(st.x, d);
    const float ka = g * gt * ea, kb = g * gs * eb;
    int v = lo + in * 8;
    Raw8<T> r[2];  // (loads two steps ahead; a value is read before the one at its place is written)
    load8(r[0], z + v, hi - v);
    load8(r[1], z + v + W * 512, hi - v - W * 512);
    meet();
    for (; v < hi; v += W * 512) {
        float x[8];
        raw8_f(x, r[0]);
        r[0] = r[1];
        load8(r[1], z + v + W * 1024, hi - v - W * 1024);
        dl_grad8<MODE>(d, x, f, ka, kb);
        if (d.stream) store8<true>(dz + v, x, hi - v);
        else store8(dz + v, x, hi - v);
    }
    meet();  // (waits for the stores: those below come after them)
    for (int j = in; j < k; j += 64 * W) {
        const int i = sidx[slot][j];
        if (i < 0) continue;
        float p = 0.0f;
        bool first = true;
        for (int o = 0; o < k; ++o)
            if (sidx[slot][o] == i) {
                p += sp[slot][o];
                if (o < j) first = false;
            }
        if (first) dz[i] = from_f<T>(dl_grad(d, sz[slot][j], f, ea, eb, gt, gs, g, p, i == label));
    }
    if (in == 0 && own_label) {
        bool listed = false;
        for (int o = 0; o < k; ++o) listed |= sidx[slot][o] == label;
        if (!listed) dz[label] = from_f<T>(dl_grad(d, sz[slot][TOP], f, ea, eb, gt, gs, g, 0.0f, true));
    }
}

// Few classes: 16 lanes a row, NZ values of z and one entry a lane in registers.
template <typename T, int NZ>
struct Tiny {
    float z[NZ], t, ref, mass;
    int i, label;

    __device__ inline float logit(int v) const {  // of class v, by all lanes of the row
        float r = 0.0f;
#pragma unroll
        for (int k = 0; k < NZ; ++k) {
            const float o = __shfl(z[k], v & 15, 16);
            if (v >> 4 == k) r = o;
        }
        return r;
    }
    __device__ inline void load(const DistillArgs& d, int64_t row, int lane) {
        const T* p = (const T*)d.z + row * d.ldz;
        const int64_t base = dl_shared(d, row);
        i = -1;
        t = -DL_INF;
        if (d.wt != 0.0f && lane < d.k) {
            i = d.idx[base * d.k + lane];
            t = to_f<T>(((const T*)d.t)[base * d.k + lane]);
        }
        label = d.y ? d.y[base] : -1;
#pragma unroll
        for (int k = 0; k < NZ; ++k) z[k] = lane + 16 * k < d.V ? to_f<T>(p[lane + 16 * k]) : -DL_INF;
        if ((unsigned)i >= (unsigned)d.V) {
            i = -1;
            t = -DL_INF;
        }
        if ((unsigned)label >= (unsigned)d.V) label = -1;
        const float m = dl_max<16>(t);
        ref = m == -DL_INF ? 0.0f : m;
        mass = dl_sum<16>(i >= 0 ? exp2f((t - ref) * d.ct) : 0.0f);
    }
};

template <typename T, int MODE, int NZ>
__global__ __launch_bounds__(256) void distill_loss_tiny_kernel(DistillArgs d) {
    const int lane = threadIdx.x & 15;
    const int64_t row = d.row0 + (int64_t)blockIdx.x * 16 + (threadIdx.x >> 4);
    if (row >= d.n) return;
    Tiny<T, NZ> r;
    r.load(d, row, lane);
    int has = (r.mass == 0.0f ? 0 : 1) | (r.label >= 0 ? 2 : 0);
    if (d.ids && (unsigned)d.ids[row] >= (unsigned)d.K) has = 0;
    float top = r.z[0];
#pragma unroll
    for (int k = 1; k < NZ; ++k) top = fmaxf(top, r.z[k]);
    Sums s = {dl_max<16>(top), 0.0f, 0.0f};
    dl_add<MODE>(s, r.z, d);
    s.a = dl_sum<16>(s.a);
    if (MODE != 1) s.b = dl_sum<16>(s.b);
    const Ref f = dl_ref(s.m, d);
    const float la = logf(s.a), lb = MODE != 1 ? logf(s.b) : la;
    const int at = r.i >= 0 ? r.i : 0;
    float zi = 0.0f;
#pragma unroll
    for (int k = 0; k < NZ; ++k) {
        const float o = __shfl(r.z[k], at & 15, 16);
        if (at >> 4 == k) zi = o;
    }
    const float zy = r.logit(r.label >= 0 ? r.label : 0);
    float kl = 0.0f;
    if (r.i >= 0) {
        const float e = r.t - r.ref, p = exp2f(e * d.ct) / r.mass;
        if (p != 0.0f) kl = p * ((e * d.inv_t - logf(r.mass)) - (dl_t(zi, f, d) * DL_LN2 - la));
    }
    kl = dl_sum<16>(kl);
    if (lane != 0) return;
    if (s.a == 0.0f) has = 0;  // every logit is -inf
    float loss = 0.0f;
    if (has & 1) loss += d.wt * kl;
    if (has & 2) loss += d.ws * (lb - dl_s(zy, f, d) * DL_LN2);
    d.loss[row] = loss;
    d.stats[row] = make_float4(s.m, 1.0f / s.a, 1.0f / (MODE != 1 ? s.b : s.a), (float)has);
}

template <typename T, int NZ>
__global__ __launch_bounds__(256) void distill_grad_tiny_kernel(DistillArgs d) {
    const int lane = threadIdx.x & 15;
    const int64_t row = d.row0 + (int64_t)blockIdx.x * 16 + (threadIdx.x >> 4);
    if (row >= d.n) return;
    T* dz = (T*)d.dz + row * d.lddz;
    const float4 st = d.stats[row];
    const float g = d.g ? d.g[row] : 1.0f;
    Tiny<T, NZ> r;
    r.load(d, row, lane);
    const int has = g == 0.0f ? 0 : (int)st.w;
    const float gt = has & 1 ? d.gt : 0.0f, gs = has & 2 ? d.gs : 0.0f;
    const float ea = has & 1 ? st.y : 0.0f, eb = has & 2 ? st.z : 0.0f;
    const int label = has & 2 ? r.label : -1;
    const Ref f = dl_ref(st.x, d);
    const float p = r.i >= 0 && has & 1 ? exp2f((r.t - r.ref) * d.ct) / r.mass : 0.0f;
    float sum[NZ];
#pragma unroll
    for (int k = 0; k < NZ; ++k) sum[k] = 0.0f;
    const int top = has & 1 ? d.k : 0;
    for (int j = 0; j < top; ++j) {
        const int ij = __shfl(r.i, j, 16);
        const float pj = __shfl(p, j, 16);
#pragma unroll
        for (int k = 0; k < NZ; ++k)
            if (ij == lane + 16 * k) sum[k] += pj;
    }
#pragma unroll
    for (int k = 0; k < NZ; ++k) {
        const int v = lane + 16 * k;
        if (v < d.V) dz[v] = from_f<T>(has == 0 ? 0.0f : dl_grad(d, r.z[k], f, ea, eb, gt, gs, g, sum[k], v == label));
    }
}

}  // namespace pnn
