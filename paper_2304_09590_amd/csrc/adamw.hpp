// adamw.hpp -- a step of AdamW over many tensors: with gradient g and step number t,
//
//   m <- beta1 m + (1 - beta1) g,  v <- beta2 v + (1 - beta2) g^2
//   p <- p (1 - lr decay) - lr / (1 - beta1^t) m / (sqrt(v / (1 - beta2^t)) + eps)
//
// Moments are held in fp32, or in 8 bits a value with a scale for each 256 of a tensor: the largest size among them.
// A code stands for scale 2^((c - top) / 8), eight levels an octave (9 % apart) from the scale down, 0 for 0: of m a
// sign and 127 levels (16 octaves), of v 255 (32).  The step itself takes the moments before they are rounded.
//
// Rounding goes to one of the two levels about a value at random, in proportion, so that it is right in the mean.
// To the nearest, v would stand still: beta2 = 0.999 moves it by 0.1 % a step, and only g^2 above 45 v by half a level.
// What lies below v's lowest level becomes that level, never 0: a step divides by it.  The random bits are a
// function of the seed, the step, the tensor, the block and the place, so the same call gives the same bits.
//
// Bound by bytes: with fp32 gradients 28 a value, or 16 and the scales in 8 bits, 2 more for a copy.  34.3 million values
// with copies: 193 us in 32 bits (5.3 TB/s), 120 to 141 us in 8 (5.2 to 4.4 TB/s: cards differ, and a pass among others takes
// less than one under the profiler), where instructions take 0.83 of the cycles.  What brought the latter there from 251 us: levels from LDS instead of their formula and codes without branches
// (187 -> 160), global addresses with scalar bases instead of flat ones (160 -> 118, at gradients alike; 138 at unlike
// ones), whole chunks without looking for ends (138 -> 125), and the places below (58 ns for each of 1,024 workgroups).
#pragma once
#include <stddef.h>

#include "groups.hpp"

namespace pnn {

constexpr int AD_BLOCK = 256;        // values of a scale
constexpr int AD_CHUNK = 4096;       // values that a workgroup takes at a time: four blocks a wave
constexpr int AD_TENSORS = 48;       // of a launch that lays out a plan (they are its arguments, at most 4 KB)

// Workgroups that end count themselves in AD_GROUPS places, a line of memory each, and the last one of a place in
// steps[1]: additions to one place take 58 ns each, one after another (34 million values in 32 bits, one place for 1,024
// workgroups 212 us, for 2,048 269, for 8,375 538).
constexpr int AD_GROUPS = 32;

// A plan is these places (zeros between calls) and the chunks of all tensors, so that a workgroup finds what it works on
// in one load.
constexpr int AD_HEAD = AD_GROUPS * 64;  // bytes
struct AdamChunk {
    float* p;
    const void* g;
    void *m, *v;
    float *sm, *sv;
    bf16_t* copy;
    int n;                           // values
    uint32_t block;                  // number of its first block in the tensor
    uint32_t tensor;                 // place of the tensor in the call
    uint32_t kind;                   // of the states and gradients that the plan was laid out for
};
constexpr uint32_t ad_kind(size_t state_size, size_t g_size) { return (uint32_t)(state_size << 8 | g_size); }

struct AdamTensor {
    float* p;
    const void* g;
    void *m, *v;
    float *sm, *sv;
    bf16_t* copy;
    int64_t n;
};
struct AdamPlanArgs {
    AdamTensor t[AD_TENSORS];
    uint32_t first[AD_TENSORS + 1];  // first chunk of each tensor in `plan`
    int count, number;               // tensors, and the place of the first in the call
    int state_size, g_size;          // bytes of a moment and of a gradient
    uint32_t* places;                // (nullable) set to zero
    AdamChunk* plan;
};

__global__ __launch_bounds__(256) void adamw_plan_kernel(AdamPlanArgs a) {
    if (a.places && blockIdx.x == 0)
        for (int i = threadIdx.x; i < AD_HEAD / 4; i += 256) a.places[i] = 0;
    const uint32_t chunks = a.first[a.count];
    for (uint32_t c = blockIdx.x * 256 + threadIdx.x; c < chunks; c += gridDim.x * 256) {
        int i = 0, end = a.count;  // the last tensor whose first chunk is at most c
        while (end - i > 1) {
            const int mid = (i + end) >> 1;
            if (a.first[mid] <= c) i = mid;
            else end = mid;
        }
        const AdamTensor& t = a.t[i];
        const int64_t at = (int64_t)(c - a.first[i]) * AD_CHUNK, block = at / AD_BLOCK;
        AdamChunk x;
        x.p = t.p + at;
        x.g = (const char*)t.g + at * a.g_size;
        x.m = (char*)t.m + at * a.state_size;
        x.v = (char*)t.v + at * a.state_size;
        x.sm = t.sm ? t.sm + block : nullptr;
        x.sv = t.sv ? t.sv + block : nullptr;
        x.copy = t.copy ? t.copy + at : nullptr;
        x.n = t.n - at < AD_CHUNK ? (int)(t.n - at) : AD_CHUNK;
        x.block = (uint32_t)block;
        x.tensor = (uint32_t)(a.number + i);
        x.kind = ad_kind(a.state_size, a.g_size);
        a.plan[c] = x;
    }
}

struct AdamArgs {
    const AdamChunk* plan;
    uint32_t* places;
    uint32_t chunks;
    float b1, c1, b2, c2;            // beta, 1 - beta
    float ln1, ln2;                  // log beta
    float lr, eps, decay;
    const float* lr_dev;             // (nullable) instead of lr
    uint32_t seed;
    int32_t* steps;                  // steps done; workgroups that are done with the call
};

// 32 bits that look random, from 32 (multiplications by odd parts of sqrt 2 and sqrt 3 between folds of the high bits)
__device__ inline uint32_t ad_mix(uint32_t x) {
    x ^= x >> 16;
    x *= 0x6A09E667u;
    x ^= x >> 15;
    x *= 0xBB67AE85u;
    return x ^ x >> 16;
}

// the value of code c (of top) without its scale: an eighth of an octave by selection, the octave in the exponent
__device__ inline float ad_level(int c, int top) {
    const int k = c - top + 8 * 32, i = k & 7;  // (top is 127 or 255, one less than a multiple of 8)
    const float lo = i & 2 ? (i & 1 ? 1.29683955f : 1.18920712f) : (i & 1 ? 1.09050773f : 1.0f);
    const float hi = i & 2 ? (i & 1 ? 1.83400809f : 1.68179283f) : (i & 1 ? 1.54221083f : 1.41421356f);
    const float f = __uint_as_float(__float_as_uint(i & 4 ? hi : lo) + ((uint32_t)((k >> 3) - 32) << 23));
    return c == 0 ? 0.0f : f;
}

// Levels in LDS, TOP + 1 of them, with 0 below the first and the last one again above it.
template <int TOP>
struct AdamLevels {
    float at[TOP + 3];
    __device__ inline void fill(int tid, int threads) {
        for (int c = tid; c < TOP + 3; c += threads) at[c] = c == 0 ? 0.0f : ad_level(c - 1 < TOP ? c - 1 : TOP, TOP);
    }
    __device__ inline float of(int c) const { return at[c + 1]; }
};

// x -> its logarithm in levels, top at the scale (the logarithm's instruction takes no subnormals: a scale below 1 and
// its values are multiplied by 2^64 first)
struct AdamLog {
    float up, zero;
    __device__ inline float of(float x) const { return __builtin_fmaf(8.0f, __builtin_amdgcn_logf(x * up), zero); }
};
__device__ inline AdamLog ad_log(float scale, int top) {
    AdamLog l;
    l.up = scale < 1.0f ? 0x1p64f : 1.0f;
    l.zero = (float)top - 8.0f * __builtin_amdgcn_logf(scale * l.up);
    return l;
}

// The code of x >= 0: one of the two levels about it, the upper one if u (in 0..1) is below its share.  `log` is the
// logarithm in levels, off by far less than half a one: the level nearest to it is one of the two, and a comparison with
// it finds the other.  Products and differences are rounded as written, so that a code is what the formulas say to the
// last bit.
template <int TOP, int LOWEST>
__device__ inline int ad_code(const AdamLevels<TOP>& levels, float x, float scale, float log, float u) {
#pragma clang fp contract(off)
    // (no number, or no scale: some code, which the caller leaves out)
    const int k = (int)__builtin_rintf(__builtin_amdgcn_fmed3f(log, 0.0f, (float)TOP));
    const float* l = levels.at + k;
    const float lower = l[0] * scale, near = l[1] * scale, upper = l[2] * scale;
    const bool over = x >= near;
    const float below = over ? near : lower, above = over ? upper : near;
    int c = over ? k : k - 1;
    c += u * (above - below) < x - below ? 1 : 0;
    if (LOWEST > 0) c = c < LOWEST && x > 0.0f ? LOWEST : c;
    return c;
}

// the root, by the instruction (one unit in the last place; it takes no subnormals)
__device__ inline float ad_root(float x) {
    const bool small = x < 0x1p-90f;
    return __builtin_amdgcn_sqrtf(small ? x * 0x1p64f : x) * (small ? 0x1p-32f : 1.0f);
}

// the moments and the step of one value
struct AdamRates { float b1, c1, b2, c2, keep, step, root, eps; };
__device__ inline void ad_value(const AdamRates& r, float g, float& p, float& m, float& v) {
    {
#pragma clang fp contract(off)
        m = r.b1 * m + r.c1 * g;
        v = r.b2 * v + r.c2 * g * g;
    }
    // (an error of some units here is far below the rounding of p)
    p = p * r.keep - r.step * m * __builtin_amdgcn_rcpf(ad_root(v * r.root) + r.eps);
}

__device__ inline float ad_scalar(float v);
__device__ inline AdamRates ad_rates(const AdamArgs& a, int t) {
    AdamRates r = {a.b1, a.c1, a.b2, a.c2, 0, 0, 0, a.eps};
    const float lr = a.lr_dev ? a.lr_dev[0] : a.lr;
    r.keep = ad_scalar(1.0f - lr * a.decay);
    // (1 - beta^t without the loss of digits for small t)
    r.step = ad_scalar(lr / -expm1f((float)t * a.ln1));
    r.root = ad_scalar(1.0f / -expm1f((float)t * a.ln2));
    return r;
}

// Memory that is known to be global: addresses that come out of memory (a plan's) are not, and accesses to any kind of
// memory would wait for LDS too.
#define PNN_GLOBAL __attribute__((address_space(1)))

// four neighbouring values, the first nv of them (the others 0)
__device__ inline void ad_load4(float (&v)[4], const PNN_GLOBAL float* p, int nv) {
    if (nv >= 4) {
        const f4 q = *(const PNN_GLOBAL f4_a4*)p;
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = q[i];
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = i < nv ? p[i] : 0.0f;
    }
}
__device__ inline void ad_load4(float (&v)[4], const PNN_GLOBAL bf16_t* p, int nv) {
    if (nv >= 4) {
        const u2v q = *(const PNN_GLOBAL u2v_a2*)p;
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = i & 1 ? bf_hi(q[i >> 1]) : bf_lo(q[i >> 1]);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = i < nv ? bf2f(p[i]) : 0.0f;
    }
}
typedef uint32_t u1_a1 __attribute__((aligned(1)));
__device__ inline uint32_t ad_load4(const PNN_GLOBAL uint8_t* p, int nv) {
    if (nv >= 4) return *(const PNN_GLOBAL u1_a1*)p;
    uint32_t q = 0;
#pragma unroll
    for (int i = 0; i < 3; ++i)
        if (i < nv) q |= (uint32_t)p[i] << (8 * i);
    return q;
}
__device__ inline void ad_store4(PNN_GLOBAL float* p, const float (&v)[4], int nv) {
    if (nv >= 4) {
        *(PNN_GLOBAL f4_a4*)p = f4{v[0], v[1], v[2], v[3]};
    } else {
#pragma unroll
        for (int i = 0; i < 3; ++i)
            if (i < nv) p[i] = v[i];
    }
}
__device__ inline void ad_store4(PNN_GLOBAL bf16_t* p, const float (&v)[4], int nv) {
    if (nv >= 4) {
        *(PNN_GLOBAL u2v_a2*)p = u2v{cvt_pk_bf16(v[0], v[1]), cvt_pk_bf16(v[2], v[3])};
    } else {
#pragma unroll
        for (int i = 0; i < 3; ++i)
            if (i < nv) p[i] = f2bf(v[i]);
    }
}
__device__ inline void ad_store4(PNN_GLOBAL uint8_t* p, uint32_t q, int nv) {
    if (nv >= 4) {
        *(PNN_GLOBAL u1_a1*)p = q;
    } else {
#pragma unroll
        for (int i = 0; i < 3; ++i)
            if (i < nv) p[i] = (uint8_t)(q >> (8 * i));
    }
}

// a chunk of the plan, the same for all lanes (in scalar registers: accesses then add a lane's place to a scalar base)
template <typename TG, typename TS>
struct AdamPlace {
    PNN_GLOBAL float* p;
    const PNN_GLOBAL TG* g;
    PNN_GLOBAL TS *m, *v;
    PNN_GLOBAL float *sm, *sv;
    PNN_GLOBAL bf16_t* copy;
    int n;
    uint32_t block, tensor, kind;
    __device__ inline AdamPlace(const AdamChunk* plan, uint32_t c, int lane) {
        constexpr int WORDS = sizeof(AdamChunk) / 4;
        const uint32_t w = ((const uint32_t*)(plan + c))[lane < WORDS ? lane : 0];
        auto word = [&](int i) { return (uint32_t)__builtin_amdgcn_readlane((int)w, i); };
        auto at = [&](size_t offset) { return (uint64_t)word((int)offset / 4 + 1) << 32 | word((int)offset / 4); };
        p = (PNN_GLOBAL float*)at(offsetof(AdamChunk, p));
        g = (const PNN_GLOBAL TG*)at(offsetof(AdamChunk, g));
        m = (PNN_GLOBAL TS*)at(offsetof(AdamChunk, m));
        v = (PNN_GLOBAL TS*)at(offsetof(AdamChunk, v));
        sm = (PNN_GLOBAL float*)at(offsetof(AdamChunk, sm));
        sv = (PNN_GLOBAL float*)at(offsetof(AdamChunk, sv));
        copy = (PNN_GLOBAL bf16_t*)at(offsetof(AdamChunk, copy));
        n = (int)word(offsetof(AdamChunk, n) / 4);
        block = word(offsetof(AdamChunk, block) / 4);
        tensor = word(offsetof(AdamChunk, tensor) / 4);
        kind = word(offsetof(AdamChunk, kind) / 4);
    }
};
__device__ inline float ad_scalar(float v) { return __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(v))); }

// the largest of a wave's sizes; NaN if one is infinite or none (sizes are compared as integers, which order them
// with infinities and NaN last)
__device__ inline uint32_t ad_size(float v) { return __float_as_uint(v) & 0x7fffffffu; }
__device__ inline float ad_scale(const float (&x)[4]) {
    uint32_t v = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k) v = ad_size(x[k]) > v ? ad_size(x[k]) : v;
    v = lanes_reduce<64>(v, [](uint32_t a, uint32_t b) { return a > b ? a : b; });
    return v < 0x7f800000u ? __uint_as_float(v) : __builtin_nanf("");
}

// A wave takes blocks of 256 values, four neighbouring ones a lane, all loads of a chunk in flight together.
template <int BITS, typename TG, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void adamw_kernel(AdamArgs a) {
    constexpr int NB = AD_CHUNK / AD_BLOCK / WAVES;  // blocks of a wave
    __shared__ AdamLevels<127> m_levels;
    __shared__ AdamLevels<255> v_levels;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    if (BITS == 8) {
        m_levels.fill(tid, 64 * WAVES);
        v_levels.fill(tid, 64 * WAVES);
        __syncthreads();
    }
    typedef typename std::conditional<BITS == 32, float, uint8_t>::type TS;
    const int done = __hip_atomic_load(a.steps, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    AdamRates r;
    int t = 0;
    for (uint32_t c = blockIdx.x; c < a.chunks; c += gridDim.x) {
        const AdamPlace<TG, TS> x(a.plan, c, lane);
        // (a plan for other states or gradients, which all of its chunks are: nothing is touched, no workgroup counts the step)
        if (x.kind != ad_kind(sizeof(TS), sizeof(TG))) return;
        const int b0 = wave * NB, first = b0 * AD_BLOCK + lane * 4;
        auto work = [&](auto full) {  // (a whole chunk: no ends to look for)
            constexpr bool FULL = decltype(full)::value;
            float p[NB][4], g[NB][4], m[NB][4], v[NB][4], sm[NB], sv[NB];
            uint32_t qm[NB], qv[NB];
#pragma unroll
            for (int b = 0; b < NB; ++b) {
                const int at = first + b * AD_BLOCK, nv = FULL ? 4 : x.n - at;
                ad_load4(p[b], x.p + at, nv);
                ad_load4(g[b], x.g + at, nv);
                if constexpr (BITS == 32) {
                    ad_load4(m[b], x.m + at, nv);
                    ad_load4(v[b], x.v + at, nv);
                } else {
                    qm[b] = ad_load4(x.m + at, nv);
                    qv[b] = ad_load4(x.v + at, nv);
                    const bool in = FULL || at - lane * 4 < x.n;
                    sm[b] = in ? x.sm[b0 + b] : 0.0f;
                    sv[b] = in ? x.sv[b0 + b] : 0.0f;
                }
            }
            if (t == 0) {  // (behind the first loads)
                t = __builtin_amdgcn_readfirstlane(done) + 1;
                r = ad_rates(a, t);
            }
            const uint32_t key = BITS == 8 ? ad_mix(ad_mix(a.seed + 0x6A09E667u * (uint32_t)t) + x.tensor) : 0;
#pragma unroll
            for (int b = 0; b < NB; ++b) {
                const int at = first + b * AD_BLOCK, nv = FULL ? 4 : x.n - at;
                if (!FULL && at - lane * 4 >= x.n) break;  // (the same for a wave)
                if (BITS == 8) {
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const int cm = qm[b] >> (8 * k) & 255, cv = qv[b] >> (8 * k) & 255;
                        m[b][k] = m_levels.of(cm & 127) * (cm & 128 ? -sm[b] : sm[b]);
                        v[b][k] = v_levels.of(cv) * sv[b];
                    }
                }
#pragma unroll
                for (int k = 0; k < 4; ++k) ad_value(r, g[b][k], p[b][k], m[b][k], v[b][k]);
                ad_store4(x.p + at, p[b], nv);
                if (x.copy) ad_store4(x.copy + at, p[b], nv);
                if constexpr (BITS == 32) {
                    ad_store4(x.m + at, m[b], nv);
                    ad_store4(x.v + at, v[b], nv);
                } else {
                    // (a value that is no number makes its block's scale one that is none; lanes past the end hold zeros)
                    const float nm = ad_scale(m[b]), nw = ad_scale(v[b]);
                    const uint32_t place = ad_mix(key + x.block + (uint32_t)(b0 + b)) + (uint32_t)(lane * 4);
                    const AdamLog lm = ad_log(nm, 127), lv = ad_log(nw, 255);
                    uint32_t om = 0, ov = 0;
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const uint32_t bits = ad_mix(place + (uint32_t)k);
                        const float um = __builtin_fmaf((float)(bits >> 16), 0x1p-16f, 0x1p-17f);
                        const float uv = __builtin_fmaf((float)(bits & 0xffff), 0x1p-16f, 0x1p-17f);
                        const float size = __builtin_fabsf(m[b][k]);
                        const int cm = ad_code<127, 0>(m_levels, size, nm, lm.of(size), um);
                        const int cv = ad_code<255, 1>(v_levels, v[b][k], nw, lv.of(v[b][k]), uv);
                        om |= ((uint32_t)cm | (__float_as_uint(m[b][k]) >> 24 & 128)) << (8 * k);
                        ov |= (uint32_t)cv << (8 * k);
                    }
                    om = nm > 0.0f ? om : 0;
                    ov = nw > 0.0f ? ov : 0;
                    ad_store4(x.m + at, om, nv);
                    ad_store4(x.v + at, ov, nv);
                    if (lane == 0) {
                        x.sm[b0 + b] = nm;
                        x.sv[b0 + b] = nw;
                    }
                }
            }
        };
        if (x.n == AD_CHUNK) work(std::true_type{});
        else work(std::false_type{});
    }
    // the last workgroup to come here counts the step: all others have read the count
    __syncthreads();
    if (tid == 0) {
        bool last = true;
        if (gridDim.x > AD_GROUPS) {
            const uint32_t place = blockIdx.x % AD_GROUPS, those = (gridDim.x - place + AD_GROUPS - 1) / AD_GROUPS;
            last = atomicAdd(a.places + place * 16, 1u) == those - 1;
            if (last) a.places[place * 16] = 0;
        }
        const int most = gridDim.x < AD_GROUPS ? (int)gridDim.x : AD_GROUPS;
        if (last && atomicAdd(a.steps + 1, 1) == most - 1) {
            a.steps[0] = done + 1;
            a.steps[1] = 0;
        }
    }
}

// What 8-bit states stand for: 34.3 million values in 66 to 69 us, 5.3 to 5.0 TB/s.
__global__ __launch_bounds__(256) void adamw_values_kernel(const uint8_t* qm, const uint8_t* qv, const float* sm, const float* sv, int64_t n,
                                                           float* m, float* v) {
    __shared__ AdamLevels<127> m_levels;
    __shared__ AdamLevels<255> v_levels;
    m_levels.fill(threadIdx.x, 256);
    v_levels.fill(threadIdx.x, 256);
    __syncthreads();
    for (int64_t at = (blockIdx.x * 256ll + threadIdx.x) * 4; at < n; at += gridDim.x * 1024ll) {
        const int nv = n - at < 4 ? (int)(n - at) : 4;
        const uint32_t cm = ad_load4((const PNN_GLOBAL uint8_t*)qm + at, nv), cv = ad_load4((const PNN_GLOBAL uint8_t*)qv + at, nv);
        const float fm = sm[at / AD_BLOCK], fv = sv[at / AD_BLOCK];
        float om[4], ov[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            om[k] = m_levels.of(cm >> (8 * k) & 127) * (cm >> (8 * k) & 128 ? -fm : fm);
            ov[k] = v_levels.of(cv >> (8 * k) & 255) * fv;
        }
        ad_store4((PNN_GLOBAL float*)m + at, om, nv);
        ad_store4((PNN_GLOBAL float*)v + at, ov, nv);
    }
}

}  // namespace pnn
