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
// Bound by bytes: with fp32 gradients 28 a value, or 16 and the scales in 8 bits.
#pragma once
#include "groups.hpp"

namespace pnn {

constexpr int AD_TENSORS = 48;       // of a launch (they are kernel arguments, at most 4 KB)
constexpr int AD_BLOCK = 256;        // values of a scale
constexpr int AD_CHUNK = 4096;       // values that a workgroup takes at a time

struct AdamTensor {
    float* p;
    const void* g;
    void *m, *v;
    float *sm, *sv;
    bf16_t* copy;
    int64_t n;
};
struct AdamArgs {
    AdamTensor t[AD_TENSORS];
    uint32_t first[AD_TENSORS + 1];  // first chunk of each tensor
    int count, number;               // tensors, and the number of the first in the call
    float b1, c1, b2, c2;            // beta, 1 - beta
    float ln1, ln2;                  // log beta
    float lr, eps, decay;
    const float* lr_dev;             // (nullable) instead of lr
    uint32_t seed;
    int32_t* steps;                  // steps done; workgroups that have read it
    bool last;                       // the call's last launch: it counts the step
};

// 32 bits that look random, from 32 (multiplications by odd parts of sqrt 2 and sqrt 3 between folds of the high bits)
__device__ inline uint32_t ad_mix(uint32_t x) {
    x ^= x >> 16;
    x *= 0x6A09E667u;
    x ^= x >> 15;
    x *= 0xBB67AE85u;
    return x ^ x >> 16;
}

// 2^(i / 8)
__device__ inline float ad_eighth(int i) {
    const float e[8] = {1.0f, 1.09050773f, 1.18920712f, 1.29683955f, 1.41421356f, 1.54221083f, 1.68179283f, 1.83400809f};
    return e[i];
}

// the value of code c (of top) without its scale: an eighth of an octave from a table in LDS, the octave in the exponent
__device__ inline float ad_level(const float* eighths, int c, int top) {
    const int k = c - top + 8 * 32;  // (top is 127 or 255, one less than a multiple of 8)
    const float f = __uint_as_float(__float_as_uint(eighths[k & 7]) + ((uint32_t)((k >> 3) - 32) << 23));
    return c == 0 ? 0.0f : f;
}

// The code of x >= 0: one of the two levels about it, the upper one if u (in 0..1) is below its share.
// Products and differences are rounded as written, so that a code is what the formulas say to the last bit.
__device__ inline int ad_code(const float* eighths, float x, float scale, int top, int lowest, float u) {
#pragma clang fp contract(off)
    const float up = scale < 1.0f ? 18446744073709551616.0f : 1.0f;  // (2^64: the logarithm's instruction takes no subnormals)
    const float at = 8.0f * (__builtin_amdgcn_logf(x * up) - __builtin_amdgcn_logf(scale * up)) + (float)top;
    int c = at > 0.0f ? (int)at : 0;
    c = c > top ? top : c;
    // (the estimate is off by less than a level)
    if (c < top && ad_level(eighths, c + 1, top) * scale <= x) ++c;
    else if (c > 0 && ad_level(eighths, c, top) * scale > x) --c;
    if (c < top) {
        const float below = ad_level(eighths, c, top) * scale, above = ad_level(eighths, c + 1, top) * scale;
        if (u * (above - below) < x - below) ++c;
    }
    c = c > lowest ? c : lowest;
    return x > 0.0f ? c : 0;
}

// the moments and the step of one value
struct AdamRates { float b1, c1, b2, c2, keep, step, root, eps; };
__device__ inline void ad_value(const AdamRates& r, float g, float& p, float& m, float& v) {
    {
#pragma clang fp contract(off)
        m = r.b1 * m + r.c1 * g;
        v = r.b2 * v + r.c2 * g * g;
    }
    p = p * r.keep - r.step * m / (sqrtf(v * r.root) + r.eps);
}

__device__ inline AdamRates ad_rates(const AdamArgs& a, int t) {
    AdamRates r = {a.b1, a.c1, a.b2, a.c2, 0, 0, 0, a.eps};
    const float lr = a.lr_dev ? a.lr_dev[0] : a.lr;
    r.keep = 1.0f - lr * a.decay;
    // (1 - beta^t without the loss of digits for small t)
    r.step = lr / -expm1f((float)t * a.ln1);
    r.root = 1.0f / -expm1f((float)t * a.ln2);
    return r;
}

// four neighbouring values, the first nv of them (the others 0)
__device__ inline void ad_load4(float (&v)[4], const float* p, int nv) {
    if (nv >= 4) {
        const f4 q = *(const f4_a4*)p;
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = q[i];
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = i < nv ? p[i] : 0.0f;
    }
}
__device__ inline void ad_load4(float (&v)[4], const bf16_t* p, int nv) {
    typedef uint32_t u2v __attribute__((ext_vector_type(2)));
    typedef u2v u2v_a2 __attribute__((aligned(2)));
    if (nv >= 4) {
        const u2v q = *(const u2v_a2*)p;
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = i & 1 ? bf_hi(q[i >> 1]) : bf_lo(q[i >> 1]);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = i < nv ? bf2f(p[i]) : 0.0f;
    }
}
typedef uint32_t u1_a1 __attribute__((aligned(1)));
__device__ inline uint32_t ad_load4(const uint8_t* p, int nv) {
    if (nv >= 4) return *(const u1_a1*)p;
    uint32_t q = 0;
#pragma unroll
    for (int i = 0; i < 3; ++i)
        if (i < nv) q |= (uint32_t)p[i] << (8 * i);
    return q;
}
__device__ inline void ad_store4(float* p, const float (&v)[4], int nv) {
    if (nv >= 4) {
        *(f4_a4*)p = f4{v[0], v[1], v[2], v[3]};
    } else {
#pragma unroll
        for (int i = 0; i < 3; ++i)
            if (i < nv) p[i] = v[i];
    }
}
__device__ inline void ad_store4(bf16_t* p, const float (&v)[4], int nv) {
    typedef uint32_t u2v __attribute__((ext_vector_type(2)));
    typedef u2v u2v_a2 __attribute__((aligned(2)));
    if (nv >= 4) {
        *(u2v_a2*)p = u2v{cvt_pk_bf16(v[0], v[1]), cvt_pk_bf16(v[2], v[3])};
    } else {
#pragma unroll
        for (int i = 0; i < 3; ++i)
            if (i < nv) p[i] = f2bf(v[i]);
    }
}
__device__ inline void ad_store4(uint8_t* p, uint32_t q, int nv) {
    if (nv >= 4) {
        *(u1_a1*)p = q;
    } else {
#pragma unroll
        for (int i = 0; i < 3; ++i)
            if (i < nv) p[i] = (uint8_t)(q >> (8 * i));
    }
}

// the largest of a wave's sizes; NaN if one is infinite or none
__device__ inline float ad_scale(float v) {
    v = row_allmax16(v);
    v = fmaxf(v, __shfl_xor(v, 16));
    v = fmaxf(v, __shfl_xor(v, 32));
    return v < __builtin_huge_valf() ? v : __builtin_nanf("");
}

// a wave takes 256 values, a scale's block, at a time: four a lane
template <int BITS, typename TG>
__global__ __launch_bounds__(256) void adamw_kernel(AdamArgs a) {
    __shared__ float eighths[8];
    __shared__ int done;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    if (tid < 8) eighths[tid] = ad_eighth(tid);
    if (tid == 0) done = __hip_atomic_load(a.steps, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __syncthreads();
    const int t = done + 1;
    const AdamRates r = ad_rates(a, t);
    const uint32_t chunks = a.first[a.count];
    for (uint32_t c = blockIdx.x; c < chunks; c += gridDim.x) {
        int i = 0, end = a.count;  // the last tensor whose first chunk is at most c
        while (end - i > 1) {
            const int mid = (i + end) >> 1;
            if (a.first[mid] <= c) i = mid;
            else end = mid;
        }
        const AdamTensor& x = a.t[i];
        const int64_t base = (int64_t)(c - a.first[i]) * AD_CHUNK;
        for (int b = wave; b < AD_CHUNK / AD_BLOCK; b += 4) {
            const int64_t start = base + b * AD_BLOCK, at = start + lane * 4;
            if (start >= x.n) break;
            const int nv = x.n - at < 4 ? (int)(x.n - at) : 4;
            float p[4], g[4], m[4], v[4];
            ad_load4(p, x.p + at, nv);
            ad_load4(g, (const TG*)x.g + at, nv);
            if (BITS == 32) {
                ad_load4(m, (const float*)x.m + at, nv);
                ad_load4(v, (const float*)x.v + at, nv);
            } else {
                const uint32_t qm = ad_load4((const uint8_t*)x.m + at, nv), qv = ad_load4((const uint8_t*)x.v + at, nv);
                const float sm = x.sm[start / AD_BLOCK], sv = x.sv[start / AD_BLOCK];
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const int cm = qm >> (8 * k) & 255, cv = qv >> (8 * k) & 255;
                    m[k] = ad_level(eighths, cm & 127, 127) * sm;
                    if (cm & 128) m[k] = -m[k];
                    v[k] = ad_level(eighths, cv, 255) * sv;
                }
            }
#pragma unroll
            for (int k = 0; k < 4; ++k) ad_value(r, g[k], p[k], m[k], v[k]);
            ad_store4(x.p + at, p, nv);
            if (x.copy) ad_store4(x.copy + at, p, nv);
            if (BITS == 32) {
                ad_store4((float*)x.m + at, m, nv);
                ad_store4((float*)x.v + at, v, nv);
            } else {
                // (a value that is no number makes its block's scale one that is none)
                float tm = 0.0f, tv = 0.0f;
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    if (k >= nv) break;
                    tm = m[k] != m[k] ? __builtin_huge_valf() : fmaxf(tm, __builtin_fabsf(m[k]));
                    tv = v[k] != v[k] ? __builtin_huge_valf() : fmaxf(tv, v[k]);
                }
                const float sm = ad_scale(tm), sv = ad_scale(tv);
                const uint32_t block = (uint32_t)(start / AD_BLOCK);
                const uint32_t key = ad_mix(ad_mix(ad_mix(a.seed + 0x6A09E667u * (uint32_t)t) + (uint32_t)(a.number + i)) + block);
                uint32_t qm = 0, qv = 0;
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const uint32_t bits = ad_mix(key + (uint32_t)(lane * 4 + k));
                    const float um = ((float)(bits >> 16) + 0.5f) * 0x1p-16f, uv = ((float)(bits & 0xffff) + 0.5f) * 0x1p-16f;
                    const int cm = sm > 0.0f ? ad_code(eighths, __builtin_fabsf(m[k]), sm, 127, 0, um) : 0;
                    const int cv = sv > 0.0f ? ad_code(eighths, v[k], sv, 255, 1, uv) : 0;
                    qm |= (uint32_t)(m[k] < 0.0f ? cm | 128 : cm) << (8 * k);
                    qv |= (uint32_t)cv << (8 * k);
                }
                ad_store4((uint8_t*)x.m + at, qm, nv);
                ad_store4((uint8_t*)x.v + at, qv, nv);
                if (lane == 0) {
                    x.sm[block] = sm;
                    x.sv[block] = sv;
                }
            }
        }
    }
    // the last workgroup to come here counts the step: all others have read the count
    if (a.last && tid == 0 && atomicAdd(a.steps + 1, 1) == (int)gridDim.x - 1) {
        a.steps[0] = t;
        a.steps[1] = 0;
    }
}

// what 8-bit states stand for
__global__ __launch_bounds__(256) void adamw_values_kernel(const uint8_t* qm, const uint8_t* qv, const float* sm, const float* sv, int64_t n,
                                                           float* m, float* v) {
    __shared__ float eighths[8];
    if (threadIdx.x < 8) eighths[threadIdx.x] = ad_eighth(threadIdx.x);
    __syncthreads();
    for (int64_t at = (blockIdx.x * 256ll + threadIdx.x) * 4; at < n; at += gridDim.x * 1024ll) {
        const int nv = n - at < 4 ? (int)(n - at) : 4;
        const uint32_t cm = ad_load4(qm + at, nv), cv = ad_load4(qv + at, nv);
        const float fm = sm[at / AD_BLOCK], fv = sv[at / AD_BLOCK];
        float om[4], ov[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            om[k] = ad_level(eighths, cm >> (8 * k) & 127, 127) * fm;
            if (cm >> (8 * k) & 128) om[k] = -om[k];
            ov[k] = ad_level(eighths, cv >> (8 * k) & 255, 255) * fv;
        }
        ad_store4(m + at, om, nv);
        ad_store4(v + at, ov, nv);
    }
}

}  // namespace pnn
