// codes.hpp -- rows as 8-bit codes: q = the integer nearest to 127 x / max |x| of the row, scale = max |x| / 127.
//
// Ties go to the even one, and which integer is nearest is decided exactly: where the quotient in 32 bits comes near
// the middle between two integers k and k + 1, 254 x is compared with (2 k + 1) max |x|, both as a product and what it
// leaves.  (Half of the maximum is such a middle, 63.5, and common among bf16 values.)  Rows of codes are padded with zeros
// to a multiple of 16, so that products read whole 16-byte pieces.  Bound by the bytes of x and the codes.
#pragma once
#include "groups.hpp"

namespace pnn {

struct CodesArgs {
    const void* x;
    int64_t ldx, n;
    int width;                // values of a row
    int8_t* q;
    int64_t ldq;
    float* scale;
};

// the integer nearest to 127 v / top, for any size of top
__device__ inline int codes_exact(float v, float top) {
    const double a = 254.0 * __builtin_fabs((double)v), k = __builtin_floor(a / (2.0 * (double)top));
    const double middle = (2.0 * k + 1.0) * (double)top;  // (k may be one too low where the quotient is a whole number)
    const int q = (int)k + (a > middle || (a == middle && ((int)k & 1)) ? 1 : 0);
    return v < 0.0f ? -q : q;
}
// The same from a quotient t, off by less than 1.6e-5, and the integer q nearest to it: q, or the next one on t's side.
// Products a and b are nearly equal, so their difference is exact, and so is that of what they leave.
__device__ inline float codes_middle(float v, float top, float t, float q) {
#pragma clang fp contract(off)
    const float side = __builtin_copysignf(1.0f, t - q), twice = 2.0f * q + side;
    const float a = 254.0f * v, b = twice * top;
    const float d = ((a - b) + (__builtin_fmaf(254.0f, v, -a) - __builtin_fmaf(twice, top, -b))) * side;
    const bool odd = __builtin_rintf(0.5f * q) != 0.5f * q;
    return __builtin_fabsf(t - q) > 0.49f && (d > 0.0f || (d == 0.0f && odd)) ? q + side : q;
}

// Sixteen values of a row as loaded, zeros behind its end: eight neighbouring ones at `at`, eight more 8 G further on.
template <typename T, int G>
struct Codes16 {
    Raw8<T> half[2];
    __device__ inline void load(const T* x, int at, int width) {
#pragma unroll
        for (int h = 0; h < 2; ++h) load8(half[h], x + at + 8 * G * h, width - at - 8 * G * h);
    }
    // the largest size as an integer, which orders infinities and NaN last
    __device__ inline uint32_t top() const {
        uint32_t m = 0;
        if constexpr (sizeof(T) == 2) {  // (two at a time)
            typedef uint16_t us2 __attribute__((ext_vector_type(2)));
            us2 both = {0, 0};
#pragma unroll
            for (int i = 0; i < 8; ++i) both = __builtin_elementwise_max(both, __builtin_bit_cast(us2, half[i / 4].v[i % 4] & 0x7fff7fffu));
            m = (uint32_t)(both[0] > both[1] ? both[0] : both[1]) << 16;
        } else {
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const uint32_t u = __float_as_uint(half[i / 8].v[i / 4 % 2][i % 4]) & 0x7fffffffu;
                m = u > m ? u : m;
            }
        }
        return m;
    }
};

// G threads a row, 16 values of it each at a time; a row that one step holds is read once, and the next one's values are
// loaded while this one's are turned.  32,768 rows of 1,024 in fp32: 28 us (6.1 TB/s; x fits the memory-side cache), in bf16
// 24 to 27 (38 with the middles decided in fp64, in every wave).
template <typename T, int G>
__global__ __launch_bounds__(256) void codes_kernel(CodesArgs a) {
    __shared__ uint32_t red[4];
    constexpr int ROWS = 256 / G;
    const int tx = threadIdx.x % G, ty = threadIdx.x / G;
    const int padded = (a.width + 15) / 16 * 16;
    const bool once = padded <= G * 16;
    const auto larger = [](uint32_t x, uint32_t y) { return x > y ? x : y; };
    auto row = [&](int64_t r0) { return (const T*)a.x + (r0 + ty < a.n ? r0 + ty : a.n - 1) * a.ldx; };
    const int64_t step = (int64_t)gridDim.x * ROWS;
    int64_t r0 = (int64_t)blockIdx.x * ROWS;
    Codes16<T, G> now, next;
    if (r0 < a.n) now.load(row(r0), tx * 8, a.width);
    for (; r0 < a.n; r0 += step, now = next) {
        const int64_t r = r0 + ty;
        const T* x = row(r0);
        uint32_t m = now.top();
        if (r0 + step < a.n) next.load(row(r0 + step), tx * 8, a.width);
        if (!once)
            for (int c = tx * 8 + G * 16; c < padded; c += G * 16) {
                Codes16<T, G> more;
                more.load(x, c, a.width);
                m = larger(m, more.top());
            }
        m = lanes_reduce<(G < 64 ? 16 : 64)>(m, larger);
        if (G > 64) {
            __syncthreads();
            if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = m;
            __syncthreads();
            m = red[ty * (G / 64)];
#pragma unroll
            for (int w = 1; w < G / 64; ++w) m = larger(m, red[ty * (G / 64) + w]);
        }
        const bool bad = m >= 0x7f800000u;
        const float top = __uint_as_float(m);
        // (the quotient in 32 bits is off by at most 127 * 2^-23, below 1.6e-5; outside 1e-20..1e20 products or what they
        // leave may leave the range)
        const bool wild = !(top > 1e-20f && top < 1e20f);
        const float by = bad || wild ? 0.0f : 127.0f / top;
        if (r >= a.n) continue;
        if (tx == 0) a.scale[r] = bad ? __builtin_nanf("") : top / 127.0f;
        for (int c = tx * 8; c < padded; c += G * 16) {
            Codes16<T, G> w = now;
            if (c != tx * 8) w.load(x, c, a.width);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int at = c + 8 * G * h;
                if (at >= padded) break;
                // added to 1.5 * 2^23, a quotient is rounded to an integer whose low byte is the sum's
                constexpr float TO_INT = 12582912.0f;
                float v[8], far = 0.0f;
                uint32_t q[8];
                raw8_f(v, w.half[h]);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float t = v[i] * by, sum = t + TO_INT;
                    q[i] = __float_as_uint(sum);
                    far = fmaxf(far, __builtin_fabsf(t - (sum - TO_INT)));
                }
                if (wild) {
#pragma unroll 1
                    for (int i = 0; i < 8; ++i) {
                        const uint32_t code = top > 0.0f && !bad ? (uint32_t)codes_exact(v[0], top) : 0;
#pragma unroll
                        for (int j = 0; j < 7; ++j) {  // (one copy of its code: the values pass by)
                            v[j] = v[j + 1];
                            q[j] = q[j + 1];
                        }
                        q[7] = code;
                    }
                } else if (far > 0.499984f) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const float t = v[i] * by;
                        q[i] = __float_as_uint(codes_middle(v[i], top, t, (t + TO_INT) - TO_INT) + TO_INT);
                    }
                }
                uint32_t word[2];
#pragma unroll
                for (int i = 0; i < 2; ++i)
                    word[i] = bad ? 0 : __builtin_amdgcn_perm(__builtin_amdgcn_perm(q[4 * i + 3], q[4 * i + 2], 0x0c0c0400u),
                                                              __builtin_amdgcn_perm(q[4 * i + 1], q[4 * i], 0x0c0c0400u), 0x05040100u);
                *(u2v*)(a.q + r * a.ldq + at) = u2v{word[0], word[1]};
            }
        }
    }
}

}  // namespace pnn
