// codes.hpp -- rows as 8-bit codes: q = the integer nearest to 127 x / max |x| of the row, scale = max |x| / 127.
//
// Ties go to the even one, and which integer is nearest is decided exactly: where the quotient in 32 bits comes near
// the middle between two integers k and k + 1, 254 |x| is compared with (2 k + 1) max |x|, both exact in 64 bits.
// (Half of the maximum is such a middle, 63.5, and common among bf16 values.)  Rows of codes are padded with zeros to a multiple of 16, so that products
// read whole 16-byte pieces.  Bound by the bytes of x and the codes.
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

// the integer nearest to 127 v / top
__device__ inline int codes_exact(float v, float top) {
    const double a = 254.0 * __builtin_fabs((double)v), k = __builtin_floor(a / (2.0 * (double)top));
    const double middle = (2.0 * k + 1.0) * (double)top;  // (k may be one too low where the quotient is a whole number)
    const int q = (int)k + (a > middle || (a == middle && ((int)k & 1)) ? 1 : 0);
    return v < 0.0f ? -q : q;
}

// G threads a row, 16 values of it each at a time; a row that one step holds is read once
template <typename T, int G>
__global__ __launch_bounds__(256) void codes_kernel(CodesArgs a) {
    __shared__ float red[4];
    constexpr int ROWS = 256 / G;
    const int tx = threadIdx.x % G, ty = threadIdx.x / G;
    const int padded = (a.width + 15) / 16 * 16;
    for (int64_t r0 = (int64_t)blockIdx.x * ROWS; r0 < a.n; r0 += (int64_t)gridDim.x * ROWS) {
        const bool in = r0 + ty < a.n;
        const int64_t r = in ? r0 + ty : a.n - 1;
        const T* x = (const T*)a.x + r * a.ldx;
        Raw8<T> raw[2];
        float top = 0.0f;  // (an infinity for a row that holds one or a NaN)
        for (int c = tx * 16; c < padded; c += G * 16) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                float v[8];
                load8(raw[h], x + c + 8 * h, a.width - c - 8 * h);
                raw8_f(v, raw[h]);
#pragma unroll
                for (int i = 0; i < 8; ++i) top = v[i] != v[i] ? __builtin_huge_valf() : fmaxf(top, __builtin_fabsf(v[i]));
            }
        }
#pragma unroll
        for (int d = 1; d < G && d < 64; d <<= 1) top = fmaxf(top, __shfl_xor(top, d));
        if (G > 64) {
            __syncthreads();
            if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = top;
            __syncthreads();
            top = fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
        }
        const bool bad = !(top < __builtin_huge_valf());
        // (the quotient in 32 bits is off by at most 127 * 2^-23, 1.6e-5; below 1e-30 the factor would leave the range)
        const bool small = top < 1e-30f;
        const float by = bad || small ? 0.0f : 127.0f / top;
        if (!in) continue;
        if (tx == 0) a.scale[r] = bad ? __builtin_nanf("") : top / 127.0f;
        for (int c = tx * 16; c < padded; c += G * 16) {
            uint32_t word[4] = {0, 0, 0, 0};
            float v[2][8];
            bool middle = small && top > 0.0f;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                if (padded > G * 16) load8(raw[h], x + c + 8 * h, a.width - c - 8 * h);
                raw8_f(v[h], raw[h]);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float t = bad ? 0.0f : v[h][i] * by, q = __builtin_rintf(t);
                    middle |= __builtin_fabsf(t - q) > 0.4999f;
                    word[2 * h + i / 4] |= (uint32_t)((int)q & 255) << (8 * (i % 4));
                }
            }
            if (middle && !bad) {
                word[0] = word[1] = word[2] = word[3] = 0;
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    word[i / 4] |= (uint32_t)(codes_exact(v[i / 8][i % 8], top) & 255) << (8 * (i % 4));
            }
            *(u4v*)(a.q + r * a.ldq + c) = u4v{word[0], word[1], word[2], word[3]};
        }
    }
}

}  // namespace pnn
