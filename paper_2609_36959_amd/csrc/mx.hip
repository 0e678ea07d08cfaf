// Microscaled 4-bit rows: quantisation, and the experts' products on them.
#include "few.hpp"

namespace cobalt {
namespace {

__device__ __forceinline__ float wide(uint16_t v) { return __uint_as_float((uint32_t)v << 16); }

// One thread per block of 32 values.
__global__ __launch_bounds__(256) void quantize_kernel(const u32x4* __restrict__ x, int64_t blocks,
                                                       u32x4* __restrict__ codes,
                                                       uint8_t* __restrict__ scales) {
    const int64_t b = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (b >= blocks) return;
    uint32_t v[16];
    uint32_t big = 0;
    for (int i = 0; i < 4; ++i) {
        const u32x4 q = x[b * 4 + i];
        for (int j = 0; j < 4; ++j) {
            v[i * 4 + j] = q[j];
            big = max(big, max(q[j] & 0x7fffu, (q[j] >> 16) & 0x7fffu));
        }
    }
    u32x4 out = {0, 0, 0, 0};
    if (big >= 0x7f80u) {
        scales[b] = 255;
        codes[b] = out;
        return;
    }
    // biased exponent of the largest; that of a subnormal one is below 2^-125
    const int ex = max((int)(big >> 7) - 2, 0);
    scales[b] = (uint8_t)ex;
    const float inv = __uint_as_float((uint32_t)(254 - ex) << 23);  // 2^(127 - ex)
    for (int i = 0; i < 32; ++i) {
        const float f = wide((uint16_t)(i & 1 ? v[i / 2] >> 16 : v[i / 2])) * inv;
        const float m = fabsf(f);
        const uint32_t c = (m > 0.25f) + (m >= 0.75f) + (m > 1.25f) + (m >= 1.75f) + (m > 2.5f) +
                           (m >= 3.5f) + (m > 5.0f);
        out[i / 8] |= (c | (__float_as_uint(f) >> 31 << 3)) << (i % 8 * 4);
    }
    codes[b] = out;
}

__device__ __forceinline__ float e2m1(uint32_t c) {
    const uint32_t m = c & 7;
    const float v = m < 4 ? 0.5f * m : m < 6 ? (float)(m - 2) : 2.0f * (m - 4);
    return c & 8 ? -v : v;
}
__device__ __forceinline__ float e8m0(uint32_t b) {
    // 2^-127 is subnormal
    return b == 255 ? __uint_as_float(0x7fc00000u) : b == 0 ? __uint_as_float(0x00400000u)
                                                            : __uint_as_float(b << 23);
}

__global__ __launch_bounds__(256) void dequantize_kernel(const u32x4* __restrict__ codes,
                                                         const uint8_t* __restrict__ scales,
                                                         int64_t blocks, u32x4* __restrict__ y) {
    const int64_t b = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (b >= blocks) return;
    const u32x4 q = codes[b];
    const float s = e8m0(scales[b]);
    for (int i = 0; i < 4; ++i) {
        u32x4 o;
        for (int j = 0; j < 4; ++j) {
            const uint32_t c = q[i] >> (8 * j);
            o[j] = pack_bf16_rne(e2m1(c & 15) * s, e2m1((c >> 4) & 15) * s);
        }
        y[b * 4 + i] = o;
    }
}

}  // namespace

cobalt_status launch_mx_quantize(const void* x, int64_t R, int64_t n, void* codes, void* scales,
                                 hipStream_t s) {
    const int64_t blocks = R * (n / 32);
    quantize_kernel<<<(unsigned)((blocks + 255) / 256), 256, 0, s>>>((const u32x4*)x, blocks,
                                                                     (u32x4*)codes,
                                                                     (uint8_t*)scales);
    COBALT_LAUNCH_CHECK();
    return COBALT_OK;
}

cobalt_status launch_mx_dequantize(const void* codes, const void* scales, int64_t R, int64_t n,
                                   void* y, hipStream_t s) {
    const int64_t blocks = R * (n / 32);
    dequantize_kernel<<<(unsigned)((blocks + 255) / 256), 256, 0, s>>>(
        (const u32x4*)codes, (const uint8_t*)scales, blocks, (u32x4*)y);
    COBALT_LAUNCH_CHECK();
    return COBALT_OK;
}

cobalt_status launch_mx_gate_up(const Groups& g, const void* xc, const void* xs, Rows rows,
                                int64_t d, int64_t f, const void* wc, const void* ws, Act act,
                                void* h, hipStream_t s) {
    return by_bool(d % 256 == 0, [&](auto whole) {
        typedef MxRows<whole()> Side;
        return gate_up(g, Side(xc, xs, d), rows, Side(wc, ws, d), f, act, h, nullptr, s);
    });
}

cobalt_status launch_mx_down(const Groups& g, const void* hc, const void* hs, int64_t d, int64_t f,
                             const void* wc, const void* ws, Rows rows, void* out, hipStream_t s) {
    return by_bool(f % 256 == 0, [&](auto whole) {
        typedef MxRows<whole()> Side;
        return down(g, Side(hc, hs, f), Side(wc, ws, f), d, rows, out, s);
    });
}

}  // namespace cobalt
