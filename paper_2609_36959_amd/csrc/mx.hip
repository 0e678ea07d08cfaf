// Microscaled 4-bit rows: quantisation, and the experts' products on them in
// plain form.
#include "simple.hpp"

namespace cobalt {
namespace {

__device__ __forceinline__ float wide(uint16_t v) { return __uint_as_float((uint32_t)v << 16); }
__device__ __forceinline__ uint16_t narrow(float v) { return (uint16_t)pack_bf16_rne(v, 0.0f); }

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

// Value k of row r.
struct MxRows {
    const uint8_t* codes;
    const uint8_t* scales;
    int64_t n;
    __device__ uint16_t operator()(int64_t r, int64_t k) const {
        const uint32_t c = codes[(r * n + k) / 2] >> (k & 1 ? 4 : 0);
        return narrow(e2m1(c & 15) * e8m0(scales[(r * n + k) / 32]));
    }
};

template <Act A>
__global__ __launch_bounds__(256) void gate_up_kernel(Groups g, MxRows x, Rows rows, int64_t d,
                                                      int64_t f, MxRows w, uint16_t* h) {
    __shared__ float gate[kTile][kTile + 1];
    const int nt = (int)((f + kTile - 1) / kTile);
    Tile t;
    if (!find_tile(g, kTile, blockIdx.x / nt, &t)) return;
    const int64_t n0 = (int64_t)(blockIdx.x % nt) * kTile;
    for (int side = 0; side < 2; ++side) {
        const int64_t w0 = ((int64_t)t.e * 2 + side) * f;
        simple_product(
            t.hi - t.lo, n0, f, d,
            [&](int m, int64_t k) {
                const int64_t r = rows.of(t.lo + m);
                return r < 0 ? (uint16_t)0 : x(r, k);
            },
            [&](int64_t n, int64_t k) { return w(w0 + n, k); },
            [&](int m, int64_t n, float v) {
                if (side == 0)
                    gate[m][n - n0] = act<A>(v);
                else
                    h[(int64_t)(t.lo + m) * f + n] = narrow(gate[m][n - n0] * v);
            });
    }
}

__global__ __launch_bounds__(256) void down_kernel(Groups g, MxRows h, int64_t d, int64_t f,
                                                   MxRows w, Rows rows, uint16_t* out) {
    const int nt = (int)((d + kTile - 1) / kTile);
    Tile t;
    if (!find_tile(g, kTile, blockIdx.x / nt, &t)) return;
    const int64_t w0 = (int64_t)t.e * d;
    simple_product(
        t.hi - t.lo, (int64_t)(blockIdx.x % nt) * kTile, d, f,
        [&](int m, int64_t k) { return h(t.lo + m, k); },
        [&](int64_t n, int64_t k) { return w(w0 + n, k); },
        [&](int m, int64_t n, float v) {
            const int64_t r = rows.of(t.lo + m);
            if (r >= 0) out[r * d + n] = narrow(v);
        });
}

unsigned grid(const Groups& g, int64_t n) {
    return (unsigned)(most_tiles(g.M, g.E, kTile) * ((n + kTile - 1) / kTile));
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
    const auto k = act == Act::kSilu ? gate_up_kernel<Act::kSilu> : gate_up_kernel<Act::kGelu>;
    k<<<grid(g, f), 256, 0, s>>>(g, MxRows{(const uint8_t*)xc, (const uint8_t*)xs, d}, rows, d, f,
                                 MxRows{(const uint8_t*)wc, (const uint8_t*)ws, d}, (uint16_t*)h);
    COBALT_LAUNCH_CHECK();
    return COBALT_OK;
}

cobalt_status launch_mx_down(const Groups& g, const void* hc, const void* hs, int64_t d, int64_t f,
                             const void* wc, const void* ws, Rows rows, void* out, hipStream_t s) {
    down_kernel<<<grid(g, d), 256, 0, s>>>(g, MxRows{(const uint8_t*)hc, (const uint8_t*)hs, f}, d,
                                           f, MxRows{(const uint8_t*)wc, (const uint8_t*)ws, f},
                                           rows, (uint16_t*)out);
    COBALT_LAUNCH_CHECK();
    return COBALT_OK;
}

}  // namespace cobalt
