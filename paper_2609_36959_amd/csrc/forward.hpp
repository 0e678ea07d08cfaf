// The two forward products of the experts, for rows and weights in bf16 or in
// 4 bits with scales.
#pragma once

#include "tile.hpp"

namespace cobalt {

// Rows of `bytes` bytes at v; kWhole: whole steps.
template <bool kW>
struct Bf16Rows {
    template <typename S>
    using Math = Bf16Math<S>;
    static constexpr bool kScaled = false, kWhole = kW;
    const char* v;
    int64_t bytes;
    __host__ __device__ Bf16Rows(const void* p, const void*, int64_t n)
        : v((const char*)p), bytes(2 * n) {}
    __device__ __forceinline__ const char* row(int64_t r) const { return v + r * bytes; }
};
// Rows of `bytes` bytes of codes at v, `scales` bytes of scales at s.
template <bool kW>
struct MxRows {
    template <typename S>
    using Math = MxMath<S, kW>;
    static constexpr bool kScaled = true, kWhole = kW;
    const char* v;
    const char* s;
    int64_t bytes, scales;
    __host__ __device__ MxRows(const void* p, const void* q, int64_t n)
        : v((const char*)p), s((const char*)q), bytes(n / 2), scales(n / 32) {}
    __device__ __forceinline__ const char* row(int64_t r) const { return v + r * bytes; }
    __device__ __forceinline__ const char* scale_row(int64_t r) const { return s + r * scales; }
};

// A tile's operands: q row r is place lo + r's row of x; p row r is row
// far(r) + near(r) of w, with far(r) the same for 32 neighbours.
// A place without a row reads weights in its place, and its results are not
// used.
template <typename S, typename Side, typename F, typename G>
__device__ __forceinline__ void product_of_rows(char* lds, const Tile& t, const Side& x,
                                                const Rows& rows, const Side& w, F&& far,
                                                G&& near, Acc<S::kTM>& acc) {
    RowOperand<S, S::kBM, false, Side::kWhole> q;
    RowOperand<S, S::kBN, true, Side::kWhole> p;
    typename Side::template Math<S> math;
    const auto place = [&](int r) { return rows.of(min(t.lo + r, t.hi - 1)); };
    q.start(x.bytes, 0, [&](int r) {
        const int64_t at = place(r);
        return at < 0 ? w.row(far(0)) : x.row(at);
    });
    p.start(w.bytes, [&](int r) { return w.row(far(r)); },
            [&](int r) { return (uint32_t)near(r) * (uint32_t)w.bytes; });
    if constexpr (Side::kScaled)
        math.start(
            x.scales,
            [&](int r) {
                const int64_t at = place(r);
                return at < 0 ? w.scale_row(far(0)) : x.scale_row(at);
            },
            w.scale_row(far(wave_id() * 32)),
            [&](int r) { return (uint32_t)near(r) * (uint32_t)w.scales; });
    multiply<S>(lds, q, p, math, (int)((x.bytes + kStepBytes - 1) / kStepBytes), acc);
}

// h = act(gate) * up. The weight rows of a tile: a wave's 64 are 32 gate rows
// and the 32 up rows of the same columns, in the order that gives a lane eight
// consecutive columns of both, so that the product needs no other lane.
template <typename S, Act A, typename Side>
__global__ __launch_bounds__(S::kThreads) void gate_up_kernel(Groups g, uint32_t b0, Side x, Rows rows,
                                                      Side w, int64_t f, uint16_t* h,
                                                      uint16_t* gu) {
    constexpr int TM = S::kTM, kBM = S::kBM, kBN = S::kBN, kWN = S::kWN;
    __shared__
        __attribute__((aligned(1024))) char lds[tile_lds<S, typename Side::template Math<S>>()];
    const TileAt at = tile_at(b0 + blockIdx.x, (uint32_t)((f + kBN / 2 - 1) / (kBN / 2)));
    Tile t;
    if (!find_tile(g, kBM, at.m, &t)) return;
    const int64_t n0 = (int64_t)at.n * (kBN / 2);
    Acc<TM> acc;
    const int last = (int)min(f - 1 - n0, (int64_t)kBN);
    // row r is an up row where r / 32 is odd
    product_of_rows<S>(
        lds, t, x, rows, w,
        [&](int r) { return ((int64_t)t.e * 2 + ((r >> 5) & 1)) * f + n0; },
        [&](int r) {
            const int i = r & 15;
            return min((r >> 6) * 32 + (i >> 2) * 8 + ((r >> 4) & 1) * 4 + (i & 3), last);
        },
        acc);
    const int lane = threadIdx.x & 63, wv = wave_id();
    const int64_t n = n0 + wv % kWN * 32 + (lane >> 4) * 8;
    if (n >= f) return;
#pragma unroll
    for (int y = 0; y < TM; ++y) {
        const int64_t i = t.lo + wv / kWN * (TM * 16) + y * 16 + (lane & 15);
        if (i >= t.hi) continue;
        if (rows.of(i) < 0)
#pragma unroll
            for (int k = 0; k < 4; ++k) acc[y][k] = f32x4{0, 0, 0, 0};
        if (gu) {
            *(u32x4*)(gu + i * 2 * f + n) = pack8(acc[y][0], acc[y][1]);
            *(u32x4*)(gu + i * 2 * f + f + n) = pack8(acc[y][2], acc[y][3]);
        }
        f32x4 v[2];
#pragma unroll
        for (int k = 0; k < 8; ++k)
            v[k / 4][k % 4] = act<A>(acc[y][k / 4][k % 4]) * acc[y][2 + k / 4][k % 4];
        *(u32x4*)(h + i * f + n) = pack8(v[0], v[1]);
    }
}

// out = w h. The order of a wave's 64 weight rows gives a lane sixteen
// consecutive columns.
template <typename S, typename Side>
__global__ __launch_bounds__(S::kThreads) void down_kernel(Groups g, uint32_t b0, Side h, Side w,
                                                   int64_t d, Rows rows, uint16_t* out) {
    constexpr int TM = S::kTM, kBM = S::kBM, kBN = S::kBN, kWN = S::kWN;
    __shared__
        __attribute__((aligned(1024))) char lds[tile_lds<S, typename Side::template Math<S>>()];
    const TileAt at = tile_at(b0 + blockIdx.x, (uint32_t)((d + kBN - 1) / kBN));
    Tile t;
    if (!find_tile(g, kBM, at.m, &t)) return;
    const int64_t n0 = (int64_t)at.n * kBN;
    Acc<TM> acc;
    const int last = (int)min(d - 1 - n0, (int64_t)kBN);
    product_of_rows<S>(
        lds, t, h, Rows{nullptr, g.M}, w,
        [&](int) { return t.e * d + n0; },
        [&](int r) {
            const int i = r & 15;
            return min((r >> 6) * 64 + (i >> 2) * 16 + ((r >> 4) & 3) * 4 + (i & 3), last);
        },
        acc);
    const int lane = threadIdx.x & 63, wv = wave_id();
    const int64_t n = n0 + wv % kWN * 64 + (lane >> 4) * 16;
#pragma unroll
    for (int y = 0; y < TM; ++y) {
        const int64_t i = t.lo + wv / kWN * (TM * 16) + y * 16 + (lane & 15);
        if (i >= t.hi) continue;
        const int64_t r = rows.of(i);
        if (r < 0) continue;
#pragma unroll
        for (int k = 0; k < 2; ++k)
            if (n + 8 * k < d)
                *(u32x4*)(out + r * d + n + 8 * k) = pack8(acc[y][2 * k], acc[y][2 * k + 1]);
    }
}

}  // namespace cobalt
