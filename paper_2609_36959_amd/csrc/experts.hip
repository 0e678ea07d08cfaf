// The experts' products in bf16 and their gradients.
#include "few.hpp"

namespace cobalt {
namespace {

template <int TM, Act A, bool kWhole>
__global__ __launch_bounds__(512) void down_gradient_kernel(Groups g, uint32_t b0,
                                                            const char* dout, Rows rows, int64_t d,
                                                            int64_t f, const char* w,
                                                            const uint16_t* gu, uint16_t* dgu) {
    constexpr int kBM = TM * 16 * kWM;
    __shared__ __attribute__((aligned(1024))) char lds[tile_lds<TM, Bf16Math<TM>>()];
    const TileAt at = tile_at(b0 + blockIdx.x, (uint32_t)((f + kBN - 1) / kBN));
    Tile t;
    if (!find_tile(g, kBM, at.m, &t)) return;
    const int64_t n0 = (int64_t)at.n * kBN;
    const char* we = w + (int64_t)t.e * d * f * 2;
    RowOperand<kBM, false, kWhole> q;
    ColumnOperand<kBN, kWhole> p;
    start_rows(q, t, dout, rows, we, d * 2);
    p.start(we + n0 * 2, f - n0, f * 2, d, nullptr, d);
    Acc<TM> acc;
    Bf16Math<TM> math;
    multiply<TM>(lds, q, p, math, (int)((d * 2 + kStepBytes - 1) / kStepBytes), acc);
    const int lane = threadIdx.x & 63, wv = wave_id();
#pragma unroll
    for (int y = 0; y < TM; ++y) {
        const int64_t i = t.lo + wv / kWN * (TM * 16) + y * 16 + (lane & 15);
        if (i >= t.hi) continue;
        const bool ok = rows.of(i) >= 0;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int64_t n = n0 + wv % kWN * 64 + k * 16 + (lane >> 4) * 4;
            if (n >= f) continue;
            const u32x2 gb = *(const u32x2*)(gu + i * 2 * f + n);
            const u32x2 ub = *(const u32x2*)(gu + i * 2 * f + f + n);
            f32x4 dg, du;
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                const float gv = c & 1 ? high(gb[c / 2]) : low(gb[c / 2]);
                const float uv = c & 1 ? high(ub[c / 2]) : low(ub[c / 2]);
                const float v = ok ? acc[y][k][c] : 0.0f;
                dg[c] = v * uv * act_slope<A>(gv);
                du[c] = v * act<A>(gv);
            }
            *(u32x2*)(dgu + i * 2 * f + n) = pack4(dg);
            *(u32x2*)(dgu + i * 2 * f + f + n) = pack4(du);
        }
    }
}

template <int TM, bool kWhole>
__global__ __launch_bounds__(512) void gate_up_gradient_kernel(Groups g, uint32_t b0,
                                                               const char* dgu, int64_t d,
                                                               int64_t f, const char* w, Rows rows,
                                                               uint16_t* dx) {
    constexpr int kBM = TM * 16 * kWM;
    __shared__ __attribute__((aligned(1024))) char lds[tile_lds<TM, Bf16Math<TM>>()];
    const TileAt at = tile_at(b0 + blockIdx.x, (uint32_t)((d + kBN - 1) / kBN));
    Tile t;
    if (!find_tile(g, kBM, at.m, &t)) return;
    const int64_t n0 = (int64_t)at.n * kBN;
    const char* we = w + (int64_t)t.e * 2 * f * d * 2;
    RowOperand<kBM, false, kWhole> q;
    ColumnOperand<kBN, kWhole> p;
    start_rows(q, t, dgu, Rows{nullptr, g.M}, we, f * 4);
    p.start(we + n0 * 2, d - n0, d * 2, 2 * f, nullptr, 2 * f);
    Acc<TM> acc;
    Bf16Math<TM> math;
    multiply<TM>(lds, q, p, math, (int)((f * 4 + kStepBytes - 1) / kStepBytes), acc);
    const int lane = threadIdx.x & 63, wv = wave_id();
#pragma unroll
    for (int y = 0; y < TM; ++y) {
        const int64_t i = t.lo + wv / kWN * (TM * 16) + y * 16 + (lane & 15);
        if (i >= t.hi) continue;
        const int64_t r = rows.of(i);
        if (r < 0) continue;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int64_t n = n0 + wv % kWN * 64 + k * 16 + (lane >> 4) * 4;
            if (n < d) *(u32x2*)(dx + r * d + n) = pack4(acc[y][k]);
        }
    }
}

// Tiles of all experts' gradients, expert by expert.
template <bool kFloat, bool kAdd>
__global__ __launch_bounds__(512) void weight_gradient_kernel(Groups g, uint32_t b0, uint32_t mt,
                                                              const char* a, int64_t na,
                                                              Rows a_rows, const char* b,
                                                              int64_t nb, Rows b_rows, void* dw) {
    constexpr int TM = 8, kBM = TM * 16 * kWM;
    __shared__ __attribute__((aligned(1024))) char lds[tile_lds<TM, Bf16Math<TM>>()];
    const TileAt at = tile_at(b0 + blockIdx.x, (uint32_t)((nb + kBN - 1) / kBN));
    const uint32_t e = at.m / mt;
    if (e >= (uint32_t)g.E) return;
    const int64_t m0 = (int64_t)(at.m % mt) * kBM, n0 = (int64_t)at.n * kBN;
    const int lo = min(max(g.off[e], 0), g.M), hi = min(max(g.off[e + 1], 0), g.M);
    Acc<TM> acc = {};
    Bf16Math<TM> math;
    if (hi > lo) {
        ColumnOperand<kBM, false> q;
        ColumnOperand<kBN, false> p;
        // without an index the places are the rows
        const auto start = [&](auto& o, const char* v, int64_t n, int64_t c0, const Rows& rows) {
            o.start(v + (rows.idx ? 0 : lo * n * 2) + c0 * 2, n - c0, n * 2, hi - lo,
                    rows.idx ? rows.idx + lo : nullptr, rows.idx ? rows.n : hi - lo);
        };
        start(q, a, na, m0, a_rows);
        start(p, b, nb, n0, b_rows);
        multiply<TM>(lds, q, p, math, (hi - lo + 63) / 64, acc);
    }
    const int lane = threadIdx.x & 63, wv = wave_id();
#pragma unroll
    for (int y = 0; y < TM; ++y) {
        const int64_t m = m0 + wv / kWN * (TM * 16) + y * 16 + (lane & 15);
        if (m >= na) continue;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int64_t n = n0 + wv % kWN * 64 + k * 16 + (lane >> 4) * 4;
            if (n >= nb) continue;
            const int64_t i = ((int64_t)e * na + m) * nb + n;
            if constexpr (!kFloat) {
                *(u32x2*)((uint16_t*)dw + i) = pack4(acc[y][k]);
            } else {
                f32x4* to = (f32x4*)((float*)dw + i);
                *to = kAdd ? *to + acc[y][k] : acc[y][k];
            }
        }
    }
}

}  // namespace

cobalt_status launch_gate_up(const Groups& g, const void* x, Rows rows, int64_t d, int64_t f,
                             const void* w_in, Act act, void* h, void* gate_up_out,
                             hipStream_t s) {
    return by_bool(d % 64 == 0, [&](auto whole) {
        typedef Bf16Rows<whole()> Side;
        return gate_up(g, Side(x, nullptr, d), rows, Side(w_in, nullptr, d), f, act, h,
                       gate_up_out, s);
    });
}

cobalt_status launch_down(const Groups& g, const void* h, int64_t d, int64_t f,
                          const void* w_down, Rows rows, void* out, hipStream_t s) {
    return by_bool(f % 64 == 0, [&](auto whole) {
        typedef Bf16Rows<whole()> Side;
        return down(g, Side(h, nullptr, f), Side(w_down, nullptr, f), d, rows, out, s);
    });
}

cobalt_status launch_down_gradient(const Groups& g, const void* dout, Rows rows, int64_t d,
                                   int64_t f, const void* w_down, const void* gate_up, Act act,
                                   void* dgate_up, hipStream_t s) {
    return by_act(act, [&](auto a) {
        return by_bool(d % 64 == 0, [&](auto whole) {
            return by_height(g, [&](auto tm) {
                return over_tiles(most_tiles(g.M, g.E, tm * 32), tiles(f, kBN),
                                  [&](uint32_t b0, unsigned n) {
                                      down_gradient_kernel<tm(), a(), whole()><<<n, 512, 0, s>>>(
                                          g, b0, (const char*)dout, rows, d, f,
                                          (const char*)w_down, (const uint16_t*)gate_up,
                                          (uint16_t*)dgate_up);
                                  });
            });
        });
    });
}

cobalt_status launch_gate_up_gradient(const Groups& g, const void* dgate_up, int64_t d, int64_t f,
                                      const void* w_in, Rows rows, void* dx, hipStream_t s) {
    return by_bool(f % 32 == 0, [&](auto whole) {
        return by_height(g, [&](auto tm) {
            return over_tiles(most_tiles(g.M, g.E, tm * 32), tiles(d, kBN),
                              [&](uint32_t b0, unsigned n) {
                                  gate_up_gradient_kernel<tm(), whole()><<<n, 512, 0, s>>>(
                                      g, b0, (const char*)dgate_up, d, f, (const char*)w_in, rows,
                                      (uint16_t*)dx);
                              });
        });
    });
}

cobalt_status launch_weight_gradient(const Groups& g, const void* a, int64_t na, bool a_rows,
                                     const void* b, int64_t nb, bool b_rows, Rows rows, void* dw,
                                     bool f32, bool add, void* ws, hipStream_t s) {
    const Rows places{nullptr, g.M};
    const int64_t mt = tiles(na, 256);
    return over_tiles(mt * g.E, tiles(nb, kBN), [&](uint32_t b0, unsigned n) {
        const auto k = !f32 ? weight_gradient_kernel<false, false>
                       : add ? weight_gradient_kernel<true, true>
                             : weight_gradient_kernel<true, false>;
        k<<<n, 512, 0, s>>>(g, b0, (uint32_t)mt, (const char*)a, na, a_rows ? rows : places,
                            (const char*)b, nb, b_rows ? rows : places, dw);
    });
}

size_t expert_backward_workspace_bytes(int64_t, int, int64_t, int64_t) { return 256; }

}  // namespace cobalt
