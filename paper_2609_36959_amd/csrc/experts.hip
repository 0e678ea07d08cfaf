// The experts' products in bf16 and their gradients.
#include "few.hpp"

namespace cobalt {
namespace {

template <typename S, Act A, bool kWhole>
__global__ __launch_bounds__(S::kThreads) void down_gradient_kernel(Groups g, uint32_t b0,
                                                            const char* dout, Rows rows, int64_t d,
                                                            int64_t f, const char* w,
                                                            const uint16_t* gu, uint16_t* dgu) {
    constexpr int TM = S::kTM, kBM = S::kBM, kBN = S::kBN, kWN = S::kWN;
    __shared__ __attribute__((aligned(1024))) char lds[tile_lds<S, Bf16Math<S>>()];
    const TileAt at = tile_at(b0 + blockIdx.x, (uint32_t)((f + kBN - 1) / kBN));
    Tile t;
    if (!find_tile(g, kBM, at.m, &t)) return;
    const int64_t n0 = (int64_t)at.n * kBN;
    const char* we = w + (int64_t)t.e * d * f * 2;
    RowOperand<S, kBM, false, kWhole> q;
    ColumnOperand<S, kBN, kWhole, false> p;
    start_rows(q, t, dout, rows, we, d * 2);
    p.start(we + n0 * 2, f - n0, f * 2, (int)d, nullptr, 0);
    Acc<TM> acc;
    Bf16Math<S> math;
    multiply<S>(lds, q, p, math, (int)((d * 2 + kStepBytes - 1) / kStepBytes), acc);
    store_rows<S>(lds, acc, [&](int m, int c, const f32x4 (&v)[2]) {
        const int64_t i = t.lo + m, n = n0 + c;
        if (i >= t.hi || n >= f) return;
        const bool ok = rows.of(i) >= 0;
        const u32x4 gb = *(const u32x4*)(gu + i * 2 * f + n);
        const u32x4 ub = *(const u32x4*)(gu + i * 2 * f + f + n);
        f32x4 dg[2], du[2];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const float gv = k & 1 ? high(gb[k / 2]) : low(gb[k / 2]);
            const float uv = k & 1 ? high(ub[k / 2]) : low(ub[k / 2]);
            const float dh = ok ? v[k / 4][k % 4] : 0.0f;
            dg[k / 4][k % 4] = dh * uv * act_slope<A>(gv);
            du[k / 4][k % 4] = dh * act<A>(gv);
        }
        *(u32x4*)(dgu + i * 2 * f + n) = pack8(dg[0], dg[1]);
        *(u32x4*)(dgu + i * 2 * f + f + n) = pack8(du[0], du[1]);
    });
}

template <typename S, bool kWhole>
__global__ __launch_bounds__(S::kThreads) void gate_up_gradient_kernel(Groups g, uint32_t b0,
                                                               const char* dgu, int64_t d,
                                                               int64_t f, const char* w, Rows rows,
                                                               uint16_t* dx) {
    constexpr int TM = S::kTM, kBM = S::kBM, kBN = S::kBN, kWN = S::kWN;
    __shared__ __attribute__((aligned(1024))) char lds[tile_lds<S, Bf16Math<S>>()];
    const TileAt at = tile_at(b0 + blockIdx.x, (uint32_t)((d + kBN - 1) / kBN));
    Tile t;
    if (!find_tile(g, kBM, at.m, &t)) return;
    const int64_t n0 = (int64_t)at.n * kBN;
    const char* we = w + (int64_t)t.e * 2 * f * d * 2;
    RowOperand<S, kBM, false, kWhole> q;
    ColumnOperand<S, kBN, kWhole, false> p;
    start_rows(q, t, dgu, Rows{nullptr, g.M}, we, f * 4);
    p.start(we + n0 * 2, d - n0, d * 2, (int)(2 * f), nullptr, 0);
    Acc<TM> acc;
    Bf16Math<S> math;
    multiply<S>(lds, q, p, math, (int)((f * 4 + kStepBytes - 1) / kStepBytes), acc);
    store_rows<S>(lds, acc, [&](int m, int c, const f32x4 (&v)[2]) {
        const int64_t i = t.lo + m, n = n0 + c;
        if (i >= t.hi || n >= d) return;
        const int64_t r = rows.of(i);
        if (r >= 0) *(u32x4*)(dx + r * d + n) = pack8(v[0], v[1]);
    });
}

// Tiles of all experts' gradients, expert by expert.
template <typename S, bool kFloat, bool kAdd, bool kGatherA, bool kGatherB>
__global__ __launch_bounds__(S::kThreads) void weight_gradient_kernel(
    Groups g, uint32_t b0, uint32_t mt, const char* a, int64_t na, const char* b, int64_t nb,
    Rows rows, void* dw) {
    constexpr int TM = S::kTM, kBM = S::kBM, kBN = S::kBN;
    __shared__ __attribute__((aligned(1024))) char lds[tile_lds<S, Bf16Math<S>>()];
    const TileAt at = tile_at(b0 + blockIdx.x, (uint32_t)((nb + kBN - 1) / kBN));
    const uint32_t e = at.m / mt;
    if (e >= (uint32_t)g.E) return;
    const int64_t m0 = (int64_t)(at.m % mt) * kBM, n0 = (int64_t)at.n * kBN;
    const int lo = min(max(g.off[e], 0), g.M), hi = min(max(g.off[e + 1], 0), g.M);
    Acc<TM> acc = {};
    if (hi > lo) {
        ColumnOperand<S, kBM, false, kGatherA> q;
        ColumnOperand<S, kBN, false, kGatherB> p;
        Bf16Math<S> math;
        q.start(a + (kGatherA ? 0 : lo * na * 2) + m0 * 2, na - m0, na * 2, hi - lo,
                rows.idx + lo, rows.n);
        p.start(b + (kGatherB ? 0 : lo * nb * 2) + n0 * 2, nb - n0, nb * 2, hi - lo,
                rows.idx + lo, rows.n);
        multiply<S>(lds, q, p, math, (hi - lo + 63) / 64, acc);
    }
    store_rows<S>(lds, acc, [&](int r, int c, const f32x4 (&v)[2]) {
        const int64_t m = m0 + r, n = n0 + c;
        if (m >= na || n >= nb) return;
        const int64_t i = ((int64_t)e * na + m) * nb + n;
        if constexpr (!kFloat) {
            *(u32x4*)((uint16_t*)dw + i) = pack8(v[0], v[1]);
        } else {
            f32x4* to = (f32x4*)((float*)dw + i);
            to[0] = kAdd ? to[0] + v[0] : v[0];
            to[1] = kAdd ? to[1] + v[1] : v[1];
        }
    });
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
            return by_shape(g, f, tiles(d, 64), [&](auto shape) {
                typedef decltype(shape) S;
                return over_tiles(most_tiles(g.M, g.E, S::kBM), tiles(f, S::kBN),
                                  [&](uint32_t b0, unsigned n) {
                                      down_gradient_kernel<S, a(), whole()>
                                          <<<n, S::kThreads, 0, s>>>(
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
        return by_shape(g, d, tiles(2 * f, 64), [&](auto shape) {
            typedef decltype(shape) S;
            return over_tiles(most_tiles(g.M, g.E, S::kBM), tiles(d, S::kBN),
                              [&](uint32_t b0, unsigned n) {
                                  gate_up_gradient_kernel<S, whole()><<<n, S::kThreads, 0, s>>>(
                                      g, b0, (const char*)dgate_up, d, f, (const char*)w_in, rows,
                                      (uint16_t*)dx);
                              });
        });
    });
}

cobalt_status launch_weight_gradient(const Groups& g, const void* a, int64_t na, bool a_rows,
                                     const void* b, int64_t nb, Rows rows, void* dw,
                                     bool f32, bool add, void* ws, hipStream_t s) {
    const auto run = [&](auto shape, auto in_float, auto in_add, auto ga, auto gb) {
        typedef decltype(shape) S;
        const int64_t mt = tiles(na, S::kBM);
        return over_tiles(mt * g.E, tiles(nb, S::kBN), [&](uint32_t b0, unsigned n) {
            weight_gradient_kernel<S, in_float(), in_add(), ga(), gb()>
                <<<n, S::kThreads, 0, s>>>(g, b0, (uint32_t)mt, (const char*)a, na,
                                           (const char*)b, nb, rows, dw);
        });
    };
    // rows without an index are the places; one operand at most has one
    const std::true_type yes;
    const std::false_type no;
    const auto gather = [&](auto shape, auto in_float, auto in_add) {
        if (!rows.idx) return run(shape, in_float, in_add, no, no);
        return a_rows ? run(shape, in_float, in_add, yes, no)
                      : run(shape, in_float, in_add, no, yes);
    };
    const auto by_type = [&](auto shape) {
        if (!f32) return gather(shape, no, no);
        return add ? gather(shape, yes, yes) : gather(shape, yes, no);
    };
    return by_type(Shape<4, 8>());
}

size_t expert_backward_workspace_bytes(int64_t, int, int64_t, int64_t) { return 256; }

}  // namespace cobalt
