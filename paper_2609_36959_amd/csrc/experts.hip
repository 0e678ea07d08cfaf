// The experts' products in bf16: plain form.
#include "simple.hpp"

namespace cobalt {
namespace {

__device__ __forceinline__ float wide(uint16_t v) { return __uint_as_float((uint32_t)v << 16); }
__device__ __forceinline__ uint16_t narrow(float v) { return (uint16_t)pack_bf16_rne(v, 0.0f); }

// tmp[i][n] fp32-free form: one workgroup makes the gate tile, then the up tile
template <Act A>
__global__ __launch_bounds__(256) void gate_up_kernel(Groups g, const uint16_t* x, Rows rows,
                                                      int64_t d, int64_t f, const uint16_t* w,
                                                      uint16_t* h, uint16_t* gu) {
    __shared__ float gate[kTile][kTile + 1];
    const int nt = (int)((f + kTile - 1) / kTile);
    Tile t;
    if (!find_tile(g, kTile, blockIdx.x / nt, &t)) return;
    const int64_t n0 = (int64_t)(blockIdx.x % nt) * kTile;
    const auto a = [&](int m, int64_t k) {
        const int64_t r = rows.of(t.lo + m);
        return r < 0 ? (uint16_t)0 : x[r * d + k];
    };
    for (int side = 0; side < 2; ++side) {
        const uint16_t* we = w + ((int64_t)t.e * 2 + side) * f * d;
        simple_product(
            t.hi - t.lo, n0, f, d, a, [&](int64_t n, int64_t k) { return we[n * d + k]; },
            [&](int m, int64_t n, float v) {
                const int64_t i = t.lo + m;
                if (gu) gu[i * 2 * f + side * f + n] = narrow(v);
                if (side == 0)
                    gate[m][n - n0] = act<A>(v);
                else
                    h[i * f + n] = narrow(gate[m][n - n0] * v);
            });
    }
}

__global__ __launch_bounds__(256) void down_kernel(Groups g, const uint16_t* h, int64_t d,
                                                   int64_t f, const uint16_t* w, Rows rows,
                                                   uint16_t* out) {
    const int nt = (int)((d + kTile - 1) / kTile);
    Tile t;
    if (!find_tile(g, kTile, blockIdx.x / nt, &t)) return;
    const uint16_t* we = w + (int64_t)t.e * d * f;
    simple_product(
        t.hi - t.lo, (int64_t)(blockIdx.x % nt) * kTile, d, f,
        [&](int m, int64_t k) { return h[(int64_t)(t.lo + m) * f + k]; },
        [&](int64_t n, int64_t k) { return we[n * f + k]; },
        [&](int m, int64_t n, float v) {
            const int64_t r = rows.of(t.lo + m);
            if (r >= 0) out[r * d + n] = narrow(v);
        });
}

template <Act A>
__global__ __launch_bounds__(256) void down_gradient_kernel(Groups g, const uint16_t* dout,
                                                            Rows rows, int64_t d, int64_t f,
                                                            const uint16_t* w,
                                                            const uint16_t* gu, uint16_t* dgu) {
    const int nt = (int)((f + kTile - 1) / kTile);
    Tile t;
    if (!find_tile(g, kTile, blockIdx.x / nt, &t)) return;
    const uint16_t* we = w + (int64_t)t.e * d * f;
    simple_product(
        t.hi - t.lo, (int64_t)(blockIdx.x % nt) * kTile, f, d,
        [&](int m, int64_t k) {
            const int64_t r = rows.of(t.lo + m);
            return r < 0 ? (uint16_t)0 : dout[r * d + k];
        },
        [&](int64_t n, int64_t k) { return we[k * f + n]; },
        [&](int m, int64_t n, float v) {
            const int64_t i = t.lo + m;
            const float gv = wide(gu[i * 2 * f + n]), uv = wide(gu[i * 2 * f + f + n]);
            dgu[i * 2 * f + n] = narrow(v * uv * act_slope<A>(gv));
            dgu[i * 2 * f + f + n] = narrow(v * act<A>(gv));
        });
}

__global__ __launch_bounds__(256) void gate_up_gradient_kernel(Groups g, const uint16_t* dgu,
                                                               int64_t d, int64_t f,
                                                               const uint16_t* w, Rows rows,
                                                               uint16_t* dx) {
    const int nt = (int)((d + kTile - 1) / kTile);
    Tile t;
    if (!find_tile(g, kTile, blockIdx.x / nt, &t)) return;
    const uint16_t* we = w + (int64_t)t.e * 2 * f * d;
    simple_product(
        t.hi - t.lo, (int64_t)(blockIdx.x % nt) * kTile, d, 2 * f,
        [&](int m, int64_t k) { return dgu[(int64_t)(t.lo + m) * 2 * f + k]; },
        [&](int64_t n, int64_t k) { return we[k * d + n]; },
        [&](int m, int64_t n, float v) {
            const int64_t r = rows.of(t.lo + m);
            if (r >= 0) dx[r * d + n] = narrow(v);
        });
}

__global__ __launch_bounds__(256) void weight_gradient_kernel(Groups g, const uint16_t* a,
                                                              int64_t na, bool a_rows,
                                                              const uint16_t* b, int64_t nb,
                                                              bool b_rows, Rows rows, void* dw,
                                                              bool f32, bool add) {
    const int nt = (int)((nb + kTile - 1) / kTile), mt = (int)((na + kTile - 1) / kTile);
    const int e = blockIdx.x / (nt * mt), tile = blockIdx.x % (nt * mt);
    const int64_t m0 = (int64_t)(tile / nt) * kTile;
    const int lo = min(max(g.off[e], 0), g.M), hi = min(max(g.off[e + 1], 0), g.M);
    simple_product(
        (int)(na - m0 < kTile ? na - m0 : kTile), (int64_t)(tile % nt) * kTile, nb,
        hi > lo ? hi - lo : 0,
        [&](int m, int64_t k) {
            const int64_t r = a_rows ? rows.of(lo + k) : lo + k;
            return r < 0 ? (uint16_t)0 : a[r * na + m0 + m];
        },
        [&](int64_t n, int64_t k) {
            const int64_t r = b_rows ? rows.of(lo + k) : lo + k;
            return r < 0 ? (uint16_t)0 : b[r * nb + n];
        },
        [&](int m, int64_t n, float v) {
            const int64_t at = ((int64_t)e * na + m0 + m) * nb + n;
            if (!f32)
                ((uint16_t*)dw)[at] = narrow(v);
            else
                ((float*)dw)[at] = add ? ((float*)dw)[at] + v : v;
        });
}

unsigned grid(const Groups& g, int64_t n) {
    return (unsigned)(most_tiles(g.M, g.E, kTile) * ((n + kTile - 1) / kTile));
}

}  // namespace

cobalt_status launch_gate_up(const Groups& g, const void* x, Rows rows, int64_t d, int64_t f,
                             const void* w_in, Act act, void* h, void* gate_up, hipStream_t s) {
    const auto k = act == Act::kSilu ? gate_up_kernel<Act::kSilu> : gate_up_kernel<Act::kGelu>;
    k<<<grid(g, f), 256, 0, s>>>(g, (const uint16_t*)x, rows, d, f, (const uint16_t*)w_in,
                                 (uint16_t*)h, (uint16_t*)gate_up);
    COBALT_LAUNCH_CHECK();
    return COBALT_OK;
}

cobalt_status launch_down(const Groups& g, const void* h, int64_t d, int64_t f,
                          const void* w_down, Rows rows, void* out, hipStream_t s) {
    down_kernel<<<grid(g, d), 256, 0, s>>>(g, (const uint16_t*)h, d, f, (const uint16_t*)w_down,
                                           rows, (uint16_t*)out);
    COBALT_LAUNCH_CHECK();
    return COBALT_OK;
}

cobalt_status launch_down_gradient(const Groups& g, const void* dout, Rows rows, int64_t d,
                                   int64_t f, const void* w_down, const void* gate_up, Act act,
                                   void* dgate_up, hipStream_t s) {
    const auto k =
        act == Act::kSilu ? down_gradient_kernel<Act::kSilu> : down_gradient_kernel<Act::kGelu>;
    k<<<grid(g, f), 256, 0, s>>>(g, (const uint16_t*)dout, rows, d, f, (const uint16_t*)w_down,
                                 (const uint16_t*)gate_up, (uint16_t*)dgate_up);
    COBALT_LAUNCH_CHECK();
    return COBALT_OK;
}

cobalt_status launch_gate_up_gradient(const Groups& g, const void* dgate_up, int64_t d, int64_t f,
                                      const void* w_in, Rows rows, void* dx, hipStream_t s) {
    gate_up_gradient_kernel<<<grid(g, d), 256, 0, s>>>(g, (const uint16_t*)dgate_up, d, f,
                                                       (const uint16_t*)w_in, rows, (uint16_t*)dx);
    COBALT_LAUNCH_CHECK();
    return COBALT_OK;
}

cobalt_status launch_weight_gradient(const Groups& g, const void* a, int64_t na, bool a_rows,
                                     const void* b, int64_t nb, bool b_rows, Rows rows, void* dw,
                                     bool f32, bool add, void* ws, hipStream_t s) {
    const int64_t tiles = (na + kTile - 1) / kTile * ((nb + kTile - 1) / kTile);
    weight_gradient_kernel<<<(unsigned)(tiles * g.E), 256, 0, s>>>(
        g, (const uint16_t*)a, na, a_rows, (const uint16_t*)b, nb, b_rows, rows, dw, f32, add);
    COBALT_LAUNCH_CHECK();
    return COBALT_OK;
}

size_t expert_backward_workspace_bytes(int64_t, int, int64_t, int64_t) { return 256; }

}  // namespace cobalt
