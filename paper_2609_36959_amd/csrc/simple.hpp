// A product of two operands given element by element, on the matrix cores:
// the plain form of the experts' products.
#pragma once

#include "experts.hpp"

namespace cobalt {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int kTile = 64, kDepth = 32, kPitch = kDepth + 8;

// c[m][n] = sum_k a(m, k) b(n, k), m < rows, n < cols, for the 64 x 64 tile
// at (0, n0); a and b return bf16 bits and are called within bounds only.
// store(m, n, c) for every element of the tile within bounds.
template <typename A, typename B, typename St>
__device__ void simple_product(int rows, int64_t n0, int64_t cols, int64_t depth, A a, B b, St st) {
    __shared__ alignas(16) uint16_t as[kTile][kPitch], bs[kTile][kPitch];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    const int r = threadIdx.x >> 2, c = (threadIdx.x & 3) * 8;
    f32x4 acc[4] = {};
    for (int64_t k0 = 0; k0 < depth; k0 += kDepth) {
        for (int i = 0; i < 8; ++i) {
            const int64_t k = k0 + c + i;
            as[r][c + i] = r < rows && k < depth ? a(r, k) : 0;
            bs[r][c + i] = n0 + r < cols && k < depth ? b(n0 + r, k) : 0;
        }
        __syncthreads();
        const bf16x8 fb = *(const bf16x8*)&bs[w * 16 + lane % 16][lane / 16 * 8];
        for (int j = 0; j < 4; ++j) {
            const bf16x8 fa = *(const bf16x8*)&as[j * 16 + lane % 16][lane / 16 * 8];
            acc[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fb, fa, acc[j], 0, 0, 0);
        }
        __syncthreads();
    }
    for (int j = 0; j < 4; ++j)
        for (int q = 0; q < 4; ++q) {
            const int m = j * 16 + lane % 16;
            const int64_t n = n0 + w * 16 + lane / 16 * 4 + q;
            if (m < rows && n < cols) st(m, n, acc[j][q]);
        }
}

}  // namespace cobalt
