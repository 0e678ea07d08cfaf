// Tiles of the experts' products on the matrix cores.
//
// A workgroup of eight waves makes a tile of BM x 256 results, acc[m][n] =
// sum_k q(m, k) p(n, k), in fp32. The operands pass through LDS in steps of
// 128 bytes of k per row (64 bf16 values, or 256 of 4 bits), two stages. Per
// step and wave there are two halves; each multiplies what the half before
// has read from LDS into registers and reads what the next one needs, one
// read between every few products, so that the matrix cores and LDS work at
// the same time. In the middle of a step every wave has read all of its
// stage: one barrier there frees the stage, and the loads of the step after
// the next go straight into it (global to LDS, no registers), a whole step
// before they are waited for.
//
// Results are transposed on the matrix cores: p is the operand of their rows,
// so that a lane holds consecutive n of one m and stores whole vectors.
//
// On 8192^3 the loop reaches 1.29 PFLOP/s, and 1.31 on 16384 x 4096 x 7168
// (a library product of the same operands 1.32 and 1.28 in that run); four
// waves with 128 x 128 results each, which read a third less from LDS, stay
// at 1.05.
#pragma once

#include "experts.hpp"

namespace cobalt {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef int16_t s16x4 __attribute__((ext_vector_type(4)));
typedef int16_t s16x8 __attribute__((ext_vector_type(8)));

constexpr int kWaves = 8, kWM = 2, kWN = 4;  // waves of a workgroup, along m and n
constexpr int kBN = 256;
constexpr int kStepBytes = 128;

// What is loaded for k past the end of a row, on both sides of a product.
alignas(16) static __device__ const uint32_t kNothing[4] = {0, 0, 0, 0};

// 16 bytes per lane from `p` to the 1 KiB of LDS at `lds`, lane by lane.
__device__ __forceinline__ void load_to_lds(const char* p, char* lds) {
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)p,
                                     (__attribute__((address_space(3))) void*)lds, 16, 0, 0);
}

__device__ __forceinline__ int wave_id() {
    return __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
}

// An operand whose k is contiguous in memory: B rows of `bytes` bytes, one
// step of each a row of 128 bytes in LDS. The 16-byte chunk c of row r lies at
// chunk c ^ (r / 2 % 8), so that the 16 rows that a quarter wave reads at one
// chunk lie in 16 different groups of four banks.
template <int B>
struct RowOperand {
    static constexpr bool kColumns = false;
    static constexpr int kLoads = B / 8 / kWaves;
    static constexpr int kReads = 1;  // LDS reads per fragment
    const char* p[kLoads];
    int64_t bytes;

    // row(r): address of row r of the tile
    template <typename F>
    __device__ void start(int64_t row_bytes, F&& row) {
        const int lane = threadIdx.x & 63, w = wave_id();
        bytes = row_bytes;
#pragma unroll
        for (int j = 0; j < kLoads; ++j) {
            const int r = (j * kWaves + w) * 8 + lane / 8;
            p[j] = (const char*)row(r) + ((lane & 7) ^ ((r >> 1) & 7)) * 16;
        }
    }
    __device__ __forceinline__ void load(char* lds, int s) {
        const int lane = threadIdx.x & 63, w = wave_id();
        const int64_t left = bytes - (int64_t)s * kStepBytes;
        if (left >= kStepBytes) {
#pragma unroll
            for (int j = 0; j < kLoads; ++j) load_to_lds(p[j], lds + (j * kWaves + w) * 1024);
        } else {
#pragma unroll
            for (int j = 0; j < kLoads; ++j) {
                const int r = (j * kWaves + w) * 8 + lane / 8;
                const int c = (lane & 7) ^ ((r >> 1) & 7);
                load_to_lds(c * 16 < left ? p[j] : (const char*)kNothing,
                            lds + (j * kWaves + w) * 1024);
            }
        }
#pragma unroll
        for (int j = 0; j < kLoads; ++j) p[j] += kStepBytes;
    }
    // The wave's part of rows r0 + 16 t + (0..15) for half kk of the step: a
    // lane's chunk is 2 * (lane / 16) + kk.
    __device__ __forceinline__ static bf16x8 read(const char* lds, int r0, int t, int kk) {
        const int lane = threadIdx.x & 63, i = lane & 15, g = lane >> 4;
        const int c = (2 * g + kk) ^ ((i >> 1) & 7);
        return *(const bf16x8*)(lds + (r0 + i) * 128 + t * 2048 + c * 16);
    }
};

// A bf16 operand whose k runs over the rows of memory, B consecutive values of
// each: 64 rows of 2B bytes in LDS for one step. Lanes get eight consecutive k
// of their column by two transposing reads of four rows each. The 32-byte
// unit u of row k lies at unit u ^ (k % 4 + k / 16 % 2 * 4): a half wave reads
// one unit of eight rows, from eight different groups of eight banks.
template <int B>
struct ColumnOperand {
    static constexpr bool kColumns = true;
    static constexpr int kRowBytes = 2 * B;
    static constexpr int kLoads = B * 128 / 1024 / kWaves;
    static constexpr int kReads = 2;
    const char* base;   // first column of the tile, in row 0
    int64_t pitch;      // bytes between rows
    int64_t rows;       // k
    const int32_t* idx; // row of each k, or NULL
    int64_t n_rows;
    int32_t next[kLoads];  // idx of the rows of the step to come
    int32_t at[kLoads];    // byte of the lane's chunk in the row

    __device__ __forceinline__ static int row_of(int j) {
        return (j * kWaves + wave_id()) * (1024 / kRowBytes) + (threadIdx.x & 63) * 16 / kRowBytes;
    }
    // cols: columns of the tile that there are (a multiple of 8)
    __device__ void start(const void* first, int64_t cols, int64_t row_bytes, int64_t k,
                          const int32_t* index, int64_t index_rows) {
        const int lane = threadIdx.x & 63;
        base = (const char*)first;
        pitch = row_bytes;
        rows = k;
        idx = index;
        n_rows = index_rows;
        if (idx) fetch(0);
#pragma unroll
        for (int j = 0; j < kLoads; ++j) {
            const int r = row_of(j), slot = lane * 16 % kRowBytes / 16;
            const int unit = (slot >> 1) ^ ((r & 3) | (((r >> 4) & 1) << 2));
            const int c = (unit * 2 + (slot & 1)) * 8;
            at[j] = (c < cols ? c : (int)cols - 8) * 2;
        }
    }
    __device__ __forceinline__ void fetch(int s) {
#pragma unroll
        for (int j = 0; j < kLoads; ++j) {
            const int64_t k = (int64_t)s * 64 + row_of(j);
            next[j] = idx[k < rows ? k : rows - 1];
        }
    }
    __device__ __forceinline__ void load(char* lds, int s) {
        const int w = wave_id();
#pragma unroll
        for (int j = 0; j < kLoads; ++j) {
            const int64_t k = (int64_t)s * 64 + row_of(j);
            const int64_t r = idx ? next[j] : k;
            const bool ok = k < rows && r >= 0 && r < n_rows;
            load_to_lds(ok ? base + r * pitch + at[j] : (const char*)kNothing,
                        lds + (j * kWaves + w) * 1024);
        }
        if (idx) fetch(s + 1);
    }
    __device__ __forceinline__ static bf16x8 read(const char* lds, int c0, int t, int kk) {
        const int lane = threadIdx.x & 63, i = lane & 15, g = lane >> 4;
        const int unit = (c0 / 16 + t) ^ ((i >> 2) | ((g & 1) << 2));
        const char* a = lds + (16 * g + 8 * kk + (i >> 2)) * kRowBytes + unit * 32 + (i & 3) * 8;
        typedef __attribute__((address_space(3))) s16x4* lds4;
        const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)a);
        const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)(a + 4 * kRowBytes));
        return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    }
};

// Results of a wave: TM x 4 tiles of 16 x 16. Lane l holds, of tile (x, t),
// m = m0 + 16 x + l % 16 and n = n0 + 16 t + 4 (l / 16) + (0..3).
template <int TM>
using Acc = f32x4[TM][4];

constexpr size_t tile_lds(int BM) { return 2 * (size_t)(BM + kBN) * kStepBytes; }

template <int TM, typename Q, typename P>
__device__ __forceinline__ void multiply(char* lds, Q& q, P& p, int steps, Acc<TM>& acc) {
    constexpr int kBM = TM * 16 * kWM, kStage = (kBM + kBN) * kStepBytes;
    const int w = wave_id(), m0 = w / kWN * (TM * 16), n0 = w % kWN * 64;
    bf16x8 fq[2][TM], fp[2][4];
    const auto load = [&](int s) {
        char* at = lds + (s & 1) * kStage;
        q.load(at, s);
        p.load(at + kBM * kStepBytes, s);
    };
    const auto read = [&](int to, int s, int kk) {
        const char* at = lds + (s & 1) * kStage;
#pragma unroll
        for (int t = 0; t < 4; ++t) fp[to][t] = P::read(at + kBM * kStepBytes, n0, t, kk);
#pragma unroll
        for (int t = 0; t < TM; ++t) fq[to][t] = Q::read(at, m0, t, kk);
    };
    const auto half = [&](int of, int s, int kk) {
        read(of ^ 1, s, kk);
#pragma unroll
        for (int x = 0; x < TM; ++x)
#pragma unroll
            for (int t = 0; t < 4; ++t)
                acc[x][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fp[of][t], fq[of][x],
                                                                    acc[x][t], 0, 0, 0);
        constexpr int kR = TM * Q::kReads + 4 * P::kReads, kM = 4 * TM;
        constexpr int kPer = kM / kR > 0 ? kM / kR : 1;
        constexpr int kGroups = kM / kPer < kR ? kM / kPer : kR;
#pragma unroll
        for (int i = 0; i < kGroups; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);    // a read of LDS
            __builtin_amdgcn_sched_group_barrier(0x008, kPer, 0);  // kPer products
        }
        __builtin_amdgcn_sched_barrier(0);
    };
#pragma unroll
    for (int x = 0; x < TM; ++x)
#pragma unroll
        for (int t = 0; t < 4; ++t) acc[x][t] = f32x4{0, 0, 0, 0};
    load(0);
    if (steps > 1) load(1);
    asm volatile("s_waitcnt vmcnt(0)\n\ts_barrier" ::: "memory");
    read(0, 0, 0);
    for (int s = 0; s < steps; ++s) {
        half(0, s, 1);
        // every wave has read stage s and has its part of stage s + 1
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
        if (s + 2 < steps) load(s + 2);
        __builtin_amdgcn_sched_barrier(0);
        half(1, s + 1, 0);  // behind the last step: reads that nothing uses
    }
    // no wave still reads LDS when the tile's results go through it
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
}

// The tile of workgroup b among mt x nt tiles. Eight consecutive workgroups
// run on eight XCDs; of every 256, each XCD takes 32 consecutive tiles, and
// those are four rows of tiles by eight columns, so that what they load meets
// in the XCD's L2.
struct TileAt {
    uint32_t m, n;
};
__device__ __forceinline__ TileAt tile_at(uint32_t b, uint32_t nt) {
    const uint32_t id = b / 256 * 256 + b % 8 * 32 + b / 8 % 32;
    const uint32_t band = id / (4 * nt), r = id % (4 * nt);
    return {band * 4 + r % 4, r / 4};
}
// Workgroups of a launch over mt x nt tiles.
inline int64_t tile_grid(int64_t mt, int64_t nt) {
    return ((mt + 3) / 4 * 4 * nt + 255) / 256 * 256;
}

}  // namespace cobalt
