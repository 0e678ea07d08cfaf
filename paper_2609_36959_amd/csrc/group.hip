// Pairs grouped by expert: a stable counting sort of the T*K pairs by their
// expert, in the order in which the experts' products take their rows.
//
// place_kernel: a workgroup takes a tile of consecutive pairs, each wave a
// segment of it. The waves count their pairs by expert in histograms of their
// own in LDS; the first place of each (wave, expert) follows from the totals
// of all tiles, the counts of the tiles before and those of the waves before.
// Then each wave goes through its segment again, 64 pairs at a time: lanes of
// the same expert find each other by one ballot per bit of the expert, so a
// pair's place is the wave's next place of its expert plus the number of its
// peers in lower lanes. No order depends on scheduling.
//
// With one tile (up to kOneTile pairs) that is the whole call, one launch.
// Above, count_kernel first writes the counts of every tile, [tiles][E], and
// each workgroup of place_kernel sums them for itself (they come out of the
// L2): that costs less than a third launch.
#include <algorithm>

#include "internal.hpp"

namespace cobalt {
namespace {

// Pairs that one workgroup sorts by itself, and the most tiles beyond.
constexpr int64_t kOneTile = 8192;
constexpr int64_t kMaxTiles = 256;

struct Cut {
    int64_t tile;   // pairs of a tile
    int tiles, waves;
    size_t lds;
};

Cut cut_pairs(int64_t P, int E) {
    Cut c;
    // 1024 to a wave keeps the walk short; at most kMaxTiles
    c.tiles = (int)std::min<int64_t>(P <= kOneTile ? 1 : (P + kOneTile - 1) / kOneTile, kMaxTiles);
    c.tile = std::max<int64_t>((P + c.tiles - 1) / c.tiles, 1);
    // as many waves as have pairs, and whose histograms leave room in LDS
    const int64_t want = std::min<int64_t>((c.tile + 63) / 64, 16);
    const int64_t room = 64 * 1024 / (4 * (int64_t)E) - 2;
    c.waves = (int)std::max<int64_t>(1, std::min(want, room));
    c.lds = (size_t)(c.waves + 2) * E * 4;
    return c;
}

__global__ __launch_bounds__(1024) void count_kernel(const int32_t* __restrict__ topk, int64_t P,
                                                     int E, int64_t tile,
                                                     uint32_t* __restrict__ counts) {
    extern __shared__ uint32_t hist[];
    for (int e = threadIdx.x; e < E; e += blockDim.x) hist[e] = 0;
    __syncthreads();
    const int64_t p0 = blockIdx.x * tile, p1 = p0 + tile < P ? p0 + tile : P;
    for (int64_t p = p0 + threadIdx.x; p < p1; p += blockDim.x) {
        const uint32_t e = (uint32_t)topk[p];
        if (e < (uint32_t)E) atomicAdd(hist + e, 1u);
    }
    __syncthreads();
    for (int e = threadIdx.x; e < E; e += blockDim.x) counts[(int64_t)blockIdx.x * E + e] = hist[e];
}

__global__ __launch_bounds__(1024) void place_kernel(
    const int32_t* __restrict__ topk, const int32_t* __restrict__ pos, int64_t P, int K, int E,
    int ebits, int64_t tile, int tiles, const uint32_t* __restrict__ counts,
    int32_t* __restrict__ rows, int32_t* __restrict__ tokens, int32_t* __restrict__ offsets) {
    extern __shared__ uint32_t lds[];
    __shared__ uint32_t wave_sum[16];
    const int waves = blockDim.x >> 6, w = threadIdx.x >> 6, lane = threadIdx.x & 63;
    uint32_t* total = lds;            // [E]: pairs of the expert, then its first place
    uint32_t* before = lds + E;       // [E]: of them, in the tiles before
    uint32_t* hist = lds + 2 * E;     // [waves][E]: of the wave, then its next place
    for (int i = threadIdx.x; i < (waves + 2) * E; i += blockDim.x) lds[i] = 0;
    __syncthreads();
    const int64_t p0 = blockIdx.x * tile, p1 = p0 + tile < P ? p0 + tile : P;
    const int64_t seg = ((p1 - p0 + waves - 1) / waves + 63) / 64 * 64;
    const int64_t s0 = p0 + w * seg, s1 = s0 + seg < p1 ? s0 + seg : p1;
    uint32_t* mine = hist + (int64_t)w * E;
    for (int64_t p = s0 + lane; p < s1; p += 64) {
        const uint32_t e = (uint32_t)topk[p];
        if (e < (uint32_t)E) atomicAdd(mine + e, 1u);
    }
    if (tiles > 1) {
        const int n = tiles * E, mid = blockIdx.x * E;
        for (int i = threadIdx.x; i < n; i += blockDim.x) {
            const uint32_t c = counts[i];
            if (c == 0) continue;
            const int e = i % E;
            atomicAdd(total + e, c);
            if (i < mid) atomicAdd(before + e, c);
        }
    }
    __syncthreads();
    // first place of each expert: each thread sums a run of experts, the runs
    // are scanned over the workgroup
    const int per = (E + blockDim.x - 1) / blockDim.x;
    const int e0 = min((int)threadIdx.x * per, E), e1 = min(e0 + per, E);
    uint32_t sum = 0;
    for (int e = e0; e < e1; ++e) {
        if (tiles == 1) {
            uint32_t c = 0;
            for (int v = 0; v < waves; ++v) c += hist[v * E + e];
            total[e] = c;
        }
        sum += total[e];
    }
    uint32_t incl = sum;
    for (int o = 1; o < 64; o <<= 1) {
        const uint32_t up = __shfl_up(incl, o, 64);
        if (lane >= o) incl += up;
    }
    if (lane == 63) wave_sum[w] = incl;
    __syncthreads();
    uint32_t first = incl - sum;
    for (int v = 0; v < w; ++v) first += wave_sum[v];
    for (int e = e0; e < e1; ++e) {
        const uint32_t c = total[e];
        if (blockIdx.x == 0) offsets[e] = (int32_t)first;
        uint32_t next = first + before[e];
        for (int v = 0; v < waves; ++v) {
            const uint32_t n = hist[v * E + e];
            hist[v * E + e] = next;
            next += n;
        }
        first += c;
    }
    uint32_t placed = 0;
    for (int v = 0; v < waves; ++v) placed += wave_sum[v];
    if (blockIdx.x == 0 && threadIdx.x == 0) offsets[E] = (int32_t)placed;
    __syncthreads();
    for (int64_t b = s0; b < s1; b += 64) {
        const int64_t p = b + lane;
        const uint32_t e = p < s1 ? (uint32_t)topk[p] : ~0u;
        const bool valid = e < (uint32_t)E;
        uint64_t peers = __ballot(valid);
        for (int k = 0; k < ebits; ++k) {
            const uint64_t bal = __ballot((e >> k) & 1u);
            peers &= (e >> k) & 1u ? bal : ~bal;
        }
        if (valid) {
            const int rank = __popcll(peers & ((uint64_t(1) << lane) - 1));
            const uint32_t at = mine[e] + rank;
            if (rank == 0) mine[e] += __popcll(peers);
            rows[at] = pos ? pos[p] : (int32_t)p;
            if (tokens) tokens[at] = (int32_t)((uint32_t)p / (uint32_t)K);
        }
    }
    // places behind the last pair
    for (int64_t i = p0 + threadIdx.x; i < p1; i += blockDim.x) {
        if (i < placed) continue;
        rows[i] = -1;
        if (tokens) tokens[i] = -1;
    }
}

}  // namespace

// The counts of every tile. Fewer pairs never take more tiles.
size_t expert_group_workspace_bytes(int64_t T, int K, int E) {
    const Cut c = cut_pairs(T * K, E);
    return std::max<size_t>(((size_t)c.tiles * E * 4 + 255) / 256 * 256, 256);
}

cobalt_status launch_expert_group(const int32_t* topk, const int32_t* pos, int64_t T, int K, int E,
                                  int32_t* rows, int32_t* tokens, int32_t* offsets, void* ws,
                                  hipStream_t s) {
    const int64_t P = T * K;
    const Cut c = cut_pairs(P, E);
    int ebits = 0;
    while ((1 << ebits) < E) ++ebits;
    if (c.tiles > 1) {
        count_kernel<<<c.tiles, 1024, (size_t)E * 4, s>>>(topk, P, E, c.tile, (uint32_t*)ws);
        COBALT_LAUNCH_CHECK();
    }
    place_kernel<<<c.tiles, c.waves * 64, c.lds, s>>>(topk, pos, P, K, E, ebits, c.tile, c.tiles,
                                                      (const uint32_t*)ws, rows, tokens, offsets);
    COBALT_LAUNCH_CHECK();
    return COBALT_OK;
}

}  // namespace cobalt
