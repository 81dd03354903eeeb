// Slots (row, choice) sorted by network, stably: network g's slots are the rows
// off[g] .. off[g + 1) of the grouping, in the slots' order.
//
// A counting sort.  A wave takes 64 slots at a time, in order: the lanes with the same
// digit are found with a ballot per bit, a slot's rank is the wave's count of its digit
// so far plus the lanes before it, and no atomic decides an order.  Up to 4096 slots are
// one block's; more are counted per block, the counts summed over the blocks, and the
// slots placed.  Up to 2048 networks are one digit, more two digits, the lower first.
#include "evox_mix.hpp"

namespace evox {

namespace {

constexpr int kWaves = 4, kRounds = 16, kThreads = 64 * kWaves, kTile = kThreads * kRounds;
constexpr int kMaxBins = 2048, kFewTiles = 16;

struct Pass {
    const int32_t *key;   // of the slots in this pass's order, outside 0 .. G - 1: none
    const int32_t *slot;  // their slots, or null: slot i is the i-th
    const int32_t *have;  // how many, or null: n
    int64_t n;
    int32_t G, shift, bits;
    int32_t bins, tiles;
    int32_t *count;       // [tiles][bins]: counts, then what the tiles before have
    int32_t *total;       // [bins]
    // an intermediate pass's results, or the last one's
    int32_t *key_out, *slot_out, *have_out;
    int32_t *off, *pos, *src, *sorted;
};

__device__ __forceinline__ int64_t pass_size(const Pass &p) { return p.have ? *p.have : p.n; }

// The network of the i-th slot, -1: none, or past the end (loaded from the last one
// then: loads behind a branch wait for each other).
__device__ __forceinline__ int slot_key(const Pass &p, int64_t i, int64_t n)
{
    const int key = p.key[i < n ? i : n - 1];
    return i < n && key >= 0 && key < p.G ? key : -1;
}

__global__ __launch_bounds__(kThreads) void k_route_count(Pass p)
{
    __shared__ int hist[kMaxBins];
    for (int b = threadIdx.x; b < p.bins; b += kThreads) hist[b] = 0;
    __syncthreads();
    const int64_t n = pass_size(p), base = (int64_t)blockIdx.x * kTile;
    int key[kRounds];
    if (base < n)
#pragma unroll
        for (int r = 0; r < kRounds; ++r) key[r] = slot_key(p, base + r * kThreads + threadIdx.x, n);
    else
#pragma unroll
        for (int r = 0; r < kRounds; ++r) key[r] = -1;
#pragma unroll
    for (int r = 0; r < kRounds; ++r)
        if (key[r] >= 0) atomicAdd(&hist[key[r] >> p.shift & (p.bins - 1)], 1);
    __syncthreads();
    for (int b = threadIdx.x; b < p.bins; b += kThreads) p.count[(int64_t)blockIdx.x * p.bins + b] = hist[b];
}

// count[t][b] = sum of the counts of the tiles before t, total[b] = of all: a block per
// 16 digits, 64 shares of the tiles.
__global__ __launch_bounds__(1024) void k_route_scan(Pass p)
{
    __shared__ int share[64][16];
    const int b = blockIdx.x * 16 + threadIdx.x % 16, w = threadIdx.x / 16;
    const int per = (p.tiles + 63) / 64, t0 = w * per, t1 = min(t0 + per, p.tiles);
    int s = 0;
    if (b < p.bins)
#pragma unroll 8
        for (int t = t0; t < t1; ++t) s += p.count[(int64_t)t * p.bins + b];
    share[w][threadIdx.x % 16] = s;
    __syncthreads();
    if (b >= p.bins) return;
    s = 0;
    for (int j = 0; j < w; ++j) s += share[j][threadIdx.x % 16];
    for (int t = t0; t < t1; ++t) {
        const int c = p.count[(int64_t)t * p.bins + b];
        p.count[(int64_t)t * p.bins + b] = s;
        s += c;
    }
    if (w == 63) p.total[b] = s;
}

// ONE: this tile is all.  SUMMED: count and total come from the scan; else the tile
// adds the counts before it itself.
template <bool ONE, bool SUMMED>
__global__ __launch_bounds__(kThreads) void k_route_place(Pass p)
{
    extern __shared__ int lds[];  // [kWaves][bins], [bins]
    __shared__ int sums[kWaves];
    const int wave = threadIdx.x / 64, lane = threadIdx.x % 64, tile = blockIdx.x, bins = p.bins;
    const int mine = wave * bins, base = kWaves * bins;
    for (int b = threadIdx.x; b < kWaves * bins; b += kThreads) lds[b] = 0;
    const int64_t n = pass_size(p);
    const int64_t first = (int64_t)tile * kTile;
    // rounds of this tile: the waves' shares follow each other
    const int64_t left = n - first;
    const int rounds = left <= 0 ? 0 : left >= kTile ? kRounds : (int)((left + kThreads - 1) / kThreads);
    const int64_t at = first + (int64_t)wave * rounds * 64 + lane;
    int key[kRounds], rank[kRounds];
    if (rounds)
#pragma unroll
        for (int r = 0; r < kRounds; ++r) key[r] = slot_key(p, r < rounds ? at + r * 64 : n, n);
    __syncthreads();
#pragma unroll
    for (int r = 0; r < kRounds; ++r)
        if (r < rounds) {
            const int d = key[r] >> p.shift & (bins - 1);
            const bool in = key[r] >= 0;
            uint64_t peers = __ballot(in);
            for (int b = 0; b < p.bits; ++b) {
                const uint64_t set = __ballot(d >> b & 1);
                peers &= d >> b & 1 ? set : ~set;
            }
            const int before = __popcll(peers & (((uint64_t)1 << lane) - 1));
            const int so_far = lds[mine + d];
            rank[r] = so_far + before;
            // (a wave's LDS accesses stay in their order; the compiler is told to keep it)
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            if (in && before == 0) lds[mine + d] = so_far + __popcll(peers);
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        }
    __syncthreads();
    // the digits' places: those of lower digits, of earlier tiles, of earlier waves
    const int per = (bins + kThreads - 1) / kThreads, b0 = threadIdx.x * per, b1 = min(b0 + per, bins);
    int s = 0;
    for (int b = b0; b < b1; ++b) {
        int all = 0, before = 0;
        if constexpr (ONE) {
            for (int w = 0; w < kWaves; ++w) all += lds[w * bins + b];
        } else if constexpr (SUMMED) {
            all = p.total[b];
            before = p.count[(int64_t)tile * bins + b];
        } else {
            for (int t = 0; t < p.tiles; ++t) {
                const int c = p.count[(int64_t)t * bins + b];
                all += c;
                before += t < tile ? c : 0;
            }
        }
        int at_wave = before;
        for (int w = 0; w < kWaves; ++w) {
            const int c = lds[w * bins + b];
            lds[w * bins + b] = at_wave;
            at_wave += c;
        }
        lds[base + b] = s;
        s += all;
    }
    int sum = s;
    for (int o = 1; o < 64; o *= 2) {
        const int v = __shfl_up(sum, o);
        if (lane >= o) sum += v;
    }
    if (lane == 63) sums[wave] = sum;
    __syncthreads();
    int lower = sum - s;
    for (int w = 0; w < wave; ++w) lower += sums[w];
    for (int b = b0; b < b1; ++b) lds[base + b] += lower;
    if (tile == 0) {
        const int all = sums[0] + sums[1] + sums[2] + sums[3];
        if (p.off) {  // (the digit is the network)
            for (int b = b0; b < b1; ++b)
                if (b <= p.G) p.off[b] = lds[base + b];
            if (threadIdx.x == 0) p.off[p.G] = all;
        }
        if (p.have_out && threadIdx.x == 0) *p.have_out = all;
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < kRounds; ++r)
        if (r < rounds && at + r * 64 < n) {
            const int64_t i = at + r * 64;
            const int slot = p.slot ? p.slot[i] : (int)i;
            if (key[r] < 0) {
                if (!p.slot) p.pos[slot] = -1;
                continue;
            }
            const int d = key[r] >> p.shift & (bins - 1);
            const int to = lds[base + d] + lds[mine + d] + rank[r];
            if (p.key_out) {
                p.key_out[to] = key[r];
                p.slot_out[to] = slot;
            } else {
                p.pos[slot] = to;
                if (p.src) p.src[to] = slot;
                if (p.sorted) p.sorted[to] = key[r];
            }
        }
}

// off[g] = the first of the sorted keys that is g or more.
__global__ __launch_bounds__(256) void k_route_bounds(Pass p, int32_t *off)
{
    const int64_t g = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (g > p.G) return;
    int lo = 0, hi = (int)pass_size(p);
    while (lo < hi) {
        const int mid = lo + (hi - lo) / 2;
        if (p.sorted[mid] < g) lo = mid + 1;
        else hi = mid;
    }
    off[g] = lo;
}

struct Scratch {
    int64_t tiles;
    int bins, bits;  // of the widest digit
    int passes;
    size_t count, total, have, key, slot, key2, end;
};
Scratch layout(const RouteArgs &a)
{
    Scratch s{};
    int bits = 0;
    while (((int64_t)1 << bits) < a.G) ++bits;
    s.passes = ((int64_t)1 << bits) <= kMaxBins ? 1 : 2;
    s.bits = s.passes == 1 ? bits : (bits + 1) / 2;
    s.bins = 1 << s.bits;
    s.tiles = (a.n + kTile - 1) / kTile;
    const auto take = [&](size_t ints) {
        const size_t at = s.end;
        s.end += (ints * 4 + 255) / 256 * 256;
        return at;
    };
    s.count = take(s.tiles > 1 ? (size_t)s.tiles * s.bins : 0);
    s.total = take(s.bins);
    s.have = take(1);
    s.key = take(s.passes == 2 ? a.n : 0);
    s.slot = take(s.passes == 2 ? a.n : 0);
    s.key2 = take(s.passes == 2 ? a.n : 0);
    return s;
}

hipError_t run(Pass p, hipStream_t s)
{
    const size_t lds = (size_t)(kWaves + 1) * p.bins * 4;
    if (p.tiles <= 1) hipLaunchKernelGGL((k_route_place<true, false>), dim3(1), dim3(kThreads), lds, s, p);
    else {
        hipLaunchKernelGGL(k_route_count, dim3(p.tiles), dim3(kThreads), 0, s, p);
        if (p.tiles <= kFewTiles) hipLaunchKernelGGL((k_route_place<false, false>), dim3(p.tiles), dim3(kThreads), lds, s, p);
        else {
            hipLaunchKernelGGL(k_route_scan, dim3((p.bins + 15) / 16), dim3(1024), 0, s, p);
            hipLaunchKernelGGL((k_route_place<false, true>), dim3(p.tiles), dim3(kThreads), lds, s, p);
        }
    }
    return hipGetLastError();
}

}  // namespace

size_t route_scratch(const RouteArgs &a) { return layout(a).end; }

hipError_t launch_route(const RouteArgs &a, hipStream_t s)
{
    const Scratch l = layout(a);
    char *m = (char *)a.scratch;
    Pass p{};
    p.key = a.ids;
    p.n = a.n;
    p.G = (int32_t)a.G;
    p.bits = l.bits;
    p.bins = l.bins;
    p.tiles = (int32_t)l.tiles;
    p.count = (int32_t *)(m + l.count);
    p.total = (int32_t *)(m + l.total);
    p.pos = a.pos;
    if (l.passes == 1) {
        p.off = a.off;
        p.src = a.src;
        return run(p, s);
    }
    p.have_out = (int32_t *)(m + l.have);
    p.key_out = (int32_t *)(m + l.key);
    p.slot_out = (int32_t *)(m + l.slot);
    hipError_t e = run(p, s);
    if (e != hipSuccess) return e;
    p.have = p.have_out;
    p.have_out = nullptr;
    p.key = p.key_out;
    p.slot = p.slot_out;
    p.shift = l.bits;
    p.key_out = nullptr;
    p.slot_out = nullptr;
    p.src = a.src;
    p.sorted = (int32_t *)(m + l.key2);
    if ((e = run(p, s)) != hipSuccess) return e;
    hipLaunchKernelGGL(k_route_bounds, dim3((unsigned)((a.G + 256) / 256)), dim3(256), 0, s, p, a.off);
    return hipGetLastError();
}

}  // namespace evox
