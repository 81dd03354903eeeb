// Slots (row, choice) sorted by network, stably: network g's slots are the rows
// off[g] .. off[g + 1) of the grouping, in the slots' order.
//
// A counting sort.  A wave takes 64 slots at a time, in order: the lanes with the same
// digit are found with a ballot per bit, a slot's rank is the wave's count of its digit
// so far plus the lanes before it, and no atomic decides an order.  Up to 2048 slots are
// one block's.  Of up to 16 tiles of as many each counts all slots itself, in one launch;
// more are counted per tile and placed by a second launch, which adds up the tiles' counts
// itself while they are few, else from a third one between.  Up to 2048 networks are one
// digit, more two digits, the lower first.
//
// Bound by latency: few blocks, and in each a chain of loads, ranks, LDS sums and scattered
// stores (20,014 slots of 100 networks: loads and counts 3.5 us, ranks 2, the digits' places
// 1, stores 1.5).  So a tile is 8 waves' of four rounds where the digits are few (LDS holds a
// count per wave and digit): 16 waves' of 4096 slots 8.4 us, 4 waves' of 1024 7.0, but 11.8
// against 7.9 of 262,144 slots, where each tile adds up four times as many counts; all ballots
// come before the first count, and all loads before both.  Up to 1024 slots, and up to 4096 where
// digits would be wide or two, are ranked by comparison instead.
#include "evox_mix.hpp"

namespace evox {

namespace {

constexpr int kTile = 2048, kMaxBins = 2048;
constexpr int kWideBins = 512;   // digits at most, for 8 waves
constexpr int kSummed = 16384;   // counts of all tiles that each block adds up itself

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

// The networks of a thread's slots i0, i0 + step, ..: -1 for none and past the end, n.
// All loads first (those past the end are of the last slot, and nothing is looked at
// before the last is on its way).
template <int ROUNDS>
__device__ __forceinline__ void slot_keys(const Pass &p, int64_t base, int i0, int step, int64_t n, int *key)
{
    const int last = (int)min(n - base, (int64_t)kTile) - 1;
    if (last < 0) {
#pragma unroll
        for (int r = 0; r < ROUNDS; ++r) key[r] = -1;
        return;
    }
    const int32_t *k = p.key + base;
#pragma unroll
    for (int r = 0; r < ROUNDS; ++r) key[r] = k[min(i0 + r * step, last)];
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int r = 0; r < ROUNDS; ++r) key[r] = i0 + r * step <= last && key[r] >= 0 && key[r] < p.G ? key[r] : -1;
}

template <int W>
__global__ __launch_bounds__(64 * W) void k_route_count(Pass p)
{
    constexpr int threads = 64 * W, rounds = kTile / threads;
    __shared__ int hist[W == 8 ? kWideBins : kMaxBins];
    for (int b = threadIdx.x; b < p.bins; b += threads) hist[b] = 0;
    const int64_t n = pass_size(p), base = (int64_t)blockIdx.x * kTile;
    int key[rounds];
    slot_keys<rounds>(p, base, threadIdx.x, threads, n, key);
    __syncthreads();
#pragma unroll
    for (int r = 0; r < rounds; ++r)
        if (key[r] >= 0) atomicAdd(&hist[key[r] >> p.shift & (p.bins - 1)], 1);
    __syncthreads();
    for (int b = threadIdx.x; b < p.bins; b += threads) p.count[(int64_t)blockIdx.x * p.bins + b] = hist[b];
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

// Where a tile has the counts of all and of the tiles before it from: it is all (ONE), it
// counts every slot itself (HERE), it adds the tiles' counts (ADDED), or from the scan (SUMMED).
enum Counts { ONE = 0, HERE = 1, ADDED = 2, SUMMED = 3 };

// HERE: each digit has `copies` places, a lane's own as far as they go, so that lanes of
// one digit seldom wait for each other, however the slots lie; in one the slots of earlier
// tiles are counted by 2^16 and the others by 1 (behind the last digit's: of no network).
// By graph replays, 100 networks: 4096 slots 6.3 us, 7.3 (8.8 where one network has them all) by
// two launches; 20,014 7.8, 8.1 (9.5); 32,768 8.8, 7.8 (9.2), where the host has a launch less to make
// (3 us).  2048 digits have two places each, and 32,768 slots of one then take 29 us, 19 by
// three launches: so many are for up to 8 tiles (16,384: 22 and 24).
constexpr int kPlacesHere = 4096, kTilesHere = 16;
typedef int Four __attribute__((ext_vector_type(4), aligned(4)));
constexpr int kBatch = 4;  // loads at a time, of four slots each
__device__ __forceinline__ void load_here(const Pass &p, int q0, int threads, int whole, Four *key)
{
#pragma unroll
    for (int r = 0; r < kBatch; ++r) key[r] = *reinterpret_cast<const Four *>(p.key + 4 * max(min(q0 + r * threads, whole - 1), 0));
}
template <int W>
__device__ __forceinline__ void count_here(const Pass &p, int n, Four *key, int *hist, int *total, int *before)
{
    constexpr int threads = 64 * W;
    const int bins = p.bins, copies = min(kPlacesHere / bins, 64), mine = threadIdx.x & (copies - 1);
    const int first = blockIdx.x * kTile, whole = n / 4;
    const bool single = p.G <= bins;
    const auto one = [&](int k, int by) {
        const int digit = single ? k : k >> p.shift & (bins - 1), d = (uint32_t)k < (uint32_t)p.G ? digit : bins;
        atomicAdd(&hist[d * copies + mine], by);
    };
    for (int q0 = threadIdx.x; q0 < whole;) {
#pragma unroll
        for (int r = 0; r < kBatch; ++r)
            if (q0 + r * threads < whole) {
                const int by = 4 * (q0 + r * threads) < first ? 0x10000 : 1;
#pragma unroll
                for (int e = 0; e < 4; ++e) one(key[r][e], by);
            }
        q0 += threads * kBatch;
        if (q0 < whole) load_here(p, q0, threads, whole, key);
    }
    if ((int)threadIdx.x < n % 4) one(p.key[4 * whole + threadIdx.x], 4 * whole < first ? 0x10000 : 1);
    __syncthreads();
    if (copies >= 8) {
        for (int u = threadIdx.x; u < bins * copies / 8; u += threads) {
            const int4 x = reinterpret_cast<const int4 *>(hist)[2 * u], y = reinterpret_cast<const int4 *>(hist)[2 * u + 1];
            const int s = x.x + x.y + x.z + x.w + y.x + y.y + y.z + y.w, b = u * 8 / copies, early = (int)((uint32_t)s >> 16);
            atomicAdd(&total[b], (s & 0xffff) + early);
            atomicAdd(&before[b], early);
        }
    } else
        for (int b = threadIdx.x; b < bins; b += threads) {
            int s = 0;
            for (int e = 0; e < copies; ++e) s += hist[b * copies + e];
            before[b] = (int)((uint32_t)s >> 16);
            total[b] = (s & 0xffff) + before[b];
        }
    __syncthreads();
    for (int b = threadIdx.x; b < W * bins; b += threads) hist[b] = 0;
    __syncthreads();
}

template <int W, int FROM>
__host__ __device__ constexpr int lds_base(int bins)
{
    return FROM == HERE && W * bins < kPlacesHere + 64 ? kPlacesHere + 64 : W * bins;
}

template <int W, int FROM>
__global__ __launch_bounds__(64 * W) void k_route_place(Pass p)
{
    constexpr int threads = 64 * W, kRounds = kTile / threads;
    extern __shared__ __attribute__((aligned(16))) int lds[];  // counts of the waves, [W][bins]; places, all counts, counts before, [bins] each
    __shared__ int sums[W];
    const int wave = threadIdx.x / 64, lane = threadIdx.x % 64, tile = blockIdx.x, bins = p.bins;
    const int mine = wave * bins, base = lds_base<W, FROM>(bins), total = base + bins, before_at = total + bins;
    const int64_t n = pass_size(p);
    const int64_t first = (int64_t)tile * kTile;
    // rounds of this tile: the waves' shares follow each other
    const int64_t left = n - first;
    const int rounds = left <= 0 ? 0 : left >= kTile ? kRounds : (int)((left + threads - 1) / threads);
    const int at = wave * rounds * 64 + lane;
    int key[kRounds], slot[kRounds];
    Four others[FROM == HERE ? kBatch : 1];
    if constexpr (FROM == HERE) load_here(p, threadIdx.x, threads, (int)n / 4, others);
    slot_keys<kRounds>(p, first, at, 64, n, key);
    if (p.slot && left > 0)
#pragma unroll
        for (int r = 0; r < kRounds; ++r) slot[r] = p.slot[min(first + at + r * 64, n - 1)];
    else
#pragma unroll
        for (int r = 0; r < kRounds; ++r) slot[r] = (int)first + at + r * 64;
    for (int b = threadIdx.x; b < base + 3 * bins; b += threads) lds[b] = 0;
    __syncthreads();
    if constexpr (FROM == HERE) count_here<W>(p, (int)n, others, lds, lds + total, lds + before_at);
    if constexpr (FROM == ADDED) {
        const int wide = min(bins, threads), part = threadIdx.x / wide, parts = threads / wide;
        for (int b = threadIdx.x % wide; b < bins; b += wide) {
            int all = 0, before = 0;
#pragma unroll 4
            for (int t = part; t < p.tiles; t += parts) {
                const int c = p.count[(int64_t)t * bins + b];
                all += c;
                before += t < tile ? c : 0;
            }
            atomicAdd(&lds[total + b], all);
            atomicAdd(&lds[before_at + b], before);
        }
    }
    // the lanes of a slot's digit: how many in all, and before it
    int many[kRounds], rank[kRounds];
#pragma unroll
    for (int r = 0; r < kRounds; ++r)
        if (r < rounds) {
            const int d = key[r] >> p.shift & (bins - 1);
            uint64_t peers = __ballot(key[r] >= 0);
            for (int b = 0; b < p.bits; ++b) {
                const uint64_t set = __ballot(d >> b & 1);
                peers &= d >> b & 1 ? set : ~set;
            }
            rank[r] = __popcll(peers & (((uint64_t)1 << lane) - 1));
            many[r] = __popcll(peers);
        }
#pragma unroll
    for (int r = 0; r < kRounds; ++r)
        if (r < rounds) {
            const int d = key[r] >> p.shift & (bins - 1);
            const int so_far = lds[mine + d];
            // (a wave's LDS accesses stay in their order; the compiler is told to keep it)
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            if (key[r] >= 0 && rank[r] == 0) lds[mine + d] = so_far + many[r];
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            rank[r] += so_far;
        }
    __syncthreads();
    // the digits' places: those of lower digits, of earlier tiles, of earlier waves
    const int per = (bins + threads - 1) / threads, b0 = min((int)threadIdx.x * per, bins), b1 = min(b0 + per, bins);
    int s = 0;
    for (int b = b0; b < b1; ++b) {
        int at_wave = FROM == ONE ? 0 : FROM == SUMMED ? p.count[(int64_t)tile * bins + b] : lds[before_at + b], all = 0, c[W];
#pragma unroll
        for (int w = 0; w < W; ++w) c[w] = lds[w * bins + b];
#pragma unroll
        for (int w = 0; w < W; ++w) {
            lds[w * bins + b] = at_wave;
            at_wave += c[w];
            all += c[w];
        }
        lds[base + b] = s;
        s += FROM == ONE ? all : FROM == SUMMED ? p.total[b] : lds[total + b];
    }
    int sum = s;
    for (int o = 1; o < 64; o *= 2) {
        const int v = __shfl_up(sum, o);
        if (lane >= o) sum += v;
    }
    if (lane == 63) sums[wave] = sum;
    __syncthreads();
    int lower = sum - s, all = 0;
#pragma unroll
    for (int w = 0; w < W; ++w) {
        lower += w < wave ? sums[w] : 0;
        all += sums[w];
    }
    for (int b = b0; b < b1; ++b) lds[base + b] += lower;
    if (tile == 0) {
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
        if (r < rounds && first + at + r * 64 < n) {
            if (key[r] < 0) {
                if (!p.slot) p.pos[slot[r]] = -1;
                continue;
            }
            const int d = key[r] >> p.shift & (bins - 1);
            const int to = lds[base + d] + lds[mine + d] + rank[r];
            if (p.key_out) {
                p.key_out[to] = key[r];
                p.slot_out[to] = slot[r];
            } else {
                p.pos[slot[r]] = to;
                if (p.src) p.src[to] = slot[r];
                if (p.sorted) p.sorted[to] = key[r];
            }
        }
}

// Few slots: a slot's row is the number of (network, slot) pairs below its own, by comparison
// with all, 16 slots a block, each over 16 lanes that share the pairs between them.  They also
// find the next pair above theirs: a network's last slot writes the offsets from its own
// network's to the next one's.  Of n slots in n^2 comparisons: 8 of 256 networks 3.0 us (by digits
// 3.7), 1000 of 512 4.5 (5.8), 2048 of 512 5.8 (5.7), of 8849 6.0 (18.6), 4096 of 1024 8.4 (11.6), of
// 8849 8.6 (19.5); so up to 1024, and up to 4096 where a digit is wide or there are two.  More
// networks than evox_gate chooses from go by digits: the one block of 8 slots of 200,000 24 us.
constexpr int kRank = 4096, kRankAny = 1024, kRankG = 32768, kRankSlots = 16;
constexpr int kRankOf = 12;  // bits of a pair that are the slot's
static_assert(kRank <= 1 << kRankOf && kRankG <= 1 << (30 - kRankOf), "pairs are below INT32_MAX");
__global__ __launch_bounds__(256) void k_route_rank(Pass p)
{
    constexpr int kNone = INT32_MAX;
    __shared__ __attribute__((aligned(16))) int pairs[kRank];
    __shared__ int keys[kRankSlots], ranks[kRankSlots], nexts[kRankSlots];
    const int n = (int)p.n, padded = (n + 63) & ~63, base = blockIdx.x * kRankSlots;
    for (int i = threadIdx.x; i < padded; i += 256) {
        const int key = p.key[min(i, n - 1)];
        pairs[i] = i < n && key >= 0 && key < p.G ? key << kRankOf | i : kNone;
    }
    __syncthreads();
    const int slot = threadIdx.x / 16, part = threadIdx.x % 16, i = base + slot;
    const int mine = i < n ? pairs[i] : kNone;
    int rank = 0;
    uint32_t above = UINT32_MAX;  // the least distance to a pair above, less 1
#pragma unroll 4
    for (int j = 4 * part; j < padded; j += 64) {
        const int4 q = *reinterpret_cast<const int4 *>(&pairs[j]);
        rank += (q.x < mine) + (q.y < mine) + (q.z < mine) + (q.w < mine);
        // (those below, and itself, are 2^31 - 1 away or more)
        above = min(min(above, min((uint32_t)(q.x - mine - 1), (uint32_t)(q.y - mine - 1))),
                    min((uint32_t)(q.z - mine - 1), (uint32_t)(q.w - mine - 1)));
    }
    rank = (int)lanes_all((uint32_t)rank, 16, [](uint32_t a, uint32_t b) { return a + b; });
    above = lanes_all(above, 16, [](uint32_t a, uint32_t b) { return a < b ? a : b; });
    if (part == 0) {
        const bool in = mine != kNone;
        // the network after this one that has slots, or the end: only the last slot of one differs
        const int next = above < (uint32_t)(kNone - mine) ? mine + 1 + (int)above : kNone;
        keys[slot] = in ? mine >> kRankOf : p.G;
        ranks[slot] = rank;
        nexts[slot] = !in ? -1 : next < kNone ? next >> kRankOf : p.G;
        if (i < n) {
            p.pos[i] = in ? rank : -1;
            if (in && p.src) p.src[rank] = i;
        }
    }
    __syncthreads();
    for (int e = 0; e < kRankSlots; ++e) {
        const int key = keys[e], row = ranks[e];
        for (int g = key + 1 + threadIdx.x; g <= nexts[e]; g += 256) p.off[g] = row + 1;
        // the first of all, or (no slot has a network) slot 0
        if (row == 0 && (key < p.G || base + e == 0))
            for (int g = threadIdx.x; g <= key; g += 256) p.off[g] = 0;
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

template <int W>
void run(const Pass &p, hipStream_t s)
{
    const dim3 grid(p.tiles), block(64 * W);
    const auto place = [&](auto from) {
        constexpr int FROM = decltype(from)::value;
        const size_t lds = (size_t)(lds_base<W, FROM>(p.bins) + 3 * p.bins) * 4;
        hipLaunchKernelGGL((k_route_place<W, FROM>), FROM == ONE ? dim3(1) : grid, block, lds, s, p);
    };
    if (p.tiles <= 1) return place(std::integral_constant<int, ONE>{});
    if (p.tiles <= kTilesHere && p.tiles * p.bins <= kSummed) return place(std::integral_constant<int, HERE>{});
    hipLaunchKernelGGL(k_route_count<W>, grid, block, 0, s, p);
    if ((int64_t)p.tiles * p.bins <= kSummed) return place(std::integral_constant<int, ADDED>{});
    hipLaunchKernelGGL(k_route_scan, dim3((p.bins + 15) / 16), dim3(1024), 0, s, p);
    place(std::integral_constant<int, SUMMED>{});
}
hipError_t run(const Pass &p, hipStream_t s)
{
    if (p.bins <= kWideBins) run<8>(p, s);
    else run<4>(p, s);
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
    if (a.n <= (l.passes == 2 || l.bins > kWideBins ? kRank : kRankAny) && a.G <= kRankG) {
        p.off = a.off;
        p.src = a.src;
        hipLaunchKernelGGL(k_route_rank, dim3((unsigned)(a.n == 0 ? 1 : (a.n + kRankSlots - 1) / kRankSlots)), dim3(256), 0, s, p);
        return hipGetLastError();
    }
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
