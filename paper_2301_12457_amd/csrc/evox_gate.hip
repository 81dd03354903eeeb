// The gate of a mixture: the k largest logits of every row and their softmax weights,
// and the logits' gradient from the weights'.
//
// Two ways to choose: k rounds over logits that lie in registers (a row over L lanes of a
// wave, a power of two, k at least, so that lane j keeps the j-th choice; above 64 lanes'
// worth over a block; each lane has NIT chunks of 16 bytes), or one pass over the row with
// the best so far sorted over the lanes of a wave or several.  Bound by instructions: bf16 65,536 x 256, k 8, weights
// over all, 815 of a wave for eight rows, 14.1 us (floor 5.8); fp32 keys are of 64 bits.  The
// gradient is bound by memory (f16 20,000 x 1001 17 us, 81 MB, floor 12.5).
#include "evox_mix.hpp"

namespace evox {

namespace {

// Logits as numbers whose order is theirs, ties to the lower column: of 16 bits the
// order in the upper half and 65535 - column below it, of 32 bits the same in 64.  -0 is
// 0, NaN above +inf; kNone and what is below it: not there (-inf).
template <typename T>
struct GateKey {
    typedef uint32_t type;
    static constexpr uint32_t kInf = std::is_same<T, bf16_t>::value ? 0x7f80u : 0x7c00u;
    static constexpr uint32_t kNone = (0x8000u - kInf) << 16 | 0xffffu;

    // a chunk's keys: two logits at a time, o = 0x8000 +- |z|'s bits
    static __device__ __forceinline__ void chunk(typename NetVec<T>::reg v, int column, uint32_t *key)
    {
        typedef short two __attribute__((ext_vector_type(2)));
        typedef unsigned short utwo __attribute__((ext_vector_type(2)));
        const uint4 w = __builtin_bit_cast(uint4, v);
        const uint32_t u[4] = {w.x, w.y, w.z, w.w};
        utwo most = 0;
        const uint32_t below = (0xffffu - (uint32_t)column) * 0x10001u - 0x10000u;  // of both columns of the first pair
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const two sign = __builtin_bit_cast(two, u[i]) >> 15;
            const uint32_t s = __builtin_bit_cast(uint32_t, sign), a = u[i] & 0x7fff7fffu;
            const two o = __builtin_bit_cast(two, a ^ s) - sign;
            const uint32_t order = __builtin_bit_cast(uint32_t, o) ^ 0x80008000u, c = below - 0x20002u * i;
            key[2 * i] = __builtin_amdgcn_perm(order, c, 0x05040100u);
            key[2 * i + 1] = __builtin_amdgcn_perm(order, c, 0x07060302u);
            most = __builtin_elementwise_max(most, __builtin_bit_cast(utwo, a));
        }
        if (max(most[0], most[1]) > kInf)  // a NaN
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if ((u[j / 2] >> j % 2 * 16 & 0x7fffu) > kInf) key[j] = 0xffff0000u | (0xffffu - (uint32_t)column - j);
    }
    static __device__ __forceinline__ int column(uint32_t k) { return (int)(0xffffu - (k & 0xffffu)); }
    static __device__ __forceinline__ float value(uint32_t k)
    {
        const uint32_t o = k >> 16;
        if (o == 0xffffu) return __builtin_nanf("");
        const uint16_t u = (uint16_t)(o >= 0x8000u ? o - 0x8000u : (0x8000u - o) | 0x8000u);
        return (float)__builtin_bit_cast(T, u);
    }
};
template <>
struct GateKey<float> {
    typedef uint64_t type;
    static constexpr uint64_t kNone = (uint64_t)0x00800000u << 32 | 0xffffffffu;

    static __device__ __forceinline__ void chunk(NetVec<float>::reg v, int column, uint64_t *key)
    {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint32_t u = __float_as_uint(v[j]), s = (uint32_t)((int32_t)u >> 31), a = u & 0x7fffffffu;
            const uint32_t o = ((a ^ s) - s) ^ 0x80000000u;
            key[j] = (uint64_t)(a > 0x7f800000u ? 0xffffffffu : o) << 32 | (0xffffffffu - (uint32_t)column - j);
        }
    }
    static __device__ __forceinline__ int column(uint64_t k) { return (int)(0xffffffffu - (uint32_t)k); }
    static __device__ __forceinline__ float value(uint64_t k)
    {
        const uint32_t o = (uint32_t)(k >> 32);
        if (o == 0xffffffffu) return __builtin_nanf("");
        return __uint_as_float(o >= 0x80000000u ? o - 0x80000000u : (0x80000000u - o) | 0x80000000u);
    }
};

// A row's chunks, -inf past its end; whole: the lanes' chunks are the row's exactly.
template <typename T, int NIT>
__device__ __forceinline__ void load_row(const T *z, int lane, int L, int G, bool whole, typename NetVec<T>::reg *v)
{
    constexpr int N = NetVec<T>::N;
    if (whole) {
#pragma unroll
        for (int i = 0; i < NIT; ++i) v[i] = *reinterpret_cast<const typename NetVec<T>::mem *>(z + (lane + i * L) * N);
        return;
    }
    if (G >= N) {
#pragma unroll
        for (int i = 0; i < NIT; ++i) v[i] = load_early(z, lane + i * L, G);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < NIT; ++i) {
            if ((lane + i * L) * N < G) settle<T>(v[i], lane + i * L, G, (T)-INFINITY);
            else
#pragma unroll
                for (int j = 0; j < N; ++j) v[i][j] = (T)-INFINITY;
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < NIT; ++i)
#pragma unroll
        for (int j = 0; j < N; ++j) v[i][j] = (lane + i * L) * N + j < G ? z[j] : (T)-INFINITY;
}

// f(g) with g(z) = e^(z - top) times a factor that all of a row's have.  16 bits: 2^(z log2 e
// - c), c the rounded top log2 e, in one multiply-add (what c is off by is the factor); of
// tops where that would be more than e^0.04, and of fp32, the difference first, factor 1.  The
// row's own top decides, though a wave without such rows computes one form alone: a
// row's bits are not its neighbours' to change.
template <typename T, typename F>
__device__ __forceinline__ void with_exp(float top, F &&f)
{
    if constexpr (sizeof(T) == 2) {
        const float c = top * 1.44269504f;
        const auto near = [=](float z) { return __builtin_amdgcn_exp2f(fmaf(z, 1.44269504f, -c)); };
        const bool large = fabsf(top) >= 0x1p19f && fabsf(top) < INFINITY;  // (of NaN and infinities both are the same)
        if (!__any(large)) f(near);
        else f([=](float z) { return large ? exp_fast(z - top) : near(z); });
    } else f([=](float z) { return exp_near(z - top); });
}

// Over the block of a wide row: the waves meet in LDS (two places in turn, so that one
// barrier is enough).
template <typename V, typename F>
__device__ __forceinline__ V block_all(V v, V *lds, F &&f)
{
    const int wave = threadIdx.x / 64, waves = blockDim.x / 64;
    if (threadIdx.x % 64 == 0) lds[wave] = v;
    __syncthreads();
    v = lds[0];
    for (int w = 1; w < waves; ++w) v = f(v, lds[w]);
    return v;
}

// ---------------------------------------------------------------------------
// The j-th choice is the largest key below the one before it, K: with unsigned wrap,
// key - K of the keys below K is larger than of all others, and the largest of them is
// the nearest, so that a round is one subtraction and half a maximum per logit and
// nothing is marked as taken (k <= G: there is always a key below).
// ---------------------------------------------------------------------------
template <typename T, int NIT, bool WIDE>
__global__ __launch_bounds__(WIDE ? 1024 : 256) void k_gate(GateArgs a, int L, bool whole)
{
    constexpr int N = NetVec<T>::N;
    typedef typename GateKey<T>::type Key;
    __shared__ Key lds_key[WIDE ? 2 : 1][16];
    __shared__ float lds_sum[16];
    const int lane = WIDE ? threadIdx.x : threadIdx.x & (L - 1), G = a.G;
    const int64_t t = WIDE ? net_block() : net_block() * (256 / L) + threadIdx.x / L;
    if (WIDE && t >= a.T) return;  // the whole block
    typename NetVec<T>::reg v[NIT];
    load_row<T, NIT>((const T *)a.z + min(t, a.T - 1) * a.ldz, lane, L, G, whole, v);
    Key key[NIT][N];
#pragma unroll
    for (int i = 0; i < NIT; ++i) GateKey<T>::chunk(v[i], (lane + i * L) * N, key[i]);
    const auto row_max = [&](Key d, int r) {
        d = lanes_max(d, WIDE ? 64 : L);
        if constexpr (WIDE) d = block_all(d, lds_key[r & 1], [](Key x, Key y) { return x > y ? x : y; });
        return d;
    };
    Key K = 0;
#pragma unroll
    for (int i = 0; i < NIT; ++i)
#pragma unroll
        for (int j = 0; j < N; ++j) K = key[i][j] > K ? key[i][j] : K;
    K = row_max(K, 0);
    const Key first = K;
    Key mine = lane == 0 ? K : 0;
    for (int r = 1; r < a.k; ++r) {
        Key d = 0;
#pragma unroll
        for (int i = 0; i < NIT; ++i)
#pragma unroll
            for (int j = 0; j < N; ++j) {
                const Key e = key[i][j] - K;
                d = e > d ? e : d;
            }
        K += row_max(d, r);
        if (lane == r) mine = K;
    }
    const bool there = mine > GateKey<T>::kNone;
    const float top = first > GateKey<T>::kNone ? GateKey<T>::value(first) : 0.0f;
    float e, s;
    with_exp<T>(top, [&](auto above) {
        e = there ? above(GateKey<T>::value(mine)) : 0.0f;
        s = lane < a.k ? e : 0.0f;
        if (a.over == GATE_ALL) {
            s = 0.0f;
#pragma unroll
            for (int i = 0; i < NIT; ++i)
#pragma unroll
                for (int j = 0; j < N; ++j) s += above((float)v[i][j]);
        }
    });
    s = lanes_sum(s, WIDE ? 64 : L);
    if constexpr (WIDE) s = block_all(s, lds_sum, [](float x, float y) { return x + y; });
    if (t < a.T && lane < a.k) {
        a.ids[t * a.k + lane] = there ? GateKey<T>::column(mine) : -1;
        a.w[t * a.k + lane] = there ? e / s : 0.0f;
    }
}

// ---------------------------------------------------------------------------
// Many choices, or long rows: a wave (of few rows several) takes a row in segments of 64 lanes' four chunks and
// keeps the best so far sorted over its lanes.  What is above the k-th of them joins a list of
// up to 64 in LDS (few do after the first segment: of N logits in any order about k ln N);
// a full list is sorted over the lanes and its first 32 merged with the best (32 are k's
// most).  Logits in ascending order, the worst, fill a list with every 64.  The softmax
// over all runs along, each lane with its own maximum.
// ---------------------------------------------------------------------------
// The value of lane ^ M: neighbours and mirrors by DPP, rows and halves by gfx950's swaps.
template <int M>
__device__ __forceinline__ uint32_t lane_xor(uint32_t v)
{
    if constexpr (M == 1) return lane_dpp<0xB1>(v);
    else if constexpr (M == 2) return lane_dpp<0x4E>(v);
    else if constexpr (M == 3) return lane_dpp<0x1B>(v);
    else if constexpr (M == 7) return lane_dpp<0x141>(v);
    else if constexpr (M == 15) return lane_dpp<0x140>(v);
    else if constexpr (M == 4) return lane_xor<3>(lane_xor<7>(v));
    else if constexpr (M == 8) return lane_dpp<0x128>(v);
    else if constexpr (M == 16) {
        const auto r = __builtin_amdgcn_permlane16_swap(v, v, false, false);
        return threadIdx.x & 16 ? r[0] : r[1];
    } else if constexpr (M == 32) {
        const auto r = __builtin_amdgcn_permlane32_swap(v, v, false, false);
        return threadIdx.x & 32 ? r[0] : r[1];
    } else if constexpr (M == 31) return lane_xor<16>(lane_xor<15>(v));
    else return lane_xor<32>(lane_xor<31>(v));  // 63
}
template <int M>
__device__ __forceinline__ uint64_t lane_xor(uint64_t v)
{
    return (uint64_t)lane_xor<M>((uint32_t)(v >> 32)) << 32 | lane_xor<M>((uint32_t)v);
}
// Of lanes l and l ^ M the larger to the one whose bit B is clear.
template <int M, int B, typename Key>
__device__ __forceinline__ Key exchange(Key v)
{
    const Key o = lane_xor<M>(v);
    return (v > o) == !(threadIdx.x & B) ? v : o;
}
// Descending over 2 S lanes: of a bitonic sequence, and of any (S doubling; a mirror makes
// two sorted halves bitonic).
template <int S, typename Key>
__device__ __forceinline__ Key merge_lanes(Key v)
{
    v = exchange<S, S>(v);
    if constexpr (S > 1) v = merge_lanes<S / 2>(v);
    return v;
}
template <int S, typename Key>
__device__ __forceinline__ Key sort_lanes(Key v)
{
    if constexpr (S > 1) v = sort_lanes<S / 2>(v);
    v = exchange<2 * S - 1, S>(v);
    if constexpr (S > 1) v = merge_lanes<S / 2>(v);
    return v;
}
__device__ __forceinline__ uint32_t lane_value(uint32_t v, int l) { return (uint32_t)__builtin_amdgcn_readlane((int)v, l); }
__device__ __forceinline__ uint64_t lane_value(uint64_t v, int l)
{
    return (uint64_t)lane_value((uint32_t)(v >> 32), l) << 32 | lane_value((uint32_t)v, l);
}

// W: waves of a row (1, or a block's), each with its own segments, best and list; the best are
// merged two at a time through LDS.
constexpr int kStreamChunks = 4;  // per lane and segment
template <typename T, int W>
__global__ __launch_bounds__(W == 1 ? 256 : 64 * W) void k_gate_stream(GateArgs a)
{
    constexpr int N = NetVec<T>::N, C = kStreamChunks, kSegment = 64 * C * N;
    typedef typename GateKey<T>::type Key;
    __shared__ Key lists[W == 1 ? 4 : W][64];
    __shared__ float sums[W];
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), G = a.G;
    const int64_t t = W == 1 ? net_block() * 4 + wave : net_block();
    if (t >= a.T) return;  // the whole wave, or block
    const T *z = (const T *)a.z + t * a.ldz;
    Key *list = lists[wave];
    Key best = 0, bar = GateKey<T>::kNone;  // (lanes 0 .. 31), and what is not above it
    int count = 0;
    const auto flush = [&]() {
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        Key v = lane < count ? list[lane] : 0;
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        v = sort_lanes<32>(v);
        v = lane_xor<31>(v);
        best = merge_lanes<16>(v > best ? v : best);
        const Key last = lane_value(best, a.k - 1);
        bar = last > bar ? last : bar;
        count = 0;
    };
    float run = -INFINITY, sum = 0.0f;
    for (int base = W == 1 ? 0 : wave * kSegment; base < G; base += W * kSegment) {
        typename NetVec<T>::reg v[C];
        load_row<T, C>(z + base, lane, 64, G - base, G - base >= kSegment, v);
        if (a.over == GATE_ALL) {
            float top = run;
#pragma unroll
            for (int i = 0; i < C; ++i)
#pragma unroll
                for (int j = 0; j < N; ++j) top = fmaxf(top, (float)v[i][j]);
            const float from = top == -INFINITY ? 0.0f : top;  // (nothing yet: every term 0)
            float s = 0.0f;
#pragma unroll
            for (int i = 0; i < C; ++i)
#pragma unroll
                for (int j = 0; j < N; ++j) {
                    const float x = (float)v[i][j] - from;
                    s += sizeof(T) == 2 ? exp_fast(x) : exp_near(x);
                }
            sum = fmaf(sum, exp_near(run - from), s);
            run = top;
        }
#pragma unroll
        for (int i = 0; i < C; ++i) {
            Key key[N];
            GateKey<T>::chunk(v[i], base + (lane + i * 64) * N, key);
#pragma unroll
            for (int j = 0; j < N; ++j) {
                uint64_t in = __ballot(key[j] > bar);
                if (in == 0) continue;
                if (count + __popcll(in) > 64) {
                    flush();
                    in = __ballot(key[j] > bar);
                }
                if (in >> lane & 1) list[count + __popcll(in & (((uint64_t)1 << lane) - 1))] = key[j];
                count += __popcll(in);
            }
        }
    }
    if (count > 0) flush();
    if constexpr (W > 1) {
        for (int s = 1; s < W; s *= 2) {
            list[lane] = best;
            __syncthreads();
            if (wave % (2 * s) == 0) {
                const Key other = lists[wave + s][lane ^ 31];
                best = merge_lanes<16>(other > best ? other : best);
            }
        }
        if (threadIdx.x == 0) lists[1][0] = best;  // (read by wave 0 alone so far)
        __syncthreads();
    }
    const bool there = lane < a.k && best > GateKey<T>::kNone;
    const Key first = W == 1 ? lane_value(best, 0) : lists[1][0];
    const float top = first > GateKey<T>::kNone ? GateKey<T>::value(first) : 0.0f;
    const float e = there ? exp_near(GateKey<T>::value(best) - top) : 0.0f;
    float s = lanes_sum(a.over == GATE_ALL ? sum * exp_near(run - top) : e, 64);
    if constexpr (W > 1) {
        if (lane == 0) sums[wave] = s;
        __syncthreads();
        if (wave > 0) return;
        if (a.over == GATE_ALL)
            for (int w = 1; w < W; ++w) s += sums[w];
    }
    if (lane < a.k) {
        a.ids[t * a.k + lane] = there ? GateKey<T>::column(best) : -1;
        a.w[t * a.k + lane] = there ? e / s : 0.0f;
    }
}

// ---------------------------------------------------------------------------
// Its gradient: S = sum of w dw; -p S everywhere (over the chosen: 0), then the chosen
// columns' own values behind them, w (dw - S): lane j that of choice j (columns given
// twice get the sum of all their slots, the same in every one's lane).  The block's or
// wave's first values are in memory by then (the fence between).
// ---------------------------------------------------------------------------
// Whether another of the first k lanes (up to 32, and a group of at least as many) has this
// lane's id too, -1 aside: all of them come by in the order of a Gray code, a step an exchange with
// lane ^ a power of two (f16 16,680 x 4261, k 31: 61 us, 100 with every id and share by a permute
// through LDS).
__device__ __forceinline__ bool lane_twice(int id, int k)
{
    uint32_t other = (uint32_t)id;
    bool twice = false;
#pragma unroll
    for (int i = 1; i < 32; ++i) {
        if ((i & (i - 1)) == 0 && i >= k) break;
        other = i & 1 ? lane_xor<1>(other) : i & 2 ? lane_xor<2>(other) : i & 4 ? lane_xor<4>(other) : i & 8 ? lane_xor<8>(other) : lane_xor<16>(other);
        twice |= other == (uint32_t)id;
    }
    return twice && id >= 0;
}

template <typename T, int NIT, bool WIDE>
__global__ __launch_bounds__(WIDE ? 1024 : 256) void k_gate_grad(GateArgs a, int L, bool whole)
{
    constexpr int N = NetVec<T>::N;
    typedef typename NetVec<T>::reg reg;
    __shared__ float lds[3][16];
    const int lane = WIDE ? threadIdx.x : threadIdx.x & (L - 1), G = a.G, k = a.k;
    const int64_t t = WIDE ? net_block() : net_block() * (256 / L) + threadIdx.x / L;
    if (WIDE && t >= a.T) return;
    const bool live = t < a.T;
    T *dz = (T *)a.dz + t * a.lddz;
    const bool all = a.over == GATE_ALL;
    reg v[NIT];
    if (all) load_row<T, NIT>((const T *)a.z + min(t, a.T - 1) * a.ldz, lane, L, G, whole, v);
    int id = -1;
    float w = 0.0f, dw = 0.0f;
    if (live && lane < k) {
        id = a.ids_in[t * k + lane];
        w = a.w_in[t * k + lane];
        dw = a.dw[t * k + lane];
    }
    const auto put = [&]() {
#pragma unroll
        for (int i = 0; i < NIT; ++i)
            if (live && (lane + i * L) * N < G) store_chunk(dz, lane + i * L, G, v[i]);
    };
    if (!all) {  // (before anything waits for the choices)
#pragma unroll
        for (int i = 0; i < NIT; ++i)
#pragma unroll
            for (int j = 0; j < N; ++j) v[i][j] = (T)0.0f;
        put();
    }
    if (live && lane < k) {
        if (id < 0 || id >= G) {
            id = -1;
            w = dw = 0.0f;
        }
    }
    float S = lanes_sum(w * dw, WIDE ? 64 : L);
    const auto add = [](float x, float y) { return x + y; };
    if (all) {
        if constexpr (WIDE) S = block_all(S, lds[0], add);
        float top = -INFINITY;
#pragma unroll
        for (int i = 0; i < NIT; ++i)
#pragma unroll
            for (int j = 0; j < N; ++j) top = fmaxf(top, (float)v[i][j]);
        const auto most = [](float x, float y) { return fmaxf(x, y); };
        top = __uint_as_float(lanes_all(__float_as_uint(top), WIDE ? 64 : L, [](uint32_t x, uint32_t y) {
            return __float_as_uint(fmaxf(__uint_as_float(x), __uint_as_float(y)));
        }));
        if constexpr (WIDE) top = block_all(top, lds[1], most);
        if (top == -INFINITY) top = 0.0f;  // (nothing there: every probability 0)
        // fp32 exponentials take the logits' registers; of 16 bits up to 32 a lane have their own
        float e[NIT][N];
        float total = 0.0f;
#pragma unroll
        for (int i = 0; i < NIT; ++i)
#pragma unroll
            for (int j = 0; j < N; ++j) {
                const float x = (float)v[i][j] - top;
                e[i][j] = sizeof(T) == 2 ? exp_fast(x) : exp_near(x);
                total += e[i][j];
            }
        total = lanes_sum(total, WIDE ? 64 : L);
        if constexpr (WIDE) total = block_all(total, lds[2], add);
        const float f = total == 0.0f ? 0.0f : -S / total;
#pragma unroll
        for (int i = 0; i < NIT; ++i)
#pragma unroll
            for (int j = 0; j < N; ++j) v[i][j] = (T)(f * e[i][j]);
        put();
    }
    // (the choices of a row are lanes of one wave, a wide row's of the first)
    const float share = w * (dw - S);
    float own = share;
    if ((!WIDE || threadIdx.x < 64) && __any(lane_twice(id, k))) {
        own = 0.0f;
        for (int j = 0; j < k; ++j) {
            const int other = __shfl(id, j, WIDE ? 64 : L);
            const float more = __shfl(share, j, WIDE ? 64 : L);
            if (other == id) own += more;
        }
    }
    __threadfence_block();
    if constexpr (WIDE) __syncthreads();
    else __builtin_amdgcn_wave_barrier();
    if (id >= 0) dz[id] = (T)own;
}

// Lanes per row: four chunks each (eight lanes of 32 logits share a round's exchanges and
// bookkeeping among more rows than sixteen of 16), fewer where there are not four waves
// for every SIMD then; at least k lanes.  Rows of more than a wave's over a block.
struct GateShape {
    int L, nit;
    bool wide;
};
template <typename T>
GateShape gate_shape(const GateArgs &a)
{
    constexpr int N = NetVec<T>::N;
    const int chunks = (a.G + N - 1) / N;
    GateShape g{1, 1, chunks > 256};
    if (g.wide) {
        g.L = 256;
        while (g.L < 1024 && chunks > 2 * g.L) g.L *= 2;
        g.nit = 2;
    } else {
        while (g.L < 64 && (chunks > 4 * g.L || (chunks > g.L && a.T * g.L < 64 * 4096))) g.L *= 2;
        while (g.L < a.k) g.L *= 2;
    }
    while (chunks > g.nit * g.L) g.nit *= 2;
    return g;
}
template <typename T, typename F>
hipError_t gate_launch(const GateArgs &a, F &&f)
{
    constexpr int N = NetVec<T>::N;
    const GateShape g = gate_shape<T>(a);
    const dim3 grid = net_grid(g.wide ? a.T : (a.T + 256 / g.L - 1) / (256 / g.L)), block(g.wide ? g.L : 256);
    const bool whole = !g.wide && a.G == g.nit * g.L * N;
    if (g.wide) {
        if (g.nit <= 2) f(std::integral_constant<int, 2>{}, std::true_type{}, grid, block, g.L, whole);
        else if (g.nit <= 4) f(std::integral_constant<int, 4>{}, std::true_type{}, grid, block, g.L, whole);
        else f(std::integral_constant<int, 8>{}, std::true_type{}, grid, block, g.L, whole);
    } else if (g.nit <= 1) f(std::integral_constant<int, 1>{}, std::false_type{}, grid, block, g.L, whole);
    else if (g.nit <= 2) f(std::integral_constant<int, 2>{}, std::false_type{}, grid, block, g.L, whole);
    else f(std::integral_constant<int, 4>{}, std::false_type{}, grid, block, g.L, whole);
    return hipGetLastError();
}

// How a gate is taken: 0 by rounds, else streamed by so many waves a row.  By instructions
// of a wave (fitted to 430 sizes, within 2 % of the fastest in the mean, 30 % at worst): a
// round of the first is s subtractions and maxima, of 64 bits five instructions, and the row's
// exchanges; the second has its segments, a sort or two, little for each choice, and merges.
// Up to 2048 waves run at once at a wave's own pace, 4096 of rows with several at 0.8 of it.  By rounds and
// streamed by 1, 4 and 16 waves: bf16 32,768 x 2048, k 8 40 us and 45, k 32 114 and 58; fp32 256 x
// 8192, k 16 28 us and 21, 11, 10; 1024 x 8192, k 16 71 and 22, 16, 34; 16 x 512, k 2 3.6 and 5.3.
template <typename T>
int gate_streams(const GateArgs &a)
{
    constexpr int N = NetVec<T>::N;
    constexpr bool wide = sizeof(T) == 4;  // (keys of 64 bits)
    const GateShape g = gate_shape<T>(a);
    const int64_t s = (int64_t)g.nit * N, waves = g.wide ? g.L / 64 : 1;
    const int64_t meet = g.wide ? 12 + (wide ? 8 : 2) * waves : (wide ? 25 : 12);
    const int64_t rounds = 5 * s + a.k * (wide ? 5 * s + meet : 3 * s / 2 + meet);
    const int64_t segments = (a.G + 64 * kStreamChunks * N - 1) / (64 * kStreamChunks * N);
    const auto time = [](int64_t c, int64_t w) { return c * (w < 2048 ? 2048 : w); };
    int64_t best = time(rounds, g.wide ? a.T * waves : (a.T * g.L + 63) / 64);
    int choice = 0;
    for (int w = 1, step = 0; w <= 16; w *= 4, step += 2) {
        const int64_t of = (segments + w - 1) / w;
        const int64_t c = (wide ? of * 352 + 370 + 13 * a.k : of * 384 + 240 + 12 * a.k) + step * (wide ? 80 : 50);
        const int64_t all = time(c, w > 1 && a.T * w <= 4096 ? a.T * w * 5 / 8 : a.T * w);
        if (all < best) {
            best = all;
            choice = w;
        }
    }
    return choice;
}

}  // namespace

hipError_t launch_gate(const GateArgs &a, hipStream_t s)
{
    return net_dispatch(a.dtype, [&](auto type) {
        typedef typename NetElement<decltype(type)::value>::type T;
        const int waves = gate_streams<T>(a);
        if (waves == 1) hipLaunchKernelGGL((k_gate_stream<T, 1>), net_grid((a.T + 3) / 4), dim3(256), 0, s, a);
        else if (waves == 4) hipLaunchKernelGGL((k_gate_stream<T, 4>), net_grid(a.T), dim3(256), 0, s, a);
        else if (waves == 16) hipLaunchKernelGGL((k_gate_stream<T, 16>), net_grid(a.T), dim3(1024), 0, s, a);
        if (waves) return hipGetLastError();
        return gate_launch<T>(a, [&](auto nit, auto wide, dim3 grid, dim3 block, int L, bool whole) {
            if constexpr (decltype(wide)::value && sizeof(T) == 2 && decltype(nit)::value == 8) return;  // (four hold any row)
            else hipLaunchKernelGGL((k_gate<T, decltype(nit)::value, decltype(wide)::value>), grid, block, 0, s, a, L, whole);
        });
    });
}

hipError_t launch_gate_grad(const GateArgs &a, hipStream_t s)
{
    return net_dispatch(a.dtype, [&](auto type) {
        typedef typename NetElement<decltype(type)::value>::type T;
        return gate_launch<T>(a, [&](auto nit, auto wide, dim3 grid, dim3 block, int L, bool whole) {
            if constexpr (decltype(wide)::value && sizeof(T) == 2 && decltype(nit)::value == 8) return;
            else hipLaunchKernelGGL((k_gate_grad<T, decltype(nit)::value, decltype(wide)::value>), grid, block, 0, s, a, L, whole);
        });
    });
}

}  // namespace evox
