// One AdamW step over a list of tensors:
//     m = b1 m + (1 - b1) g,   v = b2 v + (1 - b2) g^2,
//     p = p - lr wd p - (lr / (1 - b1^t)) m / (sqrt(v) / sqrt(1 - b2^t) + eps)
// with p in its own type or, with a master, in fp32 beside it.
//
// Bound by memory: every number is read once and written once.  The tensors are a table
// in device memory, made once, and tiles are numbered through all of them, so that a step is
// one launch (36 tensors per launch, in the kernel's arguments: 128 small ones 20 us).  The
// step's count is on the device: every block reads it, and the last one that has moves it on.
//
// 8-bit states: a group of 256 elements of a row (or a shorter row's all) is 32
// lanes' (fewer for short rows), 8 elements each; m is e4m3 numbers times the group's
// largest |m| / 448, and of v its root is held the same way: e4m3 spans 2^18 of the
// group's largest number, for v then 2^36.  Rounding is 2^-4 of a number at most where it is
// normal, at least 2^-6 of the scale (1 / 28,672 of the largest), and 2^-10 of the scale below.
// A root above 0 is never rounded to 0, where an m beside it would divide by eps
// alone: it is 2^-9 of the scale at least (1 / 229,376 of the largest), so an element whose gradients
// are below that beside a large one's takes steps that are as much smaller.  The update itself
// is made from the fp32 moments, before they are rounded.
#include "evox_mix.hpp"

namespace evox {

namespace {

constexpr int kPasses = 2;              // groups per lane and tile
constexpr uint32_t kPlaces = 32;        // counters of the blocks that have read the clock, 128 bytes apart
template <int BITS>
inline constexpr int kWidth = BITS == 8 ? 8 : 4;  // elements per lane

// A group is L lanes' elements of a row.
struct Groups {
    int shift;        // L = 2^shift
    int64_t per_row, groups;
};
Groups groups_of(int32_t bits, int64_t rows, int64_t n)
{
    const int E = bits == 8 ? kWidth<8> : kWidth<32>, most = bits == 8 ? 5 : 6;
    Groups g;
    g.shift = 0;
    while (g.shift < most && ((int64_t)E << g.shift) < n) ++g.shift;
    g.per_row = (n + ((int64_t)E << g.shift) - 1) / ((int64_t)E << g.shift);
    g.groups = rows * g.per_row;
    return g;
}
uint32_t tiles_of(const Groups &g) { return (uint32_t)((g.groups + (kPasses * 256 >> g.shift) - 1) / (kPasses * 256 >> g.shift)); }

// A tensor in the table: the caller's, its groups, and a division by the
// groups of a row (n / d = (t + (n - t) / 2) / 2^(s - 1) with t the upper half of n mul,
// Granlund and Montgomery, 1994).
struct Item {
    void *p;
    const void *g;
    void *m, *v;
    float *m_scale, *v_scale, *master;
    int64_t n, ldp, ldg, lds;
    uint32_t groups, per_row, mul;
    uint16_t shift, lanes;
    uint64_t reserved;             // (whole 16 bytes)
};
static_assert(sizeof(Item) % 16 == 0, "the table's items");
struct Step {
    const Item *t;
    const uint32_t *start;         // first tile of each
    int32_t count;
    float beta1, beta2, in1, in2, eps;  // in1, in2: 1 - beta1, 1 - beta2
    float lr, decay, log1, log2;   // the betas' logarithms
    const float *lr_dev;
    int64_t *clock;                // steps done, and blocks of this one that have read it
};

Item item_of(const AdamTensor &t, const Groups &g)
{
    Item x{};
    x.p = t.p;
    x.g = t.g;
    x.m = t.m;
    x.v = t.v;
    x.m_scale = t.m_scale;
    x.v_scale = t.v_scale;
    x.master = t.master;
    x.n = t.n;
    x.ldp = t.ldp;
    x.ldg = t.ldg;
    x.lds = t.lds;
    x.groups = (uint32_t)g.groups;
    x.per_row = (uint32_t)g.per_row;
    x.lanes = (uint16_t)g.shift;
    int s = 0;
    while (((uint64_t)1 << s) < x.per_row) ++s;
    x.shift = (uint16_t)(s ? s - 1 : 0);
    x.mul = (uint32_t)((((((uint64_t)1 << s) - x.per_row) << 32) / x.per_row) + 1);
    return x;
}

template <typename T, int E>
struct Packed {
    typedef T reg __attribute__((ext_vector_type(E)));
    typedef T mem __attribute__((ext_vector_type(E), aligned(sizeof(T))));
};
// What a lane does with its E elements where they pass the row's end: all load the row's
// last E there (no branch, so that all loads are on their way together).
//   OVERLAP  and update and store those; the elements that the lane before has too come out
//            the same (it is of the same group, whose loads all come before its stores)
//   SETTLE   moves them to their places, 0 behind them, and stores what is the row's: where a
//            group has no more than part of one lane's, so that the lane before is of another
//            group, in another wave perhaps, which may have stored already
//   TINY     rows of fewer than E elements, one by one
enum RowEnd { OVERLAP = 0, SETTLE = 1, TINY = 2 };
template <int END, int E, typename T>
__device__ __forceinline__ typename Packed<T, E>::reg get(const T *row, int64_t col, int64_t n)
{
    if constexpr (END != TINY) return __builtin_nontemporal_load(reinterpret_cast<const typename Packed<T, E>::mem *>(row + min(col, n - E)));
    typename Packed<T, E>::reg v;
#pragma unroll
    for (int e = 0; e < E; ++e) v[e] = e < n ? row[e] : (T)0;
    return v;
}
template <int E, typename T>
__device__ __forceinline__ void settle_row(typename Packed<T, E>::reg &v, int64_t col, int64_t n)
{
    const int past = (int)min(col + E - n, (int64_t)E);
    if (past <= 0) return;
#pragma unroll
    for (int b = 1; b < E; b *= 2)
        if (past & b)
#pragma unroll
            for (int j = 0; j + b < E; ++j) v[j] = v[j + b];
#pragma unroll
    for (int j = 0; j < E; ++j)
        if (j >= E - past) v[j] = (T)0;
}
template <int E, typename T>
__device__ __forceinline__ void put(T *p, int n, typename Packed<T, E>::reg v)
{
    if (n >= E) *reinterpret_cast<typename Packed<T, E>::mem *>(p) = v;
    else
#pragma unroll
        for (int e = 0; e < E; ++e)
            if (e < n) p[e] = v[e];
}

typedef Packed<uint8_t, 8>::reg Bytes8;
__device__ __forceinline__ void from8(Bytes8 bytes, float scale, float *v)
{
    const uint2 b = __builtin_bit_cast(uint2, bytes);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int w = (int)(i ? b.y : b.x);
        const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8(w, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(w, true);
        v[4 * i] = lo[0] * scale;
        v[4 * i + 1] = lo[1] * scale;
        v[4 * i + 2] = hi[0] * scale;
        v[4 * i + 3] = hi[1] * scale;
    }
}
// The group's scale, and its numbers by it.  What is below 2^-100 counts as 0; infinities
// and NaN count for nothing in it (*odd: some lane of the wave has one) and are held as NaN.
// L: lanes of the group.
__device__ __forceinline__ float scale8(const float *v, int L, float *ratio, bool *odd)
{
    float most = 0.0f;  // NaN if one is
#pragma unroll
    for (int e = 0; e < 8; ++e) most = __builtin_elementwise_maximum(most, fabsf(v[e]));
    *odd = __any(!(most < INFINITY));
    if (*odd) {
        most = 0.0f;
#pragma unroll
        for (int e = 0; e < 8; ++e) most = fabsf(v[e]) < INFINITY ? fmaxf(most, fabsf(v[e])) : most;
    }
    const float m = __uint_as_float(lanes_max(__float_as_uint(most), L));
    *ratio = m > 0x1p-100f ? 448.0f / m : 0.0f;  // (rounded once: its error is all of the group's)
    return m * (1.0f / 448.0f);
}
template <bool ROOT>
__device__ __forceinline__ Bytes8 to8(const float *v, float ratio, bool odd)
{
    float q[8], least = 1.0f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        q[e] = v[e] * ratio;
        if (ROOT) least = fminf(least, q[e]);
    }
    if (ROOT && least < 0x1p-9f)
#pragma unroll
        for (int e = 0; e < 8; ++e) q[e] = v[e] > 0.0f ? fmaxf(q[e], 0x1p-9f) : q[e];
    if (odd)
#pragma unroll
        for (int e = 0; e < 8; ++e) q[e] = fabsf(v[e]) < INFINITY ? q[e] : __builtin_nanf("");
    uint32_t b[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int w = __builtin_amdgcn_cvt_pk_fp8_f32(q[4 * i], q[4 * i + 1], 0, false);
        b[i] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(q[4 * i + 2], q[4 * i + 3], w, true);
    }
    return __builtin_bit_cast(Bytes8, make_uint2(b[0], b[1]));
}

// The constants of a step: m = beta1 m + in1 g, v = beta2 v + in2 g^2, p - shrink p -
// m / (r root + eps) with r the root of v and the rate in root and eps.  Of 8 bits the scales take
// the betas, m's once and v's squared, and the codes are exact (v's over 2^8, their scale times it,
// so that the square of a scale is no nearer to 0 than v): a rounding less on the larger term than
// by the numbers that they stand for, squared.  Of 805 million numbers m has 2827 and v 108 next to
// another e4m3 number than in 64 bits; by those numbers 2976 and 137.
struct Rates {
    float beta1, beta2, in1, in2, root, eps, shrink;
};

// A lane's elements through the step, from their registers into them.
template <typename T, int BITS, bool MASTER>
struct Lane {
    static constexpr int E = kWidth<BITS>;
    typedef typename std::conditional<MASTER, float, T>::type P;      // what is updated: p or its master
    typedef typename std::conditional<BITS == 8, uint8_t, float>::type S;
    typename Packed<P, E>::reg p;
    typename Packed<T, E>::reg g;
    typename Packed<S, E>::reg m, v;
    float m_scale, v_scale;

    __device__ __forceinline__ void step(const Rates &a, int L)
    {
        float m1[E], v1[E], r[E];
        float sm = 0.0f;
        if constexpr (BITS == 8) {
            const float wide = v_scale * 0x1p8f, sv = wide * wide * a.beta2;
            sm = m_scale * a.beta1;
            from8(m, 1.0f, m1);
            from8(v, 0x1p-8f, r);
#pragma unroll
            for (int e = 0; e < E; ++e) v1[e] = r[e] * r[e] * sv;
        } else {
#pragma unroll
            for (int e = 0; e < E; ++e) {
                m1[e] = m[e] * a.beta1;
                v1[e] = v[e] * a.beta2;
            }
        }
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const float x = (float)p[e], d = (float)g[e];
            m1[e] = BITS == 8 ? fmaf(m1[e], sm, d * a.in1) : fmaf(d, a.in1, m1[e]);
            v1[e] = fmaf(d * a.in2, d, v1[e]);
            r[e] = __builtin_amdgcn_sqrtf(v1[e]);
            p[e] = (P)fmaf(m1[e], __builtin_amdgcn_rcpf(fmaf(r[e], a.root, a.eps)), fmaf(x, -a.shrink, x));
        }
        if constexpr (BITS == 8) {
            float mr, vr;
            bool mo, vo;
            m_scale = scale8(m1, L, &mr, &mo);
            v_scale = scale8(r, L, &vr, &vo);
            m = to8<false>(m1, mr, mo);
            v = to8<true>(r, vr, vo);
        } else {
#pragma unroll
            for (int e = 0; e < E; ++e) {
                m[e] = m1[e];
                v[e] = v1[e];
            }
        }
    }
    __device__ __forceinline__ typename Packed<T, E>::reg rounded() const
    {
        typename Packed<T, E>::reg low;
#pragma unroll
        for (int e = 0; e < E; ++e) low[e] = (T)p[e];
        return low;
    }
};

template <typename T, int BITS, bool MASTER>
__global__ __launch_bounds__(256) void k_adamw(const Step a)
{
    typedef Lane<T, BITS, MASTER> Mine;
    typedef typename Mine::P P;
    typedef typename Mine::S S;
    constexpr int E = Mine::E;
    const int64_t done = __hip_atomic_load(a.clock, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    // the tensor of this tile: the last that starts at it or before (64 probes at a time)
    int lo = 0, hi = a.count;
    uint32_t begin = 0;
    while (hi - lo > 1) {
        const int step = (hi - lo + 63) / 64, at = lo + (int)(threadIdx.x % 64) * step;
        const uint32_t first = a.start[min(at, hi - 1)];
        const int n = __popcll(__ballot(at < hi && first <= blockIdx.x));
        begin = __builtin_amdgcn_readlane(first, n - 1);
        lo += (n - 1) * step;
        hi = min(lo + step, hi);
    }
    lo = __builtin_amdgcn_readfirstlane(lo);
    const Item x = a.t[lo];
    const uint32_t index = blockIdx.x - begin;

    // The step's number and what it makes of the constants, asked for after the first loads
    // are on their way; 1 - b^t = -expm1(t log b) (fp32: within 3 roundings of it).  Once every
    // thread has it (the barrier) the block counts itself: in one of 32 places, whose last
    // block counts the place (one place for 1554 blocks: 44 us of 97).
    const auto rates_of = [&]() {
        asm volatile("" ::"v"((uint32_t)done));  // (here it is in a register: the load is done)
        const int64_t t = max(done + 1, (int64_t)1);
        __syncthreads();
        if (threadIdx.x == 0) {
            const uint32_t place = blockIdx.x % kPlaces, mates = (gridDim.x - place + kPlaces - 1) / kPlaces;
            uint32_t *of = (uint32_t *)(a.clock + 16 * (1 + place)), *all = (uint32_t *)(a.clock + 1);
            const auto count = [](uint32_t *c) { return __hip_atomic_fetch_add(c, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); };
            if (count(of) == mates - 1) {
                *of = 0;
                if (count(all) == min(gridDim.x, kPlaces) - 1) {
                    *all = 0;
                    a.clock[0] = t;
                }
            }
        }
        const float lr = a.lr_dev ? *a.lr_dev : a.lr;
        // (the quotient's sign is the rate's; a rate of 0, or one whose reciprocal is not a
        // number of any use, is an infinite divisor)
        const float rate = lr / expm1f((float)t * a.log1), turn = 1.0f / rate;
        const bool some = fabsf(rate) > 1e-30f;
        // (an eps whose quotient is below 2^-126 counts as that: the reciprocal of less is infinite,
        // and m = 0 by it no number)
        const float eps = copysignf(fmaxf(fabsf(turn * a.eps), 0x1p-126f), turn);
        return Rates{a.beta1, a.beta2, a.in1, a.in2, some ? turn / sqrtf(-expm1f((float)t * a.log2)) : 0.0f,
                     some ? eps : INFINITY, lr * a.decay};
    };
    if (x.groups == 0) {  // (a table without elements is one tile of nothing: the count moves on)
        rates_of();
        return;
    }

    constexpr int kElements = kPasses * 256 * E;
    if (x.per_row == x.groups && (int64_t)(index + 1) * kElements <= x.n) {
        // Within a tensor of one row: no ends to look at, addresses that differ by the lane
        // alone.  Streamed past the caches: bf16 with 8-bit states, 100.7 million elements 166 us,
        // 6.1 TB/s, 192 with cached stores, 215 with cached loads too (and then as long with next
        // to no arithmetic); f32, 16.8 million 78 us, 6.0 TB/s, 85 with cached stores.
        const int64_t base = (int64_t)index * kElements;
        const T *g = (const T *)x.g + base;
        T *p = (T *)x.p + base;
        P *q = MASTER ? (P *)x.master + base : (P *)p;
        S *m = (S *)x.m + base, *v = (S *)x.v + base;
        float *ms = x.m_scale + base / kAdamBlock, *vs = x.v_scale + base / kAdamBlock;
        const auto load = [&](Mine &l, int u) {
            const uint32_t i = (u * 256 + threadIdx.x) * E;
            l.g = __builtin_nontemporal_load((const typename Packed<T, E>::mem *)(g + i));
            l.p = __builtin_nontemporal_load((const typename Packed<P, E>::mem *)(q + i));
            l.m = __builtin_nontemporal_load((const typename Packed<S, E>::mem *)(m + i));
            l.v = __builtin_nontemporal_load((const typename Packed<S, E>::mem *)(v + i));
            if constexpr (BITS == 8) {
                l.m_scale = ms[i / kAdamBlock];
                l.v_scale = vs[i / kAdamBlock];
            }
        };
        const auto stream = [](auto *to, auto v) {
            typedef typename Packed<typename std::remove_pointer<decltype(to)>::type, E>::mem mem;
            __builtin_nontemporal_store((mem)v, (mem *)to);
        };
        Mine ls[kPasses];
#pragma unroll
        for (int u = 0; u < kPasses; ++u) load(ls[u], u);
        __builtin_amdgcn_sched_barrier(0);
        const Rates rates = rates_of();
#pragma unroll
        for (int u = 0; u < kPasses; ++u) {
            Mine &l = ls[u];
            const uint32_t i = (u * 256 + threadIdx.x) * E;
            l.step(rates, 32);
            stream(m + i, l.m);
            stream(v + i, l.v);
            stream(q + i, l.p);
            if constexpr (MASTER)
                stream(p + i, l.rounded());
            if constexpr (BITS == 8)
                if (threadIdx.x % 32 == 0) {
                    ms[i / kAdamBlock] = l.m_scale;
                    vs[i / kAdamBlock] = l.v_scale;
                }
        }
        return;
    }

    const int shift = x.lanes, lane = threadIdx.x & ((1 << shift) - 1);
    const auto passes = [&](auto end) {
        constexpr int END = decltype(end)::value;
        Mine ls[kPasses];
        uint32_t groups[kPasses];
        int64_t ops[kPasses], oss[kPasses], cols[kPasses];  // the rows' places in p and in the states, the lane's in the row
#pragma unroll
        for (int u = 0; u < kPasses; ++u) {
            Mine &l = ls[u];
            uint32_t &group = groups[u];
            int64_t &op = ops[u], &os = oss[u], &col = cols[u];
            group = (index * kPasses + u) * (256 >> shift) + (threadIdx.x >> shift);
            const uint32_t gr = min(group, x.groups - 1);
            uint32_t r = 0;
            if (x.per_row == 1) r = gr;
            else if (x.per_row != x.groups) {
                const uint32_t d = __umulhi(gr, x.mul);
                r = (d + ((gr - d) >> 1)) >> x.shift;
            }
            int64_t og = 0;
            op = os = 0;
            if (x.per_row != x.groups) {
                op = r * x.ldp;
                og = r * x.ldg;
                os = r * x.lds;
            }
            col = ((int64_t)(gr - r * x.per_row) << shift | lane) * E;
            l.g = get<END, E>((const T *)x.g + og, col, x.n);
            l.p = get<END, E>(MASTER ? (const P *)x.master + os : (const P *)x.p + op, col, x.n);
            l.m = get<END, E>((const S *)x.m + os, col, x.n);
            l.v = get<END, E>((const S *)x.v + os, col, x.n);
            if constexpr (BITS == 8) {
                l.m_scale = x.m_scale[gr];
                l.v_scale = x.v_scale[gr];
            }
        }
        __builtin_amdgcn_sched_barrier(0);
        const Rates rates = rates_of();
#pragma unroll
        for (int u = 0; u < kPasses; ++u) {
            Mine &l = ls[u];
            const uint32_t group = groups[u];
            const bool live = group < x.groups;
            const int64_t op = ops[u], os = oss[u];
            int64_t col = cols[u];
            int n = live ? (int)min(max(x.n - col, (int64_t)0), (int64_t)E) : 0;
            if constexpr (END == OVERLAP) {
                if (n > 0) n = E;
                col = min(col, x.n - E);
            }
            if (END == SETTLE && !__all(n >= E)) {
                settle_row<E, T>(l.g, col, x.n);
                settle_row<E, P>(l.p, col, x.n);
                settle_row<E, S>(l.m, col, x.n);
                settle_row<E, S>(l.v, col, x.n);
            }
            l.step(rates, 1 << shift);
            // (rows rarely start with a cache line: stores of parts of one are put together in the
            // cache, 37.5 us of 4096 rows of 1830, 40.7 past it)
            const auto store = [&](auto *to, auto v) {
                if constexpr (END == OVERLAP) {
                    typedef typename Packed<typename std::remove_pointer<decltype(to)>::type, E>::mem mem;
                    if (n > 0) *(mem *)to = v;
                } else put<E>(to, n, v);
            };
            store((S *)x.m + os + col, l.m);
            store((S *)x.v + os + col, l.v);
            if constexpr (MASTER) {
                store(x.master + os + col, l.p);
                store((T *)x.p + op + col, l.rounded());
            } else store((T *)x.p + op + col, l.p);
            if constexpr (BITS == 8)
                if (live && lane == 0) {
                    x.m_scale[group] = l.m_scale;
                    x.v_scale[group] = l.v_scale;
                }
        }
    };
    const int tail = (int)(x.n & ((E << shift) - 1));  // of the row's last group
    if (x.n < E) passes(std::integral_constant<int, TINY>{});
    else if (tail > 0 && tail < E) passes(std::integral_constant<int, SETTLE>{});
    else passes(std::integral_constant<int, OVERLAP>{});
}

}  // namespace

int64_t adam_groups(int32_t bits, int64_t rows, int64_t n) { return groups_of(bits, rows, n).groups; }

size_t adam_table(int64_t count) { return (size_t)(count + 1) * (sizeof(Item) + 4); }

int64_t adam_fill_table(int32_t bits, const AdamTensor *t, int64_t count, void *host)
{
    // (tensors without elements are empty items whose tile is the next one's too: the search
    // finds the last)
    Item *items = (Item *)host;
    uint32_t *start = (uint32_t *)(items + count + 1);
    int64_t tiles = 0;
    for (int64_t i = 0; i < count; ++i) {
        start[i] = (uint32_t)tiles;
        items[i] = Item{};
        if (t[i].rows == 0 || t[i].n == 0) continue;
        const Groups g = groups_of(bits, t[i].rows, t[i].n);
        items[i] = item_of(t[i], g);
        tiles += tiles_of(g);
        if (tiles > INT32_MAX) return -1;
    }
    items[count] = Item{};
    start[count] = (uint32_t)tiles;
    return tiles;
}

hipError_t launch_adamw(const AdamCall &c, hipStream_t s)
{
    Step a{};
    a.t = (const Item *)c.table;
    a.start = (const uint32_t *)(a.t + c.count + 1);
    a.count = (int32_t)c.count;
    a.lr = (float)c.lr;
    a.decay = (float)c.decay;
    a.log1 = (float)log(c.beta1);  // (of 0: -inf, and 1 - b^t = 1)
    a.log2 = (float)log(c.beta2);
    a.beta1 = (float)c.beta1;
    a.beta2 = (float)c.beta2;
    a.in1 = (float)(1.0 - c.beta1);
    a.in2 = (float)(1.0 - c.beta2);
    a.eps = (float)c.eps;
    a.lr_dev = c.lr_dev;
    a.clock = c.clock;
    if (c.tiles == 0) {  // the empty item behind the others
        a.t += c.count;
        a.count = 1;
    }
    return net_dispatch(c.dtype, [&](auto type) {
        typedef typename NetElement<decltype(type)::value>::type T;
        const dim3 grid(c.tiles == 0 ? 1 : (unsigned)c.tiles), block(256);
        const auto launch = [&](auto bits, auto master) {
            hipLaunchKernelGGL((k_adamw<T, decltype(bits)::value, decltype(master)::value>), grid, block, 0, s, a);
        };
        const auto with = [&](auto master) {
            if (c.bits == 8) launch(std::integral_constant<int, 8>{}, master);
            else launch(std::integral_constant<int, 32>{}, master);
        };
        if constexpr (sizeof(T) == 2) {  // (fp32 parameters are their own)
            if (c.master) with(std::true_type{});
            else with(std::false_type{});
        } else with(std::false_type{});
        return hipGetLastError();
    });
}

}  // namespace evox
