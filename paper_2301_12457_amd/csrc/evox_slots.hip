// Rows of data to the networks' grouping and back: dispatch, combine and combine's
// gradient, over the slots that evox_route has placed.
//
// Bound by memory.  Each works from the row of data's side: a lane has a chunk of 16
// bytes of row t and meets the k rows of the grouping at pos[t][..], so a row of data is
// read or written once however many networks it has, and the sums over its slots
// stay in registers, in the slots' order.
#include "evox_mix.hpp"

namespace evox {

namespace {

// How a row lies over lanes: WAVES, whole ones (the row is then the same in all lanes of a wave,
// and so are its slots), or SPREAD bytes a lane: 16, of shorter rows the largest power of two that
// they have (f16 k 7, 714,000 rows of 7, combine 7 us and gradient 14; 13 and 35 with a lane per row
// and its elements one by one).
constexpr int WAVES = 0;
template <typename T, int SPREAD>
struct Chunk {
    static constexpr int N = (SPREAD == WAVES ? 16 : SPREAD) / (int)sizeof(T);
    typedef T reg __attribute__((ext_vector_type(N)));
    typedef T mem __attribute__((ext_vector_type(N), aligned(sizeof(T))));
};

// Chunk c of a row of n; the last one is the row's last N elements, of which the chunk before has
// some too: two lanes store the same there, and loads and stores need no branch.  NT: past
// the caches.  So are the networks' rows read (PAST): whole waves' that start with lines (bf16 k 8,
// 32,768 rows of 2048 27.8 us, 30.2 through), others where they are more than the last cache holds
// (f32 k 2, 400 MB just written, rows of 2048: 100 us, 115 through; f16 k 8, 160 MB of 1001: 43, 31),
// narrower ones where both hold (f16 2.3 million rows of 64 66 us, 73 through); narrow rows that
// share their lines with the next one's reader do not (of 40 86 us through the caches, 114 past
// them).  Stores of whole waves go past them too (dispatch 219 us, 232 through; f32 20,014 rows of
// 1001 24, 29; combine's y, f16 k 4, 100,000 rows of 1001 168, 202; where all fits the last cache as
// long), of narrower rows not (f16 562,000 rows of 40 35, 54 past).
template <int SPREAD, bool NT, typename T>
__device__ __forceinline__ typename Chunk<T, SPREAD>::reg chunk_of(const T *row, int c, int n)
{
    constexpr int N = Chunk<T, SPREAD>::N;
    typedef typename Chunk<T, SPREAD>::mem mem;
    const mem *p = reinterpret_cast<const mem *>(row + min(c * N, n - N));
    if constexpr (NT) return __builtin_nontemporal_load(p);
    else return *p;
}
template <int SPREAD, bool NT, typename T>
__device__ __forceinline__ void put_chunk(T *row, int c, int n, typename Chunk<T, SPREAD>::reg v)
{
    constexpr int N = Chunk<T, SPREAD>::N;
    typedef typename Chunk<T, SPREAD>::mem mem;
    mem *p = reinterpret_cast<mem *>(row + min(c * N, n - N));
    if constexpr (NT) __builtin_nontemporal_store((mem)v, p);
    else *p = v;
}

// K slots of row t from j0 on: their rows, -1 where there is none, and weights.
template <int K, int SPREAD>
struct Places {
    int32_t m[K];
    float w[K];
    __device__ __forceinline__ Places(const SlotArgs &a, int64_t t, int j0, bool live = true)
    {
#pragma unroll
        for (int j = 0; j < K; ++j) {
            const int64_t at = t * a.k + min(j0 + j, a.k - 1);
            m[j] = live && j0 + j < a.k ? a.pos[at] : -1;
            w[j] = a.w ? a.w[at] : 1.0f;
        }
#pragma unroll
        for (int j = 0; j < K; ++j) {
            if (m[j] >= a.M) m[j] = -1;
            if constexpr (SPREAD == WAVES) {
                m[j] = __builtin_amdgcn_readfirstlane(m[j]);
                w[j] = __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(w[j])));
            }
        }
    }
};

// The row of this lane's group of L, over 256 threads per block.
template <int SPREAD>
__device__ __forceinline__ int64_t row_of(int L)
{
    const int in_block = threadIdx.x / L;
    return net_block() * (256 / L) + (SPREAD == WAVES ? __builtin_amdgcn_readfirstlane(in_block) : in_block);
}

// Stores to many long rows at a time go faster from fewer blocks at once, 32 KB of LDS that nothing
// uses for each (five per CU): from two 310 us, from eight 248, from five 238 (bf16 262,144 rows of
// 2048, with the sort), from blocks that go on from row to row 240 (1280) to 298 (768).  Taken by what a
// row of data stores, as measured on 12,000 and 16,384 rows in 41 lengths and counts, with it and without:
// bf16 rows of 1152, k 8 55 us and 60, k 12 80 and 89, of 1536, k 5 45 and 48, of 2048, k 8 100 and 102,
// k 20 188 and 189; below the borders, not: of 1152, k 5 43 and 33, k 6 47 and 43, k 9 53 and 50.  By
// lines (k_dispatch_lines) of 16 bits also not where a round has five slots or fewer: f16 rows of 2047, k 5
// 82 and 79, k 9 115 and 108, but k 6 88 and 95, of 1029, k 8 67 and 73; f32 ones gain
// at few (of 545, k 5 42 and 47) and else differ by 2 %.  Up to 4096 rows all is the same.
// The stores bound it: of bf16 262,144 x 2048 in the rows' own order 204 us, in the sorted one 225,
// by chance 234; the floor is 186.
constexpr int kFewBlocksLds = 32768;
template <typename T>
bool few_blocks(const SlotArgs &a, bool lines)
{
    const int rounds = (a.k + 7) / 8;
    if (a.T < 8192) return false;
    if (lines && sizeof(T) == 4) return true;
    if (lines && 2 * a.k < 11 * rounds) return false;
    return a.k * a.D * (int64_t)sizeof(T) >= (rounds == 1 ? 15360 : 23040);
}

// Rows that do not start with a line, over whole waves: chunks are counted from the line in
// which the row of the grouping starts, so that all stores but the row's first and last are
// of whole lines, and each slot loads its own from the row of data, which the L1 has (bf16 k 8,
// 146,408 rows of 2049 146 us, 171 by the row of data's own chunks; f32 k 2, 73,206 164, 185;
// rows of up to a wave's 1 KB are as long or longer: of 257 246, 239).
constexpr int kLine = 128;
template <typename T, int K>
__device__ __forceinline__ void put_lines(const SlotArgs &a, const T *x, const Places<K, WAVES> &p, int lane, int L)
{
    constexpr int N = NetVec<T>::N;
    typedef typename NetVec<T>::mem mem;
    const int D = (int)a.D;
    int before[K];
#pragma unroll
    for (int j = 0; j < K; ++j) before[j] = (int)((uintptr_t)((T *)a.out + p.m[j] * a.ldo) % kLine / sizeof(T));
    for (int c = lane * N; c < D + kLine / (int)sizeof(T) - 1; c += L * N) {
        typename NetVec<T>::reg v[K];
#pragma unroll
        for (int j = 0; j < K; ++j) v[j] = *reinterpret_cast<const mem *>(x + min(max(c - before[j], 0), D - N));
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int j = 0; j < K; ++j) {
            if (p.m[j] < 0) continue;
            auto o = v[j];
            if (a.w)
#pragma unroll
                for (int e = 0; e < N; ++e) o[e] = (T)(p.w[j] * (float)v[j][e]);
            const int at = c - before[j];
            if (at > -N && at < D)
                __builtin_nontemporal_store((mem)o, reinterpret_cast<mem *>((T *)a.out + p.m[j] * a.ldo + min(max(at, 0), D - N)));
        }
    }
}
template <typename T>
bool by_lines(const SlotArgs &a, int L)
{
    return L > 64 && ((uintptr_t)a.out | a.ldo * sizeof(T)) % kLine;
}
template <typename T, int K>
__global__ __launch_bounds__(256) void k_dispatch_lines(SlotArgs a, int L)
{
    const int64_t t = row_of<WAVES>(L);
    if (t >= a.T) return;
    for (int j0 = 0; j0 < a.k; j0 += K)
        put_lines(a, (const T *)a.x + t * a.ldx, Places<K, WAVES>(a, t, j0), threadIdx.x & (L - 1), L);
}

template <typename T, int K, int SPREAD>
__global__ __launch_bounds__(256) void k_dispatch(SlotArgs a, int L)
{
    constexpr int N = Chunk<T, SPREAD>::N;
    const int lane = threadIdx.x & (L - 1), D = (int)a.D;
    const int64_t t = row_of<SPREAD>(L);
    if (t >= a.T) return;
    const T *x = (const T *)a.x + t * a.ldx;
    for (int j0 = 0; j0 < a.k; j0 += K) {
        const Places<K, SPREAD> p(a, t, j0);
        for (int c = lane; c * N < D; c += L) {
            const auto v = chunk_of<SPREAD, false>(x, c, D);
#pragma unroll
            for (int j = 0; j < K; ++j) {
                if (p.m[j] < 0) continue;
                auto o = v;
                if (a.w)
#pragma unroll
                    for (int e = 0; e < N; ++e) o[e] = (T)(p.w[j] * (float)v[e]);
                put_chunk<SPREAD, SPREAD == WAVES>((T *)a.out + p.m[j] * a.ldo, c, D, o);
            }
        }
    }
}

template <typename T, int K, int SPREAD, bool PAST>
__global__ __launch_bounds__(256) void k_combine(SlotArgs a, int L)
{
    constexpr int N = Chunk<T, SPREAD>::N;
    typedef typename Chunk<T, SPREAD>::reg reg;
    const int lane = threadIdx.x & (L - 1), D = (int)a.D;
    const int64_t t = row_of<SPREAD>(L);
    if (t >= a.T) return;
    const Places<K, SPREAD> first(a, t, 0);
    for (int c = lane; c * N < D; c += L) {
        reg r;
        if (a.x) r = chunk_of<SPREAD, false>((const T *)a.x + t * a.ldx, c, D);
        float s[N];
#pragma unroll
        for (int e = 0; e < N; ++e) s[e] = 0.0f;
        const auto add = [&](const Places<K, SPREAD> &p) {
            reg v[K];
#pragma unroll
            for (int j = 0; j < K; ++j)
                if (p.m[j] >= 0) v[j] = chunk_of<SPREAD, PAST>((const T *)a.xs + p.m[j] * a.lds, c, D);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int j = 0; j < K; ++j)
                if (p.m[j] >= 0)
#pragma unroll
                    for (int e = 0; e < N; ++e) s[e] = fmaf(p.w[j], (float)v[j][e], s[e]);
        };
        add(first);
        for (int j0 = K; j0 < a.k; j0 += K) add(Places<K, SPREAD>(a, t, j0));
        if (a.x)
#pragma unroll
            for (int e = 0; e < N; ++e) s[e] += (float)r[e];
        reg o;
#pragma unroll
        for (int e = 0; e < N; ++e) o[e] = (T)s[e];
        T *y = (T *)a.y + t * a.ldy;
        const int twice = c * N + N - D;
        if (a.x == a.y && twice > 0) {
            // r in y's place: of what the chunk before has too, r may be gone by now
#pragma unroll
            for (int e = 0; e < N; ++e)
                if (e >= twice) y[D - N + e] = o[e];
        } else put_chunk<SPREAD, SPREAD == WAVES>(y, c, D, o);
    }
}

// dw, and dxs where given.  A row lies over L lanes of a wave or, WIDE, over a block of two
// or four.
template <typename T, int K, int SPREAD, bool PAST, bool WIDE>
__global__ __launch_bounds__(256) void k_combine_grad(SlotArgs a, int L)
{
    constexpr int N = Chunk<T, SPREAD>::N;
    typedef typename Chunk<T, SPREAD>::reg reg;
    __shared__ float lds[2][4][K];
    const int lane = WIDE ? threadIdx.x : threadIdx.x & (L - 1), D = (int)a.D;
    const int64_t t = WIDE ? net_block() : row_of<SPREAD>(L);
    if (WIDE && t >= a.T) return;
    const bool live = t < a.T;
    const T *dy = (const T *)a.x + t * a.ldx;
    int turn = 0;
    for (int j0 = 0; j0 < a.k; j0 += K, turn ^= 1) {
        const Places<K, SPREAD> p(a, live ? t : 0, j0, live);
        float s[K];
#pragma unroll
        for (int j = 0; j < K; ++j) s[j] = 0.0f;
        for (int c = lane; live && c * N < D; c += L) {
            const reg d = chunk_of<SPREAD, false>(dy, c, D);
            reg v[K];
#pragma unroll
            for (int j = 0; j < K; ++j)
                if (p.m[j] >= 0) v[j] = chunk_of<SPREAD, PAST>((const T *)a.xs + p.m[j] * a.lds, c, D);
            __builtin_amdgcn_sched_barrier(0);
            // (of a last chunk, the elements that the one before it has are not this lane's to sum)
            const int twice = c * N + N - D;
            float own[N];
#pragma unroll
            for (int e = 0; e < N; ++e) own[e] = e < twice ? 0.0f : (float)d[e];
#pragma unroll
            for (int j = 0; j < K; ++j) {
                if (p.m[j] < 0) continue;
#pragma unroll
                for (int e = 0; e < N; ++e) s[j] = e < twice ? s[j] : fmaf(own[e], (float)v[j][e], s[j]);
                if (a.out) {
                    auto o = d;
                    if (a.w)
#pragma unroll
                        for (int e = 0; e < N; ++e) o[e] = (T)(p.w[j] * (float)d[e]);
                    put_chunk<SPREAD, SPREAD == WAVES>((T *)a.out + p.m[j] * a.ldo, c, D, o);
                }
            }
        }
#pragma unroll
        for (int j = 0; j < K; ++j) s[j] = lanes_sum(s[j], WIDE ? 64 : L);
        if constexpr (WIDE) {
            const int wave = threadIdx.x / 64;
            if (threadIdx.x % 64 == 0)
#pragma unroll
                for (int j = 0; j < K; ++j) lds[turn][wave][j] = s[j];
            __syncthreads();
#pragma unroll
            for (int j = 0; j < K; ++j) {
                s[j] = lds[turn][0][j] + lds[turn][1][j];
                if (L == 256) s[j] = (s[j] + lds[turn][2][j]) + lds[turn][3][j];
            }
        }
        if (live && lane == 0)
#pragma unroll
            for (int j = 0; j < K; ++j)
                if (j0 + j < a.k) a.dw[t * a.k + j0 + j] = s[j];
    }
}

// dw alone of rows over whole waves, a wave each.  Its lanes add up in four parts what the
// four waves of a block have, so that dw is the same bits with dxs and without.
template <typename T, int K, bool PAST>
__global__ __launch_bounds__(256) void k_combine_dw(SlotArgs a)
{
    constexpr int N = NetVec<T>::N;
    typedef typename NetVec<T>::reg reg;
    const int lane = threadIdx.x % 64, D = (int)a.D;
    const int64_t t = row_of<WAVES>(64);
    if (t >= a.T) return;
    const T *dy = (const T *)a.x + t * a.ldx;
    for (int j0 = 0; j0 < a.k; j0 += K) {
        const Places<K, WAVES> p(a, t, j0);
        float s[4][K];
#pragma unroll
        for (int q = 0; q < 4; ++q)
#pragma unroll
            for (int j = 0; j < K; ++j) s[q][j] = 0.0f;
        for (int c0 = lane; c0 * N < D; c0 += 256)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int c = c0 + 64 * q;
                if (c * N >= D) break;
                const reg d = chunk_of<WAVES, false>(dy, c, D);
                reg v[K];
#pragma unroll
                for (int j = 0; j < K; ++j)
                    if (p.m[j] >= 0) v[j] = chunk_of<WAVES, PAST>((const T *)a.xs + p.m[j] * a.lds, c, D);
                __builtin_amdgcn_sched_barrier(0);
                const int twice = c * N + N - D;
                float own[N];
#pragma unroll
                for (int e = 0; e < N; ++e) own[e] = e < twice ? 0.0f : (float)d[e];
#pragma unroll
                for (int j = 0; j < K; ++j)
                    if (p.m[j] >= 0)
#pragma unroll
                        for (int e = 0; e < N; ++e) s[q][j] = e < twice ? s[q][j] : fmaf(own[e], (float)v[j][e], s[q][j]);
            }
#pragma unroll
        for (int j = 0; j < K; ++j) {
#pragma unroll
            for (int q = 0; q < 4; ++q) s[q][j] = lanes_sum(s[q][j], 64);
            const float sum = ((s[0][j] + s[1][j]) + s[2][j]) + s[3][j];
            if (lane == 0 && j0 + j < a.k) a.dw[t * a.k + j0 + j] = sum;
        }
    }
}

// Elements per lane, and lanes per row up to `most`.
template <typename T>
int chunk_elements(int64_t D)
{
    int n = NetVec<T>::N;
    while (n > D) n /= 2;
    return n;
}
template <typename T>
int row_lanes(int64_t D, int most)
{
    const int64_t n = chunk_elements<T>(D), chunks = (D + n - 1) / n;
    int L = 1;
    while (L < most && L < chunks) L *= 2;
    return L;
}
dim3 row_grid(int64_t T, int L) { return net_grid((T + 256 / L - 1) / (256 / L)); }

// f(integral K, integral spread, integral past): slots at a time, by k, the row's lanes, and
// (READS: rows of the networks are read) whether past the caches.
constexpr int64_t kLastCache = (int64_t)1 << 28;
template <typename T>
int64_t slot_bytes(const SlotArgs &a) { return a.T * a.k * a.D * (int64_t)sizeof(T); }
template <bool READS, typename T, typename F>
hipError_t with_slots(const SlotArgs &a, int L, F &&f)
{
    const auto spread = [&](auto K) {
        const int bytes = chunk_elements<T>(a.D) * (int)sizeof(T);
        const bool even = ((uintptr_t)a.xs | a.lds * sizeof(T)) % kLine == 0, many = slot_bytes<T>(a) >= kLastCache;
        const auto reads = [&](auto spread, bool past) {
            if constexpr (READS) {
                if (past) return f(K, spread, std::true_type{});
            }
            f(K, spread, std::false_type{});
        };
        if (L >= 64) reads(std::integral_constant<int, WAVES>{}, even || many);
        else if (bytes == 16) reads(std::integral_constant<int, 16>{}, even && many);
        else if (bytes == 8) f(K, std::integral_constant<int, 8>{}, std::false_type{});
        else if (bytes == 4) f(K, std::integral_constant<int, 4>{}, std::false_type{});
        else if constexpr (sizeof(T) == 2) f(K, std::integral_constant<int, 2>{}, std::false_type{});
    };
    if (a.k == 1) spread(std::integral_constant<int, 1>{});
    else if (a.k == 2) spread(std::integral_constant<int, 2>{});
    else if (a.k <= 4) spread(std::integral_constant<int, 4>{});
    else spread(std::integral_constant<int, 8>{});
    return hipGetLastError();
}

}  // namespace

hipError_t launch_dispatch(const SlotArgs &a, hipStream_t s)
{
    return net_dispatch(a.dtype, [&](auto type) {
        typedef typename NetElement<decltype(type)::value>::type T;
        const int L = row_lanes<T>(a.D, 256);
        return with_slots<false, T>(a, L, [&](auto K, auto spread, auto past) {
            const bool lines = by_lines<T>(a, L);
            const int lds = decltype(K)::value == 8 && L == 256 && few_blocks<T>(a, lines) ? kFewBlocksLds : 0;
            if (lines)
                hipLaunchKernelGGL((k_dispatch_lines<T, decltype(K)::value>), row_grid(a.T, L), dim3(256), lds, s, a, L);
            else
                hipLaunchKernelGGL((k_dispatch<T, decltype(K)::value, decltype(spread)::value>), row_grid(a.T, L), dim3(256), lds, s, a, L);
        });
    });
}

hipError_t launch_combine(const SlotArgs &a, hipStream_t s)
{
    return net_dispatch(a.dtype, [&](auto type) {
        typedef typename NetElement<decltype(type)::value>::type T;
        // (one or two slots: a chunk for every second lane is worse than two for each; f32 rows of 264
        // 106 us, 88 on 64 lanes; k 7 as long)
        int L = row_lanes<T>(a.D, 256);
        const int64_t chunks = (a.D + NetVec<T>::N - 1) / NetVec<T>::N;
        if (L > 64 && a.k <= 2 && 4 * chunks <= 3 * L) L /= 2;
        return with_slots<true, T>(a, L, [&](auto K, auto spread, auto past) {
            hipLaunchKernelGGL((k_combine<T, decltype(K)::value, decltype(spread)::value, decltype(past)::value>), row_grid(a.T, L), dim3(256), 0, s, a, L);
        });
    });
}

// Of many large rows both results are faster apart, all reads before all writes, though dy is
// read for each: from four slots and what the last cache holds on.  In one kernel and in two, by bytes
// of slots: f16 rows of 4096, k 4 128 MB 60 us and 65, 256 MB 105 and 104, 700 MB 318 and 290; k 2 102 and
// 120, 351 and 364; k 3 101 and 110, 329 and 295; f32 rows of 4096, k 16 61 and 56, 128 and 110, 303 and
// 259; of 1001, k 4 58 and 61, 110 and 119, 340 and 325, k 8 55 and 61, 117 and 118, 321 and 307.
constexpr int kWaveRows = 4096;  // rows that a wave each fills the chip with
hipError_t launch_combine_grad(const SlotArgs &a, hipStream_t s)
{
    if (!a.dw) return launch_dispatch(a, s);  // (the rows alone are a dispatch of dy)
    return net_dispatch(a.dtype, [&](auto type) {
        typedef typename NetElement<decltype(type)::value>::type T;
        const int L = row_lanes<T>(a.D, 256);
        if (a.out && L == 256 && a.k >= 4 && slot_bytes<T>(a) >= kLastCache) {
            SlotArgs dw = a;
            dw.out = nullptr;
            const hipError_t e = launch_combine_grad(dw, s);
            return e == hipSuccess ? launch_dispatch(a, s) : e;
        }
        return with_slots<true, T>(a, L, [&](auto K, auto spread, auto past) {
            constexpr int k = decltype(K)::value;
            constexpr int u = decltype(spread)::value;
            constexpr bool n = decltype(past)::value;
            if (L <= 64) hipLaunchKernelGGL((k_combine_grad<T, k, u, n, false>), row_grid(a.T, L), dim3(256), 0, s, a, L);
            else if constexpr (u == WAVES) {
                if (!a.out && a.T >= kWaveRows) hipLaunchKernelGGL((k_combine_dw<T, k, n>), row_grid(a.T, 64), dim3(256), 0, s, a);
                else hipLaunchKernelGGL((k_combine_grad<T, k, WAVES, n, true>), net_grid(a.T), dim3(L), 0, s, a, L);
            }
        });
    });
}

}  // namespace evox
