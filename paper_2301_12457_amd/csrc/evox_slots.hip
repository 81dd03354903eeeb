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

// load_early past the caches: the networks' rows are read once (bf16 combine of 262,144 rows
// of 2048 225 us without, 212; f16 gradient of 65,536 rows of 4096 246, 223).
template <typename T>
__device__ __forceinline__ typename NetVec<T>::reg load_stream(const T *row, int c, int n)
{
    constexpr int N = NetVec<T>::N;
    if (n < N) return load_chunk(row, c, n, (T)0.0f);
    return __builtin_nontemporal_load(reinterpret_cast<const typename NetVec<T>::mem *>(row + min(c * N, n - N)));
}

// K slots of row t from j0 on: their rows, -1 where there is none, and weights.  UNI: t is
// the same in all lanes of the wave (rows of a wave and more), and so is all of this.
template <int K, bool UNI>
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
            if constexpr (UNI) {
                m[j] = __builtin_amdgcn_readfirstlane(m[j]);
                w[j] = __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(w[j])));
            }
        }
    }
};

// The row of this lane's group of L, over 256 threads per block.
template <bool UNI>
__device__ __forceinline__ int64_t row_of(int L)
{
    const int in_block = threadIdx.x / L;
    return net_block() * (256 / L) + (UNI ? __builtin_amdgcn_readfirstlane(in_block) : in_block);
}

template <typename T, int K, bool UNI>
__global__ __launch_bounds__(256) void k_dispatch(SlotArgs a, int L)
{
    constexpr int N = NetVec<T>::N;
    const int lane = threadIdx.x & (L - 1), D = (int)a.D;
    const int64_t t = row_of<UNI>(L);
    if (t >= a.T) return;
    const T *x = (const T *)a.x + t * a.ldx;
    for (int j0 = 0; j0 < a.k; j0 += K) {
        const Places<K, UNI> p(a, t, j0);
        for (int c = lane; c * N < D; c += L) {
            const auto v = load_chunk(x, c, D, (T)0.0f);
#pragma unroll
            for (int j = 0; j < K; ++j) {
                if (p.m[j] < 0) continue;
                auto o = v;
                if (a.w)
#pragma unroll
                    for (int e = 0; e < N; ++e) o[e] = (T)(p.w[j] * (float)v[e]);
                store_chunk<T, true>((T *)a.out + p.m[j] * a.ldo, c, D, o);
            }
        }
    }
}

template <typename T, int K, bool UNI>
__global__ __launch_bounds__(256) void k_combine(SlotArgs a, int L)
{
    constexpr int N = NetVec<T>::N;
    typedef typename NetVec<T>::reg reg;
    const int lane = threadIdx.x & (L - 1), D = (int)a.D;
    const int64_t t = row_of<UNI>(L);
    if (t >= a.T) return;
    const Places<K, UNI> first(a, t, 0);
    for (int c = lane; c * N < D; c += L) {
        reg r;
        if (a.x) r = load_early((const T *)a.x + t * a.ldx, c, D);
        float s[N];
#pragma unroll
        for (int e = 0; e < N; ++e) s[e] = 0.0f;
        const auto add = [&](const Places<K, UNI> &p) {
            reg v[K];
#pragma unroll
            for (int j = 0; j < K; ++j)
                if (p.m[j] >= 0) v[j] = load_stream((const T *)a.xs + p.m[j] * a.lds, c, D);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int j = 0; j < K; ++j)
                if (p.m[j] >= 0)
#pragma unroll
                    for (int e = 0; e < N; ++e) s[e] = fmaf(p.w[j], (float)v[j][e], s[e]);
        };
        add(first);
        for (int j0 = K; j0 < a.k; j0 += K) add(Places<K, UNI>(a, t, j0));
        if (a.x)
#pragma unroll
            for (int e = 0; e < N; ++e) s[e] += (float)r[e];
        reg o;
#pragma unroll
        for (int e = 0; e < N; ++e) o[e] = (T)s[e];
        settle(o, c, D, (T)0.0f);  // (the row's last chunk was summed where it was loaded)
        store_chunk((T *)a.y + t * a.ldy, c, D, o);
    }
}

// A row lies over L lanes of a wave or, WIDE, over a block.
template <typename T, int K, bool UNI, bool WIDE>
__global__ __launch_bounds__(256) void k_combine_grad(SlotArgs a, int L)
{
    constexpr int N = NetVec<T>::N;
    typedef typename NetVec<T>::reg reg;
    __shared__ float lds[2][4][K];
    const int lane = WIDE ? threadIdx.x : threadIdx.x & (L - 1), D = (int)a.D;
    const int64_t t = WIDE ? net_block() : row_of<UNI>(L);
    if (WIDE && t >= a.T) return;
    const bool live = t < a.T;
    const T *dy = (const T *)a.x + t * a.ldx;
    int turn = 0;
    for (int j0 = 0; j0 < a.k; j0 += K, turn ^= 1) {
        const Places<K, UNI> p(a, live ? t : 0, j0, live);
        float s[K];
#pragma unroll
        for (int j = 0; j < K; ++j) s[j] = 0.0f;
        for (int c = lane; live && c * N < D; c += L) {
            reg d = load_early(dy, c, D), v[K];
            if (a.dw)
#pragma unroll
                for (int j = 0; j < K; ++j)
                    if (p.m[j] >= 0) v[j] = load_stream((const T *)a.xs + p.m[j] * a.lds, c, D);
            __builtin_amdgcn_sched_barrier(0);
            settle(d, c, D, (T)0.0f);
#pragma unroll
            for (int j = 0; j < K; ++j) {
                if (p.m[j] < 0) continue;
                if (a.dw) {
                    settle(v[j], c, D, (T)0.0f);
#pragma unroll
                    for (int e = 0; e < N; ++e) s[j] = fmaf((float)d[e], (float)v[j][e], s[j]);
                }
                if (a.out) {
                    auto o = d;
                    if (a.w)
#pragma unroll
                        for (int e = 0; e < N; ++e) o[e] = (T)(p.w[j] * (float)d[e]);
                    store_chunk<T, true>((T *)a.out + p.m[j] * a.ldo, c, D, o);
                }
            }
        }
        if (!a.dw) continue;
#pragma unroll
        for (int j = 0; j < K; ++j) s[j] = lanes_sum(s[j], WIDE ? 64 : L);
        if constexpr (WIDE) {
            const int wave = threadIdx.x / 64;
            if (threadIdx.x % 64 == 0)
#pragma unroll
                for (int j = 0; j < K; ++j) lds[turn][wave][j] = s[j];
            __syncthreads();
#pragma unroll
            for (int j = 0; j < K; ++j) s[j] = ((lds[turn][0][j] + lds[turn][1][j]) + lds[turn][2][j]) + lds[turn][3][j];
        }
        if (live && lane == 0)
#pragma unroll
            for (int j = 0; j < K; ++j)
                if (j0 + j < a.k) a.dw[t * a.k + j0 + j] = s[j];
    }
}

// Lanes per row: a chunk each, up to `most`.
template <typename T>
int row_lanes(int64_t D, int most)
{
    const int64_t chunks = (D + NetVec<T>::N - 1) / NetVec<T>::N;
    int L = 1;
    while (L < most && L < chunks) L *= 2;
    return L;
}
dim3 row_grid(int64_t T, int L) { return net_grid((T + 256 / L - 1) / (256 / L)); }

// f(integral K, bool UNI): slots at a time, by k, and whether a row takes whole waves.
template <typename F>
hipError_t with_slots(int k, int L, F &&f)
{
    const auto uni = [&](auto K) {
        if (L >= 64) f(K, std::true_type{});
        else f(K, std::false_type{});
    };
    if (k == 1) uni(std::integral_constant<int, 1>{});
    else if (k == 2) uni(std::integral_constant<int, 2>{});
    else if (k <= 4) uni(std::integral_constant<int, 4>{});
    else uni(std::integral_constant<int, 8>{});
    return hipGetLastError();
}

}  // namespace

hipError_t launch_dispatch(const SlotArgs &a, hipStream_t s)
{
    return net_dispatch(a.dtype, [&](auto type) {
        typedef typename NetElement<decltype(type)::value>::type T;
        const int L = row_lanes<T>(a.D, 256);
        return with_slots(a.k, L, [&](auto K, auto uni) {
            hipLaunchKernelGGL((k_dispatch<T, decltype(K)::value, decltype(uni)::value>), row_grid(a.T, L), dim3(256), 0, s, a, L);
        });
    });
}

hipError_t launch_combine(const SlotArgs &a, hipStream_t s)
{
    return net_dispatch(a.dtype, [&](auto type) {
        typedef typename NetElement<decltype(type)::value>::type T;
        const int L = row_lanes<T>(a.D, 256);
        return with_slots(a.k, L, [&](auto K, auto uni) {
            hipLaunchKernelGGL((k_combine<T, decltype(K)::value, decltype(uni)::value>), row_grid(a.T, L), dim3(256), 0, s, a, L);
        });
    });
}

hipError_t launch_combine_grad(const SlotArgs &a, hipStream_t s)
{
    return net_dispatch(a.dtype, [&](auto type) {
        typedef typename NetElement<decltype(type)::value>::type T;
        const int L = row_lanes<T>(a.D, 256);
        return with_slots(a.k, L, [&](auto K, auto uni) {
            constexpr int k = decltype(K)::value;
            constexpr bool u = decltype(uni)::value;
            if (L <= 64) hipLaunchKernelGGL((k_combine_grad<T, k, u, false>), row_grid(a.T, L), dim3(256), 0, s, a, L);
            else if constexpr (u) hipLaunchKernelGGL((k_combine_grad<T, k, true, true>), net_grid(a.T), dim3(256), 0, s, a, 256);
        });
    });
}

}  // namespace evox
