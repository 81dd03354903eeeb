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

// The place of slot (t, j): -1 where there is no such row.
__device__ __forceinline__ int64_t slot_row(const SlotArgs &a, int64_t t, int j)
{
    const int m = a.pos[t * a.k + j];
    return m >= 0 && m < a.M ? m : -1;
}

template <typename T>
__global__ __launch_bounds__(256) void k_dispatch(SlotArgs a, int L)
{
    constexpr int N = NetVec<T>::N;
    const int lane = threadIdx.x & (L - 1), D = (int)a.D;
    const int64_t t = net_block() * (256 / L) + threadIdx.x / L;
    if (t >= a.T) return;
    const T *x = (const T *)a.x + t * a.ldx;
    for (int c = lane; c * N < D; c += L) {
        const auto v = load_chunk(x, c, D, (T)0.0f);
        for (int j = 0; j < a.k; ++j) {
            const int64_t m = slot_row(a, t, j);
            if (m < 0) continue;
            auto o = v;
            if (a.w) {
                const float w = a.w[t * a.k + j];
#pragma unroll
                for (int e = 0; e < N; ++e) o[e] = (T)(w * (float)v[e]);
            }
            store_chunk((T *)a.out + m * a.ldo, c, D, o);
        }
    }
}

template <typename T>
__global__ __launch_bounds__(256) void k_combine(SlotArgs a, int L)
{
    constexpr int N = NetVec<T>::N;
    const int lane = threadIdx.x & (L - 1), D = (int)a.D;
    const int64_t t = net_block() * (256 / L) + threadIdx.x / L;
    if (t >= a.T) return;
    const T *r = (const T *)a.x + t * a.ldx;
    T *y = (T *)a.y + t * a.ldy;
    for (int c = lane; c * N < D; c += L) {
        float s[N];
#pragma unroll
        for (int e = 0; e < N; ++e) s[e] = 0.0f;
        for (int j = 0; j < a.k; ++j) {
            const int64_t m = slot_row(a, t, j);
            if (m < 0) continue;
            const float w = a.w ? a.w[t * a.k + j] : 1.0f;
            const auto v = load_chunk((const T *)a.xs + m * a.lds, c, D, (T)0.0f);
#pragma unroll
            for (int e = 0; e < N; ++e) s[e] = fmaf(w, (float)v[e], s[e]);
        }
        typename NetVec<T>::reg o;
        if (a.x) {
            const auto v = load_chunk(r, c, D, (T)0.0f);
#pragma unroll
            for (int e = 0; e < N; ++e) s[e] += (float)v[e];
        }
#pragma unroll
        for (int e = 0; e < N; ++e) o[e] = (T)s[e];
        store_chunk(y, c, D, o);
    }
}

// K slots at a time (a row of data is read once for each K of its slots).  A row
// lies over L lanes of a wave or, WIDE, over a block.
template <typename T, int K, bool WIDE>
__global__ __launch_bounds__(256) void k_combine_grad(SlotArgs a, int L)
{
    constexpr int N = NetVec<T>::N;
    __shared__ float lds[2][4][K];
    const int lane = WIDE ? threadIdx.x : threadIdx.x & (L - 1), D = (int)a.D;
    const int64_t t = WIDE ? net_block() : net_block() * (256 / L) + threadIdx.x / L;
    if (WIDE && t >= a.T) return;
    const bool live = t < a.T;
    const T *dy = (const T *)a.x + t * a.ldx;
    int turn = 0;
    for (int j0 = 0; j0 < a.k; j0 += K, turn ^= 1) {
        int64_t m[K];
        float w[K], s[K];
#pragma unroll
        for (int j = 0; j < K; ++j) {
            m[j] = live && j0 + j < a.k ? slot_row(a, t, j0 + j) : -1;
            w[j] = m[j] >= 0 && a.w ? a.w[t * a.k + j0 + j] : 1.0f;
            s[j] = 0.0f;
        }
        for (int c = lane; live && c * N < D; c += L) {
            const auto d = load_chunk(dy, c, D, (T)0.0f);
#pragma unroll
            for (int j = 0; j < K; ++j) {
                if (m[j] < 0) continue;
                if (a.dw) {
                    const auto v = load_chunk((const T *)a.xs + m[j] * a.lds, c, D, (T)0.0f);
#pragma unroll
                    for (int e = 0; e < N; ++e)
                        if (c * N + e < D) s[j] = fmaf((float)d[e], (float)v[e], s[j]);
                }
                if (a.out) {
                    auto o = d;
                    if (a.w)
#pragma unroll
                        for (int e = 0; e < N; ++e) o[e] = (T)(w[j] * (float)d[e]);
                    store_chunk((T *)a.out + m[j] * a.ldo, c, D, o);
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

}  // namespace

hipError_t launch_dispatch(const SlotArgs &a, hipStream_t s)
{
    return net_dispatch(a.dtype, [&](auto type) {
        typedef typename NetElement<decltype(type)::value>::type T;
        const int L = row_lanes<T>(a.D, 256);
        hipLaunchKernelGGL(k_dispatch<T>, row_grid(a.T, L), dim3(256), 0, s, a, L);
        return hipGetLastError();
    });
}

hipError_t launch_combine(const SlotArgs &a, hipStream_t s)
{
    return net_dispatch(a.dtype, [&](auto type) {
        typedef typename NetElement<decltype(type)::value>::type T;
        const int L = row_lanes<T>(a.D, 256);
        hipLaunchKernelGGL(k_combine<T>, row_grid(a.T, L), dim3(256), 0, s, a, L);
        return hipGetLastError();
    });
}

hipError_t launch_combine_grad(const SlotArgs &a, hipStream_t s)
{
    return net_dispatch(a.dtype, [&](auto type) {
        typedef typename NetElement<decltype(type)::value>::type T;
        const int L = row_lanes<T>(a.D, 256);
        const auto launch = [&](auto K) {
            constexpr int k = decltype(K)::value;
            if (L > 64) hipLaunchKernelGGL((k_combine_grad<T, k, true>), net_grid(a.T), dim3(256), 0, s, a, 256);
            else hipLaunchKernelGGL((k_combine_grad<T, k, false>), row_grid(a.T, L), dim3(256), 0, s, a, L);
            return hipGetLastError();
        };
        if (a.k == 1) return launch(std::integral_constant<int, 1>{});
        if (a.k == 2) return launch(std::integral_constant<int, 2>{});
        return launch(std::integral_constant<int, 4>{});
    });
}

}  // namespace evox
