// The layers' products in tiles (evox_tile.hpp), one element type per
// compilation (-DEVOX_NET_TYPE).
#include "evox_tile.hpp"

namespace evox {

namespace {

typedef NetElement<EVOX_NET_TYPE>::type Elem;

// Blocks in the order of their XCD (block b of a launch runs on XCD b mod 8):
// each XCD takes one contiguous eighth of the units, so neighbouring units
// share its L2.  -1 past the last.
__device__ __forceinline__ int64_t xcd_unit(int64_t units)
{
    const int64_t b = net_block(), per = (units + 7) / 8, u = b % 8 * per + b / 8;
    return b / 8 < per && u < units ? u : -1;
}
int64_t xcd_blocks(int64_t units) { return (units + 7) / 8 * 8; }

// Units in bands of (at most) kBand tiles along j, i next, j within the band
// last: the 32 blocks that an XCD runs at a time share kBand tiles of one operand
// and 32 / kBand of the other.
constexpr int kBand = 4;
__host__ __device__ __forceinline__ int64_t band_of(int64_t tj) { return tj < kBand ? tj : kBand; }
__host__ __device__ __forceinline__ int64_t banded(int64_t tj)  // whole bands' tiles
{
    return (tj + band_of(tj) - 1) / band_of(tj) * band_of(tj);
}
__device__ __forceinline__ void unit_ij(int64_t u, int64_t ti, int64_t tj, int64_t *i, int64_t *j)
{
    const int64_t w = band_of(tj), band = u / (w * ti), in = u - band * (w * ti);
    *i = in / w;
    *j = band * w + in % w;
}

typedef NetVec<Elem>::reg Reg;
typedef NetVec<Elem>::mem Mem;

// n <= N neighbours of a row: added to v, and rounded from v.
__device__ __forceinline__ void add_row(const Elem *p, float *v, int n)
{
    constexpr int N = NetVec<Elem>::N;
    const Reg t = load_chunk(p, 0, n, (Elem)0.0f);
#pragma unroll
    for (int e = 0; e < N; ++e) v[e] += (float)t[e];
}
__device__ __forceinline__ void store_row(Elem *p, const float *v, int n)
{
    constexpr int N = NetVec<Elem>::N;
    Reg t;
#pragma unroll
    for (int e = 0; e < N; ++e) t[e] = (Elem)v[e];
    store_chunk(p, 0, n, t);
}

template <int B>
struct TileShape;
template <>
struct TileShape<64> {
    static constexpr int WI = 1, WJ = 2, sh = 6;
};
template <>
struct TileShape<128> {
    static constexpr int WI = 2, WJ = 2, sh = 7;
};
template <>
struct TileShape<256> {
    [[maybe_unused]] static constexpr int WI = 4, WJ = 2, sh = 8;  // 16 bits
};
template <int B, bool PM, bool QM>
using Product = TileProduct<Elem, PM, QM, B, B, TileShape<B>::WI, TileShape<B>::WJ>;

// y = act(x W^T + b) + r: i = output, j = row, k = input.
template <int B>
__global__ __launch_bounds__(64 * TileShape<B>::WI * TileShape<B>::WJ, 2) void k_linear_tile(LinearArgs a, int64_t ti,
                                                                                     int64_t tj, int64_t units)
{
    __shared__ __attribute__((aligned(16))) char lds[Product<B, false, false>::kLds];
    const int64_t u = xcd_unit(units);
    if (u < 0) return;
    int64_t it, jt;
    unit_ij(u, ti, tj, &it, &jt);
    const NetTile t = net_tile(a.rows, TileShape<B>::sh, jt);
    if (t.g < 0) return;
    const int i0 = (int)it * B, ni = min((int)a.n_out - i0, B), nj = (int)(t.hi - t.lo);
    const int64_t x0 = a.x_shared ? t.lo - t.g * a.rows.n : t.lo;
    const TileOp<Elem> P{(const Elem *)a.w + t.g * a.w_stride + i0 * a.ldw, a.ldw, ni},
        Q{(const Elem *)a.x + x0 * a.ldx, a.ldx, nj};
    Product<B, false, false> p;
    p.run(P, Q, a.n_in, lds);
    const Elem *b = a.b ? (const Elem *)a.b + t.g * a.b_stride + i0 : nullptr;
    p.results(ni, nj, lds, [&](int j, int i, float *v, int n) {
        const int64_t m = t.lo + j;
        if (b) add_row(b + i, v, n);
        if (a.z) store_row((Elem *)a.z + m * a.ldz + i0 + i, v, n);
        act_values<sizeof(Elem) == 2, NetVec<Elem>::N>(a.act, v);
        if (a.r) add_row((const Elem *)a.r + m * a.ldr + i0 + i, v, n);
        store_row((Elem *)a.y + m * a.ldy + i0 + i, v, n);
    });
}

// dx = d W: i = input, j = row, k = output.
template <int B>
__global__ __launch_bounds__(64 * TileShape<B>::WI * TileShape<B>::WJ, 2) void k_linear_dx_tile(LinearGradArgs a, const Elem *d,
                                                                                      int64_t ldd, int64_t ti,
                                                                                      int64_t tj, int64_t units)
{
    __shared__ __attribute__((aligned(16))) char lds[Product<B, true, false>::kLds];
    const int64_t u = xcd_unit(units);
    if (u < 0) return;
    int64_t it, jt;
    unit_ij(u, ti, tj, &it, &jt);
    const NetTile t = net_tile(a.rows, TileShape<B>::sh, jt);
    if (t.g < 0) return;
    const int i0 = (int)it * B, ni = min((int)a.n_in - i0, B), nj = (int)(t.hi - t.lo);
    const TileOp<Elem> P{(const Elem *)a.w + t.g * a.w_stride + i0, a.ldw, ni}, Q{d + t.lo * ldd, ldd, nj};
    Product<B, true, false> p;
    p.run(P, Q, a.n_out, lds);
    p.results(ni, nj, lds, [&](int j, int i, float *v, int n) {
        store_row((Elem *)a.dx + (t.lo + j) * a.lddx + i0 + i, v, n);
    });
}

// dW = d^T x: i = input, j = output, k = row of the network.
template <int B>
__global__ __launch_bounds__(64 * TileShape<B>::WI * TileShape<B>::WJ, 2) void k_linear_dw_tile(LinearGradArgs a, const Elem *d,
                                                                                     int64_t ldd, int64_t ti, int64_t tj,
                                                                                     int64_t units)
{
    __shared__ __attribute__((aligned(16))) char lds[Product<B, true, true>::kLds];
    const int64_t u = xcd_unit(units);
    if (u < 0) return;
    const int64_t per = banded(tj) * ti, g = u / per;
    int64_t it, jt, lo, hi;
    unit_ij(u - g * per, ti, tj, &it, &jt);
    if (jt >= tj) return;
    net_rows(a.rows, g, &lo, &hi);
    const int i0 = (int)it * B, ni = min((int)a.n_in - i0, B), j0 = (int)jt * B, nj = min((int)a.n_out - j0, B);
    const TileOp<Elem> P{(const Elem *)a.x + (a.x_shared ? 0 : lo) * a.ldx + i0, a.ldx, ni}, Q{d + lo * ldd + j0, ldd, nj};
    Product<B, true, true> p;
    p.run(P, Q, hi - lo, lds);
    p.results(ni, nj, lds, [&](int j, int i, float *v, int n) {
        store_row((Elem *)a.dw + g * a.dw_stride + (j0 + j) * a.lddw + i0 + i, v, n);
    });
}

// f(tile side) for size 0, 1, 2.
template <typename F>
hipError_t with_tile(int size, F &&f)
{
    if (size == 0) return f(std::integral_constant<int, 64>{});
    if constexpr (sizeof(Elem) == 2)
        if (size == 2) return f(std::integral_constant<int, 256>{});
    return f(std::integral_constant<int, 128>{});
}
template <typename G, typename K, typename... A>
hipError_t launch_tiles(K *kernel, int64_t units, hipStream_t s, A... args)
{
    hipLaunchKernelGGL(kernel, net_grid(xcd_blocks(units)), dim3(G::kThreads), 0, s, args..., units);
    return hipGetLastError();
}

}  // namespace

template <>
hipError_t launch_linear_tiles<EVOX_NET_TYPE>(const LinearArgs &a, int size, hipStream_t s)
{
    return with_tile(size, [&](auto b) {
        constexpr int B = b.value;
        typedef Product<B, false, false> G;
        const int64_t ti = (a.n_out + B - 1) / B, tj = net_tiles(a.rows, TileShape<B>::sh);
        return launch_tiles<G>(k_linear_tile<B>, banded(tj) * ti, s, a, ti, tj);
    });
}

template <>
hipError_t launch_linear_dx_tiles<EVOX_NET_TYPE>(const LinearGradArgs &a, const void *d, int64_t ldd, int size,
                                                 hipStream_t s)
{
    return with_tile(size, [&](auto b) {
        constexpr int B = b.value;
        typedef Product<B, true, false> G;
        const int64_t ti = (a.n_in + B - 1) / B, tj = net_tiles(a.rows, TileShape<B>::sh);
        return launch_tiles<G>(k_linear_dx_tile<B>, banded(tj) * ti, s, a, (const Elem *)d, ldd, ti, tj);
    });
}

template <>
hipError_t launch_linear_dw_tiles<EVOX_NET_TYPE>(const LinearGradArgs &a, const void *d, int64_t ldd, int size,
                                                 hipStream_t s)
{
    return with_tile(size, [&](auto b) {
        constexpr int B = b.value;
        typedef Product<B, true, true> G;
        const int64_t ti = (a.n_in + B - 1) / B, tj = (a.n_out + B - 1) / B;
        return launch_tiles<G>(k_linear_dw_tile<B>, a.rows.G * banded(tj) * ti, s, a, (const Elem *)d, ldd, ti, tj);
    });
}

}  // namespace evox
