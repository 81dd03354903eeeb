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

// n <= N neighbours of a row rounded from v.
__device__ __forceinline__ void store_row(Elem *p, const float *v, int n)
{
    constexpr int N = NetVec<Elem>::N;
    Reg t;
#pragma unroll
    for (int e = 0; e < N; ++e) t[e] = (Elem)v[e];
    store_chunk(p, 0, n, t);
}

// Results as they are (the gradients).
struct PlainOut {
    Elem *p;
    int64_t ld;
    __device__ __forceinline__ void begin(int, int) {}
    __device__ __forceinline__ Reg load(int, int, int) { return (Reg){}; }
    __device__ __forceinline__ void store(int j, int i, float *v, int n, Reg) { store_row(p + j * ld + i, v, n); }
};
// One share's sums of K, in fp32.
struct PartOut {
    float *p;
    int64_t ld;
    __device__ __forceinline__ void begin(int, int) {}
    __device__ __forceinline__ Reg load(int, int, int) { return (Reg){}; }
    __device__ __forceinline__ void store(int j, int i, float *v, int n, Reg)
    {
#pragma unroll
        for (int e = 0; e < NetVec<Elem>::N; ++e)
            if (e < n) p[j * ld + i + e] = v[e];
    }
};
// Share z of K: whole K tiles.
__device__ __forceinline__ void share_of(int64_t K, int splits, int z, int64_t *k0, int64_t *k1)
{
    const int64_t per = (K + splits * kTileK<Elem> - 1) / (splits * kTileK<Elem>) * kTileK<Elem>;
    *k0 = z * per < K ? z * per : K;
    *k1 = *k0 + per < K ? *k0 + per : K;
}

// The layer's epilogue; the pointers are at the tile's origin.
struct LayerOut {
    const Elem *b, *r;
    Elem *z, *y;
    int64_t ldr, ldz, ldy;
    int act;
    Reg bias;
    __device__ __forceinline__ void begin(int i, int n) { bias = b ? load_chunk(b + i, 0, n, (Elem)0.0f) : (Reg){}; }
    __device__ __forceinline__ Reg load(int j, int i, int n)
    {
        return r ? load_chunk(r + j * ldr + i, 0, n, (Elem)0.0f) : (Reg){};
    }
    __device__ __forceinline__ void store(int j, int i, float *v, int n, Reg res)
    {
        constexpr int N = NetVec<Elem>::N;
        if (b)
#pragma unroll
            for (int e = 0; e < N; ++e) v[e] += (float)bias[e];
        if (z) store_row(z + j * ldz + i, v, n);
        act_values<sizeof(Elem) == 2, N>(act, v);
        if (r)
#pragma unroll
            for (int e = 0; e < N; ++e) v[e] += (float)res[e];
        store_row(y + j * ldy + i, v, n);
    }
};

// Tile shapes, BI x BJ by WI x WJ waves.
template <int ID>
struct Shape {
    static constexpr bool k32 = sizeof(Elem) == 4;
    static constexpr int BI = ID == 0 ? 64 : ID == 1 ? 128 : 256;
    static constexpr int BJ = k32 ? (ID == 3 ? 128 : 64) : ID == 0 ? 64 : ID == 3 ? 256 : 128;
    static constexpr int WI = BI / 64, WJ = 2, kThreads = 64 * WI * WJ;
    static constexpr int sh = BJ == 64 ? 6 : BJ == 128 ? 7 : 8;
};
constexpr int kPairShift = 5;  // rows of a network per pair tile, as a power of two
bool pairs(const LinearGradArgs &a) { return (a.rows.M + a.rows.G - 1) / a.rows.G <= (int64_t)1 << kPairShift; }

template <int ID, bool PM, bool QM>
using Product = TileProduct<Elem, PM, QM, Shape<ID>::BI, Shape<ID>::BJ, Shape<ID>::WI, Shape<ID>::WJ>;

// y = act(x W^T + b) + r: i = output, j = row, k = input.
template <int ID>
__global__ __launch_bounds__(Shape<ID>::kThreads, 2) void k_linear_tile(LinearArgs a, int64_t ti,
                                                                                     int64_t tj, int64_t units)
{
    __shared__ __attribute__((aligned(16))) char lds[Product<ID, false, false>::kLds];
    const int64_t u = xcd_unit(units);
    if (u < 0) return;
    int64_t it, jt;
    unit_ij(u, ti, tj, &it, &jt);
    const NetTile t = net_tile(a.rows, Shape<ID>::sh, jt);
    if (t.g < 0) return;
    const int i0 = (int)it * Shape<ID>::BI, ni = min((int)a.n_out - i0, Shape<ID>::BI), nj = (int)(t.hi - t.lo);
    const int64_t x0 = a.x_shared ? t.lo - t.g * a.rows.n : t.lo;
    const TileOp<Elem> P{(const Elem *)a.w + t.g * a.w_stride + i0 * a.ldw, a.ldw, ni},
        Q{(const Elem *)a.x + x0 * a.ldx, a.ldx, nj};
    Product<ID, false, false> p;
    p.clear();
    p.run(P, Q, a.n_in, lds);
    LayerOut out{a.b ? (const Elem *)a.b + t.g * a.b_stride + i0 : nullptr,
                 a.r ? (const Elem *)a.r + t.lo * a.ldr + i0 : nullptr,
                 a.z ? (Elem *)a.z + t.lo * a.ldz + i0 : nullptr, (Elem *)a.y + t.lo * a.ldy + i0,
                 a.ldr, a.ldz, a.ldy, a.act, {}};
    p.results(ni, nj, lds, out);
}

// dx = d W: i = input, j = row, k = output.
// LOW: of both numbers of d.
template <int ID, bool LOW>
__global__ __launch_bounds__(Shape<ID>::kThreads, 2) void k_linear_dx_tile(LinearGradArgs a, const Elem *d, const Elem *low,
                                                                                      int64_t ldd, int64_t ti, int64_t tj,
                                                                                      int splits, float *part, int64_t units)
{
    __shared__ __attribute__((aligned(16))) char lds[Product<ID, true, false>::kLds];
    const int64_t us = xcd_unit(units), u = us / splits;
    if (us < 0) return;
    int64_t it, jt, k0, k1;
    unit_ij(u, ti, tj, &it, &jt);
    share_of(a.n_out, splits, (int)(us - u * splits), &k0, &k1);
    const NetTile t = net_tile(a.rows, Shape<ID>::sh, jt);
    if (t.g < 0) return;
    const int i0 = (int)it * Shape<ID>::BI, ni = min((int)a.n_in - i0, Shape<ID>::BI), nj = (int)(t.hi - t.lo);
    const TileOp<Elem> P{(const Elem *)a.w + t.g * a.w_stride + k0 * a.ldw + i0, a.ldw, ni}, Q{d + t.lo * ldd + k0, ldd, nj};
    Product<ID, true, false> p;
    if constexpr (LOW) p.run_split(P, Q, TileOp<Elem>{low + t.lo * ldd + k0, ldd, nj}, k1 - k0, lds);
    else {
        p.clear();
        p.run(P, Q, k1 - k0, lds);
    }
    if (splits > 1) {
        PartOut out{part + ((us - u * splits) * a.rows.M + t.lo) * a.n_in + i0, a.n_in};
        p.results(ni, nj, lds, out);
        return;
    }
    PlainOut out{(Elem *)a.dx + t.lo * a.lddx + i0, a.lddx};
    p.results(ni, nj, lds, out);
}

#if EVOX_NET_TYPE
// dx of few rows per network from both numbers of d: 32 rows of the one and of the
// other in a tile of 64, so that the weights, which bound it, are read once (bf16 1500x2
// rows 520x300: the gradient 379 us, with the weights read twice 480).
__global__ __launch_bounds__(Shape<0>::kThreads, 2) void k_linear_dx_pair(LinearGradArgs a, const Elem *d, const Elem *low, int64_t ldd,
                                                                          int64_t ti, int64_t tj, int splits, float *part,
                                                                          int64_t units)
{
    typedef Product<0, true, false> G;
    __shared__ __attribute__((aligned(16))) char lds[G::kLds];
    const int64_t us = xcd_unit(units), u = us / splits;
    if (us < 0) return;
    int64_t it, jt, k0, k1;
    unit_ij(u, ti, tj, &it, &jt);
    share_of(a.n_out, splits, (int)(us - u * splits), &k0, &k1);
    const NetTile t = net_tile(a.rows, kPairShift, jt);
    if (t.g < 0) return;
    const int i0 = (int)it * 64, ni = min((int)a.n_in - i0, 64), nj = (int)(t.hi - t.lo);
    const TileOp<Elem> P{(const Elem *)a.w + t.g * a.w_stride + k0 * a.ldw + i0, a.ldw, ni}, Q{d + t.lo * ldd + k0, ldd, nj};
    G p;
    p.clear();
    p.run<true>(P, Q, k1 - k0, lds, low + t.lo * ldd + k0);
    if (splits > 1) {
        PartOut out{part + ((us - u * splits) * a.rows.M + t.lo) * a.n_in + i0, a.n_in};
        p.results_pair(ni, nj, lds, out);
        return;
    }
    PlainOut out{(Elem *)a.dx + t.lo * a.lddx + i0, a.lddx};
    p.results_pair(ni, nj, lds, out);
}
#endif

// dW = d^T x: i = input, j = output, k = row of the network.
template <int ID, bool LOW>
__global__ __launch_bounds__(Shape<ID>::kThreads, 2) void k_linear_dw_tile(LinearGradArgs a, const Elem *d, const Elem *low,
                                                                                      int64_t ldd, int64_t ti, int64_t tj,
                                                                                      int splits, float *part, int64_t units)
{
    __shared__ __attribute__((aligned(16))) char lds[Product<ID, true, true>::kLds];
    const int64_t us = xcd_unit(units), u = us / splits, z = us - u * splits;
    if (us < 0) return;
    const int64_t per = banded(tj) * ti, g = u / per;
    int64_t it, jt, lo, hi, k0, k1;
    unit_ij(u - g * per, ti, tj, &it, &jt);
    if (jt >= tj) return;
    net_rows(a.rows, g, &lo, &hi);
    share_of(hi - lo, splits, (int)z, &k0, &k1);
    const int i0 = (int)it * Shape<ID>::BI, ni = min((int)a.n_in - i0, Shape<ID>::BI), j0 = (int)jt * Shape<ID>::BJ,
              nj = min((int)a.n_out - j0, Shape<ID>::BJ);
    const TileOp<Elem> P{(const Elem *)a.x + ((a.x_shared ? 0 : lo) + k0) * a.ldx + i0, a.ldx, ni}, Q{d + (lo + k0) * ldd + j0, ldd, nj};
    Product<ID, true, true> p;
    if constexpr (LOW) p.run_split(P, Q, TileOp<Elem>{low + (lo + k0) * ldd + j0, ldd, nj}, k1 - k0, lds);
    else {
        p.clear();
        p.run(P, Q, k1 - k0, lds);
    }
    if (splits > 1) {
        PartOut out{part + ((z * a.rows.G + g) * a.n_out + j0) * a.n_in + i0, a.n_in};
        p.results(ni, nj, lds, out);
        return;
    }
    PlainOut out{(Elem *)a.dw + g * a.dw_stride + j0 * a.lddw + i0, a.lddw};
    p.results(ni, nj, lds, out);
}

// The shape with the least estimated time: rounds of resident blocks times a
// block's work, its products plus 96 of them per row of K staged (which is how
// the shapes' times compare where all fill the chip: bf16 16x2048 4096x4096 1543,
// 1406, 1183 us in shapes 1, 2, 3, fp32 16x256 2048x2048 267, 260, 190; where
// they do not, the smaller win: fp32 4096 rows 1024x1024 64, 63, 77, bf16 1024 rows
// 1024x1024 15 in shape 0, then 19, 22, 32).  jt(BJ): tiles along j.  A CU holds
// (by LDS and registers) 3, 2, 1, 1 blocks of the fp32 shapes and 5, 2, 1, 1 of the
// 16-bit ones.
template <typename J>
int best_shape(int64_t ni, J &&jt)
{
    constexpr int per32[4] = {3, 2, 1, 1}, per16[4] = {5, 2, 1, 1};
    int best = 0;
    double least = 0.0;
    auto cost = [&](auto id) {
        typedef Shape<id.value> S;
        const int per = S::k32 ? per32[id.value] : per16[id.value];
        const int64_t blocks = (ni + S::BI - 1) / S::BI * jt(S::BJ), slots = 256 * per;
        const double rounds = blocks < slots ? (double)((blocks + 255) / 256) : (double)per * ((blocks + slots - 1) / slots);
        const double c = rounds * ((double)S::BI * S::BJ + 96.0 * (S::BI + S::BJ));
        if (id.value == 0 || c < least) {
            least = c;
            best = id.value;
        }
    };
    using std::integral_constant;
    cost(integral_constant<int, 0>{});
    cost(integral_constant<int, 1>{});
    cost(integral_constant<int, 2>{});
    cost(integral_constant<int, 3>{});
    return best;
}
template <typename F>
hipError_t with_shape(int shape, F &&f)
{
    using std::integral_constant;
    switch (shape) {
    case 0: return f(integral_constant<int, 0>{});
    case 1: return f(integral_constant<int, 1>{});
    case 2: return f(integral_constant<int, 2>{});
    default: return f(integral_constant<int, 3>{});
    }
}
// Tiles of BJ rows over the networks: ragged ones leave half a tile each, on average.
auto row_tiles(const NetRows &r)
{
    return [&r](int BJ) { return r.off ? r.M / BJ + (r.G + 1) / 2 : r.G * ((r.n + BJ - 1) / BJ); };
}
template <typename G, typename K, typename... A>
hipError_t launch_tiles(K *kernel, int64_t units, hipStream_t s, A... args)
{
    hipLaunchKernelGGL(kernel, net_grid(xcd_blocks(units)), dim3(G::kThreads), 0, s, args..., units);
    return hipGetLastError();
}

}  // namespace

template <>
int linear_tiles_shape<EVOX_NET_TYPE>(const LinearArgs &a)
{
    return best_shape(a.n_out, row_tiles(a.rows));
}
// (shares of K are for few tiles: the smallest ones; 4: a pair)
template <>
int linear_dx_tiles_shape<EVOX_NET_TYPE>(const LinearGradArgs &a, int splits)
{
    if (sizeof(Elem) == 2 && a.act > ACT_RELU && pairs(a)) return 4;
    return splits > 1 ? 0 : best_shape(a.n_in, row_tiles(a.rows));
}
template <>
int linear_dw_tiles_shape<EVOX_NET_TYPE>(const LinearGradArgs &a, int splits)
{
    return splits > 1 ? 0 : best_shape(a.n_in, [&](int BJ) { return a.rows.G * ((a.n_out + BJ - 1) / BJ); });
}

template <>
hipError_t launch_linear_tiles<EVOX_NET_TYPE>(const LinearArgs &a, hipStream_t s)
{
    return with_shape(linear_tiles_shape<EVOX_NET_TYPE>(a), [&](auto id) {
        constexpr int ID = id.value, B = Shape<ID>::BI;
        typedef Product<ID, false, false> G;
        const int64_t ti = (a.n_out + B - 1) / B, tj = net_tiles(a.rows, Shape<ID>::sh);
        return launch_tiles<G>(k_linear_tile<ID>, banded(tj) * ti, s, a, ti, tj);
    });
}

template <>
hipError_t launch_linear_dx_tiles<EVOX_NET_TYPE>(const LinearGradArgs &a, const void *d, const void *low, int64_t ldd,
                                                 int splits, float *part, hipStream_t s)
{
#if EVOX_NET_TYPE
    if (low && pairs(a)) {
        const int64_t ti = (a.n_in + 63) / 64, tj = net_tiles(a.rows, kPairShift);
        return launch_tiles<Product<0, true, false>>(k_linear_dx_pair, banded(tj) * ti * splits, s, a, (const Elem *)d,
                                                     (const Elem *)low, ldd, ti, tj, splits, part);
    }
#endif
    return with_shape(linear_dx_tiles_shape<EVOX_NET_TYPE>(a, splits), [&](auto id) {
        constexpr int ID = id.value, B = Shape<ID>::BI;
        typedef Product<ID, true, false> G;
        const int64_t ti = (a.n_in + B - 1) / B, tj = net_tiles(a.rows, Shape<ID>::sh);
        const auto go = [&](auto kernel) {
            return launch_tiles<G>(kernel, banded(tj) * ti * splits, s, a, (const Elem *)d, (const Elem *)low, ldd, ti, tj,
                                   splits, part);
        };
        if constexpr (sizeof(Elem) == 2)
            if (low) return go(k_linear_dx_tile<ID, true>);
        return go(k_linear_dx_tile<ID, false>);
    });
}

template <>
hipError_t launch_linear_dw_tiles<EVOX_NET_TYPE>(const LinearGradArgs &a, const void *d, const void *low, int64_t ldd,
                                                 int splits, float *part, hipStream_t s)
{
    return with_shape(linear_dw_tiles_shape<EVOX_NET_TYPE>(a, splits), [&](auto id) {
        constexpr int ID = id.value, B = Shape<ID>::BI, BJ = Shape<ID>::BJ;
        typedef Product<ID, true, true> G;
        const int64_t ti = (a.n_in + B - 1) / B, tj = (a.n_out + BJ - 1) / BJ;
        const auto go = [&](auto kernel) {
            return launch_tiles<G>(kernel, a.rows.G * banded(tj) * ti * splits, s, a, (const Elem *)d, (const Elem *)low, ldd,
                                   ti, tj, splits, part);
        };
        if constexpr (sizeof(Elem) == 2)
            if (low) return go(k_linear_dw_tile<ID, true>);
        return go(k_linear_dw_tile<ID, false>);
    });
}

}  // namespace evox
