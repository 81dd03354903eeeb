// Linear layers of a population of networks: y = act(x W_g^T + b_g) + r and
// its gradient.
#include <type_traits>

#include "evox_net.hpp"

namespace evox {

namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4u __attribute__((ext_vector_type(4), aligned(4)));
typedef __bf16 bf16x4u __attribute__((ext_vector_type(4), aligned(2)));
typedef _Float16 f16x4u __attribute__((ext_vector_type(4), aligned(2)));
template <typename T>
struct Quad;
template <>
struct Quad<float> {
    typedef f32x4u mem;
};
template <>
struct Quad<bf16_t> {
    typedef bf16x4u mem;
};
template <>
struct Quad<f16_t> {
    typedef f16x4u mem;
};

unsigned net_grid(int64_t n)
{
    const int64_t b = (n + 255) / 256;
    return (unsigned)(b < 1 ? 1 : b > ((int64_t)1 << 20) ? (int64_t)1 << 20 : b);
}

// ---------------------------------------------------------------------------
// One 16 x 16 tile of products over 16 bytes of K per lane: lane l brings
// elements k = KV (l / 16) .. + KV of row l % 16 of either operand (any split of
// k over the instruction's slots is a valid product, since both use the same
// one) and receives rows 4 (l / 16) .. + 4 of A against row l % 16 of B.
// ---------------------------------------------------------------------------
template <typename T>
struct Mma {
    typedef typename NetVec<T>::reg reg;
    static constexpr int KV = NetVec<T>::N, KS = 4 * KV;  // k per lane, per step
};
__device__ __forceinline__ f32x4 mma16(NetVec<bf16_t>::reg a, NetVec<bf16_t>::reg b, f32x4 c)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f32x4 mma16(NetVec<f16_t>::reg a, NetVec<f16_t>::reg b, f32x4 c)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f32x4 mma16(NetVec<float>::reg a, NetVec<float>::reg b, f32x4 c)
{
#pragma unroll
    for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[e], b[e], c, 0, 0, 0);
    return c;
}

// The epilogue of four neighbouring outputs o .. o + 3 of row m: bias,
// pre-activation, activation, residual, one rounding each.
template <typename T>
__device__ __forceinline__ void linear_out(const LinearArgs &a, int g, int64_t m, int o, f32x4 v)
{
    typedef typename Quad<T>::mem quad;
    const int n = (int)a.n_out;
    if (o >= n) return;
    const T *b = a.b ? (const T *)a.b + g * a.b_stride + o : nullptr;
    const T *r = a.r ? (const T *)a.r + m * a.ldr + o : nullptr;
    T *z = a.z ? (T *)a.z + m * a.ldz + o : nullptr, *y = (T *)a.y + m * a.ldy + o;
    if (o + 4 <= n) {
        quad t;
        if (b) {
            t = *reinterpret_cast<const quad *>(b);
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] += (float)t[j];
        }
        if (z) {
#pragma unroll
            for (int j = 0; j < 4; ++j) t[j] = (T)v[j];
            *reinterpret_cast<quad *>(z) = t;
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = act_value(a.act, v[j]);
        if (r) {
            t = *reinterpret_cast<const quad *>(r);
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] += (float)t[j];
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) t[j] = (T)v[j];
        *reinterpret_cast<quad *>(y) = t;
        return;
    }
#pragma unroll
    for (int j = 0; j < 3; ++j) {
        if (o + j >= n) continue;
        float s = v[j] + (b ? (float)b[j] : 0.0f);
        if (z) z[j] = (T)s;
        s = act_value(a.act, s);
        y[j] = (T)(s + (r ? (float)r[j] : 0.0f));
    }
}

// ---------------------------------------------------------------------------
// Few rows per network, or narrow layers: a wave computes 16 RB rows x 16 NB
// outputs with both operands straight from memory in the matrix cores' layout,
// 16 bytes per lane; rows past the network's end repeat its last one (their
// results are dropped), k past the end is zero.  WK waves share a tile's K
// where the tiles alone are too few to fill the chip, and add their sums in
// order.  Bound by the weights' bytes: each is read once.
// ---------------------------------------------------------------------------
template <typename T, int RB, int NB, int WK>
__global__ __launch_bounds__(256) void k_linear_thin(LinearArgs a, int sh, uint32_t out_tiles, int64_t units)
{
    typedef typename Mma<T>::reg reg;
    constexpr int KV = Mma<T>::KV, KS = Mma<T>::KS, U = RB + NB <= 2 ? 8 : RB + NB <= 4 ? 4 : 2;
    __shared__ f32x4 part[WK > 1 ? 4 / WK * (WK - 1) * RB * NB * 64 : 1];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x % 64, l16 = lane % 16,
              q = lane / 16, wk = wave % WK, wt = wave / WK;
    const int64_t unit = (int64_t)blockIdx.x * (4 / WK) + wt;
    NetTile t;
    t.g = -1;
    const int64_t tile = unit / out_tiles;
    const int o0 = (int)(unit - tile * out_tiles) * 16 * NB;
    if (unit < units) t = net_tile(a.rows, sh, tile);
    f32x4 acc[RB][NB];
#pragma unroll
    for (int r = 0; r < RB; ++r)
#pragma unroll
        for (int n = 0; n < NB; ++n) acc[r][n] = (f32x4){0.0f, 0.0f, 0.0f, 0.0f};
    if (t.g >= 0) {
        const int K = (int)a.n_in, steps = (K + KS - 1) / KS, per = (steps + WK - 1) / WK, s1 = min(steps, (wk + 1) * per),
                  full = min(s1, K / KS);
        const int64_t x0 = a.x_shared ? (int64_t)t.g * a.rows.n : 0;
        const T *xr[RB], *wr[NB];
#pragma unroll
        for (int r = 0; r < RB; ++r)
            xr[r] = (const T *)a.x + (min(t.lo + r * 16 + l16, t.hi - 1) - x0) * a.ldx + q * KV;
#pragma unroll
        for (int n = 0; n < NB; ++n)
            wr[n] = (const T *)a.w + t.g * a.w_stride + min((int64_t)o0 + n * 16 + l16, a.n_out - 1) * a.ldw + q * KV;
        typedef typename NetVec<T>::mem mem;
        auto steps_of = [&](int s, auto count) {
            constexpr int C = decltype(count)::value;
            reg xv[C][RB], wv[C][NB];
#pragma unroll
            for (int u = 0; u < C; ++u) {
#pragma unroll
                for (int n = 0; n < NB; ++n) wv[u][n] = *reinterpret_cast<const mem *>(wr[n] + (s + u) * KS);
#pragma unroll
                for (int r = 0; r < RB; ++r) xv[u][r] = *reinterpret_cast<const mem *>(xr[r] + (s + u) * KS);
            }
#pragma unroll
            for (int u = 0; u < C; ++u)
#pragma unroll
                for (int r = 0; r < RB; ++r)
#pragma unroll
                    for (int n = 0; n < NB; ++n) acc[r][n] = mma16(wv[u][n], xv[u][r], acc[r][n]);
        };
        int s = wk * per;
        for (; s + U <= full; s += U) steps_of(s, std::integral_constant<int, U>{});
        if constexpr (U > 4)
            for (; s + 4 <= full; s += 4) steps_of(s, std::integral_constant<int, 4>{});
        for (; s < full; ++s) steps_of(s, std::integral_constant<int, 1>{});
        if (s < s1) {  // the last step of a K that is no multiple of KS
            const int k = s * KS + q * KV;
            reg xv[RB], wv[NB];
#pragma unroll
            for (int n = 0; n < NB; ++n) wv[n] = load_chunk(wr[n] - q * KV, k / KV, K, (T)0.0f);
#pragma unroll
            for (int r = 0; r < RB; ++r) xv[r] = load_chunk(xr[r] - q * KV, k / KV, K, (T)0.0f);
#pragma unroll
            for (int r = 0; r < RB; ++r)
#pragma unroll
                for (int n = 0; n < NB; ++n) acc[r][n] = mma16(wv[n], xv[r], acc[r][n]);
        }
    }
    if constexpr (WK > 1) {
        if (wk > 0)
#pragma unroll
            for (int r = 0; r < RB; ++r)
#pragma unroll
                for (int n = 0; n < NB; ++n) part[(((wt * (WK - 1) + wk - 1) * RB + r) * NB + n) * 64 + lane] = acc[r][n];
        __syncthreads();
        if (wk > 0) return;
#pragma unroll
        for (int k = 1; k < WK; ++k)
#pragma unroll
            for (int r = 0; r < RB; ++r)
#pragma unroll
                for (int n = 0; n < NB; ++n) acc[r][n] += part[(((wt * (WK - 1) + k - 1) * RB + r) * NB + n) * 64 + lane];
    }
    if (t.g < 0) return;
#pragma unroll
    for (int r = 0; r < RB; ++r) {
        const int64_t m = t.lo + r * 16 + l16;
        if (m < t.hi)
#pragma unroll
            for (int n = 0; n < NB; ++n) linear_out<T>(a, t.g, m, o0 + n * 16 + 4 * q, acc[r][n]);
    }
}

// d = dy act'(z), rounded to the element type.
template <typename T>
__device__ __forceinline__ float grad_of_z(const LinearGradArgs &a, int64_t m, int64_t o)
{
    const float d = (float)((const T *)a.dy)[m * a.lddy + o];
    if (a.act == ACT_NONE) return d;
    return d * act_slope(a.act, (float)((const T *)a.z)[m * a.ldz + o]);
}

template <typename T>
__global__ __launch_bounds__(256) void k_linear_dx(LinearGradArgs a)
{
    const T *w = (const T *)a.w;
    T *dx = (T *)a.dx;
    for (int64_t q = (int64_t)blockIdx.x * 256 + threadIdx.x; q < a.rows.M * a.n_in; q += (int64_t)gridDim.x * 256) {
        const int64_t m = q / a.n_in, i = q % a.n_in, g = net_of_row(a.rows, m);
        if (g < 0) continue;
        float s = 0.0f;
        for (int64_t o = 0; o < a.n_out; ++o)
            s = fmaf((float)(T)grad_of_z<T>(a, m, o), (float)w[g * a.w_stride + o * a.ldw + i], s);
        dx[m * a.lddx + i] = (T)s;
    }
}

// Column n_in of a network's gradient is db.
template <typename T>
__global__ __launch_bounds__(256) void k_linear_dw(LinearGradArgs a)
{
    const T *x = (const T *)a.x;
    T *dw = (T *)a.dw, *db = (T *)a.db;
    const int64_t cols = a.n_in + 1;
    for (int64_t q = (int64_t)blockIdx.x * 256 + threadIdx.x; q < a.rows.G * a.n_out * cols;
         q += (int64_t)gridDim.x * 256) {
        const int64_t i = q % cols, o = q / cols % a.n_out, g = q / cols / a.n_out;
        if (i < a.n_in ? !dw : !db) continue;
        int64_t lo, hi;
        net_rows(a.rows, g, &lo, &hi);
        float s = 0.0f;
        for (int64_t m = lo; m < hi; ++m) {
            const float d = grad_of_z<T>(a, m, o);
            if (i == a.n_in) s += d;
            else s = fmaf((float)(T)d, (float)x[(a.x_shared ? m - lo : m) * a.ldx + i], s);
        }
        if (i == a.n_in) db[g * a.db_stride + o] = (T)s;
        else dw[g * a.dw_stride + o * a.lddw + i] = (T)s;
    }
}

}  // namespace

hipError_t launch_linear(const LinearArgs &a, hipStream_t s)
{
    return net_dispatch(a.dtype, [&](auto t) {
        using T = decltype(t);
        // rows of a wave's tile by the mean rows per network
        const int64_t mean = (a.rows.M + a.rows.G - 1) / a.rows.G;
        const int rb = mean <= 16 ? 1 : mean <= 32 ? 2 : 4, sh = rb == 1 ? 4 : rb == 2 ? 5 : 6, nb = rb == 1 ? 1 : 2;
        const uint32_t out_tiles = (uint32_t)((a.n_out + 16 * nb - 1) / (16 * nb));
        const int64_t units = net_tiles(a.rows, sh) * out_tiles;
        const int64_t steps = (a.n_in + Mma<T>::KS - 1) / Mma<T>::KS;
        const bool split = units < 4096 && steps >= 16;
        const unsigned blocks = (unsigned)(split ? units : (units + 3) / 4);
        auto go = [&](auto r, auto n) {
            if (split)
                hipLaunchKernelGGL((k_linear_thin<T, r.value, n.value, 4>), dim3(blocks), dim3(256), 0, s, a, sh,
                                   out_tiles, units);
            else
                hipLaunchKernelGGL((k_linear_thin<T, r.value, n.value, 1>), dim3(blocks), dim3(256), 0, s, a, sh,
                                   out_tiles, units);
        };
        using std::integral_constant;
        if (rb == 1) go(integral_constant<int, 1>{}, integral_constant<int, 1>{});
        else if (rb == 2) go(integral_constant<int, 2>{}, integral_constant<int, 2>{});
        else go(integral_constant<int, 4>{}, integral_constant<int, 2>{});
        return hipGetLastError();
    });
}

size_t linear_grad_scratch(const LinearGradArgs &) { return 256; }

hipError_t launch_linear_grad(const LinearGradArgs &a, hipStream_t s)
{
    return net_dispatch(a.dtype, [&](auto t) {
        if (a.dx && a.rows.M)
            hipLaunchKernelGGL((k_linear_dx<decltype(t)>), dim3(net_grid(a.rows.M * a.n_in)), dim3(256), 0, s, a);
        if (a.dw || a.db)
            hipLaunchKernelGGL((k_linear_dw<decltype(t)>), dim3(net_grid(a.rows.G * a.n_out * (a.n_in + 1))),
                               dim3(256), 0, s, a);
        return hipGetLastError();
    });
}

}  // namespace evox
