// Linear layers of a population of networks: y = act(x W_g^T + b_g) + r and
// its gradient.
#include "evox_tile.hpp"

namespace evox {

namespace {

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
        float f[4] = {v[0], v[1], v[2], v[3]};
        act_values<sizeof(T) == 2, 4>(a.act, f);
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = f[j];
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
        s = act_value<sizeof(T) == 2>(a.act, s);
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
    const int64_t unit = net_block() * (4 / WK) + wt;
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

// d = dy act'(z), rounded to the element type (where a.act is not none and a
// product needs it), and the tiles' column sums of the unrounded d (where db is
// wanted): a block takes 2^kDzShift rows of a network and 256 chunks of 16 bytes
// of their columns, L lanes to a row, and adds its row slots in order.
constexpr int kDzShift = 4;

template <typename T>
__global__ __launch_bounds__(256) void k_linear_dz(LinearGradArgs a, int L, T *d, int64_t ldd, float *sums)
{
    constexpr int N = NetVec<T>::N;
    typedef typename NetVec<T>::reg reg;
    extern __shared__ float slots_sum[];  // [256 / L - 1][N][L]
    const int64_t cols = (a.n_out + 256 * N - 1) / (256 * N), tile = net_block() / cols;
    const NetTile t = net_tile(a.rows, kDzShift, tile);
    if (t.g < 0) return;
    const int lane = threadIdx.x & (L - 1), slot = threadIdx.x / L, slots = 256 / L, n = (int)a.n_out,
              c = (int)(net_block() - tile * cols) * 256 + lane;
    float s[N];
#pragma unroll
    for (int j = 0; j < N; ++j) s[j] = 0.0f;
    if (c * N < n)
        for (int64_t m = t.lo + slot; m < t.hi; m += slots) {
            const reg dy = load_chunk((const T *)a.dy + m * a.lddy, c, n, (T)0.0f);
            if (a.act == ACT_NONE) {
#pragma unroll
                for (int j = 0; j < N; ++j) s[j] += (float)dy[j];
                continue;
            }
            const reg z = load_chunk((const T *)a.z + m * a.ldz, c, n, (T)0.0f);
            float v[N];
#pragma unroll
            for (int j = 0; j < N; ++j) v[j] = (float)z[j];
            act_slopes<sizeof(T) == 2, N>(a.act, v);
            reg out;
#pragma unroll
            for (int j = 0; j < N; ++j) {
                v[j] *= (float)dy[j];
                s[j] += v[j];
                out[j] = (T)v[j];
            }
            if (d) store_chunk(d + m * ldd, c, n, out);
        }
    if (!sums) return;
    if (slot > 0)
#pragma unroll
        for (int j = 0; j < N; ++j) slots_sum[((slot - 1) * N + j) * L + lane] = s[j];
    __syncthreads();
    if (slot > 0 || c * N >= n) return;
    for (int r = 0; r < slots - 1; ++r)
#pragma unroll
        for (int j = 0; j < N; ++j) s[j] += slots_sum[(r * N + j) * L + lane];
#pragma unroll
    for (int j = 0; j < N; ++j)
        if (c * N + j < n) sums[tile * n + c * N + j] = s[j];
}

// db from a network's tiles, in order.
template <typename T>
__global__ __launch_bounds__(256) void k_linear_db(LinearGradArgs a, const float *sums)
{
    const int o = blockIdx.x * 256 + threadIdx.x;
    if (o >= a.n_out) return;
    for (int64_t g = blockIdx.y; g < a.rows.G; g += gridDim.y) {
        int64_t lo, hi;
        net_rows(a.rows, g, &lo, &hi);
        const int64_t t0 = net_first_tile(a.rows, kDzShift, g), n = (hi - lo + (1 << kDzShift) - 1) >> kDzShift;
        float s = 0.0f;
        for (int64_t t = 0; t < n; ++t) s += sums[(t0 + t) * a.n_out + o];
        ((T *)a.db)[g * a.db_stride + o] = (T)s;
    }
}

// The scratch: d, then the tiles' column sums.
struct GradScratch {
    int64_t ldd;
    size_t sums, end;
};
GradScratch grad_layout(const LinearGradArgs &a)
{
    GradScratch g;
    const size_t e = a.dtype == NET_F32 ? 4 : 2;
    g.ldd = (a.n_out + 7) / 8 * 8;
    g.sums = (e * (size_t)a.rows.M * (size_t)g.ldd + 255) / 256 * 256;
    g.end = g.sums + 4 * ((size_t)(a.rows.M >> kDzShift) + (size_t)a.rows.G) * (size_t)a.n_out;
    return g;
}

// Tiles of 64 where either side of the result is no more than that or larger
// ones would leave CUs without a block; of 256 (16 bits) where they fill the chip.
int tile_size(int32_t dtype, int64_t ni, int64_t nj, int64_t results)
{
    if (ni <= 64 || nj <= 64 || results < (int64_t)256 * 128 * 128) return 0;
    if (dtype != NET_F32 && ni >= 192 && nj >= 192 && results >= (int64_t)512 * 256 * 256) return 2;
    return 1;
}

}  // namespace

hipError_t launch_linear(const LinearArgs &a, hipStream_t s)
{
    return net_dispatch(a.dtype, [&](auto t) {
        using T = typename NetElement<t.value>::type;
        const int64_t mean = (a.rows.M + a.rows.G - 1) / a.rows.G;
        if (mean > 32 && a.n_out > 32 && a.n_in >= 64)
            return launch_linear_tiles<t.value>(a, tile_size(a.dtype, a.n_out, mean, a.rows.M * a.n_out), s);
        // rows of a wave's tile by the mean rows per network
        const int rb = mean <= 16 ? 1 : mean <= 32 ? 2 : 4, sh = rb == 1 ? 4 : rb == 2 ? 5 : 6, nb = rb == 1 ? 1 : 2;
        const uint32_t out_tiles = (uint32_t)((a.n_out + 16 * nb - 1) / (16 * nb));
        const int64_t units = net_tiles(a.rows, sh) * out_tiles;
        const int64_t steps = (a.n_in + Mma<T>::KS - 1) / Mma<T>::KS;
        const bool split = units < 4096 && steps >= 16;
        const dim3 blocks = net_grid(split ? units : (units + 3) / 4);
        auto go = [&](auto r, auto n) {
            if (split)
                hipLaunchKernelGGL((k_linear_thin<T, r.value, n.value, 4>), blocks, dim3(256), 0, s, a, sh,
                                   out_tiles, units);
            else
                hipLaunchKernelGGL((k_linear_thin<T, r.value, n.value, 1>), blocks, dim3(256), 0, s, a, sh,
                                   out_tiles, units);
        };
        using std::integral_constant;
        if (rb == 1) go(integral_constant<int, 1>{}, integral_constant<int, 1>{});
        else if (rb == 2) go(integral_constant<int, 2>{}, integral_constant<int, 2>{});
        else go(integral_constant<int, 4>{}, integral_constant<int, 2>{});
        return hipGetLastError();
    });
}

size_t linear_grad_scratch(const LinearGradArgs &a) { return grad_layout(a).end; }

hipError_t launch_linear_grad(const LinearGradArgs &a, hipStream_t s)
{
    return net_dispatch(a.dtype, [&](auto t) {
        using T = typename NetElement<t.value>::type;
        constexpr int N = NetVec<T>::N;
        const GradScratch l = grad_layout(a);
        const bool own = a.act != ACT_NONE && (a.dx || a.dw);
        T *d = own ? (T *)a.scratch : nullptr;
        float *sums = a.db ? (float *)((char *)a.scratch + l.sums) : nullptr;
        hipError_t e = hipSuccess;
        if (a.rows.M > 0 && (d || sums)) {
            int L = 4;
            while (L < 256 && L * N < a.n_out) L *= 2;
            const int64_t cols = (a.n_out + 256 * N - 1) / (256 * N);
            hipLaunchKernelGGL((k_linear_dz<T>), net_grid(net_tiles(a.rows, kDzShift) * cols), dim3(256),
                               sizeof(float) * N * (256 - L), s, a, L, d, l.ldd, sums);
            if ((e = hipGetLastError()) != hipSuccess) return e;
        }
        if (a.db) {
            hipLaunchKernelGGL((k_linear_db<T>),
                               dim3((unsigned)((a.n_out + 255) / 256), (unsigned)(a.rows.G < 32768 ? a.rows.G : 32768)),
                               dim3(256), 0, s, a, sums);
            if ((e = hipGetLastError()) != hipSuccess) return e;
        }
        const void *dd = own ? d : a.dy;
        const int64_t ldd = own ? l.ldd : a.lddy, mean = (a.rows.M + a.rows.G - 1) / a.rows.G;
        if (a.dx)
            e = launch_linear_dx_tiles<t.value>(a, dd, ldd, tile_size(a.dtype, a.n_in, mean, a.rows.M * a.n_in), s);
        if (e == hipSuccess && a.dw)
            e = launch_linear_dw_tiles<t.value>(a, dd, ldd,
                                                tile_size(a.dtype, a.n_in, a.n_out, a.rows.G * a.n_in * a.n_out), s);
        return e;
    });
}

}  // namespace evox
