// Linear layers of a population of networks: y = act(x W_g^T + b_g) + r and its
// gradient.  Here: the choice of kernels, and those that need no LDS tiles (few
// rows, narrow layers, short sums); evox_linear_tile.hip has the rest.
#include "evox.h"
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
// Up to four neighbours p[0 .. n), zeros after them.
template <typename T>
__device__ __forceinline__ f32x4 load_quad(const T *p, int n)
{
    f32x4 v = (f32x4)(0.0f);
    if (n >= 4) {
        const typename Quad<T>::mem t = *reinterpret_cast<const typename Quad<T>::mem *>(p);
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = (float)t[j];
    } else {
#pragma unroll
        for (int j = 0; j < 3; ++j)
            if (j < n) v[j] = (float)p[j];
    }
    return v;
}
template <typename T>
__device__ __forceinline__ void store_quad(T *p, int n, f32x4 v)
{
    if (n >= 4) {
        typename Quad<T>::mem t;
#pragma unroll
        for (int j = 0; j < 4; ++j) t[j] = (T)v[j];
        *reinterpret_cast<typename Quad<T>::mem *>(p) = t;
    } else {
#pragma unroll
        for (int j = 0; j < 3; ++j)
            if (j < n) p[j] = (T)v[j];
    }
}

// ---------------------------------------------------------------------------
// Few rows per network, or narrow layers: a wave computes 16 RB rows x 16 NB
// outputs with both operands straight from memory in the matrix cores' layout,
// 16 bytes per lane; rows past the network's end repeat its last one (their
// results are dropped), k past the end is zero.  WK waves share a tile's K where
// the tiles alone are too few to fill the chip or K is long, and add their sums
// in order.  The weights, each read once, bound it: bf16 256 networks, one row
// through 2048x2048, 347 us, 6.19 TB/s of the copy's 6.45 (16 x 32 tiles: 436 us);
// fp32 4096 networks' one row 32x32, 7.8 us, a launch and the chain of its loads.
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
    f32x4 bias[NB];
#pragma unroll
    for (int n = 0; n < NB; ++n) {
        const int o = o0 + n * 16 + 4 * q;
        bias[n] = t.g >= 0 && a.b && wk == 0 ? load_quad((const T *)a.b + t.g * a.b_stride + o, (int)a.n_out - o) : (f32x4)(0.0f);
    }
    if (t.g >= 0) {
        const int K = (int)a.n_in, steps = (K + KS - 1) / KS, per = (steps + WK - 1) / WK, s1 = min(steps, (wk + 1) * per),
                  full = min(s1, K / KS);
        const int64_t x0 = a.x_shared ? (int64_t)t.g * a.rows.n : 0;
        // (row pitches are below 2^31: one multiply-add per address)
        const T *xr[RB], *wr[NB], *xb = (const T *)a.x + (t.lo - x0) * a.ldx + q * KV,
                                  *wb = (const T *)a.w + t.g * a.w_stride + o0 * a.ldw + q * KV;
        const int rows = (int)(t.hi - t.lo), outs = (int)a.n_out - o0;
#pragma unroll
        for (int r = 0; r < RB; ++r)
            xr[r] = xb + (int64_t)min(r * 16 + l16, rows - 1) * (int)a.ldx;
#pragma unroll
        for (int n = 0; n < NB; ++n)
            wr[n] = wb + (int64_t)min(n * 16 + l16, outs - 1) * (int)a.ldw;
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
    // a lane's rows l16, l16 + 16, ... of the tile, its outputs o0 + 4 q, + 16, ...
    const int rows = (int)(t.hi - t.lo) - l16, outs = (int)a.n_out - o0 - 4 * q;
    T *y = (T *)a.y + t.lo * a.ldy + o0 + (int64_t)l16 * (int)a.ldy + 4 * q;
    T *z = a.z ? (T *)a.z + t.lo * a.ldz + o0 + (int64_t)l16 * (int)a.ldz + 4 * q : nullptr;
    // the residual's loads all before the first store (which may take its place)
    f32x4 res[RB][NB];
    if (a.r) {
        const T *from = (const T *)a.r + t.lo * a.ldr + o0 + (int64_t)l16 * (int)a.ldr + 4 * q;
#pragma unroll
        for (int r = 0; r < RB; ++r)
#pragma unroll
            for (int n = 0; n < NB; ++n)
                if (r * 16 < rows) res[r][n] = load_quad(from + r * 16 * a.ldr + n * 16, outs - n * 16);
    }
#pragma unroll
    for (int r = 0; r < RB; ++r) {
        if (r * 16 >= rows) continue;
#pragma unroll
        for (int n = 0; n < NB; ++n) {
            if (outs <= n * 16) continue;
            f32x4 v = acc[r][n] + bias[n];
            if (z) store_quad(z + r * 16 * a.ldz + n * 16, outs - n * 16, v);
            if (a.act != ACT_NONE) {
                float f[4] = {v[0], v[1], v[2], v[3]};
                act_values<sizeof(T) == 2, 4>(a.act, f);
                v = (f32x4){f[0], f[1], f[2], f[3]};
            }
            if (a.r) v += res[r][n];
            store_quad(y + r * 16 * a.ldy + n * 16, outs - n * 16, v);
        }
    }
}

// d = dy act'(z) in the element type (where a.act is not none and a
// product needs it), and the tiles' column sums of d in fp32 (where db is
// wanted): a block takes 2^sh rows of a network and L chunks of 16 bytes of their
// columns, and adds its 256 / L row slots in order.  Apart from
// the products, so that a slope is computed once per element and not once per
// tile that reads it.  In 16 bits d leaves as two numbers of the type (d_split; of
// relu's d, dy or 0, one holds all), whose products are added: rounded to one, it
// would put an error of sqrt(K) roundoffs into every sum of K terms, however small
// the sum (relative rms of the bf16 gradient against 64 bits 2.3e-3 instead of
// 1.7e-3, the results' own rounding).  That costs the products twice their time:
// bf16 64x512 ragged rows 1024x1024 with GELU 450 us, 287 in one number.  bf16 32,768
// rows of 1024 with GELU: 54 us, 5.0 TB/s (50 for one number), bound by the slopes'
// arithmetic and the wait for two loads; in the dx and dw tiles' own loads the slopes
// would be computed 8 times over there.  L: the most lanes among those that leave the
// fewest idle; 2^sh: 16 rows, up to 256 where there are more than 4096 blocks (300,000
// rows of 1109: 18,750 tiles took 671 us to join).
struct DzShape {
    int sh, L;
    int64_t cols;  // blocks per row
};
DzShape dz_shape(const LinearGradArgs &a)
{
    const int64_t chunks = (a.n_out + (a.dtype == NET_F32 ? 3 : 7)) / (a.dtype == NET_F32 ? 4 : 8);
    DzShape s{4, 4, 0};
    while (s.L < 32 && s.L < chunks) s.L *= 2;
    for (int L = 64; L <= 256; L *= 2)
        if ((chunks + L - 1) / L * L <= (chunks + s.L - 1) / s.L * s.L) s.L = L;
    s.cols = (chunks + s.L - 1) / s.L;
    while (s.sh < 8 && (a.rows.M >> s.sh) * s.cols > 4096) ++s.sh;
    return s;
}

template <typename T>
__global__ __launch_bounds__(256) void k_linear_dz(LinearGradArgs a, int sh, int L, int64_t cols, T *d, T *low, int64_t ldd,
                                                     float *sums)
{
    constexpr int N = NetVec<T>::N;
    typedef typename NetVec<T>::reg reg;
    extern __shared__ float slots_sum[];  // [256 / L - 1][N][L]
    const int64_t tile = net_block() / cols;
    const NetTile t = net_tile(a.rows, sh, tile);
    if (t.g < 0) return;
    const int lane = threadIdx.x & (L - 1), slot = threadIdx.x / L, slots = 256 / L, n = (int)a.n_out,
              c = (int)(net_block() - tile * cols) * L + lane;
    float s[N];
#pragma unroll
    for (int j = 0; j < N; ++j) s[j] = 0.0f;
    if (c * N < n)
        for (int64_t m = t.lo + slot; m < t.hi; m += slots) {
            reg dy = load_early((const T *)a.dy + m * a.lddy, c, n);
            if (a.act == ACT_NONE) {
                settle(dy, c, n, (T)0.0f);
#pragma unroll
                for (int j = 0; j < N; ++j) s[j] += (float)dy[j];
                continue;
            }
            reg z = load_early((const T *)a.z + m * a.ldz, c, n);
            settle(dy, c, n, (T)0.0f);
            settle(z, c, n, (T)0.0f);
            float v[N];
#pragma unroll
            for (int j = 0; j < N; ++j) v[j] = (float)z[j];
            act_slopes<sizeof(T) == 2, N>(a.act, v);
            reg out, rest;
#pragma unroll
            for (int j = 0; j < N; ++j) {
                v[j] *= (float)dy[j];
                s[j] += v[j];
                out[j] = (T)v[j];
            }
            if (low)
#pragma unroll
                for (int j = 0; j < N; ++j) {
                    T h, l;
                    d_split(v[j], h, l);
                    out[j] = h;
                    rest[j] = l;
                }
            if (d) store_chunk(d + m * ldd, c, n, out);
            if (low) store_chunk(low + m * ldd, c, n, rest);
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
    if (t.only) {
        reg out;
#pragma unroll
        for (int j = 0; j < N; ++j) out[j] = (T)s[j];
        store_chunk((T *)a.db + t.g * a.db_stride, c, n, out);
        return;
    }
    sums += net_slot(t.lo, t.index, sh) * n + c * N;
#pragma unroll
    for (int j = 0; j < N; ++j)
        if (c * N + j < n) sums[j] = s[j];
}

// Sums over a network's rows: dw[o][i] (n_in of them per output; 0: none), then db.
template <typename T>
struct GradSums {
    T *dw, *db;
    int64_t n_out, n_in, lddw, dw_stride, db_stride;
    __device__ void operator()(int64_t g, int64_t e, float s) const
    {
        if (e >= n_out * n_in) {
            if (db) db[g * db_stride + e - n_out * n_in] = (T)s;
        } else if (dw) {
            const int64_t o = (int64_t)((uint32_t)e / (uint32_t)n_in);
            dw[g * dw_stride + o * lddw + e - o * n_in] = (T)s;
        }
    }
};

// ---------------------------------------------------------------------------
// The whole gradient of narrow layers (both widths at most 64) in one pass: a
// block takes 2^sh rows of one network, W stays in LDS, and 16 F rows per wave at a
// time d = dy act'(z) (not rounded: all of it is fp32 here) and x pass through
// LDS into the fp32 matrix cores; every operand is read once and dx written
// once.  Blocks of two waves for up to 32 rows per network, else four (two / four:
// fp32 32x32 8 rows 90 / 147 us, 32 rows 33 / 44, 64 rows 23 / 25, 200 rows 35 / 27).
// Wave w has rows 16 F w .. + 16 F of dx, and of the dw tiles every WAVES-th; with widths
// up to 16 (F = 4) its own rows' share of the one dw tile (1.8M rows 8x1
// 89 us; before whole chunks of padding were left out 120, with F = 1 149).  fp32
// 4096x32 rows 32x32: 101 MB in 30 us, floor 16; three to four waves per SIMD (LDS
// and registers) each wait for three loads in a row.  In separate passes through
// the 64-tiles it took 72 us; W's and x's loads ahead of d's cost as much in
// occupancy as they gained.
// ---------------------------------------------------------------------------
constexpr int kNarrow = 64;

template <typename T, int WAVES, int F>
__global__ __launch_bounds__(64 * WAVES, 3) void k_linear_grad_narrow(LinearGradArgs a, int sh, float *part)
{
    constexpr int N = NetVec<T>::N, TH = 64 * WAVES, R = 16 * WAVES * F, kDw = F > 1 ? 1 : 16 / WAVES;
    typedef typename NetVec<T>::reg reg;
    extern __shared__ __attribute__((aligned(16))) float lds[];
    const NetTile t = net_tile(a.rows, sh, net_block());
    if (t.g < 0) return;
    const int ni = (int)a.n_in, no = (int)a.n_out, ti = (ni + 15) / 16, to = (no + 15) / 16, pi = ti * 16 + 4,
              po = to * 16 + 4;
    float *W = lds, *X = W + (a.dx ? to * 16 * pi : 0), *D = X + R * pi;
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid / 64), l16 = tid % 16, q = tid % 64 / 16;
    // a chunk of a row of the type to a row of LDS
    auto put = [&](float *row, int c, reg v) {
#pragma unroll
        for (int j = 0; j < N; j += 4) *reinterpret_cast<f32x4 *>(row + c * N + j) = (f32x4){(float)v[j], (float)v[j + 1], (float)v[j + 2], (float)v[j + 3]};
    };
    // (k / ci and k / co by a multiplication, exact for k < 65536 / 15)
    // chunks per row: in blocks of many rows those that hold anything, the tiles' padding
    // being zero once and for all (1.8M rows 8x1 142 -> 89 us; of one or two rounds
    // 4096x32 rows 31x20 31 -> 33, so not there)
    const bool skip = t.hi - t.lo > 2 * R;
    const int ci = skip ? (ni + N - 1) / N : ti * 16 / N, co = skip ? (no + N - 1) / N : to * 16 / N, mi = (65535 + ci) / ci,
              mo = (65535 + co) / co, shares = TH / (to * 16);  // threads per column
    if (skip) {
        f32x4 *const all = reinterpret_cast<f32x4 *>(lds);
        for (int k = tid; k < ((int)(X - lds) + R * (pi + po)) / 4; k += TH) all[k] = (f32x4)(0.0f);
        __syncthreads();
    }
    if (a.dx) {
        const T *w = (const T *)a.w + t.g * a.w_stride;
#pragma unroll 2
        for (int k = tid; k < to * 16 * ci; k += TH) {
            const int o = (k * mi >> 16), c = k - o * ci;
            put(W + o * pi, c, o < no ? load_chunk(w + o * a.ldw, c, ni, (T)0.0f) : (reg){});
        }
    }
    f32x4 dw[kDw];
#pragma unroll
    for (int s = 0; s < kDw; ++s) dw[s] = (f32x4)(0.0f);
    float db = 0.0f;
    const int64_t x0 = a.x_shared ? (int64_t)t.g * a.rows.n : 0;
    for (int64_t m0 = t.lo; m0 < t.hi; m0 += R) {
        if (m0 > t.lo) __syncthreads();
        // two chunks of d per round, their loads first
#pragma unroll 1
        for (int k0 = tid; k0 < R * co; k0 += 2 * TH) {
            reg dy[2] = {}, z[2] = {};
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const int k = k0 + u * TH, r = (k * mo >> 16), c = k - r * co;
                if (k >= R * co || m0 + r >= t.hi) continue;
                dy[u] = load_early((const T *)a.dy + (m0 + r) * a.lddy, c, no);
                if (a.act != ACT_NONE) z[u] = load_early((const T *)a.z + (m0 + r) * a.ldz, c, no);
            }
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const int k = k0 + u * TH, r = (k * mo >> 16), c = k - r * co;
                if (k >= R * co) continue;
                settle(dy[u], c, no, (T)0.0f);
                settle(z[u], c, no, (T)0.0f);
                float v[N];
#pragma unroll
                for (int j = 0; j < N; ++j) v[j] = (float)z[u][j];
                act_slopes<sizeof(T) == 2, N>(a.act, v);
#pragma unroll
                for (int j = 0; j < N; ++j) v[j] *= (float)dy[u][j];
#pragma unroll
                for (int j = 0; j < N; j += 4) *reinterpret_cast<f32x4 *>(D + r * po + c * N + j) = (f32x4){v[j], v[j + 1], v[j + 2], v[j + 3]};
            }
        }
        if (a.dw)
#pragma unroll 2
            for (int k = tid; k < R * ci; k += TH) {
                const int r = (k * mi >> 16), c = k - r * ci;
                put(X + r * pi, c, m0 + r < t.hi ? load_chunk((const T *)a.x + (m0 + r - x0) * a.ldx, c, ni, (T)0.0f) : (reg){});
            }
        __syncthreads();
        if (a.dx)
            for (int f = 0; f < F; ++f) {
                const int64_t m = m0 + (wave * F + f) * 16 + l16;
                const float *d = D + ((wave * F + f) * 16 + l16) * po;
                for (int i = 0; i < ti; ++i) {
                    f32x4 acc = (f32x4)(0.0f);
                    for (int k = 0; k < to; ++k) {
                        const f32x4 b = *reinterpret_cast<const f32x4 *>(d + k * 16 + 4 * q);
                        f32x4 w;
#pragma unroll
                        for (int e = 0; e < 4; ++e) w[e] = W[(k * 16 + 4 * q + e) * pi + i * 16 + l16];
                        acc = mma16(w, b, acc);
                    }
                    if (m < t.hi) store_quad((T *)a.dx + m * a.lddx + i * 16 + 4 * q, ni - (i * 16 + 4 * q), acc);
                }
            }
        if (a.dw)
#pragma unroll
            for (int s = 0; s < kDw; ++s) {
                const int u = F > 1 ? 0 : wave + s * WAVES;
                if (u >= ti * to) continue;
                const int o = u / ti, i = u - o * ti, k0 = F > 1 ? wave * 16 * F : 0;
#pragma unroll 1
                for (int k = k0; k < k0 + (F > 1 ? 16 * F : R); k += 16) {
                    f32x4 p, d;
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        p[e] = X[(k + 4 * q + e) * pi + i * 16 + l16];
                        d[e] = D[(k + 4 * q + e) * po + o * 16 + l16];
                    }
                    dw[s] = mma16(p, d, dw[s]);
                }
            }
        // db: a column per thread, the rows shared by the threads left over
        if (tid < shares * to * 16) {
#pragma unroll 4
            for (int r = tid / (to * 16); r < R; r += shares) db += D[r * po + tid % (to * 16)];
        }
    }
    __syncthreads();
    float *const join = X;  // [TH] db, then (F > 1) [WAVES][64] of the dw tile's quads
    join[tid] = db;
    if constexpr (F > 1) *reinterpret_cast<f32x4 *>(join + TH + 4 * tid) = dw[0];
    __syncthreads();
    for (int s = 1; tid < no && s < shares; ++s) db += join[s * to * 16 + tid];
    if constexpr (F > 1) {
        if (wave == 0)
#pragma unroll
            for (int w = 1; w < WAVES; ++w) dw[0] += *reinterpret_cast<const f32x4 *>(join + TH + 4 * (w * 64 + tid));
    }
    // the results, or this tile's sums
    float *sums = part + net_slot(t.lo, t.index, sh) * no * (ni + 1);
    if (a.dw)
#pragma unroll
        for (int s = 0; s < kDw; ++s) {
            const int u = wave + s * WAVES;
            if (u >= ti * to) continue;  // (F > 1: wave 0 alone)
            const int o = u / ti * 16 + l16, i = (u - u / ti * ti) * 16 + 4 * q;
            if (o < no)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    if (i + e >= ni) continue;
                    if (t.only) ((T *)a.dw)[t.g * a.dw_stride + o * a.lddw + i + e] = (T)dw[s][e];
                    else sums[o * ni + i + e] = dw[s][e];
                }
        }
    if (a.db && tid < no) {
        if (t.only) ((T *)a.db)[t.g * a.db_stride + tid] = (T)db;
        else sums[no * ni + tid] = db;
    }
}

// Rows per tile of the narrow gradient, as a power of two: about 2048 tiles, of
// 64 .. 4096 rows; whole networks of up to 4096 where these are enough for the chip
// (their results need no sums).  least: the fewest rows with or without offsets, for
// the scratch's size, which is asked for without them.
int narrow_shift(const LinearGradArgs &a, bool least = false)
{
    int sh = 6;
    while (sh < 12 && ((a.rows.M >> sh) > 2048 || (!least && !a.rows.off && a.rows.G >= 512 && a.rows.n > (int64_t)1 << sh))) ++sh;
    return sh;
}
// 16 bits, both widths above 48: the tiles' 16-bit products are no slower than fp32
// ones (bf16 100x1000 rows 64x64 without an activation 45 us, with tanh 58, here 60;
// 64x48 51 without, here 50).
bool narrow(const LinearGradArgs &a)
{
    return a.n_in <= kNarrow && a.n_out <= kNarrow && (a.dtype == NET_F32 || a.n_in <= 48 || a.n_out <= 48);
}

// ---------------------------------------------------------------------------
// The whole gradient of few inputs (up to 32) and more than 64 outputs in one pass:
// a block takes 64 rows of a network and goes over the outputs 64 at a time.  d
// passes through LDS as above, dx's sums stay in registers, and dw and db of the 64
// rows are written at every step, as results or as the tile's sums; dy and z are
// read once and d is never stored.  Bound by the slopes, the fp32 matrix cores (whose
// tiles one input fills as 16 do) and the steps' barriers, 3.4 us a step at three to
// four blocks per CU: bf16 300,000 rows 16x1109 with GELU 627 us, in separate passes
// through the tiles 1199 with d in one number (fp32 950, 2599); fp32 1408x51 rows 1x564
// 143, 399; bf16 856x581 rows 29x408 657, 682.  Where blocks are few and their steps
// many the tiles are faster: in 16 bits from more than 16 steps on (bf16 with tanh
// 16x334 rows 6x2204, 100 blocks of 35 steps, 108, 92; 10x320 rows 8x945, 60 of 15, 44,
// 76, without an activation 40, 41; 8x1280, 20 steps, 55, 59, without 50, 36), in fp32
// from 12.
// ---------------------------------------------------------------------------
constexpr int kFewInputs = 32, kFewShift = 6;

template <typename T, int TI>
__global__ __launch_bounds__(256, 3) void k_linear_grad_few(LinearGradArgs a, float *part)
{
    constexpr int N = NetVec<T>::N, R = 1 << kFewShift, C = 64, CI = TI * 16 / N, CO = C / N, pi = TI * 16 + 4, po = C + 4,
                  KD = R * CO / 256, KW = (C * CI + 255) / 256;
    typedef typename NetVec<T>::reg reg;
    __shared__ __attribute__((aligned(16))) float X[R * pi], W[C * pi], D[R * po];
    __shared__ float join[256];
    const NetTile t = net_tile(a.rows, kFewShift, net_block());
    if (t.g < 0) return;
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid / 64), l16 = tid % 16, q = tid % 64 / 16,
              ni = (int)a.n_in, no = (int)a.n_out, rows = (int)(t.hi - t.lo);
    auto put = [&](float *row, int c, reg v) {
#pragma unroll
        for (int j = 0; j < N; j += 4) *reinterpret_cast<f32x4 *>(row + c * N + j) = (f32x4){(float)v[j], (float)v[j + 1], (float)v[j + 2], (float)v[j + 3]};
    };
    if (a.dw) {
        const T *x = (const T *)a.x + (t.lo - (a.x_shared ? (int64_t)t.g * a.rows.n : 0)) * a.ldx;
#pragma unroll
        for (int k = tid; k < R * CI; k += 256) {
            const int r = k / CI, c = k % CI;
            put(X + r * pi, c, r < rows ? load_chunk(x + r * a.ldx, c, ni, (T)0.0f) : (reg){});
        }
    }
    const T *w = (const T *)a.w + t.g * a.w_stride, *pd = (const T *)a.dy + t.lo * a.lddy, *pz = (const T *)a.z + t.lo * a.ldz;
    reg dy[KD], z[KD], wv[KW];
    // the next 64 outputs' d and weights, in flight over a step
    const auto load = [&](int o0) {
#pragma unroll
        for (int u = 0; u < KD; ++u) {
            const int r = (tid + u * 256) / CO, c = (tid + u * 256) % CO + o0 / N;
            dy[u] = z[u] = (reg){};
            if (r >= rows || c * N >= no) continue;
            dy[u] = load_early(pd + r * a.lddy, c, no);
            if (a.act != ACT_NONE) z[u] = load_early(pz + r * a.ldz, c, no);
        }
        if (a.dx)
#pragma unroll
            for (int u = 0; u < KW; ++u) {
                const int o = (tid + u * 256) / CI + o0, c = (tid + u * 256) % CI;
                wv[u] = (reg){};
                if (tid + u * 256 < C * CI && o < no && c * N < ni) wv[u] = load_early(w + o * a.ldw, c, ni);
            }
    };
    f32x4 dx[TI];
#pragma unroll
    for (int i = 0; i < TI; ++i) dx[i] = (f32x4)(0.0f);
    float *sums = part + net_slot(t.lo, t.index, kFewShift) * no * (ni + 1);
    load(0);
#pragma unroll 1
    for (int o0 = 0; o0 < no; o0 += C) {
        if (o0 > 0) __syncthreads();
#pragma unroll
        for (int u = 0; u < KD; ++u) {
            const int r = (tid + u * 256) / CO, c = (tid + u * 256) % CO;
            settle(dy[u], c + o0 / N, no, (T)0.0f);
            settle(z[u], c + o0 / N, no, (T)0.0f);
            float v[N];
#pragma unroll
            for (int j = 0; j < N; ++j) v[j] = (float)z[u][j];
            act_slopes<sizeof(T) == 2, N>(a.act, v);
#pragma unroll
            for (int j = 0; j < N; ++j) v[j] *= (float)dy[u][j];
#pragma unroll
            for (int j = 0; j < N; j += 4) *reinterpret_cast<f32x4 *>(D + r * po + c * N + j) = (f32x4){v[j], v[j + 1], v[j + 2], v[j + 3]};
        }
        if (a.dx)
#pragma unroll
            for (int u = 0; u < KW; ++u) {
                const int o = (tid + u * 256) / CI, c = (tid + u * 256) % CI;
                settle(wv[u], c, ni, (T)0.0f);
                if (tid + u * 256 < C * CI) put(W + o * pi, c, wv[u]);
            }
        if (o0 + C < no) load(o0 + C);
        __syncthreads();
        if (a.dx) {
            const float *d = D + (wave * 16 + l16) * po + 4 * q;
#pragma unroll
            for (int k = 0; k < C; k += 16) {
                const f32x4 b = *reinterpret_cast<const f32x4 *>(d + k);
#pragma unroll
                for (int i = 0; i < TI; ++i) {
                    f32x4 p;
#pragma unroll
                    for (int e = 0; e < 4; ++e) p[e] = W[(k + 4 * q + e) * pi + i * 16 + l16];
                    dx[i] = mma16(p, b, dx[i]);
                }
            }
        }
        const int o = o0 + wave * 16 + l16;
        if (a.dw) {
            f32x4 dw[TI];
#pragma unroll
            for (int i = 0; i < TI; ++i) dw[i] = (f32x4)(0.0f);
#pragma unroll
            for (int k = 0; k < R; k += 16) {
                f32x4 d;
#pragma unroll
                for (int e = 0; e < 4; ++e) d[e] = D[(k + 4 * q + e) * po + wave * 16 + l16];
#pragma unroll
                for (int i = 0; i < TI; ++i) {
                    f32x4 p;
#pragma unroll
                    for (int e = 0; e < 4; ++e) p[e] = X[(k + 4 * q + e) * pi + i * 16 + l16];
                    dw[i] = mma16(p, d, dw[i]);
                }
            }
            if (o < no)
#pragma unroll
                for (int i = 0; i < TI; ++i) {
                    const int at = i * 16 + 4 * q;
                    if (t.only) store_quad((T *)a.dw + t.g * a.dw_stride + o * a.lddw + at, ni - at, dw[i]);
                    else store_quad(sums + (int64_t)o * ni + at, ni - at, dw[i]);
                }
        }
        if (a.db) {
            float s = 0.0f;
#pragma unroll
            for (int r = 0; r < R / 4; ++r) s += D[(tid / 64 * (R / 4) + r) * po + tid % 64];
            join[tid] = s;
            __syncthreads();
            if (tid < C && o0 + tid < no) {
                s += join[C + tid] + join[2 * C + tid] + join[3 * C + tid];
                if (t.only) ((T *)a.db)[t.g * a.db_stride + o0 + tid] = (T)s;
                else sums[(int64_t)no * ni + o0 + tid] = s;
            }
        }
    }
    const int m = wave * 16 + l16;
    if (a.dx && m < rows)
#pragma unroll
        for (int i = 0; i < TI; ++i)
            store_quad((T *)a.dx + (t.lo + m) * a.lddx + i * 16 + 4 * q, ni - (i * 16 + 4 * q), dx[i]);
}
bool few_inputs(const LinearGradArgs &a)
{
    const int64_t steps = a.dtype == NET_F32 ? 12 : 16;
    return a.n_in <= kFewInputs && a.n_out > kNarrow && (a.n_out <= steps * 64 || (a.rows.M >> kFewShift) + a.rows.G >= 512);
}

// ---------------------------------------------------------------------------
// Gradient products of a short sum: dx of few outputs (DW = false: rows m of a
// tile, k the outputs) and dw of few rows per network (rows o, k the network's
// rows).  Either is out[r][c] = sum_k p[k][c] q(r, k) with p and the result dense
// along c, so the matrix cores' tiles would be mostly padding and the bytes bound
// it: a thread takes four rows by one chunk of 16 bytes of columns, the block 16
// rows (a tile's, or outputs) by L chunks.  For sums of at most 8 outputs or 4
// rows over at least 64 columns: the whole gradient of 1566 networks' 2 rows
// 304x1 takes 25 us, 101 in tiles; of 100,000 rows 1000x16 (bf16) 163, in tiles 143.
// LOW: of both numbers of d, a kernel of its own: in one with a branch the gradient
// without an activation of bf16 500x3 rows 1000x1000 took 577 us, 539 so.
// ---------------------------------------------------------------------------
constexpr int kShortRows = 16, kShortShift = 4, kShortOutputs = 8, kShortMean = 4;

template <typename T, bool DW, bool LOW>
__global__ __launch_bounds__(256) void k_linear_short(LinearGradArgs a, const T *d, const T *low, int64_t ldd, int L, int64_t units)
{
    constexpr int N = NetVec<T>::N;
    typedef typename NetVec<T>::reg reg;
    const int64_t cols = (a.n_in + L * N - 1) / (L * N), unit = net_block() / cols;
    const int lane = threadIdx.x & (L - 1), slot = threadIdx.x / L, slots = 256 / L, ni = (int)a.n_in,
              c = (int)(net_block() - unit * cols) * L + lane;
    if (unit >= units) return;
    int g, R;
    int64_t K;
    const T *p, *q, *ql;
    T *out;
    int64_t ldp, ldo;
    if constexpr (DW) {
        const int64_t tiles = (a.n_out + kShortRows - 1) / kShortRows;
        g = (int)(unit / tiles);
        const int o0 = (int)(unit - g * tiles) * kShortRows;
        int64_t lo, hi;
        net_rows(a.rows, g, &lo, &hi);
        R = min((int)a.n_out - o0, kShortRows);
        K = hi - lo;
        p = (const T *)a.x + (a.x_shared ? 0 : lo) * a.ldx;
        ldp = a.ldx;
        q = d + lo * ldd + o0;
        ql = low + lo * ldd + o0;
        out = (T *)a.dw + g * a.dw_stride + o0 * a.lddw;
        ldo = a.lddw;
    } else {
        const NetTile t = net_tile(a.rows, kShortShift, unit);
        if (t.g < 0) return;
        R = (int)(t.hi - t.lo);
        K = a.n_out;
        p = (const T *)a.w + t.g * a.w_stride;
        ldp = a.ldw;
        q = d + t.lo * ldd;
        ql = low + t.lo * ldd;
        out = (T *)a.dx + t.lo * a.lddx;
        ldo = a.lddx;
    }
    if (c * N >= ni) return;
    // up to four of d's neighbours
    const auto load_d = [&](int64_t at, int n) -> f32x4 {
        const f32x4 h = load_quad(q + at, n);
        if constexpr (LOW) return h * d_up<T> + load_quad(ql + at, n) * d_down<T>;
        else return h;
    };
    for (int r0 = slot * 4; r0 < R; r0 += slots * 4) {
        float acc[4][N];
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int j = 0; j < N; ++j) acc[r][j] = 0.0f;
        const int rows = R - r0;
        // four k at a time (zeros past the last)
        for (int64_t k = 0; k < K; k += 4) {
            const int left = K - k < 4 ? (int)(K - k) : 4;
            reg pv[4];
            f32x4 qv[4];  // DW: [k] over rows, else [row] over k
#pragma unroll
            for (int e = 0; e < 4; ++e) pv[e] = e < left ? load_chunk(p + (k + e) * ldp, c, ni, (T)0.0f) : (reg){};
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if constexpr (DW) qv[e] = e < left ? load_d((k + e) * ldd + r0, rows) : (f32x4)(0.0f);
                else qv[e] = e < rows ? load_d((r0 + e) * ldd + k, left) : (f32x4)(0.0f);
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
                for (int r = 0; r < 4; ++r)
#pragma unroll
                    for (int j = 0; j < N; ++j) acc[r][j] = fmaf(DW ? qv[e][r] : qv[r][e], (float)pv[e][j], acc[r][j]);
        }
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            if (r >= rows) continue;
            reg v;
#pragma unroll
            for (int j = 0; j < N; ++j) v[j] = (T)acc[r][j];
            store_chunk(out + (r0 + r) * ldo, c, ni, v);
        }
    }
}

// dx and dw of so few tiles that most CUs would idle through a long K: its shares
// are summed by blocks of their own, into fp32 partial results that are then added
// in order: about four blocks per CU, of at least 256 of K.  Decided by the sizes
// alone (the scratch is sized by them), for tiles of 64 a side.  fp32 5 networks'
// 12 rows 331x1756 49 us, 125 without; half as many blocks: bf16 300,000 rows 18x1109
// 1364 us, 1296 so, fp32 4096 rows 1024x1024 194, 183, bf16 20,000 rows 300x300 90, 102.
int grad_splits(int64_t tiles, int64_t K)
{
    int64_t s = 1024 / (tiles < 1 ? 1 : tiles);
    if (s > K / 256) s = K / 256;
    return s < 2 ? 1 : s > 64 ? 64 : (int)s;
}
int dx_splits(const LinearGradArgs &a)
{
    const int64_t rows = (a.rows.M + 63) / 64;
    return grad_splits((a.n_in + 63) / 64 * (rows > a.rows.G ? rows : a.rows.G), a.n_out);
}
int dw_splits(const LinearGradArgs &a)
{
    return grad_splits(a.rows.G * ((a.n_in + 63) / 64) * ((a.n_out + 63) / 64), (a.rows.M + a.rows.G - 1) / a.rows.G);
}

// out[r][c] = sum over the splits, of `rows` rows of n at part[z][r][c]; row r is at
// (r / per) stride + (r % per) ld of the result.  Rows of no network stay.
template <typename T>
__global__ __launch_bounds__(256) void k_linear_join(NetRows rows, const float *part, int splits, int64_t count, int64_t n,
                                                     T *out, int64_t per, int64_t stride, int64_t ld, bool by_row)
{
    const int64_t total = count * n;
    for (int64_t e = net_block() * 256 + threadIdx.x; e < total; e += (int64_t)gridDim.x * gridDim.y * 256) {
        const int64_t r = e / n, c = e - r * n;
        if (by_row && rows.off && net_of_row(rows, r) < 0) continue;
        float s = part[e];
        for (int z = 1; z < splits; ++z) s += part[z * total + e];
        out[r / per * stride + r % per * ld + c] = (T)s;
    }
}

// The scratch: d (in 16 bits its two numbers, for any activation), then the tiles'
// column sums, then the partial products; of narrow layers, the tiles' sums.
struct GradScratch {
    int64_t ldd = 0;
    size_t low = 0, sums = 0, part = 0, end = 0;
};
GradScratch grad_layout(const LinearGradArgs &a)
{
    GradScratch g;
    if (narrow(a) || few_inputs(a)) {
        g.end = 4 * (size_t)net_slots(a.rows.M, few_inputs(a) ? kFewShift : narrow_shift(a, true)) * (size_t)(a.n_out * (a.n_in + 1));
        return g;
    }
    const size_t e = a.dtype == NET_F32 ? 4 : 2;
    g.ldd = (a.n_out + 7) / 8 * 8;
    g.low = (e * (size_t)a.rows.M * (size_t)g.ldd + 255) / 256 * 256;
    g.sums = a.dtype == NET_F32 ? g.low : 2 * g.low;
    g.part = (g.sums + 4 * (size_t)net_slots(a.rows.M, dz_shape(a).sh) * (size_t)a.n_out + 255) / 256 * 256;
    const size_t dx = dx_splits(a) > 1 ? (size_t)dx_splits(a) * (size_t)a.rows.M * (size_t)a.n_in : 0;
    const size_t dw = dw_splits(a) > 1 ? (size_t)dw_splits(a) * (size_t)(a.rows.G * a.n_out) * (size_t)a.n_in : 0;
    g.end = g.part + 4 * (dx > dw ? dx : dw);
    return g;
}

int64_t mean_rows(const NetRows &r) { return (r.M + r.G - 1) / r.G; }

// The tiles, for their reuse, where their padding (64 rows, outputs and k) is
// not most of them (without / with, us: bf16 512x512 24 rows 39 / 38, 48 rows 52 / 44,
// fp32 77 / 78, 157 / 83; 500 rows 256x32 bf16 11 / 10, fp32 24 / 30, 256x48 15 / 10,
// 38 / 30; 500 rows 64x300 24 / 28, 44 / 44, fp32 96x300 60 / 53), and where they are
// not too few for the chip (tiles of 64 a side: 128, one network's 512 rows
// 2048x1024, 18 / 22, 34 / 64; 192, 1024 rows 4096x768, 46 / 39, 93 / 118; 256, 1024 rows
// 1024x1024, 18 / 14, 35 / 37; 384, 1024 rows 2048x1536, 46 / 24, 95 / 64).
template <typename T>
bool wide(const LinearArgs &a)
{
    return mean_rows(a.rows) > 24 && a.n_out > 32 && a.n_in >= (sizeof(T) == 2 ? 128 : 64);
}
template <typename T>
bool tiles(const LinearArgs &a)
{
    return wide<T>(a) && net_tiles(a.rows, 6) * ((a.n_out + 63) / 64) > (sizeof(T) == 2 ? 128 : 256);
}

// Short sums: of few outputs (dx) or rows (dw; in fp32 dx too, whose tiles would
// split every weight for two rows: 207x2 rows 3496x386 521 us, 611 in tiles, 1500x2 rows
// 520x300 428, 547; bf16 1500x1 rows 100x300 312, 98, others even).
template <typename T>
bool short_dx(const LinearGradArgs &a)
{
    return (a.n_out <= kShortOutputs || (sizeof(T) == 4 && mean_rows(a.rows) <= kShortMean)) && a.n_in >= 64;
}
bool short_dw(const LinearGradArgs &a) { return mean_rows(a.rows) <= kShortMean && a.n_in >= 64; }

}  // namespace

void linear_kernels(const LinearGradArgs &a, int32_t *forward, int32_t *dx, int32_t *dw)
{
    net_dispatch(a.dtype, [&](auto t) {
        using T = typename NetElement<t.value>::type;
        LinearArgs l{};
        l.rows = a.rows;
        l.n_in = a.n_in;
        l.n_out = a.n_out;
        const auto of_tiles = [](int shape, int splits) { return EVOX_KERNEL_TILES + shape + (splits > 1 ? EVOX_KERNEL_SHARES : 0); };
        *forward = tiles<T>(l) ? of_tiles(linear_tiles_shape<t.value>(l), 1) : EVOX_KERNEL_ROWS;
        if (narrow(a)) *dx = *dw = EVOX_KERNEL_NARROW;
        else if (few_inputs(a)) *dx = *dw = EVOX_KERNEL_FEW_INPUTS;
        else {
            *dx = short_dx<T>(a) ? (int)EVOX_KERNEL_SHORT : of_tiles(linear_dx_tiles_shape<t.value>(a, dx_splits(a)), dx_splits(a));
            *dw = short_dw(a) ? (int)EVOX_KERNEL_SHORT : of_tiles(linear_dw_tiles_shape<t.value>(a, dw_splits(a)), dw_splits(a));
        }
        return hipSuccess;
    });
}

hipError_t launch_linear(const LinearArgs &a, hipStream_t s)
{
    return net_dispatch(a.dtype, [&](auto t) {
        using T = typename NetElement<t.value>::type;
        if (tiles<T>(a)) return launch_linear_tiles<t.value>(a, s);
        const int64_t mean = mean_rows(a.rows);
        // rows of a wave's tile by the mean rows per network (few k steps of 16 bits or
        // outputs: smaller tiles, more waves at a time: 200 rows 32x200 bf16 12.1, with 64 x
        // 32 13.0 us); one 16 x 16 tile where larger ones would leave most of the chip
        // without a wave (one network's 3000 rows 512x24 9.3, 10.9 us; fp32 512 rows 2048x256,
        // 128 tiles of 32 x 32, 17.6, 19.0; 4x128 rows 1024x512, 256 of them, 17.4, 12.4)
        const bool few_steps = a.n_in <= 2 * Mma<T>::KS && (sizeof(T) == 2 || a.n_out <= 16);
        int rb = mean <= 16 ? 1 : mean <= 32 || few_steps || wide<T>(a) ? 2 : 4, nb = rb == 1 || a.n_out <= 16 ? 1 : 2;
        const int64_t steps = (a.n_in + Mma<T>::KS - 1) / Mma<T>::KS;
        const auto units_of = [&](int r, int n) {
            return net_tiles(a.rows, r == 1 ? 4 : r == 2 ? 5 : 6) * ((a.n_out + 16 * n - 1) / (16 * n));
        };
        if (steps >= 16 && units_of(rb, nb) < 192) rb = nb = 1;
        const int sh = rb == 1 ? 4 : rb == 2 ? 5 : 6;
        const uint32_t out_tiles = (uint32_t)((a.n_out + 16 * nb - 1) / (16 * nb));
        const int64_t units = units_of(rb, nb);
        // a long K to four waves (one / four, us: bf16 one row 2048x2048 380 / 347, 8 rows
        // 1024x1024 868 / 958; fp32 761 / 698, 1734 / 1681, 8 rows 512x512 215 / 213), and a
        // shorter one where tiles are few (one network's 16 rows 2048x1024 17 / 9)
        const bool split = (units < 4096 && steps >= 16) || (rb < 4 && steps >= (sizeof(T) == 2 ? 64 : 32));
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
        else if (rb == 2 && nb == 1) go(integral_constant<int, 2>{}, integral_constant<int, 1>{});
        else if (rb == 2) go(integral_constant<int, 2>{}, integral_constant<int, 2>{});
        else if (nb == 1) go(integral_constant<int, 4>{}, integral_constant<int, 1>{});
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
        const int64_t mean = mean_rows(a.rows);
        hipError_t e = hipSuccess;
        if (narrow(a) || few_inputs(a)) {
            const int sh = few_inputs(a) ? kFewShift : narrow_shift(a);
            float *part = (float *)a.scratch;
            auto go = [&](auto waves, auto f) {
                const int64_t ti = (a.n_in + 15) / 16 * 16, to = (a.n_out + 15) / 16 * 16;
                const size_t lds = sizeof(float) * ((a.dx ? to * (ti + 4) : 0) + 16 * waves.value * f.value * (ti + 4 + to + 4));
                hipLaunchKernelGGL((k_linear_grad_narrow<T, waves.value, f.value>), net_grid(net_tiles(a.rows, sh)),
                                   dim3(64 * waves.value), lds, s, a, sh, part);
                return hipGetLastError();
            };
            if (a.rows.M > 0) {
                using std::integral_constant;
                const dim3 few = net_grid(net_tiles(a.rows, sh));
                if (few_inputs(a) && a.n_in <= 16) {
                    hipLaunchKernelGGL((k_linear_grad_few<T, 1>), few, dim3(256), 0, s, a, part);
                    e = hipGetLastError();
                } else if (few_inputs(a)) {
                    hipLaunchKernelGGL((k_linear_grad_few<T, 2>), few, dim3(256), 0, s, a, part);
                    e = hipGetLastError();
                } else if (mean <= 32) e = go(integral_constant<int, 2>{}, integral_constant<int, 1>{});
                else if (mean > 128 && a.n_in <= 16 && a.n_out <= 16) e = go(integral_constant<int, 4>{}, integral_constant<int, 4>{});
                else e = go(integral_constant<int, 4>{}, integral_constant<int, 1>{});
            }
            if (e != hipSuccess || (!a.dw && !a.db) || (a.rows.M > 0 && !a.rows.off && net_single(a.rows, sh))) return e;
            return launch_net_sums(a.rows, part, a.n_out * (a.n_in + 1), sh, s,
                                   GradSums<T>{(T *)a.dw, (T *)a.db, a.n_out, a.n_in, a.lddw, a.dw_stride, a.db_stride});
        }
        const DzShape dz = dz_shape(a);
        const bool own = a.act != ACT_NONE && (a.dx || a.dw);
        T *d = own ? (T *)a.scratch : nullptr;
        T *low = own && sizeof(T) == 2 && a.act > ACT_RELU ? (T *)((char *)a.scratch + l.low) : nullptr;
        float *sums = a.db ? (float *)((char *)a.scratch + l.sums) : nullptr;
        if (a.rows.M > 0 && (d || sums)) {
            hipLaunchKernelGGL((k_linear_dz<T>), net_grid(net_tiles(a.rows, dz.sh) * dz.cols), dim3(256),
                               sizeof(float) * N * (256 - dz.L), s, a, dz.sh, dz.L, dz.cols, d, low, l.ldd, sums);
            if ((e = hipGetLastError()) != hipSuccess) return e;
        }
        if (a.db && !(a.rows.M > 0 && !a.rows.off && net_single(a.rows, dz.sh))) {
            e = launch_net_sums(a.rows, sums, a.n_out, dz.sh, s,
                                GradSums<T>{nullptr, (T *)a.db, a.n_out, 0, 0, 0, a.db_stride});
            if (e != hipSuccess) return e;
        }
        const void *dd = own ? d : a.dy;
        const int64_t ldd = own ? l.ldd : a.lddy;
        float *part = (float *)((char *)a.scratch + l.part);
        int L = 1;  // of short sums
        while (L < 256 && L * N < a.n_in) L *= 2;
        const int64_t cols = (a.n_in + L * N - 1) / (L * N);
        const auto short_sums = [&](auto dw, int64_t units) {
            constexpr bool DW = dw.value;
            auto kernel = k_linear_short<T, DW, false>;
            if constexpr (sizeof(T) == 2)
                if (low) kernel = k_linear_short<T, DW, true>;
            hipLaunchKernelGGL(kernel, net_grid(units * cols), dim3(256), 0, s, a, (const T *)dd, low, ldd, L, units);
            return hipGetLastError();
        };
        if (a.dx && short_dx<T>(a)) e = short_sums(std::false_type{}, net_tiles(a.rows, kShortShift));
        else if (a.dx) {
            const int splits = dx_splits(a);
            e = launch_linear_dx_tiles<t.value>(a, dd, low, ldd, splits, part, s);
            if (e == hipSuccess && splits > 1) {
                hipLaunchKernelGGL((k_linear_join<T>), net_grid((a.rows.M * a.n_in + 255) / 256), dim3(256), 0, s, a.rows,
                                   part, splits, a.rows.M, a.n_in, (T *)a.dx, a.rows.M, (int64_t)0, a.lddx, true);
                e = hipGetLastError();
            }
        }
        if (e != hipSuccess || !a.dw) return e;
        if (short_dw(a)) return short_sums(std::true_type{}, a.rows.G * ((a.n_out + kShortRows - 1) / kShortRows));
        const int splits = dw_splits(a);
        e = launch_linear_dw_tiles<t.value>(a, dd, low, ldd, splits, part, s);
        if (e != hipSuccess || splits == 1) return e;
        const int64_t rows = a.rows.G * a.n_out;
        hipLaunchKernelGGL((k_linear_join<T>), net_grid((rows * a.n_in + 255) / 256), dim3(256), 0, s, a.rows, part, splits,
                           rows, a.n_in, (T *)a.dw, a.n_out, a.dw_stride, a.lddw, false);
        return hipGetLastError();
    });
}

}  // namespace evox
