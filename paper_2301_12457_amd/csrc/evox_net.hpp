// Layers, norms and losses of a population of networks: the kernels' arguments,
// element types and the rows of each network.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>
#include <type_traits>

namespace evox {

enum NetType { NET_F32 = 0, NET_BF16 = 1, NET_F16 = 2 };
enum NetAct { ACT_NONE = 0, ACT_RELU = 1, ACT_TANH = 2, ACT_GELU = 3, ACT_SILU = 4, ACT_COUNT = 5 };
constexpr int64_t kNetMaxG = (int64_t)1 << 20, kNetMaxWidth = (int64_t)1 << 20;

// The rows of the networks: off[g] .. off[g + 1), or n each.
struct NetRows {
    const int32_t *off;
    int64_t G, M, n;  // n = M / G where off is null
};

struct LinearArgs {
    NetRows rows;
    int32_t dtype, act, x_shared;
    int64_t n_in, n_out;
    const void *x, *w, *b, *r;
    void *z, *y;
    int64_t ldx, ldw, w_stride, b_stride, ldr, ldz, ldy;
};
struct LinearGradArgs {
    NetRows rows;
    int32_t dtype, act, x_shared;
    int64_t n_in, n_out;
    const void *x, *w, *z, *dy;
    void *dx, *dw, *db;
    int64_t ldx, ldw, w_stride, ldz, lddy, lddx, lddw, dw_stride, db_stride;
    void *scratch;
};
struct NormArgs {
    NetRows rows;
    int32_t dtype;
    int64_t D;
    const void *x, *gamma, *beta, *dy;
    void *y, *dx, *dgamma, *dbeta;
    float *mean, *rstd;              // written by the norm
    const float *mean_in, *rstd_in;  // read by its gradient
    int64_t ldx, ldy, lddx, p_stride, dp_stride;
    float eps;
    void *scratch;
};
struct XentArgs {
    NetRows rows;
    int32_t dtype, labels_shared;
    int64_t C;
    const void *logits;
    const int32_t *labels;
    float *fit;
    void *dz;
    int64_t ldz, lddz;
    void *scratch;
};
hipError_t launch_linear(const LinearArgs &a, hipStream_t s);
size_t linear_grad_scratch(const LinearGradArgs &a);  // of the sizes alone
hipError_t launch_linear_grad(const LinearGradArgs &a, hipStream_t s);
hipError_t launch_layernorm(const NormArgs &a, hipStream_t s);
size_t layernorm_grad_scratch(const NormArgs &a);
hipError_t launch_layernorm_grad(const NormArgs &a, hipStream_t s);
size_t xent_scratch(const XentArgs &a);
hipError_t launch_xent(const XentArgs &a, hipStream_t s);

// The large cases: tiles through LDS (one file per element type).  d: dy act'(z)
// in the element type, low: its second number (d_split) or null.  splits > 1: K in so
// many shares, partial results to part[z].
template <int TYPE>
hipError_t launch_linear_tiles(const LinearArgs &a, hipStream_t s);
template <int TYPE>
hipError_t launch_linear_dx_tiles(const LinearGradArgs &a, const void *d, const void *low, int64_t ldd, int splits,
                                  float *part, hipStream_t s);
template <int TYPE>
hipError_t launch_linear_dw_tiles(const LinearGradArgs &a, const void *d, const void *low, int64_t ldd, int splits,
                                  float *part, hipStream_t s);

// The tile shape that the same calls take (0 .. 3; 4: dx of a pair).
template <int TYPE>
int linear_tiles_shape(const LinearArgs &a);
template <int TYPE>
int linear_dx_tiles_shape(const LinearGradArgs &a, int splits);
template <int TYPE>
int linear_dw_tiles_shape(const LinearGradArgs &a, int splits);

// Which kernels a layer and its gradient take (enum evox_layer_kernel).
void linear_kernels(const LinearGradArgs &a, int32_t *forward, int32_t *dx, int32_t *dw);

typedef __bf16 bf16_t;
typedef _Float16 f16_t;

template <int TYPE>
struct NetElement {
    typedef f16_t type;
};
template <>
struct NetElement<NET_F32> {
    typedef float type;
};
template <>
struct NetElement<NET_BF16> {
    typedef bf16_t type;
};

// d = dy act'(z) for 16-bit products as two numbers of the type: the rounded one and
// what it leaves, d = d_up<T> high + d_down<T> low within u^2 |d| (u: the type's
// roundoff).  f16's range is narrower than d's (a slope may be 1.13, or 2^-20): its
// first number is d / 2, so that none overflows, its second 2^10 times as large, so
// that 2^-35 is still kept.  An infinity or NaN is the first one's alone.
template <typename T>
inline constexpr float d_up = std::is_same<T, f16_t>::value ? 2.0f : 1.0f;
template <typename T>
inline constexpr float d_down = std::is_same<T, f16_t>::value ? 0x1p-10f : 1.0f;
template <typename T>
__device__ __forceinline__ void d_split(float d, T &high, T &low)
{
    high = (T)(d * (1.0f / d_up<T>));
    const float r = d - (float)high * d_up<T>;
    low = (T)(fabsf(r) < INFINITY ? r * (1.0f / d_down<T>) : 0.0f);
}

// Type-dependent launches: f is called with an integral constant, the type.
template <typename F>
hipError_t net_dispatch(int32_t dtype, F &&f)
{
    if (dtype == NET_F32) return f(std::integral_constant<int, NET_F32>{});
    if (dtype == NET_BF16) return f(std::integral_constant<int, NET_BF16>{});
    return f(std::integral_constant<int, NET_F16>{});
}

// Sixteen bytes of a row: loads and stores need only the element's alignment
// (gfx950 takes a dwordx4 at any address).
template <typename T>
struct NetVec {
    static constexpr int N = 16 / (int)sizeof(T);
    typedef T reg __attribute__((ext_vector_type(N)));
    typedef T mem __attribute__((ext_vector_type(N), aligned(sizeof(T))));
};

// Elements [c N, c N + N) of a row of n, `fill` past its end.  NT: stored with the
// streaming hint.
template <typename T>
__device__ __forceinline__ typename NetVec<T>::reg load_chunk(const T *row, int c, int n, T fill)
{
    constexpr int N = NetVec<T>::N;
    const int at = c * N;
    if (at + N <= n) return *reinterpret_cast<const typename NetVec<T>::mem *>(row + at);
    typename NetVec<T>::reg v;
#pragma unroll
    for (int j = 0; j < N; ++j) v[j] = at + j < n ? row[at + j] : fill;
    return v;
}
// The same in two steps, for loads that are to stay in flight: rows' last chunks
// are loaded from the row's last N elements, without the wait that a branch for
// them would bring (f16 norm gradient of 67,392 rows of 2625: 427 us with it, 285
// without; fp32 narrow gradient of 4096x32 rows 31x31 45, 39), and settle(), at
// their first use, moves these to their places.  Rows whose
// other chunks other lanes may have written by then take load_chunk.
template <typename T>
__device__ __forceinline__ typename NetVec<T>::reg load_early(const T *row, int c, int n)
{
    constexpr int N = NetVec<T>::N;
    if (n < N) return load_chunk(row, c, n, (T)0.0f);
    return *reinterpret_cast<const typename NetVec<T>::mem *>(row + min(c * N, n - N));
}
template <typename T>
__device__ __forceinline__ void settle(typename NetVec<T>::reg &v, int c, int n, T fill)
{
    constexpr int N = NetVec<T>::N;
    const int past = c * N + N - n;
    if (past <= 0) return;
    if (n >= N)
#pragma unroll
        for (int b = 1; b < N; b *= 2)
            if (past & b)
#pragma unroll
                for (int j = 0; j + b < N; ++j) v[j] = v[j + b];
#pragma unroll
    for (int j = 0; j < N; ++j)
        if (j >= N - past) v[j] = fill;
}
template <typename T, bool NT = false>
__device__ __forceinline__ void store_chunk(T *row, int c, int n, typename NetVec<T>::reg v)
{
    constexpr int N = NetVec<T>::N;
    const int at = c * N;
    if (at + N <= n) {
        auto *p = reinterpret_cast<typename NetVec<T>::mem *>(row + at);
        if constexpr (NT) __builtin_nontemporal_store((typename NetVec<T>::mem)v, p);
        else *p = v;
        return;
    }
#pragma unroll
    for (int j = 0; j < N; ++j)
        if (at + j < n) row[at + j] = v[j];
}

__device__ __forceinline__ int64_t net_off(const NetRows &r, int64_t g)
{
    const int64_t o = r.off[g];
    return o < 0 ? 0 : o > r.M ? r.M : o;
}

// Grids of any number of blocks: HIP bounds the threads of a grid dimension by
// 2^32, so the blocks are laid over two.
inline dim3 net_grid(int64_t blocks)
{
    const int64_t x = (int64_t)1 << 20;
    return blocks <= x ? dim3((unsigned)blocks) : dim3((unsigned)x, (unsigned)((blocks + x - 1) / x));
}
__device__ __forceinline__ int64_t net_block() { return (int64_t)blockIdx.y * gridDim.x + blockIdx.x; }

// The rows [lo, hi) of network g, within [0, M] whatever off holds.
__device__ __forceinline__ void net_rows(const NetRows &r, int64_t g, int64_t *lo, int64_t *hi)
{
    if (!r.off) {
        *lo = g * r.n;
        *hi = *lo + r.n;
        return;
    }
    const int64_t b = net_off(r, g + 1);
    *lo = net_off(r, g);
    *hi = b < *lo ? *lo : b;
}

// The network of a row: the last g with off[g] <= row (networks without rows
// share their offset with the next), or -1 where the row belongs to none.
__device__ __forceinline__ int net_of_row(const NetRows &r, int64_t row)
{
    if (!r.off) return (int)((uint32_t)row / (uint32_t)r.n);
    int lo = -1, hi = (int)r.G;  // off[lo] <= row < off[hi]
    while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if (r.off[mid] <= row) lo = mid;
        else hi = mid;
    }
    return lo >= 0 && row < r.off[lo + 1] ? lo : -1;
}

// Tiles of 2^sh rows that stay within a network, numbered so that a network's
// first tile needs its own offset alone: T(g) = (off[g] >> sh) + g.  T grows by
// at least the network's tile count from one network to the next (by one more
// where its rows do not fill their tiles), so (M >> sh) + G numbers hold all,
// some of them of no rows.  With as many rows for each, T(g) = g ceil(n / 2^sh).
struct NetTile {
    int g;           // -1: no rows
    int index;       // of the network's tiles
    int64_t lo, hi;  // rows
    bool only;       // the network has no other tile
};
__host__ __device__ __forceinline__ int64_t net_tiles(const NetRows &r, int sh)
{
    const int64_t per = (r.n + ((int64_t)1 << sh) - 1) >> sh;
    return r.off ? (r.M >> sh) + r.G : r.G * per;
}
__device__ __forceinline__ int64_t net_first_tile(const NetRows &r, int sh, int64_t g)
{
    return r.off ? (net_off(r, g) >> sh) + g : g * ((r.n + ((int64_t)1 << sh) - 1) >> sh);
}
// The tile's network by 64 probes at a time, one per lane (all lanes of the
// wave must call with the same t).
__device__ __forceinline__ NetTile net_tile(const NetRows &r, int sh, int64_t t)
{
    NetTile o;
    o.g = -1;
    if (t >= net_tiles(r, sh)) return o;
    if (!r.off) {
        const uint32_t per = (uint32_t)((r.n + ((int64_t)1 << sh) - 1) >> sh);
        const uint32_t g = (uint32_t)t / per;
        o.index = (int)((uint32_t)t - g * per);
        o.lo = (int64_t)g * r.n + ((int64_t)o.index << sh);
        o.hi = (int64_t)(g + 1) * r.n;
        o.g = (int)g;
        o.only = per == 1;
    } else {
        int lo = 0, hi = (int)r.G;
        const int lane = threadIdx.x % 64;
        while (hi - lo > 1) {
            const int step = (hi - lo + 63) / 64, p = lo + lane * step;
            const bool in = p < hi && net_first_tile(r, sh, p) <= t;
            const int n = __popcll(__ballot(in));
            if (n == 0) return o;
            lo += (n - 1) * step;
            hi = lo + step < hi ? lo + step : hi;
        }
        int64_t a, b;
        net_rows(r, lo, &a, &b);
        const int64_t i = t - ((a >> sh) + lo);
        o.lo = a + (i << sh);
        o.hi = b;
        o.index = (int)i;
        if (i < 0 || o.lo >= b) return o;
        o.g = lo;
        o.only = b - a <= ((int64_t)1 << sh);
    }
    if (o.hi > o.lo + ((int64_t)1 << sh)) o.hi = o.lo + ((int64_t)1 << sh);
    // the same in every lane: scalar registers, and scalar bases for the rows' addresses
    o.g = __builtin_amdgcn_readfirstlane(o.g);
    o.index = __builtin_amdgcn_readfirstlane(o.index);
    o.lo = __builtin_amdgcn_readfirstlane((int)o.lo);
    o.hi = __builtin_amdgcn_readfirstlane((int)o.hi);
    o.only = __builtin_amdgcn_readfirstlane((int)o.only);
    return o;
}

// Sums over a network's rows: the network's only tile writes its result, several
// leave fp32 partial sums, added in the tiles' order by k_net_sums.  A partial's
// place is its tile's first row over 2^sh, doubled, plus one after the network's
// first tile: a network of several tiles covers whole blocks of 2^sh rows, so no
// two such tiles meet, and 2 (M / 2^sh + 1) places are enough for any offsets
// (a place per tile would be one per network, even of a single row).
__device__ __forceinline__ int64_t net_slot(int64_t lo, int index, int sh) { return 2 * (lo >> sh) + (index > 0); }
__host__ __device__ __forceinline__ int64_t net_slots(int64_t M, int sh) { return 2 * ((M >> sh) + 1); }
// Whether every network has at most one tile, for certain.
inline bool net_single(const NetRows &r, int sh) { return r.off ? r.M <= ((int64_t)1 << sh) : r.n <= ((int64_t)1 << sh); }

// out(g, e, sum) for the networks of several tiles and those without rows (sum
// 0): E elements by S shares of the tiles per block, 64 by 4, or 16 by 64 where
// networks have more than 64 tiles on average (the narrow gradient of 500,000 rows
// 32x32 of one network, 1954 tiles of 1056 elements: 76 us, 123 with 64 by 4).  A
// block takes several networks' where there would be more than 8192 blocks
// (bf16 gradient of 517 networks' 38 rows 29x3006: 544 us, 679 with one per block).
template <typename F, int E, int S>
__global__ __launch_bounds__(E * S) void k_net_sums(NetRows rows, const float *part, int64_t width, int sh, F out)
{
    __shared__ float share[S][E];
    const int64_t e = (int64_t)blockIdx.x * E + threadIdx.x % E;
    const int w = threadIdx.x / E;
    for (int64_t g = blockIdx.y; g < rows.G; g += gridDim.y) {
        int64_t lo, hi;
        net_rows(rows, g, &lo, &hi);
        const int64_t n = (hi - lo + ((int64_t)1 << sh) - 1) >> sh, per = (n + S - 1) / S;
        if (n == 1) continue;
        float s = 0.0f;
        if (e < width) {
            const int64_t t1 = (w + 1) * per < n ? (w + 1) * per : n;
#pragma unroll 8
            for (int64_t t = w * per; t < t1; ++t) s += part[net_slot(lo + (t << sh), (int)t, sh) * width + e];
        }
        share[w][threadIdx.x % E] = s;
        __syncthreads();
        if (w == 0 && e < width) {
            for (int k = 1; k < S; ++k) s += share[k][threadIdx.x];
            out(g, e, s);
        }
        __syncthreads();
    }
}
template <typename F>
hipError_t launch_net_sums(const NetRows &rows, const float *part, int64_t width, int sh, hipStream_t s, F out)
{
    const bool many = (rows.M >> sh) / rows.G > 64;
    const int64_t x = (width + (many ? 15 : 63)) / (many ? 16 : 64), most = x < 8192 ? 8192 / x : 1;
    const dim3 grid((unsigned)x, (unsigned)(rows.G < most ? rows.G : most));
    if (many) hipLaunchKernelGGL((k_net_sums<F, 16, 64>), grid, dim3(1024), 0, s, rows, part, width, sh, out);
    else hipLaunchKernelGGL((k_net_sums<F, 64, 4>), grid, dim3(256), 0, s, rows, part, width, sh, out);
    return hipGetLastError();
}

// Activations and their slopes.  For results of 16 bits the hardware's exp2
// and reciprocal (1 ulp) stand in for expf and the division, and the normal
// distribution's upper tail is Q(x) = e^(-x^2/2) t (a1 + .. + a7 t^6) / 2, t = 1 /
// (1 + p x) (the form of Abramowitz and Stegun 7.1.26; the coefficients minimise the
// larger of the error over 1.5e-7 and the relative one over 1e-5, x up to 13.6: at most
// 1e-7 and 3.1e-6.  Their own five are within 7.5e-8, but a bf16 GELU(-8) came out 1e-2
// off); tanh below 0.15 is its series.  A GELU is then 16
// multiply-adds and two transcendental instructions instead of about 60
// instructions of erff, 268M of which cost more than a quarter of the layer that
// they follow (16x2048 rows 4096x4096).  fp32 takes erfc, which keeps its digits where
// 1 + erf cancels (a tenth of GELU(-5) was off, below -5.5 all of it): 4096x32 rows
// 32x32 16.5 us, 14.8 by 1 + erf.
__device__ __forceinline__ float exp_fast(float x) { return __builtin_amdgcn_exp2f(x * 1.44269504f); }

// e^x within 2 ulp for results that are normal numbers: the rounding of x log2 e
// put back, e^x = 2^h (1 + l ln 2).
__device__ __forceinline__ float exp_near(float x)
{
    const float c = fmaxf(x, -200.0f), l = fmaf(c, 1.92596299e-8f, fmaf(c, 1.44269502f, -(c * 1.44269502f)));
    const float e = __builtin_amdgcn_exp2f(x * 1.44269502f);
    return fmaf(e, l * 0.69314718f, e);
}

// Q(|z|) and e^(-z^2/2).
__device__ __forceinline__ float normal_tail(float z, float *e)
{
    *e = __builtin_amdgcn_exp2f(z * z * -0.72134752f);
    const float t = __builtin_amdgcn_rcpf(fmaf(fabsf(z), 0.256326199f, 1.0f));
    float p = fmaf(t, -0.157882705f, 0.528239012f);
    p = fmaf(t, p, -0.305762857f);
    p = fmaf(t, p, 0.39424786f);
    p = fmaf(t, p, 0.1218144f);
    p = fmaf(t, p, 0.215542689f);
    p = fmaf(t, p, 0.203801587f);
    return 0.5f * p * t * *e;
}

// (-inf has the value 0 of GELU's and SiLU's limits; NaN passes)
template <bool FAST>
__device__ __forceinline__ float act_value(int act, float z)
{
    switch (act) {
    case ACT_RELU: return z < 0.0f ? 0.0f : z;  // NaN passes
    case ACT_TANH: {
        if constexpr (!FAST) return tanhf(z);
        const float s = z * z, t = exp_fast(-2.0f * fabsf(z)), r = (1.0f - t) * __builtin_amdgcn_rcpf(1.0f + t);
        const float near = z * fmaf(s, fmaf(s, fmaf(s, -17.0f / 315.0f, 2.0f / 15.0f), -1.0f / 3.0f), 1.0f);
        return s < 0.0225f ? near : copysignf(r, z);
    }
    case ACT_GELU: {
        if constexpr (!FAST) return 0.5f * fmaxf(z, -126.0f) * erfcf(z * -0.70710678f);
        float e;
        const float q = normal_tail(z, &e);  // NaN where z is
        return fmaf(-fminf(fabsf(z), 30.0f), q, fmaxf(z, 0.0f));
    }
    case ACT_SILU:
        if constexpr (!FAST) return fmaxf(z, -126.0f) / (1.0f + expf(-z));
        return fmaxf(z, -126.0f) * __builtin_amdgcn_rcpf(1.0f + exp_fast(-z));
    default: return z;
    }
}

template <bool FAST>
__device__ __forceinline__ float act_slope(int act, float z)
{
    const float zc = fminf(fmaxf(z, -126.0f), 126.0f);  // infinities have slope 0 or 1
    switch (act) {
    case ACT_RELU: return z > 0.0f ? 1.0f : z == z ? 0.0f : z;
    case ACT_TANH: {  // 4 t / (1 + t)^2, t = e^(-2 |z|): no cancellation
        const float t = FAST ? exp_fast(-2.0f * fabsf(z)) : exp_near(-2.0f * fabsf(z)), r = __builtin_amdgcn_rcpf(1.0f + t);
        const float far = 4.0f * t * r * r;
        if constexpr (FAST) return far;
        // near 0 the roundings of t and 1 + t are most of it (rms 6.7e-8 below 1, so 2.3e-8):
        // there 1 - z^2 p(z^2), fitted within 1.2e-9
        const float s = z * z;
        float p = fmaf(s, -0.00235370733f, 0.0134551786f);
        p = fmaf(s, p, -0.0409715064f);
        p = fmaf(s, p, 0.095073618f);
        p = fmaf(s, p, -0.196208805f);
        p = fmaf(s, p, 0.377689391f);
        p = fmaf(s, p, -0.666660488f);
        p = fmaf(s, p, 0.999999881f);
        return s < 0.81f ? fmaf(-s, p, 1.0f) : far;
    }
    case ACT_GELU: {
        if constexpr (FAST) {
            float e;
            const float q = normal_tail(z, &e);
            return fmaf(zc * 0.39894228f, e, z < 0.0f ? q : 1.0f - q);
        }
        return 0.5f * erfcf(z * -0.70710678f) + zc * 0.39894228f * expf(-0.5f * z * z);
    }
    case ACT_SILU: {
        const float s = FAST ? __builtin_amdgcn_rcpf(1.0f + exp_fast(-z)) : 1.0f / (1.0f + expf(-z));
        return s * (1.0f + zc * (1.0f - s));
    }
    default: return 1.0f;
    }
}

// N neighbours at a time: one branch for all of them.
template <bool FAST, int N>
__device__ __forceinline__ void act_values(int act, float *v)
{
#define EVOX_ACT_ALL(A)                                             \
    case A:                                                         \
        _Pragma("unroll") for (int e = 0; e < N; ++e) v[e] = act_value<FAST>(A, v[e]); \
        break;
    switch (act) {
        EVOX_ACT_ALL(ACT_RELU)
        EVOX_ACT_ALL(ACT_TANH)
        EVOX_ACT_ALL(ACT_GELU)
        EVOX_ACT_ALL(ACT_SILU)
    default: break;
    }
#undef EVOX_ACT_ALL
}
template <bool FAST, int N>
__device__ __forceinline__ void act_slopes(int act, float *z)
{
#define EVOX_ACT_ALL(A)                                             \
    case A:                                                         \
        _Pragma("unroll") for (int e = 0; e < N; ++e) z[e] = act_slope<FAST>(A, z[e]); \
        break;
    switch (act) {
        EVOX_ACT_ALL(ACT_NONE)
        EVOX_ACT_ALL(ACT_RELU)
        EVOX_ACT_ALL(ACT_TANH)
        EVOX_ACT_ALL(ACT_GELU)
        EVOX_ACT_ALL(ACT_SILU)
    }
#undef EVOX_ACT_ALL
}

}  // namespace evox
