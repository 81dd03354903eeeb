// One AdamW step over a list of tensors:
//     m = b1 m + (1 - b1) g,   v = b2 v + (1 - b2) g^2,
//     p = p - lr wd p - (lr / (1 - b1^t)) m / (sqrt(v) / sqrt(1 - b2^t) + eps)
// with p in its own type or, with a master, in fp32 beside it.
//
// Bound by memory: every number is read once and written once.  The tensors travel in the
// kernel's arguments, so that nothing is copied to the device and a step can be captured;
// tiles are numbered through all of them.  The step's count is on the device: every
// block reads it, and the last one that has moves it on.
//
// 8-bit states: a group of 256 elements of a row (or a shorter row's all) is 32
// lanes' (fewer for short rows), 8 elements each; m is e4m3 numbers times the group's
// largest |m| / 448, and of v its root is held the same way: e4m3 spans 2^18 of the
// group's largest number, for v then 2^36, with 2^-4 of a root's value at most in
// rounding.  A root above 0 is never rounded to 0, where an m beside it would divide by eps
// alone.  The update itself is made from the fp32 moments, before they are rounded.
#include "evox_mix.hpp"

namespace evox {

namespace {

constexpr int kPasses = 2;  // groups per lane
template <int BITS>
inline constexpr int kWidth = BITS == 8 ? 8 : 4;  // elements per lane

struct Groups {
    int L, per_row;  // lanes per group, groups per row
    int64_t groups, tiles;
};
template <int BITS>
__host__ __device__ __forceinline__ Groups groups_of(int64_t rows, int64_t n)
{
    constexpr int E = kWidth<BITS>, most = BITS == 8 ? kAdamBlock / E : 64;
    Groups g;
    g.L = 1;
    while (g.L < most && g.L * E < n) g.L *= 2;
    g.per_row = (int)((n + g.L * E - 1) / (g.L * E));
    g.groups = rows * g.per_row;
    const int per_tile = kPasses * 256 / g.L;
    g.tiles = (g.groups + per_tile - 1) / per_tile;
    return g;
}

template <typename T, int E>
struct Packed {
    typedef T reg __attribute__((ext_vector_type(E)));
    typedef T mem __attribute__((ext_vector_type(E), aligned(sizeof(T))));
};
template <typename T, int E>
__device__ __forceinline__ void read(const T *p, int n, float *v)
{
    if (n >= E) {
        const typename Packed<T, E>::reg r = *reinterpret_cast<const typename Packed<T, E>::mem *>(p);
#pragma unroll
        for (int e = 0; e < E; ++e) v[e] = (float)r[e];
        return;
    }
#pragma unroll
    for (int e = 0; e < E; ++e) v[e] = e < n ? (float)p[e] : 0.0f;
}
template <typename T, int E>
__device__ __forceinline__ void write(T *p, int n, const float *v)
{
    if (n >= E) {
        typename Packed<T, E>::reg r;
#pragma unroll
        for (int e = 0; e < E; ++e) r[e] = (T)v[e];
        *reinterpret_cast<typename Packed<T, E>::mem *>(p) = r;
        return;
    }
#pragma unroll
    for (int e = 0; e < E; ++e)
        if (e < n) p[e] = (T)v[e];
}

struct Bytes8 {
    uint32_t w[2];
};
__device__ __forceinline__ Bytes8 read8(const uint8_t *p, int n)
{
    Bytes8 b{{0, 0}};
    if (n >= 8) __builtin_memcpy(&b, p, 8);
    else
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (e < n) b.w[e / 4] |= (uint32_t)p[e] << e % 4 * 8;
    return b;
}
__device__ __forceinline__ void write8(uint8_t *p, int n, Bytes8 b)
{
    if (n >= 8) __builtin_memcpy(p, &b, 8);
    else
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (e < n) p[e] = (uint8_t)(b.w[e / 4] >> e % 4 * 8);
}
__device__ __forceinline__ void from8(Bytes8 b, float scale, float *v)
{
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)b.w[i], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)b.w[i], true);
        v[4 * i] = lo[0] * scale;
        v[4 * i + 1] = lo[1] * scale;
        v[4 * i + 2] = hi[0] * scale;
        v[4 * i + 3] = hi[1] * scale;
    }
}
// The group's scale, and its numbers by it.  What is below 2^-100 counts as 0;
// an infinity or NaN makes the scale NaN, and with it all that the group stands for.
__device__ __forceinline__ float scale8(const float *v, int L, float *ratio)
{
    uint32_t most = 0;  // as integers: NaN is above all
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const uint32_t u = __float_as_uint(v[e]) & 0x7fffffffu;
        most = u > most ? u : most;
    }
    const float m = __uint_as_float(lanes_max(most, L));
    const bool finite = m < INFINITY;
    *ratio = finite && m > 0x1p-100f ? 448.0f / m : 0.0f;
    return finite ? m * (1.0f / 448.0f) : __builtin_nanf("");
}
template <bool ROOT>
__device__ __forceinline__ Bytes8 to8(const float *v, float ratio)
{
    Bytes8 b;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        float q[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            q[e] = ratio > 0.0f ? v[4 * i + e] * ratio : 0.0f;
            if (ROOT && v[4 * i + e] > 0.0f) q[e] = fmaxf(q[e], 0x1p-9f);
        }
        int w = __builtin_amdgcn_cvt_pk_fp8_f32(q[0], q[1], 0, false);
        b.w[i] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(q[2], q[3], w, true);
    }
    return b;
}

// b^t
__device__ __forceinline__ double power(double b, int64_t t)
{
    double r = 1.0;
    for (; t > 0; t >>= 1, b *= b)
        if (t & 1) r *= b;
    return r;
}

template <typename T, int BITS, bool MASTER>
__global__ __launch_bounds__(256) void k_adamw(AdamArgs a)
{
    constexpr int E = kWidth<BITS>;
    int lo = 0, hi = a.count;
    while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if (a.start[mid] <= blockIdx.x) lo = mid;
        else hi = mid;
    }
    const AdamTensor &x = a.t[lo];
    const Groups gr = groups_of<BITS>(x.rows, x.n);
    const int L = gr.L, lane = threadIdx.x & (L - 1);
    const int64_t tile = blockIdx.x - a.start[lo];

    const int64_t t = max(a.clock[0] + 1, (int64_t)1);
    const double lr = a.lr_dev ? (double)*a.lr_dev : a.lr;
    const float rate = (float)(lr / (1.0 - power(a.b1, t))), root = (float)(1.0 / sqrt(1.0 - power(a.b2, t))),
                shrink = (float)(lr * a.decay);

    for (int u = 0; u < kPasses; ++u) {
        const int64_t group = (tile * kPasses + u) * (256 / L) + threadIdx.x / L;
        const bool live = group < gr.groups;
        const int64_t row = live ? group / gr.per_row : 0, b = live ? group - row * gr.per_row : 0;
        const int64_t col = (b * L + lane) * E;
        const int n = live ? (int)min(max(x.n - col, (int64_t)0), (int64_t)E) : 0;
        float p[E], g[E], m[E], v[E], r[E];
        read<T, E>((const T *)x.g + row * x.ldg + col, n, g);
        if constexpr (MASTER) read<float, E>(x.master + row * x.lds + col, n, p);
        else read<T, E>((const T *)x.p + row * x.ldp + col, n, p);
        if constexpr (BITS == 8) {
            const Bytes8 mb = read8((const uint8_t *)x.m + row * x.lds + col, n), vb = read8((const uint8_t *)x.v + row * x.lds + col, n);
            const int64_t s = row * gr.per_row + b;
            from8(mb, live ? x.m_scale[s] : 0.0f, m);
            from8(vb, live ? x.v_scale[s] : 0.0f, v);
#pragma unroll
            for (int e = 0; e < E; ++e) v[e] *= v[e];
        } else {
            read<float, E>((const float *)x.m + row * x.lds + col, n, m);
            read<float, E>((const float *)x.v + row * x.lds + col, n, v);
        }
#pragma unroll
        for (int e = 0; e < E; ++e) {
            m[e] = m[e] * a.beta1 + g[e] * a.one_minus1;
            v[e] = v[e] * a.beta2 + (g[e] * g[e]) * a.one_minus2;
            r[e] = sqrtf(v[e]);
            p[e] = (p[e] - p[e] * shrink) - rate * (m[e] / (r[e] * root + a.eps));
        }
        if constexpr (MASTER) write<float, E>(x.master + row * x.lds + col, n, p);
        write<T, E>((T *)x.p + row * x.ldp + col, n, p);
        if constexpr (BITS == 8) {
            float mr, vr;
            const float ms = scale8(m, L, &mr), vs = scale8(r, L, &vr);
            write8((uint8_t *)x.m + row * x.lds + col, n, to8<false>(m, mr));
            write8((uint8_t *)x.v + row * x.lds + col, n, to8<true>(r, vr));
            if (live && lane == 0) {
                x.m_scale[row * gr.per_row + b] = ms;
                x.v_scale[row * gr.per_row + b] = vs;
            }
        } else {
            write<float, E>((float *)x.m + row * x.lds + col, n, m);
            write<float, E>((float *)x.v + row * x.lds + col, n, v);
        }
    }
    // this block has its count (in every thread's registers behind the barrier)
    if (!a.last) return;
    __syncthreads();
    if (threadIdx.x == 0) {
        __threadfence();
        uint32_t *ticket = (uint32_t *)(a.clock + 1);
        if (atomicAdd(ticket, 1u) == gridDim.x - 1) {
            *ticket = 0;
            a.clock[0] = t;
        }
    }
}

}  // namespace

int64_t adam_tiles(int32_t bits, int64_t rows, int64_t n)
{
    return bits == 8 ? groups_of<8>(rows, n).tiles : groups_of<32>(rows, n).tiles;
}

hipError_t launch_adamw(const AdamCall &c, const AdamTensor *t, int64_t count, hipStream_t s)
{
    AdamArgs a{};
    a.lr = c.lr;
    a.decay = c.decay;
    a.b1 = c.beta1;
    a.b2 = c.beta2;
    a.beta1 = (float)c.beta1;
    a.beta2 = (float)c.beta2;
    a.one_minus1 = (float)(1.0 - c.beta1);
    a.one_minus2 = (float)(1.0 - c.beta2);
    a.eps = (float)c.eps;
    a.lr_dev = c.lr_dev;
    a.clock = c.clock;
    int64_t i = 0;
    do {
        a.count = 0;
        uint32_t tiles = 0;
        // as many tensors as the arguments hold (tensors without elements are left out;
        // all with a master or none)
        for (; i < count && a.count < kAdamTensors; ++i) {
            const int64_t n = t[i].rows && t[i].n ? adam_tiles(c.bits, t[i].rows, t[i].n) : 0;
            if (n == 0) continue;
            if (tiles + n > INT32_MAX) break;
            a.start[a.count] = tiles;
            a.t[a.count++] = t[i];
            tiles += (uint32_t)n;
        }
        a.start[a.count] = tiles;
        a.last = i == count;
        if (tiles == 0) {
            if (!a.last) continue;
            // nothing to update in the last launch: the count moves on all the same
            tiles = 1;
            a.count = 1;
            a.t[0] = AdamTensor{};
            a.start[0] = 0;
        }
        const bool master = a.t[0].master != nullptr;
        const hipError_t e = net_dispatch(c.dtype, [&](auto type) {
            typedef typename NetElement<decltype(type)::value>::type T;
            const dim3 grid(tiles), block(256);
            if (c.bits == 8) {
                if (master) hipLaunchKernelGGL((k_adamw<T, 8, true>), grid, block, 0, s, a);
                else hipLaunchKernelGGL((k_adamw<T, 8, false>), grid, block, 0, s, a);
            } else if (master) hipLaunchKernelGGL((k_adamw<T, 32, true>), grid, block, 0, s, a);
            else hipLaunchKernelGGL((k_adamw<T, 32, false>), grid, block, 0, s, a);
            return hipGetLastError();
        });
        if (e != hipSuccess) return e;
    } while (i < count);
    return hipSuccess;
}

}  // namespace evox
