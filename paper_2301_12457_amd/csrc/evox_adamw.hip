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

constexpr int kBatch = 2, kPasses = 8;  // groups per lane whose loads are in flight together, and per tile
constexpr int kTensors = 36;            // per launch: the arguments hold 4 KB
constexpr uint32_t kPlaces = 32;        // counters of the blocks that have read the clock, 128 bytes apart
constexpr int kBlocks = 2048;           // eight per CU, which go on from tile to tile
template <int BITS>
inline constexpr int kWidth = BITS == 8 ? 8 : 4;  // elements per lane

// A group is L lanes' elements of a row.
struct Groups {
    int shift;        // L = 2^shift
    int64_t per_row, groups;
};
Groups groups_of(int32_t bits, int64_t rows, int64_t n)
{
    const int E = bits == 8 ? kWidth<8> : kWidth<32>, most = bits == 8 ? 5 : 6;
    Groups g;
    g.shift = 0;
    while (g.shift < most && ((int64_t)E << g.shift) < n) ++g.shift;
    g.per_row = (n + ((int64_t)E << g.shift) - 1) / ((int64_t)E << g.shift);
    g.groups = rows * g.per_row;
    return g;
}
uint32_t tiles_of(const Groups &g) { return (uint32_t)((g.groups + (kPasses * 256 >> g.shift) - 1) / (kPasses * 256 >> g.shift)); }

// A tensor in the kernel's arguments: the caller's, its groups, and a division by the
// groups of a row (n / d = (t + (n - t) / 2) / 2^(s - 1) with t the upper half of n mul,
// Granlund and Montgomery, 1994).
struct Item {
    void *p;
    const void *g;
    void *m, *v;
    float *m_scale, *v_scale, *master;
    int64_t n, ldp, ldg, lds;
    uint32_t groups, per_row, mul;
    uint16_t shift, lanes;
};
struct Step {
    Item t[kTensors];
    uint32_t start[kTensors + 1];  // first tile of each
    int32_t count, last;
    float beta1, beta2, one_minus1, one_minus2, eps;
    float lr, decay, log1, log2;   // the betas' logarithms
    const float *lr_dev;
    int64_t *clock;                // steps done, and blocks of this one that have read it
};
static_assert(sizeof(Step) <= 4096, "kernel arguments");

Item item_of(const AdamTensor &t, const Groups &g)
{
    Item x{};
    x.p = t.p;
    x.g = t.g;
    x.m = t.m;
    x.v = t.v;
    x.m_scale = t.m_scale;
    x.v_scale = t.v_scale;
    x.master = t.master;
    x.n = t.n;
    x.ldp = t.ldp;
    x.ldg = t.ldg;
    x.lds = t.lds;
    x.groups = (uint32_t)g.groups;
    x.per_row = (uint32_t)g.per_row;
    x.lanes = (uint16_t)g.shift;
    int s = 0;
    while (((uint64_t)1 << s) < x.per_row) ++s;
    x.shift = (uint16_t)(s ? s - 1 : 0);
    x.mul = (uint32_t)((((((uint64_t)1 << s) - x.per_row) << 32) / x.per_row) + 1);
    return x;
}

template <typename T, int E>
struct Packed {
    typedef T reg __attribute__((ext_vector_type(E)));
    typedef T mem __attribute__((ext_vector_type(E), aligned(sizeof(T))));
};
// A lane's E elements of a row: loaded from the row's last E where they pass its end (no
// branch, so that all loads of a batch are on their way together), and then moved to their
// places with 0 behind them.  TINY: rows of fewer than E, element by element.
template <bool TINY, int E, typename T>
__device__ __forceinline__ typename Packed<T, E>::reg get(const T *row, int64_t col, int64_t n)
{
    if constexpr (!TINY) return *reinterpret_cast<const typename Packed<T, E>::mem *>(row + min(col, n - E));
    typename Packed<T, E>::reg v;
#pragma unroll
    for (int e = 0; e < E; ++e) v[e] = e < n ? row[e] : (T)0;
    return v;
}
template <int E, typename T>
__device__ __forceinline__ void settle_row(typename Packed<T, E>::reg &v, int64_t col, int64_t n)
{
    const int past = (int)min(col + E - n, (int64_t)E);
    if (past <= 0) return;
#pragma unroll
    for (int b = 1; b < E; b *= 2)
        if (past & b)
#pragma unroll
            for (int j = 0; j + b < E; ++j) v[j] = v[j + b];
#pragma unroll
    for (int j = 0; j < E; ++j)
        if (j >= E - past) v[j] = (T)0;
}
template <int E, typename T>
__device__ __forceinline__ void put(T *p, int n, typename Packed<T, E>::reg v)
{
    if (n >= E) *reinterpret_cast<typename Packed<T, E>::mem *>(p) = v;
    else
#pragma unroll
        for (int e = 0; e < E; ++e)
            if (e < n) p[e] = v[e];
}

typedef Packed<uint8_t, 8>::reg Bytes8;
__device__ __forceinline__ void from8(Bytes8 bytes, float scale, float *v)
{
    const uint2 b = __builtin_bit_cast(uint2, bytes);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int w = (int)(i ? b.y : b.x);
        const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8(w, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(w, true);
        v[4 * i] = lo[0] * scale;
        v[4 * i + 1] = lo[1] * scale;
        v[4 * i + 2] = hi[0] * scale;
        v[4 * i + 3] = hi[1] * scale;
    }
}
// The group's scale, and its numbers by it.  What is below 2^-100 counts as 0;
// an infinity or NaN makes the scale NaN, and with it all that the group stands for (its
// numbers are then 0).
__device__ __forceinline__ float scale8(const float *v, int L, float *ratio)
{
    float most = 0.0f;  // NaN if one is
#pragma unroll
    for (int e = 0; e < 8; ++e) most = __builtin_elementwise_maximum(most, fabsf(v[e]));
    // (as integers: NaN is above all)
    const float m = __uint_as_float(lanes_max(__float_as_uint(most) & 0x7fffffffu, L));
    const bool finite = m < INFINITY;
    *ratio = !finite ? -1.0f : m > 0x1p-100f ? 448.0f / m : 0.0f;
    return finite ? m * (1.0f / 448.0f) : __builtin_nanf("");
}
template <bool ROOT>
__device__ __forceinline__ Bytes8 to8(const float *v, float ratio)
{
    float q[8], least = 1.0f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        q[e] = v[e] * ratio;
        if (ROOT) least = fminf(least, q[e]);
    }
    if (ROOT && least < 0x1p-9f)
#pragma unroll
        for (int e = 0; e < 8; ++e) q[e] = v[e] > 0.0f ? fmaxf(q[e], 0x1p-9f) : q[e];
    uint32_t b[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int w = __builtin_amdgcn_cvt_pk_fp8_f32(q[4 * i], q[4 * i + 1], 0, false);
        b[i] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(q[4 * i + 2], q[4 * i + 3], w, true);
        if (ratio < 0.0f) b[i] = 0;
    }
    return __builtin_bit_cast(Bytes8, make_uint2(b[0], b[1]));
}

template <typename T, int BITS, bool MASTER>
__global__ __launch_bounds__(256) void k_adamw(const Step a)
{
    constexpr int E = kWidth<BITS>;
    typedef typename std::conditional<MASTER, float, T>::type P;
    typedef typename std::conditional<BITS == 8, uint8_t, float>::type S;
    // the step's number; 1 - b^t = -expm1(t log b) (fp32: within 3 roundings of it)
    const int64_t t = max(__hip_atomic_load(a.clock, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) + 1, (int64_t)1);
    asm volatile("" ::"v"((uint32_t)t));  // (here it is in a register: the load is done)
    const float lr = a.lr_dev ? *a.lr_dev : a.lr;
    const float rate = lr / -expm1f((float)t * a.log1), root = 1.0f / sqrtf(-expm1f((float)t * a.log2)), shrink = lr * a.decay;
    // every thread has t behind the barrier, and the block counts itself: in one of 32 places,
    // whose last block counts the place (one place for 1554 blocks: 44 us of 97)
    __syncthreads();
    if (a.last && threadIdx.x == 0) {
        const uint32_t place = blockIdx.x % kPlaces, mates = (gridDim.x - place + kPlaces - 1) / kPlaces;
        uint32_t *of = (uint32_t *)(a.clock + 16 * (1 + place)), *all = (uint32_t *)(a.clock + 1);
        const auto count = [](uint32_t *c) { return __hip_atomic_fetch_add(c, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); };
        if (count(of) == mates - 1) {
            *of = 0;
            if (count(all) == min(gridDim.x, kPlaces) - 1) {
                *all = 0;
                a.clock[0] = t;
            }
        }
    }

    for (uint32_t tile = blockIdx.x; tile < a.start[a.count]; tile += gridDim.x) {
        int lo = 0, hi = a.count;
        while (hi - lo > 1) {
            const int mid = (lo + hi) / 2;
            if (a.start[mid] <= tile) lo = mid;
            else hi = mid;
        }
        const Item &x = a.t[lo];
        const int shift = x.lanes, lane = threadIdx.x & ((1 << shift) - 1);
        const uint32_t first = (tile - a.start[lo]) * (kPasses * 256 >> shift) + (threadIdx.x >> shift);
        const auto batch = [&](auto tiny, int u0) {
            constexpr bool TINY = decltype(tiny)::value;
            typename Packed<P, E>::reg pv[kBatch];
            typename Packed<T, E>::reg gv[kBatch];
            typename Packed<S, E>::reg mv[kBatch], vv[kBatch];
            float ms[kBatch], vs[kBatch];
            int64_t op[kBatch], os[kBatch], col[kBatch];  // the rows' places in p, and in the states
            int n[kBatch];
            uint32_t group[kBatch];
            bool inside = true;
#pragma unroll
            for (int u = 0; u < kBatch; ++u) {
                group[u] = first + (u0 + u) * (256 >> shift);
                const uint32_t gr = min(group[u], x.groups - 1);
                uint32_t r = 0;
                if (x.per_row == 1) r = gr;
                else if (x.per_row != x.groups) {
                    const uint32_t q = __umulhi(gr, x.mul);
                    r = (q + ((gr - q) >> 1)) >> x.shift;
                }
                int64_t og = 0;
                op[u] = os[u] = 0;
                if (x.per_row != x.groups) {
                    op[u] = r * x.ldp;
                    og = r * x.ldg;
                    os[u] = r * x.lds;
                }
                col[u] = ((int64_t)(gr - r * x.per_row) << shift | lane) * E;
                n[u] = group[u] < x.groups ? (int)min(max(x.n - col[u], (int64_t)0), (int64_t)E) : 0;
                inside &= n[u] >= E;
                gv[u] = get<TINY, E>((const T *)x.g + og, col[u], x.n);
                pv[u] = get<TINY, E>(MASTER ? (const P *)x.master + os[u] : (const P *)x.p + op[u], col[u], x.n);
                mv[u] = get<TINY, E>((const S *)x.m + os[u], col[u], x.n);
                vv[u] = get<TINY, E>((const S *)x.v + os[u], col[u], x.n);
                if constexpr (BITS == 8) {
                    ms[u] = x.m_scale[gr];
                    vs[u] = x.v_scale[gr];
                }
            }
            inside = __all(inside);
            if (!TINY && !inside)
#pragma unroll
                for (int u = 0; u < kBatch; ++u) {
                    settle_row<E, T>(gv[u], col[u], x.n);
                    settle_row<E, P>(pv[u], col[u], x.n);
                    settle_row<E, S>(mv[u], col[u], x.n);
                    settle_row<E, S>(vv[u], col[u], x.n);
                }
#pragma unroll
            for (int u = 0; u < kBatch; ++u) {
                float m[E], v[E], r[E];
                if constexpr (BITS == 8) {
                    from8(mv[u], ms[u], m);
                    from8(vv[u], vs[u], v);
#pragma unroll
                    for (int e = 0; e < E; ++e) v[e] *= v[e];
                } else {
#pragma unroll
                    for (int e = 0; e < E; ++e) {
                        m[e] = mv[u][e];
                        v[e] = vv[u][e];
                    }
                }
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    const float g = (float)gv[u][e], p = (float)pv[u][e];
                    m[e] = fmaf(m[e], a.beta1, g * a.one_minus1);
                    v[e] = fmaf(v[e], a.beta2, (g * g) * a.one_minus2);
                    r[e] = __builtin_amdgcn_sqrtf(v[e]);
                    pv[u][e] = (P)fmaf(m[e] * __builtin_amdgcn_rcpf(fmaf(r[e], root, a.eps)), -rate, fmaf(p, -shrink, p));
                }
                if constexpr (BITS == 8) {
                    float mr, vr;
                    const float new_m = scale8(m, 1 << shift, &mr), new_v = scale8(r, 1 << shift, &vr);
                    mv[u] = to8<false>(m, mr);
                    vv[u] = to8<true>(r, vr);
                    if (group[u] < x.groups && lane == 0) {
                        x.m_scale[group[u]] = new_m;
                        x.v_scale[group[u]] = new_v;
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < E; ++e) {
                        mv[u][e] = m[e];
                        vv[u][e] = v[e];
                    }
                }
                const int64_t at = os[u] + col[u];
                const int left = inside ? E : n[u];
                put<E>((S *)x.m + at, left, mv[u]);
                put<E>((S *)x.v + at, left, vv[u]);
                if constexpr (MASTER) {
                    put<E>(x.master + at, left, pv[u]);
                    typename Packed<T, E>::reg low;
#pragma unroll
                    for (int e = 0; e < E; ++e) low[e] = (T)pv[u][e];
                    put<E>((T *)x.p + op[u] + col[u], left, low);
                } else put<E>((T *)x.p + op[u] + col[u], left, pv[u]);
            }
        };
        for (int u0 = 0; u0 < kPasses; u0 += kBatch) {
            if (((tile - a.start[lo]) * kPasses + u0) * (256 >> shift) >= x.groups) break;
            if (x.n >= E) batch(std::false_type{}, u0);
            else batch(std::true_type{}, u0);
        }
    }
}

}  // namespace

int64_t adam_groups(int32_t bits, int64_t rows, int64_t n) { return groups_of(bits, rows, n).groups; }

hipError_t launch_adamw(const AdamCall &c, const AdamTensor *t, int64_t count, hipStream_t s)
{
    Step a{};
    a.lr = (float)c.lr;
    a.decay = (float)c.decay;
    a.log1 = (float)log(c.beta1);  // (of 0: -inf, and 1 - b^t = 1)
    a.log2 = (float)log(c.beta2);
    a.beta1 = (float)c.beta1;
    a.beta2 = (float)c.beta2;
    a.one_minus1 = (float)(1.0 - c.beta1);
    a.one_minus2 = (float)(1.0 - c.beta2);
    a.eps = (float)c.eps;
    a.lr_dev = c.lr_dev;
    a.clock = c.clock;
    const bool master = count > 0 && t[0].master;
    int64_t i = 0;
    do {
        a.count = 0;
        uint32_t tiles = 0;
        // as many tensors as the arguments hold (those without elements are left out)
        for (; i < count && a.count < kTensors; ++i) {
            if (t[i].rows == 0 || t[i].n == 0) continue;
            const Groups g = groups_of(c.bits, t[i].rows, t[i].n);
            const uint32_t n = tiles_of(g);
            if (n > UINT32_MAX / 2 - tiles) break;
            a.start[a.count] = tiles;
            a.t[a.count++] = item_of(t[i], g);
            tiles += n;
        }
        a.start[a.count] = tiles;
        a.last = i == count;
        if (tiles == 0 && !a.last) continue;  // (in the last launch the count moves on all the same)
        const hipError_t e = net_dispatch(c.dtype, [&](auto type) {
            typedef typename NetElement<decltype(type)::value>::type T;
            const dim3 grid(tiles == 0 ? 1 : tiles < kBlocks ? tiles : kBlocks), block(256);
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
