// Layer norm and cross-entropy over the rows of a population of networks.
//
// All four kernels are bound by memory: they read every row once, keep it in
// registers (but the norm's gradient of the longest rows, which reads them twice), and
// write their results once.  A row lies over L lanes (a power
// of two, 1 .. 64, or a block of 256 .. 1024 threads), each with NIT chunks of
// 16 bytes; row sums are butterflies over the L lanes (and LDS across waves)
// in fp32.
#include "evox_net.hpp"

namespace evox {

namespace {

// Lanes per row and chunks per lane for n elements in chunks of N: up to 16 lanes
// two chunks per lane (so that a wave's load covers whole lines of a row), then
// `per` up to a wave per row of at most PER, then a block per row: PER per lane of
// 128 .. 1024 threads, then as many as it takes.
struct RowShape {
    int L, nit, threads;
    bool wide;
};
template <int PER>
RowShape row_shape(int64_t n, int N)
{
    const int64_t chunks = (n + N - 1) / N;
    RowShape s{1, 1, 256, chunks > 64 * PER};
    if (s.wide) {
        s.L = 256;
        while (s.L < 1024 && chunks > PER * s.L) s.L += 64;
        while (chunks > (int64_t)s.nit * s.L) s.nit *= 2;
        s.L = s.threads = (int)((chunks + s.nit * 64 - 1) / (s.nit * 64)) * 64;
        return s;
    }
    while (s.L < 64 && chunks > (s.L < 16 ? 2 : PER) * s.L) s.L *= 2;
    while (chunks > (int64_t)s.nit * s.L) s.nit *= 2;
    return s;
}

// f(integral NIT, bool WIDE): the instantiation of a shape.
template <int V>
struct Int {
    static constexpr int v = V;
};
template <typename T, int PER, typename F>
hipError_t with_shape(const RowShape &s, F &&f)
{
    if (!s.wide) {
        if (s.nit == 1) f(Int<1>{}, Int<0>{});
        else if (PER == 2 || s.nit == 2) f(Int<2>{}, Int<0>{});
        else f(Int<PER>{}, Int<0>{});
    } else {
        if (PER == 2 && s.nit == 1) f(Int<PER == 2 ? 1 : 2>{}, Int<1>{});  // (PER = 4: 257 chunks on 256 lanes at least)
        else if (s.nit <= 2) f(Int<2>{}, Int<1>{});
        else if (s.nit == 4) f(Int<4>{}, Int<1>{});
        else if constexpr (sizeof(T) == 4) f(Int<8>{}, Int<1>{});  // 16 bits: 4 x 1024 chunks hold EVOX_MAX_D
    }
    return hipGetLastError();
}

// Sums (maxima) over the L lanes of a row; wide rows are a whole block, whose
// waves meet in LDS.
template <bool WIDE, bool MAX>
__device__ __forceinline__ float row_all(float v, int L, float *lds)
{
    for (int o = WIDE ? 32 : L / 2; o > 0; o /= 2) {
        const float w = __shfl_xor(v, o);
        v = MAX ? fmaxf(v, w) : v + w;
    }
    if constexpr (WIDE) {
        const int wave = threadIdx.x / 64, waves = blockDim.x / 64;
        __syncthreads();
        if (threadIdx.x % 64 == 0) lds[wave] = v;
        __syncthreads();
        v = lds[0];
        for (int w = 1; w < waves; ++w) v = MAX ? fmaxf(v, lds[w]) : v + lds[w];
    }
    return v;
}
// lds: not the place of the call before (its reads need no wait then).
template <bool WIDE>
__device__ __forceinline__ void row_sum2(float &a, float &b, int L, float2 *lds)
{
    for (int o = WIDE ? 32 : L / 2; o > 0; o /= 2) {
        a += __shfl_xor(a, o);
        b += __shfl_xor(b, o);
    }
    if constexpr (WIDE) {
        const int wave = threadIdx.x / 64, waves = blockDim.x / 64;
        if (threadIdx.x % 64 == 0) lds[wave] = make_float2(a, b);
        __syncthreads();
        float2 v = lds[0];
        for (int w = 1; w < waves; ++w) {
            v.x += lds[w].x;
            v.y += lds[w].y;
        }
        a = v.x;
        b = v.y;
    }
}

// ---------------------------------------------------------------------------
// Layer norm: the mean first, then the variance of the centred row (both from
// the row in registers, so a large mean costs no digits).  Bound by memory: f16
// 65,536 rows of 1024 50 us, 5.4 TB/s of the copy's 6.45 (its floor 42).  Results
// with the streaming hint (f16 16,384 rows of 1024 17.1 us, 19.3 without; on the
// loads it does nothing).  Two to four chunks per lane (four / two: f16 65,536 rows
// of 300 22 / 28 us, of 1024 50 / 52; of 100 16 / 13, so from 16 lanes on).
// ---------------------------------------------------------------------------
template <typename T, int NIT, bool WIDE>
__global__ __launch_bounds__(WIDE ? 1024 : 256) void k_layernorm(NormArgs a, int L)
{
    constexpr int N = NetVec<T>::N;
    __shared__ float lds[16];
    const int lane = WIDE ? threadIdx.x : threadIdx.x & (L - 1), D = (int)a.D;
    const int64_t m = WIDE ? net_block() : net_block() * (256 / L) + threadIdx.x / L;
    const bool live = m < a.rows.M;
    const T *x = (const T *)a.x + m * a.ldx;
    typename NetVec<T>::reg v[NIT];
    if (live)
#pragma unroll
        for (int i = 0; i < NIT; ++i)
            if ((lane + i * L) * N < D) v[i] = load_chunk(x, lane + i * L, D, (T)0.0f);
    const int g = live ? net_of_row(a.rows, m) : -1;
    if (WIDE && g < 0) return;  // the whole block
    float s = 0.0f;
    if (live)
#pragma unroll
        for (int i = 0; i < NIT; ++i)
            if ((lane + i * L) * N < D)
#pragma unroll
                for (int j = 0; j < N; ++j) s += (float)v[i][j];
    const float inv = 1.0f / (float)D, mean = row_all<WIDE, false>(s, L, lds) * inv;
    s = 0.0f;
    if (live)
#pragma unroll
        for (int i = 0; i < NIT; ++i)
            if ((lane + i * L) * N < D)
#pragma unroll
                for (int j = 0; j < N; ++j) {
                    const float c = (lane + i * L) * N + j < D ? (float)v[i][j] - mean : 0.0f;
                    s = fmaf(c, c, s);
                }
    const float rstd = 1.0f / sqrtf(row_all<WIDE, false>(s, L, lds) * inv + a.eps);
    if (g < 0) return;
    const T *ga = (const T *)a.gamma + g * a.p_stride, *be = (const T *)a.beta + g * a.p_stride;
    T *y = (T *)a.y + m * a.ldy;
#pragma unroll
    for (int i = 0; i < NIT; ++i) {
        const int c = lane + i * L;
        if (c * N < D) {
            const auto gv = load_chunk(ga, c, D, (T)0.0f), bv = load_chunk(be, c, D, (T)0.0f);
#pragma unroll
            for (int j = 0; j < N; ++j) v[i][j] = (T)fmaf(((float)v[i][j] - mean) * rstd, (float)gv[j], (float)bv[j]);
            store_chunk<T, true>(y, c, D, v[i]);
        }
    }
    if (lane == 0) {
        if (a.mean) a.mean[m] = mean;
        if (a.rstd) a.rstd[m] = rstd;
    }
}

// ---------------------------------------------------------------------------
// Its gradient.  A block takes a tile of one network's rows: every lane keeps
// the sums of dy h and dy of its own columns over the rows it meets, the row
// slots of the block add theirs in a fixed order; k_net_sums adds a network's tiles.
// Rows whose chunks and sums do not fit the registers together (fp32, eight
// chunks per lane; 16 bits, four) are read a second time, the others' loads run a
// row ahead of the sums.  fp32 20,000 ragged rows of 1001: 62 us with its sums' 5
// (floor 37), 77 with four chunks per lane, where there is no room for the row
// ahead; f16 134,784 rows of 1000 194 us, 239 without it and with gamma loaded per
// row; 67,392 rows of 2625 285, of one chunk per lane 398.  fp32 rows of 1000 reach
// 4.5 TB/s; bound by the loads in flight and, above 16,384 columns, by the
// second reading (f16 8192 rows of 32,768 522 us; held, with spills, 710).
// ---------------------------------------------------------------------------
template <typename T, int NIT, bool WIDE>
__global__ __launch_bounds__(WIDE ? 1024 : 256) void k_layernorm_grad(NormArgs a, int L, int sh)
{
    constexpr int N = NetVec<T>::N;
    typedef typename NetVec<T>::reg reg;
    // which rows fit the registers: x and dy from one pass to the next; gamma; the row ahead
    constexpr bool kHold = NIT * (8 + 2 * N) < 96, kGamma = NIT * (12 + 2 * N) <= 72, kAhead = NIT * (20 + 2 * N) <= 72;
    extern __shared__ float sums[];  // [3 waves][2][NIT][N][L] (narrow rows)
    __shared__ float2 lds[2][16];
    const NetTile t = net_tile(a.rows, sh, net_block());
    if (t.g < 0) return;
    const int lane = WIDE ? threadIdx.x : threadIdx.x & (L - 1), slot = WIDE ? 0 : threadIdx.x / L, slots = WIDE ? 1 : 256 / L,
              D = (int)a.D;
    const T *ga = (const T *)a.gamma + t.g * a.p_stride;
    float sg[NIT][N], sb[NIT][N];
#pragma unroll
    for (int i = 0; i < NIT; ++i)
#pragma unroll
        for (int j = 0; j < N; ++j) sg[i][j] = sb[i][j] = 0.0f;
    const float inv = 1.0f / (float)D;
    struct Row {
        reg x[kHold ? NIT : 1], dy[kHold ? NIT : 1];
        float mean, rstd;
    };
    const auto load = [&](Row &r, int64_t m) {
        r.mean = r.rstd = 0.0f;
        if (m >= t.hi) return;
        if constexpr (kHold)
#pragma unroll
            for (int i = 0; i < NIT; ++i) {
                const int c = lane + i * L;
                if (c * N >= D) continue;
                r.x[i] = load_early((const T *)a.x + m * a.ldx, c, D);
                r.dy[i] = load_early((const T *)a.dy + m * a.ldy, c, D);
            }
        r.mean = a.mean_in[m];
        r.rstd = a.rstd_in[m];
    };
    reg g[kGamma ? NIT : 1];
    if constexpr (kGamma)
#pragma unroll
        for (int i = 0; i < NIT; ++i)
            if ((lane + i * L) * N < D) g[i] = load_chunk(ga, lane + i * L, D, (T)0.0f);
    Row next;
    if constexpr (kAhead) load(next, t.lo + slot);
    // every slot makes as many rounds (the row sums need all lanes)
    int turn = 0;
    for (int64_t m0 = t.lo; m0 < t.hi; m0 += slots, turn ^= 1) {
        const int64_t m = m0 + slot;
        const bool live = m < t.hi;
        const T *x = (const T *)a.x + m * a.ldx, *dy = (const T *)a.dy + m * a.ldy;
        Row r;
        if constexpr (kAhead) {
            r = next;
            load(next, m + slots);
        } else load(r, m);
        float s1 = 0.0f, s2 = 0.0f;
        if (live)
#pragma unroll
            for (int i = 0; i < NIT; ++i) {
                const int c = lane + i * L, k = kHold ? i : 0;
                if (c * N >= D) continue;
                if constexpr (kHold) {
                    settle(r.x[i], c, D, (T)0.0f);
                    settle(r.dy[i], c, D, (T)0.0f);
                } else {
                    r.x[0] = load_chunk(x, c, D, (T)0.0f);
                    r.dy[0] = load_chunk(dy, c, D, (T)0.0f);
                }
                if constexpr (!kGamma) g[0] = load_chunk(ga, c, D, (T)0.0f);
#pragma unroll
                for (int j = 0; j < N; ++j) {
                    const float p = (float)r.dy[k][j] * (float)g[kGamma ? i : 0][j];
                    s1 += p;
                    s2 = fmaf(p, ((float)r.x[k][j] - r.mean) * r.rstd, s2);
                }
            }
        row_sum2<WIDE>(s1, s2, L, lds[turn]);
        if (!live) continue;
        s1 *= inv;
        s2 *= inv;
#pragma unroll
        for (int i = 0; i < NIT; ++i) {
            const int c = lane + i * L, k = kHold ? i : 0;
            if (c * N >= D) continue;
            if constexpr (!kHold) {
                r.x[0] = load_chunk(x, c, D, (T)0.0f);
                r.dy[0] = load_chunk(dy, c, D, (T)0.0f);
            }
            if constexpr (!kGamma) g[0] = load_chunk(ga, c, D, (T)0.0f);
            reg out;
#pragma unroll
            for (int j = 0; j < N; ++j) {
                const float h = ((float)r.x[k][j] - r.mean) * r.rstd, d = (float)r.dy[k][j];
                sg[i][j] = fmaf(d, h, sg[i][j]);
                sb[i][j] += d;
                out[j] = (T)(r.rstd * (fmaf(d, (float)g[kGamma ? i : 0][j], -s1) - h * s2));
            }
            if (a.dx) store_chunk<T, true>((T *)a.dx + m * a.lddx, c, D, out);
        }
    }
    if (!a.dgamma) return;
    if constexpr (!WIDE) {
        // over the slots of a wave in registers, then the waves in order
        for (int o = L; o < 64; o *= 2)
#pragma unroll
            for (int i = 0; i < NIT; ++i)
#pragma unroll
                for (int j = 0; j < N; ++j) {
                    sg[i][j] += __shfl_xor(sg[i][j], o);
                    sb[i][j] += __shfl_xor(sb[i][j], o);
                }
        const int wave = threadIdx.x / 64, wl = threadIdx.x % 64;
        if (wave > 0 && wl < L)
#pragma unroll
            for (int i = 0; i < NIT; ++i)
#pragma unroll
                for (int j = 0; j < N; ++j) {
                    sums[((((wave - 1) * 2 + 0) * NIT + i) * N + j) * L + lane] = sg[i][j];
                    sums[((((wave - 1) * 2 + 1) * NIT + i) * N + j) * L + lane] = sb[i][j];
                }
        __syncthreads();
        if (threadIdx.x >= L) return;
#pragma unroll
        for (int r = 0; r < 3; ++r)
#pragma unroll
            for (int i = 0; i < NIT; ++i)
#pragma unroll
                for (int j = 0; j < N; ++j) {
                    sg[i][j] += sums[(((r * 2 + 0) * NIT + i) * N + j) * L + lane];
                    sb[i][j] += sums[(((r * 2 + 1) * NIT + i) * N + j) * L + lane];
                }
    }
    float *part = (float *)a.scratch + net_slot(t.lo, t.index, sh) * 2 * D;
#pragma unroll
    for (int i = 0; i < NIT; ++i) {
        const int c = lane + i * L;
        if (c * N >= D) continue;
        if (t.only) {
            typename NetVec<T>::reg g, b;
#pragma unroll
            for (int j = 0; j < N; ++j) {
                g[j] = (T)sg[i][j];
                b[j] = (T)sb[i][j];
            }
            store_chunk((T *)a.dgamma + t.g * a.dp_stride, c, D, g);
            store_chunk((T *)a.dbeta + t.g * a.dp_stride, c, D, b);
            continue;
        }
#pragma unroll
        for (int j = 0; j < N; ++j)
            if (c * N + j < D) {
                part[c * N + j] = sg[i][j];
                part[D + c * N + j] = sb[i][j];
            }
    }
}

template <typename T>
struct NormSums {
    T *dgamma, *dbeta;
    int64_t stride, D;
    __device__ void operator()(int64_t g, int64_t e, float s) const
    {
        if (e < D) dgamma[g * stride + e] = (T)s;
        else dbeta[g * stride + e - D] = (T)s;
    }
};

// Rows per tile of the gradient, as a power of two: 64 (its sums are then 4 % or
// less of the rows' traffic), 256 of a few columns, fewer where that leaves less than
// two blocks per CU (wide rows: 1.5; bf16 2000 rows of 8192 in 500 tiles 52 us, in
// 1000 76; 8192 rows of 4096 in 512 tiles 67, in 256 92).
int norm_tile_shift(const NormArgs &a)
{
    const int least = a.D > 2048 ? 0 : 3;  // rows over a block or waves: few of them fill neither registers nor chip
    int sh = a.D <= 16 ? 8 : 6;  // (a lane per row: as many rows as threads)
    while (sh > least && (a.rows.M >> sh) < (a.D > 2048 ? 400 : 512)) --sh;
    return sh;
}

// ---------------------------------------------------------------------------
// Cross-entropy.  A block takes a tile of one network's rows; a row's logits
// stay in registers from the maximum to the gradient.  The tile's loss (fp64)
// and count go to the scratch and are added per network in order.  The
// gradient needs the network's count first: where a tile is the whole network
// the block counts the labels itself, else k_xent_count has.  bf16 8192 rows of
// 32,768 in 16 ragged networks: 248 us, 4.3 TB/s (floor 166); bound by a row's loads,
// exponentials and two block-wide reductions in turn, with one other block per CU
// to fill in; 10 us are the count's and the fitness's launches.  fp32 4096x32 rows
// of 10: one launch of 6.8 us.
// ---------------------------------------------------------------------------
constexpr int kCountShift = 12;  // labels per block of k_xent_count

__device__ __forceinline__ int xent_label(const XentArgs &a, int64_t g, int64_t m)
{
    return a.labels[a.labels_shared ? m - g * a.rows.n : m];
}
__device__ __forceinline__ bool xent_counts(const XentArgs &a, int label) { return label >= 0 && label < a.C; }

// e^(v - top) for v <= top: of fp32 logits within 2 ulp, of 16-bit ones with the
// rounding of the exponent left in, far below the probability's own.  v - top
// comes first (its parts may be the type's lowest value).  Of -inf 0, of NaN NaN.
template <typename T>
__device__ __forceinline__ float exp_below(float v, float top)
{
    if constexpr (sizeof(T) == 2) return exp_fast(v - top);
    else return exp_near(v - top);
}

struct XentScratch {
    double *loss;    // [tiles]
    int32_t *count;  // [tiles] rows that count
    int32_t *labels; // [tiles of 2^kCountShift rows] the same, before the gradient
};
__host__ __device__ __forceinline__ XentScratch xent_layout(const XentArgs &a, int sh)
{
    const int64_t n = net_tiles(a.rows, sh);
    XentScratch s;
    s.loss = (double *)a.scratch;
    s.count = (int32_t *)(s.loss + n);
    s.labels = s.count + n;
    return s;
}

__global__ __launch_bounds__(256) void k_xent_count(XentArgs a, int sh)
{
    __shared__ int waves[4];
    const NetTile t = net_tile(a.rows, kCountShift, net_block());
    if (t.g < 0) return;
    int n = 0;
    for (int64_t m = t.lo + threadIdx.x; m < t.hi; m += 256) n += xent_counts(a, xent_label(a, t.g, m));
    for (int o = 32; o > 0; o /= 2) n += __shfl_xor(n, o);
    if (threadIdx.x % 64 == 0) waves[threadIdx.x / 64] = n;
    __syncthreads();
    if (threadIdx.x == 0) xent_layout(a, sh).labels[net_block()] = waves[0] + waves[1] + waves[2] + waves[3];
}

// Tiles of 2^sh rows; whole: a tile is a whole network (rows may be more).
template <typename T, int NIT, bool WIDE>
__global__ __launch_bounds__(WIDE ? 1024 : 256, WIDE && NIT <= 4 ? 8 : 1) void k_xent(XentArgs a, int L, int sh, bool whole)
{
    constexpr int N = NetVec<T>::N;
    // fp32 exponentials take their logits' registers; those of long 16-bit rows are
    // computed again, so that two blocks of 1024 threads fit a CU
    constexpr bool kAgain = sizeof(T) == 2 && NIT == 4;
    __shared__ float lds[16];
    __shared__ double wave_loss[16];
    __shared__ int wave_count[16];
    NetTile t;
    if (whole) {
        if (net_block() >= a.rows.G) return;
        t.g = (int)net_block();
        t.lo = t.g * a.rows.n;
        t.hi = t.lo + a.rows.n;
    } else {
        t = net_tile(a.rows, sh, net_block());
        if (t.g < 0) return;
    }
    const int lane = WIDE ? threadIdx.x : threadIdx.x & (L - 1), slot = WIDE ? 0 : threadIdx.x / L, slots = WIDE ? 1 : blockDim.x / L,
              C = (int)a.C;
    // narrow rows: the first one's logits are on their way while the labels are
    // counted (a wide row's registers would not last)
    typename NetVec<T>::reg first[WIDE ? 1 : NIT];
    int label = -1;
    if constexpr (!WIDE)
        if (t.lo + slot < t.hi) {
            label = xent_label(a, t.g, t.lo + slot);
#pragma unroll
            for (int i = 0; i < NIT; ++i)
                if ((lane + i * L) * N < C)
                    first[i] = load_chunk((const T *)a.logits + (t.lo + slot) * a.ldz, lane + i * L, C, (T)-INFINITY);
        }
    float scale = 0.0f;
    if (a.dz) {
        int n = 0;
        const int wl = threadIdx.x % 64;
        if (whole) {
            for (int64_t m = t.lo + wl; m < t.hi; m += 64) n += xent_counts(a, xent_label(a, t.g, m));
        } else {
            int64_t lo, hi;
            net_rows(a.rows, t.g, &lo, &hi);
            const int64_t t0 = net_first_tile(a.rows, kCountShift, t.g),
                          k = (hi - lo + ((int64_t)1 << kCountShift) - 1) >> kCountShift;
            const int32_t *labels = xent_layout(a, sh).labels;
            for (int64_t i = wl; i < k; i += 64) n += labels[t0 + i];
        }
        for (int o = 32; o > 0; o /= 2) n += __shfl_xor(n, o);
        scale = 1.0f / (float)n;  // not used where no row counts
    }
    double loss = 0.0;
    int count = 0;
    for (int64_t m0 = t.lo; m0 < t.hi; m0 += slots) {
        const int64_t m = m0 + slot;
        const bool live = m < t.hi;
        if ((WIDE || m0 > t.lo) && live) label = xent_label(a, t.g, m);
        const bool counts = live && xent_counts(a, label);
        typename NetVec<T>::reg v[NIT];
        if (counts)
#pragma unroll
            for (int i = 0; i < NIT; ++i) {
                if ((lane + i * L) * N >= C) continue;
                if constexpr (!WIDE)
                    if (m0 == t.lo) {
                        v[i] = first[i];
                        continue;
                    }
                v[i] = load_chunk((const T *)a.logits + m * a.ldz, lane + i * L, C, (T)-INFINITY);
            }
        float top = -INFINITY, sum = 0.0f;
        // the label's logit, before the gradient may take its place
        const float at = counts ? (float)((const T *)a.logits)[m * a.ldz + label] : 0.0f;
        if (counts)
#pragma unroll
            for (int i = 0; i < NIT; ++i)
                if ((lane + i * L) * N < C)
#pragma unroll
                    for (int j = 0; j < N; ++j) top = fmaxf(top, (float)v[i][j]);
        top = row_all<WIDE, true>(top, L, lds);
        // past the row's end v is -inf: nothing, but in a row of -inf alone, all NaN anyway
        float e16[kAgain || sizeof(T) == 4 ? 1 : NIT][N];
        auto e = [&](int i, int j) -> float {
            if constexpr (sizeof(T) == 4) return v[i][j];
            else if constexpr (kAgain) return exp_below<T>((float)v[i][j], top);
            else return e16[i][j];
        };
        if (counts)
#pragma unroll
            for (int i = 0; i < NIT; ++i)
                if ((lane + i * L) * N < C)
#pragma unroll
                    for (int j = 0; j < N; ++j) {
                        const float p = exp_below<T>((float)v[i][j], top);
                        if constexpr (sizeof(T) == 4) v[i][j] = p;
                        else if constexpr (!kAgain) e16[i][j] = p;
                        sum += p;
                    }
        sum = row_all<WIDE, false>(sum, L, lds);
        if (lane == 0 && counts) {
            loss += (double)(logf(sum) + (top - at));
            ++count;
        }
        if (a.dz && live) {
            T *dz = (T *)a.dz + m * a.lddz;
            if (!counts) {
#pragma unroll
                for (int i = 0; i < NIT; ++i)
                    if ((lane + i * L) * N < C) store_chunk<T, true>(dz, lane + i * L, C, (typename NetVec<T>::reg){});
                continue;
            }
            const float f = scale / sum;
#pragma unroll
            for (int i = 0; i < NIT; ++i) {
                const int c = lane + i * L;
                if (c * N >= C) continue;
                typename NetVec<T>::reg out;
#pragma unroll
                for (int j = 0; j < N; ++j) out[j] = (T)(e(i, j) * f);
                if (c == label / N)  // the label's chunk: (p - 1) scale, rounded once
#pragma unroll
                    for (int j = 0; j < N; ++j)
                        if (j == label % N) out[j] = (T)fmaf(e(i, j), f, -scale);
                store_chunk<T, true>(dz, c, C, out);
            }
        }
    }
    // the slots' losses in a fixed order: over the lanes, then the waves
    for (int o = 32; o > 0; o /= 2) {
        loss += __shfl_xor(loss, o);
        count += __shfl_xor(count, o);
    }
    const int wave = threadIdx.x / 64, waves = blockDim.x / 64;
    if (threadIdx.x % 64 == 0) {
        wave_loss[wave] = loss;
        wave_count[wave] = count;
    }
    __syncthreads();
    if (threadIdx.x > 0) return;
    for (int w = 1; w < waves; ++w) {
        loss += wave_loss[w];
        count += wave_count[w];
    }
    if (whole) {
        a.fit[t.g] = (float)(loss / (double)count);
    } else {
        const XentScratch s = xent_layout(a, sh);
        s.loss[net_block()] = loss;
        s.count[net_block()] = count;
    }
}

// fit[g] from the network's tiles, a wave per network.
__global__ __launch_bounds__(256) void k_xent_fit(XentArgs a, int sh)
{
    const int64_t g = (int64_t)blockIdx.x * 4 + threadIdx.x / 64;
    if (g >= a.rows.G) return;
    int64_t lo, hi;
    net_rows(a.rows, g, &lo, &hi);
    const int64_t t0 = net_first_tile(a.rows, sh, g), k = (hi - lo + ((int64_t)1 << sh) - 1) >> sh;
    const XentScratch s = xent_layout(a, sh);
    double loss = 0.0;
    int64_t count = 0;
    for (int64_t i = threadIdx.x % 64; i < k; i += 64) {
        loss += s.loss[t0 + i];
        count += s.count[t0 + i];
    }
    for (int o = 32; o > 0; o /= 2) {
        loss += __shfl_xor(loss, o);
        count += __shfl_xor(count, o);
    }
    if (threadIdx.x % 64 == 0) a.fit[g] = (float)(loss / (double)count);
}

// Whether every network is one block's: as many rows for each, and either
// networks enough to fill the chip or little work in each (fp32 rows of 10: 4096x32
// 9 us, in tiles with a count and a sum 22; 1024x500 18, 24; 16x1000 of 16 15, 19).
bool xent_whole(const XentArgs &a)
{
    return !a.rows.off && a.rows.n <= 4096 && (a.rows.G >= 1024 || a.rows.n * a.C <= 16384);
}
// Rows per tile, as a power of two: 256 (a lane each, of rows of a few classes),
// fewer where that leaves less than eight blocks per CU (a few classes: two; 200,000
// rows of 10 21 us, 25 so; bf16 8192 ragged rows of 32,768 249 us, with two blocks 316).
int xent_tile_shift(const XentArgs &a)
{
    int sh = 8;
    while (sh > 1 && (a.rows.M >> sh) < (a.C <= 16 ? 512 : 2048)) --sh;
    return sh;
}

}  // namespace

hipError_t launch_layernorm(const NormArgs &a, hipStream_t s)
{
    return net_dispatch(a.dtype, [&](auto t) {
        using T = typename NetElement<t.value>::type;
        const RowShape r = row_shape<4>(a.D, NetVec<T>::N);
        const int64_t per = r.wide ? 1 : 256 / r.L;
        return with_shape<T, 4>(r, [&](auto nit, auto wide) {
            hipLaunchKernelGGL((k_layernorm<T, nit.v, wide.v>), net_grid((a.rows.M + per - 1) / per),
                               dim3(r.threads), 0, s, a, r.L);
        });
    });
}

size_t layernorm_grad_scratch(const NormArgs &a)
{
    return 8 * (size_t)net_slots(a.rows.M, norm_tile_shift(a)) * (size_t)a.D;
}

hipError_t launch_layernorm_grad(const NormArgs &a, hipStream_t s)
{
    return net_dispatch(a.dtype, [&](auto t) {
        using T = typename NetElement<t.value>::type;
        const RowShape r = row_shape<2>(a.D, NetVec<T>::N);
        const int sh = norm_tile_shift(a);
        const int64_t tiles = net_tiles(a.rows, sh);
        hipError_t e = hipSuccess;
        if (a.rows.M > 0)
            e = with_shape<T, 2>(r, [&](auto nit, auto wide) {
                const size_t lds = wide.v ? 0 : sizeof(float) * 2 * nit.v * NetVec<T>::N * 3 * r.L;
                hipLaunchKernelGGL((k_layernorm_grad<T, nit.v, wide.v>), net_grid(tiles), dim3(r.threads), lds, s,
                                   a, r.L, sh);
            });
        if (e != hipSuccess || !a.dgamma || (a.rows.M > 0 && !a.rows.off && net_single(a.rows, sh))) return e;
        return launch_net_sums(a.rows, (const float *)a.scratch, 2 * a.D, sh, s,
                               NormSums<T>{(T *)a.dgamma, (T *)a.dbeta, a.dp_stride, a.D});
    });
}

size_t xent_scratch(const XentArgs &a)
{
    return 12 * (size_t)((a.rows.M >> xent_tile_shift(a)) + a.rows.G) +
           4 * (size_t)((a.rows.M >> kCountShift) + a.rows.G);
}

hipError_t launch_xent(const XentArgs &a, hipStream_t s)
{
    return net_dispatch(a.dtype, [&](auto t) {
        using T = typename NetElement<t.value>::type;
        const RowShape r = row_shape<4>(a.C, NetVec<T>::N);
        const bool whole = xent_whole(a);
        const int sh = xent_tile_shift(a);
        if (a.dz && !whole)
            hipLaunchKernelGGL(k_xent_count, net_grid(net_tiles(a.rows, kCountShift)), dim3(256), 0, s, a, sh);
        hipError_t e = hipSuccess;
        if (a.rows.M > 0 || whole)
            e = with_shape<T, 4>(r, [&](auto nit, auto wide) {
                // no more threads than a whole network's rows keep busy
                int threads = r.threads;
                while (whole && !wide.v && threads > 64 && a.rows.n * r.L <= threads / 2) threads /= 2;
                hipLaunchKernelGGL((k_xent<T, nit.v, wide.v>),
                                   net_grid(whole ? a.rows.G : net_tiles(a.rows, sh)), dim3(threads), 0, s, a,
                                   r.L, sh, whole);
            });
        if (e != hipSuccess || whole) return e;
        hipLaunchKernelGGL(k_xent_fit, dim3((unsigned)((a.rows.G + 3) / 4)), dim3(256), 0, s, a, sh);
        return hipGetLastError();
    });
}

}  // namespace evox
