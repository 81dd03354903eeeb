// Matrix products of the layers' large cases: tiles staged through LDS into the
// bf16 / f16 matrix cores.
//
// A block computes D[j][i] = sum_k P[i][k] Q[j][k] for a BJ x BI tile of a
// row-major result: i runs along the result's rows (its contiguous dimension),
// so that a lane's four results of a 16 x 16 tile are neighbours.  Either
// operand is k-contiguous (element (r, k) at r ld + k) or k-major (k ld + r),
// and is staged as rows of K: a k-major operand is transposed in registers, 8 k
// by 4 rows per thread (fp32: by 1), on its way to LDS.
//
// 16 bits: LDS rows of 64 k (128 bytes) in eight 16-byte chunks, chunk c of row
// r at c ^ f(r), f(r) = (r ^ r / 4) mod 8: the eight lanes that an LDS access
// serves at a time touch different chunks both when they read 8 consecutive rows
// (matrix operands, k-contiguous writes) and when they write every fourth row
// (k-major writes).
//
// 32 bits: an element is the exact sum of three bf16 numbers x = h + m + l (each
// the rounding of what the ones before leave), staged as three planes; of the
// nine products of pieces the six down to 2^-16 are summed, the rest are at most
// 2^-24 of the term (rms 2^-27).  Six bf16 products cost 6/16 of an fp32 one.  Below
// 2^56 no piece is infinite and no sum of up to 2^15 terms overflows (a longer one only
// where its magnitudes' sum does); a block that meets a larger
// number or an infinity computes its tile again with fp32 products
// (v_mfma_f32_32x32x2f32).  A NaN is one in its own row either way.  A number
// below 2^-100 loses its bits under 2^-126, as fp32 with flushed subnormals does.
//
// Gradients of 16 bits: d is two numbers of the type (d_split), K is run through once
// for each, the small one first; their products are added in the same registers.
//
// What it reaches: bf16 16x2048 ragged rows 4096x4096 with GELU and residual 1.15 -
// 1.25 ms, 880 - 960 TFLOP/s (a large library product 1440; the matrix cores are
// 51 % busy, LDS reads and writes take about as long as the products, and 6 % is
// the ragged tiles' padding); fp32 16x256 rows
// 2048x2048 176 - 190 us, 181 - 195 TFLOP/s (the library's fp32 product 154); fp32
// 100 networks of 100 ragged rows 1001x1000 240 - 256 us.  Not kept: 256 x 256 tiles by four waves of 128 x 128 (a third less LDS
// traffic, one wave per SIMD: 30 % slower); raised wave priority around the
// products; the LDS writes in the first quarter of a tile.
#pragma once

#include "evox_net.hpp"

namespace evox {

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2u __attribute__((ext_vector_type(2), aligned(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2u __attribute__((ext_vector_type(2), aligned(2)));
typedef uint32_t u32x4u __attribute__((ext_vector_type(4), aligned(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

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

// One 32 x 32 tile over 16 k: lane l brings k = 8 (l / 32) .. + 8 of row l % 32 of
// either operand and receives rows 8 b + 4 (l / 32) .. + 4 (b = 0 .. 3) of A
// against row l % 32 of B.
typedef float f32x16 __attribute__((ext_vector_type(16)));
__device__ __forceinline__ f32x16 mma32(NetVec<bf16_t>::reg a, NetVec<bf16_t>::reg b, f32x16 c)
{
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f32x16 mma32(NetVec<f16_t>::reg a, NetVec<f16_t>::reg b, f32x16 c)
{
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
}

constexpr float kTileBig = 0x1p56f;

// The two numbers rounded to bf16, packed; the three pieces of a pair.
__device__ __forceinline__ uint32_t net_pack_bf16(float a, float b)
{
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2){a, b}, bf16x2));
}
__device__ __forceinline__ void net_split2(float a, float b, uint32_t &h, uint32_t &m, uint32_t &l)
{
    h = net_pack_bf16(a, b);
    const float a1 = a - __uint_as_float(h << 16), b1 = b - __uint_as_float(h & 0xffff0000u);
    m = net_pack_bf16(a1, b1);
    l = net_pack_bf16(a1 - __uint_as_float(m << 16), b1 - __uint_as_float(m & 0xffff0000u));
}

// A barrier for LDS alone: __syncthreads() also waits for the global loads in
// flight, which here are the next tiles' operands.
__device__ __forceinline__ void lds_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// K per staged tile and bytes of one staged operand of R rows.
template <typename T>
constexpr int kTileK = sizeof(T) == 4 ? 32 : 64;
template <typename T, int R>
constexpr int kStageBytes = sizeof(T) == 4 ? 3 * 64 * R : 128 * R;

// LDS byte of chunk c (8 k) of row r.
__device__ __forceinline__ int chunk16(int r, int c) { return r * 128 + ((c ^ ((r ^ (r >> 2)) & 7)) << 4); }
__device__ __forceinline__ int chunk32(int r, int c)
{
    return (r >> 1) * 128 + (((r & 1) << 2 | (c ^ ((r >> 1) & 3))) << 4);
}

// One operand's next K tile in registers: TH threads, R rows of which n exist.
// k-contiguous rows past n repeat row n - 1 and k-major ones are zero (neither
// reaches a result); k past K is zero.
template <typename T, bool MAJOR, int R, int TH>
struct Stage;

template <typename T, int R, int TH>
struct Stage16c {
    static constexpr int P = R * 8 / TH, kLoads = P, kStores = P;
    u32x4 v[P];
    const T *row[P];
    __device__ __forceinline__ void init(const T *src, int64_t ld, int n)
    {
#pragma unroll
        for (int p = 0; p < P; ++p) {
            const int r = threadIdx.x / 8 + p * (TH / 8);
            row[p] = src + (int64_t)(r < n ? r : n - 1) * ld;
        }
    }
    // the first half of the rows of one operand, the second of another of as many rows
    __device__ __forceinline__ void init_pair(const T *src, const T *other, int64_t ld, int n)
    {
#pragma unroll
        for (int p = 0; p < P; ++p) {
            const int r = threadIdx.x / 8 + p * (TH / 8), h = r % (R / 2);
            row[p] = (r < R / 2 ? src : other) + (int64_t)(h < n ? h : n - 1) * ld;
        }
    }
    __device__ __forceinline__ bool whole() const { return true; }
    __device__ __forceinline__ void load_piece(int p, int64_t k0)  // k0 + 64 <= K
    {
        v[p] = *reinterpret_cast<const u32x4u *>(row[p] + k0 + 8 * (threadIdx.x % 8));
    }
    __device__ __forceinline__ void load(int64_t k0, int64_t K)
    {
        if (k0 + 64 <= K) {
#pragma unroll
            for (int p = 0; p < P; ++p) load_piece(p, k0);
            return;
        }
#pragma unroll
        for (int p = 0; p < P; ++p)
            v[p] = __builtin_bit_cast(u32x4, load_chunk(row[p] + k0, threadIdx.x % 8, (int)(K - k0), (T)0.0f));
    }
    __device__ __forceinline__ void store_piece(int p, char *lds, float &)
    {
        *reinterpret_cast<u32x4 *>(lds + chunk16(threadIdx.x / 8 + p * (TH / 8), threadIdx.x % 8)) = v[p];
    }
};

template <typename T, int R, int TH>
struct Stage16m {
    static constexpr int P = (R * 2 + TH - 1) / TH, kQuads = R / 4, kLoads = 8 * P, kStores = 4 * P;
    u32x2 v[P][8];
    const T *base[P];  // the thread's patches at k = 0
    int64_t ld;
    int n;
    // threads past the patches repeat the first ones' work
    static __device__ __forceinline__ int thread() { return R * 2 < TH ? threadIdx.x % (R * 2) : threadIdx.x; }
    __device__ __forceinline__ void init(const T *s, int64_t l, int rows)
    {
        ld = l;
        n = rows;
#pragma unroll
        for (int p = 0; p < P; ++p) {
            const int q = thread() + p * TH;
            base[p] = s + (int64_t)(q / kQuads * 8) * l + q % kQuads * 4;
        }
    }
    __device__ __forceinline__ bool whole() const { return n == R; }
    __device__ __forceinline__ void load_piece(int i, int64_t k0)  // and all R rows exist
    {
        v[i / 8][i % 8] = *reinterpret_cast<const u32x2u *>(base[i / 8] + (k0 + i % 8) * ld);
    }
    __device__ __forceinline__ void load(int64_t k0, int64_t K)
    {
#pragma unroll
        for (int p = 0; p < P; ++p) {
            const int q = thread() + p * TH, r = q % kQuads * 4, k = q / kQuads * 8;
            const T *at = base[p] + k0 * ld;
            if (k0 + k + 8 <= K && r + 4 <= n) {
#pragma unroll
                for (int j = 0; j < 8; ++j) v[p][j] = *reinterpret_cast<const u32x2u *>(at + j * ld);
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    T e[4];
#pragma unroll
                    for (int x = 0; x < 4; ++x) e[x] = k0 + k + j < K && r + x < n ? at[j * ld + x] : (T)0.0f;
                    v[p][j] = __builtin_bit_cast(u32x2, e);
                }
            }
        }
    }
    __device__ __forceinline__ void store_piece(int i, char *lds, float &)
    {
        const int p = i / 4, x = i % 4, q = thread() + p * TH, r = q % kQuads * 4, c = q / kQuads;
        u32x4 t;
#pragma unroll
        for (int j = 0; j < 4; ++j)
            t[j] = __builtin_amdgcn_perm(v[p][2 * j + 1][x / 2], v[p][2 * j][x / 2], x % 2 ? 0x07060302u : 0x05040100u);
        *reinterpret_cast<u32x4 *>(lds + chunk16(r + x, c)) = t;
    }
};

// The pieces of 8 consecutive k of row r into their planes.
template <int R>
__device__ __forceinline__ void store_pieces(char *lds, int r, int c, const float *f, float &big)
{
    u32x4 h, m, l;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        big = fmaxf(big, fmaxf(fabsf(f[2 * j]), fabsf(f[2 * j + 1])));
        uint32_t a, b, d;
        net_split2(f[2 * j], f[2 * j + 1], a, b, d);
        h[j] = a;
        m[j] = b;
        l[j] = d;
    }
    char *at = lds + chunk32(r, c);
    *reinterpret_cast<u32x4 *>(at) = h;
    *reinterpret_cast<u32x4 *>(at + 64 * R) = m;
    *reinterpret_cast<u32x4 *>(at + 128 * R) = l;
}

template <int R, int TH>
struct Stage32c {
    static constexpr int P = (R * 4 + TH - 1) / TH, kStores = P;
    f32x4 v[P][2];
    const float *row[P];
    // threads past the chunks repeat the first ones' work
    static __device__ __forceinline__ int thread() { return R * 4 < TH ? threadIdx.x % (R * 4) : threadIdx.x; }
    __device__ __forceinline__ void init(const float *src, int64_t ld, int n)
    {
#pragma unroll
        for (int p = 0; p < P; ++p) {
            const int r = thread() / 4 + p * (TH / 4);
            row[p] = src + (int64_t)(r < n ? r : n - 1) * ld;
        }
    }
    __device__ __forceinline__ bool whole() const { return true; }
    __device__ __forceinline__ void load_piece(int p, int64_t k0)  // k0 + 32 <= K
    {
#pragma unroll
        for (int h = 0; h < 2; ++h)
            v[p][h] = *reinterpret_cast<const NetVec<float>::mem *>(row[p] + k0 + 8 * (thread() % 4) + 4 * h);
    }
    __device__ __forceinline__ void load(int64_t k0, int64_t K)
    {
        if (k0 + 32 <= K) {
#pragma unroll
            for (int p = 0; p < P; ++p) load_piece(p, k0);
            return;
        }
#pragma unroll
        for (int p = 0; p < P; ++p)
#pragma unroll
            for (int h = 0; h < 2; ++h) v[p][h] = load_chunk(row[p] + k0, 2 * (thread() % 4) + h, (int)(K - k0), 0.0f);
    }
    __device__ __forceinline__ void store_piece(int p, char *lds, float &big)
    {
        float f[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) f[j] = v[p][j / 4][j % 4];
        store_pieces<R>(lds, thread() / 4 + p * (TH / 4), thread() % 4, f, big);
    }
};

// k-major: 8 k of one row per thread and piece, a wave's loads 256 bytes of a k.
template <int R, int TH>
struct Stage32m {
    static constexpr int P = (R * 4 + TH - 1) / TH, kStores = P;
    float v[P][8];
    const float *base[P];  // the thread's elements at k = 0
    int64_t ld;
    int n;
    static __device__ __forceinline__ int thread() { return R * 4 < TH ? threadIdx.x % (R * 4) : threadIdx.x; }
    __device__ __forceinline__ void init(const float *s, int64_t l, int rows)
    {
        ld = l;
        n = rows;
#pragma unroll
        for (int p = 0; p < P; ++p) {
            const int q = thread() + p * TH;
            base[p] = s + (int64_t)(q / R * 8) * l + q % R;
        }
    }
    __device__ __forceinline__ bool whole() const { return n == R; }
    __device__ __forceinline__ void load_piece(int p, int64_t k0)  // and all R rows exist
    {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[p][j] = base[p][(k0 + j) * ld];
    }
    __device__ __forceinline__ void load(int64_t k0, int64_t K)
    {
#pragma unroll
        for (int p = 0; p < P; ++p) {
            const int q = thread() + p * TH, r = q % R, k = q / R * 8;
#pragma unroll
            for (int j = 0; j < 8; ++j) v[p][j] = k0 + k + j < K && r < n ? base[p][(k0 + j) * ld] : 0.0f;
        }
    }
    __device__ __forceinline__ void store_piece(int p, char *lds, float &big)
    {
        const int q = thread() + p * TH;
        store_pieces<R>(lds, q % R, q / R, v[p], big);
    }
};
template <int R, int TH>
struct Stage<float, false, R, TH> : Stage32c<R, TH> {};
template <int R, int TH>
struct Stage<float, true, R, TH> : Stage32m<R, TH> {};
template <typename T, int R, int TH>
struct Stage<T, false, R, TH> : Stage16c<T, R, TH> {};
template <typename T, int R, int TH>
struct Stage<T, true, R, TH> : Stage16m<T, R, TH> {};

// An operand's tile: element (r, k) for r < n, k < K.
template <typename T>
struct TileOp {
    const T *p;
    int64_t ld;
    int n;
};

// The tile's product and its results.  Waves: WI along i by WJ along j, each
// TI x TJ tiles of 32 x 32 (which read each operand register half as often as
// tiles of 16 would, and leave more registers: the bf16 gradient of 64x512
// 1024x1024 312 -> 288 us).
template <typename T, bool PM, bool QM, int BI, int BJ, int WI, int WJ>
struct TileProduct {
    static constexpr int kThreads = 64 * WI * WJ, BK = kTileK<T>;
    static constexpr bool kSplit = sizeof(T) == 4;
    static constexpr int S = 32, TI = BI / WI / S, TJ = BJ / WJ / S;
    static constexpr int kBuffers = 2;
    static constexpr int kBuffer = kStageBytes<T, BI> + kStageBytes<T, BJ>;
    static constexpr int kPitch = BI / WI + 4;  // floats per row of a wave's results in LDS, S rows at a time
    static constexpr int kOutBytes = WI * WJ * S * kPitch * 4;
    static constexpr int kLds = kBuffers * kBuffer > kOutBytes ? kBuffers * kBuffer : kOutBytes;

    f32x16 acc[TI][TJ];
    int wi, wj, row, q;  // the lane's row of a tile and k group

    __device__ __forceinline__ TileProduct()
    {
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
        wi = wave % WI;
        wj = wave / WI;
        row = threadIdx.x % S;
        q = threadIdx.x % 64 / S;
    }
    __device__ __forceinline__ void clear()
    {
#pragma unroll
        for (int i = 0; i < TI; ++i)
#pragma unroll
            for (int j = 0; j < TJ; ++j) acc[i][j] = (f32x16)(0.0f);
    }
    __device__ __forceinline__ void scale(float f)
    {
#pragma unroll
        for (int i = 0; i < TI; ++i)
#pragma unroll
            for (int j = 0; j < TJ; ++j) acc[i][j] *= f;
    }

    // One K tile (64 k) of 16-bit products in 4 TJ slots of TI products: slot k
    // reads the operand of slot k + 2, and with kNext writes a share of the next
    // tile to LDS (first half of the slots) or loads a share of the one after
    // (second half).  The order is held by the scheduling barriers: left to itself
    // the compiler reads one operand and waits for it before every TI products,
    // and writes and loads in a burst.
    template <bool kNext, typename SP, typename SQ>
    __device__ __forceinline__ void compute16(const char *lds, char *next, SP &sp, SQ &sq, int64_t k0, float &big)
    {
        typedef typename NetVec<T>::reg reg;
        constexpr int kSlots = 4 * TJ, kHalf = 2 * TJ, kW = SP::kStores + SQ::kStores, kV = SP::kLoads + SQ::kLoads;
        reg p[2][TI], s[3];
        auto read_p = [&](int h, int i) {
            p[h % 2][i] = *reinterpret_cast<const reg *>(lds + chunk16((wi * TI + i) * 32 + row, 2 * h + q));
        };
        auto read_s = [&](int k) {
            s[k % 3] = *reinterpret_cast<const reg *>(lds + kStageBytes<T, BI> +
                                                      chunk16((wj * TJ + k % TJ) * 32 + row, 2 * (k / TJ) + q));
        };
        read_s(0);
#pragma unroll
        for (int i = 0; i < TI; ++i) read_p(0, i);
        read_s(1);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int k = 0; k < kSlots; ++k) {
            if (k + 2 < kSlots) read_s(k + 2);
            if (k < 3 * TJ)
#pragma unroll
                for (int i = TI * (k % TJ) / TJ; i < TI * (k % TJ + 1) / TJ; ++i) read_p(k / TJ + 1, i);
            if constexpr (kNext) {
                if (k < kHalf) {
#pragma unroll
                    for (int w = kW * k / kHalf; w < kW * (k + 1) / kHalf; ++w)
                        if (w < SP::kStores) sp.store_piece(w, next, big);
                        else sq.store_piece(w - SP::kStores, next + kStageBytes<T, BI>, big);
                } else {
#pragma unroll
                    for (int v = kV * (k - kHalf) / kHalf; v < kV * (k - kHalf + 1) / kHalf; ++v)
                        if (v < SP::kLoads) sp.load_piece(v, k0);
                        else sq.load_piece(v - SP::kLoads, k0);
                }
            }
#pragma unroll
            for (int i = 0; i < TI; ++i) acc[i][k % TJ] = mma32(p[k / TJ % 2][i], s[k % 3], acc[i][k % TJ]);
            __builtin_amdgcn_sched_barrier(0);
        }
    }
    // The same for a K tile (32 k) of fp32: two halves of 16 k with TJ slots each, a
    // slot the six products of the pieces for TI tiles.  A share of the next tile is
    // split, written and its registers loaded again in one slot, its vector
    // instructions in the shadow of the matrix ones.
    template <bool kNext, typename SP, typename SQ>
    __device__ __forceinline__ void compute32(const char *lds, char *next, SP &sp, SQ &sq, int64_t k0, float &big)
    {
        typedef NetVec<bf16_t>::reg reg;
        constexpr int kSlots = 2 * TJ, kW = SP::kStores + SQ::kStores;
        reg p[2][TI][3], s[2][3];
        auto read_p = [&](int h, int i) {
#pragma unroll
            for (int u = 0; u < 3; ++u)
                p[h][i][u] = *reinterpret_cast<const reg *>(lds + u * 64 * BI + chunk32((wi * TI + i) * S + row, 2 * h + q));
        };
        auto read_s = [&](int k) {
#pragma unroll
            for (int u = 0; u < 3; ++u)
                s[k % 2][u] = *reinterpret_cast<const reg *>(lds + kStageBytes<T, BI> + u * 64 * BJ +
                                                             chunk32((wj * TJ + k % TJ) * S + row, 2 * (k / TJ) + q));
        };
        read_s(0);
#pragma unroll
        for (int i = 0; i < TI; ++i) read_p(0, i);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int k = 0; k < kSlots; ++k) {
            if (k + 1 < kSlots) read_s(k + 1);
            if (k < TJ)
#pragma unroll
                for (int i = TI * k / TJ; i < TI * (k + 1) / TJ; ++i) read_p(1, i);
            if constexpr (kNext) {
#pragma unroll
                for (int w = kW * k / kSlots; w < kW * (k + 1) / kSlots; ++w) {
                    if (w < SP::kStores) {
                        sp.store_piece(w, next, big);
                        sp.load_piece(w, k0);
                    } else {
                        sq.store_piece(w - SP::kStores, next + kStageBytes<T, BI>, big);
                        sq.load_piece(w - SP::kStores, k0);
                    }
                }
            }
            // the small products first
#pragma unroll
            for (int sum = 2; sum >= 0; --sum)
#pragma unroll
                for (int u = 0; u <= sum; ++u)
#pragma unroll
                    for (int i = 0; i < TI; ++i)
                        acc[i][k % TJ] = mma32(p[k / TJ][i][u], s[k % 2][sum - u], acc[i][k % TJ]);
            if constexpr (kNext)
#pragma unroll
                for (int m = 0; m < 6 * TI; ++m) {
                    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                    __builtin_amdgcn_sched_group_barrier(0x002, 7, 0);
                }
            __builtin_amdgcn_sched_barrier(0);
        }
    }
    template <bool kNext, typename SP, typename SQ>
    __device__ __forceinline__ void compute(const char *lds, char *next, SP &sp, SQ &sq, int64_t k0, float &big)
    {
        if constexpr (kSplit) compute32<kNext>(lds, next, sp, sq, k0, big);
        else compute16<kNext>(lds, next, sp, sq, k0, big);
    }

    // With fp32 products, straight from memory.
    __device__ __forceinline__ void again(const TileOp<T> &P, const TileOp<T> &Q, int64_t K)
    {
        clear();
        auto at = [&](const TileOp<T> &o, bool major, int r, int64_t k) -> float {
            if (k >= K) return 0.0f;
            r = r < o.n ? r : o.n - 1;
            return (float)(major ? o.p[k * o.ld + r] : o.p[(int64_t)r * o.ld + k]);
        };
#pragma unroll 1
        for (int64_t k = 0; k < K; k += 2) {
            float p[TI], s[TJ];
#pragma unroll
            for (int i = 0; i < TI; ++i) p[i] = at(P, PM, (wi * TI + i) * S + row, k + q);
#pragma unroll
            for (int j = 0; j < TJ; ++j) s[j] = at(Q, QM, (wj * TJ + j) * S + row, k + q);
#pragma unroll
            for (int j = 0; j < TJ; ++j)
#pragma unroll
                for (int i = 0; i < TI; ++i) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x2f32(p[i], s[j], acc[i][j], 0, 0, 0);
        }
    }

    template <typename SP, typename SQ>
    __device__ __forceinline__ void store_all(char *lds, SP &sp, SQ &sq, float &big)
    {
#pragma unroll
        for (int w = 0; w < SP::kStores; ++w) sp.store_piece(w, lds, big);
#pragma unroll
        for (int w = 0; w < SQ::kStores; ++w) sq.store_piece(w, lds + kStageBytes<T, BI>, big);
    }

    // The product, added to acc; ends with all waves past their last use of LDS.  PAIR:
    // Q's rows in the first half of the tile, R's (R.p, as many) in the second.
    template <bool PAIR = false>
    __device__ __forceinline__ void run(const TileOp<T> &P, const TileOp<T> &Q, int64_t K, char *lds, const T *R = nullptr)
    {
        Stage<T, PM, BI, kThreads> sp;
        Stage<T, QM, BJ, kThreads> sq;
        if (K <= 0) return;
        sp.init(P.p, P.ld, P.n);
        if constexpr (PAIR) sq.init_pair(Q.p, R, Q.ld, Q.n);
        else sq.init(Q.p, Q.ld, Q.n);
        float big = 0.0f;
        const int64_t tiles = (K + BK - 1) / BK;
        sp.load(0, K);
        sq.load(0, K);
        store_all(lds, sp, sq, big);
        if (tiles > 1) {
            sp.load(BK, K);
            sq.load(BK, K);
        }
        lds_barrier();
        int64_t t = 0;
        // while the tile two ahead is whole
        if (sp.whole() && sq.whole())
            for (const int64_t full = K / BK; t + 2 < full; ++t) {
                compute<true>(lds + t % 2 * kBuffer, lds + (t + 1) % 2 * kBuffer, sp, sq, (t + 2) * BK, big);
                lds_barrier();
            }
        for (; t < tiles; ++t) {
            if (t + 1 < tiles) {
                store_all(lds + (t + 1) % 2 * kBuffer, sp, sq, big);
                if (t + 2 < tiles) {
                    sp.load((t + 2) * BK, K);
                    sq.load((t + 2) * BK, K);
                }
            }
            compute<false>(lds + t % 2 * kBuffer, nullptr, sp, sq, 0, big);
            lds_barrier();
        }
        if constexpr (kSplit)
            if (__syncthreads_or(!(big < kTileBig))) again(P, Q, K);
    }

    // The product of P and d_up Q + d_down R, K once for each of the two, the small one
    // first.
    __device__ __forceinline__ void run_split(const TileOp<T> &P, const TileOp<T> &Q, const TileOp<T> &R, int64_t K, char *lds)
    {
        clear();
        run(P, R, K, lds);
        if constexpr (d_up<T> != 1.0f) scale(d_down<T> / d_up<T>);
        run(P, Q, K, lds);
        if constexpr (d_up<T> != 1.0f) scale(d_up<T>);
    }

    // A wave's sub-tiles j to its own part of LDS, S rows of kPitch.
    __device__ __forceinline__ void sub_tile(int j, float *mine) const
    {
#pragma unroll
        for (int k = 0; k < TI; ++k)
#pragma unroll
            for (int b = 0; b < 4; ++b) {  // the lane's quads of the tile
                f32x4 t;
#pragma unroll
                for (int e = 0; e < 4; ++e) t[e] = acc[k][j][4 * b + e];
                *reinterpret_cast<f32x4 *>(mine + row * kPitch + k * S + 8 * b + 4 * q) = t;
            }
    }

    // The results of a pair, two waves of one sub-tile each: row j of the one and of the
    // other, d_up and d_down times; every wave stores half of the rows.
    template <typename F>
    __device__ __forceinline__ void results_pair(int ni, int nj, char *lds, F &out)
    {
        static_assert(WI == 1 && WJ == 2 && TJ == 1, "two waves");
        constexpr int N = NetVec<T>::N, kLanes = BI / N, kRows = 64 / kLanes;
        float *all = reinterpret_cast<float *>(lds);
        sub_tile(0, all + wj * S * kPitch);
        lds_barrier();
        const int lane = threadIdx.x % 64, i = lane % kLanes * N, n = ni - i < N ? ni - i : N;
        for (int r = wj * (S / 2) + lane / kLanes; r < (wj + 1) * (S / 2); r += kRows) {
            if (r >= nj || n <= 0) continue;
            float v[N];
#pragma unroll
            for (int e = 0; e < N; ++e) v[e] = all[r * kPitch + i + e] * d_up<T> + all[(S + r) * kPitch + i + e] * d_down<T>;
            out.store(r, i, v, n, {});
        }
    }

    // The results, S rows of every wave at a time through LDS (the wave's own part
    // of it).  A lane gets n <= N neighbours i .. i + n - 1 of a row j at a time (N:
    // 16 bytes of the element type, a row's in consecutive lanes), always the same
    // i: out.begin(i, n) loads what belongs to the columns once, out.load(j, i, n)
    // what belongs to the row (for all of a lane's rows before the first is done, so
    // that their latencies overlap), out.store(j, i, v, n, loaded) is the result.
    template <typename F>
    __device__ __forceinline__ void results(int ni, int nj, char *lds, F &out)
    {
        constexpr int N = NetVec<T>::N, kRow = BI / WI, kLanes = kRow / N, kRows = 64 / kLanes, kIter = S / kRows;
        float *mine = reinterpret_cast<float *>(lds) + (wj * WI + wi) * S * kPitch;
        const int lane = threadIdx.x % 64, c = lane % kLanes * N, i = wi * kRow + c, n = ni - i < N ? ni - i : N;
        if (n > 0) out.begin(i, n);
#pragma unroll
        for (int j = 0; j < TJ; ++j) {
            typename NetVec<T>::reg loaded[kIter];
            const int r0 = (wj * TJ + j) * S + lane / kLanes;
#pragma unroll
            for (int it = 0; it < kIter; ++it)
                if (r0 + it * kRows < nj && n > 0) loaded[it] = out.load(r0 + it * kRows, i, n);
            sub_tile(j, mine);
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
            for (int it = 0; it < kIter; ++it) {
                if (r0 + it * kRows >= nj || n <= 0) continue;
                float v[N];
#pragma unroll
                for (int e = 0; e < N; e += 4) {
                    const f32x4 t = *reinterpret_cast<const f32x4 *>(mine + (lane / kLanes + it * kRows) * kPitch + c + e);
#pragma unroll
                    for (int x = 0; x < 4; ++x) v[e + x] = t[x];
                }
                out.store(r0 + it * kRows, i, v, n, loaded[it]);
            }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        }
    }
};

}  // namespace evox
