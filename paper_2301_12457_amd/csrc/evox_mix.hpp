// Mixtures of networks (gate, route, dispatch, combine) and the optimizer's step:
// the kernels' arguments.
#pragma once

#include "evox_net.hpp"

namespace evox {

enum GateOver { GATE_CHOSEN = 0, GATE_ALL = 1 };
constexpr int kGateMaxK = 32, kSlotsMaxK = 1024;

struct GateArgs {
    int32_t dtype, over;
    int64_t T;
    int32_t G, k;
    const void *z;
    int64_t ldz, lddz;
    int32_t *ids;
    float *w;
    const int32_t *ids_in;  // of the gradient
    const float *w_in, *dw;
    void *dz;
};
hipError_t launch_gate(const GateArgs &a, hipStream_t s);
hipError_t launch_gate_grad(const GateArgs &a, hipStream_t s);

struct RouteArgs {
    int64_t n;  // slots, T k
    int64_t G;
    const int32_t *ids;
    int32_t *off, *pos, *src;
    void *scratch;
};
size_t route_scratch(const RouteArgs &a);  // of the sizes alone
hipError_t launch_route(const RouteArgs &a, hipStream_t s);

struct SlotArgs {
    int32_t dtype;
    int64_t T, M, D;
    int32_t k;
    const int32_t *pos;
    const float *w;
    const void *x;   // [T][D]: dispatch's rows, combine's residual, the gradient's dy
    const void *xs;  // [M][D]: rows of the networks, read
    void *y;         // combine's result [T][D]
    void *out;       // rows of the networks, written
    float *dw;
    int64_t ldx, ldy, lds, ldo;
};
hipError_t launch_dispatch(const SlotArgs &a, hipStream_t s);
hipError_t launch_combine(const SlotArgs &a, hipStream_t s);
hipError_t launch_combine_grad(const SlotArgs &a, hipStream_t s);

// One tensor of a step: [rows][n] at pitches (states and master at one).
struct AdamTensor {
    void *p;
    const void *g;
    void *m, *v;
    float *m_scale, *v_scale, *master;
    int64_t rows, n, ldp, ldg, lds;
};
struct AdamCall {
    int32_t dtype, bits, master;
    double lr, beta1, beta2, eps, decay;
    const float *lr_dev;
    int64_t *clock;
    const void *table;
    int64_t count, tiles;
};
constexpr int kAdamBlock = 256;  // elements per scale of an 8-bit state
int64_t adam_groups(int32_t bits, int64_t rows, int64_t n);  // below 2^31 for each tensor
size_t adam_table(int64_t count);                            // bytes
int64_t adam_fill_table(int32_t bits, const AdamTensor *t, int64_t count, void *host);  // its tiles
hipError_t launch_adamw(const AdamCall &c, hipStream_t s);

// Lanes of a wave in groups of L (a power of two): the maximum or sum over a group in
// every lane of it, by lane exchanges in registers (no LDS): neighbours, pairs, halves
// of eight and of sixteen by DPP, rows and halves of the wave by gfx950's swaps.  All
// lanes of the wave take part; L the same in all.
template <int CTRL>
__device__ __forceinline__ uint32_t lane_dpp(uint32_t v)
{
    return (uint32_t)__builtin_amdgcn_mov_dpp((int)v, CTRL, 0xf, 0xf, true);
}
template <typename F>
__device__ __forceinline__ uint32_t lanes_all(uint32_t v, int L, F &&f)
{
    if (L > 1) v = f(v, lane_dpp<0xB1>(v));   // lane ^ 1
    if (L > 2) v = f(v, lane_dpp<0x4E>(v));   // lane ^ 2
    if (L > 4) v = f(v, lane_dpp<0x141>(v));  // mirrored in eight: the other four
    if (L > 8) v = f(v, lane_dpp<0x140>(v));  // mirrored in sixteen: the other eight
    if (L > 16) {
        const auto r = __builtin_amdgcn_permlane16_swap(v, v, false, false);
        v = f(r[0], r[1]);
    }
    if (L > 32) {
        const auto r = __builtin_amdgcn_permlane32_swap(v, v, false, false);
        v = f(r[0], r[1]);
    }
    return v;
}
__device__ __forceinline__ uint32_t lanes_max(uint32_t v, int L)
{
    return lanes_all(v, L, [](uint32_t a, uint32_t b) { return a > b ? a : b; });
}
__device__ __forceinline__ float lanes_sum(float v, int L)
{
    return __uint_as_float(lanes_all(__float_as_uint(v), L, [](uint32_t a, uint32_t b) {
        return __float_as_uint(__uint_as_float(a) + __uint_as_float(b));
    }));
}
template <int CTRL>
__device__ __forceinline__ uint64_t lane_dpp64(uint64_t v)
{
    return (uint64_t)lane_dpp<CTRL>((uint32_t)(v >> 32)) << 32 | lane_dpp<CTRL>((uint32_t)v);
}
__device__ __forceinline__ uint64_t lanes_max(uint64_t v, int L)
{
    const auto f = [](uint64_t a, uint64_t b) { return a > b ? a : b; };
    if (L > 1) v = f(v, lane_dpp64<0xB1>(v));
    if (L > 2) v = f(v, lane_dpp64<0x4E>(v));
    if (L > 4) v = f(v, lane_dpp64<0x141>(v));
    if (L > 8) v = f(v, lane_dpp64<0x140>(v));
    if (L > 16) {
        const auto h = __builtin_amdgcn_permlane16_swap((uint32_t)(v >> 32), (uint32_t)(v >> 32), false, false);
        const auto l = __builtin_amdgcn_permlane16_swap((uint32_t)v, (uint32_t)v, false, false);
        v = f((uint64_t)h[0] << 32 | l[0], (uint64_t)h[1] << 32 | l[1]);
    }
    if (L > 32) {
        const auto h = __builtin_amdgcn_permlane32_swap((uint32_t)(v >> 32), (uint32_t)(v >> 32), false, false);
        const auto l = __builtin_amdgcn_permlane32_swap((uint32_t)v, (uint32_t)v, false, false);
        v = f((uint64_t)h[0] << 32 | l[0], (uint64_t)h[1] << 32 | l[1]);
    }
    return v;
}

}  // namespace evox
