// Layers, norms and losses of a population of networks: the kernels' arguments,
// element types and the rows of each network.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

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

typedef __bf16 bf16_t;
typedef _Float16 f16_t;

// Type-dependent launches: f is called with a value of the element type.
template <typename F>
hipError_t net_dispatch(int32_t dtype, F &&f)
{
    if (dtype == NET_F32) return f(float{});
    if (dtype == NET_BF16) return f(bf16_t{});
    return f(f16_t{});
}

// The rows [lo, hi) of network g, within [0, M] whatever off holds.
__device__ __forceinline__ void net_rows(const NetRows &r, int64_t g, int64_t *lo, int64_t *hi)
{
    if (!r.off) {
        *lo = g * r.n;
        *hi = *lo + r.n;
        return;
    }
    const int64_t a = r.off[g], b = r.off[g + 1];
    *lo = a < 0 ? 0 : a > r.M ? r.M : a;
    *hi = b < *lo ? *lo : b > r.M ? r.M : b;
}

// The network of a row: the last g with off[g] <= row (networks without rows
// share their offset with the next), or -1 where the row belongs to none.
__device__ __forceinline__ int64_t net_of_row(const NetRows &r, int64_t row)
{
    if (!r.off) return row / r.n;
    int64_t lo = -1, hi = r.G;  // off[lo] <= row < off[hi]
    while (hi - lo > 1) {
        const int64_t mid = (lo + hi) / 2;
        if (r.off[mid] <= row) lo = mid;
        else hi = mid;
    }
    return lo >= 0 && row < r.off[lo + 1] ? lo : -1;
}

__device__ __forceinline__ float act_value(int act, float z)
{
    switch (act) {
    case ACT_RELU: return z < 0.0f ? 0.0f : z;  // NaN passes
    case ACT_TANH: return tanhf(z);
    case ACT_GELU: return 0.5f * z * (1.0f + erff(z * 0.70710678f));
    case ACT_SILU: return z / (1.0f + expf(-z));
    default: return z;
    }
}

__device__ __forceinline__ float act_slope(int act, float z)
{
    switch (act) {
    case ACT_RELU: return z > 0.0f ? 1.0f : z == z ? 0.0f : z;
    case ACT_TANH: {
        const float t = tanhf(z);
        return (1.0f - t) * (1.0f + t);
    }
    case ACT_GELU:
        return 0.5f * (1.0f + erff(z * 0.70710678f)) + z * 0.39894228f * expf(-0.5f * z * z);
    case ACT_SILU: {
        const float s = 1.0f / (1.0f + expf(-z));
        return s * (1.0f + z * (1.0f - s));
    }
    default: return 1.0f;
    }
}

}  // namespace evox
