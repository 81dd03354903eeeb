// Layer norm and cross-entropy over the rows of a population of networks, one
// thread per row (or per column of a network's gradient).
#include "evox_net.hpp"

namespace evox {

namespace {

unsigned net_grid(int64_t n)
{
    const int64_t b = (n + 255) / 256;
    return (unsigned)(b < 1 ? 1 : b > ((int64_t)1 << 20) ? (int64_t)1 << 20 : b);
}

template <typename T>
__global__ __launch_bounds__(256) void k_layernorm(NormArgs a)
{
    for (int64_t m = (int64_t)blockIdx.x * 256 + threadIdx.x; m < a.rows.M; m += (int64_t)gridDim.x * 256) {
        const int64_t g = net_of_row(a.rows, m);
        if (g < 0) continue;
        const T *x = (const T *)a.x + m * a.ldx, *ga = (const T *)a.gamma + g * a.p_stride,
                *be = (const T *)a.beta + g * a.p_stride;
        T *y = (T *)a.y + m * a.ldy;
        float s = 0.0f, v = 0.0f;
        for (int64_t j = 0; j < a.D; ++j) s += (float)x[j];
        const float mean = s / (float)a.D;
        for (int64_t j = 0; j < a.D; ++j) {
            const float c = (float)x[j] - mean;
            v = fmaf(c, c, v);
        }
        const float rstd = 1.0f / sqrtf(v / (float)a.D + a.eps);
        for (int64_t j = 0; j < a.D; ++j)
            y[j] = (T)fmaf(((float)x[j] - mean) * rstd, (float)ga[j], (float)be[j]);
        if (a.mean) a.mean[m] = mean;
        if (a.rstd) a.rstd[m] = rstd;
    }
}

template <typename T>
__global__ __launch_bounds__(256) void k_layernorm_dx(NormArgs a)
{
    for (int64_t m = (int64_t)blockIdx.x * 256 + threadIdx.x; m < a.rows.M; m += (int64_t)gridDim.x * 256) {
        const int64_t g = net_of_row(a.rows, m);
        if (g < 0) continue;
        const T *x = (const T *)a.x + m * a.ldx, *dy = (const T *)a.dy + m * a.ldy,
                *ga = (const T *)a.gamma + g * a.p_stride;
        T *dx = (T *)a.dx + m * a.lddx;
        const float mean = a.mean_in[m], rstd = a.rstd_in[m];
        float s1 = 0.0f, s2 = 0.0f;
        for (int64_t j = 0; j < a.D; ++j) {
            const float p = (float)dy[j] * (float)ga[j];
            s1 += p;
            s2 = fmaf(p, ((float)x[j] - mean) * rstd, s2);
        }
        s1 /= (float)a.D;
        s2 /= (float)a.D;
        for (int64_t j = 0; j < a.D; ++j)
            dx[j] = (T)(rstd * ((float)dy[j] * (float)ga[j] - s1 - ((float)x[j] - mean) * rstd * s2));
    }
}

template <typename T>
__global__ __launch_bounds__(256) void k_layernorm_dp(NormArgs a)
{
    for (int64_t q = (int64_t)blockIdx.x * 256 + threadIdx.x; q < a.rows.G * a.D; q += (int64_t)gridDim.x * 256) {
        const int64_t g = q / a.D, j = q % a.D;
        int64_t lo, hi;
        net_rows(a.rows, g, &lo, &hi);
        float sg = 0.0f, sb = 0.0f;
        for (int64_t m = lo; m < hi; ++m) {
            const float dy = (float)((const T *)a.dy)[m * a.ldy + j];
            const float h = ((float)((const T *)a.x)[m * a.ldx + j] - a.mean_in[m]) * a.rstd_in[m];
            sb += dy;
            sg = fmaf(dy, h, sg);
        }
        ((T *)a.dgamma)[g * a.dp_stride + j] = (T)sg;
        ((T *)a.dbeta)[g * a.dp_stride + j] = (T)sb;
    }
}

__device__ __forceinline__ int xent_label(const XentArgs &a, int64_t g, int64_t m)
{
    return a.labels[a.labels_shared ? m - g * a.rows.n : m];
}

// Fitness of a network, and its count of rows (in the scratch).
template <typename T>
__global__ __launch_bounds__(256) void k_xent_fit(XentArgs a)
{
    for (int64_t g = (int64_t)blockIdx.x * 256 + threadIdx.x; g < a.rows.G; g += (int64_t)gridDim.x * 256) {
        int64_t lo, hi, count = 0;
        net_rows(a.rows, g, &lo, &hi);
        double sum = 0.0;
        for (int64_t m = lo; m < hi; ++m) {
            const T *z = (const T *)a.logits + m * a.ldz;
            const int lab = xent_label(a, g, m);
            if (lab < 0 || lab >= a.C) continue;
            float top = -INFINITY, s = 0.0f;
            for (int64_t c = 0; c < a.C; ++c) top = fmaxf(top, (float)z[c]);
            for (int64_t c = 0; c < a.C; ++c) s += expf((float)z[c] - top);
            sum += (double)(logf(s) + (top - (float)z[lab]));
            ++count;
        }
        a.fit[g] = (float)(sum / (double)count);
        ((float *)a.scratch)[g] = (float)count;
    }
}

template <typename T>
__global__ __launch_bounds__(256) void k_xent_grad(XentArgs a)
{
    for (int64_t m = (int64_t)blockIdx.x * 256 + threadIdx.x; m < a.rows.M; m += (int64_t)gridDim.x * 256) {
        const int64_t g = net_of_row(a.rows, m);
        if (g < 0) continue;
        const T *z = (const T *)a.logits + m * a.ldz;
        T *dz = (T *)a.dz + m * a.lddz;
        const int lab = xent_label(a, g, m);
        if (lab < 0 || lab >= a.C) {
            for (int64_t c = 0; c < a.C; ++c) dz[c] = (T)0.0f;
            continue;
        }
        float top = -INFINITY, s = 0.0f;
        for (int64_t c = 0; c < a.C; ++c) top = fmaxf(top, (float)z[c]);
        for (int64_t c = 0; c < a.C; ++c) s += expf((float)z[c] - top);
        const float count = ((const float *)a.scratch)[g];
        for (int64_t c = 0; c < a.C; ++c)
            dz[c] = (T)((expf((float)z[c] - top) / s - (c == lab ? 1.0f : 0.0f)) / count);
    }
}

}  // namespace

hipError_t launch_layernorm(const NormArgs &a, hipStream_t s)
{
    return net_dispatch(a.dtype, [&](auto t) {
        hipLaunchKernelGGL((k_layernorm<decltype(t)>), dim3(net_grid(a.rows.M)), dim3(256), 0, s, a);
        return hipGetLastError();
    });
}

size_t layernorm_grad_scratch(const NormArgs &) { return 256; }

hipError_t launch_layernorm_grad(const NormArgs &a, hipStream_t s)
{
    return net_dispatch(a.dtype, [&](auto t) {
        using T = decltype(t);
        if (a.dgamma)  // first: dx may take dy's place
            hipLaunchKernelGGL((k_layernorm_dp<T>), dim3(net_grid(a.rows.G * a.D)), dim3(256), 0, s, a);
        if (a.dx && a.rows.M) hipLaunchKernelGGL((k_layernorm_dx<T>), dim3(net_grid(a.rows.M)), dim3(256), 0, s, a);
        return hipGetLastError();
    });
}

size_t xent_scratch(const XentArgs &a) { return 4 * (size_t)a.rows.G; }

hipError_t launch_xent(const XentArgs &a, hipStream_t s)
{
    return net_dispatch(a.dtype, [&](auto t) {
        using T = decltype(t);
        hipLaunchKernelGGL((k_xent_fit<T>), dim3(net_grid(a.rows.G)), dim3(256), 0, s, a);
        if (a.dz && a.rows.M) hipLaunchKernelGGL((k_xent_grad<T>), dim3(net_grid(a.rows.M)), dim3(256), 0, s, a);
        return hipGetLastError();
    });
}

}  // namespace evox
