// Linear layers of a population of networks: y = act(x W_g^T + b_g) + r and
// its gradient, one thread per result.
#include "evox_net.hpp"

namespace evox {

namespace {

unsigned net_grid(int64_t n)
{
    const int64_t b = (n + 255) / 256;
    return (unsigned)(b < 1 ? 1 : b > ((int64_t)1 << 20) ? (int64_t)1 << 20 : b);
}

template <typename T>
__global__ __launch_bounds__(256) void k_linear(LinearArgs a)
{
    const T *x = (const T *)a.x, *w = (const T *)a.w, *b = (const T *)a.b, *r = (const T *)a.r;
    T *z = (T *)a.z, *y = (T *)a.y;
    for (int64_t q = (int64_t)blockIdx.x * 256 + threadIdx.x; q < a.rows.M * a.n_out; q += (int64_t)gridDim.x * 256) {
        const int64_t m = q / a.n_out, o = q % a.n_out, g = net_of_row(a.rows, m);
        if (g < 0) continue;
        const T *xr = x + (a.x_shared ? m - g * a.rows.n : m) * a.ldx, *wr = w + g * a.w_stride + o * a.ldw;
        float s = 0.0f;
        for (int64_t k = 0; k < a.n_in; ++k) s = fmaf((float)xr[k], (float)wr[k], s);
        if (b) s += (float)b[g * a.b_stride + o];
        if (z) z[m * a.ldz + o] = (T)s;
        s = act_value(a.act, s);
        if (r) s += (float)r[m * a.ldr + o];
        y[m * a.ldy + o] = (T)s;
    }
}

// d = dy act'(z), rounded to the element type.
template <typename T>
__device__ __forceinline__ float grad_of_z(const LinearGradArgs &a, int64_t m, int64_t o)
{
    const float d = (float)((const T *)a.dy)[m * a.lddy + o];
    if (a.act == ACT_NONE) return d;
    return d * act_slope(a.act, (float)((const T *)a.z)[m * a.ldz + o]);
}

template <typename T>
__global__ __launch_bounds__(256) void k_linear_dx(LinearGradArgs a)
{
    const T *w = (const T *)a.w;
    T *dx = (T *)a.dx;
    for (int64_t q = (int64_t)blockIdx.x * 256 + threadIdx.x; q < a.rows.M * a.n_in; q += (int64_t)gridDim.x * 256) {
        const int64_t m = q / a.n_in, i = q % a.n_in, g = net_of_row(a.rows, m);
        if (g < 0) continue;
        float s = 0.0f;
        for (int64_t o = 0; o < a.n_out; ++o)
            s = fmaf((float)(T)grad_of_z<T>(a, m, o), (float)w[g * a.w_stride + o * a.ldw + i], s);
        dx[m * a.lddx + i] = (T)s;
    }
}

// Column n_in of a network's gradient is db.
template <typename T>
__global__ __launch_bounds__(256) void k_linear_dw(LinearGradArgs a)
{
    const T *x = (const T *)a.x;
    T *dw = (T *)a.dw, *db = (T *)a.db;
    const int64_t cols = a.n_in + 1;
    for (int64_t q = (int64_t)blockIdx.x * 256 + threadIdx.x; q < a.rows.G * a.n_out * cols;
         q += (int64_t)gridDim.x * 256) {
        const int64_t i = q % cols, o = q / cols % a.n_out, g = q / cols / a.n_out;
        if (i < a.n_in ? !dw : !db) continue;
        int64_t lo, hi;
        net_rows(a.rows, g, &lo, &hi);
        float s = 0.0f;
        for (int64_t m = lo; m < hi; ++m) {
            const float d = grad_of_z<T>(a, m, o);
            if (i == a.n_in) s += d;
            else s = fmaf((float)(T)d, (float)x[(a.x_shared ? m - lo : m) * a.ldx + i], s);
        }
        if (i == a.n_in) db[g * a.db_stride + o] = (T)s;
        else dw[g * a.dw_stride + o * a.lddw + i] = (T)s;
    }
}

}  // namespace

hipError_t launch_linear(const LinearArgs &a, hipStream_t s)
{
    return net_dispatch(a.dtype, [&](auto t) {
        hipLaunchKernelGGL((k_linear<decltype(t)>), dim3(net_grid(a.rows.M * a.n_out)), dim3(256), 0, s, a);
        return hipGetLastError();
    });
}

size_t linear_grad_scratch(const LinearGradArgs &) { return 256; }

hipError_t launch_linear_grad(const LinearGradArgs &a, hipStream_t s)
{
    return net_dispatch(a.dtype, [&](auto t) {
        if (a.dx && a.rows.M)
            hipLaunchKernelGGL((k_linear_dx<decltype(t)>), dim3(net_grid(a.rows.M * a.n_in)), dim3(256), 0, s, a);
        if (a.dw || a.db)
            hipLaunchKernelGGL((k_linear_dw<decltype(t)>), dim3(net_grid(a.rows.G * a.n_out * (a.n_in + 1))),
                               dim3(256), 0, s, a);
        return hipGetLastError();
    });
}

}  // namespace evox
