// Layer norm of rows with the residual sum before it, and its gradients
// (include/gear.h).  With t a row, u = (t - mean) r, r = 1 / sqrt(var + eps):
//   y = u w + b,   dx = r (g - mean(g) - u mean(g u)) + dt,  g = dy w,
//   dw = sum_rows dy u,   db = sum_rows dy.
//
// The mean is taken first and the squares around it, with what the mean itself was
// off by taken out again: sums of t and t^2 would cancel where |mean| exceeds the
// deviation.
#include "element.h"
#include "gear_internal.h"

namespace gear {
namespace {

constexpr int kThreads = 256;

struct Args {
    const void *x, *residual, *weight, *bias, *dy, *dtotal;
    void *y, *total, *dx, *dweight, *dbias;
    float* saved;
    float* work;  // [blocks][2][D]
    int64_t n, D;
    int64_t x_row, residual_row, dy_row, dtotal_row;
    int32_t param_dtype, blocks;
    float eps;
};

__device__ __forceinline__ float param_at(const void* p, int32_t dtype, int64_t i, float none) {
    if (p == nullptr) return none;
    if (dtype == GEAR_DTYPE_F32) return static_cast<const float*>(p)[i];
    if (dtype == GEAR_DTYPE_BF16) return (float)static_cast<const __bf16*>(p)[i];
    return (float)static_cast<const _Float16*>(p)[i];
}
__device__ __forceinline__ void param_put(void* p, int32_t dtype, int64_t i, float v) {
    if (dtype == GEAR_DTYPE_F32) static_cast<float*>(p)[i] = v;
    else if (dtype == GEAR_DTYPE_BF16) static_cast<__bf16*>(p)[i] = (__bf16)v;
    else static_cast<_Float16*>(p)[i] = (_Float16)v;
}

__device__ __forceinline__ float wave_add(float v) {
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) v += __shfl_xor(v, off);
    return v;
}

// Two sums over the workgroup, in every thread.
__device__ __forceinline__ void block_add2(float& a, float& b, float (*s)[2]) {
    a = wave_add(a);
    b = wave_add(b);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) {
        s[threadIdx.x >> 6][0] = a;
        s[threadIdx.x >> 6][1] = b;
    }
    __syncthreads();
    a = b = 0.0f;
#pragma unroll
    for (int k = 0; k < kThreads / 64; k++) {
        a += s[k][0];
        b += s[k][1];
    }
}

// Rows of any length, an element a lane and load.
template <typename E>
__global__ __launch_bounds__(kThreads) void forward_kernel(const Args a) {
    __shared__ float s[kThreads / 64][2];
    for (int64_t row = blockIdx.x; row < a.n; row += gridDim.x) {
        const E* x = static_cast<const E*>(a.x) + row * a.x_row;
        const E* r = a.residual ? static_cast<const E*>(a.residual) + row * a.residual_row : nullptr;
        const auto value = [&](int64_t j) {
            const float v = (float)x[j];
            return r ? (float)(E)(v + (float)r[j]) : v;
        };
        float sum = 0.0f, none = 0.0f;
        for (int64_t j = threadIdx.x; j < a.D; j += kThreads) sum += value(j);
        block_add2(sum, none, s);
        const float c = sum / (float)a.D;
        float off = 0.0f, sq = 0.0f;
        for (int64_t j = threadIdx.x; j < a.D; j += kThreads) {
            const float d = value(j) - c;
            off += d;
            sq = fmaf(d, d, sq);
        }
        block_add2(off, sq, s);
        off /= (float)a.D;
        const float var = fmaxf(fmaf(-off, off, sq / (float)a.D), 0.0f);
        const float rstd = 1.0f / sqrtf(var + a.eps);
        E* y = static_cast<E*>(a.y) + row * a.D;
        E* t = a.total ? static_cast<E*>(a.total) + row * a.D : nullptr;
        for (int64_t j = threadIdx.x; j < a.D; j += kThreads) {
            const float v = value(j);
            if (t) t[j] = (E)v;
            y[j] = (E)fmaf((v - c - off) * rstd, param_at(a.weight, a.param_dtype, j, 1.0f),
                           param_at(a.bias, a.param_dtype, j, 0.0f));
        }
        if (a.saved && threadIdx.x == 0) {
            a.saved[2 * row] = c + off;
            a.saved[2 * row + 1] = rstd;
        }
    }
}

template <typename E>
__global__ __launch_bounds__(kThreads) void dx_kernel(const Args a) {
    __shared__ float s[kThreads / 64][2];
    for (int64_t row = blockIdx.x; row < a.n; row += gridDim.x) {
        const E* t = static_cast<const E*>(a.x) + row * a.x_row;
        const E* dy = static_cast<const E*>(a.dy) + row * a.dy_row;
        const float mean = a.saved[2 * row], rstd = a.saved[2 * row + 1];
        float g = 0.0f, gu = 0.0f;
        for (int64_t j = threadIdx.x; j < a.D; j += kThreads) {
            const float v = (float)dy[j] * param_at(a.weight, a.param_dtype, j, 1.0f);
            g += v;
            gu = fmaf(v, ((float)t[j] - mean) * rstd, gu);
        }
        block_add2(g, gu, s);
        g /= (float)a.D;
        gu /= (float)a.D;
        for (int64_t j = threadIdx.x; j < a.D; j += kThreads) {
            const float v = (float)dy[j] * param_at(a.weight, a.param_dtype, j, 1.0f);
            const float u = ((float)t[j] - mean) * rstd;
            float o = (v - g - u * gu) * rstd;
            if (a.dtotal) o += (float)(static_cast<const E*>(a.dtotal) + row * a.dtotal_row)[j];
            (static_cast<E*>(a.dx) + row * a.D)[j] = (E)o;
        }
    }
}

// Sums over a slice of the rows, a lane per column: slice blockIdx.y of a.blocks.
template <typename E>
__global__ __launch_bounds__(kThreads) void columns_kernel(const Args a) {
    const int64_t j = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    if (j >= a.D) return;
    const int64_t first = a.n * blockIdx.y / a.blocks, end = a.n * (blockIdx.y + 1) / a.blocks;
    float dw = 0.0f, db = 0.0f;
    for (int64_t row = first; row < end; row++) {
        const float dy = (float)(static_cast<const E*>(a.dy) + row * a.dy_row)[j];
        const float t = (float)(static_cast<const E*>(a.x) + row * a.x_row)[j];
        dw = fmaf(dy, (t - a.saved[2 * row]) * a.saved[2 * row + 1], dw);
        db += dy;
    }
    a.work[(2 * (int64_t)blockIdx.y) * a.D + j] = dw;
    a.work[(2 * (int64_t)blockIdx.y + 1) * a.D + j] = db;
}

__global__ __launch_bounds__(kThreads) void finish_kernel(const Args a) {
    const int64_t j = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    if (j >= a.D) return;
    float dw = 0.0f, db = 0.0f;
    for (int k = 0; k < a.blocks; k++) {
        dw += a.work[(2 * (int64_t)k) * a.D + j];
        db += a.work[(2 * (int64_t)k + 1) * a.D + j];
    }
    if (a.dweight) param_put(a.dweight, a.param_dtype, j, dw);
    if (a.dbias) param_put(a.dbias, a.param_dtype, j, db);
}

constexpr int64_t kMaxValues = 1ll << 40, kMaxD = 1 << 20;
int blocks_of(int64_t n) { return (int)(n < 1 ? 1 : n < 512 ? n : 512); }
int64_t work_bytes_of(const gear_norm_desc& d) { return 2 * blocks_of(d.n) * d.D * (int64_t)sizeof(float); }

const char* flaw(const gear_norm_desc* d) {
    if (d == nullptr) return "NULL descriptor";
    if (float_bytes(d->dtype) == 0) return "dtype must be F16, BF16 or F32";
    if (d->param_dtype != d->dtype && d->param_dtype != GEAR_DTYPE_F32) return "param_dtype must be dtype or F32";
    if (d->n < 0 || d->D < 1 || d->D > kMaxD || d->n > kMaxValues / d->D) return "size out of range";
    if (d->x_row < 0 || d->residual_row < 0 || d->dy_row < 0 || d->dtotal_row < 0) return "negative stride";
    if (!(d->eps >= 0.0f) || d->eps > 3e38f) return "eps below 0 or not finite";
    return nullptr;
}

Args args_of(const gear_norm_desc& d, const void* x, const void* weight) {
    Args a{};
    a.x = x;
    a.weight = weight;
    a.n = d.n;
    a.D = d.D;
    a.x_row = d.x_row;
    a.residual_row = d.residual_row;
    a.dy_row = d.dy_row;
    a.dtotal_row = d.dtotal_row;
    a.param_dtype = d.param_dtype;
    a.eps = d.eps;
    return a;
}

}  // namespace
}  // namespace gear

extern "C" int gear_layer_norm_sizes(const gear_norm_desc* d, int64_t* work_bytes) {
    using namespace gear;
    if (const char* w = flaw(d)) return fail(GEAR_E_INVAL, std::string("gear_layer_norm_sizes: ") + w);
    if (work_bytes) *work_bytes = work_bytes_of(*d);
    return GEAR_OK;
}

extern "C" int gear_layer_norm(const gear_norm_desc* d, const void* d_x, const void* d_residual, const void* d_weight,
                               const void* d_bias, void* d_y, void* d_total, float* d_saved, void* stream) {
    using namespace gear;
    if (const char* w = flaw(d)) return fail(GEAR_E_INVAL, std::string("gear_layer_norm: ") + w);
    if (d->n == 0) return GEAR_OK;
    if (d_x == nullptr || d_y == nullptr) return fail(GEAR_E_INVAL, "gear_layer_norm: NULL x or y");
    if (d_total != nullptr && d_residual == nullptr) return fail(GEAR_E_INVAL, "gear_layer_norm: total without a residual");
    Args a = args_of(*d, d_x, d_weight);
    a.residual = d_residual;
    a.bias = d_bias;
    a.y = d_y;
    a.total = d_total;
    a.saved = d_saved;
    (void)hipGetLastError();  // an error pending from an earlier HIP call is not this call's
    const dim3 grid((unsigned)(a.n < 4096 ? a.n : 4096));
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (d->dtype == GEAR_DTYPE_F32) hipLaunchKernelGGL(forward_kernel<float>, grid, dim3(kThreads), 0, s, a);
    else if (d->dtype == GEAR_DTYPE_BF16) hipLaunchKernelGGL(forward_kernel<__bf16>, grid, dim3(kThreads), 0, s, a);
    else hipLaunchKernelGGL(forward_kernel<_Float16>, grid, dim3(kThreads), 0, s, a);
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? GEAR_OK : hip_fail(e, "gear_layer_norm: launch");
}

extern "C" int gear_layer_norm_backward(const gear_norm_desc* d, const void* d_t, const float* d_saved,
                                        const void* d_weight, const void* d_dy, const void* d_dtotal, void* d_dx,
                                        void* d_dweight, void* d_dbias, void* d_work, int64_t work_bytes,
                                        void* stream) {
    using namespace gear;
    if (const char* w = flaw(d)) return fail(GEAR_E_INVAL, std::string("gear_layer_norm_backward: ") + w);
    const bool params = d_dweight != nullptr || d_dbias != nullptr;
    if (d->n > 0 && (d_t == nullptr || d_saved == nullptr || d_dy == nullptr))
        return fail(GEAR_E_INVAL, "gear_layer_norm_backward: NULL t, saved or dy");
    if (params && (d_work == nullptr || work_bytes < work_bytes_of(*d)))
        return fail(GEAR_E_INVAL, "gear_layer_norm_backward: workspace smaller than gear_layer_norm_sizes states");
    Args a = args_of(*d, d_t, d_weight);
    a.saved = const_cast<float*>(d_saved);
    a.dy = d_dy;
    a.dtotal = d_dtotal;
    a.dx = d_dx;
    a.dweight = d_dweight;
    a.dbias = d_dbias;
    a.work = static_cast<float*>(d_work);
    a.blocks = blocks_of(a.n);
    (void)hipGetLastError();  // an error pending from an earlier HIP call is not this call's
    hipStream_t s = static_cast<hipStream_t>(stream);
    hipError_t e = hipSuccess;
    if (d_dx != nullptr && a.n > 0) {
        const dim3 grid((unsigned)(a.n < 4096 ? a.n : 4096));
        if (d->dtype == GEAR_DTYPE_F32) hipLaunchKernelGGL(dx_kernel<float>, grid, dim3(kThreads), 0, s, a);
        else if (d->dtype == GEAR_DTYPE_BF16) hipLaunchKernelGGL(dx_kernel<__bf16>, grid, dim3(kThreads), 0, s, a);
        else hipLaunchKernelGGL(dx_kernel<_Float16>, grid, dim3(kThreads), 0, s, a);
        e = hipGetLastError();
        if (e != hipSuccess) return hip_fail(e, "gear_layer_norm_backward: row launch");
    }
    if (!params) return GEAR_OK;
    const dim3 grid((unsigned)((a.D + kThreads - 1) / kThreads), (unsigned)a.blocks);
    if (d->dtype == GEAR_DTYPE_F32) hipLaunchKernelGGL(columns_kernel<float>, grid, dim3(kThreads), 0, s, a);
    else if (d->dtype == GEAR_DTYPE_BF16) hipLaunchKernelGGL(columns_kernel<__bf16>, grid, dim3(kThreads), 0, s, a);
    else hipLaunchKernelGGL(columns_kernel<_Float16>, grid, dim3(kThreads), 0, s, a);
    e = hipGetLastError();
    if (e != hipSuccess) return hip_fail(e, "gear_layer_norm_backward: column launch");
    hipLaunchKernelGGL(finish_kernel, dim3(grid.x), dim3(kThreads), 0, s, a);
    e = hipGetLastError();
    return e == hipSuccess ? GEAR_OK : hip_fail(e, "gear_layer_norm_backward: sum launch");
}
