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

// Sum over groups of G neighbouring lanes, in each of them.
template <int CTRL>
__device__ __forceinline__ float from_lane(float v) {
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, 0xf, 0xf, false));
}
template <int G>
__device__ __forceinline__ float lanes_add(float v) {
    if (G >= 2) v += from_lane<0xB1>(v);    // quad_perm: the other of two
    if (G >= 4) v += from_lane<0x4E>(v);    // quad_perm: the other two of four
    if (G >= 8) v += from_lane<0x141>(v);   // row_half_mirror: the other four of eight
    if (G >= 16) v += from_lane<0x140>(v);  // row_mirror: the other eight of 16
    if (G >= 32) v += __shfl_xor(v, 16);
    if (G >= 64) v += __shfl_xor(v, 32);
    return v;
}
__device__ __forceinline__ float wave_add(float v) { return lanes_add<64>(v); }

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

// Rows of any length, an element a lane and load, read again for each pass: beyond 32768 values, which LDS no longer
// holds.  Memory, and the cache from the second pass on, bound it.
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

// --- rows held in registers -----------------------------------------------------

constexpr int kLaneValues = 16;  // of a row, in a lane's registers

// G lanes share a row (or a workgroup of G > 64 does), each with NV pieces of VE
// neighbouring values, piece k at (k G + lane) VE.  The row's last piece ends with the
// row, so that it is read as a whole too; what it has in common with the piece
// before, `skip` values, does not count in sums.
template <typename E>
struct Lane {
    static constexpr int VE = 16 / sizeof(E);
    typedef typename Vec<E, VE>::raw Raw;
    typedef Vec<E, VE> V;
};
template <typename E, int G, int NV>
struct Share {
    static constexpr int VE = Lane<E>::VE;
    int32_t at[NV], skip[NV];

    __device__ __forceinline__ Share(int lane, int64_t D) {
#pragma unroll
        for (int k = 0; k < NV; k++) {
            const int32_t col = (k * G + lane) * VE, last = (int32_t)D - VE;
            at[k] = col < last ? col : last;
            skip[k] = col - at[k] < VE ? col - at[k] : VE;
        }
    }
    // Whether the row reaches piece k of any lane; the same in all of them.
    static __device__ __forceinline__ bool reached(int k, int64_t D) { return k * G * VE < D; }
};
// f of every value of a piece that counts.
template <int VE, typename F>
__device__ __forceinline__ void counted(int skip, F f) {
    if (skip == 0) {
#pragma unroll
        for (int j = 0; j < VE; j++) f(j);
    } else {
#pragma unroll
        for (int j = 0; j < VE; j++)
            if (j >= skip) f(j);
    }
}

// Sums over the lanes of a row.  Workgroups' sums take the two places of `s` in
// turn, so that one barrier serves.
template <int G, int K>
__device__ __forceinline__ void row_add(float (&v)[K], float* s, int& turn) {
#pragma unroll
    for (int q = 0; q < K; q++) v[q] = lanes_add<(G < 64 ? G : 64)>(v[q]);
    if constexpr (G > 64) {
        constexpr int W = G / 64;
        float* p = s + turn * 2 * W;
        turn ^= 1;
        if ((threadIdx.x & 63) == 0) {
#pragma unroll
            for (int q = 0; q < K; q++) p[q * W + (threadIdx.x >> 6)] = v[q];
        }
        __syncthreads();
#pragma unroll
        for (int q = 0; q < K; q++) v[q] = lanes_add<W>(p[q * W + (threadIdx.x & (W - 1))]);
    }
}

template <int N>
__device__ __forceinline__ void params_at(const void* p, int32_t dtype, int64_t i, float none, float (&f)[N]) {
    if (p == nullptr) {
#pragma unroll
        for (int j = 0; j < N; j++) f[j] = none;
    } else if (dtype == GEAR_DTYPE_F32) {
        Vec<float, N>::unpack(Vec<float, N>::load(static_cast<const float*>(p) + i), f);
    } else if (dtype == GEAR_DTYPE_BF16) {
        Vec<__bf16, N>::unpack(Vec<__bf16, N>::load(static_cast<const __bf16*>(p) + i), f);
    } else {
        Vec<_Float16, N>::unpack(Vec<_Float16, N>::load(static_cast<const _Float16*>(p) + i), f);
    }
}
// Workgroups of 1024 have 128 registers a lane: they read the parameters again for
// each row, from the cache, through a pointer that hides that they are the same.
constexpr bool keeps(int threads) { return threads <= 256; }
__device__ __forceinline__ const void* hidden(const void* p) {
    asm volatile("" : "+s"(p));
    return p;
}

// One read and one write of each value; memory bounds it: 262144 rows of 512 bf16 with a residual, 1.07 GB, 196 us, 5.5 TB/s.
// Rows off a line are bound by latency too: 37000 of 1003 fp16, 148 MB, 32 us.  A row of 64 lanes' size in one
// launch for a single step: 64 rows of 1024, 3.6 us.
// Without a residual a row's values are on their way while the row before is worked on
// (37000 rows of 1003 fp16: 32 us, and 41 otherwise; with one, which reads twice as much, it
// gains nothing).  With STREAM rows pass by the caches.
template <typename E, int G, int NV, int THREADS, bool RES, bool STREAM>
__global__ __launch_bounds__(THREADS, THREADS <= 256 && RES && sizeof(E) == 4 ? 3 : 4) void forward_rows(const Args a) {
    constexpr int VE = Lane<E>::VE, R = THREADS / G;
    typedef typename Lane<E>::V V;
    typedef typename Lane<E>::Raw Raw;
    __shared__ float s[G > 64 ? 4 * G / 64 : 1];
    int turn = 0;
    const int lane = threadIdx.x % G;
    const Share<E, G, NV> at(lane, a.D);
    constexpr bool KEEP = keeps(THREADS), AHEAD = !RES;
    float w[NV][VE], b[NV][VE];
#pragma unroll
    for (int k = 0; k < NV; k++) {
        if (!KEEP || !at.reached(k, a.D)) continue;
        params_at<VE>(a.weight, a.param_dtype, at.at[k], 1.0f, w[k]);
        params_at<VE>(a.bias, a.param_dtype, at.at[k], 0.0f, b[k]);
    }
    const float per = 1.0f / (float)a.D;
    const auto fetch = [&](int64_t row, Raw (&raw)[NV], Raw (&res)[NV]) {
        const E* x = static_cast<const E*>(a.x) + row * a.x_row;
        const E* r = static_cast<const E*>(a.residual) + row * a.residual_row;
#pragma unroll
        for (int k = 0; k < NV; k++) {
            if (!at.reached(k, a.D)) continue;
            raw[k] = V::template load<STREAM>(x + at.at[k]);
            if (RES) res[k] = V::template load<STREAM>(r + at.at[k]);
        }
    };
    Raw next_raw[NV], next_res[NV];
    const int64_t first = (int64_t)blockIdx.x * R + threadIdx.x / G, stride = (int64_t)gridDim.x * R;
    if (AHEAD && first < a.n) fetch(first, next_raw, next_res);
    for (int64_t row = first; row < a.n; row += stride) {
        Raw raw[NV], res[NV];
        if (AHEAD) {
#pragma unroll
            for (int k = 0; k < NV; k++) {
                raw[k] = next_raw[k];
                if (RES) res[k] = next_res[k];
            }
            if (row + stride < a.n) fetch(row + stride, next_raw, next_res);
        } else {
            fetch(row, raw, res);
        }
        float t[NV][VE];
        float sum[1] = {0.0f};
#pragma unroll
        for (int k = 0; k < NV; k++) {
            if (!at.reached(k, a.D)) continue;
            V::unpack(raw[k], t[k]);
            if (RES) {
                float r[VE];
                V::unpack(res[k], r);
#pragma unroll
                for (int j = 0; j < VE; j++) t[k][j] += r[j];
                const Raw whole = V::round(t[k]);
                V::unpack(whole, t[k]);
                if (a.total && at.skip[k] < VE) V::template store<STREAM>(static_cast<E*>(a.total) + row * a.D + at.at[k], t[k]);
            }
            counted<VE>(at.skip[k], [&](int j) { sum[0] += t[k][j]; });
        }
        row_add<G>(sum, s, turn);
        const float c = sum[0] * per;
        float v[2] = {0.0f, 0.0f};
#pragma unroll
        for (int k = 0; k < NV; k++) {
            if (!at.reached(k, a.D)) continue;
#pragma unroll
            for (int j = 0; j < VE; j++) t[k][j] -= c;
            counted<VE>(at.skip[k], [&](int j) {
                v[0] += t[k][j];
                v[1] = fmaf(t[k][j], t[k][j], v[1]);
            });
        }
        row_add<G>(v, s, turn);
        const float off = v[0] * per;
        const float var = fmaxf(fmaf(-off, off, v[1] * per), 0.0f);
        const float rstd = v[1] == v[1] ? 1.0f / sqrtf(var + a.eps) : v[1];
#pragma unroll
        for (int k = 0; k < NV; k++) {
            if (!at.reached(k, a.D)) continue;
            float y[VE], wk[VE], bk[VE];
            if (!KEEP) {
                params_at<VE>(hidden(a.weight), a.param_dtype, at.at[k], 1.0f, wk);
                params_at<VE>(hidden(a.bias), a.param_dtype, at.at[k], 0.0f, bk);
            }
#pragma unroll
            for (int j = 0; j < VE; j++) y[j] = fmaf((t[k][j] - off) * rstd, KEEP ? w[k][j] : wk[j], KEEP ? b[k][j] : bk[j]);
            if (at.skip[k] < VE) V::template store<STREAM>(static_cast<E*>(a.y) + row * a.D + at.at[k], y);
        }
        if (a.saved && lane == 0) {
            a.saved[2 * row] = c + off;
            a.saved[2 * row + 1] = rstd;
        }
    }
}

// Longer rows lie in LDS between the passes, each lane's pieces its own; CAP values of a
// row, 20352 where two workgroups share a unit: 1024 rows of 20000 fp32 and a residual 68 us,
// 76 with the row in registers and one workgroup a unit.
template <typename E, int CAP, bool RES>
__global__ __launch_bounds__(1024, CAP > 20352 ? 4 : 8) void forward_long(const Args a) {
    constexpr int VE = Lane<E>::VE, T = 1024, STEP = 2, NV = (CAP + T * VE - 1) / (T * VE);
    typedef typename Lane<E>::V V;
    typedef typename Lane<E>::Raw Raw;
    typedef float Values __attribute__((ext_vector_type(4)));
    __shared__ Values held[(CAP + VE - 1) / VE][VE / 4];
    __shared__ float s[4 * T / 64];
    int turn = 0;
    const float per = 1.0f / (float)a.D;
    const int32_t last = (int32_t)a.D - VE;
    for (int64_t row = blockIdx.x; row < a.n; row += gridDim.x) {
        const E* x = static_cast<const E*>(a.x) + row * a.x_row;
        const E* r = static_cast<const E*>(a.residual) + row * a.residual_row;
        float sum[1] = {0.0f};
#pragma unroll 1
        for (int k0 = 0; k0 < NV; k0 += STEP) {
            Raw raw[STEP], res[STEP];
#pragma unroll
            for (int k = 0; k < STEP; k++) {
                const int32_t col = ((k0 + k) * T + (int32_t)threadIdx.x) * VE, at = col < last ? col : last;
                if (col >= a.D) continue;
                raw[k] = V::load(x + at);
                if (RES) res[k] = V::load(r + at);
            }
#pragma unroll
            for (int k = 0; k < STEP; k++) {
                const int32_t p = (k0 + k) * T + (int32_t)threadIdx.x, col = p * VE, at = col < last ? col : last;
                if (col >= a.D) continue;
                float t[VE];
                V::unpack(raw[k], t);
                if (RES) {
                    float q[VE];
                    V::unpack(res[k], q);
#pragma unroll
                    for (int j = 0; j < VE; j++) t[j] += q[j];
                    const Raw whole = V::round(t);
                    V::unpack(whole, t);
                    if (a.total) V::store(static_cast<E*>(a.total) + row * a.D + at, t);
                }
                counted<VE>(col - at, [&](int j) { sum[0] += t[j]; });
#pragma unroll
                for (int j = 0; j < VE; j += 4) held[p][j / 4] = Values{t[j], t[j + 1], t[j + 2], t[j + 3]};
            }
        }
        row_add<T>(sum, s, turn);
        const float c = sum[0] * per;
        float v[2] = {0.0f, 0.0f};
#pragma unroll 2
        for (int32_t p = threadIdx.x; p * VE < a.D; p += T) {
            const int32_t col = p * VE, at = col < last ? col : last;
#pragma unroll
            for (int j = 0; j < VE; j += 4) {
                const Values t = held[p][j / 4] - c;
#pragma unroll
                for (int i = 0; i < 4; i++) {
                    if (j + i < col - at) continue;
                    v[0] += t[i];
                    v[1] = fmaf(t[i], t[i], v[1]);
                }
            }
        }
        row_add<T>(v, s, turn);
        const float off = v[0] * per;
        const float var = fmaxf(fmaf(-off, off, v[1] * per), 0.0f);
        const float rstd = v[1] == v[1] ? 1.0f / sqrtf(var + a.eps) : v[1];
#pragma unroll 2
        for (int32_t p = threadIdx.x; p * VE < a.D; p += T) {
            const int32_t col = p * VE, at = col < last ? col : last;
            float y[VE], w[VE], b[VE];
            params_at<VE>(a.weight, a.param_dtype, at, 1.0f, w);
            params_at<VE>(a.bias, a.param_dtype, at, 0.0f, b);
#pragma unroll
            for (int j = 0; j < VE; j++) y[j] = fmaf((held[p][j / 4][j % 4] - c - off) * rstd, w[j], b[j]);
            V::store(static_cast<E*>(a.y) + row * a.D + at, y);
        }
        if (a.saved && threadIdx.x == 0) {
            a.saved[2 * row] = c + off;
            a.saved[2 * row + 1] = rstd;
        }
    }
}

// dx of rows, and with PARAMS what a workgroup's rows add to dweight and dbias, in registers over all its rows.
// Memory bounds it: 262144 rows of 512 bf16, 1.08 GB, 197 us, 5.5 TB/s; 37000 of 1003 fp16, 225 MB, 47 us (latency, and
// rows off a line); the next row's loads on their way did not help here (59 us: registers).
template <typename E, int G, int NV, int THREADS, bool PARAMS, bool STREAM>
__global__ __launch_bounds__(THREADS, THREADS > 256 ? 4 : 3) void backward_rows(const Args a) {
    constexpr int VE = Lane<E>::VE, R = THREADS / G;
    typedef typename Lane<E>::V V;
    typedef typename Lane<E>::Raw Raw;
    __shared__ float s[G > 64 ? 4 * G / 64 : 1];
    int turn = 0;
    const int lane = threadIdx.x % G;
    const Share<E, G, NV> at(lane, a.D);
    // LATE: dtotal waits for registers.
    constexpr bool KEEP = keeps(THREADS), LATE = NV * VE > kLaneValues;
    float w[NV][VE], dw[NV][VE], db[NV][VE];
#pragma unroll
    for (int k = 0; k < NV; k++) {
        if (KEEP && at.reached(k, a.D)) params_at<VE>(a.weight, a.param_dtype, at.at[k], 1.0f, w[k]);
#pragma unroll
        for (int j = 0; j < VE; j++) dw[k][j] = db[k][j] = 0.0f;
    }
    const float per = 1.0f / (float)a.D;
    for (int64_t row = (int64_t)blockIdx.x * R + threadIdx.x / G; row < a.n; row += (int64_t)gridDim.x * R) {
        const E* t = static_cast<const E*>(a.x) + row * a.x_row;
        const E* dy = static_cast<const E*>(a.dy) + row * a.dy_row;
        const float mean = a.saved[2 * row], rstd = a.saved[2 * row + 1];
        Raw rt[NV], rd[NV], rs[NV];
#pragma unroll
        for (int k = 0; k < NV; k++) {
            if (!at.reached(k, a.D)) continue;
            rt[k] = V::template load<STREAM>(t + at.at[k]);
            rd[k] = V::template load<STREAM>(dy + at.at[k]);
            if (!LATE && a.dtotal) rs[k] = V::template load<STREAM>(static_cast<const E*>(a.dtotal) + row * a.dtotal_row + at.at[k]);
        }
        float v[2] = {0.0f, 0.0f};
#pragma unroll
        for (int k = 0; k < NV; k++) {
            if (!at.reached(k, a.D)) continue;
            float u[VE], d[VE], wk[VE];
            V::unpack(rt[k], u);
            V::unpack(rd[k], d);
            if (!KEEP) params_at<VE>(hidden(a.weight), a.param_dtype, at.at[k], 1.0f, wk);
            counted<VE>(at.skip[k], [&](int j) {
                const float x = (u[j] - mean) * rstd, g = d[j] * (KEEP ? w[k][j] : wk[j]);
                v[0] += g;
                v[1] = fmaf(g, x, v[1]);
                if (PARAMS) {
                    dw[k][j] = fmaf(d[j], x, dw[k][j]);
                    db[k][j] += d[j];
                }
            });
        }
        row_add<G>(v, s, turn);
        const float g0 = v[0] * per, gu = v[1] * per;
        if (a.dx) {
#pragma unroll
            for (int k = 0; k < NV; k++) {
                if (!at.reached(k, a.D)) continue;
                float u[VE], d[VE], o[VE], wk[VE];
                V::unpack(rt[k], u);
                V::unpack(rd[k], d);
                if (!KEEP) params_at<VE>(hidden(a.weight), a.param_dtype, at.at[k], 1.0f, wk);
#pragma unroll
                for (int j = 0; j < VE; j++)
                    o[j] = (d[j] * (KEEP ? w[k][j] : wk[j]) - g0 - (u[j] - mean) * rstd * gu) * rstd;
                if (a.dtotal) {
                    if (LATE) rs[k] = V::template load<STREAM>(static_cast<const E*>(a.dtotal) + row * a.dtotal_row + at.at[k]);
                    V::unpack(rs[k], u);
#pragma unroll
                    for (int j = 0; j < VE; j++) o[j] += u[j];
                }
                if (at.skip[k] < VE) V::template store<STREAM>(static_cast<E*>(a.dx) + row * a.D + at.at[k], o);
            }
        }
    }
    if constexpr (PARAMS) {
        // Rows of the same wave, then of the workgroup's waves.
        constexpr int W = G > 64 ? 1 : THREADS / 64, N = (G < 64 ? G : 64) * VE;
        __shared__ float part[W > 1 ? W * N : 1];
        float* out = a.work + 2 * (int64_t)blockIdx.x * a.D;
#pragma unroll
        for (int q = 0; q < 2; q++) {
#pragma unroll
            for (int k = 0; k < NV; k++) {
                if (!at.reached(k, a.D)) continue;
                float v[VE];
#pragma unroll
                for (int j = 0; j < VE; j++) {
                    v[j] = q == 0 ? dw[k][j] : db[k][j];
#pragma unroll
                    for (int off = G; off < 64; off <<= 1) v[j] += __shfl_xor(v[j], off);
                }
                if constexpr (W == 1) {
#pragma unroll
                    for (int j = 0; j < VE; j++)
                        if (j >= at.skip[k]) out[q * a.D + at.at[k] + j] = v[j];
                } else {
                    __syncthreads();
                    if ((threadIdx.x & 63) < G) {
#pragma unroll
                        for (int j = 0; j < VE; j++) part[(threadIdx.x >> 6) * N + lane * VE + j] = v[j];
                    }
                    __syncthreads();
                    if (threadIdx.x < G) {
#pragma unroll
                        for (int j = 0; j < VE; j++) {
                            float sum = 0.0f;
#pragma unroll
                            for (int i = 0; i < W; i++) sum += part[i * N + lane * VE + j];
                            if (j >= at.skip[k]) out[q * a.D + at.at[k] + j] = sum;
                        }
                    }
                }
            }
        }
    }
}

// --- rows shorter than a piece ----------------------------------------------------

// A lane takes a row; a row is shorter than a 16-byte load.
template <typename E, bool RES>
__global__ __launch_bounds__(kThreads) void forward_tiny(const Args a) {
    constexpr int VE = Lane<E>::VE;
    const float per = 1.0f / (float)a.D;
    const int D = (int)a.D;
    for (int64_t row = (int64_t)blockIdx.x * kThreads + threadIdx.x; row < a.n; row += (int64_t)gridDim.x * kThreads) {
        float t[VE], c = 0.0f, off = 0.0f, sq = 0.0f;
#pragma unroll
        for (int j = 0; j < VE; j++) {
            t[j] = 0.0f;
            if (j >= D) continue;
            t[j] = (float)(static_cast<const E*>(a.x) + row * a.x_row)[j];
            if (RES) {
                const E whole = (E)(t[j] + (float)(static_cast<const E*>(a.residual) + row * a.residual_row)[j]);
                if (a.total) (static_cast<E*>(a.total) + row * D)[j] = whole;
                t[j] = (float)whole;
            }
            c += t[j];
        }
        c *= per;
#pragma unroll
        for (int j = 0; j < VE; j++) {
            if (j >= D) continue;
            t[j] -= c;
            off += t[j];
            sq = fmaf(t[j], t[j], sq);
        }
        off *= per;
        const float var = fmaxf(fmaf(-off, off, sq * per), 0.0f);
        const float rstd = sq == sq ? 1.0f / sqrtf(var + a.eps) : sq;
#pragma unroll
        for (int j = 0; j < VE; j++) {
            if (j >= D) continue;
            (static_cast<E*>(a.y) + row * D)[j] = (E)fmaf((t[j] - off) * rstd, param_at(a.weight, a.param_dtype, j, 1.0f),
                                                          param_at(a.bias, a.param_dtype, j, 0.0f));
        }
        if (a.saved) {
            a.saved[2 * row] = c + off;
            a.saved[2 * row + 1] = rstd;
        }
    }
}
template <typename E, bool PARAMS>
__global__ __launch_bounds__(kThreads) void backward_tiny(const Args a) {
    constexpr int VE = Lane<E>::VE;
    __shared__ float s[kThreads / 64][2 * VE];
    const float per = 1.0f / (float)a.D;
    const int D = (int)a.D;
    float dw[VE], db[VE];
#pragma unroll
    for (int j = 0; j < VE; j++) dw[j] = db[j] = 0.0f;
    for (int64_t row = (int64_t)blockIdx.x * kThreads + threadIdx.x; row < a.n; row += (int64_t)gridDim.x * kThreads) {
        const float mean = a.saved[2 * row], rstd = a.saved[2 * row + 1];
        float u[VE], g[VE], g0 = 0.0f, gu = 0.0f;
#pragma unroll
        for (int j = 0; j < VE; j++) {
            u[j] = g[j] = 0.0f;
            if (j >= D) continue;
            u[j] = ((float)(static_cast<const E*>(a.x) + row * a.x_row)[j] - mean) * rstd;
            const float dy = (float)(static_cast<const E*>(a.dy) + row * a.dy_row)[j];
            g[j] = dy * param_at(a.weight, a.param_dtype, j, 1.0f);
            g0 += g[j];
            gu = fmaf(g[j], u[j], gu);
            if (PARAMS) {
                dw[j] = fmaf(dy, u[j], dw[j]);
                db[j] += dy;
            }
        }
        g0 *= per;
        gu *= per;
        if (a.dx == nullptr) continue;
#pragma unroll
        for (int j = 0; j < VE; j++) {
            if (j >= D) continue;
            float o = (g[j] - g0 - u[j] * gu) * rstd;
            if (a.dtotal) o += (float)(static_cast<const E*>(a.dtotal) + row * a.dtotal_row)[j];
            (static_cast<E*>(a.dx) + row * D)[j] = (E)o;
        }
    }
    if constexpr (PARAMS) {
#pragma unroll
        for (int j = 0; j < VE; j++) {
            dw[j] = wave_add(dw[j]);
            db[j] = wave_add(db[j]);
        }
        if ((threadIdx.x & 63) == 0) {
#pragma unroll
            for (int j = 0; j < VE; j++) {
                s[threadIdx.x >> 6][j] = dw[j];
                s[threadIdx.x >> 6][VE + j] = db[j];
            }
        }
        __syncthreads();
        const int q = threadIdx.x / VE, j = threadIdx.x % VE;
        if (q < 2 && j < D) {
            float v = 0.0f;
#pragma unroll
            for (int i = 0; i < kThreads / 64; i++) v += s[i][q * VE + j];
            a.work[(2 * (int64_t)blockIdx.x + q) * D + j] = v;
        }
    }
}

// --- sums over rows ---------------------------------------------------------------

// A slice blockIdx.y of the rows, a piece of columns a lane, for rows too long to keep two sums a value in registers.
// Reads both inputs again, partly from the last-level cache: 1024 rows of 20000 fp32, 164 MB, 28 us.
template <typename E>
__global__ __launch_bounds__(kThreads) void columns_kernel(const Args a) {
    constexpr int VE = Lane<E>::VE;
    typedef typename Lane<E>::V V;
    const int64_t col = ((int64_t)blockIdx.x * kThreads + threadIdx.x) * VE, last = a.D - VE;
    if (col >= a.D) return;
    const int64_t at = col < last ? col : last;
    const int64_t first = a.n * blockIdx.y / a.blocks, end = a.n * (blockIdx.y + 1) / a.blocks;
    float dw[VE], db[VE];
#pragma unroll
    for (int j = 0; j < VE; j++) dw[j] = db[j] = 0.0f;
#pragma unroll 4
    for (int64_t row = first; row < end; row++) {
        float t[VE], dy[VE];
        V::unpack(V::load(static_cast<const E*>(a.x) + row * a.x_row + at), t);
        V::unpack(V::load(static_cast<const E*>(a.dy) + row * a.dy_row + at), dy);
        const float mean = a.saved[2 * row], rstd = a.saved[2 * row + 1];
#pragma unroll
        for (int j = 0; j < VE; j++) {
            dw[j] = fmaf(dy[j], (t[j] - mean) * rstd, dw[j]);
            db[j] += dy[j];
        }
    }
    // The last piece's first values are the piece before's too: the same sums twice.
    Vec<float, VE>::store(a.work + 2 * (int64_t)blockIdx.y * a.D + at, dw);
    Vec<float, VE>::store(a.work + (2 * (int64_t)blockIdx.y + 1) * a.D + at, db);
}

// Adds the workgroups' sums: 64 columns a workgroup, of dweight or of dbias, a wave for every 16th.  7 to 8 us, a launch
// and a chain of loads.  One workgroup that leaves the sums itself saves this launch, but takes 3 us for each round of rows:
// no gain from two rounds on.
constexpr int kFinishThreads = 1024;
__global__ __launch_bounds__(kFinishThreads) void finish_kernel(const Args a) {
    constexpr int W = kFinishThreads / 64;
    __shared__ float s[W][64];
    const int64_t j = (int64_t)blockIdx.x * 64 + (threadIdx.x & 63);
    const int q = blockIdx.y;
    void* out = q == 0 ? a.dweight : a.dbias;
    if (out == nullptr) return;
    float v = 0.0f;
    if (j < a.D) {
#pragma unroll 8
        for (int k = threadIdx.x >> 6; k < a.blocks; k += W) v += a.work[(2 * (int64_t)k + q) * a.D + j];
    }
    s[threadIdx.x >> 6][threadIdx.x & 63] = v;
    __syncthreads();
    if (threadIdx.x < 64 && j < a.D) {
        v = 0.0f;
#pragma unroll
        for (int k = 0; k < W; k++) v += s[k][threadIdx.x];
        param_put(out, a.param_dtype, j, v);
    }
}

typedef void (*Kernel)(const Args);
struct Choice {
    Kernel kernel;
    int threads, rows;  // rows that a workgroup runs at a time
    int blocks;         // workgroups that the GPU runs at a time
};
constexpr int kCUs = 256;

template <typename E, int G, int NV, bool RES, bool STREAM = false>
Choice forward_of() {
    constexpr int T = G > 256 ? G : 256;
    return {forward_rows<E, G, NV, T, RES, STREAM>, T, T / G, kCUs * 1024 / T};
}
template <typename E, bool RES>
Choice forward_choice(int64_t D, bool stream) {
    constexpr int VE = Lane<E>::VE, NV = kLaneValues / VE;
    if (D < VE) return {forward_tiny<E, RES>, kThreads, kThreads, kCUs * 8};
    if (D > 32768) return {forward_kernel<E>, kThreads, 1, 4096};
    if (D <= 4 * kLaneValues) return forward_of<E, 4, NV, RES>();
    if (D <= 16 * kLaneValues) return forward_of<E, 16, NV, RES>();
    if (D <= 32 * kLaneValues) return stream ? forward_of<E, 32, NV, RES, true>() : forward_of<E, 32, NV, RES>();
    if (D <= 64 * kLaneValues) return stream ? forward_of<E, 64, NV, RES, true>() : forward_of<E, 64, NV, RES>();
    if (D <= 256 * kLaneValues) return stream ? forward_of<E, 256, NV, RES, true>() : forward_of<E, 256, NV, RES>();
    if (D <= 1024 * kLaneValues) return forward_of<E, 1024, NV, RES>();
    if (D <= 20352) return {forward_long<E, 20352, RES>, 1024, 1, kCUs * 2};
    return {forward_long<E, 32768, RES>, 1024, 1, kCUs};
}
template <typename E, int G, int NV, bool PARAMS, bool STREAM = false>
Choice backward_of() {
    constexpr int T = G > 256 ? G : 256;
    return {backward_rows<E, G, NV, T, PARAMS, STREAM>, T, T / G, kCUs * 1024 / T};
}
// Rows beyond kSumsD have their sums over rows in a launch of their own.
constexpr int64_t kSumsD = 16384;
template <typename E, bool PARAMS>
Choice backward_choice(int64_t D, bool stream) {
    constexpr int VE = Lane<E>::VE, NV = kLaneValues / VE;
    if (D < VE) return {backward_tiny<E, PARAMS>, kThreads, kThreads, kCUs * 4};
    if (D > 32768) return {dx_kernel<E>, kThreads, 1, 4096};
    if (D <= 4 * kLaneValues) return backward_of<E, 4, NV, PARAMS>();
    if (D <= 16 * kLaneValues) return backward_of<E, 16, NV, PARAMS>();
    if (D <= 32 * kLaneValues) return stream ? backward_of<E, 32, NV, PARAMS, true>() : backward_of<E, 32, NV, PARAMS>();
    if (D <= 64 * kLaneValues) return stream ? backward_of<E, 64, NV, PARAMS, true>() : backward_of<E, 64, NV, PARAMS>();
    if (D <= 256 * kLaneValues) return stream ? backward_of<E, 256, NV, PARAMS, true>() : backward_of<E, 256, NV, PARAMS>();
    if (D <= 1024 * kLaneValues) return backward_of<E, 1024, NV, PARAMS>();
    if constexpr (!PARAMS) return backward_of<E, 1024, 2 * NV, false>();
    return {};
}

constexpr int64_t kMaxValues = 1ll << 40, kMaxD = 1 << 20;
// Rows of whole lines that no cache holds pass by it: 262144 rows of 512 bf16, forward
// and backward, 393 us, and 425 through the caches; rows off a line gain nothing (37000
// of 1003: 94 and 92).
bool streams(int32_t dtype, int64_t n, int64_t D) {
    const int64_t row = D * float_bytes(dtype);
    return row % 128 == 0 && n * row >= (128ll << 20);
}
template <bool RES>
Choice forward_by_type(int32_t dtype, int64_t n, int64_t D) {
    const bool stream = streams(dtype, n, D);
    return dtype == GEAR_DTYPE_F32 ? forward_choice<float, RES>(D, stream)
           : dtype == GEAR_DTYPE_BF16 ? forward_choice<__bf16, RES>(D, stream) : forward_choice<_Float16, RES>(D, stream);
}
template <bool PARAMS>
Choice backward_by_type(int32_t dtype, int64_t n, int64_t D) {
    const bool stream = streams(dtype, n, D);
    return dtype == GEAR_DTYPE_F32 ? backward_choice<float, PARAMS>(D, stream)
           : dtype == GEAR_DTYPE_BF16 ? backward_choice<__bf16, PARAMS>(D, stream) : backward_choice<_Float16, PARAMS>(D, stream);
}
int grid_of(const Choice& c, int64_t n) {
    const int64_t want = (n + c.rows - 1) / c.rows;
    return (int)(want < c.blocks ? want : c.blocks);
}

// Workgroups, or slices of rows, that leave sums.  Each leaves 2 D of them, so it
// should have some rows to add: 8 at a time per row it holds, where that leaves a workgroup for every unit.
int sums_of(const gear_norm_desc& d) {
    if (d.n == 0) return 0;
    if (d.D > kSumsD) {
        const int64_t across = (d.D + 4 * kThreads - 1) / (4 * kThreads);
        int64_t slices = 2048 / across < 1 ? 1 : 2048 / across;
        if (slices > (d.n + 7) / 8) slices = (d.n + 7) / 8;
        return (int)slices;
    }
    const Choice c = backward_by_type<true>(d.dtype, d.n, d.D);
    const int64_t most = grid_of(c, d.n), few = most < kCUs ? most : kCUs;
    const int64_t want = (d.n + 8 * c.rows - 1) / (8 * c.rows);
    return (int)(want < few ? few : want < most ? want : most);
}
int64_t work_bytes_of(const gear_norm_desc& d) { return (2 * sums_of(d) * d.D + 1) * (int64_t)sizeof(float); }

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
    const Choice c = d_residual ? forward_by_type<true>(d->dtype, a.n, a.D) : forward_by_type<false>(d->dtype, a.n, a.D);
    hipLaunchKernelGGL(c.kernel, dim3(grid_of(c, a.n)), dim3(c.threads), 0, static_cast<hipStream_t>(stream), a);
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
    a.blocks = params ? sums_of(*d) : 0;
    (void)hipGetLastError();  // an error pending from an earlier HIP call is not this call's
    hipStream_t s = static_cast<hipStream_t>(stream);
    hipError_t e = hipSuccess;
    const bool apart = a.D > kSumsD;  // the sums over rows have a launch of their own
    if (a.n > 0 && (d_dx != nullptr || (params && !apart))) {
        const Choice c = params && !apart ? backward_by_type<true>(d->dtype, a.n, a.D) : backward_by_type<false>(d->dtype, a.n, a.D);
        hipLaunchKernelGGL(c.kernel, dim3(params && !apart ? a.blocks : grid_of(c, a.n)), dim3(c.threads), 0, s, a);
        e = hipGetLastError();
        if (e != hipSuccess) return hip_fail(e, "gear_layer_norm_backward: row launch");
    }
    if (!params) return GEAR_OK;
    if (a.n > 0 && apart) {
        const int64_t per = (int64_t)kThreads * 16 / float_bytes(d->dtype);
        const dim3 grid((unsigned)((a.D + per - 1) / per), (unsigned)a.blocks);
        if (d->dtype == GEAR_DTYPE_F32) hipLaunchKernelGGL(columns_kernel<float>, grid, dim3(kThreads), 0, s, a);
        else if (d->dtype == GEAR_DTYPE_BF16) hipLaunchKernelGGL(columns_kernel<__bf16>, grid, dim3(kThreads), 0, s, a);
        else hipLaunchKernelGGL(columns_kernel<_Float16>, grid, dim3(kThreads), 0, s, a);
        e = hipGetLastError();
        if (e != hipSuccess) return hip_fail(e, "gear_layer_norm_backward: column launch");
    }
    hipLaunchKernelGGL(finish_kernel, dim3((unsigned)((a.D + 63) / 64), 2), dim3(kFinishThreads), 0, s, a);
    e = hipGetLastError();
    return e == hipSuccess ? GEAR_OK : hip_fail(e, "gear_layer_norm_backward: sum launch");
}
