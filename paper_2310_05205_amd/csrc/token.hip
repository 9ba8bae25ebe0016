// The loss of a token head and its gradients, without the logits
// (include/gear.h).  With z = h W^T, lse = log sum_v exp z_v, y the target:
//   logp = z_y - lse,  e_v = exp(z_v - lse) - [v = y],
//   dh = c sum_v e_v W_v,  dW_v = sum_rows c e_v h,  c the row's share of the loss.
//
// Every product is C[j][i] = sum_k X[i][k] Y[j][k] of two operands whose k lie next
// to each other, so one tile loop serves all:
//   logits   X = W,           Y = h,             k = D   (i tokens, j rows)
//   dW       X = h^T,         Y = (c e)^T,       k = n   (i of D,   j tokens)
//   dh       X = W^T,         Y = e,             k = V   (i of D,   j rows)
// The transposed operands are copies that this call makes, and e is written in both
// orders, a piece of the vocabulary at a time.  The copies pad k to whole steps with
// zeros, so odd sizes and alignments end there.
//
// 32-bit values are cut into three bf16 parts a = a1 + a2 + a3 (8 bits each); the six
// products a1 b1, a1 b2, a2 b1, a2 b2, a1 b3, a3 b1 leave an error of 2^-25 of |a b|,
// and matrix instructions of 16-bit types are 16 times as fast as those of 32.
#include <math.h>

#include <type_traits>

#include "element.h"
#include "gear_internal.h"

namespace gear {
namespace {

constexpr int kStep = 64;                 // k of one step: 128 bytes a row
constexpr int kThreads = 256;
constexpr int64_t kPieceValues = 1 << 27;  // values of e formed at a time, at most
constexpr int64_t kPieceTokens = 1 << 16;
constexpr int kParts = 512;               // workgroups that look at the rows

typedef __bf16 B8 __attribute__((ext_vector_type(8)));
typedef _Float16 H8 __attribute__((ext_vector_type(8)));
typedef float F4 __attribute__((ext_vector_type(4)));

template <typename T>
struct Matrix;
template <>
struct Matrix<__bf16> {
    typedef B8 V8;
    // e lies in [-1, 1]; bf16 reaches far below what counts.
    static constexpr float kScale = 1.0f;
    static __device__ __forceinline__ F4 mfma(V8 x, V8 y, F4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, y, c, 0, 0, 0); }
};
template <>
struct Matrix<_Float16> {
    typedef H8 V8;
    // fp16 ends at 65504, and its precision at 2^-14: e is held times 2^14, so that it is
    // rounded like any fp16 value down to 2^-28.
    static constexpr float kScale = 16384.0f;
    static __device__ __forceinline__ F4 mfma(V8 x, V8 y, F4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(x, y, c, 0, 0, 0); }
};

// Type of the products, and parts of a value, for elements E.
template <typename E>
struct Parts {
    typedef E T;
    static constexpr int kCount = 1;
};
template <>
struct Parts<float> {
    typedef __bf16 T;
    static constexpr int kCount = 3;
};
// The products of parts (first, second) that a step of k goes through.
constexpr int kPairs[6][2] = {{0, 0}, {0, 1}, {1, 0}, {1, 1}, {0, 2}, {2, 0}};

// An operand: `rows` rows of `k` values at stride ld; 32-bit operands have their parts `part` apart.
struct Operand {
    const void* p;
    int64_t rows, ld, part;
};

// What a row adds: its target, or -1 where it takes no part, and its weight.
struct Row {
    int32_t target;
    float weight;
};
// Of all rows; made by one workgroup.
struct Totals {
    float share;     // 1 / denom
    float weight;    // largest |weight| of a row that takes part
};

struct Args {
    const void* target;
    const uint8_t* mask;
    const float *weight, *grad_loss, *lse_in;
    float *loss, *logp, *lse;
    Row* rows;
    Totals* totals;
    double* sums;      // [kParts]
    int64_t* counts;   // [kParts]
    float* tops;       // [kParts]
    float* part_max;   // [tiles of tokens][n]
    float* part_sum;
    float* at_target;  // [n]: the target's logit
    int64_t n, D, V, mask_group, weight_group;
    int32_t target_dtype, tiles, parts;
    float denom, grad_scale;
};

// --- rows ---------------------------------------------------------------------

template <typename T>
__device__ __forceinline__ T wave_add(T v) {
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) v += __shfl_xor(v, off);
    return v;
}
// Targets and weights of the rows, how many take part, and their largest weight.
__global__ __launch_bounds__(kThreads) void rows_kernel(const Args a) {
    __shared__ int64_t s_count[kThreads / 64];
    __shared__ float s_top[kThreads / 64];
    int64_t count = 0;
    float top = 0.0f;
    for (int64_t r = (int64_t)blockIdx.x * kThreads + threadIdx.x; r < a.n; r += (int64_t)gridDim.x * kThreads) {
        const int64_t y = a.target_dtype == GEAR_DTYPE_I32   ? (int64_t)static_cast<const int32_t*>(a.target)[r]
                          : a.target_dtype == GEAR_DTYPE_I64 ? static_cast<const int64_t*>(a.target)[r]
                                                             : (int64_t)static_cast<const uint8_t*>(a.target)[r];
        const bool on = y >= 0 && y < a.V && (a.mask == nullptr || a.mask[r / a.mask_group] != 0);
        const float w = !on ? 0.0f : a.weight ? a.weight[r / a.weight_group] : 1.0f;
        a.rows[r] = Row{on ? (int32_t)y : -1, w};
        count += on ? 1 : 0;
        // A NaN or an infinity has to stay: it makes every gradient of the head one.
        if (on && !(fabsf(w) <= top)) top = fabsf(w);
    }
    count = wave_add(count);
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) {
        const float o = __shfl_xor(top, off);
        if (!(o <= top)) top = o;
    }
    if ((threadIdx.x & 63) == 0) {
        s_count[threadIdx.x >> 6] = count;
        s_top[threadIdx.x >> 6] = top;
    }
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int k = 1; k < kThreads / 64; k++) {
            count += s_count[k];
            if (!(s_top[k] <= top)) top = s_top[k];
        }
        a.counts[blockIdx.x] = count;
        a.tops[blockIdx.x] = top;
    }
}
__global__ __launch_bounds__(64) void totals_kernel(const Args a) {
    int64_t count = 0;
    float top = 0.0f;
    for (int k = threadIdx.x; k < a.parts; k += 64) {
        count += a.counts[k];
        if (!(a.tops[k] <= top)) top = a.tops[k];
    }
    count = wave_add(count);
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) {
        const float o = __shfl_xor(top, off);
        if (!(o <= top)) top = o;
    }
    if (threadIdx.x == 0) {
        a.totals->share = 1.0f / (a.denom > 0.0f ? a.denom : count > 0 ? (float)count : 1.0f);
        a.totals->weight = top;
    }
}

// Joins the tiles' maxima and sums: lse, logp, and a sum of the losses per workgroup.
__global__ __launch_bounds__(kThreads) void lse_kernel(const Args a) {
    __shared__ double s[kThreads / 64];
    double sum = 0.0;
    for (int64_t r = (int64_t)blockIdx.x * kThreads + threadIdx.x; r < a.n; r += (int64_t)gridDim.x * kThreads) {
        float m = -INFINITY;
        for (int t = 0; t < a.tiles; t++) m = fmaxf(m, a.part_max[t * a.n + r]);
        const float from = m == -INFINITY ? 0.0f : m;
        float S = 0.0f;
        for (int t = 0; t < a.tiles; t++) S += a.part_sum[t * a.n + r] * fast_exp(a.part_max[t * a.n + r] - from);
        const float lse = from + __builtin_amdgcn_logf(S) * kLn2;
        const Row row = a.rows[r];
        const bool on = row.target >= 0;
        const float lp = on ? (a.at_target[r] - from) - __builtin_amdgcn_logf(S) * kLn2 : 0.0f;
        if (a.logp) a.logp[r] = lp;
        if (a.lse) a.lse[r] = on ? lse : 0.0f;
        // A weight of 0 leaves 0 of an infinite term.
        if (on && !(row.weight == 0.0f && lp == -INFINITY)) sum -= (double)row.weight * (double)lp;
    }
    sum = wave_add(sum);
    if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = sum;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int k = 1; k < kThreads / 64; k++) sum += s[k];
        a.sums[blockIdx.x] = sum;
    }
}
__global__ __launch_bounds__(64) void loss_kernel(const Args a) {
    double sum = 0.0;
    for (int k = threadIdx.x; k < a.parts; k += 64) sum += a.sums[k];
    sum = wave_add(sum);
    if (threadIdx.x == 0) *a.loss = (float)(sum * (double)a.totals->share);
}

// --- operands -----------------------------------------------------------------

// A value's parts.  Each is the rest so far, rounded; one that rounds to an infinity is cut instead.
template <typename T, int N>
__device__ __forceinline__ void cut(float v, T (&part)[N]) {
    if (N == 1) {
        part[0] = (T)v;
        return;
    }
#pragma unroll
    for (int k = 0; k < N; k++) {
        T h = (T)v;
        if (!(fabsf((float)h) < INFINITY) && fabsf(v) < INFINITY) h = __builtin_bit_cast(T, (uint16_t)(__builtin_bit_cast(uint32_t, v) >> 16));
        part[k] = h;
        v = fabsf(v) < INFINITY ? v - (float)h : 0.0f;
    }
}

// Rows copied to rows of whole steps, zeros behind their end.
template <typename E>
__global__ __launch_bounds__(kThreads) void copy_kernel(const E* src, int64_t rows, int64_t cols, int64_t ld_src,
                                                        typename Parts<E>::T* dst, int64_t ld, int64_t part) {
    typedef typename Parts<E>::T T;
    constexpr int N = Parts<E>::kCount;
    const int64_t per_row = ld / 8;
    for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < rows * per_row; i += (int64_t)gridDim.x * kThreads) {
        const int64_t r = i / per_row, c = i % per_row * 8;
        typename Matrix<T>::V8 out[N];
#pragma unroll
        for (int j = 0; j < 8; j++) {
            T p[N];
            cut<T, N>(c + j < cols ? (float)src[r * ld_src + c + j] : 0.0f, p);
#pragma unroll
            for (int k = 0; k < N; k++) out[k][j] = p[k];
        }
#pragma unroll
        for (int k = 0; k < N; k++) *reinterpret_cast<typename Matrix<T>::V8*>(dst + k * part + r * ld + c) = out[k];
    }
}

// The transpose: dst[c][r], zeros behind the last row, and in place of rows that take no part.
template <typename E>
__global__ __launch_bounds__(kThreads) void turn_kernel(const E* src, int64_t rows, int64_t cols, int64_t ld_src,
                                                        typename Parts<E>::T* dst, int64_t ld, int64_t part,
                                                        const Row* only) {
    typedef typename Parts<E>::T T;
    constexpr int N = Parts<E>::kCount;
    __shared__ float tile[64][65];
    const int64_t down = ld / 64, across = (cols + 63) / 64;
    for (int64_t t = blockIdx.x; t < down * across; t += gridDim.x) {
        const int64_t r0 = t % down * 64, c0 = t / down * 64;
        __syncthreads();
#pragma unroll
        for (int k = 0; k < 16; k++) {
            const int i = k * 4 + threadIdx.x / 64, j = threadIdx.x % 64;
            const bool in = r0 + i < rows && c0 + j < cols && (only == nullptr || only[r0 + i].target >= 0);
            tile[i][j] = in ? (float)src[(r0 + i) * ld_src + c0 + j] : 0.0f;
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < 16; k++) {
            const int i = threadIdx.x % 64, j = k * 4 + threadIdx.x / 64;
            if (c0 + j < cols) {
                T p[N];
                cut<T, N>(tile[i][j], p);
#pragma unroll
                for (int q = 0; q < N; q++) dst[q * part + (c0 + j) * ld + r0 + i] = p[q];
            }
        }
    }
}

// --- the tile loop --------------------------------------------------------------

// 16 bytes a lane from memory to LDS, lane after lane from `to` on.
__device__ __forceinline__ void load_lds(const void* from, void* to) {
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)from,
                                     (__attribute__((address_space(3))) void*)to, 16, 0, 0);
}

// A tile of BM x BN of the product by WM x WN waves, each with MI x NJ squares of 16.
// An operand's tile lies in LDS as rows of 128 bytes; the 16-byte pieces of a row are
// exchanged by the row's number, so that lanes reading a column of pieces meet all banks.
template <typename T, int BM, int BN, int WM, int WN, int PAIRS>
struct Tile {
    static constexpr int kWaves = WM * WN, MI = BM / WM / 16, NJ = BN / WN / 16;
    static constexpr int kBytes = (BM + BN) * kStep * 2;  // of one step
    typedef typename Matrix<T>::V8 V8;

    template <int ROWS>
    static __device__ __forceinline__ void fetch(const Operand& o, int part, int64_t row0, int64_t k, char* lds) {
        const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
        const int r = lane >> 3, piece = (lane & 7) ^ r;
        const T* p = static_cast<const T*>(o.p) + part * o.part + k + piece * 8;
#pragma unroll
        for (int i = 0; i < ROWS / 8 / kWaves; i++) {
            const int block = i * kWaves + wave;
            int64_t row = row0 + block * 8 + r;
            row = row < o.rows ? row : o.rows - 1;  // rows past the end: any, their products are not used
            load_lds(p + row * o.ld, lds + block * 1024);
        }
    }
    static __device__ __forceinline__ V8 piece_at(const char* lds, int row, int piece) {
        return *reinterpret_cast<const V8*>(lds + row * 128 + ((piece ^ (row & 7)) << 4));
    }

    // acc[i][j][q]: row wave_m + 16 i + 4 (lane / 16) + q of X, row wave_n + 16 j + lane % 16 of Y.
    static __device__ __forceinline__ void run(const Operand& x, const Operand& y, int64_t x0, int64_t y0, int64_t k0,
                                               int steps, char* lds, F4 (&acc)[MI][NJ]) {
        const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
        const int m = wave / WN * MI * 16 + (lane & 15), n = wave % WN * NJ * 16 + (lane & 15);
#pragma unroll
        for (int i = 0; i < MI; i++)
#pragma unroll
            for (int j = 0; j < NJ; j++) acc[i][j] = F4{0.0f, 0.0f, 0.0f, 0.0f};
        int pair = 0, at = 0;  // of the step that is fetched next
        const auto fetch_next = [&](char* to) {
            const int px = PAIRS == 1 ? 0 : kPairs[pair][0], py = PAIRS == 1 ? 0 : kPairs[pair][1];
            fetch<BM>(x, px, x0, k0 + (int64_t)at * kStep, to);
            fetch<BN>(y, py, y0, k0 + (int64_t)at * kStep, to + BM * 128);
            if (++at == steps) {
                at = 0;
                pair++;
            }
        };
        const int total = steps * PAIRS;
        if (total > 0) fetch_next(lds);
        for (int t = 0; t < total; t++) {
            __syncthreads();  // step t is there, and step t - 1 read
            if (t + 1 < total) fetch_next(lds + ((t + 1) & 1) * kBytes);
            const char* xs = lds + (t & 1) * kBytes;
            const char* ys = xs + BM * 128;
#pragma unroll
            for (int k = 0; k < kStep / 32; k++) {
                V8 fx[MI], fy[NJ];
#pragma unroll
                for (int i = 0; i < MI; i++) fx[i] = piece_at(xs, m + i * 16, k * 4 + (lane >> 4));
#pragma unroll
                for (int j = 0; j < NJ; j++) fy[j] = piece_at(ys, n + j * 16, k * 4 + (lane >> 4));
#pragma unroll
                for (int i = 0; i < MI; i++)
#pragma unroll
                    for (int j = 0; j < NJ; j++) acc[i][j] = Matrix<T>::mfma(fx[i], fy[j], acc[i][j]);
            }
        }
        __syncthreads();
    }
};

constexpr int kBM = 128, kBN = 128, kWM = 2, kWN = 2;

// Maximum and sum of exponentials of a tile's logits, per row, and the targets' logits;
// `first` is the token of the head's first row.
template <typename T, int PAIRS>
__global__ __launch_bounds__(kThreads) void logits_kernel(const Args a, const Operand head, const Operand hidden,
                                                          int steps, int64_t first, int32_t tiles) {
    typedef Tile<T, kBM, kBN, kWM, kWN, PAIRS> Tl;
    __shared__ __attribute__((aligned(16))) char lds[2 * Tl::kBytes];
    const int64_t v0 = (int64_t)(blockIdx.x % tiles) * kBM, r0 = (int64_t)(blockIdx.x / tiles) * kBN;
    F4 acc[Tl::MI][Tl::NJ];
    Tl::run(head, hidden, v0, r0, 0, steps, lds, acc);
    const int64_t tile = (first + v0) / kBM;
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, wm = wave / kWN, wn = wave % kWN;
    float* s_max = reinterpret_cast<float*>(lds);  // [kWM][kBN]
    float* s_sum = s_max + kWM * kBN;
    const int64_t v = first + v0 + wm * Tl::MI * 16 + (lane >> 4) * 4;
#pragma unroll
    for (int j = 0; j < Tl::NJ; j++) {
        const int in = wn * Tl::NJ * 16 + j * 16 + (lane & 15);
        const int64_t r = r0 + in;
        const int32_t y = r < a.n ? a.rows[r].target : -1;
        float m = -INFINITY;
#pragma unroll
        for (int i = 0; i < Tl::MI; i++)
#pragma unroll
            for (int q = 0; q < 4; q++) {
                if (v + i * 16 + q >= a.V) acc[i][j][q] = -INFINITY;
                else if (v + i * 16 + q == y) a.at_target[r] = acc[i][j][q];
                m = fmaxf(m, acc[i][j][q]);
            }
        m = fmaxf(m, __shfl_xor(m, 16));
        m = fmaxf(m, __shfl_xor(m, 32));
        const float from = m == -INFINITY ? 0.0f : m;
        float S = 0.0f;
#pragma unroll
        for (int i = 0; i < Tl::MI; i++)
#pragma unroll
            for (int q = 0; q < 4; q++) S += fast_exp(acc[i][j][q] - from);
        S += __shfl_xor(S, 16);
        S += __shfl_xor(S, 32);
        if (lane < 16) {
            s_max[wm * kBN + in] = m;
            s_sum[wm * kBN + in] = S;
        }
    }
    __syncthreads();
    for (int in = threadIdx.x; in < kBN; in += kThreads) {
        if (r0 + in >= a.n) continue;
        float m = -INFINITY;
        for (int k = 0; k < kWM; k++) m = fmaxf(m, s_max[k * kBN + in]);
        const float from = m == -INFINITY ? 0.0f : m;
        float S = 0.0f;
        for (int k = 0; k < kWM; k++) S += s_sum[k * kBN + in] * fast_exp(s_max[k * kBN + in] - from);
        a.part_max[tile * a.n + r0 + in] = m;
        a.part_sum[tile * a.n + r0 + in] = S;
    }
}

// e of a piece of the vocabulary: e[n][ld], and with the rows' weights over their
// largest, turned, we[tokens][ld_turned].
struct Errors {
    void *e, *we;      // either may be NULL
    int64_t ld, part, ld_turned, part_turned;
    int64_t first;     // token of the piece
    int32_t tiles;     // tiles of tokens in the piece
};
template <typename T, int PAIRS>
__global__ __launch_bounds__(kThreads) void errors_kernel(const Args a, const Operand head, const Operand hidden,
                                                          int steps, const Errors o) {
    typedef Tile<T, kBM, kBN, kWM, kWN, PAIRS> Tl;
    constexpr int N = PAIRS == 1 ? 1 : 3;
    __shared__ __attribute__((aligned(16))) char lds[2 * Tl::kBytes];
    const int64_t v0 = (int64_t)(blockIdx.x % o.tiles) * kBM, r0 = (int64_t)(blockIdx.x / o.tiles) * kBN;
    F4 acc[Tl::MI][Tl::NJ];
    Tl::run(head, hidden, v0, r0, 0, steps, lds, acc);
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, wm = wave / kWN, wn = wave % kWN;
    const float top = a.totals->weight;
#pragma unroll
    for (int j = 0; j < Tl::NJ; j++) {
        const int64_t r = r0 + wn * Tl::NJ * 16 + j * 16 + (lane & 15);
        const Row row = r < a.n ? a.rows[r] : Row{-1, 0.0f};
        const bool on = row.target >= 0;
        const float lse = on ? a.lse_in[r] : 0.0f;
        const float w = on && top != 0.0f ? row.weight / top : 0.0f;
#pragma unroll
        for (int i = 0; i < Tl::MI; i++) {
            const int64_t v = v0 + wm * Tl::MI * 16 + i * 16 + (lane >> 4) * 4;
            typedef T T4 __attribute__((ext_vector_type(4)));
            T4 e[N];
            T we[N][4];
#pragma unroll
            for (int q = 0; q < 4; q++) {
                float x = 0.0f;
                if (on && o.first + v + q < a.V) {
                    x = fast_exp(acc[i][j][q] - lse);
                    if (o.first + v + q == row.target) x -= 1.0f;
                }
                x *= Matrix<T>::kScale;
                T p[N];
                cut<T, N>(x, p);
#pragma unroll
                for (int k = 0; k < N; k++) e[k][q] = p[k];
                cut<T, N>(on ? x * w : 0.0f, p);
#pragma unroll
                for (int k = 0; k < N; k++) we[k][q] = p[k];
            }
            if (o.e && r < a.n && v < o.ld) {
#pragma unroll
                for (int k = 0; k < N; k++) *reinterpret_cast<T4*>(static_cast<T*>(o.e) + k * o.part + r * o.ld + v) = e[k];
            }
            if (o.we && r < o.ld_turned) {
#pragma unroll
                for (int q = 0; q < 4; q++)
#pragma unroll
                    for (int k = 0; k < N; k++)
                        if (v + q < o.ld) static_cast<T*>(o.we)[k * o.part_turned + (v + q) * o.ld_turned + r] = we[k][q];
            }
        }
    }
}

// dW of a piece: out[token][D], times what the errors were held by.
template <typename E, typename T, int PAIRS>
__global__ __launch_bounds__(kThreads) void dhead_kernel(const Args a, const Operand x, const Operand y, int steps, E* out) {
    typedef Tile<T, kBM, kBN, kWM, kWN, PAIRS> Tl;
    __shared__ __attribute__((aligned(16))) char lds[2 * Tl::kBytes];
    const int across = (int)((a.D + kBM - 1) / kBM);
    const int64_t d0 = (int64_t)(blockIdx.x % across) * kBM, v0 = (int64_t)(blockIdx.x / across) * kBN;
    F4 acc[Tl::MI][Tl::NJ];
    Tl::run(x, y, d0, v0, 0, steps, lds, acc);
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, wm = wave / kWN, wn = wave % kWN;
    const float by = a.totals->weight * a.totals->share * a.grad_scale * (a.grad_loss ? *a.grad_loss : 1.0f) / Matrix<T>::kScale;
#pragma unroll
    for (int j = 0; j < Tl::NJ; j++) {
        const int64_t v = v0 + wn * Tl::NJ * 16 + j * 16 + (lane & 15);
        if (v >= y.rows) continue;
#pragma unroll
        for (int i = 0; i < Tl::MI; i++) {
            const int64_t d = d0 + wm * Tl::MI * 16 + i * 16 + (lane >> 4) * 4;
            float f[4];
#pragma unroll
            for (int q = 0; q < 4; q++) f[q] = acc[i][j][q] * by;
            if (d + 4 <= a.D) {
                Vec<E, 4>::store(out + v * a.D + d, f);
            } else {
#pragma unroll
                for (int q = 0; q < 4; q++)
                    if (d + q < a.D) out[v * a.D + d + q] = (E)f[q];
            }
        }
    }
}

// dh of a piece, added to what the pieces before left: slab[split][n][ld], a split of the piece's tokens each.
template <typename T, int PAIRS>
__global__ __launch_bounds__(kThreads) void dhidden_kernel(const Args a, const Operand x, const Operand y, int steps,
                                                           int splits, float* slab, int64_t ld, int add) {
    typedef Tile<T, kBM, kBN, kWM, kWN, PAIRS> Tl;
    __shared__ __attribute__((aligned(16))) char lds[2 * Tl::kBytes];
    const int across = (int)((a.D + kBM - 1) / kBM);
    const int split = blockIdx.x % splits, tile = blockIdx.x / splits;
    const int64_t d0 = (int64_t)(tile % across) * kBM, r0 = (int64_t)(tile / across) * kBN;
    const int from = (int)((int64_t)steps * split / splits), to = (int)((int64_t)steps * (split + 1) / splits);
    F4 acc[Tl::MI][Tl::NJ];
    Tl::run(x, y, d0, r0, (int64_t)from * kStep, to - from, lds, acc);
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, wm = wave / kWN, wn = wave % kWN;
#pragma unroll
    for (int j = 0; j < Tl::NJ; j++) {
        const int64_t r = r0 + wn * Tl::NJ * 16 + j * 16 + (lane & 15);
        if (r >= a.n) continue;
#pragma unroll
        for (int i = 0; i < Tl::MI; i++) {
            const int64_t d = d0 + wm * Tl::MI * 16 + i * 16 + (lane >> 4) * 4;
            if (d >= ld) continue;
            F4* at = reinterpret_cast<F4*>(slab + (split * a.n + r) * ld + d);
            *at = add ? *at + acc[i][j] : acc[i][j];
        }
    }
}

// The splits' sums, times the row's share.
template <typename E>
__global__ __launch_bounds__(kThreads) void rows_out_kernel(const Args a, const float* slab, int64_t ld, int splits,
                                                            float held, E* out) {
    const float by = a.totals->share * a.grad_scale * (a.grad_loss ? *a.grad_loss : 1.0f) / held;
    for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < a.n * a.D; i += (int64_t)gridDim.x * kThreads) {
        const int64_t r = i / a.D, d = i % a.D;
        const Row row = a.rows[r];
        float v = 0.0f;
        if (row.target >= 0) {
            for (int k = 0; k < splits; k++) v += slab[(k * a.n + r) * ld + d];
            v *= row.weight * by;
        }
        out[i] = (E)v;
    }
}

// --- the plan -------------------------------------------------------------------

inline int64_t up(int64_t x, int64_t m) { return (x + m - 1) / m * m; }

// Where everything lies in the workspace.
struct Plan {
    int parts = 0;                       // of a value
    int64_t ldk = 0, ldn = 0, ldv = 0;   // padded D, n and tokens of a piece
    int64_t piece = 0, loss_piece = 0;   // tokens of a piece, backward and forward
    int tiles = 0;                       // tiles of tokens
    int splits = 0;
    int64_t rows = 0, totals = 0, sums = 0, counts = 0, tops = 0, at_target = 0, part_max = 0, part_sum = 0;
    int64_t hidden = 0, head = 0, head_piece = 0, hidden_t = 0, head_t = 0, e = 0, we = 0, slab = 0;
    int64_t bytes_loss = 0, bytes_backward = 0;
};

bool plain_rows(int32_t dtype, const void* p, int64_t row, int64_t D) {
    return dtype != GEAR_DTYPE_F32 && D % kStep == 0 && row % 8 == 0 && reinterpret_cast<uintptr_t>(p) % 16 == 0;
}

// The workspace holds what any alignment of the operands needs.
Plan plan_of(const gear_token_desc& d) {
    Plan p;
    p.parts = d.dtype == GEAR_DTYPE_F32 ? 3 : 1;
    p.ldk = up(d.D, kStep);
    p.ldn = up(d.n, kStep);
    p.tiles = (int)((d.V + kBM - 1) / kBM);
    int64_t piece = kPieceValues / (d.n > 0 ? d.n : 1) / p.parts / kBM * kBM;
    piece = piece < kBM ? kBM : piece > kPieceTokens ? kPieceTokens : piece;
    p.piece = piece < d.V ? piece : d.V;
    p.loss_piece = kPieceTokens < d.V ? kPieceTokens : d.V;
    p.ldv = up(p.piece, kStep);
    // Few tiles of dh share the GPU's 256 units by splitting the tokens.
    const int64_t tiles = (d.D + kBM - 1) / kBM * ((d.n + kBN - 1) / kBN), steps = p.ldv / kStep;
    p.splits = 1;
    while (tiles * p.splits < 512 && p.splits * 8 <= steps && p.splits < 16) p.splits *= 2;
    int64_t at = 0;
    const auto take = [&](int64_t bytes) {
        const int64_t here = at;
        at += up(bytes, 256);
        return here;
    };
    p.rows = take(d.n * (int64_t)sizeof(Row));
    p.totals = take(sizeof(Totals));
    p.sums = take(kParts * sizeof(double));
    p.counts = take(kParts * sizeof(int64_t));
    p.tops = take(kParts * sizeof(float));
    p.hidden = take(d.n * p.ldk * p.parts * 2);
    const int64_t common = at;
    p.at_target = take(d.n * 4);
    p.part_max = take(d.n * (int64_t)p.tiles * 4);
    p.part_sum = take(d.n * (int64_t)p.tiles * 4);
    p.head = take(p.loss_piece * p.ldk * p.parts * 2);
    p.bytes_loss = at;
    at = common;
    p.head_piece = take(p.piece * p.ldk * p.parts * 2);
    p.hidden_t = take(d.D * p.ldn * p.parts * 2);
    p.head_t = take(d.D * p.ldv * p.parts * 2);
    p.e = take(d.n * p.ldv * p.parts * 2);
    p.we = take(p.ldv * p.ldn * p.parts * 2);
    p.slab = take(p.splits * d.n * p.ldk * 4);
    p.bytes_backward = at;
    return p;
}

const char* flaw(const gear_token_desc* d) {
    if (d == nullptr) return "NULL descriptor";
    if (float_bytes(d->dtype) == 0) return "dtype must be F16, BF16 or F32";
    if (d->target_dtype != GEAR_DTYPE_U8 && d->target_dtype != GEAR_DTYPE_I32 && d->target_dtype != GEAR_DTYPE_I64)
        return "target dtype must be U8, I32 or I64";
    if (d->n < 0 || d->n > GEAR_TOKEN_MAX || d->V < 1 || d->V > GEAR_TOKEN_MAX || d->D < 1 || d->D > 65536 ||
        d->n * d->V > (1ll << 36))
        return "size out of range";
    if ((d->hidden_row < d->D && d->n > 1) || (d->head_row < d->D && d->V > 1)) return "row stride below D";
    if (d->mask_group < 1 || d->weight_group < 1) return "group below 1";
    if (!(d->denom >= 0.0f) || d->denom > 3e38f) return "denom below 0 or not finite";
    if (!(fabsf(d->grad_scale) < 3e38f)) return "grad_scale not finite";
    return nullptr;
}

unsigned some_blocks(int64_t items, int64_t most) {
    const int64_t b = (items + kThreads - 1) / kThreads;
    return (unsigned)(b < 1 ? 1 : b < most ? b : most);
}

Args args_of(const gear_token_desc& d, const Plan& p, char* work) {
    Args a{};
    a.target = d.d_target;
    a.mask = d.d_mask;
    a.weight = d.d_weight;
    a.rows = reinterpret_cast<Row*>(work + p.rows);
    a.totals = reinterpret_cast<Totals*>(work + p.totals);
    a.sums = reinterpret_cast<double*>(work + p.sums);
    a.counts = reinterpret_cast<int64_t*>(work + p.counts);
    a.tops = reinterpret_cast<float*>(work + p.tops);
    a.n = d.n;
    a.D = d.D;
    a.V = d.V;
    a.mask_group = d.mask_group;
    a.weight_group = d.weight_group;
    a.target_dtype = d.target_dtype;
    a.tiles = p.tiles;
    a.parts = (int32_t)some_blocks(d.n, kParts);
    a.denom = d.denom;
    a.grad_scale = d.grad_scale;
    return a;
}

template <typename E>
struct Call {
    typedef typename Parts<E>::T T;
    static constexpr int N = Parts<E>::kCount, PAIRS = N == 1 ? 1 : 6;
    const gear_token_desc& d;
    const Plan p;
    char* work;
    hipStream_t s;

    hipError_t copy(const void* src, int64_t rows, int64_t ld_src, int64_t to) const {
        hipLaunchKernelGGL(copy_kernel<E>, dim3(some_blocks(rows * (p.ldk / 8), 8192)), dim3(kThreads), 0, s,
                           static_cast<const E*>(src), rows, d.D, ld_src, reinterpret_cast<T*>(work + to), p.ldk,
                           rows * p.ldk);
        return hipGetLastError();
    }
    hipError_t turn(const void* src, int64_t rows, int64_t ld_src, int64_t ld, int64_t to, const Row* only) const {
        const int64_t tiles = ld / 64 * ((d.D + 63) / 64);
        hipLaunchKernelGGL(turn_kernel<E>, dim3((unsigned)(tiles < 16384 ? tiles : 16384)), dim3(kThreads), 0, s,
                           static_cast<const E*>(src), rows, d.D, ld_src, reinterpret_cast<T*>(work + to), ld, d.D * ld, only);
        return hipGetLastError();
    }
    // The operand of rows as they lie, or of a copy.
    hipError_t operand(const void* src, int64_t rows, int64_t ld_src, int64_t to, Operand& o) const {
        if (plain_rows(d.dtype, src, ld_src, d.D)) {
            o = Operand{src, rows, ld_src, 0};
            return hipSuccess;
        }
        o = Operand{work + to, rows, p.ldk, rows * p.ldk};
        return copy(src, rows, ld_src, to);
    }
    hipError_t rows(const Args& a) const {
        hipLaunchKernelGGL(rows_kernel, dim3(a.parts), dim3(kThreads), 0, s, a);
        hipLaunchKernelGGL(totals_kernel, dim3(1), dim3(64), 0, s, a);
        return hipGetLastError();
    }

    hipError_t loss(Args a, const void* hidden, const void* head) const {
        a.at_target = reinterpret_cast<float*>(work + p.at_target);
        a.part_max = reinterpret_cast<float*>(work + p.part_max);
        a.part_sum = reinterpret_cast<float*>(work + p.part_sum);
        hipError_t e = rows(a);
        if (e != hipSuccess) return e;
        if (a.n > 0) {
            Operand x, y;
            if ((e = operand(hidden, a.n, d.hidden_row, p.hidden, y)) != hipSuccess) return e;
            for (int64_t first = 0; first < a.V; first += p.loss_piece) {
                const int64_t tokens = a.V - first < p.loss_piece ? a.V - first : p.loss_piece;
                const int tiles = (int)((tokens + kBM - 1) / kBM);
                const E* from = static_cast<const E*>(head) + first * d.head_row;
                if ((e = operand(from, tokens, d.head_row, p.head, x)) != hipSuccess) return e;
                hipLaunchKernelGGL((logits_kernel<T, PAIRS>), dim3((unsigned)(tiles * ((a.n + kBN - 1) / kBN))),
                                   dim3(kThreads), 0, s, a, x, y, (int)(p.ldk / kStep), first, tiles);
                if ((e = hipGetLastError()) != hipSuccess) return e;
            }
        }
        hipLaunchKernelGGL(lse_kernel, dim3(a.parts), dim3(kThreads), 0, s, a);
        hipLaunchKernelGGL(loss_kernel, dim3(1), dim3(64), 0, s, a);
        return hipGetLastError();
    }

    hipError_t backward(const Args& a, const void* hidden, const void* head, void* dhidden, void* dhead) const {
        hipError_t e = rows(a);
        if (e != hipSuccess) return e;
        Operand x, y;
        if ((e = operand(hidden, a.n, d.hidden_row, p.hidden, y)) != hipSuccess) return e;
        if (dhead && (e = turn(hidden, a.n, d.hidden_row, p.ldn, p.hidden_t, a.rows)) != hipSuccess) return e;
        const int across = (int)((a.D + kBM - 1) / kBM);
        float* slab = reinterpret_cast<float*>(work + p.slab);
        for (int64_t first = 0; first < a.V; first += p.piece) {
            const int64_t tokens = a.V - first < p.piece ? a.V - first : p.piece, ldv = up(tokens, kStep);
            const E* from = static_cast<const E*>(head) + first * d.head_row;
            if ((e = operand(from, tokens, d.head_row, p.head_piece, x)) != hipSuccess) return e;
            Errors o{};
            o.e = dhidden ? work + p.e : nullptr;
            o.we = dhead ? work + p.we : nullptr;
            o.ld = ldv;
            o.part = a.n * ldv;
            o.ld_turned = p.ldn;
            o.part_turned = ldv * p.ldn;
            o.first = first;
            o.tiles = (int32_t)((ldv + kBM - 1) / kBM);
            hipLaunchKernelGGL((errors_kernel<T, PAIRS>), dim3((unsigned)(o.tiles * ((p.ldn + kBN - 1) / kBN))),
                               dim3(kThreads), 0, s, a, x, y, (int)(p.ldk / kStep), o);
            if ((e = hipGetLastError()) != hipSuccess) return e;
            if (dhead) {
                const Operand ht{work + p.hidden_t, a.D, p.ldn, a.D * p.ldn};
                const Operand we{work + p.we, tokens, p.ldn, ldv * p.ldn};
                hipLaunchKernelGGL((dhead_kernel<E, T, PAIRS>), dim3((unsigned)(across * ((tokens + kBN - 1) / kBN))),
                                   dim3(kThreads), 0, s, a, ht, we, (int)(p.ldn / kStep), static_cast<E*>(dhead) + first * a.D);
                if ((e = hipGetLastError()) != hipSuccess) return e;
            }
            if (dhidden) {
                if ((e = turn(from, tokens, d.head_row, ldv, p.head_t, nullptr)) != hipSuccess) return e;
                const Operand wt{work + p.head_t, a.D, ldv, a.D * ldv};
                const Operand er{work + p.e, a.n, ldv, a.n * ldv};
                hipLaunchKernelGGL((dhidden_kernel<T, PAIRS>),
                                   dim3((unsigned)(p.splits * across * ((a.n + kBN - 1) / kBN))), dim3(kThreads), 0, s, a,
                                   wt, er, (int)(ldv / kStep), p.splits, slab, p.ldk, first > 0 ? 1 : 0);
                if ((e = hipGetLastError()) != hipSuccess) return e;
            }
        }
        if (dhidden) {
            hipLaunchKernelGGL(rows_out_kernel<E>, dim3(some_blocks(a.n * a.D, 8192)), dim3(kThreads), 0, s, a, slab, p.ldk,
                               p.splits, Matrix<T>::kScale, static_cast<E*>(dhidden));
            e = hipGetLastError();
        }
        return e;
    }
};

// Zeros, 16 bits at a time: the head's gradient without rows.
__global__ __launch_bounds__(kThreads) void zero_kernel(uint16_t* p, int64_t n) {
    for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < n; i += (int64_t)gridDim.x * kThreads) p[i] = 0;
}

template <typename F>
hipError_t by_type(int32_t dtype, F f) {
    return dtype == GEAR_DTYPE_F32 ? f(0.0f) : dtype == GEAR_DTYPE_BF16 ? f((__bf16)0.0f) : f((_Float16)0.0f);
}

}  // namespace
}  // namespace gear

extern "C" int gear_token_loss_sizes(const gear_token_desc* d, int64_t* loss_bytes, int64_t* backward_bytes) {
    using namespace gear;
    if (const char* w = flaw(d)) return fail(GEAR_E_INVAL, std::string("gear_token_loss_sizes: ") + w);
    const Plan p = plan_of(*d);
    if (loss_bytes) *loss_bytes = p.bytes_loss;
    if (backward_bytes) *backward_bytes = p.bytes_backward;
    return GEAR_OK;
}

extern "C" int gear_token_loss(const gear_token_desc* d, const void* d_hidden, const void* d_head, float* d_loss,
                               float* d_logp, float* d_lse, void* d_work, int64_t work_bytes, void* stream) {
    using namespace gear;
    if (const char* w = flaw(d)) return fail(GEAR_E_INVAL, std::string("gear_token_loss: ") + w);
    if (d_loss == nullptr) return fail(GEAR_E_INVAL, "gear_token_loss: NULL loss");
    if (d->n > 0 && (d_hidden == nullptr || d_head == nullptr || d->d_target == nullptr))
        return fail(GEAR_E_INVAL, "gear_token_loss: NULL hidden, head or target");
    const Plan p = plan_of(*d);
    if (d_work == nullptr || work_bytes < p.bytes_loss || reinterpret_cast<uintptr_t>(d_work) % 16 != 0)
        return fail(GEAR_E_INVAL, "gear_token_loss: workspace smaller than gear_token_loss_sizes states, or not aligned to 16 bytes");
    char* work = static_cast<char*>(d_work);
    Args a = args_of(*d, p, work);
    a.loss = d_loss;
    a.logp = d_logp;
    a.lse = d_lse;
    (void)hipGetLastError();  // an error pending from an earlier HIP call is not this call's
    hipStream_t s = static_cast<hipStream_t>(stream);
    const hipError_t e = by_type(d->dtype, [&](auto type) {
        return Call<decltype(type)>{*d, p, work, s}.loss(a, d_hidden, d_head);
    });
    return e == hipSuccess ? GEAR_OK : hip_fail(e, "gear_token_loss: launch");
}

extern "C" int gear_token_loss_backward(const gear_token_desc* d, const void* d_hidden, const void* d_head,
                                        const float* d_lse, const float* d_grad_loss, void* d_dhidden, void* d_dhead,
                                        void* d_work, int64_t work_bytes, void* stream) {
    using namespace gear;
    if (const char* w = flaw(d)) return fail(GEAR_E_INVAL, std::string("gear_token_loss_backward: ") + w);
    if (d->n > 0 && (d_hidden == nullptr || d_head == nullptr || d->d_target == nullptr || d_lse == nullptr))
        return fail(GEAR_E_INVAL, "gear_token_loss_backward: NULL hidden, head, target or lse");
    const Plan p = plan_of(*d);
    if (d_work == nullptr || work_bytes < p.bytes_backward || reinterpret_cast<uintptr_t>(d_work) % 16 != 0)
        return fail(GEAR_E_INVAL,
                    "gear_token_loss_backward: workspace smaller than gear_token_loss_sizes states, or not aligned to 16 bytes");
    char* work = static_cast<char*>(d_work);
    Args a = args_of(*d, p, work);
    a.lse_in = d_lse;
    a.grad_loss = d_grad_loss;
    (void)hipGetLastError();  // an error pending from an earlier HIP call is not this call's
    hipStream_t s = static_cast<hipStream_t>(stream);
    hipError_t e = hipSuccess;
    if (d->n == 0) {
        if (d_dhead == nullptr) return GEAR_OK;
        const int64_t n = d->V * d->D * float_bytes(d->dtype) / 2;
        hipLaunchKernelGGL(zero_kernel, dim3(some_blocks(n, 8192)), dim3(kThreads), 0, s, static_cast<uint16_t*>(d_dhead), n);
        e = hipGetLastError();
    } else if (d_dhidden != nullptr || d_dhead != nullptr) {
        e = by_type(d->dtype, [&](auto type) {
            return Call<decltype(type)>{*d, p, work, s}.backward(a, d_hidden, d_head, d_dhidden, d_dhead);
        });
    }
    return e == hipSuccess ? GEAR_OK : hip_fail(e, "gear_token_loss_backward: launch");
}
