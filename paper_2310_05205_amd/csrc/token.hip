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
// 32-bit values are cut into two fp16 parts, a 2^s = a1 + a2 (11 bits each), s making the largest
// finite value 2^14 to 2^15, of a row for the logits, which so depend on their own row and token
// alone, and of the tensor for the turned copies, whose k runs over the rows; a part is off by
// 2^-22 of the value, or by 2^-39 of the largest where the value is far below it.  The products a1 b1, a1 b2 and a2 b1 leave out
// 2^-22 of |a b| at most.  Matrix instructions of 16-bit types are 16 times as fast as those of 32
// bits, so three of them take a fifth of the time.  (Three bf16 parts need no scale and leave
// 2^-25, but six products: 1000 x 512 x 8192, forward and backward, took 245 us with them and takes 158.)
#include <math.h>

#include <type_traits>

#include "element.h"
#include "gear_internal.h"

namespace gear {
namespace {

constexpr int kStep = 64;                 // k of one step: 128 bytes a row
constexpr int kThreads = 512;             // of the kernels that are not products
constexpr int64_t kPieceValues = 1 << 27;  // values of e formed at a time, at most
constexpr int64_t kPieceTokens = 1 << 16;
constexpr int kParts = 512;               // workgroups that look at the rows
constexpr int64_t kSoloRows = 8192;       // one looks at so many

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
    typedef _Float16 T;
    static constexpr int kCount = 2;
};
// The products of parts (first, second), small ones first.
constexpr int kPairs[3][2] = {{1, 0}, {0, 1}, {0, 0}};

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
    float weight;    // largest |weight| of a row that takes part, NaN where one is
};
// Powers of two that 32-bit hidden values and the head are multiplied by before they are cut and turned.
struct Scales {
    int32_t hidden, head;
};

struct Args {
    const void* target;
    const uint8_t* mask;
    const float *weight, *grad_loss, *lse_in;
    float *loss, *logp, *lse;
    Row* rows;
    Totals* totals;
    Scales* scales;    // of 32-bit values, turned
    int32_t *hidden_scale, *head_scale;  // of each row, and of each token of a piece
    uint32_t* largest; // [2][kParts]: largest finite magnitudes of hidden and head, a workgroup each
    double* sums;      // [kParts]
    int64_t* counts;   // [kParts]
    float* tops;       // [kParts]
    float2* part;      // [n][tiles]: maximum and sum of a tile of tokens
    float* at_target;  // [n]: the target's logit
    int64_t n, D, V, mask_group, weight_group;
    int32_t target_dtype, tiles, row_parts, lse_parts, max_parts;
    float denom, grad_scale;
};

// --- rows ---------------------------------------------------------------------

template <typename T>
__device__ __forceinline__ T lanes_add(T v, int lanes) {
    for (int off = lanes / 2; off > 0; off >>= 1) v += __shfl_xor(v, off);
    return v;
}
// The larger magnitude, or NaN where either is one: of weights, it makes every gradient of the head NaN.
__device__ __forceinline__ float larger(float top, float w) { return top != top || fabsf(w) <= top ? top : fabsf(w); }

__device__ __forceinline__ Row row_of(const Args& a, int64_t r) {
    const int64_t y = a.target_dtype == GEAR_DTYPE_I32   ? (int64_t)static_cast<const int32_t*>(a.target)[r]
                      : a.target_dtype == GEAR_DTYPE_I64 ? static_cast<const int64_t*>(a.target)[r]
                                                         : (int64_t)static_cast<const uint8_t*>(a.target)[r];
    const bool on = y >= 0 && y < a.V && (a.mask == nullptr || a.mask[r / a.mask_group] != 0);
    const float w = !on ? 0.0f : a.weight ? a.weight[r / a.weight_group] : 1.0f;
    return Row{on ? (int32_t)y : -1, w};
}
__device__ __forceinline__ Totals totals_of(const Args& a, int64_t count, float top) {
    return Totals{1.0f / (a.denom > 0.0f ? a.denom : count > 0 ? (float)count : 1.0f), top};
}

// Targets and weights of the rows, how many take part, and their largest weight;
// workgroup `block` of a.row_parts.
__device__ __forceinline__ void look_at_rows(const Args& a, int block) {
    __shared__ int64_t s_count[kThreads / 64];
    __shared__ float s_top[kThreads / 64];
    int64_t count = 0;
    float top = 0.0f;
#pragma unroll 4
    for (int64_t r = (int64_t)block * kThreads + threadIdx.x; r < a.n; r += (int64_t)a.row_parts * kThreads) {
        const Row row = row_of(a, r);
        a.rows[r] = row;
        count += row.target >= 0 ? 1 : 0;
        if (row.target >= 0) top = larger(top, row.weight);
    }
    count = lanes_add(count, 64);
    for (int off = 32; off > 0; off >>= 1) top = larger(top, __shfl_xor(top, off));
    if ((threadIdx.x & 63) == 0) {
        s_count[threadIdx.x >> 6] = count;
        s_top[threadIdx.x >> 6] = top;
    }
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int k = 1; k < kThreads / 64; k++) {
            count += s_count[k];
            top = larger(top, s_top[k]);
        }
        if (a.row_parts == 1) {
            *a.totals = totals_of(a, count, top);
        } else {
            a.counts[block] = count;
            a.tops[block] = top;
        }
    }
}
__global__ __launch_bounds__(64) void totals_kernel(const Args a) {
    int64_t count = 0;
    float top = 0.0f;
    for (int k = threadIdx.x; k < a.row_parts; k += 64) {
        count += a.counts[k];
        top = larger(top, a.tops[k]);
    }
    count = lanes_add(count, 64);
    for (int off = 32; off > 0; off >>= 1) top = larger(top, __shfl_xor(top, off));
    if (threadIdx.x == 0) *a.totals = totals_of(a, count, top);
}

// Joins the tiles' maxima and sums, LANES lanes a row: lse, logp, and a sum of the
// losses and a count of the rows that take part per workgroup; the loss where there is but one.
// Two passes over a row's tiles, the second from the cache; latency bounds it: 4096 rows of 128
// tiles 7 us, 16 rows of 512 tiles in one workgroup 6, 320 rows of one tile 3.
template <int LANES>
__global__ __launch_bounds__(kThreads) void lse_kernel(const Args a) {
    __shared__ double s[kThreads / 64];
    __shared__ int64_t s_count[kThreads / 64];
    const int lane = threadIdx.x % LANES;
    double sum = 0.0;
    int64_t count = 0;
    for (int64_t r = ((int64_t)blockIdx.x * kThreads + threadIdx.x) / LANES; r < a.n;
         r += (int64_t)gridDim.x * kThreads / LANES) {
        const float2* part = a.part + r * a.tiles;
        const Row row = row_of(a, r);
        const bool on = row.target >= 0;
        const float z = on ? a.at_target[r] : 0.0f;
        float top = -INFINITY, S = 0.0f;
#pragma unroll 8
        for (int t = lane; t < a.tiles; t += LANES) top = fmaxf(top, part[t].x);
#pragma unroll
        for (int off = LANES / 2; off > 0; off >>= 1) top = fmaxf(top, __shfl_xor(top, off));
        const float from = top == -INFINITY ? 0.0f : top;
#pragma unroll 8
        for (int t = lane; t < a.tiles; t += LANES) S = fmaf(part[t].y, fast_exp(part[t].x - from), S);
        S = lanes_add(S, LANES);
        if (lane != 0) continue;
        const float log_S = __builtin_amdgcn_logf(S) * kLn2;
        const float lp = on ? (z - from) - log_S : 0.0f;
        if (a.logp) a.logp[r] = lp;
        if (a.lse) a.lse[r] = on ? from + log_S : 0.0f;
        count += on ? 1 : 0;
        // A weight of 0 leaves 0 of an infinite term.
        if (on && !(row.weight == 0.0f && lp == -INFINITY)) sum -= (double)row.weight * (double)lp;
    }
    sum = lanes_add(sum, 64);
    count = lanes_add(count, 64);
    if ((threadIdx.x & 63) == 0) {
        s[threadIdx.x >> 6] = sum;
        s_count[threadIdx.x >> 6] = count;
    }
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int k = 1; k < kThreads / 64; k++) {
            sum += s[k];
            count += s_count[k];
        }
        if (gridDim.x == 1) {
            *a.loss = (float)(sum * (double)totals_of(a, count, 0.0f).share);
        } else {
            a.sums[blockIdx.x] = sum;
            a.counts[blockIdx.x] = count;
        }
    }
}
__global__ __launch_bounds__(64) void loss_kernel(const Args a) {
    double sum = 0.0;
    int64_t count = 0;
    for (int k = threadIdx.x; k < a.lse_parts; k += 64) {
        sum += a.sums[k];
        count += a.counts[k];
    }
    sum = lanes_add(sum, 64);
    count = lanes_add(count, 64);
    if (threadIdx.x == 0) *a.loss = (float)(sum * (double)totals_of(a, count, 0.0f).share);
}

// --- operands -----------------------------------------------------------------

// A value's parts: each is the rest so far, rounded.  An infinity or a NaN is one in both.
template <typename T, int N>
__device__ __forceinline__ void cut(float v, T (&part)[N]) {
#pragma unroll
    for (int k = 0; k < N; k++) {
        part[k] = (T)v;
        v -= (float)part[k];
    }
}

// The power of two that takes `top`, a finite magnitude, to 2^14 .. 2^15; none for 0.
__device__ __forceinline__ int32_t scale_for(uint32_t top) {
    return top == 0 ? 0 : 15 - __builtin_amdgcn_frexp_expf(__builtin_bit_cast(float, top));
}
// The larger of `top` and a magnitude, in the magnitudes' order, unless that is not finite.
__device__ __forceinline__ uint32_t larger_finite(uint32_t top, float f) {
    const uint32_t m = __builtin_bit_cast(uint32_t, f) & 0x7FFFFFFFu;
    return m < 0x7F800000u && m > top ? m : top;
}
// Largest finite magnitudes of 32-bit hidden rows that take part and of the head: a.max_parts workgroups each.  1000 and 8192
// rows of 512: 5.5 us, latency.  A workgroup that turns rows could look at all of them itself and save this launch,
// which gains 1.8 us at 4000 values and loses 2.5 at 24000.
__global__ __launch_bounds__(kThreads) void largest_kernel(const Args a, const float* hidden, int64_t hidden_row,
                                                           const float* head, int64_t head_row) {
    __shared__ uint32_t s[kThreads / 64];
    const bool first = (int)blockIdx.x < a.max_parts;
    const int64_t rows = first ? a.n : a.V, ld = first ? hidden_row : head_row;
    const float* p = first ? hidden : head;
    const int64_t pieces = (a.D + 3) / 4;
    uint32_t top = 0;
    for (int64_t i = (int64_t)(blockIdx.x % a.max_parts) * kThreads + threadIdx.x; i < rows * pieces;
         i += (int64_t)a.max_parts * kThreads) {
        const int64_t r = i / pieces, c = i % pieces * 4;
        if (first && row_of(a, r).target < 0) continue;
        float f[4] = {0.0f, 0.0f, 0.0f, 0.0f};
        if (c + 4 <= a.D) {
            Vec<float, 4>::unpack(Vec<float, 4>::load(p + r * ld + c), f);
        } else {
#pragma unroll
            for (int q = 0; q < 4; q++)
                if (c + q < a.D) f[q] = p[r * ld + c + q];
        }
#pragma unroll
        for (int q = 0; q < 4; q++) top = larger_finite(top, f[q]);
    }
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) top = max(top, (uint32_t)__shfl_xor((int)top, off));
    if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = top;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int k = 1; k < kThreads / 64; k++) top = max(top, s[k]);
        a.largest[(first ? 0 : kParts) + blockIdx.x % a.max_parts] = top;
    }
}
// The scale of hidden values (q = 0) or of the head from those, in every thread of a workgroup.
__device__ __forceinline__ int32_t find_scale(const Args& a, int q) {
    __shared__ uint32_t s[kThreads / 64];
    static_assert(kThreads >= kParts, "a lane for each workgroup's");
    uint32_t top = (int)threadIdx.x < a.max_parts ? a.largest[q * kParts + threadIdx.x] : 0;
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) top = max(top, (uint32_t)__shfl_xor((int)top, off));
    if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = top;
    __syncthreads();
    for (int k = 0; k < kThreads / 64; k++) top = max(top, s[k]);
    return scale_for(top);
}

// The parts of 8 values in a row, to `to` and, `part` values apart, behind it.
template <typename T, int N>
__device__ __forceinline__ void put8(const float (&f)[8], T* to, int64_t part) {
    typename Matrix<T>::V8 out[N];
#pragma unroll
    for (int j = 0; j < 8; j++) {
        T p[N];
        cut<T, N>(f[j], p);
#pragma unroll
        for (int k = 0; k < N; k++) out[k][j] = p[k];
    }
#pragma unroll
    for (int k = 0; k < N; k++) *reinterpret_cast<typename Matrix<T>::V8*>(to + k * part) = out[k];
}
// 8 values of a row of `left`, zeros behind its end.
template <typename E>
__device__ __forceinline__ void get8(const E* p, int64_t left, float (&f)[8]) {
    if (left >= 8) {
        Vec<E, 8>::unpack(Vec<E, 8>::load(p), f);
    } else {
#pragma unroll
        for (int j = 0; j < 8; j++) f[j] = j < left ? (float)p[j] : 0.0f;
    }
}

// A copy of rows as rows of whole steps (ld), 32-bit ones each times the power of two that it
// leaves in `scale`, or turned: dst[column][row], zeros behind the last row.  `on`: rows that take no
// part become zeros.
struct Job {
    const void* src;
    void* dst;
    int32_t* scale;
    int64_t rows, cols, ld_src, len, ld, part;  // len: of a row of dst, in whole steps
    int32_t first;  // workgroup
    int32_t on;
};
struct Jobs {
    Job copy[2], turn[2];
    int32_t row_blocks, blocks;  // workgroups that look at the rows, the first ones; of all
};
// Lanes that copy a 32-bit row of so many pieces of 8 values.
__host__ __device__ __forceinline__ int lanes_of(int64_t pieces) { return pieces <= 8 ? 8 : pieces <= 16 ? 16 : pieces <= 32 ? 32 : 64; }
template <typename E>
__device__ __forceinline__ void run_copy(const Job& j, int block, int blocks) {
    typedef typename Parts<E>::T T;
    const int64_t per_row = j.len / 8;
    if constexpr (Parts<E>::kCount == 1) {
        for (int64_t i = (int64_t)block * kThreads + threadIdx.x; i < j.rows * per_row; i += (int64_t)blocks * kThreads) {
            const int64_t r = i / per_row, c = i % per_row * 8;
            float f[8];
            get8(static_cast<const E*>(j.src) + r * j.ld_src + c, j.cols - c, f);
            put8<T, 1>(f, static_cast<T*>(j.dst) + r * j.ld + c, j.part);
        }
    } else {
        // A row is read for its scale, then again, from the cache.
        const int lanes = lanes_of(per_row), lane = threadIdx.x & (lanes - 1);
        for (int64_t r = ((int64_t)block * kThreads + threadIdx.x) / lanes; r < j.rows; r += (int64_t)blocks * (kThreads / lanes)) {
            const E* row = static_cast<const E*>(j.src) + r * j.ld_src;
            float f[8];
            uint32_t top = 0;
            for (int64_t c = lane * 8; c < j.cols; c += lanes * 8) {
                get8(row + c, j.cols - c, f);
#pragma unroll
                for (int q = 0; q < 8; q++) top = larger_finite(top, f[q]);
            }
            for (int off = lanes / 2; off > 0; off >>= 1) top = max(top, (uint32_t)__shfl_xor((int)top, off));
            const int32_t by = scale_for(top);
            if (lane == 0) j.scale[r] = by;
            for (int64_t c = lane * 8; c < j.len; c += lanes * 8) {
                get8(row + c, j.cols - c, f);
#pragma unroll
                for (int q = 0; q < 8; q++) f[q] = ldexpf(f[q], by);
                put8<T, 2>(f, static_cast<T*>(j.dst) + r * j.ld + c, j.part);
            }
        }
    }
}
template <typename E>
__device__ __forceinline__ void run_turn(const Args& a, const Job& j, int32_t by, int block, int blocks, float (*tile)[65]) {
    typedef typename Parts<E>::T T;
    static_assert(kThreads == 512, "a lane takes 8 values of the tile");
    const int64_t down = j.len / 64, across = (j.cols + 63) / 64;
    const int at = threadIdx.x >> 3, k = (threadIdx.x & 7) * 8;
    for (int64_t t = block; t < down * across; t += blocks) {
        // Neighbouring workgroups go along the rows, so that lines are read whole.
        const int64_t c0 = t % across * 64, r0 = t / across * 64;
        float f[8];
        const bool in = r0 + at < j.rows && (!j.on || row_of(a, r0 + at).target >= 0);
        get8(static_cast<const E*>(j.src) + (r0 + at) * j.ld_src + c0 + k, in ? j.cols - c0 - k : 0, f);
        __syncthreads();
#pragma unroll
        for (int q = 0; q < 8; q++) tile[at][k + q] = Parts<E>::kCount > 1 ? ldexpf(f[q], by) : f[q];
        __syncthreads();
        if (c0 + at < j.cols) {
#pragma unroll
            for (int q = 0; q < 8; q++) f[q] = tile[k + q][at];
            put8<T, Parts<E>::kCount>(f, static_cast<T*>(j.dst) + (c0 + at) * j.ld + r0 + k, j.part);
        }
    }
}
// What has to be done before a product, in one launch: workgroups for each job; copies of
// the head and of hidden rows, then hidden rows and the head turned.  Memory bounds it: 50001 fp16
// rows of 1003 copied 50 us (205 MB), copied and turned 100; 32768 bf16 rows of 1024 turned 30 (151 MB,
// the hidden rows' among them).
template <typename E>
__global__ __launch_bounds__(kThreads) void prepare_kernel(const Args a, const Jobs jobs) {
    __shared__ float tile[64][65];
    const int b = blockIdx.x;
    if (b < jobs.row_blocks) return look_at_rows(a, b);
    const int copy1 = jobs.copy[1].first, turn0 = jobs.turn[0].first, turn1 = jobs.turn[1].first;
    if (b < copy1) return run_copy<E>(jobs.copy[0], b - jobs.copy[0].first, copy1 - jobs.copy[0].first);
    if (b < turn0) return run_copy<E>(jobs.copy[1], b - copy1, turn0 - copy1);
    const int q = b < turn1 ? 0 : 1, first = q == 0 ? turn0 : turn1;
    const Job& turn = jobs.turn[q];
    int32_t by = 0;
    if constexpr (Parts<E>::kCount > 1) {
        by = find_scale(a, q);
        if (b == first && threadIdx.x == 0) (q == 0 ? a.scales->hidden : a.scales->head) = by;
    }
    run_turn<E>(a, turn, by, b - first, (q == 0 ? turn1 : jobs.blocks) - first, tile);
}

// --- the tile loop --------------------------------------------------------------

// 16 bytes a lane from memory to LDS, lane after lane from `to` on.
__device__ __forceinline__ void load_lds(const void* from, void* to) {
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)from,
                                     (__attribute__((address_space(3))) void*)to, 16, 0, 0);
}
// All waves here, all LDS reads of before done, and all but the last LOADS loads.
template <int LOADS>
__device__ __forceinline__ void meet() {
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(LOADS) : "memory");
}

// A tile of BM x BN of the product by WM x WN waves, each with MI x NJ squares of 16.  A wave reads MI + NJ
// fragments for MI NJ matrix instructions, so large tiles keep LDS behind them: at 256 x 256 a step of 32 needs 768 cycles
// of LDS reads and 1024 of matrix instructions, at 128 x 128 with 4 waves as many as each other.  The rest is
// waiting for the step's loads and for the slowest wave at the barrier: at k of 4096 1250 TFLOP/s, the instructions
// and barriers alone 1614 (the clock falls to 1.9 GHz).  Tried and slower: steps of 32 in four or five stages, 256 x 128 tiles with two workgroups a unit (19 %), 4 waves of 128 x 128.
// Of a step, an operand's tile lies in LDS as rows of ROW bytes, a tile for each of its N parts; the
// 16-byte pieces of a row are exchanged by the row's number, so that lanes reading a column of
// pieces meet all banks.  STAGES steps are on their way or in use.
template <int BM_, int BN_, int WM_, int WN_, int STAGES_, int N_ = 1>
struct Shape {
    static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_, STAGES = STAGES_, N = N_;
    static constexpr int kWaves = WM * WN, kThreads = 64 * kWaves, MI = BM / WM / 16, NJ = BN / WN / 16;
    static constexpr int ROW = N == 1 ? 128 : 64, K = ROW / 2;  // bytes and values of a row in a step
    static constexpr int kBytes = (BM + BN) * ROW * N;          // of a step
    static constexpr int kLds = STAGES * kBytes > BM * BN * 2 ? STAGES * kBytes : BM * BN * 2;
    static constexpr int kWavesPerSimd = kLds > 80 * 1024 ? kWaves / 4 : kWaves / 2;
    static constexpr int kRows = 1024 / ROW;                    // of a wave's load
    static constexpr int kLoads = (BM + BN) / kRows / kWaves * N;  // of a wave for one step
    static_assert(BM / kRows % kWaves == 0 && BN / kRows % kWaves == 0, "waves fetch alike");
};
// For N parts.
template <int N>
struct Shapes {
    typedef Shape<256, 256, 2, 4, 2> Big;
    typedef Shape<128, 128, 2, 2, 2> Middle;
    typedef Shape<64, 64, 2, 2, 4> Small;
};
template <>
struct Shapes<2> {
    typedef Shape<256, 256, 2, 4, 2, 2> Big;
    typedef Shape<128, 128, 2, 2, 2, 2> Middle;
    typedef Shape<64, 64, 2, 2, 4, 2> Small;
};

template <typename T, typename S>
struct Tile {
    static constexpr int MI = S::MI, NJ = S::NJ, N = S::N;
    typedef typename Matrix<T>::V8 V8;

    static __device__ __forceinline__ int exchanged(int row, int piece) {
        return S::ROW == 128 ? piece ^ (row & 7) : piece ^ ((row >> 1) & 3);
    }
    template <int ROWS>
    static __device__ __forceinline__ void fetch(const Operand& o, int64_t row0, int64_t k, char* lds) {
        const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
        const int r = lane / (S::ROW / 16), piece = exchanged(r, lane % (S::ROW / 16));
#pragma unroll
        for (int part = 0; part < N; part++) {
            const T* p = static_cast<const T*>(o.p) + part * o.part + k + piece * 8;
#pragma unroll
            for (int i = 0; i < ROWS / S::kRows / S::kWaves; i++) {
                const int block = i * S::kWaves + wave;
                int64_t row = row0 + block * S::kRows + r;
                row = row < o.rows ? row : o.rows - 1;  // rows past the end: any, their products are not used
                load_lds(p + row * o.ld, lds + part * ROWS * S::ROW + block * 1024);
            }
        }
    }
    static __device__ __forceinline__ V8 piece_at(const char* lds, int row, int piece) {
        return *reinterpret_cast<const V8*>(lds + row * S::ROW + (exchanged(row, piece) << 4));
    }

    // acc[i][j][q]: row wave_m + 16 i + 4 (lane / 16) + q of X, row wave_n + 16 j + lane % 16 of Y; `steps` of kStep.
    static __device__ __forceinline__ void run(const Operand& x, const Operand& y, int64_t x0, int64_t y0, int64_t k0,
                                               int steps, char* lds, F4 (&acc)[MI][NJ]) {
        const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
        const int m = wave / S::WN * MI * 16 + (lane & 15), n = wave % S::WN * NJ * 16 + (lane & 15);
#pragma unroll
        for (int i = 0; i < MI; i++)
#pragma unroll
            for (int j = 0; j < NJ; j++) acc[i][j] = F4{0.0f, 0.0f, 0.0f, 0.0f};
        int at = 0, next = 0;  // the step that is fetched next, and its place
        const auto fetch_next = [&]() {
            char* to = lds + next * S::kBytes;
            fetch<S::BM>(x, x0, k0 + (int64_t)at * S::K, to);
            fetch<S::BN>(y, y0, k0 + (int64_t)at * S::K, to + S::BM * S::ROW * N);
            at++;
            next = next + 1 == S::STAGES ? 0 : next + 1;
        };
        const int total = steps * (kStep / S::K);
        int here = 0;
        meet<0>();  // the last tile's reads
        for (int t = 0; t < S::STAGES - 1 && t < total; t++) fetch_next();
        for (int t = 0; t < total; t++) {
            // Step t is there, and step t - 1 read, whose place step t + STAGES - 1 takes.
            if (t + S::STAGES - 2 < total) meet<(S::STAGES - 2) * S::kLoads>();
            else meet<0>();
            const char* xs = lds + here * S::kBytes;
            const char* ys = xs + S::BM * S::ROW * N;
            here = here + 1 == S::STAGES ? 0 : here + 1;
#pragma unroll
            for (int k = 0; k < S::K / 32; k++) {
                V8 fx[N][MI], fy[N][NJ];
#pragma unroll
                for (int part = 0; part < N; part++) {
#pragma unroll
                    for (int j = 0; j < NJ; j++) fy[part][j] = piece_at(ys + part * S::BN * S::ROW, n + j * 16, k * 4 + (lane >> 4));
#pragma unroll
                    for (int i = 0; i < MI; i++) fx[part][i] = piece_at(xs + part * S::BM * S::ROW, m + i * 16, k * 4 + (lane >> 4));
                }
                if (k == 0) {
                    // Behind the first reads, which the matrix instructions wait for: 1250 TFLOP/s of logits at k of 4096,
                    // and 1200 before them.
                    __builtin_amdgcn_sched_barrier(0);
                    if (t + S::STAGES - 1 < total) fetch_next();
                    __builtin_amdgcn_sched_barrier(0);
                }
                __builtin_amdgcn_s_setprio(1);
                constexpr int PAIRS = N == 1 ? 1 : 3;
#pragma unroll
                for (int pair = 0; pair < PAIRS; pair++)
#pragma unroll
                    for (int i = 0; i < MI; i++)
#pragma unroll
                        for (int j = 0; j < NJ; j++)
                            acc[i][j] = Matrix<T>::mfma(fx[N == 1 ? 0 : kPairs[pair][0]][i], fy[N == 1 ? 0 : kPairs[pair][1]][j], acc[i][j]);
                __builtin_amdgcn_s_setprio(0);
            }
        }
        meet<0>();
    }
};

// Which tile of tm x tn workgroup `b` takes.  Workgroups go round the 8 XCDs; each XCD
// takes neighbouring tiles, 8 down before the next column, so that its L2 serves their rows.
struct Place {
    int m, n;
};
__device__ __forceinline__ Place place_of(int b, int tm, int tn) {
    const int total = tm * tn, xcd = b & 7, per = total >> 3, rest = total & 7;
    const int id = xcd * per + (xcd < rest ? xcd : rest) + (b >> 3);
    const int width = 8 * tn, group = id / width, first = group * 8, in = id - group * width;
    const int high = tm - first < 8 ? tm - first : 8;
    return Place{first + in % high, in / high};
}

// Products of rows from `r` on, every 16th, of scaled values, and of tokens from `t` of the piece on.
template <typename S>
__device__ __forceinline__ void unscale(const Args& a, F4 (&acc)[S::MI][S::NJ], int64_t t, int64_t r) {
    int32_t row[S::NJ];
#pragma unroll
    for (int j = 0; j < S::NJ; j++) row[j] = r + j * 16 < a.n ? a.hidden_scale[r + j * 16] : 0;
#pragma unroll
    for (int i = 0; i < S::MI; i++) {
        // The tokens' scales go on to whole tiles; what lies behind the last one is not used.
        const int4 token = *reinterpret_cast<const int4*>(a.head_scale + t + i * 16);
#pragma unroll
        for (int j = 0; j < S::NJ; j++) {
            acc[i][j][0] = ldexpf(acc[i][j][0], -token.x - row[j]);
            acc[i][j][1] = ldexpf(acc[i][j][1], -token.y - row[j]);
            acc[i][j][2] = ldexpf(acc[i][j][2], -token.z - row[j]);
            acc[i][j][3] = ldexpf(acc[i][j][3], -token.w - row[j]);
        }
    }
}

// Maximum and sum of exponentials of a tile's logits, per row, and the targets' logits;
// `first` is the token of the head's first row.  4096 x 1024 x 32768 bf16: 260 to 281 us, 980 to 1060 TFLOP/s (torch's
// product, which writes the logits, 258); a tile's first loads and its 128 exponentials a lane are 7 of its 35 us, in
// which the matrix instructions stand still.  Few rows are bound by the head's bytes: 16 rows of 2048 and 32768
// tokens 23 us, 5.8 TB/s.
template <typename T, typename S>
__global__ __launch_bounds__(S::kThreads, S::kWavesPerSimd) void logits_kernel(const Args a, const Operand head,
                                                                               const Operand hidden, int steps,
                                                                               int64_t first, int tm, int tn) {
    typedef Tile<T, S> Tl;
    __shared__ __attribute__((aligned(16))) char lds[S::STAGES * S::kBytes];
    const Place at = place_of(blockIdx.x, tm, tn);
    const int64_t v0 = (int64_t)at.m * S::BM, r0 = (int64_t)at.n * S::BN;
    F4 acc[Tl::MI][Tl::NJ];
    Tl::run(head, hidden, v0, r0, 0, steps, lds, acc);
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, wm = wave / S::WN, wn = wave % S::WN;
    float* s_max = reinterpret_cast<float*>(lds);  // [WM][BN]
    float* s_sum = s_max + S::WM * S::BN;
    const int64_t v = first + v0 + wm * Tl::MI * 16 + (lane >> 4) * 4;
    if (S::N > 1) unscale<S>(a, acc, v - first, r0 + wn * Tl::NJ * 16 + (lane & 15));
    if (first + v0 + S::BM > a.V) {
#pragma unroll
        for (int i = 0; i < Tl::MI; i++)
#pragma unroll
            for (int j = 0; j < Tl::NJ; j++)
#pragma unroll
                for (int q = 0; q < 4; q++)
                    if (v + i * 16 + q >= a.V) acc[i][j][q] = -INFINITY;
    }
#pragma unroll
    for (int j = 0; j < Tl::NJ; j++) {
        const int in = wn * Tl::NJ * 16 + j * 16 + (lane & 15);
        const int64_t r = r0 + in;
        const int64_t y = (r < a.n ? row_of(a, r).target : -1) - v;
        float m = -INFINITY;
#pragma unroll
        for (int i = 0; i < Tl::MI; i++)
#pragma unroll
            for (int q = 0; q < 4; q++) m = fmaxf(m, acc[i][j][q]);
        if (y >= 0 && y < Tl::MI * 16 && (y & 15) < 4) {
#pragma unroll
            for (int i = 0; i < Tl::MI; i++)
#pragma unroll
                for (int q = 0; q < 4; q++)
                    if (y == i * 16 + q) a.at_target[r] = acc[i][j][q];
        }
        m = fmaxf(m, __shfl_xor(m, 16));
        m = fmaxf(m, __shfl_xor(m, 32));
        const float top = m == -INFINITY ? 0.0f : m;
        float sum = 0.0f;
#pragma unroll
        for (int i = 0; i < Tl::MI; i++)
#pragma unroll
            for (int q = 0; q < 4; q++) sum += fast_exp(acc[i][j][q] - top);
        sum += __shfl_xor(sum, 16);
        sum += __shfl_xor(sum, 32);
        if (lane < 16) {
            s_max[wm * S::BN + in] = m;
            s_sum[wm * S::BN + in] = sum;
        }
    }
    __syncthreads();
    for (int in = threadIdx.x; in < S::BN; in += S::kThreads) {
        if (r0 + in >= a.n) continue;
        float m = -INFINITY;
#pragma unroll
        for (int k = 0; k < S::WM; k++) m = fmaxf(m, s_max[k * S::BN + in]);
        const float from = m == -INFINITY ? 0.0f : m;
        float sum = 0.0f;
#pragma unroll
        for (int k = 0; k < S::WM; k++) sum += s_sum[k * S::BN + in] * fast_exp(s_max[k * S::BN + in] - from);
        a.part[(r0 + in) * a.tiles + (first + v0) / S::BM] = float2{m, sum};
    }
}

// A tile of 16-bit values goes through LDS, so that memory is written in whole rows of
// the tile.  It has `ROWS` rows of COLS values; pieces of 8 bytes are exchanged by the
// row's number.
template <int COLS>
__device__ __forceinline__ char* spot(char* lds, int row, int col) {
    static_assert(COLS >= 64, "16 pieces a row");
    return lds + row * COLS * 2 + ((col / 4 ^ ((row & 15) << 2) % (COLS / 4)) << 3);
}

// Four lanes' four 16-bit values each, turned: lane k of four gets value k of all four.
__device__ __forceinline__ uint2 turned(uint2 x) {
    const int lane = threadIdx.x & 3;
    const auto other = [](uint32_t v) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0xB1, 0xf, 0xf, false); };
    const auto across = [](uint32_t v) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x4E, 0xf, 0xf, false); };
    // Even lanes take the low halves of their own and the next lane's words, odd ones the high halves.
    const uint32_t pick = lane & 1 ? 0x03020706u : 0x05040100u;
    const uint32_t A = __builtin_amdgcn_perm(other(x.x), x.x, pick), B = __builtin_amdgcn_perm(other(x.y), x.y, pick);
    const uint32_t got = across(lane & 2 ? A : B);
    return lane & 2 ? uint2{got, B} : uint2{A, got};
}

// e of a piece of the vocabulary: e[n][ld], and with the rows' weights over their
// largest, turned, we[tokens][ld_turned].  Both orders, as matrix operands have their k in a row.  The logits' kernel
// but for its end, which writes: 345 to 365 us where that one takes 258 to 281, 537 MB in 86 us.
struct Errors {
    void *e, *we;      // either may be NULL
    int64_t tokens, rows;  // of the piece and of all, in whole steps
    int64_t ld, part, ld_turned, part_turned;
    int64_t first;     // token of the piece
};
template <typename T, typename S>
__global__ __launch_bounds__(S::kThreads, S::kWavesPerSimd) void errors_kernel(const Args a, const Operand head,
                                                                               const Operand hidden, int steps,
                                                                               const Errors o, int tm, int tn) {
    typedef Tile<T, S> Tl;
    constexpr int N = S::N;
    __shared__ __attribute__((aligned(16))) char lds[S::kLds];
    const Place at = place_of(blockIdx.x, tm, tn);
    const int64_t v0 = (int64_t)at.m * S::BM, r0 = (int64_t)at.n * S::BN;
    F4 acc[Tl::MI][Tl::NJ];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, wm = wave / S::WN, wn = wave % S::WN;
    const int vt = wm * Tl::MI * 16 + (lane >> 4) * 4, rt = wn * Tl::NJ * 16 + (lane & 15);  // in the tile
    // What the rows need is read before the products, whose first wait is for it too, rather than after them (4096 x 1024
    // x 32768: 7 us less), where registers are left.
    const float top = a.totals->weight;
    Row rows[Tl::NJ];
    float lses[Tl::NJ], w[Tl::NJ];
    const auto look = [&]() {
#pragma unroll
        for (int j = 0; j < Tl::NJ; j++) {
            const int64_t r = r0 + rt + j * 16;
            rows[j] = r < a.n ? a.rows[r] : Row{-1, 0.0f};
            lses[j] = r < a.n ? a.lse_in[r] : 0.0f;
        }
    };
    if (N == 1) look();
    Tl::run(head, hidden, v0, r0, 0, steps, lds, acc);
    if (N > 1) look();
    if (S::N > 1) unscale<S>(a, acc, v0 + vt, r0 + rt);
#pragma unroll
    for (int j = 0; j < Tl::NJ; j++) {
        const Row row = rows[j];
        const bool on = row.target >= 0;
        const float lse = on ? lses[j] : 0.0f;
        w[j] = on && top != 0.0f ? row.weight / top : 0.0f;
#pragma unroll
        for (int i = 0; i < Tl::MI; i++)
#pragma unroll
            for (int q = 0; q < 4; q++) {
                const float x = fast_exp(acc[i][j][q] - lse);
                acc[i][j][q] = on ? Matrix<T>::kScale * x : 0.0f;
            }
        const int64_t y = row.target - (o.first + v0 + vt);
        if (on && y >= 0 && y < Tl::MI * 16 && (y & 15) < 4) {
#pragma unroll
            for (int i = 0; i < Tl::MI; i++)
#pragma unroll
                for (int q = 0; q < 4; q++)
                    if (y == i * 16 + q) acc[i][j][q] -= Matrix<T>::kScale;
        }
    }
    if (o.first + v0 + S::BM > a.V) {
        const int64_t left = a.V - o.first - v0 - vt;
#pragma unroll
        for (int i = 0; i < Tl::MI; i++)
#pragma unroll
            for (int j = 0; j < Tl::NJ; j++)
#pragma unroll
                for (int q = 0; q < 4; q++)
                    if (i * 16 + q >= left) acc[i][j][q] = 0.0f;
    }
    // The parts of both orders in turn; a part is taken off what remains.
    typedef T T4 __attribute__((ext_vector_type(4)));
    typedef uint32_t Line __attribute__((ext_vector_type(4)));
#pragma unroll
    for (int order = 0; order < 2; order++) {
        void* out = order == 0 ? o.e : o.we;
        if (out == nullptr) continue;
#pragma unroll
        for (int part = 0; part < N; part++) {
            if (order + part > 0) __syncthreads();
#pragma unroll
            for (int j = 0; j < Tl::NJ; j++)
#pragma unroll
                for (int i = 0; i < Tl::MI; i++) {
                    F4 x = order == 0 ? acc[i][j] : acc[i][j] * w[j];
                    // A product rounded to 32 bits: folded into the cut it would be rounded otherwise for one part
                    // than for the other.  And it is cut anew: parts kept from the last time would fill the registers.
                    if (N > 1) asm volatile("" : "+v"(x));
                    T4 e;
                    if constexpr (N == 1) {
                        e = __builtin_convertvector(x, T4);
                    } else {
#pragma unroll
                        for (int q = 0; q < 4; q++) {
                            T p[N];
                            cut<T, N>(x[q], p);
                            e[q] = p[part];
                        }
                    }
                    uint2 bits = __builtin_bit_cast(uint2, e);
                    if (order == 0) {
                        *reinterpret_cast<uint2*>(spot<S::BM>(lds, rt + j * 16, vt + i * 16)) = bits;
                    } else {
                        // Lane k of four has token vt + k, and the four lanes' rows.
                        bits = turned(bits);
                        *reinterpret_cast<uint2*>(spot<S::BN>(lds, vt + i * 16 + (lane & 3), (rt + j * 16) & ~3)) = bits;
                    }
                }
            __syncthreads();
            // 16 bytes a lane, rows of the tile after each other.
            constexpr int COLS[2] = {S::BM, S::BN}, ROWS[2] = {S::BN, S::BM};
            const int64_t row0 = order == 0 ? r0 : v0, col0 = order == 0 ? v0 : r0;
            const int64_t rows = order == 0 ? a.n : o.tokens, cols = order == 0 ? o.tokens : o.rows;
            const int64_t ld = order == 0 ? o.ld : o.ld_turned;
            T* to = static_cast<T*>(out) + part * (order == 0 ? o.part : o.part_turned);
#pragma unroll 4
            for (int k = threadIdx.x; k < ROWS[order] * (COLS[order] / 8); k += S::kThreads) {
                const int row = k / (COLS[order] / 8), col = k % (COLS[order] / 8) * 8;
                const char* from = order == 0 ? spot<S::BM>(lds, row, col) : spot<S::BN>(lds, row, col);
                if (row0 + row < rows && col0 + col < cols)
                    *reinterpret_cast<Line*>(to + (row0 + row) * ld + col0 + col) = *reinterpret_cast<const Line*>(from);
            }
        }
    }
}

// Times f 2^e, which together may lie in range where neither alone does.
struct Factor {
    float m;
    int32_t e;
    __device__ __forceinline__ Factor(float f, int32_t exponent)
        : m(__builtin_amdgcn_frexp_mantf(f)), e(__builtin_amdgcn_frexp_expf(f) + exponent) {}
    __device__ __forceinline__ float operator()(float x) const { return ldexpf(x * m, e); }
};

// Both gradients of a piece in one launch, the workgroups of dh first: their k is longer.  4096 x 1024 x 32768 bf16:
// 484 to 507 us, 1090 to 1140 TFLOP/s (torch's products one after the other 551); 1519 x 1003 x 50001 fp16: 340 to 360, 850 to
// 900, 3.8 rounds of tiles and rows of dW off a line.
struct Gradients {
    Operand wt, er;         // of dh: W^T, e
    Operand ht, we;         // of dW: h^T, (c e)^T
    float* slab;            // [splits][n][ld]: dh so far; a split of the piece's tokens each
    float* slab_head;       // [splits_n][tokens][ld]: dW where the rows are split
    void* dhead;            // the piece's first row
    void* dhidden;          // where dh is one sum, written here and not to the slab
    int64_t ld;
    int32_t steps_v, steps_n, splits, splits_n, add;
    int32_t dh_blocks, tm, tn_rows, tn_tokens;  // tiles across D, down the rows and the tokens
};
// What the sums of a row of dh, per weight, and of dW are multiplied by.
template <typename T>
__device__ __forceinline__ float rows_factor(const Args& a) {
    return a.totals->share * a.grad_scale * (a.grad_loss ? *a.grad_loss : 1.0f) / Matrix<T>::kScale;
}
template <typename T>
__device__ __forceinline__ float head_factor(const Args& a) {
    return a.totals->weight * rows_factor<T>(a);
}
// A tile of a gradient, columns from d0 and `rows` - row0 rows at most, each times by[j] 2^e, or 0 where it is not on.
template <typename E, typename S>
__device__ __forceinline__ void put_tile(const F4 (&acc)[S::MI][S::NJ], char* lds, E* out, int64_t rows, int64_t D, int64_t row0,
                                         int64_t d0, int nt, int dt, const float (&by)[S::NJ], const bool (&on)[S::NJ], int32_t e) {
    if constexpr (sizeof(E) == 4) {
        // 16 bytes a lane as they are.
#pragma unroll
        for (int j = 0; j < S::NJ; j++) {
            const int64_t r = row0 + nt + j * 16;
            if (r >= rows) continue;
            const Factor times(by[j], e);
#pragma unroll
            for (int i = 0; i < S::MI; i++) {
                const int64_t d = d0 + dt + i * 16;
                float f[4];
#pragma unroll
                for (int q = 0; q < 4; q++) f[q] = on[j] ? times(acc[i][j][q]) : 0.0f;
                if (d + 4 <= D) {
                    Vec<E, 4>::store(out + r * D + d, f);
                } else {
#pragma unroll
                    for (int q = 0; q < 4; q++)
                        if (d + q < D) out[r * D + d + q] = (E)f[q];
                }
            }
        }
    } else {
        typedef E E4 __attribute__((ext_vector_type(4)));
        typedef uint32_t Line __attribute__((ext_vector_type(4)));
        typedef Line LooseLine __attribute__((aligned(2)));
#pragma unroll
        for (int j = 0; j < S::NJ; j++)
#pragma unroll
            for (int i = 0; i < S::MI; i++) {
                E4 f;
#pragma unroll
                for (int q = 0; q < 4; q++) f[q] = on[j] ? (E)(acc[i][j][q] * by[j]) : (E)0.0f;
                *reinterpret_cast<uint2*>(spot<S::BM>(lds, nt + j * 16, dt + i * 16)) = __builtin_bit_cast(uint2, f);
            }
        __syncthreads();
#pragma unroll 4
        for (int k = threadIdx.x; k < S::BN * (S::BM / 8); k += S::kThreads) {
            const int row = k / (S::BM / 8), col = k % (S::BM / 8) * 8;
            if (row0 + row >= rows || d0 + col >= D) continue;
            E* to = out + (row0 + row) * D + d0 + col;
            const char* from = spot<S::BM>(lds, row, col);
            if (d0 + col + 8 <= D) {
                *reinterpret_cast<LooseLine*>(to) = *reinterpret_cast<const Line*>(from);
            } else {
                for (int q = 0; q < 8 && d0 + col + q < D; q++) to[q] = reinterpret_cast<const E*>(from)[q];
            }
        }
    }
}
template <typename E, typename T, typename S>
__global__ __launch_bounds__(S::kThreads, S::kWavesPerSimd) void gradients_kernel(const Args a, const Gradients g) {
    typedef Tile<T, S> Tl;
    __shared__ __attribute__((aligned(16))) char lds[S::kLds];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, wm = wave / S::WN, wn = wave % S::WN;
    const int dt = wm * Tl::MI * 16 + (lane >> 4) * 4, nt = wn * Tl::NJ * 16 + (lane & 15);  // in the tile
    F4 acc[Tl::MI][Tl::NJ];
    float by[Tl::NJ];
    bool on[Tl::NJ];
    if ((int)blockIdx.x < g.dh_blocks) {
        const int split = blockIdx.x % g.splits;
        const Place at = place_of(blockIdx.x / g.splits, g.tm, g.tn_rows);
        const int64_t d0 = (int64_t)at.m * S::BM, r0 = (int64_t)at.n * S::BN;
        const int from = (int)((int64_t)g.steps_v * split / g.splits), to = (int)((int64_t)g.steps_v * (split + 1) / g.splits);
        Tl::run(g.wt, g.er, d0, r0, (int64_t)from * kStep, to - from, lds, acc);
        if (g.dhidden) {
            const float all = rows_factor<T>(a);
#pragma unroll
            for (int j = 0; j < Tl::NJ; j++) {
                const int64_t r = r0 + nt + j * 16;
                const Row row = r < a.n ? a.rows[r] : Row{-1, 0.0f};
                on[j] = row.target >= 0;
                by[j] = row.weight * all;
            }
            put_tile<E, S>(acc, lds, static_cast<E*>(g.dhidden), a.n, a.D, r0, d0, nt, dt, by, on, sizeof(E) == 4 ? -a.scales->head : 0);
            return;
        }
#pragma unroll
        for (int j = 0; j < Tl::NJ; j++) {
            const int64_t r = r0 + nt + j * 16;
            if (r >= a.n) continue;
#pragma unroll
            for (int i = 0; i < Tl::MI; i++) {
                const int64_t d = d0 + dt + i * 16;
                if (d >= g.ld) continue;
                F4* to = reinterpret_cast<F4*>(g.slab + (split * a.n + r) * g.ld + d);
                *to = g.add ? *to + acc[i][j] : acc[i][j];
            }
        }
        return;
    }
    const int split = (blockIdx.x - g.dh_blocks) % g.splits_n;
    const Place at = place_of((blockIdx.x - g.dh_blocks) / g.splits_n, g.tm, g.tn_tokens);
    const int64_t d0 = (int64_t)at.m * S::BM, v0 = (int64_t)at.n * S::BN;
    const int from = (int)((int64_t)g.steps_n * split / g.splits_n), to = (int)((int64_t)g.steps_n * (split + 1) / g.splits_n);
    Tl::run(g.ht, g.we, d0, v0, (int64_t)from * kStep, to - from, lds, acc);
    if (g.splits_n > 1) {
#pragma unroll
        for (int j = 0; j < Tl::NJ; j++) {
            const int64_t v = v0 + nt + j * 16;
            if (v >= g.we.rows) continue;
#pragma unroll
            for (int i = 0; i < Tl::MI; i++) {
                const int64_t d = d0 + dt + i * 16;
                if (d < g.ld) *reinterpret_cast<F4*>(g.slab_head + (split * g.we.rows + v) * g.ld + d) = acc[i][j];
            }
        }
        return;
    }
    const float all = head_factor<T>(a);
#pragma unroll
    for (int j = 0; j < Tl::NJ; j++) {
        on[j] = true;
        by[j] = all;
    }
    put_tile<E, S>(acc, lds, static_cast<E*>(g.dhead), g.we.rows, a.D, v0, d0, nt, dt, by, on, sizeof(E) == 4 ? -a.scales->hidden : 0);
}

// Sums over the splits of dW of a piece, and of dh after the last piece, times what
// each is to be multiplied by: dh of a.n rows, or none, then `tokens` rows of dW, or none.  4 splits of 4096 x 1024
// in 32 bits: 18 us (76 MB, latency at this size).
template <typename E, typename T>
__global__ __launch_bounds__(kThreads) void splits_kernel(const Args a, const Gradients g, int64_t tokens, E* dhidden) {
    const int64_t per_row = (a.D + 3) / 4, rows = dhidden ? a.n : 0;
    const float by = rows_factor<T>(a);
    for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < (rows + tokens) * per_row;
         i += (int64_t)gridDim.x * kThreads) {
        const int64_t r = i / per_row, d = i % per_row * 4;
        const bool head = r >= rows;
        const float* slab = head ? g.slab_head + (r - rows) * g.ld + d : g.slab + r * g.ld + d;
        const int64_t next = (head ? tokens : a.n) * g.ld;
        const int splits = head ? g.splits_n : g.splits;
        E* out = head ? static_cast<E*>(g.dhead) + (r - rows) * a.D + d : dhidden + r * a.D + d;
        const Row row = head ? Row{0, 0.0f} : a.rows[r];
        F4 v = {0.0f, 0.0f, 0.0f, 0.0f};
        if (row.target >= 0) {
#pragma unroll 4
            for (int k = 0; k < splits; k++) v += *reinterpret_cast<const F4*>(slab + k * next);
            const float f = head ? head_factor<T>(a) : row.weight * by;
            if constexpr (sizeof(E) == 4) {
                const Factor times(f, head ? -a.scales->hidden : -a.scales->head);
#pragma unroll
                for (int q = 0; q < 4; q++) v[q] = times(v[q]);
            } else {
                v *= f;
            }
        }
        const float f[4] = {v[0], v[1], v[2], v[3]};
        if (d + 4 <= a.D) {
            Vec<E, 4>::store(out, f);
        } else {
#pragma unroll
            for (int q = 0; q < 4; q++)
                if (d + q < a.D) out[q] = (E)f[q];
        }
    }
}

// --- the plan -------------------------------------------------------------------

inline int64_t up(int64_t x, int64_t m) { return (x + m - 1) / m * m; }
// Rows that begin whole kilobytes apart would meet in few channels of the L2.
inline int64_t pitch(int64_t len) { return len % 512 == 0 ? len + 64 : len; }
inline int64_t tiles(int64_t x, int64_t m) { return (x + m - 1) / m; }

// Sizes of tiles.  Few rows leave the products to memory, and small tiles keep many
// steps on their way; few tiles leave units idle, and small ones are more (300 rows of 2048, 1000
// tokens, bf16: 58 us, and 84 with middle ones; 8192 x 512 x 1000, 512 middle tiles: 99 with small
// ones and 88); otherwise big ones where they fill the GPU.
enum Size { kSmall, kMiddle, kBig };
Size size_of(int64_t m, int64_t n, int64_t rows) {
    if (rows <= 64) return kSmall;
    if (tiles(m, 128) * tiles(n, 128) < 256) return kSmall;
    return tiles(m, 256) * tiles(n, 256) >= 192 ? kBig : kMiddle;
}
// Workgroups of a product that splits should fill the GPU's 256 units with: as many as LDS holds, but one of two of the
// middle tiles of two parts, whose splits beyond that cost more than they share (fp32, backward: 1000 x 512 x 8192 135 to 138 us
// so and 147 with two, 3000 x 1024 x 3000 230 and 246; five other sizes within 1%).
int64_t slots_of(Size s, int parts) { return s == kBig || (s == kMiddle && parts > 1) ? 256 : 512; }
int edge(Size s) { return s == kBig ? 256 : s == kMiddle ? 128 : 64; }

// Where everything lies in the workspace.
struct Plan {
    int parts = 0;                       // of a value
    int64_t ldk = 0, ldn = 0, ldv = 0;   // padded D, n and tokens of a piece
    int64_t piece = 0, loss_piece = 0;   // tokens of a piece, backward and forward
    Size logits = kMiddle, errors = kMiddle, gradients = kMiddle;
    int tiles = 0;                       // tiles of tokens, forward
    int splits = 0, splits_n = 0;        // of the tokens for dh, of the rows for dW
    bool direct = false;                 // dh is one sum
    int64_t rows = 0, totals = 0, scales = 0, hidden_scale = 0, head_scale = 0, largest = 0, sums = 0, counts = 0, tops = 0, at_target = 0, part = 0;
    int64_t hidden = 0, head = 0, head_piece = 0, hidden_t = 0, head_t = 0, e = 0, we = 0, slab = 0, slab_head = 0;
    int64_t bytes_loss = 0, bytes_backward = 0;
};

bool plain_rows(int32_t dtype, const void* p, int64_t row, int64_t D) {
    return dtype != GEAR_DTYPE_F32 && D % kStep == 0 && row % 8 == 0 && reinterpret_cast<uintptr_t>(p) % 16 == 0;
}

// The workspace holds what any alignment of the operands needs.
Plan plan_of(const gear_token_desc& d) {
    Plan p;
    p.parts = d.dtype == GEAR_DTYPE_F32 ? Parts<float>::kCount : 1;
    p.ldk = up(d.D, kStep);
    p.ldn = up(d.n, kStep);
    int64_t piece = kPieceValues / (d.n > 0 ? d.n : 1) / p.parts / 256 * 256;
    piece = piece < 256 ? 256 : piece > kPieceTokens ? kPieceTokens : piece;
    p.piece = piece < d.V ? piece : d.V;
    p.loss_piece = kPieceTokens < d.V ? kPieceTokens : d.V;
    p.ldv = up(p.piece, kStep);
    p.logits = size_of(p.loss_piece, d.n, d.n);
    p.errors = size_of(p.piece, d.n, d.n);
    p.gradients = d.n <= 64 ? kSmall : size_of(d.D, p.piece + d.n, d.n);
    p.tiles = (int)tiles(d.V, edge(p.logits));
    // Few tiles of dh share the GPU by splitting the tokens, while they then run all at once: 24 big tiles (1519 x 1003 x 50001
    // fp16, backward) take 625 us in 8 splits and 657 in 16, of which the second half would follow the first and the slab be
    // twice as large (1500 x 1024 x 20000 bf16: 218 and 255).  And from 16 steps on: one sum is written as dh itself, and
    // splits cost their slab and a launch (fp32, rows of 64, forward and backward: 500 rows and tokens 38.7 us whole and 41.2
    // in two; 1000 rows and tokens 46.2 whole and 44.5 in four).
    const int64_t slots = slots_of(p.gradients, p.parts);
    const int64_t dh = tiles(d.D, edge(p.gradients)) * tiles(d.n, edge(p.gradients)), steps = p.ldv / kStep;
    p.splits = 1;
    while (dh * p.splits * 2 <= slots && steps >= 16 && p.splits * 8 <= steps && p.splits < 16) p.splits *= 2;
    p.direct = p.splits == 1 && p.piece >= d.V;
    // So do few tiles of dW, splitting the rows: 65536 rows of 64, a head of 18, bf16, forward and backward take 93 us so
    // and 1490 with the rows in one piece.
    const int64_t dw = tiles(d.D, edge(p.gradients)) * tiles(p.piece, edge(p.gradients));
    p.splits_n = 1;
    const int64_t steps_n = p.ldn / kStep;
    while (dw * p.splits_n * 2 <= slots && steps_n >= 16 && p.splits_n * 8 <= steps_n && p.splits_n < 64) p.splits_n *= 2;
    int64_t at = 0;
    const auto take = [&](int64_t bytes) {
        const int64_t here = at;
        at += up(bytes, 256);
        return here;
    };
    p.rows = take(d.n * (int64_t)sizeof(Row));
    p.totals = take(sizeof(Totals));
    p.scales = take(sizeof(Scales));
    // Whole tiles of tokens.
    p.hidden_scale = take(p.parts > 1 ? d.n * 4 : 0);
    p.head_scale = take(p.parts > 1 ? up(p.piece > p.loss_piece ? p.piece : p.loss_piece, 256) * 4 : 0);
    p.largest = take(2 * kParts * sizeof(uint32_t));
    p.sums = take(kParts * sizeof(double));
    p.counts = take(kParts * sizeof(int64_t));
    p.tops = take(kParts * sizeof(float));
    p.hidden = take(d.n * pitch(p.ldk) * p.parts * 2);
    const int64_t common = at;
    p.at_target = take(d.n * 4);
    p.part = take(d.n * (int64_t)p.tiles * (int64_t)sizeof(float2));
    p.head = take(p.loss_piece * pitch(p.ldk) * p.parts * 2);
    p.bytes_loss = at;
    at = common;
    p.head_piece = take(p.piece * pitch(p.ldk) * p.parts * 2);
    p.hidden_t = take(d.D * pitch(p.ldn) * p.parts * 2);
    p.head_t = take(d.D * (p.ldv + 64) * p.parts * 2);
    p.e = take(d.n * (p.ldv + 64) * p.parts * 2);
    p.we = take(p.ldv * pitch(p.ldn) * p.parts * 2);
    if (!p.direct) p.slab = take(p.splits * d.n * p.ldk * 4);
    if (p.splits_n > 1) p.slab_head = take(p.splits_n * p.piece * p.ldk * 4);
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
    a.scales = reinterpret_cast<Scales*>(work + p.scales);
    a.hidden_scale = reinterpret_cast<int32_t*>(work + p.hidden_scale);
    a.head_scale = reinterpret_cast<int32_t*>(work + p.head_scale);
    a.largest = reinterpret_cast<uint32_t*>(work + p.largest);
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
    a.row_parts = d.n <= kSoloRows ? 1 : (int32_t)some_blocks(d.n, kParts);
    a.max_parts = (int32_t)some_blocks((d.n > d.V ? d.n : d.V) * ((d.D + 3) / 4), kParts);
    a.denom = d.denom;
    a.grad_scale = d.grad_scale;
    return a;
}

template <typename E>
struct Call {
    typedef typename Parts<E>::T T;
    static constexpr int N = Parts<E>::kCount;
    typedef typename Shapes<N>::Big Big;
    typedef typename Shapes<N>::Middle Middle;
    typedef typename Shapes<N>::Small Small;
    const gear_token_desc& d;
    const Plan p;
    char* work;
    hipStream_t s;

    // An operand of rows as they lie, or of a copy that `job` makes.
    Operand operand(const void* src, int64_t rows, int64_t ld_src, int64_t to, int32_t* scale, Job& job) const {
        if (plain_rows(d.dtype, src, ld_src, d.D)) return Operand{src, rows, ld_src, 0};
        job = Job{src, work + to, scale, rows, d.D, ld_src, p.ldk, pitch(p.ldk), rows * pitch(p.ldk), 0, 0};
        return Operand{work + to, rows, pitch(p.ldk), rows * pitch(p.ldk)};
    }
    // A turned copy: d.D rows of ld values.
    Operand turned_operand(const void* src, int64_t rows, int64_t ld_src, int64_t len, int64_t to, bool on, Job& job) const {
        const int64_t ld = pitch(len);
        job = Job{src, work + to, nullptr, rows, d.D, ld_src, len, ld, d.D * ld, 0, on ? 1 : 0};
        return Operand{work + to, d.D, ld, d.D * ld};
    }
    // The scales of 32-bit values: before anything is turned.
    hipError_t look(const Args& a, const void* hidden, const void* head) const {
        if constexpr (N > 1) {
            hipLaunchKernelGGL(largest_kernel, dim3(2 * a.max_parts), dim3(kThreads), 0, s, a, static_cast<const float*>(hidden),
                               d.hidden_row, static_cast<const float*>(head), d.head_row);
            return hipGetLastError();
        }
        return hipSuccess;
    }
    // Nothing to do costs no launch.
    hipError_t prepare(const Args& a, Jobs& j, bool rows) const {
        int32_t at = j.row_blocks = rows ? a.row_parts : 0;
        for (Job& c : j.copy) {
            c.first = at;
            if (c.src) at += (int32_t)some_blocks(c.rows * (N > 1 ? lanes_of(c.len / 8) : c.len / 8), 4096);
        }
        for (Job& c : j.turn) {
            c.first = at;
            if (c.src) at += (int32_t)(tiles(c.len, 64) * tiles(c.cols, 64) < 8192 ? tiles(c.len, 64) * tiles(c.cols, 64) : 8192);
        }
        j.blocks = at;
        if (at == 0) return hipSuccess;
        hipLaunchKernelGGL(prepare_kernel<E>, dim3((unsigned)at), dim3(kThreads), 0, s, a, j);
        if (rows && a.row_parts > 1) hipLaunchKernelGGL(totals_kernel, dim3(1), dim3(64), 0, s, a);
        return hipGetLastError();
    }

    template <typename S>
    hipError_t logits(const Args& a, const Operand& x, const Operand& y, int64_t first) const {
        const int tm = (int)tiles(x.rows, S::BM), tn = (int)tiles(a.n, S::BN);
        hipLaunchKernelGGL((logits_kernel<T, S>), dim3((unsigned)(tm * tn)), dim3(S::kThreads), 0, s, a, x, y,
                           (int)(p.ldk / kStep), first, tm, tn);
        return hipGetLastError();
    }
    template <int LANES>
    hipError_t join(Args a) const {
        // One workgroup where it has few rounds, and a launch less.
        const int64_t want = tiles(a.n * LANES, kThreads);
        a.lse_parts = (int32_t)(want <= 4 ? 1 : want < kParts ? want : kParts);
        hipLaunchKernelGGL(lse_kernel<LANES>, dim3(a.lse_parts), dim3(kThreads), 0, s, a);
        if (a.lse_parts > 1) hipLaunchKernelGGL(loss_kernel, dim3(1), dim3(64), 0, s, a);
        return hipGetLastError();
    }
    hipError_t loss(Args a, const void* hidden, const void* head) const {
        a.at_target = reinterpret_cast<float*>(work + p.at_target);
        a.part = reinterpret_cast<float2*>(work + p.part);
        hipError_t e = hipSuccess;
        for (int64_t first = 0; first < a.V && a.n > 0; first += p.loss_piece) {
            const int64_t tokens = a.V - first < p.loss_piece ? a.V - first : p.loss_piece;
            Jobs j{};
            const Operand x = operand(static_cast<const E*>(head) + first * d.head_row, tokens, d.head_row, p.head, a.head_scale, j.copy[0]);
            Operand y = operand(hidden, a.n, d.hidden_row, p.hidden, a.hidden_scale, j.copy[1]);
            if (first > 0) j.copy[1] = Job{};
            if ((e = prepare(a, j, false)) != hipSuccess) return e;
            e = p.logits == kBig ? logits<Big>(a, x, y, first) : p.logits == kMiddle ? logits<Middle>(a, x, y, first)
                                                                                      : logits<Small>(a, x, y, first);
            if (e != hipSuccess) return e;
        }
        return p.tiles <= 4 ? join<1>(a) : p.tiles <= 32 ? join<8>(a) : join<64>(a);
    }

    template <typename S>
    hipError_t errors(const Args& a, const Operand& x, const Operand& y, const Errors& o) const {
        const int tm = (int)tiles(o.tokens, S::BM), tn = (int)tiles(p.ldn, S::BN);
        hipLaunchKernelGGL((errors_kernel<T, S>), dim3((unsigned)(tm * tn)), dim3(S::kThreads), 0, s, a, x, y,
                           (int)(p.ldk / kStep), o, tm, tn);
        return hipGetLastError();
    }
    template <typename S>
    hipError_t gradients(const Args& a, Gradients g, bool dhidden, bool dhead, int64_t tokens) const {
        g.tm = (int)tiles(a.D, S::BM);
        g.tn_rows = (int)tiles(a.n, S::BN);
        g.tn_tokens = (int)tiles(tokens, S::BN);
        g.dh_blocks = dhidden ? g.splits * g.tm * g.tn_rows : 0;
        const int blocks = g.dh_blocks + (dhead ? g.splits_n * g.tm * g.tn_tokens : 0);
        hipLaunchKernelGGL((gradients_kernel<E, T, S>), dim3((unsigned)blocks), dim3(S::kThreads), 0, s, a, g);
        return hipGetLastError();
    }
    hipError_t backward(const Args& a, const void* hidden, const void* head, void* dhidden, void* dhead) const {
        hipError_t e = look(a, hidden, head);
        if (e != hipSuccess) return e;
        float* slab = reinterpret_cast<float*>(work + p.slab);
        for (int64_t first = 0; first < a.V; first += p.piece) {
            const int64_t tokens = a.V - first < p.piece ? a.V - first : p.piece, ldv = up(tokens, kStep);
            const E* from = static_cast<const E*>(head) + first * d.head_row;
            Jobs j{};
            Gradients g{};
            const Operand x = operand(from, tokens, d.head_row, p.head_piece, a.head_scale, j.copy[0]);
            const Operand y = operand(hidden, a.n, d.hidden_row, p.hidden, a.hidden_scale, j.copy[1]);
            if (dhead) g.ht = turned_operand(hidden, a.n, d.hidden_row, p.ldn, p.hidden_t, true, j.turn[0]);
            if (dhidden) g.wt = turned_operand(from, tokens, d.head_row, ldv, p.head_t, false, j.turn[1]);
            if (first > 0) j.copy[1] = j.turn[0] = Job{};  // made for the first piece
            if ((e = prepare(a, j, first == 0)) != hipSuccess) return e;
            Errors o{};
            o.e = dhidden ? work + p.e : nullptr;
            o.we = dhead ? work + p.we : nullptr;
            o.tokens = ldv;
            o.rows = p.ldn;
            o.ld = pitch(ldv);
            o.part = a.n * o.ld;
            o.ld_turned = pitch(p.ldn);
            o.part_turned = ldv * o.ld_turned;
            o.first = first;
            e = p.errors == kBig ? errors<Big>(a, x, y, o) : p.errors == kMiddle ? errors<Middle>(a, x, y, o)
                                                                                  : errors<Small>(a, x, y, o);
            if (e != hipSuccess) return e;
            g.er = Operand{work + p.e, a.n, o.ld, o.part};
            g.we = Operand{work + p.we, tokens, o.ld_turned, o.part_turned};
            g.slab = slab;
            g.slab_head = reinterpret_cast<float*>(work + p.slab_head);
            g.dhead = dhead ? static_cast<E*>(dhead) + first * a.D : nullptr;
            g.dhidden = p.direct ? dhidden : nullptr;
            g.ld = p.ldk;
            g.steps_v = (int32_t)(ldv / kStep);
            g.steps_n = (int32_t)(p.ldn / kStep);
            g.splits = p.splits;
            g.splits_n = p.splits_n;
            g.add = first > 0 ? 1 : 0;
            e = p.gradients == kBig      ? gradients<Big>(a, g, dhidden != nullptr, dhead != nullptr, tokens)
                : p.gradients == kMiddle ? gradients<Middle>(a, g, dhidden != nullptr, dhead != nullptr, tokens)
                                         : gradients<Small>(a, g, dhidden != nullptr, dhead != nullptr, tokens);
            if (e != hipSuccess) return e;
            // What is left in splits: dW of this piece, dh after the last.
            const bool last = first + p.piece >= a.V;
            const int64_t heads = dhead && p.splits_n > 1 ? tokens : 0, rows = dhidden && last && !p.direct ? a.n : 0;
            if (heads + rows == 0) continue;
            hipLaunchKernelGGL((splits_kernel<E, T>), dim3(some_blocks((heads + rows) * ((a.D + 3) / 4), 8192)), dim3(kThreads), 0,
                               s, a, g, heads, rows ? static_cast<E*>(dhidden) : nullptr);
            if ((e = hipGetLastError()) != hipSuccess) return e;
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
