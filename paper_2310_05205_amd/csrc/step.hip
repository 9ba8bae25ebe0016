// The optimizer's step of many tensors at once, and the norm of their gradients
// (include/gear.h).  A value is read, updated in 32 bits and written in one pass;
// the averages are held in 32 bits, or in e4m3 with a scale per 256 values:
//   m = q s,  v = (q' s')^2,  s = max |.| / 448 over the block.
// The second average is held by its root: e4m3 reaches over 17 powers of two below a
// block's largest, and the root needs half of what v itself would.  The first one of a
// value without a gradient is rounded towards 0: to nearest, beta1 m is m again where
// 1 - beta1 of it is less than half a step of e4m3 (multiples of 2^-9 up to 4 of them at
// 0.9, values of any size at 0.95), and the parameter would go on moving.
//
// Tensors travel in the kernel's arguments, 56 a launch, so a call needs no table
// on the device and a captured call keeps its own.
//
// The bytes bound it: 218 M bf16 values with masters and 32-bit averages, their norm
// among it, take 1120 to 1280 us (boxes differ), 5.1 to 5.9 TB/s; a plain copy reaches 5.1.
#include <math.h>

#include "element.h"
#include "gear_internal.h"

namespace gear {
namespace {

constexpr int kThreads = 256;
constexpr int kValues = 8;                           // values a lane takes at a time
constexpr int kRound = kThreads * kValues;           // values of a workgroup at a time
// Values of a workgroup: four rounds, or one where the whole step has few (26000 values in 13
// tensors: the update takes 8.6 us with four, 5 with one).
constexpr int kChunk = 4 * kRound;
constexpr int64_t kFewValues = 1 << 21;
constexpr int kItems = 56;                           // tensors of one launch
constexpr int kGrads = 160;                          // gradients of one launch of the norm
constexpr int kGroup = GEAR_STEP_BLOCK / kValues;    // lanes of an 8-bit block
constexpr int kNormBlocks = 1024;
constexpr float kTop = 448.0f, kLeast = 0.001953125f;  // e4m3: its largest value, and its least above 0
constexpr float kNothing = 7.888609e-31f;              // 2^-100

struct Item {
    const void* grad;
    void *param, *m, *v;
    float *master, *ms, *vs;
    int64_t n;
};
struct Grad {
    const void* grad;
    int64_t n;
};
template <typename I, int N>
struct List {
    I item[N];
    uint32_t first[N + 1];  // chunks before each tensor
    int32_t count, chunk;   // values of a chunk
};
typedef List<Item, kItems> Items;
typedef List<Grad, kGrads> Grads;

// What a step multiplies by; made once on the device.
struct Factors {
    float grad, decay, rate, root;  // factor, 1 - lr weight_decay, lr / (1 - beta1^s), (1 - beta2^s)^-1/2
    int32_t skip;
};

// The tensor that a chunk belongs to.
template <typename L>
__device__ __forceinline__ int item_of(const L& t, uint32_t chunk) {
    int lo = 0, hi = t.count;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (t.first[mid] <= chunk) lo = mid;
        else hi = mid;
    }
    return lo;
}

template <int N, bool STREAM, typename E>
__device__ __forceinline__ void load(const E* p, int64_t left, float (&f)[N]) {
    if (left >= N) {
        Vec<E, N>::unpack(Vec<E, N>::template load<STREAM>(p), f);
    } else {
#pragma unroll
        for (int j = 0; j < N; j++) f[j] = j < left ? (float)p[j] : 0.0f;
    }
}
template <int N, bool STREAM, typename E>
__device__ __forceinline__ void store(E* p, int64_t left, const float (&f)[N]) {
    if (left >= N) {
        Vec<E, N>::template store<STREAM>(p, f);
    } else {
#pragma unroll
        for (int j = 0; j < N; j++)
            if (j < left) p[j] = (E)f[j];
    }
}

typedef uint32_t Bytes __attribute__((ext_vector_type(2)));
typedef Bytes LooseBytes __attribute__((aligned(1)));
// The root by the hardware's instruction, which is within one unit, of normal numbers alone: what is smaller is scaled.
__device__ __forceinline__ float root_of(float v) {
    const bool small = v < 1.2621774e-29f;  // 2^-96
    const float r = __builtin_amdgcn_sqrtf(small ? v * 1.8446744e19f : v);
    return small ? r * 2.3283064e-10f : r;
}
template <bool STREAM>
__device__ __forceinline__ void load8(const uint8_t* p, int64_t left, float scale, float (&f)[kValues]) {
    Bytes b = {0, 0};
    if (left >= kValues) {
        const LooseBytes* at = reinterpret_cast<const LooseBytes*>(p);
        b = STREAM ? __builtin_nontemporal_load(at) : *at;
    } else {
#pragma unroll
        for (int j = 0; j < kValues; j++)
            if (j < left) b[j / 4] |= (uint32_t)p[j] << (8 * (j % 4));
    }
#pragma unroll
    for (int j = 0; j < kValues; j += 4) {
        const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)b[j / 4], false);
        const auto hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)b[j / 4], true);
        f[j] = lo[0] * scale;
        f[j + 1] = lo[1] * scale;
        f[j + 2] = hi[0] * scale;
        f[j + 3] = hi[1] * scale;
    }
}
// The e4m3 value next to x, |x| <= kTop, towards 0.  2^-20 more than x: what was such a value before roundings stays one.
__device__ __forceinline__ float towards_0(float x) {
    const float a = fminf(fabsf(x) * (1.0f + 9.5367432e-07f), kTop);
    const float normal = __builtin_bit_cast(float, __builtin_bit_cast(uint32_t, a) & 0xFFF00000u);  // 3 bits after the first
    return copysignf(a < 8.0f * kLeast ? truncf(a * (1.0f / kLeast)) * kLeast : normal, x);
}
// A lane's values of a block, under the block's scale, which is returned: to nearest, what is not 0 to no less than kLeast;
// those of the bits `fading` towards 0.
template <bool STREAM>
__device__ __forceinline__ float store8(uint8_t* p, int64_t left, const float (&f)[kValues], uint32_t fading) {
    float top = 0.0f;
#pragma unroll
    for (int j = 0; j < kValues; j++) top = fmaxf(top, fabsf(f[j]));
#pragma unroll
    for (int off = 1; off < kGroup; off <<= 1) top = fmaxf(top, __shfl_xor(top, off));
    const bool some = top >= kNothing;
    const float inv = some ? kTop * __builtin_amdgcn_rcpf(top) : 0.0f;
    Bytes b;
#pragma unroll
    for (int j = 0; j < kValues; j += 4) {
        float q[4];
#pragma unroll
        for (int k = 0; k < 4; k++) {
            const float x = f[j + k] * inv;
            q[k] = x;
            // Comparisons that a NaN passes through.
            if (fabsf(x) > kTop) q[k] = copysignf(kTop, x);
            if (fabsf(x) < kLeast) q[k] = f[j + k] != 0.0f && some ? copysignf(kLeast, x) : 0.0f;
            if ((fading >> (j + k) & 1) != 0 && x == x) q[k] = towards_0(x);
        }
        int w = __builtin_amdgcn_cvt_pk_fp8_f32(q[0], q[1], 0, false);
        w = __builtin_amdgcn_cvt_pk_fp8_f32(q[2], q[3], w, true);
        b[j / 4] = (uint32_t)w;
    }
    if (left >= kValues) {
        LooseBytes* at = reinterpret_cast<LooseBytes*>(p);
        if (STREAM) __builtin_nontemporal_store(b, at);
        else *at = b;
    } else {
#pragma unroll
        for (int j = 0; j < kValues; j++)
            if (j < left) p[j] = (uint8_t)(b[j / 4] >> (8 * (j % 4)));
    }
    return some ? top * (1.0f / kTop) : 0.0f;
}

// The step's factors, and the step counted; one lane, 2 to 5 us.  In its own launch, as all workgroups of the update read
// what it writes.
__global__ void factors_kernel(Factors* out, int64_t* step, const float* d_lr, const float* d_factor, double lr,
                               double log1, double log2, double weight_decay) {
    const float factor = d_factor ? *d_factor : 1.0f;
    if (d_lr) lr = (double)*d_lr;
    Factors f{};
    f.skip = !(fabsf(factor) < INFINITY) || !(fabs(lr) < (double)INFINITY);
    if (!f.skip) {
        const double s = (double)(*step + 1);
        *step += 1;
        f.grad = factor;
        f.decay = (float)(1.0 - lr * weight_decay);
        f.rate = (float)(lr / -expm1(s * log1));
        f.root = (float)sqrt(1.0 / -expm1(s * log2));
    }
    *out = f;
}

struct Betas {
    float b1, c1, b2, c2, eps;  // c = 1 - b
};

// One read and one write of everything a value has; memory bounds it: 147 M bf16 values with masters and 32-bit averages, 28
// bytes each, 760 us, 5.4 TB/s; 54 M with 8-bit averages, 16 bytes each, 159 us, 5.4 TB/s.
template <typename E, bool MASTER, bool BITS8, bool STREAM>
__global__ __launch_bounds__(kThreads) void update_kernel(const Items t, const Betas b, const Factors* factors) {
    const Factors f = *factors;
    if (f.skip) return;
    for (uint32_t chunk = blockIdx.x; chunk < t.first[t.count]; chunk += gridDim.x) {
        const int k = item_of(t, chunk);
        const Item& it = t.item[k];
        const int64_t base = (int64_t)(chunk - t.first[k]) * t.chunk;
        const int64_t end = it.n - base < t.chunk ? it.n : base + t.chunk;
        // Whole lanes of a block stay together: its scale is theirs together.
        for (int64_t at = base; at < end; at += kRound) {
            const int64_t i = at + threadIdx.x * kValues, left = end - i;
            float g[kValues], p[kValues], m[kValues], v[kValues];
            load<kValues, STREAM>(static_cast<const E*>(it.grad) + i, left, g);
            if (MASTER) load<kValues, STREAM>(it.master + i, left, p);
            else load<kValues, STREAM>(static_cast<const E*>(it.param) + i, left, p);
            if (BITS8) {
                const bool in = left > 0;
                load8<STREAM>(static_cast<const uint8_t*>(it.m) + i, left, in ? it.ms[i / GEAR_STEP_BLOCK] : 0.0f, m);
                load8<STREAM>(static_cast<const uint8_t*>(it.v) + i, left, in ? it.vs[i / GEAR_STEP_BLOCK] : 0.0f, v);
#pragma unroll
                for (int j = 0; j < kValues; j++) v[j] *= v[j];
            } else {
                load<kValues, STREAM>(static_cast<const float*>(it.m) + i, left, m);
                load<kValues, STREAM>(static_cast<const float*>(it.v) + i, left, v);
            }
            float r[kValues];
            uint32_t fading = 0;  // values without a gradient
#pragma unroll
            for (int j = 0; j < kValues; j++) {
                const float x = g[j] * f.grad;
                fading |= x == 0.0f ? 1u << j : 0u;
                m[j] = b.b1 * m[j] + b.c1 * x;
                v[j] = b.b2 * v[j] + b.c2 * (x * x);
                r[j] = root_of(v[j]);
                // eps is a normal number, and so its reciprocal is finite.
                p[j] = p[j] * f.decay - f.rate * m[j] * __builtin_amdgcn_rcpf(r[j] * f.root + b.eps);
            }
            if (MASTER) store<kValues, STREAM>(it.master + i, left, p);
            store<kValues, STREAM>(static_cast<E*>(it.param) + i, left, p);
            if (BITS8) {
                const float sm = store8<STREAM>(static_cast<uint8_t*>(it.m) + i, left, m, fading);
                const float sv = store8<STREAM>(static_cast<uint8_t*>(it.v) + i, left, r, 0);
                if (left > 0 && (threadIdx.x & (kGroup - 1)) == 0) {
                    it.ms[i / GEAR_STEP_BLOCK] = sm;
                    it.vs[i / GEAR_STEP_BLOCK] = sv;
                }
            } else {
                store<kValues, STREAM>(static_cast<float*>(it.m) + i, left, m);
                store<kValues, STREAM>(static_cast<float*>(it.v) + i, left, v);
            }
        }
    }
}

template <int THREADS>
__device__ __forceinline__ double block_add(double v, double* s) {
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) v += __shfl_xor(v, off);
    if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0.0;
#pragma unroll
    for (int k = 0; k < THREADS / 64; k++) v += s[k];
    return v;
}

// What a group of kThreads adds to the sum of squares: every `stride`-th chunk from `first` on.
template <typename E>
__device__ __forceinline__ double squares(const Grads& t, uint32_t first, uint32_t stride, int lane) {
    double sum = 0.0;
    for (uint32_t chunk = first; chunk < t.first[t.count]; chunk += stride) {
        const int k = item_of(t, chunk);
        const Grad& it = t.item[k];
        const int64_t base = (int64_t)(chunk - t.first[k]) * t.chunk;
        const int64_t end = it.n - base < t.chunk ? it.n : base + t.chunk;
        if (end - base == kChunk) {
            // Four rounds' loads on their way together.
            typename Vec<E, kValues>::raw raw[4];
#pragma unroll
            for (int q = 0; q < 4; q++) raw[q] = Vec<E, kValues>::load(static_cast<const E*>(it.grad) + base + q * kRound + lane * kValues);
#pragma unroll
            for (int q = 0; q < 4; q++) {
                float g[kValues];
                Vec<E, kValues>::unpack(raw[q], g);
#pragma unroll
                for (int j = 0; j < kValues; j++) sum = fma((double)g[j], (double)g[j], sum);
            }
            continue;
        }
        for (int64_t at = base; at < end; at += kRound) {
            const int64_t i = at + lane * kValues;
            float g[kValues];
            load<kValues, false>(static_cast<const E*>(it.grad) + i, end - i, g);
#pragma unroll
            for (int j = 0; j < kValues; j++) sum = fma((double)g[j], (double)g[j], sum);
        }
    }
    return sum;
}

// A sum per workgroup; `add` to those of the launches before.  218 M bf16 values take 99 to 124 us, 3.5 to 4.4 TB/s, 61 M 41
// to 43, where reads reach 6.9 TB/s: a workgroup asks for its next chunk when the squares of this one, in 64 bits, are added.
template <typename E>
__global__ __launch_bounds__(kThreads) void squares_kernel(const Grads t, double* sums, int add) {
    __shared__ double s[kThreads / 64];
    const double sum = block_add<kThreads>(squares<E>(t, blockIdx.x, gridDim.x, threadIdx.x), s);
    if (threadIdx.x == 0) sums[blockIdx.x] = sum + (add ? sums[blockIdx.x] : 0.0);
}

struct Limit {
    float scale, max_norm;
    float *norm, *factor;

    __device__ __forceinline__ void put(double sum) const {
        const double x = sqrt(sum) * (double)scale;
        *norm = (float)x;
        const double by = x > (double)max_norm ? (double)max_norm / x : 1.0;
        *factor = fabsf((float)x) < INFINITY ? (float)((double)scale * by) : NAN;
    }
};
__global__ __launch_bounds__(kThreads) void norm_kernel(const double* sums, int blocks, const Limit limit) {
    __shared__ double s[kThreads / 64];
    double sum = 0.0;
    for (int k = threadIdx.x; k < blocks; k += kThreads) sum += sums[k];
    sum = block_add<kThreads>(sum, s);
    if (threadIdx.x == 0) limit.put(sum);
}

// Few gradients of one type: one workgroup and no second launch (26000 values in 13 tensors: 8 us; norm and step together
// 20 us, and 23.4 with two launches for the norm).
constexpr int kSoloThreads = 1024;
constexpr uint32_t kSoloChunks = 32;
template <typename E>
__global__ __launch_bounds__(kSoloThreads) void solo_kernel(const Grads t, const Limit limit) {
    __shared__ double s[kSoloThreads / 64];
    const int groups = kSoloThreads / kThreads, group = threadIdx.x / kThreads;
    const double sum = block_add<kSoloThreads>(squares<E>(t, group, groups, threadIdx.x % kThreads), s);
    if (threadIdx.x == 0) limit.put(sum);
}

constexpr int64_t kMaxN = 1ll << 40;

const char* flaw(const gear_step_tensor* t, int64_t count) {
    if (count < 0 || (count > 0 && t == nullptr)) return "NULL or negative list of tensors";
    for (int64_t i = 0; i < count; i++) {
        if (float_bytes(t[i].dtype) == 0) return "dtype must be F16, BF16 or F32";
        if (t[i].n < 0 || t[i].n > kMaxN) return "size out of range";
        if (t[i].n > 0 && t[i].d_grad == nullptr) return "NULL gradient";
    }
    return nullptr;
}
const char* flaw(const gear_adamw_desc* d, const gear_step_tensor* t, int64_t count) {
    if (d == nullptr) return "NULL descriptor";
    if (d->state_bits != 32 && d->state_bits != 8) return "state_bits must be 32 or 8";
    if (!(d->lr >= 0.0) || !(d->lr < 3e38) || !(d->weight_decay >= 0.0) || !(d->weight_decay < 3e38))
        return "lr or weight_decay below 0 or not finite";
    if (!(d->beta1 >= 0.0 && d->beta1 < 1.0) || !(d->beta2 >= 0.0 && d->beta2 < 1.0)) return "betas must lie in [0, 1)";
    if (!((float)d->eps >= 1.17549435e-38f) || !(d->eps < 3e38)) return "eps must be 2^-126 or more, and finite";
    for (int64_t i = 0; i < count; i++) {
        if (t[i].n == 0) continue;
        if (t[i].d_param == nullptr || t[i].d_exp_avg == nullptr || t[i].d_exp_avg_sq == nullptr)
            return "NULL parameter or average";
        if (d->state_bits == 8 && (t[i].d_exp_avg_scale == nullptr || t[i].d_exp_avg_sq_scale == nullptr))
            return "8-bit averages need their scales";
        if (t[i].d_master != nullptr && t[i].dtype == GEAR_DTYPE_F32) return "a 32-bit parameter has no master";
    }
    return nullptr;
}

void set(Item& to, const gear_step_tensor& t) {
    to = Item{t.d_grad, t.d_param, t.d_exp_avg, t.d_exp_avg_sq, t.d_master, t.d_exp_avg_scale, t.d_exp_avg_sq_scale, t.n};
}
void set(Grad& to, const gear_step_tensor& t) { to = Grad{t.d_grad, t.n}; }

// Fills `out` with tensors from `i` on that `want` accepts; true when there are any.
template <typename I, int N, typename F>
bool gather(const gear_step_tensor* t, int64_t count, int64_t& i, List<I, N>& out, F want) {
    out.count = 0;
    out.first[0] = 0;
    for (; i < count && out.count < N; i++) {
        if (t[i].n == 0 || !want(t[i])) continue;
        const uint64_t chunks = (uint64_t)((t[i].n + out.chunk - 1) / out.chunk);
        if (out.first[out.count] + chunks > 0xFFFFFFFFull) break;  // the next launch's
        set(out.item[out.count], t[i]);
        out.first[out.count + 1] = (uint32_t)(out.first[out.count] + chunks);
        out.count++;
    }
    return out.count > 0;
}
int64_t values_of(const gear_step_tensor* t, int64_t count) {
    int64_t n = 0;
    for (int64_t i = 0; i < count; i++) n += t[i].n;
    return n;
}

typedef void (*Update)(const Items, const Betas, const Factors*);
template <bool BITS8, bool STREAM = false>
Update update_of(int32_t dtype, bool master) {
    if (dtype == GEAR_DTYPE_F32) return update_kernel<float, false, BITS8, STREAM>;
    if (dtype == GEAR_DTYPE_BF16) return master ? update_kernel<__bf16, true, BITS8, STREAM> : update_kernel<__bf16, false, BITS8, STREAM>;
    return master ? update_kernel<_Float16, true, BITS8, STREAM> : update_kernel<_Float16, false, BITS8, STREAM>;
}
// With 8-bit averages, what no cache holds until the next step passes by it: 123 M values
// with masters, a step with its norm, 414 us, and 464 through the caches.  With 32-bit averages
// that gains nothing (218 M values: 1306 and 1278).
constexpr int64_t kStreamValues = 16 << 20;

}  // namespace
}  // namespace gear

extern "C" int gear_step_sizes(int64_t* norm_bytes, int64_t* adamw_bytes) {
    using namespace gear;
    if (norm_bytes) *norm_bytes = 3 * (int64_t)(kNormBlocks * sizeof(double));
    if (adamw_bytes) *adamw_bytes = (int64_t)sizeof(Factors);
    return GEAR_OK;
}

extern "C" int gear_grad_norm(const gear_step_tensor* tensors, int64_t count, float scale, float max_norm,
                              float* d_norm, float* d_factor, void* d_work, int64_t work_bytes, void* stream) {
    using namespace gear;
    if (const char* w = flaw(tensors, count)) return fail(GEAR_E_INVAL, std::string("gear_grad_norm: ") + w);
    if (!(scale > 0.0f) || !(scale < 3e38f)) return fail(GEAR_E_INVAL, "gear_grad_norm: scale must be above 0 and finite");
    if (!(max_norm > 0.0f)) return fail(GEAR_E_INVAL, "gear_grad_norm: max_norm must be above 0");
    if (d_norm == nullptr || d_factor == nullptr) return fail(GEAR_E_INVAL, "gear_grad_norm: NULL norm or factor");
    int64_t need = 0;
    gear_step_sizes(&need, nullptr);
    if (d_work == nullptr || work_bytes < need)
        return fail(GEAR_E_INVAL, "gear_grad_norm: workspace smaller than gear_step_sizes states");
    double* sums = static_cast<double*>(d_work);
    hipStream_t s = static_cast<hipStream_t>(stream);
    (void)hipGetLastError();  // an error pending from an earlier HIP call is not this call's
    const Limit limit{scale, max_norm, d_norm, d_factor};
    int blocks = 0;  // sums that the launches so far have left
    Grads items;
    const int64_t values = values_of(tensors, count);
    items.chunk = values < kFewValues ? kRound : kChunk;
    hipError_t e = hipSuccess;
    const int32_t types[3] = {GEAR_DTYPE_F32, GEAR_DTYPE_BF16, GEAR_DTYPE_F16};
    for (const int32_t type : types) {
        int64_t i = 0;
        if (!gather(tensors, count, i, items, [&](const gear_step_tensor& t) { return t.dtype == type; })) continue;
        if (items.first[items.count] > kSoloChunks || i < count) break;
        bool others = false;
        for (int64_t k = 0; k < count; k++) others |= tensors[k].n > 0 && tensors[k].dtype != type;
        if (others) break;
        const auto kernel = type == GEAR_DTYPE_F32 ? solo_kernel<float>
                            : type == GEAR_DTYPE_BF16 ? solo_kernel<__bf16> : solo_kernel<_Float16>;
        hipLaunchKernelGGL(kernel, dim3(1), dim3(kSoloThreads), 0, s, items, limit);
        e = hipGetLastError();
        return e == hipSuccess ? GEAR_OK : hip_fail(e, "gear_grad_norm: launch");
    }
    for (const int32_t type : types) {
        // Each type has sums of its own.
        int used = 0;
        int64_t i = 0;
        while (gather(tensors, count, i, items, [&](const gear_step_tensor& t) { return t.dtype == type; })) {
            // Later launches add to all sums of the first, so they are as many workgroups.
            const int64_t most = values / items.chunk + count;
            const int grid = (int)(most < kNormBlocks ? most : kNormBlocks);
            const auto kernel = type == GEAR_DTYPE_F32 ? squares_kernel<float>
                                : type == GEAR_DTYPE_BF16 ? squares_kernel<__bf16> : squares_kernel<_Float16>;
            hipLaunchKernelGGL(kernel, dim3(grid), dim3(kThreads), 0, s, items, sums + blocks, used ? 1 : 0);
            e = hipGetLastError();
            if (e != hipSuccess) return hip_fail(e, "gear_grad_norm: launch");
            used = grid;
        }
        blocks += used;
    }
    hipLaunchKernelGGL(norm_kernel, dim3(1), dim3(kThreads), 0, s, sums, blocks, limit);
    e = hipGetLastError();
    return e == hipSuccess ? GEAR_OK : hip_fail(e, "gear_grad_norm: sum launch");
}

extern "C" int gear_adamw(const gear_adamw_desc* d, const gear_step_tensor* tensors, int64_t count, int64_t* d_step,
                          void* d_work, int64_t work_bytes, void* stream) {
    using namespace gear;
    if (const char* w = flaw(tensors, count)) return fail(GEAR_E_INVAL, std::string("gear_adamw: ") + w);
    if (const char* w = flaw(d, tensors, count)) return fail(GEAR_E_INVAL, std::string("gear_adamw: ") + w);
    if (d_step == nullptr) return fail(GEAR_E_INVAL, "gear_adamw: NULL step");
    if (d_work == nullptr || work_bytes < (int64_t)sizeof(Factors))
        return fail(GEAR_E_INVAL, "gear_adamw: workspace smaller than gear_step_sizes states");
    Factors* factors = static_cast<Factors*>(d_work);
    hipStream_t s = static_cast<hipStream_t>(stream);
    (void)hipGetLastError();  // an error pending from an earlier HIP call is not this call's
    hipLaunchKernelGGL(factors_kernel, dim3(1), dim3(1), 0, s, factors, d_step, d->d_lr, d->d_factor, d->lr,
                       log(d->beta1), log(d->beta2), d->weight_decay);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return hip_fail(e, "gear_adamw: factor launch");
    const Betas b{(float)d->beta1, (float)(1.0 - d->beta1), (float)d->beta2, (float)(1.0 - d->beta2), (float)d->eps};
    Items items;
    const int64_t values = values_of(tensors, count);
    items.chunk = values < kFewValues ? kRound : kChunk;
    const bool past = d->state_bits == 8 && values >= kStreamValues;
    const int32_t types[3] = {GEAR_DTYPE_F32, GEAR_DTYPE_BF16, GEAR_DTYPE_F16};
    for (const int32_t type : types) {
        for (int master = 0; master < 2; master++) {
            int64_t i = 0;
            while (gather(tensors, count, i, items, [&](const gear_step_tensor& t) {
                return t.dtype == type && (t.d_master != nullptr) == (master != 0);
            })) {
                const Update kernel = d->state_bits == 32 ? update_of<false>(type, master != 0)
                                      : past ? update_of<true, true>(type, master != 0) : update_of<true>(type, master != 0);
                const uint32_t chunks = items.first[items.count];
                const uint32_t grid = chunks < (1u << 20) ? chunks : 1u << 20;
                hipLaunchKernelGGL(kernel, dim3(grid), dim3(kThreads), 0, s, items, b, factors);
                e = hipGetLastError();
                if (e != hipSuccess) return hip_fail(e, "gear_adamw: launch");
            }
        }
    }
    return GEAR_OK;
}
