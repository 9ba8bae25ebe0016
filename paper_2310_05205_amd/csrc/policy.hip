// The clipped policy loss of rows of logits, its gradient, and the actions'
// log-probabilities alone (include/gear.h).  With z a row's logits, m their
// largest and d = z - m:
//   S = sum e^d,  lp = d[action] - log S,  H = log S - (sum d e^d) / S,
//   dz_j = s ((1[j = action] - p_j) c + entropy p_j (log p_j + H)),  p_j = e^d_j / S,
// where c is the derivative of the clipped and KL terms for lp and s the
// row's weight over the denominator.
//
// Logits are read and gradients written, with some operations per element:
// memory bounds it.
#include "element.h"
#include "gear_internal.h"

namespace gear {
namespace {

constexpr int kThreads = 256, kWaves = kThreads / 64;
constexpr int kSums = 5;              // loss, clipped term, KL term, entropy, clipped rows
constexpr int kCountBlocks = 256;     // workgroups that count the rows that take part
constexpr int kMaxBlocks = 4096;      // workgroups of the row kernel
constexpr int64_t kCountOff = 0, kSumOff = kCountBlocks * (int64_t)sizeof(int64_t);

struct Args {
    const void* logits;
    void* grad;
    const void* action;
    const uint8_t* mask;
    const float *old_logp, *ref_logp, *adv, *weight, *grad_loss;
    float *loss, *stats, *logp, *entropy;
    int64_t* counts;  // [kCountBlocks]
    float* sums;      // [blocks][kSums]
    int64_t n, V, row_stride, mask_group, adv_group, weight_group;
    int32_t action_dtype, count_blocks;
    float lo, hi, kl, ent, denom, grad_scale;
};

__device__ __forceinline__ int64_t action_of(const Args& a, int64_t row) {
    if (a.action_dtype == GEAR_DTYPE_I32) return static_cast<const int32_t*>(a.action)[row];
    if (a.action_dtype == GEAR_DTYPE_I64) return static_cast<const int64_t*>(a.action)[row];
    return static_cast<const uint8_t*>(a.action)[row];
}
__device__ __forceinline__ bool takes_part(const Args& a, int64_t row, int64_t action) {
    return action >= 0 && action < a.V && (a.mask == nullptr || a.mask[row / a.mask_group] != 0);
}

__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) v = fmaxf(v, __shfl_xor(v, off));
    return v;
}
template <typename T>
__device__ __forceinline__ T wave_add(T v) {
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) v += __shfl_xor(v, off);
    return v;
}

// Rows that take part, per workgroup.
__global__ __launch_bounds__(kThreads) void count_kernel(const Args a) {
    __shared__ int64_t s[kWaves];
    int64_t c = 0;
    for (int64_t r = (int64_t)blockIdx.x * kThreads + threadIdx.x; r < a.n; r += (int64_t)gridDim.x * kThreads)
        c += takes_part(a, r, action_of(a, r)) ? 1 : 0;
    c = wave_add(c);
    if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = c;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int k = 1; k < kWaves; k++) c += s[k];
        a.counts[blockIdx.x] = c;
    }
}

// What the sums are divided by, in every lane of the wave.
__device__ __forceinline__ float denominator(const Args& a) {
    if (a.denom > 0.0f) return a.denom;
    int64_t c = 0;
    for (int k = threadIdx.x & 63; k < a.count_blocks; k += 64) c += a.counts[k];
    c = wave_add(c);
    return c > 0 ? (float)c : 1.0f;
}

struct Row {
    float lp, H;   // log-probability of the action, entropy
    float c, s;    // derivative of the loss for lp, factor of the gradient
    float sums[kSums];
};

// A row's terms from its largest logit, its sums and the action's logit.
template <bool LOSS>
__device__ __forceinline__ Row row_terms(const Args& a, int64_t row, float m, float S, float dS, float za, float denom) {
    Row r{};
    if (m == -INFINITY) {  // no distribution
        r.lp = -INFINITY;
        return r;
    }
    const float log_S = fast_log(S);
    r.lp = (za - m) - log_S;
    r.H = log_S - dS / S;
    if (!LOSS) return r;
    const float A = a.adv[row / a.adv_group], w = a.weight ? a.weight[row / a.weight_group] : 1.0f;
    const float ratio = expf(r.lp - a.old_logp[row]);
    const float free = ratio * A, held = fminf(fmaxf(ratio, a.lo), a.hi) * A;
    const bool clipped = held < free;
    const float pg = clipped ? -held : -free;
    r.c = clipped ? 0.0f : -free;
    float kl = 0.0f, row_loss = pg;
    if (a.ref_logp) {
        const float q = a.ref_logp[row] - r.lp, e = expm1f(q);
        kl = e - q;
        if (a.kl != 0.0f) {
            row_loss += a.kl * kl;
            r.c -= a.kl * e;
        }
    }
    if (a.ent != 0.0f) row_loss -= a.ent * r.H;
    r.s = w * a.grad_scale * (a.grad_loss ? *a.grad_loss : 1.0f) / denom;
    r.sums[0] = w * row_loss;
    r.sums[1] = pg;
    r.sums[2] = kl;
    r.sums[3] = r.H;
    r.sums[4] = clipped ? 1.0f : 0.0f;
    return r;
}

// Gradient of one logit that is not the action's: d = z - m.
__device__ __forceinline__ float slope(const Args& a, const Row& r, float d, float inv_S, float log_S) {
    const float p = fast_exp(d) * inv_S;
    return r.s * p * (a.ent * (fmaxf(d, -3e38f) - log_S + r.H) - r.c);
}

// A workgroup per row, which reads it three times.
template <typename E, bool LOSS>
__global__ __launch_bounds__(kThreads) void row_kernel(const Args a) {
    __shared__ float s_max[kWaves], s_sum[kWaves], s_dsum[kWaves];
    const int wave = threadIdx.x >> 6;
    const float denom = LOSS ? denominator(a) : 1.0f;
    float total[kSums] = {};
    for (int64_t row = blockIdx.x; row < a.n; row += gridDim.x) {
        const int64_t action = action_of(a, row);
        E* g = LOSS && a.grad ? static_cast<E*>(a.grad) + row * a.V : nullptr;
        if (!takes_part(a, row, action)) {
            if (threadIdx.x == 0) {
                if (a.logp) a.logp[row] = 0.0f;
                if (a.entropy) a.entropy[row] = 0.0f;
            }
            if (g)
                for (int64_t j = threadIdx.x; j < a.V; j += kThreads) g[j] = (E)0.0f;
            continue;
        }
        const E* z = static_cast<const E*>(a.logits) + row * a.row_stride;
        const float za = (float)z[action];
        float m = -INFINITY;
        for (int64_t j = threadIdx.x; j < a.V; j += kThreads) m = fmaxf(m, (float)z[j]);
        m = wave_max(m);
        if ((threadIdx.x & 63) == 0) s_max[wave] = m;
        __syncthreads();
#pragma unroll
        for (int k = 0; k < kWaves; k++) m = fmaxf(m, s_max[k]);
        float S = 0.0f, dS = 0.0f;
        if (m != -INFINITY) {
            for (int64_t j = threadIdx.x; j < a.V; j += kThreads) {
                const float d = (float)z[j] - m, e = fast_exp(d);
                S += e;
                dS += e * fmaxf(d, -3e38f);
            }
        }
        S = wave_add(S);
        dS = wave_add(dS);
        if ((threadIdx.x & 63) == 0) {
            s_sum[wave] = S;
            s_dsum[wave] = dS;
        }
        __syncthreads();
        S = dS = 0.0f;
#pragma unroll
        for (int k = 0; k < kWaves; k++) {
            S += s_sum[k];
            dS += s_dsum[k];
        }
        const Row r = row_terms<LOSS>(a, row, m, S, dS, za, denom);
        if (threadIdx.x == 0) {
            if (a.logp) a.logp[row] = r.lp;
            if (a.entropy) a.entropy[row] = r.H;
#pragma unroll
            for (int k = 0; k < kSums; k++) total[k] += r.sums[k];
        }
        if (g) {
            const float inv_S = 1.0f / S, log_S = fast_log(S);
            for (int64_t j = threadIdx.x; j < a.V; j += kThreads) {
                float v = 0.0f;
                if (m != -INFINITY) {
                    v = slope(a, r, (float)z[j] - m, inv_S, log_S);
                    if (j == action) v += r.s * r.c;
                }
                g[j] = (E)v;
            }
        }
    }
    if (LOSS && threadIdx.x == 0) {
#pragma unroll
        for (int k = 0; k < kSums; k++) a.sums[(int64_t)blockIdx.x * kSums + k] = total[k];
    }
}

// Adds the workgroups' sums, in 64 bits and always in the same order.
__global__ __launch_bounds__(64) void finish_kernel(const Args a, int32_t blocks) {
    const float denom = denominator(a);
    for (int k = 0; k < kSums; k++) {
        double v = 0.0;
        for (int b = threadIdx.x; b < blocks; b += 64) v += (double)a.sums[(int64_t)b * kSums + k];
        v = wave_add(v) / (double)denom;
        if (threadIdx.x == 0) {
            if (k == 0) *a.loss = (float)v;
            else if (a.stats) a.stats[k - 1] = (float)v;
        }
    }
}

int64_t work_bytes_of(const gear_policy_desc&) { return kSumOff + (int64_t)kMaxBlocks * kSums * (int64_t)sizeof(float); }

const char* flaw(const gear_policy_desc* d) {
    if (d == nullptr) return "NULL descriptor";
    if (float_bytes(d->dtype) == 0) return "dtype must be F16, BF16 or F32";
    if (d->action_dtype != GEAR_DTYPE_U8 && d->action_dtype != GEAR_DTYPE_I32 && d->action_dtype != GEAR_DTYPE_I64)
        return "action dtype must be U8, I32 or I64";
    if (d->n < 0 || d->V < 1 || d->V >= (1ll << 31) || d->n > (1ll << 40) / d->V) return "size out of range";
    if (d->row_stride < d->V && d->n > 1) return "row_stride below V";
    if (d->mask_group < 1 || d->adv_group < 1 || d->weight_group < 1) return "group below 1";
    return nullptr;
}
const char* loss_flaw(const gear_policy_desc* d) {
    if (const char* w = flaw(d)) return w;
    if (!(d->clip_low >= 0.0f) || !(d->clip_high >= 0.0f)) return "clip range below 0";
    if (!(d->denom >= 0.0f) || d->denom > 3e38f) return "denom below 0 or not finite";
    if (!(fabsf(d->kl) < 3e38f) || !(fabsf(d->entropy) < 3e38f) || !(fabsf(d->grad_scale) < 3e38f))
        return "coefficient not finite";
    return nullptr;
}

Args args_of(const gear_policy_desc& d, const void* logits) {
    Args a{};
    a.logits = logits;
    a.action = d.d_action;
    a.mask = d.d_mask;
    a.n = d.n;
    a.V = d.V;
    a.row_stride = d.row_stride;
    a.mask_group = d.mask_group;
    a.adv_group = d.adv_group;
    a.weight_group = d.weight_group;
    a.action_dtype = d.action_dtype;
    return a;
}

template <bool LOSS>
hipError_t launch_rows(const Args& a, int32_t dtype, int blocks, hipStream_t s) {
    void (*k)(const Args) = dtype == GEAR_DTYPE_F32 ? row_kernel<float, LOSS>
                            : dtype == GEAR_DTYPE_BF16 ? row_kernel<__bf16, LOSS> : row_kernel<_Float16, LOSS>;
    hipLaunchKernelGGL(k, dim3(blocks), dim3(kThreads), 0, s, a);
    return hipGetLastError();
}

}  // namespace
}  // namespace gear

extern "C" int gear_policy_sizes(const gear_policy_desc* d, int64_t* work_bytes) {
    using namespace gear;
    if (const char* w = loss_flaw(d)) return fail(GEAR_E_INVAL, std::string("gear_policy_sizes: ") + w);
    if (work_bytes) *work_bytes = work_bytes_of(*d);
    return GEAR_OK;
}

extern "C" int gear_policy_loss(const gear_policy_desc* d, const void* d_logits, const float* d_old_logp,
                                const float* d_ref_logp, const float* d_adv, const float* d_weight,
                                const float* d_grad_loss, float* d_loss, float* d_stats, float* d_logp,
                                float* d_entropy, void* d_grad, void* d_work, int64_t work_bytes, void* stream) {
    using namespace gear;
    if (const char* w = loss_flaw(d)) return fail(GEAR_E_INVAL, std::string("gear_policy_loss: ") + w);
    if (d_loss == nullptr) return fail(GEAR_E_INVAL, "gear_policy_loss: NULL loss");
    if (d->n > 0 && (d_logits == nullptr || d->d_action == nullptr || d_old_logp == nullptr || d_adv == nullptr))
        return fail(GEAR_E_INVAL, "gear_policy_loss: NULL logits, action, old_logp or adv");
    if (d_grad == d_logits && d_grad != nullptr && d->row_stride != d->V && d->n > 1)
        return fail(GEAR_E_INVAL, "gear_policy_loss: the gradient may take the logits' place when row_stride is V only");
    if (d_work == nullptr || work_bytes < work_bytes_of(*d))
        return fail(GEAR_E_INVAL, "gear_policy_loss: workspace smaller than gear_policy_sizes states");
    Args a = args_of(*d, d_logits);
    a.grad = d_grad;
    a.old_logp = d_old_logp;
    a.ref_logp = d_ref_logp;
    a.adv = d_adv;
    a.weight = d_weight;
    a.grad_loss = d_grad_loss;
    a.loss = d_loss;
    a.stats = d_stats;
    a.logp = d_logp;
    a.entropy = d_entropy;
    a.counts = reinterpret_cast<int64_t*>(static_cast<char*>(d_work) + kCountOff);
    a.sums = reinterpret_cast<float*>(static_cast<char*>(d_work) + kSumOff);
    a.lo = 1.0f - d->clip_low;
    a.hi = 1.0f + d->clip_high;
    a.kl = d->kl;
    a.ent = d->entropy;
    a.denom = d->denom;
    a.grad_scale = d->grad_scale;
    hipStream_t s = static_cast<hipStream_t>(stream);
    (void)hipGetLastError();  // an error pending from an earlier HIP call is not this call's
    hipError_t e = hipSuccess;
    if (!(a.denom > 0.0f)) {
        const int64_t want = (a.n + kThreads - 1) / kThreads;
        a.count_blocks = (int32_t)(want < 1 ? 1 : want < kCountBlocks ? want : kCountBlocks);
        hipLaunchKernelGGL(count_kernel, dim3(a.count_blocks), dim3(kThreads), 0, s, a);
        e = hipGetLastError();
        if (e != hipSuccess) return hip_fail(e, "gear_policy_loss: count launch");
    }
    const int blocks = (int)(a.n < kMaxBlocks ? a.n : kMaxBlocks);
    if (blocks > 0) {
        e = launch_rows<true>(a, d->dtype, blocks, s);
        if (e != hipSuccess) return hip_fail(e, "gear_policy_loss: row launch");
    }
    hipLaunchKernelGGL(finish_kernel, dim3(1), dim3(64), 0, s, a, blocks);
    e = hipGetLastError();
    return e == hipSuccess ? GEAR_OK : hip_fail(e, "gear_policy_loss: sum launch");
}

extern "C" int gear_action_logp(const gear_policy_desc* d, const void* d_logits, float* d_logp, float* d_entropy,
                                void* stream) {
    using namespace gear;
    if (const char* w = flaw(d)) return fail(GEAR_E_INVAL, std::string("gear_action_logp: ") + w);
    if (d->n == 0) return GEAR_OK;
    if (d_logits == nullptr || d->d_action == nullptr) return fail(GEAR_E_INVAL, "gear_action_logp: NULL logits or action");
    Args a = args_of(*d, d_logits);
    a.logp = d_logp;
    a.entropy = d_entropy;
    (void)hipGetLastError();  // an error pending from an earlier HIP call is not this call's
    const int blocks = (int)(a.n < kMaxBlocks ? a.n : kMaxBlocks);
    const hipError_t e = launch_rows<false>(a, d->dtype, blocks, static_cast<hipStream_t>(stream));
    return e == hipSuccess ? GEAR_OK : hip_fail(e, "gear_action_logp: launch");
}
