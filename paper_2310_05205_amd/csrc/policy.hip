// The clipped policy loss of rows of logits, its gradient, and the actions'
// log-probabilities alone (include/gear.h).  With z a row's logits, m their
// largest and d = z - m:
//   S = sum e^d,  lp = d[action] - log S,  H = log S - (sum d e^d) / S,
//   dz_j = s ((1[j = action] - p_j) c + entropy p_j (log p_j + H)),  p_j = e^d_j / S,
// where c is the derivative of the clipped and KL terms for lp and s the
// row's weight over the denominator.
//
// Logits are read and gradients written once: 4 bytes an element of 16-bit
// types.  The element's operations (widen, running maximum, two exponentials,
// two sums, narrow) keep the vector units busy for three quarters of the time that
// memory needs or more, so they are counted as carefully as the bytes.
#include "element.h"
#include "gear_internal.h"

namespace gear {
namespace {

constexpr int kThreads = 256;
constexpr int kSums = 5;               // loss, clipped term, KL term, entropy, clipped rows
constexpr int kCountBlocks = 512;      // workgroups that count the rows that take part
constexpr int kMaxBlocks = 2048;       // workgroups of the row kernels
constexpr int kSoloThreads = 1024;     // calls of one workgroup
// Small calls run in one workgroup, without the launches that count rows before
// and add sums after: in fp32 16 x 18 take 10.3 us so and 15.3 otherwise, 1024 x 18
// 14.5 and 15.0, 256 x 128 14.8 and 15.2, 2048 x 18 20.8 and 15.0.
constexpr int64_t kSoloLogits = 1 << 15, kSoloActions = 1024;  // at most 256 pieces a row
constexpr int64_t kCountOff = 0, kSumOff = kCountBlocks * (int64_t)sizeof(int64_t);
// Where a logit's distance stops mattering: 2^d is 0 well above it, and a
// multiple of it stays finite.
constexpr float kFloor = -1e4f;

// Quotients by a number fixed for the launch: for dividends below 2^31, the
// high part of a product with ceil(2^(31 + l) / d), 2^l >= d, which is exact.
struct Divisor {
    int64_t d;
    uint32_t mul, shift;  // mul 0: divide
};
Divisor divisor(int64_t d, int64_t dividends) {
    Divisor r{d, 0, 0};
    if (dividends >= (1ll << 31) || d > dividends) {
        // Nothing below d: the quotient is 0, which mul 0 would compute too.
        return r;
    }
    uint32_t l = 0;
    while ((1ll << l) < d) l++;
    r.mul = (uint32_t)(((1ull << (31 + l)) + (uint64_t)d - 1) / (uint64_t)d);
    r.shift = 31 + l;
    return r;
}
__device__ __forceinline__ int64_t quotient(int64_t x, const Divisor& d) {
    if (d.mul) return (int64_t)(((uint64_t)(uint32_t)x * d.mul) >> d.shift);
    return x / d.d;
}

struct Args {
    const void* logits;
    void* grad;
    const void* action;
    const uint8_t* mask;
    const float *old_logp, *ref_logp, *adv, *weight, *grad_loss;
    float *loss, *stats, *logp, *entropy;
    int64_t* counts;  // [kCountBlocks]
    float* sums;      // [kSums][kMaxBlocks]
    int64_t n, V, row_stride;
    Divisor mask_group, adv_group, weight_group;
    int32_t action_dtype, count_blocks;
    float lo, hi, kl, ent, denom, grad_scale;
};

__device__ __forceinline__ int64_t action_of(const Args& a, int64_t row) {
    if (a.action_dtype == GEAR_DTYPE_I32) return static_cast<const int32_t*>(a.action)[row];
    if (a.action_dtype == GEAR_DTYPE_I64) return static_cast<const int64_t*>(a.action)[row];
    return static_cast<const uint8_t*>(a.action)[row];
}
__device__ __forceinline__ bool takes_part(const Args& a, int64_t row, int64_t action) {
    return (action >= 0) & (action < a.V) && (a.mask == nullptr || a.mask[quotient(row, a.mask_group)] != 0);
}

template <int G>
__device__ __forceinline__ float group_max(float v) {
#pragma unroll
    for (int off = G / 2; off > 0; off >>= 1) v = fmaxf(v, __shfl_xor(v, off));
    return v;
}
template <int G, typename T>
__device__ __forceinline__ T group_add(T v) {
#pragma unroll
    for (int off = G / 2; off > 0; off >>= 1) v += __shfl_xor(v, off);
    return v;
}

// Sum of one value per lane over the workgroup, in the first wave's lanes; `s` holds a value per wave.
template <int THREADS, typename T>
__device__ __forceinline__ T block_add(T v, T* s) {
    v = group_add<64>(v);
    if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = v;
    __syncthreads();
    return group_add<THREADS / 64>(s[threadIdx.x % (THREADS / 64)]);
}

// Rows that take part, of which a thread takes 16 neighbouring ones at a time.
constexpr int kCountRows = 16;
template <int THREADS>
__device__ __forceinline__ int64_t count_rows(const Args& a, int64_t* s) {
    int64_t c = 0;
    for (int64_t r = ((int64_t)blockIdx.x * THREADS + threadIdx.x) * kCountRows; r < a.n;
         r += (int64_t)gridDim.x * THREADS * kCountRows) {
        if (a.action_dtype == GEAR_DTYPE_I32 && a.mask_group.d == 1 && r + kCountRows <= a.n) {
            int32_t act[kCountRows];
            uint32_t mask[kCountRows / 4];
            __builtin_memcpy(act, static_cast<const int32_t*>(a.action) + r, sizeof(act));
            if (a.mask) __builtin_memcpy(mask, a.mask + r, sizeof(mask));
#pragma unroll
            for (int k = 0; k < kCountRows; k++) {
                const bool on = a.mask == nullptr || ((mask[k / 4] >> (8 * (k % 4))) & 0xFFu) != 0;
                c += on && (uint32_t)act[k] < (uint32_t)a.V ? 1 : 0;
            }
        } else {
            const int64_t end = r + kCountRows < a.n ? r + kCountRows : a.n;
            for (int64_t k = r; k < end; k++) c += takes_part(a, k, action_of(a, k)) ? 1 : 0;
        }
    }
    return block_add<THREADS>(c, s);
}

// Rows that take part, per workgroup: 5 us for 2097152 rows under a mask, which is
// mostly the launch.
__global__ __launch_bounds__(kThreads) void count_kernel(const Args a) {
    __shared__ int64_t s[kThreads / 64];
    const int64_t c = count_rows<kThreads>(a, s);
    if (threadIdx.x == 0) a.counts[blockIdx.x] = c;
}

// What the sums are divided by, in every lane of the wave.
__device__ __forceinline__ float denominator(const Args& a) {
    if (a.denom > 0.0f) return a.denom;
    int64_t c = 0;
#pragma unroll 8
    for (int k = threadIdx.x & 63; k < a.count_blocks; k += 64) c += a.counts[k];
    c = group_add<64>(c);
    return c > 0 ? (float)c : 1.0f;
}

// Distances from a row's largest logit m, in powers of two: 0 for m itself, so
// that a row's only possible action has log-probability 0.
struct Scale {
    float m;
    __device__ __forceinline__ float operator()(float z) const { return (z - m) * kLog2e; }
};
__device__ __forceinline__ Scale scale_of(float m) { return Scale{m == -INFINITY ? 0.0f : m}; }  // a row of -inf sums to 0

// Adds a piece's 2^d and d 2^d.  With TAME no logit is far enough out for its d,
// or a multiple of it, to be infinite, and need not be kept from it.
template <bool TAME, int VE>
__device__ __forceinline__ void add_piece(const float (&f)[VE], const Scale& dist, float& S, float& dS) {
#pragma unroll
    for (int j = 0; j < VE; j++) {
        const float d = dist(f[j]), e = __builtin_amdgcn_exp2f(d);
        S += e;
        dS = fmaf(e, TAME ? d : fmaxf(d, kFloor), dS);
    }
}
constexpr float kTame = 1e9f;

// Sums against logit m become sums against logit `top`, which is no smaller.
struct Sums {
    float m, S, dS;
};
__device__ __forceinline__ void rescale(float m, float top, float& S, float& dS) {
    const float d = fmaxf((m - scale_of(top).m) * kLog2e, kFloor), e = __builtin_amdgcn_exp2f(d);
    dS = e * fmaf(d, S, dS);
    S *= e;
}

// What a row has beside its logits, read while they are on their way.
struct Inputs {
    float old, ref, A, w;
};
__device__ __forceinline__ Inputs inputs_of(const Args& a, int64_t row) {
    Inputs in;
    in.old = a.old_logp[row];
    in.ref = a.ref_logp ? a.ref_logp[row] : 0.0f;
    in.A = a.adv[quotient(row, a.adv_group)];
    in.w = a.weight ? a.weight[quotient(row, a.weight_group)] : 1.0f;
    return in;
}

// exp(q) - 1 and exp(q) - 1 - q, the latter without cancellation near 0: there by
// the exponential's series, whose first omitted term is below 2^-30 of the result.
__device__ __forceinline__ void exp_less_one(float q, float& e, float& k) {
#pragma clang fp contract(off)
    float p = 1.0f / 40320.0f;
    p = fmaf(p, q, 1.0f / 5040.0f);
    p = fmaf(p, q, 1.0f / 720.0f);
    p = fmaf(p, q, 1.0f / 120.0f);
    p = fmaf(p, q, 1.0f / 24.0f);
    p = fmaf(p, q, 1.0f / 6.0f);
    p = fmaf(p, q, 0.5f);
    const float near_k = p * q * q, far_e = fast_exp(q) - 1.0f;
    const bool near = fabsf(q) < 0.25f;
    k = near ? near_k : far_e - q;
    e = near ? q + near_k : far_e;
}

struct Row {
    float lp, H;  // log-probability of the action, entropy
    float c, s;   // derivative of the loss for lp, factor of the gradient
    float sums[kSums];
};

// A row's terms from the sums of 2^d and of d 2^d, and the action's d.  The
// operations are spelled out, so that lp and H come out the same in every kernel.
template <bool LOSS>
__device__ __forceinline__ Row row_terms(const Args& a, const Inputs& in, float S, float dS, float da, float scale) {
#pragma clang fp contract(off)
    Row r{};
    // All -inf, no distribution.  The sum says so: it is 1 or more with any other logit and NaN with a NaN, which
    // the maximum passes over.
    if (S == 0.0f) {
        r.lp = -INFINITY;
        return r;
    }
    const float log_S = __builtin_amdgcn_logf(S);
    r.lp = (da - log_S) * kLn2;
    r.H = (log_S - dS * __builtin_amdgcn_rcpf(S)) * kLn2;
    if (!LOSS) return r;
    // The ratio and the KL term are exponentials that may pass fp32.  Where an advantage or a weight of 0 multiplies
    // them, 0 is left, not NaN.
    const float lr = r.lp - in.old, ratio = fast_exp(lr);
    const float free = in.A == 0.0f && fabsf(lr) < INFINITY ? 0.0f : ratio * in.A;
    const float held = fminf(fmaxf(ratio, a.lo), a.hi) * in.A;
    const bool clipped = held < free;
    const float pg = clipped ? -held : -free;
    r.c = clipped ? 0.0f : -free;
    float kl = 0.0f, row_loss = pg;
    if (a.ref_logp) {
        float e;
        exp_less_one(in.ref - r.lp, e, kl);
        if (a.kl != 0.0f) {
            row_loss += a.kl * kl;
            r.c -= a.kl * e;
        }
    }
    if (a.ent != 0.0f) row_loss -= a.ent * r.H;
    if (in.w == 0.0f) {
        if (fabsf(row_loss) == INFINITY) row_loss = 0.0f;
        if (fabsf(r.c) == INFINITY) r.c = 0.0f;
    }
    r.s = in.w * scale;
    r.sums[0] = in.w * row_loss;
    r.sums[1] = pg;
    r.sums[2] = kl;
    r.sums[3] = r.H;
    r.sums[4] = clipped ? 1.0f : 0.0f;
    return r;
}

// dz_j = 2^d_j (k1 d_j + k0), and k2 more for the action.
struct Slope {
    float k0, k1, k2;
    template <bool TAME>
    __device__ __forceinline__ float at(float d) const {
        return __builtin_amdgcn_exp2f(d) * fmaf(k1, TAME ? d : fmaxf(d, kFloor), k0);
    }
    __device__ __forceinline__ float operator()(float d) const { return at<false>(d); }
};
__device__ __forceinline__ Slope slope_of(const Args& a, const Row& r, float S) {
    const float f = r.s * __builtin_amdgcn_rcpf(S), g = a.ent * kLn2;
    return Slope{f * (a.ent * r.H - g * __builtin_amdgcn_logf(S) - r.c), f * g, r.s * r.c};
}

// The sums of a call that one workgroup ran, or this workgroup's share of them.
template <int THREADS, bool SOLO>
__device__ __forceinline__ void leave_sums(const Args& a, const float (&total)[kSums], float denom,
                                           double (*s)[THREADS / 64]) {
    constexpr int kWaves = THREADS / 64;
#pragma unroll
    for (int k = 0; k < kSums; k++) {
        const double v = group_add<64>((double)total[k]);
        if ((threadIdx.x & 63) == 0) s[k][threadIdx.x >> 6] = v;
    }
    __syncthreads();
    if (threadIdx.x >= 64) return;
#pragma unroll
    for (int k = 0; k < kSums; k++) {
        const double v = group_add<kWaves>(s[k][threadIdx.x % kWaves]);
        if (threadIdx.x == 0) {
            if (!SOLO) a.sums[k * kMaxBlocks + blockIdx.x] = (float)v;
            else if (k == 0) *a.loss = (float)(v / (double)denom);
            else if (a.stats) a.stats[k - 1] = (float)(v / (double)denom);
        }
    }
}

// 16 bytes of a row as four words: the vectors of 16-bit elements that the
// language offers are taken apart into a register per element as soon as one is replaced.
template <typename E>
struct Piece {
    static constexpr int VE = 16 / sizeof(E), kPerWord = 4 / sizeof(E);
    typedef uint32_t words __attribute__((ext_vector_type(4)));
    words w;

    static __device__ __forceinline__ uint32_t lowest() {  // a word of -inf
        const E e[kPerWord] = {};
        E f[kPerWord];
#pragma unroll
        for (int k = 0; k < kPerWord; k++) f[k] = e[k] - (E)INFINITY;
        return __builtin_bit_cast(uint32_t, f);
    }
    typedef words loose __attribute__((aligned(2)));
    // Streaming loads where a wave takes whole lines of a row: 8% of the time at
    // 32768 actions.  Where it takes parts of many rows' lines, the rest has to stay in the cache.
    template <bool STREAM>
    __device__ __forceinline__ void load(const E* p) {
        if (STREAM) w = __builtin_nontemporal_load(reinterpret_cast<const loose*>(p));
        else w = *reinterpret_cast<const loose*>(p);
    }
    __device__ __forceinline__ void fill() { w = words{lowest(), lowest(), lowest(), lowest()}; }
    // The first n elements become -inf.
    __device__ __forceinline__ void drop(int n) {
#pragma unroll
        for (int k = 0; k < 4; k++) {
            if (kPerWord == 2 && n == 2 * k + 1) w[k] = (w[k] & 0xFFFF0000u) | (lowest() & 0xFFFFu);
            if (n >= kPerWord * (k + 1)) w[k] = lowest();
        }
    }
    // A row of V < VE elements, the rest -inf.
    __device__ __forceinline__ void gather(const E* p, int V) {
        fill();
#pragma unroll
        for (int j = 0; j < VE; j++)
            if (j < V) {
                if constexpr (sizeof(E) == 4) {
                    w[j] = __builtin_bit_cast(uint32_t, p[j]);
                } else {
                    uint16_t h16;
                    __builtin_memcpy(&h16, p + j, 2);
                    const uint32_t h = h16;
                    w[j / 2] = j % 2 ? (w[j / 2] & 0xFFFFu) | (h << 16) : (w[j / 2] & 0xFFFF0000u) | h;
                }
            }
    }
    __device__ __forceinline__ void unpack(float (&f)[VE]) const {
#pragma unroll
        for (int k = 0; k < 4; k++) {
            E e[kPerWord];
            const uint32_t u = w[k];
            __builtin_memcpy(e, &u, 4);
#pragma unroll
            for (int h = 0; h < kPerWord; h++) f[kPerWord * k + h] = (float)e[h];
        }
    }
    // Keeps the compiler from holding on to what it computed from the piece:
    // unpacked values kept from one pass to the next take several times its registers.
    __device__ __forceinline__ void forget() { asm volatile("" : "+v"(w)); }
};

// Lane `mine`'s piece number i of a row shared by G lanes, which take its pieces
// in turn: past the row's end, the rest of its last piece that no other lane has, or -inf.
template <typename E, int G>
__device__ __forceinline__ void load_piece(Piece<E>& v, const E* z, int V, int mine, int i) {
    constexpr int VE = Piece<E>::VE;
    const int first = i * G * VE;
    if (first + G * VE <= V) {
        v.template load<(G >= 64)>(z + first + mine * VE);
    } else if (first < V) {
        const int base = first + mine * VE, over = base + VE - V;
        v.template load<(G >= 64)>(z + (over < 0 ? base : V - VE));
        if (over > 0) v.drop(over);
    } else {
        v.fill();
    }
}

// Writes the gradient of the elements that load_piece gave to this lane.
template <typename E, int G, bool TINY, bool TAME>
__device__ __forceinline__ void store_piece(E* g, const Piece<E>& v, int V, int mine, int i, const Slope& slope,
                                            const Scale& dist) {
    constexpr int VE = Piece<E>::VE;
    const int base = (i * G + mine) * VE;
    float f[VE], o[VE];
    v.unpack(f);
#pragma unroll
    for (int j = 0; j < VE; j++) o[j] = slope.template at<TAME>(dist(f[j]));
    if (!TINY && ((i + 1) * G * VE <= V || base + VE <= V)) {
        Vec<E, VE>::store(g + base, o);
    } else {
        const int at = TINY ? 0 : V - VE;
#pragma unroll
        for (int j = 0; j < VE; j++)
            if (at + j >= base && at + j < V) g[at + j] = (E)o[j];
    }
}

// The gradient's factor beside denom, grad_scale's, and the loss's own gradient.
__device__ __forceinline__ float scale_by(const Args& a, float denom) {
    return a.grad_scale * (a.grad_loss ? *a.grad_loss : 1.0f) / denom;
}

// Rows held in registers: G lanes share a row, each with up to NV pieces of 16
// bytes, so that a row is read once and its gradient written once.  With TINY,
// rows are shorter than a piece.  2097152 rows of 16 bf16 take 48 us, of which the
// vector units' share is about 31 and memory's 28; 320 rows of 18 fp32, in one
// workgroup without the launches before and after, 8.4 us, mostly dependent loads.
template <typename E, int G, int NV, int THREADS, int WAVES, bool TINY, bool LOSS>
__global__ __launch_bounds__(THREADS, WAVES) void held_kernel(const Args a) {
    constexpr int VE = Piece<E>::VE, kGroups = THREADS / G, kWaves = THREADS / 64;
    constexpr bool kSolo = THREADS == kSoloThreads;  // the one workgroup of its call
    __shared__ double s_add[kSums][kWaves];
    __shared__ int64_t s_count[kWaves];
    const int lane = threadIdx.x % G, V = (int)a.V;
    float denom = 1.0f, scale = 1.0f;
    if (LOSS) {
        if (kSolo && !(a.denom > 0.0f)) {
            const int64_t c = count_rows<THREADS>(a, s_count);
            denom = c > 0 ? (float)c : 1.0f;
        } else {
            denom = denominator(a);
        }
        scale = scale_by(a, denom);
    }
    float total[kSums] = {};  // of the group's rows, in its lane 0
    for (int64_t first = (int64_t)blockIdx.x * kGroups; first < a.n; first += (int64_t)gridDim.x * kGroups) {
        const int64_t row = first + threadIdx.x / G;
        const bool used = row < a.n;
        const int64_t action = used ? action_of(a, row) : -1;
        const bool on = used && takes_part(a, row, action);
        const E* z = static_cast<const E*>(a.logits) + row * a.row_stride;
        Piece<E> v[NV];
        float za = 0.0f;
        Inputs in{};
        // The lane's number, hidden so that what follows from it for each piece is not kept from row to row.
        int mine = lane;
        asm volatile("" : "+v"(mine));
        if (on) {
#pragma unroll
            for (int i = 0; i < NV; i++) {
                if (TINY) v[i].gather(z, V);
                else load_piece<E, G>(v[i], z, V, mine, i);
            }
            za = (float)z[action];
            if (LOSS) in = inputs_of(a, row);
        } else {
#pragma unroll
            for (int i = 0; i < NV; i++) v[i].fill();
        }
        float m = -INFINITY, S = 0.0f, dS = 0.0f;
#pragma unroll
        for (int i = 0; i < NV; i++) {
            float f[VE];
            v[i].unpack(f);
#pragma unroll
            for (int j = 0; j < VE; j++) m = fmaxf(m, f[j]);
            v[i].forget();
        }
        m = group_max<G>(m);
        const Scale dist = scale_of(m);
#pragma unroll
        for (int i = 0; i < NV; i++) {
            float f[VE];
            v[i].unpack(f);
            add_piece<false>(f, dist, S, dS);
            v[i].forget();
        }
        S = group_add<G>(S);
        dS = group_add<G>(dS);
        Row r{};
        if (on) r = row_terms<LOSS>(a, in, S, dS, dist(za), scale);
        if (used && lane == 0) {
            if (a.logp) a.logp[row] = r.lp;
            if (a.entropy) a.entropy[row] = r.H;
#pragma unroll
            for (int k = 0; k < kSums; k++) total[k] += r.sums[k];
        }
        if (LOSS && a.grad && used) {
            // Rows without part or distribution hold only -inf, and get zeros.
            E* g = static_cast<E*>(a.grad) + row * a.V;
            const bool some = on && S != 0.0f;
            const Slope slope = some ? slope_of(a, r, S) : Slope{};
            asm volatile("" : "+v"(mine));
#pragma unroll
            for (int i = 0; i < NV; i++)
                if (i * G * VE < V) store_piece<E, G, TINY, false>(g, v[i], V, mine, i, slope, dist);
            // The action's, over the value just written by the same lane.
            if (some && lane == (TINY ? 0 : (int)action / VE % G)) g[action] = (E)(slope(dist(za)) + slope.k2);
        }
    }
    if (LOSS) leave_sums<THREADS, kSolo>(a, total, denom, s_add);
}

// Rows that a workgroup shares.  Each lane sums its pieces two at a time as they
// arrive, against the largest logit it has seen so far, so one barrier a row
// is enough.  For the gradient a lane holds all its pieces; without one nothing
// is held, and few registers let two of the longest rows share a CU.  4096 rows of
// 32768 bf16 take 110 us (537 MB, 4.9 TB/s; vector units busy for about 85), 1519
// of 50001 fp16, most of them off a line's start, 78 us; log-probabilities of
// 2048 rows of 131072 bf16 97 us (5.5 TB/s).
template <typename E, int NV, int THREADS, bool LOSS>
__global__ __launch_bounds__(THREADS, LOSS ? 4 : 8) void block_kernel(const Args a) {
    constexpr int VE = Piece<E>::VE, G = THREADS, kWaves = THREADS / 64, kHeld = LOSS ? NV : 4;
    // Rows take these in turn: a row's are read after its only barrier.
    __shared__ Sums s_wave[2][kWaves];
    __shared__ Inputs s_in[2];
    __shared__ float s_za[2];
    __shared__ float s_total[kSums];  // thread 0's
    __shared__ double s_add[kSums][kWaves];
    const int V = (int)a.V;  // at most 2^17
    const float denom = LOSS ? denominator(a) : 1.0f, scale = LOSS ? scale_by(a, denom) : 1.0f;
    if (threadIdx.x < kSums) s_total[threadIdx.x] = 0.0f;
    __syncthreads();
    int turn = 0;
    for (int64_t row = blockIdx.x; row < a.n; row += gridDim.x) {
        const int64_t action = action_of(a, row);
        const E* z = static_cast<const E*>(a.logits) + row * a.row_stride;
        E* g = static_cast<E*>(a.grad) + row * a.V;
        // The lane's number, hidden so that what follows from it for each piece is not kept from row to row.
        int mine = threadIdx.x;
        asm volatile("" : "+v"(mine));
        if (takes_part(a, row, action)) {
            Piece<E> v[kHeld];
            if (LOSS) {
#pragma unroll
                for (int i = 0; i < kHeld; i++) load_piece<E, G>(v[i], z, V, mine, i);
            }
            float za = 0.0f, m = -INFINITY, S = 0.0f, dS = 0.0f;
            bool tame = true;  // the wave's pieces; the row's largest logit is looked at below
            Inputs in{};
            if (threadIdx.x == 0) {
                za = (float)z[action];
                if (LOSS) in = inputs_of(a, row);
            }
#pragma unroll 1
            for (int i0 = 0; i0 < NV; i0 += kHeld) {
                if (!LOSS) {
#pragma unroll
                    for (int i = 0; i < kHeld; i++) load_piece<E, G>(v[i], z, V, mine, i0 + i);
                }
#pragma unroll
                for (int i = 0; i < kHeld; i += 2) {
                    if ((i0 + i) * G * VE < V) {
                        float f[VE], h[VE];
                        v[i].unpack(f);
                        v[i + 1].unpack(h);
                        float top = m, low = kTame;
#pragma unroll
                        for (int j = 0; j < VE; j++) {
                            top = fmaxf(fmaxf(top, f[j]), h[j]);
                            low = fminf(fminf(low, f[j]), h[j]);
                        }
                        rescale(m, top, S, dS);
                        m = top;
                        if (__all(low > -kTame && top < kTame)) {
                            add_piece<true>(f, scale_of(m), S, dS);
                            add_piece<true>(h, scale_of(m), S, dS);
                        } else {
                            tame = false;
                            add_piece<false>(f, scale_of(m), S, dS);
                            add_piece<false>(h, scale_of(m), S, dS);
                        }
                        v[i].forget();
                        v[i + 1].forget();
                    }
                }
            }
            const float top = group_max<64>(m);
            rescale(m, top, S, dS);
            S = group_add<64>(S);
            dS = group_add<64>(dS);
            if ((threadIdx.x & 63) == 0) s_wave[turn][threadIdx.x >> 6] = Sums{top, S, dS};
            if (threadIdx.x == 0) {
                s_za[turn] = za;
                s_in[turn] = in;
            }
            __syncthreads();
            const Sums w = s_wave[turn][threadIdx.x % kWaves];
            m = group_max<kWaves>(w.m);
            S = w.S;
            dS = w.dS;
            rescale(w.m, m, S, dS);
            S = group_add<kWaves>(S);
            dS = group_add<kWaves>(dS);
            za = s_za[turn];
            in = s_in[turn];
            turn ^= 1;
            const Scale dist = scale_of(m);
            const Row r = row_terms<LOSS>(a, in, S, dS, dist(za), scale);
            if (threadIdx.x == 0) {
                if (a.logp) a.logp[row] = r.lp;
                if (a.entropy) a.entropy[row] = r.H;
#pragma unroll
                for (int k = 0; k < kSums; k++)
                    if (LOSS) s_total[k] += r.sums[k];
            }
            if (LOSS) {
                const bool some = S != 0.0f;
                const Slope slope = some ? slope_of(a, r, S) : Slope{};
                asm volatile("" : "+v"(mine));
                if (a.grad && tame && m < kTame) {
#pragma unroll
                    for (int i = 0; i < kHeld; i++)
                        if (i * G * VE < V) store_piece<E, G, false, true>(g, v[i], V, mine, i, slope, dist);
                } else if (a.grad) {
#pragma unroll
                    for (int i = 0; i < kHeld; i++)
                        if (i * G * VE < V) store_piece<E, G, false, false>(g, v[i], V, mine, i, slope, dist);
                }
                // The action's, over the value just written by the same lane.
                if (a.grad && some && mine == (int)action / VE % G) g[action] = (E)(slope(dist(za)) + slope.k2);
            }
        } else {
            if (threadIdx.x == 0) {
                if (a.logp) a.logp[row] = 0.0f;
                if (a.entropy) a.entropy[row] = 0.0f;
            }
            if (LOSS && a.grad) {
                const float zero[VE] = {};
                for (int j = mine * VE; j < V; j += G * VE) {
                    if (j + VE <= V) Vec<E, VE>::store(g + j, zero);
                    else
                        for (int k = j; k < V; k++) g[k] = (E)0.0f;
                }
            }
        }
    }
    if (LOSS) {
        float total[kSums] = {};
        if (threadIdx.x == 0) {
#pragma unroll
            for (int k = 0; k < kSums; k++) total[k] = s_total[k];
        }
        leave_sums<THREADS, false>(a, total, denom, s_add);
    }
}

// Rows longer than registers hold, of more than 131072 logits in 16 bits or 65536
// in 32: a workgroup per row, which reads it three times (log-probabilities
// twice), an element a lane and load.  Slow: 1024 rows of 151936 bf16 take 679 us,
// log-probabilities 442, where rows of 131072 take 132 and 49; of 128256 fp32 637
// and 397, where 65536 take 123 and 44.
template <typename E, bool LOSS>
__global__ __launch_bounds__(kSoloThreads) void long_kernel(const Args a) {
    constexpr int kWaves = kSoloThreads / 64;
    __shared__ float s_max[kWaves], s_sum[kWaves], s_dsum[kWaves];
    __shared__ double s_add[kSums][kWaves];
    const int wave = threadIdx.x >> 6;
    const float denom = LOSS ? denominator(a) : 1.0f;
    const float scale = LOSS ? scale_by(a, denom) : 1.0f;
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
                for (int64_t j = threadIdx.x; j < a.V; j += kSoloThreads) g[j] = (E)0.0f;
            continue;
        }
        const E* z = static_cast<const E*>(a.logits) + row * a.row_stride;
        const float za = (float)z[action];
        Inputs in{};
        if (LOSS) in = inputs_of(a, row);
        float m = -INFINITY;
        for (int64_t j = threadIdx.x; j < a.V; j += kSoloThreads) m = fmaxf(m, (float)z[j]);
        m = group_max<64>(m);
        if ((threadIdx.x & 63) == 0) s_max[wave] = m;
        __syncthreads();
#pragma unroll
        for (int k = 0; k < kWaves; k++) m = fmaxf(m, s_max[k]);
        const Scale dist = scale_of(m);
        float S = 0.0f, dS = 0.0f;
        for (int64_t j = threadIdx.x; j < a.V; j += kSoloThreads) {
            const float d = dist((float)z[j]), e = __builtin_amdgcn_exp2f(d);
            S += e;
            dS = fmaf(e, fmaxf(d, kFloor), dS);
        }
        S = group_add<64>(S);
        dS = group_add<64>(dS);
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
        const Row r = row_terms<LOSS>(a, in, S, dS, dist(za), scale);
        if (threadIdx.x == 0) {
            if (a.logp) a.logp[row] = r.lp;
            if (a.entropy) a.entropy[row] = r.H;
#pragma unroll
            for (int k = 0; k < kSums; k++) total[k] += r.sums[k];
        }
        if (g) {
            const Slope slope = S != 0.0f ? slope_of(a, r, S) : Slope{};
            for (int64_t j = threadIdx.x; j < a.V; j += kSoloThreads) {
                const float o = slope(dist((float)z[j]));
                g[j] = (E)(j == action ? o + slope.k2 : o);
            }
        }
    }
    if (LOSS) leave_sums<kSoloThreads, false>(a, total, denom, s_add);
}

// Adds the workgroups' sums, a wave for each, in 64 bits and always in the same
// order: 4.7 us for 2048, a launch and dependent loads.
__global__ __launch_bounds__(64 * kSums) void finish_kernel(const Args a, int32_t blocks) {
    const float denom = denominator(a);
    const int k = threadIdx.x >> 6;
    double v = 0.0;
#pragma unroll 8
    for (int b = threadIdx.x & 63; b < blocks; b += 64) v += (double)a.sums[k * kMaxBlocks + b];
    v = group_add<64>(v) / (double)denom;
    if ((threadIdx.x & 63) == 0) {
        if (k == 0) *a.loss = (float)v;
        else if (a.stats) a.stats[k - 1] = (float)v;
    }
}

typedef void (*Kernel)(const Args);
struct Choice {
    Kernel kernel;
    int threads, rows;  // rows that a workgroup runs at a time
    int blocks;         // workgroups that the GPU runs at a time
};
constexpr int kCUs = 256;
constexpr int resident(int threads, int waves) { return kCUs * waves * 4 / (threads / 64); }
template <typename E, int G, int NV, int WAVES, bool LOSS, bool TINY = false>
Choice held(bool solo) {
    // 64 lanes with more than 4 pieces each have more actions than one workgroup takes on.
    if constexpr (LOSS && NV <= 4) {
        if (solo) return {held_kernel<E, G, NV, kSoloThreads, 4, TINY, true>, kSoloThreads, kSoloThreads / G, 1};
    }
    constexpr int W = LOSS ? WAVES : NV > 8 ? 5 : 8;
    return {held_kernel<E, G, NV, kThreads, W, TINY, LOSS>, kThreads, kThreads / G, resident(kThreads, W)};
}
template <typename E, int NV, int THREADS, bool LOSS>
Choice block() {
    return {block_kernel<E, NV, THREADS, LOSS>, THREADS, 1, resident(THREADS, LOSS ? 4 : 8)};
}

// The kernel for rows of V: as few lanes as hold a row in four pieces each, so
// that what is done once per row is done by few (2097152 rows of 16 bf16: 116 us
// with two lanes a row, 78 with one, everything else as it then was), then up to 16
// pieces, which leaves more workgroups to hide one's barrier (4096 rows of 32768
// bf16: 115 us with 256 lanes of 16, 127 with 512 of 8).  A wave keeps rows of up to
// 12 pieces a lane to itself: 16384 rows of 2047, 2304, 4096, 5000 and 7000 bf16
// take it 45, 61, 70, 94 and (16 pieces) 116 us, and a workgroup 87, 96, 90, 117
// and 127, but 120 and 117 at 8192; log-probabilities likewise, 50 and 50 there.
// Rows of 65 to 128 pieces take 64 lanes with at most two each; 32 lanes with four
// were not tried.
// How many lanes share a row, and so the order of its sums, depends on V alone.
template <typename E, bool LOSS>
Choice choose(int64_t V, bool solo) {
    constexpr int VE = 16 / sizeof(E);
    const int64_t pieces = (V + VE - 1) / VE;
    static_assert(resident(kThreads, 8) <= kMaxBlocks, "the sums have a place per workgroup");
    if (V < VE) return held<E, 1, 1, 8, LOSS, true>(solo);
    if (pieces <= 1) return held<E, 1, 1, 8, LOSS>(solo);
    if (pieces <= 2) return held<E, 1, 2, 6, LOSS>(solo);
    if (pieces <= 4) return held<E, 1, 4, 4, LOSS>(solo);
    if (pieces <= 8) return held<E, 2, 4, 6, LOSS>(solo);
    if (pieces <= 16) return held<E, 4, 4, 6, LOSS>(solo);
    if (pieces <= 32) return held<E, 8, 4, 6, LOSS>(solo);
    if (pieces <= 64) return held<E, 16, 4, 6, LOSS>(solo);
    if (pieces <= 256) return held<E, 64, 4, 6, LOSS>(solo);
    if (pieces <= 512) return held<E, 64, 8, 4, LOSS>(solo);
    if (pieces <= 768) return held<E, 64, 12, 4, LOSS>(solo);
    if (pieces <= 1024) return block<E, 4, 256, LOSS>();
    if (pieces <= 4096) return block<E, 16, 256, LOSS>();
    if (pieces <= 8192) return block<E, 16, 512, LOSS>();
    if (pieces <= 16384) return block<E, 16, 1024, LOSS>();
    return {long_kernel<E, LOSS>, kSoloThreads, 1, resident(kSoloThreads, 4)};
}

int64_t work_bytes_of(const gear_policy_desc&) { return kSumOff + (int64_t)kSums * kMaxBlocks * (int64_t)sizeof(float); }

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
    a.mask_group = divisor(d.mask_group, d.n);
    a.adv_group = divisor(d.adv_group, d.n);
    a.weight_group = divisor(d.weight_group, d.n);
    a.action_dtype = d.action_dtype;
    return a;
}

template <bool LOSS>
hipError_t launch_rows(const Args& a, int32_t dtype, bool solo, int* blocks, hipStream_t s) {
    const Choice c = dtype == GEAR_DTYPE_F32 ? choose<float, LOSS>(a.V, solo)
                     : dtype == GEAR_DTYPE_BF16 ? choose<__bf16, LOSS>(a.V, solo) : choose<_Float16, LOSS>(a.V, solo);
    const int64_t want = (a.n + c.rows - 1) / c.rows;
    *blocks = (int)(want < c.blocks ? want : c.blocks);
    hipLaunchKernelGGL(c.kernel, dim3(*blocks), dim3(c.threads), 0, s, a);
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
    // Few logits: one workgroup does it all, and the launches saved are worth
    // more than the others would bring.
    const bool solo = a.n > 0 && a.n <= kSoloLogits / a.V && a.V <= kSoloActions;
    hipError_t e = hipSuccess;
    int blocks = 0;
    if (!solo && !(a.denom > 0.0f)) {
        const int64_t want = (a.n + kThreads * kCountRows - 1) / (kThreads * kCountRows);
        a.count_blocks = (int32_t)(want < 1 ? 1 : want < kCountBlocks ? want : kCountBlocks);
        hipLaunchKernelGGL(count_kernel, dim3(a.count_blocks), dim3(kThreads), 0, s, a);
        e = hipGetLastError();
        if (e != hipSuccess) return hip_fail(e, "gear_policy_loss: count launch");
    }
    if (a.n > 0) {
        e = launch_rows<true>(a, d->dtype, solo, &blocks, s);
        if (e != hipSuccess) return hip_fail(e, "gear_policy_loss: row launch");
        if (solo) return GEAR_OK;
    }
    hipLaunchKernelGGL(finish_kernel, dim3(1), dim3(64 * kSums), 0, s, a, blocks);
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
    int blocks = 0;
    const hipError_t e = launch_rows<false>(a, d->dtype, false, &blocks, static_cast<hipStream_t>(stream));
    return e == hipSuccess ? GEAR_OK : hip_fail(e, "gear_action_logp: launch");
}
