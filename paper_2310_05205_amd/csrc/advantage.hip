// Advantages and returns of collected windows (include/gear.h): a scan over
// each window from its last step back,
//   A_t = delta_t + k_t A_{t+1},  delta_t = r_t + gamma V_{t+1} - V_t,  k_t = gamma lambda,
// with V_{t+1} and k_t dropped after a step that ended its episode.
//
// A few bytes in and eight out per step, so memory bounds long windows and
// the launch short ones.  2 to 64 lanes share a window, 4 neighbouring steps each,
// or 64 lanes 8: a lane composes its steps' maps c -> delta + k c, the lanes' maps
// are composed by a suffix scan in registers, and each lane then runs its steps
// from the value that comes in.  Longer windows repeat that from the end with
// the value carried.  Few long windows are split into segments: one launch
// reduces each to its map, and in the next every segment composes the maps
// after it.
//
// Instructions count as much as bytes: types known only at run time, and maps
// composed step by step where k is the same for all, took twice the time.
#include "element.h"
#include "gear_internal.h"

namespace gear {
namespace {

constexpr int kThreads = 256;
constexpr int kFew = 4, kMany = 8;     // steps of a lane in a tile
constexpr int64_t kWantGroups = 8192;  // waves that fill the GPU
// Calls of fewer windows, of at least so many tiles each, are split.  In fp32, split
// and not: 1 window of 2100 steps (5 tiles) 10.4 and 9.2 us, 1 of 4200 11 and 15, 256
// of 4200 11 and 14, 256 of 16400 22 and 43, 1024 of 4200 21 and 17, 4096 of 600 18 and 10.
constexpr int64_t kWholeWindows = 1024, kSplitTiles = 6;
constexpr int64_t kMaxBlocks = 1 << 22;

// c -> P c + Z with P in [0, 1], or Z whatever c (P = -1): a step that ended
// its episode passes nothing on, not even a NaN.
struct Map {
    float P, Z;
};
__device__ __forceinline__ float apply(Map m, float c) { return m.P < 0.0f ? m.Z : fmaf(m.P, c, m.Z); }
// `late` first, then `early`.  A product of discounts does not fall below `least`,
// the smallest number above 0 unless the discount itself is 0: a product of 0
// would make a NaN of an infinity that the steps carry on.
__device__ __forceinline__ Map compose(Map early, Map late, float least) {
    return Map{early.P < 0.0f || late.P < 0.0f ? -1.0f : fmaxf(early.P * late.P, least), apply(early, late.Z)};
}

struct Args {
    const void *reward, *value;
    const uint8_t* done;
    const int32_t* lengths;
    float *adv, *ret;
    Map* maps;  // [B][S] when S > 1
    int64_t B, L, reward_b, value_b, done_b;
    int64_t seg_tiles;
    int32_t S;
    float gamma, decay;
};

// Neighbouring elements as they lie in memory: reading does not look at them,
// so that all of a tile's are on their way before any is converted.
template <typename E, int PER>
struct Steps {
    static constexpr int kWords = PER * sizeof(E) / 4, kPiece = kWords < 4 ? kWords : 4;
    typedef uint32_t piece __attribute__((ext_vector_type(kPiece)));
    uint32_t w[kWords];

    __device__ __forceinline__ void load(const E* p) {
        typedef piece loose __attribute__((aligned(sizeof(E))));
#pragma unroll
        for (int k = 0; k < kWords; k += kPiece) {
            const piece v = *reinterpret_cast<const loose*>(reinterpret_cast<const char*>(p) + 4 * k);
#pragma unroll
            for (int j = 0; j < kPiece; j++) w[k + j] = v[j];
        }
    }
    // The first `count`, the rest 0.
    __device__ __forceinline__ void load_some(const E* p, int count) {
#pragma unroll
        for (int k = 0; k < kWords; k++) w[k] = 0;
#pragma unroll
        for (int j = 0; j < PER; j++) {
            if (j >= count) continue;
            if constexpr (sizeof(E) == 4) w[j] = __builtin_bit_cast(uint32_t, p[j]);
            else w[j / 2] |= (uint32_t)__builtin_bit_cast(uint16_t, p[j]) << (16 * (j % 2));
        }
    }
    __device__ __forceinline__ float at(int j) const {
        if constexpr (sizeof(E) == 4) return __uint_as_float(w[j]);
        else return (float)__builtin_bit_cast(E, (uint16_t)(w[j / 2] >> (16 * (j % 2))));
    }
};
template <int PER>
__device__ __forceinline__ void store_steps(float* p, const float (&f)[PER], int room) {
    if (room == PER) {
#pragma unroll
        for (int j = 0; j < PER; j += 4) {
            const float g[4] = {f[j], f[j + 1], f[j + 2], f[j + 3]};
            Vec<float, 4>::store(p + j, g);
        }
    } else {
#pragma unroll
        for (int j = 0; j < PER; j++)
            if (j < room) p[j] = f[j];
    }
}
template <int PER>
__device__ __forceinline__ int clamp_steps(int64_t n) { return n < 0 ? 0 : n < PER ? (int)n : PER; }

// Inclusive scan of the G lanes' maps, each with the later ones after it.
template <int G>
__device__ __forceinline__ Map suffix(Map m, int lane, float least) {
#pragma unroll
    for (int off = 1; off < G; off <<= 1) {
        const Map o = {__shfl_down(m.P, off, G), __shfl_down(m.Z, off, G)};
        if (lane + off < G) m = compose(m, o, least);
    }
    return m;
}

// G lanes share a window or, with S > 1, a segment of one.  8192 windows of 32
// fp32 steps take 3.4 us, a launch and two dependent loads; 19 of 262147 bf16
// steps 9 us for the maps and 15 for the results, 40 MB written and 25 read
// in each: latency and instructions, with memory's share about 10.  One window of
// 4194304 fp32 steps takes 73 us for 10 us of bytes: each of its 8192 segments reads
// the maps of all later ones.  Four of 1048576 take 32.
template <typename ER, typename EV, int G, int PER, bool MAPS>
__global__ __launch_bounds__(kThreads) void advantage_kernel(const Args a) {
    const int lane = threadIdx.x % G;
    const float least = a.decay > 0.0f ? 0x1p-149f : 0.0f;
    const int64_t tile = (int64_t)G * PER, tiles = (a.L + tile - 1) / tile;
    const int64_t per_block = kThreads / G, units = a.B * a.S;
    // Every lane of a wave runs the same rounds, because the scan shuffles.
    for (int64_t first = (int64_t)blockIdx.x * per_block; first < units; first += (int64_t)gridDim.x * per_block) {
        const int64_t unit = first + threadIdx.x / G;
        const bool used = unit < units;
        const int64_t b = used ? unit / a.S : 0, seg = used ? unit - b * a.S : 0;
        int64_t n = a.L;
        if (a.lengths) n = a.lengths[b] < 0 ? 0 : a.lengths[b] < a.L ? a.lengths[b] : a.L;
        if (!used) n = 0;
        float carry = 0.0f;
        Map whole = {1.0f, 0.0f};
        if (!MAPS && a.S > 1) {
            // The maps of the later segments, a share of neighbouring ones to a lane.
            const Map* maps = a.maps + b * a.S + seg + 1;
            const int64_t later = used ? a.S - 1 - seg : 0, share = (later + G - 1) / G;
            Map m = {1.0f, 0.0f};
#pragma unroll 4
            for (int64_t k = share - 1; k >= 0; k--)
                if (lane * share + k < later) m = compose(maps[lane * share + k], m, least);
            m = suffix<G>(m, lane, least);
            carry = apply(Map{__shfl(m.P, 0, G), __shfl(m.Z, 0, G)}, 0.0f);
        }
        const int64_t k1 = (seg + 1) * a.seg_tiles < tiles ? (seg + 1) * a.seg_tiles : tiles;
        for (int64_t k = k1 - 1; k >= seg * a.seg_tiles; k--) {
            const int64_t t = k * tile + lane * PER;
            const int count = clamp_steps<PER>(n - t);
            const ER* reward = static_cast<const ER*>(a.reward) + b * a.reward_b + t;
            const EV* value = static_cast<const EV*>(a.value) + b * a.value_b + t;
            const uint8_t* done = a.done + b * a.done_b + t;
            Steps<ER, PER> rw;
            Steps<EV, PER> vw;
            Steps<EV, 4 / sizeof(EV)> last;  // the value after the lane's steps
            uint32_t ended[PER / 4] = {};
            if (__all(count == PER)) {
                rw.load(reward);
                vw.load(value);
                last.load_some(value + PER, 1);
                if (a.done) __builtin_memcpy(ended, done, PER);
            } else {
                rw.load_some(reward, count);
                vw.load_some(value, count);
                last.load_some(value + count, count > 0 ? 1 : 0);
#pragma unroll
                for (int j = 0; j < PER; j++)
                    if (a.done && j < count) ended[j / 4] |= (uint32_t)done[j] << (8 * (j % 4));
            }
            float delta[PER], v[PER], z = 0.0f, power = 1.0f;
            bool cut[PER], any = false;
#pragma unroll
            for (int j = PER - 1; j >= 0; j--) {
                v[j] = vw.at(j);
                cut[j] = (ended[j / 4] & (0xFFu << (8 * (j % 4)))) != 0;
                const float next = j + 1 < count ? v[j + 1 < PER ? j + 1 : j] : last.at(0);
                delta[j] = rw.at(j) + (cut[j] ? 0.0f : a.gamma * next) - v[j];
                if (j < count) {
                    z = cut[j] ? delta[j] : fmaf(a.decay, z, delta[j]);
                    power *= a.decay;
                    any |= cut[j];
                }
            }
            const Map mine = suffix<G>(Map{any ? -1.0f : fmaxf(power, least), z}, lane, least);
            if (!MAPS) {
                const Map later = {__shfl_down(mine.P, 1, G), __shfl_down(mine.Z, 1, G)};
                float c = lane + 1 < G ? apply(later, carry) : carry, A[PER], R[PER];
#pragma unroll
                for (int j = PER - 1; j >= 0; j--) {
                    if (j < count) c = cut[j] ? delta[j] : fmaf(a.decay, c, delta[j]);
                    A[j] = j < count ? c : 0.0f;
                    R[j] = j < count ? c + v[j] : 0.0f;
                }
                const int room = used ? clamp_steps<PER>(a.L - t) : 0;
                store_steps<PER>(a.adv + b * a.L + t, A, room);
                if (a.ret) store_steps<PER>(a.ret + b * a.L + t, R, room);
            }
            const Map head = {__shfl(mine.P, 0, G), __shfl(mine.Z, 0, G)};
            if (MAPS) whole = compose(head, whole, least);
            else carry = apply(head, carry);
        }
        if (MAPS && used && lane == 0) a.maps[b * a.S + seg] = whole;
    }
}

struct Plan {
    int G, per;
    int64_t seg_tiles;
    int32_t S;
};
Plan plan_of(const gear_advantages_desc& d) {
    Plan p;
    p.G = 2;
    while (p.G < 64 && (int64_t)p.G * kFew < d.L) p.G *= 2;
    p.per = (int64_t)p.G * kFew < d.L ? kMany : kFew;
    const int64_t tile = (int64_t)p.G * p.per, tiles = (d.L + tile - 1) / tile;
    int64_t S = d.B > 0 && d.B < kWholeWindows && tiles >= kSplitTiles ? kWantGroups / d.B : 1;
    if (S > tiles) S = tiles;
    if (S < 1) S = 1;
    p.seg_tiles = (tiles + S - 1) / S;
    p.S = p.seg_tiles > 0 ? (int32_t)((tiles + p.seg_tiles - 1) / p.seg_tiles) : 1;
    return p;
}
int64_t work_bytes_of(const gear_advantages_desc& d) {
    const Plan p = plan_of(d);
    return p.S > 1 ? p.S * d.B * (int64_t)sizeof(Map) : 0;
}

const char* flaw(const gear_advantages_desc* d) {
    if (d == nullptr) return "NULL descriptor";
    if (float_bytes(d->reward_dtype) == 0 || float_bytes(d->value_dtype) == 0) return "dtype must be F16, BF16 or F32";
    const int64_t most = 1ll << 40;
    if (d->B < 0 || d->L < 0 || d->B > most || d->L > most || (d->L > 0 && d->B > most / d->L)) return "size out of range";
    if (!(d->gamma >= 0.0f && d->gamma <= 1.0f) || !(d->lambda >= 0.0f && d->lambda <= 1.0f))
        return "gamma and lambda must lie in [0, 1]";
    return nullptr;
}

typedef void (*Kernel)(const Args);
template <typename ER, typename EV, bool MAPS>
Kernel kernel_for(const Plan& p) {
    if constexpr (!MAPS) {  // windows of one tile of few steps a lane are not split
        if (p.per == kFew) {
            switch (p.G) {
                case 2: return advantage_kernel<ER, EV, 2, kFew, false>;
                case 4: return advantage_kernel<ER, EV, 4, kFew, false>;
                case 8: return advantage_kernel<ER, EV, 8, kFew, false>;
                case 16: return advantage_kernel<ER, EV, 16, kFew, false>;
                case 32: return advantage_kernel<ER, EV, 32, kFew, false>;
                default: return advantage_kernel<ER, EV, 64, kFew, false>;
            }
        }
    }
    return advantage_kernel<ER, EV, 64, kMany, MAPS>;
}
template <typename ER, bool MAPS>
Kernel kernel_for(const Plan& p, int32_t value_dtype) {
    if (value_dtype == GEAR_DTYPE_F32) return kernel_for<ER, float, MAPS>(p);
    return value_dtype == GEAR_DTYPE_BF16 ? kernel_for<ER, __bf16, MAPS>(p) : kernel_for<ER, _Float16, MAPS>(p);
}
template <bool MAPS>
Kernel kernel_for(const Plan& p, int32_t reward_dtype, int32_t value_dtype) {
    if (reward_dtype == GEAR_DTYPE_F32) return kernel_for<float, MAPS>(p, value_dtype);
    return reward_dtype == GEAR_DTYPE_BF16 ? kernel_for<__bf16, MAPS>(p, value_dtype)
                                           : kernel_for<_Float16, MAPS>(p, value_dtype);
}

}  // namespace
}  // namespace gear

extern "C" int gear_advantages_sizes(const gear_advantages_desc* d, int64_t* work_bytes) {
    using namespace gear;
    if (const char* w = flaw(d)) return fail(GEAR_E_INVAL, std::string("gear_advantages_sizes: ") + w);
    if (work_bytes) *work_bytes = work_bytes_of(*d);
    return GEAR_OK;
}

extern "C" int gear_advantages(const gear_advantages_desc* d, const void* d_reward, const void* d_value, float* d_adv,
                               float* d_ret, void* d_work, int64_t work_bytes, void* stream) {
    using namespace gear;
    if (const char* w = flaw(d)) return fail(GEAR_E_INVAL, std::string("gear_advantages: ") + w);
    if (d->B == 0 || d->L == 0) return GEAR_OK;
    if (d_reward == nullptr || d_value == nullptr || d_adv == nullptr)
        return fail(GEAR_E_INVAL, "gear_advantages: NULL pointer argument");
    const int64_t need = work_bytes_of(*d);
    if (need > 0 && (d_work == nullptr || work_bytes < need))
        return fail(GEAR_E_INVAL, "gear_advantages: workspace smaller than gear_advantages_sizes states");
    const Plan p = plan_of(*d);
    Args a{};
    a.reward = d_reward;
    a.value = d_value;
    a.done = d->d_done;
    a.lengths = d->d_lengths;
    a.adv = d_adv;
    a.ret = d_ret;
    a.maps = static_cast<Map*>(d_work);
    a.B = d->B;
    a.L = d->L;
    a.reward_b = d->reward_b;
    a.value_b = d->value_b;
    a.done_b = d->done_b;
    a.seg_tiles = p.seg_tiles;
    a.S = p.S;
    a.gamma = d->gamma;
    a.decay = d->gamma * d->lambda;
    hipStream_t s = static_cast<hipStream_t>(stream);
    (void)hipGetLastError();  // an error pending from an earlier HIP call is not this call's
    const int64_t per_block = kThreads / p.G, want = (d->B * p.S + per_block - 1) / per_block;
    const unsigned blocks = (unsigned)(want < kMaxBlocks ? want : kMaxBlocks);
    if (p.S > 1) {
        hipLaunchKernelGGL(kernel_for<true>(p, d->reward_dtype, d->value_dtype), dim3(blocks), dim3(kThreads), 0, s, a);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return hip_fail(e, "gear_advantages: launch");
    }
    hipLaunchKernelGGL(kernel_for<false>(p, d->reward_dtype, d->value_dtype), dim3(blocks), dim3(kThreads), 0, s, a);
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? GEAR_OK : hip_fail(e, "gear_advantages: launch");
}
