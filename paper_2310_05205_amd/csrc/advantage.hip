// Advantages and returns of collected windows (include/gear.h): a scan over
// each window from its last step back,
//   A_t = delta_t + k_t A_{t+1},  delta_t = r_t + gamma V_{t+1} - V_t,  k_t = gamma lambda,
// with V_{t+1} and k_t dropped after a step that ended its episode.
//
// A few bytes in and eight out per step, so memory bounds long windows and
// the launch short ones.  2 to 64 lanes share a window, four steps each: a
// lane composes its steps' maps c -> delta + k c, the lanes' maps are composed
// by a suffix scan in registers, and each lane then runs its steps from the
// value that comes in.  Longer windows repeat that from the end with the
// value carried.  Few long windows are split into segments: one launch
// reduces each to its map, and in the next every segment composes the maps
// after it.
#include "element.h"
#include "gear_internal.h"

namespace gear {
namespace {

constexpr int kPer = 4;            // steps of a lane in a tile
constexpr int kThreads = 256;
constexpr int64_t kWantGroups = 4096;  // waves that fill the GPU
constexpr int64_t kMinSegTiles = 4;
constexpr int64_t kMaxBlocks = 1 << 22;

// c -> P c + Z with P in [0, 1], or Z whatever c (P = -1): a step that ended
// its episode passes nothing on, not even a NaN.
struct Map {
    float P, Z;
};
__device__ __forceinline__ float apply(Map m, float c) { return m.P < 0.0f ? m.Z : fmaf(m.P, c, m.Z); }
// `late` first, then `early`.
__device__ __forceinline__ Map compose(Map early, Map late) {
    return Map{early.P < 0.0f || late.P < 0.0f ? -1.0f : early.P * late.P, apply(early, late.Z)};
}

struct Args {
    const void *reward, *value;
    const uint8_t* done;
    const int32_t* lengths;
    float *adv, *ret;
    Map* maps;  // [S][B] when S > 1
    int64_t B, L, reward_b, value_b, done_b;
    int64_t seg_tiles;
    int32_t S, reward_dtype, value_dtype;
    float gamma, decay;
};

// Elements [i, i + count) of an array as floats.
template <typename E>
__device__ __forceinline__ void load_steps(const void* p, int64_t i, int count, float (&f)[kPer]) {
    const E* e = static_cast<const E*>(p) + i;
    if (count == kPer) {
        Vec<E, kPer>::unpack(Vec<E, kPer>::load(e), f);
    } else {
#pragma unroll
        for (int j = 0; j < kPer; j++) f[j] = j < count ? (float)e[j] : 0.0f;
    }
}
__device__ __forceinline__ void load_steps(const void* p, int32_t dtype, int64_t i, int count, float (&f)[kPer]) {
    if (dtype == GEAR_DTYPE_F32) load_steps<float>(p, i, count, f);
    else if (dtype == GEAR_DTYPE_BF16) load_steps<__bf16>(p, i, count, f);
    else load_steps<_Float16>(p, i, count, f);
}

// G lanes share a window or, with S > 1, a segment of one.
template <int G, bool MAPS>
__global__ __launch_bounds__(kThreads) void advantage_kernel(const Args a) {
    const int lane = threadIdx.x % G;
    const int64_t tile = (int64_t)G * kPer, tiles = (a.L + tile - 1) / tile;
    const int64_t per_block = kThreads / G, units = a.B * a.S;
    // Every lane of a wave runs the same rounds, because the scan shuffles.
    for (int64_t first = (int64_t)blockIdx.x * per_block; first < units; first += (int64_t)gridDim.x * per_block) {
        const int64_t unit = first + threadIdx.x / G;
        const bool used = unit < units;
        const int64_t seg = used ? unit / a.B : 0, b = used ? unit - seg * a.B : 0;
        int64_t n = a.L;
        if (a.lengths) n = a.lengths[b] < 0 ? 0 : a.lengths[b] < a.L ? a.lengths[b] : a.L;
        if (!used) n = 0;
        float carry = 0.0f;
        Map whole = {1.0f, 0.0f};
        if (!MAPS && a.S > 1) {
            // The maps of the later segments, 64 at a time from the last on.
            const int64_t later = a.S - 1 - seg;
            for (int64_t base = (a.S - 1) / G * G; base >= 0; base -= G) {
                const int64_t k = base + lane;
                Map m = {1.0f, 0.0f};
                if (used && k < later) m = a.maps[(seg + 1 + k) * a.B + b];
#pragma unroll
                for (int off = 1; off < G; off <<= 1) {
                    const Map o = {__shfl_down(m.P, off, G), __shfl_down(m.Z, off, G)};
                    if (lane + off < G) m = compose(m, o);
                }
                carry = apply(Map{__shfl(m.P, 0, G), __shfl(m.Z, 0, G)}, carry);
            }
        }
        int64_t k1 = (seg + 1) * a.seg_tiles < tiles ? (seg + 1) * a.seg_tiles : tiles;
        for (int64_t k = k1 - 1; k >= seg * a.seg_tiles; k--) {
            const int64_t t = k * tile + lane * kPer;
            const int count = n - t >= kPer ? kPer : n > t ? (int)(n - t) : 0;
            const int room = a.L - t >= kPer ? kPer : a.L > t ? (int)(a.L - t) : 0;
            float r[kPer] = {}, v[kPer] = {}, after[kPer] = {};
            Map m[kPer];
            if (count > 0) {
                load_steps(a.reward, a.reward_dtype, b * a.reward_b + t, count, r);
                load_steps(a.value, a.value_dtype, b * a.value_b + t, count, v);
                load_steps(a.value, a.value_dtype, b * a.value_b + t + 1, count, after);
            }
            uint32_t ended = 0;
            if (a.done && count > 0) {
                const uint8_t* p = a.done + b * a.done_b + t;
                if (count == kPer) __builtin_memcpy(&ended, p, kPer);
                else
                    for (int j = 0; j < count; j++) ended |= (uint32_t)p[j] << (8 * j);
            }
            Map mine = {1.0f, 0.0f};
#pragma unroll
            for (int j = kPer - 1; j >= 0; j--) {
                const bool cut = ((ended >> (8 * j)) & 0xFFu) != 0;
                m[j] = Map{1.0f, 0.0f};
                if (j < count) m[j] = Map{cut ? -1.0f : a.decay, r[j] + (cut ? 0.0f : a.gamma * after[j]) - v[j]};
                mine = compose(m[j], mine);
            }
#pragma unroll
            for (int off = 1; off < G; off <<= 1) {
                const Map o = {__shfl_down(mine.P, off, G), __shfl_down(mine.Z, off, G)};
                if (lane + off < G) mine = compose(mine, o);
            }
            if (!MAPS) {
                const Map next = {__shfl_down(mine.P, 1, G), __shfl_down(mine.Z, 1, G)};
                float c = lane + 1 < G ? apply(next, carry) : carry;
                float A[kPer], R[kPer];
#pragma unroll
                for (int j = kPer - 1; j >= 0; j--) {
                    c = apply(m[j], c);
                    A[j] = j < count ? c : 0.0f;
                    R[j] = j < count ? c + v[j] : 0.0f;
                }
                const int64_t o = b * a.L + t;
                if (used && room == kPer) {
                    Vec<float, kPer>::store(a.adv + o, A);
                    if (a.ret) Vec<float, kPer>::store(a.ret + o, R);
                } else if (used) {
#pragma unroll
                    for (int j = 0; j < kPer; j++)
                        if (j < room) {
                            a.adv[o + j] = A[j];
                            if (a.ret) a.ret[o + j] = R[j];
                        }
                }
            }
            const Map head = {__shfl(mine.P, 0, G), __shfl(mine.Z, 0, G)};
            if (MAPS) whole = compose(head, whole);
            else carry = apply(head, carry);
        }
        if (MAPS && used && lane == 0) a.maps[seg * a.B + b] = whole;
    }
}

struct Plan {
    int G;
    int64_t seg_tiles;
    int32_t S;
};
Plan plan_of(const gear_advantages_desc& d) {
    Plan p;
    p.G = 2;
    while (p.G < 64 && (int64_t)p.G * kPer < d.L) p.G *= 2;
    const int64_t tile = (int64_t)p.G * kPer, tiles = (d.L + tile - 1) / tile;
    int64_t S = d.B > 0 ? kWantGroups / d.B : 1;
    if (S > tiles / kMinSegTiles) S = tiles / kMinSegTiles;
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
template <bool MAPS>
Kernel kernel_for(int G) {
    switch (G) {
        case 2: return advantage_kernel<2, MAPS>;
        case 4: return advantage_kernel<4, MAPS>;
        case 8: return advantage_kernel<8, MAPS>;
        case 16: return advantage_kernel<16, MAPS>;
        case 32: return advantage_kernel<32, MAPS>;
        default: return advantage_kernel<64, MAPS>;
    }
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
    a.reward_dtype = d->reward_dtype;
    a.value_dtype = d->value_dtype;
    a.gamma = d->gamma;
    a.decay = d->gamma * d->lambda;
    hipStream_t s = static_cast<hipStream_t>(stream);
    (void)hipGetLastError();  // an error pending from an earlier HIP call is not this call's
    const int64_t per_block = kThreads / p.G, want = (d->B * p.S + per_block - 1) / per_block;
    const unsigned blocks = (unsigned)(want < kMaxBlocks ? want : kMaxBlocks);
    if (p.S > 1) {
        hipLaunchKernelGGL(kernel_for<true>(p.G), dim3(blocks), dim3(kThreads), 0, s, a);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return hip_fail(e, "gear_advantages: launch");
    }
    hipLaunchKernelGGL(kernel_for<false>(p.G), dim3(blocks), dim3(kThreads), 0, s, a);
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? GEAR_OK : hip_fail(e, "gear_advantages: launch");
}
