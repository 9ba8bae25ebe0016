// The gated linear recurrence over collected windows (include/gear.h):
//   h_t = a_t h_{t-1} + u_t,  a = gate, u = x             (value form)
//                             a = f, u = (1 - f) x, f = sigmoid(gate)
// and its gradients, from the last step back:
//   G_t = dy_t + a_{t+1} G_{t+1},  dx_t = G_t du/dx,  dgate_t = G_t dh_t/dgate,
// where a reset makes h_{t-1} count as 0 and cuts the chain in both directions.
//
// Both directions read and write every element once and do a few operations
// on it, so memory bounds them.  A lane owns the 8 bytes of neighbouring
// channels of one window and walks its steps in tiles of 16, whose loads are
// all issued before the first is used.  Windows and channels give the
// parallelism; where they are too few to fill the GPU, the steps are split
// into segments: one launch reduces every segment to what it does to a state
// carried through it (an affine map), one applies the maps in order, and the
// last runs every segment from its own first state.
#include "element.h"
#include "gear_internal.h"

namespace gear {
namespace {

constexpr int kSteps = GEAR_RECURRENCE_STEPS;  // steps of a tile
constexpr int kForwardBytes = 8, kBackwardBytes = 4;  // neighbouring channels of a lane
constexpr int kThreads = 256;
constexpr int kWantLanes = 2048 * 64;  // lanes that fill the GPU
constexpr int64_t kMaxBlocks = 1 << 22;

// A map c -> P c + Z of a carried value; a reset inside it cuts the value
// off, which P holds as these bits (a NaN that no operation makes), because
// 0 c would be NaN for an infinite c.
constexpr uint32_t kCutBits = 0x7FC0DEADu;
struct Map {
    float P, Z;
};
__device__ __forceinline__ float apply(Map m, float c) {
    return __float_as_uint(m.P) == kCutBits ? m.Z : fmaf(m.P, c, m.Z);
}

// `early` first, then `late`.
__device__ __forceinline__ Map compose(Map late, Map early) {
    const bool cut = __float_as_uint(late.P) == kCutBits || __float_as_uint(early.P) == kCutBits;
    return Map{cut ? __uint_as_float(kCutBits) : late.P * early.P, apply(late, early.Z)};
}

struct Args {
    const void *gate, *x, *dy;
    const float *state, *saved, *dfinal;
    void *y, *dgate, *dx;
    float *final_state, *out_saved, *dstate;
    const uint8_t* reset;
    const int32_t* lengths;
    Map* maps;            // [S][B][D] when S > 1; their first states after carry_kernel
    int64_t B, T, D, gate_b, gate_t, x_b, x_t, dy_b, dy_t, reset_b;
    int64_t groups;       // of VE channels in a window
    int64_t lanes;        // B * groups
    int64_t seg_tiles;    // tiles of a segment
    int32_t S;
};

// A lane's place: window b, first channel c, and the steps of its window.
struct Place {
    int64_t b, c, n;
};
template <int VE>
__device__ __forceinline__ Place place_of(const Args& a, int64_t q) {
    Place p;
    p.b = q / a.groups;
    p.c = (q - p.b * a.groups) * VE;
    // The last group of a width that VE does not divide moves back: the
    // channels it shares are computed twice, with the same results.
    if (p.c > a.D - VE) p.c = a.D - VE;
    p.n = a.T;
    if (a.lengths) {
        const int64_t n = a.lengths[p.b];
        p.n = n < 0 ? 0 : n < a.T ? n : a.T;
    }
    return p;
}

// Resets of steps [t0, t0 + count), one bit each.
__device__ __forceinline__ uint32_t resets(const Args& a, int64_t b, int64_t t0, int count) {
    if (a.reset == nullptr) return 0;
    const uint8_t* r = a.reset + b * a.reset_b + t0;
    uint32_t bits = 0;
    if (count == kSteps) {
        uint32_t w[kSteps / 4];
        __builtin_memcpy(w, r, sizeof(w));
#pragma unroll
        for (int i = 0; i < kSteps; i++) bits |= ((w[i / 4] >> (8 * (i % 4))) & 0xFFu) != 0 ? 1u << i : 0u;
    } else {
        for (int i = 0; i < count; i++) bits |= r[i] != 0 ? 1u << i : 0u;
    }
    return bits;
}

// Decay and input weight of a gate.  With e = exp(-g) they are 1 / (1 + e) and
// e / (1 + e), neither of which cancels; where e is large the latter is 1,
// and its product would fail as the decay underflows.  A NaN stays one.
template <int FORM>
__device__ __forceinline__ void gates(float g, float& f, float& w) {
    if (FORM == GEAR_GATE_VALUE) {
        f = g;
        w = 1.0f;
    } else {
        const float e = fast_exp(-g);
        f = __builtin_amdgcn_rcpf(1.0f + e);
        w = e > 0x1p30f ? 1.0f : e * f;
    }
}

// What the lanes of a wave have in common at a tile: every step of it and no
// reset, every step, or anything else.  The first two run without a branch
// per step, so that the steps' gates are computed side by side.
enum { kPlain = 0, kCuts = 1, kAny = 2 };
__device__ __forceinline__ int mode_of(int count, uint32_t r) {
    if (!__all(count == kSteps)) return kAny;
    return __any(r != 0) ? kCuts : kPlain;
}

template <typename E, int VE>
struct Tile {
    typename Vec<E, VE>::raw v[kSteps];
    template <int MODE>
    __device__ __forceinline__ void load(const E* p, int64_t stride, int count) {
#pragma unroll
        for (int i = 0; i < kSteps; i++)
            if (MODE != kAny || i < count) v[i] = Vec<E, VE>::load(p + i * stride);
    }
};

__device__ __forceinline__ int clamp_count(int64_t n) { return n < 0 ? 0 : n < kSteps ? (int)n : kSteps; }

// A lane's pointers at its window and channels.
template <typename E>
struct Rows {
    const E *gate, *x, *dy;
    E *y, *dgate, *dx;
};
template <typename E>
__device__ __forceinline__ Rows<E> rows_of(const Args& a, const Place& p) {
    Rows<E> r;
    r.gate = static_cast<const E*>(a.gate) + p.b * a.gate_b + p.c;
    r.x = static_cast<const E*>(a.x) + p.b * a.x_b + p.c;
    r.dy = a.dy ? static_cast<const E*>(a.dy) + p.b * a.dy_b + p.c : nullptr;
    r.y = static_cast<E*>(a.y) + p.b * a.T * a.D + p.c;
    r.dgate = static_cast<E*>(a.dgate) + p.b * a.T * a.D + p.c;
    r.dx = static_cast<E*>(a.dx) + p.b * a.T * a.D + p.c;
    return r;
}

// `count` steps of the recurrence from step t0 on; zeros up to `room`.
template <typename E, int VE, int FORM, bool MAPS, int MODE>
__device__ __forceinline__ void forward_tile(const Args& a, const Rows<E>& rows, int64_t t0, int count, int room,
                                             uint32_t r, float (&h)[VE], float (&P)[VE]) {
#pragma clang fp contract(off)  // the modes round alike: lanes that share channels may run different ones
    Tile<E, VE> g, x;
    g.template load<MODE>(rows.gate + t0 * a.gate_t, a.gate_t, count);
    x.template load<MODE>(rows.x + t0 * a.x_t, a.x_t, count);
    E* y = rows.y + t0 * a.D;
#pragma unroll
    for (int s = 0; s < kSteps; s++) {
        if (MODE != kAny || s < count) {
            float gv[VE], xv[VE];
            Vec<E, VE>::unpack(g.v[s], gv);
            Vec<E, VE>::unpack(x.v[s], xv);
            const bool z = MODE != kPlain && ((r >> s) & 1u);
#pragma unroll
            for (int j = 0; j < VE; j++) {
                float f, w;
                gates<FORM>(gv[j], f, w);
                const float u = FORM == GEAR_GATE_VALUE ? xv[j] : w * xv[j];
                h[j] = z ? u : fmaf(f, h[j], u);
                if (MAPS) P[j] *= f;
            }
            if (!MAPS && a.y) Vec<E, VE>::store(y + s * a.D, h);
        } else if (!MAPS && s < room && a.y) {
            const float zero[VE] = {};
            Vec<E, VE>::store(y + s * a.D, zero);
        }
    }
}

// Segments forward: with MAPS, reduces each to its map; else the whole recurrence.
template <typename E, int VE, int FORM, bool MAPS>
__global__ __launch_bounds__(kThreads) void forward_kernel(const Args a) {
    const int64_t BD = a.B * a.D, tiles = (a.T + kSteps - 1) / kSteps;
    for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < a.lanes * a.S;
         i += (int64_t)gridDim.x * kThreads) {
        const int64_t seg = i / a.lanes;
        const Place p = place_of<VE>(a, i - seg * a.lanes);
        const Rows<E> rows = rows_of<E>(a, p);
        const int64_t at = p.b * a.D + p.c;
        float h[VE], P[VE];
        bool cut = false;
#pragma unroll
        for (int j = 0; j < VE; j++) {
            P[j] = 1.0f;
            h[j] = MAPS || !a.state ? 0.0f : a.state[at + j];
            if (!MAPS && a.S > 1) h[j] = a.maps[seg * BD + at + j].P;
        }
        const int64_t k1 = (seg + 1) * a.seg_tiles < tiles ? (seg + 1) * a.seg_tiles : tiles;
        for (int64_t k = seg * a.seg_tiles; k < k1; k++) {
            const int64_t t0 = k * kSteps;
            const int count = clamp_count(p.n - t0), room = clamp_count(a.T - t0);
            if (!MAPS && a.out_saved && k > 0) Vec<float, VE>::store(a.out_saved + (k - 1) * BD + at, h);
            const uint32_t r = resets(a, p.b, t0, count);
            cut |= r != 0;
            const int mode = mode_of(count, r);
            if (mode == kPlain) forward_tile<E, VE, FORM, MAPS, kPlain>(a, rows, t0, count, room, r, h, P);
            else if (mode == kCuts) forward_tile<E, VE, FORM, MAPS, kCuts>(a, rows, t0, count, room, r, h, P);
            else forward_tile<E, VE, FORM, MAPS, kAny>(a, rows, t0, count, room, r, h, P);
        }
        if (MAPS) {
#pragma unroll
            for (int j = 0; j < VE; j++)
                a.maps[seg * BD + at + j] = Map{cut ? __uint_as_float(kCutBits) : P[j], h[j]};
        } else if (a.final_state && seg == a.S - 1) {
            Vec<float, VE>::store(a.final_state + at, h);
        }
    }
}

// Applies every channel's maps in order (the last segment first when
// BACKWARD) and leaves the value each segment starts from in its map.  A
// workgroup takes 64 channels; its waves compose a run of segments each, the
// runs' maps lead to every run's first value, and the waves go through their
// runs again.  (A thread per channel took 261 us for 1024 segments of 512.)
constexpr int kCarryWaves = 16, kCarryAhead = 8;
template <bool BACKWARD>
__global__ __launch_bounds__(64 * kCarryWaves) void carry_kernel(Map* __restrict__ maps, const float* __restrict__ first,
                                                                int64_t channels, int32_t S) {
    __shared__ Map s_run[kCarryWaves][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t i = (int64_t)blockIdx.x * 64 + lane;
    const bool used = i < channels;
    const int32_t run = (S + kCarryWaves - 1) / kCarryWaves;
    const int32_t s0 = wave * run < S ? wave * run : S, s1 = s0 + run < S ? s0 + run : S;
    Map whole = {1.0f, 0.0f};
    if (used) {
        for (int32_t s = s0; s < s1; s += kCarryAhead) {
            Map m[kCarryAhead];
#pragma unroll
            for (int k = 0; k < kCarryAhead; k++)
                if (s + k < s1) m[k] = maps[(BACKWARD ? S - 1 - (s + k) : s + k) * channels + i];
#pragma unroll
            for (int k = 0; k < kCarryAhead; k++)
                if (s + k < s1) whole = compose(m[k], whole);
        }
    }
    s_run[wave][lane] = whole;
    __syncthreads();
    if (!used) return;
    float c = first ? first[i] : 0.0f;
    for (int k = 0; k < wave; k++) c = apply(s_run[k][lane], c);
    for (int32_t s = s0; s < s1; s += kCarryAhead) {
        Map m[kCarryAhead];
#pragma unroll
        for (int k = 0; k < kCarryAhead; k++)
            if (s + k < s1) m[k] = maps[(BACKWARD ? S - 1 - (s + k) : s + k) * channels + i];
#pragma unroll
        for (int k = 0; k < kCarryAhead; k++) {
            if (s + k < s1) {
                maps[(BACKWARD ? S - 1 - (s + k) : s + k) * channels + i].P = c;
                c = apply(m[k], c);
            }
        }
    }
}

// A tile backward: G comes in as the gradient of the state after it and goes
// out as that of the state before it.  h is the state before it, from which
// the states inside are recomputed in 32 bits: read back from y they would carry
// its rounding into h_{t-1} - x_t.
template <typename E, int VE, int FORM, bool MAPS, int MODE>
__device__ __forceinline__ void backward_tile(const Args& a, const Rows<E>& rows, int64_t t0, int count, int room,
                                              uint32_t r, float (&h)[VE], float (&G)[VE], float (&P)[VE]) {
#pragma clang fp contract(off)  // as forward_tile
    Tile<E, VE> g, x, d;
    g.template load<MODE>(rows.gate + t0 * a.gate_t, a.gate_t, count);
    if (!MAPS) x.template load<MODE>(rows.x + t0 * a.x_t, a.x_t, count);
    if (rows.dy) d.template load<MODE>(rows.dy + t0 * a.dy_t, a.dy_t, count);
    // Per step: decay, input weight, and what the gate's gradient is a multiple of.
    float F[kSteps][VE], W[kSteps][VE], Q[kSteps][VE];
#pragma unroll
    for (int s = 0; s < kSteps; s++) {
        if (MODE != kAny || s < count) {
            float gv[VE], xv[VE];
            Vec<E, VE>::unpack(g.v[s], gv);
            if (!MAPS) Vec<E, VE>::unpack(x.v[s], xv);
            const bool z = MODE != kPlain && ((r >> s) & 1u);
#pragma unroll
            for (int j = 0; j < VE; j++) {
                gates<FORM>(gv[j], F[s][j], W[s][j]);
                if (!MAPS) {
                    const float before = z ? 0.0f : h[j];
                    const float u = FORM == GEAR_GATE_VALUE ? xv[j] : W[s][j] * xv[j];
                    Q[s][j] = FORM == GEAR_GATE_VALUE ? before : before - xv[j];
                    h[j] = z ? u : fmaf(F[s][j], h[j], u);
                }
            }
        }
    }
    E* dgate = rows.dgate + t0 * a.D;
    E* dx = rows.dx + t0 * a.D;
#pragma unroll
    for (int s = kSteps - 1; s >= 0; s--) {
        if (MODE != kAny || s < count) {
            float dv[VE] = {}, og[VE], ox[VE];
            if (rows.dy) Vec<E, VE>::unpack(d.v[s], dv);
            const bool z = MODE != kPlain && ((r >> s) & 1u);
#pragma unroll
            for (int j = 0; j < VE; j++) {
                const float f = F[s][j], t = G[j] + dv[j];
                if (!MAPS) {
                    ox[j] = FORM == GEAR_GATE_VALUE ? t : t * W[s][j];
                    og[j] = FORM == GEAR_GATE_VALUE ? t * Q[s][j] : ox[j] * Q[s][j] * f;
                }
                G[j] = z ? 0.0f : f * t;
                if (MAPS) P[j] *= f;
            }
            if (!MAPS) {
                Vec<E, VE>::store(dgate + s * a.D, og);
                Vec<E, VE>::store(dx + s * a.D, ox);
            }
        } else if (!MAPS && s < room) {
            const float zero[VE] = {};
            Vec<E, VE>::store(dgate + s * a.D, zero);
            Vec<E, VE>::store(dx + s * a.D, zero);
        }
    }
}

// Segments backward: with MAPS, reduces each to what it does to the gradient
// that comes in at its end; else the gradients.
template <typename E, int VE, int FORM, bool MAPS>
__global__ __launch_bounds__(kThreads) void backward_kernel(const Args a) {
    const int64_t BD = a.B * a.D, tiles = (a.T + kSteps - 1) / kSteps;
    for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < a.lanes * a.S;
         i += (int64_t)gridDim.x * kThreads) {
        const int64_t seg = i / a.lanes;
        const Place p = place_of<VE>(a, i - seg * a.lanes);
        const Rows<E> rows = rows_of<E>(a, p);
        const int64_t at = p.b * a.D + p.c;
        float G[VE], P[VE];
        bool cut = false;
#pragma unroll
        for (int j = 0; j < VE; j++) {
            P[j] = 1.0f;
            G[j] = MAPS || !a.dfinal ? 0.0f : a.dfinal[at + j];
            if (!MAPS && a.S > 1) G[j] = a.maps[seg * BD + at + j].P;
        }
        const int64_t k1 = (seg + 1) * a.seg_tiles < tiles ? (seg + 1) * a.seg_tiles : tiles;
        for (int64_t k = k1 - 1; k >= seg * a.seg_tiles; k--) {
            const int64_t t0 = k * kSteps;
            const int count = clamp_count(p.n - t0), room = clamp_count(a.T - t0);
            const uint32_t r = resets(a, p.b, t0, count);
            cut |= r != 0;
            float h[VE] = {};
            if (!MAPS && count > 0) {
                const float* from = k > 0 ? a.saved + (k - 1) * BD + at : a.state ? a.state + at : nullptr;
                if (from) {
#pragma unroll
                    for (int j = 0; j < VE; j++) h[j] = from[j];
                }
            }
            const int mode = mode_of(count, r);
            if (mode == kPlain) backward_tile<E, VE, FORM, MAPS, kPlain>(a, rows, t0, count, room, r, h, G, P);
            else if (mode == kCuts) backward_tile<E, VE, FORM, MAPS, kCuts>(a, rows, t0, count, room, r, h, G, P);
            else backward_tile<E, VE, FORM, MAPS, kAny>(a, rows, t0, count, room, r, h, G, P);
        }
        if (MAPS) {
#pragma unroll
            for (int j = 0; j < VE; j++)
                a.maps[seg * BD + at + j] = Map{cut ? __uint_as_float(kCutBits) : P[j], G[j]};
        } else if (a.dstate && seg == 0) {
            Vec<float, VE>::store(a.dstate + at, G);
        }
    }
}

typedef void (*Kernel)(const Args);
struct Kernels {
    Kernel maps, whole;
};
template <typename E, int VE, int FORM, bool BACKWARD>
Kernels kernels_of() {
    if constexpr (BACKWARD) return {backward_kernel<E, VE, FORM, true>, backward_kernel<E, VE, FORM, false>};
    else return {forward_kernel<E, VE, FORM, true>, forward_kernel<E, VE, FORM, false>};
}
template <typename E, bool BACKWARD>
Kernels kernels_for(int32_t form, bool wide) {
    constexpr int VE = (BACKWARD ? kBackwardBytes : kForwardBytes) / sizeof(E);
    if (form == GEAR_GATE_VALUE)
        return wide ? kernels_of<E, VE, GEAR_GATE_VALUE, BACKWARD>() : kernels_of<E, 1, GEAR_GATE_VALUE, BACKWARD>();
    return wide ? kernels_of<E, VE, GEAR_GATE_SIGMOID, BACKWARD>() : kernels_of<E, 1, GEAR_GATE_SIGMOID, BACKWARD>();
}

// How a call is cut: channels per lane, lanes, segments.
struct Plan {
    int ve;
    int64_t groups, lanes, tiles, seg_tiles;
    int32_t S;
};
Plan plan_of(const gear_recurrence_desc& d, bool backward, bool in_place) {
    Plan p;
    const int full = (backward ? kBackwardBytes : kForwardBytes) / float_bytes(d.dtype);
    // Widths below a lane's are taken channel by channel, as are odd ones
    // whose states are updated in place: lanes that share channels must not
    // read what another has written.
    p.ve = d.D < full || (in_place && d.D % full != 0) ? 1 : full;
    p.groups = (d.D + p.ve - 1) / p.ve;
    p.lanes = d.B * p.groups;
    p.tiles = (d.T + kSteps - 1) / kSteps;
    int64_t S = p.lanes > 0 ? kWantLanes / p.lanes : 1;
    if (S > p.tiles) S = p.tiles;
    if (S < 1) S = 1;
    p.seg_tiles = (p.tiles + S - 1) / S;
    p.S = p.seg_tiles > 0 ? (int32_t)((p.tiles + p.seg_tiles - 1) / p.seg_tiles) : 1;
    return p;
}
int64_t work_bytes_of(const gear_recurrence_desc& d) {
    const int32_t f = plan_of(d, false, false).S, b = plan_of(d, true, false).S, S = f > b ? f : b;
    return S > 1 ? (int64_t)S * d.B * d.D * (int64_t)sizeof(Map) : 0;
}
int64_t saved_bytes_of(const gear_recurrence_desc& d) {
    const int64_t tiles = (d.T + kSteps - 1) / kSteps;
    return tiles > 1 ? (tiles - 1) * d.B * d.D * (int64_t)sizeof(float) : 0;
}

unsigned blocks_for(int64_t items) {
    const int64_t b = (items + kThreads - 1) / kThreads;
    return (unsigned)(b < kMaxBlocks ? b : kMaxBlocks);
}

// NULL when the descriptor is sound, else what is wrong with it.
const char* flaw(const gear_recurrence_desc* d) {
    if (d == nullptr) return "NULL descriptor";
    if (float_bytes(d->dtype) == 0) return "dtype must be F16, BF16 or F32";
    if (d->form != GEAR_GATE_VALUE && d->form != GEAR_GATE_SIGMOID) return "unknown gate form";
    if (d->B < 0 || d->T < 0 || d->D < 0) return "negative size";
    // Element counts up to 2^40 keep every byte offset far inside 64 bits.
    const int64_t most = 1ll << 40;
    if (d->B > most || d->T > most || d->D > most) return "size out of range";
    if (d->B > 0 && d->T > 0 && d->D > 0 && (d->B > most / d->T || d->B * d->T > most / d->D)) return "size out of range";
    if (d->B > 0 && d->D > 0 && d->B > most / d->D) return "size out of range";
    return nullptr;
}

template <typename E>
int run(const Args& base, const Plan& p, int32_t form, bool backward, const char* what, hipStream_t s) {
    const Kernels k = backward ? kernels_for<E, true>(form, p.ve > 1) : kernels_for<E, false>(form, p.ve > 1);
    const int64_t BD = base.B * base.D;
    if (p.S > 1) {
        hipLaunchKernelGGL(k.maps, dim3(blocks_for(p.lanes * p.S)), dim3(kThreads), 0, s, base);
        hipError_t e = hipGetLastError();
        if (e != hipSuccess) return hip_fail(e, what);
        hipLaunchKernelGGL(backward ? carry_kernel<true> : carry_kernel<false>, dim3((unsigned)((BD + 63) / 64)),
                           dim3(64 * kCarryWaves), 0, s, base.maps, backward ? base.dfinal : base.state, BD, p.S);
        e = hipGetLastError();
        if (e != hipSuccess) return hip_fail(e, what);
    }
    hipLaunchKernelGGL(k.whole, dim3(blocks_for(p.lanes * p.S)), dim3(kThreads), 0, s, base);
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? GEAR_OK : hip_fail(e, what);
}

int dispatch(const Args& base, const Plan& p, const gear_recurrence_desc& d, bool backward, const char* what,
             hipStream_t s) {
    if (p.lanes == 0) return GEAR_OK;
    (void)hipGetLastError();  // an error pending from an earlier HIP call is not this call's
    if (d.dtype == GEAR_DTYPE_F32) return run<float>(base, p, d.form, backward, what, s);
    if (d.dtype == GEAR_DTYPE_BF16) return run<__bf16>(base, p, d.form, backward, what, s);
    return run<_Float16>(base, p, d.form, backward, what, s);
}

Args args_of(const gear_recurrence_desc& d, const Plan& p, void* work) {
    Args a{};
    a.reset = d.d_reset;
    a.lengths = d.d_lengths;
    a.maps = static_cast<Map*>(work);
    a.B = d.B;
    a.T = d.T;
    a.D = d.D;
    a.gate_b = d.gate_b;
    a.gate_t = d.gate_t;
    a.x_b = d.x_b;
    a.x_t = d.x_t;
    a.dy_b = d.dy_b;
    a.dy_t = d.dy_t;
    a.reset_b = d.reset_b;
    a.groups = p.groups;
    a.lanes = p.lanes;
    a.seg_tiles = p.seg_tiles;
    a.S = p.S;
    return a;
}

}  // namespace
}  // namespace gear

extern "C" int gear_recurrence_sizes(const gear_recurrence_desc* d, int64_t* saved_bytes, int64_t* work_bytes) {
    using namespace gear;
    if (const char* w = flaw(d)) return fail(GEAR_E_INVAL, std::string("gear_recurrence_sizes: ") + w);
    if (saved_bytes) *saved_bytes = saved_bytes_of(*d);
    if (work_bytes) *work_bytes = work_bytes_of(*d);
    return GEAR_OK;
}

extern "C" int gear_recurrence(const gear_recurrence_desc* d, const void* d_gate, const void* d_x,
                               const float* d_state, void* d_y, float* d_final, float* d_saved, void* d_work,
                               int64_t work_bytes, void* stream) {
    using namespace gear;
    if (const char* w = flaw(d)) return fail(GEAR_E_INVAL, std::string("gear_recurrence: ") + w);
    const bool any = d->B > 0 && d->T > 0 && d->D > 0;
    if (any && (d_gate == nullptr || d_x == nullptr)) return fail(GEAR_E_INVAL, "gear_recurrence: NULL gate or x");
    const bool in_place = d_final != nullptr && d_final == d_state;
    if (in_place && d->T > 1) return fail(GEAR_E_INVAL, "gear_recurrence: d_final may be d_state for one step only");
    const int64_t need = work_bytes_of(*d);
    if (need > 0 && (d_work == nullptr || work_bytes < need))
        return fail(GEAR_E_INVAL, "gear_recurrence: workspace smaller than gear_recurrence_sizes states");
    const Plan p = plan_of(*d, false, in_place);
    Args a = args_of(*d, p, d_work);
    a.gate = d_gate;
    a.x = d_x;
    a.state = d_state;
    a.y = d_y;
    a.final_state = d_final;
    a.out_saved = d_saved;
    return dispatch(a, p, *d, false, "gear_recurrence: launch", static_cast<hipStream_t>(stream));
}

extern "C" int gear_recurrence_backward(const gear_recurrence_desc* d, const void* d_gate, const void* d_x,
                                        const float* d_state, const float* d_saved, const void* d_dy,
                                        const float* d_dfinal, void* d_dgate, void* d_dx, float* d_dstate,
                                        void* d_work, int64_t work_bytes, void* stream) {
    using namespace gear;
    if (const char* w = flaw(d)) return fail(GEAR_E_INVAL, std::string("gear_recurrence_backward: ") + w);
    const bool any = d->B > 0 && d->T > 0 && d->D > 0;
    if (any && (d_gate == nullptr || d_x == nullptr || d_dgate == nullptr || d_dx == nullptr))
        return fail(GEAR_E_INVAL, "gear_recurrence_backward: NULL gate, x, dgate or dx");
    if (saved_bytes_of(*d) > 0 && d_saved == nullptr)
        return fail(GEAR_E_INVAL, "gear_recurrence_backward: NULL saved states");
    const int64_t need = work_bytes_of(*d);
    if (need > 0 && (d_work == nullptr || work_bytes < need))
        return fail(GEAR_E_INVAL, "gear_recurrence_backward: workspace smaller than gear_recurrence_sizes states");
    const Plan p = plan_of(*d, true, false);
    Args a = args_of(*d, p, d_work);
    a.gate = d_gate;
    a.x = d_x;
    a.state = d_state;
    a.saved = d_saved;
    a.dy = d_dy;
    a.dfinal = d_dfinal;
    a.dgate = d_dgate;
    a.dx = d_dx;
    a.dstate = d_dstate;
    return dispatch(a, p, *d, true, "gear_recurrence_backward: launch", static_cast<hipStream_t>(stream));
}
