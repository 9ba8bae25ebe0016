// The gated linear recurrence over collected windows (include/gear.h):
//   h_t = a_t h_{t-1} + u_t,  a = gate, u = x             (value form)
//                             a = f, u = (1 - f) x, f = sigmoid(gate)
// and its gradients, from the last step back:
//   G_t = dy_t + a_{t+1} G_{t+1},  dx_t = G_t du/dx,  dgate_t = G_t dh_t/dgate,
// where a reset makes h_{t-1} count as 0 and cuts the chain in both directions.
//
// Both directions read and write every element once and do a few operations
// on it, so memory bounds them.  A lane owns 8 (backward 4) bytes of neighbouring
// channels of one window and walks its steps in tiles of 16, loading an input's
// part of a tile as a whole.  Windows and channels give the
// parallelism; where they are too few to fill the GPU, the steps are split
// into segments, one to a wave: one launch reduces every segment, and every
// workgroup's run of segments, to what it does to a value carried through it
// (an affine map), one applies the runs' maps in order, and the last goes
// through every segment from its own first value.
#include <type_traits>

#include "element.h"
#include "gear_internal.h"

namespace gear {
namespace {

constexpr int kSteps = GEAR_RECURRENCE_STEPS;  // steps of a tile
// Neighbouring channels of a lane: 8 bytes of them forward; two backward, which
// holds three fp32 values for every step of each.  Of 16-bit types four took 473 us
// for forward and backward of 8192 x 32 x 512, two 423; of fp32 one took 332 us for 4 x 16384 x
// 512, two 305.
constexpr int kForwardBytes = 8, kBackwardChannels = 2;
constexpr int kThreads = 256;
// Calls of fewer lanes and at least so many tiles are split.  Splitting reads the
// inputs twice and takes three launches; not splitting leaves the GPU waiting for
// one tile of each lane at a time, 2.5 to 4 us.  Forward of B x T x 512 in
// bf16, split and not: 128 x 512 (16384 lanes) 82 and 131 us, 256 x 512 (32768) 137
// and 137, 512 x 512 271 and 161; 1 x 64 (4 tiles) 15 and 13, 1 x 128 20 and 23,
// 128 x 64 24 and 20, 128 x 128 32 and 37.  Backward: 64 x 512 (16384 lanes) 59 and
// 99, 128 x 512 106 and 107, 256 x 512 198 and 130; 64 x 64 16 and 14, 64 x 128 23 and 27.
// The bounds were set for these.  Elsewhere, forward and backward: fp32 64 x 512 x
// 512 69 / 93 and 77 / 125, but 96 x 512 x 512 102 / 148 and 84 / 136; bf16 64 x 512 x
// 1003 96 / 133 and 148 / 131, but 128 x 512 x 1003 190 and 168 forward; 4096 x 256 x 8
// 51 / 70 and 129 / 124.
constexpr int kWholeLanes = 512 * 64, kSplitTiles = 6;
constexpr int kWantLanes = 8192 * 64;   // lanes that a split call is cut into, at most:
constexpr int kMostSegments = 1024;     // more segments of long windows cost more in maps than they gain
constexpr int64_t kMaxBlocks = 1 << 22;
constexpr int kRun = 8;  // segments of a workgroup of a split call, a wave each
constexpr int32_t kMostExponent = 1 << 20;  // of a segment's decays: those of all segments together fit 31 bits

// What a segment does to the value c carried through it: c -> P c + Z, with a P of
// 0 from a reset on.  A sigmoid's decays are 1 at most: what their product loses
// below 2^-149 no later step raises again.
struct DecayMap {
    float P, Z;
    __device__ __forceinline__ float apply(float c) const { return fmaf(P, c, Z); }
    // `early` before this one.
    __device__ __forceinline__ DecayMap after(DecayMap early) const { return {P * early.P, apply(early.Z)}; }
};
// Gates as given may exceed 1, and their product P 2^n has an exponent of its own:
// fp32 alone would pass into an infinity, or into a 0, which loses what later
// steps raise again.  A P of 0 leaves nothing of any c, which may have grown to an
// infinity before a reset.
struct GrowthMap {
    float P, Z;
    int32_t n;
    __device__ __forceinline__ float apply(float c) const {
        const int32_t e = n < -1024 ? -1024 : n > 1024 ? 1024 : n;
        return fmaf(P, __builtin_amdgcn_ldexpf(P == 0.0f ? 0.0f : c, e), Z);
    }
    __device__ __forceinline__ GrowthMap after(GrowthMap early) const {
        const float p = P * early.P;
        return {__builtin_amdgcn_frexp_mantf(p), apply(early.Z), n + early.n + __builtin_amdgcn_frexp_expf(p)};
    }
};
template <int FORM>
using Map = std::conditional_t<FORM == GEAR_GATE_VALUE, GrowthMap, DecayMap>;

// The product of a segment's decays so far.
template <int FORM>
struct Product {
    float P = 1.0f;
    __device__ __forceinline__ void multiply(float f) { P *= f; }
    __device__ __forceinline__ void end_tile() {}
    __device__ __forceinline__ DecayMap map(float Z, bool cut) const { return {cut ? 0.0f : P, Z}; }
};
template <>
struct Product<GEAR_GATE_VALUE> {
    float P = 1.0f;
    int32_t n = 0;
    __device__ __forceinline__ void multiply(float f) {  // 16 factors of at least 0.5 stay in range
        P *= __builtin_amdgcn_frexp_mantf(f);
        n += __builtin_amdgcn_frexp_expf(f);
    }
    __device__ __forceinline__ void end_tile() {
        n += __builtin_amdgcn_frexp_expf(P);
        P = __builtin_amdgcn_frexp_mantf(P);
        n = n < -kMostExponent ? -kMostExponent : n > kMostExponent ? kMostExponent : n;
    }
    __device__ __forceinline__ GrowthMap map(float Z, bool cut) const { return {cut ? 0.0f : P, Z, n}; }
};

// A map gives the value of the steps as long as its two parts do not cancel and
// none of them overflows.  Where a Z, or a value carried from run to run, is
// this large (growth, an infinity, a NaN), the call is not trusted to maps: its
// lanes go through all their steps, as in calls that are not split.
constexpr float kTrusted = 0x1p40f;
__device__ __forceinline__ bool trusted(float v) { return fabsf(v) < kTrusted; }

struct Args {
    const void *gate, *x, *dy;
    const float *state, *saved, *dfinal;
    void *y, *dgate, *dx;
    float *final_state, *out_saved, *dstate;
    const uint8_t* reset;
    const int32_t* lengths;
    void* maps;           // of split calls: Map<FORM>[runs * kRun][B][D], one per segment, and [runs][B][D], one per
                          // run, whose first value carry_kernel leaves in P
    int32_t* doubt;       // whether carry_kernel found one that is not trusted
    int64_t B, T, D, gate_b, gate_t, x_b, x_t, dy_b, dy_t, reset_b;
    int64_t groups;       // of VE channels in a window
    int64_t lanes;        // B * groups
    int64_t seg_tiles;    // tiles of a segment
    int64_t columns;      // of 64 lanes
    int32_t runs;         // of kRun segments; 0 for a call that is not split
    bool stream;          // write past the caches
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

// Reset flags of the steps of a tile: read before the tile, so that they need
// not be waited for, and looked at after its loads are on their way.
struct Flags {
    uint32_t w[kSteps / 4];
    __device__ __forceinline__ void load(const Args& a, int64_t b, int64_t t0, int count) {
#pragma unroll
        for (int i = 0; i < kSteps / 4; i++) w[i] = 0;
        const uint8_t* r = a.reset + b * a.reset_b + t0;
        if (count == kSteps) __builtin_memcpy(w, r, sizeof(w));
        else
#pragma unroll
            for (int i = 0; i < kSteps; i++)
                if (i < count) w[i / 4] |= (uint32_t)r[i] << (8 * (i % 4));
    }
    __device__ __forceinline__ bool any() const { return (w[0] | w[1] | w[2] | w[3]) != 0; }
    __device__ __forceinline__ bool at(int s) const { return (w[s / 4] & (0xFFu << (8 * (s % 4)))) != 0; }
};
static_assert(kSteps == 16, "four words of flags");

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

// Hides where a pointer comes from.  A tile's addresses follow from its first;
// left to itself the compiler keeps a pointer per step from tile to tile, 96 registers.
// The pointer also loses its address space: accesses through it are flat ones, all
// of which are waited for before any is used, in the 16-bit sigmoid forward the
// gates before those of x go out.
template <typename P>
__device__ __forceinline__ void hide(P*& p) {
    asm volatile("" : "+v"(p));
}

// Loads go past the caches at every width, which suits rows of whole lines.  Where
// rows are narrower a load touches up to a line per lane, and the next step wants
// the same lines: forward and backward of 134 M bf16 elements in windows of 32 steps
// take 137 and 227 us with 512 channels, 178 and 241 with 64, 294 and 482 with 20,
// 413 and 606 with 8, 844 and 1542 with one.
template <typename E, int VE>
struct Tile {
    typename Vec<E, VE>::raw v[kSteps];
    // With FULL every lane of the wave has all steps, and no step takes a branch:
    // their gates are computed side by side.
    template <bool FULL>
    __device__ __forceinline__ void load(const E* p, int64_t stride, int count) {
        hide(p);
#pragma unroll
        for (int i = 0; i < kSteps; i++) {
            if (FULL || i < count) v[i] = Vec<E, VE>::template load<true>(p);
            p += stride;
        }
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
template <typename E, int VE, int FORM, bool RESET, bool MAPS, bool FULL, bool STREAM>
__device__ __forceinline__ void forward_tile(const Args& a, const Rows<E>& rows, int64_t t0, int count, int room,
                                             const Flags& flags, float (&h)[VE], Product<FORM> (&P)[VE]) {
#pragma clang fp contract(off)  // full and other tiles round alike: lanes that share channels may have either
    Tile<E, VE> g, x;
    g.template load<FULL>(rows.gate + t0 * a.gate_t, a.gate_t, count);
    x.template load<FULL>(rows.x + t0 * a.x_t, a.x_t, count);
    E* y = rows.y + t0 * a.D;
    hide(y);
#pragma unroll
    for (int s = 0; s < kSteps; s++) {
        if (FULL || s < count) {
            float gv[VE], xv[VE];
            Vec<E, VE>::unpack(g.v[s], gv);
            Vec<E, VE>::unpack(x.v[s], xv);
            const bool z = RESET && flags.at(s);
#pragma unroll
            for (int j = 0; j < VE; j++) {
                float f, w;
                gates<FORM>(gv[j], f, w);
                const float u = FORM == GEAR_GATE_VALUE ? xv[j] : w * xv[j];
                h[j] = z ? u : fmaf(f, h[j], u);
                if (MAPS) P[j].multiply(f);
            }
            if (!MAPS && a.y) Vec<E, VE>::template store<STREAM>(y, h);
        } else if (!MAPS && s < room && a.y) {
            const float zero[VE] = {};
            Vec<E, VE>::store(y, zero);
        }
        y += a.D;
    }
}

// A wave's part of a split call: 64 lanes' channels, one segment of their
// steps.  A workgroup has neighbouring segments of the same lanes.
struct Part {
    int64_t q, seg;  // lane among the call's; segment from the start, or for the backward pass from the end
    int32_t run;
    bool used;
};
__device__ __forceinline__ Part part_of(const Args& a) {
    Part w;
    w.run = (int32_t)(blockIdx.x / a.columns);
    w.q = ((int64_t)blockIdx.x - w.run * a.columns) * 64 + (threadIdx.x & 63);
    w.used = w.q < a.lanes;
    if (!w.used) w.q = 0;
    w.seg = (int64_t)w.run * kRun + (threadIdx.x >> 6);
    return w;
}

// Leaves a wave's map, and the first wave its workgroup's, with a Z of NaN where
// that of a segment, or of the segments so far, is not trusted.
template <int FORM, int VE>
__device__ __forceinline__ void leave_maps(const Args& a, const Part& w, int64_t at, const Map<FORM> (&m)[VE],
                                           Map<FORM> (*s)[VE][64]) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    Map<FORM>* const maps = static_cast<Map<FORM>*>(a.maps);
    const int64_t BD = a.B * a.D, run_maps = (int64_t)a.runs * kRun * BD;
    if (blockIdx.x == 0 && threadIdx.x == 0) *a.doubt = 0;  // for the next launch
#pragma unroll
    for (int j = 0; j < VE; j++) {
        s[wave][j][lane] = m[j];
        if (w.used) maps[w.seg * BD + at + j] = m[j];
    }
    __syncthreads();
    if (wave > 0) return;
#pragma unroll
    for (int j = 0; j < VE; j++) {
        Map<FORM> all = m[j];
        bool sound = trusted(all.Z);
#pragma unroll
        for (int k = 1; k < kRun; k++) {
            const Map<FORM> next = s[k][j][lane];
            all = next.after(all);
            sound = sound && trusted(next.Z) && trusted(all.Z);
        }
        if (!sound) all.Z = NAN;
        if (w.used) maps[run_maps + w.run * BD + at + j] = all;
    }
}

// The value a wave's segment starts from: its run's, through the run's earlier segments.
template <int FORM, int VE>
__device__ __forceinline__ void first_of(const Args& a, const Part& w, int64_t at, float (&c)[VE]) {
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const Map<FORM>* const maps = static_cast<const Map<FORM>*>(a.maps);
    const int64_t BD = a.B * a.D, run_maps = (int64_t)a.runs * kRun * BD;
#pragma unroll
    for (int j = 0; j < VE; j++) c[j] = maps[run_maps + w.run * BD + at + j].P;
    for (int k = 0; k < wave; k++) {
#pragma unroll
        for (int j = 0; j < VE; j++) c[j] = maps[((int64_t)w.run * kRun + k) * BD + at + j].apply(c[j]);
    }
}

// The steps of lane q from tile k0 to tile k1, from state h.
template <typename E, int VE, int FORM, bool RESET, bool MAPS>
__device__ __forceinline__ bool forward_tiles(const Args& a, const Place& p, int64_t at, bool used, int64_t k0, int64_t k1,
                                              float (&h)[VE], Product<FORM> (&P)[VE]) {
    const Rows<E> rows = rows_of<E>(a, p);
    const int64_t BD = a.B * a.D;
    bool cut = false;
    for (int64_t k = k0; k < k1; k++) {
        const int64_t t0 = k * kSteps;
        const int count = used ? clamp_count(p.n - t0) : 0, room = used ? clamp_count(a.T - t0) : 0;
        if (!MAPS && used && a.out_saved && k > 0) Vec<float, VE>::store(a.out_saved + (k - 1) * BD + at, h);
        Flags flags;
        if (RESET) flags.load(a, p.b, t0, count);
        if (!__all(count == kSteps))
            forward_tile<E, VE, FORM, RESET, MAPS, false, false>(a, rows, t0, count, room, flags, h, P);
        else if (!MAPS && a.stream)
            forward_tile<E, VE, FORM, RESET, MAPS, true, true>(a, rows, t0, count, room, flags, h, P);
        else forward_tile<E, VE, FORM, RESET, MAPS, true, false>(a, rows, t0, count, room, flags, h, P);
        if (RESET) cut |= flags.any();
        if (MAPS) {
#pragma unroll
            for (int j = 0; j < VE; j++) P[j].end_tile();
        }
    }
    return cut;
}

// Windows that are not split, a lane per piece of channels.  At 8192 x 32 x 512
// bf16 with resets it takes 139 us for the 840 MB it reads and writes (saved
// states included), 6.0 TB/s: memory bounds it.
template <typename E, int VE, int FORM, bool RESET>
__global__ __launch_bounds__(kThreads) void forward_kernel(const Args a) {
    for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < a.lanes; i += (int64_t)gridDim.x * kThreads) {
        const Place p = place_of<VE>(a, i);
        const int64_t at = p.b * a.D + p.c;
        float h[VE];
        Product<FORM> P[VE];
#pragma unroll
        for (int j = 0; j < VE; j++) h[j] = a.state ? a.state[at + j] : 0.0f;
        forward_tiles<E, VE, FORM, RESET, false>(a, p, at, true, 0, (a.T + kSteps - 1) / kSteps, h, P);
        if (a.final_state) Vec<float, VE>::store(a.final_state + at, h);
    }
}

// Segments: with MAPS, reduces each to its map; else goes through it.  What the
// first launch reads the second reads again, from the last-level cache where it
// fits: at 4 x 16384 x 512 fp32 the two take 48 and 81 us and the carry between
// them 6.4 (a map of gates as given costs 4 us more than one of plain products);
// at 1 x 131072 x 512 bf16 49, 69 and 6.0.
template <typename E, int VE, int FORM, bool RESET, bool MAPS>
__global__ __launch_bounds__(64 * kRun) void forward_split_kernel(const Args a) {
    __shared__ Map<FORM> s[MAPS ? kRun : 1][VE][64];
    const Part w = part_of(a);
    const Place p = place_of<VE>(a, w.q);
    const int64_t at = p.b * a.D + p.c, tiles = (a.T + kSteps - 1) / kSteps;
    const int64_t k0 = w.seg * a.seg_tiles < tiles ? w.seg * a.seg_tiles : tiles;
    int64_t k1 = k0 + a.seg_tiles < tiles ? k0 + a.seg_tiles : tiles;
    float h[VE] = {};
    Product<FORM> P[VE];
    if (MAPS) {
        const bool cut = forward_tiles<E, VE, FORM, RESET, MAPS>(a, p, at, w.used, k0, k1, h, P);
        Map<FORM> m[VE];
#pragma unroll
        for (int j = 0; j < VE; j++) m[j] = P[j].map(h[j], cut);
        leave_maps<FORM, VE>(a, w, at, m, s);
    } else {
        const int32_t doubt = *a.doubt;
        first_of<FORM, VE>(a, w, at, h);
        // In doubt the first segment's wave takes all tiles.
        if (doubt) k1 = w.seg == 0 ? tiles : k0;
        forward_tiles<E, VE, FORM, RESET, MAPS>(a, p, at, w.used, k0, k1, h, P);
        if (w.used && a.final_state && k0 < k1 && k1 == tiles) Vec<float, VE>::store(a.final_state + at, h);
    }
}

// Applies every channel's run maps in order and leaves the value each run
// starts from in its map.  A workgroup takes 64 channels; each of its waves
// composes a share of the runs, the shares' maps lead to every share's first
// value, and the waves go through their shares again.
constexpr int kCarryWaves = 16, kCarryAhead = 16;
template <int FORM>
__global__ __launch_bounds__(64 * kCarryWaves) void carry_kernel(const Args a, const float* __restrict__ first) {
    const int64_t channels = a.B * a.D;
    const int32_t runs = a.runs;
    Map<FORM>* __restrict__ const maps = static_cast<Map<FORM>*>(a.maps) + (int64_t)runs * kRun * channels;
    __shared__ Map<FORM> s_share[kCarryWaves][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int64_t i = (int64_t)blockIdx.x * 64 + lane;
    const bool used = i < channels;
    if (!used) i = channels - 1;
    const int32_t share = (runs + kCarryWaves - 1) / kCarryWaves;
    const int32_t s0 = wave * share < runs ? wave * share : runs, s1 = s0 + share < runs ? s0 + share : runs;
    Map<FORM> whole = Product<FORM>().map(0.0f, false), m[kCarryAhead];
    bool sound = true;
    for (int32_t s = s0; s < s1; s += kCarryAhead) {
        // Places past the share read its last map again and are not used.
#pragma unroll
        for (int k = 0; k < kCarryAhead; k++) m[k] = maps[(s + k < s1 ? s + k : s1 - 1) * channels + i];
#pragma unroll
        for (int k = 0; k < kCarryAhead; k++) {
            if (s + k < s1) {
                whole = m[k].after(whole);
                sound = sound && trusted(m[k].Z) && trusted(whole.Z);
            }
        }
    }
    s_share[wave][lane] = whole;
    __syncthreads();
    if (!used) return;
    float c = first ? first[i] : 0.0f;
    for (int k = 0; k < wave; k++) c = s_share[k][lane].apply(c);
    for (int32_t s = s0; s < s1; s += kCarryAhead) {
        if (share > kCarryAhead) {
#pragma unroll
            for (int k = 0; k < kCarryAhead; k++) m[k] = maps[(s + k < s1 ? s + k : s1 - 1) * channels + i];
        }
#pragma unroll
        for (int k = 0; k < kCarryAhead; k++) {
            if (s + k < s1) {
                sound = sound && trusted(c);
                maps[(s + k) * channels + i].P = c;
                c = m[k].apply(c);
            }
        }
    }
    if (!sound) *a.doubt = 1;
}

// A tile backward: G comes in as the gradient of the state after it and goes
// out as that of the state before it.  h is the state before it, from which
// the states inside are recomputed in 32 bits: read back from y they would carry
// its rounding into h_{t-1} - x_t.
template <typename E, int VE, int FORM, bool RESET, bool MAPS, bool FULL, bool STREAM>
__device__ __forceinline__ void backward_tile(const Args& a, const Rows<E>& rows, int64_t t0, int count, int room,
                                              const Flags& flags, float (&h)[VE], float (&G)[VE],
                                              Product<FORM> (&P)[VE]) {
#pragma clang fp contract(off)  // as forward_tile
    Tile<E, VE> g, x, d;
    g.template load<FULL>(rows.gate + t0 * a.gate_t, a.gate_t, count);
    if (!MAPS) x.template load<FULL>(rows.x + t0 * a.x_t, a.x_t, count);
    if (rows.dy) d.template load<FULL>(rows.dy + t0 * a.dy_t, a.dy_t, count);
    // Per step: decay, input weight, and what the gate's gradient is a multiple of.
    float F[kSteps][VE], W[kSteps][VE], Q[kSteps][VE];
#pragma unroll
    for (int s = 0; s < kSteps; s++) {
        if (FULL || s < count) {
            float gv[VE], xv[VE];
            Vec<E, VE>::unpack(g.v[s], gv);
            if (!MAPS) Vec<E, VE>::unpack(x.v[s], xv);
            const bool z = RESET && flags.at(s);
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
    E* dgate = rows.dgate + (t0 + kSteps - 1) * a.D;
    E* dx = rows.dx + (t0 + kSteps - 1) * a.D;
    hide(dgate);
    hide(dx);
#pragma unroll
    for (int s = kSteps - 1; s >= 0; s--) {
        if (FULL || s < count) {
            float dv[VE] = {}, og[VE], ox[VE];
            if (rows.dy) Vec<E, VE>::unpack(d.v[s], dv);
            const bool z = RESET && flags.at(s);
#pragma unroll
            for (int j = 0; j < VE; j++) {
                const float f = F[s][j], t = G[j] + dv[j];
                if (!MAPS) {
                    ox[j] = FORM == GEAR_GATE_VALUE ? t : t * W[s][j];
                    og[j] = FORM == GEAR_GATE_VALUE ? t * Q[s][j] : ox[j] * Q[s][j] * f;
                }
                G[j] = z ? 0.0f : f * t;
                if (MAPS) P[j].multiply(f);
            }
            if (!MAPS) {
                Vec<E, VE>::template store<STREAM>(dgate, og);
                Vec<E, VE>::template store<STREAM>(dx, ox);
            }
        } else if (!MAPS && s < room) {
            const float zero[VE] = {};
            Vec<E, VE>::store(dgate, zero);
            Vec<E, VE>::store(dx, zero);
        }
        dgate -= a.D;
        dx -= a.D;
    }
}

// The steps of lane q back from tile k1 to tile k0.
template <typename E, int VE, int FORM, bool RESET, bool MAPS>
__device__ __forceinline__ bool backward_tiles(const Args& a, const Place& p, int64_t at, bool used, int64_t k0, int64_t k1,
                                               float (&G)[VE], Product<FORM> (&P)[VE]) {
    const Rows<E> rows = rows_of<E>(a, p);
    const int64_t BD = a.B * a.D;
    bool cut = false;
    for (int64_t k = k1 - 1; k >= k0; k--) {
        const int64_t t0 = k * kSteps;
        const int count = used ? clamp_count(p.n - t0) : 0, room = used ? clamp_count(a.T - t0) : 0;
        Flags flags;
        if (RESET) flags.load(a, p.b, t0, count);
        float h[VE] = {};
        if (!MAPS && count > 0) {
            const float* from = k > 0 ? a.saved + (k - 1) * BD + at : a.state ? a.state + at : nullptr;
            if (from) {
#pragma unroll
                for (int j = 0; j < VE; j++) h[j] = from[j];
            }
        }
        if (!__all(count == kSteps))
            backward_tile<E, VE, FORM, RESET, MAPS, false, false>(a, rows, t0, count, room, flags, h, G, P);
        else if (!MAPS && a.stream)
            backward_tile<E, VE, FORM, RESET, MAPS, true, true>(a, rows, t0, count, room, flags, h, G, P);
        else backward_tile<E, VE, FORM, RESET, MAPS, true, false>(a, rows, t0, count, room, flags, h, G, P);
        if (RESET) cut |= flags.any();
        if (MAPS) {
#pragma unroll
            for (int j = 0; j < VE; j++) P[j].end_tile();
        }
    }
    return cut;
}

// Windows that are not split.  Three inputs read, two gradients written: 8192 x 32
// x 512 bf16 with resets in 227 us, 1.36 GB with the saved states, 6.0 TB/s.
template <typename E, int VE, int FORM, bool RESET>
__global__ __launch_bounds__(kThreads) void backward_kernel(const Args a) {
    for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < a.lanes; i += (int64_t)gridDim.x * kThreads) {
        const Place p = place_of<VE>(a, i);
        const int64_t at = p.b * a.D + p.c;
        float G[VE];
        Product<FORM> P[VE];
#pragma unroll
        for (int j = 0; j < VE; j++) G[j] = a.dfinal ? a.dfinal[at + j] : 0.0f;
        backward_tiles<E, VE, FORM, RESET, false>(a, p, at, true, 0, (a.T + kSteps - 1) / kSteps, G, P);
        if (a.dstate) Vec<float, VE>::store(a.dstate + at, G);
    }
}

// Segments are numbered from the end here: the gradient is carried from there.
// At 4 x 16384 x 512 fp32 the maps take 48 us and the gradients 120 (679 MB, 5.7 TB/s).
template <typename E, int VE, int FORM, bool RESET, bool MAPS>
__global__ __launch_bounds__(64 * kRun) void backward_split_kernel(const Args a) {
    __shared__ Map<FORM> s[MAPS ? kRun : 1][VE][64];
    const Part w = part_of(a);
    const Place p = place_of<VE>(a, w.q);
    const int64_t at = p.b * a.D + p.c, tiles = (a.T + kSteps - 1) / kSteps;
    const int64_t k1 = tiles - w.seg * a.seg_tiles > 0 ? tiles - w.seg * a.seg_tiles : 0;
    int64_t k0 = k1 - a.seg_tiles > 0 ? k1 - a.seg_tiles : 0;
    float G[VE] = {};
    Product<FORM> P[VE];
    if (MAPS) {
        const bool cut = backward_tiles<E, VE, FORM, RESET, MAPS>(a, p, at, w.used, k0, k1, G, P);
        Map<FORM> m[VE];
#pragma unroll
        for (int j = 0; j < VE; j++) m[j] = P[j].map(G[j], cut);
        leave_maps<FORM, VE>(a, w, at, m, s);
    } else {
        const int32_t doubt = *a.doubt;
        first_of<FORM, VE>(a, w, at, G);
        if (doubt) k0 = w.seg == 0 ? 0 : k1;  // as forward
        backward_tiles<E, VE, FORM, RESET, MAPS>(a, p, at, w.used, k0, k1, G, P);
        if (w.used && a.dstate && k0 < k1 && k0 == 0) Vec<float, VE>::store(a.dstate + at, G);
    }
}

typedef void (*Kernel)(const Args);
struct Kernels {
    Kernel whole, maps, split;
};
template <typename E, int VE, int FORM, bool RESET, bool BACKWARD>
Kernels kernels_of() {
    if constexpr (BACKWARD)
        return {backward_kernel<E, VE, FORM, RESET>, backward_split_kernel<E, VE, FORM, RESET, true>,
                backward_split_kernel<E, VE, FORM, RESET, false>};
    else
        return {forward_kernel<E, VE, FORM, RESET>, forward_split_kernel<E, VE, FORM, RESET, true>,
                forward_split_kernel<E, VE, FORM, RESET, false>};
}
template <typename E, int VE, bool BACKWARD>
Kernels kernels_for(int32_t form, bool reset) {
    if (form == GEAR_GATE_VALUE)
        return reset ? kernels_of<E, VE, GEAR_GATE_VALUE, true, BACKWARD>() : kernels_of<E, VE, GEAR_GATE_VALUE, false, BACKWARD>();
    return reset ? kernels_of<E, VE, GEAR_GATE_SIGMOID, true, BACKWARD>() : kernels_of<E, VE, GEAR_GATE_SIGMOID, false, BACKWARD>();
}
template <typename E, bool BACKWARD>
Kernels kernels_for(int32_t form, bool reset, bool wide) {
    constexpr int VE = BACKWARD ? kBackwardChannels : kForwardBytes / (int)sizeof(E);
    return wide ? kernels_for<E, VE, BACKWARD>(form, reset) : kernels_for<E, 1, BACKWARD>(form, reset);
}

// How a call is cut: channels per lane; for a split one, segments of tiles and runs of them.
struct Plan {
    int ve;
    int64_t groups, lanes, columns, seg_tiles;
    int32_t runs;
};
Plan plan_of(const gear_recurrence_desc& d, bool backward, bool in_place) {
    Plan p;
    const int full = backward ? kBackwardChannels : kForwardBytes / float_bytes(d.dtype);
    // Widths below a lane's are taken channel by channel, as are odd ones
    // whose states are updated in place: lanes that share channels must not
    // read what another has written.
    p.ve = d.D < full || (in_place && d.D % full != 0) ? 1 : full;
    p.groups = (d.D + p.ve - 1) / p.ve;
    p.lanes = d.B * p.groups;
    p.columns = (p.lanes + 63) / 64;
    p.seg_tiles = 0;
    p.runs = 0;
    const int64_t tiles = (d.T + kSteps - 1) / kSteps;
    if (tiles < kSplitTiles || p.lanes == 0 || p.lanes >= kWholeLanes) return p;
    int64_t S = kWantLanes / p.lanes;
    if (S > kMostSegments) S = kMostSegments;
    if (S > tiles) S = tiles;
    p.seg_tiles = (tiles + S - 1) / S;
    S = (tiles + p.seg_tiles - 1) / p.seg_tiles;
    p.runs = (int32_t)((S + kRun - 1) / kRun);
    return p;
}
int64_t map_bytes(const gear_recurrence_desc& d) { return d.form == GEAR_GATE_VALUE ? sizeof(GrowthMap) : sizeof(DecayMap); }
int64_t work_bytes_of(const gear_recurrence_desc& d) {
    const int32_t f = plan_of(d, false, false).runs, b = plan_of(d, true, false).runs;
    const int64_t runs = f > b ? f : b;
    return runs ? runs * (kRun + 1) * d.B * d.D * map_bytes(d) + (int64_t)sizeof(int32_t) : 0;
}
int64_t saved_bytes_of(const gear_recurrence_desc& d) {
    const int64_t tiles = (d.T + kSteps - 1) / kSteps;
    return tiles > 1 ? (tiles - 1) * d.B * d.D * (int64_t)sizeof(float) : 0;
}

// Outputs that the last-level cache cannot hold are written past it, where a
// wave writes whole lines of 128 bytes: forward and backward of 8192 x 32 x 512 in
// bf16 took 422 us without and 367 with.  Outputs that it holds for the next
// reader stay in it (1 x 131072 x 512 in bf16: 126 and 130 us).  Rows that share
// lines go through it, which suits outputs whose memory it already holds: 37 x 1000
// x 1003 in fp16 took 192 us through it and 252 past it where every pass wrote the
// same memory, but 239 and 214 where the outputs of the pass before were kept.
constexpr int64_t kCacheBytes = 192ll << 20;  // of 256 MB, beside what else is in use
bool streams(const gear_recurrence_desc& d, const void* out, const void* other, int outputs) {
    const int64_t row = d.D * float_bytes(d.dtype);
    const uintptr_t at = reinterpret_cast<uintptr_t>(out) | reinterpret_cast<uintptr_t>(other);
    return row % 128 == 0 && at % 128 == 0 && outputs * d.B * d.T * row > kCacheBytes;
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
    const Kernels k = backward ? kernels_for<E, true>(form, base.reset != nullptr, p.ve > 1)
                               : kernels_for<E, false>(form, base.reset != nullptr, p.ve > 1);
    const int64_t BD = base.B * base.D;
    if (p.runs == 0) {
        hipLaunchKernelGGL(k.whole, dim3(blocks_for(p.lanes)), dim3(kThreads), 0, s, base);
        const hipError_t e = hipGetLastError();
        return e == hipSuccess ? GEAR_OK : hip_fail(e, what);
    }
    const dim3 grid((unsigned)(p.columns * p.runs)), block(64 * kRun);
    hipLaunchKernelGGL(k.maps, grid, block, 0, s, base);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return hip_fail(e, what);
    hipLaunchKernelGGL(form == GEAR_GATE_VALUE ? carry_kernel<GEAR_GATE_VALUE> : carry_kernel<GEAR_GATE_SIGMOID>,
                       dim3((unsigned)((BD + 63) / 64)), dim3(64 * kCarryWaves), 0, s, base,
                       backward ? base.dfinal : base.state);
    e = hipGetLastError();
    if (e != hipSuccess) return hip_fail(e, what);
    hipLaunchKernelGGL(k.split, grid, block, 0, s, base);
    e = hipGetLastError();
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
    a.maps = work;
    a.doubt = reinterpret_cast<int32_t*>(static_cast<char*>(work) + (int64_t)p.runs * (kRun + 1) * d.B * d.D * map_bytes(d));
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
    a.columns = p.columns;
    a.runs = p.runs;
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
    a.stream = streams(*d, d_y, nullptr, 1);
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
    a.stream = streams(*d, d_dgate, d_dx, 2);
    return dispatch(a, p, *d, true, "gear_recurrence_backward: launch", static_cast<hipStream_t>(stream));
}
