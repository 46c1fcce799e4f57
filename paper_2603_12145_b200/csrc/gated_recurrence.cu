// gated_recurrence.cu -- the gated linear recurrence behind the C ABI of gated_recurrence.h: sequences, gradients, single
// tokens.
//
// A thread walks the time axis with the states of V neighbouring channels in registers (two where sizes, strides and
// pointers allow, so that a warp's access covers whole lines and one instruction works on both; else one), kSteps steps at
// a time; the next steps' loads are in flight meanwhile.  The lanes of a warp share a sequence, so that a ballot gives them its
// resets.
//
// Few rows: the time axis is cut into segments.  A first pass finds what each segment makes of a zero state and the sum of
// its L, k_carry chains them, and the second pass starts every segment from its state.  With many rows there is one
// segment and one pass; shape_of chooses.
//
// Backward, the state at the start of every kSaved steps is saved by the forward pass; a thread goes back through them,
// forms the states and gates of the kSaved steps in registers, and then walks these backwards.  (Four steps: eight need twice the
// registers, and the saved states are then an eighth of what a pass reads instead of a sixteenth.)
//
// Arithmetic of a step.  With d = e^L - 1 to full relative precision (a polynomial for small L, where 1 - e^L would cancel),
// the decay is h + d h in one multiply-add and the gain sqrt(1 - e^(2 L)) = sqrt(-d (2 + d)): no second exponential, and no
// rounding of a decay just below one, which a slow channel would gather step after step.  Backward, 1 - sigmoid(v) is e^-v
// sigmoid(v): no cancellation there either.  Per element: three exponentials, two reciprocals, one reciprocal square root.
//
// What bounds it: the special-function unit, 6 results per element at 16 per cycle and SM, forward (512 x 128 x 1,152 in
// bfloat16 146 us, 75.5 M elements: 100 us of it), issue backward (288 us; 166 instructions per pair of elements), HBM in
// the single token (16,384 x 1,152 rows 53 us, 302 MB, 5.7 TB/s).  A prompt of 8,192 steps of one row and 2,048 channels
// takes 75 us, two passes of segments; 64 single tokens take 12 us, the host's part.
#include <new>
#include <type_traits>

#include "../../include/gated_recurrence.h"
#include "on_device.cuh"
#include "vectors.cuh"

namespace {

using namespace vals;

constexpr int kThreads = 128;
constexpr int kWarps = kThreads / 32;
constexpr int kSteps = 8;                // steps of a tile, forward
constexpr int kSaved = 4;                // steps between saved states, and of a tile, backward
constexpr int kStepThreads = 256;

__device__ __forceinline__ void allow_next() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void wait_for_previous() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

template <int V>
__device__ __forceinline__ Vals<V> load_floats(const float *src)
{
    if (src == nullptr) return all<V>(0.0f);
    if constexpr (V == 1)
        return src[0];
    else
        return pair(src[0], src[1]);
}
__device__ __forceinline__ void store_floats(float *dst, float v) { dst[0] = v; }
__device__ __forceinline__ void store_floats(float *dst, Pair v)
{
    dst[0] = lo(v);
    dst[1] = hi(v);
}

// ---- the functions of a step

constexpr float kLog2e = 1.4426950408889634f;

__device__ __forceinline__ float rsq(float v)
{
    float r;
    asm("rsqrt.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
    return r;
}

// e^-v of binary32 gates, `most` bounding -v = n.  The rounded exponent t = n log2 e alone would be off by |v| 2^-24 of the result (62
// units of 2^-24 for gates down to -80): 2^t is multiplied by 1 + (n - t ln 2), which leaves t times ln 2's own rounding, 2e-9 (6
// units in all; 256 x 128 x 1,152 forward 110 against 109 us).  Below e^-104 nothing is left, and an infinite exponent has no
// difference.  Gates of 16 bits do without: their own rounding moves the result by more.
template <typename F>
__device__ __forceinline__ F exp_minus(F v, float most)
{
    constexpr int V = sizeof(F) / 4;
    const F n = each([&](float e) { return ssm_k::at_least(ssm_k::at_most(-e, most), -104.0f); }, v);
    const F t = mul(n, all<V>(kLog2e)), e = each([](float x) { return ex2(x); }, t);
    return fma(e, fma(t, all<V>(-ssm_k::kLn2), n), e);
}

// 1 / (1 + e^-v), T the type that v comes in.  (Beyond e^88 the reciprocal is below the normal numbers: zero.)
template <typename T, typename F>
__device__ __forceinline__ F sigmoid(F v)
{
    constexpr int V = sizeof(F) / 4;
    F e;
    if constexpr (sizeof(T) == 4)
        e = exp_minus(v, 88.0f);
    else
        e = each([](float x) { return ex2(x); }, mul(v, all<V>(-kLog2e)));
    return each([](float x) { return rcp(x); }, add(e, all<V>(1.0f)));
}

// The same, and 1 - sigmoid(v) to full relative precision.  (The exponential stays within 2^126: its product with
// the sigmoid is one, not infinity times zero.)
template <typename T, typename F>
__device__ __forceinline__ F sigmoid(F v, F &rest)
{
    constexpr int V = sizeof(F) / 4;
    F e;
    if constexpr (sizeof(T) == 4)
        e = exp_minus(v, 87.3f);
    else
        e = each([](float x) { return ex2(ssm_k::at_most(x, 126.0f)); }, mul(v, all<V>(-kLog2e)));
    const F s = each([](float x) { return rcp(x); }, add(e, all<V>(1.0f)));
    rest = mul(e, s);
    return s;
}

// e^L - 1, L <= 0: the series up to L^5 above -1/8 (the next term is under 5e-8 of the sum), else from the exponential, whose
// error then counts eightfold at most.  (The exponent's own rounding is |L| e^L 2^-24 of one: nothing.)
template <typename F>
__device__ __forceinline__ F decay_less_one(F L)
{
    constexpr int V = sizeof(F) / 4;
    F p = fma(L, all<V>(1.0f / 120.0f), all<V>(1.0f / 24.0f));
    p = fma(p, L, all<V>(1.0f / 6.0f));
    p = fma(p, L, all<V>(0.5f));
    p = fma(mul(p, L), L, L);
    const F large = add(each([](float e) { return ex2(e); }, mul(L, all<V>(kLog2e))), all<V>(-1.0f));
    return each([](float l, float small, float big) { return l > -0.125f ? small : big; }, L, p, large);
}

// e^L h from d = e^L - 1, with one rounding; an infinity stays one (d h and h would cancel to a NaN).
template <typename F>
__device__ __forceinline__ F decayed(F d, F h)
{
    return each([](float v, float w) { return fabsf(w) == __int_as_float(0x7F800000) ? w : v; }, fma(d, h, h), h);
}

// 1 - e^(2 L) = -d (2 + d)
template <typename F>
__device__ __forceinline__ F square_gain(F d)
{
    constexpr int V = sizeof(F) / 4;
    const F minus = mul(d, all<V>(-1.0f));
    return fma(minus, d, add(minus, minus));
}

// 1 / sqrt(square); zero where nothing is left of it.  (A NaN passes, and the negative square of a growing state gives one.)
template <typename F>
__device__ __forceinline__ F inverse_root(F square)
{
    return each([](float s) { return fabsf(s) < 1.2e-38f ? 0.0f : rsq(s); }, square);
}

// The state after a step: gates and input of the step, the state before it.
template <typename F>
__device__ __forceinline__ F advance(F d, F in, F x, F before)
{
    const F square = square_gain(d);
    return fma(mul(square, inverse_root(square)), mul(in, x), decayed(d, before));
}

// ---- arguments

template <typename T>
struct Seq {
    T *ptr;
    int64_t sb, st;
    __device__ __forceinline__ T *row(int64_t b, int64_t t) const { return ptr + b * sb + t * st; }
};

struct Shape {
    int64_t batch;
    int time, channels;
    int segments, segment_steps;     // the latter a multiple of kSteps, and so of kSaved
    int slots;                       // backward: rows of sums; a warp takes several (row, segment) pairs
};

template <typename T>
struct Params {
    Seq<const T> x, r, i, dy;
    Seq<const uint8_t> reset;
    Seq<T> y, dx, dr, di;
    const float *a, *state, *dstate_out;
    float *state_out, *dstate, *saved, *da;
    float *carry;                    // [batch][segments][channels]: a segment's end, then its start
    float *span;                     // [batch][segments][channels]: sum of L, positive where a reset cuts the segment
    float *part;                     // [slots][channels]
};

// Which (row, segment) and which channels this warp works on.
template <int V>
struct Place {
    int64_t unit, b;
    int segment, t0, t1, c;
    bool live;                       // lanes past the last channel go along
    __device__ Place(const Shape &s, int64_t unit_, int tile) : unit(unit_)
    {
        b = unit / s.segments;
        segment = static_cast<int>(unit - b * s.segments);
        t0 = segment * s.segment_steps;
        t1 = min(s.time, t0 + s.segment_steps);
        c = (tile * 32 + static_cast<int>(threadIdx.x & 31)) * V;
        live = c < s.channels;
        if (!live) c = 0;
    }
};

// Steps [t, t + K) that start an episode, as bits.
template <int K, typename T>
__device__ __forceinline__ uint32_t resets_at(const Params<T> &p, int64_t b, int t, int t1)
{
    if (p.reset.ptr == nullptr) return 0;
    const int lane = threadIdx.x & 31;
    return __ballot_sync(0xFFFFFFFFu, lane < K && t + lane < t1 && *p.reset.row(b, t + lane) != 0);
}

// K steps of a sequence; steps past the end are zeros.
template <typename T, int V, int K>
struct Block {
    Packed<T, V> v[K];
    __device__ __forceinline__ void load(const Seq<const T> &q, const Place<V> &at, int t)
    {
        const T *ptr = q.row(at.b, t) + at.c;
        if (t + K <= at.t1) {
#pragma unroll
            for (int k = 0; k < K; ++k) {
                v[k] = packed_load<T, V>(ptr);
                ptr += q.st;
            }
        } else {
#pragma unroll
            for (int k = 0; k < K; ++k) {
                v[k] = t + k < at.t1 ? packed_load<T, V>(ptr) : packed_zero<T, V>();
                ptr += q.st;
            }
        }
    }
};

// kEnds: the first pass over segments.  (Binary32 in three blocks per SM: 1 x 4,096 x 2,048 53 us, 62 with the two that 206 registers
// leave.)
template <typename T, int V, bool kEnds>
__global__ void __launch_bounds__(kThreads, sizeof(T) != 2 ? 3 : kEnds ? 4 : 5)
k_forward(const Shape s, const Params<T> p)
{
    using F = Vals<V>;
    allow_next();
    wait_for_previous();
    const int tiles = (s.channels + 32 * V - 1) / (32 * V);
    const int64_t warp = static_cast<int64_t>(blockIdx.x) * kWarps + (threadIdx.x >> 5);
    if (warp >= s.batch * s.segments * tiles) return;
    const Place<V> at(s, warp / tiles, static_cast<int>(warp % tiles));
    const F a = load_floats<V>(p.a + at.c);
    F h = all<V>(0.0f), span = h;
    if (!kEnds)
        h = load_floats<V>(s.segments > 1 ? p.carry + at.unit * s.channels + at.c
                                          : p.state == nullptr ? nullptr : p.state + at.b * s.channels + at.c);
    Block<T, V, kSteps> nx, nr, ni;
    nx.load(p.x, at, at.t0);
    nr.load(p.r, at, at.t0);
    ni.load(p.i, at, at.t0);
    float *saved = nullptr;
    if (!kEnds && p.saved != nullptr)
        saved = p.saved + (at.b * ((s.time + kSaved - 1) / kSaved) + at.t0 / kSaved) * s.channels + at.c;
    T *py = kEnds ? nullptr : p.y.row(at.b, at.t0) + at.c;
    bool cut = false;
    for (int t = at.t0; t < at.t1; t += kSteps) {
        const Block<T, V, kSteps> x = nx, r = nr, i = ni;
        const uint32_t resets = resets_at<kSteps>(p, at.b, t, at.t1);
        if (t + kSteps < at.t1) {
            nx.load(p.x, at, t + kSteps);
            nr.load(p.r, at, t + kSteps);
            ni.load(p.i, at, t + kSteps);
        }
        // Plain: all steps are there and none starts an episode, the common case
        auto work = [&](auto plain) {
#pragma unroll
            for (int k = 0; k < kSteps; ++k) {
                if (!plain.value) {
                    if (t + k >= at.t1) break;
                    if ((resets >> k) & 1u) {
                        cut = true;
                        h = all<V>(0.0f);
                    }
                }
                if (!kEnds && k % kSaved == 0 && saved != nullptr) {
                    if (at.live) store_floats(saved, h);
                    saved += s.channels;
                }
                const F L = mul(a, sigmoid<T>(widen(r.v[k])));
                h = advance(decay_less_one(L), sigmoid<T>(widen(i.v[k])), widen(x.v[k]), h);
                if constexpr (kEnds) {
                    span = add(span, L);
                } else {
                    if (at.live) packed_store<T, V>(py, narrow<T>(h));
                    py += p.y.st;
                }
            }
        };
        if (resets == 0 && t + kSteps <= at.t1)
            work(std::true_type{});
        else
            work(std::false_type{});
    }
    if (!at.live) return;
    if constexpr (kEnds) {
        store_floats(p.carry + at.unit * s.channels + at.c, h);
        store_floats(p.span + at.unit * s.channels + at.c, cut ? all<V>(1.0f) : span);
    } else if (at.t1 == s.time && p.state_out != nullptr) {
        store_floats(p.state_out + at.b * s.channels + at.c, h);
    }
}

// Chains the segments of a row: each end is replaced by the value that enters the segment.  From the first segment on
// (forward: states) or from the last one back (gradients).  A block takes 32 channels; its warps take a run of segments each, find
// what it makes of a zero, chain the runs before theirs and go through their own again.
constexpr int kAhead = 16;
constexpr int kCarryWarps = 16;          // at most

// The value behind a segment, or a run of them: `end` is what a zero became, L the sum of its logarithms (positive: a reset).
__device__ __forceinline__ float carried(float h, float end, float L)
{
    return L > 0.0f ? end : decayed(decay_less_one(L), h) + end;
}

__global__ void __launch_bounds__(32 * kCarryWarps)
k_carry(const Shape s, float *carry, const float *span, const float *start, const int backward)
{
    __shared__ float s_end[kCarryWarps][32], s_span[kCarryWarps][32];
    allow_next();
    wait_for_previous();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    const int tiles = (s.channels + 31) / 32;
    const int64_t b = blockIdx.x / tiles;
    const int c = static_cast<int>(blockIdx.x % tiles) * 32 + lane;
    const bool live = c < s.channels;
    const int64_t index = b * s.channels + (live ? c : 0);
    const int64_t step = backward ? -s.channels : s.channels;
    const int64_t base = b * s.segments * s.channels + (live ? c : 0) + (backward ? static_cast<int64_t>(s.segments - 1) * s.channels : 0);
    const int per = (s.segments + warps - 1) / warps, first = min(warp * per, s.segments), last = min(first + per, s.segments);
    float end[kAhead] = {}, sum[kAhead] = {};
    auto fetch = [&](int from) {
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            const bool in = from + k < last;
            end[k] = in ? carry[base + (from + k) * step] : 0.0f;
            sum[k] = in ? span[base + (from + k) * step] : 0.0f;
        }
    };
    float h = 0.0f, L = 0.0f;
    bool cut = false;
    if (per <= kAhead) fetch(first);
    if (warp + 1 < warps) {                              // (nobody asks for the last run)
        for (int g = first; g < last; g += kAhead) {
            if (per > kAhead) fetch(g);
#pragma unroll
            for (int k = 0; k < kAhead; ++k) {           // (a segment that is not there: nothing changes)
                h = carried(h, end[k], sum[k]);
                cut = cut || sum[k] > 0.0f;
                L += sum[k];
            }
        }
    }
    s_end[warp][lane] = h;
    s_span[warp][lane] = cut ? 1.0f : L;
    __syncthreads();
    h = start == nullptr ? 0.0f : start[index];
    for (int w = 0; w < warp; ++w) h = carried(h, s_end[w][lane], s_span[w][lane]);
    for (int g = first; g < last; g += kAhead) {
        if (per > kAhead) fetch(g);
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            if (g + k >= last) break;
            if (live) carry[base + (g + k) * step] = h;
            h = carried(h, end[k], sum[k]);
        }
    }
}

// (16-bit types: four blocks per SM, 287 us at 512 x 128 x 1152 against 390 with the two or three that more registers leave;
// binary32 would spill.)
template <typename T, int V, bool kEnds>
__global__ void __launch_bounds__(kThreads, sizeof(T) == 2 && !kEnds ? 4 : 1)
k_backward(const Shape s, const Params<T> p)
{
    using F = Vals<V>;
    allow_next();
    wait_for_previous();
    const int tiles = (s.channels + 32 * V - 1) / (32 * V);
    const int64_t warp = static_cast<int64_t>(blockIdx.x) * kWarps + (threadIdx.x >> 5);
    const int64_t units = s.batch * s.segments, slot = warp / tiles, slots = kEnds ? units : s.slots;
    if (slot >= slots) return;
    const int tile = static_cast<int>(warp % tiles);
    const int chunks = (s.time + kSaved - 1) / kSaved;
    const F zero = all<V>(0.0f), one = all<V>(1.0f);
    F da = zero;
    int c = 0;
    bool live = false;
    for (int64_t unit = slot; unit < units; unit += slots) {
        const Place<V> at(s, unit, tile);
        c = at.c;
        live = at.live;
        const F a = load_floats<V>(p.a + c);
        F g = zero, span = zero;         // g: what comes from behind the step
        if (!kEnds)
            g = load_floats<V>(s.segments > 1 ? p.carry + unit * s.channels + c
                                              : p.dstate_out == nullptr ? nullptr : p.dstate_out + at.b * s.channels + c);
        bool cut = false;
        constexpr int K = kSaved;
        Block<T, V, K> nx, nr, ni, ndy;
        F nh = zero;
        auto fetch = [&](int t) {
            nr.load(p.r, at, t);
            ndy.load(p.dy, at, t);
            if (!kEnds) {
                nx.load(p.x, at, t);
                ni.load(p.i, at, t);
                nh = load_floats<V>(p.saved + (at.b * chunks + t / K) * s.channels + c);
            }
        };
        const int last = at.t0 + (at.t1 - 1 - at.t0) / K * K;
        fetch(last);
        for (int t = last; t >= at.t0; t -= K) {
            const Block<T, V, K> x = nx, r = nr, i = ni, dy = ndy;
            const uint32_t resets = resets_at<K>(p, at.b, t, at.t1);
            F h = nh;
            if (t > at.t0) fetch(t - K);
            auto work = [&](auto plain) {
                if constexpr (kEnds) {
#pragma unroll
                    for (int k = K - 1; k >= 0; --k) {
                        if (!plain.value && t + k >= at.t1) continue;
                        const F L = mul(a, sigmoid<T>(widen(r.v[k]))), gt = add(g, widen(dy.v[k]));
                        g = fma(decay_less_one(L), gt, gt);
                        span = add(span, L);
                        if (!plain.value && (resets >> k) & 1u) {
                            cut = true;
                            g = zero;
                        }
                    }
                } else {
                    // the steps' gates and the states before them
                    F gate[K], slope[K], in[K], out[K], d[K], inverse[K], before[K];
#pragma unroll
                    for (int k = 0; k < K; ++k) {
                        F rest;
                        gate[k] = sigmoid<T>(widen(r.v[k]), rest);
                        in[k] = sigmoid<T>(widen(i.v[k]), out[k]);
                        const F L = mul(a, gate[k]);
                        slope[k] = mul(L, rest);             // dL / dr
                        d[k] = decay_less_one(L);
                        const F square = square_gain(d[k]);
                        inverse[k] = inverse_root(square);
                        before[k] = h;
                        if (!plain.value && (resets >> k) & 1u) before[k] = zero;
                        h = fma(mul(square, inverse[k]), mul(in[k], widen(x.v[k])), fma(d[k], before[k], before[k]));
                    }
                    F sum = zero;        // of these steps' terms of da: shorter chains
                    T *pdx = p.dx.row(at.b, t + K - 1) + c, *pdr = p.dr.row(at.b, t + K - 1) + c, *pdi = p.di.row(at.b, t + K - 1) + c;
#pragma unroll
                    for (int k = K - 1; k >= 0; --k) {
                        if (plain.value || t + k < at.t1) {
                            const F u = mul(in[k], widen(x.v[k])), gt = add(g, widen(dy.v[k]));
                            const F into = mul(gt, mul(square_gain(d[k]), inverse[k]));
                            const F keep = add(d[k], one);
                            const F dL = mul(mul(gt, keep), fma(mul(u, all<V>(-1.0f)), mul(keep, inverse[k]), before[k]));
                            sum = fma(dL, gate[k], sum);
                            g = fma(d[k], gt, gt);
                            if (!plain.value && (resets >> k) & 1u) g = zero;
                            if (live) {
                                packed_store<T, V>(pdx, narrow<T>(mul(into, in[k])));
                                packed_store<T, V>(pdr, narrow<T>(mul(dL, slope[k])));
                                packed_store<T, V>(pdi, narrow<T>(mul(mul(into, u), out[k])));
                            }
                        }
                        pdx -= p.dx.st;
                        pdr -= p.dr.st;
                        pdi -= p.di.st;
                    }
                    da = add(da, sum);
                }
            };
            if (resets == 0 && t + K <= at.t1)
                work(std::true_type{});
            else
                work(std::false_type{});
        }
        if (!live) continue;
        if constexpr (kEnds) {
            store_floats(p.carry + unit * s.channels + c, g);
            store_floats(p.span + unit * s.channels + c, cut ? one : span);
        } else if (at.segment == 0 && p.dstate != nullptr) {
            store_floats(p.dstate + at.b * s.channels + c, g);
        }
    }
    if constexpr (!kEnds) {
        if (live) store_floats(p.part + slot * s.channels + c, da);
    }
}

// da: a block takes 32 channels of the slots' sums, its warps share the slots.
constexpr int kJoinWarps = 8;

__global__ void __launch_bounds__(32 * kJoinWarps)
k_join(const float *part, int slots, int channels, float *da)
{
    __shared__ float s[kJoinWarps][32];
    allow_next();
    wait_for_previous();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, c = blockIdx.x * 32 + lane;
    float sum = 0.0f;
    if (c < channels) {
#pragma unroll 8
        for (int i = warp; i < slots; i += kJoinWarps) sum += part[static_cast<int64_t>(i) * channels + c];
    }
    s[warp][lane] = sum;
    __syncthreads();
    if (warp != 0 || c >= channels) return;
#pragma unroll
    for (int i = 1; i < kJoinWarps; ++i) sum += s[i][lane];
    da[c] = sum;
}

// One token: every thread takes V neighbouring channels of a row.
template <typename T>
struct Step {
    const T *x, *r, *i;
    T *y;
    const uint8_t *done;
    int64_t x_stride, r_stride, i_stride, y_stride, done_stride;
    const float *a, *state;
    float *state_out;
    int64_t n;
    int channels;
};

template <typename T, int V>
__global__ void __launch_bounds__(kStepThreads)
k_step(const Step<T> p)
{
    const int vectors = p.channels / V;
    const int64_t index = static_cast<int64_t>(blockIdx.x) * kStepThreads + threadIdx.x;
    if (index >= p.n * vectors) return;
    const int64_t n = index / vectors;
    const int c = static_cast<int>(index - n * vectors) * V;
    const Packed<T, V> x = packed_load<T, V>(p.x + n * p.x_stride + c), r = packed_load<T, V>(p.r + n * p.r_stride + c),
                       i = packed_load<T, V>(p.i + n * p.i_stride + c);
    const Packed<float, V> state = packed_load<float, V>(p.state + n * p.channels + c);
    const bool fresh = p.done != nullptr && p.done[n * p.done_stride] != 0;
    float h[V];
    if constexpr (V == 1) {
        h[0] = advance(decay_less_one(mul(__ldg(p.a + c), sigmoid<T>(widen(r)))), sigmoid<T>(widen(i)), widen(x),
                       fresh ? 0.0f : packed_get<float, 1>(state, 0));
    } else {
#pragma unroll
        for (int e = 0; e < V; e += 2) {
            auto two = [&](const auto &v) { return pair(packed_get<T, V>(v, e), packed_get<T, V>(v, e + 1)); };
            const Pair before = fresh ? pair(0.0f, 0.0f) : pair(packed_get<float, V>(state, e), packed_get<float, V>(state, e + 1));
            const Pair a = pair(__ldg(p.a + c + e), __ldg(p.a + c + e + 1));
            const Pair v = advance(decay_less_one(mul(a, sigmoid<T>(two(r)))), sigmoid<T>(two(i)), two(x), before);
            h[e] = lo(v);
            h[e + 1] = hi(v);
        }
    }
    packed_store<float, V>(p.state_out + n * p.channels + c, packed_of<float, V>(h));
    packed_store<T, V>(p.y + n * p.y_stride + c, packed_of<T, V>(h));
}

// ---------------------------------------------------------------- host side

constexpr int64_t kMaxBlocks = 0x7FFFFFFF;

int64_t div_up(int64_t a, int64_t b) { return (a + b - 1) / b; }

bool aligned(const void *ptr, size_t bytes) { return reinterpret_cast<uintptr_t>(ptr) % bytes == 0; }

}  // namespace

struct gated_recurrence {
    int channels = 0, type = 0;
    int device = 0, sms = 0;
    cudaStream_t stream = nullptr;
    int64_t launches = 0;
};

namespace {

int element_bytes(const gated_recurrence *p) { return p->type == GATED_RECURRENCE_F32 ? 4 : 2; }

bool sizes_ok(int64_t batch, int64_t time) { return batch >= 1 && time >= 1 && batch <= kMaxBlocks && time <= kMaxBlocks / 2; }

// The cut of the time axis, for warps of 64 channels, by what it would take in nanoseconds.  A warp by itself goes through eight
// steps in about 1,000 forward and 1,900 backward (800 in the pass that looks for a segment's end); the device through
// 500 elements a nanosecond forward, 260 backward (700), however they are cut.  Chaining costs two more launches and
// about 20 per segment.  (In bfloat16, 1 x 8,192 x 1,024: forward 43 us in 171 segments, 62 in 94; 64 x 512 x 512: 62 uncut,
// 78 in 5; backward 133 and 104.)
Shape shape_of(const gated_recurrence *p, int64_t batch, int64_t time, bool backward)
{
    Shape s = {};
    s.batch = batch;
    s.time = static_cast<int>(time);
    s.channels = p->channels;
    const int64_t tiles = div_up(p->channels, 64), warps = batch * tiles;
    const int64_t resident = static_cast<int64_t>(p->sms) * (backward ? 16 : 20);
    const int64_t chunks = div_up(time, kSteps);
    const double elements = static_cast<double>(batch) * time * p->channels;
    auto passes = [&](int64_t steps8, bool ends) {
        auto pass = [&](double chain, double rate) {
            const double alone = chain * steps8, all = elements / rate;
            return alone > all ? alone + 0.5 * all : all + 0.5 * alone;
        };
        return (backward ? pass(1900, 260) : pass(1000, 500)) + (!ends ? 0 : backward ? pass(800, 700) : 0.9 * pass(1000, 500));
    };
    s.segments = 1;
    s.segment_steps = static_cast<int>(chunks * kSteps);
    double best = passes(chunks * div_up(warps, resident), false);
    const int64_t round = resident / warps;              // segments that fill the device once
    auto consider = [&](int64_t n) {
        if (n < 2 || n > chunks) return;
        const int64_t per = div_up(chunks, n), segments = div_up(chunks, per);
        const double cost = passes(per * div_up(segments * warps, resident), true) + 6000 + 20.0 * segments;
        if (cost >= best) return;
        best = cost;
        s.segments = static_cast<int>(segments);
        s.segment_steps = static_cast<int>(per * kSteps);
    };
    for (int64_t n = 2; n < round; n += n / 2) consider(n);
    for (int64_t n = 1; n <= 4; ++n) consider(n * round);
    const int64_t units = batch * s.segments;
    int64_t slots = div_up(resident, tiles);
    if (slots > units) slots = units;
    s.slots = static_cast<int>(div_up(units, div_up(units, slots)));
    return s;
}

struct Scratch {
    size_t carry, span, part, total;
};

size_t align16(size_t v) { return (v + 15) & ~static_cast<size_t>(15); }

Scratch scratch_of(const Shape &s, bool backward)
{
    Scratch w = {};
    const size_t states = s.segments > 1 ? static_cast<size_t>(s.batch) * s.segments * s.channels * sizeof(float) : 0;
    w.span = align16(states);
    w.part = align16(w.span + states);
    w.total = backward ? align16(w.part + static_cast<size_t>(s.slots) * s.channels * sizeof(float)) : w.part;
    return w;
}

int check_seq(const gated_recurrence_seq &q, size_t bytes)
{
    if (q.ptr == nullptr) return GATED_RECURRENCE_ENULL;
    if (q.stride_b < 0 || q.stride_t < 0) return GATED_RECURRENCE_EINVAL;
    return aligned(q.ptr, bytes) ? GATED_RECURRENCE_OK : GATED_RECURRENCE_EALIGN;
}

// Do rows of `row` elements, of which `many` are `step` apart and these in turn `few` times `jump`, stay clear of
// one another?  They do where a jump passes all the steps; else the i-th jump has to land between two steps.
bool rows_apart(int64_t row, int64_t many, int64_t step, int64_t few, int64_t jump)
{
    if ((many > 1 && step < row) || (few > 1 && jump < row)) return false;
    if (many == 1 || few == 1) return true;
    using wide = __int128;
    if (jump >= static_cast<wide>(many - 1) * step + row || step >= static_cast<wide>(few - 1) * jump + row) return true;
    for (int64_t i = 1; i < few; ++i) {
        const wide at = static_cast<wide>(i) * jump, below = at / step;
        if (below < many && at - below * step < row) return false;
        if (below + 1 < many && (below + 1) * step - at < row) return false;
    }
    return true;
}

int check_out(const gated_recurrence_seq &q, size_t bytes, int64_t row, int64_t batch, int64_t time)
{
    const int rc = check_seq(q, bytes);
    if (rc != GATED_RECURRENCE_OK) return rc;
    const bool apart = batch < time ? rows_apart(row, time, q.stride_t, batch, q.stride_b)
                                    : rows_apart(row, batch, q.stride_b, time, q.stride_t);
    return apart ? GATED_RECURRENCE_OK : GATED_RECURRENCE_EINVAL;
}

int check(const gated_recurrence *p, const gated_recurrence_args *a, bool backward)
{
    if (p == nullptr || a == nullptr) return GATED_RECURRENCE_ENULL;
    if (!sizes_ok(a->batch, a->time)) return GATED_RECURRENCE_EINVAL;
    const size_t e = element_bytes(p);
    int rc;
    for (const gated_recurrence_seq *q : {&a->x, &a->r, &a->i})
        if ((rc = check_seq(*q, e)) != GATED_RECURRENCE_OK) return rc;
    if (a->reset.ptr != nullptr && (rc = check_seq(a->reset, 1)) != GATED_RECURRENCE_OK) return rc;
    if (a->a == nullptr) return GATED_RECURRENCE_ENULL;
    const float *floats[] = {a->a, a->state, a->state_out, a->saved, a->dstate_out, a->dstate, a->da};
    for (const float *v : floats)
        if (!aligned(v, 4)) return GATED_RECURRENCE_EALIGN;
    if (!aligned(a->workspace, 16)) return GATED_RECURRENCE_EALIGN;
    if (!backward) {
        if (a->state != nullptr && a->state == a->state_out) return GATED_RECURRENCE_EINVAL;
        return check_out(a->y, e, p->channels, a->batch, a->time);
    }
    if ((rc = check_seq(a->dy, e)) != GATED_RECURRENCE_OK) return rc;
    if (a->saved == nullptr || a->da == nullptr) return GATED_RECURRENCE_ENULL;
    for (const gated_recurrence_seq *q : {&a->dx, &a->dr, &a->di})
        if ((rc = check_out(*q, e, p->channels, a->batch, a->time)) != GATED_RECURRENCE_OK) return rc;
    return GATED_RECURRENCE_OK;
}

// A launch that may start while the kernel before it on the stream still runs: its blocks wait there for its results.
template <typename... Args>
bool launch_after(cudaStream_t stream, int64_t blocks, unsigned threads, void (*kernel)(Args...), Args... args)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(blocks));
    cfg.blockDim = dim3(threads);
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, args...) == cudaSuccess;
}

template <typename T>
Seq<T> seq_of(const gated_recurrence_seq &q) { return {static_cast<T *>(q.ptr), q.stride_b, q.stride_t}; }

// V elements of every row start on a boundary of their size.
bool pairs_ok(const gated_recurrence_seq &q, size_t e)
{
    return q.ptr == nullptr || (aligned(q.ptr, 2 * e) && q.stride_b % 2 == 0 && q.stride_t % 2 == 0);
}

template <typename T, int V>
int launch(gated_recurrence *p, const Shape &s, const Params<T> &k, bool backward)
{
    const int64_t tiles = div_up(s.channels, 32 * V), units = s.batch * s.segments;
    const int64_t blocks = div_up(units * tiles, kWarps);
    const int64_t chains = s.batch * div_up(s.channels, 32);
    if (blocks > kMaxBlocks || chains > kMaxBlocks) return GATED_RECURRENCE_EINVAL;
    bool ok = true;
    int launched = 0;
    // with few segments one warp has them all in its registers
    const int64_t carry_warps = s.segments <= kAhead ? 1 : s.segments > 8 * kCarryWarps ? kCarryWarps : div_up(s.segments, 8);
    if (s.segments > 1) {
        ok = backward ? (k_backward<T, V, true><<<static_cast<unsigned>(blocks), kThreads, 0, p->stream>>>(s, k), cudaGetLastError() == cudaSuccess)
                      : (k_forward<T, V, true><<<static_cast<unsigned>(blocks), kThreads, 0, p->stream>>>(s, k), cudaGetLastError() == cudaSuccess);
        ok = ok && launch_after(p->stream, chains, static_cast<unsigned>(32 * carry_warps), k_carry, s, k.carry,
                                static_cast<const float *>(k.span), backward ? k.dstate_out : k.state, backward ? 1 : 0);
        launched += 2;
    }
    if (ok && backward) {
        const int64_t grid = div_up(s.slots * tiles, kWarps);
        if (s.segments > 1) ok = launch_after(p->stream, grid, kThreads, k_backward<T, V, false>, s, k);
        else {
            k_backward<T, V, false><<<static_cast<unsigned>(grid), kThreads, 0, p->stream>>>(s, k);
            ok = cudaGetLastError() == cudaSuccess;
        }
        ok = ok && launch_after(p->stream, div_up(s.channels, 32), 32 * kJoinWarps, k_join, static_cast<const float *>(k.part),
                                s.slots, s.channels, k.da);
        launched += 2;
    } else if (ok) {
        if (s.segments > 1) ok = launch_after(p->stream, blocks, kThreads, k_forward<T, V, false>, s, k);
        else {
            k_forward<T, V, false><<<static_cast<unsigned>(blocks), kThreads, 0, p->stream>>>(s, k);
            ok = cudaGetLastError() == cudaSuccess;
        }
        launched += 1;
    }
    if (!ok) {
        cudaGetLastError();
        return GATED_RECURRENCE_ECUDA;
    }
    p->launches += launched;
    return GATED_RECURRENCE_OK;
}

template <typename T>
int run(gated_recurrence *p, const gated_recurrence_args *a, bool backward)
{
    const Shape s = shape_of(p, a->batch, a->time, backward);
    const Scratch w = scratch_of(s, backward);
    if (w.total > 0 && a->workspace == nullptr) return GATED_RECURRENCE_ENULL;
    if (w.total > a->workspace_bytes) return GATED_RECURRENCE_ENOMEM;
    uint8_t *base = static_cast<uint8_t *>(a->workspace);
    Params<T> k = {};
    k.x = seq_of<const T>(a->x);
    k.r = seq_of<const T>(a->r);
    k.i = seq_of<const T>(a->i);
    k.reset = seq_of<const uint8_t>(a->reset);
    k.a = a->a;
    k.saved = a->saved;
    if (w.total > 0) {
        k.carry = reinterpret_cast<float *>(base + w.carry);
        k.span = reinterpret_cast<float *>(base + w.span);
        k.part = reinterpret_cast<float *>(base + w.part);
    }
    bool pairs = p->channels % 2 == 0;
    for (const gated_recurrence_seq *q : {&a->x, &a->r, &a->i}) pairs = pairs && pairs_ok(*q, sizeof(T));
    if (backward) {
        k.dy = seq_of<const T>(a->dy);
        k.dx = seq_of<T>(a->dx);
        k.dr = seq_of<T>(a->dr);
        k.di = seq_of<T>(a->di);
        k.dstate_out = a->dstate_out;
        k.dstate = a->dstate;
        k.da = a->da;
        for (const gated_recurrence_seq *q : {&a->dy, &a->dx, &a->dr, &a->di}) pairs = pairs && pairs_ok(*q, sizeof(T));
    } else {
        k.y = seq_of<T>(a->y);
        k.state = a->state;
        k.state_out = a->state_out;
        pairs = pairs && pairs_ok(a->y, sizeof(T));
    }
    return pairs ? launch<T, 2>(p, s, k, backward) : launch<T, 1>(p, s, k, backward);
}

int call(gated_recurrence *p, const gated_recurrence_args *a, bool backward)
{
    const int rc = check(p, a, backward);
    if (rc != GATED_RECURRENCE_OK) return rc;
    const OnDevice on(p->device);
    if (!on.ok()) return GATED_RECURRENCE_ECUDA;
    if (p->type == GATED_RECURRENCE_F32) return run<float>(p, a, backward);
    return p->type == GATED_RECURRENCE_BF16 ? run<__nv_bfloat16>(p, a, backward) : run<__half>(p, a, backward);
}

template <typename T>
int step(gated_recurrence *p, const Step<T> &s, bool quads)
{
    const int64_t blocks = div_up(s.n * (p->channels / (quads ? 4 : 1)), kStepThreads);
    if (blocks > kMaxBlocks) return GATED_RECURRENCE_EINVAL;
    if (quads)
        k_step<T, 4><<<static_cast<unsigned>(blocks), kStepThreads, 0, p->stream>>>(s);
    else
        k_step<T, 1><<<static_cast<unsigned>(blocks), kStepThreads, 0, p->stream>>>(s);
    if (cudaGetLastError() != cudaSuccess) return GATED_RECURRENCE_ECUDA;
    p->launches += 1;
    return GATED_RECURRENCE_OK;
}

}  // namespace

extern "C" {

int gated_recurrence_create(gated_recurrence **out, int channels, int type)
{
    if (out == nullptr) return GATED_RECURRENCE_ENULL;
    *out = nullptr;
    if (channels < 1 || channels > GATED_RECURRENCE_MAX_CHANNELS) return GATED_RECURRENCE_EINVAL;
    if (type != GATED_RECURRENCE_F32 && type != GATED_RECURRENCE_BF16 && type != GATED_RECURRENCE_F16)
        return GATED_RECURRENCE_EINVAL;
    gated_recurrence *p = new (std::nothrow) gated_recurrence;
    if (p == nullptr) return GATED_RECURRENCE_ENOMEM;
    p->channels = channels;
    p->type = type;
    if (cudaGetDevice(&p->device) != cudaSuccess ||
        cudaDeviceGetAttribute(&p->sms, cudaDevAttrMultiProcessorCount, p->device) != cudaSuccess) {
        cudaGetLastError();
        delete p;
        return GATED_RECURRENCE_ECUDA;
    }
    *out = p;
    return GATED_RECURRENCE_OK;
}

int gated_recurrence_destroy(gated_recurrence *p)
{
    if (p == nullptr) return GATED_RECURRENCE_ENULL;
    delete p;
    return GATED_RECURRENCE_OK;
}

int gated_recurrence_set_stream(gated_recurrence *p, void *cuda_stream)
{
    if (p == nullptr) return GATED_RECURRENCE_ENULL;
    p->stream = static_cast<cudaStream_t>(cuda_stream);
    return GATED_RECURRENCE_OK;
}

size_t gated_recurrence_saved_bytes(const gated_recurrence *p, int64_t batch, int64_t time)
{
    if (p == nullptr || !sizes_ok(batch, time)) return 0;
    return static_cast<size_t>(batch) * div_up(time, kSaved) * p->channels * sizeof(float);
}

size_t gated_recurrence_workspace_bytes(const gated_recurrence *p, int64_t batch, int64_t time, int backward)
{
    if (p == nullptr || !sizes_ok(batch, time)) return 0;
    return scratch_of(shape_of(p, batch, time, backward != 0), backward != 0).total;
}

int gated_recurrence_forward(gated_recurrence *p, const gated_recurrence_args *a) { return call(p, a, false); }

int gated_recurrence_backward(gated_recurrence *p, const gated_recurrence_args *a) { return call(p, a, true); }

int gated_recurrence_step(gated_recurrence *p, const void *x, int64_t x_stride, const void *r, int64_t r_stride,
                          const void *i, int64_t i_stride, const uint8_t *done, int64_t done_stride, const float *a,
                          const float *state, float *state_out, void *y, int64_t y_stride, int64_t n)
{
    if (p == nullptr) return GATED_RECURRENCE_ENULL;
    if (n < 1 || n > kMaxBlocks) return GATED_RECURRENCE_EINVAL;
    if (x == nullptr || r == nullptr || i == nullptr || a == nullptr || state == nullptr || state_out == nullptr || y == nullptr)
        return GATED_RECURRENCE_ENULL;
    if (x_stride < 0 || r_stride < 0 || i_stride < 0 || done_stride < 0 || (n > 1 && y_stride < p->channels))
        return GATED_RECURRENCE_EINVAL;
    const size_t e = element_bytes(p);
    if (!aligned(x, e) || !aligned(r, e) || !aligned(i, e) || !aligned(y, e) || !aligned(a, 4) || !aligned(state, 4) ||
        !aligned(state_out, 4))
        return GATED_RECURRENCE_EALIGN;
    const OnDevice on(p->device);
    if (!on.ok()) return GATED_RECURRENCE_ECUDA;
    const bool quads = p->channels % 4 == 0 && aligned(x, 4 * e) && aligned(r, 4 * e) && aligned(i, 4 * e) && aligned(y, 4 * e) &&
                       aligned(state, 16) && aligned(state_out, 16) && x_stride % 4 == 0 && r_stride % 4 == 0 &&
                       i_stride % 4 == 0 && y_stride % 4 == 0;
    auto of = [&](auto zero) {
        using T = decltype(zero);
        const Step<T> s = {static_cast<const T *>(x), static_cast<const T *>(r), static_cast<const T *>(i), static_cast<T *>(y),
                           done, x_stride, r_stride, i_stride, y_stride, done_stride, a, state, state_out, n, p->channels};
        return step<T>(p, s, quads);
    };
    if (p->type == GATED_RECURRENCE_F32) return of(float{});
    return p->type == GATED_RECURRENCE_BF16 ? of(__nv_bfloat16{}) : of(__half{});
}

int64_t gated_recurrence_launch_count(const gated_recurrence *p) { return p ? p->launches : 0; }

const char *gated_recurrence_strerror(int code)
{
    switch (code) {
    case GATED_RECURRENCE_OK: return "ok";
    case GATED_RECURRENCE_EINVAL: return "invalid size, stride or type";
    case GATED_RECURRENCE_ENULL: return "required pointer is NULL";
    case GATED_RECURRENCE_EALIGN: return "pointer not aligned to its element";
    case GATED_RECURRENCE_ECUDA: return "CUDA call or launch failed";
    case GATED_RECURRENCE_ENOMEM: return "allocation failed, or the workspace is too small";
    default: return "unknown error";
    }
}

}  // extern "C"
