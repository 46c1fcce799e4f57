// gated_recurrence.cu -- the gated linear recurrence behind the C ABI of gated_recurrence.h: sequences, gradients, single
// tokens.
//
// A thread walks the time axis with the states of V neighbouring channels in registers (two where sizes, strides and
// pointers allow, so that a warp's access covers whole lines; else one), kSteps steps at a time; the next steps' loads are
// in flight meanwhile.  The lanes of a warp share a sequence, so that a ballot gives them its resets.
//
// Few rows: the time axis is cut into segments.  A first pass finds what each segment makes of a zero state and the sum of
// its L, k_carry chains them, and the second pass starts every segment from its state.  With many rows there is one
// segment and one pass.
//
// Backward, the state at the start of every kSteps steps is saved by the forward pass; a thread goes back through them,
// forms the states and gates of the kSteps steps in registers, and then walks these backwards.
//
// Arithmetic of a step.  With e = e^L - 1 to full relative precision (a polynomial for small L, where 1 - e^L would cancel),
// the decay is h + e h in one multiply-add and the gain sqrt(1 - e^(2 L)) = sqrt(-e (2 + e)): no second exponential, and no
// rounding of a decay just below one, which a slow channel would gather step after step.  A sigmoid is kept as the smaller of
// s and 1 - s with the argument's sign, so that both are at hand to full relative precision.  Per element: three exponentials, two
// reciprocals, one reciprocal square root.
#include <new>

#include "../../include/gated_recurrence.h"
#include "on_device.cuh"
#include "vectors.cuh"

namespace {

constexpr int kThreads = 128;
constexpr int kWarps = kThreads / 32;
constexpr int kSteps = 8;                // steps between saved states
constexpr int kStepThreads = 256;

__device__ __forceinline__ void allow_next() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void wait_for_previous() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

// ---- scalar functions

constexpr float kLog2e = 1.4426950408889634f;

__device__ __forceinline__ float ex2(float v)
{
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
    return r;
}

__device__ __forceinline__ float rcp(float v)
{
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
    return r;
}

__device__ __forceinline__ float rsq(float v)
{
    float r;
    asm("rsqrt.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
    return r;
}

// v or the bound, whichever is larger; a NaN stays.
__device__ __forceinline__ float at_least(float v, float bound)
{
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(v), "f"(bound));
    return r;
}

// e^v for v in [-104, 0].  v log2 e is formed in two parts: rounded to one binary32 number its error would be that of the
// exponent, |v| 2^-24 relative in the result.  A 16-bit argument's own step is far coarser: T decides.
template <typename T>
__device__ __forceinline__ float exp_of(float v)
{
    const float t = v * kLog2e;
    if (sizeof(T) == 2) return ex2(t);
    constexpr float kLog2eLow = 1.9259629911e-8f;   // log2 e - float(log2 e)
    constexpr float kLn2 = 0.6931471805599453f;
    const float low = fmaf(v, kLog2eLow, fmaf(v, kLog2e, -t));
    const float e = ex2(t);
    return fmaf(e * kLn2, low, e);
}

// The smaller of sigmoid(v) and 1 - sigmoid(v), with v's sign.
template <typename T>
__device__ __forceinline__ float signed_sigmoid(float v)
{
    const float e = exp_of<T>(at_least(-fabsf(v), -104.0f));
    return copysignf(e * rcp(1.0f + e), v);
}
__device__ __forceinline__ float sigmoid_of(float s) { return __float_as_int(s) < 0 ? -s : 1.0f - s; }
__device__ __forceinline__ float rest_of(float s) { return __float_as_int(s) < 0 ? 1.0f + s : s; }      // 1 - sigmoid

// e^L - 1, L <= 0: the series up to L^7 below 0.35 (the next term is under 2e-8 of the sum), else from the exponential, whose
// error then counts at most twofold.
__device__ __forceinline__ float decay_less_one(float L)
{
    float p = 1.0f / 5040.0f;
    p = fmaf(p, L, 1.0f / 720.0f);
    p = fmaf(p, L, 1.0f / 120.0f);
    p = fmaf(p, L, 1.0f / 24.0f);
    p = fmaf(p, L, 1.0f / 6.0f);
    p = fmaf(p, L, 0.5f);
    const float small = fmaf(p * L, L, L), large = exp_of<float>(at_least(L, -104.0f)) - 1.0f;
    return L > -0.35f ? small : large;
}

// e^L h from d = e^L - 1, with one rounding; an infinity stays one (d h and h would cancel to a NaN).
__device__ __forceinline__ float decayed(float d, float h)
{
    const float v = fmaf(d, h, h);
    return fabsf(h) == __int_as_float(0x7F800000) ? h : v;
}

// 1 / sqrt(1 - e^(2 L)) from e = e^L - 1; zero where nothing is left of it.
__device__ __forceinline__ float inverse_gain(float e, float &square)
{
    square = -e * (2.0f + e);
    return square < 1.2e-38f ? 0.0f : rsq(square);       // a NaN passes
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
    int segments, segment_steps;     // the latter a multiple of kSteps
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

// Steps [t, t + kSteps) that start an episode, as bits.
template <typename T>
__device__ __forceinline__ uint32_t resets_at(const Params<T> &p, int64_t b, int t, int t1)
{
    if (p.reset.ptr == nullptr) return 0;
    const int lane = threadIdx.x & 31;
    return __ballot_sync(0xFFFFFFFFu, lane < kSteps && t + lane < t1 && *p.reset.row(b, t + lane) != 0);
}

template <typename T, int V>
struct Block {                       // kSteps steps of a sequence
    Packed<T, V> v[kSteps];
    __device__ __forceinline__ void load(const Seq<const T> &q, const Place<V> &at, int t)
    {
        const T *ptr = q.row(at.b, t) + at.c;
#pragma unroll
        for (int k = 0; k < kSteps; ++k) {
            v[k] = t + k < at.t1 ? packed_load<T, V>(ptr) : packed_zero<T, V>();
            ptr += q.st;
        }
    }
};

template <int V>
__device__ __forceinline__ void load_floats(float (&dst)[V], const float *src)
{
#pragma unroll
    for (int e = 0; e < V; ++e) dst[e] = src == nullptr ? 0.0f : src[e];
}

// kEnds: the first pass over segments.
template <typename T, int V, bool kEnds>
__global__ void __launch_bounds__(kThreads)
k_forward(const Shape s, const Params<T> p)
{
    allow_next();
    wait_for_previous();
    const int tiles = (s.channels + 32 * V - 1) / (32 * V);
    const int64_t warp = static_cast<int64_t>(blockIdx.x) * kWarps + (threadIdx.x >> 5);
    if (warp >= s.batch * s.segments * tiles) return;
    const Place<V> at(s, warp / tiles, static_cast<int>(warp % tiles));
    float a[V], h[V], span[V];
    load_floats<V>(a, p.a + at.c);
    if (kEnds || (s.segments == 1 && p.state == nullptr)) {
#pragma unroll
        for (int e = 0; e < V; ++e) h[e] = 0.0f;
    } else {
        load_floats<V>(h, s.segments > 1 ? p.carry + at.unit * s.channels + at.c : p.state + at.b * s.channels + at.c);
    }
#pragma unroll
    for (int e = 0; e < V; ++e) span[e] = 0.0f;
    Block<T, V> nx, nr, ni;
    nx.load(p.x, at, at.t0);
    nr.load(p.r, at, at.t0);
    ni.load(p.i, at, at.t0);
    bool cut = false;
    for (int t = at.t0; t < at.t1; t += kSteps) {
        const Block<T, V> x = nx, r = nr, i = ni;
        const uint32_t resets = resets_at(p, at.b, t, at.t1);
        if (t + kSteps < at.t1) {
            nx.load(p.x, at, t + kSteps);
            nr.load(p.r, at, t + kSteps);
            ni.load(p.i, at, t + kSteps);
        }
        if (!kEnds && p.saved != nullptr && at.live) {
            float *dst = p.saved + (at.b * ((s.time + kSteps - 1) / kSteps) + t / kSteps) * s.channels + at.c;
#pragma unroll
            for (int e = 0; e < V; ++e) dst[e] = h[e];
        }
        T *py = kEnds ? nullptr : p.y.row(at.b, t) + at.c;
#pragma unroll
        for (int k = 0; k < kSteps; ++k) {
            if (t + k >= at.t1) break;
            if ((resets >> k) & 1u) {
                cut = true;
#pragma unroll
                for (int e = 0; e < V; ++e) h[e] = 0.0f;
            }
            float out[V];
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const float L = a[e] * sigmoid_of(signed_sigmoid<T>(packed_get<T, V>(r.v[k], e)));
                const float d = decay_less_one(L);
                float square;
                const float inverse = inverse_gain(d, square);
                const float u = sigmoid_of(signed_sigmoid<T>(packed_get<T, V>(i.v[k], e))) * packed_get<T, V>(x.v[k], e);
                h[e] = fmaf(square * inverse, u, decayed(d, h[e]));
                out[e] = h[e];
                if (kEnds) span[e] += L;
            }
            if (!kEnds) {
                if (at.live) packed_store<T, V>(py, packed_of<T, V>(out));
                py += p.y.st;
            }
        }
    }
    if (!at.live) return;
    if (kEnds) {
#pragma unroll
        for (int e = 0; e < V; ++e) {
            p.carry[at.unit * s.channels + at.c + e] = h[e];
            p.span[at.unit * s.channels + at.c + e] = cut ? 1.0f : span[e];
        }
    } else if (at.t1 == s.time && p.state_out != nullptr) {
#pragma unroll
        for (int e = 0; e < V; ++e) p.state_out[at.b * s.channels + at.c + e] = h[e];
    }
}

// Chains the segments of a row: each end is replaced by the value that enters the segment.  From the first segment on
// (forward: states) or from the last one back (gradients).
constexpr int kAhead = 8;

__global__ void __launch_bounds__(kThreads)
k_carry(const Shape s, float *carry, const float *span, const float *start, const int backward)
{
    allow_next();
    wait_for_previous();
    const int64_t index = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x;
    if (index >= s.batch * s.channels) return;
    const int64_t b = index / s.channels;
    const int c = static_cast<int>(index - b * s.channels);
    const int64_t base = b * s.segments * s.channels + c;
    float h = start == nullptr ? 0.0f : start[index];
    for (int g0 = 0; g0 < s.segments; g0 += kAhead) {
        float end[kAhead], sum[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            const int g = min(g0 + k, s.segments - 1);
            const int64_t at = base + static_cast<int64_t>(backward ? s.segments - 1 - g : g) * s.channels;
            end[k] = carry[at];
            sum[k] = span[at];
        }
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            if (g0 + k >= s.segments) break;
            carry[base + static_cast<int64_t>(backward ? s.segments - 1 - g0 - k : g0 + k) * s.channels] = h;
            h = sum[k] > 0.0f ? end[k] : decayed(decay_less_one(sum[k]), h) + end[k];
        }
    }
}

template <typename T, int V, bool kEnds>
__global__ void __launch_bounds__(kThreads)
k_backward(const Shape s, const Params<T> p)
{
    allow_next();
    wait_for_previous();
    const int tiles = (s.channels + 32 * V - 1) / (32 * V);
    const int64_t warp = static_cast<int64_t>(blockIdx.x) * kWarps + (threadIdx.x >> 5);
    const int64_t units = s.batch * s.segments, slot = warp / tiles, slots = kEnds ? units : s.slots;
    if (slot >= slots) return;
    const int tile = static_cast<int>(warp % tiles);
    const int chunks = (s.time + kSteps - 1) / kSteps;
    float a[V], da[V];
    int c = 0;
    bool live = false;
#pragma unroll
    for (int e = 0; e < V; ++e) da[e] = 0.0f;
    for (int64_t unit = slot; unit < units; unit += slots) {
        const Place<V> at(s, unit, tile);
        c = at.c;
        live = at.live;
        load_floats<V>(a, p.a + c);
        float g[V], span[V];             // g: what comes from behind the step
        if (kEnds) {
#pragma unroll
            for (int e = 0; e < V; ++e) g[e] = span[e] = 0.0f;
        } else {
            load_floats<V>(g, s.segments > 1 ? p.carry + unit * s.channels + c
                                             : p.dstate_out == nullptr ? nullptr : p.dstate_out + at.b * s.channels + c);
        }
        bool cut = false;
        Block<T, V> nx, nr, ni, ndy;
        float nh[V];
        auto fetch = [&](int t) {
            nr.load(p.r, at, t);
            ndy.load(p.dy, at, t);
            if (!kEnds) {
                nx.load(p.x, at, t);
                ni.load(p.i, at, t);
                load_floats<V>(nh, p.saved + (at.b * chunks + t / kSteps) * s.channels + c);
            }
        };
        const int last = at.t0 + (at.t1 - 1 - at.t0) / kSteps * kSteps;
        fetch(last);
        for (int t = last; t >= at.t0; t -= kSteps) {
            const Block<T, V> x = nx, r = nr, i = ni, dy = ndy;
            const uint32_t resets = resets_at(p, at.b, t, at.t1);
            float h[V];
            if (!kEnds) {
#pragma unroll
                for (int e = 0; e < V; ++e) h[e] = nh[e];
            }
            if (t > at.t0) fetch(t - kSteps);
            if constexpr (kEnds) {
#pragma unroll
                for (int k = kSteps - 1; k >= 0; --k) {
                    if (t + k >= at.t1) continue;
#pragma unroll
                    for (int e = 0; e < V; ++e) {
                        const float L = a[e] * sigmoid_of(signed_sigmoid<T>(packed_get<T, V>(r.v[k], e)));
                        g[e] += packed_get<T, V>(dy.v[k], e);
                        g[e] = decayed(decay_less_one(L), g[e]);
                        span[e] += L;
                    }
                    if ((resets >> k) & 1u) {
                        cut = true;
#pragma unroll
                        for (int e = 0; e < V; ++e) g[e] = 0.0f;
                    }
                }
            } else {
                // the steps' gates and the states before them
                float sr[kSteps][V], si[kSteps][V], d[kSteps][V], inverse[kSteps][V], before[kSteps][V];
#pragma unroll
                for (int k = 0; k < kSteps; ++k) {
                    const bool fresh = (resets >> k) & 1u;
#pragma unroll
                    for (int e = 0; e < V; ++e) {
                        sr[k][e] = signed_sigmoid<T>(packed_get<T, V>(r.v[k], e));
                        si[k][e] = signed_sigmoid<T>(packed_get<T, V>(i.v[k], e));
                        d[k][e] = decay_less_one(a[e] * sigmoid_of(sr[k][e]));
                        float square;
                        inverse[k][e] = inverse_gain(d[k][e], square);
                        before[k][e] = fresh ? 0.0f : h[e];
                        h[e] = fmaf(square * inverse[k][e], sigmoid_of(si[k][e]) * packed_get<T, V>(x.v[k], e),
                                    decayed(d[k][e], before[k][e]));
                    }
                }
                float sum[V];                // of these steps' terms of da: shorter chains
#pragma unroll
                for (int e = 0; e < V; ++e) sum[e] = 0.0f;
                T *pdx = p.dx.row(at.b, t) + c, *pdr = p.dr.row(at.b, t) + c, *pdi = p.di.row(at.b, t) + c;
#pragma unroll
                for (int k = kSteps - 1; k >= 0; --k) {
                    if (t + k >= at.t1) continue;
                    float dx[V], dr[V], di[V];
#pragma unroll
                    for (int e = 0; e < V; ++e) {
                        const float gate = sigmoid_of(sr[k][e]), in = sigmoid_of(si[k][e]), xv = packed_get<T, V>(x.v[k], e);
                        const float gt = g[e] + packed_get<T, V>(dy.v[k], e);
                        const float square = -d[k][e] * (2.0f + d[k][e]);
                        const float gain = gt * (square * inverse[k][e]);
                        dx[e] = gain * in;
                        di[e] = dx[e] * xv * rest_of(si[k][e]);
                        const float decay = 1.0f + d[k][e];
                        const float dL = gt * decay * (before[k][e] - in * xv * decay * inverse[k][e]);
                        dr[e] = dL * (a[e] * gate) * rest_of(sr[k][e]);
                        sum[e] = fmaf(dL, gate, sum[e]);
                        g[e] = (resets >> k) & 1u ? 0.0f : decayed(d[k][e], gt);
                    }
                    if (live) {
                        packed_store<T, V>(pdx + k * p.dx.st, packed_of<T, V>(dx));
                        packed_store<T, V>(pdr + k * p.dr.st, packed_of<T, V>(dr));
                        packed_store<T, V>(pdi + k * p.di.st, packed_of<T, V>(di));
                    }
                }
#pragma unroll
                for (int e = 0; e < V; ++e) da[e] += sum[e];
            }
        }
        if (!live) continue;
        if (kEnds) {
#pragma unroll
            for (int e = 0; e < V; ++e) {
                p.carry[unit * s.channels + c + e] = g[e];
                p.span[unit * s.channels + c + e] = cut ? 1.0f : span[e];
            }
        } else if (at.segment == 0 && p.dstate != nullptr) {
#pragma unroll
            for (int e = 0; e < V; ++e) p.dstate[at.b * s.channels + c + e] = g[e];
        }
    }
    if constexpr (!kEnds) {
        if (!live) return;
#pragma unroll
        for (int e = 0; e < V; ++e) p.part[slot * s.channels + c + e] = da[e];
    }
}

// da: a block takes 32 channels of the slots' sums, eight warps share the slots.
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
#pragma unroll
    for (int e = 0; e < V; ++e) {
        const float before = fresh ? 0.0f : packed_get<float, V>(state, e);
        const float d = decay_less_one(__ldg(p.a + c + e) * sigmoid_of(signed_sigmoid<T>(packed_get<T, V>(r, e))));
        float square;
        const float inverse = inverse_gain(d, square);
        const float u = sigmoid_of(signed_sigmoid<T>(packed_get<T, V>(i, e))) * packed_get<T, V>(x, e);
        h[e] = fmaf(square * inverse, u, decayed(d, before));
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

// The cut of the time axis, for warps of 64 channels.  One segment costs one pass over its steps, several cost two: the
// cut pays where the rows alone give less than half of the warps that the device holds.  The segments then fill one or a
// few whole rounds of them, whichever is the shortest.
Shape shape_of(const gated_recurrence *p, int64_t batch, int64_t time, bool backward)
{
    Shape s = {};
    s.batch = batch;
    s.time = static_cast<int>(time);
    s.channels = p->channels;
    const int64_t tiles = div_up(p->channels, 64), warps = batch * tiles;
    const int64_t resident = static_cast<int64_t>(p->sms) * (backward ? 12 : 24);
    const int64_t chunks = div_up(time, kSteps);
    s.segments = 1;
    s.segment_steps = static_cast<int>(chunks * kSteps);
    if (resident / warps >= 2 && chunks >= 4) {
        int64_t best = -1, best_per = chunks;
        for (int rounds = 1; rounds <= 4; ++rounds) {
            const int64_t most = rounds * resident / warps;
            const int64_t per = div_up(chunks, most < chunks ? most : chunks);
            const int64_t cost = div_up(div_up(chunks, per) * warps, resident) * (2 * per + 1);   // a segment's start: half a chunk
            if (best < 0 || cost < best) {
                best = cost;
                best_per = per;
            }
        }
        s.segments = static_cast<int>(div_up(chunks, best_per));
        s.segment_steps = static_cast<int>(best_per * kSteps);
    }
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
    if (blocks > kMaxBlocks || div_up(s.batch * s.channels, kThreads) > kMaxBlocks) return GATED_RECURRENCE_EINVAL;
    bool ok = true;
    int launched = 0;
    if (s.segments > 1) {
        ok = backward ? (k_backward<T, V, true><<<static_cast<unsigned>(blocks), kThreads, 0, p->stream>>>(s, k), cudaGetLastError() == cudaSuccess)
                      : (k_forward<T, V, true><<<static_cast<unsigned>(blocks), kThreads, 0, p->stream>>>(s, k), cudaGetLastError() == cudaSuccess);
        ok = ok && launch_after(p->stream, div_up(s.batch * s.channels, kThreads), kThreads, k_carry, s, k.carry,
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
    return static_cast<size_t>(batch) * div_up(time, kSteps) * p->channels * sizeof(float);
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
