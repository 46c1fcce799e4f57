// ssm_scan_forward.cu -- the selective scan over a sequence and its single-token form.
//
// k_scan_forward: a thread owns one channel (or, beyond 16 states, a 16-state part of one) and
// walks the time axis with the recurrent state in registers:
//     e = 2^(delta a log2 e),  h = e h + (delta x) b,  y += c h        per state
// on packed pairs of states.  A warp's 32 channels are neighbours, so every access to x, dt, z
// and y is one contiguous piece per step at any alignment; b and c, which all channels of a
// group share, are staged as binary32 in shared memory, four steps at a time, the next four
// steps' loads in flight meanwhile.
//
// What bounds it: per step and channel 20 results of the special-function unit (16 decays, softplus
// and gate two each; 16 per clock and SM) and some 155 instructions per warp.  512 x 128 x 1152 x
// 16 states in bfloat16: 0.515 ms with the saved states, the special-function unit 59 % busy, the
// schedulers 57 %, shared-memory returns 50 %; 16 warps per SM at 126 registers.  Tried and slower:
// two channels per thread (half the shared-memory reads, 0.68 ms: a quarter of the warps), tiles of 2
// and 8 steps, part of the decays as polynomials on the multiply-add pipe (0.52 - 0.57 ms).
//
// Few rows: the time axis is cut into segments that run side by side.  k_scan_summary forms
// each segment's end state from a zero start; since the decay over a whole segment is
// exp(a * sum delta), k_scan_carry joins the segments with one exponential per state and
// segment, and k_scan_forward then runs every segment from its true start.  1 x 8192 x 2048 x 16
// states: 98 + 7 + 118 us in 37 segments (a single segment would keep 16 of 148 SMs busy).
#include "ssm_kernels.cuh"

namespace ssm_k {
namespace {

constexpr int kThreads = 128;
constexpr int kTile = 4;     // steps whose loads are in flight together

template <int NP>
__device__ __forceinline__ void load_pairs(Pair (&dst)[NP / 2], const float *src)   // 16-byte aligned
{
#pragma unroll
    for (int i = 0; i < NP / 4; ++i) {
        const ulonglong2 v = reinterpret_cast<const ulonglong2 *>(src)[i];
        dst[2 * i].v = v.x;
        dst[2 * i + 1].v = v.y;
    }
}

// Minus infinity: the input of a step past the end, whose softplus is zero and leaves the state as it is.
template <typename T>
constexpr uint32_t kNoStep = 0;
template <>
constexpr uint32_t kNoStep<float> = 0xFF800000u;
template <>
constexpr uint32_t kNoStep<__nv_bfloat16> = 0xFF80u;
template <>
constexpr uint32_t kNoStep<__half> = 0xFC00u;

template <typename T, int NP, int LN, bool kSummary>
__global__ void __launch_bounds__(kThreads, LN > 1 ? 3 : 4)
k_scan_forward(const ScanShape s, const ScanParams p, const ScanSeqs<T> q, const int tiles)
{
    constexpr int NS = NP * LN;
    constexpr int kWidth = (kSummary ? 1 : 2) * NS;               // staged values per step: b (and c)
    constexpr int kStage = (kTile * kWidth + kThreads - 1) / kThreads;
    __shared__ __align__(16) float s_bc[2][kTile][kWidth];
    allow_next();
    wait_for_previous();
    const int tid = threadIdx.x;
    int64_t unit = blockIdx.x;
    const int tile = static_cast<int>(unit % (tiles * s.groups));
    unit /= tiles * s.groups;
    const int seg = static_cast<int>(unit % s.segments);
    const int64_t b = unit / s.segments;
    if (kSummary && seg == s.segments - 1) return;                // nobody asks for the last segment's end
    const int g = tile / tiles;
    const int part = tid % LN;
    const int local = (tile - g * tiles) * (kThreads / LN) + tid / LN;
    const bool live = local < s.group_channels;
    const bool warp_live = (tile - g * tiles) * (kThreads / LN) + (tid & ~31) / LN < s.group_channels;
    const int d = g * s.group_channels + (live ? local : 0);
    const int t0 = seg * s.segment_steps;
    const int t1 = min(s.time, t0 + s.segment_steps);

    Pair a2[NP / 2], h[NP / 2];
#pragma unroll
    for (int i = 0; i < NP; i += 2) {
        const int n = part * NP + i;
        const float *row = p.a + static_cast<int64_t>(d) * s.states;
        a2[i / 2] = pair(live && n < s.states ? row[n] * kLog2e : 0.0f,
                         live && n + 1 < s.states ? row[n + 1] * kLog2e : 0.0f);
        h[i / 2] = pair(0.0f, 0.0f);
    }
    if (!kSummary && live) {
        if (s.segments > 1) {
#pragma unroll
            for (int i = 0; i < NP / 4; ++i) {
                const int64_t at = ((b * s.segments + seg) * s.quads + part * (NP / 4) + i) * s.channels + d;
                const float4 v = reinterpret_cast<const float4 *>(p.carry)[at];
                h[2 * i] = pair(v.x, v.y);
                h[2 * i + 1] = pair(v.z, v.w);
            }
        } else if (p.state != nullptr) {
            const float *row = p.state + (b * s.channels + d) * s.states;
#pragma unroll
            for (int i = 0; i < NP; i += 2) {
                const int n = part * NP + i;
                h[i / 2] = pair(n < s.states ? row[n] : 0.0f, n + 1 < s.states ? row[n + 1] : 0.0f);
            }
        }
    }
    const float bias = p.dt_bias != nullptr && live ? p.dt_bias[d] : 0.0f;
    const float skip = p.d != nullptr && live ? p.d[d] : 0.0f;
    const bool gated = !kSummary && q.z.ptr != nullptr;

    // the next tile's values, in flight while the current one is worked on
    uint32_t nx[kTile], ndt[kTile], nz[kTile], nbc[kStage];
    uint8_t nreset = 0;
    const T *px = q.x.row(b, t0) + d, *pdt = q.dt.row(b, t0) + d, *pz = gated ? q.z.row(b, t0) + d : nullptr;
    T *py = kSummary ? nullptr : q.y.row(b, t0) + d;
    const T *pbc[kStage];
#pragma unroll
    for (int k = 0; k < kStage; ++k) {
        const int i = k * kThreads + tid;
        const Seq<const T> &src = (i / NS) % (kWidth / NS) == 0 ? q.b : q.c;
        pbc[k] = i < kTile * kWidth && i % NS < s.states ? src.row(b, t0 + i / kWidth) + g * s.states + i % NS : nullptr;
    }
    auto fetch = [&](int t) {
        if (warp_live) {
#pragma unroll
            for (int k = 0; k < kTile; ++k) {
                const bool in = live && t + k < t1;
                nx[k] = in ? load_bits(px) : 0;
                ndt[k] = in ? load_bits(pdt) : kNoStep<T>;
                px += q.x.st;
                pdt += q.dt.st;
                if (!kSummary) {
                    nz[k] = in && gated ? load_bits(pz) : 0;
                    pz += q.z.st;
                }
            }
        }
#pragma unroll
        for (int k = 0; k < kStage; ++k) {
            const int i = k * kThreads + tid;
            const int64_t st = (i / NS) % (kWidth / NS) == 0 ? q.b.st : q.c.st;
            nbc[k] = pbc[k] != nullptr && t + i / kWidth < t1 ? load_bits(pbc[k]) : 0;
            if (pbc[k] != nullptr) pbc[k] += kTile * st;
        }
        // a lane per step; a ballot shows a tile's resets to the whole warp
        const int lane = tid & 31;
        nreset = q.reset.ptr != nullptr && lane < kTile && t + lane < t1 ? *q.reset.row(b, t + lane) : 0;
    };
    fetch(t0);

    float span = 0.0f;
    bool cut = false;
    int buf = 0;
    for (int t = t0; t < t1; t += kTile, buf ^= 1) {
        // everything that does not wait for the recurrence, for all steps of the tile side by side
        float delta[kTile], xv[kTile], gate[kTile];
#pragma unroll
        for (int k = 0; k < kTile; k += 2) {
            const Pair step = softplus(pair(from_bits<T>(ndt[k]) + bias, from_bits<T>(ndt[k + 1]) + bias));
            delta[k] = lo(step);
            delta[k + 1] = hi(step);
            xv[k] = from_bits<T>(nx[k]);
            xv[k + 1] = from_bits<T>(nx[k + 1]);
            if (!kSummary) {
                const Pair z = pair(from_bits<T>(nz[k]), from_bits<T>(nz[k + 1]));
                const Pair f = mul(z, gate_sigmoid<T>(z));
                gate[k] = gated ? lo(f) : 1.0f;
                gate[k + 1] = gated ? hi(f) : 1.0f;
            }
        }
#pragma unroll
        for (int k = 0; k < kStage; ++k) {
            const int i = k * kThreads + tid;
            if (i < kTile * kWidth) (&s_bc[buf][0][0])[i] = from_bits<T>(nbc[k]);
        }
        const uint32_t resets = __ballot_sync(0xFFFFFFFFu, nreset != 0);
        __syncthreads();
        if (t + kTile < t1) fetch(t + kTile);
        if (!warp_live) continue;
        if (!kSummary && p.saved != nullptr && t % kScanChunk == 0 && live) {
#pragma unroll
            for (int i = 0; i < NP / 4; ++i) {
                const int64_t at = ((b * s.chunks + t / kScanChunk) * s.quads + part * (NP / 4) + i) * s.channels + d;
                reinterpret_cast<float4 *>(p.saved)[at] =
                    make_float4(lo(h[2 * i]), hi(h[2 * i]), lo(h[2 * i + 1]), hi(h[2 * i + 1]));
            }
        }
        const bool stores = live && part == 0;
#pragma unroll
        for (int k = 0; k < kTile; ++k) {
            if ((resets >> k) & 1u) {
                cut = true;
#pragma unroll
                for (int i = 0; i < NP / 2; ++i) h[i] = pair(0.0f, 0.0f);
            }
            span += delta[k];
            const Pair dd = pair(delta[k], delta[k]), dx = pair(delta[k] * xv[k], delta[k] * xv[k]);
            Pair bb[NP / 2], cc[NP / 2];
            load_pairs<NP>(bb, &s_bc[buf][k][part * NP]);
            if (!kSummary) load_pairs<NP>(cc, &s_bc[buf][k][NS * (kWidth / NS - 1) + part * NP]);
            Pair acc[2];
#pragma unroll
            for (int i = 0; i < NP / 2; ++i) {
                h[i] = fma(decay(a2[i], dd), h[i], mul(dx, bb[i]));
                if (!kSummary) acc[i & 1] = i < 2 ? mul(cc[i], h[i]) : fma(cc[i], h[i], acc[i & 1]);
            }
            if (!kSummary) {
                const Pair sum = add(acc[0], acc[1]);
                float y = lo(sum) + hi(sum);
#pragma unroll
                for (int m = 1; m < LN; m *= 2) y += __shfl_xor_sync(0xFFFFFFFFu, y, m);
                y = fmaf(skip, xv[k], y) * gate[k];
                if (stores && t + k < t1) *py = from_f32<T>(y);
                py += q.y.st;
            }
        }
    }
    if (!live) return;
    if (kSummary) {
#pragma unroll
        for (int i = 0; i < NP / 4; ++i) {
            const int64_t at = ((b * s.segments + seg) * s.quads + part * (NP / 4) + i) * s.channels + d;
            reinterpret_cast<float4 *>(p.carry)[at] =
                make_float4(lo(h[2 * i]), hi(h[2 * i]), lo(h[2 * i + 1]), hi(h[2 * i + 1]));
        }
        if (part == 0) p.span[(b * s.segments + seg) * s.channels + d] = cut ? -1.0f : span;
    } else if (t1 == s.time && p.state_out != nullptr) {
        float *row = p.state_out + (b * s.channels + d) * s.states;
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            const int n = part * NP + i;
            if (n < s.states) row[n] = i & 1 ? hi(h[i / 2]) : lo(h[i / 2]);
        }
    }
}

// Turns the segments' ends (from a zero start) into their starts, in place, kAhead segments' loads in flight together.
__global__ void __launch_bounds__(256)
k_scan_carry(const ScanShape s, const ScanParams p)
{
    allow_next();
    wait_for_previous();
    const int64_t i = static_cast<int64_t>(blockIdx.x) * blockDim.x + threadIdx.x;
    const int64_t per_row = static_cast<int64_t>(s.quads) * s.channels;
    if (i >= s.batch * per_row) return;
    const int64_t b = i / per_row;
    const int quad = static_cast<int>((i - b * per_row) / s.channels);
    const int d = static_cast<int>(i % s.channels);
    float a[4], h[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const int n = 4 * quad + e;
        const bool in = n < s.states;
        a[e] = in ? p.a[static_cast<int64_t>(d) * s.states + n] * kLog2e : 0.0f;
        h[e] = in && p.state != nullptr ? p.state[(b * s.channels + d) * s.states + n] : 0.0f;
    }
    float4 *slots = reinterpret_cast<float4 *>(p.carry) + (b * s.segments * s.quads + quad) * s.channels + d;
    const float *spans = p.span + b * s.segments * s.channels + d;
    const int64_t stride = static_cast<int64_t>(s.quads) * s.channels;
    for (int seg0 = 0; seg0 < s.segments; seg0 += kAhead) {
        float4 end[kAhead];
        float span[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {               // the last segment's end is nobody's start
            const bool in = seg0 + k < s.segments - 1;
            end[k] = in ? slots[(seg0 + k) * stride] : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
            span[k] = in ? spans[static_cast<int64_t>(seg0 + k) * s.channels] : 0.0f;
        }
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            if (seg0 + k >= s.segments) break;
            slots[(seg0 + k) * stride] = make_float4(h[0], h[1], h[2], h[3]);
            const float ends[4] = {end[k].x, end[k].y, end[k].z, end[k].w};
#pragma unroll
            for (int e = 0; e < 4; ++e) h[e] = span[k] < 0.0f ? ends[e] : fmaf(decay(a[e], span[k]), h[e], ends[e]);
        }
    }
}

template <typename T, int NP, int LN>
int launch(const ScanShape &s, const ScanParams &p, const ScanSeqs<T> &q, cudaStream_t stream)
{
    const int per_block = kThreads / LN;
    const int tiles = (s.group_channels + per_block - 1) / per_block;
    const unsigned blocks = static_cast<unsigned>(s.batch * s.segments * s.groups * tiles);
    if (s.segments == 1) {
        k_scan_forward<T, NP, LN, false><<<blocks, kThreads, 0, stream>>>(s, p, q, tiles);
        return cudaGetLastError() == cudaSuccess ? 1 : -1;
    }
    k_scan_forward<T, NP, LN, true><<<blocks, kThreads, 0, stream>>>(s, p, q, tiles);
    const int64_t threads = s.batch * s.quads * s.channels;
    const bool ok = cudaGetLastError() == cudaSuccess &&
                    launch_after(stream, dim3(static_cast<unsigned>((threads + 255) / 256)), 256, 0, k_scan_carry, s, p) &&
                    launch_after(stream, dim3(blocks), kThreads, 0, k_scan_forward<T, NP, LN, false>, s, p, q, tiles);
    return ok ? 3 : -1;
}

// ---- one token
//
// The state passes through memory once; 4 states make one 16-byte access and neighbouring lanes
// hold neighbouring quads, so a warp's accesses to the state are contiguous.  A block keeps its
// channels' parameters and walks rows, four at a time.  What a channel needs once per row (the
// step's softplus, the gate, the result) is spread over the lanes that share the channel, a row or
// two for each, and the others' reach it by shuffles: computed by every lane it would be three
// quarters of the instructions.  16,384 rows x 1152 x 16 states: 490 us, 5.2 TB/s of 2.57 GB
// (0.80 of the measured copy bandwidth; 603 us with the scalars in every lane).  64 registers for four blocks per
// SM: the binary32 form spills (48 bytes of stores per thread) and takes 524 us, 5.2 TB/s of 2.71 GB; without whole
// vectors (15 states: 132 to 164 bytes) it is 0.80 ms in binary32, 0.97 in bfloat16, 0.92 in binary16.

constexpr int kStepThreads = 256;
constexpr int kStepRows = 4;    // rows whose states are in flight together

// Four neighbouring elements of a row of b or c, as they lie in memory.
template <typename T>
struct Four {
    uint32_t w[sizeof(T)];
    __device__ __forceinline__ float at(int e) const
    {
        if (sizeof(T) == 4) return __uint_as_float(w[e]);
        return from_bits<T>(e & 1 ? w[e / 2] >> 16 : w[e / 2] & 0xFFFFu);
    }
};

template <typename T>
__device__ __forceinline__ Four<T> load_four(const T *p)     // aligned to its size
{
    Four<T> v;
    if constexpr (sizeof(T) == 4)
        asm volatile("ld.global.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.w[0]), "=r"(v.w[1]), "=r"(v.w[2]), "=r"(v.w[3]) : "l"(p));
    else
        asm volatile("ld.global.v2.u32 {%0, %1}, [%2];" : "=r"(v.w[0]), "=r"(v.w[1]) : "l"(p));
    return v;
}

template <typename T>
__device__ __forceinline__ Four<T> gather_four(const T *p, int count)
{
    uint32_t v[4];
    for (int e = 0; e < 4; ++e) v[e] = e < count ? load_bits(p + e) : 0;
    Four<T> r;
    for (int i = 0; i < static_cast<int>(sizeof(T)); ++i) r.w[i] = sizeof(T) == 4 ? v[i] : v[2 * i & 3] | v[(2 * i + 1) & 3] << 16;
    return r;
}

// kAligned: states, rows of b and c come in whole, aligned quads.
template <typename T, int LPC, bool kAligned>
__global__ void __launch_bounds__(kStepThreads, 4)
k_scan_step(const StepParams p, const T *__restrict__ x, const T *__restrict__ dt, const T *__restrict__ z,
            const T *__restrict__ bv, const T *__restrict__ cv, T *__restrict__ y, const int rows_per_block)
{
    constexpr int kChannels = kStepThreads / LPC;
    constexpr int kShare = LPC < kStepRows ? LPC : kStepRows, kOwn = kStepRows / kShare;   // rows whose scalars a lane forms
    static_assert(kStepRows == 4, "spread4 and the exchanges below");
    const int lane = threadIdx.x & 31;
    const int part = threadIdx.x % LPC;
    const int own0 = part % kShare * kOwn;
    const int c0 = blockIdx.x * kChannels + threadIdx.x / LPC;
    const int n0 = 4 * part;
    const bool live = c0 < p.channels;
    const bool holds = live && n0 < p.states;          // the thread has states
    const int d = live ? c0 : 0;
    const int g = d / p.group_channels;
    float a2[4];
#pragma unroll
    for (int e = 0; e < 4; ++e)
        a2[e] = holds && n0 + e < p.states ? p.a[static_cast<int64_t>(d) * p.states + n0 + e] * kLog2e : 0.0f;
    const float bias = p.dt_bias != nullptr ? p.dt_bias[d] : 0.0f;
    const float skip = p.d != nullptr ? p.d[d] : 0.0f;
    const int64_t r0 = static_cast<int64_t>(blockIdx.y) * rows_per_block;
    const int64_t r1 = r0 + rows_per_block < p.n ? r0 + rows_per_block : p.n;
    const int64_t state_row = static_cast<int64_t>(p.channels) * p.states;
    const int from = holds ? n0 : 0;
    const T *zs = z != nullptr ? z : x;                // without a gate x stands in for z
    const int64_t z_stride = z != nullptr ? p.z_stride : p.x_stride;
    for (int64_t r = r0; r < r1; r += kStepRows) {
        // All loads of the rows first, none of them conditional: lanes without states read the first ones.
        float4 h[kStepRows];
        uint32_t xv[kOwn], dv[kOwn], zv[kOwn];
        Four<T> bb[kStepRows], cc[kStepRows];
        uint8_t clear[kStepRows];
#pragma unroll
        for (int k = 0; k < kStepRows; ++k) {
            const int64_t row = r + k < r1 ? r + k : r1 - 1;
            const float *src = p.state + row * state_row + static_cast<int64_t>(d) * p.states + from;
            const T *b4 = bv + row * p.b_stride + g * p.states + from, *c4 = cv + row * p.c_stride + g * p.states + from;
            if (kAligned) {
                asm volatile("ld.global.L1::no_allocate.v4.f32 {%0, %1, %2, %3}, [%4];"
                             : "=f"(h[k].x), "=f"(h[k].y), "=f"(h[k].z), "=f"(h[k].w) : "l"(src));
                bb[k] = load_four(b4);
                cc[k] = load_four(c4);
            } else {
                const int count = min(4, p.states - from);
                h[k] = make_float4(src[0], count > 1 ? src[1] : 0.0f, count > 2 ? src[2] : 0.0f, count > 3 ? src[3] : 0.0f);
                bb[k] = gather_four(b4, count);
                cc[k] = gather_four(c4, count);
            }
            clear[k] = p.done != nullptr ? p.done[row * p.done_stride] : 0;
        }
#pragma unroll
        for (int i = 0; i < kOwn; ++i) {
            const int64_t row = r + own0 + i < r1 ? r + own0 + i : r1 - 1;
            xv[i] = load_bits(x + row * p.x_stride + d);
            dv[i] = load_bits(dt + row * p.dt_stride + d);
            zv[i] = load_bits(zs + row * z_stride + d);
        }
        float delta[kOwn], dx[kOwn];
#pragma unroll
        for (int i = 0; i < kOwn; ++i) {
            delta[i] = softplus(from_bits<T>(dv[i]) + bias);
            dx[i] = delta[i] * from_bits<T>(xv[i]);
        }
        float sum[kStepRows];
#pragma unroll
        for (int k = 0; k < kStepRows; ++k) {
            if (clear[k]) h[k] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
            const int source = lane - part + k / kOwn;
            const float step = kShare > 1 ? __shfl_sync(0xFFFFFFFFu, delta[k % kOwn], source) : delta[k % kOwn];
            const float input = kShare > 1 ? __shfl_sync(0xFFFFFFFFu, dx[k % kOwn], source) : dx[k % kOwn];
            float v[4] = {h[k].x, h[k].y, h[k].z, h[k].w};
            sum[k] = 0.0f;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                v[e] = fmaf(decay(a2[e], step), v[e], input * bb[k].at(e));
                sum[k] = fmaf(cc[k].at(e), v[e], sum[k]);
            }
            if (!holds) sum[k] = 0.0f;
            if (holds && r + k < r1) {
                float *dst = p.state_out + (r + k) * state_row + static_cast<int64_t>(d) * p.states + n0;
                if (kAligned) {
                    *reinterpret_cast<float4 *>(dst) = make_float4(v[0], v[1], v[2], v[3]);
                } else {
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (n0 + e < p.states) dst[e] = v[e];
                }
            }
        }
#pragma unroll
        for (int m = kShare; m < LPC; m *= 2)
#pragma unroll
            for (int k = 0; k < kStepRows; ++k) sum[k] += __shfl_xor_sync(0xFFFFFFFFu, sum[k], m);
        float mine[kOwn];
        if constexpr (kShare == 4) {
            mine[0] = spread4(sum, lane);
        } else {
#pragma unroll
            for (int i = 0; i < kOwn; ++i) {
                mine[i] = sum[i];
                if constexpr (kShare == 2) {
                    const float keep = part & 1 ? sum[2 + i] : sum[i], give = part & 1 ? sum[i] : sum[2 + i];
                    mine[i] = keep + __shfl_xor_sync(0xFFFFFFFFu, give, 1);
                }
            }
        }
#pragma unroll
        for (int i = 0; i < kOwn; ++i) {
            float out = fmaf(skip, from_bits<T>(xv[i]), mine[i]);
            if (z != nullptr) {
                const float zf = from_bits<T>(zv[i]);
                out *= zf * sigmoid(zf);
            }
            const int64_t row = r + own0 + i;
            if (live && part < kShare && row < r1) y[row * p.y_stride + d] = from_f32<T>(out);
        }
    }
}

template <typename T>
bool whole_quads(const T *ptr, int64_t stride)
{
    return reinterpret_cast<uintptr_t>(ptr) % (4 * sizeof(T)) == 0 && stride % 4 == 0;
}

template <typename T, int LPC>
int launch_step(const StepParams &p, const T *x, const T *dt, const T *z, const T *b, const T *c, T *y,
                cudaStream_t stream)
{
    const int per_block = kStepThreads / LPC;
    const unsigned tiles = static_cast<unsigned>((p.channels + per_block - 1) / per_block);
    // rows per block: enough blocks for eight per SM, then longer walks that reuse the parameters
    int64_t chunks = (static_cast<int64_t>(8) * p.sms + tiles - 1) / tiles;
    if (chunks < (p.n + 63) / 64) chunks = (p.n + 63) / 64;
    if (chunks > (p.n + kStepRows - 1) / kStepRows) chunks = (p.n + kStepRows - 1) / kStepRows;
    if (chunks > 65535) chunks = 65535;
    const int64_t rows = (p.n + chunks - 1) / chunks;
    const dim3 grid(tiles, static_cast<unsigned>((p.n + rows - 1) / rows));
    if (p.states % 4 == 0 && whole_quads(b, p.b_stride) && whole_quads(c, p.c_stride))
        k_scan_step<T, LPC, true><<<grid, kStepThreads, 0, stream>>>(p, x, dt, z, b, c, y, static_cast<int>(rows));
    else
        k_scan_step<T, LPC, false><<<grid, kStepThreads, 0, stream>>>(p, x, dt, z, b, c, y, static_cast<int>(rows));
    return cudaGetLastError() == cudaSuccess ? 1 : -1;
}

}  // namespace

template <typename T>
int launch_scan_forward(const ScanShape &s, const ScanParams &p, const ScanSeqs<T> &q, cudaStream_t stream)
{
    if (s.states <= 4) return launch<T, 4, 1>(s, p, q, stream);
    if (s.states <= 8) return launch<T, 8, 1>(s, p, q, stream);
    if (s.states <= 16) return launch<T, 16, 1>(s, p, q, stream);
    if (s.states <= 32) return launch<T, 16, 2>(s, p, q, stream);
    return launch<T, 16, 4>(s, p, q, stream);
}

template <typename T>
int launch_scan_step(const StepParams &p, const T *x, const T *dt, const T *z, const T *b, const T *c, T *y,
                     cudaStream_t stream)
{
    if (p.states <= 4) return launch_step<T, 1>(p, x, dt, z, b, c, y, stream);
    if (p.states <= 8) return launch_step<T, 2>(p, x, dt, z, b, c, y, stream);
    if (p.states <= 16) return launch_step<T, 4>(p, x, dt, z, b, c, y, stream);
    if (p.states <= 32) return launch_step<T, 8>(p, x, dt, z, b, c, y, stream);
    return launch_step<T, 16>(p, x, dt, z, b, c, y, stream);
}

#define SSM_INSTANTIATE(T)                                                                                     \
    template int launch_scan_forward<T>(const ScanShape &, const ScanParams &, const ScanSeqs<T> &,            \
                                        cudaStream_t);                                                         \
    template int launch_scan_step<T>(const StepParams &, const T *, const T *, const T *, const T *,           \
                                     const T *, T *, cudaStream_t);
SSM_INSTANTIATE(float)
SSM_INSTANTIATE(__nv_bfloat16)
SSM_INSTANTIATE(__half)

}  // namespace ssm_k
