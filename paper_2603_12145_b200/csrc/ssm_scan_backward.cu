// ssm_scan_backward.cu -- gradients of the selective scan.
//
//     dh_t   = g_t c_t + E_t,    E_{t-1} = a_t dh_t  (zero where t starts an episode),   a_t = exp(delta_t A)
//     dc_t   = sum_d g h_t       db_t = sum_d dh_t delta x
//     pull   = sum_n dh_t b      S    = sum_n A dh_t a_t h_{t-1}
//     dx     = D g + delta pull  d delta = S + x pull   dA += delta dh_t a_t h_{t-1}
// with g = dy z sigmoid(z).  The recurrence of E runs backwards and needs h_t, which the forward
// pass saved at the start of every chunk of steps.
//
// A thread owns 4 channels x 4 states, a warp 32 channels x 16 states: sums over channels (db,
// dc) and over states (pull, S, y) are each formed over four values in registers first, and
// both then take eight or four lanes.  Halving exchanges leave every lane with one total: of
// the lane's own channel for the sums over states, of one (b or c, state) for the sums over
// channels, so that the per-channel arithmetic is spread over the warp without repetition.
//
// Per chunk of 16 steps the warp first brings its channels' x, dt, z and dy, all loads in flight
// together, and leaves what the steps need of them in shared memory.  It runs the recurrence
// forward once, keeping h at every fourth step; then it takes the groups of four steps from the
// last to the first, recomputes a_t and a_t h_{t-1} of the four steps into registers and walks
// them backwards.  Beyond 16 states the blocks of 16 states follow one another within the chunk.
//
// What bounds it: 425 instructions per warp, step and 32 channels x 16 states, 33 of them for the
// special-function unit, with 8 warps per SM: a_t and a_t h_{t-1} of four steps take 128 of
// the 255 registers.  512 x 128 x 1152 x 16 states in bfloat16: 1.90 ms, the schedulers 45 % busy.
// Chunks of 16 steps keep two blocks on an SM (84 KB each); with 32 it would be one.  Tried and
// slower: the next chunk's loads spread over the groups of this one (2.57 ms, spills).
//
// db and dc of a block's 128 channels are added in shared memory, those of different blocks by
// k_scan_dbc; dA, dD and d dt_bias stay with the block over all its rows and are added by
// k_scan_params: fixed orders, no atomics.
#include "ssm_kernels.cuh"

namespace ssm_k {
namespace {

constexpr int kGroup = 4;      // steps walked backwards out of registers
constexpr int kChunk = kScanChunk;

__device__ __forceinline__ Pair zero_pair() { return Pair{0ull}; }

// v[0..7] over the eight lanes that share lane & 3: lane gets the total of
// v[4 * bit 4 + 2 * bit 3 + bit 2 of lane].
__device__ __forceinline__ float spread8(const float (&v)[8], int lane)
{
    const bool b4 = lane & 16, b3 = lane & 8, b2 = lane & 4;
    float k[4], m[2];
#pragma unroll
    for (int i = 0; i < 4; ++i) k[i] = (b4 ? v[4 + i] : v[i]) + __shfl_xor_sync(0xFFFFFFFFu, b4 ? v[i] : v[4 + i], 16);
#pragma unroll
    for (int i = 0; i < 2; ++i) m[i] = (b3 ? k[2 + i] : k[i]) + __shfl_xor_sync(0xFFFFFFFFu, b3 ? k[i] : k[2 + i], 8);
    return (b2 ? m[1] : m[0]) + __shfl_xor_sync(0xFFFFFFFFu, b2 ? m[0] : m[1], 4);
}

__device__ __forceinline__ void load4(Pair (&dst)[2], const float *src)   // 16-byte aligned
{
    const ulonglong2 v = *reinterpret_cast<const ulonglong2 *>(src);
    dst[0].v = v.x;
    dst[1].v = v.y;
}

__device__ __forceinline__ void store4(float *dst, const Pair (&src)[2])
{
    *reinterpret_cast<ulonglong2 *>(dst) = make_ulonglong2(src[0].v, src[1].v);
}

// What a step needs of the lane's own channel, binary32 [step][32] each.
enum Scalar { kDelta, kDeltaX, kG, kX, kSig, kW, kScalars };   // kSig: sigmoid(dt + bias), kW: dy (z sigmoid(z))'

template <int SB>
struct Smem {
    static constexpr int kStates = 16 * SB;
    static constexpr int kThreads = scan_back_channels(kStates), kWarps = kThreads / 32;
    static constexpr int kBc = kChunk * 2 * kStates * 2;                // floats: every value twice
    static constexpr int kCheck = (kChunk / kGroup) * 16 * 32;          // per warp: h at every fourth step
    static constexpr int kScal = kScalars * kChunk * 32;                // per warp
    static constexpr int kAcc = SB > 1 ? kChunk * 3 * 32 : 0;           // per warp: y, pull, S of earlier state blocks
    static constexpr int kCarry = SB > 1 ? SB * 16 * 32 : 0;            // per warp: E; as many again: dA
    static constexpr int kWarp = kCheck + kScal + kAcc + 2 * kCarry;
    static constexpr int kBytes = (kBc + kWarps * kWarp) * 4;
};

__device__ __forceinline__ void load_bc(Pair (&dst)[4], const float *src)   // four states' values, each twice
{
    const ulonglong2 v = reinterpret_cast<const ulonglong2 *>(src)[0], w = reinterpret_cast<const ulonglong2 *>(src)[1];
    dst[0].v = v.x;
    dst[1].v = v.y;
    dst[2].v = w.x;
    dst[3].v = w.y;
}

__device__ __forceinline__ void clear(Pair (&h)[4][2])
{
#pragma unroll
    for (int n = 0; n < 4; ++n) h[n][0] = h[n][1] = zero_pair();
}

// A log2 e of the thread's 4 channels and 4 states, zero where one does not exist.
__device__ __forceinline__ void load_rates(Pair (&a2)[4][2], const ScanParams &p, const ScanShape &s, int channel, int channels,
                                           int state)
{
#pragma unroll
    for (int n = 0; n < 4; ++n) {
        float v[4];
#pragma unroll
        for (int c = 0; c < 4; ++c)
            v[c] = c < channels && state + n < s.states
                       ? p.a[static_cast<int64_t>(channel + c) * s.states + state + n] * kLog2e : 0.0f;
        a2[n][0] = pair(v[0], v[1]);
        a2[n][1] = pair(v[2], v[3]);
    }
}

__device__ __forceinline__ void load_saved(float4 (&h)[4], const ScanParams &p, const ScanShape &s, int64_t b, int chunk, int quad,
                                           int channel, int channels)
{
    const float4 *src = reinterpret_cast<const float4 *>(p.saved) + ((b * s.chunks + chunk) * s.quads + quad) * s.channels + channel;
#pragma unroll
    for (int c = 0; c < 4; ++c)
        h[c] = c < channels && quad < s.quads ? src[c] : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
}

// Four states per channel to four channels per state.
__device__ __forceinline__ void turn(Pair (&h)[4][2], const float4 (&v)[4])
{
#pragma unroll
    for (int c = 0; c < 2; ++c) {
        h[0][c] = pair(v[2 * c].x, v[2 * c + 1].x);
        h[1][c] = pair(v[2 * c].y, v[2 * c + 1].y);
        h[2][c] = pair(v[2 * c].z, v[2 * c + 1].z);
        h[3][c] = pair(v[2 * c].w, v[2 * c + 1].w);
    }
}

// Asks for a line that will be needed soon.
__device__ __forceinline__ void prefetch(const void *ptr) { asm volatile("prefetch.global.L2 [%0];" ::"l"(ptr)); }

template <typename T, int SB>
__global__ void __launch_bounds__(Smem<SB>::kThreads, 2)
k_scan_backward(const ScanShape s, const ScanParams p, const ScanSeqs<T> q, const int tiles)
{
    using S = Smem<SB>;
    constexpr int NS = S::kStates, kThreads = S::kThreads, kWarps = S::kWarps;
    constexpr int kStage = (kChunk * 2 * NS + kThreads - 1) / kThreads;   // values of b and c per thread and chunk
    allow_next();
    wait_for_previous();
    extern __shared__ __align__(16) float smem[];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    float *s_bc = smem;                                  // [step][b|c][NS][2]
    float *s_check = smem + S::kBc + warp * S::kWarp;    // [step / 4][4 states][32 lanes][4 channels]
    float *s_scal = s_check + S::kCheck;                 // [Scalar][step][32]
    float *s_acc = s_scal + S::kScal;                    // [step][y|pull|S][32]
    float *s_e = s_acc + S::kAcc;                        // [SB][4 states][32 lanes][4 channels]
    float *s_da = s_e + S::kCarry;

    const int tile = static_cast<int>(blockIdx.x % (tiles * s.groups));
    const int slot = static_cast<int>(blockIdx.x / (tiles * s.groups));
    const int g = tile / tiles;
    const int tile_in_group = tile - g * tiles;
    const int local0 = tile_in_group * kThreads + warp * 32;
    const int d0 = g * s.group_channels + local0;        // the warp's first channel
    const bool warp_live = local0 < s.group_channels;
    const int warps = min(kWarps, (s.group_channels - tile_in_group * kThreads + 31) / 32);
    const bool live = local0 + lane < s.group_channels;  // the lane's own channel
    const int own = live ? d0 + lane : 0;
    const int ch = 4 * (lane >> 2);                      // the thread's first channel within the warp
    const int quad = lane & 3;                           // the thread's states within a block of 16
    const int live4 = min(4, s.group_channels - (local0 + ch));   // how many of its channels exist (may be <= 0)
    const float bias = p.dt_bias != nullptr && live ? p.dt_bias[own] : 0.0f;
    const float skip = p.d != nullptr && live ? p.d[own] : 0.0f;
    const bool gated = q.z.ptr != nullptr;
    const int total_at = (lane & 16) + 4 * quad + ((lane >> 2) & 3);   // which sum over channels spread8 leaves here
    float dd = 0.0f, ddt_bias = 0.0f;
    // Rates, E and dA of the state block at hand: with a single block they stay here, else E and dA are in
    // shared memory between chunks
    Pair a2[4][2], e[4][2], da[4][2];
    if (SB == 1) load_rates(a2, p, s, d0 + ch, live4, 4 * quad);
    clear(da);
    if (SB > 1)
        for (int i = 0; i < 4 * SB; ++i) store4(s_da + (i * 32 + lane) * 4, da[0]);

    for (int64_t unit = slot; unit < s.batch * s.segments; unit += s.slots) {
        const int64_t b = unit / s.segments;
        const int seg = static_cast<int>(unit - b * s.segments);
        const int c_first = seg * (s.segment_steps / kChunk);
        const int c_last = min(s.chunks, c_first + s.segment_steps / kChunk) - 1;

        // gradient that arrives from the steps after the segment
        for (int sb = 0; sb < SB; ++sb) {
            float in[4][4];
#pragma unroll
            for (int c = 0; c < 4; ++c)
#pragma unroll
                for (int n = 0; n < 4; ++n) {
                    const int state = sb * 16 + 4 * quad + n;
                    in[n][c] = 0.0f;
                    if (c >= live4 || state >= s.states) continue;
                    if (seg < s.segments - 1)
                        in[n][c] = p.carry[(((b * s.segments + seg) * s.quads + sb * 4 + quad) * s.channels + d0 + ch + c) * 4 + n];
                    else if (p.dstate_out != nullptr)
                        in[n][c] = p.dstate_out[(b * s.channels + d0 + ch + c) * s.states + state];
                }
#pragma unroll
            for (int n = 0; n < 4; ++n) {
                e[n][0] = pair(in[n][0], in[n][1]);
                e[n][1] = pair(in[n][2], in[n][3]);
                if (SB > 1) store4(s_e + ((sb * 4 + n) * 32 + lane) * 4, e[n]);
            }
        }

        for (int chunk = c_last; chunk >= c_first; --chunk) {
            const int tc = chunk * kChunk;
            const int steps = min(kChunk, s.time - tc);
            const int groups = (steps + kGroup - 1) / kGroup;
            float4 hv[4];
            if (SB == 1) load_saved(hv, p, s, b, chunk, quad, d0 + ch, live4);
            uint32_t bc[kStage];
#pragma unroll
            for (int i = 0; i < kStage; ++i) {
                const int at = i * kThreads + tid;
                const int k = at / (2 * NS), n = at % NS;
                const Seq<const T> &src = (at / NS) & 1 ? q.c : q.b;
                bc[i] = k < steps && n < s.states ? load_bits(src.row(b, tc + k) + g * s.states + n) : 0;
            }
            uint32_t resets = 0;
            if (q.reset.ptr != nullptr)
                resets = __ballot_sync(0xFFFFFFFFu, lane < steps && *q.reset.row(b, tc + min(lane, steps - 1)) != 0);
            if (chunk > c_first && live) {      // the chunk that follows: a lane asks for its row of two sequences
                const int t = tc - kChunk + (lane & 15);
                prefetch((lane < 16 ? q.x : q.dt).row(b, t) + d0);
                if (lane < 16)      // and the first block of saved states: a line holds eight channels of a quad
                    prefetch(reinterpret_cast<const float4 *>(p.saved) +
                             ((b * s.chunks + chunk - 1) * s.quads + min(lane >> 2, s.quads - 1)) * s.channels + d0 +
                             min(8 * (lane & 3), s.group_channels - local0 - 1));
                prefetch((lane < 16 || !gated ? q.dy : q.z).row(b, t) + d0);
            }
            if (warp_live) {
                // All of the chunk's loads first, none of them conditional (a value that may also be a constant
                // would be waited for where the two meet): beyond the end the last step is read again, a lane without a channel
                // reads the first one, and without a gate x stands in for z.
                uint32_t x[kChunk], dt[kChunk], dy[kChunk], z[kChunk];
                const Seq<const T> &sz = gated ? q.z : q.x;
                const T *px = q.x.row(b, tc) + own, *pdt = q.dt.row(b, tc) + own, *pdy = q.dy.row(b, tc) + own;
                const T *pz = sz.row(b, tc) + own;
#pragma unroll
                for (int k = 0; k < kChunk; ++k) {
                    x[k] = load_bits(px);
                    dt[k] = load_bits(pdt);
                    dy[k] = load_bits(pdy);
                    z[k] = load_bits(pz);
                    if (k + 1 < steps) {
                        px += q.x.st;
                        pdt += q.dt.st;
                        pdy += q.dy.st;
                        pz += sz.st;
                    }
                }
#pragma unroll
                for (int k = 0; k < kChunk; k += 2) {
                    float *dst = s_scal + k * 32 + lane;
                    const bool in0 = live && k < steps, in1 = live && k + 1 < steps;
                    const Pair xv = pair(in0 ? from_bits<T>(x[k]) : 0.0f, in1 ? from_bits<T>(x[k + 1]) : 0.0f);
                    const Pair dyv = pair(in0 ? from_bits<T>(dy[k]) : 0.0f, in1 ? from_bits<T>(dy[k + 1]) : 0.0f);
                    Pair sig;
                    const Pair step = softplus(pair(from_bits<T>(dt[k]) + bias, from_bits<T>(dt[k + 1]) + bias), &sig);
                    const Pair delta = pair(in0 ? lo(step) : 0.0f, in1 ? hi(step) : 0.0f);
                    auto keep = [&](int which, Pair v) {
                        dst[which * kChunk * 32] = lo(v);
                        dst[which * kChunk * 32 + 32] = hi(v);
                    };
                    keep(kDelta, delta);
                    keep(kDeltaX, mul(delta, xv));
                    keep(kX, xv);
                    keep(kSig, sig);
                    if (gated) {
                        const Pair zv = pair(in0 ? from_bits<T>(z[k]) : 0.0f, in1 ? from_bits<T>(z[k + 1]) : 0.0f);
                        const Pair sg = gate_sigmoid<T>(zv), zs = mul(zv, sg);
                        keep(kG, mul(dyv, zs));
                        keep(kW, mul(dyv, fma(zs, fma(sg, pair(-1.0f, -1.0f), pair(1.0f, 1.0f)), sg)));
                    } else {
                        keep(kG, dyv);
                    }
                }
            }
#pragma unroll
            for (int i = 0; i < kStage; ++i) {
                const float v = from_bits<T>(bc[i]);
                if (i * kThreads + tid < kChunk * 2 * NS)
                    *reinterpret_cast<float2 *>(s_bc + 2 * (i * kThreads + tid)) = make_float2(v, v);
            }
            __syncthreads();

            for (int sb = 0; sb < SB; ++sb) {
                if (warp_live) {
                    if (SB > 1) {
                        load_rates(a2, p, s, d0 + ch, live4, sb * 16 + 4 * quad);
                        load_saved(hv, p, s, b, chunk, sb * 4 + quad, d0 + ch, live4);
                    }
                    Pair h[4][2];
                    turn(h, hv);
                    const float *bc4 = s_bc + (sb * 16 + 4 * quad) * 2;   // the thread's states of b; c is 2 NS further
                    const float *sc4 = s_scal + ch;                       // its channels' scalars

                    // forward over the chunk: h before every group of steps
#pragma unroll 1
                    for (int grp = 0;; ++grp) {
#pragma unroll
                        for (int n = 0; n < 4; ++n) store4(s_check + ((grp * 4 + n) * 32 + lane) * 4, h[n]);
                        if (grp == groups - 1) break;
#pragma unroll
                        for (int j = 0; j < kGroup; ++j) {
                            const int k = grp * kGroup + j;
                            Pair delta[2], dtx[2], bb[4];
                            load4(delta, sc4 + (kDelta * kChunk + k) * 32);
                            load4(dtx, sc4 + (kDeltaX * kChunk + k) * 32);
                            load_bc(bb, bc4 + (2 * k) * NS * 2);
                            if ((resets >> k) & 1u) clear(h);
#pragma unroll
                            for (int n = 0; n < 4; ++n)
#pragma unroll
                                for (int c = 0; c < 2; ++c)
                                    h[n][c] = fma(decay(a2[n][c], delta[c]), h[n][c], mul(dtx[c], bb[n]));
                        }
                    }
                    if (SB > 1) {
#pragma unroll
                        for (int n = 0; n < 4; ++n) {
                            load4(e[n], s_e + ((sb * 4 + n) * 32 + lane) * 4);
                            load4(da[n], s_da + ((sb * 4 + n) * 32 + lane) * 4);
                        }
                    }

                    T *pdx = q.dx.row(b, tc + groups * kGroup) + own, *pddt = q.ddt.row(b, tc + groups * kGroup) + own;
                    T *pdz = gated ? q.dz.row(b, tc + groups * kGroup) + own : nullptr;
#pragma unroll 1
                    for (int grp = groups - 1; grp >= 0; --grp) {
#pragma unroll
                        for (int n = 0; n < 4; ++n) load4(h[n], s_check + ((grp * 4 + n) * 32 + lane) * 4);
                        __syncwarp();
                        Pair at[kGroup][4][2], ah[kGroup][4][2];
                        float yp[kGroup];
#pragma unroll
                        for (int j = 0; j < kGroup; ++j) {
                            const int k = grp * kGroup + j;
                            Pair delta[2], dtx[2], bb[4], cc[4];
                            load4(delta, sc4 + (kDelta * kChunk + k) * 32);
                            load4(dtx, sc4 + (kDeltaX * kChunk + k) * 32);
                            load_bc(bb, bc4 + (2 * k) * NS * 2);
                            load_bc(cc, bc4 + (2 * k + 1) * NS * 2);
                            if ((resets >> k) & 1u) clear(h);
                            Pair y2[2] = {zero_pair(), zero_pair()};
#pragma unroll
                            for (int n = 0; n < 4; ++n)
#pragma unroll
                                for (int c = 0; c < 2; ++c) {
                                    at[j][n][c] = decay(a2[n][c], delta[c]);
                                    ah[j][n][c] = mul(at[j][n][c], h[n][c]);
                                    h[n][c] = fma(dtx[c], bb[n], ah[j][n][c]);
                                    y2[c] = fma(cc[n], h[n][c], y2[c]);
                                }
                            const float yv[4] = {lo(y2[0]), hi(y2[0]), lo(y2[1]), hi(y2[1])};
                            yp[j] = spread4(yv, lane);
                        }
#pragma unroll
                        for (int j = kGroup - 1; j >= 0; --j) {
                            const int k = grp * kGroup + j;
                            Pair delta[2], dtx[2], gg[2], bb[4], cc[4];
                            load4(delta, sc4 + (kDelta * kChunk + k) * 32);
                            load4(dtx, sc4 + (kDeltaX * kChunk + k) * 32);
                            load4(gg, sc4 + (kG * kChunk + k) * 32);
                            load_bc(bb, bc4 + (2 * k) * NS * 2);
                            load_bc(cc, bc4 + (2 * k + 1) * NS * 2);
                            Pair pull[2] = {zero_pair(), zero_pair()}, sa[2] = {zero_pair(), zero_pair()};
                            float dbc[8];
#pragma unroll
                            for (int n = 0; n < 4; ++n) {
                                Pair db2 = zero_pair(), dc2 = zero_pair();
#pragma unroll
                                for (int c = 0; c < 2; ++c) {
                                    const Pair ht = fma(dtx[c], bb[n], ah[j][n][c]);
                                    dc2 = c == 0 ? mul(gg[c], ht) : fma(gg[c], ht, dc2);
                                    const Pair dh = fma(gg[c], cc[n], e[n][c]);
                                    db2 = c == 0 ? mul(dtx[c], dh) : fma(dtx[c], dh, db2);
                                    pull[c] = n == 0 ? mul(bb[n], dh) : fma(bb[n], dh, pull[c]);
                                    const Pair qq = mul(dh, ah[j][n][c]);
                                    sa[c] = n == 0 ? mul(a2[n][c], qq) : fma(a2[n][c], qq, sa[c]);
                                    da[n][c] = fma(delta[c], qq, da[n][c]);
                                    e[n][c] = mul(at[j][n][c], dh);
                                }
                                dbc[n] = lo(db2) + hi(db2);
                                dbc[4 + n] = lo(dc2) + hi(dc2);
                            }
                            if ((resets >> k) & 1u) clear(e);
                            const float total = spread8(dbc, lane);
                            const float pv[4] = {lo(pull[0]), hi(pull[0]), lo(pull[1]), hi(pull[1])};
                            const float sv[4] = {lo(sa[0]), hi(sa[0]), lo(sa[1]), hi(sa[1])};
                            float own_pull = spread4(pv, lane), own_s = spread4(sv, lane), own_y = yp[j];
                            // the group's place in s_check has been read: its first words take the sums over channels
                            s_check[grp * 512 + j * 32 + total_at] = total;
                            if (SB > 1) {
                                float *acc = s_acc + (3 * k) * 32 + lane;
                                if (sb > 0) {
                                    own_y += acc[0];
                                    own_pull += acc[32];
                                    own_s += acc[64];
                                }
                                acc[0] = own_y;
                                acc[32] = own_pull;
                                acc[64] = own_s;
                            }
                            pdx -= q.dx.st;
                            pddt -= q.ddt.st;
                            pdz -= q.dz.st;
                            if (sb == SB - 1 && live && k < steps) {
                                const float *own_scal = s_scal + k * 32 + lane;
                                const float x = own_scal[kX * kChunk * 32], gr = own_scal[kG * kChunk * 32];
                                const float dx = fmaf(own_scal[kDelta * kChunk * 32], own_pull, skip * gr);
                                const float ddt = fmaf(x, own_pull, kLn2 * own_s) * own_scal[kSig * kChunk * 32];
                                *pdx = from_f32<T>(dx);
                                *pddt = from_f32<T>(ddt);
                                if (gated) *pdz = from_f32<T>(own_scal[kW * kChunk * 32] * fmaf(skip, x, own_y));
                                ddt_bias += ddt;
                                dd = fmaf(gr, x, dd);
                            }
                        }
                    }
                    if (SB > 1) {
#pragma unroll
                        for (int n = 0; n < 4; ++n) {
                            store4(s_e + ((sb * 4 + n) * 32 + lane) * 4, e[n]);
                            store4(s_da + ((sb * 4 + n) * 32 + lane) * 4, da[n]);
                        }
                    }
                }
                __syncthreads();
                // the block's channels together, the steps spread over the warps
                for (int k = warp; k < steps; k += kWarps) {
                    float sum = 0.0f;
                    for (int w = 0; w < warps; ++w)
                        sum += smem[S::kBc + w * S::kWarp + (k / kGroup) * 512 + (k % kGroup) * 32 + lane];
                    const int64_t row = (static_cast<int64_t>(tile_in_group) * s.batch + b) * s.time + tc + k;
                    p.dbc_part[((row * s.groups + g) * 2 + (lane >> 4)) * NS + sb * 16 + (lane & 15)] = sum;
                }
                __syncthreads();
            }
        }

        if (seg == 0 && p.dstate != nullptr && warp_live) {
            for (int sb = 0; sb < SB; ++sb) {
#pragma unroll
                for (int n = 0; n < 4; ++n) {
                    const int state = sb * 16 + 4 * quad + n;
                    if (SB > 1) load4(e[n], s_e + ((sb * 4 + n) * 32 + lane) * 4);
                    const float out[4] = {lo(e[n][0]), hi(e[n][0]), lo(e[n][1]), hi(e[n][1])};
#pragma unroll
                    for (int c = 0; c < 4; ++c)
                        if (c < live4 && state < s.states)
                            p.dstate[(b * s.channels + d0 + ch + c) * s.states + state] = out[c];
                }
            }
        }
    }

    if (!warp_live) return;
    for (int sb = 0; sb < SB; ++sb) {
        const int q4 = sb * 4 + quad;
#pragma unroll
        for (int n = 0; n < 4; ++n) {
            if (SB > 1) load4(da[n], s_da + ((sb * 4 + n) * 32 + lane) * 4);
            const float out[4] = {lo(da[n][0]), hi(da[n][0]), lo(da[n][1]), hi(da[n][1])};
#pragma unroll
            for (int c = 0; c < 4; ++c)
                if (c < live4 && q4 < s.quads)
                    p.da_part[((static_cast<int64_t>(slot) * s.quads + q4) * s.channels + d0 + ch + c) * 4 + n] = out[c];
        }
    }
    if (live) {
        p.dd_part[(static_cast<int64_t>(slot) * 2) * s.channels + own] = dd;
        p.dd_part[(static_cast<int64_t>(slot) * 2 + 1) * s.channels + own] = ddt_bias;
    }
}

// The recurrence of E over a segment from a zero end, a channel (or a 16-state part) per thread
// as in the forward kernel.
template <typename T, int NP, int LN>
__global__ void __launch_bounds__(128)
k_scan_back_summary(const ScanShape s, const ScanParams p, const ScanSeqs<T> q, const int tiles)
{
    constexpr int NS = NP * LN, kTile = 8;
    __shared__ __align__(16) float s_c[kTile][NS];
    __shared__ uint8_t s_reset[kTile];
    allow_next();
    wait_for_previous();
    const int tid = threadIdx.x;
    int64_t unit = blockIdx.x;
    const int tile = static_cast<int>(unit % (tiles * s.groups));
    unit /= tiles * s.groups;
    const int seg = static_cast<int>(unit % s.segments);
    const int64_t b = unit / s.segments;
    if (seg == 0) return;                             // nothing lies before the first segment
    const int g = tile / tiles;
    const int part = tid % LN;
    const int local = (tile - g * tiles) * (128 / LN) + tid / LN;
    const bool live = local < s.group_channels;
    const int d = g * s.group_channels + (live ? local : 0);
    const int t0 = seg * s.segment_steps;
    const int t1 = min(s.time, t0 + s.segment_steps);
    Pair a2[NP / 2], e[NP / 2];
#pragma unroll
    for (int i = 0; i < NP; i += 2) {
        const int n = part * NP + i;
        const float *row = p.a + static_cast<int64_t>(d) * s.states;
        a2[i / 2] = pair(live && n < s.states ? row[n] * kLog2e : 0.0f,
                         live && n + 1 < s.states ? row[n + 1] * kLog2e : 0.0f);
        e[i / 2] = zero_pair();
    }
    const float bias = p.dt_bias != nullptr && live ? p.dt_bias[d] : 0.0f;
    const bool gated = q.z.ptr != nullptr;
    float span = 0.0f;
    bool cut = false;
    for (int t = t0 + (t1 - 1 - t0) / kTile * kTile; t >= t0; t -= kTile) {
        float dt[kTile], gr[kTile];
#pragma unroll
        for (int k = 0; k < kTile; ++k) {
            const bool in = live && t + k < t1;
            dt[k] = in ? to_f32(q.dt.row(b, t + k)[d]) : 0.0f;
            gr[k] = in ? to_f32(q.dy.row(b, t + k)[d]) : 0.0f;
            if (gated) {
                const float z = in ? to_f32(q.z.row(b, t + k)[d]) : 0.0f;
                gr[k] *= z * sigmoid(z);
            }
        }
        __syncthreads();
        for (int i = tid; i < kTile * NS; i += 128) {
            const int k = i / NS, n = i % NS;
            s_c[k][n] = t + k < t1 && n < s.states ? to_f32(q.c.row(b, t + k)[g * s.states + n]) : 0.0f;
        }
        if (tid < kTile) s_reset[tid] = q.reset.ptr != nullptr && t + tid < t1 ? *q.reset.row(b, t + tid) : 0;
        __syncthreads();
#pragma unroll
        for (int k = kTile - 1; k >= 0; --k) {
            if (t + k >= t1) continue;
            const float delta = softplus(dt[k] + bias);
            const Pair dd = pair(delta, delta), gg = pair(gr[k], gr[k]);
            const bool first = s_reset[k] != 0;
            cut |= first;
            span += delta;
#pragma unroll
            for (int i = 0; i < NP / 2; ++i) {
                Pair c;
                c.v = *reinterpret_cast<const unsigned long long *>(&s_c[k][part * NP + 2 * i]);
                e[i] = first ? zero_pair() : mul(decay(a2[i], dd), fma(gg, c, e[i]));
            }
        }
    }
    if (!live) return;
#pragma unroll
    for (int i = 0; i < NP / 4; ++i) {
        const int64_t at = ((b * s.segments + seg) * s.quads + part * (NP / 4) + i) * s.channels + d;
        reinterpret_cast<float4 *>(p.carry)[at] = make_float4(lo(e[2 * i]), hi(e[2 * i]), lo(e[2 * i + 1]), hi(e[2 * i + 1]));
    }
    if (part == 0) p.span[(b * s.segments + seg) * s.channels + d] = cut ? -1.0f : span;
}

// Turns what leaves each segment at its start (from a zero end) into what arrives at its end, in place.
__global__ void __launch_bounds__(256)
k_scan_back_carry(const ScanShape s, const ScanParams p)
{
    allow_next();
    wait_for_previous();
    const int64_t i = static_cast<int64_t>(blockIdx.x) * blockDim.x + threadIdx.x;
    const int64_t per_row = static_cast<int64_t>(s.quads) * s.channels;
    if (i >= s.batch * per_row) return;
    const int64_t b = i / per_row;
    const int quad = static_cast<int>((i - b * per_row) / s.channels);
    const int d = static_cast<int>(i % s.channels);
    float a[4], e[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const int n = 4 * quad + k;
        const bool in = n < s.states;
        a[k] = in ? p.a[static_cast<int64_t>(d) * s.states + n] * kLog2e : 0.0f;
        e[k] = in && p.dstate_out != nullptr ? p.dstate_out[(b * s.channels + d) * s.states + n] : 0.0f;
    }
    float4 *slots = reinterpret_cast<float4 *>(p.carry) + (b * s.segments * s.quads + quad) * s.channels + d;
    const float *spans = p.span + b * s.segments * s.channels + d;
    const int64_t stride = static_cast<int64_t>(s.quads) * s.channels;
    for (int seg0 = s.segments - 1; seg0 >= 0; seg0 -= kAhead) {
        float4 out[kAhead];
        float span[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {               // what leaves the first segment goes to dstate
            const bool in = seg0 - k > 0;
            out[k] = in ? slots[(seg0 - k) * stride] : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
            span[k] = in ? spans[static_cast<int64_t>(seg0 - k) * s.channels] : 0.0f;
        }
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            if (seg0 - k < 0) break;
            slots[(seg0 - k) * stride] = make_float4(e[0], e[1], e[2], e[3]);
            const float outs[4] = {out[k].x, out[k].y, out[k].z, out[k].w};
#pragma unroll
            for (int i = 0; i < 4; ++i) e[i] = span[k] < 0.0f ? outs[i] : fmaf(decay(a[i], span[k]), e[i], outs[i]);
        }
    }
}

// db and dc: the sum over the blocks of a group's channels, in block order.
template <typename T>
__global__ void __launch_bounds__(256)
k_scan_dbc(const ScanShape s, const ScanParams p, const ScanSeqs<T> q, const int tiles, const int padded)
{
    allow_next();
    wait_for_previous();
    const int64_t i = static_cast<int64_t>(blockIdx.x) * blockDim.x + threadIdx.x;
    const int64_t rows = s.batch * s.time * s.groups;
    const int n = static_cast<int>(i % padded);
    const int64_t which_row = i / padded;             // (row, b | c)
    if (which_row >= 2 * rows || n >= s.states) return;
    float sum = 0.0f;
    for (int k = 0; k < tiles; ++k) sum += p.dbc_part[(k * 2 * rows + which_row) * padded + n];
    const int64_t row = which_row >> 1;
    const int g = static_cast<int>(row % s.groups);
    const int64_t bt = row / s.groups;
    const int64_t b = bt / s.time;
    const Seq<T> &dst = which_row & 1 ? q.dc : q.db;
    dst.row(b, bt - b * s.time)[g * s.states + n] = from_f32<T>(sum);
}

// dA, dD, d dt_bias: the sum over the slots.  32 neighbouring channels per warp, every eighth
// slot per warp, the eight sums added in order.  blockIdx.y: a quad of states, or the last: dD and d dt_bias.
__global__ void __launch_bounds__(256)
k_scan_params(const ScanShape s, const ScanParams p)
{
    allow_next();
    wait_for_previous();
    __shared__ float4 part[8][32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int d = blockIdx.x * 32 + lane;
    const int quad = blockIdx.y;
    const bool rates = quad < s.quads;
    float4 sum = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    if (d < s.channels) {
#pragma unroll 4
        for (int k = warp; k < s.slots; k += 8) {
            float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
            if (rates) {
                v = reinterpret_cast<const float4 *>(p.da_part)[(static_cast<int64_t>(k) * s.quads + quad) * s.channels + d];
            } else {
                v.x = p.dd_part[(static_cast<int64_t>(k) * 2) * s.channels + d];
                v.y = p.dd_part[(static_cast<int64_t>(k) * 2 + 1) * s.channels + d];
            }
            sum = make_float4(sum.x + v.x, sum.y + v.y, sum.z + v.z, sum.w + v.w);
        }
    }
    part[warp][lane] = sum;
    __syncthreads();
    if (warp != 0 || d >= s.channels) return;
    for (int w = 1; w < 8; ++w) {
        const float4 v = part[w][lane];
        sum = make_float4(sum.x + v.x, sum.y + v.y, sum.z + v.z, sum.w + v.w);
    }
    if (rates) {
        const float out[4] = {sum.x, sum.y, sum.z, sum.w};
        for (int n = 0; n < 4; ++n)
            if (4 * quad + n < s.states) p.da[static_cast<int64_t>(d) * s.states + 4 * quad + n] = out[n];
    } else {
        if (p.dd != nullptr) p.dd[d] = sum.x;
        if (p.ddt_bias != nullptr) p.ddt_bias[d] = sum.y;
    }
}

template <typename T, int NP, int LN>
void launch_summary(const ScanShape &s, const ScanParams &p, const ScanSeqs<T> &q, cudaStream_t stream)
{
    const int tiles = (s.group_channels + 128 / LN - 1) / (128 / LN);
    const unsigned blocks = static_cast<unsigned>(s.batch * s.segments * s.groups * tiles);
    k_scan_back_summary<T, NP, LN><<<blocks, 128, 0, stream>>>(s, p, q, tiles);
}

template <typename T, int SB>
int launch(const ScanShape &s, const ScanParams &p, const ScanSeqs<T> &q, cudaStream_t stream)
{
    using S = Smem<SB>;
    static_assert(S::kBytes <= 227 * 1024, "one block's shared memory");
    constexpr int kThreads = S::kThreads;
    const int tiles = (s.group_channels + kThreads - 1) / kThreads;
    if (cudaFuncSetAttribute(k_scan_backward<T, SB>, cudaFuncAttributeMaxDynamicSharedMemorySize, S::kBytes) != cudaSuccess)
        return -1;
    const dim3 blocks(static_cast<unsigned>(tiles * s.groups) * s.slots);
    int launched = 3;
    if (s.segments > 1) {
        if (s.states <= 4)
            launch_summary<T, 4, 1>(s, p, q, stream);
        else if (s.states <= 8)
            launch_summary<T, 8, 1>(s, p, q, stream);
        else
            launch_summary<T, 16, SB>(s, p, q, stream);
        const int64_t threads = s.batch * s.quads * s.channels;
        if (cudaGetLastError() != cudaSuccess ||
            !launch_after(stream, dim3(static_cast<unsigned>((threads + 255) / 256)), 256, 0, k_scan_back_carry, s, p) ||
            !launch_after(stream, blocks, kThreads, S::kBytes, k_scan_backward<T, SB>, s, p, q, tiles))
            return -1;
        launched += 2;
    } else {
        k_scan_backward<T, SB><<<blocks, kThreads, S::kBytes, stream>>>(s, p, q, tiles);
        if (cudaGetLastError() != cudaSuccess) return -1;
    }
    const int64_t values = s.batch * s.time * s.groups * 2 * S::kStates;
    const dim3 grid(static_cast<unsigned>((s.channels + 31) / 32), static_cast<unsigned>(s.quads + 1));
    const bool ok = launch_after(stream, dim3(static_cast<unsigned>((values + 255) / 256)), 256, 0, k_scan_dbc<T>, s, p, q, tiles,
                                 static_cast<int>(S::kStates)) &&
                    launch_after(stream, grid, 256, 0, k_scan_params, s, p);
    return ok ? launched : -1;
}

}  // namespace

template <typename T>
int launch_scan_backward(const ScanShape &s, const ScanParams &p, const ScanSeqs<T> &q, cudaStream_t stream)
{
    if (s.states <= 16) return launch<T, 1>(s, p, q, stream);
    if (s.states <= 32) return launch<T, 2>(s, p, q, stream);
    return launch<T, 4>(s, p, q, stream);
}

template int launch_scan_backward<float>(const ScanShape &, const ScanParams &, const ScanSeqs<float> &, cudaStream_t);
template int launch_scan_backward<__nv_bfloat16>(const ScanShape &, const ScanParams &, const ScanSeqs<__nv_bfloat16> &,
                                                 cudaStream_t);
template int launch_scan_backward<__half>(const ScanShape &, const ScanParams &, const ScanSeqs<__half> &, cudaStream_t);

}  // namespace ssm_k
