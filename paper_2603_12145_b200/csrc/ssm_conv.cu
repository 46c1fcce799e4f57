// ssm_conv.cu -- the short causal convolution: sequence, gradients, single token.
//
// All three should be bound by memory: a thread takes V = 4 neighbouring channels (one 8- or
// 16-byte access, where sizes, strides and pointers allow; else V = 1) and walks a run of steps
// with the last width - 1 inputs in registers, so that each input is read once plus width - 1
// steps per run; the next tile's loads are in flight while a tile is computed.  Arithmetic is on
// pairs of channels.  The lanes of a warp share a sequence, so that a ballot gives them the
// resets of a tile; a tile without one, the common case, takes a path that does not look at them.
// A reset clears the window, which drops every tap from before the episode.
//
// 1024 x 128 x 1152 in bfloat16: forward 120 us (5.0 TB/s of 0.6 GB, a copy of the same bytes takes
// 100 us), backward 222 us (4.1 TB/s of 0.9 GB, schedulers 56 % busy).  In binary32: forward 199 us (6.1 TB/s),
// backward 511 us (3.5 TB/s).  Backward, four blocks per SM leave 128 registers: with width 4 some values are
// spilled (52 bytes of stores per thread in bfloat16, 44 in binary16, 256 in binary32).
//
// The backward kernel walks forward too: step t gives dpre_t, which goes into the pending
// gradients of x_t .. x_{t-width+1} (as far back as the episode reaches); the oldest one is
// then complete.  Its thread keeps its channels through all its runs, so dw and dbias stay in
// registers until the end; each thread's sums go to a row of their own and a second kernel adds
// the rows in a fixed order.
#include <cstring>
#include <type_traits>

#include "ssm_kernels.cuh"

namespace ssm_k {
namespace {

constexpr int kThreads = 128;

// V neighbouring elements as they lie in memory: one access, and nothing is taken apart before it is needed (an
// extraction right behind a load would wait for it).
template <int Bytes>
struct Words;
template <>
struct Words<2> {
    using type = uint16_t;
};
template <>
struct Words<4> {
    using type = uint32_t;
};
template <>
struct Words<8> {
    using type = uint2;
};
template <>
struct Words<16> {
    using type = uint4;
};

template <typename T, int V>
struct Vec {
    typename Words<sizeof(T) * V>::type w;
};

template <typename T, int V>
__device__ __forceinline__ Vec<T, V> load_vec(const T *p)
{
    return Vec<T, V>{*reinterpret_cast<const decltype(Vec<T, V>::w) *>(p)};
}

template <typename T, int V>
__device__ __forceinline__ void store_vec(T *p, const Vec<T, V> &v)
{
    *reinterpret_cast<decltype(Vec<T, V>::w) *>(p) = v.w;
}

template <typename T, int V>
__device__ __forceinline__ Vec<T, V> zero_vec()
{
    return Vec<T, V>{};
}

// V channels as pairs (a single channel leaves the upper half at zero).
template <typename T, int V>
__device__ __forceinline__ void widen(Pair (&dst)[(V + 1) / 2], const Vec<T, V> &v)
{
    T e[V];
    memcpy(e, &v.w, sizeof(e));
#pragma unroll
    for (int i = 0; i < V; i += 2) dst[i / 2] = pair(to_f32(e[i]), i + 1 < V ? to_f32(e[i + 1 < V ? i + 1 : i]) : 0.0f);
}

template <typename T>
__device__ __forceinline__ uint32_t narrow_two(Pair v);     // 16-bit types: both in one conversion
template <>
__device__ __forceinline__ uint32_t narrow_two<__nv_bfloat16>(Pair v)
{
    const __nv_bfloat162 r = __floats2bfloat162_rn(lo(v), hi(v));
    return *reinterpret_cast<const uint32_t *>(&r);
}
template <>
__device__ __forceinline__ uint32_t narrow_two<__half>(Pair v)
{
    const __half2 r = __floats2half2_rn(lo(v), hi(v));
    return *reinterpret_cast<const uint32_t *>(&r);
}

template <typename T, int V>
__device__ __forceinline__ Vec<T, V> narrow(const Pair (&src)[(V + 1) / 2])
{
    Vec<T, V> v;
    if constexpr (sizeof(T) == 2 && V == 4) {
        v.w = make_uint2(narrow_two<T>(src[0]), narrow_two<T>(src[1]));
    } else {
        T e[V];
#pragma unroll
        for (int i = 0; i < V; ++i) e[i] = from_f32<T>(i & 1 ? hi(src[i / 2]) : lo(src[i / 2]));
        memcpy(&v.w, e, sizeof(e));
    }
    return v;
}

// The activation's sigmoid: for a 16-bit result the exponent's rounding (|u| 2^-24 relative) is far below the result's.
template <typename T>
__device__ __forceinline__ Pair sigmoid_for(Pair u)
{
    if (sizeof(T) == 4) return pair(sigmoid(lo(u)), sigmoid(hi(u)));
    const Pair v = mul(u, pair(-kLog2e, -kLog2e));
    const Pair w = add(pair(ex2(lo(v)), ex2(hi(v))), pair(1.0f, 1.0f));
    return pair(rcp(lo(w)), rcp(hi(w)));
}

// The lane's part of a run of steps.
template <typename T>
struct Run {
    int64_t b;
    int t0, t1;
    __device__ Run(const ConvShape &s, int64_t unit)
    {
        b = unit / s.runs;
        t0 = static_cast<int>(unit - b * s.runs) * s.run;
        t1 = min(s.time, t0 + s.run);
    }
    // Lane k < count: does step t + k < end start an episode?  A ballot over the lanes, taken when the
    // tile is worked on, gives all of them the tile's resets.
    static __device__ uint8_t reset_of_lane(const ConvSeqs<T> &q, int64_t b, int t, int count, int end)
    {
        const int lane = threadIdx.x & 31;
        return q.reset.ptr != nullptr && lane < count && t + lane < end ? *q.reset.row(b, t + lane) : 0;
    }
};

// The window before step t0: win[j] = x[t0 - 1 - j], from the history before the sequence, zero
// where an episode starts between it and t0 - 1.  All loads are in flight together.
template <typename T, int V, int W>
__device__ __forceinline__ void load_window(Pair (&win)[W - 1][(V + 1) / 2], const ConvShape &s, const ConvSeqs<T> &q,
                                            int64_t b, int t0, int c)
{
    Vec<T, V> v[W - 1];
    bool starts[W - 1];
#pragma unroll
    for (int j = 0; j < W - 1; ++j) {
        const int t = t0 - 1 - j;
        v[j] = zero_vec<T, V>();
        if (t >= 0)
            v[j] = load_vec<T, V>(q.x.row(b, t) + c);
        else if (q.history != nullptr)
            v[j] = load_vec<T, V>(q.history + (b * (W - 1) + (W - 1 + t)) * s.channels + c);
        starts[j] = q.reset.ptr != nullptr && t >= 0 && *q.reset.row(b, t) != 0;
    }
    bool seen = true;
#pragma unroll
    for (int j = 0; j < W - 1; ++j) {
        widen<T, V>(win[j], seen ? v[j] : zero_vec<T, V>());
        seen = seen && !starts[j];
    }
}

template <int V>
__device__ __forceinline__ void load_params(Pair (&dst)[(V + 1) / 2], const float *src, int stride)
{
#pragma unroll
    for (int e = 0; e < V; e += 2)
        dst[e / 2] = src == nullptr ? Pair{0ull} : pair(src[e * stride], e + 1 < V ? src[(e + 1) * stride] : 0.0f);
}

template <typename T, int V, int W>
__global__ void __launch_bounds__(kThreads)
k_conv_forward(const ConvShape s, const ConvParams p, const ConvSeqs<T> q)
{
    constexpr int kTile = 8, P = (V + 1) / 2;
    const int vecs = s.channels / V, tiles = (vecs + 31) / 32;
    const int64_t warp = (static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x) / 32;
    const int64_t unit = warp / tiles;
    if (unit >= s.batch * s.runs) return;
    const int vec = static_cast<int>(warp - unit * tiles) * 32 + (threadIdx.x & 31);
    const bool live = vec < vecs;
    const int c = (live ? vec : 0) * V;
    const Run<T> r(s, unit);
    Pair w[W][P], bias[P], win[W - 1][P];
#pragma unroll
    for (int k = 0; k < W; ++k) load_params<V>(w[k], p.w + static_cast<int64_t>(c) * W + k, W);
    load_params<V>(bias, p.bias != nullptr ? p.bias + c : nullptr, 1);
    const T *px = q.x.row(r.b, r.t0) + c;
    T *py = q.y.row(r.b, r.t0) + c;
    Vec<T, V> next[kTile];
    auto fetch = [&](int t) {
#pragma unroll
        for (int k = 0; k < kTile; ++k) {
            next[k] = live && t + k < r.t1 ? load_vec<T, V>(px) : zero_vec<T, V>();
            px += q.x.st;
        }
    };
    fetch(r.t0);
    load_window<T, V, W>(win, s, q, r.b, r.t0, c);
    uint8_t next_reset = Run<T>::reset_of_lane(q, r.b, r.t0, kTile, r.t1);
    for (int t = r.t0; t < r.t1; t += kTile) {
        Vec<T, V> x[kTile];
#pragma unroll
        for (int k = 0; k < kTile; ++k) x[k] = next[k];
        const uint32_t resets = __ballot_sync(0xFFFFFFFFu, next_reset != 0);
        if (t + kTile < r.t1) {
            fetch(t + kTile);
            next_reset = Run<T>::reset_of_lane(q, r.b, t + kTile, kTile, r.t1);
        }
#pragma unroll
        for (int k = 0; k < kTile; ++k) {
            if (t + k >= r.t1) break;
            if ((resets >> k) & 1u) {
#pragma unroll
                for (int j = 0; j < W - 1; ++j)
#pragma unroll
                    for (int i = 0; i < P; ++i) win[j][i] = Pair{0ull};
            }
            Pair xv[P], out[P];
            widen<T, V>(xv, x[k]);
#pragma unroll
            for (int i = 0; i < P; ++i) {
                Pair u = bias[i];
#pragma unroll
                for (int j = W - 2; j >= 0; --j) u = fma(w[W - 2 - j][i], win[j][i], u);
                u = fma(w[W - 1][i], xv[i], u);
                out[i] = mul(u, sigmoid_for<T>(u));
#pragma unroll
                for (int j = W - 2; j > 0; --j) win[j][i] = win[j - 1][i];
                win[0][i] = xv[i];
            }
            if (live) store_vec<T, V>(py, narrow<T, V>(out));
            py += q.y.st;
        }
    }
    if (r.t1 == s.time && q.history_out != nullptr && live) {
#pragma unroll
        for (int j = 0; j < W - 1; ++j)
            store_vec<T, V>(q.history_out + (r.b * (W - 1) + (W - 2 - j)) * s.channels + c, narrow<T, V>(win[j]));
    }
}

template <typename T, int V, int W>
__global__ void __launch_bounds__(kThreads, 4)
k_conv_backward(const ConvShape s, const ConvParams p, const ConvSeqs<T> q)
{
    allow_next();
    wait_for_previous();
    constexpr int kTile = 4, P = (V + 1) / 2;
    const int vecs = s.channels / V, tiles = (vecs + 31) / 32;
    const int64_t warp = (static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x) / 32;
    const int slot = static_cast<int>(warp / tiles);
    if (slot >= s.slots) return;
    const int vec = static_cast<int>(warp - static_cast<int64_t>(slot) * tiles) * 32 + (threadIdx.x & 31);
    const bool live = vec < vecs;
    const int c = (live ? vec : 0) * V;
    const Pair zero = Pair{0ull}, one = pair(1.0f, 1.0f);
    Pair w[W][P], bias[P], dw[W][P], dbias[P];
#pragma unroll
    for (int k = 0; k < W; ++k) load_params<V>(w[k], p.w + static_cast<int64_t>(c) * W + k, W);
    load_params<V>(bias, p.bias != nullptr ? p.bias + c : nullptr, 1);
#pragma unroll
    for (int i = 0; i < P; ++i) {
#pragma unroll
        for (int k = 0; k < W; ++k) dw[k][i] = zero;
        dbias[i] = zero;
    }
    for (int64_t unit = slot; unit < s.batch * s.runs; unit += s.slots) {
        const Run<T> r(s, unit);
        const int t2 = r.t1 + W - 1;        // the gradients of the run's last inputs come from the steps up to here
        const int t3 = min(t2, s.time);     // steps that exist
        Pair win[W - 1][P], pend[W][P];
#pragma unroll
        for (int j = 0; j < W; ++j)
#pragma unroll
            for (int i = 0; i < P; ++i) pend[j][i] = zero;
        int age = W;                      // steps since the episode began, as far as the run's own inputs go
        const T *px = q.x.row(r.b, r.t0) + c, *pdy = q.dy.row(r.b, r.t0) + c;
        T *pdx = q.dx.row(r.b, r.t0) + c;
        Vec<T, V> nx[kTile], ndy[kTile];
        auto fetch = [&](int t) {
#pragma unroll
            for (int k = 0; k < kTile; ++k) {
                const bool in = live && t + k < t3;
                nx[k] = in ? load_vec<T, V>(px) : zero_vec<T, V>();
                ndy[k] = in ? load_vec<T, V>(pdy) : zero_vec<T, V>();
                px += q.x.st;
                pdy += q.dy.st;
            }
        };
        fetch(r.t0);
        load_window<T, V, W>(win, s, q, r.b, r.t0, c);
        uint8_t next_reset = Run<T>::reset_of_lane(q, r.b, r.t0, kTile, t3);
        for (int t = r.t0; t < t2; t += kTile) {
            Vec<T, V> x[kTile], dy[kTile];
#pragma unroll
            for (int k = 0; k < kTile; ++k) {
                x[k] = nx[k];
                dy[k] = ndy[k];
            }
            const uint32_t resets = __ballot_sync(0xFFFFFFFFu, next_reset != 0);
            if (t + kTile < t2) {
                fetch(t + kTile);
                next_reset = Run<T>::reset_of_lane(q, r.b, t + kTile, kTile, t3);
            }
            // kPlain: every step of the tile is the run's own, in one episode with its taps, and completes a gradient
            auto walk = [&](auto plain) {
                constexpr bool kPlain = decltype(plain)::value;
#pragma unroll
                for (int k = 0; k < kTile; ++k) {
                    if (!kPlain) {
                        if (t + k >= t2) break;
                        age = (resets >> k) & 1u ? 0 : age + 1;
                        if (age == 0) {
#pragma unroll
                            for (int j = 0; j < W - 1; ++j)
#pragma unroll
                                for (int i = 0; i < P; ++i) win[j][i] = zero;
                        }
                    }
                    Pair xv[P], dyv[P];
                    widen<T, V>(xv, x[k]);
                    widen<T, V>(dyv, dy[k]);
#pragma unroll
                    for (int i = 0; i < P; ++i) {
                        Pair u = bias[i];
#pragma unroll
                        for (int j = W - 2; j >= 0; --j) u = fma(w[W - 2 - j][i], win[j][i], u);
                        u = fma(w[W - 1][i], xv[i], u);
                        const Pair sg = sigmoid_for<T>(u);
                        // (u sigmoid(u))' = sg + u sg (1 - sg) = sg + (u sg) - (u sg) sg
                        const Pair us = mul(u, sg);
                        Pair dpre = mul(dyv[i], fma(us, fma(sg, pair(-1.0f, -1.0f), one), sg));
                        // past the end of the sequence there is no step: not 0 * slope, which a NaN would survive
                        if (!kPlain && t + k >= s.time) dpre = zero;
                        if (kPlain || t + k < r.t1) {
                            dbias[i] = add(dbias[i], dpre);
                            dw[W - 1][i] = fma(dpre, xv[i], dw[W - 1][i]);
#pragma unroll
                            for (int j = 0; j < W - 1; ++j) dw[W - 2 - j][i] = fma(dpre, win[j][i], dw[W - 2 - j][i]);
                        }
#pragma unroll
                        for (int j = W - 1; j > 0; --j)
                            pend[j][i] = kPlain || age >= j ? fma(dpre, w[W - 1 - j][i], pend[j - 1][i]) : pend[j - 1][i];
                        pend[0][i] = mul(dpre, w[W - 1][i]);
#pragma unroll
                        for (int j = W - 2; j > 0; --j) win[j][i] = win[j - 1][i];
                        win[0][i] = xv[i];
                    }
                    if (kPlain || t + k - (W - 1) >= r.t0) {
                        if (live) store_vec<T, V>(pdx, narrow<T, V>(pend[W - 1]));
                        pdx += q.dx.st;
                    }
                }
            };
            if (resets == 0 && age >= W - 1 && t >= r.t0 + W - 1 && t + kTile <= r.t1)
                walk(std::true_type());
            else
                walk(std::false_type());
        }
    }
    if (!live) return;
#pragma unroll
    for (int k = 0; k <= W; ++k)
        store_vec<float, V>(p.part + (static_cast<int64_t>(slot) * (W + 1) + k) * s.channels + c,
                            narrow<float, V>(k < W ? dw[k < W ? k : 0] : dbias));
}

// Adds the slots' rows of one (tap, channel): a warp takes 32 neighbouring channels at a time,
// each of the block's eight warps every eighth row, and the eight sums are added in order.
__global__ void __launch_bounds__(256)
k_conv_params(const ConvShape s, const ConvParams p)
{
    allow_next();
    wait_for_previous();
    __shared__ float part[8][32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int c = blockIdx.x * 32 + lane;
    const int k = blockIdx.y;
    float sum = 0.0f;
    if (c < s.channels) {
        const float *src = p.part + static_cast<int64_t>(k) * s.channels + c;
        const int64_t step = static_cast<int64_t>(s.width + 1) * s.channels;
#pragma unroll 8
        for (int r = warp; r < s.slots; r += 8) sum += src[r * step];
    }
    part[warp][lane] = sum;
    __syncthreads();
    if (warp != 0 || c >= s.channels) return;
    float total = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) total += part[i][lane];
    if (k < s.width)
        p.dw[static_cast<int64_t>(c) * s.width + k] = total;
    else if (p.dbias != nullptr)
        p.dbias[c] = total;
}

template <typename T, int V, int W>
__global__ void __launch_bounds__(kThreads)
k_conv_step(const ConvShape s, const ConvParams p, const T *__restrict__ x, const int64_t x_stride,
            const uint8_t *__restrict__ done, const int64_t done_stride, const T *history, T *history_out,
            T *__restrict__ y, const int64_t y_stride)
{
    constexpr int P = (V + 1) / 2;
    const int vecs = s.channels / V;
    const int64_t i = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x;
    const int64_t row = i / vecs;
    if (row >= s.batch) return;
    const int c = static_cast<int>(i - row * vecs) * V;
    const bool clear = done != nullptr && done[row * done_stride] != 0;
    const T *src = history + row * (W - 1) * s.channels + c;
    T *dst = history_out + row * (W - 1) * s.channels + c;
    Vec<T, V> taps[W];
#pragma unroll
    for (int k = 0; k < W - 1; ++k) taps[k] = load_vec<T, V>(src + k * s.channels);
    taps[W - 1] = load_vec<T, V>(x + row * x_stride + c);
    if (clear) {
#pragma unroll
        for (int k = 0; k < W - 1; ++k) taps[k] = zero_vec<T, V>();
    }
    Pair x4[W][P], out[P];
#pragma unroll
    for (int k = 0; k < W; ++k) widen<T, V>(x4[k], taps[k]);
    load_params<V>(out, p.bias != nullptr ? p.bias + c : nullptr, 1);
#pragma unroll
    for (int k = 0; k < W; ++k) {
        Pair w[P];
        load_params<V>(w, p.w + static_cast<int64_t>(c) * W + k, W);
#pragma unroll
        for (int i = 0; i < P; ++i) out[i] = fma(w[i], x4[k][i], out[i]);
    }
#pragma unroll
    for (int i = 0; i < P; ++i) out[i] = mul(out[i], sigmoid_for<T>(out[i]));
    store_vec<T, V>(y + row * y_stride + c, narrow<T, V>(out));
#pragma unroll
    for (int k = 0; k < W - 1; ++k) store_vec<T, V>(dst + k * s.channels, taps[k + 1]);
}

unsigned blocks_for(int64_t threads) { return static_cast<unsigned>((threads + kThreads - 1) / kThreads); }

// rows of `vecs` vectors, a whole number of warps each
int64_t warp_threads(int64_t rows, int vecs) { return rows * ((vecs + 31) / 32) * 32; }

template <typename T>
bool fits(const Seq<T> &q, int v)
{
    return reinterpret_cast<uintptr_t>(q.ptr) % (v * sizeof(T)) == 0 && q.sb % v == 0 && q.st % v == 0;
}

bool fits(const void *ptr, size_t bytes) { return reinterpret_cast<uintptr_t>(ptr) % bytes == 0; }

}  // namespace

#define SSM_BY_WIDTH(KERNEL, T, V, BLOCKS, ...)                                          \
    do {                                                                                 \
        if (s.width == 2)                                                                \
            KERNEL<T, V, 2><<<BLOCKS, kThreads, 0, stream>>>(__VA_ARGS__);               \
        else if (s.width == 3)                                                           \
            KERNEL<T, V, 3><<<BLOCKS, kThreads, 0, stream>>>(__VA_ARGS__);               \
        else                                                                             \
            KERNEL<T, V, 4><<<BLOCKS, kThreads, 0, stream>>>(__VA_ARGS__);               \
    } while (0)

template <typename T>
int launch_conv_forward(const ConvShape &s, const ConvParams &p, const ConvSeqs<T> &q, cudaStream_t stream)
{
    constexpr int V = 4;
    if (s.channels % V == 0 && fits(q.x, V) && fits(q.y, V) && fits(q.history, V * sizeof(T)) &&
        fits(q.history_out, V * sizeof(T))) {
        const unsigned blocks = blocks_for(warp_threads(s.batch * s.runs, s.channels / V));
        SSM_BY_WIDTH(k_conv_forward, T, V, blocks, s, p, q);
    } else {
        const unsigned blocks = blocks_for(warp_threads(s.batch * s.runs, s.channels));
        SSM_BY_WIDTH(k_conv_forward, T, 1, blocks, s, p, q);
    }
    return cudaGetLastError() == cudaSuccess ? 1 : -1;
}

template <typename T>
int launch_conv_backward(const ConvShape &s, const ConvParams &p, const ConvSeqs<T> &q, cudaStream_t stream)
{
    constexpr int V = 4;
    if (s.channels % V == 0 && fits(q.x, V) && fits(q.dy, V) && fits(q.dx, V) && fits(q.history, V * sizeof(T))) {
        const unsigned blocks = blocks_for(warp_threads(s.slots, s.channels / V));
        SSM_BY_WIDTH(k_conv_backward, T, V, blocks, s, p, q);
    } else {
        const unsigned blocks = blocks_for(warp_threads(s.slots, s.channels));
        SSM_BY_WIDTH(k_conv_backward, T, 1, blocks, s, p, q);
    }
    const dim3 grid(static_cast<unsigned>((s.channels + 31) / 32), static_cast<unsigned>(s.width + 1));
    const bool ok = cudaGetLastError() == cudaSuccess && launch_after(stream, grid, 256, 0, k_conv_params, s, p);
    return ok ? 2 : -1;
}

template <typename T>
int launch_conv_step(const ConvShape &s, const ConvParams &p, const T *x, int64_t x_stride, const uint8_t *done,
                     int64_t done_stride, const T *history, T *history_out, T *y, int64_t y_stride,
                     cudaStream_t stream)
{
    constexpr int V = 4;
    constexpr size_t kBytes = V * sizeof(T);
    if (s.channels % V == 0 && x_stride % V == 0 && y_stride % V == 0 && fits(x, kBytes) && fits(y, kBytes) &&
        fits(history, kBytes) && fits(history_out, kBytes)) {
        const unsigned blocks = blocks_for(s.batch * (s.channels / V));
        SSM_BY_WIDTH(k_conv_step, T, V, blocks, s, p, x, x_stride, done, done_stride, history, history_out, y, y_stride);
    } else {
        const unsigned blocks = blocks_for(s.batch * s.channels);
        SSM_BY_WIDTH(k_conv_step, T, 1, blocks, s, p, x, x_stride, done, done_stride, history, history_out, y, y_stride);
    }
    return cudaGetLastError() == cudaSuccess ? 1 : -1;
}

#define SSM_INSTANTIATE(T)                                                                                     \
    template int launch_conv_forward<T>(const ConvShape &, const ConvParams &, const ConvSeqs<T> &,            \
                                        cudaStream_t);                                                         \
    template int launch_conv_backward<T>(const ConvShape &, const ConvParams &, const ConvSeqs<T> &,           \
                                         cudaStream_t);                                                        \
    template int launch_conv_step<T>(const ConvShape &, const ConvParams &, const T *, int64_t,                \
                                     const uint8_t *, int64_t, const T *, T *, T *, int64_t, cudaStream_t);
SSM_INSTANTIATE(float)
SSM_INSTANTIATE(__nv_bfloat16)
SSM_INSTANTIATE(__half)

}  // namespace ssm_k
