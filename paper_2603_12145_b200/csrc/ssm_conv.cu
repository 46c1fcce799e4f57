// ssm_conv.cu -- the short causal convolution: sequence, gradients, single token.
//
// All three are bound by memory: a thread takes V neighbouring channels (one 8- or 16-byte
// access where sizes, strides and pointers allow, else one element) and walks a run of steps
// with the last width - 1 inputs in registers, so that each input is read once plus width - 1
// steps per run; the loads of the next steps are in flight while a step is computed.
// A reset clears the window, which drops every tap from before the episode.
//
// The backward kernel walks forward too: step t gives dpre_t, which goes into the pending
// gradients of x_t .. x_{t-width+1} (as far back as the episode reaches); the oldest one is
// then complete.  Its thread keeps its channels through all its runs, so dw and dbias stay in
// registers until the end; each thread's sums go to a row of their own and a second kernel adds
// the rows in a fixed order.
#include "ssm_kernels.cuh"

namespace ssm_k {
namespace {

constexpr int kThreads = 128;

template <typename T, int V>
struct alignas(sizeof(T) * V) Vec {
    T e[V];
};

template <typename T, int V>
__device__ __forceinline__ Vec<T, V> load_vec(const T *p)
{
    return *reinterpret_cast<const Vec<T, V> *>(p);
}

template <typename T, int V>
__device__ __forceinline__ Vec<T, V> zero_vec()
{
    Vec<T, V> v;
#pragma unroll
    for (int e = 0; e < V; ++e) v.e[e] = from_f32<T>(0.0f);
    return v;
}

// The window before step t0: win[j] = x[t0 - 1 - j], from the history before the sequence, zero
// where an episode starts between it and t0 - 1.
template <typename T, int V, int W>
__device__ __forceinline__ void load_window(float (&win)[W - 1][V], const ConvShape &s, const ConvSeqs<T> &q,
                                            int64_t b, int t0, int c)
{
    bool seen = true;
#pragma unroll
    for (int j = 0; j < W - 1; ++j) {
        const int t = t0 - 1 - j;
        Vec<T, V> v = zero_vec<T, V>();
        if (seen) {
            if (t >= 0)
                v = load_vec<T, V>(q.x.row(b, t) + c);
            else if (q.history != nullptr)
                v = load_vec<T, V>(q.history + (b * (W - 1) + (W - 1 + t)) * s.channels + c);
            if (q.reset.ptr != nullptr && t >= 0 && *q.reset.row(b, t) != 0) seen = false;
        }
#pragma unroll
        for (int e = 0; e < V; ++e) win[j][e] = to_f32(v.e[e]);
    }
}

template <typename T, int V, int W>
__global__ void __launch_bounds__(kThreads)
k_conv_forward(const ConvShape s, const ConvParams p, const ConvSeqs<T> q)
{
    constexpr int kTile = 8;
    const int vecs = s.channels / V;
    const int64_t i = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x;
    const int64_t unit = i / vecs;
    if (unit >= s.batch * s.runs) return;
    const int c = static_cast<int>(i - unit * vecs) * V;
    const int64_t b = unit / s.runs;
    const int t0 = static_cast<int>(unit - b * s.runs) * s.run;
    const int t1 = min(s.time, t0 + s.run);
    float w[W][V], bias[V], win[W - 1][V];
#pragma unroll
    for (int e = 0; e < V; ++e) {
#pragma unroll
        for (int k = 0; k < W; ++k) w[k][e] = p.w[static_cast<int64_t>(c + e) * W + k];
        bias[e] = p.bias != nullptr ? p.bias[c + e] : 0.0f;
    }
    load_window<T, V, W>(win, s, q, b, t0, c);
    for (int t = t0; t < t1; t += kTile) {
        Vec<T, V> x[kTile];
        uint8_t reset[kTile];
#pragma unroll
        for (int k = 0; k < kTile; ++k) {
            const bool in = t + k < t1;
            x[k] = in ? load_vec<T, V>(q.x.row(b, t + k) + c) : zero_vec<T, V>();
            reset[k] = in && q.reset.ptr != nullptr ? *q.reset.row(b, t + k) : 0;
        }
#pragma unroll
        for (int k = 0; k < kTile; ++k) {
            if (t + k >= t1) break;
            if (reset[k]) {
#pragma unroll
                for (int j = 0; j < W - 1; ++j)
#pragma unroll
                    for (int e = 0; e < V; ++e) win[j][e] = 0.0f;
            }
            Vec<T, V> out;
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const float xv = to_f32(x[k].e[e]);
                float u = bias[e];
#pragma unroll
                for (int j = W - 2; j >= 0; --j) u = fmaf(w[W - 2 - j][e], win[j][e], u);
                u = fmaf(w[W - 1][e], xv, u);
                out.e[e] = from_f32<T>(u * sigmoid(u));
#pragma unroll
                for (int j = W - 2; j > 0; --j) win[j][e] = win[j - 1][e];
                win[0][e] = xv;
            }
            *reinterpret_cast<Vec<T, V> *>(q.y.row(b, t + k) + c) = out;
        }
    }
    if (t1 == s.time && q.history_out != nullptr) {
#pragma unroll
        for (int j = 0; j < W - 1; ++j) {
            Vec<T, V> out;
#pragma unroll
            for (int e = 0; e < V; ++e) out.e[e] = from_f32<T>(win[j][e]);
            *reinterpret_cast<Vec<T, V> *>(q.history_out + (b * (W - 1) + (W - 2 - j)) * s.channels + c) = out;
        }
    }
}

template <typename T, int V, int W>
__global__ void __launch_bounds__(kThreads)
k_conv_backward(const ConvShape s, const ConvParams p, const ConvSeqs<T> q)
{
    constexpr int kTile = 8;
    const int vecs = s.channels / V;
    const int64_t i = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x;
    const int slot = static_cast<int>(i / vecs);
    if (slot >= s.slots) return;
    const int c = static_cast<int>(i - static_cast<int64_t>(slot) * vecs) * V;
    float w[W][V], bias[V], dw[W][V], dbias[V];
#pragma unroll
    for (int e = 0; e < V; ++e) {
#pragma unroll
        for (int k = 0; k < W; ++k) {
            w[k][e] = p.w[static_cast<int64_t>(c + e) * W + k];
            dw[k][e] = 0.0f;
        }
        bias[e] = p.bias != nullptr ? p.bias[c + e] : 0.0f;
        dbias[e] = 0.0f;
    }
    for (int64_t unit = slot; unit < s.batch * s.runs; unit += s.slots) {
        const int64_t b = unit / s.runs;
        const int t0 = static_cast<int>(unit - b * s.runs) * s.run;
        const int t1 = min(s.time, t0 + s.run);
        const int t2 = t1 + W - 1;        // the gradients of the run's last inputs come from the steps up to here
        float win[W - 1][V], pend[W][V];
        load_window<T, V, W>(win, s, q, b, t0, c);
#pragma unroll
        for (int j = 0; j < W; ++j)
#pragma unroll
            for (int e = 0; e < V; ++e) pend[j][e] = 0.0f;
        int age = W;                      // steps since the episode began, as far as the run's own inputs go
        for (int t = t0; t < t2; t += kTile) {
            Vec<T, V> x[kTile], dy[kTile];
            uint8_t reset[kTile];
#pragma unroll
            for (int k = 0; k < kTile; ++k) {
                const bool in = t + k < t2 && t + k < s.time;
                x[k] = in ? load_vec<T, V>(q.x.row(b, t + k) + c) : zero_vec<T, V>();
                dy[k] = in ? load_vec<T, V>(q.dy.row(b, t + k) + c) : zero_vec<T, V>();
                reset[k] = in && q.reset.ptr != nullptr ? *q.reset.row(b, t + k) : 0;
            }
#pragma unroll
            for (int k = 0; k < kTile; ++k) {
                if (t + k >= t2) break;
                age = reset[k] ? 0 : age + 1;
                const bool own = t + k < t1;
                const bool inside = t + k < s.time;
                Vec<T, V> out;
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    if (reset[k]) {
#pragma unroll
                        for (int j = 0; j < W - 1; ++j) win[j][e] = 0.0f;
                    }
                    const float xv = to_f32(x[k].e[e]);
                    float u = bias[e];
#pragma unroll
                    for (int j = W - 2; j >= 0; --j) u = fmaf(w[W - 2 - j][e], win[j][e], u);
                    u = fmaf(w[W - 1][e], xv, u);
                    const float sg = sigmoid(u);
                    // past the end of the sequence there is no step: not 0 * slope, which a NaN would survive
                    const float dpre = inside ? to_f32(dy[k].e[e]) * fmaf(u * sg, 1.0f - sg, sg) : 0.0f;
                    if (own) {
                        dbias[e] += dpre;
                        dw[W - 1][e] = fmaf(dpre, xv, dw[W - 1][e]);
#pragma unroll
                        for (int j = 0; j < W - 1; ++j) dw[W - 2 - j][e] = fmaf(dpre, win[j][e], dw[W - 2 - j][e]);
                    }
#pragma unroll
                    for (int j = W - 1; j > 0; --j)
                        pend[j][e] = age >= j ? fmaf(dpre, w[W - 1 - j][e], pend[j - 1][e]) : pend[j - 1][e];
                    pend[0][e] = dpre * w[W - 1][e];
                    out.e[e] = from_f32<T>(pend[W - 1][e]);
#pragma unroll
                    for (int j = W - 2; j > 0; --j) win[j][e] = win[j - 1][e];
                    win[0][e] = xv;
                }
                if (t + k - (W - 1) >= t0) *reinterpret_cast<Vec<T, V> *>(q.dx.row(b, t + k - (W - 1)) + c) = out;
            }
        }
    }
#pragma unroll
    for (int k = 0; k <= W; ++k) {
        Vec<float, V> out;
#pragma unroll
        for (int e = 0; e < V; ++e) out.e[e] = k < W ? dw[k < W ? k : 0][e] : dbias[e];
        *reinterpret_cast<Vec<float, V> *>(p.part + (static_cast<int64_t>(slot) * (W + 1) + k) * s.channels + c) = out;
    }
}

// Adds the slots' rows of one (tap, channel): a warp takes 32 neighbouring channels at a time,
// each of the block's eight warps every eighth row, and the eight sums are added in order.
__global__ void __launch_bounds__(256)
k_conv_params(const ConvShape s, const ConvParams p)
{
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
    Vec<T, V> out;
#pragma unroll
    for (int e = 0; e < V; ++e) {
        float u = p.bias != nullptr ? p.bias[c + e] : 0.0f;
#pragma unroll
        for (int k = 0; k < W; ++k) u = fmaf(p.w[static_cast<int64_t>(c + e) * W + k], to_f32(taps[k].e[e]), u);
        out.e[e] = from_f32<T>(u * sigmoid(u));
    }
    *reinterpret_cast<Vec<T, V> *>(y + row * y_stride + c) = out;
#pragma unroll
    for (int k = 0; k < W - 1; ++k) *reinterpret_cast<Vec<T, V> *>(dst + k * s.channels) = taps[k + 1];
}

unsigned blocks_for(int64_t threads) { return static_cast<unsigned>((threads + kThreads - 1) / kThreads); }

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
    constexpr int V = 8 / sizeof(T);
    if (s.channels % V == 0 && fits(q.x, V) && fits(q.y, V) && fits(q.history, 8) && fits(q.history_out, 8)) {
        const unsigned blocks = blocks_for(s.batch * s.runs * (s.channels / V));
        SSM_BY_WIDTH(k_conv_forward, T, V, blocks, s, p, q);
    } else {
        const unsigned blocks = blocks_for(s.batch * s.runs * s.channels);
        SSM_BY_WIDTH(k_conv_forward, T, 1, blocks, s, p, q);
    }
    return cudaGetLastError() == cudaSuccess ? 1 : -1;
}

template <typename T>
int launch_conv_backward(const ConvShape &s, const ConvParams &p, const ConvSeqs<T> &q, cudaStream_t stream)
{
    constexpr int V = 8 / sizeof(T);
    if (s.channels % V == 0 && fits(q.x, V) && fits(q.dy, V) && fits(q.dx, V) && fits(q.history, 8)) {
        const unsigned blocks = blocks_for(static_cast<int64_t>(s.slots) * (s.channels / V));
        SSM_BY_WIDTH(k_conv_backward, T, V, blocks, s, p, q);
    } else {
        const unsigned blocks = blocks_for(static_cast<int64_t>(s.slots) * s.channels);
        SSM_BY_WIDTH(k_conv_backward, T, 1, blocks, s, p, q);
    }
    const dim3 grid(static_cast<unsigned>((s.channels + 31) / 32), static_cast<unsigned>(s.width + 1));
    k_conv_params<<<grid, 256, 0, stream>>>(s, p);
    return cudaGetLastError() == cudaSuccess ? 2 : -1;
}

template <typename T>
int launch_conv_step(const ConvShape &s, const ConvParams &p, const T *x, int64_t x_stride, const uint8_t *done,
                     int64_t done_stride, const T *history, T *history_out, T *y, int64_t y_stride,
                     cudaStream_t stream)
{
    constexpr int V = 8 / sizeof(T);
    if (s.channels % V == 0 && x_stride % V == 0 && y_stride % V == 0 && fits(x, 8) && fits(y, 8) &&
        fits(history, 8) && fits(history_out, 8)) {
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
