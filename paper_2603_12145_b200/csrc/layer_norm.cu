// layer_norm.cu -- the layer norm of a residual stream behind the C ABI of layer_norm.h.
//
// A row stays in the registers of the threads that share it, as the words it was loaded in: the sum, the mean, the
// variance (from differences to the mean) and the result come from one reading of memory.  A row of up to 96 vectors of
// 16 bytes (binary32: 128) belongs to 4 to 32 lanes of a warp, which reduce by shuffles; a wider one to a block, whose warps
// exchange their sums through shared memory with one barrier per reduction (two alternating slots).  Of R threads each holds
// the vectors index, index + R, ..., so that a warp's access is contiguous.  Blocks go through several rows, as many as fit on
// the device at once, and the next row's loads are in flight while a row is reduced.  Rows that do not begin on boundaries of
// 16 bytes are read between these or by single elements (offered()).
//
// The backward kernel keeps dw and db of its thread's columns in registers over all its rows: per row only the two sums of dx
// cross threads.  The row groups of a warp are added by exchanges, a block's warps in shared memory, blocks leave a row of
// sums each and k_join adds them, all in a fixed order.
//
// What bounds them: memory, and issue close behind it.  In bfloat16 on a B200, 65,536 x 576 with residual takes 52 us forward
// (302 MB, 5.8 TB/s) and 55 us backward (5.5 TB/s), 8,192 x 8,192 without takes 51 us (5.2 TB/s) and 89 us (4.5 TB/s: one
// block per SM, which waits for its row's sums); 64 rows take 5 us on the device, less than the call on the host.
#include <cmath>
#include <new>
#include <type_traits>

#include "../../include/layer_norm.h"
#include "on_device.cuh"
#include "vectors.cuh"

namespace {

using namespace vals;

// Who shares a row: lanes of a warp, a block of up to 256 threads, a block of kMost.
enum Form { kLanes, kBlock, kLargest };
// How a row lies in its threads' accesses: some have none in the last round, all have all, or the row begins and ends inside an
// access (kShifted: at any alignment that all arrays share; the rows of a thread are a multiple of a vector's elements apart, so that
// all begin alike and its columns stay the same).
enum Fit { kSome, kAll, kShifted };
constexpr int kNarrowThreads = 128;      // block of the kernels whose rows belong to lanes of a warp
constexpr int kMost = 512;               // threads that share a wide row, at most

__device__ __forceinline__ void allow_next() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void wait_for_previous() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

template <typename T>
struct Rows {
    T *ptr;
    int64_t stride;
    __device__ __forceinline__ T *row(int64_t i) const { return ptr + i * stride; }
};

template <typename T>
struct Forward {
    Rows<const T> x, residual;
    Rows<T> sum, y;
    const float *w, *b;
    float2 *saved;
    int64_t n;
    int width, lanes;
    int shift, turn;         // kShifted: elements from a boundary to the first row, and from row to row, modulo a vector
    float eps;
};

template <typename T>
struct Backward {
    Rows<const T> dy, s, dsum;
    Rows<T> dx;
    const float *w;
    const float2 *saved;
    float *part;             // [blocks][2][width], or nullptr: no dw, db
    int64_t n;
    int width, lanes;
    int shift, turn;
};

// Sums over the threads that share a row: R lanes, or the block.
template <bool kWide>
struct Team {
    int size, index;         // threads of the row, and which of them this is
    int slot = 0;
    float2 *shared;          // [2][kMost / 32]

    __device__ float2 total(float2 v)
    {
        if (kWide) {
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) {
                v.x += __shfl_xor_sync(0xFFFFFFFFu, v.x, o);
                v.y += __shfl_xor_sync(0xFFFFFFFFu, v.y, o);
            }
            float2 *s = shared + slot * (kMost / 32);
            slot ^= 1;
            const int lane = index & 31, warps = size >> 5;
            if (lane == 0) s[index >> 5] = v;
            __syncthreads();
            v = s[lane & (warps - 1)];               // (their number is a power of two)
            for (int o = warps >> 1; o > 0; o >>= 1) {
                v.x += __shfl_xor_sync(0xFFFFFFFFu, v.x, o);
                v.y += __shfl_xor_sync(0xFFFFFFFFu, v.y, o);
            }
        } else {
            for (int o = size >> 1; o > 0; o >>= 1) {
                v.x += __shfl_xor_sync(0xFFFFFFFFu, v.x, o);
                v.y += __shfl_xor_sync(0xFFFFFFFFu, v.y, o);
            }
        }
        return v;
    }
    __device__ float total(float v)
    {
        if constexpr (kWide) {
            return total(make_float2(v, 0.0f)).x;
        } else {
            for (int o = size >> 1; o > 0; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
            return v;
        }
    }
    __device__ void totals(float2 (&v)[1]) { v[0] = total(v[0]); }
    __device__ void totals(float2 (&v)[2])              // (lanes of a warp)
    {
        for (int o = size >> 1; o > 0; o >>= 1) {
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                v[r].x += __shfl_xor_sync(0xFFFFFFFFu, v[r].x, o);
                v[r].y += __shfl_xor_sync(0xFFFFFFFFu, v[r].y, o);
            }
        }
    }
    __device__ void totals(float (&v)[1]) { v[0] = total(v[0]); }
    __device__ void totals(float (&v)[2])
    {
        const float2 t = total(make_float2(v[0], v[1]));
        v[0] = t.x;
        v[1] = t.y;
    }
};

// Rows that a thread shares at a time, forward: two of few 16-bit elements, which are bound by arithmetic and exchanges, for one
// round of these and the parameters read once (bfloat16 without residual: 8,192 x 8,192 51 against 70 us, 65,536 x 256
// 12.4 against 14.4, x 576 30 against 34; binary32 is near memory's rate with one, 65,536 x 512 46 and 47 us).  24 elements only
// where no access is masked and no barrier waits: x 768 41 against 43, but x 696 43 against 40, 32,768 x 1,032 43 against 33.
template <typename T, int V, int C, int R, Form kForm, Fit kFit>
constexpr int kRowsOf = sizeof(T) == 2 && V > 1 && kFit != kShifted && C * V + R <= (kForm == kLanes && kFit == kAll ? 24 : 20) ? 2 : 1;
// Backward by lanes of a warp likewise (65,536 x 576 with dsum 55.5 against 59.4 us, x 256 24.6 against 26.7); a block's threads
// have no registers for it.
template <typename T, int V, int C, int R, Form kForm, Fit kFit>
constexpr int kBackwardRowsOf = kForm == kLanes ? kRowsOf<T, V, C, R, kForm, kFit> : 1;

// Units of one or two neighbouring parameters (from L1: every row reads them)
template <int W, int N>
__device__ __forceinline__ void load_params(Vals<W> (&dst)[N], const float *src, float absent)
{
    if (src == nullptr) {
#pragma unroll
        for (int i = 0; i < N; ++i) dst[i] = all<W>(absent);
    } else if constexpr (W == 1) {
        dst[0] = __ldg(src);
    } else if constexpr (N == 1) {
        const float2 f = __ldg(reinterpret_cast<const float2 *>(src));
        dst[0] = pair(f.x, f.y);
    } else {
#pragma unroll
        for (int i = 0; i < N; i += 2) {
            const float4 f = __ldg(reinterpret_cast<const float4 *>(src + 2 * i));
            dst[i] = pair(f.x, f.y);
            dst[i + 1] = pair(f.z, f.w);
        }
    }
}

__device__ __forceinline__ void store_unit(float *dst, float v) { *dst = v; }
__device__ __forceinline__ void store_unit(float *dst, Pair v) { *reinterpret_cast<float2 *>(dst) = make_float2(lo(v), hi(v)); }

// A thread's share of a row: C accesses of V elements, index, index + size, ... of the row's `vectors`, and R elements of the rest
// behind C * size vectors.
template <typename T, int V, int C, int R, Fit kFit>
struct Mine {
    static constexpr int W = V == 1 ? 1 : 2, N = (V + 1) / 2, kUnits = C * N + R / 2;
    using Unit = Vals<W>;

    struct Words {                       // as they lie in memory
        Packed<T, V> v[C];
        Packed<T, R == 0 ? V : R> rest;
        __device__ __forceinline__ Unit get(int u) const
        {
            if constexpr (R > 0)
                if (u >= C * N) return widen_at(rest, u - C * N);
            return widen_at(v[u / N], u % N);
        }
        __device__ __forceinline__ void set(int u, Unit f)
        {
            if constexpr (R > 0) {
                if (u >= C * N) {
                    narrow_at(rest, u - C * N, f);
                    return;
                }
            }
            narrow_at(v[u / N], u % N, f);
        }
    };

    int size, index, vectors;
    int shift, width;                    // (kShifted)

    // The share of the rows that begin `first`, `first` + a multiple of V, ... rows behind the first one.
    template <typename P>
    static __device__ __forceinline__ Mine of(int size, int index, const P &p, int64_t first)
    {
        if (kFit != kShifted) return {size, index, p.width / V, 0, p.width};
        const int shift = (p.shift + static_cast<int>(first % V) * p.turn) % V;
        return {size, index, (shift + p.width + V - 1) / V, shift, p.width};
    }
    // The access that begins with element `at` has elements [from, to) of the row.
    __device__ __forceinline__ int from(int at) const { return kFit == kShifted ? max(0, -at) : 0; }
    __device__ __forceinline__ int to(int at) const { return kFit == kShifted ? min(V, width - at) : V; }
    __device__ __forceinline__ bool partial(int at) const { return kFit == kShifted && (at < 0 || at + V > width); }

    // f(first unit, how many, the element that they begin with, whether they are there) for each access
    template <typename F>
    __device__ __forceinline__ void each_access(F f) const
    {
#pragma unroll
        for (int c = 0; c < C; ++c)
            f(c * N, std::integral_constant<int, N>{}, (c * size + index) * V - (kFit == kShifted ? shift : 0), kFit == kAll || c * size + index < vectors);
        if constexpr (R > 0) f(C * N, std::integral_constant<int, R / 2>{}, C * size * V + index * R, true);
    }
    // Zeros where there is nothing.  kShifted: what lies beside the row comes along until trim(), but not of the first and the
    // last row (`outer`), where it may be outside the array.
    __device__ __forceinline__ Words load(const T *row, bool outer) const
    {
        Words w;
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int i = c * size + index, at = i * V - (kFit == kShifted ? shift : 0);
            if (kFit != kAll && i >= vectors) w.v[c] = packed_zero<T, V>();
            else w.v[c] = one_access(row, at, outer);
        }
        if constexpr (R > 0) w.rest = packed_load<T, R>(row + C * size * V + index * R);
        return w;
    }
    __device__ __forceinline__ Packed<T, V> one_access(const T *row, int at, bool outer) const
    {
        if constexpr (kFit == kShifted)
            if (outer && partial(at)) return packed_load_part<T, V>(row + at, from(at), to(at));
        return packed_load<T, V>(row + at);
    }
    __device__ __forceinline__ void trim(Words &w) const
    {
        if constexpr (kFit == kShifted) {
#pragma unroll
            for (int c = 0; c < C; ++c) {
                const int at = (c * size + index) * V - shift;
                if (partial(at)) packed_trim<T, V>(w.v[c], from(at), to(at));
            }
        }
    }
    __device__ __forceinline__ void store(T *row, const Words &w) const
    {
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int i = c * size + index, at = i * V - (kFit == kShifted ? shift : 0);
            if (kFit == kAll || i < vectors) store_access(row, at, w.v[c]);
        }
        if constexpr (R > 0) packed_store<T, R>(row + C * size * V + index * R, w.rest);
    }
    template <int E>
    __device__ __forceinline__ void store_access(T *row, int at, const Packed<T, E> &v) const
    {
        if constexpr (kFit == kShifted)
            if (partial(at)) return packed_store_part<T, V>(row + at, v, from(at), to(at));
        packed_store<T, E>(row + at, v);
    }
    // Units of parameters that stay in registers: `absent` where there are none.
    template <int E>
    __device__ __forceinline__ void params(Unit (&dst)[E], const float *src, int at, bool in, float absent) const
    {
        if constexpr (kFit == kShifted) {
#pragma unroll
            for (int i = 0; i < E; ++i) {
                auto one = [&](int e) { return src != nullptr && in && e >= 0 && e < width ? __ldg(src + e) : absent; };
                dst[i] = pair(one(at + 2 * i), one(at + 2 * i + 1));
            }
        } else {
            load_params<W>(dst, src != nullptr && in ? src + at : nullptr, absent);
        }
    }
};

// Rows of this warp or block, one after the other.
struct Turns {
    int64_t first, step;
    int behind;              // which of the warp's rows this lane has: all go round while the first of them is there
    template <bool kWide>
    static __device__ __forceinline__ Turns of(int lanes, int rows = 1)
    {
        const int per_block = kWide ? rows : kNarrowThreads / lanes * rows;
        return {static_cast<int64_t>(blockIdx.x) * per_block + (kWide ? 0 : static_cast<int>(threadIdx.x) / lanes * rows),
                static_cast<int64_t>(gridDim.x) * per_block, kWide ? 0 : static_cast<int>(threadIdx.x & 31) / lanes * rows};
    }
};

template <typename T, int V, int C, int R, Form kForm, Fit kFit>
__global__ void __launch_bounds__(kForm == kLargest ? kMost : kForm == kBlock ? kMost / 2 : kNarrowThreads)
k_forward(const Forward<T> p)
{
    constexpr bool kWide = kForm != kLanes;
    using M = Mine<T, V, C, R, kFit>;
    using U = typename M::Unit;
    constexpr int W = M::W;
    __shared__ float2 s_sum[kWide ? 2 * (kMost / 32) : 1];
    Team<kWide> team;
    team.size = kWide ? static_cast<int>(blockDim.x) : p.lanes;
    team.index = static_cast<int>(threadIdx.x) & (team.size - 1);
    team.shared = s_sum;
    constexpr int kRows = kRowsOf<T, V, C, R, kForm, kFit>;
    const Turns turns = Turns::of<kWide>(p.lanes, kRows);
    const M mine = M::of(team.size, team.index, p, turns.first);
    const float inverse = 1.0f / static_cast<float>(p.width);
    const bool added = p.residual.ptr != nullptr;
    typename M::Words nx[kRows] = {}, nr[kRows] = {};
    auto fetch = [&](int64_t first) {        // behind the last row that one again: no zeros to be put in place
#pragma unroll
        for (int r = 0; r < kRows; ++r) {
            if (kFit == kShifted && first + r >= p.n) return;          // (that one may lie otherwise)
            const int64_t row = first + r < p.n ? first + r : p.n - 1;
            const bool outer = row == 0 || row + 1 == p.n;
            nx[r] = mine.load(p.x.row(row), outer);
            if (added) nr[r] = mine.load(p.residual.row(row), outer);
        }
    };
    fetch(turns.first);
    // The parameters stay in registers where there is room (bfloat16, no residual: 65,536 x 256 14.7 against 18.7 us, 32,768 x 1,032 33
    // against 41; of single elements 65,536 x 577 120 against 157); blocks that share a binary32 row lose warps by it (8,192 x 4,096
    // 51 against 49).
    constexpr bool kHeld = V == 1 ? C <= 8 : C * V + R <= (sizeof(T) == 2 ? 24 : kWide ? 0 : 18);
    U held_w[kHeld ? M::kUnits : 1], held_b[kHeld ? M::kUnits : 1];
    if constexpr (kHeld) {
        mine.each_access([&](int u0, auto n, int at, bool in) {
            U w[n.value], b[n.value];
            mine.params(w, p.w, at, in, 1.0f);
            mine.params(b, p.b, at, in, 0.0f);
#pragma unroll
            for (int i = 0; i < n.value; ++i) {
                held_w[u0 + i] = w[i];
                held_b[u0 + i] = b[i];
            }
        });
    }
    for (int64_t row = turns.first; row - turns.behind < p.n; row += turns.step) {
        U s[kRows][M::kUnits];
        float mean[kRows], scale[kRows];
#pragma unroll
        for (int r = 0; r < kRows; ++r) {
            if (added) {
#pragma unroll
                for (int u = 0; u < M::kUnits; ++u) nx[r].set(u, add(nx[r].get(u), nr[r].get(u)));     // rounded to the type
                if (row + r < p.n) mine.store(p.sum.row(row + r), nx[r]);
            }
            mine.trim(nx[r]);
            U sum = all<W>(0.0f);
#pragma unroll
            for (int u = 0; u < M::kUnits; ++u) {
                s[r][u] = nx[r].get(u);
                sum = add(sum, s[r][u]);
            }
            mean[r] = sum_of(sum);
        }
        fetch(row + turns.step);
        team.totals(mean);
#pragma unroll
        for (int r = 0; r < kRows; ++r) {
            mean[r] *= inverse;
            U square = all<W>(0.0f);
            mine.each_access([&](int u0, auto n, int at, bool in) {
                if (!in) return;
#pragma unroll
                for (int i = 0; i < n.value; ++i) s[r][u0 + i] = add(s[r][u0 + i], all<W>(-mean[r]));
                if (mine.partial(at)) {                  // (nothing beside the row)
                    const int from = mine.from(at), to = mine.to(at);
                    if constexpr (kFit == kShifted) {
#pragma unroll
                        for (int i = 0; i < n.value; ++i)
                            s[r][u0 + i] = pair(2 * i >= from && 2 * i < to ? lo(s[r][u0 + i]) : 0.0f, 2 * i + 1 >= from && 2 * i + 1 < to ? hi(s[r][u0 + i]) : 0.0f);
                    }
                }
#pragma unroll
                for (int i = 0; i < n.value; ++i) square = fma(s[r][u0 + i], s[r][u0 + i], square);
            });
            scale[r] = sum_of(square);
        }
        team.totals(scale);
#pragma unroll
        for (int r = 0; r < kRows; ++r) {
            scale[r] = rsqrtf(fmaf(scale[r], inverse, p.eps));
            if (row + r >= p.n) continue;
            if (p.saved != nullptr && team.index == 0) p.saved[row + r] = make_float2(mean[r], scale[r]);
            T *const py = p.y.row(row + r);
            mine.each_access([&](int u0, auto n, int at, bool in) {
                if (!in) return;
                Packed<T, W * n.value> out;
                U w[n.value], b[n.value];
                if constexpr (kHeld) {
#pragma unroll
                    for (int i = 0; i < n.value; ++i) {
                        w[i] = held_w[u0 + i];
                        b[i] = held_b[u0 + i];
                    }
                } else {
                    load_params<W>(w, p.w != nullptr ? p.w + at : nullptr, 1.0f);
                    load_params<W>(b, p.b != nullptr ? p.b + at : nullptr, 0.0f);
                }
#pragma unroll
                for (int i = 0; i < n.value; ++i) narrow_at(out, i, fma(mul(s[r][u0 + i], all<W>(scale[r])), w[i], b[i]));
                mine.store_access(py, at, out);
            });
        }
    }
}

template <typename T, int V, int C, int R, Form kForm, Fit kFit>
__global__ void __launch_bounds__(kForm == kLanes || (V == 8 && C == 3) ? kNarrowThreads : kForm == kBlock ? kMost / 2 : kMost)
k_backward(const Backward<T> p)
{
    constexpr bool kWide = kForm != kLanes;
    using M = Mine<T, V, C, R, kFit>;
    using U = typename M::Unit;
    constexpr int W = M::W;
    extern __shared__ float s_part[];                      // narrow rows: [warps][2][width], the sums of a warp's row groups
    __shared__ float2 s_sum[kWide ? 2 * (kMost / 32) : 1];
    allow_next();
    Team<kWide> team;
    team.size = kWide ? static_cast<int>(blockDim.x) : p.lanes;
    team.index = static_cast<int>(threadIdx.x) & (team.size - 1);
    team.shared = s_sum;
    constexpr int kRows = kBackwardRowsOf<T, V, C, R, kForm, kFit>;
    const Turns turns = Turns::of<kWide>(p.lanes, kRows);
    const M mine = M::of(team.size, team.index, p, turns.first);
    const float inverse = 1.0f / static_cast<float>(p.width);
    const bool added = p.dsum.ptr != nullptr;
    U dw[M::kUnits], db[M::kUnits];
#pragma unroll
    for (int u = 0; u < M::kUnits; ++u) dw[u] = db[u] = all<W>(0.0f);
    typename M::Words ns[kRows] = {}, ndy[kRows] = {}, nd[kRows] = {};
    float2 nstat[kRows] = {};
    auto fetch = [&](int64_t first) {
#pragma unroll
        for (int r = 0; r < kRows; ++r) {
            if (kFit == kShifted && first + r >= p.n) return;
            const int64_t row = first + r < p.n ? first + r : p.n - 1;
            nstat[r] = __ldg(p.saved + row);
            const bool outer = row == 0 || row + 1 == p.n;
            ns[r] = mine.load(p.s.row(row), outer);
            ndy[r] = mine.load(p.dy.row(row), outer);
            if (added) nd[r] = mine.load(p.dsum.row(row), outer);
        }
    };
    fetch(turns.first);
    // The weights take a third of the accesses if every row fetches them: in registers where there is room, that is, not in
    // blocks for rows of binary32 (bfloat16: 65,536 x 576 61 against 73 us, 8,192 x 8,192 98 against 131; binary32: 32,768 x 512
    // 49 against 54, but 16,384 x 1,024 75 against 67; single elements: 16,384 x 1,003 64 against 81.)
    constexpr bool kHeld = V == 1 ? C <= 8 : sizeof(T) == 2 || !kWide;
    U held[kHeld ? M::kUnits : 1];
    if constexpr (kHeld) {
        mine.each_access([&](int u0, auto n, int at, bool in) {
            U w[n.value];
            mine.params(w, p.w, at, in, 1.0f);
#pragma unroll
            for (int i = 0; i < n.value; ++i) held[u0 + i] = w[i];
        });
    }
    auto weights = [&](auto &w, int u0, int at) {
        if constexpr (kHeld) {
#pragma unroll
            for (int i = 0; i < static_cast<int>(sizeof(w) / sizeof(w[0])); ++i) w[i] = held[u0 + i];
        } else {
            load_params<W>(w, p.w != nullptr ? p.w + at : nullptr, 1.0f);
        }
    };
    for (int64_t row = turns.first; row - turns.behind < p.n; row += turns.step) {
        typename M::Words s[kRows], dy[kRows], d[kRows];
        float mean[kRows], scale[kRows];
        float2 sums[kRows];
#pragma unroll
        for (int r = 0; r < kRows; ++r) {
            s[r] = ns[r];
            dy[r] = ndy[r];
            d[r] = nd[r];
            mine.trim(s[r]);
            mine.trim(dy[r]);
            mean[r] = nstat[r].x;
            scale[r] = nstat[r].y;
        }
        fetch(row + turns.step);
#pragma unroll
        for (int r = 0; r < kRows; ++r) {
            const bool live = row + r < p.n;
            U sum = all<W>(0.0f), along = sum;
            mine.each_access([&](int u0, auto n, int at, bool in) {
                if (!in || !live) return;
                U w[n.value];
                weights(w, u0, at);
#pragma unroll
                for (int i = 0; i < n.value; ++i) {
                    const int u = u0 + i;
                    const U z = mul(add(s[r].get(u), all<W>(-mean[r])), all<W>(scale[r])), g = dy[r].get(u), h = mul(g, w[i]);
                    sum = add(sum, h);
                    along = fma(h, z, along);
                    dw[u] = fma(g, z, dw[u]);
                    db[u] = add(db[u], g);
                }
            });
            sums[r] = make_float2(sum_of(sum), sum_of(along));
        }
        team.totals(sums);
#pragma unroll
        for (int r = 0; r < kRows; ++r) {
            if (row + r >= p.n) continue;
            const U slope = all<W>(-scale[r] * sums[r].y * inverse), shift = all<W>(-scale[r] * sums[r].x * inverse);
            T *const px = p.dx.row(row + r);
            mine.each_access([&](int u0, auto n, int at, bool in) {
                if (!in) return;
                Packed<T, W * n.value> out;
                U w[n.value];
                weights(w, u0, at);
#pragma unroll
                for (int i = 0; i < n.value; ++i) {
                    const int u = u0 + i;
                    const U z = mul(add(s[r].get(u), all<W>(-mean[r])), all<W>(scale[r]));
                    U x = fma(mul(dy[r].get(u), w[i]), all<W>(scale[r]), fma(z, slope, shift));
                    if (added) x = add(x, d[r].get(u));
                    narrow_at(out, i, x);
                }
                mine.store_access(px, at, out);
            });
        }
    }
    if (p.part == nullptr) return;
    float *part = p.part + static_cast<int64_t>(blockIdx.x) * 2 * p.width;
    auto leave = [&](float *to) {
        mine.each_access([&](int u0, auto n, int at, bool in) {
            if (!in) return;
#pragma unroll
            for (int i = 0; i < n.value; ++i) {
                if constexpr (kFit == kShifted) {
                    auto one = [&](int e, float w, float b) {
                        if (e < 0 || e >= p.width) return;
                        to[e] = w;
                        to[p.width + e] = b;
                    };
                    one(at + 2 * i, lo(dw[u0 + i]), lo(db[u0 + i]));
                    one(at + 2 * i + 1, hi(dw[u0 + i]), hi(db[u0 + i]));
                } else {
                    store_unit(to + at + W * i, dw[u0 + i]);
                    store_unit(to + p.width + at + W * i, db[u0 + i]);
                }
            }
        });
    };
    if constexpr (kWide) {
        leave(part);
    } else {
        // a warp's row groups by exchanges (kShifted: it has one), the warps one after the other
        const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
        for (int o = 16; o >= team.size; o >>= 1) {
#pragma unroll
            for (int u = 0; u < M::kUnits; ++u) {
                dw[u] = each([&](float x) { return x + __shfl_xor_sync(0xFFFFFFFFu, x, o); }, dw[u]);
                db[u] = each([&](float x) { return x + __shfl_xor_sync(0xFFFFFFFFu, x, o); }, db[u]);
            }
        }
        if (lane < team.size) leave(s_part + warp * 2 * p.width);
        __syncthreads();
        for (int i = threadIdx.x; i < 2 * p.width; i += kNarrowThreads) {
            float sum = s_part[i];
#pragma unroll
            for (int w = 1; w < kNarrowThreads / 32; ++w) sum += s_part[w * 2 * p.width + i];
            part[i] = sum;
        }
    }
}

// dw and db: a block takes 32 columns of the `rows` rows of sums, its warps share the rows.
constexpr int kJoinWarps = 32;

__global__ void __launch_bounds__(32 * kJoinWarps)
k_join(const float *part, int rows, int width, float *dw, float *db)
{
    __shared__ float s[kJoinWarps][32];
    wait_for_previous();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int column = blockIdx.x * 32 + lane;
    float sum = 0.0f;
    if (column < 2 * width) {
        const float *at = part + column;
#pragma unroll 8
        for (int r = warp; r < rows; r += kJoinWarps) sum += at[static_cast<int64_t>(r) * 2 * width];
    }
    s[warp][lane] = sum;
    __syncthreads();
    if (warp != 0 || column >= 2 * width) return;
#pragma unroll
    for (int i = 1; i < kJoinWarps; ++i) sum += s[i][lane];
    if (column < width)
        dw[column] = sum;
    else
        db[column - width] = sum;
}

// ---------------------------------------------------------------- host side

int64_t div_up(int64_t a, int64_t b) { return (a + b - 1) / b; }

bool aligned(const void *ptr, size_t bytes) { return reinterpret_cast<uintptr_t>(ptr) % bytes == 0; }

// How a row is shared: `lanes` threads with C accesses each.
struct Share {
    int lanes, count;
    bool wide;
    int rest;                // elements per lane behind `count` whole rounds of a warp's accesses
};

// Vectors of 16 bytes: up to three (of four elements four) per lane of a warp; then, per thread of a block, up to two of eight
// elements (three in blocks of up to 128 threads, which have the registers) or four of four.  Single elements: up to 8 per
// lane, then up to 8 (16 in the largest blocks).  Measured in bfloat16: 32,768 x 1,024 backward 57 us as blocks of 64
// threads, 74 us as a warp with four vectors per lane.
Share share_of(int vectors, int V, bool with_rest)
{
    Share s = {4, 1, false, 0};
    while (s.lanes < 32 && s.lanes * (V > 1 ? 2 : 4) < vectors) s.lanes *= 2;
    if (vectors > s.lanes * (V == 1 ? 8 : V == 4 ? 4 : 3)) {
        s.wide = true;
        s.lanes = 64;
        while (s.lanes < kMost && s.lanes * (V == 1 ? 8 : V == 4 ? 4 : s.lanes <= kNarrowThreads ? 3 : 2) < vectors) s.lanes *= 2;
    }
    s.count = static_cast<int>(div_up(vectors, s.lanes));
    // a warp's last round would leave three or two of four lanes without work: the rest of 64 or 128 elements by twos or fours
    // (65,536 x 576 in bfloat16: 126 against 142 us forward and backward)
    if (with_rest && V == 8 && !s.wide && vectors > 32 && (vectors % 32 == 8 || vectors % 32 == 16)) {
        s.count = vectors / 32;
        s.rest = vectors % 32 / 4;
    }
    return s;
}
static_assert(kMost * 16 >= LAYER_NORM_MAX_WIDTH && kMost * 2 * 8 >= LAYER_NORM_MAX_WIDTH && kMost * 4 * 4 >= LAYER_NORM_MAX_WIDTH,
              "the widest row: single elements, vectors of 8, vectors of 4");

template <int N>
using Count = std::integral_constant<int, N>;

template <Form kForm>
using Of = std::integral_constant<Form, kForm>;
template <Fit kFit>
using As = std::integral_constant<Fit, kFit>;

// The accesses that a call's arrays allow: single elements, vectors of 16 bytes on their boundaries, or vectors on boundaries that the
// rows begin and end between.
enum Access { kSingle, kWhole, kBetween, kAccesses };

// Calls f with V, C, R, the form of the kernel and how rows fit for this share of a row of `vectors`.  (kAll instead of kSome: bfloat16,
// 16,384 x 4,096 backward 97 against 104 us.)
template <typename T, typename F>
bool with_counts(const Share &s, int vectors, Access access, F f)
{
    using V = Count<16 / sizeof(T)>;
    using One = Count<1>;
    using None = Count<0>;
    using No = As<kSome>;
    using Yes = As<kAll>;
    const bool largest = s.lanes == kMost;
    if (access == kSingle) {
        if (!s.wide) return s.count <= 4 ? f(One{}, Count<4>{}, None{}, Of<kLanes>{}, No{}) : f(One{}, Count<8>{}, None{}, Of<kLanes>{}, No{});
        if (s.count > 8) return f(One{}, Count<16>{}, None{}, Of<kLargest>{}, No{});
        return largest ? f(One{}, Count<8>{}, None{}, Of<kLargest>{}, No{}) : f(One{}, Count<8>{}, None{}, Of<kBlock>{}, No{});
    }
    if constexpr (sizeof(T) == 2) {
        auto with_rest = [&](auto c) { return s.rest == 2 ? f(V{}, c, Count<2>{}, Of<kLanes>{}, Yes{}) : f(V{}, c, Count<4>{}, Of<kLanes>{}, Yes{}); };
        if (s.rest > 0) return s.count == 1 ? with_rest(Count<1>{}) : with_rest(Count<2>{});
    }
    auto with_count = [&](auto all) {
        if (s.wide) {
            if constexpr (sizeof(T) == 4) {
                if (s.count <= 3) return largest ? f(V{}, Count<3>{}, None{}, Of<kLargest>{}, all) : f(V{}, Count<3>{}, None{}, Of<kBlock>{}, all);
                return largest ? f(V{}, Count<4>{}, None{}, Of<kLargest>{}, all) : f(V{}, Count<4>{}, None{}, Of<kBlock>{}, all);
            } else {
                if (s.count == 3) return f(V{}, Count<3>{}, None{}, Of<kBlock>{}, all);
                return largest ? f(V{}, Count<2>{}, None{}, Of<kLargest>{}, all) : f(V{}, Count<2>{}, None{}, Of<kBlock>{}, all);
            }
        }
        if constexpr (sizeof(T) == 4)
            if (s.count == 4) return f(V{}, Count<4>{}, None{}, Of<kLanes>{}, all);
        if (s.count <= 1) return f(V{}, Count<1>{}, None{}, Of<kLanes>{}, all);
        return s.count == 2 ? f(V{}, Count<2>{}, None{}, Of<kLanes>{}, all) : f(V{}, Count<3>{}, None{}, Of<kLanes>{}, all);
    };
    if constexpr (sizeof(T) == 2) {                      // (offered(): by whole warps and small blocks)
        auto between = [&](auto form) {
            return s.count <= 2 ? f(V{}, Count<2>{}, None{}, form, As<kShifted>{}) : f(V{}, Count<3>{}, None{}, form, As<kShifted>{});
        };
        if (access == kBetween) return s.wide ? between(Of<kBlock>{}) : between(Of<kLanes>{});
    }
    return vectors == s.lanes * s.count ? with_count(Yes{}) : with_count(No{});
}

int element_bytes(int type) { return type == LAYER_NORM_F32 ? 4 : 2; }

}  // namespace

struct layer_norm {
    int width = 0, type = 0;
    float eps = 0.0f;
    int device = 0, sms = 0;
    int forward_blocks[kAccesses] = {}, backward_blocks[kAccesses] = {};     // that an SM holds; none where rows are not read this way
    int backward_rows[kAccesses] = {};       // that a thread takes at a time
    cudaStream_t stream = nullptr;
    int64_t launches = 0;
};

namespace {

int vectors_of(const layer_norm *p, Access access)
{
    const int V = 16 / element_bytes(p->type);
    return access == kSingle ? p->width : access == kWhole ? p->width / V : (p->width + 2 * (V - 1)) / V;
}

Share share_for(const layer_norm *p, Access access)
{
    return share_of(vectors_of(p, access), access == kSingle ? 1 : 16 / element_bytes(p->type), access == kWhole);
}

// Whether rows of this width are read this way at all.  Between boundaries 16-bit rows of 257 to about 3,000 elements (65,536 x 577
// in bfloat16 with residual 95 against 186 us forward, 127 against 223 backward; 32,768 x 1,501 81 and 111 against 198 and 236):
// shorter ones are as fast by single elements (x 255 71 and 72 against 62 and 74), the backward pass of larger
// blocks is slower (16,384 x 4,001 399 against 264), binary32 too (65,536 x 255 66 and 80 against 61 and 66).
bool offered(const layer_norm *p, Access access)
{
    if (access == kWhole) return p->width % (16 / element_bytes(p->type)) == 0;
    return access == kSingle || (p->type != LAYER_NORM_F32 && p->width > 256 && share_for(p, access).lanes <= kNarrowThreads);
}

size_t backward_smem(const layer_norm *p, const Share &s) { return s.wide ? 0 : kNarrowThreads / 32 * 2 * sizeof(float) * p->width; }

// Whole rounds of resident blocks, so that all end together.  Between boundaries, the rows of a thread begin alike: as many blocks as
// make its rows whole vectors' elements apart, unless it has one row.
int64_t blocks_for(const layer_norm *p, Access access, int64_t n, int per_sm, int rows)
{
    const Share s = share_for(p, access);
    const int64_t per_block = static_cast<int64_t>(s.wide ? 1 : kNarrowThreads / s.lanes) * rows;
    const int64_t units = div_up(n, per_block), blocks = div_up(units, div_up(units, static_cast<int64_t>(p->sms) * per_sm));
    if (access != kBetween || blocks == units) return blocks;
    const int64_t V = 16 / element_bytes(p->type), alike = per_block >= V ? 1 : V / per_block;
    return div_up(blocks, alike) * alike;
}

int64_t backward_blocks(const layer_norm *p, int64_t n, Access access)
{
    return blocks_for(p, access, n, p->backward_blocks[access], p->backward_rows[access]);
}

template <typename T>
bool count_blocks(layer_norm *p)
{
    for (const Access access : {kSingle, kWhole, kBetween}) {
        if (!offered(p, access)) continue;
        const Share s = share_for(p, access);
        const int threads = s.wide ? s.lanes : kNarrowThreads;
        const bool ok = with_counts<T>(s, vectors_of(p, access), access, [&](auto v, auto c, auto r, auto form, auto fit) {
            p->backward_rows[access] = kBackwardRowsOf<T, v.value, c.value, r.value, form.value, fit.value>;
            return cudaOccupancyMaxActiveBlocksPerMultiprocessor(&p->forward_blocks[access], k_forward<T, v.value, c.value, r.value, form.value, fit.value>,
                                                                 threads, 0) == cudaSuccess &&
                   cudaOccupancyMaxActiveBlocksPerMultiprocessor(&p->backward_blocks[access], k_backward<T, v.value, c.value, r.value, form.value, fit.value>,
                                                                 threads, backward_smem(p, s)) == cudaSuccess;
        });
        if (!ok || p->forward_blocks[access] < 1 || p->backward_blocks[access] < 1) return false;
    }
    return true;
}

// How a call's arrays can be read: add() takes each, access() decides.  Whole vectors need the parameters (params_whole) and all rows on
// boundaries; between boundaries the rows have to lie alike and the width has to be offered, the parameters lie as they like (whole
// rows with other parameters come here too); else single elements.
struct Lie {
    const layer_norm *p;
    int64_t n;
    int bytes, shift = -1, turn = 0;
    bool whole = true, alike = true;
    void add(const void *ptr, int64_t stride)
    {
        if (ptr == nullptr) return;
        const int V = 16 / bytes;
        const int at = static_cast<int>(reinterpret_cast<uintptr_t>(ptr) / bytes % V), step = n == 1 ? 0 : static_cast<int>(stride % V);
        whole = whole && at == 0 && step == 0;
        alike = alike && (n == 1 || stride >= V) && (shift < 0 || (at == shift && step == turn));
        shift = at;
        turn = step;
    }
    Access access(bool params_whole) const
    {
        if (whole && params_whole && offered(p, kWhole)) return kWhole;
        return alike && offered(p, kBetween) ? kBetween : kSingle;
    }
};

bool check_in(const void *ptr, int64_t stride, int bytes, int *rc)
{
    if (stride < 0) *rc = LAYER_NORM_EINVAL;
    else if (!aligned(ptr, bytes)) *rc = LAYER_NORM_EALIGN;
    return *rc == LAYER_NORM_OK;
}

bool check_out(const void *ptr, int64_t stride, int64_t n, int width, int bytes, int *rc)
{
    if (n > 1 && stride < width) *rc = LAYER_NORM_EINVAL;
    else if (!aligned(ptr, bytes)) *rc = LAYER_NORM_EALIGN;
    return *rc == LAYER_NORM_OK;
}

template <typename T>
Rows<const T> in_rows(const void *ptr, int64_t stride) { return {static_cast<const T *>(ptr), stride}; }
template <typename T>
Rows<T> out_rows(void *ptr, int64_t stride) { return {static_cast<T *>(ptr), stride}; }

template <typename T>
int run_forward(layer_norm *p, Forward<T> f, Access access)
{
    const Share s = share_for(p, access);
    f.lanes = s.lanes;
    const bool ok = with_counts<T>(s, vectors_of(p, access), access, [&](auto v, auto c, auto r, auto form, auto fit) {
        const int64_t blocks = blocks_for(p, access, f.n, p->forward_blocks[access], kRowsOf<T, v.value, c.value, r.value, form.value, fit.value>);
        k_forward<T, v.value, c.value, r.value, form.value, fit.value>
            <<<static_cast<unsigned>(blocks), s.wide ? s.lanes : kNarrowThreads, 0, p->stream>>>(f);
        return cudaGetLastError() == cudaSuccess;
    });
    if (!ok) return LAYER_NORM_ECUDA;
    p->launches += 1;
    return LAYER_NORM_OK;
}

template <typename T>
int run_backward(layer_norm *p, Backward<T> b, Access access, float *dw, float *db)
{
    const Share s = share_for(p, access);
    b.lanes = s.lanes;
    const int64_t blocks = backward_blocks(p, b.n, access);
    const size_t smem = backward_smem(p, s);
    const bool ok = with_counts<T>(s, vectors_of(p, access), access, [&](auto v, auto c, auto r, auto form, auto fit) {
        k_backward<T, v.value, c.value, r.value, form.value, fit.value>
            <<<static_cast<unsigned>(blocks), s.wide ? s.lanes : kNarrowThreads, smem, p->stream>>>(b);
        return cudaGetLastError() == cudaSuccess;
    });
    if (!ok) return LAYER_NORM_ECUDA;
    p->launches += 1;
    if (b.part == nullptr) return LAYER_NORM_OK;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(div_up(2 * static_cast<int64_t>(p->width), 32)));
    cfg.blockDim = dim3(32 * kJoinWarps);
    cfg.stream = p->stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    if (cudaLaunchKernelEx(&cfg, k_join, static_cast<const float *>(b.part), static_cast<int>(blocks), p->width, dw, db) !=
        cudaSuccess) {
        cudaGetLastError();
        return LAYER_NORM_ECUDA;
    }
    p->launches += 1;
    return LAYER_NORM_OK;
}

template <typename T>
int forward_of(layer_norm *p, const void *x, int64_t x_stride, const void *residual, int64_t residual_stride, const float *w,
               const float *b, void *sum, int64_t sum_stride, void *y, int64_t y_stride, float *saved, int64_t n)
{
    Forward<T> f = {};
    f.x = in_rows<T>(x, x_stride);
    f.residual = in_rows<T>(residual, residual_stride);
    f.sum = out_rows<T>(sum, sum_stride);
    f.y = out_rows<T>(y, y_stride);
    f.w = w;
    f.b = b;
    f.saved = reinterpret_cast<float2 *>(saved);
    f.n = n;
    f.width = p->width;
    f.eps = p->eps;
    Lie lie = {p, n, sizeof(T)};
    lie.add(x, x_stride);
    lie.add(residual, residual_stride);
    lie.add(sum, sum_stride);
    lie.add(y, y_stride);
    f.shift = lie.shift;
    f.turn = lie.turn;
    return run_forward<T>(p, f, lie.access(aligned(w, 16) && aligned(b, 16)));
}

template <typename T>
int backward_of(layer_norm *p, const void *dy, int64_t dy_stride, const void *s, int64_t s_stride, const float *w,
                const float *saved, const void *dsum, int64_t dsum_stride, void *dx, int64_t dx_stride, float *dw, float *db,
                void *workspace, int64_t n)
{
    Backward<T> f = {};
    f.dy = in_rows<T>(dy, dy_stride);
    f.s = in_rows<T>(s, s_stride);
    f.dsum = in_rows<T>(dsum, dsum_stride);
    f.dx = out_rows<T>(dx, dx_stride);
    f.w = w;
    f.saved = reinterpret_cast<const float2 *>(saved);
    f.part = dw != nullptr ? static_cast<float *>(workspace) : nullptr;
    f.n = n;
    f.width = p->width;
    Lie lie = {p, n, sizeof(T)};
    lie.add(dy, dy_stride);
    lie.add(s, s_stride);
    lie.add(dsum, dsum_stride);
    lie.add(dx, dx_stride);
    f.shift = lie.shift;
    f.turn = lie.turn;
    return run_backward<T>(p, f, lie.access(aligned(w, 16)), dw, db);
}

bool rows_ok(int64_t n) { return n >= 1 && n <= 0x7FFFFFFF; }

}  // namespace

extern "C" {

int layer_norm_create(layer_norm **out, int width, float eps, int type)
{
    if (out == nullptr) return LAYER_NORM_ENULL;
    *out = nullptr;
    if (width < 1 || width > LAYER_NORM_MAX_WIDTH) return LAYER_NORM_EINVAL;
    if (!(eps > 0.0f) || std::isinf(eps)) return LAYER_NORM_EINVAL;
    if (type != LAYER_NORM_F32 && type != LAYER_NORM_BF16 && type != LAYER_NORM_F16) return LAYER_NORM_EINVAL;
    layer_norm *p = new (std::nothrow) layer_norm;
    if (p == nullptr) return LAYER_NORM_ENOMEM;
    p->width = width;
    p->eps = eps;
    p->type = type;
    if (cudaGetDevice(&p->device) != cudaSuccess ||
        cudaDeviceGetAttribute(&p->sms, cudaDevAttrMultiProcessorCount, p->device) != cudaSuccess ||
        !(type == LAYER_NORM_F32 ? count_blocks<float>(p) : type == LAYER_NORM_BF16 ? count_blocks<__nv_bfloat16>(p) : count_blocks<__half>(p))) {
        cudaGetLastError();
        delete p;
        return LAYER_NORM_ECUDA;
    }
    *out = p;
    return LAYER_NORM_OK;
}

int layer_norm_destroy(layer_norm *p)
{
    if (p == nullptr) return LAYER_NORM_ENULL;
    delete p;
    return LAYER_NORM_OK;
}

int layer_norm_set_stream(layer_norm *p, void *cuda_stream)
{
    if (p == nullptr) return LAYER_NORM_ENULL;
    p->stream = static_cast<cudaStream_t>(cuda_stream);
    return LAYER_NORM_OK;
}

int layer_norm_forward(layer_norm *p, const void *x, int64_t x_stride, const void *residual, int64_t residual_stride,
                       const float *w, const float *b, void *sum, int64_t sum_stride, void *y, int64_t y_stride,
                       float *saved, int64_t n)
{
    if (p == nullptr) return LAYER_NORM_ENULL;
    if (!rows_ok(n)) return LAYER_NORM_EINVAL;            // first: an empty batch comes without pointers
    if (x == nullptr || y == nullptr || (residual == nullptr) != (sum == nullptr)) return LAYER_NORM_ENULL;
    const int e = element_bytes(p->type);
    int rc = LAYER_NORM_OK;
    if (!check_in(x, x_stride, e, &rc) || !check_out(y, y_stride, n, p->width, e, &rc)) return rc;
    if (residual != nullptr &&
        (!check_in(residual, residual_stride, e, &rc) || !check_out(sum, sum_stride, n, p->width, e, &rc)))
        return rc;
    if (!aligned(w, 4) || !aligned(b, 4) || !aligned(saved, 8)) return LAYER_NORM_EALIGN;
    const OnDevice on(p->device);
    if (!on.ok()) return LAYER_NORM_ECUDA;
    auto call = p->type == LAYER_NORM_F32 ? forward_of<float> : p->type == LAYER_NORM_BF16 ? forward_of<__nv_bfloat16> : forward_of<__half>;
    return call(p, x, x_stride, residual, residual_stride, w, b, sum, sum_stride, y, y_stride, saved, n);
}

size_t layer_norm_workspace_bytes(const layer_norm *p, int64_t n)
{
    if (p == nullptr || !rows_ok(n)) return 0;
    // rows are shared out by how they lie: room for each way
    int64_t rows = 0;
    for (const Access access : {kSingle, kWhole, kBetween}) {
        if (p->backward_blocks[access] < 1) continue;
        const int64_t blocks = backward_blocks(p, n, access);
        if (blocks > rows) rows = blocks;
    }
    return static_cast<size_t>(rows) * 2 * p->width * sizeof(float);
}

int layer_norm_backward(layer_norm *p, const void *dy, int64_t dy_stride, const void *s, int64_t s_stride,
                        const float *w, const float *saved, const void *dsum, int64_t dsum_stride, void *dx,
                        int64_t dx_stride, float *dw, float *db, void *workspace, size_t workspace_bytes, int64_t n)
{
    if (p == nullptr) return LAYER_NORM_ENULL;
    if (!rows_ok(n)) return LAYER_NORM_EINVAL;
    if (dy == nullptr || s == nullptr || saved == nullptr || dx == nullptr || (dw == nullptr) != (db == nullptr))
        return LAYER_NORM_ENULL;
    const int e = element_bytes(p->type);
    int rc = LAYER_NORM_OK;
    if (!check_in(dy, dy_stride, e, &rc) || !check_in(s, s_stride, e, &rc) || !check_out(dx, dx_stride, n, p->width, e, &rc))
        return rc;
    if (dsum != nullptr && !check_in(dsum, dsum_stride, e, &rc)) return rc;
    if (!aligned(w, 4) || !aligned(dw, 4) || !aligned(db, 4) || !aligned(saved, 8) || !aligned(workspace, 16))
        return LAYER_NORM_EALIGN;
    if (dw != nullptr) {
        if (workspace == nullptr) return LAYER_NORM_ENULL;
        if (layer_norm_workspace_bytes(p, n) > workspace_bytes) return LAYER_NORM_ENOMEM;
    }
    const OnDevice on(p->device);
    if (!on.ok()) return LAYER_NORM_ECUDA;
    auto call = p->type == LAYER_NORM_F32 ? backward_of<float> : p->type == LAYER_NORM_BF16 ? backward_of<__nv_bfloat16> : backward_of<__half>;
    return call(p, dy, dy_stride, s, s_stride, w, saved, dsum, dsum_stride, dx, dx_stride, dw, db, workspace, n);
}

int64_t layer_norm_launch_count(const layer_norm *p) { return p ? p->launches : 0; }

const char *layer_norm_strerror(int code)
{
    switch (code) {
    case LAYER_NORM_OK: return "ok";
    case LAYER_NORM_EINVAL: return "invalid size, stride, eps or type";
    case LAYER_NORM_ENULL: return "required pointer is NULL";
    case LAYER_NORM_EALIGN: return "pointer not aligned to its element";
    case LAYER_NORM_ECUDA: return "CUDA call or launch failed";
    case LAYER_NORM_ENOMEM: return "allocation failed, or the workspace is too small";
    default: return "unknown error";
    }
}

}  // extern "C"
