// orthogonal.cu -- the orthogonalised update behind the C ABI of orthogonal.h, on sm_100a tensor cores.
//
// k_product is one matrix product D = A B^T on CTA pairs (tcgen05, cta_group::2): a pair's tile is 256 rows of A by 64, 128
// or 256 rows of B; each block of the pair stages 128 rows of A and half of the rows of B per 64 reduction elements, the
// leader issues M = 256 instructions into one of two accumulator buffers, and eight epilogue warps per block empty the
// other one meanwhile.  Three epilogues make a step of the iteration:
//
//   kGram     A = X X^T.  Symmetric: only tiles with elements on or above the diagonal are computed, and each element
//             above it is written to both places.  Off the diagonal binary16 (O), on it binary32 (d) and a zero in O.
//   kSquare   B = b A + c A A, symmetric too.  A = diag(d) + O, so A A = O O + (d_i + d_j) O_ij off the diagonal, O O + d_i^2 on
//             it: the product has O alone, the rest is binary32 in the epilogue.  B again as P (binary16) and e (binary32).
//   kApply    X' = (a + e_i) X + P X, with X as the pair hi + lo in the first term and hi as the operand; the last step
//             writes the update instead.
//
// Why the diagonals are apart: in the last steps A is near the identity and B near -2.7 of it, so that a X + B X cancels.
// Rounded to binary16 these diagonals alone put 1e-3 to 3e-3 of error into the result; centred around the polynomial's middle
// instead, a dominant direction's rounding runs into the small ones (3e-2).  Why hi + lo: rounded anew in every step, what the
// large directions lose comes out 3.4 times larger per step in the small ones (4e-2 for a momentum of few directions).
//
// Operands lie in memory as they are: where the reduction runs along rows, TMA brings boxes of 64 elements of the row by 64
// reduction rows and the instruction reads them MN-major; nothing is transposed, and a tall matrix is worked on as
// X' = X (a + e_j) + X P.
#include <cmath>
#include <new>

#include <cuda_fp16.h>

#include "../../include/orthogonal.h"
#include "on_device.cuh"
#include "sm100.cuh"
#include "vectors.cuh"

namespace {

constexpr int kBK = 64;                          // reduction elements per stage
constexpr int kRowsPerBlock = 128;               // rows of A per block; a pair's tile has twice as many
constexpr int kTileM = 2 * kRowsPerBlock;
constexpr int kStages = 6;
constexpr int kABytes = kRowsPerBlock * kBK * 2;
constexpr int kBBytes = 128 * kBK * 2;           // at most 128 rows of B per block
constexpr int kStageBytes = kABytes + kBBytes;
constexpr int kAccCols = 256;
constexpr int kTmemCols = 2 * kAccCols;
constexpr int kEpilogueWarps = 8;
constexpr int kThreads = 64 + 32 * kEpilogueWarps;
constexpr int kSmem = kStages * kStageBytes + 256 + 1024;
static_assert(kSmem <= 227 * 1024, "shared memory of a block");

constexpr int kRowThreads = 256;                 // blocks of the kernels that read and write rows
constexpr int kMostParts = 128;                  // partial sums of squares per matrix

// Operands are held times 2^13: an element of a normalised matrix of a million is about 2^-10, of A and B up to 2^2.
constexpr float kScale = 8192.0f;
constexpr float kUnscale = 1.0f / kScale;

enum Mode { kGram, kSquare, kApply, kLast };

struct Product {
    int m, n, k;            // rows of A, rows of B, reduction length, of one matrix
    int batch;
    int a_rows, b_rows;     // 1: the operand is stored [k][rows] (MN-major), 0: [rows][k]
    int tile_n;             // columns of D per tile: 256, 128 or 64
    int m_tiles, n_tiles;
    int tiles;              // of one matrix: those that are computed
    int steps;              // ceil(k / 64)
    int tall;               // rows > cols: the diagonal's factors go with columns
    int ld;                 // elements between rows of X
    int ldk;                // of O and P
    int dk;                 // elements between the diagonals of two matrices
    float a, b, c;
    __half *o, *p;
    float *d, *e;
    const __half *hi, *lo;
    __half *hi_next, *lo_next;
    __nv_bfloat16 *out;     // kLast
    int64_t out_batch, out_row;
    int out_whole;          // rows of the update start on 16-byte boundaries
    int *err;
};

__device__ __forceinline__ void allow_next() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void wait_for_previous() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

// MN-major operand tile with the 128-byte swizzle: boxes of 64 elements (128 bytes) by 64 reduction
// rows; the next 64 elements are a box (8192 bytes, leading offset) further, the next 8
// reduction rows 1024 bytes (stride offset).
__device__ __forceinline__ uint64_t smem_desc_rows(uint32_t addr)
{
    return static_cast<uint64_t>((addr >> 4) & 0x3FFFu) | (512ull << 16) | (64ull << 32) | (1ull << 46) | (2ull << 61);
}

// Tile load of matrix z by this block of the pair; `bar` is a shared::cluster address and may be the peer's barrier.
__device__ __forceinline__ void tma_load_matrix(uint32_t dst, const CUtensorMap *map, int x, int y, int z, uint32_t bar)
{
    asm volatile(
        "cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes"
        " [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(dst),
        "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar)
        : "memory");
}

struct Tile {
    int z, row, col;         // matrix, first row and column
};

// Symmetric products: row block I has the column tiles from the one of its first diagonal element on.
template <int kMode>
__device__ __forceinline__ Tile tile_at(const Product &p, int index)
{
    Tile t;
    t.z = index / p.tiles;
    int i = index - t.z * p.tiles;
    if (kMode == kGram || kMode == kSquare) {
        const int per = kTileM / p.tile_n;
        int r = 0;
        while (i >= p.n_tiles - r * per) {
            i -= p.n_tiles - r * per;
            ++r;
        }
        t.row = r * kTileM;
        t.col = (r * per + i) * p.tile_n;
    } else {
        // neighbours share the columns' operand
        t.row = i % p.m_tiles * kTileM;
        t.col = i / p.m_tiles * p.tile_n;
    }
    return t;
}

__device__ __forceinline__ uint32_t pack2(float a, float b)
{
    const __half2 v = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t *>(&v);
}

__device__ __forceinline__ float2 unpack2(uint32_t w) { return __half22float2(*reinterpret_cast<const __half2 *>(&w)); }

// 16 elements of a row that lies in memory in pieces of 8; columns from `width` (a multiple of 8) on are not there.
__device__ __forceinline__ void load16(uint32_t (&w)[8], const __half *src, int c, int width)
{
    const uint4 none = make_uint4(0, 0, 0, 0);
    const uint4 u = c < width ? *reinterpret_cast<const uint4 *>(src + c) : none;
    const uint4 v = c + 8 < width ? *reinterpret_cast<const uint4 *>(src + c + 8) : none;
    w[0] = u.x, w[1] = u.y, w[2] = u.z, w[3] = u.w, w[4] = v.x, w[5] = v.y, w[6] = v.z, w[7] = v.w;
}

__device__ __forceinline__ void store16(void *row, int c, int width, const uint32_t (&w)[8])
{
    uint4 *dst = reinterpret_cast<uint4 *>(static_cast<uint16_t *>(row) + c);
    if (c < width) dst[0] = make_uint4(w[0], w[1], w[2], w[3]);
    if (c + 8 < width) dst[1] = make_uint4(w[4], w[5], w[6], w[7]);
}

// Elements (i, j0 .. j0 + 15) of a symmetric matrix of k rows: those above the diagonal to both places, a zero on it.
__device__ __forceinline__ void store_symmetric(__half *base, int ldk, int k, int i, int j0, const float (&v)[16])
{
    __half *mirror = base + static_cast<int64_t>(j0) * ldk + i;
    if (j0 > i) {
        uint32_t w[8];
#pragma unroll
        for (int q = 0; q < 8; ++q) w[q] = pack2(v[2 * q], v[2 * q + 1]);
        store16(base + static_cast<int64_t>(i) * ldk, j0, ldk, w);
#pragma unroll
        for (int q = 0; q < 16; ++q) {
            if (j0 + q < k)
                *reinterpret_cast<uint16_t *>(mirror + static_cast<int64_t>(q) * ldk) =
                    static_cast<uint16_t>(q & 1 ? w[q / 2] >> 16 : w[q / 2]);
        }
    } else if (j0 + 15 >= i) {
#pragma unroll
        for (int q = 0; q < 16; ++q) {
            const int j = j0 + q;
            if (j < i || j >= k) continue;
            const __half h = j == i ? __float2half_rn(0.0f) : __float2half_rn(v[q]);
            base[static_cast<int64_t>(i) * ldk + j] = h;
            mirror[static_cast<int64_t>(q) * ldk] = h;
        }
    }
}

template <int kMode>
__global__ void __launch_bounds__(kThreads, 1)
k_product(const __grid_constant__ CUtensorMap tm_a, const __grid_constant__ CUtensorMap tm_b, const __grid_constant__ Product p)
{
    extern __shared__ uint8_t smem_raw[];
    const uint32_t raw = smem_u32(smem_raw);
    const uint32_t stages = (raw + 1023u) & ~1023u;
    const uint32_t bars = stages + kStages * kStageBytes;
    uint8_t *bars_ptr = smem_raw + (bars - raw);
    const uint32_t full0 = bars, empty0 = bars + 8 * kStages;
    const uint32_t acc_full0 = bars + 16 * kStages, acc_empty0 = acc_full0 + 16;
    volatile uint32_t *tmem_slot = reinterpret_cast<volatile uint32_t *>(bars_ptr + 16 * kStages + 32);
    volatile int *abort_flag = reinterpret_cast<volatile int *>(bars_ptr + 16 * kStages + 32 + 8);

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = cluster_cta_rank();
    const int pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;
    const int b_half = p.tile_n / 2;
    const int all = p.tiles * p.batch;

    if (threadIdx.x == 0) {
        for (int s = 0; s < kStages; ++s) {
            mbar_init(full0 + 8 * s, 1);
            mbar_init(empty0 + 8 * s, 1);
        }
        for (int b = 0; b < 2; ++b) {
            mbar_init(acc_full0 + 8 * b, 1);
            mbar_init(acc_empty0 + 8 * b, 2 * kEpilogueWarps);
        }
        *abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    allow_next();
    if (warp == 1) tmem_alloc(smem_u32(const_cast<uint32_t *>(tmem_slot)), kTmemCols);
    tc_fence_before_sync();
    cluster_sync_all();
    tc_fence_after_sync();
    const uint32_t tmem_base = *tmem_slot;
    wait_for_previous();                     // operands are its results, and outputs what it still reads

    if (warp == 0) {
        if (lane == 0) {
            asm volatile("fence.proxy.async.global;" ::: "memory");    // the previous kernel wrote the operands by plain stores
            uint32_t s = 0, ph = 0;
            bool ok = true;
            const int b_boxes = (b_half + 63) / 64;
            const uint32_t bytes = kABytes + (p.b_rows ? b_boxes * 64 * kBK * 2 : b_half * kBK * 2);
            for (int index = pair; ok && index < all; index += pairs) {
                const Tile t = tile_at<kMode>(p, index);
                const int a0 = t.row + static_cast<int>(rank) * kRowsPerBlock, b0 = t.col + static_cast<int>(rank) * b_half;
                for (int kc = 0; kc < p.steps; ++kc) {
                    if (!mbar_wait(empty0 + 8 * s, ph ^ 1u, abort_flag)) {
                        ok = false;
                        break;
                    }
                    const uint32_t dst = stages + s * kStageBytes;
                    const uint32_t full = map_to_rank(full0 + 8 * s, 0);
                    if (rank == 0) mbar_expect_tx(full0 + 8 * s, 2 * bytes);
                    if (p.a_rows) {
                        tma_load_matrix(dst, &tm_a, a0, kc * kBK, t.z, full);
                        tma_load_matrix(dst + kABytes / 2, &tm_a, a0 + 64, kc * kBK, t.z, full);
                    } else {
                        tma_load_matrix(dst, &tm_a, kc * kBK, a0, t.z, full);
                    }
                    if (p.b_rows) {
                        for (int i = 0; i < b_boxes; ++i)
                            tma_load_matrix(dst + kABytes + i * 64 * kBK * 2, &tm_b, b0 + 64 * i, kc * kBK, t.z, full);
                    } else {
                        tma_load_matrix(dst + kABytes, &tm_b, kc * kBK, b0, t.z, full);
                    }
                    if (++s == kStages) {
                        s = 0;
                        ph ^= 1u;
                    }
                }
            }
            // do not leave while the leader's instructions may still read this block's stages
            for (int i = 0; i < kStages && ok; ++i) {
                ok = mbar_wait(empty0 + 8 * s, ph ^ 1u, abort_flag);
                if (++s == kStages) {
                    s = 0;
                    ph ^= 1u;
                }
            }
        }
    } else if (warp == 1) {
        if (lane == 0 && rank == 0) {
            const uint32_t idesc = (1u << 4) | (static_cast<uint32_t>(p.a_rows) << 15) | (static_cast<uint32_t>(p.b_rows) << 16) |
                                   (static_cast<uint32_t>(p.tile_n >> 3) << 17) | (static_cast<uint32_t>(kTileM >> 4) << 24);
            // 16 reduction elements: 32 bytes along a K-major row, 16 rows of 128 bytes MN-major
            const uint32_t a_step = p.a_rows ? 2048 >> 4 : 32 >> 4, b_step = p.b_rows ? 2048 >> 4 : 32 >> 4;
            uint32_t s = 0, ph = 0;
            bool ok = true;
            int it = 0;
            for (int index = pair; ok && index < all; index += pairs, ++it) {
                const uint32_t buf = it & 1, use = (it >> 1) & 1;
                if (!mbar_wait(acc_empty0 + 8 * buf, use ^ 1u, abort_flag)) break;
                tc_fence_after_sync();
                const uint32_t d = tmem_base + buf * kAccCols;
                for (int kc = 0; kc < p.steps; ++kc) {
                    if (!mbar_wait(full0 + 8 * s, ph, abort_flag)) {
                        ok = false;
                        break;
                    }
                    tc_fence_after_sync();
                    const uint32_t addr = stages + s * kStageBytes;
                    const uint64_t ad = p.a_rows ? smem_desc_rows(addr) : smem_desc(addr);
                    const uint64_t bd = p.b_rows ? smem_desc_rows(addr + kABytes) : smem_desc(addr + kABytes);
#pragma unroll
                    for (int k = 0; k < kBK / 16; ++k)
                        umma_bf16(d, ad + a_step * k, bd + b_step * k, idesc, kc > 0 || k > 0);
                    umma_commit_pair(empty0 + 8 * s);
                    if (++s == kStages) {
                        s = 0;
                        ph ^= 1u;
                    }
                }
                if (ok) umma_commit_pair(acc_full0 + 8 * buf);
            }
        }
    } else {
        const int q = warp & 3;
        const int half = (warp - 2) >> 2;                // which half of the columns
        const uint32_t lane_base = tmem_base + (static_cast<uint32_t>(q * 32) << 16);
        int it = 0;
        for (int index = pair; index < all; index += pairs, ++it) {
            const uint32_t buf = it & 1, use = (it >> 1) & 1;
            const Tile t = tile_at<kMode>(p, index);
            const int row = t.row + static_cast<int>(rank) * kRowsPerBlock + q * 32 + lane;
            const bool live = row < p.m;
            const uint32_t t0 = lane_base + buf * kAccCols;
            const bool ready = mbar_wait(acc_full0 + 8 * buf, use, abort_flag);
            if (!__all_sync(0xFFFFFFFFu, ready)) break;
            tc_fence_after_sync();
            const int c_end = (half + 1) * (p.tile_n / 2);
            if (kMode == kGram || kMode == kSquare) {
                const int64_t square = static_cast<int64_t>(t.z) * p.m * p.ldk;
                const int64_t diagonal = static_cast<int64_t>(t.z) * p.dk;
                const float di = kMode == kSquare && live ? p.d[diagonal + row] : 0.0f;
#pragma unroll 1
                for (int c = half * (p.tile_n / 2); c < c_end; c += 16) {
                    const int j0 = t.col + c;
                    uint32_t acc[16];
                    tmem_ld16(t0 + c, acc);
                    if (kMode == kGram) {
                        tmem_wait_ld();
                        if (live && j0 < p.n && j0 + 15 >= row) {
                            float v[16];
#pragma unroll
                            for (int e = 0; e < 16; ++e) {
                                v[e] = __uint_as_float(acc[e]) * kUnscale;
                                if (j0 + e == row) p.d[diagonal + row] = v[e] * kUnscale;
                            }
                            store_symmetric(p.o + square, p.ldk, p.m, row, j0, v);
                        }
                    } else {
                        const bool any = live && j0 < p.n && j0 + 15 >= row;
                        uint32_t ow[8] = {0, 0, 0, 0, 0, 0, 0, 0};
                        if (any) load16(ow, p.o + square + static_cast<int64_t>(row) * p.ldk, j0, p.ldk);
                        tmem_wait_ld();
                        if (any) {
                            float v[16];
#pragma unroll
                            for (int e = 0; e < 16; e += 4) {
                                // (the diagonals are padded to whole pieces of 16)
                                const float4 dj = *reinterpret_cast<const float4 *>(p.d + diagonal + j0 + e);
                                const float2 o0 = unpack2(ow[e / 2]), o1 = unpack2(ow[e / 2 + 1]);
                                const float o[4] = {o0.x, o0.y, o1.x, o1.y}, ds[4] = {dj.x, dj.y, dj.z, dj.w};
#pragma unroll
                                for (int f = 0; f < 4; ++f) {
                                    const float s = __uint_as_float(acc[e + f]) * kUnscale;
                                    v[e + f] = fmaf(p.c, fmaf(di + ds[f], o[f], s), p.b * o[f]);
                                    if (j0 + e + f == row)
                                        p.e[diagonal + row] = fmaf(p.c, fmaf(di, di, s * kUnscale), p.b * di);
                                }
                            }
                            store_symmetric(p.p + square, p.ldk, p.m, row, j0, v);
                        }
                    }
                }
            } else {
                const int64_t diagonal = static_cast<int64_t>(t.z) * p.dk;
                const int64_t at = (static_cast<int64_t>(t.z) * p.m + (live ? row : 0)) * p.ld;
                const float factor = p.a + (p.tall || !live ? 0.0f : p.e[diagonal + row]);
#pragma unroll 1
                for (int c = half * (p.tile_n / 2); c < c_end; c += 16) {
                    const int j0 = t.col + c;
                    uint32_t acc[16], hw[8], lw[8];
                    tmem_ld16(t0 + c, acc);
                    const bool any = live && j0 < p.n;
                    if (any) {
                        load16(hw, p.hi + at, j0, p.ld);
                        load16(lw, p.lo + at, j0, p.ld);
                    }
                    tmem_wait_ld();
                    if (!any) continue;
                    float v[16];
#pragma unroll
                    for (int e = 0; e < 16; e += 4) {
                        float f[4] = {factor, factor, factor, factor};
                        if (p.tall) {
                            const float4 ej = *reinterpret_cast<const float4 *>(p.e + diagonal + j0 + e);
                            f[0] += ej.x, f[1] += ej.y, f[2] += ej.z, f[3] += ej.w;
                        }
#pragma unroll
                        for (int g = 0; g < 4; g += 2) {
                            const float2 h = unpack2(hw[(e + g) / 2]), l = unpack2(lw[(e + g) / 2]);
                            v[e + g] = fmaf(f[g], h.x + l.x, __uint_as_float(acc[e + g]) * kUnscale);
                            v[e + g + 1] = fmaf(f[g + 1], h.y + l.y, __uint_as_float(acc[e + g + 1]) * kUnscale);
                        }
                    }
                    if (kMode == kApply) {
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            hw[e] = pack2(v[2 * e], v[2 * e + 1]);
                            const float2 h = unpack2(hw[e]);
                            lw[e] = pack2(v[2 * e] - h.x, v[2 * e + 1] - h.y);
                        }
                        store16(p.hi_next + at, j0, p.ld, hw);
                        store16(p.lo_next + at, j0, p.ld, lw);
                    } else {
                        __nv_bfloat16 *dst = p.out + t.z * p.out_batch + row * p.out_row;
                        if (p.out_whole) {
#pragma unroll
                            for (int e = 0; e < 8; ++e) hw[e] = pack_bf16(v[2 * e] * kUnscale, v[2 * e + 1] * kUnscale);
                            store16(dst, j0, p.n, hw);
                        } else {
#pragma unroll
                            for (int e = 0; e < 16; ++e)
                                if (j0 + e < p.n) dst[j0 + e] = __float2bfloat16_rn(v[e] * kUnscale);
                        }
                    }
                }
            }
            tc_fence_before_sync();
            __syncwarp();
            if (lane == 0) mbar_arrive_cluster(map_to_rank(acc_empty0 + 8 * buf, 0));
        }
    }

    tc_fence_before_sync();
    __syncthreads();
    if (*abort_flag) {
        if (threadIdx.x == 0) atomicExch(p.err, 1);
        const unsigned long long t0 = global_timer_ns();
        while (global_timer_ns() - t0 < kDrainNs) __nanosleep(1000);
    }
    cluster_sync_all();
    if (warp == 1) {
        __syncwarp();
        tc_fence_after_sync();
        tmem_dealloc(tmem_base, kTmemCols);
    }
}

// ---- the norm, and the first X

struct Start {
    int rows, cols, ld;
    int parts;               // blocks per matrix
    int whole;               // rows of G start on 16-byte boundaries
    int64_t g_batch, g_row;
    double eps;
    double *squares;         // [batch][parts]
    __half *hi, *lo;
};

// Eight elements of a row of G, from column c.
template <typename T>
__device__ __forceinline__ void load8(float (&v)[8], const T *row, int c, int cols, bool whole)
{
    constexpr int V = 16 / sizeof(T);
    if (whole && c + 8 <= cols) {
#pragma unroll
        for (int i = 0; i < 8; i += V) {
            const Packed<T, V> w = packed_load<T, V>(row + c + i);
#pragma unroll
            for (int e = 0; e < V; ++e) v[i + e] = packed_get<T, V>(w, e);
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = c + e < cols ? packed_get<T, 1>(packed_load<T, 1>(row + c + e), 0) : 0.0f;
    }
}

// The block's part of a matrix: pieces of eight elements, every parts-th run of kRowThreads.
template <typename F>
__device__ __forceinline__ void each_piece(const Start &s, int part, F f)
{
    const int per_row = s.ld / 8;
    const int64_t pieces = static_cast<int64_t>(s.rows) * per_row;
    for (int64_t i = static_cast<int64_t>(part) * kRowThreads + threadIdx.x; i < pieces; i += static_cast<int64_t>(s.parts) * kRowThreads) {
        const int64_t row = i / per_row;
        f(row, static_cast<int>(i - row * per_row) * 8);
    }
}

__device__ double block_sum(double v)
{
    __shared__ double s[kRowThreads / 32];
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
    if ((threadIdx.x & 31) == 0) s[threadIdx.x >> 5] = v;
    __syncthreads();
    v = 0.0;
#pragma unroll
    for (int i = 0; i < kRowThreads / 32; ++i) v += s[i];
    return v;
}

template <typename T>
__global__ void __launch_bounds__(kRowThreads)
k_squares(const Start s, const T *g)
{
    allow_next();
    const int part = blockIdx.x, z = blockIdx.y;
    double sum = 0.0;
    each_piece(s, part, [&](int64_t row, int c) {
        float v[8];
        load8<T>(v, g + z * s.g_batch + row * s.g_row, c, s.cols, s.whole);
#pragma unroll
        for (int e = 0; e < 8; ++e) sum = fma(static_cast<double>(v[e]), static_cast<double>(v[e]), sum);
    });
    sum = block_sum(sum);
    if (threadIdx.x == 0) s.squares[z * s.parts + part] = sum;
}

template <typename T>
__global__ void __launch_bounds__(kRowThreads)
k_start(const Start s, const T *g)
{
    allow_next();
    wait_for_previous();
    const int part = blockIdx.x, z = blockIdx.y;
    const double sum = block_sum(threadIdx.x < s.parts ? s.squares[z * s.parts + threadIdx.x] : 0.0);
    const float factor = static_cast<float>(static_cast<double>(kScale) / (sqrt(sum) + s.eps));
    each_piece(s, part, [&](int64_t row, int c) {
        float v[8];
        load8<T>(v, g + z * s.g_batch + row * s.g_row, c, s.cols, s.whole);
        uint32_t hw[4], lw[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            v[2 * e] *= factor;
            v[2 * e + 1] *= factor;
            hw[e] = pack2(v[2 * e], v[2 * e + 1]);
            const float2 h = unpack2(hw[e]);
            lw[e] = pack2(v[2 * e] - h.x, v[2 * e + 1] - h.y);
        }
        const int64_t at = (static_cast<int64_t>(z) * s.rows + row) * s.ld + c;
        *reinterpret_cast<uint4 *>(s.hi + at) = make_uint4(hw[0], hw[1], hw[2], hw[3]);
        *reinterpret_cast<uint4 *>(s.lo + at) = make_uint4(lw[0], lw[1], lw[2], lw[3]);
    });
}

// ---------------------------------------------------------------- host side

int64_t div_up(int64_t a, int64_t b) { return (a + b - 1) / b; }

// A stack of matrices [batch][rows][cols] of binary16 with `ld` elements between rows, in boxes of 64 columns by box_rows.
bool encode(CUtensorMap *m, const __half *base, int64_t batch, int64_t rows, int64_t cols, int64_t ld, uint32_t box_rows)
{
    const cuuint64_t dims[3] = {static_cast<cuuint64_t>(cols), static_cast<cuuint64_t>(rows), static_cast<cuuint64_t>(batch)};
    const cuuint64_t strides[2] = {static_cast<cuuint64_t>(ld) * 2, static_cast<cuuint64_t>(ld) * rows * 2};
    const cuuint32_t box[3] = {kBK, box_rows, 1};
    const cuuint32_t elem_strides[3] = {1, 1, 1};
    return tensor_map_encoder()(m, CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 3, const_cast<__half *>(base), dims, strides, box, elem_strides,
                                CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                                CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

bool aligned(const void *ptr, size_t bytes) { return reinterpret_cast<uintptr_t>(ptr) % bytes == 0; }

}  // namespace

struct orthogonal {
    int rows = 0, cols = 0, steps = 0, type = 0;
    float a = 0, b = 0, c = 0, eps = 0;
    int device = 0, sms = 0, pairs = 0;
    cudaStream_t stream = nullptr;
    int64_t launches = 0;
    int *err = nullptr;
};

namespace {

int short_side(const orthogonal *p) { return p->rows < p->cols ? p->rows : p->cols; }
int64_t pad8(int64_t v) { return div_up(v, 8) * 8; }
int64_t pad16(int64_t v) { return div_up(v, 16) * 16; }

// Everything a call keeps between its kernels.
struct Layout {
    int64_t ld, ldk, dk;
    size_t hi[2], lo[2], o, p, d, e, squares, total;
};

Layout layout_of(const orthogonal *p, int64_t batch)
{
    Layout w = {};
    const int64_t k = short_side(p);
    w.ld = pad8(p->cols);
    w.ldk = pad8(k);
    w.dk = pad16(k);
    size_t at = 0;
    auto take = [&](size_t bytes) {
        const size_t here = at;
        at += (bytes + 255) & ~static_cast<size_t>(255);
        return here;
    };
    const size_t x = static_cast<size_t>(batch) * p->rows * w.ld * 2, s = static_cast<size_t>(batch) * k * w.ldk * 2;
    for (int i = 0; i < 2; ++i) {
        w.hi[i] = take(x);
        w.lo[i] = take(x);
    }
    w.o = take(s);
    w.p = take(s);
    w.d = take(static_cast<size_t>(batch) * w.dk * 4);
    w.e = take(static_cast<size_t>(batch) * w.dk * 4);
    w.squares = take(static_cast<size_t>(batch) * kMostParts * sizeof(double));
    w.total = at;
    return w;
}

// Column tiles of the symmetric products, or all tiles, of an m x n result.
int64_t tiles_of(int64_t m, int64_t n, int tile_n, bool symmetric)
{
    const int64_t m_tiles = div_up(m, kTileM), n_tiles = div_up(n, tile_n);
    if (!symmetric) return m_tiles * n_tiles;
    int64_t tiles = 0;
    for (int64_t r = 0; r < m_tiles; ++r) tiles += n_tiles - r * (kTileM / tile_n);
    return tiles;
}

// Rounds of tiles times a tile's cost: half the columns cost more than half, since the rows of A are shared by fewer.
void choose_tile(const orthogonal *p, Product &q, bool symmetric)
{
    const int widths[3] = {256, 128, 64};
    int64_t best = -1;
    for (int w : widths) {
        const int64_t tiles = tiles_of(q.m, q.n, w, symmetric);
        const int64_t cost = div_up(tiles * q.batch, p->pairs) * (w + 128);
        if (best < 0 || cost < best) {
            best = cost;
            q.tile_n = w;
            q.tiles = static_cast<int>(tiles);
        }
    }
    q.m_tiles = static_cast<int>(div_up(q.m, kTileM));
    q.n_tiles = static_cast<int>(div_up(q.n, q.tile_n));
    q.steps = static_cast<int>(div_up(q.k, kBK));
}

template <typename... Params, typename... Args>
bool launch_after(cudaStream_t stream, dim3 grid, unsigned threads, size_t smem, bool pairs, void (*kernel)(Params...), const Args &...args)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = 2;
    attr[1].val.clusterDim.y = 1;
    attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = pairs ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, kernel, args...) == cudaSuccess;
}

// An operand of a product: a stack of [rows][cols] matrices, read along or across its rows.
struct Operand {
    const __half *base;
    int64_t rows, cols, ld;
    int by_rows;             // 1: the reduction runs down the rows
};

template <int kMode>
bool launch_product(orthogonal *p, Product q, const Operand &a, const Operand &b)
{
    q.a_rows = a.by_rows;
    q.b_rows = b.by_rows;
    CUtensorMap tm_a, tm_b;
    if (!encode(&tm_a, a.base, q.batch, a.rows, a.cols, a.ld, a.by_rows ? kBK : kRowsPerBlock) ||
        !encode(&tm_b, b.base, q.batch, b.rows, b.cols, b.ld, b.by_rows ? kBK : q.tile_n / 2))
        return false;
    const int64_t all = static_cast<int64_t>(q.tiles) * q.batch;
    const unsigned pairs = static_cast<unsigned>(all < p->pairs ? all : p->pairs);
    if (!launch_after(p->stream, dim3(2 * pairs), kThreads, kSmem, true, k_product<kMode>, tm_a, tm_b, q)) return false;
    p->launches += 1;
    return true;
}

template <typename T>
int run(orthogonal *p, const T *g, int64_t g_batch, int64_t g_row, __nv_bfloat16 *out, int64_t out_batch, int64_t out_row,
        uint8_t *base, int64_t batch)
{
    const Layout w = layout_of(p, batch);
    const int k = short_side(p);
    const bool tall = p->rows > p->cols;
    auto half = [&](size_t at) { return reinterpret_cast<__half *>(base + at); };
    auto single = [&](size_t at) { return reinterpret_cast<float *>(base + at); };

    Start s = {};
    s.rows = p->rows;
    s.cols = p->cols;
    s.ld = static_cast<int>(w.ld);
    // about eight pieces per thread
    const int64_t parts = div_up(static_cast<int64_t>(p->rows) * (w.ld / 8), 8 * kRowThreads);
    s.parts = static_cast<int>(parts < kMostParts ? parts : kMostParts);
    s.g_batch = g_batch;
    s.g_row = g_row;
    s.whole = aligned(g, 16) && (p->rows == 1 || g_row * sizeof(T) % 16 == 0) && (batch == 1 || g_batch * sizeof(T) % 16 == 0);
    s.eps = p->eps;
    s.squares = reinterpret_cast<double *>(base + w.squares);
    s.hi = half(w.hi[0]);
    s.lo = half(w.lo[0]);
    const dim3 grid(static_cast<unsigned>(s.parts), static_cast<unsigned>(batch));
    k_squares<T><<<grid, kRowThreads, 0, p->stream>>>(s, g);
    if (cudaGetLastError() != cudaSuccess) return ORTHOGONAL_ECUDA;
    if (!launch_after(p->stream, grid, kRowThreads, 0, false, k_start<T>, s, g)) {
        cudaGetLastError();
        return ORTHOGONAL_ECUDA;
    }
    p->launches += 2;

    Product q = {};
    q.batch = static_cast<int>(batch);
    q.tall = tall;
    q.ld = static_cast<int>(w.ld);
    q.ldk = static_cast<int>(w.ldk);
    q.dk = static_cast<int>(w.dk);
    q.a = p->a;
    q.b = p->b;
    q.c = p->c;
    q.o = half(w.o);
    q.p = half(w.p);
    q.d = single(w.d);
    q.e = single(w.e);
    q.out = out;
    q.out_batch = out_batch;
    q.out_row = out_row;
    q.out_whole = p->cols % 8 == 0 && aligned(out, 16) && (p->rows == 1 || out_row % 8 == 0) && (batch == 1 || out_batch % 8 == 0);
    q.err = p->err;
    Product gram = q, square = q, apply = q;
    gram.m = gram.n = square.m = square.n = square.k = k;
    gram.k = tall ? p->rows : p->cols;
    apply.m = p->rows;
    apply.n = p->cols;
    apply.k = k;
    choose_tile(p, gram, true);
    choose_tile(p, square, true);
    choose_tile(p, apply, false);
    const Operand o = {q.o, k, k, w.ldk, 0}, pp = {q.p, k, k, w.ldk, 0};
    for (int i = 0; i < p->steps; ++i) {
        const __half *hi = half(w.hi[i & 1]);
        const Operand x = {hi, p->rows, p->cols, w.ld, 0}, xt = {hi, p->rows, p->cols, w.ld, 1};
        apply.hi = hi;
        apply.lo = half(w.lo[i & 1]);
        apply.hi_next = half(w.hi[(i + 1) & 1]);
        apply.lo_next = half(w.lo[(i + 1) & 1]);
        const bool last = i + 1 == p->steps;
        const bool ok = launch_product<kGram>(p, gram, tall ? xt : x, tall ? xt : x) && launch_product<kSquare>(p, square, o, o) &&
                        (last ? launch_product<kLast>(p, apply, tall ? x : pp, tall ? pp : xt)
                              : launch_product<kApply>(p, apply, tall ? x : pp, tall ? pp : xt));
        if (!ok) {
            cudaGetLastError();
            return ORTHOGONAL_ECUDA;
        }
    }
    return ORTHOGONAL_OK;
}

bool batch_ok(const orthogonal *p, int64_t batch)
{
    // matrices and tiles are 32-bit in the kernels, and a grid's second dimension counts matrices
    return batch >= 1 && batch <= 65535 &&
           batch * div_up(p->rows, kTileM) * div_up(p->cols, 64) < 0x7FFFFFFF;
}

bool prepare_kernels(int *pairs, int sms)
{
    if (!raise_dynamic_smem(reinterpret_cast<const void *>(k_product<kGram>), kSmem) ||
        !raise_dynamic_smem(reinterpret_cast<const void *>(k_product<kSquare>), kSmem) ||
        !raise_dynamic_smem(reinterpret_cast<const void *>(k_product<kApply>), kSmem) ||
        !raise_dynamic_smem(reinterpret_cast<const void *>(k_product<kLast>), kSmem))
        return false;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(sms & ~1));
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = kSmem;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = 2;
    attr[0].val.clusterDim.y = 1;
    attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    int clusters = 0;
    if (cudaOccupancyMaxActiveClusters(&clusters, k_product<kGram>, &cfg) != cudaSuccess || clusters < 1) return false;
    *pairs = clusters < sms / 2 ? clusters : sms / 2;
    return true;
}

}  // namespace

extern "C" {

int orthogonal_create(orthogonal **out, int rows, int cols, int steps, float a, float b, float c, float eps, int type)
{
    if (out == nullptr) return ORTHOGONAL_ENULL;
    *out = nullptr;
    if (rows < 1 || rows > ORTHOGONAL_MAX_SIDE || cols < 1 || cols > ORTHOGONAL_MAX_SIDE) return ORTHOGONAL_EINVAL;
    if (steps < 1 || steps > ORTHOGONAL_MAX_STEPS) return ORTHOGONAL_EINVAL;
    if (!std::isfinite(a) || !std::isfinite(b) || !std::isfinite(c) || !std::isfinite(eps) || !(eps > 0.0f)) return ORTHOGONAL_EINVAL;
    if (type != ORTHOGONAL_F32 && type != ORTHOGONAL_BF16 && type != ORTHOGONAL_F16) return ORTHOGONAL_EINVAL;
    if (tensor_map_encoder() == nullptr) return ORTHOGONAL_ECUDA;
    orthogonal *p = new (std::nothrow) orthogonal;
    if (p == nullptr) return ORTHOGONAL_ENOMEM;
    p->rows = rows;
    p->cols = cols;
    p->steps = steps;
    p->a = a;
    p->b = b;
    p->c = c;
    p->eps = eps;
    p->type = type;
    if (cudaGetDevice(&p->device) != cudaSuccess ||
        cudaDeviceGetAttribute(&p->sms, cudaDevAttrMultiProcessorCount, p->device) != cudaSuccess ||
        !prepare_kernels(&p->pairs, p->sms)) {
        cudaGetLastError();
        delete p;
        return ORTHOGONAL_ECUDA;
    }
    if (cudaMalloc(reinterpret_cast<void **>(&p->err), sizeof(int)) != cudaSuccess) {
        cudaGetLastError();
        delete p;
        return ORTHOGONAL_ENOMEM;
    }
    if (cudaMemset(p->err, 0, sizeof(int)) != cudaSuccess) {
        cudaGetLastError();
        cudaFree(p->err);
        delete p;
        return ORTHOGONAL_ECUDA;
    }
    *out = p;
    return ORTHOGONAL_OK;
}

int orthogonal_destroy(orthogonal *p)
{
    if (p == nullptr) return ORTHOGONAL_ENULL;
    const OnDevice on(p->device);
    cudaStreamSynchronize(p->stream);
    cudaFree(p->err);
    delete p;
    return ORTHOGONAL_OK;
}

int orthogonal_set_stream(orthogonal *p, void *cuda_stream)
{
    if (p == nullptr) return ORTHOGONAL_ENULL;
    p->stream = static_cast<cudaStream_t>(cuda_stream);
    return ORTHOGONAL_OK;
}

size_t orthogonal_workspace_bytes(const orthogonal *p, int64_t batch)
{
    if (p == nullptr || !batch_ok(p, batch)) return 0;
    return layout_of(p, batch).total;
}

int orthogonal_update(orthogonal *p, const void *g, int64_t g_stride_batch, int64_t g_stride_row, void *update,
                      int64_t update_stride_batch, int64_t update_stride_row, void *workspace, size_t workspace_bytes,
                      int64_t batch)
{
    if (p == nullptr) return ORTHOGONAL_ENULL;
    if (!batch_ok(p, batch)) return ORTHOGONAL_EINVAL;     // first: an empty batch comes without pointers
    if (g == nullptr || update == nullptr || workspace == nullptr) return ORTHOGONAL_ENULL;
    if (g_stride_batch < 0 || g_stride_row < 0) return ORTHOGONAL_EINVAL;
    if (p->rows > 1 && update_stride_row < p->cols) return ORTHOGONAL_EINVAL;
    // the update's matrices one behind the other
    if (batch > 1 && update_stride_batch < (p->rows - 1) * (p->rows > 1 ? update_stride_row : 0) + p->cols) return ORTHOGONAL_EINVAL;
    if (!aligned(g, p->type == ORTHOGONAL_F32 ? 4 : 2) || !aligned(update, 2) || !aligned(workspace, 256)) return ORTHOGONAL_EALIGN;
    if (orthogonal_workspace_bytes(p, batch) > workspace_bytes) return ORTHOGONAL_ENOMEM;
    const OnDevice on(p->device);
    if (!on.ok()) return ORTHOGONAL_ECUDA;
    __nv_bfloat16 *out = static_cast<__nv_bfloat16 *>(update);
    uint8_t *base = static_cast<uint8_t *>(workspace);
    if (p->type == ORTHOGONAL_F32)
        return run(p, static_cast<const float *>(g), g_stride_batch, g_stride_row, out, update_stride_batch, update_stride_row, base, batch);
    if (p->type == ORTHOGONAL_BF16)
        return run(p, static_cast<const __nv_bfloat16 *>(g), g_stride_batch, g_stride_row, out, update_stride_batch, update_stride_row,
                   base, batch);
    return run(p, static_cast<const __half *>(g), g_stride_batch, g_stride_row, out, update_stride_batch, update_stride_row, base, batch);
}

int orthogonal_status(orthogonal *p)
{
    if (p == nullptr) return ORTHOGONAL_ENULL;
    const OnDevice on(p->device);
    if (!on.ok() || cudaStreamSynchronize(p->stream) != cudaSuccess) return ORTHOGONAL_ECUDA;
    int flag = 0;
    if (cudaMemcpy(&flag, p->err, sizeof(int), cudaMemcpyDeviceToHost) != cudaSuccess) return ORTHOGONAL_ECUDA;
    if (flag != 0) {
        cudaMemset(p->err, 0, sizeof(int));
        return ORTHOGONAL_ETIMEOUT;
    }
    return ORTHOGONAL_OK;
}

int64_t orthogonal_launch_count(const orthogonal *p) { return p ? p->launches : 0; }

const char *orthogonal_strerror(int code)
{
    switch (code) {
    case ORTHOGONAL_OK: return "ok";
    case ORTHOGONAL_EINVAL: return "invalid size, stride, type, steps, coefficient or eps";
    case ORTHOGONAL_ENULL: return "required pointer is NULL";
    case ORTHOGONAL_EALIGN: return "pointer not aligned to its element";
    case ORTHOGONAL_ECUDA: return "CUDA call or launch failed";
    case ORTHOGONAL_ENOMEM: return "allocation failed, or the workspace is too small";
    case ORTHOGONAL_ETIMEOUT: return "a kernel gave up a bounded wait; its output is invalid";
    default: return "unknown error";
    }
}

}  // extern "C"
