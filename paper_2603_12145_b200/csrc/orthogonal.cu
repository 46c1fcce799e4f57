// orthogonal.cu -- the orthogonalised update behind the C ABI of orthogonal.h, on sm_100a tensor cores.
//
// A step of the iteration is three matrix products D = A B^T with an epilogue each:
//
//   gram      A = X X^T.  Symmetric: only tiles with elements on or above the diagonal are computed, and each element
//             above it is written to both places.  Off the diagonal binary16 (O), on it binary32 (d) and a zero in O.
//   square    B = b A + c A A, symmetric too.  A = diag(d) + O, so A A = O O + (d_i + d_j) O_ij off the diagonal, O O + d_i^2 on
//             it: the product has O alone, the rest is binary32 in the epilogue.  B again as P (binary16) and e (binary32).
//   apply     X' = (a + e_i) X + P X, with X as the pair hi + lo in the first term and hi as the operand; the last step
//             writes the update instead.
//
// k_iterate runs all of them in one launch, on CTA pairs that stay (tcgen05, cta_group::2): a pair's tile is 256 rows of A
// by 64, 128 or 256 rows of B; each block of the pair stages 128 rows of A and half of the rows of B per 64 reduction
// elements, the leader issues M = 256 instructions into one of two accumulator buffers, and eight epilogue warps per block
// empty the other one meanwhile.  Where a product has fewer tiles than there are pairs, two or four pairs of a cluster share
// a tile's reduction and exchange their parts through distributed shared memory.  Between products all blocks wait for a
// counter in memory.  k_squares and k_start bring G into X first.  A matrix whose short side is at most 128 takes k_small
// instead: the whole iteration in the shared memory of one cluster.
//
// What bounds it, on a B200 (five steps): 2,048 x 8,192 in bfloat16 takes 630 to 645 us, 720 at the power cap, for 0.56 TFLOP (890
// and 775 TFLOP/s): a last round of tiles that not all pairs have, epilogues and waits between products.  1,728 x 576 in
// binary32 takes 127 us: fifteen products of 8 us each, of which the operands' way from L2 (about 80 KB a microsecond into each
// SM) is a third and the rest is latency: the wait for all blocks 1.3 us, first loads 0.6, epilogue, stores and their
// fence 3.  As separate launches, each started while the one before ends, it took 181 us (and 855 for 2,048 x 8,192).
// Eight matrices 384 x 64 take 33 us in k_small.
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
constexpr int kABytes = kRowsPerBlock * kBK * 2;
constexpr int kRing = 5 * 32 * 1024;             // stages take turns in it: five of 256 columns, up to eight of fewer
constexpr int kStages = 8;
constexpr int kAccCols = 256;
constexpr int kTmemCols = 2 * kAccCols;
constexpr int kEpilogueWarps = 8;
constexpr int kThreads = 64 + 32 * kEpilogueWarps;
// Pairs that may share a tile's reduction, in a cluster of four or eight blocks, and the columns of such a tile, at most.
constexpr int kShares[2] = {2, 4};
__host__ __device__ constexpr int share_cols(int share) { return share == 2 ? 256 : 128; }
__host__ __device__ constexpr int exchange_bytes(int share) { return (share - 1) * kRowsPerBlock * (share_cols(share) / share) * 4; }
constexpr int kBlock = 32 * 64;                  // 32 rows x 32 columns of 16 bits on their way between registers and memory
constexpr int kSets = 2;                         // per epilogue warp: one worked on, the other on its way in; two planes each
constexpr int kStaging = 2 * kSets * kBlock;
// (what pairs exchange and what is staged take turns: a product does one or the other)
constexpr int kBesides = kEpilogueWarps * kStaging;
constexpr int kBarrierBytes = 512;
constexpr int kColumns = kEpilogueWarps * 32 * 4;   // per epilogue warp: the diagonal's elements of its 32 columns
constexpr int kSmem = kRing + kBesides + kBarrierBytes + kColumns + 1024;
static_assert(kSmem <= 227 * 1024 && exchange_bytes(2) <= kBesides && exchange_bytes(4) <= kBesides, "shared memory of a block");

constexpr int kRowThreads = 256;                 // blocks of the kernels that read and write rows
constexpr int kMostParts = 592;                  // partial sums of squares per matrix

// X is held times 2^13: an element of a normalised matrix of a million is about 2^-10, and hi + lo then has 22 bits of it.  A
// and B are held as they are (up to 3 in magnitude; what is below binary16's normal numbers, 2^-14, is off by 2^-25 at most).
constexpr float kScale = 8192.0f;
constexpr float kUnscale = 1.0f / kScale;
constexpr float kUnscale2 = kUnscale * kUnscale;

// A product of the iteration, and how it is cut.
struct Product {
    int m, n, k;            // rows of A, rows of B, reduction length, of one matrix
    int a_rows, b_rows;     // 1: the operand is stored [k][rows] (MN-major), 0: [rows][k]
    int symmetric;          // only tiles with elements on or above the diagonal
    int tile_n;             // columns of D per tile: 256, 128 or 64
    int m_tiles, n_tiles;
    int tiles;              // of one matrix: those that are computed
    int steps;              // ceil(k / 64)
    int shared;             // 1: the pairs of a cluster share each tile's reduction
};

struct Iteration {
    Product gram, square, apply;
    int batch, steps;
    int tall;               // rows > cols: the diagonal's factors go with columns
    int share;              // pairs per cluster: 1, 2 or 4
    int ldk;                // of O and P
    int dk;                 // elements between the diagonals of two matrices
    float a, b, c;
    __half *o, *p;
    float *d, *e;
    __half *hi[2], *lo[2];
    __nv_bfloat16 *out;
    int64_t out_batch, out_row;
    int out_whole;          // rows of the update start on 16-byte boundaries
    unsigned *arrived;      // blocks that have finished a product, all products so far
    int *err;
};

// The operands, by product and by which of X's two places holds it; and blocks of 32 x 32 of what the epilogues read and write.
struct Maps {
    CUtensorMap gram_a[2], gram_b[2], square_a, square_b, apply_a[2], apply_b[2];
    CUtensorMap hi[2], lo[2], o, p, out;
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

// The mbarrier at this shared-memory offset in both blocks of the pair whose first block has rank `leader` in the cluster
// receives one arrival once every instruction issued so far by this thread is done.
__device__ __forceinline__ void umma_commit(uint32_t bar, uint32_t leader)
{
    asm volatile(
        "tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar),
        "h"(static_cast<uint16_t>(3u << leader))
        : "memory");
}

struct Tile {
    int z, row, col;         // matrix, first row and column
};

// Symmetric products: row block I has the column tiles from the one of its first diagonal element on.
__device__ __forceinline__ Tile tile_at(const Product &p, int index)
{
    Tile t;
    t.z = index / p.tiles;
    int i = index - t.z * p.tiles;
    if (p.symmetric) {
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

// Bytes of the columns' operand in a stage: whole boxes of 64 columns where the reduction runs along rows.
__device__ __forceinline__ uint32_t b_bytes(const Product &p)
{
    const int half = p.tile_n / 2;
    return static_cast<uint32_t>(p.b_rows ? (half + 63) / 64 * 64 : half) * kBK * 2;
}

// Which tiles a pair works on, and which steps of their reduction.
struct Walk {
    int index, step, end, k0, k1;
    __device__ Walk(const Iteration &q, const Product &p)
    {
        const int pair = static_cast<int>(blockIdx.x >> 1), pairs = static_cast<int>(gridDim.x >> 1);
        const int sub = p.shared ? pair % q.share : 0;
        index = p.shared ? pair / q.share : pair;
        step = p.shared ? pairs / q.share : pairs;
        end = p.tiles * q.batch;
        k0 = p.shared ? p.steps * sub / q.share : 0;
        k1 = p.shared ? p.steps * (sub + 1) / q.share : p.steps;
    }
};

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

// Elements (i, j0 .. j0 + 15) of a symmetric matrix of k rows to their places across the diagonal; neighbouring lanes have
// neighbouring rows.
__device__ __forceinline__ void store_mirrored(__half *base, int ldk, int k, int i, int j0, const uint32_t (&w)[8])
{
    if (i >= k) return;
    uint16_t *dst = reinterpret_cast<uint16_t *>(base + static_cast<int64_t>(j0) * ldk + i);
#pragma unroll
    for (int q = 0; q < 16; ++q) {
        if (j0 + q < k) *dst = static_cast<uint16_t>(q & 1 ? w[q / 2] >> 16 : w[q / 2]);
        dst += ldk;
    }
}

// The lane's row of a staged block (64-byte swizzle): 16-byte piece i.
__device__ __forceinline__ uint32_t piece16(uint32_t block, int lane, int i) { return block + lane * 64 + ((i ^ ((lane >> 1) & 3)) << 4); }

__device__ __forceinline__ void put16(uint32_t block, int lane, int h, const uint32_t (&w)[8])
{
#pragma unroll
    for (int i = 0; i < 2; ++i)
        asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(piece16(block, lane, 2 * h + i)), "r"(w[4 * i]), "r"(w[4 * i + 1]),
                     "r"(w[4 * i + 2]), "r"(w[4 * i + 3])
                     : "memory");
}

__device__ __forceinline__ void get16(uint32_t block, int lane, int h, uint32_t (&w)[8])
{
#pragma unroll
    for (int i = 0; i < 2; ++i)
        asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];"
                     : "=r"(w[4 * i]), "=r"(w[4 * i + 1]), "=r"(w[4 * i + 2]), "=r"(w[4 * i + 3])
                     : "r"(piece16(block, lane, 2 * h + i))
                     : "memory");
}

// A 32 x 32 block of matrix z, with this block's own barrier.
__device__ __forceinline__ void tma_load_block(uint32_t dst, const CUtensorMap *map, int x, int y, int z, uint32_t bar)
{
    asm volatile(
        "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(dst),
        "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar)
        : "memory");
}

__device__ __forceinline__ void prefetch_map(const CUtensorMap *map) { asm volatile("prefetch.tensormap [%0];" ::"l"(map) : "memory"); }

__device__ __forceinline__ void tma_store_block(const CUtensorMap *map, int x, int y, int z, uint32_t src)
{
    asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.tile.bulk_group [%0, {%1, %2, %3}], [%4];" ::"l"(map), "r"(x), "r"(y),
                 "r"(z), "r"(src)
                 : "memory");
}

__device__ __forceinline__ void bulk_commit() { asm volatile("cp.async.bulk.commit_group;" ::: "memory"); }
// The copies' reads of shared memory are done.
__device__ __forceinline__ void bulk_wait_read() { asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory"); }
__device__ __forceinline__ void bulk_wait() { asm volatile("cp.async.bulk.wait_group 0;" ::: "memory"); }
__device__ __forceinline__ void fence_async() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

__device__ __forceinline__ unsigned load_acquire(const unsigned *p)
{
    unsigned v;
    asm volatile("ld.acquire.gpu.global.u32 %0, [%1];" : "=r"(v) : "l"(p) : "memory");
    return v;
}

__device__ __forceinline__ void add_release(unsigned *p)
{
    asm volatile("red.release.gpu.global.add.u32 [%0], 1;" ::"l"(p) : "memory");
}

__device__ __forceinline__ unsigned add_acq_rel(uint32_t p)
{
    unsigned v;
    asm volatile("atom.acq_rel.cta.shared::cta.add.u32 %0, [%1], 1;" : "=r"(v) : "r"(p) : "memory");
    return v;
}

// Waits until `target` blocks have finished; gives up as mbar_wait does.
__device__ bool wait_arrived(const unsigned *arrived, unsigned target, volatile int *abort_flag)
{
    unsigned long long t0 = 0;
    for (uint32_t spin = 0;; ++spin) {
        if (load_acquire(arrived) >= target) return true;
        if ((spin & 63u) == 63u) {
            if (*abort_flag) return false;
            const unsigned long long now = global_timer_ns();
            if (t0 == 0) {
                t0 = now;
            } else if (now - t0 > kWaitLimitNs) {
                *abort_flag = 1;
                return false;
            }
        }
    }
}

__device__ __forceinline__ void mbar_arrive(uint32_t bar)
{
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}

// What this thread (and those it synchronised with) wrote to the other block's shared memory is there for who waits.
__device__ __forceinline__ void mbar_arrive_release_cluster(uint32_t cluster_addr)
{
    asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(cluster_addr) : "memory");
}

// mbar_wait for a barrier on which other blocks of the cluster arrive, having written to this one's shared memory.
__device__ bool mbar_wait_cluster(uint32_t bar, uint32_t parity, volatile int *abort_flag)
{
    unsigned long long t0 = 0;
    for (uint32_t spin = 0;; ++spin) {
        uint32_t ok;
        asm volatile(
            "{\n\t.reg .pred p;\n\t"
            "mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n\t"
            "selp.u32 %0, 1, 0, p;\n\t}"
            : "=r"(ok)
            : "r"(bar), "r"(parity)
            : "memory");
        if (ok) return true;
        if ((spin & 63u) == 63u) {
            if (*abort_flag) return false;
            const unsigned long long now = global_timer_ns();
            if (t0 == 0) {
                t0 = now;
            } else if (now - t0 > kWaitLimitNs) {
                *abort_flag = 1;
                return false;
            }
        }
    }
}

__device__ __forceinline__ void store_remote(uint32_t cluster_addr, const uint32_t *v)
{
    asm volatile("st.shared::cluster.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(cluster_addr), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3])
                 : "memory");
}

__device__ __forceinline__ float4 load_shared4(uint32_t addr)
{
    float4 v;
    asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr) : "memory");
    return v;
}

// ---- epilogues: elements (row, j0 .. j0 + 15) of a product to what is stored of them.  Rows and columns past
// the matrix go along; nothing of them is kept.

// A from the products of X, to O with a zero on the diagonal, which goes to d
__device__ __forceinline__ void finish_gram(const Iteration &q, int z, int row, int j0, const float (&acc)[16], uint32_t (&w)[8])
{
    float v[16];
#pragma unroll
    for (int e = 0; e < 16; ++e) v[e] = acc[e] * kUnscale2;
    if (j0 <= row && row < j0 + 16 && row < q.gram.m) {
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            if (j0 + e == row) {
                q.d[static_cast<int64_t>(z) * q.dk + row] = v[e];
                v[e] = 0.0f;
            }
        }
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) w[e] = pack2(v[2 * e], v[2 * e + 1]);
}

// B from O's products, O itself and the diagonal d, of which di is the row's and d the columns': likewise to P and e.  w: O in, P out.
__device__ __forceinline__ void finish_square(const Iteration &q, int z, int row, int j0, float di, const float *d, const float (&acc)[16], uint32_t (&w)[8])
{
    if (j0 >= q.gram.m) return;
    const int64_t diagonal = static_cast<int64_t>(z) * q.dk;
    float v[16];
#pragma unroll
    for (int e = 0; e < 16; e += 4) {
        // (the diagonals are padded to whole pieces of 16)
        const float4 dj = *reinterpret_cast<const float4 *>(d + e);
        const float2 o0 = unpack2(w[e / 2]), o1 = unpack2(w[e / 2 + 1]);
        const float o[4] = {o0.x, o0.y, o1.x, o1.y}, ds[4] = {dj.x, dj.y, dj.z, dj.w};
#pragma unroll
        for (int f = 0; f < 4; ++f) v[e + f] = fmaf(q.c, fmaf(di + ds[f], o[f], acc[e + f]), q.b * o[f]);
    }
    if (j0 <= row && row < j0 + 16 && row < q.gram.m) {
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            if (j0 + e == row) {
                q.e[diagonal + row] = fmaf(q.c, fmaf(di, di, acc[e]), q.b * di);
                v[e] = 0.0f;
            }
        }
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) w[e] = pack2(v[2 * e], v[2 * e + 1]);
}

// X' from X = hi + lo in, hi and lo out; of the last product the update instead of hi.  factor: a, and e of the row where the
// diagonal goes with rows; by_columns: e where it goes with columns, else nullptr.
__device__ __forceinline__ void finish_apply(const Iteration &q, bool last, float factor, const float *by_columns, const float (&acc)[16],
                                             uint32_t (&hi)[8], uint32_t (&lo)[8])
{
    float v[16];
#pragma unroll
    for (int e = 0; e < 16; e += 4) {
        float f[4] = {factor, factor, factor, factor};
        if (by_columns != nullptr) {
            const float4 ej = *reinterpret_cast<const float4 *>(by_columns + e);
            f[0] += ej.x, f[1] += ej.y, f[2] += ej.z, f[3] += ej.w;
        }
#pragma unroll
        for (int g = 0; g < 4; g += 2) {
            const float2 h = unpack2(hi[(e + g) / 2]), l = unpack2(lo[(e + g) / 2]);
            v[e + g] = fmaf(f[g], h.x + l.x, acc[e + g]);
            v[e + g + 1] = fmaf(f[g + 1], h.y + l.y, acc[e + g + 1]);
        }
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        if (last) {
            hi[e] = pack_bf16(v[2 * e] * kUnscale, v[2 * e + 1] * kUnscale);
        } else {
            hi[e] = pack2(v[2 * e], v[2 * e + 1]);
            const float2 h = unpack2(hi[e]);
            lo[e] = pack2(v[2 * e] - h.x, v[2 * e + 1] - h.y);
        }
    }
}

// The whole iteration: one block per SM, all at once on the device; blocks wait for one another between products.
__global__ void __launch_bounds__(kThreads, 1)
k_iterate(const __grid_constant__ Maps maps, const __grid_constant__ Iteration q)
{
    extern __shared__ uint8_t smem_raw[];
    const uint32_t raw = smem_u32(smem_raw);
    const uint32_t stages = (raw + 1023u) & ~1023u;
    const uint32_t besides = stages + kRing;
    const uint32_t bars = besides + kBesides;
    uint8_t *bars_ptr = smem_raw + (bars - raw);
    const uint32_t full0 = bars, empty0 = bars + 8 * kStages;
    const uint32_t acc_full0 = bars + 16 * kStages, acc_empty0 = acc_full0 + 16;
    const uint32_t ready = acc_empty0 + 16, received = ready + 8, staged0 = received + 8;        // the last: kSets per epilogue warp
    uint8_t *words = bars_ptr + 16 * kStages + 48 + 8 * kSets * kEpilogueWarps;
    volatile uint32_t *tmem_slot = reinterpret_cast<volatile uint32_t *>(words);
    volatile int *abort_flag = reinterpret_cast<volatile int *>(words + 4);
    unsigned *finished = reinterpret_cast<unsigned *>(words + 8);     // epilogue warps, all products so far

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t cluster_rank = cluster_cta_rank(), rank = cluster_rank & 1;            // pairs are neighbours in the cluster
    const uint32_t leader = cluster_rank & ~1u;

    if (threadIdx.x == 0) {
        for (int s = 0; s < kStages; ++s) {
            mbar_init(full0 + 8 * s, 1);
            mbar_init(empty0 + 8 * s, 1);
        }
        for (int b = 0; b < 2; ++b) {
            mbar_init(acc_full0 + 8 * b, 1);
            mbar_init(acc_empty0 + 8 * b, 2 * kEpilogueWarps);
        }
        mbar_init(ready, 1);
        mbar_init(received, q.share > 1 ? (q.share - 1) * kEpilogueWarps / 2 : 1);
        for (int i = 0; i < kSets * kEpilogueWarps; ++i) mbar_init(staged0 + 8 * i, 1);
        *abort_flag = 0;
        *finished = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    if (warp == 1) tmem_alloc(smem_u32(const_cast<uint32_t *>(tmem_slot)), kTmemCols);
    tc_fence_before_sync();
    cluster_sync_all();
    tc_fence_after_sync();
    const uint32_t tmem_base = *tmem_slot;

    const int products = 3 * q.steps;
    if (warp == 0) {
        if (lane == 0) {
            uint32_t used = 0;                           // bit s: parity of the stage's uses so far
            bool ok = true;
            for (int i = 0; ok && i < products; ++i) {
                const int kind = i % 3, from = i / 3 & 1;
                const Product &p = kind == 0 ? q.gram : kind == 1 ? q.square : q.apply;
                const CUtensorMap *tm_a = kind == 0 ? &maps.gram_a[from] : kind == 1 ? &maps.square_a : &maps.apply_a[from];
                const CUtensorMap *tm_b = kind == 0 ? &maps.gram_b[from] : kind == 1 ? &maps.square_b : &maps.apply_b[from];
                prefetch_map(tm_a);                      // (1 % at the middle sizes)
                prefetch_map(tm_b);
                if (i > 0) ok = wait_arrived(q.arrived, static_cast<unsigned>(i) * gridDim.x, abort_flag);
                mbar_arrive(ready);
                // some of the operands were written by plain stores (a fence of all memory: 137 against 130 us)
                asm volatile("fence.proxy.async.global;" ::: "memory");
                const int b_half = p.tile_n / 2, b_boxes = (b_half + 63) / 64;
                const uint32_t bytes = kABytes + b_bytes(p);
                const uint32_t depth = min(static_cast<uint32_t>(kStages), kRing / bytes);
                uint32_t s = 0;                          // (nothing of the last product is in the ring any more)
                for (Walk w(q, p); ok && w.index < w.end; w.index += w.step) {
                    const Tile t = tile_at(p, w.index);
                    const int a0 = t.row + static_cast<int>(rank) * kRowsPerBlock, b0 = t.col + static_cast<int>(rank) * b_half;
                    for (int kc = w.k0; kc < w.k1; ++kc) {
                        if (!mbar_wait(empty0 + 8 * s, ((used >> s) & 1) ^ 1u, abort_flag)) {
                            ok = false;
                            break;
                        }
                        const uint32_t dst = stages + s * bytes;
                        const uint32_t full = map_to_rank(full0 + 8 * s, leader);
                        if (rank == 0) mbar_expect_tx(full0 + 8 * s, 2 * bytes);
                        if (p.a_rows) {
                            tma_load_matrix(dst, tm_a, a0, kc * kBK, t.z, full);
                            tma_load_matrix(dst + kABytes / 2, tm_a, a0 + 64, kc * kBK, t.z, full);
                        } else {
                            tma_load_matrix(dst, tm_a, kc * kBK, a0, t.z, full);
                        }
                        if (p.b_rows) {
                            for (int b = 0; b < b_boxes; ++b)
                                tma_load_matrix(dst + kABytes + b * 64 * kBK * 2, tm_b, b0 + 64 * b, kc * kBK, t.z, full);
                        } else {
                            tma_load_matrix(dst + kABytes, tm_b, kc * kBK, b0, t.z, full);
                        }
                        used ^= 1u << s;
                        if (++s == depth) s = 0;
                    }
                }
            }
            // do not leave while the leader's instructions may still read this block's stages
            for (int s = 0; s < kStages && ok; ++s) ok = mbar_wait(empty0 + 8 * s, ((used >> s) & 1) ^ 1u, abort_flag);
        }
    } else if (warp == 1) {
        if (lane == 0 && rank == 0) {
            uint32_t used = 0;
            bool ok = true;
            int it = 0;
            for (int i = 0; ok && i < products; ++i) {
                const int kind = i % 3;
                const Product &p = kind == 0 ? q.gram : kind == 1 ? q.square : q.apply;
                const uint32_t idesc = (1u << 4) | (static_cast<uint32_t>(p.a_rows) << 15) | (static_cast<uint32_t>(p.b_rows) << 16) |
                                       (static_cast<uint32_t>(p.tile_n >> 3) << 17) | (static_cast<uint32_t>(kTileM >> 4) << 24);
                // 16 reduction elements: 32 bytes along a K-major row, 16 rows of 128 bytes MN-major
                const uint32_t a_step = p.a_rows ? 2048 >> 4 : 32 >> 4, b_step = p.b_rows ? 2048 >> 4 : 32 >> 4;
                const uint32_t bytes = kABytes + b_bytes(p), depth = min(static_cast<uint32_t>(kStages), kRing / bytes);
                uint32_t s = 0;
                for (Walk w(q, p); ok && w.index < w.end; w.index += w.step, ++it) {
                    const uint32_t buf = it & 1, use = (it >> 1) & 1;
                    if (!mbar_wait(acc_empty0 + 8 * buf, use ^ 1u, abort_flag)) {
                        ok = false;
                        break;
                    }
                    tc_fence_after_sync();
                    const uint32_t d = tmem_base + buf * kAccCols;
                    for (int kc = w.k0; kc < w.k1; ++kc) {
                        if (!mbar_wait(full0 + 8 * s, (used >> s) & 1, abort_flag)) {
                            ok = false;
                            break;
                        }
                        tc_fence_after_sync();
                        const uint32_t addr = stages + s * bytes;
                        const uint64_t ad = p.a_rows ? smem_desc_rows(addr) : smem_desc(addr);
                        const uint64_t bd = p.b_rows ? smem_desc_rows(addr + kABytes) : smem_desc(addr + kABytes);
#pragma unroll
                        for (int k = 0; k < kBK / 16; ++k)
                            umma_bf16(d, ad + a_step * k, bd + b_step * k, idesc, kc > w.k0 || k > 0);
                        umma_commit(empty0 + 8 * s, leader);
                        used ^= 1u << s;
                        if (++s == depth) s = 0;
                    }
                    if (ok) umma_commit(acc_full0 + 8 * buf, leader);
                }
            }
        }
    } else {
        const int quarter = warp & 3;
        const int half = (warp - 2) >> 2;                // which half of the columns
        const uint32_t lane_base = tmem_base + (static_cast<uint32_t>(quarter * 32) << 16);
        const int row_in_block = quarter * 32 + lane;
        const uint32_t stage = besides + (warp - 2) * kStaging, staged = staged0 + 8 * kSets * (warp - 2);
        float *columns = reinterpret_cast<float *>(bars_ptr + kBarrierBytes) + 32 * (warp - 2);
        uint32_t staged_phase = 0;                       // bit b: parity of the next arrival in set b
        bool ok = true;
        int it = 0, exchanges = 0;
        for (int i = 0; ok && i < products; ++i) {
            const int kind = i % 3, from = i / 3 & 1;
            const bool last = i + 1 == products;
            const Product &p = kind == 0 ? q.gram : kind == 1 ? q.square : q.apply;
            __half *symmetric = kind == 0 ? q.o : q.p;
            ok = __all_sync(0xFFFFFFFFu, mbar_wait(ready, i & 1, abort_flag));
            if (lane == 0) asm volatile("fence.proxy.async.global;" ::: "memory");
            for (Walk w(q, p); ok && w.index < w.end; w.index += w.step, ++it) {
                const uint32_t buf = it & 1, use = (it >> 1) & 1;
                const Tile t = tile_at(p, w.index);
                const int row0 = t.row + static_cast<int>(rank) * kRowsPerBlock + quarter * 32, row = row0 + lane;
                const bool live = row < p.m;
                const uint32_t t0 = lane_base + buf * kAccCols;
                const int64_t diagonal = static_cast<int64_t>(t.z) * q.dk;
                // the square blocks on the diagonal are computed whole, those above it are written to both places
                const bool mirrored = kind != 2 && t.col >= t.row + kTileM;
                const float factor = kind == 1 ? (live ? q.d[diagonal + row] : 0.0f)
                                               : kind == 2 && !q.tall && live ? q.a + q.e[diagonal + row] : q.a;
                if (!p.shared) {
                    const int sets = p.tile_n / 64, first = t.col + half * (p.tile_n / 2);
                    // set s, columns [first + 32 s, + 32) of what the epilogue reads, into buffer s % kSets
                    auto bring = [&](int s) {
                        const uint32_t dst = stage + (s % kSets) * (2 * kBlock), bar = staged + 8 * (s % kSets);
                        mbar_expect_tx(bar, kind == 1 ? kBlock : 2 * kBlock);
                        if (kind == 1) {
                            tma_load_block(dst, &maps.o, first + 32 * s, row0, t.z, bar);
                        } else {
                            tma_load_block(dst, &maps.hi[from], first + 32 * s, row0, t.z, bar);
                            tma_load_block(dst + kBlock, &maps.lo[from], first + 32 * s, row0, t.z, bar);
                        }
                    };
                    // d or e of the columns [first + 32 s, + 32), a set ahead
                    const float *diagonals = kind == 1 ? q.d + diagonal : kind == 2 && q.tall ? q.e + diagonal : nullptr;
                    auto fetch_column = [&](int s) {
                        const int c = first + 32 * s + lane;
                        return diagonals != nullptr && s < sets && c < p.n ? diagonals[c] : 0.0f;
                    };
                    float column = fetch_column(0);
                    if (lane == 0) {
                        bulk_wait_read();                // the buffers: the previous tile's results have left
                        if (kind != 0)
                            for (int s = 0; s < kSets && s < sets; ++s) bring(s);
                    }
                    __syncwarp();
                    ok = __all_sync(0xFFFFFFFFu, mbar_wait(acc_full0 + 8 * buf, use, abort_flag));
                    if (!ok) break;
                    tc_fence_after_sync();
#pragma unroll 1
                    for (int s = 0; s < sets; ++s) {
                        const uint32_t block = stage + (s % kSets) * (2 * kBlock);
                        const int f = first + 32 * s;
                        if (kind != 0) {
                            const bool here = mbar_wait(staged + 8 * (s % kSets), (staged_phase >> (s % kSets)) & 1, abort_flag);
                            staged_phase ^= 1u << (s % kSets);
                            ok = __all_sync(0xFFFFFFFFu, here);
                            if (!ok) break;
                        } else if (s >= kSets) {
                            if (lane == 0) bulk_wait_read();
                            __syncwarp();
                        }
                        if (diagonals != nullptr) {
                            columns[lane] = column;
                            column = fetch_column(s + 1);
                            __syncwarp();
                        }
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            uint32_t raw_acc[16], u[8], v[8];
                            tmem_ld16(t0 + half * (p.tile_n / 2) + 32 * s + 16 * h, raw_acc);
                            if (kind != 0) get16(block, lane, h, u);
                            if (kind == 2) get16(block + kBlock, lane, h, v);
                            tmem_wait_ld();
                            float acc[16];
#pragma unroll
                            for (int e = 0; e < 16; ++e) acc[e] = __uint_as_float(raw_acc[e]);
                            const int j0 = f + 16 * h;
                            if (kind == 0) finish_gram(q, t.z, row, j0, acc, u);
                            else if (kind == 1) finish_square(q, t.z, row, j0, factor, columns + 16 * h, acc, u);
                            else finish_apply(q, last, factor, q.tall ? columns + 16 * h : nullptr, acc, u, v);
                            if (last && !q.out_whole) {
                                __nv_bfloat16 *dst = q.out + t.z * q.out_batch + row * q.out_row;
                                if (live) {
#pragma unroll
                                    for (int e = 0; e < 16; ++e)
                                        if (j0 + e < p.n)
                                            *reinterpret_cast<uint16_t *>(dst + j0 + e) = static_cast<uint16_t>(e & 1 ? u[e / 2] >> 16 : u[e / 2]);
                                }
                                continue;
                            }
                            put16(block, lane, h, u);
                            if (kind == 2 && !last) put16(block + kBlock, lane, h, v);
                            if (mirrored) store_mirrored(symmetric + static_cast<int64_t>(t.z) * p.m * q.ldk, q.ldk, p.m, row, j0, u);
                        }
                        fence_async();
                        __syncwarp();
                        if (lane == 0) {
                            if (f < p.n && row0 < p.m && !(last && !q.out_whole)) {
                                const CUtensorMap *to = kind == 0 ? &maps.o : kind == 1 ? &maps.p : last ? &maps.out : &maps.hi[from ^ 1];
                                tma_store_block(to, f, row0, t.z, block);
                                if (kind == 2 && !last) tma_store_block(&maps.lo[from ^ 1], f, row0, t.z, block + kBlock);
                            }
                            bulk_commit();
                            if (kind != 0 && s + kSets < sets) {     // into this buffer
                                bulk_wait_read();
                                bring(s + kSets);
                            }
                        }
                        __syncwarp();
                    }
                    if (!ok) break;
                } else {
                    ok = __all_sync(0xFFFFFFFFu, mbar_wait(acc_full0 + 8 * buf, use, abort_flag));
                    if (!ok) break;
                    tc_fence_after_sync();
                    // the other pairs' parts go to them: [source][4 columns][row][4], a warp's stores are contiguous
                    const int part = p.tile_n / q.share, sub = static_cast<int>(cluster_rank >> 1);
                    for (int c = half * (p.tile_n / 2); c < (half + 1) * (p.tile_n / 2); c += 16) {
                        const int to = c / part;
                        if (to == sub) continue;
                        uint32_t acc[16];
                        tmem_ld16(t0 + c, acc);
                        tmem_wait_ld();
                        const int slot = sub < to ? sub : sub - 1;
                        const uint32_t base = map_to_rank(besides + (slot * (part / 4) + (c - to * part) / 4) * (kRowsPerBlock * 16) + row_in_block * 16,
                                                          2 * to + rank);
#pragma unroll
                        for (int e = 0; e < 4; ++e) store_remote(base + e * (kRowsPerBlock * 16), acc + 4 * e);
                    }
                    __syncwarp();
                    if (lane == 0) {
                        for (int to = 0; to < q.share; ++to) {
                            // (a part lies in one half of the tile's columns)
                            if (to != sub && to * part / (p.tile_n / 2) == half)
                                mbar_arrive_release_cluster(map_to_rank(received, 2 * to + rank));
                        }
                    }
                    const int c0 = sub * part + 16 * half, c1 = (sub + 1) * part;
                    const int64_t at = static_cast<int64_t>(t.z) * p.m * q.ldk + static_cast<int64_t>(live ? row : 0) * q.ldk;
                    ok = __all_sync(0xFFFFFFFFu, mbar_wait_cluster(received, exchanges & 1, abort_flag));
                    ++exchanges;
                    if (!ok) break;
#pragma unroll 1
                    for (int c = c0; c < c1; c += 32) {
                        const int j0 = t.col + c;
                        uint32_t raw_acc[16], u[8] = {0, 0, 0, 0, 0, 0, 0, 0};
                        tmem_ld16(t0 + c, raw_acc);
                        if (kind == 1 && live) load16(u, q.o + at, j0, q.ldk);
                        tmem_wait_ld();
                        // in the order of the reduction: the parts before this pair's, its own, those after it
                        float acc[16];
#pragma unroll
                        for (int e = 0; e < 16; ++e) acc[e] = 0.0f;
                        for (int src = 0; src < q.share; ++src) {
                            const int slot = src < sub ? src : src - 1;
                            const uint32_t base = besides + (slot * (part / 4) + (c - sub * part) / 4) * (kRowsPerBlock * 16) + row_in_block * 16;
#pragma unroll
                            for (int e = 0; e < 16; e += 4) {
                                const float4 v = src == sub ? make_float4(__uint_as_float(raw_acc[e]), __uint_as_float(raw_acc[e + 1]),
                                                                          __uint_as_float(raw_acc[e + 2]), __uint_as_float(raw_acc[e + 3]))
                                                            : load_shared4(base + e / 4 * (kRowsPerBlock * 16));
                                acc[e] += v.x, acc[e + 1] += v.y, acc[e + 2] += v.z, acc[e + 3] += v.w;
                            }
                        }
                        if (kind == 0) finish_gram(q, t.z, row, j0, acc, u);
                        else finish_square(q, t.z, row, j0, factor, q.d + diagonal + j0, acc, u);
                        if (live) store16(symmetric + at, j0, q.ldk, u);
                        if (mirrored) store_mirrored(symmetric + static_cast<int64_t>(t.z) * p.m * q.ldk, q.ldk, p.m, row, j0, u);
                    }
                }
                tc_fence_before_sync();
                __syncwarp();
                if (lane == 0) mbar_arrive_cluster(map_to_rank(acc_empty0 + 8 * buf, leader));
            }
            // The block has finished this product when its eighth warp has: what the others wrote is passed on through the count
            // (one release for the device instead of one per warp: 1,728 x 576 138 against 144 us).
            __syncwarp();
            if (lane == 0) {
                bulk_wait();
                if (!last && add_acq_rel(smem_u32(finished)) % kEpilogueWarps == kEpilogueWarps - 1) add_release(q.arrived);
            }
        }
    }

    tc_fence_before_sync();
    __syncthreads();
    if (*abort_flag) {
        if (threadIdx.x == 0) atomicExch(q.err, 1);
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

// 2^13 / (|G| + eps) as two factors: of a very small matrix it is beyond binary32, and the first, a power of two, is then
// taken ahead.
struct Factor {
    float first, second;
    __device__ __forceinline__ Factor(double squares, double eps)
    {
        const double whole = static_cast<double>(kScale) / (sqrt(squares) + eps);
        const bool large = whole > 0x1p100;
        first = large ? 0x1p100f : 1.0f;
        second = static_cast<float>(large ? whole * 0x1p-100 : whole);
    }
    __device__ __forceinline__ float of(float v) const { return v * first * second; }
};

struct Start {
    int rows, cols, ld;
    int parts;               // blocks per matrix
    int whole;               // rows of G start on 16-byte boundaries
    int64_t g_batch, g_row;
    double eps;
    double *squares;         // [batch][parts]
    unsigned *arrived;       // the iteration's counter, set to zero here
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
    if (part == 0 && z == 0 && threadIdx.x == 0) *s.arrived = 0;
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
    double sum = 0.0;
    for (int i = threadIdx.x; i < s.parts; i += kRowThreads) sum += s.squares[z * s.parts + i];
    sum = block_sum(sum);
    const Factor factor(sum, s.eps);
    each_piece(s, part, [&](int64_t row, int c) {
        float v[8];
        load8<T>(v, g + z * s.g_batch + row * s.g_row, c, s.cols, s.whole);
        uint32_t hw[4], lw[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            v[2 * e] = factor.of(v[2 * e]);
            v[2 * e + 1] = factor.of(v[2 * e + 1]);
            hw[e] = pack2(v[2 * e], v[2 * e + 1]);
            const float2 h = unpack2(hw[e]);
            lw[e] = pack2(v[2 * e] - h.x, v[2 * e + 1] - h.y);
        }
        const int64_t at = (static_cast<int64_t>(z) * s.rows + row) * s.ld + c;
        *reinterpret_cast<uint4 *>(s.hi + at) = make_uint4(hw[0], hw[1], hw[2], hw[3]);
        *reinterpret_cast<uint4 *>(s.lo + at) = make_uint4(lw[0], lw[1], lw[2], lw[3]);
    });
}

// ---- a short side of up to 128: the whole iteration on the chip
//
// A cluster of up to eight blocks keeps X in shared memory, each block a slice of the long side's columns (a tall matrix is
// turned while it is read and written).  Of a step only the products X X^T cross blocks: each block sends the rows of its
// part to the blocks that own them, the owners add them up in order and send A's rows to everyone; A A, B and the slice of B X
// are each block's own.  Nothing waits for a whole cluster: a block that has received every part of this step knows that all
// others are past what they read of the last one.
//
// Operand tiles are boxes of 64 columns by KP rows with the 128-byte swizzle, as TMA would write them: read along the rows by
// X X^T, and down the rows (MN-major) by B X.  Instructions have 128 rows; with KP = 64 the upper half of them
// computes on whatever lies behind the box, and nobody reads it, but for P, which is there twice: B X then comes out in all
// lanes of the tensor memory, and all warps work on it.

constexpr int kSmallThreads = 512;
constexpr int kSmallQuads = kSmallThreads / 128;         // warps that share 32 rows: each takes a part of the columns
constexpr int kSmallWarps = kSmallThreads / 32;
constexpr int kSmallMost = 8;                            // blocks of a cluster
constexpr int kGroup = 256;                              // columns of X that one accumulator buffer holds

template <int KP>
struct Small {
    static constexpr int kBox = KP * 128;                // 64 columns of KP rows
    static constexpr int kSquare = KP / 64 * kBox;       // O
    static constexpr int kP = 128 / KP * kSquare;        // P: 128 rows
    static constexpr int kParts = KP * KP * 4;           // the parts of the rows that a block owns, from everyone
    static constexpr int kFloats = 2 * KP * 4;           // d, e
    static constexpr int kRest = 512;                    // barriers, sums
    // slices: as many boxes as there is room for
    static constexpr int kBoxes = KP == 64 ? 11 : 3;
    static constexpr int bytes(int boxes, int blocks)
    {
        const int used = 2 * boxes * kBox + kSquare + kP + (blocks > 1 ? kParts : 0) + kFloats + kRest + 1024;
        const int least = 120 * 1024;                    // one block per SM, since each takes all of the tensor memory
        return used > least ? used : least;
    }
};
static_assert(Small<64>::bytes(Small<64>::kBoxes, 2) <= 227 * 1024 && Small<128>::bytes(Small<128>::kBoxes, 2) <= 227 * 1024, "shared memory of a block");

struct SmallArgs {
    int k, l;                // short and long side
    int tall;
    int boxes;               // of a block's slice
    int steps;
    float a, b, c;
    double eps;
    int64_t g_batch, g_row;
    int g_whole;             // runs of eight elements of G's rows start on 16-byte boundaries
    __nv_bfloat16 *out;
    int64_t out_batch, out_row;
    int out_whole;
    int *err;
};

__device__ __forceinline__ void umma_one(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t accumulate)
{
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d_tmem),
        "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate)
        : "memory");
}

__device__ __forceinline__ void umma_commit_one(uint32_t bar)
{
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}

__device__ __forceinline__ uint32_t cluster_size()
{
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(r));
    return r;
}

__device__ __forceinline__ void put_piece(uint32_t addr, uint32_t a, uint32_t b, uint32_t c, uint32_t d)
{
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}

__device__ __forceinline__ uint4 get_piece(uint32_t addr)
{
    uint4 v;
    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr) : "memory");
    return v;
}

// Eight columns [8 piece, 8 piece + 8) of a row, in boxes of 64 columns.
template <int KP>
__device__ __forceinline__ uint32_t small_piece(uint32_t base, int row, int piece)
{
    return base + (piece >> 3) * Small<KP>::kBox + row * 128 + (((piece & 7) ^ (row & 7)) << 4);
}

template <typename T, int KP>
__global__ void __launch_bounds__(kSmallThreads, 1)
k_small(const __grid_constant__ SmallArgs p, const T *g)
{
    using S = Small<KP>;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t raw = smem_u32(smem_raw);
    const uint32_t hi0 = (raw + 1023u) & ~1023u, lo0 = hi0 + p.boxes * S::kBox;
    const uint32_t o0 = lo0 + p.boxes * S::kBox, p0 = o0 + S::kSquare;
    const uint32_t blocks = cluster_size(), rank = cluster_cta_rank();
    const uint32_t parts0 = p0 + S::kP, floats0 = parts0 + (blocks > 1 ? S::kParts : 0);
    uint8_t *floats_ptr = smem_raw + (floats0 - raw);
    float *d = reinterpret_cast<float *>(floats_ptr), *e = d + KP;
    const uint32_t bars = floats0 + S::kFloats;
    const uint32_t done0 = bars, parts_full = bars + 16, o_full = bars + 24;      // done0: two, one per accumulator buffer
    double *sums = reinterpret_cast<double *>(floats_ptr + S::kFloats + 32);      // [kSmallWarps], [kSmallMost]
    volatile uint32_t *tmem_slot = reinterpret_cast<volatile uint32_t *>(floats_ptr + S::kFloats + 32 + 8 * (kSmallWarps + kSmallMost));
    volatile int *abort_flag = reinterpret_cast<volatile int *>(tmem_slot + 1);

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int quarter = warp & 3, part = warp >> 2, row = quarter * 32 + lane;
    const int64_t z = blockIdx.x / blocks;
    const int slice = static_cast<int>(rank) * p.boxes * 64;         // the block's first column
    const T *gz = g + z * p.g_batch;

    if (threadIdx.x == 0) {
        mbar_init(done0, 1);
        mbar_init(done0 + 8, 1);
        mbar_init(parts_full, kSmallWarps * blocks);
        mbar_init(o_full, kSmallWarps * blocks);
        *abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 0) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(
                         smem_u32(const_cast<uint32_t *>(tmem_slot))),
                     "r"(512u)
                     : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }

    // G comes once: its numbers' upper and lower halves lie where hi and lo will, until the norm is known.  A unit is eight
    // elements of a row of G, along X's row or (tall) down eight of them; several are under way at a time.
    const int columns = p.boxes * 64;
    const int units = columns * (KP / 8);
    for (int i = threadIdx.x; i < 2 * p.boxes * S::kBox / 16; i += kSmallThreads) put_piece(hi0 + 16 * i, 0, 0, 0, 0);
    if (threadIdx.x < 2 * KP) d[threadIdx.x] = 0.0f;
    __syncthreads();
    double sum = 0.0;
    constexpr int kUnits = 4;
    for (int u0 = threadIdx.x; u0 < units; u0 += kUnits * kSmallThreads) {
        float v[kUnits][8];
        int r[kUnits], c[kUnits];
#pragma unroll
        for (int j = 0; j < kUnits; ++j) {
            const int u = u0 + j * kSmallThreads, box = u / (KP * 8);
            r[j] = p.tall ? u / 64 % (KP / 8) * 8 : u / 8 % KP;
            c[j] = box * 64 + (p.tall ? u % 64 : u % 8 * 8);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[j][i] = 0.0f;
            if (u >= units || r[j] >= p.k || slice + c[j] >= p.l) continue;
            if (p.tall)
                load8<T>(v[j], gz + (slice + c[j]) * p.g_row, r[j], p.k, p.g_whole);
            else
                load8<T>(v[j], gz + r[j] * p.g_row, slice + c[j], p.l, p.g_whole);
        }
#pragma unroll
        for (int j = 0; j < kUnits; ++j) {
            if (u0 + j * kSmallThreads >= units || r[j] >= p.k) continue;
            uint32_t w[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                sum = fma(static_cast<double>(v[j][i]), static_cast<double>(v[j][i]), sum);
                w[i] = __float_as_uint(v[j][i]);
            }
            if (!p.tall) {
                put_piece(small_piece<KP>(hi0, r[j], c[j] >> 3), __byte_perm(w[0], w[1], 0x7632), __byte_perm(w[2], w[3], 0x7632),
                          __byte_perm(w[4], w[5], 0x7632), __byte_perm(w[6], w[7], 0x7632));
                put_piece(small_piece<KP>(lo0, r[j], c[j] >> 3), __byte_perm(w[0], w[1], 0x5410), __byte_perm(w[2], w[3], 0x5410),
                          __byte_perm(w[4], w[5], 0x5410), __byte_perm(w[6], w[7], 0x5410));
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    if (r[j] + i >= p.k) break;
                    const uint32_t at = small_piece<KP>(0, r[j] + i, c[j] >> 3) + 2 * (c[j] & 7);
                    asm volatile("st.shared.u16 [%0], %1;" ::"r"(hi0 + at), "h"(static_cast<uint16_t>(w[i] >> 16)) : "memory");
                    asm volatile("st.shared.u16 [%0], %1;" ::"r"(lo0 + at), "h"(static_cast<uint16_t>(w[i])) : "memory");
                }
            }
        }
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, o);
    if (lane == 0) sums[warp] = sum;
    __syncthreads();
    sum = 0.0;
    for (int i = 0; i < kSmallWarps; ++i) sum += sums[i];
    cluster_sync_all();                                              // every block's barriers and memory are there
    if (blocks > 1) {
        if (threadIdx.x < blocks) {
            const uint32_t at = map_to_rank(smem_u32(sums + kSmallWarps + rank), threadIdx.x);
            asm volatile("st.shared::cluster.f64 [%0], %1;" ::"r"(at), "d"(sum) : "memory");
        }
        cluster_sync_all();
        sum = 0.0;
        for (uint32_t i = 0; i < blocks; ++i) sum += sums[kSmallWarps + i];
    }
    const Factor factor(sum, p.eps);
    for (int i = threadIdx.x; i < p.boxes * S::kBox / 16; i += kSmallThreads) {
        const uint4 up = get_piece(hi0 + 16 * i), low = get_piece(lo0 + 16 * i);
        const uint32_t h[4] = {up.x, up.y, up.z, up.w}, l[4] = {low.x, low.y, low.z, low.w};
        uint32_t hw[4], lw[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float x = factor.of(__uint_as_float(__byte_perm(l[j], h[j], 0x5410))), y = factor.of(__uint_as_float(__byte_perm(l[j], h[j], 0x7632)));
            hw[j] = pack2(x, y);
            const float2 f = unpack2(hw[j]);
            lw[j] = pack2(x - f.x, y - f.y);
        }
        put_piece(hi0 + 16 * i, hw[0], hw[1], hw[2], hw[3]);
        put_piece(lo0 + 16 * i, lw[0], lw[1], lw[2], lw[3]);
    }
    fence_async();
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    const uint32_t tmem = *tmem_slot, lanes = tmem + (static_cast<uint32_t>(quarter * 32) << 16);

    // f16 in, f32 out, 128 rows; KP columns along the rows of both, or `n` down the rows of the second operand
    const uint32_t idesc_square = (1u << 4) | ((KP >> 3) << 17) | ((128u >> 4) << 24);
    auto idesc_apply = [](int n) { return (1u << 4) | (1u << 16) | (static_cast<uint32_t>(n >> 3) << 17) | ((128u >> 4) << 24); };
    const int groups = (columns + kGroup - 1) / kGroup;
    uint32_t done_phase = 0;                                         // bit b: parity of the next commit to buffer b
    bool ok = true;
    auto wait_done = [&](int b) {
        ok = mbar_wait(done0 + 8 * b, (done_phase >> b) & 1, abort_flag) && ok;
        done_phase ^= 1u << b;
        tc_fence_after_sync();
    };
    auto issue_group = [&](int gr) {                                 // columns [256 gr, + n) of P X into buffer gr & 1
        const int n = min(kGroup, columns - gr * kGroup);
        const uint32_t idesc = idesc_apply(n);
        const uint32_t x = hi0 + gr * (kGroup / 64) * S::kBox;
        // MN-major: the next 64 columns are a box further, the next 8 rows 1024 bytes
        const uint64_t bd = static_cast<uint64_t>((x >> 4) & 0x3FFFu) | (static_cast<uint64_t>(S::kBox >> 4) << 16) | (64ull << 32) |
                            (1ull << 46) | (2ull << 61);
        for (int i = 0; i < KP / 16; ++i)
            umma_one(tmem + (gr & 1) * kGroup, smem_desc(p0 + (i >> 2) * S::kBox) + 2 * (i & 3), bd + (2048 >> 4) * i, idesc, i > 0);
        umma_commit_one(done0 + 8 * (gr & 1));
    };
    constexpr int kPart = KP / kSmallQuads;                          // columns of a symmetric product that a warp takes
    const bool mine = quarter * 32 < KP;                             // (whole warps)

    for (int step = 0; step < p.steps; ++step) {
        const bool last = step + 1 == p.steps;
        if (threadIdx.x == 0) {
            for (int b = 0; b < p.boxes; ++b)
                for (int i = 0; i < 4; ++i) {
                    const uint64_t x = smem_desc(hi0 + b * S::kBox) + 2 * i;
                    umma_one(tmem, x, x, idesc_square, b > 0 || i > 0);
                }
            umma_commit_one(done0);
        }
        wait_done(0);
        if (blocks == 1) {
#pragma unroll 1
            for (int c = part * kPart; mine && c < (part + 1) * kPart; c += 16) {
                uint32_t acc[16], w[8];
                tmem_ld16(lanes + c, acc);
                tmem_wait_ld();
                float v[16];
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    v[i] = __uint_as_float(acc[i]) * kUnscale2;
                    if (c + i == row) {
                        d[row] = v[i];
                        v[i] = 0.0f;
                    }
                }
#pragma unroll
                for (int i = 0; i < 8; ++i) w[i] = pack2(v[2 * i], v[2 * i + 1]);
                put_piece(small_piece<KP>(o0, row, c >> 3), w[0], w[1], w[2], w[3]);
                put_piece(small_piece<KP>(o0, row, (c >> 3) + 1), w[4], w[5], w[6], w[7]);
            }
        } else {
            const int own = KP / static_cast<int>(blocks);           // rows that a block adds up
            // [source][4 columns][row][4]: the rows of an owner lie together
            const int to = row / own, local = row - to * own;
            const uint32_t base = mine ? map_to_rank(parts0 + ((rank * (KP / 4)) * own + local) * 16, to) : 0;
#pragma unroll 1
            for (int c = part * kPart; mine && c < (part + 1) * kPart; c += 16) {
                uint32_t acc[16];
                tmem_ld16(lanes + c, acc);
                tmem_wait_ld();
#pragma unroll
                for (int i = 0; i < 4; ++i) store_remote(base + ((c >> 2) + i) * own * 16, acc + 4 * i);
            }
            __syncwarp();
            if (lane < blocks) mbar_arrive_release_cluster(map_to_rank(parts_full, lane));
            ok = mbar_wait_cluster(parts_full, step & 1, abort_flag) && ok;
            for (int u = threadIdx.x; u < own * (KP / 8); u += kSmallThreads) {
                const int r = u % own, piece = u / own, i = static_cast<int>(rank) * own + r;
                float v[8] = {0, 0, 0, 0, 0, 0, 0, 0};
                for (uint32_t src = 0; src < blocks; ++src) {
                    const uint32_t at = parts0 + ((src * (KP / 4) + 2 * piece) * own + r) * 16;
                    const float4 x = load_shared4(at), y = load_shared4(at + own * 16);
                    v[0] += x.x, v[1] += x.y, v[2] += x.z, v[3] += x.w, v[4] += y.x, v[5] += y.y, v[6] += y.z, v[7] += y.w;
                }
                float diagonal = 0.0f;
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    v[j] *= kUnscale2;
                    if (8 * piece + j == i) {
                        diagonal = v[j];
                        v[j] = 0.0f;
                    }
                }
                const uint32_t w[4] = {pack2(v[0], v[1]), pack2(v[2], v[3]), pack2(v[4], v[5]), pack2(v[6], v[7])};
                for (uint32_t other = 0; other < blocks; ++other) {
                    store_remote(map_to_rank(small_piece<KP>(o0, i, piece), other), w);
                    if (piece == i >> 3)
                        asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(map_to_rank(smem_u32(d + i), other)), "f"(diagonal) : "memory");
                }
            }
            __syncwarp();
            if (lane < blocks) mbar_arrive_release_cluster(map_to_rank(o_full, lane));
            ok = mbar_wait_cluster(o_full, step & 1, abort_flag) && ok;
        }
        fence_async();
        tc_fence_before_sync();
        __syncthreads();
        tc_fence_after_sync();
        if (threadIdx.x == 0) {
            for (int i = 0; i < KP / 16; ++i) {
                const uint64_t o = smem_desc(o0 + (i >> 2) * S::kBox) + 2 * (i & 3);
                umma_one(tmem + kGroup, o, o, idesc_square, i > 0);
            }
            umma_commit_one(done0 + 8);
        }
        const float di = mine ? d[row] : 0.0f;
        wait_done(1);
#pragma unroll 1
        for (int c = part * kPart; mine && c < (part + 1) * kPart; c += 16) {
            uint32_t acc[16], w[8];
            tmem_ld16(lanes + kGroup + c, acc);
            const uint4 o_lo = get_piece(small_piece<KP>(o0, row, c >> 3)), o_hi = get_piece(small_piece<KP>(o0, row, (c >> 3) + 1));
            const uint32_t ow[8] = {o_lo.x, o_lo.y, o_lo.z, o_lo.w, o_hi.x, o_hi.y, o_hi.z, o_hi.w};
            tmem_wait_ld();
            float v[16];
#pragma unroll
            for (int i = 0; i < 16; i += 2) {
                const float2 o = unpack2(ow[i / 2]);
                const float2 dj = *reinterpret_cast<const float2 *>(d + c + i);
                const float s0 = __uint_as_float(acc[i]), s1 = __uint_as_float(acc[i + 1]);
                v[i] = fmaf(p.c, fmaf(di + dj.x, o.x, s0), p.b * o.x);
                v[i + 1] = fmaf(p.c, fmaf(di + dj.y, o.y, s1), p.b * o.y);
                if (c + i == row) {
                    e[row] = fmaf(p.c, fmaf(di, di, s0), p.b * di);
                    v[i] = 0.0f;
                }
                if (c + i + 1 == row) {
                    e[row] = fmaf(p.c, fmaf(di, di, s1), p.b * di);
                    v[i + 1] = 0.0f;
                }
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) w[i] = pack2(v[2 * i], v[2 * i + 1]);
            for (int copy = 0; copy < S::kP; copy += S::kSquare) {
                put_piece(small_piece<KP>(p0 + copy, row, c >> 3), w[0], w[1], w[2], w[3]);
                put_piece(small_piece<KP>(p0 + copy, row, (c >> 3) + 1), w[4], w[5], w[6], w[7]);
            }
        }
        fence_async();
        tc_fence_before_sync();
        __syncthreads();
        tc_fence_after_sync();
        if (threadIdx.x == 0) {
            issue_group(0);
            if (groups > 1) issue_group(1);
        }
        // the row of B X that this lane has, and the runs of 16 columns that are this warp's
        constexpr int kRuns = kSmallQuads * 128 / KP;
        const int here = row % KP, run = part * (128 / KP) + row / KP;
        const float scale = p.a + e[here];
        for (int gr = 0; gr < groups; ++gr) {
            const int n = min(kGroup, columns - gr * kGroup);
            wait_done(gr & 1);
#pragma unroll 1
            for (int c = 16 * run; c < n; c += 16 * kRuns) {
                uint32_t acc[16];
                tmem_ld16(lanes + (gr & 1) * kGroup + c, acc);
                const int piece = (gr * kGroup + c) >> 3;
                const uint4 h0 = get_piece(small_piece<KP>(hi0, here, piece)), h1 = get_piece(small_piece<KP>(hi0, here, piece + 1));
                const uint4 l0 = get_piece(small_piece<KP>(lo0, here, piece)), l1 = get_piece(small_piece<KP>(lo0, here, piece + 1));
                const uint32_t hw[8] = {h0.x, h0.y, h0.z, h0.w, h1.x, h1.y, h1.z, h1.w};
                const uint32_t lw[8] = {l0.x, l0.y, l0.z, l0.w, l1.x, l1.y, l1.z, l1.w};
                tmem_wait_ld();
                float v[16];
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float2 h = unpack2(hw[i]), l = unpack2(lw[i]);
                    v[2 * i] = fmaf(scale, h.x + l.x, __uint_as_float(acc[2 * i]));
                    v[2 * i + 1] = fmaf(scale, h.y + l.y, __uint_as_float(acc[2 * i + 1]));
                }
                if (!last) {
                    uint32_t nh[8], nl[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        nh[i] = pack2(v[2 * i], v[2 * i + 1]);
                        const float2 h = unpack2(nh[i]);
                        nl[i] = pack2(v[2 * i] - h.x, v[2 * i + 1] - h.y);
                    }
                    put_piece(small_piece<KP>(hi0, here, piece), nh[0], nh[1], nh[2], nh[3]);
                    put_piece(small_piece<KP>(hi0, here, piece + 1), nh[4], nh[5], nh[6], nh[7]);
                    put_piece(small_piece<KP>(lo0, here, piece), nl[0], nl[1], nl[2], nl[3]);
                    put_piece(small_piece<KP>(lo0, here, piece + 1), nl[4], nl[5], nl[6], nl[7]);
                } else if (here < p.k) {
                    const int j0 = slice + 8 * piece;
                    if (p.tall) {                                    // neighbouring lanes have neighbouring columns of the update
                        __nv_bfloat16 *dst = p.out + z * p.out_batch + j0 * p.out_row + here;
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            if (j0 + i < p.l) *dst = __float2bfloat16_rn(v[i] * kUnscale);
                            dst += p.out_row;
                        }
                    } else {
                        __nv_bfloat16 *dst = p.out + z * p.out_batch + here * p.out_row;
                        if (p.out_whole) {
                            uint32_t w[8];
#pragma unroll
                            for (int i = 0; i < 8; ++i) w[i] = pack_bf16(v[2 * i] * kUnscale, v[2 * i + 1] * kUnscale);
                            store16(dst, j0, p.l, w);
                        } else {
#pragma unroll
                            for (int i = 0; i < 16; ++i)
                                if (j0 + i < p.l) dst[j0 + i] = __float2bfloat16_rn(v[i] * kUnscale);
                        }
                    }
                }
            }
            if (gr + 2 < groups) {                                   // this buffer is free again
                tc_fence_before_sync();
                __syncthreads();
                tc_fence_after_sync();
                if (threadIdx.x == 0) issue_group(gr + 2);
            }
        }
        fence_async();
        tc_fence_before_sync();
        __syncthreads();
        tc_fence_after_sync();
    }
    if (!ok) atomicExch(p.err, 1);                                   // (whichever thread gave up)
    cluster_sync_all();                                              // the others may still write here
    if (warp == 0) {
        __syncwarp();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u) : "memory");
    }
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

// The same in blocks of 32 x 32; type: of 16 bits, strides in elements.
bool encode_blocks(CUtensorMap *m, CUtensorMapDataType type, const void *base, int64_t batch, int64_t rows, int64_t cols, int64_t ld, int64_t stack)
{
    const cuuint64_t dims[3] = {static_cast<cuuint64_t>(cols), static_cast<cuuint64_t>(rows), static_cast<cuuint64_t>(batch)};
    const cuuint64_t strides[2] = {static_cast<cuuint64_t>(ld) * 2, static_cast<cuuint64_t>(stack) * 2};
    const cuuint32_t box[3] = {32, 32, 1};
    const cuuint32_t elem_strides[3] = {1, 1, 1};
    return tensor_map_encoder()(m, type, 3, const_cast<void *>(base), dims, strides, box, elem_strides, CU_TENSOR_MAP_INTERLEAVE_NONE,
                                CU_TENSOR_MAP_SWIZZLE_64B, CU_TENSOR_MAP_L2_PROMOTION_L2_128B,
                                CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

bool aligned(const void *ptr, size_t bytes) { return reinterpret_cast<uintptr_t>(ptr) % bytes == 0; }

}  // namespace

struct orthogonal {
    int rows = 0, cols = 0, steps = 0, type = 0;
    float a = 0, b = 0, c = 0, eps = 0;
    int device = 0, sms = 0;
    int pairs = 0, clusters[2] = {0, 0};     // of two blocks, and of 2 kShares[i], that the device holds at once
    cudaStream_t stream = nullptr;
    int64_t launches = 0;
    int *err = nullptr;
};

namespace {

int short_side(const orthogonal *p) { return p->rows < p->cols ? p->rows : p->cols; }
int64_t pad8(int64_t v) { return div_up(v, 8) * 8; }
int64_t pad16(int64_t v) { return div_up(v, 16) * 16; }

// How k_small cuts the long side: blocks of a cluster and boxes of 64 columns for each.  A box costs a block about a sixth of
// what crossing blocks does, and matrices that do not fit on the device at once follow one another.  False where the
// matrix is not for it: a short side over 128, or too long a one.
bool small_cut(const orthogonal *p, int64_t batch, int *blocks, int *boxes)
{
    const int k = short_side(p), l = p->rows > p->cols ? p->rows : p->cols;
    if (k > 128) return false;
    const int most = k <= 64 ? Small<64>::kBoxes : Small<128>::kBoxes;
    const int64_t all = div_up(l, 64);
    int64_t best = -1;
    for (int n = 1; n <= kSmallMost; n *= 2) {
        const int64_t each = div_up(all, n);
        const int64_t cost = (each + (n > 1 ? 12 : 6)) * div_up(batch, p->sms / n);
        if (each > most || (best >= 0 && cost >= best)) continue;
        best = cost;
        *blocks = n;
        *boxes = static_cast<int>(each);
    }
    return best >= 0;
}

// Everything a call keeps between its kernels.
struct Layout {
    int64_t ld, ldk, dk;
    size_t hi[2], lo[2], o, p, d, e, squares, arrived, total;
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
    w.arrived = take(sizeof(unsigned));
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

// Chooses the tiles of a product for `pairs` pairs in clusters of `share` and returns what it costs, in units of 1.6 ns.  A block
// brings in 128 rows of A and half the columns of B per step, at about 80 KB a microsecond whatever the tile (measured: 0.42 us
// a step for 256 columns, 0.31 for 128, 0.28 for 64); the wait for the other blocks, the first loads and the last stores come
// to 3 us, a set of 64 columns in the epilogue to half a microsecond, exchanging the parts of a shared tile to 2 us.
int64_t choose_tile(Product &q, int64_t batch, int64_t pairs, int share)
{
    q.steps = static_cast<int>(div_up(q.k, kBK));
    q.m_tiles = static_cast<int>(div_up(q.m, kTileM));
    int64_t best = -1;
    for (int w : {256, 128, 64}) {
        const int64_t tiles = tiles_of(q.m, q.n, w, q.symmetric);
        for (int shared = 0; shared <= (share > 1 && q.symmetric && w <= share_cols(share) ? 1 : 0); ++shared) {
            // (a shared tile takes a step for each pair, and each cluster one tile)
            if (shared && (q.steps < share || tiles * batch > pairs / share)) continue;
            const int64_t rounds = shared ? 1 : div_up(tiles * batch, pairs), steps = shared ? div_up(q.steps, share) : q.steps;
            const int64_t cost = rounds * steps * (w / 2 + 128) + 1800 + w / 64 * 300 + (shared ? 1250 : 0);
            if (best >= 0 && cost >= best) continue;
            best = cost;
            q.tile_n = w;
            q.tiles = static_cast<int>(tiles);
            q.shared = shared;
        }
    }
    q.n_tiles = static_cast<int>(div_up(q.n, q.tile_n));
    return best;
}

// An operand of a product: a stack of [rows][cols] matrices, read along or across its rows.
struct Operand {
    const __half *base;
    int64_t rows, cols, ld;
};

bool encode_operand(CUtensorMap *m, const Operand &x, int64_t batch, int by_rows, int box_rows)
{
    return encode(m, x.base, batch, x.rows, x.cols, x.ld, by_rows ? kBK : box_rows);
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

    const bool out_whole = p->cols % 8 == 0 && aligned(out, 16) && (p->rows == 1 || out_row % 8 == 0) && (batch == 1 || out_batch % 8 == 0);
    const bool g_whole = aligned(g, 16) && (p->rows == 1 || g_row * sizeof(T) % 16 == 0) && (batch == 1 || g_batch * sizeof(T) % 16 == 0);
    int blocks, boxes;
    if (small_cut(p, batch, &blocks, &boxes)) {
        SmallArgs r = {};
        r.k = k;
        r.l = tall ? p->rows : p->cols;
        r.tall = tall;
        r.boxes = boxes;
        r.steps = p->steps;
        r.a = p->a;
        r.b = p->b;
        r.c = p->c;
        r.eps = p->eps;
        r.g_batch = g_batch;
        r.g_row = g_row;
        r.g_whole = g_whole;
        r.out = out;
        r.out_batch = out_batch;
        r.out_row = out_row;
        r.out_whole = out_whole;
        r.err = p->err;
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3(static_cast<unsigned>(batch * blocks));
        cfg.blockDim = dim3(kSmallThreads);
        cfg.dynamicSmemBytes = k <= 64 ? Small<64>::bytes(boxes, blocks) : Small<128>::bytes(boxes, blocks);
        cfg.stream = p->stream;
        cudaLaunchAttribute attr[1];
        attr[0].id = cudaLaunchAttributeClusterDimension;
        attr[0].val.clusterDim.x = static_cast<unsigned>(blocks);
        attr[0].val.clusterDim.y = 1;
        attr[0].val.clusterDim.z = 1;
        cfg.attrs = attr;
        cfg.numAttrs = 1;
        if (cudaLaunchKernelEx(&cfg, k <= 64 ? k_small<T, 64> : k_small<T, 128>, r, g) != cudaSuccess) {
            cudaGetLastError();
            return ORTHOGONAL_ECUDA;
        }
        p->launches += 1;
        return ORTHOGONAL_OK;
    }

    Start s = {};
    s.rows = p->rows;
    s.cols = p->cols;
    s.ld = static_cast<int>(w.ld);
    // a piece per thread where there are few, several where there are many
    const int64_t parts = div_up(static_cast<int64_t>(p->rows) * (w.ld / 8), kRowThreads);
    s.parts = static_cast<int>(parts < kMostParts ? parts : kMostParts);
    s.g_batch = g_batch;
    s.g_row = g_row;
    s.whole = g_whole;
    s.eps = p->eps;
    s.squares = reinterpret_cast<double *>(base + w.squares);
    s.arrived = reinterpret_cast<unsigned *>(base + w.arrived);
    s.hi = half(w.hi[0]);
    s.lo = half(w.lo[0]);
    const dim3 grid(static_cast<unsigned>(s.parts), static_cast<unsigned>(batch));
    k_squares<T><<<grid, kRowThreads, 0, p->stream>>>(s, g);
    if (cudaGetLastError() != cudaSuccess) return ORTHOGONAL_ECUDA;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(kRowThreads);
    cfg.stream = p->stream;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    if (cudaLaunchKernelEx(&cfg, k_start<T>, s, g) != cudaSuccess) {
        cudaGetLastError();
        return ORTHOGONAL_ECUDA;
    }

    Iteration q = {};
    q.batch = static_cast<int>(batch);
    q.steps = p->steps;
    q.tall = tall;
    q.ldk = static_cast<int>(w.ldk);
    q.dk = static_cast<int>(w.dk);
    q.a = p->a;
    q.b = p->b;
    q.c = p->c;
    q.o = half(w.o);
    q.p = half(w.p);
    q.d = single(w.d);
    q.e = single(w.e);
    for (int i = 0; i < 2; ++i) {
        q.hi[i] = half(w.hi[i]);
        q.lo[i] = half(w.lo[i]);
    }
    q.out = out;
    q.out_batch = out_batch;
    q.out_row = out_row;
    q.out_whole = out_whole;
    q.arrived = s.arrived;
    q.err = p->err;
    q.gram.m = q.gram.n = q.square.m = q.square.n = q.square.k = k;
    q.gram.k = tall ? p->rows : p->cols;
    q.gram.symmetric = q.square.symmetric = 1;
    q.gram.a_rows = q.gram.b_rows = tall;
    q.apply.m = p->rows;
    q.apply.n = p->cols;
    q.apply.k = k;
    q.apply.b_rows = !tall;
    // pairs by themselves, or in clusters that can share a reduction: whichever a step of the iteration is shortest with
    int64_t most = p->pairs;                             // pairs on the device
    auto cost = [&](Iteration &r, int64_t pairs, int share) {
        r.share = share;
        return choose_tile(r.gram, batch, pairs, share) + choose_tile(r.square, batch, pairs, share) + choose_tile(r.apply, batch, pairs, share);
    };
    int64_t best = cost(q, most, 1);
    for (int i = 0; i < 2; ++i) {
        Iteration other = q;
        const int64_t pairs = static_cast<int64_t>(p->clusters[i]) * kShares[i];
        if (pairs == 0) continue;
        const int64_t c = cost(other, pairs, kShares[i]);
        if (c >= best) continue;
        best = c;
        most = pairs;
        q = other;
    }

    Maps maps;
    const Operand o = {q.o, k, k, w.ldk}, pp = {q.p, k, k, w.ldk};
    bool ok = encode_operand(&maps.square_a, o, batch, 0, kRowsPerBlock) && encode_operand(&maps.square_b, o, batch, 0, q.square.tile_n / 2);
    for (int i = 0; i < 2; ++i) {
        const Operand x = {q.hi[i], p->rows, p->cols, w.ld};
        ok = ok && encode_operand(&maps.gram_a[i], x, batch, q.gram.a_rows, kRowsPerBlock) &&
             encode_operand(&maps.gram_b[i], x, batch, q.gram.b_rows, q.gram.tile_n / 2) &&
             encode_operand(&maps.apply_a[i], tall ? x : pp, batch, q.apply.a_rows, kRowsPerBlock) &&
             encode_operand(&maps.apply_b[i], tall ? pp : x, batch, q.apply.b_rows, q.apply.tile_n / 2);
        for (int low = 0; low < 2; ++low)
            ok = ok && encode_blocks(low ? &maps.lo[i] : &maps.hi[i], CU_TENSOR_MAP_DATA_TYPE_FLOAT16, low ? q.lo[i] : q.hi[i], batch,
                                     p->rows, p->cols, w.ld, w.ld * p->rows);
    }
    for (int b = 0; b < 2; ++b)
        ok = ok && encode_blocks(b ? &maps.p : &maps.o, CU_TENSOR_MAP_DATA_TYPE_FLOAT16, b ? q.p : q.o, batch, k, k, w.ldk, w.ldk * k);
    // (of a single row or matrix the stride does not matter, but it has to be one)
    if (q.out_whole) {
        const int64_t row = p->rows > 1 ? out_row : p->cols;
        ok = ok && encode_blocks(&maps.out, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, out, batch, p->rows, p->cols, row, batch > 1 ? out_batch : row * p->rows);
    } else {
        maps.out = maps.hi[0];
    }
    if (!ok) return ORTHOGONAL_ECUDA;
    // as many blocks as there is work for, in whole clusters
    auto wanted = [&](const Product &r) {
        const int64_t tiles = static_cast<int64_t>(r.tiles) * batch;
        return r.shared ? tiles * q.share : tiles;
    };
    int64_t pairs = wanted(q.gram);
    if (wanted(q.square) > pairs) pairs = wanted(q.square);
    if (wanted(q.apply) > pairs) pairs = wanted(q.apply);
    pairs = div_up(pairs, q.share) * q.share;
    if (pairs > most) pairs = most;
    cfg.gridDim = dim3(static_cast<unsigned>(2 * pairs));
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = kSmem;
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = static_cast<unsigned>(2 * q.share);
    attr[0].val.clusterDim.y = 1;
    attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeCooperative;     // all blocks at once: they wait for one another
    attr[1].val.cooperative = 1;
    cfg.numAttrs = 2;
    if (cudaLaunchKernelEx(&cfg, k_iterate, maps, q) != cudaSuccess) {
        cudaGetLastError();
        return ORTHOGONAL_ECUDA;
    }
    p->launches += 3;
    return ORTHOGONAL_OK;
}

bool batch_ok(const orthogonal *p, int64_t batch)
{
    // matrices and tiles are 32-bit in the kernels, and a grid's second dimension counts matrices
    return batch >= 1 && batch <= 65535 &&
           batch * div_up(p->rows, kTileM) * div_up(p->cols, 64) < 0x7FFFFFFF;
}

template <typename T>
bool raise_small()
{
    return raise_dynamic_smem(reinterpret_cast<const void *>(k_small<T, 64>), 227 * 1024) &&
           raise_dynamic_smem(reinterpret_cast<const void *>(k_small<T, 128>), 227 * 1024);
}

// Clusters of `blocks` blocks of k_iterate that the device holds at once, 0 if none.
int resident_clusters(int blocks, int sms)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(sms / blocks * blocks));
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = kSmem;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = static_cast<unsigned>(blocks);
    attr[0].val.clusterDim.y = 1;
    attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    int clusters = 0;
    if (cudaOccupancyMaxActiveClusters(&clusters, k_iterate, &cfg) != cudaSuccess) {
        cudaGetLastError();
        return 0;
    }
    return clusters < sms / blocks ? clusters : sms / blocks;
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
        !raise_dynamic_smem(reinterpret_cast<const void *>(k_iterate), kSmem) || !raise_small<float>() ||
        !raise_small<__nv_bfloat16>() || !raise_small<__half>()) {
        cudaGetLastError();
        delete p;
        return ORTHOGONAL_ECUDA;
    }
    p->pairs = resident_clusters(2, p->sms);
    for (int i = 0; i < 2; ++i) p->clusters[i] = resident_clusters(2 * kShares[i], p->sms);
    if (p->pairs < 1) {
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
    int blocks, boxes;
    return small_cut(p, batch, &blocks, &boxes) ? 0 : layout_of(p, batch).total;
}

int orthogonal_update(orthogonal *p, const void *g, int64_t g_stride_batch, int64_t g_stride_row, void *update,
                      int64_t update_stride_batch, int64_t update_stride_row, void *workspace, size_t workspace_bytes,
                      int64_t batch)
{
    if (p == nullptr) return ORTHOGONAL_ENULL;
    if (!batch_ok(p, batch)) return ORTHOGONAL_EINVAL;     // first: an empty batch comes without pointers
    const size_t need = orthogonal_workspace_bytes(p, batch);
    if (g == nullptr || update == nullptr || (need > 0 && workspace == nullptr)) return ORTHOGONAL_ENULL;
    if (g_stride_batch < 0 || g_stride_row < 0) return ORTHOGONAL_EINVAL;
    if (p->rows > 1 && update_stride_row < p->cols) return ORTHOGONAL_EINVAL;
    // the update's matrices one behind the other
    if (batch > 1 && update_stride_batch < (p->rows - 1) * (p->rows > 1 ? update_stride_row : 0) + p->cols) return ORTHOGONAL_EINVAL;
    if (!aligned(g, p->type == ORTHOGONAL_F32 ? 4 : 2) || !aligned(update, 2) || !aligned(workspace, 256)) return ORTHOGONAL_EALIGN;
    if (need > workspace_bytes) return ORTHOGONAL_ENOMEM;
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
