// gated_ffn.cu -- the gated feed-forward block (forward, backward) as sm_100a kernels behind the
// C ABI of gated_ffn.h.
//
// k_product is one matrix product D = A B^T on CTA pairs (tcgen05, cta_group::2) with three
// epilogues.  A pair's tile is 256 rows of A by 256 (or 192, 128) rows of B; each block of the pair
// stages 128 rows of A and half of the rows of B per 64 reduction elements, the leader issues
// M = 256 instructions into one of two 256-column accumulator buffers, and eight epilogue warps
// per block empty the other one meanwhile.
//
//   kGated    forward: the leader stages 128 gate rows of W_in as its half of B, its peer the
//             128 rows of the other projection, so that columns c and 128 + c of every
//             accumulator row are g and u of one hidden unit: act(g) u is formed in registers.
//   kSlope    backward: D = dy W_out; the epilogue reads g and u and writes dg and du.
//   kStore    the remaining products.
//
// A thread's accumulators are one row of the tile, so that its own stores would touch a line each.
// kGated and kSlope move several times the bytes of their accumulators: there every warp passes
// blocks of 32 rows x 32 columns through shared memory (swizzled, no bank conflicts) and TMA
// copies them out, and g and u in.
//
// g and u are kept for the backward pass as the upper 24 bits of their binary32 values, in a plane of 16
// and a plane of 8 bits: rounded to the type they would add an error as large as the result's own
// rounding to dx and dW_in.
//
// Operands lie in memory as they are: where the reduction runs along rows (W_in in dx, W_out in
// dhidden, both operands of a weight gradient) TMA brings boxes of 64 elements of the row by 64
// reduction rows and the instruction reads them MN-major; nothing is transposed.
//
// Work of kStore: whole rounds of tiles, one tile per pair; the tiles of a last, incomplete round
// are one stretch of 64-element steps cut evenly over the pairs, so that all pairs finish together
// whatever the number of tiles; a tile that a cut divides goes to scratch in binary32 and k_join
// adds its pieces in order.
//
// What bounds it (65,536 x 576 x 1,536 / 8,192 x 2,048 x 8,192, silu, bfloat16, each kernel by itself):
//     kGated   231 us, 1.00 PFLOP/s / 390 us, 1.41 PFLOP/s   epilogue (805 MB written, 3.5 TB/s) / tensor cores
//     kSlope   199 us, 0.58 PFLOP/s / 287 us, 0.96 PFLOP/s   memory (679 MB read and 403 written, 5.4 TB/s, 0.83 of
//              a copy: the kept g and u are more than half of it) / epilogue
//     kStore   y 110 us, 1.06 / 187 us, 1.47; dx 201 us, 1.15 / 372 us, 1.48; dW_in 250 us, 0.93 / 405 us, 1.36;
//              dW_out 135 us, 0.86 / 208 us, 1.32 PFLOP/s
// The products with 576 columns move 57 to 64 KB of operands from L2 per 0.29 us of a tile's arithmetic, 8.5 to 10.5 TB/s
// (11 to 14 by L2's own count, which has fills and results in it); wider tiles would need more accumulator
// columns than there are.  dW_out has 576 rows, which three tiles of 256 round up to 768: a quarter of its work is
// padding (1.15 PFLOP/s with it).
//
// k_rows: up to 64 rows of x, bound by reading the weights: one row through 2,048 x 8,192 takes 16.8 us from a
// graph, 6.0 TB/s.  A block owns 16 rows of the weights
// (of each projection), its warps split the reduction, and each lane's 16-byte loads of the
// weights go straight into the operands of warp-wide matrix instructions: a dot product does not
// care in which order its terms come, so a lane's eight consecutive elements serve as the
// fragment positions of two instructions, for the weights and for x alike.
#include <cstring>
#include <new>

#include <cuda_fp16.h>

#include "../../include/gated_ffn.h"
#include "on_device.cuh"
#include "sm100.cuh"

namespace {

constexpr int kBK = 64;                          // reduction elements per stage
constexpr int kRowsPerBlock = 128;               // rows of A per block; a pair's tile has twice as many
constexpr int kTileM = 2 * kRowsPerBlock;
constexpr int kStagesMost = 6;
constexpr int kABytes = kRowsPerBlock * kBK * 2;
constexpr int kBBytes = 128 * kBK * 2;           // at most 128 rows of B per block
constexpr int kStageBytes = kABytes + kBBytes;
constexpr int kAccCols = 256;
constexpr int kTmemCols = 2 * kAccCols;
constexpr int kEpilogueWarps = 8;
constexpr int kThreads = 64 + 32 * kEpilogueWarps;
constexpr int kBarrierBytes = 512;
constexpr int kMinSteps = 4;                     // a piece of a divided tile is at least this long

enum Mode { kStore, kGated, kSlope };

// A block of 32 rows x 32 columns on its way between registers and memory: 16-bit elements 64 bytes per row
// (64-byte swizzle), 8-bit elements 32 bytes per row (32-byte swizzle).
constexpr int kBlock16 = 32 * 64;
constexpr int kBlock8 = 32 * 32;
constexpr int kPreBytes = 2 * kBlock16 + 2 * kBlock8;    // g and u: upper planes, then lower planes

// Stages of the ring and staging bytes per epilogue warp: kGated holds g and u and the hidden units, kSlope
// kSets sets of g and u (one worked on and then overwritten with dg and du, the others on their way in).
constexpr int kSets = 2;
__host__ __device__ constexpr int stages_of(int mode) { return mode == kStore ? 6 : mode == kGated ? 5 : 6 - kSets; }
__host__ __device__ constexpr int staging_of(int mode) { return mode == kStore ? 0 : mode == kGated ? kPreBytes + kBlock16 : kSets * kPreBytes; }
__host__ __device__ constexpr int smem_of(int mode)
{
    return stages_of(mode) * kStageBytes + kEpilogueWarps * staging_of(mode) + kBarrierBytes + 1024;
}
static_assert(smem_of(kStore) <= 227 * 1024 && smem_of(kGated) <= 227 * 1024 && smem_of(kSlope) <= 227 * 1024,
              "shared memory of a block");
static_assert(kPreBytes % 1024 == 0 && (kPreBytes + kBlock16) % 1024 == 0, "swizzled blocks need their alignment");

template <typename T>
struct Type;
template <>
struct Type<__nv_bfloat16> {
    static constexpr uint32_t kFormat = 1;       // operand format field of the instruction descriptor
    static constexpr CUtensorMapDataType kMap = CU_TENSOR_MAP_DATA_TYPE_BFLOAT16;
    static __device__ __forceinline__ uint32_t pack(float a, float b) { return pack_bf16(a, b); }
    static __device__ __forceinline__ float2 unpack(uint32_t w) { return make_float2(bf16_lo(w), bf16_hi(w)); }
};
template <>
struct Type<__half> {
    static constexpr uint32_t kFormat = 0;
    static constexpr CUtensorMapDataType kMap = CU_TENSOR_MAP_DATA_TYPE_FLOAT16;
    static __device__ __forceinline__ uint32_t pack(float a, float b)
    {
        const __half2 v = __floats2half2_rn(a, b);
        return *reinterpret_cast<const uint32_t *>(&v);
    }
    static __device__ __forceinline__ float2 unpack(uint32_t w) { return __half22float2(*reinterpret_cast<const __half2 *>(&w)); }
};

// ---- activation: act(v) = v sigmoid(s(v)), s(v) = v (silu) or 2 c (v + k v^3) (gelu, since
// (1 + tanh w) / 2 = sigmoid(2 w)); act'(v) = sg + v sg (1 - sg) s'(v)

constexpr float kGelu2C = 1.5957691216057308f;   // 2 sqrt(2 / pi)
constexpr float kGeluK = 0.044715f;

template <bool kGelu>
__device__ __forceinline__ float act_sigmoid(float v)
{
    const float s = kGelu ? kGelu2C * fmaf(kGeluK * v * v, v, v) : v;
    return rcp_approx(1.0f + ex2_approx(-kLog2e * s));
}

template <bool kGelu>
__device__ __forceinline__ float act_slope(float v, float sg)
{
    const float rise = v * sg * (1.0f - sg);
    return kGelu ? fmaf(rise, kGelu2C * fmaf(3.0f * kGeluK * v, v, 1.0f), sg) : sg + rise;
}

// ---- the product

struct Product {
    int64_t m;              // rows of A and D
    int n;                  // rows of B, columns of D (kGated: hidden units)
    int64_t k;              // reduction length
    int a_rows, b_rows;     // 1: the operand is stored [k][rows] (MN-major), 0: [rows][k]
    int tile_n;             // columns of D per tile: 256, 192 or 128; kGated: 128 or 64 hidden units, twice as many columns
    int m_tiles, n_tiles;
    int m_first;            // 1: consecutive tiles run down the rows, 0: along the columns
    int steps;              // ceil(k / 64)
    int rounds;             // whole rounds of tiles
    int cuts;               // pairs that share the rest (0: none)
    void *out;              // kStore: D
    int64_t out_stride;
    int keep;               // kGated: write g and u
    float *pieces;          // [cuts][2] tiles in the order of piece_at
    int *err;
};

// The stretches of reduction steps a pair works through, in order.  Every role of the block runs its own copy.
struct Walk {
    const Product &p;
    int pair, pairs, tiles;
    int round = 0;
    int64_t at, end, begin;      // steps of the shared rest
    int tile, k0, k1, piece;     // the current stretch; piece: -1 whole tile, else which of the pair's two slots

    __device__ Walk(const Product &q, int pair_, int pairs_) : p(q), pair(pair_), pairs(pairs_), tiles(q.m_tiles * q.n_tiles)
    {
        const int64_t rest = static_cast<int64_t>(tiles - p.rounds * pairs) * p.steps;
        begin = at = pair < p.cuts ? rest * pair / p.cuts : 0;
        end = pair < p.cuts ? rest * (pair + 1) / p.cuts : 0;
    }
    __device__ bool next()
    {
        if (round < p.rounds) {
            tile = round * pairs + pair;
            ++round;
            k0 = 0;
            k1 = p.steps;
            piece = -1;
            return tile < tiles;
        }
        if (at >= end) return false;
        const int64_t t = at / p.steps;
        tile = p.rounds * pairs + static_cast<int>(t);
        k0 = static_cast<int>(at - t * p.steps);
        const int64_t left = end - at;
        k1 = left < p.steps - k0 ? k0 + static_cast<int>(left) : p.steps;
        piece = k0 == 0 && k1 == p.steps ? -1 : (at == begin ? 0 : 1);
        at += k1 - k0;
        return true;
    }
    __device__ int row_tile() const { return p.m_first ? tile % p.m_tiles : tile / p.n_tiles; }
    __device__ int col_tile() const { return p.m_first ? tile / p.m_tiles : tile % p.n_tiles; }
};

// A kernel's start on the device ahead of the end of the one before it: what precedes wait_for_previous() must
// not touch that one's results.  Every block waits, so that kernels end in the order of the stream.
__device__ __forceinline__ void allow_next() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void wait_for_previous() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

// MN-major operand tile with the 128-byte swizzle: boxes of 64 elements (128 bytes) by 64 reduction
// rows; the next 64 elements are a box (8192 bytes, leading offset) further, the next 8
// reduction rows 1024 bytes (stride offset).
__device__ __forceinline__ uint64_t smem_desc_rows(uint32_t addr)
{
    return static_cast<uint64_t>((addr >> 4) & 0x3FFFu) | (512ull << 16) | (64ull << 32) | (1ull << 46) | (2ull << 61);
}

// Place of a piece's block of 32 rows (0..7) and 16 columns (0..15) in the scratch, in float4.
__device__ __forceinline__ int64_t piece_at(int pair, int slot, int rows, int cols)
{
    return (((static_cast<int64_t>(pair) * 2 + slot) * (kTileM / 32) + rows) * (kAccCols / 16) + cols) * 128;
}

// Columns [c, c + 16) of a row of `width` columns (a multiple of 8).
__device__ __forceinline__ void store16(void *row, int c, int width, const uint32_t (&w)[8])
{
    uint4 *dst = reinterpret_cast<uint4 *>(static_cast<uint16_t *>(row) + c);
    if (c < width) dst[0] = make_uint4(w[0], w[1], w[2], w[3]);
    if (c + 8 < width) dst[1] = make_uint4(w[4], w[5], w[6], w[7]);
}

// The lane's row of a staged block: 16-byte piece i.
__device__ __forceinline__ uint32_t piece16(uint32_t block, int lane, int i) { return block + lane * 64 + ((i ^ ((lane >> 1) & 3)) << 4); }
__device__ __forceinline__ uint32_t piece8(uint32_t block, int lane, int i) { return block + lane * 32 + ((i ^ ((lane >> 2) & 1)) << 4); }

__device__ __forceinline__ void put(uint32_t addr, uint32_t a, uint32_t b, uint32_t c, uint32_t d)
{
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}

__device__ __forceinline__ uint4 get(uint32_t addr)
{
    uint4 v;
    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr) : "memory");
    return v;
}

// Elements [8 i, 8 i + 8) of the lane's row, as the upper 24 bits of binary32 numbers in the two planes.
__device__ __forceinline__ void put_upper(uint32_t block, int lane, int i, const uint32_t *v)
{
    put(piece16(block, lane, i), __byte_perm(v[0], v[1], 0x7632), __byte_perm(v[2], v[3], 0x7632),
        __byte_perm(v[4], v[5], 0x7632), __byte_perm(v[6], v[7], 0x7632));
}

__device__ __forceinline__ uint32_t third_bytes(uint32_t a, uint32_t b, uint32_t c, uint32_t d)
{
    return __byte_perm(__byte_perm(a, b, 0x0051), __byte_perm(c, d, 0x0051), 0x5410);
}

// Element e (0..3) of a word pair of the upper plane and a word of the lower one.
__device__ __forceinline__ float join24(uint32_t upper, uint32_t lower, int e)
{
    // result bytes, low to high: 0, lower[e], the two bytes of upper's half e & 1
    const uint32_t shifted = __byte_perm(lower, 0, 0x4404 | (e << 4));           // 0, lower[e], 0, 0
    return __uint_as_float(__byte_perm(shifted, upper, e & 1 ? 0x7610 : 0x5410));
}

// A block of one plane (0: g, 1: u) of a [rows][2][columns] array, with this block's own barrier.
__device__ __forceinline__ void tma_load_plane(uint32_t dst, const CUtensorMap *map, int x, int plane, int y, uint32_t bar)
{
    asm volatile(
        "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(dst),
        "l"(map), "r"(x), "r"(plane), "r"(y), "r"(bar)
        : "memory");
}

__device__ __forceinline__ void tma_store_plane(const CUtensorMap *map, int x, int plane, int y, uint32_t src)
{
    asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.tile.bulk_group [%0, {%1, %2, %3}], [%4];" ::"l"(map), "r"(x),
                 "r"(plane), "r"(y), "r"(src)
                 : "memory");
}

// 8 consecutive accumulator columns of this thread's lane.
__device__ __forceinline__ void tmem_ld8(uint32_t taddr, uint32_t (&v)[8])
{
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7])
                 : "r"(taddr)
                 : "memory");
}

__device__ __forceinline__ void tma_store(const CUtensorMap *map, int x, int y, uint32_t src)
{
    asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.tile.bulk_group [%0, {%1, %2}], [%3];" ::"l"(map), "r"(x),
                 "r"(y), "r"(src)
                 : "memory");
}

__device__ __forceinline__ void bulk_commit() { asm volatile("cp.async.bulk.commit_group;" ::: "memory"); }
// The copies' reads of shared memory are done.
__device__ __forceinline__ void bulk_wait_read() { asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory"); }
__device__ __forceinline__ void bulk_wait() { asm volatile("cp.async.bulk.wait_group 0;" ::: "memory"); }
__device__ __forceinline__ void fence_async() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

// The memory that the epilogues of kGated and kSlope reach by TMA.  [g | u] and [dg | du] are [rows][2][hidden]
// to the copies: a block at the last columns of one projection must not run into the other.
struct Maps {
    CUtensorMap out;            // kGated: hidden units [rows][hidden]; kSlope: [dg | du]
    CUtensorMap upper, lower;   // planes of [g | u]
};

template <typename T, int kMode, bool kGelu>
__global__ void __launch_bounds__(kThreads, 1)
k_product(const __grid_constant__ CUtensorMap tm_a, const __grid_constant__ CUtensorMap tm_b,
          const __grid_constant__ Maps maps, const __grid_constant__ Product p)
{
    constexpr int kStages = stages_of(kMode);
    extern __shared__ uint8_t smem_raw[];
    const uint32_t raw = smem_u32(smem_raw);
    const uint32_t tiles = (raw + 1023u) & ~1023u;
    const uint32_t staging = tiles + kStages * kStageBytes;
    const uint32_t bars = staging + kEpilogueWarps * staging_of(kMode);
    uint8_t *bars_ptr = smem_raw + (bars - raw);
    const uint32_t full0 = bars, empty0 = bars + 8 * kStages;
    const uint32_t acc_full0 = bars + 16 * kStagesMost, acc_empty0 = acc_full0 + 16;
    const uint32_t pre_full0 = acc_empty0 + 16;              // two per epilogue warp (kSlope)
    volatile uint32_t *tmem_slot = reinterpret_cast<volatile uint32_t *>(bars_ptr + 16 * kStagesMost + 32 + 128);
    volatile int *abort_flag = reinterpret_cast<volatile int *>(bars_ptr + 16 * kStagesMost + 32 + 128 + 8);

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = cluster_cta_rank();
    const int pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;
    const int tile_n = kMode == kGated ? 2 * p.tile_n : p.tile_n;     // accumulator columns
    const int b_half = tile_n / 2;

    if (threadIdx.x == 0) {
        for (int s = 0; s < kStages; ++s) {
            mbar_init(full0 + 8 * s, 1);
            mbar_init(empty0 + 8 * s, 1);
        }
        for (int b = 0; b < 2; ++b) {
            mbar_init(acc_full0 + 8 * b, 1);
            mbar_init(acc_empty0 + 8 * b, 2 * kEpilogueWarps);
        }
        for (int i = 0; i < 2 * kEpilogueWarps; ++i) mbar_init(pre_full0 + 8 * i, 1);
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
    wait_for_previous();                     // operands may be its results, and outputs what it still reads

    if (warp == 0) {
        if (lane == 0) {
            uint32_t s = 0, ph = 0;
            bool ok = true;
            const int b_boxes = (b_half + 63) / 64;
            const uint32_t bytes = kABytes + (p.b_rows ? b_boxes * 64 * kBK * 2 : b_half * kBK * 2);
            Walk w(p, pair, pairs);
            while (ok && w.next()) {
                const int a0 = w.row_tile() * kTileM + static_cast<int>(rank) * kRowsPerBlock;
                const int b0 = kMode == kGated ? w.col_tile() * p.tile_n + static_cast<int>(rank) * p.n
                                               : w.col_tile() * tile_n + static_cast<int>(rank) * b_half;
                for (int kc = w.k0; kc < w.k1; ++kc) {
                    if (!mbar_wait(empty0 + 8 * s, ph ^ 1u, abort_flag)) {
                        ok = false;
                        break;
                    }
                    const uint32_t dst = tiles + s * kStageBytes;
                    const uint32_t full = map_to_rank(full0 + 8 * s, 0);
                    if (rank == 0) mbar_expect_tx(full0 + 8 * s, 2 * bytes);
                    if (p.a_rows) {
                        tma_load_2d(dst, &tm_a, a0, kc * kBK, full);
                        tma_load_2d(dst + kABytes / 2, &tm_a, a0 + 64, kc * kBK, full);
                    } else {
                        tma_load_2d(dst, &tm_a, kc * kBK, a0, full);
                    }
                    if (p.b_rows) {
                        for (int i = 0; i < b_boxes; ++i)
                            tma_load_2d(dst + kABytes + i * 64 * kBK * 2, &tm_b, b0 + 64 * i, kc * kBK, full);
                    } else {
                        tma_load_2d(dst + kABytes, &tm_b, kc * kBK, b0, full);
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
            const uint32_t idesc = (1u << 4) | (Type<T>::kFormat << 7) | (Type<T>::kFormat << 10) |
                                   (static_cast<uint32_t>(p.a_rows) << 15) | (static_cast<uint32_t>(p.b_rows) << 16) |
                                   (static_cast<uint32_t>(tile_n >> 3) << 17) | (static_cast<uint32_t>(kTileM >> 4) << 24);
            // 16 reduction elements: 32 bytes along a K-major row, 16 rows of 128 bytes MN-major
            const uint32_t a_step = p.a_rows ? 2048 >> 4 : 32 >> 4, b_step = p.b_rows ? 2048 >> 4 : 32 >> 4;
            uint32_t s = 0, ph = 0;
            bool ok = true;
            int it = 0;
            for (Walk w(p, pair, pairs); ok && w.next(); ++it) {
                const uint32_t buf = it & 1, use = (it >> 1) & 1;
                if (!mbar_wait(acc_empty0 + 8 * buf, use ^ 1u, abort_flag)) break;
                tc_fence_after_sync();
                const uint32_t d = tmem_base + buf * kAccCols;
                for (int kc = w.k0; kc < w.k1; ++kc) {
                    if (!mbar_wait(full0 + 8 * s, ph, abort_flag)) {
                        ok = false;
                        break;
                    }
                    tc_fence_after_sync();
                    const uint32_t addr = tiles + s * kStageBytes;
                    const uint64_t ad = p.a_rows ? smem_desc_rows(addr) : smem_desc(addr);
                    const uint64_t bd = p.b_rows ? smem_desc_rows(addr + kABytes) : smem_desc(addr + kABytes);
#pragma unroll
                    for (int k = 0; k < kBK / 16; ++k)
                        umma_bf16(d, ad + a_step * k, bd + b_step * k, idesc, kc > w.k0 || k > 0);
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
        const uint32_t stage = staging + (warp - 2) * staging_of(kMode);
        const uint32_t pre_full = pre_full0 + 16 * (warp - 2);
        uint32_t pre_phase = 0;                          // bit b: parity of the next arrival in buffer b
        int it = 0;
        for (Walk w(p, pair, pairs); w.next(); ++it) {
            const uint32_t buf = it & 1, use = (it >> 1) & 1;
            const int row_in_block = q * 32 + lane;
            const int64_t row = static_cast<int64_t>(w.row_tile()) * kTileM + static_cast<int>(rank) * kRowsPerBlock + row_in_block;
            const int row0 = static_cast<int>(row) - lane;   // the warp's first row
            const bool live = row < p.m;
            const uint32_t t0 = lane_base + buf * kAccCols;
            // kSlope: set i of the tile's four, columns [f, f + 32) of g and u, into buffer i & 1
            auto bring = [&](int i) {
                const int f = w.col_tile() * tile_n + half * (tile_n / 2) + 32 * i;
                const uint32_t dst = stage + (i % kSets) * kPreBytes, bar = pre_full + 8 * (i % kSets);
                mbar_expect_tx(bar, kPreBytes);
                tma_load_plane(dst, &maps.upper, f, 0, row0, bar);
                tma_load_plane(dst + kBlock16, &maps.upper, f, 1, row0, bar);
                tma_load_plane(dst + 2 * kBlock16, &maps.lower, f, 0, row0, bar);
                tma_load_plane(dst + 2 * kBlock16 + kBlock8, &maps.lower, f, 1, row0, bar);
            };
            if (kMode == kSlope && lane == 0) {
                bulk_wait_read();                        // the buffers: the previous tile's results have left
                for (int i = 0; i < kSets; ++i) bring(i);
            }
            const bool ready = mbar_wait(acc_full0 + 8 * buf, use, abort_flag);
            if (!__all_sync(0xFFFFFFFFu, ready)) break;
            tc_fence_after_sync();
            if (kMode == kGated) {
#pragma unroll 1
                for (int c = half * (p.tile_n / 2); c < (half + 1) * (p.tile_n / 2); c += 32) {
                    const int f = w.col_tile() * p.tile_n + c;
                    if (lane == 0) bulk_wait_read();     // the blocks staged before have left
                    __syncwarp();
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        uint32_t g[16], u[16], hw[8];
                        tmem_ld16(t0 + c + 16 * h, g);
                        tmem_ld16(t0 + p.tile_n + c + 16 * h, u);
                        tmem_wait_ld();
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            const float g0 = __uint_as_float(g[2 * i]), g1 = __uint_as_float(g[2 * i + 1]);
                            const float u0 = __uint_as_float(u[2 * i]), u1 = __uint_as_float(u[2 * i + 1]);
                            hw[i] = Type<T>::pack(g0 * act_sigmoid<kGelu>(g0) * u0, g1 * act_sigmoid<kGelu>(g1) * u1);
                        }
                        put(piece16(stage + kPreBytes, lane, 2 * h), hw[0], hw[1], hw[2], hw[3]);
                        put(piece16(stage + kPreBytes, lane, 2 * h + 1), hw[4], hw[5], hw[6], hw[7]);
                        if (p.keep) {
                            put_upper(stage, lane, 2 * h, g);
                            put_upper(stage, lane, 2 * h + 1, g + 8);
                            put_upper(stage + kBlock16, lane, 2 * h, u);
                            put_upper(stage + kBlock16, lane, 2 * h + 1, u + 8);
                            put(piece8(stage + 2 * kBlock16, lane, h), third_bytes(g[0], g[1], g[2], g[3]),
                                third_bytes(g[4], g[5], g[6], g[7]), third_bytes(g[8], g[9], g[10], g[11]),
                                third_bytes(g[12], g[13], g[14], g[15]));
                            put(piece8(stage + 2 * kBlock16 + kBlock8, lane, h), third_bytes(u[0], u[1], u[2], u[3]),
                                third_bytes(u[4], u[5], u[6], u[7]), third_bytes(u[8], u[9], u[10], u[11]),
                                third_bytes(u[12], u[13], u[14], u[15]));
                        }
                    }
                    fence_async();
                    __syncwarp();
                    if (lane == 0 && f < p.n && row0 < p.m) {
                        tma_store(&maps.out, f, row0, stage + kPreBytes);
                        if (p.keep) {
                            tma_store_plane(&maps.upper, f, 0, row0, stage);
                            tma_store_plane(&maps.upper, f, 1, row0, stage + kBlock16);
                            tma_store_plane(&maps.lower, f, 0, row0, stage + 2 * kBlock16);
                            tma_store_plane(&maps.lower, f, 1, row0, stage + 2 * kBlock16 + kBlock8);
                        }
                        bulk_commit();
                    }
                }
            } else if (kMode == kSlope) {
                const int sets = tile_n / 64;
#pragma unroll 1
                for (int i = 0; i < sets; ++i) {
                    const int c = half * (tile_n / 2) + 32 * i, f = w.col_tile() * tile_n + c;
                    const uint32_t pre = stage + (i % kSets) * kPreBytes;
                    const bool here = mbar_wait(pre_full + 8 * (i % kSets), (pre_phase >> (i % kSets)) & 1, abort_flag);
                    pre_phase ^= 1u << (i % kSets);
                    if (!__all_sync(0xFFFFFFFFu, here)) break;
#pragma unroll
                    for (int h = 0; h < 4; ++h) {        // 8 columns at a time
                        uint32_t d[8];
                        tmem_ld8(t0 + c + 8 * h, d);
                        const uint4 gu = get(piece16(pre, lane, h)), uu = get(piece16(pre + kBlock16, lane, h));
                        const uint4 gl4 = get(piece8(pre + 2 * kBlock16, lane, h >> 1));
                        const uint4 ul4 = get(piece8(pre + 2 * kBlock16 + kBlock8, lane, h >> 1));
                        const uint32_t gw[4] = {gu.x, gu.y, gu.z, gu.w}, uw[4] = {uu.x, uu.y, uu.z, uu.w};
                        const uint32_t gl[2] = {h & 1 ? gl4.z : gl4.x, h & 1 ? gl4.w : gl4.y};
                        const uint32_t ul[2] = {h & 1 ? ul4.z : ul4.x, h & 1 ? ul4.w : ul4.y};
                        tmem_wait_ld();
                        uint32_t og[4], ou[4];
#pragma unroll
                        for (int e = 0; e < 8; e += 2) {
                            float dg[2], du[2];
#pragma unroll
                            for (int m = 0; m < 2; ++m) {
                                const float g = join24(gw[e / 2], gl[e / 4], (e + m) & 3);
                                const float u = join24(uw[e / 2], ul[e / 4], (e + m) & 3);
                                const float dh = __uint_as_float(d[e + m]), sg = act_sigmoid<kGelu>(g);
                                dg[m] = dh * u * act_slope<kGelu>(g, sg);
                                du[m] = dh * g * sg;
                            }
                            og[e / 2] = Type<T>::pack(dg[0], dg[1]);
                            ou[e / 2] = Type<T>::pack(du[0], du[1]);
                        }
                        put(piece16(pre, lane, h), og[0], og[1], og[2], og[3]);
                        put(piece16(pre + kBlock16, lane, h), ou[0], ou[1], ou[2], ou[3]);
                    }
                    fence_async();
                    __syncwarp();
                    if (lane == 0) {
                        if (f < p.n && row0 < p.m) {
                            tma_store_plane(&maps.out, f, 0, row0, pre);
                            tma_store_plane(&maps.out, f, 1, row0, pre + kBlock16);
                        }
                        bulk_commit();
                        if (i + kSets < sets) {          // into this buffer
                            bulk_wait_read();
                            bring(i + kSets);
                        }
                    }
                }
            } else if (w.piece >= 0) {
                // [32 rows][16 columns][4][row][4 columns]: a warp's stores, and k_join's loads, are contiguous
                float4 *dst = reinterpret_cast<float4 *>(p.pieces) + piece_at(pair, w.piece, static_cast<int>(rank) * 4 + q, 0) + lane;
#pragma unroll 1
                for (int c = half * (tile_n / 2); c < (half + 1) * (tile_n / 2); c += 16) {
                    uint32_t d[16];
                    tmem_ld16(t0 + c, d);
                    tmem_wait_ld();
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        dst[(c / 16) * 128 + 32 * i] =
                            make_float4(__uint_as_float(d[4 * i]), __uint_as_float(d[4 * i + 1]), __uint_as_float(d[4 * i + 2]),
                                        __uint_as_float(d[4 * i + 3]));
                }
            } else {
                const int c0 = w.col_tile() * tile_n;
                uint16_t *orow = static_cast<uint16_t *>(p.out) + (live ? row : 0) * p.out_stride;
#pragma unroll 1
                for (int c = half * (tile_n / 2); c < (half + 1) * (tile_n / 2); c += 16) {
                    uint32_t d[16], o[8];
                    tmem_ld16(t0 + c, d);
                    tmem_wait_ld();
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        o[i] = Type<T>::pack(__uint_as_float(d[2 * i]), __uint_as_float(d[2 * i + 1]));
                    if (live) store16(orow, c0 + c, p.n, o);
                }
            }
            tc_fence_before_sync();
            __syncwarp();
            if (lane == 0) mbar_arrive_cluster(map_to_rank(acc_empty0 + 8 * buf, 0));
        }
        if (kMode != kStore && lane == 0) bulk_wait();
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

// Adds the pieces of the tiles that were divided: a warp takes 32 rows x 16 columns, a lane a row.
template <typename T>
__global__ void __launch_bounds__(256)
k_join(const Product p, const int pairs)
{
    allow_next();
    wait_for_previous();                                 // in every block: this kernel must not end before that one
    const int index = blockIdx.y;                        // tile of the shared rest
    const int tile = p.rounds * pairs + index;
    const int64_t rest = static_cast<int64_t>(p.m_tiles * p.n_tiles - p.rounds * pairs) * p.steps;
    const int64_t lo = static_cast<int64_t>(index) * p.steps, hi = lo + p.steps;
    // the pairs whose stretch meets [lo, hi): pair i has [rest i / cuts, rest (i + 1) / cuts)
    int first = static_cast<int>(lo * p.cuts / rest);
    while (rest * (first + 1) / p.cuts <= lo) ++first;
    while (first > 0 && rest * first / p.cuts > lo) --first;
    int last = first + 1;
    while (last < p.cuts && rest * last / p.cuts < hi) ++last;
    if (last == first + 1) return;                       // one pair did all of it
    const int part = blockIdx.x * 8 + (threadIdx.x >> 5), lane = threadIdx.x & 31;
    const int rows = part / (kAccCols / 16), cols = part % (kAccCols / 16);
    const int c0 = (p.m_first ? tile / p.m_tiles : tile % p.n_tiles) * p.tile_n + 16 * cols;
    const int64_t row = static_cast<int64_t>(p.m_first ? tile % p.m_tiles : tile / p.n_tiles) * kTileM + rows * 32 + lane;
    if (16 * cols >= p.tile_n || c0 >= p.n) return;
    float4 sum[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) sum[j] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    for (int i = first; i < last; ++i) {
        // the slot of its first stretch if that lies in this tile, else of its last
        const int slot = rest * i / p.cuts / p.steps == index ? 0 : 1;
        const float4 *src = reinterpret_cast<const float4 *>(p.pieces) + piece_at(i, slot, rows, cols) + lane;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float4 v = src[32 * j];
            sum[j] = make_float4(sum[j].x + v.x, sum[j].y + v.y, sum[j].z + v.z, sum[j].w + v.w);
        }
    }
    if (row >= p.m) return;
    uint32_t out[8];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        out[2 * j] = Type<T>::pack(sum[j].x, sum[j].y);
        out[2 * j + 1] = Type<T>::pack(sum[j].z, sum[j].w);
    }
    store16(static_cast<uint16_t *>(p.out) + row * p.out_stride, c0, p.n, out);
}

// ---- few rows

// Rows of x that take k_rows: its blocks read x from L2 once per 16 rows of the weights, k_product's time hardly
// depends on so few rows.  576 x 1,536: 32 rows 8.6, 64 rows 12.1 against 19.7 us; 2,048 x 8,192: 32 rows 41 against 43,
// 64 rows 75 against 44 us: up to 32 rows always, up to 64 while model * hidden is below 4 M.
constexpr int kRowsMax = 64;
inline bool few_rows(int64_t n, int64_t weights) { return n <= 32 || (n <= kRowsMax && weights <= (int64_t{4} << 20)); }


template <typename T>
__device__ __forceinline__ void mma_16x8x16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3,
                                            uint32_t b0, uint32_t b1)
{
    if constexpr (Type<T>::kFormat == 1)
        asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
            "{%0, %1, %2, %3};"
            : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
            : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
    else
        asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
            "{%0, %1, %2, %3};"
            : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
            : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

struct Rows {
    const void *x;
    int64_t x_stride;
    const void *w;              // kGated: [2 * width][k]; else [width][k]
    void *out;
    int64_t out_stride;
    uint16_t *upper;            // kGated: planes of [g | u], or nullptr
    uint8_t *lower;
    int lower_width;
    int n, width, k;            // rows of x, rows of w (one projection), reduction length
    int gelu;
};

// NT: groups of 8 rows of x.  The warps split the reduction: as many as give enough loads in flight (16 where a
// block reads one projection, 8 where it reads both) and as the sums of NT = 8 leave room for.
template <bool kGatedRows, int NT>
struct RowsShape {
    static constexpr int kWarps = (kGatedRows ? 8 : 16) / (NT == 8 ? 2 : 1);
    static constexpr int kDepth = NT <= 2 ? (kGatedRows ? 4 : 8) : 2;    // chunks of 32 reduction elements in flight
};

template <typename T, bool kGatedRows, int NT>
__global__ void __launch_bounds__(32 * RowsShape<kGatedRows, NT>::kWarps)
k_rows(const Rows p)
{
    constexpr int P = kGatedRows ? 2 : 1;
    constexpr int kDepth = RowsShape<kGatedRows, NT>::kDepth, kWarps = RowsShape<kGatedRows, NT>::kWarps;
    __shared__ float s_sum[kWarps][P][16][NT * 8 + 1];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int g = lane >> 2, t = lane & 3;
    const int f0 = blockIdx.x * 16;
    const uint16_t *w = static_cast<const uint16_t *>(p.w);
    const uint16_t *x = static_cast<const uint16_t *>(p.x);
    if (kGatedRows) allow_next();
    bool waited = kGatedRows;
    float acc[P][NT][4];
#pragma unroll
    for (int i = 0; i < P; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[i][j][e] = 0.0f;
    const int chunks = (p.k + 31) / 32;
    const uint4 none = make_uint4(0, 0, 0, 0);
    for (int c0 = warp; c0 < chunks; c0 += kWarps * kDepth) {
        uint4 wv[kDepth][P][2], xv[kDepth][NT];
#pragma unroll
        for (int s = 0; s < kDepth; ++s) {
            const int k = (c0 + s * kWarps) * 32 + 8 * t;
#pragma unroll
            for (int i = 0; i < P; ++i)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int f = f0 + g + 8 * h;
                    wv[s][i][h] = k < p.k && f < p.width
                                      ? __ldg(reinterpret_cast<const uint4 *>(w + (static_cast<int64_t>(i) * p.width + f) * p.k + k))
                                      : none;
                }
        }
        if (!waited) {       // the weights are under way; x is the previous kernel's result
            wait_for_previous();
            waited = true;
        }
#pragma unroll
        for (int s = 0; s < kDepth; ++s) {
            const int k = (c0 + s * kWarps) * 32 + 8 * t;
#pragma unroll
            for (int j = 0; j < NT; ++j) {
                const int r = 8 * j + g;
                xv[s][j] = k < p.k && r < p.n ? *reinterpret_cast<const uint4 *>(x + r * p.x_stride + k) : none;
            }
        }
#pragma unroll
        for (int s = 0; s < kDepth; ++s)
#pragma unroll
            for (int i = 0; i < P; ++i)
#pragma unroll
                for (int j = 0; j < NT; ++j) {
                    mma_16x8x16<T>(acc[i][j], wv[s][i][0].x, wv[s][i][1].x, wv[s][i][0].y, wv[s][i][1].y, xv[s][j].x, xv[s][j].y);
                    mma_16x8x16<T>(acc[i][j], wv[s][i][0].z, wv[s][i][1].z, wv[s][i][0].w, wv[s][i][1].w, xv[s][j].z, xv[s][j].w);
                }
    }
#pragma unroll
    for (int i = 0; i < P; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) s_sum[warp][i][g + 8 * (e >> 1)][8 * j + 2 * t + (e & 1)] = acc[i][j][e];
    __syncthreads();
    if (!waited) wait_for_previous();
    for (int i = threadIdx.x; i < 16 * NT * 8; i += 32 * kWarps) {
        const int f = i % 16, r = i / 16;
        if (r >= p.n || f0 + f >= p.width) continue;
        float v[P];
#pragma unroll
        for (int e = 0; e < P; ++e) {
            v[e] = 0.0f;
            for (int k = 0; k < kWarps; ++k) v[e] += s_sum[k][e][f][r];
        }
        T *out = static_cast<T *>(p.out) + r * p.out_stride + f0 + f;
        if constexpr (kGatedRows) {
            *out = static_cast<T>(v[0] * (p.gelu ? act_sigmoid<true>(v[0]) : act_sigmoid<false>(v[0])) * v[1]);
            if (p.upper != nullptr) {
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const uint32_t bits = __float_as_uint(v[e]);
                    p.upper[(static_cast<int64_t>(r) * 2 + e) * p.width + f0 + f] = static_cast<uint16_t>(bits >> 16);
                    p.lower[(static_cast<int64_t>(r) * 2 + e) * p.lower_width + f0 + f] = static_cast<uint8_t>(bits >> 8);
                }
            }
        } else {
            *out = static_cast<T>(v[0]);
        }
    }
}

// ---------------------------------------------------------------- host side

// An operand in the type T: rows x cols (cols contiguous), boxes of 64 columns by box_rows rows.
bool encode(CUtensorMapDataType type, CUtensorMap *m, const void *base, int64_t rows, int64_t cols, int64_t stride,
            uint32_t box_rows)
{
    const cuuint64_t dims[2] = {static_cast<cuuint64_t>(cols), static_cast<cuuint64_t>(rows)};
    const cuuint64_t strides[1] = {static_cast<cuuint64_t>(stride) * 2};
    const cuuint32_t box[2] = {kBK, box_rows};
    const cuuint32_t elem_strides[2] = {1, 1};
    return tensor_map_encoder()(m, type, 2, const_cast<void *>(base), dims, strides, box, elem_strides,
                                CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                                CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// [rows][2][cols] seen by copies of 32 columns of one plane x 32 rows.  pitch: bytes between planes (a row is two).
bool encode_planes(CUtensorMapDataType type, CUtensorMap *m, const void *base, int64_t rows, int64_t cols, int64_t pitch,
                   CUtensorMapSwizzle swizzle)
{
    const cuuint64_t dims[3] = {static_cast<cuuint64_t>(cols), 2, static_cast<cuuint64_t>(rows)};
    const cuuint64_t strides[2] = {static_cast<cuuint64_t>(pitch), static_cast<cuuint64_t>(2 * pitch)};
    const cuuint32_t box[3] = {32, 1, 32};
    const cuuint32_t elem_strides[3] = {1, 1, 1};
    return tensor_map_encoder()(m, type, 3, const_cast<void *>(base), dims, strides, box, elem_strides,
                                CU_TENSOR_MAP_INTERLEAVE_NONE, swizzle, CU_TENSOR_MAP_L2_PROMOTION_L2_128B,
                                CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

bool encode_blocks(CUtensorMapDataType type, CUtensorMap *m, const void *base, int64_t rows, int64_t cols)
{
    const cuuint64_t dims[2] = {static_cast<cuuint64_t>(cols), static_cast<cuuint64_t>(rows)};
    const cuuint64_t strides[1] = {static_cast<cuuint64_t>(cols) * 2};
    const cuuint32_t box[2] = {32, 32};
    const cuuint32_t elem_strides[2] = {1, 1};
    return tensor_map_encoder()(m, type, 2, const_cast<void *>(base), dims, strides, box, elem_strides,
                                CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_64B,
                                CU_TENSOR_MAP_L2_PROMOTION_L2_128B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// g and u as the caller keeps them: the upper planes [n][2][hidden] of 16 bits, then, 256-byte aligned, the
// lower ones [n][2][hidden rounded up to 16] of 8 bits (the copies want rows of whole 16-byte pieces).
int64_t lower_width(int hidden) { return (hidden + 15) / 16 * 16; }
size_t upper_bytes(int64_t n, int hidden) { return (static_cast<size_t>(n) * hidden * 4 + 255) & ~static_cast<size_t>(255); }

}  // namespace

struct gated_ffn {
    int model = 0, hidden = 0, activation = 0, type = 0;
    int device = 0, sms = 0, pairs = 0;
    cudaStream_t stream = nullptr;
    int64_t launches = 0;
    int *err = nullptr;
};

namespace {

int64_t div_up(int64_t a, int64_t b) { return (a + b - 1) / b; }

struct Operand {
    const void *ptr;
    int64_t stride;   // elements between stored rows
    int by_rows;      // 1: stored [k][rows]
};

// Sizes and the cut of D[m][n] = A B^T.
Product plan(const gated_ffn *p, int mode, int64_t m, int n, int64_t k)
{
    Product q = {};
    q.m = m;
    q.n = n;
    q.k = k;
    if (mode == kStore) {
        // an incomplete round is shared by all pairs: the narrowest total width wins, the widest tile among equals
        q.tile_n = 256;
        const int widths[2] = {192, 128};
        for (int w : widths)
            if (div_up(n, w) * w < div_up(n, q.tile_n) * q.tile_n) q.tile_n = w;
    } else {
        // Whole rounds only: the fewest rounds times a tile's cost.  Half the columns cost more than half (the rows of A
        // are shared by fewer): 0.7 measured (1,003 x 1,000 x 2,504: three rounds of 64 units 24.5 us, two of 128 22.1 us), so a
        // narrow tile pays where the wide ones are too few for the pairs.
        const int widths[3] = {256, 192, 128};
        int64_t best = -1;
        for (int w : widths) {
            const int units = mode == kGated ? w / 2 : w;
            if (mode == kGated && w == 192) continue;      // its halves of 48 units are no multiple of a staged block
            const int64_t cost = div_up(div_up(m, kTileM) * div_up(n, units), p->pairs) * (w + 192);
            if (best < 0 || cost < best) {
                best = cost;
                q.tile_n = units;
            }
        }
    }
    q.m_tiles = static_cast<int>(div_up(m, kTileM));
    q.n_tiles = static_cast<int>(div_up(n, q.tile_n));
    // Neighbouring tiles, worked on at the same time, share the operand of the longer side; the
    // shorter side's operand is the smaller one and stays in L2.
    q.m_first = q.m_tiles <= q.n_tiles;
    q.steps = static_cast<int>(div_up(k, kBK));
    const int64_t tiles = static_cast<int64_t>(q.m_tiles) * q.n_tiles;
    q.rounds = static_cast<int>(tiles / p->pairs);
    const int64_t rest = tiles % p->pairs;
    // an incomplete round is cut over all pairs unless it is nearly complete: joining pieces costs
    // about a sixth of a round
    if (rest > 0 && (mode != kStore || 6 * rest > 5 * p->pairs)) {
        ++q.rounds;
    } else if (rest > 0) {
        int64_t cuts = rest * q.steps / kMinSteps;
        if (cuts < rest) cuts = rest;
        q.cuts = static_cast<int>(cuts < p->pairs ? cuts : p->pairs);
    }
    q.err = p->err;
    return q;
}

size_t pieces_bytes(const Product &q) { return static_cast<size_t>(q.cuts) * 2 * kTileM * kAccCols * sizeof(float); }

// A launch that may start while the kernel before it on the stream still runs (the kernels say where they wait for it).
template <typename... Params, typename... Args>
bool launch_overlapped(cudaStream_t stream, dim3 grid, unsigned threads, void (*kernel)(Params...), Args... args)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(threads);
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, args...) == cudaSuccess;
}

// after_own: the launch before it on the stream is one of this call's, which allow it to start early.
template <typename T, int kMode>
int launch_product(gated_ffn *p, Product q, const Operand &a, const Operand &b, const Maps &maps, bool after_own)
{
    CUtensorMap tm_a, tm_b;
    const CUtensorMapDataType type = Type<T>::kMap;
    const int64_t b_total = kMode == kGated ? 2 * static_cast<int64_t>(q.n) : q.n;
    const uint32_t b_box = kMode == kGated ? q.tile_n : q.tile_n / 2;
    q.a_rows = a.by_rows;
    q.b_rows = b.by_rows;
    const bool ok = (a.by_rows ? encode(type, &tm_a, a.ptr, q.k, q.m, a.stride, kBK)
                               : encode(type, &tm_a, a.ptr, q.m, q.k, a.stride, kRowsPerBlock)) &&
                    (b.by_rows ? encode(type, &tm_b, b.ptr, q.k, b_total, b.stride, kBK)
                               : encode(type, &tm_b, b.ptr, b_total, q.k, b.stride, b_box));
    if (!ok) return GATED_FFN_ECUDA;
    const int64_t tiles = static_cast<int64_t>(q.m_tiles) * q.n_tiles;
    // a full grid, unless there is less than one round (then the walk's rounds count that grid's pairs)
    int pairs = p->pairs;
    if (q.rounds == 0) pairs = q.cuts;
    else if (q.cuts == 0 && tiles < pairs) pairs = static_cast<int>(tiles);
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(2 * pairs));
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = smem_of(kMode);
    cfg.stream = p->stream;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = 2;
    attr[0].val.clusterDim.y = 1;
    attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = after_own ? 2 : 1;
    auto kernel = kMode != kStore && p->activation == GATED_FFN_GELU ? k_product<T, kMode, kMode != kStore> : k_product<T, kMode, false>;
    if (cudaLaunchKernelEx(&cfg, kernel, tm_a, tm_b, maps, q) != cudaSuccess) {
        cudaGetLastError();
        return GATED_FFN_ECUDA;
    }
    p->launches += 1;
    if (q.cuts > 1) {
        const dim3 grid((kTileM / 32) * (kAccCols / 16) / 8, static_cast<unsigned>(tiles - static_cast<int64_t>(q.rounds) * pairs));
        if (!launch_overlapped(p->stream, grid, 256, k_join<T>, q, pairs)) {
            cudaGetLastError();
            return GATED_FFN_ECUDA;
        }
        p->launches += 1;
    }
    return GATED_FFN_OK;
}

template <typename T, bool kGatedRows, int NT>
bool launch_rows_of(gated_ffn *p, const Rows &r)
{
    const dim3 grid(static_cast<unsigned>(div_up(r.width, 16)));
    constexpr unsigned kThreadsOf = 32 * RowsShape<kGatedRows, NT>::kWarps;
    if (!kGatedRows) return launch_overlapped(p->stream, grid, kThreadsOf, k_rows<T, kGatedRows, NT>, r);
    k_rows<T, kGatedRows, NT><<<grid, kThreadsOf, 0, p->stream>>>(r);
    return cudaGetLastError() == cudaSuccess;
}

template <typename T, bool kGatedRows>
int launch_rows(gated_ffn *p, const Rows &r)
{
    const bool ok = r.n <= 8    ? launch_rows_of<T, kGatedRows, 1>(p, r)
                    : r.n <= 16 ? launch_rows_of<T, kGatedRows, 2>(p, r)
                    : r.n <= 32 ? launch_rows_of<T, kGatedRows, 4>(p, r)
                                : launch_rows_of<T, kGatedRows, 8>(p, r);
    if (!ok) {
        cudaGetLastError();
        return GATED_FFN_ECUDA;
    }
    p->launches += 1;
    return GATED_FFN_OK;
}

// The maps of kGated (out: hidden) and kSlope (out: [dg | du]).
template <typename T>
bool encode_maps(const gated_ffn *p, Maps *m, bool slope, void *out, const void *pre, int64_t n)
{
    const int64_t f = p->hidden;
    bool ok = slope ? encode_planes(Type<T>::kMap, &m->out, out, n, f, 2 * f, CU_TENSOR_MAP_SWIZZLE_64B)
                    : encode_blocks(Type<T>::kMap, &m->out, out, n, f);
    if (pre != nullptr)
        ok = ok && encode_planes(CU_TENSOR_MAP_DATA_TYPE_UINT16, &m->upper, pre, n, f, 2 * f, CU_TENSOR_MAP_SWIZZLE_64B) &&
             encode_planes(CU_TENSOR_MAP_DATA_TYPE_UINT8, &m->lower, static_cast<const uint8_t *>(pre) + upper_bytes(n, p->hidden),
                           n, f, lower_width(p->hidden), CU_TENSOR_MAP_SWIZZLE_32B);
    return ok;
}

template <typename T>
int run_forward(gated_ffn *p, const void *x, int64_t x_stride, const void *w_in, const void *w_out, void *pre,
                void *hidden, void *y, int64_t y_stride, float *scratch, int64_t n)
{
    Maps maps = {};
    if (few_rows(n, static_cast<int64_t>(p->model) * p->hidden)) {
        Rows r = {};
        r.x = x;
        r.x_stride = x_stride;
        r.w = w_in;
        r.out = hidden;
        r.out_stride = p->hidden;
        if (pre != nullptr) {
            r.upper = static_cast<uint16_t *>(pre);
            r.lower = static_cast<uint8_t *>(pre) + upper_bytes(n, p->hidden);
            r.lower_width = static_cast<int>(lower_width(p->hidden));
        }
        r.n = static_cast<int>(n);
        r.width = p->hidden;
        r.k = p->model;
        r.gelu = p->activation == GATED_FFN_GELU;
        const int rc = launch_rows<T, true>(p, r);
        if (rc != GATED_FFN_OK) return rc;
        Rows s = {};
        s.x = hidden;
        s.x_stride = p->hidden;
        s.w = w_out;
        s.out = y;
        s.out_stride = y_stride;
        s.n = static_cast<int>(n);
        s.width = p->model;
        s.k = p->hidden;
        return launch_rows<T, false>(p, s);
    }
    Product q = plan(p, kGated, n, p->hidden, p->model);
    q.keep = pre != nullptr;
    if (!encode_maps<T>(p, &maps, false, hidden, pre, n)) return GATED_FFN_ECUDA;
    const int rc = launch_product<T, kGated>(p, q, {x, x_stride, 0}, {w_in, p->model, 0}, maps, false);
    if (rc != GATED_FFN_OK) return rc;
    Product r = plan(p, kStore, n, p->model, p->hidden);
    r.out = y;
    r.out_stride = y_stride;
    r.pieces = scratch;
    return launch_product<T, kStore>(p, r, {hidden, p->hidden, 0}, {w_out, p->hidden, 0}, maps, true);
}

struct BackwardPlan {
    Product slope, dx, dw_in, dw_out;
    size_t dpre, pieces, total;
};

BackwardPlan plan_backward(const gated_ffn *p, int64_t n)
{
    BackwardPlan b;
    b.slope = plan(p, kSlope, n, p->hidden, p->model);
    b.dx = plan(p, kStore, n, p->model, 2 * static_cast<int64_t>(p->hidden));
    b.dw_in = plan(p, kStore, 2 * static_cast<int64_t>(p->hidden), p->model, n);
    b.dw_out = plan(p, kStore, p->model, p->hidden, n);
    b.dpre = 0;
    b.pieces = (static_cast<size_t>(n) * 2 * p->hidden * 2 + 255) & ~static_cast<size_t>(255);
    // the products follow one another on the stream: one set of pieces serves all
    size_t most = pieces_bytes(b.dx);
    if (pieces_bytes(b.dw_in) > most) most = pieces_bytes(b.dw_in);
    if (pieces_bytes(b.dw_out) > most) most = pieces_bytes(b.dw_out);
    b.total = b.pieces + most;
    return b;
}

template <typename T>
int run_backward(gated_ffn *p, const void *dy, int64_t dy_stride, const void *x, int64_t x_stride, const void *w_in,
                 const void *w_out, const void *pre, const void *hidden, void *dx, int64_t dx_stride, void *dw_in,
                 void *dw_out, uint8_t *scratch, int64_t n)
{
    BackwardPlan b = plan_backward(p, n);
    void *dpre = scratch + b.dpre;
    float *pieces = reinterpret_cast<float *>(scratch + b.pieces);
    const int64_t f = p->hidden, d = p->model;
    Maps maps = {};
    if (!encode_maps<T>(p, &maps, true, dpre, pre, n)) return GATED_FFN_ECUDA;
    int rc = launch_product<T, kSlope>(p, b.slope, {dy, dy_stride, 0}, {w_out, f, 1}, maps, false);
    if (rc != GATED_FFN_OK) return rc;
    b.dx.pieces = b.dw_in.pieces = b.dw_out.pieces = pieces;
    if (dx != nullptr) {
        b.dx.out = dx;
        b.dx.out_stride = dx_stride;
        rc = launch_product<T, kStore>(p, b.dx, {dpre, 2 * f, 0}, {w_in, d, 1}, maps, true);
        if (rc != GATED_FFN_OK) return rc;
    }
    b.dw_in.out = dw_in;
    b.dw_in.out_stride = d;
    rc = launch_product<T, kStore>(p, b.dw_in, {dpre, 2 * f, 1}, {x, x_stride, 1}, maps, true);
    if (rc != GATED_FFN_OK) return rc;
    b.dw_out.out = dw_out;
    b.dw_out.out_stride = f;
    return launch_product<T, kStore>(p, b.dw_out, {dy, dy_stride, 1}, {hidden, f, 1}, maps, true);
}

bool aligned16(const void *v) { return reinterpret_cast<uintptr_t>(v) % 16 == 0; }

bool rows_ok(const gated_ffn *p, int64_t n)
{
    // rows and tile counts are 32-bit in the kernels
    return n >= 1 && n <= 0x7FFFFF00 &&
           div_up(n, kTileM) * div_up(2 * static_cast<int64_t>(p->hidden > p->model ? p->hidden : p->model), 128) < 0x7FFFFFFF;
}

bool stride_ok(int64_t stride, int64_t width) { return stride >= width && stride % 8 == 0; }

template <typename T>
bool prepare_kernels(int *pairs, int sms)
{
    if (!raise_dynamic_smem(reinterpret_cast<const void *>(k_product<T, kStore, false>), smem_of(kStore)) ||
        !raise_dynamic_smem(reinterpret_cast<const void *>(k_product<T, kGated, false>), smem_of(kGated)) ||
        !raise_dynamic_smem(reinterpret_cast<const void *>(k_product<T, kGated, true>), smem_of(kGated)) ||
        !raise_dynamic_smem(reinterpret_cast<const void *>(k_product<T, kSlope, false>), smem_of(kSlope)) ||
        !raise_dynamic_smem(reinterpret_cast<const void *>(k_product<T, kSlope, true>), smem_of(kSlope)))
        return false;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(sms & ~1));
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = smem_of(kStore);
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = 2;
    attr[0].val.clusterDim.y = 1;
    attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    int clusters = 0;
    if (cudaOccupancyMaxActiveClusters(&clusters, k_product<T, kStore, false>, &cfg) != cudaSuccess || clusters < 1) return false;
    *pairs = clusters < sms / 2 ? clusters : sms / 2;
    return true;
}

}  // namespace

extern "C" {

int gated_ffn_create(gated_ffn **out, int model, int hidden, int activation, int type)
{
    if (out == nullptr) return GATED_FFN_ENULL;
    *out = nullptr;
    if (model < 8 || model > GATED_FFN_MAX_WIDTH || model % 8 != 0) return GATED_FFN_EINVAL;
    if (hidden < 8 || hidden > GATED_FFN_MAX_WIDTH || hidden % 8 != 0) return GATED_FFN_EINVAL;
    if (activation != GATED_FFN_SILU && activation != GATED_FFN_GELU) return GATED_FFN_EINVAL;
    if (type != GATED_FFN_BF16 && type != GATED_FFN_F16) return GATED_FFN_EINVAL;
    if (tensor_map_encoder() == nullptr) return GATED_FFN_ECUDA;
    gated_ffn *p = new (std::nothrow) gated_ffn;
    if (p == nullptr) return GATED_FFN_ENOMEM;
    p->model = model;
    p->hidden = hidden;
    p->activation = activation;
    p->type = type;
    bool ok = cudaGetDevice(&p->device) == cudaSuccess &&
              cudaDeviceGetAttribute(&p->sms, cudaDevAttrMultiProcessorCount, p->device) == cudaSuccess;
    ok = ok && (type == GATED_FFN_BF16 ? prepare_kernels<__nv_bfloat16>(&p->pairs, p->sms)
                                       : prepare_kernels<__half>(&p->pairs, p->sms));
    if (!ok) {
        cudaGetLastError();
        delete p;
        return GATED_FFN_ECUDA;
    }
    if (cudaMalloc(reinterpret_cast<void **>(&p->err), sizeof(int)) != cudaSuccess) {
        cudaGetLastError();
        delete p;
        return GATED_FFN_ENOMEM;
    }
    if (cudaMemset(p->err, 0, sizeof(int)) != cudaSuccess) {
        cudaGetLastError();
        cudaFree(p->err);
        delete p;
        return GATED_FFN_ECUDA;
    }
    *out = p;
    return GATED_FFN_OK;
}

int gated_ffn_destroy(gated_ffn *p)
{
    if (p == nullptr) return GATED_FFN_ENULL;
    const OnDevice on(p->device);
    cudaStreamSynchronize(p->stream);
    cudaFree(p->err);
    delete p;
    return GATED_FFN_OK;
}

int gated_ffn_set_stream(gated_ffn *p, void *cuda_stream)
{
    if (p == nullptr) return GATED_FFN_ENULL;
    p->stream = static_cast<cudaStream_t>(cuda_stream);
    return GATED_FFN_OK;
}

size_t gated_ffn_workspace_bytes(const gated_ffn *p, int64_t n, int backward)
{
    if (p == nullptr || !rows_ok(p, n)) return 0;
    if (backward) return plan_backward(p, n).total;
    return few_rows(n, static_cast<int64_t>(p->model) * p->hidden) ? 0 : pieces_bytes(plan(p, kStore, n, p->model, p->hidden));
}

size_t gated_ffn_pre_bytes(const gated_ffn *p, int64_t n)
{
    if (p == nullptr || !rows_ok(p, n)) return 0;
    return upper_bytes(n, p->hidden) + static_cast<size_t>(n) * 2 * lower_width(p->hidden);
}

int gated_ffn_forward(gated_ffn *p, const void *x, int64_t x_stride, const void *w_in, const void *w_out, void *pre,
                      void *hidden, void *y, int64_t y_stride, void *workspace, size_t workspace_bytes, int64_t n)
{
    if (p == nullptr) return GATED_FFN_ENULL;
    if (!rows_ok(p, n)) return GATED_FFN_EINVAL;      // first: an empty batch comes without pointers
    if (x == nullptr || w_in == nullptr || w_out == nullptr || hidden == nullptr || y == nullptr) return GATED_FFN_ENULL;
    if (!stride_ok(x_stride, p->model) || !stride_ok(y_stride, p->model)) return GATED_FFN_EINVAL;
    for (const void *v : {x, w_in, w_out, static_cast<const void *>(pre), static_cast<const void *>(hidden),
                          static_cast<const void *>(y), static_cast<const void *>(workspace)})
        if (!aligned16(v)) return GATED_FFN_EALIGN;
    const size_t need = gated_ffn_workspace_bytes(p, n, 0);
    if (need > 0 && workspace == nullptr) return GATED_FFN_ENULL;
    if (need > workspace_bytes) return GATED_FFN_ENOMEM;
    const OnDevice on(p->device);
    if (!on.ok()) return GATED_FFN_ECUDA;
    float *scratch = static_cast<float *>(workspace);
    return p->type == GATED_FFN_BF16
               ? run_forward<__nv_bfloat16>(p, x, x_stride, w_in, w_out, pre, hidden, y, y_stride, scratch, n)
               : run_forward<__half>(p, x, x_stride, w_in, w_out, pre, hidden, y, y_stride, scratch, n);
}

int gated_ffn_backward(gated_ffn *p, const void *dy, int64_t dy_stride, const void *x, int64_t x_stride,
                       const void *w_in, const void *w_out, const void *pre, const void *hidden, void *dx,
                       int64_t dx_stride, void *dw_in, void *dw_out, void *workspace, size_t workspace_bytes,
                       int64_t n)
{
    if (p == nullptr) return GATED_FFN_ENULL;
    if (!rows_ok(p, n)) return GATED_FFN_EINVAL;
    if (dy == nullptr || x == nullptr || w_in == nullptr || w_out == nullptr || pre == nullptr || hidden == nullptr ||
        dw_in == nullptr || dw_out == nullptr || workspace == nullptr)
        return GATED_FFN_ENULL;
    if (!stride_ok(dy_stride, p->model) || !stride_ok(x_stride, p->model) ||
        (dx != nullptr && !stride_ok(dx_stride, p->model)))
        return GATED_FFN_EINVAL;
    for (const void *v : {dy, x, w_in, w_out, pre, hidden, static_cast<const void *>(dx),
                          static_cast<const void *>(dw_in), static_cast<const void *>(dw_out),
                          static_cast<const void *>(workspace)})
        if (!aligned16(v)) return GATED_FFN_EALIGN;
    if (gated_ffn_workspace_bytes(p, n, 1) > workspace_bytes) return GATED_FFN_ENOMEM;
    const OnDevice on(p->device);
    if (!on.ok()) return GATED_FFN_ECUDA;
    uint8_t *scratch = static_cast<uint8_t *>(workspace);
    return p->type == GATED_FFN_BF16 ? run_backward<__nv_bfloat16>(p, dy, dy_stride, x, x_stride, w_in, w_out, pre,
                                                                   hidden, dx, dx_stride, dw_in, dw_out, scratch, n)
                                     : run_backward<__half>(p, dy, dy_stride, x, x_stride, w_in, w_out, pre, hidden,
                                                            dx, dx_stride, dw_in, dw_out, scratch, n);
}

int gated_ffn_status(gated_ffn *p)
{
    if (p == nullptr) return GATED_FFN_ENULL;
    const OnDevice on(p->device);
    if (!on.ok() || cudaStreamSynchronize(p->stream) != cudaSuccess) return GATED_FFN_ECUDA;
    int flag = 0;
    if (cudaMemcpy(&flag, p->err, sizeof(int), cudaMemcpyDeviceToHost) != cudaSuccess) return GATED_FFN_ECUDA;
    if (flag != 0) {
        cudaMemset(p->err, 0, sizeof(int));
        return GATED_FFN_ETIMEOUT;
    }
    return GATED_FFN_OK;
}

int64_t gated_ffn_launch_count(const gated_ffn *p) { return p ? p->launches : 0; }

const char *gated_ffn_strerror(int code)
{
    switch (code) {
    case GATED_FFN_OK: return "ok";
    case GATED_FFN_EINVAL: return "invalid size, stride, type or activation";
    case GATED_FFN_ENULL: return "required pointer is NULL";
    case GATED_FFN_EALIGN: return "pointer not 16-byte aligned";
    case GATED_FFN_ECUDA: return "CUDA call or launch failed";
    case GATED_FFN_ENOMEM: return "allocation failed, or the workspace is too small";
    case GATED_FFN_ETIMEOUT: return "a kernel gave up a bounded wait; its output is invalid";
    default: return "unknown error";
    }
}

}  // extern "C"
