// The dense products on the 5th-generation tensor cores: D = A B^T over operands in device memory, with an epilogue of the
// including file's choice on the accumulators.
//
// One persistent block per multiprocessor, its warps in roles: 16 warps of the epilogue (four to a scheduler hide what one of
// them waits for), one that fetches tiles of 128 bytes of depth by TMA into a ring of shared-memory stages (128-byte swizzle), one that
// issues tcgen05.mma.  Accumulators lie in tensor memory twice, so that the epilogue of a tile runs beside the products of the next.  CTAS = 2: two blocks of a cluster share a tile of 256
// rows; each fetches its 128 rows of A and half of B's rows, and the first one issues products over both halves, so that B
// crosses shared memory once for 256 rows.
//
// An operand is K-major (rows of depth-contiguous elements) or MN-major (its depth is the slow axis; bf16 only here).  Elements past the
// tensor's edges read as zero, which is what pads rows, columns and depth.  The tiles may be split along the depth ("splits").
//
// Every wait is bounded.  If one runs out the block raises a flag that bigcn_sync_check() reports, waits (bounded) for its own copies
// and products in flight, frees its tensor memory and returns.
#pragma once
#include <cuda.h>

#include <algorithm>

#include "bigcn_internal.cuh"
#include "tc_common.cuh"

namespace bigcn {
namespace gemm {

constexpr int kEpiWarps = 16, kProducer = 16, kIssuer = 17, kThreads = 576;
// A tile's columns are shared among four warps for each 32 rows, or among two or one where it is so narrow that four would not have 32 each; then two
// or four groups of warps take tiles in turn (169,343 rows of 256 against 40 8-bit classes in us: 26, 19 so).
__host__ __device__ constexpr int column_parts(int bn) { return bn >= 128 ? 4 : bn / 32; }
__host__ __device__ constexpr int epi_groups(int bn) { return kEpiWarps / 4 / column_parts(bn); }
__host__ __device__ constexpr int acc_buffers(int bn) { return 2 * epi_groups(bn); }
constexpr int kRows = 128;                    // rows of a block's tile: the lanes of tensor memory
constexpr int kDepthBytes = 128;              // depth of a stage
constexpr int kTries = 1 << 22;               // bound of every wait, in tries of up to about a microsecond
constexpr int kMaxStages = 8;
constexpr int kStripBytes = 32 * 64;          // a warp's strip of 32 rows x 64 bytes on its way out; see write_strip()

// Sizes of a product.  `count`, where given, holds at run time how many rows (or, with over_depth, steps of depth) the whole matrix
// has of at most `of`; this product's begin at `base` of it, so that it has at most m (or k) and at least none.  Where nothing was left
// out, an operand marked alt is read through the second map.
struct Shape {
    int m, n, k;             // rows, columns, depth (elements)
    int splits = 1;          // of the depth
    int half = 0;            // 16-bit operands: 1 for fp16, 0 for bf16
    int tries = 0;           // bound of the waits inside a block (0 = default)
    const int* count = nullptr;
    int of = 0, base = 0;
    bool over_depth = false, alt_a = false, alt_b = false;
    int tile_rows = kRows;   // rows of a tile that count (a multiple of 8; the accumulators have 128), one block to a tile, K-major A
    bool rotate = false;     // each block (or pair) begins with another step of the depth.  For operands that are read once: blocks that all begin at the first
                             // 128 bytes of rows a power of two apart keep to a part of the memory channels (131,072 8-bit classes x 2,048 for
                             // eight rows in us: 73, 47 so).  Sums of floats are then taken in an order that depends on the tile.
    int b_depth = 0;         // MN-major B: where its depth begins over again (0: it does not), so that A may come in two halves: a stage's 64, or 32, the half of the
                             // only stage, in boxes of 32 rows
    bool a_ahead = false;    // A does not come from the kernel before this one (which let this one start early): its first stages are
                             // fetched while that one runs.  No count, one block to a tile.
};

struct Unit {
    int row, col;            // first row and column of the (pair's) tile
    int k0, k1;              // stages of depth [k0, k1)
    int split;
};

// Order of the tiles: bands of kBand row tiles, and in a band columns outside, rows inside, so that what runs at a time shares rows
// and columns in L2.
struct Walk {
    int m, tiles_m, tiles_n, stages, per_split, splits, tile_rows, tile_cols;
    static constexpr int kBand = 8;
    __device__ Walk(const Shape& s, int tile_rows_, int tile_cols_, int depth)
    {
        int mm = s.m, kk = s.k;
        if (s.count) {
            const int c = max(0, *s.count - s.base);
            if (s.over_depth) kk = min(kk, c); else mm = min(mm, c);
        }
        m = mm;
        tile_rows = tile_rows_;
        tile_cols = tile_cols_;
        tiles_m = (mm + tile_rows - 1) / tile_rows;
        tiles_n = (s.n + tile_cols - 1) / tile_cols;
        stages = (kk + depth - 1) / depth;
        splits = s.splits;
        per_split = (stages + splits - 1) / splits;
    }
    __device__ int units() const { return tiles_m * tiles_n * splits; }
    __device__ Unit at(int u) const
    {
        Unit r;
        if (tiles_n == 1 && splits == 1) {       // no divisions
            r.split = 0;
            r.col = 0;
            r.row = u * tile_rows;
            r.k0 = 0;
            r.k1 = stages;
            return r;
        }
        const int tiles = max(1, tiles_m * tiles_n);
        r.split = u / tiles;
        const int t = u - r.split * tiles, band = t / (kBand * tiles_n), in = t - band * kBand * tiles_n;
        const int rows = max(1, min(kBand, tiles_m - band * kBand));
        r.col = in / rows * tile_cols;
        r.row = (band * kBand + in % rows) * tile_rows;
        r.k0 = min(stages, r.split * per_split);
        r.k1 = min(stages, r.k0 + per_split);
        return r;
    }
};

// ---- device pieces -------------------------------------------------------------------------------------------------------

__device__ __forceinline__ uint32_t cluster_rank()
{
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;\n" : "=r"(r));
    return r;
}
__device__ __forceinline__ void cluster_meet()
{
    asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;\n" ::: "memory");
}
__device__ __forceinline__ void init_barrier(uint64_t* bar, int count)
{
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;\n" ::"r"(tc::smem_u32(bar)), "r"(count) : "memory");
}
// true once the phase is complete; false when the block gave up
__device__ __forceinline__ bool wait(uint64_t* bar, uint32_t parity, volatile int* abort, int* flag, int tries)
{
    for (int it = 0; it < tries; ++it) {
        uint32_t done;
        asm volatile("{\n.reg .pred p;\nmbarrier.try_wait.parity.acquire.cta.shared::cta.b64 p, [%1], %2;\nselp.u32 %0, 1, 0, p;\n}\n"
                     : "=r"(done) : "r"(tc::smem_u32(bar)), "r"(parity) : "memory");
        if (done) return true;
        if ((it & 15) == 15 && *abort) return false;
    }
    atomicExch(flag, 1);
    *abort = 1;
    return false;
}
template <int CTAS>
__device__ __forceinline__ void expect_bytes(uint64_t* bar, uint32_t bytes)
{
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;\n" ::"r"(tc::smem_u32(bar)), "r"(bytes) : "memory");
}
// A box of the tensor at (x, y) into shared memory; the bytes are counted at `bar` (of the cluster's first block with CTAS = 2).
template <int CTAS>
__device__ __forceinline__ void copy_box(uint32_t dst, const CUtensorMap* map, int x, int y, uint64_t* bar)
{
    if constexpr (CTAS == 2)
        asm volatile("cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];\n"
                     ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(tc::smem_u32(bar) & 0xFEFFFFFFu) : "memory");
    else
        asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];\n"
                     ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(tc::smem_u32(bar)) : "memory");
}
// Counts at `bar` (of every block of the cluster) once all products issued so far are done.
template <int CTAS>
__device__ __forceinline__ void commit(uint64_t* bar)
{
    if constexpr (CTAS == 2)
        asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;\n"
                     ::"r"(tc::smem_u32(bar)), "h"((uint16_t)3) : "memory");
    else
        asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n" ::"r"(tc::smem_u32(bar)) : "memory");
}
template <bool I8, int CTAS>
__device__ __forceinline__ void product(uint32_t acc, uint64_t a, uint64_t b, uint32_t idesc, bool add)
{
#define BIGCN_MMA(KIND, GROUP)                                                                                                       \
    asm volatile("{\n.reg .pred p;\nsetp.ne.b32 p, %4, 0;\ntcgen05.mma.cta_group::" GROUP ".kind::" KIND " [%0], %1, %2, %3, p;\n}\n" \
                 ::"r"(acc), "l"(a), "l"(b), "r"(idesc), "r"(add ? 1u : 0u) : "memory")
    if constexpr (I8 && CTAS == 1) BIGCN_MMA("i8", "1");
    else if constexpr (I8) BIGCN_MMA("i8", "2");
    else if constexpr (CTAS == 1) BIGCN_MMA("f16", "1");
    else BIGCN_MMA("f16", "2");
#undef BIGCN_MMA
}
// A named barrier of `threads` threads that tells each whether all of them were ok.
__device__ __forceinline__ bool meet(int id, int threads, bool ok)
{
    uint32_t all;
    __syncwarp();
    asm volatile("{\n.reg .pred p, q;\nsetp.ne.b32 p, %3, 0;\nbarrier.cta.red.and.aligned.pred q, %1, %2, p;\nselp.u32 %0, 1, 0, q;\n}\n"
                 : "=r"(all) : "r"(id), "r"(threads), "r"(ok ? 1u : 0u) : "memory");
    return all != 0;
}
// An arrival at the barrier of the cluster's first block, after reads of tensor memory (which tcgen05.fence orders); relaxed, since one that
// released would wait for the epilogue's stores to global memory, too.
template <int CTAS>
__device__ __forceinline__ void arrive_first(uint64_t* bar)
{
    if constexpr (CTAS == 2) {
        uint32_t remote;
        asm volatile("mapa.shared::cluster.u32 %0, %1, 0;\n" : "=r"(remote) : "r"(tc::smem_u32(bar)));
        asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];\n" ::"r"(remote) : "memory");
    } else {
        asm volatile("mbarrier.arrive.relaxed.cta.shared::cta.b64 _, [%0];\n" ::"r"(tc::smem_u32(bar)) : "memory");
    }
}

// Descriptor of a shared-memory operand with 128-byte swizzle (layout type 2, descriptor version 1).  K-major: groups of 8 rows
// x 128 bytes follow each other, `sbo` = 1024 bytes apart.  MN-major: blocks of 64 elements x 64 steps of depth, 8192 bytes apart
// (`lbo`), in which groups of 8 steps are 1024 bytes apart (`sbo`).
__device__ __forceinline__ uint64_t swizzled_desc(uint32_t addr, uint32_t lbo, uint32_t sbo)
{
    return (uint64_t)((addr & 0x3FFFFu) >> 4) | (uint64_t)(lbo >> 4) << 16 | (uint64_t)(sbo >> 4) << 32 | (uint64_t)1 << 46 | (uint64_t)2 << 61;
}

template <int BN, int CTAS>
struct Config {
    static constexpr int kBRows = BN / CTAS;                     // rows of B a block holds
    static constexpr int kABytes = kRows * kDepthBytes, kBBytes = kBRows * kDepthBytes, kStage = kABytes + kBBytes;
    static constexpr int kFit = (232448 - 1024 - 512 - kEpiWarps * kStripBytes) / kStage;
    static constexpr int kStages = kFit < kMaxStages ? kFit : kMaxStages;
    static constexpr size_t kSmem = (size_t)kStages * kStage + 1024 + kEpiWarps * kStripBytes;
};

struct Control {
    uint64_t full[kMaxStages], empty[kMaxStages], acc_full[8], acc_empty[8], drained;
    uint32_t tmem;
    int abort;
};

// 32 consecutive 32-bit columns of this thread's lane; tmem_wait32() before they are used
__device__ __forceinline__ void tmem_ld32(uint32_t taddr, uint32_t (&v)[32])
{
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"
                 "%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];\n"
                 : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]),
                   "=r"(v[8]), "=r"(v[9]), "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15]),
                   "=r"(v[16]), "=r"(v[17]), "=r"(v[18]), "=r"(v[19]), "=r"(v[20]), "=r"(v[21]), "=r"(v[22]), "=r"(v[23]),
                   "=r"(v[24]), "=r"(v[25]), "=r"(v[26]), "=r"(v[27]), "=r"(v[28]), "=r"(v[29]), "=r"(v[30]), "=r"(v[31])
                 : "r"(taddr) : "memory");
}
__device__ __forceinline__ void tmem_wait32(uint32_t (&v)[32])
{
    asm volatile("tcgen05.wait::ld.sync.aligned;\n"
                 : "+r"(v[0]), "+r"(v[1]), "+r"(v[2]), "+r"(v[3]), "+r"(v[4]), "+r"(v[5]), "+r"(v[6]), "+r"(v[7]),
                   "+r"(v[8]), "+r"(v[9]), "+r"(v[10]), "+r"(v[11]), "+r"(v[12]), "+r"(v[13]), "+r"(v[14]), "+r"(v[15]),
                   "+r"(v[16]), "+r"(v[17]), "+r"(v[18]), "+r"(v[19]), "+r"(v[20]), "+r"(v[21]), "+r"(v[22]), "+r"(v[23]),
                   "+r"(v[24]), "+r"(v[25]), "+r"(v[26]), "+r"(v[27]), "+r"(v[28]), "+r"(v[29]), "+r"(v[30]), "+r"(v[31])
                 :: "memory");
}

// one column, there when it returns
__device__ __forceinline__ uint32_t tmem_ld1(uint32_t taddr)
{
    uint32_t v;
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x1.b32 {%0}, [%1];\ntcgen05.wait::ld.sync.aligned;\n" : "=r"(v) : "r"(taddr) : "memory");
    return v;
}

// What an epilogue warp works with: warp w has lanes 32 (w & 3) .. + 31 of tensor memory (rows of the tile) and part_cols(BN) columns of it, its
// `part` of the tile's; the four warps (or fewer) that share the rows are 4 apart, the first of them at `part` 0.
struct Part {
    int row;                 // first of the warp's 32 rows
    int rows;                // rows of the whole product
    int col;                 // first column
    uint32_t acc;            // its lanes and first column
    bool empty;              // no depth: the accumulators hold nothing, the sums are 0
    int part;
    int meeting;             // barrier of the warps that share the rows
    unsigned char* strip;    // kStripBytes of shared memory
};

// Columns of a warp's part.
__host__ __device__ constexpr int part_cols(int bn) { return bn / column_parts(bn); }

// body(c, v) for every 32 columns c, c + 1, .. of the warp's, as far as there are `columns`: v is the row of this lane.  done() once all
// are read from tensor memory.
template <int BN, class Done, class Body>
__device__ __forceinline__ void each_chunk(const Part& p, int columns, const Done& done, const Body& body)
{
    const int chunks = max(0, min(part_cols(BN) / 32, (columns - p.col + 31) >> 5));
    uint32_t v[32];
    if (p.empty || chunks == 0) done();
    for (int c = 0; c < chunks; ++c) {
        __syncwarp();
        if (p.empty) {
#pragma unroll
            for (int i = 0; i < 32; ++i) v[i] = 0u;
        } else {
            tmem_ld32(p.acc + 32 * c, v);
            tmem_wait32(v);
            if (c == chunks - 1) done();
        }
        body(32 * c, v);
    }
}

// 64 bytes of each lane's row, turned through shared memory so that four lanes hold the pieces of one row: put(r, piece, 16 bytes)
// for eight rows at a time.  A lane's own 64 bytes of 32 rows would be 32 half-written pairs of sectors an instruction.  Pieces of a
// row lie in an order that depends on the row, so that eight lanes meet eight groups of banks both ways.
template <class Put>
__device__ __forceinline__ void write_strip(unsigned char* strip, const uint32_t (&w)[16], const Put& put)
{
    const int lane = threadIdx.x & 31;
    __syncwarp();
#pragma unroll
    for (int i = 0; i < 4; ++i) *reinterpret_cast<uint4*>(strip + lane * 64 + 16 * (i ^ ((lane >> 1) & 3))) = make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
    __syncwarp();
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int r = 8 * i + (lane >> 2), piece = lane & 3;
        put(r, piece, *reinterpret_cast<const uint4*>(strip + r * 64 + 16 * (piece ^ ((r >> 1) & 3))));
    }
}

// The same straight to memory, all 32 rows and 64 bytes of them there: `at` is where this lane's first piece goes (row lane >> 2, piece
// lane & 3), `step` eight rows in bytes.
__device__ __forceinline__ void write_strip_whole(unsigned char* strip, const uint32_t (&w)[16], char* at, int64_t step)
{
    write_strip(strip, w, [&](int, int, const uint4& q) {
        *reinterpret_cast<uint4*>(at) = q;
        at += step;
    });
}

// The same for rows of a 16-bit type that start anywhere: put(r, bits) for the element of this lane's number, row by row.  A short loop, which costs
// the epilogue's other forms less, too (bf16, 3,269 x 64 times 34,619 and 34,624 classes in us: 137 and 106 with eight rows a turn, 119 and 84 with two).
template <class Put>
__device__ __forceinline__ void write_strip_elements(unsigned char* strip, const uint32_t (&w)[16], const Put& put)
{
    const int lane = threadIdx.x & 31;
    __syncwarp();
#pragma unroll
    for (int i = 0; i < 4; ++i) *reinterpret_cast<uint4*>(strip + lane * 64 + 16 * (i ^ ((lane >> 1) & 3))) = make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
    __syncwarp();
#pragma unroll 2
    for (int r = 0; r < 32; ++r) put(r, *reinterpret_cast<const uint16_t*>(strip + r * 64 + 16 * ((lane >> 3) ^ ((r >> 1) & 3)) + 2 * (lane & 7)));
}

// The same for 32 words (128 bytes) of each lane's row, the rows of half a warp at a time, so that eight lanes hold a row's 128 bytes: what a store costs
// beyond the multiprocessor is the 128-byte lines that it touches and the sectors that it leaves half-written, fewer of both for rows in whole (3,269 x 64
// times 34,619, 34,620 and 34,624 classes, rows from 4-, 16- and 32-byte boundaries, in us: 284, 196, 131 by 64 bytes, 197, 151, 113 so).
template <class Put>
__device__ __forceinline__ void write_wide(unsigned char* strip, const uint32_t (&v)[32], const Put& put)
{
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        __syncwarp();
        if ((lane >> 4) == h) {
#pragma unroll
            for (int i = 0; i < 8; ++i) *reinterpret_cast<uint4*>(strip + (lane & 15) * 128 + 16 * (i ^ (lane & 7))) = make_uint4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
        }
        __syncwarp();
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int r = 4 * i + (lane >> 3), piece = lane & 7;
            put(16 * h + r, piece, *reinterpret_cast<const uint4*>(strip + r * 128 + 16 * (piece ^ (r & 7))));
        }
    }
}
// For rows that start anywhere: put(r, bits) for the word of this lane's number, row by row.
template <class Put>
__device__ __forceinline__ void write_wide_elements(unsigned char* strip, const uint32_t (&v)[32], const Put& put)
{
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        __syncwarp();
        if ((lane >> 4) == h) {
#pragma unroll
            for (int i = 0; i < 8; ++i) *reinterpret_cast<uint4*>(strip + (lane & 15) * 128 + 16 * (i ^ (lane & 7))) = make_uint4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
        }
        __syncwarp();
#pragma unroll 4
        for (int r = 0; r < 16; ++r) put(16 * h + r, *reinterpret_cast<const uint32_t*>(strip + r * 128 + 16 * ((lane >> 2) ^ (r & 7)) + 4 * (lane & 3)));
    }
}

// Epi: struct with
//   Args
//   Row                            what it reads of a row (of the tile, a lane's)
//   static __device__ Row row(const Args&, int row, int rows)                    fetched while the tile before is worked on
//   template <int BN, class Done> static __device__ void tile(const Args&, const Shape&, const Unit&, const Part&, const Row&, const Done& done)
//                                  run by the epilogue warps; done() once, when the accumulators are read
//   static __device__ int* flag()  raised when a wait ran out
//   static constexpr bool kMeets   whether the warps of the same rows meet in tile()
template <bool I8, int BN, int CTAS, bool A_MN, bool B_MN, class Epi>
__global__ void __launch_bounds__(kThreads, 1)
product_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b, const __grid_constant__ CUtensorMap map_alt,
               const __grid_constant__ Shape shape, const __grid_constant__ typename Epi::Args args)
{
    using C = Config<BN, CTAS>;
    constexpr int kDepth = I8 ? 128 : 64;
    extern __shared__ unsigned char raw[];
    __shared__ Control ctl;
    unsigned char* stages = raw + ((1024u - (tc::smem_u32(raw) & 1023u)) & 1023u);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = CTAS == 2 ? cluster_rank() : 0u;
    constexpr int kGroups = epi_groups(BN), kBuffers = acc_buffers(BN), kCols = kBuffers * BN;

    if (threadIdx.x == 0) {
        for (int i = 0; i < C::kStages; ++i) {
            init_barrier(&ctl.full[i], 1);
            init_barrier(&ctl.empty[i], 1);
        }
        for (int i = 0; i < kBuffers; ++i) {
            init_barrier(&ctl.acc_full[i], 1);
            init_barrier(&ctl.acc_empty[i], kEpiWarps / kGroups * CTAS);
        }
        init_barrier(&ctl.drained, 1);
        ctl.abort = 0;
        asm volatile("fence.mbarrier_init.release.cluster;\n" ::: "memory");
    }
    if (warp == kIssuer) {
        if constexpr (CTAS == 2) {
            asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;\n" ::"r"(tc::smem_u32(&ctl.tmem)), "r"(kCols) : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;\n" ::: "memory");
        } else {
            tc::tmem_alloc(&ctl.tmem, kCols);
        }
    }
    tc::fence_before_sync();
    __syncthreads();
    if constexpr (CTAS == 2) cluster_meet();
    tc::fence_after_sync();
    const uint32_t tmem = ctl.tmem;
    volatile int* abort = &ctl.abort;
    int* const flag = Epi::flag();
    const int tries = shape.tries > 0 ? shape.tries : kTries;

    int early = 0;           // stages whose A is on its way
    const auto depth_at = [&](const Unit& t, int k) {        // of the stage k in [k0, k1)
        if (!shape.rotate) return k;
        const int steps = t.k1 - t.k0, at = k - t.k0 + (int)(blockIdx.x / CTAS % (unsigned)steps);
        return t.k0 + (at < steps ? at : at - steps);
    };
    if (CTAS == 1 && !A_MN && shape.a_ahead && threadIdx.x == kProducer * 32) {
        const Walk walk(shape, shape.tile_rows, BN, kDepth);
        if ((int)blockIdx.x < walk.units()) {
            const Unit t = walk.at(blockIdx.x);
            early = min(t.k1 - t.k0, C::kStages);
            for (int i = 0; i < early; ++i) {
                expect_bytes<CTAS>(&ctl.full[i], shape.tile_rows * kDepthBytes + C::kBBytes);
                copy_box<CTAS>(tc::smem_u32(stages + i * C::kStage), &map_a, depth_at(t, t.k0 + i) * kDepth, t.row, &ctl.full[i]);
            }
        }
    }
    pdl_enter();
    const Walk walk(shape, CTAS == 1 && !A_MN ? shape.tile_rows : kRows * CTAS, BN, kDepth);
    const uint32_t stage_bytes = (CTAS == 1 && !A_MN ? shape.tile_rows * kDepthBytes : C::kABytes) + C::kBBytes;
    const int units = walk.units(), first = blockIdx.x / CTAS, step = gridDim.x / CTAS;

    if (warp == kProducer) {
        if (lane == 0) {
            const bool whole = shape.count && *shape.count >= shape.of;
            const CUtensorMap* ma = whole && shape.alt_a ? &map_alt : &map_a;
            const CUtensorMap* mb = whole && shape.alt_b ? &map_alt : &map_b;
            int slot = 0;
            uint32_t phase = 0;
            bool ok = true;
            int64_t issued = 0;
            for (int u = first; u < units && ok; u += step) {
                const Unit t = walk.at(u);
                const int arow = t.row + (int)rank * kRows, brow = t.col + (int)rank * C::kBRows;
                for (int k = t.k0; k < t.k1; ++k) {
                    ok = wait(&ctl.empty[slot], phase ^ 1u, abort, flag, tries);
                    if (!ok) break;
                    const int at = depth_at(t, k) * kDepth;
                    const bool fetched = issued < early;
                    if (rank == 0 && !fetched) expect_bytes<CTAS>(&ctl.full[slot], stage_bytes * CTAS);
                    const uint32_t sa = tc::smem_u32(stages + slot * C::kStage), sb = sa + C::kABytes;
                    if (fetched) {
                    } else if constexpr (A_MN) {
#pragma unroll
                        for (int i = 0; i < kRows / 64; ++i) copy_box<CTAS>(sa + i * 8192, ma, arow + 64 * i, at, &ctl.full[slot]);
                    } else {
                        copy_box<CTAS>(sa, ma, at, arow, &ctl.full[slot]);
                    }
                    if constexpr (B_MN) {
                        const int at_b = shape.b_depth > 0 && at >= shape.b_depth ? at - shape.b_depth : at;
#pragma unroll
                        for (int i = 0; i < C::kBRows / 64; ++i) copy_box<CTAS>(sb + i * 8192, mb, brow + 64 * i, at_b, &ctl.full[slot]);
                        if (shape.b_depth == 32)
#pragma unroll
                            for (int i = 0; i < C::kBRows / 64; ++i) copy_box<CTAS>(sb + i * 8192 + 4096, mb, brow + 64 * i, at_b, &ctl.full[slot]);
                    } else {
                        copy_box<CTAS>(sb, mb, at, brow, &ctl.full[slot]);
                    }
                    ++issued;
                    if (++slot == C::kStages) slot = 0, phase ^= 1u;
                }
            }
            // every stage handed back: nothing of the cluster touches this block's barriers or stages any more
            for (int i = 0; i < C::kStages && ok; ++i) {
                ok = wait(&ctl.empty[slot], phase ^ 1u, abort, flag, tries);
                if (++slot == C::kStages) slot = 0, phase ^= 1u;
            }
            if (!ok) {
                // gave up: the copies that were issued have to land first.  A pair's are counted at one block's barriers, which the other block may
                // have left short, so time (a thousand times what a copy takes) stands in for them
                volatile int none = 0;
                if (CTAS == 1)
                    for (int64_t j = issued > C::kStages ? issued - C::kStages : 0; j < issued; ++j)
                        wait(&ctl.full[j % C::kStages], (uint32_t)(j / C::kStages) & 1u, &none, flag, kTries);
                for (int i = 0; i < 10; ++i) __nanosleep(1000000);
            }
        }
        __syncwarp();
    } else if (warp == kIssuer) {
        if (lane == 0 && rank == 0) {
            const uint32_t fmt = I8 || !shape.half ? 1u : 0u;
            const uint32_t idesc = (I8 ? 2u : 1u) << 4 | fmt << 7 | fmt << 10 | (A_MN ? 1u : 0u) << 15 | (B_MN ? 1u : 0u) << 16 |
                                       (uint32_t)(BN >> 3) << 17 | (uint32_t)((kRows * CTAS) >> 4) << 24;
            constexpr uint32_t step_a = A_MN ? 2048 >> 4 : 32 >> 4, step_b = B_MN ? 2048 >> 4 : 32 >> 4;
            int slot = 0, buf = 0;
            uint32_t phase = 0, acc_phase = 0;
            bool ok = true, any = false;
            for (int u = first; u < units && ok; u += step) {
                const Unit t = walk.at(u);
                ok = wait(&ctl.acc_empty[buf], acc_phase ^ 1u, abort, flag, tries);
                if (!ok) break;
                tc::fence_after_sync();
                const uint32_t acc = tmem + (uint32_t)(buf * BN);
                for (int k = t.k0; k < t.k1; ++k) {
                    ok = wait(&ctl.full[slot], phase, abort, flag, tries);
                    if (!ok) break;
                    tc::fence_after_sync();
                    const uint32_t sa = tc::smem_u32(stages + slot * C::kStage), sb = sa + C::kABytes;
                    const uint64_t da = A_MN ? swizzled_desc(sa, 8192, 1024) : swizzled_desc(sa, 16, 1024);
                    const uint64_t db = B_MN ? swizzled_desc(sb, 8192, 1024) : swizzled_desc(sb, 16, 1024);
#pragma unroll
                    for (int i = 0; i < 4; ++i) product<I8, CTAS>(acc, da + i * step_a, db + i * step_b, idesc, k > t.k0 || i > 0);
                    any = true;
                    commit<CTAS>(&ctl.empty[slot]);
                    if (++slot == C::kStages) slot = 0, phase ^= 1u;
                }
                if (!ok) break;
                commit<CTAS>(&ctl.acc_full[buf]);        // (at once where there is no depth)
                if (++buf == kBuffers) buf = 0, acc_phase ^= 1u;
            }
            if (any) {
                // all products done, whether or not an epilogue warp (which may have given up) waits for the last of them
                volatile int none = 0;
                if constexpr (CTAS == 2)
                    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.b64 [%0];\n" ::"r"(tc::smem_u32(&ctl.drained)) : "memory");
                else
                    commit<1>(&ctl.drained);
                wait(&ctl.drained, 0, &none, flag, kTries);
            }
        }
        __syncwarp();
    } else {
        constexpr int kParts = column_parts(BN);
        const int group = (warp >> 2) / kParts, begin = first + group * step, stride = kGroups * step;
        const int own = (int)rank * kRows + (warp & 3) * 32;
        Part part;
        part.rows = walk.m;
        part.part = (warp >> 2) % kParts;
        part.meeting = 1 + group * 4 + (warp & 3);
        part.strip = stages + C::kStages * C::kStage + warp * kStripBytes;
        int buf = group;
        uint32_t acc_phase = 0;
        Unit coming = walk.at(begin < units ? begin : 0);
        typename Epi::Row ahead = Epi::row(args, begin < units ? coming.row + own + lane : walk.m, walk.m);
        for (int u = begin; u < units; u += stride) {
            const Unit t = coming;
            const typename Epi::Row now = ahead;
            if (u + stride < units) {
                coming = walk.at(u + stride);
                ahead = Epi::row(args, coming.row + own + lane, walk.m);
            }
            // where an epilogue lets the warps of the same rows meet, they go on or give up together
            const bool there = __all_sync(0xffffffffu, wait(&ctl.acc_full[buf], acc_phase, abort, flag, tries));
            if constexpr (Epi::kMeets && kParts > 1) {
                if (!meet(part.meeting, 32 * kParts, there)) break;
            } else {
                if (!there) break;
            }
            tc::fence_after_sync();
            part.row = t.row + own;
            if (CTAS == 1) part.rows = min(walk.m, t.row + walk.tile_rows);
            part.col = t.col + part.part * part_cols(BN);
            part.acc = tmem + (uint32_t)(buf * BN + part.part * part_cols(BN)) + ((uint32_t)((warp & 3) * 32) << 16);
            part.empty = t.k0 >= t.k1;
            Epi::template tile<BN>(args, shape, t, part, now, [&] {
                tc::fence_before_sync();
                __syncwarp();
                if (lane == 0) arrive_first<CTAS>(&ctl.acc_empty[buf]);
            });
            if ((buf += kGroups) >= kBuffers) buf -= kBuffers, acc_phase ^= 1u;
        }
    }
    tc::fence_before_sync();
    __syncthreads();
    if constexpr (CTAS == 2) cluster_meet();
    if (warp == kIssuer) {
        tc::fence_after_sync();
        if constexpr (CTAS == 2) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;\n" ::"r"(tmem), "r"(kCols) : "memory");
        else tc::tmem_free(tmem, kCols);
    }
}

// ---- host pieces ---------------------------------------------------------------------------------------------------------

// Rows that a tile reads: of few rows no more than there are, since rows past the tensor's end cost their bytes between L2 and shared memory, too.
inline int rows_of_one_tile(int64_t rows) { return rows >= kRows ? kRows : (int)round_up(rows, 8); }

// Tensor map of a row-major matrix (rows x cols elements of `elt` bytes, `pitch` bytes from row to row; base and pitch on 16-byte
// boundaries), read in swizzled boxes of box_cols x box_rows.
cudaError_t encode_map(CUtensorMap* map, const void* base, int elt, bool integers, int64_t rows, int64_t cols, int64_t pitch, int box_cols, int box_rows);

template <bool I8, int BN, int CTAS, bool A_MN, bool B_MN, class Epi>
cudaError_t launch(cudaStream_t s, const CUtensorMap& a, const CUtensorMap& b, const CUtensorMap& alt, const Shape& shape, const typename Epi::Args& args)
{
    using C = Config<BN, CTAS>;
    auto* kernel = product_kernel<I8, BN, CTAS, A_MN, B_MN, Epi>;
    static std::atomic<uint64_t> ready{0};     // by device
    const cudaError_t e = allow_shared(kernel, C::kSmem, &ready);
    if (e != cudaSuccess) return e;
    const int64_t units = ceil_div(shape.m, CTAS == 1 && !A_MN ? shape.tile_rows : kRows * CTAS) * ceil_div(shape.n, BN) * shape.splits;
    const int clusters = (int)std::max<int64_t>(1, std::min<int64_t>(units, sm_count() / CTAS));
    cudaLaunchAttribute attr[2] = {};
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = CTAS;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(clusters * CTAS));
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = C::kSmem;
    cfg.stream = s;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, kernel, a, b, alt, shape, args);
}

}  // namespace gemm
}  // namespace bigcn
