// Softmax cross entropy of rows against a class matrix, without storing the logits, and its gradients.
//
//   z_ik = sum_j x_ij w_kj,  lse_i = log sum_k exp z_ik,  loss_i = lse_i - z_i,label(i)
//   G_ik = (exp(z_ik - lse_i) - [k = label(i)]) g_i,  g_x = G W,  g_w = G^T X            (g_i = the gradient of loss_i)
//
// All four products run on the tensor cores (dense_gemm.cuh).  The first leaves, for every row and tile of columns, the
// maximum and the sum of exp(z - maximum); a second kernel joins them.  The backward pass computes z once more, a piece of rows and classes at a time
// (kPieceBytes of G), turns it into G in its epilogue, and multiplies that piece into g_x and g_w; sums over pieces, and over
// parts of a long depth, are kept in fp32 in the workspace and added in a fixed order.  G is rounded to the operands' type, the one
// rounding besides the outputs' own: a relative error of half a step for each term of sums whose terms' errors are independent,
// which is the size of the output's rounding.  Up to 64 classes there is no such error: G is the sum of two numbers of the type, a high half and behind it a
// low one.  Tiles of G's columns are 128 wide in g_w whether or not they hold the low half, and the depth of g_x is one stage, or two from 33 classes on,
// whose class rows are fetched twice: what it costs are G's bytes, twice as many from 33 classes on (see low_half()).  In bf16 g_i is part of G.  fp16 has no exponents for a g_i of, say, 1 / n times a small
// probability, so there G holds (exp(z - lse) - [..]) 2^14 (down to 2^-28 in normal numbers), rows of g_x are multiplied by g_i 2^-14 in fp32, and X enters
// g_w as rows times g_i / max |g| (one more rounding, none where all g_i are the same), the rest in fp32.  Nor has fp16 the exponents for a g_i far below
// the largest: such a row of X goes up by a power of two 2^b and its row of G down by it, see lift_of().
//
// Rows without a label take no part: the labelled ones are listed first and, unless that is all of them, copied together, so that what
// the others hold (NaN, infinities) reaches nothing and their work is not done.  How many there are is known on the GPU only; the
// kernels read it there.
//
// Against 64 bits (2-norm, bf16): 0.0019 for the gradients of many classes, where rounding the exact ones once leaves 0.0016 (as for up to 64).
// lse and loss 3e-7: the tensor cores' sums, each cut at its step, and ex2.approx.
#include <algorithm>
#include <climits>

#include "dense_gemm.cuh"
#include "dense_types.cuh"

namespace bigcn {

namespace {

using namespace dense;

__device__ int g_loss_timeout;                // set when a wait ran out

constexpr float kLog2e = 1.4426950408889634f;
constexpr int kScan = 4096;                   // labels of a block of the listing: 1024 threads, four each

__device__ __forceinline__ float exp2_fast(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;\n" : "=f"(y) : "f"(x));
    return y;
}

// ---- the labelled rows ---------------------------------------------------------------------------------------------------

// Four consecutive labels of a thread: which are classes.
__device__ __forceinline__ void read_labels(const int64_t* labels, int64_t n, int classes, int64_t at, int64_t (&v)[4], bool (&in)[4])
{
    if (at + 4 <= n && (reinterpret_cast<uintptr_t>(labels) & 15) == 0) {
        const longlong2 a = __ldg(reinterpret_cast<const longlong2*>(labels + at)), b = __ldg(reinterpret_cast<const longlong2*>(labels + at) + 1);
        v[0] = a.x; v[1] = a.y; v[2] = b.x; v[3] = b.y;
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = at + i < n ? __ldg(labels + at + i) : -1;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) in[i] = v[i] >= 0 && v[i] < classes;
}
__device__ __forceinline__ int block_sum(int v, int* slot)
{
    v = __reduce_add_sync(0xffffffffu, v);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) slot[threadIdx.x >> 5] = v;
    __syncthreads();
    return __reduce_add_sync(0xffffffffu, (threadIdx.x & 31) < (blockDim.x >> 5) ? slot[threadIdx.x & 31] : 0);
}
__global__ void __launch_bounds__(1024) count_labels_kernel(const int64_t* __restrict__ labels, int64_t n, int classes, int* __restrict__ counts)
{
    pdl_enter();
    __shared__ int slot[32];
    int64_t v[4];
    bool in[4];
    read_labels(labels, n, classes, ((int64_t)blockIdx.x * 1024 + threadIdx.x) * 4, v, in);
    const int c = block_sum(in[0] + in[1] + in[2] + in[3], slot);
    if (threadIdx.x == 0) counts[blockIdx.x] = c;
}

struct ListArgs {
    const int64_t* labels;
    int64_t n;
    int classes;
    const int* counts;       // of the blocks (more than one)
    int* kept;               // [n] the labelled rows, ascending
    int* label;              // [n] their classes
    int* place;              // [n] of every row: where it is in `kept`, or -1
    int* count;              // how many
    float* loss;             // nullable: 0 (NaN for a label that is no class) for the others
    float* lse;
    bool words;              // both on 16-byte boundaries
    const float* of_lse;     // nullable: two values of every row,
    const float* of_g_loss;
    float* to_lse;           // [n] those of the labelled ones
    float* to_g_loss;
    unsigned* top;           // nullable: the largest magnitude of g_loss among them, as bits (0 before)
};
struct GatherArgs {
    const uint16_t* x;
    int64_t ldx, n;
    int d;
    bool whole;              // rows of x on 16-byte boundaries: where all are labelled they are read where they are
    const int* place;
    const int* count;
    uint16_t* to;            // [n rounded up to 128] rows of ldt (a multiple of 8)
    int64_t ldt;
    uint16_t* g_x;           // nullable: rows without a label become zero
    int64_t ldgx;
    bool g_whole;
    int span;                // rows of a warp at a time, at most 32
    const float* g_loss;     // fp16's gradients (else null): of every row,
    const float* top;        // and the largest magnitude among the labelled ones;
    float* lift;             // of the labelled rows: what G is multiplied by, kHalfScale 2^-b
    float* undo;             // g divided by it
    uint16_t* scaled;        // rows times g / top 2^b, as `to` lies (nullable: g_w is not wanted)
};
constexpr float kHalfScale = 16384.f;         // fp16's G is this much larger

// The power b of a row whose g is `ratio` of the largest: X enters g_w as x ratio 2^b and G as G 2^(14 - b).  Of fp16's 14 exponents below 1 in
// normal numbers rows of X give up five (x ratio 2^b stays within [2^-6, 2^-5) of x where x ratio would lie below), the others are left for small
// values of x; G, whose largest is 2^14 without b, gives up 18 at most, which leaves it 10.  So a ratio of 2^-30 still has x near 1 in normal
// numbers; without b they ended at 2^-14, and from 2^-25 on nothing of such a row was left.
__device__ __forceinline__ int lift_of(float ratio)
{
    const int exponent = (int)(__float_as_uint(ratio) >> 23 & 255u) - 127;       // (128 of infinities and NaN)
    return min(18, max(0, -6 - exponent));
}
__device__ __forceinline__ float power_of_two(int e) { return __int_as_float((127 + e) << 23); }
// How rows of x lie: on 16-byte boundaries, up to 32 words of 16 bytes or more; on 4-byte boundaries; anywhere.
enum Lie : int { kShort = 0, kLong = 1, kPairs = 2, kAnywhere = 3 };
template <int LIE>
__device__ __forceinline__ void gather_rows(const GatherArgs& a, int count, const int* places, int64_t first, int64_t warps, float top);

// kGather: at most kScan rows, whose listing every block does for itself (the first one writes it) before it gathers its share: one launch less.
template <bool kGather, int LIE>
__global__ void __launch_bounds__(1024) list_labels_kernel(const ListArgs a, const GatherArgs gather)
{
    pdl_enter();
    __shared__ int slot[32];
    __shared__ int here[kGather ? kScan : 1];
    __shared__ int total;
    const int block = kGather ? 0 : blockIdx.x;
    const bool write = !kGather || blockIdx.x == 0;
    const int64_t at = ((int64_t)block * 1024 + threadIdx.x) * 4;
    int64_t v[4];
    bool in[4];
    read_labels(a.labels, a.n, a.classes, at, v, in);         // (on their way while the blocks before are summed)
    int before = 0;
    for (int b = threadIdx.x; b < block; b += 1024) before += __ldg(a.counts + b);
    before = !kGather && gridDim.x > 1 ? block_sum(before, slot) : 0;
    const int mine = in[0] + in[1] + in[2] + in[3], lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int upto = mine;
#pragma unroll
    for (int m = 1; m < 32; m <<= 1) {
        const int o = __shfl_up_sync(0xffffffffu, upto, m);
        if (lane >= m) upto += o;
    }
    __syncthreads();
    if (lane == 31) slot[warp] = upto;
    __syncthreads();
    const int base = before + __reduce_add_sync(0xffffffffu, lane < warp ? slot[lane] : 0);
    int next = base + upto - mine, places[4];
    float none[4];
    unsigned top = 0u;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (a.top && in[i]) top = max(top, __float_as_uint(__ldg(a.of_g_loss + at + i)) & 0x7fffffffu);
        places[i] = in[i] ? next : -1;
        none[i] = v[i] < 0 ? 0.f : __uint_as_float(0x7fc00000u);
        if (in[i]) {
            if (write) {
                a.kept[next] = (int)(at + i);
                a.label[next] = (int)v[i];
                if (a.of_lse) {
                    a.to_lse[next] = __ldg(a.of_lse + at + i);
                    a.to_g_loss[next] = __ldg(a.of_g_loss + at + i);
                }
            }
            ++next;
        }
    }
    if constexpr (kGather) {
#pragma unroll
        for (int i = 0; i < 4; ++i) here[4 * threadIdx.x + i] = places[i];
    } else if (at + 4 <= a.n) {
        *reinterpret_cast<int4*>(a.place + at) = make_int4(places[0], places[1], places[2], places[3]);
    } else {
        for (int i = 0; i < 4 && at + i < a.n; ++i) a.place[at + i] = places[i];
    }
    if (write && a.loss && mine < 4) {
        if (mine == 0 && at + 4 <= a.n && a.words) {
            *reinterpret_cast<float4*>(a.loss + at) = make_float4(none[0], none[1], none[2], none[3]);
            *reinterpret_cast<float4*>(a.lse + at) = make_float4(none[0], none[1], none[2], none[3]);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (!in[i] && at + i < a.n) a.loss[at + i] = a.lse[at + i] = none[i];
        }
    }
    if (threadIdx.x == 1023) {
        total = base + upto;
        if (write && block == (kGather ? 0 : (int)gridDim.x - 1)) *a.count = base + upto;
    }
    if (a.top) {                              // (magnitudes and NaN order as bits; the largest does not depend on the order of the blocks)
        top = __reduce_max_sync(0xffffffffu, top);
        __syncthreads();
        if (lane == 0) slot[warp] = (int)top;
        __syncthreads();
        top = __reduce_max_sync(0xffffffffu, (unsigned)slot[lane]);
        if (threadIdx.x == 0 && write) atomicMax(a.top, top);
    }
    if constexpr (kGather) {
        __syncthreads();
        gather_rows<LIE>(gather, total, here, (int64_t)blockIdx.x * 32 + warp, (int64_t)gridDim.x * 32, __uint_as_float(top));
    }
}

// The next ROWS of the labelled rows that `left` names, copied by words of T, WORDS of them a lane at a time, all on their way before the first
// is stored; what is left of a row after `words` of them one by one.
template <int ROWS, int WORDS, class T, class Load>
__device__ __forceinline__ void copy_rows(const GatherArgs& a, int64_t row0, int place, uint32_t& left, int words, const Load& load)
{
    const int lane = threadIdx.x & 31;
    constexpr int kElts = sizeof(T) / 2;
    const uint16_t* from[ROWS];
    uint16_t* to[ROWS];
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
        const int at = __ffs(left) - 1;
        from[r] = left != 0u ? a.x + (row0 + at) * a.ldx : nullptr;
        to[r] = left != 0u ? a.to + (int64_t)__shfl_sync(0xffffffffu, place, at) * a.ldt : nullptr;
        left &= left - 1;
    }
    for (int base = lane; base < words; base += 32 * WORDS) {
        T v[ROWS][WORDS];
#pragma unroll
        for (int r = 0; r < ROWS; ++r)
#pragma unroll
            for (int j = 0; j < WORDS; ++j)
                if (from[r] && base + 32 * j < words) v[r][j] = load(from[r], base + 32 * j);
#pragma unroll
        for (int r = 0; r < ROWS; ++r)
#pragma unroll
            for (int j = 0; j < WORDS; ++j)
                if (from[r] && base + 32 * j < words) reinterpret_cast<T*>(to[r])[base + 32 * j] = v[r][j];
    }
#pragma unroll
    for (int r = 0; r < ROWS; ++r)
        if (from[r] && lane < a.d - words * kElts) to[r][words * kElts + lane] = __ldg(from[r] + words * kElts + lane);
}

// A warp to `span` rows at a time, whose places its lanes read together: labelled rows are copied together, the gradient of the others is
// zero; rows up to the next multiple of 128 are zero.
template <int LIE>
__device__ void gather_rows(const GatherArgs& a, int count, const int* places, int64_t first, int64_t warps, float top)
{
    const int lane = threadIdx.x & 31;
    const int64_t end = ((int64_t)count + 127) / 128 * 128;
    if (a.lift) {
        for (int64_t row = first; row < a.n; row += warps) {
            const int p = places[row];
            if (p < 0) continue;
            const float g = __ldg(a.g_loss + row), ratio = top > 0.f ? g / top : 0.f;
            const int b = lift_of(ratio);
            if (lane == 0) {
                a.lift[p] = power_of_two(14 - b);                 // kHalfScale 2^-b
                a.undo[p] = g * power_of_two(b - 14);
            }
            if (!a.scaled) continue;
            const float factor = ratio * power_of_two(b);
            for (int i = lane; i < a.d; i += 32)
                a.scaled[(int64_t)p * a.ldt + i] = __half_as_ushort(__float2half_rn(__half2float(__ushort_as_half(__ldg(a.x + row * a.ldx + i))) * factor));
        }
        for (int64_t row = count + first; a.scaled && row < end; row += warps)
            for (int i = lane; i < a.d; i += 32) a.scaled[row * a.ldt + i] = 0;
    }
    if (a.whole && count == a.n) return;
    const int words = a.d / 8;
    for (int64_t row0 = first * a.span; row0 < a.n; row0 += warps * a.span) {
        const int rows = (int)min((int64_t)a.span, a.n - row0);
        const int place = lane < rows ? places[row0 + lane] : -1;
        const uint32_t kept = __ballot_sync(0xffffffffu, place >= 0);
        uint32_t left = kept;
        if constexpr (LIE == kShort) {                        // rows of one word a lane
            while (left != 0u) copy_rows<2, 1, uint4>(a, row0, place, left, words, [&](const uint16_t* from, int i) { return __ldg(reinterpret_cast<const uint4*>(from) + i); });
        } else if constexpr (LIE == kLong) {
            while (left != 0u) copy_rows<1, 4, uint4>(a, row0, place, left, words, [&](const uint16_t* from, int i) { return __ldg(reinterpret_cast<const uint4*>(from) + i); });
        } else if constexpr (LIE == kPairs) {
            while (left != 0u) copy_rows<2, 4, uint32_t>(a, row0, place, left, a.d / 2, [&](const uint16_t* from, int i) { return __ldg(reinterpret_cast<const uint32_t*>(from) + i); });
        } else {
            // rows that begin anywhere, as words of the destination out of the two aligned ones that hold them; a row with others around it may be
            // read two bytes past either end
            while (left != 0u) copy_rows<2, 4, uint32_t>(a, row0, place, left, a.d / 2, [&](const uint16_t* from, int i) {
                if (from == a.x || from == a.x + (a.n - 1) * a.ldx) return (uint32_t)__ldg(from + 2 * i) | (uint32_t)__ldg(from + 2 * i + 1) << 16;
                const uint32_t* word = reinterpret_cast<const uint32_t*>(reinterpret_cast<uintptr_t>(from) & ~uintptr_t(3)) + i;
                return reinterpret_cast<uintptr_t>(from) & 2 ? __funnelshift_r(__ldg(word), __ldg(word + 1), 16) : __ldg(word);
            });
        }
        if (!a.g_x) continue;
        for (left = ~kept & (rows < 32 ? (1u << rows) - 1u : 0xffffffffu); left != 0u; left &= left - 1) {
            uint16_t* to = a.g_x + (row0 + __ffs(left) - 1) * a.ldgx;
            if (a.g_whole) {
                for (int w = lane; w < words; w += 32) reinterpret_cast<uint4*>(to)[w] = make_uint4(0u, 0u, 0u, 0u);
                if (lane < a.d - 8 * words) to[8 * words + lane] = 0;
            } else {
                for (int i = lane; i < a.d; i += 32) to[i] = 0;
            }
        }
    }
    for (int64_t row = count + first; row < end; row += warps)
        for (int i = lane; i < a.d; i += 32) a.to[row * a.ldt + i] = 0;
}
template <int LIE>
__global__ void __launch_bounds__(256, LIE == kShort ? 8 : 6) gather_rows_kernel(const GatherArgs a)
{
    pdl_enter();
    gather_rows<LIE>(a, __ldg(a.count), a.place, (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5), (int64_t)gridDim.x * 8, a.lift ? __ldg(a.top) : 0.f);
}

// Rows copied to 16-byte boundaries (a class matrix that does not start its rows there), in words of T where the rows allow it.
template <class T>
__global__ void __launch_bounds__(256) align_rows_kernel(const uint16_t* __restrict__ w, int64_t ldw, int64_t n, int d, uint16_t* __restrict__ to, int64_t ldt)
{
    pdl_enter();
    constexpr int kElts = sizeof(T) / 2;
    const int lane = threadIdx.x & 31, words = d / kElts;
    for (int64_t row = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5); row < n; row += (int64_t)gridDim.x * 8) {
        const T* from = reinterpret_cast<const T*>(w + row * ldw);
        T* out = reinterpret_cast<T*>(to + row * ldt);
#pragma unroll 4
        for (int i = lane; i < words; i += 32) out[i] = __ldg(from + i);
        for (int i = words * kElts + lane; i < d; i += 32) to[row * ldt + i] = __ldg(w + row * ldw + i);
    }
}

// ---- epilogues -----------------------------------------------------------------------------------------------------------

// Maximum and sum of exp(z - maximum) of a tile's columns, and the label's z.  An argument of exp2 is the difference times
// log2 e: the difference first, so that the largest term is exactly 1 and a loss near 0 keeps its digits.  The warps that share the rows
// join theirs in shared memory (they meet twice a tile), which leaves a quarter of the parts to write and to join.
struct SumExp {
    struct Args {
        const int* label;    // of the rows
        float2* part;        // [column tiles][rows]
        int64_t rows;
        float* at;           // [rows] the label's z
        const int* kept;     // one tile holds all columns: straight to the results (null otherwise)
        float* loss;
        float* lse;
    };
    static constexpr bool kMeets = true;
    static __device__ int* flag() { return &g_loss_timeout; }
    struct Row {
        int label, to;
    };
    static __device__ __forceinline__ Row row(const Args& a, int row, int rows)
    {
        return {row < rows ? __ldg(a.label + row) : INT_MIN, row < rows && a.kept ? __ldg(a.kept + row) : 0};
    }
    template <int BN, class Done>
    static __device__ __forceinline__ void tile(const Args& a, const gemm::Shape& sh, const gemm::Unit& u, const gemm::Part& p, const Row& of_row, const Done& done)
    {
        const int row = p.row + (threadIdx.x & 31);
        const int label = of_row.label >= p.col ? of_row.label - p.col : INT_MIN;          // far from any column, as the rows that are not there have it
        float m = -INFINITY, s = 0.f, at = 0.f;
        bool mine = false;
        gemm::each_chunk<BN>(p, sh.n, done, [&](int c, uint32_t (&v)[32]) {
            const int left = sh.n - (p.col + c);
            if (left < 32) {
#pragma unroll
                for (int i = 0; i < 32; ++i)
                    if (i >= left) v[i] = 0xff800000u;
            }
            float tops[4] = {m, __uint_as_float(v[0]), __uint_as_float(v[1]), __uint_as_float(v[2])};
#pragma unroll
            for (int i = 3; i < 32; ++i) tops[i & 3] = fmaxf(tops[i & 3], __uint_as_float(v[i]));
            const float top = fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3])), t = top == -INFINITY ? 0.f : top;
            float s4[4] = {s * exp2_fast((m - t) * kLog2e), 0.f, 0.f, 0.f};
#pragma unroll
            for (int i = 0; i < 32; ++i) s4[i & 3] += exp2_fast((__uint_as_float(v[i]) - t) * kLog2e);
            s = (s4[0] + s4[1]) + (s4[2] + s4[3]);
            m = top;
            const unsigned in = (unsigned)label - (unsigned)c;
            if (__any_sync(0xffffffffu, in < 32u)) {
#pragma unroll
                for (int i = 0; i < 32; ++i)
                    if (in == (unsigned)i) at = __uint_as_float(v[i]);
                mine |= in < 32u;
            }
        });
        // each warp's strip holds its own 32 pairs; those of the others that share the rows lie kStripBytes * 4 apart
        constexpr int kParts = gemm::column_parts(BN);
        const int lane = threadIdx.x & 31;
        unsigned char* const first = p.strip - p.part * (4 * gemm::kStripBytes);
        gemm::meet(p.meeting, 32 * kParts, true);
        if (p.part > 0) *reinterpret_cast<float2*>(p.strip + 8 * lane) = make_float2(m, s);
        if (mine) {
            if (a.kept) *reinterpret_cast<float*>(first + 256 + 4 * lane) = at;      // in the first warp's
            else a.at[row] = at;
        }
        gemm::meet(p.meeting, 32 * kParts, true);
        if (p.part == 0) {
#pragma unroll
            for (int w = 1; w < kParts; ++w) {
                const float2 q = *reinterpret_cast<const float2*>(first + w * (4 * gemm::kStripBytes) + 8 * lane);
                const float top = fmaxf(m, q.x), t = top == -INFINITY ? 0.f : top;
                s = s * exp2_fast((m - t) * kLog2e) + q.y * exp2_fast((q.x - t) * kLog2e);
                m = top;
            }
            if (row < p.rows && a.kept) {
                const float l = logf(s);
                a.loss[of_row.to] = (m - *reinterpret_cast<const float*>(first + 256 + 4 * lane)) + l;
                a.lse[of_row.to] = m + l;
            } else if (row < p.rows) {
                a.part[(int64_t)(u.col / BN) * a.rows + row] = make_float2(m, s);
            }
        }
    }
};

// G of a tile, rounded to the operands' type; zero past the last class and the last row, which pads the depth of what reads it.
template <int TYPE>
struct Gradient {
    struct Args {
        const int* label;
        const float* lse;    // of the labelled rows
        const float* weight; // of the labelled rows: bf16 g_loss, fp16 kHalfScale 2^-b
        int first_class;     // of the piece
        int columns;         // with those past the last class: a multiple of 64, or 32
        uint16_t* g;
        int64_t ldg;         // columns, or twice that: then the second half of a row holds what rounding the first one left
    };
    static constexpr bool kMeets = false;
    static __device__ int* flag() { return &g_loss_timeout; }
    struct Row {
        int label;
        float lse, weight;
    };
    static __device__ __forceinline__ Row row(const Args& a, int row, int rows)
    {
        if (row >= rows) return {INT_MIN, 0.f, 0.f};
        return {__ldg(a.label + row), __ldg(a.lse + row), __ldg(a.weight + row)};
    }
    template <int BN, class Done>
    static __device__ __forceinline__ void tile(const Args& a, const gemm::Shape& sh, const gemm::Unit&, const gemm::Part& p, const Row& of_row, const Done& done)
    {
        if (p.row >= (p.rows + 127) / 128 * 128) return done();       // a pair's second block past the last row: G has no such rows
        const bool there = p.row + (int)(threadIdx.x & 31) < p.rows;
        const int label = of_row.label >= a.first_class + p.col ? of_row.label - a.first_class - p.col : INT_MIN;
        const float lse = of_row.lse, weight = of_row.weight;
        gemm::each_chunk<BN>(p, a.columns, done, [&](int c, uint32_t (&v)[32]) {
            const int left = sh.n - (p.col + c);
            float f[32];
#pragma unroll
            for (int i = 0; i < 32; ++i) f[i] = exp2_fast((__uint_as_float(v[i]) - lse) * kLog2e);
            const unsigned in = (unsigned)label - (unsigned)c;
            if (__any_sync(0xffffffffu, in < 32u)) {
#pragma unroll
                for (int i = 0; i < 32; ++i)
                    if (in == (unsigned)i) f[i] -= 1.f;
            }
            uint32_t w[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) w[i] = pack2<TYPE>(f[2 * i] * weight, f[2 * i + 1] * weight);
            const auto put = [&](uint16_t* to) {
                if (!there || left < 32) {
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        if (!there || 2 * i >= left) w[i] = 0u;
                        else if (2 * i + 1 >= left) w[i] &= 0xffffu;
                    }
                }
                gemm::write_strip_whole(p.strip, w, reinterpret_cast<char*>(to), 16 * a.ldg);
            };
            const int lane = threadIdx.x & 31;
            uint16_t* const to = a.g + (int64_t)(p.row + (lane >> 2)) * a.ldg + p.col + c + 8 * (lane & 3);
            if constexpr (BN == 64) {
                if (a.ldg > a.columns) {
                    uint32_t low[16];
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const float2 high = unpack2<TYPE>(w[i]);
                        low[i] = pack2<TYPE>(fmaf(f[2 * i], weight, -high.x), fmaf(f[2 * i + 1], weight, -high.y));
                    }
                    put(to);
#pragma unroll
                    for (int i = 0; i < 16; ++i) w[i] = low[i];
                    return put(to + a.columns);
                }
            }
            put(to);
        });
    }
};

// The accumulators: times a row's factor and a common one where there are such, rounded to the output, or as they are into fp32 parts.
template <int TYPE>
struct Store {
    struct Args {
        const int* map;      // nullable: the output row of every row
        uint16_t* out;       // where there are no parts
        int64_t ldo;
        bool whole;
        float* part;         // [splits][rows][pitch], pitch a multiple of 8
        int64_t pitch, split_stride;
        bool add;            // parts: to what is there
        const float* row_factor;     // nullable
        const float* factor;         // nullable
        float constant;
    };
    static constexpr bool kMeets = false;
    static __device__ int* flag() { return &g_loss_timeout; }
    struct Row {
        int to;
        float factor;
    };
    static __device__ __forceinline__ Row row(const Args& a, int row, int rows)
    {
        return {row < rows && a.map ? __ldg(a.map + row) : row, (row < rows && a.row_factor ? __ldg(a.row_factor + row) : 1.f) * a.constant};
    }
    template <int BN, class Done>
    static __device__ __forceinline__ void tile(const Args& a, const gemm::Shape& sh, const gemm::Unit& u, const gemm::Part& p, const Row& of_row, const Done& done)
    {
        if (p.empty && a.part && a.add) return done();
        const int mapped = of_row.to;
        const float factor = TYPE == BIGCN_F16 ? of_row.factor * (a.factor ? __ldg(a.factor) : 1.f) : 1.f;
        gemm::each_chunk<BN>(p, sh.n, done, [&](int c, uint32_t (&v)[32]) {
            const int col = p.col + c;
            uint32_t w[16];
            if (a.part) {
                float* to = a.part + u.split * a.split_stride + (int64_t)p.row * a.pitch + col;
#pragma unroll
                for (int h = 0; h < 2; ++h) {
#pragma unroll
                    for (int i = 0; i < 16; ++i) w[i] = v[16 * h + i];
                    gemm::write_strip(p.strip, w, [&](int r, int piece, const uint4& q) {
                        if (p.row + r >= p.rows || col + 16 * h + 4 * piece >= a.pitch) return;
                        float4* at = reinterpret_cast<float4*>(to + r * a.pitch + 16 * h + 4 * piece);
                        float4 f = make_float4(__uint_as_float(q.x), __uint_as_float(q.y), __uint_as_float(q.z), __uint_as_float(q.w));
                        if (a.add) {
                            const float4 o = *at;
                            f.x += o.x; f.y += o.y; f.z += o.z; f.w += o.w;
                        }
                        *at = f;
                    });
                }
            } else {
#pragma unroll
                for (int i = 0; i < 16; ++i) w[i] = pack2<TYPE>(__uint_as_float(v[2 * i]) * factor, __uint_as_float(v[2 * i + 1]) * factor);
                const int lane = threadIdx.x & 31;
                if (a.whole && !a.map && p.row + 32 <= p.rows && col + 32 <= sh.n) {
                    gemm::write_strip_whole(p.strip, w, reinterpret_cast<char*>(a.out + (int64_t)(p.row + (lane >> 2)) * a.ldo + col + 8 * (lane & 3)), 16 * a.ldo);
                } else if (a.whole) {
                    gemm::write_strip(p.strip, w, [&](int r, int piece, const uint4& q) {
                        const int64_t to_row = __shfl_sync(0xffffffffu, mapped, r);
                        const int at = col + 8 * piece;
                        if (p.row + r >= p.rows || at >= sh.n) return;
                        uint16_t* to = a.out + to_row * a.ldo + at;
                        if (at + 8 <= sh.n) {
                            *reinterpret_cast<uint4*>(to) = q;
                        } else {
                            const uint16_t* e = reinterpret_cast<const uint16_t*>(&q);
#pragma unroll
                            for (int i = 0; i < 8; ++i)
                                if (at + i < sh.n) to[i] = e[i];
                        }
                    });
                } else {
                    gemm::write_strip_elements(p.strip, w, [&](int r, uint16_t bits) {
                        const int64_t to_row = __shfl_sync(0xffffffffu, mapped, r);
                        if (p.row + r < p.rows && col + lane < sh.n) a.out[to_row * a.ldo + col + lane] = bits;
                    });
                }
            }
        });
    }
};

// ---- joining the parts -----------------------------------------------------------------------------------------------------

// 256 threads to kRows rows: the parts of a row are shared among 256 / kRows threads.
template <int kRows>
__global__ void __launch_bounds__(256) join_loss_kernel(const float2* __restrict__ part, int parts, int64_t pitch, const int* __restrict__ count, int base, int rows,
                                                        const int* __restrict__ kept, const float* __restrict__ at, float* __restrict__ loss, float* __restrict__ lse)
{
    pdl_enter();
    constexpr int kSlices = 256 / kRows;
    __shared__ float ms[kSlices][kRows], ss[kSlices][kRows];
    const int r = threadIdx.x % kRows, slice = threadIdx.x / kRows;
    const int there = min(rows, __ldg(count) - base);
    for (int64_t row0 = (int64_t)blockIdx.x * kRows; row0 < there; row0 += (int64_t)gridDim.x * kRows) {
        const int64_t row = row0 + r;
        float m = -INFINITY, s = 0.f;
        if (row < there) {
            for (int p = slice; p < parts; p += kSlices) {
                const float2 q = __ldg(part + (int64_t)p * pitch + row);
                const float top = fmaxf(m, q.x), t = top == -INFINITY ? 0.f : top;
                s = s * exp2_fast((m - t) * kLog2e) + q.y * exp2_fast((q.x - t) * kLog2e);
                m = top;
            }
        }
        __syncthreads();
        ms[slice][r] = m;
        ss[slice][r] = s;
        __syncthreads();
        if (slice == 0 && row < there) {
            float top = -INFINITY, sum = 0.f;
#pragma unroll 4
            for (int i = 0; i < kSlices; ++i) top = fmaxf(top, ms[i][r]);
            const float t = top == -INFINITY ? 0.f : top;
#pragma unroll 4
            for (int i = 0; i < kSlices; ++i) sum += ss[i][r] * exp2_fast((ms[i][r] - t) * kLog2e);
            const float l = logf(sum);
            const int to = kept[base + row];
            loss[to] = (top - at[row]) + l;
            lse[to] = top + l;
        }
        __syncthreads();
    }
}

struct FinishArgs {
    const float* part;
    int splits;
    int64_t split_stride, pitch;
    const int* count;        // nullable
    int base;
    int64_t rows;
    int d;
    const int* map;          // nullable
    uint16_t* out;
    int64_t ldo;
    bool whole;
    const float* row_factor; // as Store's
    const float* factor;
    float constant;
};
// The parts of a gradient, added in order and rounded: 8 columns to a thread, and where there are many parts of few rows, kSlices threads to
// those, each with every kSlices-th part.
template <int TYPE, int kSlices>
__global__ void __launch_bounds__(256) finish_parts_kernel(const FinishArgs a)
{
    pdl_enter();
    constexpr int kItems = 256 / kSlices;
    __shared__ float sums[kSlices > 1 ? kSlices : 1][kItems][9];
    const int64_t rows = a.count ? min(a.rows, (int64_t)max(0, __ldg(a.count) - a.base)) : a.rows;
    const int words = (a.d + 7) / 8, slice = threadIdx.x / kItems, item = threadIdx.x % kItems;
    for (int64_t base = (int64_t)blockIdx.x * kItems; base < rows * words; base += (int64_t)gridDim.x * kItems) {
        const int64_t t = base + item, row = t / words;
        const int c = (int)(t - row * words) * 8;
        const bool there = t < rows * words;
        float f[8] = {};
        if (there) {
#pragma unroll 4
            for (int s = slice; s < a.splits; s += kSlices) {
                const float4* p = reinterpret_cast<const float4*>(a.part + s * a.split_stride + row * a.pitch + c);
                const float4 u = __ldg(p), v = __ldg(p + 1);
                f[0] += u.x; f[1] += u.y; f[2] += u.z; f[3] += u.w;
                f[4] += v.x; f[5] += v.y; f[6] += v.z; f[7] += v.w;
            }
        }
        if constexpr (kSlices > 1) {
            __syncthreads();
#pragma unroll
            for (int i = 0; i < 8; ++i) sums[slice][item][i] = f[i];
            __syncthreads();
            if (slice == 0) {
#pragma unroll 1
                for (int s = 1; s < kSlices; ++s)
#pragma unroll
                    for (int i = 0; i < 8; ++i) f[i] += sums[s][item][i];
            }
        }
        if (there && slice == 0) {
            const int64_t to = a.map ? __ldg(a.map + row) : row;
            if constexpr (TYPE == BIGCN_F16) {
                const float factor = (a.row_factor ? __ldg(a.row_factor + row) : 1.f) * a.constant * (a.factor ? __ldg(a.factor) : 1.f);
#pragma unroll
                for (int i = 0; i < 8; ++i) f[i] *= factor;
            }
            store_elts<TYPE, 8>(reinterpret_cast<typename Elt<TYPE>::T*>(a.out) + to * a.ldo + c, a.d - c, a.whole, f);
        }
    }
}
template <int TYPE>
cudaError_t launch_finish(cudaStream_t s, const FinishArgs& a, int* launches)
{
    const int64_t items = a.rows * ceil_div(a.d, 8);
    const bool many = a.splits >= 16;
    ++*launches;
    const dim3 grid((unsigned)std::min<int64_t>(8 * sm_count(), ceil_div(items, many ? 16 : 256)));
    return many ? launch_kernel(finish_parts_kernel<TYPE, 16>, grid, dim3(256), 0, s, a) : launch_kernel(finish_parts_kernel<TYPE, 1>, grid, dim3(256), 0, s, a);
}

// ---- plan ------------------------------------------------------------------------------------------------------------------

constexpr int64_t kPieceBytes = int64_t(512) << 20;      // of G (of its high half), and of the forward pass's parts
constexpr size_t kAlign = 256;
size_t up(size_t v) { return (v + kAlign - 1) / kAlign * kAlign; }

int tile_cols(int columns) { return columns <= 64 ? 64 : columns <= 128 ? 128 : 256; }

// How many parts a product's depth is split into, so that its tiles fill the machine.  Its 148 multiprocessors are a constant here, so that the workspace's size is
// one of the sizes alone, whichever device is current; with another number of them the parts are right and their choice is not the best.  What its rounds take, a stage of a pair's 256 x 256 tile
// at 0.42 us and of a block's at 0.15 us (measured), and where it is split another 5 us for the kernel that adds the parts and their bytes, written
// and read, at 5 TB/s.
int pick_splits(int64_t rows, int64_t columns, int64_t stages, int most)
{
    const int bn = tile_cols((int)columns);
    const bool pairs = bn == 256 && rows > gemm::kRows;
    const int units = pairs ? 74 : 148;
    const int64_t tiles = ceil_div(rows, pairs ? 256 : 128) * ceil_div(columns, bn);
    int best = 1;
    double least = 1e30;
    for (int s = 1; s <= most && (s == 1 || stages / s >= 4); ++s) {
        const double t = (double)ceil_div(tiles * s, units) * (double)ceil_div(stages, s) * (pairs ? 0.42 : 0.15) + (s > 1 ? 5.0 + 8.0 * s * (double)rows * (double)columns / 5e6 : 0.0);
        if (t < least) least = t, best = s;
    }
    return best;
}

// How far behind its high half G's low one lies (0: there is none).  In us for the gradients without it and with it, bf16: 2,708 x 64 against 7 classes 27 and 27,
// 219,149 x 232 against 4 144 and 154 (167 with the low half 64 columns on), 2,449,029 x 256 against 47, 8 % labelled, 374 and 387.  From 65 classes on
// it would be more tiles and more depth, for a rounding that counts less among more terms: in the 2-norm (with the result's 0.0016) 0.0019 against
// 65,536 classes, 0.0022 to 0.0024 against 7 and 47.
int low_half(int classes) { return classes <= 32 ? 32 : classes <= 64 ? 64 : 0; }

struct Plan {
    int64_t n_pad, ldt;                       // copied rows
    int64_t rows;                             // of a piece (a multiple of 128)
    int64_t cols;                             // classes of a piece (a multiple of 64; of 256 where there are several)
    int row_pieces, col_pieces;
    int bn, parts;                            // forward: column tile and parts of a row
    int splits_x, splits_w;
    int low;                                  // low_half()
    int bn_d;                                 // column tile of the gradients' products
    int64_t pitch;                            // of fp32 parts
    size_t bytes;
    // offsets
    size_t kept, label, place, count, counts, lse, g_loss, lift, undo, x, w, scaled, top, at, part, g, px, pw;
};

Plan make_plan(int64_t n, int d, int classes, bool backward, bool half)
{
    Plan p = {};
    p.n_pad = round_up(std::max<int64_t>(n, 1), 128);
    p.ldt = round_up(d, 8);
    p.bn = tile_cols(classes);
    size_t off = 0;
    auto take = [&](size_t bytes) { const size_t at = off; off += up(bytes); return at; };
    p.count = take(sizeof(int));
    p.counts = take((size_t)ceil_div(p.n_pad, kScan) * 4);
    p.kept = take((size_t)p.n_pad * 4);
    p.label = take((size_t)p.n_pad * 4);
    p.place = take((size_t)p.n_pad * 4);
    if (backward) {
        p.lse = take((size_t)p.n_pad * 4);
        p.g_loss = take((size_t)p.n_pad * 4);
    }
    p.x = take((size_t)p.n_pad * p.ldt * 2);
    p.w = take((size_t)classes * p.ldt * 2);                    // (the class matrix laid on boundaries, where it is not)
    if (backward && half) {
        p.scaled = take((size_t)p.n_pad * p.ldt * 2);
        p.lift = take((size_t)p.n_pad * 4);
        p.undo = take((size_t)p.n_pad * 4);
        p.top = take(sizeof(unsigned));
    }
    if (!backward) {
        p.parts = (int)ceil_div(classes, p.bn);
        p.rows = p.parts == 1 ? p.n_pad : std::min(p.n_pad, std::max<int64_t>(2048, kPieceBytes / (8 * (int64_t)p.parts) / 128 * 128));
        p.row_pieces = (int)ceil_div(p.n_pad, p.rows);
        p.col_pieces = 1;
        if (p.parts > 1) {
            p.at = take((size_t)p.rows * 4);
            p.part = take((size_t)p.rows * p.parts * 8);
        }
    } else {
        const int64_t all = round_up(classes, 64);
        p.rows = std::min(p.n_pad, std::max<int64_t>(16384, kPieceBytes / (2 * all) / 128 * 128));
        p.cols = std::min(all, std::max<int64_t>(256, kPieceBytes / (2 * p.rows) / 256 * 256));
        p.row_pieces = (int)ceil_div(p.n_pad, p.rows);
        p.col_pieces = (int)ceil_div(classes, p.cols);
        p.bn_d = tile_cols(d);
        p.pitch = round_up(d, 8);
        p.splits_x = pick_splits(std::min<int64_t>(p.rows, std::max<int64_t>(n, 1)), d, p.cols / 64, 148);
        p.splits_w = pick_splits(std::min<int64_t>(p.cols, classes), d, p.rows / 64, 148);
        p.low = low_half(classes);
        p.g = take((size_t)p.rows * std::max<int64_t>(p.cols, 2 * p.low) * 2);
        if (p.splits_x > 1 || p.col_pieces > 1) p.px = take((size_t)p.splits_x * p.n_pad * p.pitch * 4);
        if (p.splits_w > 1 || p.row_pieces > 1 || p.low) p.pw = take((size_t)p.splits_w * round_up(p.cols, 128) * p.pitch * 4);
    }
    p.bytes = off;
    return p;
}

struct Operands {
    int tries;               // bound of the products' waits (0 = default)
    const void* x;
    int64_t ldx;
    bool x_whole;
    const uint16_t* copied;
    const void* w;
    int64_t ldw;
};

// Lists the labelled rows, copies them together where that is needed, and lays the class matrix on 16-byte boundaries.
cudaError_t prepare(cudaStream_t s, const Plan& p, char* ws, int type, const void* x, int64_t ldx, const void* w, int64_t ldw, int64_t n, int d, int classes,
                    const int64_t* labels, float* loss, float* lse, const float* of_lse, const float* of_g_loss, void* g_x, int64_t ldgx, bool want_g_w, int tries, Operands* o, int* launches)
{
    int* counts = reinterpret_cast<int*>(ws + p.counts);
    unsigned* top = type == BIGCN_F16 && of_g_loss ? reinterpret_cast<unsigned*>(ws + p.top) : nullptr;
    const int blocks = (int)ceil_div(n, kScan);
    cudaError_t e = top ? cudaMemsetAsync(top, 0, sizeof(unsigned), s) : cudaSuccess;
    if (e != cudaSuccess) return e;
    if (blocks > 1) {
        ++*launches;
        e = launch_kernel(count_labels_kernel, dim3(blocks), dim3(1024), 0, s, labels, n, classes, counts);
        if (e != cudaSuccess) return e;
    }
    const ListArgs list = {labels, n, classes, counts, reinterpret_cast<int*>(ws + p.kept), reinterpret_cast<int*>(ws + p.label),
                           reinterpret_cast<int*>(ws + p.place), reinterpret_cast<int*>(ws + p.count), loss, lse,
                           (reinterpret_cast<uintptr_t>(loss) | reinterpret_cast<uintptr_t>(lse)) % 16 == 0, of_lse, of_g_loss,
                           reinterpret_cast<float*>(ws + p.lse), reinterpret_cast<float*>(ws + p.g_loss), top};
    *o = {tries, x, ldx, rows_whole(x, ldx, BIGCN_BF16, 8), reinterpret_cast<const uint16_t*>(ws + p.x), w, ldw};
    // rows of a warp at a time: as many times as it takes with 32, and the same each time
    const int resident = o->x_whole && d <= 256 ? 8 : 6;     // blocks of the kernel on a multiprocessor
    const int64_t warps = 8 * resident * sm_count();
    const int span = (int)ceil_div(n, warps * ceil_div(n, warps * 32));
    const GatherArgs gather = {static_cast<const uint16_t*>(x), ldx, n, d, o->x_whole, list.place, list.count, reinterpret_cast<uint16_t*>(ws + p.x), p.ldt,
                               static_cast<uint16_t*>(g_x), ldgx, rows_whole(g_x, ldgx, BIGCN_BF16, 8), span, of_g_loss,
                               reinterpret_cast<const float*>(top), top ? reinterpret_cast<float*>(ws + p.lift) : nullptr, top ? reinterpret_cast<float*>(ws + p.undo) : nullptr,
                               top && want_g_w ? reinterpret_cast<uint16_t*>(ws + p.scaled) : nullptr};
    ++*launches;
    const int lie = o->x_whole ? (d <= 256 ? kShort : kLong) : rows_whole(x, ldx, BIGCN_BF16, 2) ? kPairs : kAnywhere;
    if (n <= kScan) {
        const dim3 grid((unsigned)std::min<int64_t>(ceil_div(n, 32), sm_count()));
        e = launch_kernel(lie == kShort ? list_labels_kernel<true, kShort> : lie == kLong ? list_labels_kernel<true, kLong> : lie == kPairs ? list_labels_kernel<true, kPairs>
                          : list_labels_kernel<true, kAnywhere>, grid, dim3(1024), 0, s, list, gather);
    } else {
        e = launch_kernel(list_labels_kernel<false, kShort>, dim3(blocks), dim3(1024), 0, s, list, gather);
        if (e != cudaSuccess) return e;
        ++*launches;
        const dim3 grid((unsigned)std::min<int64_t>(ceil_div(n, 8 * span), resident * sm_count()));
        e = launch_kernel(lie == kShort ? gather_rows_kernel<kShort> : lie == kLong ? gather_rows_kernel<kLong> : lie == kPairs ? gather_rows_kernel<kPairs>
                          : gather_rows_kernel<kAnywhere>, grid, dim3(256), 0, s, gather);
    }
    if (e != cudaSuccess) return e;
    if (!rows_whole(w, ldw, BIGCN_BF16, 8)) {
        ++*launches;
        const dim3 grid((unsigned)std::min<int64_t>(ceil_div(classes, 8), 8 * sm_count()));
        const uint16_t* from = static_cast<const uint16_t*>(w);
        uint16_t* to = reinterpret_cast<uint16_t*>(ws + p.w);
        if (rows_whole(w, ldw, BIGCN_BF16, 4)) e = launch_kernel(align_rows_kernel<uint2>, grid, dim3(256), 0, s, from, ldw, (int64_t)classes, d, to, p.ldt);
        else if (rows_whole(w, ldw, BIGCN_BF16, 2)) e = launch_kernel(align_rows_kernel<uint32_t>, grid, dim3(256), 0, s, from, ldw, (int64_t)classes, d, to, p.ldt);
        else e = launch_kernel(align_rows_kernel<uint16_t>, grid, dim3(256), 0, s, from, ldw, (int64_t)classes, d, to, p.ldt);
        o->w = ws + p.w;
        o->ldw = p.ldt;
    }
    return e;
}

// Maps of the labelled rows from `first` on: the copied ones, and the rows where they are.
cudaError_t row_maps(CUtensorMap* copied, CUtensorMap* own, const Plan& p, const Operands& o, int64_t n, int d, int64_t first, int box_cols, int box_rows)
{
    cudaError_t e = gemm::encode_map(copied, o.copied + first * p.ldt, 2, false, p.n_pad - first, d, p.ldt * 2, box_cols, box_rows);
    if (e != cudaSuccess) return e;
    if (!o.x_whole) {
        *own = *copied;
        return e;
    }
    return gemm::encode_map(own, static_cast<const uint16_t*>(o.x) + first * o.ldx, 2, false, n - first, d, o.ldx * 2, box_cols, box_rows);
}

template <int BN, int CTAS, class Epi>
cudaError_t launch_logits(cudaStream_t s, const Plan& p, const Operands& o, int64_t n, int d, int classes, int64_t first_row, int64_t rows, int64_t first_class,
                          const int* count, int type, const typename Epi::Args& args, int* launches)
{
    CUtensorMap a, b, own;
    gemm::Shape sh;
    if (CTAS == 1) sh.tile_rows = gemm::rows_of_one_tile(rows);
    cudaError_t e = row_maps(&a, &own, p, o, n, d, first_row, 64, sh.tile_rows);
    if (e == cudaSuccess) e = gemm::encode_map(&b, static_cast<const uint16_t*>(o.w) + first_class * o.ldw, 2, false, classes, d, o.ldw * 2, 64, BN / CTAS);
    if (e != cudaSuccess) return e;
    sh.m = (int)rows;
    sh.n = classes;
    sh.k = d;
    sh.count = count;
    sh.of = (int)n;
    sh.base = (int)first_row;
    sh.alt_a = o.x_whole;
    sh.half = type == BIGCN_F16;
    sh.tries = o.tries;
    sh.rotate = rows <= gemm::kRows;          // classes are read once
    ++*launches;
    return gemm::launch<false, BN, CTAS, false, false, Epi>(s, a, b, own, sh, args);
}
template <class Epi>
cudaError_t pick_logits(cudaStream_t s, int bn, const Plan& p, const Operands& o, int64_t n, int d, int classes, int64_t first_row, int64_t rows, int64_t first_class,
                        const int* count, int type, const typename Epi::Args& args, int* launches)
{
    if (bn == 64) return launch_logits<64, 1, Epi>(s, p, o, n, d, classes, first_row, rows, first_class, count, type, args, launches);
    if (bn == 128) return launch_logits<128, 1, Epi>(s, p, o, n, d, classes, first_row, rows, first_class, count, type, args, launches);
    if (rows > gemm::kRows) return launch_logits<256, 2, Epi>(s, p, o, n, d, classes, first_row, rows, first_class, count, type, args, launches);
    return launch_logits<256, 1, Epi>(s, p, o, n, d, classes, first_row, rows, first_class, count, type, args, launches);
}

// g_x = G W (columns of W outside, its rows the depth) and g_w = G^T X.
template <int TYPE, bool A_MN>
cudaError_t launch_gradient(cudaStream_t s, int bn, const CUtensorMap& g, const CUtensorMap& b, const CUtensorMap& own, const gemm::Shape& sh, const typename Store<TYPE>::Args& args)
{
    if (bn == 64) return gemm::launch<false, 64, 1, A_MN, true, Store<TYPE>>(s, g, b, own, sh, args);
    if (bn == 128) return gemm::launch<false, 128, 1, A_MN, true, Store<TYPE>>(s, g, b, own, sh, args);
    if (sh.m > gemm::kRows) return gemm::launch<false, 256, 2, A_MN, true, Store<TYPE>>(s, g, b, own, sh, args);
    return gemm::launch<false, 256, 1, A_MN, true, Store<TYPE>>(s, g, b, own, sh, args);
}

template <int TYPE>
cudaError_t backward_as(cudaStream_t s, const void* x, int64_t ldx, const void* w, int64_t ldw, int64_t n, int d, int classes, const int64_t* labels,
                                       const float* lse, const float* g_loss, void* g_x, int64_t ldgx, void* g_w, int64_t ldgw, void* scratch, int tries, int* launches)
{
    char* ws = static_cast<char*>(scratch);
    cudaError_t e;
    constexpr int type = TYPE;
    constexpr bool half = TYPE == BIGCN_F16;
    const Plan p = make_plan(n, d, classes, true, half);
    Operands o;
    e = prepare(s, p, ws, type, x, ldx, w, ldw, n, d, classes, labels, nullptr, nullptr, lse, g_loss, g_x, ldgx, g_w != nullptr, tries, &o, launches);
    const int* count = reinterpret_cast<const int*>(ws + p.count);
    const int* kept = reinterpret_cast<const int*>(ws + p.kept);
    const int* label = reinterpret_cast<const int*>(ws + p.label);
    uint16_t* g = reinterpret_cast<uint16_t*>(ws + p.g);
    const bool parts_x = p.splits_x > 1 || p.col_pieces > 1, parts_w = p.splits_w > 1 || p.row_pieces > 1 || p.low;
    for (int c = 0; c < p.col_pieces && e == cudaSuccess; ++c) {
        const int64_t first_class = c * p.cols;
        const int here = (int)std::min<int64_t>(p.cols, classes - first_class);
        const int columns = p.low ? p.low : (int)round_up(here, 64);
        const int64_t ldg = p.low ? 2 * p.low : columns;
        for (int r = 0; r < p.row_pieces && e == cudaSuccess; ++r) {
            const int64_t first = r * p.rows, rows = std::min(p.rows, n - first);
            if (rows <= 0) break;
            const typename Gradient<TYPE>::Args ga = {label + first, reinterpret_cast<const float*>(ws + p.lse) + first, reinterpret_cast<const float*>(ws + (half ? p.lift : p.g_loss)) + first, (int)first_class, columns, g, ldg};
            e = pick_logits<Gradient<TYPE>>(s, tile_cols(here), p, o, n, d, here, first, rows, first_class, count, type, ga, launches);
            if (e != cudaSuccess) break;
            gemm::Shape sh;
            sh.n = d;
            sh.count = count;
            sh.of = (int)n;
            sh.base = (int)first;
            sh.half = half;
            sh.tries = tries;
            if (g_x) {
                CUtensorMap mg, mw;
                sh.tile_rows = gemm::rows_of_one_tile(rows);
                sh.rotate = rows <= gemm::kRows;
                e = gemm::encode_map(&mg, g, 2, false, round_up(rows, 128), ldg, ldg * 2, 64, sh.tile_rows);
                if (e == cudaSuccess) e = gemm::encode_map(&mw, static_cast<const uint16_t*>(o.w) + first_class * o.ldw, 2, false, here, d, o.ldw * 2, 64, p.low == 32 ? 32 : 64);
                if (e != cudaSuccess) break;
                sh.m = (int)rows;
                sh.k = p.low ? (int)ldg : here;                // (zeros of G meet the classes that are not there)
                sh.b_depth = p.low;
                sh.splits = p.splits_x;
                const typename Store<TYPE>::Args args = {kept + first, static_cast<uint16_t*>(g_x), ldgx, rows_whole(g_x, ldgx, BIGCN_BF16, 8),
                                          parts_x ? reinterpret_cast<float*>(ws + p.px) + first * p.pitch : nullptr, p.pitch, p.n_pad * p.pitch, c > 0,
                                          half ? reinterpret_cast<const float*>(ws + p.undo) + first : nullptr, nullptr, 1.f};
                ++*launches;
                e = launch_gradient<TYPE, false>(s, p.bn_d, mg, mw, mw, sh, args);
                if (e == cudaSuccess && parts_x && c == p.col_pieces - 1) {
                    const FinishArgs fa = {args.part, p.splits_x, args.split_stride, p.pitch, count, (int)first, rows, d, kept + first, static_cast<uint16_t*>(g_x), ldgx, args.whole, args.row_factor, args.factor, args.constant};
                    e = launch_finish<TYPE>(s, fa, launches);
                }
                if (e != cudaSuccess) break;
            }
            if (g_w) {
                CUtensorMap mg, mx, own;
                e = gemm::encode_map(&mg, g, 2, false, round_up(rows, 128), ldg, ldg * 2, 64, 64);
                if (e == cudaSuccess && half) {
                    e = gemm::encode_map(&mx, reinterpret_cast<const uint16_t*>(ws + p.scaled) + first * p.ldt, 2, false, p.n_pad - first, d, p.ldt * 2, 64, 64);
                    own = mx;
                } else if (e == cudaSuccess) {
                    e = row_maps(&mx, &own, p, o, n, d, first, 64, 64);
                }
                if (e != cudaSuccess) break;
                sh.m = p.low ? (int)ldg : here;                // the halves' sums as rows of their own, added with the other parts
                sh.k = (int)rows;
                sh.b_depth = 0;
                sh.splits = p.splits_w;
                sh.over_depth = true;
                sh.rotate = false;
                sh.alt_b = o.x_whole && !half;
                uint16_t* out = static_cast<uint16_t*>(g_w) + first_class * ldgw;
                const typename Store<TYPE>::Args args = {nullptr, out, ldgw, rows_whole(out, ldgw, BIGCN_BF16, 8), parts_w ? reinterpret_cast<float*>(ws + p.pw) : nullptr, p.pitch,
                                          (p.low ? ldg : round_up(p.cols, 128)) * p.pitch, r > 0, nullptr, half ? reinterpret_cast<const float*>(ws + p.top) : nullptr, half ? 1.f / kHalfScale : 1.f};
                ++*launches;
                e = launch_gradient<TYPE, true>(s, p.bn_d, mg, mx, own, sh, args);
                if (e == cudaSuccess && parts_w && r == p.row_pieces - 1) {
                    const FinishArgs fa = {args.part, p.low ? 2 * p.splits_w : p.splits_w, p.low ? p.low * p.pitch : args.split_stride, p.pitch, nullptr, 0, here, d, nullptr, out, ldgw, args.whole, args.row_factor, args.factor, args.constant};
                    e = launch_finish<TYPE>(s, fa, launches);
                }
            }
        }
    }
    return e;
}

}  // namespace

int class_loss_timeouts()
{
    int v = 0;
    if (cudaMemcpyFromSymbol(&v, g_loss_timeout, sizeof(int)) != cudaSuccess) return -1;
    return v;
}

size_t class_loss_scratch_bytes(int64_t n, int d, int classes, bool backward) { return make_plan(n, d, classes, backward, true).bytes; }

cudaError_t launch_class_loss(cudaStream_t s, int type, const void* x, int64_t ldx, const void* w, int64_t ldw, int64_t n, int d, int classes, const int64_t* labels,
                              float* loss, float* lse, void* scratch, int tries, int* launches)
{
    char* ws = static_cast<char*>(scratch);
    cudaError_t e;
    const Plan p = make_plan(n, d, classes, false, false);
    Operands o;
    e = prepare(s, p, ws, type, x, ldx, w, ldw, n, d, classes, labels, loss, lse, nullptr, nullptr, nullptr, 0, false, tries, &o, launches);
    const int* count = reinterpret_cast<const int*>(ws + p.count);
    const int* kept = reinterpret_cast<const int*>(ws + p.kept);
    float* at = reinterpret_cast<float*>(ws + p.at);
    float2* part = reinterpret_cast<float2*>(ws + p.part);
    for (int r = 0; r < p.row_pieces && e == cudaSuccess; ++r) {
        const int64_t first = r * p.rows, rows = std::min(p.rows, n - first);
        if (rows <= 0) break;
        const bool direct = p.parts == 1;
        const SumExp::Args args = {reinterpret_cast<const int*>(ws + p.label) + first, part, p.rows, at, direct ? kept + first : nullptr, loss, lse};
        e = pick_logits<SumExp>(s, p.bn, p, o, n, d, classes, first, rows, 0, count, type, args, launches);
        if (e != cudaSuccess || direct) continue;
        ++*launches;
        const auto blocks = [&](int rows_per_block) { return dim3((unsigned)std::min<int64_t>(ceil_div(rows, rows_per_block), 16 * sm_count())); };
        // rows side by side where there are enough of them, else threads side by side over a row's parts (512 parts of 128 rows in us: 26 with
        // 32 rows to a block, 8 with four)
        if (p.parts <= 16) e = launch_kernel(join_loss_kernel<256>, blocks(256), dim3(256), 0, s, (const float2*)part, p.parts, p.rows, count, (int)first, (int)rows, kept, (const float*)at, loss, lse);
        else if (rows >= 4096) e = launch_kernel(join_loss_kernel<32>, blocks(32), dim3(256), 0, s, (const float2*)part, p.parts, p.rows, count, (int)first, (int)rows, kept, (const float*)at, loss, lse);
        else e = launch_kernel(join_loss_kernel<4>, blocks(4), dim3(256), 0, s, (const float2*)part, p.parts, p.rows, count, (int)first, (int)rows, kept, (const float*)at, loss, lse);
    }
    return e;
}

cudaError_t launch_class_loss_backward(cudaStream_t s, int type, const void* x, int64_t ldx, const void* w, int64_t ldw, int64_t n, int d, int classes,
                                       const int64_t* labels, const float* lse, const float* g_loss, void* g_x, int64_t ldgx, void* g_w, int64_t ldgw,
                                       void* scratch, int tries, int* launches)
{
    return type == BIGCN_F16 ? backward_as<BIGCN_F16>(s, x, ldx, w, ldw, n, d, classes, labels, lse, g_loss, g_x, ldgx, g_w, ldgw, scratch, tries, launches)
                             : backward_as<BIGCN_BF16>(s, x, ldx, w, ldw, n, d, classes, labels, lse, g_loss, g_x, ldgx, g_w, ldgw, scratch, tries, launches);
}

}  // namespace bigcn
