// Rows in 8-bit integers and their product with 8-bit class rows.
//
//   s_i = max_j |x_ij| / 127,  q_ij = the integer nearest to 127 x_ij / max_j |x_ij| (halfway: the even one)
//   out_ik = (sum_j q_ij qw_kj) s_i sw_k
//
// The integers are exact: the sum of 16,384 products of 127 stays below 2^31.  The three roundings of an output (the sum to fp32, and
// two products) are fp32's, then one to the output's type.  The sum comes before the scales' product, which may leave fp32's range where the
// output does not: two scales of 2^-75 lose the digits that a sum of 2^28 brings back, and a sum of 0 times infinity is no number.  The scale
// of a row with fp32's lowest value in it, 2^121, times the sum would overflow likewise: see row_scale().
#include <climits>
#include <type_traits>

#include "dense_gemm.cuh"
#include "dense_types.cuh"

namespace bigcn {

namespace {

using namespace dense;

__device__ int g_quant_timeout;               // set when a wait ran out

struct QuantArgs {
    const void* x;
    int type;
    int64_t ldx, n;
    int d;
    bool whole;              // kAnyType: rows start on boundaries of four elements
    int8_t* q;
    int64_t ldq;
    float* scale;
    bool early;              // the next kernel may start: it waits for this one where it reads what this one writes
};

// Four values as the integers nearest to 127 x / top, in the bytes of a word.  The sum with 1.5 * 2^23 rounds x (127 / top) to an integer and holds it
// in its low bits; the quotient in it is off by 127 * 2^-23 at most (the factor's rounding, and the sum's own at the border).  Where that
// could decide one of the roundings, they are taken exactly: of 16-bit types in fp32, where 127 x is exact and a quotient is halfway between
// integers or at least 2^-20 of its size away, so that its one rounding neither meets nor misses that; of fp32 in 64 bits, where the
// same holds with 2^-32.
template <bool HALF>
__device__ __noinline__ uint32_t nearest4_exactly(float4 x, float top)
{
    const float v[4] = {x.x, x.y, x.z, x.w};
    uint32_t n[4];
    const float down = HALF && top > 1e30f ? 0x1p-10f : 1.f;                 // 127 x would overflow
#pragma unroll
    for (int i = 0; i < 4; ++i)
        n[i] = HALF ? (uint32_t)(int)rintf(__fdiv_rn(127.f * (v[i] * down), top * down)) : (uint32_t)(int)rint(127.0 * (double)v[i] / (double)top);
    return __byte_perm(__byte_perm(n[0], n[1], 0x0040), __byte_perm(n[2], n[3], 0x0040), 0x5410);
}
template <bool HALF>
__device__ __forceinline__ uint32_t nearest4(const float* x, float factor, float top, bool tiny)
{
    constexpr float kRound = 12582912.f;
    uint32_t n[4];
    float off = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float r = fmaf(x[i], factor, kRound);
        n[i] = __float_as_uint(r);
        off = fmaxf(off, fabsf(fmaf(x[i], factor, kRound - r)));
    }
    if (tiny || off > 0.49998f) return nearest4_exactly<HALF>(make_float4(x[0], x[1], x[2], x[3]), top);
    return __byte_perm(__byte_perm(n[0], n[1], 0x0040), __byte_perm(n[2], n[3], 0x0040), 0x5410);
}

// Rows to LANES threads (a warp or a block) one after the other, V values at a time, NV times; the next row is on its way while one is worked on.
template <int TYPE, int V, int LANES, int NV>
__global__ void __launch_bounds__(LANES > 32 ? LANES : 256, LANES > 32 ? 1 : NV * V > 16 ? 2 : 4) quantize_kernel(const QuantArgs a)
{
    pdl_enter();
    if (a.early) asm volatile("griddepcontrol.launch_dependents;\n" ::: "memory");
    constexpr int B = LANES > 32 ? LANES : 256, GROUPS = B / LANES;
    __shared__ uint32_t slots[2][LANES > 32 ? LANES / 32 : 1];
    const int lane = threadIdx.x % LANES;
    const int64_t step = (int64_t)gridDim.x * GROUPS;
    int64_t row = (int64_t)blockIdx.x * GROUPS + threadIdx.x / LANES;
    Raw<TYPE, V> next[NV];
    auto fetch = [&](int64_t r) {
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int c = (k * LANES + lane) * V;
            next[k].load(a.x, a.type, r * a.ldx + c, r < a.n ? a.d - c : 0, a.whole);
        }
    };
    fetch(row);
    int trip = 0;
    for (int64_t base = (int64_t)blockIdx.x * GROUPS; base < a.n; base += step, row += step, trip ^= 1) {      // the same trips for all threads of a block
        Raw<TYPE, V> w[NV];
        uint32_t top = 0u;                    // as bits, which order magnitudes, infinity and NaN
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            w[k] = next[k];
            float v[V];
            w[k].values(v, a.type);
#pragma unroll
            for (int i = 0; i < V; ++i) top = max(top, __float_as_uint(v[i]) & 0x7fffffffu);
        }
        fetch(row + step);
        if constexpr (LANES < 32) {
#pragma unroll
            for (int m = LANES / 2; m >= 1; m >>= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, m));
        } else {
            top = __reduce_max_sync(0xffffffffu, top);
        }
        if constexpr (LANES > 32) {
            uint32_t* slot = slots[trip];
            if ((threadIdx.x & 31) == 0) slot[threadIdx.x >> 5] = top;
            __syncthreads();
            top = __reduce_max_sync(0xffffffffu, (threadIdx.x & 31) < LANES / 32 ? slot[threadIdx.x & 31] : 0u);
        }
        if (row >= a.n) continue;             // (the warp's other rows go on: nothing below is done together)
        const bool finite = top < 0x7f800000u;
        const float t = __uint_as_float(top), factor = 127.f / t;
        const bool tiny = t < 1e-30f;         // 127 / t would overflow
        if (lane == 0) a.scale[row] = finite ? t / 127.f : __uint_as_float(0x7fc00000u);
        int8_t* q = a.q + row * a.ldq;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int c = (k * LANES + lane) * V;
            if (c >= a.d) break;
            float v[V];
            w[k].values(v, a.type);
            uint32_t o[V / 4];
#pragma unroll
            for (int j = 0; j < V / 4; ++j) o[j] = finite && top ? nearest4<TYPE == BIGCN_BF16 || TYPE == BIGCN_F16>(v + 4 * j, factor, t, tiny) : 0u;
            if (c + V <= a.d) {               // rows of q start on 16-byte boundaries
                if constexpr (V == 4) *reinterpret_cast<uint32_t*>(q + c) = o[0];
                else *reinterpret_cast<uint2*>(q + c) = make_uint2(o[0], o[1]);
            } else {
#pragma unroll
                for (int i = 0; i < V; ++i)
                    if (c + i < a.d) q[c + i] = (int8_t)(o[i >> 2] >> (8 * (i & 3)));
            }
        }
    }
}

template <int TYPE, int V, int LANES, int NV>
cudaError_t launch_quantize_as(cudaStream_t s, const QuantArgs& a, int* launches)
{
    constexpr int B = LANES > 32 ? LANES : 256;
    ++*launches;
    const int64_t blocks = std::min<int64_t>(ceil_div(a.n, B / LANES), (int64_t)sm_count() * (LANES > 32 ? 2048 / B : NV * V > 16 ? 2 : 4));
    return launch_kernel(quantize_kernel<TYPE, V, LANES, NV>, dim3((unsigned)blocks), dim3(B), 0, s, a);
}
// A warp to a row as long as that leaves the machine enough warps, else a block.  In us: 16,384 bf16 rows of 2,048 45 with a row of 128 threads,
// 32 with a warp; 169,343 fp32 rows of 256 53 with a warp that ends with its row, 39 with one that goes on.
template <int TYPE, int V>
cudaError_t pick_quantize(cudaStream_t s, const QuantArgs& a, int* launches)
{
    constexpr int Q = 16 / V;
    const int64_t words = ceil_div(a.d, V);
    const bool many = a.n >= 4096;
    if (words <= 8) return launch_quantize_as<TYPE, V, 8, 1>(s, a, launches);
    if (words <= 16) return launch_quantize_as<TYPE, V, 16, 1>(s, a, launches);
    if (words <= 32) return launch_quantize_as<TYPE, V, 32, 1>(s, a, launches);
    if (words <= 64) return launch_quantize_as<TYPE, V, 32, 2>(s, a, launches);
    if (words <= 32 * Q || (many && words <= 128)) return launch_quantize_as<TYPE, V, 32, 4>(s, a, launches);
    if (many && words <= 256) return launch_quantize_as<TYPE, V, 32, 8>(s, a, launches);
    if (words <= 128 * Q) return launch_quantize_as<TYPE, V, 128, Q>(s, a, launches);
    if (words <= 512 * Q) return launch_quantize_as<TYPE, V, 512, Q>(s, a, launches);
    return launch_quantize_as<TYPE, V, 1024, Q>(s, a, launches);
}

// A sum times a row's scale s and a class's t, in this order in every form of the product, so that all give the same bits.  The sum is below 2^28 and so times s
// in range up to 2^99; of a larger s 2^-64 goes in first, which is 2^32 and more, so that no t loses digits either, and where that overflows without the
// 2^64 that come last it does with them.
__device__ __forceinline__ bool large_scale(float s) { return fabsf(s) >= 0x1p96f; }
struct RowScale {
    float s, last;
};
__device__ __forceinline__ RowScale row_scale(float s)
{
    const bool large = large_scale(s);
    return {large ? s * 0x1p-64f : s, large ? 0x1p64f : 1.f};
}
__device__ __forceinline__ float scaled(int sum, const RowScale& r, float t) { return (float)sum * r.s * t * r.last; }

// Epilogue: the sums times both scales, in the output's type.
struct ScaledArgs {
    const float* s_x;
    const float* s_w;
    bool s_w_whole;
    void* out;
    int type;
    int64_t ldo;
    bool whole;              // rows of out on 16-byte boundaries
};

// A warp's part of a tile with a large scale of a row, a column at a time: so little code that the other tiles take no longer for it (with a function that
// is called instead, 92 us for 85 at 3,269 x 64 times 34,624 classes in bf16).
template <int TYPE>
__device__ __forceinline__ void large_tile(const ScaledArgs& a, const gemm::Part& p, int cols, float s)
{
    const int row = p.row + (threadIdx.x & 31);
    const RowScale scale = row_scale(s);
    typename Elt<TYPE>::T* to = static_cast<typename Elt<TYPE>::T*>(a.out) + (int64_t)row * a.ldo + p.col;
#pragma unroll 1
    for (int c = 0; c < cols; ++c) {
        const int sum = (int)gemm::tmem_ld1(p.acc + c);
        if (row < p.rows) to[c] = from_float<TYPE>(scaled(sum, scale, __ldg(a.s_w + p.col + c)));
        __syncwarp();
    }
}
__device__ __forceinline__ void times(uint32_t (&v)[32], int i, const float4& w)
{
    v[i] = __float_as_uint(__uint_as_float(v[i]) * w.x);
    v[i + 1] = __float_as_uint(__uint_as_float(v[i + 1]) * w.y);
    v[i + 2] = __float_as_uint(__uint_as_float(v[i + 2]) * w.z);
    v[i + 3] = __float_as_uint(__uint_as_float(v[i + 3]) * w.w);
}
template <int TYPE>
struct ScaledOut {
    using Args = ScaledArgs;
    static constexpr bool kMeets = false;
    static __device__ int* flag() { return &g_quant_timeout; }
    using Row = float;
    static __device__ __forceinline__ Row row(const Args& a, int row, int rows) { return row < rows ? __ldg(a.s_x + row) : 0.f; }
    template <int BN, class Done>
    static __device__ __forceinline__ void tile(const Args& a, const gemm::Shape& sh, const gemm::Unit&, const gemm::Part& p, const Row& sx, const Done& done)
    {
        if (__any_sync(0xffffffffu, large_scale(sx))) {
            large_tile<TYPE>(a, p, min(gemm::part_cols(BN), sh.n - p.col), sx);
            return done();
        }
        const int lane = threadIdx.x & 31;
        // the warp's class scales are read by all lanes at once below: from L1 by then
        if (lane < gemm::part_cols(BN) / 32 && p.col + 32 * lane < sh.n) asm volatile("prefetch.global.L1 [%0];\n" ::"l"(a.s_w + p.col + 32 * lane));
        using T = typename Elt<TYPE>::T;
        T* const at = static_cast<T*>(a.out) + (int64_t)p.row * a.ldo + p.col;
        const bool rows_there = p.row + 32 <= p.rows;
        gemm::each_chunk<BN>(p, sh.n, done, [&](int c, uint32_t (&v)[32]) {
            const int left = sh.n - (p.col + c);
            if (a.s_w_whole && left >= 32) {
                const float4* from = reinterpret_cast<const float4*>(a.s_w + p.col + c);
                if constexpr (TYPE == BIGCN_F32) {
                    // all scales first (8,192 x 256 times 10,000 classes in us: fp32 90 so, 103 with a scale read where it is needed; 3,269 x 64 times 34,624, bf16: 90
                    // and 86)
                    float4 w[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) w[i] = __ldg(from + i);
#pragma unroll
                    for (int i = 0; i < 32; ++i) v[i] = __float_as_uint((float)(int)v[i] * sx);
#pragma unroll
                    for (int i = 0; i < 8; ++i) times(v, 4 * i, w[i]);
                } else {
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
#pragma unroll
                        for (int j = 0; j < 4; ++j) v[4 * i + j] = __float_as_uint((float)(int)v[4 * i + j] * sx);
                        times(v, 4 * i, __ldg(from + i));
                    }
                }
            } else {
#pragma unroll
                for (int i = 0; i < 32; ++i) v[i] = __float_as_uint((float)(int)v[i] * sx * (i < left ? __ldg(a.s_w + p.col + c + i) : 0.f));
            }
            T* const to = at + c;
            if constexpr (TYPE == BIGCN_F32) {
                if (a.whole && rows_there && left >= 32) {
                    float* e = to + (int64_t)(lane >> 3) * a.ldo + (lane & 7) * 4;
                    gemm::write_wide(p.strip, v, [&](int, int, const uint4& q) {
                        *reinterpret_cast<uint4*>(e) = q;
                        e += 4 * a.ldo;
                    });
                } else if (a.whole) {
                    const auto put = [&](int r, int piece, const uint4& q) {
                        const int there = left - 4 * piece;
                        if (p.row + r >= p.rows || there <= 0) return;
                        float* e = to + r * a.ldo + 4 * piece;
                        if (there >= 4) {
                            *reinterpret_cast<uint4*>(e) = q;
                        } else {
                            const float* from = reinterpret_cast<const float*>(&q);
#pragma unroll
                            for (int i = 0; i < 4; ++i)
                                if (i < there) e[i] = from[i];
                        }
                    };
                    if (left > 16) {
                        gemm::write_wide(p.strip, v, put);
                    } else {
                        uint32_t w[16];
#pragma unroll
                        for (int i = 0; i < 16; ++i) w[i] = v[i];
                        gemm::write_strip(p.strip, w, put);
                    }
                } else {
                    uint32_t* e = reinterpret_cast<uint32_t*>(to) + lane;
                    const int rows = lane < left ? p.rows - p.row : 0;
                    gemm::write_wide_elements(p.strip, v, [&](int r, uint32_t q) {
                        if (r < rows) *e = q;
                        e += a.ldo;
                    });
                }
            } else {
                uint32_t w[16];
#pragma unroll
                for (int i = 0; i < 16; ++i) w[i] = pack2<TYPE>(__uint_as_float(v[2 * i]), __uint_as_float(v[2 * i + 1]));
                if (a.whole && rows_there && left >= 32) {
                    gemm::write_strip_whole(p.strip, w, reinterpret_cast<char*>(to + (int64_t)(lane >> 2) * a.ldo + (lane & 3) * 8), 16 * a.ldo);
                } else if (a.whole) {
                    gemm::write_strip(p.strip, w, [&](int r, int piece, const uint4& q) {
                        const int there = left - piece * 8;
                        if (p.row + r >= p.rows || there <= 0) return;
                        T* e = to + r * a.ldo + piece * 8;
                        if (there >= 8) {
                            *reinterpret_cast<uint4*>(e) = q;
                        } else {
                            const T* from = reinterpret_cast<const T*>(&q);
#pragma unroll
                            for (int i = 0; i < 8; ++i)
                                if (i < there) e[i] = from[i];
                        }
                    });
                } else {
                    uint16_t* e = reinterpret_cast<uint16_t*>(to) + lane;
                    const int rows = lane < left ? p.rows - p.row : 0;
                    gemm::write_strip_elements(p.strip, w, [&](int r, uint16_t q) {
                        if (r < rows) *e = q;
                        e += a.ldo;
                    });
                }
            }
        });
    }
};

// The same with classes as rows of the tiles and the few rows of x as columns: a lane has a class, so that 32 neighbours of an output row
// are stored together, and 128 class rows to a tile leave more tiles than 256 columns would.
struct ScaledAcross {
    using Args = ScaledArgs;
    static constexpr bool kMeets = false;
    static __device__ int* flag() { return &g_quant_timeout; }
    using Row = float;
    static __device__ __forceinline__ Row row(const Args& a, int row, int rows) { return row < rows ? __ldg(a.s_w + row) : 0.f; }
    template <int BN, class Done>
    static __device__ __forceinline__ void tile(const Args& a, const gemm::Shape& sh, const gemm::Unit&, const gemm::Part& p, const Row& sw, const Done& done)
    {
        static_assert(gemm::part_cols(BN) == 32, "a lane looks at the scale of one row of x");
        const int lane = threadIdx.x & 31, k = p.row + lane, cols = min(32, sh.n - p.col);
        if (__any_sync(0xffffffffu, lane < cols && large_scale(__ldg(a.s_x + p.col + lane)))) {      // a column at a time, as large_tile()
#pragma unroll 1
            for (int i = 0; i < cols; ++i) {
                const float f[1] = {scaled((int)gemm::tmem_ld1(p.acc + i), row_scale(__ldg(a.s_x + p.col + i)), sw)};
                if (k < p.rows) store_as<1>(a.out, a.type, (int64_t)(p.col + i) * a.ldo + k, 1, true, f);
                __syncwarp();
            }
            return done();
        }
        gemm::each_chunk<BN>(p, sh.n, done, [&](int c, uint32_t (&v)[32]) {
            if (k >= p.rows) return;
#pragma unroll
            for (int i = 0; i < 32; ++i) {
                const int row = p.col + c + i;
                if (row >= sh.n) break;
                const float f[1] = {(float)(int)v[i] * __ldg(a.s_x + row) * sw};
                store_as<1>(a.out, a.type, (int64_t)row * a.ldo + k, 1, true, f);
            }
        });
    }
};

// One to four rows, not yet quantised, in one launch.  Every block quantises them for itself into shared memory (their bytes times the number of
// blocks come from L2 and are few) while its first class rows are on their way; then a warp takes kGemvRows class rows at a time, 16 bytes of each a
// lane, and sums by four-byte dot products.  Bound by the class rows, which are read once: 65,536 classes x 1,024 for one row in us, with the
// 67 MB in L2 from the call before: 19.8 by two kernels with tensor memory to set up, 10.3 so; from memory 15.2 (68 % of a plain copy's rate).  More rows cost
// more dot products: few_rows_pays().
constexpr int kGemvThreads = 512, kGemvRows = 4, kGemvMax = 4, kGemvBytes = 64 * 1024;
struct GemvArgs {
    const void* x;
    int type;
    int64_t ldx;
    int n, d;
    bool whole;
    const int8_t* q_w;
    int64_t ldqw;
    const float* s_w;
    int m;
    void* out;
    int out_type;
    int64_t ldo;
};
template <int N>
__global__ void __launch_bounds__(kGemvThreads, 2) few_rows_kernel(const GemvArgs a)
{
    pdl_enter();
    extern __shared__ uint4 qs[];             // [N][words] the quantised rows
    __shared__ uint32_t slot[kGemvThreads / 32];
    __shared__ RowScale scales[N];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, words = (a.d + 15) / 16;
    const int warps = gridDim.x * (kGemvThreads / 32);
    int k = (blockIdx.x * (kGemvThreads / 32) + warp) * kGemvRows;
    uint4 w[kGemvRows];
    auto fetch = [&](int at, int word) {
#pragma unroll
        for (int j = 0; j < kGemvRows; ++j)
            w[j] = word < words && at + j < a.m ? __ldg(reinterpret_cast<const uint4*>(a.q_w + (int64_t)(at + j) * a.ldqw) + word) : make_uint4(0u, 0u, 0u, 0u);
    };
    fetch(k, lane);
    for (int r = 0; r < N; ++r) {
        const int64_t row = (int64_t)r * a.ldx;
        uint32_t top = 0u;
        for (int c = threadIdx.x * 4; c < a.d; c += kGemvThreads * 4) {
            float v[4];
            load4(a.x, a.type, row + c, r < a.n ? a.d - c : 0, a.whole, v);
#pragma unroll
            for (int i = 0; i < 4; ++i) top = max(top, __float_as_uint(v[i]) & 0x7fffffffu);
        }
        top = __reduce_max_sync(0xffffffffu, top);
        __syncthreads();
        if (lane == 0) slot[warp] = top;
        __syncthreads();
        top = __reduce_max_sync(0xffffffffu, lane < kGemvThreads / 32 ? slot[lane] : 0u);
        const bool finite = top < 0x7f800000u;
        const float t = __uint_as_float(top), factor = 127.f / t;
        if (threadIdx.x == 0) scales[r] = row_scale(finite ? t / 127.f : __uint_as_float(0x7fc00000u));
        uint32_t* q = reinterpret_cast<uint32_t*>(qs + r * words);
        for (int c = threadIdx.x * 4; c < words * 16; c += kGemvThreads * 4) {
            float v[4];
            load4(a.x, a.type, row + c, r < a.n ? a.d - c : 0, a.whole, v);
            q[c / 4] = finite && top ? nearest4<false>(v, factor, t, t < 1e-30f) : 0u;
        }
    }
    __syncthreads();
    for (; k < a.m; k += warps * kGemvRows) {
        int sum[kGemvRows][N] = {};
        for (int word = lane; word < words; word += 32) {
            uint4 now[kGemvRows];
#pragma unroll
            for (int j = 0; j < kGemvRows; ++j) now[j] = w[j];
            // the lane's next word of these rows, or its first of the next ones
            if (word + 32 < words) fetch(k, word + 32);
            else fetch(k + warps * kGemvRows, lane);
#pragma unroll
            for (int r = 0; r < N; ++r) {
                const uint4 x = qs[r * words + word];
#pragma unroll
                for (int j = 0; j < kGemvRows; ++j) {
                    sum[j][r] = __dp4a((int)now[j].x, (int)x.x, sum[j][r]);
                    sum[j][r] = __dp4a((int)now[j].y, (int)x.y, sum[j][r]);
                    sum[j][r] = __dp4a((int)now[j].z, (int)x.z, sum[j][r]);
                    sum[j][r] = __dp4a((int)now[j].w, (int)x.w, sum[j][r]);
                }
            }
        }
#pragma unroll
        for (int j = 0; j < kGemvRows; ++j)
#pragma unroll
            for (int r = 0; r < N; ++r) {
                const int total = __reduce_add_sync(0xffffffffu, sum[j][r]);
                if (lane == j * N + r && k + j < a.m && r < a.n) {
                    const float f[1] = {scaled(total, scales[r], __ldg(a.s_w + k + j))};
                    store_as<1>(a.out, a.out_type, (int64_t)r * a.ldo + k + j, 1, true, f);
                }
            }
    }
}
template <int N>
cudaError_t launch_few_rows(cudaStream_t s, const GemvArgs& a)
{
    const size_t smem = (size_t)N * ((a.d + 15) / 16) * 16;
    static std::atomic<uint64_t> ready{0};    // by device
    const cudaError_t e = allow_shared(few_rows_kernel<N>, smem, &ready);
    if (e != cudaSuccess) return e;
    const int64_t blocks = std::min<int64_t>(2 * sm_count(), ceil_div(a.m, kGemvThreads / 32 * kGemvRows));
    return launch_kernel(few_rows_kernel<N>, dim3((unsigned)blocks), dim3(kGemvThreads), smem, s, a);
}

template <int BN, int CTAS>
cudaError_t launch_product_as(cudaStream_t s, const int8_t* q_x, int64_t ldqx, const int8_t* q_w, int64_t ldqw, const gemm::Shape& shape, const ScaledArgs& args)
{
    CUtensorMap ma, mb;
    cudaError_t e = gemm::encode_map(&ma, q_x, 1, true, shape.m, shape.k, ldqx, 128, shape.tile_rows);
    if (e == cudaSuccess) e = gemm::encode_map(&mb, q_w, 1, true, shape.n, shape.k, ldqw, 128, BN / CTAS);
    if (e != cudaSuccess) return e;
    if (args.type == BIGCN_F32) return gemm::launch<true, BN, CTAS, false, false, ScaledOut<BIGCN_F32>>(s, ma, mb, ma, shape, args);
    if (args.type == BIGCN_BF16) return gemm::launch<true, BN, CTAS, false, false, ScaledOut<BIGCN_BF16>>(s, ma, mb, ma, shape, args);
    return gemm::launch<true, BN, CTAS, false, false, ScaledOut<BIGCN_F16>>(s, ma, mb, ma, shape, args);
}

template <int BN>
cudaError_t launch_across(cudaStream_t s, const int8_t* q_x, int64_t ldqx, const int8_t* q_w, int64_t ldqw, const gemm::Shape& shape, const ScaledArgs& args)
{
    CUtensorMap ma, mb;
    cudaError_t e = gemm::encode_map(&ma, q_w, 1, true, shape.m, shape.k, ldqw, 128, shape.tile_rows);
    if (e == cudaSuccess) e = gemm::encode_map(&mb, q_x, 1, true, shape.n, shape.k, ldqx, 128, BN);
    if (e != cudaSuccess) return e;
    return gemm::launch<true, BN, 1, false, false, ScaledAcross>(s, ma, mb, ma, shape, args);
}

}  // namespace

int quant_timeouts()
{
    int v = 0;
    if (cudaMemcpyFromSymbol(&v, g_quant_timeout, sizeof(int)) != cudaSuccess) return -1;
    return v;
}

// Whether that is expected to be the faster one, on a machine of 148 multiprocessors (either is right on any), of what each takes in us: from Python 11 for one launch and 14.3 for two; the class rows' bytes; and
// here the steps of a class row in one of 2,368 warps (16 bytes a lane are a load and four dot products a row, and every row's sum a reduction
// and a store), there the tiles' own time.  Measured for 1, 2, 3, 4 rows against two kernels: 65,536 classes x 1,024 15.2, 18.6, 23.7, 24.8
// against 18.3; 32,768 x 4,096 24, 28, 34, 35 against 28; 200,000 x 256 22, 29, 41, 45 against 20; 30,011 x 602 11.3, 11.3, 14.2, 14.7 against 14.3;
// 4,096 x 256 11 against 14.6.
bool few_rows_pays(int64_t n, int d, int m)
{
    if (n > kGemvMax || n * round_up(d, 16) > kGemvBytes) return false;
    const double bytes = (double)m * d, steps = (double)m * ((double)ceil_div(d, 512) * (4 * n + 6) + 12 * n);
    return std::max(11.0, 4.5 + std::max(bytes / 6.3e6, 2.5 + 3.7e-6 * steps)) <= std::max(14.3, 7.0 + std::max(bytes / 6.5e6, 6.4e-5 * m));
}
cudaError_t launch_few_rows_product(cudaStream_t s, const void* x, int type, int64_t ldx, int64_t n, int d, const int8_t* q_w, int64_t ldqw, const float* s_w, int m,
                                    void* out, int out_type, int64_t ldo, int* launches)
{
    const GemvArgs a = {x, type, ldx, (int)n, d, rows_whole(x, ldx, type, 4), q_w, ldqw, s_w, m, out, out_type, ldo};
    ++*launches;
    return n == 1 ? launch_few_rows<1>(s, a) : n == 2 ? launch_few_rows<2>(s, a) : launch_few_rows<4>(s, a);
}

bool quantized_across(int64_t n, int m) { return n <= 64 && m > 64; }

cudaError_t launch_quantize_rows(cudaStream_t s, const void* x, int type, int64_t n, int d, int64_t ldx, int8_t* q, int64_t ldq, float* scale, bool early, int* launches)
{
    const QuantArgs a = {x, type, ldx, n, d, rows_whole(x, ldx, type, 4), q, ldq, scale, early};
    if (!rows_whole(x, ldx, type, type == BIGCN_F32 ? 4 : 8)) return pick_quantize<kAnyType, 4>(s, a, launches);
    if (type == BIGCN_F32) return pick_quantize<BIGCN_F32, 4>(s, a, launches);
    if (type == BIGCN_BF16) return pick_quantize<BIGCN_BF16, 8>(s, a, launches);
    return pick_quantize<BIGCN_F16, 8>(s, a, launches);
}

cudaError_t launch_quantized_product(cudaStream_t s, const int8_t* q_x, int64_t ldqx, const float* s_x, int64_t n, int d, const int8_t* q_w, int64_t ldqw,
                                     const float* s_w, int m, void* out, int out_type, int64_t ldo, bool early, int tries, int* launches)
{
    const ScaledArgs args = {s_x, s_w, reinterpret_cast<uintptr_t>(s_w) % 16 == 0, out, out_type, ldo, rows_whole(out, ldo, out_type, 8)};
    gemm::Shape shape;
    shape.m = (int)n;
    shape.n = m;
    shape.k = d;
    shape.tries = tries;
    shape.rotate = n <= gemm::kRows;          // class rows are read once
    shape.tile_rows = gemm::rows_of_one_tile(n);
    ++*launches;
    if (quantized_across(n, m)) {
        shape.m = m;
        shape.n = (int)n;
        shape.a_ahead = early;
        // a height of the tiles with which the last round of the multiprocessors is full, or nearly so: a round costs its rows, and some 16 more
        int64_t least = INT64_MAX;
        for (int r = 128; r >= 64; r -= 8) {
            const int64_t cost = ceil_div(ceil_div(m, r), sm_count()) * (r + 16);
            if (cost < least) least = cost, shape.tile_rows = r;
        }
        if (n <= 32) return launch_across<32>(s, q_x, ldqx, q_w, ldqw, shape, args);
        return launch_across<64>(s, q_x, ldqx, q_w, ldqw, shape, args);
    }
    if (m <= 64) return launch_product_as<64, 1>(s, q_x, ldqx, q_w, ldqw, shape, args);
    if (m <= 128) return launch_product_as<128, 1>(s, q_x, ldqx, q_w, ldqw, shape, args);
    if (n > gemm::kRows) return launch_product_as<256, 2>(s, q_x, ldqx, q_w, ldqw, shape, args);
    return launch_product_as<256, 1>(s, q_x, ldqx, q_w, ldqw, shape, args);
}

}  // namespace bigcn
