// Rows in 8-bit integers and their product with 8-bit class rows.
//
//   s_i = max_j |x_ij| / 127,  q_ij = the integer nearest to 127 x_ij / max_j |x_ij| (halfway: the even one)
//   out_ik = (sum_j q_ij qw_kj) s_i sw_k
//
// The integers are exact: the sum of 16,384 products of 127 stays below 2^31.  The three roundings of an output (the sum to fp32, and
// two products) are fp32's, then one to the output's type.  The scales are multiplied first: a row with fp32's lowest value in it has a
// scale of 2^121, which times the sum would overflow where the output does not.
#include "dense_gemm.cuh"
#include "dense_types.cuh"

namespace bigcn {

namespace {

using namespace dense;

__device__ int g_quant_timeout;               // set when a wait ran out

struct QuantArgs {
    const void* x;
    int64_t ldx, n;
    int d;
    bool whole;
    int8_t* q;
    int64_t ldq;
    float* scale;
    bool early;              // the next kernel may start: it waits for this one where it reads what this one writes
};

// Four values as the integers nearest to 127 x / top, in the bytes of a word.  In fp32 the quotient is off by 127 * 3 * 2^-24 at
// most; where that could decide one of the roundings, they are taken in 64 bits, where 127 x is exact and a quotient halfway between integers
// cannot be met or missed by its rounding: with x and top of 24 bits it is halfway, or at least 2^-32 of its size away from it.  The sum with
// 1.5 * 2^23 rounds to the integer and holds it in its low bits.
__device__ __forceinline__ uint32_t nearest4(const float* x, float factor, float top, bool tiny)
{
    constexpr float kRound = 12582912.f;
    uint32_t n[4];
    float off = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float t = x[i] * factor, r = t + kRound;
        n[i] = __float_as_uint(r);
        off = fmaxf(off, fabsf(t - (r - kRound)));
    }
    if (tiny || off > 0.4999f) {
#pragma unroll
        for (int i = 0; i < 4; ++i) n[i] = (uint32_t)(int)rint(127.0 * (double)x[i] / (double)top);
    }
    return __byte_perm(__byte_perm(n[0], n[1], 0x0040), __byte_perm(n[2], n[3], 0x0040), 0x5410);
}

// One row to LANES threads (a warp or a block), V values at a time, NV times.
template <int TYPE, int V, int LANES, int NV>
__global__ void __launch_bounds__(LANES > 32 ? LANES : 256) quantize_kernel(const QuantArgs a)
{
    pdl_enter();
    if (a.early) asm volatile("griddepcontrol.launch_dependents;\n" ::: "memory");
    constexpr int B = LANES > 32 ? LANES : 256, GROUPS = B / LANES;
    __shared__ uint32_t slot[LANES > 32 ? LANES / 32 : 1];
    const int lane = threadIdx.x % LANES;
    const int64_t row = (int64_t)blockIdx.x * GROUPS + threadIdx.x / LANES;
    const auto* x = static_cast<const typename Elt<TYPE>::T*>(a.x) + row * a.ldx;
    float v[NV][V];
    uint32_t top = 0u;                        // as bits, which order magnitudes, infinity and NaN
#pragma unroll
    for (int k = 0; k < NV; ++k) {
        const int c = (k * LANES + lane) * V;
        load_elts<TYPE, V>(x + c, row < a.n ? a.d - c : 0, a.whole, v[k]);
#pragma unroll
        for (int i = 0; i < V; ++i) top = max(top, __float_as_uint(v[k][i]) & 0x7fffffffu);
    }
    top = __reduce_max_sync(0xffffffffu, top);
    if constexpr (LANES > 32) {
        if ((threadIdx.x & 31) == 0) slot[threadIdx.x >> 5] = top;
        __syncthreads();
        top = (threadIdx.x & 31) < LANES / 32 ? slot[threadIdx.x & 31] : 0u;
        top = __reduce_max_sync(0xffffffffu, top);
    }
    if (row >= a.n) return;
    const bool finite = top < 0x7f800000u;
    const float t = __uint_as_float(top), factor = 127.f / t;
    const bool tiny = t < 1e-30f;             // 127 / t would overflow
    if (lane == 0) a.scale[row] = finite ? t / 127.f : __uint_as_float(0x7fc00000u);
    int8_t* q = a.q + row * a.ldq;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
        const int c = (k * LANES + lane) * V;
        if (c >= a.d) break;
        uint32_t w[V / 4];
#pragma unroll
        for (int j = 0; j < V / 4; ++j) w[j] = finite && top ? nearest4(&v[k][4 * j], factor, t, tiny) : 0u;
        if (c + V <= a.d) {                   // rows of q start on 16-byte boundaries
            if constexpr (V == 4) *reinterpret_cast<uint32_t*>(q + c) = w[0];
            else *reinterpret_cast<uint2*>(q + c) = make_uint2(w[0], w[1]);
        } else {
#pragma unroll
            for (int i = 0; i < V; ++i)
                if (c + i < a.d) q[c + i] = (int8_t)(w[i >> 2] >> (8 * (i & 3)));
        }
    }
}

template <int TYPE, int V, int LANES, int NV>
cudaError_t launch_quantize_as(cudaStream_t s, const QuantArgs& a, int* launches)
{
    constexpr int B = LANES > 32 ? LANES : 256;
    ++*launches;
    return launch_kernel(quantize_kernel<TYPE, V, LANES, NV>, dim3((unsigned)ceil_div(a.n, B / LANES)), dim3(B), 0, s, a);
}
template <int TYPE, int V>
cudaError_t pick_quantize(cudaStream_t s, const QuantArgs& a, int* launches)
{
    constexpr int Q = 16 / V;
    const int64_t words = ceil_div(a.d, V);
    if (words <= 32) return launch_quantize_as<TYPE, V, 32, 1>(s, a, launches);
    if (words <= 64) return launch_quantize_as<TYPE, V, 32, 2>(s, a, launches);
    if (words <= 32 * Q) return launch_quantize_as<TYPE, V, 32, Q>(s, a, launches);
    if (words <= 128 * Q) return launch_quantize_as<TYPE, V, 128, Q>(s, a, launches);
    if (words <= 512 * Q) return launch_quantize_as<TYPE, V, 512, Q>(s, a, launches);
    return launch_quantize_as<TYPE, V, 1024, Q>(s, a, launches);
}

// Epilogue: the sums times both scales, in the output's type.
struct ScaledOut {
    struct Args {
        const float* s_x;
        const float* s_w;
        bool s_w_whole;
        void* out;
        int type;
        int64_t ldo;
        bool whole;          // rows of out on 16-byte boundaries
    };
    // 16 or 32 columns of a strip: 64 bytes of a row
    template <int TYPE>
    static __device__ __forceinline__ void write(const Args& a, const gemm::Part& p, int columns, int col, const float (&f)[32])
    {
        constexpr int kElts = 16 / type_bytes(TYPE), kStrips = type_bytes(TYPE) / 2;
        using T = typename Elt<TYPE>::T;
#pragma unroll
        for (int h = 0; h < kStrips; ++h) {
            uint32_t w[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                if constexpr (TYPE == BIGCN_F32) w[i] = __float_as_uint(f[16 * h + i]);
                else w[i] = pack2<TYPE>(f[2 * i], f[2 * i + 1]);
            }
            gemm::write_strip(p.strip, w, [&](int r, int piece, const uint4& v) {
                const int row = p.row + r, c = col + 16 * h + piece * kElts;
                if (row >= p.rows || c >= columns) return;
                T* to = static_cast<T*>(a.out) + (int64_t)row * a.ldo + c;
                if (a.whole && c + kElts <= columns) {
                    *reinterpret_cast<uint4*>(to) = v;
                } else {
                    const T* e = reinterpret_cast<const T*>(&v);
#pragma unroll
                    for (int i = 0; i < kElts; ++i)
                        if (c + i < columns) to[i] = e[i];
                }
            });
        }
    }
    static __device__ int* flag() { return &g_quant_timeout; }
    using Row = float;
    static __device__ __forceinline__ Row row(const Args& a, int row, int rows) { return row < rows ? __ldg(a.s_x + row) : 0.f; }
    template <int BN, class Done>
    static __device__ __forceinline__ void tile(const Args& a, const gemm::Shape& sh, const gemm::Unit&, const gemm::Part& p, const Row& sx, const Done& done)
    {
        const int lane = threadIdx.x & 31;
        // the warp's class scales are read by all lanes at once below: from L1 by then
        if (lane < gemm::part_cols(BN) / 32 && p.col + 32 * lane < sh.n) asm volatile("prefetch.global.L1 [%0];\n" ::"l"(a.s_w + p.col + 32 * lane));
        gemm::each_chunk<BN>(p, sh.n, done, [&](int c, uint32_t (&v)[32]) {
            const int col = p.col + c;
            float f[32];
            if (a.s_w_whole && col + 32 <= sh.n) {
#pragma unroll
                for (int i = 0; i < 32; i += 4) {
                    const float4 w = __ldg(reinterpret_cast<const float4*>(a.s_w + col + i));
                    f[i] = w.x; f[i + 1] = w.y; f[i + 2] = w.z; f[i + 3] = w.w;
                }
            } else {
#pragma unroll
                for (int i = 0; i < 32; ++i) f[i] = col + i < sh.n ? __ldg(a.s_w + col + i) : 0.f;
            }
#pragma unroll
            for (int i = 0; i < 32; ++i) f[i] = (float)(int)v[i] * (sx * f[i]);
            if (a.type == BIGCN_F32) write<BIGCN_F32>(a, p, sh.n, col, f);
            else if (a.type == BIGCN_BF16) write<BIGCN_BF16>(a, p, sh.n, col, f);
            else write<BIGCN_F16>(a, p, sh.n, col, f);
        });
    }
};

// The same with classes as rows of the tiles and the few rows of x as columns: a lane has a class, so that 32 neighbours of an output row
// are stored together, and 128 class rows to a tile leave more tiles than 256 columns would.
struct ScaledAcross {
    using Args = ScaledOut::Args;
    static __device__ int* flag() { return &g_quant_timeout; }
    using Row = float;
    static __device__ __forceinline__ Row row(const Args& a, int row, int rows) { return row < rows ? __ldg(a.s_w + row) : 0.f; }
    template <int BN, class Done>
    static __device__ __forceinline__ void tile(const Args& a, const gemm::Shape& sh, const gemm::Unit&, const gemm::Part& p, const Row& sw, const Done& done)
    {
        const int k = p.row + (threadIdx.x & 31);
        gemm::each_chunk<BN>(p, sh.n, done, [&](int c, uint32_t (&v)[32]) {
            if (k >= p.rows) return;
#pragma unroll
            for (int i = 0; i < 32; ++i) {
                const int row = p.col + c + i;
                if (row >= sh.n) break;
                const float f[1] = {(float)(int)v[i] * (__ldg(a.s_x + row) * sw)};
                store_as<1>(a.out, a.type, (int64_t)row * a.ldo + k, 1, true, f);
            }
        });
    }
};

template <int BN, int CTAS>
cudaError_t launch_product_as(cudaStream_t s, const int8_t* q_x, int64_t ldqx, const int8_t* q_w, int64_t ldqw, const gemm::Shape& shape, const ScaledOut::Args& args)
{
    CUtensorMap ma, mb;
    cudaError_t e = gemm::encode_map(&ma, q_x, 1, true, shape.m, shape.k, ldqx, 128, gemm::kRows);
    if (e == cudaSuccess) e = gemm::encode_map(&mb, q_w, 1, true, shape.n, shape.k, ldqw, 128, BN / CTAS);
    if (e != cudaSuccess) return e;
    return gemm::launch<true, BN, CTAS, false, false, ScaledOut>(s, ma, mb, ma, shape, args);
}

template <int BN>
cudaError_t launch_across(cudaStream_t s, const int8_t* q_x, int64_t ldqx, const int8_t* q_w, int64_t ldqw, const gemm::Shape& shape, const ScaledOut::Args& args)
{
    CUtensorMap ma, mb;
    cudaError_t e = gemm::encode_map(&ma, q_w, 1, true, shape.m, shape.k, ldqw, 128, gemm::kRows);
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

bool quantized_across(int64_t n, int m) { return n <= 64 && m > 64; }

cudaError_t launch_quantize_rows(cudaStream_t s, const void* x, int type, int64_t n, int d, int64_t ldx, int8_t* q, int64_t ldq, float* scale, bool early, int* launches)
{
    const QuantArgs a = {x, ldx, n, d, rows_whole(x, ldx, type, type == BIGCN_F32 ? 4 : 8), q, ldq, scale, early};
    if (type == BIGCN_F32) return pick_quantize<BIGCN_F32, 4>(s, a, launches);
    if (type == BIGCN_BF16) return pick_quantize<BIGCN_BF16, 8>(s, a, launches);
    return pick_quantize<BIGCN_F16, 8>(s, a, launches);
}

cudaError_t launch_quantized_product(cudaStream_t s, const int8_t* q_x, int64_t ldqx, const float* s_x, int64_t n, int d, const int8_t* q_w, int64_t ldqw,
                                     const float* s_w, int m, void* out, int out_type, int64_t ldo, bool early, int* launches)
{
    const ScaledOut::Args args = {s_x, s_w, reinterpret_cast<uintptr_t>(s_w) % 16 == 0, out, out_type, ldo, rows_whole(out, ldo, out_type, 8)};
    gemm::Shape shape;
    shape.m = (int)n;
    shape.n = m;
    shape.k = d;
    ++*launches;
    if (quantized_across(n, m)) {
        shape.m = m;
        shape.n = (int)n;
        shape.a_ahead = early;
        return launch_across<64>(s, q_x, ldqx, q_w, ldqw, shape, args);
    }
    if (m <= 64) return launch_product_as<64, 1>(s, q_x, ldqx, q_w, ldqw, shape, args);
    if (m <= 128) return launch_product_as<128, 1>(s, q_x, ldqx, q_w, ldqw, shape, args);
    if (n > gemm::kRows) return launch_product_as<256, 2>(s, q_x, ldqx, q_w, ldqw, shape, args);
    return launch_product_as<256, 1>(s, q_x, ldqx, q_w, ldqw, shape, args);
}

}  // namespace bigcn
