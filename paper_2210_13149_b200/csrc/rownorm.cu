// Layer norm of rows and its gradients.
//
//   y_ij = xhat_ij gain_j + offset_j,  xhat_ij = (x_ij - mean_i) rstd_i,  rstd_i = 1 / sqrt(var_i + eps)
//   g_x_ij = rstd_i (g_ij gain_j - a_i - xhat_ij b_i),  a_i = sum_j g_ij gain_j / d,  b_i = sum_j g_ij gain_j xhat_ij / d
//   g_gain_j = sum_i g_ij xhat_ij,  g_offset_j = sum_i g_ij                        (g = the gradient of y)
//
// Both directions are bound by the bytes of the rows where these are long (fp32 rows of 256: 85 to 97 % of a plain copy's rate), by latency and instructions where a
// lane has little of a row (bf16 rows of 24: 44 and 51 %, of 23: 20 and 18 %) or holds much of it in registers (500 columns back: 65 %).  A row is held in the registers of the lanes that read it (4 to 32 lanes of a
// warp, or a whole block for long rows), so that it is read once: the mean first, then the squares about it, which lose nothing to
// cancellation.  The columns' sums of the backward pass ride along in registers, one pair per column a thread owns, over the rows that
// its lanes take; blocks leave theirs in the workspace, and a second kernel adds them in 64 bits in a fixed order.
//
// Lanes read words of 16 bytes where the rows they read start on their boundaries, and otherwise words of 4, 2 or 1 elements, whichever the rows
// allow (the backward pass, with two types to read, then looks them up); they store what the output's rows allow.
#include <algorithm>
#include <cfloat>

#include "dense_types.cuh"

namespace bigcn {

namespace {

using namespace dense;

constexpr int kThreads = 256;

// Sum over the LANES threads of a group; every thread gets it.  `slot`: for groups of several warps (the whole block), two sets of
// words that calls alternate between.
template <int LANES, int COUNT>
__device__ __forceinline__ void group_sum(float (&v)[COUNT], float* slot)
{
#pragma unroll
    for (int m = (LANES < 32 ? LANES : 32) / 2; m >= 1; m >>= 1)
#pragma unroll
        for (int c = 0; c < COUNT; ++c) v[c] += __shfl_xor_sync(0xffffffffu, v[c], m);
    if constexpr (LANES > 32) {
        constexpr int W = LANES / 32;
        const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
        if (lane == 0)
#pragma unroll
            for (int c = 0; c < COUNT; ++c) slot[c * W + warp] = v[c];
        __syncthreads();
#pragma unroll
        for (int c = 0; c < COUNT; ++c) {
            float s = lane < W ? slot[c * W + lane] : 0.f;
#pragma unroll
            for (int m = 16; m >= 1; m >>= 1) s += __shfl_xor_sync(0xffffffffu, s, m);
            v[c] = s;
        }
    }
}

// The columns' factors of a kernel whose threads own more than 8 columns each: in shared memory, `none` past d and where there are none.  Words of
// 8 columns lie as two halves `padded` / 2 apart, so that lanes read 16 bytes next to each other.
template <int V>
__device__ __forceinline__ void stage_columns(float* to, const float* p, float none, int d, int padded)
{
    for (int c = threadIdx.x; c < padded; c += blockDim.x)
        to[V == 8 ? (c >> 2 & 1) * (padded / 2) + (c >> 3) * 4 + (c & 3) : c] = c < d && p ? __ldg(p + c) : none;
}
template <int V>
__device__ __forceinline__ void staged(const float* from, int c, int padded, float (&v)[V])
{
    if constexpr (V % 4 == 0) {
#pragma unroll
        for (int i = 0; i < V; i += 4) {
            const float4 q = *reinterpret_cast<const float4*>(from + (V == 8 ? i / 4 * (padded / 2) + (c >> 3) * 4 : c));
            v[i] = q.x; v[i + 1] = q.y; v[i + 2] = q.z; v[i + 3] = q.w;
        }
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = from[c + i];
    }
}

struct NormArgs {
    const void* x;
    int x_type;
    int64_t ldx;
    int64_t n;
    int d;
    int y_step;              // elements of y that can be stored at a time
    const float* gain;       // nullable: 1
    const float* offset;     // nullable: 0
    float eps;
    void* y;
    int y_type;
    int64_t ldy;
    float* mean;
    float* rstd;
};

// Rows of a lane's words on their way at a time, of what a row takes in registers: 32 warps of a multiprocessor with 12 registers each on their way are
// 48 KB, which covers a latency of a microsecond at the memory's rate (1,362,217 bf16 rows of 23 columns in us: 110 with one row that is converted where it is loaded, 95 so).
__host__ __device__ constexpr int rows_ahead(int registers) { return registers <= 2 ? 4 : registers <= 4 ? 3 : 1; }

// Blocks of the forward pass on a multiprocessor: 1,024 threads with 64 registers each, rows going round in all of them.
constexpr int norm_blocks(int lanes) { return lanes > 32 ? 1024 / lanes : 1024 / kThreads; }

template <int TYPE, int V, int LANES, int NV>
__global__ void __launch_bounds__(LANES > 32 ? LANES : kThreads, norm_blocks(LANES)) norm_kernel(const NormArgs a)
{
    pdl_enter();
    constexpr int B = LANES > 32 ? LANES : kThreads, GROUPS = B / LANES;
    constexpr bool kHold = NV * V <= 8;          // gain and offset stay in registers over the rows
    constexpr int kAhead = rows_ahead(NV * Raw<TYPE, V>::kWords);
    extern __shared__ __align__(16) float dyn[];  // else [2][LANES V NV]
    __shared__ float slots[2][LANES > 32 ? LANES / 32 : 1];
    const int lane = threadIdx.x % LANES;
    const float inv_d = 1.f / (float)a.d;
    float gain[kHold ? NV * V : 1], offset[kHold ? NV * V : 1];
    if constexpr (kHold) {
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const int c = (k * LANES + lane) * V + i;
                gain[k * V + i] = c < a.d && a.gain ? __ldg(a.gain + c) : 1.f;
                offset[k * V + i] = c < a.d && a.offset ? __ldg(a.offset + c) : 0.f;
            }
    } else {
        stage_columns<V>(dyn, a.gain, 1.f, a.d, LANES * V * NV);
        stage_columns<V>(dyn + LANES * V * NV, a.offset, 0.f, a.d, LANES * V * NV);
        __syncthreads();
    }
    const int64_t step = (int64_t)gridDim.x * GROUPS;
    int64_t row = (int64_t)blockIdx.x * GROUPS + threadIdx.x / LANES;
    Raw<TYPE, V> next[kAhead][NV];               // the rows after this one are on their way while this one is worked on
    auto fetch = [&](int64_t r, Raw<TYPE, V> (&to)[NV]) {
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int c = (k * LANES + lane) * V;
            to[k].load(a.x, a.x_type, r * a.ldx + c, r < a.n ? a.d - c : 0);
        }
    };
#pragma unroll
    for (int j = 0; j < kAhead; ++j) fetch(row + j * step, next[j]);
    for (int64_t base = (int64_t)blockIdx.x * GROUPS; base < a.n;)   // the same trips for all threads of a block
#pragma unroll
    for (int j = 0; j < kAhead; ++j, base += step, row += step) {
        if (kAhead > 1 && base >= a.n) break;
        float v[NV][V], sum[1] = {0.f};
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            next[j][k].values(v[k], a.x_type);
#pragma unroll
            for (int i = 0; i < V; ++i) sum[0] += v[k][i];
        }
        fetch(row + kAhead * step, next[j]);
        group_sum<LANES, 1>(sum, slots[0]);
        const float mu = sum[0] * inv_d;
        float sq[1] = {0.f};
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
            for (int i = 0; i < V; ++i) {
                v[k][i] = (k * LANES + lane) * V + i < a.d ? v[k][i] - mu : 0.f;
                sq[0] = fmaf(v[k][i], v[k][i], sq[0]);
            }
        group_sum<LANES, 1>(sq, slots[1]);
        const float r = 1.f / sqrtf(fmaf(sq[0], inv_d, a.eps));
        if (row < a.n) {
            if (lane == 0) {
                a.mean[row] = mu;
                a.rstd[row] = r;
            }
#pragma unroll
            for (int k = 0; k < NV; ++k) {
                const int c = (k * LANES + lane) * V;
                float g[V], o[V];
                if constexpr (kHold) {
#pragma unroll
                    for (int i = 0; i < V; ++i) g[i] = gain[k * V + i], o[i] = offset[k * V + i];
                } else {
                    staged<V>(dyn, c, LANES * V * NV, g);
                    staged<V>(dyn + LANES * V * NV, c, LANES * V * NV, o);
                }
#pragma unroll
                for (int i = 0; i < V; ++i) v[k][i] = fmaf(v[k][i] * r, g[i], o[i]);
            }
            store_row<NV, V>(a.y, a.y_type, row * a.ldy, lane * V, LANES * V, a.d, a.y_step, v);
        }
    }
}

struct NormBackArgs {
    const void* g;
    int g_type;
    int64_t ldg;
    const void* x;
    int x_type;
    int64_t ldx;
    int64_t n;
    int d;
    int gx_step;             // elements of g_x that can be stored at a time
    const float* gain;
    const float* mean;
    const float* rstd;
    void* gx;
    int gx_type;
    int64_t ldgx;
    float* part;             // [blocks][2][d]: the columns' sums of every block (null: not wanted)
};

// How a block of the backward pass is laid out.  Its rows come through a ring in shared memory, copied kRing - 1 rows ahead into places
// that only the thread itself reads, so that nothing but its own copies is waited for: registers hold one row of 16 to 64 bytes ahead and
// no more (89,250 bf16 rows of 500 columns in us: 102 with one row ahead in registers, 66 with two in the ring).
template <int GTYPE, int TYPE, int V, int LANES, int NV>
struct BackLayout {
    static constexpr int B = LANES > 32 ? LANES : kThreads;
    static constexpr bool kHold = NV * V <= 8;          // the gain stays in registers, else in shared memory
    static constexpr bool kShared = LANES >= 1024;      // no registers left for the columns' sums: each thread keeps its own in shared memory
    static constexpr bool kTyped = TYPE >= 0 && GTYPE >= 0;
    static constexpr int kRowBytes = NV * 4 * (Raw<GTYPE, V>::kWords + Raw<TYPE, V>::kWords);      // of a thread
    static constexpr int kRing = !kTyped || kShared ? 0 : LANES >= 512 ? 2 : NV * V > 8 ? 3 : 4;
    static constexpr int kBlocks = LANES >= 512 ? 1 : LANES > 32 ? 512 / LANES : kHold ? 3 : 2;    // a multiprocessor, by their registers
    static constexpr int kAhead = kRing || LANES > 32 ? 0 : kRowBytes <= 16 ? 4 : kRowBytes <= 32 ? 2 : 1;    // else: rows of them on their way in registers
    static constexpr int kRingBytes = kRing * kRowBytes * B;
    static size_t smem(int d) { return kRingBytes + (size_t)(kHold ? 0 : LANES * V * NV) * 4 + (LANES > 32 && !kShared ? 0 : (size_t)2 * d * 4); }
};

template <int GTYPE, int TYPE, int V, int LANES, int NV>
__global__ void __launch_bounds__(LANES > 32 ? LANES : kThreads, BackLayout<GTYPE, TYPE, V, LANES, NV>::kBlocks) norm_backward_kernel(const NormBackArgs a)
{
    pdl_enter();
    using L = BackLayout<GTYPE, TYPE, V, LANES, NV>;
    constexpr int B = L::B, GROUPS = B / LANES, kRing = L::kRing;
    constexpr bool kHold = L::kHold, kShared = L::kShared;
    constexpr int kAhead = L::kAhead, kHeld = kAhead > 0 ? kAhead : 1;
    extern __shared__ __align__(16) unsigned char raw[];       // the ring, the gain, [2][d] for the block's sums
    float* const gains = reinterpret_cast<float*>(raw + L::kRingBytes);
    float* const dyn = gains + (kHold ? 0 : LANES * V * NV);
    __shared__ float slots[2][LANES > 32 ? 2 * (LANES / 32) : 1];
    const int lane = threadIdx.x % LANES;
    const float inv_d = 1.f / (float)a.d;
    float gain[kHold ? NV * V : 1], dgain[kShared ? 1 : NV * V], doff[kShared ? 1 : NV * V];
    if constexpr (kHold) {
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const int c = (k * LANES + lane) * V + i;
                gain[k * V + i] = c < a.d && a.gain ? __ldg(a.gain + c) : 1.f;
            }
    } else {
        stage_columns<V>(gains, a.gain, 1.f, a.d, LANES * V * NV);
    }
    if constexpr (!kShared) {
#pragma unroll
        for (int k = 0; k < NV * V; ++k) dgain[k] = 0.f, doff[k] = 0.f;
    } else {
        for (int c = threadIdx.x; c < 2 * a.d; c += B) dyn[c] = 0.f;
    }
    if constexpr (!kHold || kShared) __syncthreads();
    const int64_t step = (int64_t)gridDim.x * GROUPS;
    int64_t row = (int64_t)blockIdx.x * GROUPS + threadIdx.x / LANES;
    Raw<TYPE, V> nx[kHeld][NV];
    Raw<GTYPE, V> ng[kHeld][NV];
    float nmean[kHeld], nrstd[kHeld];
    auto fetch = [&](int64_t r, int j) {
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int c = (k * LANES + lane) * V;
            nx[j][k].load(a.x, a.x_type, r * a.ldx + c, r < a.n ? a.d - c : 0);
            ng[j][k].load(a.g, a.g_type, r * a.ldg + c, r < a.n ? a.d - c : 0);
        }
        nmean[j] = r < a.n ? __ldg(a.mean + r) : 0.f;
        nrstd[j] = r < a.n ? __ldg(a.rstd + r) : 0.f;
    };
    // a thread's place in a slot of the ring: its words of x, then of g, 16-byte pieces B threads apart
    constexpr int kXBytes = Raw<TYPE, V>::kWords * 4, kGBytes = Raw<GTYPE, V>::kWords * 4;
    auto place = [&](int slot, int k, bool of_g) {
        return raw + (size_t)slot * L::kRowBytes * B + (of_g ? (size_t)NV * kXBytes * B + ((size_t)k * B + threadIdx.x) * kGBytes : ((size_t)k * B + threadIdx.x) * kXBytes);
    };
    // what a lane copies of a row is the same for all rows; its place in the matrices moves on by a constant
    int64_t sent = row;
    const typename Elt<(kRing > 0 ? TYPE : 0)>::T* from_x = static_cast<const typename Elt<(kRing > 0 ? TYPE : 0)>::T*>(a.x) + row * a.ldx + lane * V;
    const typename Elt<(kRing > 0 ? GTYPE : 0)>::T* from_g = static_cast<const typename Elt<(kRing > 0 ? GTYPE : 0)>::T*>(a.g) + row * a.ldg + lane * V;
    auto send = [&](int slot) {
        if constexpr (kRing > 0) {
            const bool live = sent < a.n;
#pragma unroll
            for (int k = 0; k < NV; ++k) {
                const int there = a.d - (k * LANES + lane) * V, count = live ? max(0, min(there, V)) : 0;
                Raw<TYPE, V>::copy_to(place(slot, k, false), count > 0 ? from_x + k * LANES * V : static_cast<const typename Elt<TYPE>::T*>(a.x), count);
                Raw<GTYPE, V>::copy_to(place(slot, k, true), count > 0 ? from_g + k * LANES * V : static_cast<const typename Elt<GTYPE>::T*>(a.g), count);
            }
            asm volatile("cp.async.commit_group;\n" ::: "memory");
            sent += step;
            from_x += step * a.ldx;
            from_g += step * a.ldg;
        }
    };
    int slot = 0;
    if constexpr (kRing > 0) {
#pragma unroll
        for (int i = 0; i < kRing - 1; ++i) send(i);
        nmean[0] = row < a.n ? __ldg(a.mean + row) : 0.f;
        nrstd[0] = row < a.n ? __ldg(a.rstd + row) : 0.f;
    }
#pragma unroll
    for (int j = 0; j < kAhead; ++j) fetch(row + j * step, j);
    int trip = 0;
    for (int64_t base = (int64_t)blockIdx.x * GROUPS; base < a.n;)
#pragma unroll
    for (int j = 0; j < kHeld; ++j, base += step, row += step, ++trip) {
        if (kHeld > 1 && base >= a.n) break;
        float xh[NV][V], gv[NV][V], sums[2] = {0.f, 0.f};
        if constexpr (kRing > 0) {
            send(slot == 0 ? kRing - 1 : slot - 1);
            asm volatile("cp.async.wait_group %0;\n" ::"n"(kRing > 0 ? kRing - 1 : 0) : "memory");
#pragma unroll
            for (int k = 0; k < NV; ++k) {
                nx[j][k].take(place(slot, k, false));
                ng[j][k].take(place(slot, k, true));
            }
            if (++slot == kRing) slot = 0;
        } else if constexpr (kAhead == 0) {
            fetch(row, j);
        }
        const float mu = nmean[j], r = nrstd[j];
        if constexpr (kRing > 0) {
            nmean[0] = row + step < a.n ? __ldg(a.mean + row + step) : 0.f;
            nrstd[0] = row + step < a.n ? __ldg(a.rstd + row + step) : 0.f;
        }
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            nx[j][k].values(xh[k], a.x_type);
            ng[j][k].values(gv[k], a.g_type);
        }
        if constexpr (kAhead > 0) fetch(row + kAhead * step, j);
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int c = (k * LANES + lane) * V;
            float w[V];
            if constexpr (kHold) {
#pragma unroll
                for (int i = 0; i < V; ++i) w[i] = gain[k * V + i];
            } else {
                staged<V>(gains, c, LANES * V * NV, w);
            }
#pragma unroll
            for (int i = 0; i < V; ++i) {
                // (where there is no element x and g are 0: its xhat adds nothing while it is a number, and nothing is kept of it)
                xh[k][i] = (xh[k][i] - mu) * r;
                const float gi = gv[k][i];
                if constexpr (kShared) {
                    if (row < a.n && c + i < a.d) {
                        dyn[c + i] = fmaf(gi, xh[k][i], dyn[c + i]);
                        dyn[a.d + c + i] += gi;
                    }
                } else {
                    dgain[k * V + i] = fmaf(gi, xh[k][i], dgain[k * V + i]);
                    doff[k * V + i] += gi;
                }
                gv[k][i] = gi * w[i];
                sums[0] += gv[k][i];
                sums[1] = fmaf(gv[k][i], xh[k][i], sums[1]);
            }
        }
        if (!(fabsf(mu * r) <= FLT_MAX)) {       // 0 - mean, times rstd, is no number then: the sum of what is there
            sums[1] = 0.f;
#pragma unroll
            for (int k = 0; k < NV; ++k)
#pragma unroll
                for (int i = 0; i < V; ++i)
                    if ((k * LANES + lane) * V + i < a.d) sums[1] = fmaf(gv[k][i], xh[k][i], sums[1]);
        }
        group_sum<LANES, 2>(sums, slots[trip & 1]);
        if (row < a.n) {
            const float sa = sums[0] * inv_d * r, sb = sums[1] * inv_d * r;
#pragma unroll
            for (int k = 0; k < NV; ++k)
#pragma unroll
                for (int i = 0; i < V; ++i) gv[k][i] = fmaf(-xh[k][i], sb, fmaf(gv[k][i], r, -sa));
            store_row<NV, V>(a.gx, a.gx_type, row * a.ldgx, lane * V, LANES * V, a.d, a.gx_step, gv);
        }
    }
    if (!a.part) return;
    float* out = a.part + (int64_t)blockIdx.x * 2 * a.d;
    if constexpr (kShared) {
        __syncthreads();
        for (int c = threadIdx.x; c < 2 * a.d; c += B) out[c] = dyn[c];
    } else if constexpr (LANES > 32) {
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const int c = (k * LANES + lane) * V + i;
                if (c < a.d) {
                    out[c] = dgain[k * V + i];
                    out[a.d + c] = doff[k * V + i];
                }
            }
    } else {
        // the groups of a warp first, then the warps one after the other
#pragma unroll
        for (int m = LANES; m < 32; m <<= 1)
#pragma unroll
            for (int k = 0; k < NV * V; ++k) {
                dgain[k] += __shfl_xor_sync(0xffffffffu, dgain[k], m);
                doff[k] += __shfl_xor_sync(0xffffffffu, doff[k], m);
            }
        for (int w = 0; w < B / 32; ++w) {
            if ((int)(threadIdx.x >> 5) == w && (threadIdx.x & 31) < LANES) {
#pragma unroll
                for (int k = 0; k < NV; ++k)
#pragma unroll
                    for (int i = 0; i < V; ++i) {
                        const int c = (k * LANES + lane) * V + i;
                        if (c < a.d) {
                            dyn[c] = w ? dyn[c] + dgain[k * V + i] : dgain[k * V + i];
                            dyn[a.d + c] = w ? dyn[a.d + c] + doff[k * V + i] : doff[k * V + i];
                        }
                    }
            }
            __syncthreads();
        }
        for (int c = threadIdx.x; c < 2 * a.d; c += B) out[c] = dyn[c];
    }
}

// out[c] = sum over the parts of part[b][c], in 64 bits: 32 columns to a block, its 32 warps take every 32nd part.
__global__ void __launch_bounds__(1024) column_sums_kernel(const float* __restrict__ part, int parts, int d, float* __restrict__ g_gain, float* __restrict__ g_offset)
{
    pdl_enter();
    __shared__ double s[32][33];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, c = blockIdx.x * 32 + lane;
    double v = 0.0;
    if (c < 2 * d)
        for (int b = warp; b < parts; b += 32) v += (double)__ldg(part + (int64_t)b * 2 * d + c);
    s[warp][lane] = v;
    __syncthreads();
    v = s[lane][warp];                           // a warp to a column
#pragma unroll
    for (int m = 16; m >= 1; m >>= 1) v += __shfl_xor_sync(0xffffffffu, v, m);
    const int col = blockIdx.x * 32 + warp;
    if (lane == 0 && col < 2 * d) {
        float* out = col < d ? g_gain : g_offset;
        if (out) out[col < d ? col : col - d] = (float)v;
    }
}

// Blocks of the backward pass: `each` for every multiprocessor, or as many as there are rows.
constexpr int kMaxParts = 512;
int backward_blocks(int64_t n, int groups, int each)
{
    return (int)std::min<int64_t>(ceil_div(n, groups), std::min(kMaxParts, each * sm_count()));
}

template <int TYPE, int V, int LANES, int NV>
cudaError_t launch_norm(cudaStream_t s, const NormArgs& a, int* launches)
{
    constexpr int B = LANES > 32 ? LANES : kThreads;
    const int64_t blocks = std::min<int64_t>(ceil_div(a.n, B / LANES), (int64_t)sm_count() * norm_blocks(LANES));
    auto* kernel = norm_kernel<TYPE, V, LANES, NV>;
    constexpr size_t smem = NV * V <= 8 ? 0 : (size_t)2 * LANES * V * NV * sizeof(float);
    static std::atomic<uint64_t> ready{0};     // by device
    const cudaError_t e = allow_shared(kernel, smem, &ready);
    if (e != cudaSuccess) return e;
    ++*launches;
    return launch_kernel(kernel, dim3((unsigned)blocks), dim3(B), smem, s, a);
}

template <int TYPE, int V>
cudaError_t pick_norm(cudaStream_t s, const NormArgs& a, int* launches)
{
    const int64_t words = ceil_div(a.d, V);
    constexpr int Q = 16 / V;                    // words per lane of the longer forms: 16 values
    if (words <= 4) return launch_norm<TYPE, V, 4, 1>(s, a, launches);
    if (words <= 8) return launch_norm<TYPE, V, 8, 1>(s, a, launches);
    if (words <= 16) return launch_norm<TYPE, V, 16, 1>(s, a, launches);
    if (words <= 32) return launch_norm<TYPE, V, 32, 1>(s, a, launches);
    if (words <= 64) return launch_norm<TYPE, V, 32, 2>(s, a, launches);
    if (words <= 32 * Q) return launch_norm<TYPE, V, 32, Q>(s, a, launches);
    if (words <= 128 * Q / 2) return launch_norm<TYPE, V, 128, Q / 2>(s, a, launches);
    if (words <= 128 * Q) return launch_norm<TYPE, V, 128, Q>(s, a, launches);
    if (words <= 256 * Q) return launch_norm<TYPE, V, 256, Q>(s, a, launches);
    if (words <= 512 * Q) return launch_norm<TYPE, V, 512, Q>(s, a, launches);
    return launch_norm<TYPE, V, 1024, Q>(s, a, launches);
}

// Rows off 16-byte boundaries, in words of V elements.
template <int TYPE, int V>
cudaError_t pick_norm_off(cudaStream_t s, const NormArgs& a, int* launches)
{
    constexpr int Q = 16 / V;
    if (a.d <= 16) return launch_norm<TYPE, V, 8, 2 / (V < 2 ? V : 2)>(s, a, launches);
    if (a.d <= 32) return launch_norm<TYPE, V, 16, 2 / (V < 2 ? V : 2)>(s, a, launches);
    if (a.d <= 64) return launch_norm<TYPE, V, 32, 2 / (V < 2 ? V : 2)>(s, a, launches);
    if (a.d <= 128) return launch_norm<TYPE, V, 32, 4 / V>(s, a, launches);
    if (a.d <= 256) return launch_norm<TYPE, V, 32, 8 / V>(s, a, launches);
    if (a.d <= 512) return launch_norm<TYPE, V, 32, Q>(s, a, launches);
    if (a.d <= 1024) return launch_norm<TYPE, V, 128, Q / 2>(s, a, launches);
    if (a.d <= 2048) return launch_norm<TYPE, V, 128, Q>(s, a, launches);
    if (a.d <= 4096) return launch_norm<TYPE, V, 512, Q / 2>(s, a, launches);
    if (a.d <= 8192) return launch_norm<TYPE, V, 512, Q>(s, a, launches);
    return launch_norm<TYPE, V, 1024, Q>(s, a, launches);
}
template <int TYPE>
cudaError_t pick_norm_step(cudaStream_t s, int step, const NormArgs& a, int* launches)
{
    if constexpr (TYPE != BIGCN_F32)
        if (step >= 4) return pick_norm_off<TYPE, 4>(s, a, launches);
    if (step >= 2) return pick_norm_off<TYPE, 2>(s, a, launches);
    return pick_norm_off<TYPE, 1>(s, a, launches);
}

template <int GTYPE, int TYPE, int V, int LANES, int NV>
cudaError_t launch_back(cudaStream_t s, const NormBackArgs& a, float* g_gain, float* g_offset, int* launches)
{
    using L = BackLayout<GTYPE, TYPE, V, LANES, NV>;
    constexpr int B = L::B;
    const size_t smem = L::smem(a.d);
    const int blocks = backward_blocks(a.n, B / LANES, std::max(1, std::min(L::kBlocks, (int)(227 * 1024 / (smem + 1024)))));
    auto* kernel = norm_backward_kernel<GTYPE, TYPE, V, LANES, NV>;
    static std::atomic<uint64_t> ready{0};     // by device
    cudaError_t e = allow_shared(kernel, smem, &ready);
    if (e != cudaSuccess) return e;
    ++*launches;
    e = launch_kernel(kernel, dim3((unsigned)blocks), dim3(B), smem, s, a);
    if (e == cudaSuccess && a.part) {
        ++*launches;
        e = launch_kernel(column_sums_kernel, dim3((unsigned)ceil_div(2 * a.d, 32)), dim3(1024), 0, s, (const float*)a.part, blocks, a.d, g_gain, g_offset);
    }
    return e;
}

template <int GTYPE, int TYPE>
cudaError_t pick_back(cudaStream_t s, const NormBackArgs& a, float* g_gain, float* g_offset, int* launches)
{
    constexpr int V = TYPE == BIGCN_F32 || GTYPE == BIGCN_F32 ? 4 : 8;
    constexpr int Q = 16 / V;
    const int64_t words = ceil_div(a.d, V);
    if (words <= 4) return launch_back<GTYPE, TYPE, V, 4, 1>(s, a, g_gain, g_offset, launches);
    if (words <= 8) return launch_back<GTYPE, TYPE, V, 8, 1>(s, a, g_gain, g_offset, launches);
    if (words <= 16) return launch_back<GTYPE, TYPE, V, 16, 1>(s, a, g_gain, g_offset, launches);
    if (words <= 32) return launch_back<GTYPE, TYPE, V, 32, 1>(s, a, g_gain, g_offset, launches);
    if (words <= 64) return launch_back<GTYPE, TYPE, V, 32, 2>(s, a, g_gain, g_offset, launches);
    if (words <= 32 * Q) return launch_back<GTYPE, TYPE, V, 32, Q>(s, a, g_gain, g_offset, launches);
    if (words <= 128 * Q / 2) return launch_back<GTYPE, TYPE, V, 128, Q / 2>(s, a, g_gain, g_offset, launches);
    if (words <= 128 * Q) return launch_back<GTYPE, TYPE, V, 128, Q>(s, a, g_gain, g_offset, launches);
    if (words <= 256 * Q) return launch_back<GTYPE, TYPE, V, 256, Q>(s, a, g_gain, g_offset, launches);
    if (words <= 512 * Q) return launch_back<GTYPE, TYPE, V, 512, Q>(s, a, g_gain, g_offset, launches);
    return launch_back<GTYPE, TYPE, V, 1024, Q>(s, a, g_gain, g_offset, launches);
}

template <int V>
cudaError_t pick_back_off(cudaStream_t s, const NormBackArgs& a, float* g_gain, float* g_offset, int* launches)
{
    constexpr int Q = 16 / V, T = kAnyType;
    if (a.d <= 16) return launch_back<T, T, V, 8, 2 / (V < 2 ? V : 2)>(s, a, g_gain, g_offset, launches);
    if (a.d <= 32) return launch_back<T, T, V, 16, 2 / (V < 2 ? V : 2)>(s, a, g_gain, g_offset, launches);
    if (a.d <= 64) return launch_back<T, T, V, 32, 2 / (V < 2 ? V : 2)>(s, a, g_gain, g_offset, launches);
    if (a.d <= 128) return launch_back<T, T, V, 32, 4 / V>(s, a, g_gain, g_offset, launches);
    if (a.d <= 256) return launch_back<T, T, V, 32, 8 / V>(s, a, g_gain, g_offset, launches);
    if (a.d <= 512) return launch_back<T, T, V, 32, Q>(s, a, g_gain, g_offset, launches);
    if (a.d <= 1024) return launch_back<T, T, V, 128, Q / 2>(s, a, g_gain, g_offset, launches);
    if (a.d <= 2048) return launch_back<T, T, V, 128, Q>(s, a, g_gain, g_offset, launches);
    if (a.d <= 4096) return launch_back<T, T, V, 512, Q / 2>(s, a, g_gain, g_offset, launches);
    if (a.d <= 8192) return launch_back<T, T, V, 512, Q>(s, a, g_gain, g_offset, launches);
    return launch_back<T, T, V, 1024, Q>(s, a, g_gain, g_offset, launches);
}

template <int GTYPE>
cudaError_t pick_back_x(cudaStream_t s, int x_type, const NormBackArgs& a, float* g_gain, float* g_offset, int* launches)
{
    if (x_type == BIGCN_F32) return pick_back<GTYPE, BIGCN_F32>(s, a, g_gain, g_offset, launches);
    if (x_type == BIGCN_BF16) return pick_back<GTYPE, BIGCN_BF16>(s, a, g_gain, g_offset, launches);
    return pick_back<GTYPE, BIGCN_F16>(s, a, g_gain, g_offset, launches);
}

}  // namespace

size_t layer_norm_scratch_bytes(int d) { return (size_t)kMaxParts * 2 * (size_t)d * sizeof(float); }

cudaError_t launch_layer_norm(cudaStream_t s, const void* x, int x_type, int64_t n, int d, int64_t ldx, const float* gain, const float* offset,
                              float eps, void* y, int y_type, int64_t ldy, float* mean, float* rstd, int* launches)
{
    NormArgs a = {x, x_type, ldx, n, d, rows_step(y, ldy, y_type, 8), gain, offset, eps, y, y_type, ldy, mean, rstd};
    if (rows_whole(x, ldx, x_type, x_type == BIGCN_F32 ? 4 : 8)) {
        if (x_type == BIGCN_F32) return pick_norm<BIGCN_F32, 4>(s, a, launches);
        if (x_type == BIGCN_BF16) return pick_norm<BIGCN_BF16, 8>(s, a, launches);
        return pick_norm<BIGCN_F16, 8>(s, a, launches);
    }
    const int step = rows_step(x, ldx, x_type, 4);
    if (x_type == BIGCN_F32) return pick_norm_step<BIGCN_F32>(s, step, a, launches);
    if (x_type == BIGCN_BF16) return pick_norm_step<BIGCN_BF16>(s, step, a, launches);
    return pick_norm_step<BIGCN_F16>(s, step, a, launches);
}

cudaError_t launch_layer_norm_backward(cudaStream_t s, const void* g, int g_type, int64_t ldg, const void* x, int x_type, int64_t ldx, int64_t n, int d,
                                       const float* gain, const float* mean, const float* rstd, void* gx, int gx_type, int64_t ldgx,
                                       float* g_gain, float* g_offset, void* scratch, int* launches)
{
    const NormBackArgs a = {g, g_type, ldg, x, x_type, ldx, n, d, rows_step(gx, ldgx, gx_type, 8), gain, mean, rstd, gx, gx_type, ldgx,
                            g_gain || g_offset ? static_cast<float*>(scratch) : nullptr};
    const int V = x_type == BIGCN_F32 || g_type == BIGCN_F32 ? 4 : 8;
    if (!rows_whole(g, ldg, g_type, V) || !rows_whole(x, ldx, x_type, V)) {
        const int step = std::min(rows_step(g, ldg, g_type, 4), rows_step(x, ldx, x_type, 4));
        if (step == 4) return pick_back_off<4>(s, a, g_gain, g_offset, launches);
        if (step == 2) return pick_back_off<2>(s, a, g_gain, g_offset, launches);
        return pick_back_off<1>(s, a, g_gain, g_offset, launches);
    }
    if (g_type == BIGCN_F32) return pick_back_x<BIGCN_F32>(s, x_type, a, g_gain, g_offset, launches);
    if (g_type == BIGCN_BF16) return pick_back_x<BIGCN_BF16>(s, x_type, a, g_gain, g_offset, launches);
    return pick_back_x<BIGCN_F16>(s, x_type, a, g_gain, g_offset, launches);
}

}  // namespace bigcn
