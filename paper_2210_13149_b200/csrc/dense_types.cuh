// Element types of the dense operators (layer norm, 8-bit products, class loss): loads to fp32 and rounded stores.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <stdint.h>

#include "bigcn_internal.cuh"

namespace bigcn {
namespace dense {

__host__ __device__ constexpr int type_bytes(int type) { return type == BIGCN_F32 ? 4 : 2; }

template <int TYPE> struct Elt;
template <> struct Elt<BIGCN_F32> { using T = float; };
template <> struct Elt<BIGCN_BF16> { using T = __nv_bfloat16; };
template <> struct Elt<BIGCN_F16> { using T = __half; };

template <int TYPE>
__device__ __forceinline__ float to_float(typename Elt<TYPE>::T v)
{
    if constexpr (TYPE == BIGCN_F32) return v;
    else if constexpr (TYPE == BIGCN_BF16) return __bfloat162float(v);
    else return __half2float(v);
}
template <int TYPE>
__device__ __forceinline__ typename Elt<TYPE>::T from_float(float v)
{
    if constexpr (TYPE == BIGCN_F32) return v;
    else if constexpr (TYPE == BIGCN_BF16) return __float2bfloat16_rn(v);
    else return __float2half_rn(v);
}
// two values as one 32-bit word of a 16-bit type, the first in the low half
template <int TYPE>
__device__ __forceinline__ uint32_t pack2(float a, float b)
{
    if constexpr (TYPE == BIGCN_BF16) {
        const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
        return *reinterpret_cast<const uint32_t*>(&h);
    } else {
        const __half2 h = __floats2half2_rn(a, b);
        return *reinterpret_cast<const uint32_t*>(&h);
    }
}
template <int TYPE>
__device__ __forceinline__ float2 unpack2(uint32_t w)
{
    if constexpr (TYPE == BIGCN_BF16) return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
    else return __half22float2(*reinterpret_cast<const __half2*>(&w));
}

// Four consecutive elements, of which the first `count` exist; the rest read as 0.  `whole`: the pointer is aligned to four, and they can be moved as a whole
// word where all of them exist.
template <int TYPE>
__device__ __forceinline__ void load4_of(const typename Elt<TYPE>::T* __restrict__ p, int count, bool whole, float (&v)[4])
{
    if (whole && count >= 4) {
        if constexpr (TYPE == BIGCN_F32) {
            const float4 w = *reinterpret_cast<const float4*>(p);
            v[0] = w.x; v[1] = w.y; v[2] = w.z; v[3] = w.w;
        } else {
            const uint2 w = *reinterpret_cast<const uint2*>(p);
            const float2 a = unpack2<TYPE>(w.x), b = unpack2<TYPE>(w.y);
            v[0] = a.x; v[1] = a.y; v[2] = b.x; v[3] = b.y;
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = i < count ? to_float<TYPE>(p[i]) : 0.f;
}
// the same with the type known at run time
__device__ __forceinline__ void load4(const void* base, int type, int64_t at, int count, bool whole, float (&v)[4])
{
    if (type == BIGCN_F32) load4_of<BIGCN_F32>(static_cast<const float*>(base) + at, count, whole, v);
    else if (type == BIGCN_BF16) load4_of<BIGCN_BF16>(static_cast<const __nv_bfloat16*>(base) + at, count, whole, v);
    else load4_of<BIGCN_F16>(static_cast<const __half*>(base) + at, count, whole, v);
}

// The first `count` of V (1, 2, 4 or 8) consecutive elements, `whole` as above for V of them (or 16 bytes).
template <int TYPE, int V>
__device__ __forceinline__ void store_elts(typename Elt<TYPE>::T* __restrict__ p, int count, bool whole, const float (&v)[V])
{
    if (whole && count >= V) {
        if constexpr (V == 1) {
            *p = from_float<TYPE>(v[0]);
        } else if constexpr (V == 2 && TYPE == BIGCN_F32) {
            *reinterpret_cast<float2*>(p) = make_float2(v[0], v[1]);
        } else if constexpr (V == 2) {
            *reinterpret_cast<uint32_t*>(p) = pack2<TYPE>(v[0], v[1]);
        } else if constexpr (TYPE == BIGCN_F32) {
#pragma unroll
            for (int i = 0; i < V; i += 4) *reinterpret_cast<float4*>(p + i) = make_float4(v[i], v[i + 1], v[i + 2], v[i + 3]);
        } else if constexpr (V == 4) {
            *reinterpret_cast<uint2*>(p) = make_uint2(pack2<TYPE>(v[0], v[1]), pack2<TYPE>(v[2], v[3]));
        } else {
            *reinterpret_cast<uint4*>(p) = make_uint4(pack2<TYPE>(v[0], v[1]), pack2<TYPE>(v[2], v[3]), pack2<TYPE>(v[4], v[5]), pack2<TYPE>(v[6], v[7]));
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < V; ++i)
        if (i < count) p[i] = from_float<TYPE>(v[i]);
}
template <int V>
__device__ __forceinline__ void store_as(void* base, int type, int64_t at, int count, bool whole, const float (&v)[V])
{
    if (type == BIGCN_F32) store_elts<BIGCN_F32, V>(static_cast<float*>(base) + at, count, whole, v);
    else if (type == BIGCN_BF16) store_elts<BIGCN_BF16, V>(static_cast<__nv_bfloat16*>(base) + at, count, whole, v);
    else store_elts<BIGCN_F16, V>(static_cast<__half*>(base) + at, count, whole, v);
}

// Words of at most `step` elements, a power of two that the address is aligned to.  A row's store looks its type up once: NV words of a
// lane, `stride` elements apart from column `c` on.
template <int TYPE, int V>
__device__ __forceinline__ void store_steps(typename Elt<TYPE>::T* p, int count, int step, const float (&v)[V])
{
    if constexpr (V == 1) {
        store_elts<TYPE, 1>(p, count, true, v);
    } else {
        if (step >= V) return store_elts<TYPE, V>(p, count, true, v);
        float lo[V / 2], hi[V / 2];
#pragma unroll
        for (int i = 0; i < V / 2; ++i) lo[i] = v[i], hi[i] = v[V / 2 + i];
        store_steps<TYPE, V / 2>(p, count, step, lo);
        store_steps<TYPE, V / 2>(p + V / 2, count - V / 2, step, hi);
    }
}
template <int TYPE, int NV, int V>
__device__ __forceinline__ void store_row_of(void* base, int64_t row_at, int c, int stride, int d, int step, const float (&v)[NV][V])
{
    auto* p = static_cast<typename Elt<TYPE>::T*>(base) + row_at;
#pragma unroll
    for (int k = 0; k < NV; ++k)
        if (c + k * stride < d) store_steps<TYPE, V>(p + c + k * stride, d - c - k * stride, step, v[k]);
}
template <int NV, int V>
__device__ __forceinline__ void store_row(void* base, int type, int64_t row_at, int c, int stride, int d, int step, const float (&v)[NV][V])
{
    if (type == BIGCN_F32) store_row_of<BIGCN_F32, NV, V>(base, row_at, c, stride, d, step, v);
    else if (type == BIGCN_BF16) store_row_of<BIGCN_BF16, NV, V>(base, row_at, c, stride, d, step, v);
    else store_row_of<BIGCN_F16, NV, V>(base, row_at, c, stride, d, step, v);
}

constexpr int kAnyType = -1;                  // a type known at run time

// V elements as they lie in memory, words of 32 bits (a 16-bit element alone in the low half of one).  Nothing is done with them where they are loaded, so
// that a row asked for ahead of its time is not waited for before it.
template <int TYPE, int V>
struct Raw {
    static constexpr int kWords = TYPE == kAnyType || TYPE == BIGCN_F32 ? V : V > 1 ? V / 2 : 1;
    uint32_t w[kWords];

    // The first `count` of V elements, zeros behind them.  whole: the address is aligned to V elements (or 16 bytes); otherwise to one.
    __device__ __forceinline__ void load(const void* base, int type, int64_t at, int count, bool whole = true)
    {
        if (TYPE == BIGCN_F32 || (TYPE == kAnyType && type == BIGCN_F32)) load_words<BIGCN_F32>(static_cast<const float*>(base) + at, count, whole);
        else load_words<BIGCN_BF16>(reinterpret_cast<const __nv_bfloat16*>(base) + at, count, whole);
    }
    template <int T>
    __device__ __forceinline__ void load_words(const typename Elt<T>::T* p, int count, bool whole)
    {
        constexpr int kUsed = T == BIGCN_F32 ? V : V > 1 ? V / 2 : 1;
        if constexpr (kUsed <= kWords) {
            const uint32_t* q = reinterpret_cast<const uint32_t*>(p);
            const unsigned short* h = reinterpret_cast<const unsigned short*>(p);
            if (count >= V && whole) {
                if constexpr (T != BIGCN_F32 && V == 1) {
                    w[0] = *h;
                } else if constexpr (kUsed == 1) {
                    w[0] = *q;
                } else if constexpr (kUsed == 2) {
                    const uint2 v = *reinterpret_cast<const uint2*>(q);
                    w[0] = v.x; w[1] = v.y;
                } else {
#pragma unroll
                    for (int i = 0; i < kUsed; i += 4) {
                        const uint4 v = *reinterpret_cast<const uint4*>(q + i);
                        w[i] = v.x; w[i + 1] = v.y; w[i + 2] = v.z; w[i + 3] = v.w;
                    }
                }
            } else if constexpr (T == BIGCN_F32) {
#pragma unroll
                for (int i = 0; i < V; ++i) w[i] = i < count ? q[i] : 0u;
            } else if (whole) {
#pragma unroll
                for (int i = 0; i < kUsed; ++i) w[i] = 2 * i + 1 < count ? q[i] : 2 * i < count ? (uint32_t)h[2 * i] : 0u;
            } else {
#pragma unroll
                for (int i = 0; i < kUsed; ++i) w[i] = (2 * i < count ? (uint32_t)h[2 * i] : 0u) | (V > 1 && 2 * i + 1 < count ? (uint32_t)h[2 * i + 1] << 16 : 0u);
            }
        }
    }
    __device__ __forceinline__ void values(float (&f)[V], int type = TYPE) const
    {
        if (TYPE == BIGCN_F32 || (TYPE == kAnyType && type == BIGCN_F32)) {
            if constexpr (kWords == V) {
#pragma unroll
                for (int i = 0; i < V; ++i) f[i] = __uint_as_float(w[i]);
            }
        } else if (TYPE == BIGCN_BF16 || (TYPE == kAnyType && type == BIGCN_BF16)) {
            halves<BIGCN_BF16>(f);
        } else {
            halves<BIGCN_F16>(f);
        }
    }
    template <int T>
    __device__ __forceinline__ void halves(float (&f)[V]) const
    {
#pragma unroll
        for (int i = 0; i < (V > 1 ? V / 2 : 1); ++i) {
            const float2 u = unpack2<T>(w[i]);
            f[2 * i] = u.x;
            if constexpr (V > 1) f[2 * i + 1] = u.y;
        }
    }
    // the same through shared memory: an asynchronous copy of `count` elements to a place of this thread's own, zeros behind them
    static __device__ __forceinline__ void copy_to(void* to, const typename Elt<TYPE < 0 ? 0 : TYPE>::T* from, int count)
    {
        constexpr int kBytes = 4 * kWords;
        const int bytes = count * type_bytes(TYPE);
        const uint32_t dst = (uint32_t)__cvta_generic_to_shared(to);
        if constexpr (kBytes == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;\n" ::"r"(dst), "l"(from), "r"(bytes) : "memory");
        else asm volatile("cp.async.ca.shared.global [%0], [%1], 8, %2;\n" ::"r"(dst), "l"(from), "r"(bytes) : "memory");
    }
    __device__ __forceinline__ void take(const void* from)
    {
        if constexpr (kWords == 4) {
            const uint4 q = *static_cast<const uint4*>(from);
            w[0] = q.x; w[1] = q.y; w[2] = q.z; w[3] = q.w;
        } else if constexpr (kWords == 2) {
            const uint2 q = *static_cast<const uint2*>(from);
            w[0] = q.x; w[1] = q.y;
        }
    }
};

// Whether rows of `ld` elements from `base` on can be moved in words of V elements.
inline bool rows_whole(const void* base, int64_t ld, int type, int V)
{
    const int64_t bytes = (int64_t)V * type_bytes(type), word = bytes < 16 ? bytes : 16;
    return reinterpret_cast<uintptr_t>(base) % word == 0 && ld * type_bytes(type) % word == 0;
}

// The widest words of at most V elements that they can be moved in.
inline int rows_step(const void* base, int64_t ld, int type, int V)
{
    while (V > 1 && !rows_whole(base, ld, type, V)) V /= 2;
    return V;
}

}  // namespace dense
}  // namespace bigcn
