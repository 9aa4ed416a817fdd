// Element types of tensors that may be binary32, binary16 or bfloat16: how a value is fetched and written, one at a time
// or eight neighbours at once.  Arithmetic is binary32; a result is rounded once, where it is written (to nearest even).
#pragma once

#include <type_traits>

#include "mkq_internal.h"

namespace mkq {

struct ElemF32 {
    using raw = float;
    static constexpr int BYTES = 4;
    __device__ static __forceinline__ float get(raw v) { return v; }
    __device__ static __forceinline__ raw put(float v) { return v; }
};
struct ElemF16 {
    using raw = uint16_t;
    static constexpr int BYTES = 2;
    __device__ static __forceinline__ float get(raw v) { return half_bits_to_float(v); }
    __device__ static __forceinline__ raw put(float v) { return float_to_half_bits(v); }
};
struct ElemBF16 {
    using raw = uint16_t;
    static constexpr int BYTES = 2;
    __device__ static __forceinline__ float get(raw v) { return __uint_as_float((uint32_t)v << 16); }
    __device__ static __forceinline__ raw put(float v) { return float_to_bf16_bits(v); }
};

// A product rounded to binary32, also where it is narrowed next: the compiler would fuse a single value's product with its rounding
// to 16 bits, but not those of a vector, and the same value would come out differently by where it lies.
__device__ __forceinline__ float product(float a, float b)
{
    float r = a * b;
    asm("" : "+v"(r));
    return r;
}

// Eight neighbours as binary32, from an address that is a multiple of 16
template <class E>
__device__ __forceinline__ void get8(const typename E::raw *p, float (&v)[8])
{
    if constexpr (E::BYTES == 4) {
        load8<float>(reinterpret_cast<const float *>(p), v);
    } else {
        const uint4 a = *reinterpret_cast<const uint4 *>(p);
        const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[2 * i] = E::get((uint16_t)(w[i] & 0xFFFFu));
            v[2 * i + 1] = E::get((uint16_t)(w[i] >> 16));
        }
    }
}

// 16 bytes that this kernel does not touch again, past the caches where STREAM
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
template <bool STREAM>
__device__ __forceinline__ void store16(void *p, uint4 v)
{
    if constexpr (STREAM) {
        const u32x4 x = {v.x, v.y, v.z, v.w};
        __builtin_nontemporal_store(x, static_cast<u32x4 *>(p));
    } else {
        *static_cast<uint4 *>(p) = v;
    }
}

template <class E, bool STREAM = false>
__device__ __forceinline__ void put8(typename E::raw *p, const float (&v)[8])
{
    if constexpr (E::BYTES == 4) {
#pragma unroll
        for (int i = 0; i < 8; i += 4)
            store16<STREAM>(p + i, make_uint4(__float_as_uint(v[i]), __float_as_uint(v[i + 1]), __float_as_uint(v[i + 2]), __float_as_uint(v[i + 3])));
    } else {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i)
            w[i] = std::is_same<E, ElemF16>::value ? pack2_f16(v[2 * i], v[2 * i + 1]) : pack2_bf16(v[2 * i], v[2 * i + 1]);
        store16<STREAM>(p, make_uint4(w[0], w[1], w[2], w[3]));
    }
}

// Host side: f(E()) for the element type of a dtype code
inline bool is_float_dtype(int dtype) { return dtype == MKQ_F32 || dtype == MKQ_F16 || dtype == MKQ_BF16; }
inline int64_t dtype_bytes(int dtype) { return dtype == MKQ_F32 ? 4 : 2; }
template <class F>
inline void with_elem(int dtype, F &&f)
{
    if (dtype == MKQ_F32) f(ElemF32());
    else if (dtype == MKQ_F16) f(ElemF16());
    else f(ElemBF16());
}
// Rows of ld elements from an address that is a multiple of 16: whether every eighth element of every row is, too
inline bool rows_aligned16(const void *p, int64_t ld, int dtype) { return aligned16(p) && (ld * dtype_bytes(dtype)) % 16 == 0; }

inline bool aligned4(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

// Workgroups of a launch: the grid's work items are counted in 32 bits
inline bool grid_ok(int64_t workgroups, int threads) { return workgroups > 0 && workgroups * threads < ((int64_t)1 << 32); }

}  // namespace mkq
