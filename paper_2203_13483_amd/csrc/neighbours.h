// Eight neighbours of a row whose address, length and stride need not fit vectors of 16 bytes: fetched and written whole, as the unit takes any
// address of an element.
#pragma once

#include "elements.h"

namespace mkq {

// 16 bytes from an address that only fits their elements (the unit takes any)
template <int BYTES>
struct __attribute__((packed, aligned(BYTES))) Loose {
    u32x4 v;
};
struct Codes {  // rows kept in 8 bits
    using raw = int8_t;
    static constexpr int BYTES = 1;
};

// Sixteen bytes without their first n elements, zeros behind them
template <int BYTES>
__device__ __forceinline__ u32x4 without_first(u32x4 v, int n)
{
    if constexpr (BYTES == 2) {
        if (n & 1)
            v = u32x4{__builtin_amdgcn_alignbit(v[1], v[0], 16), __builtin_amdgcn_alignbit(v[2], v[1], 16), __builtin_amdgcn_alignbit(v[3], v[2], 16), v[3] >> 16};
        n >>= 1;
    }
    if (n & 1) v = u32x4{v[1], v[2], v[3], 0};
    if (n & 2) v = u32x4{v[2], v[3], 0, 0};
    return n >= 4 ? u32x4{0, 0, 0, 0} : v;
}
// The elements of sixteen bytes of a row from place k on, zeros from place `end` on.  Whole vectors only, and no branch that lanes of a wave take
// apart: where the row ends among a wave's places (`edge`), its last sixteen bytes are fetched instead and moved down.  SHORT: rows may have fewer,
// which are fetched one by one.  place: the bytes of the row, or a place that all lanes share with `off` bytes to a lane's row
template <class E, bool SHORT>
__device__ __forceinline__ u32x4 fetch16(const void *place, uint32_t off, int k, int end, bool edge)
{
    constexpr int N = 16 / E::BYTES;
    const uint8_t *row = static_cast<const uint8_t *>(place);
    if (SHORT && end < N) {
        u32x4 v = {0, 0, 0, 0};
        if (k != 0) return v;
#pragma unroll
        for (int i = 0; i < N - 1; ++i)
            if (i < end) {
                const typename E::raw x = *reinterpret_cast<const typename E::raw *>(row + (off + i * E::BYTES));
                if constexpr (E::BYTES == 4) v[i] = __float_as_uint(x);
                else v[i / 2] |= (uint32_t)x << (16 * (i % 2));
            }
        return v;
    }
    const int from = edge && k + N > end ? end - N : k;
    const u32x4 v = reinterpret_cast<const Loose<E::BYTES> *>(row + (off + (uint32_t)from * E::BYTES))->v;
    return edge ? without_first<E::BYTES>(v, k - from < N ? k - from : N) : v;
}

// Eight neighbours of a row from place k on.  (Rows kept in 8 bits have zeros behind them.)
template <class E, bool SHORT = false>
struct Neighbours {
    u32x4 w[E::BYTES == 4 ? 2 : 1];
    __device__ __forceinline__ void clear()
    {
        w[0] = u32x4{0, 0, 0, 0};
        if constexpr (E::BYTES == 4) w[1] = u32x4{0, 0, 0, 0};
    }
    __device__ __forceinline__ void fetch(const void *row, int k, int end, bool edge) { fetch(row, 0u, k, end, edge); }
    __device__ __forceinline__ void fetch(const void *place, uint32_t off, int k, int end, bool edge)
    {
        if constexpr (E::BYTES == 1) {
            if (edge) k = k < end ? k : (end - 1) & ~7;
            const uint2 v = *reinterpret_cast<const uint2 *>(static_cast<const uint8_t *>(place) + (off + (uint32_t)k));
            w[0] = u32x4{v.x, v.y, 0, 0};
        } else {
            w[0] = fetch16<E, SHORT>(place, off, k, end, edge);
            if constexpr (E::BYTES == 4) w[1] = fetch16<E, SHORT>(place, off, k + 4, end, edge);
        }
    }
    __device__ __forceinline__ float get(int i) const
    {
        if constexpr (E::BYTES == 4) return __uint_as_float(w[i / 4][i % 4]);
        else if constexpr (E::BYTES == 1) return (float)(int8_t)(w[0][i / 4] >> (8 * (i % 4)));
        else return E::get((uint16_t)(w[0][i / 2] >> (16 * (i % 2))));
    }
};

// Eight neighbours of a row from place k on, those before `end`; place and off as above
template <class O>
__device__ __forceinline__ void put_neighbours(void *place, uint32_t off, int k, int end, bool edge, const float (&y)[8])
{
    uint8_t *to = static_cast<uint8_t *>(place) + (off + (uint32_t)k * O::BYTES);
    uint32_t w[8];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        if constexpr (O::BYTES == 4) {
            w[e] = __float_as_uint(y[e]);
            w[4 + e] = __float_as_uint(y[4 + e]);
        } else {
            w[e] = std::is_same<O, ElemF16>::value ? pack2_f16(in_binary32(y[2 * e]), in_binary32(y[2 * e + 1])) : pack2_bf16(y[2 * e], y[2 * e + 1]);
        }
    }
    if (edge && k + 8 > end) {
#pragma unroll
        for (int e = 0; e < 7; ++e)
            if (k + e < end) {
                if constexpr (O::BYTES == 4) reinterpret_cast<uint32_t *>(to)[e] = w[e];
                else reinterpret_cast<uint16_t *>(to)[e] = (uint16_t)(w[e / 2] >> (16 * (e % 2)));
            }
    } else {
        reinterpret_cast<Loose<O::BYTES> *>(to)->v = u32x4{w[0], w[1], w[2], w[3]};
        if constexpr (O::BYTES == 4) reinterpret_cast<Loose<4> *>(to + 16)->v = u32x4{w[4], w[5], w[6], w[7]};
    }
}

}  // namespace mkq
