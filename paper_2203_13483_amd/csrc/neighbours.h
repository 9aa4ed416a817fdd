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

// Eight neighbours of a row from place k on, as fetched.  Whole vectors only, and no branch that lanes of a wave take apart: where the row
// ends among a wave's places (`edge`), its last eight elements are fetched instead and moved down, zeros behind them.  A row of fewer than
// eight is fetched one by one.  (Rows kept in 8 bits have zeros behind them.)
template <class E>
struct Neighbours {
    u32x4 w[E::BYTES == 4 ? 2 : 1];
    __device__ __forceinline__ void clear()
    {
        w[0] = u32x4{0, 0, 0, 0};
        if constexpr (E::BYTES == 4) w[1] = u32x4{0, 0, 0, 0};
    }
    __device__ __forceinline__ void without_first(int n)
    {
        if constexpr (E::BYTES == 2) {
            u32x4 &v = w[0];
            if (n & 1)
                v = u32x4{__builtin_amdgcn_alignbit(v[1], v[0], 16), __builtin_amdgcn_alignbit(v[2], v[1], 16), __builtin_amdgcn_alignbit(v[3], v[2], 16), v[3] >> 16};
            if (n & 2) v = u32x4{v[1], v[2], v[3], 0};
            if (n & 4) v = u32x4{v[2], v[3], 0, 0};
            if (n >= 8) v = u32x4{0, 0, 0, 0};
        } else {
            u32x4 &v = w[0], &x = w[E::BYTES / 4];
            if (n & 1) {
                v = u32x4{v[1], v[2], v[3], x[0]};
                x = u32x4{x[1], x[2], x[3], 0};
            }
            if (n & 2) {
                v = u32x4{v[2], v[3], x[0], x[1]};
                x = u32x4{x[2], x[3], 0, 0};
            }
            if (n >= 4) {
                v = n >= 8 ? u32x4{0, 0, 0, 0} : x;
                x = u32x4{0, 0, 0, 0};
            }
        }
    }
    // `row`: the bytes of a row, or a place that all lanes share with `off` bytes to a lane's row
    __device__ __forceinline__ void fetch(const void *row, int k, int end, bool edge) { fetch(row, 0u, k, end, edge); }
    __device__ __forceinline__ void fetch(const void *place, uint32_t off, int k, int end, bool edge)
    {
        const uint8_t *row = static_cast<const uint8_t *>(place);
        if constexpr (E::BYTES == 1) {
            if (edge) k = k < end ? k : (end - 1) & ~7;
            const uint2 v = *reinterpret_cast<const uint2 *>(row + (off + (uint32_t)k));
            w[0] = u32x4{v.x, v.y, 0, 0};
        } else {
            if (end < 8) return fetch_short(row, off, k, end);
            const int from = edge && k + 8 > end ? end - 8 : k;
            const uint8_t *at = row + (off + (uint32_t)from * E::BYTES);
            w[0] = reinterpret_cast<const Loose<E::BYTES> *>(at)->v;
            if constexpr (E::BYTES == 4) w[1] = reinterpret_cast<const Loose<4> *>(at + 16)->v;
            if (edge) without_first(k - from < 8 ? k - from : 8);
        }
    }
    __device__ __forceinline__ void fetch_short(const uint8_t *row, uint32_t off, int k, int end)
    {
        clear();
        if (k != 0) return;
#pragma unroll
        for (int i = 0; i < 7; ++i)
            if (i < end) {
                const typename E::raw v = *reinterpret_cast<const typename E::raw *>(row + (off + i * E::BYTES));
                if constexpr (E::BYTES == 4) w[i / 4][i % 4] = __float_as_uint(v);
                else w[0][i / 2] |= (uint32_t)v << (16 * (i % 2));
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
