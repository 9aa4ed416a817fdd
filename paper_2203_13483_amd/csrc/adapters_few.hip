// Few rows of short sides: hidden values and results in one launch.  A workgroup has a tile of 16 rows, an adapter of it and 512 columns, and makes
// the hidden values for itself, as every other 512 columns' workgroup does: a launch and a round trip less for 64 KiB through the caches more.
// Measured, us a call among others: a token each of 16 requests, 768 -> 768, rank 8, binary16 11.1 instead of 15.6 (the kernel 7.9); 64 rows of 64 adapters of rank 16,
// bfloat16, 1024 -> 1024 10.9 (1025 -> 1024, in two launches, 14.6).
#include "adapters.h"

namespace mkq {

template <class X, class W, class O>
__global__ __launch_bounds__(256, W::BYTES == 4 ? 1 : 2) void few_kernel(const ShrinkParams s, const ExpandParams p)
{
    constexpr int STEP = shrink_step(X::BYTES, W::BYTES), PT = O::BYTES == 4 ? 3 : 2;
    using XRows = ShrinkRows<X, STEP>;
    using WRows = ShrinkRows<W, STEP>;
    constexpr int LDS = XRows::BYTES + WRows::BYTES;
    static_assert(LDS >= 64 * 16, "sums");
    __shared__ __attribute__((aligned(16))) uint8_t lds[4 * LDS];
    __shared__ __attribute__((aligned(16))) float hidden[16][16];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, c = lane & 15, q = lane >> 4;
    const int groups = (p.column_blocks + 3) / 4;
    unsigned b = blockIdx.x;
    const int group = b % groups;
    b /= groups;
    const int slot = b % p.slots;
    const int64_t m0 = (int64_t)(b / p.slots) * 16;
    const int block = group * 4 + wave, n0 = block * 128 + 8 * c;
    const bool mine_to_write = block < p.column_blocks;
    const int last_row = p.a.M - m0 < 16 ? (int)(p.a.M - m0) - 1 : 15;
    const int mine = adapter_of(p.a, lane < 16 ? m0 + lane : p.a.M);
    uint8_t *lds_x = lds + wave * LDS, *lds_w = lds_x + XRows::BYTES;
    v4f *sums = reinterpret_cast<v4f *>(lds);
    Neighbours<O> base[4];
    if (p.base && mine_to_write) {
        const void *at = static_cast<const typename O::raw *>(p.base) + m0 * p.ld_base;
#pragma unroll
        for (int v = 0; v < 4; ++v)
            base[v].fetch(at, (uint32_t)(4 * q + v < last_row ? 4 * q + v : last_row) * ((uint32_t)p.ld_base * O::BYTES), n0, p.N, true);
    }
    const int steps = (s.K + STEP - 1) / STEP;
    Adapters adapters(mine, slot, p.slots, lane < 16 && m0 + lane < p.a.M && mine < 0);
    int a;
    uint64_t same;
    while (adapters.next(a, same)) {
        v4f acc[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) acc[i] = v4f{0, 0, 0, 0};
        if (a < 0) {  // rows without an adapter
            if (s.hidden && group == 0 && threadIdx.x < 16 && (same >> threadIdx.x & 1))
                for (int r = 0; r < p.a.rank; ++r) s.hidden[(m0 + threadIdx.x) * p.a.rank + r] = 0.0f;
        } else {
            Block<W> rows;
            if (mine_to_write) {
                const typename W::raw *w = static_cast<const typename W::raw *>(p.w) + (int64_t)a * p.a.rank * p.N;
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    rows.rows[e].fetch(w, (uint32_t)(8 * q + e < p.a.rank ? 8 * q + e : p.a.rank - 1) * ((uint32_t)p.N * W::BYTES), n0, p.N, true);
            }
            const typename W::raw *w = static_cast<const typename W::raw *>(s.w) + (int64_t)a * p.a.rank * s.K;
            v4f sum = {0, 0, 0, 0};
            for (int i = wave; i < steps; i += 4) {
                XRows xs;
                WRows ws;
#pragma unroll
                for (int j = 0; j < XRows::N; ++j) {
                    const int row = XRows::row_of(j);
                    xs.v[j] = fetch16<X, false>(static_cast<const typename X::raw *>(s.x) + (m0 + (row < last_row ? row : last_row)) * s.ldx, 0,
                                                i * STEP + XRows::piece_of() * (16 / X::BYTES), s.K, true);
                }
#pragma unroll
                for (int j = 0; j < WRows::N; ++j) {
                    const int at = WRows::row_of(j);
                    ws.v[j] = fetch16<W, false>(w, (uint32_t)(at < p.a.rank ? at : p.a.rank - 1) * ((uint32_t)s.K * W::BYTES),
                                                i * STEP + WRows::piece_of() * (16 / W::BYTES), s.K, true);
                }
                wave_order();
                xs.put(lds_x);
                ws.put(lds_w);
                wave_order();
#pragma unroll
                for (int h = 0; h < STEP / 32; ++h) {
                    const Neighbours<X> xn = XRows::get(lds_x, h);
                    const Neighbours<W> wn = WRows::get(lds_w, h);
                    if constexpr (std::is_same<X, ElemF16>::value && std::is_same<W, ElemF16>::value) {
                        sum = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(v8h, xn.w[0]), __builtin_bit_cast(v8h, wn.w[0]), sum, 0, 0, 0);
                    } else {
                        uint4 xp[Parts<X>::N], wp[Parts<W>::N];
                        operand(xn, xp);
                        operand(wn, wp);
                        sum = multiply<3>(xp, wp, sum);
                    }
                }
            }
            __syncthreads();
            sums[wave * 64 + lane] = sum;
            __syncthreads();
            if (wave == 0) {
                const v4f all = (sums[lane] + sums[64 + lane]) + (sums[128 + lane] + sums[192 + lane]);
#pragma unroll
                for (int v = 0; v < 4; ++v) {
                    const float value = c < p.a.rank ? all[v] : 0.0f;
                    hidden[4 * q + v][c] = value;
                    if (s.hidden && group == 0 && c < p.a.rank && (same >> (4 * q + v) & 1)) s.hidden[(m0 + 4 * q + v) * p.a.rank + c] = value;
                }
            }
            __syncthreads();
            const float scale = scale_of(p.a, a);
            uint4 tp[PT];
            float v[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = q < 2 ? hidden[c][8 * (q & 1) + e] * scale : 0.0f;
            parts_of(v, tp);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                uint4 wp[Parts<W>::N];
                rows.column(i, wp);
                acc[i] = multiply<3>(tp, wp, acc[i]);
            }
        }
        if (!mine_to_write || n0 >= p.N || (a < 0 && p.base == p.out)) continue;
#pragma unroll
        for (int v = 0; v < 4; ++v)
            if (same >> (4 * q + v) & 1) {
                float y[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) y[e] = p.base ? acc[e][v] + base[v].get(e) : acc[e][v];
                put_neighbours<O>(static_cast<typename O::raw *>(p.out) + m0 * p.ld_out, (uint32_t)(4 * q + v) * ((uint32_t)p.ld_out * O::BYTES), n0, p.N, true, y);
            }
    }
}

void launch_few_kernel(const ShrinkParams &s, const ExpandParams &e, int x_dtype, int w_dtype, int out_dtype, unsigned workgroups, hipStream_t st)
{
    with_elem(x_dtype, [&](auto x) {
        with_elem(w_dtype, [&](auto w) {
            with_elem(out_dtype, [&](auto o) { few_kernel<decltype(x), decltype(w), decltype(o)><<<workgroups, 256, 0, st>>>(s, e); });
        });
    });
}

}  // namespace mkq
