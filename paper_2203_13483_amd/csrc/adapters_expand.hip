// Sums of an adapter's rows: out = base + s_a up_a^T t, dx = base + down_a^T u.
#include "adapters.h"

namespace mkq {

// t of row c from place r on, eight values, added up over the splits (ONE: there is one); t: the tile's first row
template <bool ONE>
__device__ __forceinline__ void hidden_values(const ExpandParams &p, const float *t, int c, int r, float (&v)[8])
{
    const uint32_t off = (uint32_t)(c * p.a.pitch + (r < p.a.pitch ? r : 0)) * 4;
    const int64_t split = p.a.M * p.a.pitch;
    auto load = [&](int s, float (&to)[8]) { load8(reinterpret_cast<const float *>(reinterpret_cast<const uint8_t *>(t + s * split) + off), to); };
    load(0, v);
    for (int s = 1; !ONE && s < p.a.splits; s += 3) {
        float more[3][8];
#pragma unroll
        for (int i = 0; i < 3; ++i) load(s + i < p.a.splits ? s + i : s, more[i]);
#pragma unroll
        for (int i = 0; i < 3; ++i)
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] += s + i < p.a.splits ? more[i][e] : 0.0f;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = r < p.a.pitch ? v[e] : 0.0f;
}

// A wave has 16 rows and 128 columns; lane (c, q) has columns 8 c .. 8 c + 7 of rows 4 q .. 4 q + 3.  edge: whether the matrix ends among the columns
template <class W, class O, bool ONE, class EDGE>
__device__ __forceinline__ void expand(const ExpandParams &p, int64_t m0, int block, int slot, EDGE edge)
{
    constexpr int PT = O::BYTES == 4 ? 3 : 2;  // (two leave out 2^-17 of a product, of either sign, under results of 16 bits, which end at 2^-9 or 2^-12.  With three, 8192 rows of 1024 and 4096, rank 16:
    // bfloat16 39.3 instead of 38.9 us, binary16 53.5 instead of 49.1)
    const int last_row = p.a.M - m0 < 16 ? (int)(p.a.M - m0) - 1 : 15;
    const int first_lane = threadIdx.x & 63, mine = adapter_of(p.a, first_lane < 16 ? m0 + first_lane : p.a.M);
    Neighbours<O> base[4];
    if (p.base) {
        const int q = first_lane >> 4, n0 = block * 128 + 8 * (first_lane & 15);
        const void *at = static_cast<const typename O::raw *>(p.base) + m0 * p.ld_base;
#pragma unroll
        for (int v = 0; v < 4; ++v)
            base[v].fetch(at, (uint32_t)(4 * q + v < last_row ? 4 * q + v : last_row) * ((uint32_t)p.ld_base * O::BYTES), n0, p.N, edge);
    }
    typename O::raw *out = static_cast<typename O::raw *>(p.out) + m0 * p.ld_out;
    const float *t = p.t + m0 * p.a.pitch;
    Adapters adapters(mine, slot, p.slots, first_lane < 16 && m0 + first_lane < p.a.M && mine < 0);
    int a;
    uint64_t same;
    while (adapters.next(a, same)) {
        const int lane = fresh(threadIdx.x & 63), c = lane & 15, q = lane >> 4, n0 = block * 128 + 8 * c;
        v4f acc[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) acc[i] = v4f{0, 0, 0, 0};
        if (a < 0) {  // rows without an adapter
            if (!ONE && p.keep && block == 0)
                for (int i = 0; i < 16; ++i)
                    if (same >> i & 1)
                        for (int r = lane; r < p.a.rank; r += 64) p.keep[(m0 + i) * p.keep_pitch + r] = 0.0f;
            if (p.base == p.out) continue;
        } else {
            const float scale = scale_of(p.a, a), factor = p.scaled ? scale : 1.0f;
            const typename W::raw *w = static_cast<const typename W::raw *>(p.w) + (int64_t)a * p.a.rank * p.N;
#pragma unroll 1
            for (int r0 = 0; r0 < p.a.rank; r0 += 32) {
                const int r = r0 + 8 * q;
                Block<W> rows;  // (behind the rank its last row again: t is 0 there)
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    rows.rows[e].fetch(w, (uint32_t)(r + e < p.a.rank ? r + e : p.a.rank - 1) * ((uint32_t)p.N * W::BYTES), n0, p.N, edge);
                uint4 tp[PT];
                float v[8];
                hidden_values<ONE>(p, t, c < last_row ? c : last_row, r, v);
                if (!ONE && p.keep && block == 0 && (same >> c & 1)) {
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        if (r + e < p.a.rank) p.keep[(m0 + c) * p.keep_pitch + r + e] = p.keep_scaled ? v[e] * factor : v[e];
                }
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] *= factor;
                parts_of(v, tp);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    uint4 wp[Parts<W>::N];
                    rows.column(i, wp);
                    acc[i] = multiply<3>(tp, wp, acc[i]);
                }
            }
        }
#pragma unroll
        for (int v = 0; v < 4; ++v)
            if (same >> (4 * q + v) & 1 && (!edge || n0 < p.N)) {
                float y[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) y[e] = p.base ? acc[e][v] + base[v].get(e) : acc[e][v];
                put_neighbours<O>(out, (uint32_t)(4 * q + v) * ((uint32_t)p.ld_out * O::BYTES), n0, p.N, edge, y);
            }
    }
}

template <class W, class O, bool ONE>
__global__ __launch_bounds__(256, W::BYTES == 4 || O::BYTES == 4 || !ONE ? 2 : 4) void expand_kernel(const ExpandParams p)
{
    const ColumnTask task(blockIdx.x, p.column_blocks, __builtin_amdgcn_readfirstlane(threadIdx.x >> 6));
    const int slot = task.row / p.row_groups, block = task.block;
    if (slot >= p.slots || block >= p.column_blocks) return;
    const int64_t m0 = (int64_t)(task.row - slot * p.row_groups) * 16;
    if (block * 128 + 128 > p.N) expand<W, O, ONE>(p, m0, block, slot, std::true_type());
    else expand<W, O, ONE>(p, m0, block, slot, std::false_type());
}

void launch_expand_kernel(const ExpandParams &p, int w_dtype, int out_dtype, unsigned workgroups, hipStream_t st)
{
    with_elem(w_dtype, [&](auto w) {
        with_elem(out_dtype, [&](auto o) {
            using W = decltype(w);
            using O = decltype(o);
            if (p.a.splits == 1) expand_kernel<W, O, true><<<workgroups, 256, 0, st>>>(p);
            else expand_kernel<W, O, false><<<workgroups, 256, 0, st>>>(p);
        });
    });
}

}  // namespace mkq
