// Sums of the batch's rows: d_down_a = sum_m u[m] x[m]^T, d_up_a = s_a sum_m t[m] dy[m]^T.
#include "adapters.h"

namespace mkq {

// rows: how many of the batch the adapter has.  (0 times a scale that is infinite or NaN would not be the 0 of an adapter without any.)
__device__ __forceinline__ void write_grad(const OuterParams &p, const OuterSide &side, int a, int rows, int64_t at, float v)
{
    v *= side.scaled && rows > 0 ? scale_of(p.a, a) : 1.0f;
    at += (int64_t)a * p.a.rank * side.N;
    auto write = [&](auto o) __attribute__((always_inline)) {
        using O = decltype(o);
        typename O::raw *to = static_cast<typename O::raw *>(side.grad) + at;
        if (p.accumulate) v += O::get(*to);
        *to = O::put(in_binary32(v));
    };
    if (p.grad_dtype == MKQ_F32) write(ElemF32());
    else if (p.grad_dtype == MKQ_F16) write(ElemF16());
    else write(ElemBF16());
}

// 32 rows of a piece on their way: lane (c, q) has eight neighbouring columns of rows 8 q .. 8 q + 7, and their coefficients for place c of the rank
template <class Y, int RT>
struct OuterStage {
    Block<Y> y;
    float coeff[RT][8], step[Y::BYTES == 1 ? 8 : 1];
    // rows: in lanes from `first` on, the piece's
    template <class EDGE>
    __device__ __forceinline__ void fetch(const OuterParams &p, const OuterSide &side, int chunk, int n0, EDGE edge, int rows, int first)
    {
        const int lane = threadIdx.x & 63, c = lane & 15, q = lane >> 4;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int64_t row = __shfl(rows, first + 8 * q + e, 64);
            y.rows[e].fetch(static_cast<const typename Y::raw *>(side.y) + row * side.ld, n0, side.N, edge);
            if constexpr (Y::BYTES == 1) step[e] = side.steps[row * side.groups + ((n0 < side.N ? n0 : 0) >> side.group_shift)];
#pragma unroll
            for (int r = 0; r < RT; ++r) {
                const int at = (chunk * RT + r) * 16 + c;
                coeff[r][e] = side.coeff[row * side.coeff_pitch + (at < p.a.rank ? at : 0)];
            }
        }
    }
    // left: how many of the rows are the piece's; the others are its last row again, times 0
    __device__ __forceinline__ void add(v4f (&acc)[RT][8], int left)
    {
        const int q = (threadIdx.x & 63) >> 4;
        uint4 cp[RT][3];
#pragma unroll
        for (int r = 0; r < RT; ++r) {
#pragma unroll
            for (int e = 0; e < 8; ++e) coeff[r][e] = 8 * q + e < left ? coeff[r][e] : 0.0f;
            parts_of(coeff[r], cp[r]);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            uint4 yp[Parts<Y>::N];
            if constexpr (Y::BYTES == 1) {
                float v[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = product(y.rows[e].get(i), step[e]);
                parts_of(v, yp);
            } else {
                y.column(i, yp);
            }
#pragma unroll
            for (int r = 0; r < RT; ++r) acc[r][i] = multiply<3>(cp[r], yp, acc[r][i]);
        }
    }
};

// A piece of an adapter's rows, 128 columns and RT * 16 of the rank.  The rows of the next step are asked for before those at hand are used.
template <class Y, int RT, class EDGE>
__device__ __forceinline__ void outer(const OuterParams &p, const OuterSide &side, int block, int chunk, int a, int first, int last, int pieces, float *tile,
                                      EDGE edge)
{
    const int lane = threadIdx.x & 63, c = lane & 15, q = lane >> 4, n0 = block * 128 + 8 * c, n = last - first;
    v4f acc[RT][8];
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int i = 0; i < 8; ++i) acc[r][i] = v4f{0, 0, 0, 0};
    const int32_t *order = p.plan.order + first;
    auto places = [&](int s) { return (int)order[s + lane < n ? s + lane : n - 1]; };
    if (n > 0) {
        OuterStage<Y, RT> even, odd;
        int rows = places(0);
        even.fetch(p, side, chunk, n0, edge, rows, 0);
        for (int s = 0; s < n; s += 64) {
            int next = rows;
            if (s + 64 < n) next = places(s + 64);
            if (s + 32 < n) odd.fetch(p, side, chunk, n0, edge, rows, 32);
            even.add(acc, n - s);
            rows = next;
            if (s + 64 < n) even.fetch(p, side, chunk, n0, edge, rows, 0);
            if (s + 32 < n) odd.add(acc, n - s - 32);
        }
    }
    const int start = p.plan.starts[a], part = 2 * (start / p.plan.piece) + (first - start) / p.plan.piece;
    const int columns = side.N - block * 128 < 128 ? side.N - block * 128 : 128;
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        // by way of LDS, so that neighbouring lanes write neighbouring values
        wave_order();
#pragma unroll
        for (int v = 0; v < 4; ++v)
#pragma unroll
            for (int i = 0; i < 8; i += 4)
                *reinterpret_cast<v4f *>(tile + (4 * q + v) * 128 + 8 * c + i) = v4f{acc[r][i][v], acc[r][i + 1][v], acc[r][i + 2][v], acc[r][i + 3][v]};
        wave_order();
        const int at = (chunk * RT + r) * 16, rows = p.a.rank - at < 16 ? p.a.rank - at : 16;
        const int64_t corner = (int64_t)at * side.N + block * 128;
        if (pieces > 1) {
            float *to = side.partials + (int64_t)part * p.a.rank * side.N + corner;
            const int i = lane % 32 * 4;
#pragma unroll
            for (int two = 0; two < 8; ++two) {
                const int row = 2 * two + lane / 32;
                const v4f v = *reinterpret_cast<const v4f *>(tile + row * 128 + i);
                if (row >= rows) continue;
                if (i + 4 <= columns) {
                    reinterpret_cast<Loose<4> *>(to + (int64_t)row * side.N + i)->v = __builtin_bit_cast(u32x4, v);
                } else {
#pragma unroll
                    for (int e = 0; e < 3; ++e)
                        if (i + e < columns) to[(int64_t)row * side.N + i + e] = v[e];
                }
            }
        } else {
            for (int row = 0; row < rows; ++row)
                for (int i = lane; i < columns; i += 64) write_grad(p, side, a, n, corner + (int64_t)row * side.N + i, tile[row * 128 + i]);
        }
    }
}

template <class X, class D, int RT>
__global__ __launch_bounds__(256, (X::BYTES < 4 && D::BYTES < 4 ? 4 : 3) - RT) void outer_kernel(const OuterParams p)
{
    __shared__ __attribute__((aligned(16))) float tiles[4][16 * 128];
    float *tile = tiles[threadIdx.x >> 6];
    const int blocks = p.side[0].column_blocks + p.side[1].column_blocks;
    const ColumnTask at(blockIdx.x, blocks, __builtin_amdgcn_readfirstlane(threadIdx.x >> 6));
    const int block = at.block, chunk = at.row % p.rank_chunks, task = at.row / p.rank_chunks;
    if (task >= p.plan.tasks_most || block >= blocks) return;
    const int4 what = p.plan.tasks[task];
    const int a = __builtin_amdgcn_readfirstlane(what.x), first = __builtin_amdgcn_readfirstlane(what.y), last = __builtin_amdgcn_readfirstlane(what.z);
    const int pieces = __builtin_amdgcn_readfirstlane(what.w);
    if (a < 0 || (first == last && p.accumulate)) return;
    auto run = [&](auto y, const OuterSide &side, int at) __attribute__((always_inline)) {
        if (at * 128 + 128 > side.N) outer<decltype(y), RT>(p, side, at, chunk, a, first, last, pieces, tile, std::true_type());
        else outer<decltype(y), RT>(p, side, at, chunk, a, first, last, pieces, tile, std::false_type());
    };
    if (block < p.side[0].column_blocks) run(X(), p.side[0], block);
    else run(D(), p.side[1], block - p.side[0].column_blocks);
}

// Adds up the pieces of the adapters that have several, in their order
__global__ __launch_bounds__(256) void outer_join_kernel(const OuterParams p)
{
    const int columns = p.side[0].column_blocks ? p.side[0].N : 0;
    const int64_t values0 = (int64_t)p.a.rank * columns, values = values0 + (p.side[1].column_blocks ? (int64_t)p.a.rank * p.side[1].N : 0);
    const unsigned blocks = (unsigned)((values + 255) / 256);
    const int a = (int)(blockIdx.x / blocks);
    const int start = p.plan.starts[a], count = p.plan.starts[a + 1] - start;
    if (count <= p.plan.piece) return;
    const int pieces = (count + p.plan.piece - 1) / p.plan.piece;
    int64_t i = (int64_t)(blockIdx.x - (unsigned)a * blocks) * 256 + threadIdx.x;
    if (i >= values) return;
    const bool second = i >= values0;
    const OuterSide &side = p.side[second];
    i -= second ? values0 : 0;
    const int64_t step = (int64_t)p.a.rank * side.N;
    const float *from = side.partials + (int64_t)(2 * (start / p.plan.piece)) * step + i;
    float sum = 0.0f;
    int j = 0;
    for (; j + 8 <= pieces; j += 8) {
        float v[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = from[(j + k) * step];
#pragma unroll
        for (int k = 0; k < 8; ++k) sum += v[k];
    }
    for (; j < pieces; ++j) sum += from[j * step];
    write_grad(p, side, a, count, i, sum);
}

void launch_outer_kernel(const OuterParams &p, int x_dtype, int dy_dtype, unsigned workgroups, hipStream_t st)
{
    auto with_rows = [](int dtype, auto &&f) {
        if (dtype == MKQ_I8) f(Codes());
        else with_elem(dtype, f);
    };
    with_rows(x_dtype, [&](auto x) {
        with_elem(dy_dtype, [&](auto y) {
            if (outer_tiles(p.a.rank) == 1) outer_kernel<decltype(x), decltype(y), 1><<<workgroups, 256, 0, st>>>(p);
            else outer_kernel<decltype(x), decltype(y), 2><<<workgroups, 256, 0, st>>>(p);
        });
    });
}

void launch_outer_join_kernel(const OuterParams &p, unsigned workgroups, hipStream_t st) { outer_join_kernel<<<workgroups, 256, 0, st>>>(p); }

}  // namespace mkq
