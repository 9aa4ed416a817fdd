// Shared by the kernels of the low-rank adapters and their host side.
#pragma once

#include "gemm_common.h"
#include "neighbours.h"

namespace mkq {

typedef float v4f __attribute__((ext_vector_type(4)));
typedef __bf16 v8b __attribute__((ext_vector_type(8)));

struct AdapterParams {
    const int32_t *adapter;
    const float *scales;  // [R], or NULL: 1
    int64_t M;
    int R, rank, pitch, splits;  // pitch: rank rounded up to eight
};
__device__ __forceinline__ float scale_of(const AdapterParams &p, int a) { return p.scales ? p.scales[a] : 1.0f; }
// The adapter of a row, -1 for none
__device__ __forceinline__ int adapter_of(const AdapterParams &p, int64_t row)
{
    if (row >= p.M) return -1;
    const int a = p.adapter[row];
    return a >= 0 && a < p.R ? a : -1;
}

// The adapters that lanes have (-1: none), each with its lanes as bits, in the order of the first lanes: those whose number is `slot`
// modulo `slots`, and for the first slot the lanes of `none` as an adapter of -1
struct Adapters {
    uint64_t left, none;
    int mine, turn, slots;
    __device__ __forceinline__ Adapters(int mine, int slot, int slots, bool none)
        : left(__ballot(mine >= 0)), none(slot == 0 ? __ballot(none) : 0), mine(mine), turn(slot), slots(slots) {}
    __device__ __forceinline__ bool next(int &a, uint64_t &lanes)
    {
        while (left) {
            a = __builtin_amdgcn_readlane(mine, __builtin_ctzll(left));
            lanes = __ballot(mine == a);
            left &= ~lanes;
            if (turn == 0) {
                turn = slots - 1;
                return true;
            }
            --turn;
        }
        a = -1;
        lanes = none;
        none = 0;
        return lanes != 0;
    }
};

// ---- numbers as parts -----------------------------------------------------------------------------------------------------
__device__ __forceinline__ uint32_t upper_halves(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x07060302u); }
__device__ __forceinline__ uint32_t lower_halves(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x05040100u); }
// x = sum of PARTS bfloat16 numbers, each the nearest to what is left: of three nothing is left, two leave 2^-17 of x.  (Cut off instead of rounded they
// left up to 2^-15, always with the sign of x.)  The largest of them are the first part of what lies above; nothing is left of an infinity or a NaN.
// HALVES: values of binary16, of which 2^8 is left at most (and of an infinity or a NaN something finite: beside the first part it makes no difference)
template <bool HALVES = false, int PARTS>
__device__ __forceinline__ void parts_of(const float (&x)[8], uint4 (&out)[PARTS])
{
    constexpr float MOST = 0x1.FEp127f;  // bfloat16's
    float left[8];
    bool finite[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        finite[i] = HALVES || fabsf(x[i]) < __builtin_inff();
        left[i] = !HALVES && finite[i] ? __builtin_amdgcn_fmed3f(x[i], -MOST, MOST) : x[i];
    }
#pragma unroll
    for (int p = 0; p < PARTS; ++p) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = pack2_bf16(left[2 * i], left[2 * i + 1]);
        out[p] = make_uint4(w[0], w[1], w[2], w[3]);
        if (p + 1 == PARTS) break;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float part = __uint_as_float(i % 2 ? w[i / 2] & 0xFFFF0000u : w[i / 2] << 16);
            if (HALVES) left[i] = __builtin_amdgcn_fmed3f(left[i] - part, -0x1p8f, 0x1p8f);
            else left[i] = p == 0 ? (finite[i] ? x[i] - part : 0.0f) : left[i] - part;
        }
    }
}
template <class E> struct Parts { static constexpr int N = 3; };
template <> struct Parts<ElemF16> { static constexpr int N = 2; };
template <> struct Parts<ElemBF16> { static constexpr int N = 1; };
template <> struct Parts<Codes> { static constexpr int N = 3; };
__device__ __forceinline__ v4f multiply(uint4 a, uint4 b, v4f c)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8b, a), __builtin_bit_cast(v8b, b), c, 0, 0, 0);
}
// Products of parts, the small ones first; those of places DEEP or more are left out
template <int DEEP, int PA, int PB>
__device__ __forceinline__ v4f multiply(const uint4 (&a)[PA], const uint4 (&b)[PB], v4f c)
{
#pragma unroll
    for (int sum = PA + PB - 2; sum >= 0; --sum)
#pragma unroll
        for (int i = 0; i < PA; ++i)
            if (sum < DEEP && sum - i >= 0 && sum - i < PB) c = multiply(a[i], b[sum - i], c);
    return c;
}

// A number that the compiler takes for new where it stands: what follows from it is computed there again, not kept in registers around a loop
__device__ __forceinline__ int fresh(int v)
{
    asm volatile("" : "+v"(v));
    return v;
}

// ---- the batch's rows by adapter -------------------------------------------------------------------------------------------
// order: rows with an adapter, sorted by it, in the batch's order; starts [R + 1].  An adapter's rows are summed in pieces of
// `piece` rows: task starts[a] / piece + a + j has the j-th (no two adapters' tasks meet, as starts grow by an adapter's rows).
struct PlanParams {
    int piece, tasks_most;
    int32_t *order, *starts;
    int4 *tasks;  // [tasks_most] adapter (-1: nothing to do), first and last place in order, pieces of the adapter
};
__device__ __forceinline__ int task_of(int start, int a, int piece) { return start / piece + a; }

// Blocks of 128 columns, four neighbours of a `row` of blocks a workgroup.  (Whole rows to the XCDs in turn took as long: 8192 x 4096 bfloat16 with its
// base 30.3 and 30.3 us.)
struct ColumnTask {
    int row, block;
    __device__ __forceinline__ ColumnTask(unsigned workgroup, int column_blocks, int wave)
    {
        const unsigned parts = (unsigned)(column_blocks + 3) / 4;
        row = (int)(workgroup / parts);  // (a grid has fewer than 2^24 workgroups)
        block = (int)(workgroup % parts) * 4 + wave;
    }
    static int64_t workgroups(int64_t rows, int64_t column_blocks) { return rows * ((column_blocks + 3) / 4); }
};

// ---- what the kernels take ------------------------------------------------------------------------------------------------
struct ShrinkParams {
    AdapterParams a;
    const void *x, *w;  // [M, K] of stride ldx, [R, rank, K]
    int64_t ldx;
    int K;
    int slots;          // workgroups that share a tile's adapters
    int rank_chunks;
    bool scaled;        // times the adapter's scale
    float *t;           // [splits, M, pitch], zeros behind the rank
    float *hidden;      // [M, rank], or NULL: the same
    int plans;          // workgroups in front that put the rows in order
    PlanParams plan;
};

struct ExpandParams {
    AdapterParams a;
    const float *t;   // [splits, M, pitch]
    const void *w;    // [R, rank, N]
    const void *base; // [M, N], or NULL
    void *out;
    int64_t ld_base, ld_out;
    int N, column_blocks, slots, row_groups;
    bool scaled;      // t is still to be multiplied by the adapter's scale
    bool keep_scaled; // ... as it is kept
    float *keep;      // [M, keep_pitch], or NULL: what the splits add up to
    int keep_pitch;
};

struct OuterSide {
    const float *coeff;  // [M, coeff_pitch]
    const void *y;       // [M, N] of stride ld
    const float *steps;  // of rows kept in 8 bits: [M, groups]
    int64_t ld;
    int coeff_pitch, N, column_blocks, groups, group_shift;
    bool scaled;         // the result is multiplied by the adapter's scale
    float *partials;     // [parts, rank, N]
    void *grad;          // [R, rank, N]
};
struct OuterParams {
    AdapterParams a;
    OuterSide side[2];  // d_down's and d_up's, without columns if not wanted
    int rank_chunks, grad_dtype;
    bool accumulate;
    PlanParams plan;
};
// Columns of eight rows as the matrix unit takes them: of eight rows' neighbours in lanes (c, q), tile i has the columns 8 c + i
template <class E>
struct Block {
    Neighbours<E> rows[8];
    __device__ __forceinline__ void column(int i, uint4 (&out)[Parts<E>::N]) const
    {
        if constexpr (std::is_same<E, ElemBF16>::value) {
            uint32_t w[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint32_t a = rows[2 * j].w[0][i / 2], b = rows[2 * j + 1].w[0][i / 2];
                w[j] = i % 2 ? upper_halves(a, b) : lower_halves(a, b);
            }
            out[0] = make_uint4(w[0], w[1], w[2], w[3]);
        } else {
            float v[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = rows[j].get(i);
            parts_of<std::is_same<E, ElemF16>::value>(v, out);
        }
    }
};

// ---- rows by way of LDS ----------------------------------------------------------------------------------------------------
template <class E>
__device__ __forceinline__ void operand(const Neighbours<E> &n, uint4 (&out)[Parts<E>::N])
{
    if constexpr (std::is_same<E, ElemBF16>::value) {
        out[0] = __builtin_bit_cast(uint4, n.w[0]);
    } else {
        float v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = n.get(i);
        parts_of<std::is_same<E, ElemF16>::value>(v, out);
    }
}

// Places of a row that a wave multiplies at a time: 256 bytes of the larger elements
constexpr int shrink_step(int x_bytes, int w_bytes) { return x_bytes == 4 || w_bytes == 4 ? 64 : 128; }

// Sixteen rows of a step on their way from memory to LDS: neighbouring lanes fetch neighbouring pieces of 16 bytes of a row.  (Fetched as
// the matrix unit takes them, a row a lane, every lane asked for a line of its own: dy of 8192 x 4096 bfloat16 32 instead of 17 us.)  In LDS piece i of row r is
// at i ^ r, so that sixteen rows' same pieces, and a row's sixteen pieces, are on different banks.
template <class E, int STEP>
struct ShrinkRows {
    static constexpr int PIECES = STEP * E::BYTES / 16, N = PIECES / 4;  // of a row, of a lane
    static constexpr int BYTES = 16 * STEP * E::BYTES;
    u32x4 v[N];
    __device__ static __forceinline__ int row_of(int i) { return (64 * i + (int)(threadIdx.x & 63)) / PIECES; }
    __device__ static __forceinline__ int piece_of() { return (threadIdx.x & 63) % PIECES; }
    __device__ __forceinline__ void put(uint8_t *lds) const
    {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int r = row_of(i);
            *reinterpret_cast<u32x4 *>(lds + (r * PIECES + (piece_of() ^ (r % PIECES))) * 16) = v[i];
        }
    }
    // lane (c, q): eight places from 32 h + 8 q on of row c
    __device__ static __forceinline__ Neighbours<E> get(const uint8_t *lds, int h)
    {
        const int c = threadIdx.x & 15, q = (threadIdx.x & 63) >> 4;
        Neighbours<E> n;
#pragma unroll
        for (int i = 0; i < E::BYTES / 2; ++i) {
            const int piece = (4 * h + q) * (E::BYTES / 2) + i;
            n.w[i] = *reinterpret_cast<const u32x4 *>(lds + (c * PIECES + (piece ^ (c % PIECES))) * 16);
        }
        return n;
    }
};

// Launches of what the params hold; the sources are compiled side by side
inline int rank_tiles(int rank) { return rank <= 16 ? 1 : rank <= 32 ? 2 : 4; }  // of 16, a workgroup's
void launch_shrink_kernel(const ShrinkParams &p, int x_dtype, int w_dtype, unsigned workgroups, hipStream_t st);
// shrink and expand of few rows in one launch
void launch_few_kernel(const ShrinkParams &s, const ExpandParams &e, int x_dtype, int w_dtype, int out_dtype, unsigned workgroups, hipStream_t st);
void launch_expand_kernel(const ExpandParams &p, int w_dtype, int out_dtype, unsigned workgroups, hipStream_t st);
inline int outer_tiles(int rank) { return rank <= 16 ? 1 : 2; }
void launch_outer_kernel(const OuterParams &p, int x_dtype, int dy_dtype, unsigned workgroups, hipStream_t st);
void launch_outer_join_kernel(const OuterParams &p, unsigned workgroups, hipStream_t st);

}  // namespace mkq
