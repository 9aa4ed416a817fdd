// Low-rank adapters of many requests beside a shared projection, and their gradients.  Row m has the adapter a = adapter[m]:
//
//     t[m] = down_a x[m]        out[m] = base[m] + s_a up_a^T t[m]                  (down_a [rank, K], up_a [rank, N])
//     u[m] = s_a up_a dy[m]     dx[m]  = base[m] + down_a^T u[m]
//     d_down_a = sum_m u[m] x[m]^T,   d_up_a = s_a sum_m t[m] dy[m]^T
//
// Both matrices of an adapter have their long side in rows, so three kernels do all of it: `shrink` (t, u: products along rows),
// `expand` (out, dx: sums of the adapter's rows) and `outer` (sums of the batch's rows).  Bound by the bytes of x, dy, base and out; products
// are the matrix unit's.
//
// Operands enter the products exactly: binary16 and bfloat16 as they are where both sides are the same, otherwise a number is the sum of
// one to three bfloat16 parts (binary32 three, binary16 two), and products of parts whose places add up to 2^-24 or less are left out.
// Sums are binary32.  A tile of rows may hold any adapters: it is gone through once for each of them, results are taken for the rows
// that have it, so a request's infinities and NaN stay in its rows.
#include "elements.h"
#include "gemm_common.h"

namespace mkq {

typedef float v4f __attribute__((ext_vector_type(4)));
typedef __bf16 v8b __attribute__((ext_vector_type(8)));

// 16 bytes from an address that only fits their elements (the unit takes any)
template <int BYTES>
struct __attribute__((packed, aligned(BYTES))) Loose {
    u32x4 v;
};
struct Codes {  // rows kept in 8 bits
    using raw = int8_t;
    static constexpr int BYTES = 1;
};

struct AdapterParams {
    const int32_t *adapter;
    const float *scales;  // [R], or NULL: 1
    int64_t M;
    int R, rank, splits;
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
// x = sum of `parts` numbers that are the upper halves of what is left; nothing is left of an infinity, and a NaN stays one
template <int PARTS>
__device__ __forceinline__ void parts_of(const float (&x)[8], uint4 (&out)[PARTS])
{
    uint32_t left[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) left[i] = x[i] != x[i] ? 0x7FC00000u : __float_as_uint(x[i]);
#pragma unroll
    for (int p = 0; p < PARTS; ++p) {
        out[p] = make_uint4(upper_halves(left[0], left[1]), upper_halves(left[2], left[3]), upper_halves(left[4], left[5]), upper_halves(left[6], left[7]));
        if (p + 1 == PARTS) break;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float v = __uint_as_float(left[i]), r = v - __uint_as_float(left[i] & 0xFFFF0000u);
            left[i] = fabsf(v) < __builtin_inff() ? __float_as_uint(r) : 0u;
        }
    }
}
template <class E> struct Parts { static constexpr int N = 3; };
template <> struct Parts<ElemF16> { static constexpr int N = 2; };
template <> struct Parts<ElemBF16> { static constexpr int N = 1; };
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

// Eight neighbours of a row from place k on, as fetched; zeros from place `end` on
template <class E>
struct Neighbours {
    u32x4 w[E::BYTES == 4 ? 2 : 1];
    __device__ __forceinline__ void clear()
    {
#pragma unroll
        for (auto &v : w) v = u32x4{0, 0, 0, 0};
    }
    __device__ __forceinline__ void fetch(const typename E::raw *row, int64_t k, int64_t end)
    {
        const typename E::raw *at = row + k;
        if (k + 8 <= end) {
            if constexpr (E::BYTES == 1) {
                const uint2 v = *reinterpret_cast<const uint2 *>(at);
                w[0] = u32x4{v.x, v.y, 0, 0};
            } else {
                w[0] = reinterpret_cast<const Loose<E::BYTES> *>(at)->v;
                if constexpr (E::BYTES == 4) w[1] = reinterpret_cast<const Loose<4> *>(at + 4)->v;
            }
        } else {
            typename E::raw v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = k + i < end ? at[i] : typename E::raw(0);
            if constexpr (E::BYTES == 4) {
                w[0] = u32x4{__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])};
                w[1] = u32x4{__float_as_uint(v[4]), __float_as_uint(v[5]), __float_as_uint(v[6]), __float_as_uint(v[7])};
            } else if constexpr (E::BYTES == 2) {
                w[0] = u32x4{v[0] | (uint32_t)v[1] << 16, v[2] | (uint32_t)v[3] << 16, v[4] | (uint32_t)v[5] << 16, v[6] | (uint32_t)v[7] << 16};
            } else {
                uint32_t lo = 0, hi = 0;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    lo |= (uint32_t)(uint8_t)v[i] << (8 * i);
                    hi |= (uint32_t)(uint8_t)v[4 + i] << (8 * i);
                }
                w[0] = u32x4{lo, hi, 0, 0};
            }
        }
    }
    __device__ __forceinline__ float get(int i) const
    {
        if constexpr (E::BYTES == 4) return __uint_as_float(w[i / 4][i % 4]);
        else if constexpr (E::BYTES == 1) return (float)(int8_t)(w[0][i / 4] >> (8 * (i % 4)));
        else return E::get((uint16_t)(w[0][i / 2] >> (16 * (i % 2))));
    }
};

// Eight neighbours of a row from place k on, those before `end`
template <class O>
__device__ __forceinline__ void put_neighbours(typename O::raw *row, int64_t k, int64_t end, const float (&y)[8])
{
    typename O::raw *to = row + k;
    if (k + 8 > end) {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (k + e < end) to[e] = O::put(in_binary32(y[e]));
    } else if constexpr (O::BYTES == 4) {
#pragma unroll
        for (int e = 0; e < 8; e += 4)
            reinterpret_cast<Loose<4> *>(to + e)->v = u32x4{__float_as_uint(y[e]), __float_as_uint(y[e + 1]), __float_as_uint(y[e + 2]), __float_as_uint(y[e + 3])};
    } else {
        uint32_t w[4];
#pragma unroll
        for (int e = 0; e < 4; ++e)
            w[e] = std::is_same<O, ElemF16>::value ? pack2_f16(in_binary32(y[2 * e]), in_binary32(y[2 * e + 1])) : pack2_bf16(y[2 * e], y[2 * e + 1]);
        reinterpret_cast<Loose<2> *>(to)->v = u32x4{w[0], w[1], w[2], w[3]};
    }
}

// ---- shrink ---------------------------------------------------------------------------------------------------------------
struct ShrinkParams {
    AdapterParams a;
    const void *x, *w;  // [M, K] of stride ldx, [R, rank, K]
    int64_t ldx;
    int K;
    int slots;          // workgroups that share a tile's adapters
    int rank_chunks, per_split;  // steps of 64 places of a split
    bool scaled;        // times the adapter's scale
    float *t;           // [splits, M, rank]
};
constexpr int SHRINK_STEP = 64;

template <class E>
__device__ __forceinline__ void operand(const Neighbours<E> &n, uint4 (&out)[Parts<E>::N])
{
    if constexpr (std::is_same<E, ElemBF16>::value) {
        out[0] = __builtin_bit_cast(uint4, n.w[0]);
    } else {
        float v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = n.get(i);
        parts_of(v, out);
    }
}

// Tiles of 16 rows and RT * 16 of the rank; the four waves of a workgroup take steps in turn and add up through LDS
template <class X, class W, int RT>
__global__ __launch_bounds__(256) void shrink_kernel(const ShrinkParams p)
{
    __shared__ v4f sums[4][RT][64];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, c = lane & 15, q = lane >> 4;
    unsigned b = blockIdx.x;
    const int chunk = b % p.rank_chunks;
    b /= p.rank_chunks;
    const int split = b % p.a.splits;
    b /= p.a.splits;
    const int slot = b % p.slots;
    const int64_t m0 = (int64_t)(b / p.slots) * 16;
    const int mine = adapter_of(p.a, lane < 16 ? m0 + lane : p.a.M);
    const int64_t row = m0 + c < p.a.M ? m0 + c : p.a.M - 1;
    const typename X::raw *x = static_cast<const typename X::raw *>(p.x) + row * p.ldx;
    const int steps = (p.K + SHRINK_STEP - 1) / SHRINK_STEP;
    const int from = split * p.per_split, to = from + p.per_split < steps ? from + p.per_split : steps;
    float *t = p.t + (int64_t)split * p.a.M * p.a.rank;
    Adapters adapters(mine, slot, p.slots, lane < 16 && m0 + lane < p.a.M && mine < 0);
    int a;
    uint64_t same;
    while (adapters.next(a, same)) {
        if (a < 0) {  // rows without an adapter
            for (int i = 0; i < 16; ++i)
                if (same >> i & 1)
                    for (int r = chunk * RT * 16 + (int)threadIdx.x; r < p.a.rank && r < (chunk + 1) * RT * 16; r += 256) t[(m0 + i) * p.a.rank + r] = 0.0f;
            continue;
        }
        v4f acc[RT];
        const typename W::raw *w[RT];
        bool real[RT];
#pragma unroll
        for (int r = 0; r < RT; ++r) {
            const int at = (chunk * RT + r) * 16 + c;
            acc[r] = v4f{0, 0, 0, 0};
            real[r] = at < p.a.rank;
            w[r] = static_cast<const typename W::raw *>(p.w) + ((int64_t)a * p.a.rank + (real[r] ? at : 0)) * p.K;
        }
        for (int s = from + wave; s < to; s += 4) {
            Neighbours<X> xs[2];
            Neighbours<W> ws[2][RT];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int k = s * SHRINK_STEP + h * 32 + q * 8;
                xs[h].clear();
                if (k < p.K) xs[h].fetch(x, k, p.K);
#pragma unroll
                for (int r = 0; r < RT; ++r) {
                    ws[h][r].clear();
                    if (k < p.K && real[r]) ws[h][r].fetch(w[r], k, p.K);
                }
            }
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                if constexpr (std::is_same<X, ElemF16>::value && std::is_same<W, ElemF16>::value) {
#pragma unroll
                    for (int r = 0; r < RT; ++r)
                        acc[r] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(v8h, xs[h].w[0]), __builtin_bit_cast(v8h, ws[h][r].w[0]), acc[r], 0, 0, 0);
                } else {
                    uint4 xp[Parts<X>::N], wp[Parts<W>::N];
                    operand(xs[h], xp);
#pragma unroll
                    for (int r = 0; r < RT; ++r) {
                        operand(ws[h][r], wp);
                        acc[r] = multiply<3>(xp, wp, acc[r]);
                    }
                }
            }
        }
#pragma unroll
        for (int r = 0; r < RT; ++r) sums[wave][r][lane] = acc[r];
        __syncthreads();
        const float scale = p.scaled ? scale_of(p.a, a) : 1.0f;
        for (int r = wave; r < RT; r += 4) {
            const v4f sum = (sums[0][r][lane] + sums[1][r][lane]) + (sums[2][r][lane] + sums[3][r][lane]);
            const int at = (chunk * RT + r) * 16 + c;
#pragma unroll
            for (int v = 0; v < 4; ++v)
                if (at < p.a.rank && (same >> (4 * q + v) & 1)) t[(m0 + 4 * q + v) * p.a.rank + at] = sum[v] * scale;
        }
        __syncthreads();
    }
}

// ---- expand ---------------------------------------------------------------------------------------------------------------
struct ExpandParams {
    AdapterParams a;
    const float *t;   // [splits, M, rank]
    const void *w;    // [R, rank, N]
    const void *base; // [M, N], or NULL
    void *out;
    int64_t ld_base, ld_out;
    int N, column_blocks, slots, row_groups;
    bool scaled;      // t is still to be multiplied by the adapter's scale
    bool keep_scaled; // ... as it is kept
    float *keep;      // [M, rank], or NULL: what the splits add up to
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
            parts_of(v, out);
        }
    }
};

// t of a row from place r on, eight values, added up over the splits
__device__ __forceinline__ void hidden_values(const ExpandParams &p, int64_t row, int r, float (&v)[8])
{
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = 0.0f;
    if (r >= p.a.rank) return;
    for (int s = 0; s < p.a.splits; ++s) {
        Neighbours<ElemF32> n;
        n.fetch(p.t + ((int64_t)s * p.a.M + row) * p.a.rank, r, p.a.rank);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] += n.get(e);
    }
}

// A wave has 16 RB rows and 128 columns; lane (c, q) ends with columns 8 c .. 8 c + 7 of rows 4 q .. 4 q + 3 of every 16
template <class W, class O, int RB>
__global__ __launch_bounds__(256) void expand_kernel(const ExpandParams p)
{
    constexpr int PT = O::BYTES == 4 ? 3 : 2;  // (2^-16 of a product is left out under results of 16 bits, which end at 2^-9 or 2^-12)
    const int lane = threadIdx.x & 63, c = lane & 15, q = lane >> 4;
    int64_t task = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    const int block = (int)(task % p.column_blocks);
    task /= p.column_blocks;
    const int slot = (int)(task / p.row_groups);
    if (slot >= p.slots) return;
    const int64_t m0 = (task - (int64_t)slot * p.row_groups) * (16 * RB);
    const int mine = adapter_of(p.a, lane < 16 * RB ? m0 + lane : p.a.M);
    const int64_t n0 = (int64_t)block * 128 + 8 * c;
    Adapters adapters(mine, slot, p.slots, lane < 16 * RB && m0 + lane < p.a.M && mine < 0);
    int a;
    uint64_t same;
    while (adapters.next(a, same)) {
        v4f acc[RB][8];
#pragma unroll
        for (int b = 0; b < RB; ++b)
#pragma unroll
            for (int i = 0; i < 8; ++i) acc[b][i] = v4f{0, 0, 0, 0};
        const float scale = a < 0 ? 0.0f : scale_of(p.a, a), factor = p.scaled ? scale : 1.0f;
        const typename W::raw *w = static_cast<const typename W::raw *>(p.w) + (int64_t)(a < 0 ? 0 : a) * p.a.rank * p.N;
        if (a < 0) {  // rows without an adapter
            if (p.keep && block == 0)
                for (int i = 0; i < 16 * RB; ++i)
                    if (same >> i & 1)
                        for (int r = lane; r < p.a.rank; r += 64) p.keep[(m0 + i) * p.a.rank + r] = 0.0f;
            if (p.base == p.out) continue;
        }
        for (int r0 = 0; a >= 0 && r0 < p.a.rank; r0 += 32) {
            const int r = r0 + 8 * q;
            Block<W> block_w;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                block_w.rows[e].clear();
                if (r + e < p.a.rank && n0 < p.N) block_w.rows[e].fetch(w + (int64_t)(r + e) * p.N, n0, p.N);
            }
            uint4 tp[RB][PT];
#pragma unroll
            for (int b = 0; b < RB; ++b) {
                const int64_t row = m0 + 16 * b + c < p.a.M ? m0 + 16 * b + c : p.a.M - 1;
                float v[8];
                hidden_values(p, row, r, v);
                const bool kept = p.keep && block == 0 && (same >> (16 * b + c) & 1);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float s = v[e] * factor;
                    if (kept && r + e < p.a.rank) p.keep[row * p.a.rank + r + e] = p.keep_scaled ? s : v[e];
                    v[e] = s;
                }
                parts_of(v, tp[b]);
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                uint4 wp[Parts<W>::N];
                block_w.column(i, wp);
#pragma unroll
                for (int b = 0; b < RB; ++b) acc[b][i] = multiply<PT>(tp[b], wp, acc[b][i]);
            }
        }
        if (n0 >= p.N) continue;
#pragma unroll
        for (int b = 0; b < RB; ++b)
#pragma unroll
            for (int v = 0; v < 4; ++v) {
                const int i = 16 * b + 4 * q + v;
                if (same >> i & 1) {
                    float y[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) y[e] = acc[b][e][v];
                    if (p.base) {
                        Neighbours<O> n;
                        n.fetch(static_cast<const typename O::raw *>(p.base) + (m0 + i) * p.ld_base, n0, p.N);
#pragma unroll
                        for (int e = 0; e < 8; ++e) y[e] += n.get(e);
                    }
                    put_neighbours<O>(static_cast<typename O::raw *>(p.out) + (m0 + i) * p.ld_out, n0, p.N, y);
                }
            }
    }
}

// ---- the batch's rows by adapter -------------------------------------------------------------------------------------------
// order: rows with an adapter, sorted by it, in the batch's order; starts [R + 1].  An adapter's rows are summed in pieces of
// `piece` rows: task starts[a] / piece + a + j has the j-th (no two adapters' tasks meet, as starts grow by an adapter's rows).
struct PlanParams {
    AdapterParams a;
    int piece;
    int32_t *order, *starts;
    int4 *tasks;  // [tasks_most] adapter (-1: nothing to do), first and last place in order, pieces of the adapter
    int tasks_most;
};
__device__ __forceinline__ int task_of(int start, int a, int piece) { return start / piece + a; }

// A workgroup has an adapter: each thread looks through neighbouring rows for those of the adapter and those of smaller ones
__global__ __launch_bounds__(1024) void plan_kernel(const PlanParams p)
{
    __shared__ int equal_before[16], less_before[16];
    const int a = blockIdx.x, wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int each = (int)((p.a.M + 1023) / 1024);
    const int64_t from = (int64_t)threadIdx.x * each, to = from + each < p.a.M ? from + each : p.a.M;
    int equal = 0, less = 0;
    for (int64_t m = from; m < to; ++m) {
        const int b = p.a.adapter[m];
        equal += b == a;
        less += b >= 0 && b < a;
    }
    int before = equal, all_less = less;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
        const int v = __shfl_up(before, off, 64);
        if (lane >= off) before += v;
        all_less += __shfl_xor(all_less, off, 64);
    }
    if (lane == 63) {
        equal_before[wave] = before;
        less_before[wave] = all_less;
    }
    __syncthreads();
    int start = 0, waves_before = 0, count = 0;
    for (int w = 0; w < 16; ++w) {
        start += less_before[w];
        if (w < wave) waves_before += equal_before[w];
        count += equal_before[w];
    }
    int at = start + waves_before + before - equal;
    for (int64_t m = from; m < to; ++m)
        if (p.a.adapter[m] == a) p.order[at++] = (int32_t)m;
    if (threadIdx.x == 0) {
        p.starts[a] = start;
        if (a == p.a.R - 1) p.starts[p.a.R] = start + count;
    }
    // (behind the last adapter's: fewer rows than the batch's may have an adapter)
    const int first = task_of(start, a, p.piece), next = a + 1 < p.a.R ? task_of(start + count, a + 1, p.piece) : p.tasks_most;
    const int pieces = count ? (count + p.piece - 1) / p.piece : 1;
    for (int i = first + (int)threadIdx.x; i < next; i += 1024) {
        const int j = i - first, last = (j + 1) * p.piece < count ? (j + 1) * p.piece : count;
        p.tasks[i] = j < pieces ? make_int4(a, start + j * p.piece, start + last, pieces) : make_int4(-1, 0, 0, 0);
    }
}

// ---- outer ----------------------------------------------------------------------------------------------------------------
struct OuterParams {
    AdapterParams a;
    const float *coeff;  // [M, rank]
    const void *y;       // [M, N] of stride ld
    const float *steps;  // of rows kept in 8 bits: [M, groups]
    int64_t ld;
    int N, column_blocks, rank_chunks, groups, group_shift, piece;
    bool scaled;         // the result is multiplied by the adapter's scale
    bool accumulate;
    const int32_t *order, *starts;
    const int4 *tasks;
    int tasks_most;
    float *partials;     // [parts, rank, N]
    void *grad;          // [R, rank, N]
};
template <> struct Parts<Codes> { static constexpr int N = 3; };

template <class O>
__device__ __forceinline__ void write_grad(const OuterParams &p, int a, int r, int64_t n, float v)
{
    typename O::raw *at = static_cast<typename O::raw *>(p.grad) + ((int64_t)a * p.a.rank + r) * p.N + n;
    v *= p.scaled ? scale_of(p.a, a) : 1.0f;
    if (p.accumulate) v += O::get(*at);
    *at = O::put(in_binary32(v));
}

// A wave has a piece of an adapter's rows, 128 columns and RT * 16 of the rank: 32 rows a step, lane (c, q) fetches eight neighbouring columns
// of eight of them
template <class Y, class O, int RT>
__global__ __launch_bounds__(256) void outer_kernel(const OuterParams p)
{
    const int lane = threadIdx.x & 63, c = lane & 15, q = lane >> 4;
    int64_t task = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    const int block = (int)(task % p.column_blocks);
    task /= p.column_blocks;
    const int chunk = (int)(task % p.rank_chunks);
    task /= p.rank_chunks;
    if (task >= p.tasks_most) return;
    const int4 what = p.tasks[task];
    const int a = __builtin_amdgcn_readfirstlane(what.x), first = __builtin_amdgcn_readfirstlane(what.y), last = __builtin_amdgcn_readfirstlane(what.z);
    const int pieces = __builtin_amdgcn_readfirstlane(what.w);
    if (a < 0) return;
    if (first == last && p.accumulate) return;
    const int64_t n0 = (int64_t)block * 128 + 8 * c;
    v4f acc[RT][8];
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int i = 0; i < 8; ++i) acc[r][i] = v4f{0, 0, 0, 0};
    for (int s = first; s < last; s += 32) {
        Block<Y> y;
        float step[8], coeff[RT][8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            // behind the last row: that row again, times 0
            const int place = s + 8 * q + e;
            const int64_t row = p.order[place < last ? place : last - 1];
            y.rows[e].clear();
            if (n0 < p.N) {
                y.rows[e].fetch(static_cast<const typename Y::raw *>(p.y) + row * p.ld, n0, p.N);
                if constexpr (Y::BYTES == 1) step[e] = p.steps[row * p.groups + (n0 >> p.group_shift)];
            } else {
                step[e] = 0.0f;
            }
#pragma unroll
            for (int r = 0; r < RT; ++r) {
                const int at = (chunk * RT + r) * 16 + c;
                coeff[r][e] = place < last && at < p.a.rank ? p.coeff[row * p.a.rank + at] : 0.0f;
            }
        }
        uint4 cp[RT][3];
#pragma unroll
        for (int r = 0; r < RT; ++r) parts_of(coeff[r], cp[r]);
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
    const int start = p.starts[a], part = 2 * (start / p.piece) + (first - start) / p.piece;
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int v = 0; v < 4; ++v) {
            const int at = (chunk * RT + r) * 16 + 4 * q + v;
            if (at >= p.a.rank) continue;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                if (n0 + i >= p.N) continue;
                if (pieces > 1) p.partials[((int64_t)part * p.a.rank + at) * p.N + n0 + i] = acc[r][i][v];
                else write_grad<O>(p, a, at, n0 + i, acc[r][i][v]);
            }
        }
}

// Adds up the pieces of the adapters that have several, in their order
template <class O>
__global__ __launch_bounds__(256) void outer_join_kernel(const OuterParams p)
{
    const int64_t values = (int64_t)p.a.rank * p.N;
    const unsigned blocks = (unsigned)((values + 1023) / 1024);
    const int a = (int)(blockIdx.x / blocks);
    const int start = p.starts[a], count = p.starts[a + 1] - start;
    if (count <= p.piece) return;
    const int pieces = (count + p.piece - 1) / p.piece;
    const float *from = p.partials + (int64_t)(2 * (start / p.piece)) * values;
    const int64_t first = (int64_t)(blockIdx.x - (unsigned)a * blocks) * 1024 + threadIdx.x;
    for (int u = 0; u < 4; ++u) {
        const int64_t i = first + u * 256;
        if (i >= values) return;
        float sum = 0.0f;
        for (int j = 0; j < pieces; ++j) sum += from[j * values + i];
        const int r = (int)(i / p.N);
        write_grad<O>(p, a, r, i - (int64_t)r * p.N, sum);
    }
}

// ---- host side ------------------------------------------------------------------------------------------------------------
constexpr int64_t ADAPTERS_MOST = 0x3FFFFF, SIDES_MOST = 0x7FFFFF00;
constexpr int RANK_MOST = 256;
constexpr int FEW_ROWS = 512;  // up to here a tile's adapters are shared out among workgroups

struct AdapterShape {
    int64_t M, K, N, R;
    int rank;
};
static int check_shape(const AdapterShape &d)
{
    if (d.M < 0 || d.K <= 0 || d.N <= 0 || d.R <= 0 || d.rank <= 0) return MKQ_ERR_SHAPE;
    if (d.M > SIDES_MOST || d.K > SIDES_MOST || d.N > SIDES_MOST || d.R > ADAPTERS_MOST || d.rank > RANK_MOST) return MKQ_ERR_UNSUPPORTED;
    return MKQ_OK;
}

static int least(int64_t a, int64_t b) { return (int)(a < b ? a : b); }
static int slots_of(const AdapterShape &d) { return d.M <= FEW_ROWS ? least(least(16, d.M), d.R) : 1; }
static int rank_tiles(int rank) { return rank <= 16 ? 1 : rank <= 32 ? 2 : 4; }
// Workgroups that share the places of a row: about 512 of them in all, four steps each at least
static int splits_of(const AdapterShape &d, int64_t side)
{
    const int64_t steps = ceil_div(side, SHRINK_STEP), groups = ceil_div(d.M, 16) * slots_of(d) * ceil_div(d.rank, 16 * rank_tiles(d.rank));
    int64_t n = groups == 0 || groups >= 512 ? 1 : 512 / groups;
    if (n > ceil_div(steps, 4)) n = ceil_div(steps, 4);
    if (n > 16) n = 16;
    return (int)ceil_div(steps, ceil_div(steps, n));
}

template <class F>
static void with_tiles(int tiles, F &&f)
{
    if (tiles == 1) f(std::integral_constant<int, 1>());
    else if (tiles == 2) f(std::integral_constant<int, 2>());
    else f(std::integral_constant<int, 4>());
}

static int launch_shrink(const AdapterShape &d, const AdapterParams &a, const void *x, int x_dtype, int64_t ldx, const void *w, int w_dtype, int64_t side,
                         bool scaled, float *t, hipStream_t st)
{
    const int tiles = rank_tiles(d.rank);
    const ShrinkParams p = {a, x, w, ldx, (int)side, slots_of(d), (int)ceil_div(d.rank, 16 * tiles), (int)ceil_div(ceil_div(side, SHRINK_STEP), a.splits), scaled, t};
    const int64_t workgroups = ceil_div(d.M, 16) * p.slots * a.splits * p.rank_chunks;
    if (!grid_ok(workgroups, 256)) return MKQ_ERR_UNSUPPORTED;
    with_elem(x_dtype, [&](auto x_e) {
        with_elem(w_dtype, [&](auto w_e) {
            with_tiles(tiles, [&](auto n) { shrink_kernel<decltype(x_e), decltype(w_e), decltype(n)::value><<<(unsigned)workgroups, 256, 0, st>>>(p); });
        });
    });
    return launch_status();
}

static int launch_expand(const AdapterShape &d, ExpandParams p, int w_dtype, int out_dtype, hipStream_t st)
{
    const int rows = d.M <= FEW_ROWS * 4 ? 16 : 64;
    p.column_blocks = (int)ceil_div(p.N, 128);
    p.row_groups = (int)ceil_div(d.M, rows);
    p.slots = slots_of(d);
    const int64_t workgroups = ceil_div((int64_t)p.column_blocks * p.row_groups * p.slots, 4);
    if (!grid_ok(workgroups, 256)) return MKQ_ERR_UNSUPPORTED;
    with_elem(w_dtype, [&](auto w) {
        with_elem(out_dtype, [&](auto o) {
            if (rows == 16) expand_kernel<decltype(w), decltype(o), 1><<<(unsigned)workgroups, 256, 0, st>>>(p);
            else expand_kernel<decltype(w), decltype(o), 4><<<(unsigned)workgroups, 256, 0, st>>>(p);
        });
    });
    return launch_status();
}

// Rows of a piece: about 1280 waves in all
static int piece_rows(const AdapterShape &d)
{
    const int64_t columns = ceil_div(d.K, 128) + ceil_div(d.N, 128), n = ceil_div(ceil_div(d.M * columns, 1280), 32) * 32;
    return (int)(n < 64 ? 64 : n > 2048 ? 2048 : n);
}

struct AdapterWorkspace {
    size_t t, u, order, starts, tasks, down, up, total;
    int splits, piece;
    int64_t tasks_most;
};
static AdapterWorkspace forward_workspace(const AdapterShape &d)
{
    AdapterWorkspace w = {};
    w.splits = splits_of(d, d.K);
    w.total = (size_t)w.splits * d.M * d.rank * sizeof(float);
    return w;
}
static AdapterWorkspace gradient_workspace(const AdapterShape &d)
{
    AdapterWorkspace w = {};
    auto take = [&](size_t bytes) {
        const size_t at = w.total;
        w.total += (bytes + 255) / 256 * 256;
        return at;
    };
    w.splits = splits_of(d, d.N);
    w.piece = piece_rows(d);
    w.tasks_most = d.M / w.piece + d.R;
    const size_t hidden = (size_t)d.M * d.rank * sizeof(float), parts = d.M > w.piece ? 2 * (size_t)(d.M / w.piece) + 2 : 0;
    w.t = take(w.splits > 1 ? hidden * w.splits : 0);
    w.u = take(hidden);
    w.order = take((size_t)d.M * sizeof(int32_t));
    w.starts = take((size_t)(d.R + 1) * sizeof(int32_t));
    w.tasks = take((size_t)w.tasks_most * sizeof(int4));
    w.down = take(parts * d.rank * d.K * sizeof(float));
    w.up = take(parts * d.rank * d.N * sizeof(float));
    return w;
}

template <class F>
static void with_rows(int dtype, F &&f)
{
    if (dtype == MKQ_I8) f(Codes());
    else with_elem(dtype, f);
}

static int launch_outer(const AdapterShape &d, OuterParams p, int y_dtype, int grad_dtype, hipStream_t st)
{
    p.column_blocks = (int)ceil_div(p.N, 128);
    const int tiles = d.rank <= 16 ? 1 : 2;
    p.rank_chunks = (int)ceil_div(d.rank, 16 * tiles);
    const int64_t workgroups = ceil_div((int64_t)p.tasks_most * p.column_blocks * p.rank_chunks, 4);
    const int64_t joins = d.R * ceil_div((int64_t)d.rank * p.N, 1024);
    if (!grid_ok(workgroups, 256) || !grid_ok(joins, 256)) return MKQ_ERR_UNSUPPORTED;
    with_rows(y_dtype, [&](auto y) {
        with_elem(grad_dtype, [&](auto o) {
            if (tiles == 1) outer_kernel<decltype(y), decltype(o), 1><<<(unsigned)workgroups, 256, 0, st>>>(p);
            else outer_kernel<decltype(y), decltype(o), 2><<<(unsigned)workgroups, 256, 0, st>>>(p);
            if (d.M > p.piece) outer_join_kernel<decltype(o)><<<(unsigned)joins, 256, 0, st>>>(p);
        });
    });
    return launch_status();
}

}  // namespace mkq

using namespace mkq;

extern "C" size_t mkq_low_rank_adapters_workspace_bytes(int64_t M, int64_t K, int64_t N, int rank, int64_t R)
{
    const AdapterShape d = {M, K, N, R, rank};
    return check_shape(d) != MKQ_OK || M == 0 ? 0 : forward_workspace(d).total;
}

extern "C" int mkq_low_rank_adapters(const void *x, int x_dtype, int64_t ldx, const int32_t *adapter, int64_t M, int64_t K, int64_t N, int rank,
                                     int64_t R, const void *down, const void *up, int w_dtype, const float *scales, const void *base, int64_t ld_base,
                                     void *out, int out_dtype, int64_t ld_out, float *hidden, void *workspace, size_t workspace_bytes, void *stream)
{
    if (!is_float_dtype(x_dtype) || !is_float_dtype(w_dtype) || !is_float_dtype(out_dtype)) return MKQ_ERR_DTYPE;
    const AdapterShape d = {M, K, N, R, rank};
    int status = check_shape(d);
    if (status == MKQ_ERR_SHAPE || ldx < K || ld_out < N || (base && ld_base < N)) return MKQ_ERR_SHAPE;
    if (M == 0) return MKQ_OK;
    if (!x || !adapter || !down || !up || !out) return MKQ_ERR_NULL;
    if (!aligned16(x) || !aligned4(adapter) || !aligned16(down) || !aligned16(up) || !aligned4(scales) || !aligned16(base) || !aligned16(out) || !aligned4(hidden))
        return MKQ_ERR_ALIGN;
    if (status != MKQ_OK) return status;
    if (base && !in_place_or_apart(base, out_dtype, ld_base, out, out_dtype, ld_out, M, N)) return MKQ_ERR_UNSUPPORTED;
    const AdapterWorkspace w = forward_workspace(d);
    if (!workspace || workspace_bytes < w.total) return MKQ_ERR_WORKSPACE;
    if (!aligned16(workspace)) return MKQ_ERR_ALIGN;
    const hipStream_t st = as_stream(stream);
    const AdapterParams a = {adapter, scales, M, (int)R, rank, w.splits};
    float *t = w.splits == 1 && hidden ? hidden : static_cast<float *>(workspace);
    status = launch_shrink(d, a, x, x_dtype, ldx, down, w_dtype, K, false, t, st);
    if (status != MKQ_OK) return status;
    ExpandParams e = {a, t, up, base, out, ld_base, ld_out, (int)N, 0, 0, 0, true, false, w.splits > 1 ? hidden : nullptr};
    return launch_expand(d, e, w_dtype, out_dtype, st);
}

extern "C" size_t mkq_low_rank_adapters_gradient_workspace_bytes(int64_t M, int64_t K, int64_t N, int rank, int64_t R)
{
    const AdapterShape d = {M, K, N, R, rank};
    return check_shape(d) != MKQ_OK ? 0 : gradient_workspace(d).total;
}

extern "C" int mkq_low_rank_adapters_gradient(const void *dy, int dy_dtype, int64_t ld_dy, const void *x, int x_dtype, int64_t ldx, const float *x_steps,
                                              int x_group, const int32_t *adapter, const float *hidden, int64_t M, int64_t K, int64_t N, int rank, int64_t R,
                                              const void *down, const void *up, int w_dtype, const float *scales, const void *dx_base, int64_t ld_dx_base,
                                              void *dx, int dx_dtype, int64_t ld_dx, void *d_down, void *d_up, int grad_dtype, int accumulate,
                                              void *workspace, size_t workspace_bytes, void *stream)
{
    const bool kept = x_dtype == MKQ_I8;
    if (!is_float_dtype(dy_dtype) || (!kept && !is_float_dtype(x_dtype)) || !is_float_dtype(w_dtype) || (dx && !is_float_dtype(dx_dtype)) || !is_float_dtype(grad_dtype))
        return MKQ_ERR_DTYPE;
    const AdapterShape d = {M, K, N, R, rank};
    int status = check_shape(d);
    if (status == MKQ_ERR_SHAPE || ld_dy < N || (d_down && !kept && ldx < K) || (dx && ld_dx < K) || (dx && dx_base && ld_dx_base < K) ||
        (d_down && kept && x_group != 32 && x_group != 64 && x_group != 128))
        return MKQ_ERR_SHAPE;
    if (!dx && !d_down && !d_up) return MKQ_ERR_NULL;
    if (M > 0) {
        if (!dy || !adapter || (d_down && (!x || (kept && !x_steps))) || (d_up && !hidden) || (dx && !down) || ((dx || d_down) && !up)) return MKQ_ERR_NULL;
        if (!aligned16(dy) || !aligned4(adapter) || !aligned16(x) || !aligned4(x_steps) || !aligned4(hidden) || !aligned16(down) || !aligned16(up) ||
            !aligned4(scales) || !aligned16(dx_base) || !aligned16(dx))
            return MKQ_ERR_ALIGN;
    }
    if (!aligned16(d_down) || !aligned16(d_up)) return MKQ_ERR_ALIGN;
    if (status != MKQ_OK) return status;
    const int64_t pitch = kept ? ceil_div(K, 32) * 32 : ldx;
    if (dx && M > 0) {
        if (dx_base && !in_place_or_apart(dx_base, dx_dtype, ld_dx_base, dx, dx_dtype, ld_dx, M, K)) return MKQ_ERR_UNSUPPORTED;
        // the batch's rows are read again behind dx
        if (!apart(dy, dy_dtype, ld_dy, N, dx, dx_dtype, ld_dx, K, M) || (d_down && !apart(x, x_dtype, pitch, K, dx, dx_dtype, ld_dx, K, M))) return MKQ_ERR_UNSUPPORTED;
    }
    AdapterWorkspace w = gradient_workspace(d);
    if (!workspace || workspace_bytes < w.total) return MKQ_ERR_WORKSPACE;
    if (!aligned16(workspace)) return MKQ_ERR_ALIGN;
    uint8_t *ws = static_cast<uint8_t *>(workspace);
    const hipStream_t st = as_stream(stream);
    AdapterParams a = {adapter, scales, M, (int)R, rank, dx && M > 0 ? w.splits : 1};
    float *u = reinterpret_cast<float *>(ws + w.u);
    if (M > 0 && (dx || d_down)) {
        float *t = a.splits > 1 ? reinterpret_cast<float *>(ws + w.t) : u;
        status = launch_shrink(d, a, dy, dy_dtype, ld_dy, up, w_dtype, N, a.splits == 1, t, st);
        if (status != MKQ_OK) return status;
        if (dx) {
            ExpandParams e = {a, t, down, dx_base, dx, ld_dx_base, ld_dx, (int)K, 0, 0, 0, a.splits > 1, true, a.splits > 1 ? u : nullptr};
            status = launch_expand(d, e, w_dtype, dx_dtype, st);
            if (status != MKQ_OK) return status;
        }
    }
    if (!d_down && !d_up) return MKQ_OK;
    PlanParams plan = {a, w.piece, reinterpret_cast<int32_t *>(ws + w.order), reinterpret_cast<int32_t *>(ws + w.starts), reinterpret_cast<int4 *>(ws + w.tasks), (int)w.tasks_most};
    plan_kernel<<<(unsigned)R, 1024, 0, st>>>(plan);
    status = launch_status();
    OuterParams o = {};
    o.a = a;
    o.piece = w.piece;
    o.accumulate = accumulate != 0;
    o.order = plan.order;
    o.starts = plan.starts;
    o.tasks = plan.tasks;
    o.tasks_most = (int)w.tasks_most;
    if (status == MKQ_OK && d_down) {
        o.coeff = u;
        o.y = x;
        o.steps = x_steps;
        o.ld = pitch;
        o.N = (int)K;
        o.group_shift = x_group == 32 ? 5 : x_group == 64 ? 6 : 7;
        o.groups = kept ? (int)ceil_div(K, x_group) : 0;
        o.partials = reinterpret_cast<float *>(ws + w.down);
        o.grad = d_down;
        status = launch_outer(d, o, x_dtype, grad_dtype, st);
    }
    if (status == MKQ_OK && d_up) {
        o.coeff = hidden;
        o.y = dy;
        o.ld = ld_dy;
        o.N = (int)N;
        o.scaled = true;
        o.partials = reinterpret_cast<float *>(ws + w.up);
        o.grad = d_up;
        status = launch_outer(d, o, dy_dtype, grad_dtype, st);
    }
    return status;
}
