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

// A workgroup of 256 has an adapter: each thread looks through neighbouring rows for those of the adapter and those of smaller ones
__device__ void plan(const AdapterParams &p, const PlanParams &plan, int a)
{
    __shared__ int equal_before[4], less_before[4];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int64_t each = (p.M + 1023) / 1024 * 4;
    const int64_t from = threadIdx.x * each < p.M ? threadIdx.x * each : p.M, to = from + each < p.M ? from + each : p.M;
    auto rows = [&](auto &&f) {
        int64_t m = from;
        for (; m + 16 <= to; m += 16) {
            u32x4 v[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = reinterpret_cast<const Loose<4> *>(p.adapter + m + 4 * i)->v;
#pragma unroll
            for (int i = 0; i < 16; ++i) f(m + i, (int)v[i / 4][i % 4]);
        }
        for (; m < to; ++m) f(m, p.adapter[m]);
    };
    int equal = 0, less = 0;
    rows([&](int64_t, int b) {
        equal += b == a;
        less += b >= 0 && b < a;
    });
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
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        start += less_before[w];
        if (w < wave) waves_before += equal_before[w];
        count += equal_before[w];
    }
    int at = start + waves_before + before - equal;
    if (equal)
        rows([&](int64_t m, int b) {
            if (b == a) plan.order[at++] = (int32_t)m;
        });
    if (threadIdx.x == 0) {
        plan.starts[a] = start;
        if (a == p.R - 1) plan.starts[p.R] = start + count;
    }
    // (behind the last adapter's: fewer rows than the batch's may have an adapter)
    const int first = task_of(start, a, plan.piece), next = a + 1 < p.R ? task_of(start + count, a + 1, plan.piece) : plan.tasks_most;
    const int pieces = count ? (count + plan.piece - 1) / plan.piece : 1;
    for (int i = first + (int)threadIdx.x; i < next; i += 256) {
        const int j = i - first, last = (j + 1) * plan.piece < count ? (j + 1) * plan.piece : count;
        plan.tasks[i] = j < pieces ? make_int4(a, start + j * plan.piece, start + last, pieces) : make_int4(-1, 0, 0, 0);
    }
}

// ---- shrink ---------------------------------------------------------------------------------------------------------------
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

// Places of a row that a wave multiplies at a time: 256 bytes of the larger elements
constexpr int shrink_step(int x_bytes, int w_bytes) { return x_bytes == 4 || w_bytes == 4 ? 64 : 128; }

// Sixteen rows of a step on their way from memory to LDS: neighbouring lanes fetch neighbouring pieces of 16 bytes of a row.  (Fetched as
// the matrix unit takes them, a row a lane, every lane asked for a line of its own: dy of 8192 x 4096 bfloat16 32 us.)  In LDS piece i of row r is
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

// Tiles of 16 rows and RT * 16 of the rank; the four waves of a workgroup take steps in turn and add up through LDS
template <class X, class W, int RT>
__global__ __launch_bounds__(256) void shrink_kernel(const ShrinkParams p)
{
    constexpr int STEP = shrink_step(X::BYTES, W::BYTES);
    using XRows = ShrinkRows<X, STEP>;
    using WRows = ShrinkRows<W, STEP>;
    constexpr int LDS = XRows::BYTES + RT * WRows::BYTES;  // of a wave; the sums have room in it
    static_assert(LDS >= RT * 64 * 16, "sums");
    __shared__ __attribute__((aligned(16))) uint8_t lds[4 * LDS];
    if (blockIdx.x < (unsigned)p.plans) return plan(p.a, p.plan, blockIdx.x);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, c = lane & 15, q = lane >> 4;
    unsigned b = blockIdx.x - p.plans;
    const int chunk = b % p.rank_chunks;
    b /= p.rank_chunks;
    const int split = b % p.a.splits;
    b /= p.a.splits;
    const int slot = b % p.slots;
    const int64_t m0 = (int64_t)(b / p.slots) * 16;
    const int mine = adapter_of(p.a, lane < 16 ? m0 + lane : p.a.M);
    const int steps = (p.K + STEP - 1) / STEP, per_split = (steps + p.a.splits - 1) / p.a.splits;
    const int from = split * per_split, to = from + per_split < steps ? from + per_split : steps;
    float *t = p.t + (int64_t)split * p.a.M * p.a.pitch;
    uint8_t *lds_x = lds + wave * LDS, *lds_w = lds_x + XRows::BYTES;
    v4f *sums = reinterpret_cast<v4f *>(lds);
    const typename X::raw *x[XRows::N];
#pragma unroll
    for (int i = 0; i < XRows::N; ++i) {
        const int64_t row = m0 + XRows::row_of(i);
        x[i] = static_cast<const typename X::raw *>(p.x) + (row < p.a.M ? row : p.a.M - 1) * p.ldx;
    }
    Adapters adapters(mine, slot, p.slots, lane < 16 && m0 + lane < p.a.M && mine < 0);
    int a;
    uint64_t same;
    while (adapters.next(a, same)) {
        if (a < 0) {  // rows without an adapter
            for (int i = 0; i < 16; ++i)
                if (same >> i & 1)
                    for (int r = chunk * RT * 16 + (int)threadIdx.x; r < p.a.pitch && r < (chunk + 1) * RT * 16; r += 256) {
                        t[(m0 + i) * p.a.pitch + r] = 0.0f;
                        if (p.hidden && r < p.a.rank) p.hidden[(m0 + i) * p.a.rank + r] = 0.0f;
                    }
            continue;
        }
        v4f acc[RT];
#pragma unroll
        for (int r = 0; r < RT; ++r) acc[r] = v4f{0, 0, 0, 0};
        const typename W::raw *w = static_cast<const typename W::raw *>(p.w) + (int64_t)a * p.a.rank * p.K;
        XRows xs;
        WRows ws[RT];
        auto fetch = [&](int s) {
            const bool edge = (s + 1) * STEP > p.K;
#pragma unroll
            for (int i = 0; i < XRows::N; ++i) xs.v[i] = fetch16<X, false>(x[i], 0, s * STEP + XRows::piece_of() * (16 / X::BYTES), p.K, edge);
#pragma unroll
            for (int r = 0; r < RT; ++r)
#pragma unroll
                for (int i = 0; i < WRows::N; ++i) {
                    const int at = (chunk * RT + r) * 16 + WRows::row_of(i);
                    ws[r].v[i] = fetch16<W, false>(w, (uint32_t)(at < p.a.rank ? at : p.a.rank - 1) * ((uint32_t)p.K * W::BYTES),
                                            s * STEP + WRows::piece_of() * (16 / W::BYTES), p.K, edge);
                }
        };
        if (from + wave < to) fetch(from + wave);
        for (int s = from + wave; s < to; s += 4) {
            xs.put(lds_x);
#pragma unroll
            for (int r = 0; r < RT; ++r) ws[r].put(lds_w + r * WRows::BYTES);
            if (s + 4 < to) fetch(s + 4);
            wave_order();
#pragma unroll
            for (int h = 0; h < STEP / 32; ++h) {
                const Neighbours<X> xn = XRows::get(lds_x, h);
                if constexpr (std::is_same<X, ElemF16>::value && std::is_same<W, ElemF16>::value) {
#pragma unroll
                    for (int r = 0; r < RT; ++r)
                        acc[r] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(v8h, xn.w[0]),
                                                                        __builtin_bit_cast(v8h, WRows::get(lds_w + r * WRows::BYTES, h).w[0]), acc[r], 0, 0, 0);
                } else {
                    uint4 xp[Parts<X>::N], wp[Parts<W>::N];
                    operand(xn, xp);
#pragma unroll
                    for (int r = 0; r < RT; ++r) {
                        operand(WRows::get(lds_w + r * WRows::BYTES, h), wp);
                        acc[r] = multiply<3>(xp, wp, acc[r]);
                    }
                }
            }
            wave_order();
        }
        __syncthreads();
#pragma unroll
        for (int r = 0; r < RT; ++r) sums[(wave * RT + r) * 64 + lane] = acc[r];
        __syncthreads();
        const float scale = p.scaled ? scale_of(p.a, a) : 1.0f;
        for (int r = wave; r < RT; r += 4) {
            const v4f sum = (sums[r * 64 + lane] + sums[(RT + r) * 64 + lane]) + (sums[(2 * RT + r) * 64 + lane] + sums[(3 * RT + r) * 64 + lane]);
            const int at = (chunk * RT + r) * 16 + c;
#pragma unroll
            for (int v = 0; v < 4; ++v)
                if (at < p.a.pitch && (same >> (4 * q + v) & 1)) {
                    const float value = at < p.a.rank ? sum[v] * scale : 0.0f;
                    t[(m0 + 4 * q + v) * p.a.pitch + at] = value;
                    if (p.hidden && at < p.a.rank) p.hidden[(m0 + 4 * q + v) * p.a.rank + at] = value;
                }
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
    int N, column_blocks, slots, row_groups, tiles;
    bool scaled;      // t is still to be multiplied by the adapter's scale
    bool keep_scaled; // ... as it is kept
    float *keep;      // [M, keep_pitch], or NULL: what the splits add up to
    int keep_pitch;
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

// t of row c from place r on, eight values, added up over the splits; t: that of the first row
__device__ __forceinline__ void hidden_values(const ExpandParams &p, const float *t, int c, int r, float (&v)[8])
{
    const uint32_t off = (uint32_t)(c * p.a.pitch + (r < p.a.pitch ? r : 0)) * 4;
    const int64_t split = p.a.M * p.a.pitch;
    auto load = [&](int s, float (&to)[8]) { load8(reinterpret_cast<const float *>(reinterpret_cast<const uint8_t *>(t + s * split) + off), to); };
    load(0, v);
    for (int s = 1; s < p.a.splits; s += 3) {
        float more[3][8];
#pragma unroll
        for (int i = 0; i < 3; ++i) load(s + i < p.a.splits ? s + i : s, more[i]);
#pragma unroll
        for (int i = 0; i < 3; ++i)
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] += s + i < p.a.splits ? more[i][e] : 0.0f;
    }
    if (r >= p.a.pitch)
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = 0.0f;
}

// A wave has 128 columns of `tiles` tiles of 16 rows; lane (c, q) has columns 8 c .. 8 c + 7 of rows 4 q .. 4 q + 3.  KEEP: the adapter's rows are
// kept as operands in LDS while the adapter is the same, otherwise they are fetched again for every tile (from the caches), 32 at a time.
template <class W, class O, bool KEEP>
__global__ __launch_bounds__(256, 2) void expand_kernel(const ExpandParams p)
{
    constexpr int PW = Parts<W>::N, PT = O::BYTES == 4 ? 3 : 2;  // (2^-16 of a product is left out under results of 16 bits, which end at 2^-9 or 2^-12)
    const int64_t task = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int block = (int)(task % p.column_blocks);
    const int64_t rest = task / p.column_blocks;
    const int slot = (int)(rest / p.row_groups), group = (int)(rest - (int64_t)slot * p.row_groups);
    if (slot >= p.slots) return;
    const bool edge = block * 128 + 128 > p.N;
    extern __shared__ uint4 operands[];
    uint4 *kept = operands + (KEEP ? (threadIdx.x >> 6) * ((p.a.rank + 31) / 32 * 8 * PW * 64) + (threadIdx.x & 63) : 0);
    int have = -1;
    const int64_t first = (int64_t)group * p.tiles * 16;
    // at most four tiles: a row of theirs a lane
    const int all = adapter_of(p.a, (int)(threadIdx.x & 63) < 16 * p.tiles ? first + (threadIdx.x & 63) : p.a.M);
    auto fetch_base = [&](Neighbours<O> (&to)[4], int64_t m0) {
        if (!p.base || m0 >= p.a.M) return;
        const int lane = fresh(threadIdx.x & 63), q = lane >> 4, n0 = block * 128 + 8 * (lane & 15);
        const int last_row = p.a.M - m0 < 16 ? (int)(p.a.M - m0) - 1 : 15;
        const void *at = static_cast<const typename O::raw *>(p.base) + m0 * p.ld_base;
#pragma unroll
        for (int v = 0; v < 4; ++v)
            to[v].fetch(at, (uint32_t)(4 * q + v < last_row ? 4 * q + v : last_row) * ((uint32_t)p.ld_base * O::BYTES), n0, p.N, edge);
    };
    Neighbours<O> base[4], next_base[4];
    fetch_base(next_base, first);
    for (int tile = 0; tile < p.tiles; ++tile) {
        const int64_t m0 = first + 16 * tile;
        if (m0 >= p.a.M) break;
        const int lane = fresh(threadIdx.x & 63), c = lane & 15, q = lane >> 4, n0 = block * 128 + 8 * c;
        const int last_row = p.a.M - m0 < 16 ? (int)(p.a.M - m0) - 1 : 15;
        const int mine = __shfl(all, 16 * tile + c, 64), of_tile = lane < 16 ? mine : -1;
#pragma unroll
        for (int v = 0; v < 4; ++v) base[v] = next_base[v];
        if (tile + 1 < p.tiles) fetch_base(next_base, m0 + 16);
        typename O::raw *out = static_cast<typename O::raw *>(p.out) + m0 * p.ld_out;
        const float *t = p.t + m0 * p.a.pitch;
        Adapters adapters(of_tile, slot, p.slots, lane < 16 && m0 + lane < p.a.M && mine < 0);
        int a;
        uint64_t same;
        while (adapters.next(a, same)) {
            v4f acc[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) acc[i] = v4f{0, 0, 0, 0};
            if (a < 0) {  // rows without an adapter
                if (p.keep && block == 0)
                    for (int i = 0; i < 16; ++i)
                        if (same >> i & 1)
                            for (int r = lane; r < p.a.rank; r += 64) p.keep[(m0 + i) * p.keep_pitch + r] = 0.0f;
                if (p.base == p.out) continue;
            } else {
                const float scale = scale_of(p.a, a), factor = p.scaled ? scale : 1.0f;
                const typename W::raw *w = static_cast<const typename W::raw *>(p.w) + (int64_t)a * p.a.rank * p.N;
                auto fetch = [&](Block<W> &rows, int r0) {  // (behind the rank its last row again: t is 0 there)
                    const int r = r0 + 8 * q;
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        rows.rows[e].fetch(w, (uint32_t)(r + e < p.a.rank ? r + e : p.a.rank - 1) * ((uint32_t)p.N * W::BYTES), n0, p.N, edge);
                };
                if (KEEP && a != have) {
                    for (int r0 = 0; r0 < p.a.rank; r0 += 32) {
                        Block<W> rows;
                        fetch(rows, r0);
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            uint4 wp[PW];
                            rows.column(i, wp);
#pragma unroll
                            for (int k = 0; k < PW; ++k) kept[((r0 / 32 * 8 + i) * PW + k) * 64] = wp[k];
                        }
                    }
                    have = a;
                }
                for (int r0 = 0; r0 < p.a.rank; r0 += 32) {
                    const int r = r0 + 8 * q;
                    Block<W> rows;
                    if (!KEEP) fetch(rows, r0);
                    uint4 tp[PT];
                    float v[8];
                    hidden_values(p, t, c < last_row ? c : last_row, r, v);
                    if (p.keep && block == 0 && (same >> c & 1)) {
#pragma unroll
                        for (int e = 0; e < 8; ++e)
                            if (r + e < p.a.rank) p.keep[(m0 + c) * p.keep_pitch + r + e] = p.keep_scaled ? v[e] * factor : v[e];
                    }
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[e] *= factor;
                    parts_of(v, tp);
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        uint4 wp[PW];
                        if constexpr (KEEP) {
#pragma unroll
                            for (int k = 0; k < PW; ++k) wp[k] = kept[((r0 / 32 * 8 + i) * PW + k) * 64];
                        } else {
                            rows.column(i, wp);
                        }
                        acc[i] = multiply<PT>(tp, wp, acc[i]);
                    }
                }
            }
#pragma unroll
            for (int v = 0; v < 4; ++v)
                if (same >> (4 * q + v) & 1 && n0 < p.N) {
                    float y[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) y[e] = p.base ? acc[e][v] + base[v].get(e) : acc[e][v];
                    put_neighbours<O>(out, (uint32_t)(4 * q + v) * ((uint32_t)p.ld_out * O::BYTES), n0, p.N, edge, y);
                }
        }
    }
}

// ---- outer ----------------------------------------------------------------------------------------------------------------
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
template <> struct Parts<Codes> { static constexpr int N = 3; };

__device__ __forceinline__ void write_grad(const OuterParams &p, const OuterSide &side, int a, int64_t at, float v)
{
    v *= side.scaled ? scale_of(p.a, a) : 1.0f;
    at += (int64_t)a * p.a.rank * side.N;
    auto write = [&](auto o) {
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
    __device__ __forceinline__ void fetch(const OuterParams &p, const OuterSide &side, int chunk, int n0, bool edge, int rows, int first)
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
template <class Y, int RT>
__device__ __forceinline__ void outer(const OuterParams &p, const OuterSide &side, int block, int chunk, int a, int first, int last, int pieces)
{
    const int lane = threadIdx.x & 63, c = lane & 15, q = lane >> 4, n0 = block * 128 + 8 * c, n = last - first;
    const bool edge = block * 128 + 128 > side.N;
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
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int v = 0; v < 4; ++v) {
            const int at = (chunk * RT + r) * 16 + 4 * q + v;
            if (at >= p.a.rank) continue;
            if (pieces > 1 && n0 + 8 <= side.N) {
                float *to = side.partials + ((int64_t)part * p.a.rank + at) * side.N + n0;
#pragma unroll
                for (int i = 0; i < 8; i += 4)
                    reinterpret_cast<Loose<4> *>(to + i)->v = u32x4{__float_as_uint(acc[r][i][v]), __float_as_uint(acc[r][i + 1][v]),
                                                                    __float_as_uint(acc[r][i + 2][v]), __float_as_uint(acc[r][i + 3][v])};
                continue;
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                if (n0 + i >= side.N) continue;
                if (pieces > 1) side.partials[((int64_t)part * p.a.rank + at) * side.N + n0 + i] = acc[r][i][v];
                else write_grad(p, side, a, (int64_t)at * side.N + n0 + i, acc[r][i][v]);
            }
        }
}

template <class X, class D, int RT>
__global__ __launch_bounds__(256, (X::BYTES < 4 && D::BYTES < 4 ? 4 : 3) - RT) void outer_kernel(const OuterParams p)
{
    const int blocks = p.side[0].column_blocks + p.side[1].column_blocks;
    int64_t task = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int block = (int)(task % blocks);
    task /= blocks;
    const int chunk = (int)(task % p.rank_chunks);
    task /= p.rank_chunks;
    if (task >= p.plan.tasks_most) return;
    const int4 what = p.plan.tasks[task];
    const int a = __builtin_amdgcn_readfirstlane(what.x), first = __builtin_amdgcn_readfirstlane(what.y), last = __builtin_amdgcn_readfirstlane(what.z);
    const int pieces = __builtin_amdgcn_readfirstlane(what.w);
    if (a < 0 || (first == last && p.accumulate)) return;
    if (block < p.side[0].column_blocks) outer<X, RT>(p, p.side[0], block, chunk, a, first, last, pieces);
    else outer<D, RT>(p, p.side[1], block - p.side[0].column_blocks, chunk, a, first, last, pieces);
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
    write_grad(p, side, a, i, sum);
}

// ---- host side ------------------------------------------------------------------------------------------------------------
constexpr int64_t ADAPTERS_MOST = 0x3FFFFF, SIDES_MOST = 0x7FFFFF00;
constexpr int RANK_MOST = 256;
constexpr int64_t STRIDE_MOST = (int64_t)1 << 25;  // elements between rows: 16 of them are addressed in 32 bits
constexpr int FEW_ROWS = 512;  // up to here a tile's adapters are shared out among workgroups

struct AdapterShape {
    int64_t M, K, N, R;
    int rank;
};
static int check_shape(const AdapterShape &d)
{
    if (d.M < 0 || d.K <= 0 || d.N <= 0 || d.R <= 0 || d.rank <= 0) return MKQ_ERR_SHAPE;
    if (d.M > SIDES_MOST || d.K > SIDES_MOST || d.N > SIDES_MOST || d.R > ADAPTERS_MOST || d.rank > RANK_MOST || d.K * d.rank >= (int64_t)1 << 29 || d.N * d.rank >= (int64_t)1 << 29 ||
        d.K > STRIDE_MOST || d.N > STRIDE_MOST || d.K < 8 || d.N < 8)
        return MKQ_ERR_UNSUPPORTED;
    return MKQ_OK;
}

static int least(int64_t a, int64_t b) { return (int)(a < b ? a : b); }
static int slots_of(const AdapterShape &d) { return d.M <= FEW_ROWS ? least(least(16, d.M), d.R) : 1; }
static int rank_tiles(int rank) { return rank <= 16 ? 1 : rank <= 32 ? 2 : 4; }
// Workgroups that share the places of a row: about 512 of them in all, four steps each at least
static int splits_of(const AdapterShape &d, int64_t side)
{
    const int64_t steps = ceil_div(side, 64), groups = ceil_div(d.M, 16) * slots_of(d) * ceil_div(d.rank, 16 * rank_tiles(d.rank));
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

static ShrinkParams shrink_params(const AdapterShape &d, const AdapterParams &a, const void *x, int64_t ldx, const void *w, int64_t side, bool scaled, float *t,
                                  float *hidden)
{
    ShrinkParams p = {};
    p.a = a;
    p.x = x;
    p.w = w;
    p.ldx = ldx;
    p.K = (int)side;
    p.slots = slots_of(d);
    p.rank_chunks = (int)ceil_div(d.rank, 16 * rank_tiles(d.rank));
    p.scaled = scaled;
    p.t = t;
    p.hidden = hidden;
    return p;
}
static int launch_shrink(const AdapterShape &d, const ShrinkParams &p, int x_dtype, int w_dtype, hipStream_t st)
{
    const int64_t workgroups = (p.x ? ceil_div(d.M, 16) * p.slots * p.a.splits * p.rank_chunks : 0) + p.plans;
    if (!grid_ok(workgroups, 256)) return MKQ_ERR_UNSUPPORTED;
    with_elem(x_dtype, [&](auto x_e) {
        with_elem(w_dtype, [&](auto w_e) {
            with_tiles(rank_tiles(d.rank), [&](auto n) { shrink_kernel<decltype(x_e), decltype(w_e), decltype(n)::value><<<(unsigned)workgroups, 256, 0, st>>>(p); });
        });
    });
    return launch_status();
}

static int launch_expand(const AdapterShape &d, ExpandParams p, int w_dtype, int out_dtype, hipStream_t st)
{
    p.column_blocks = (int)ceil_div(p.N, 128);
    p.slots = slots_of(d);
    // tiles of a wave: four, if 4096 waves are left then
    const int64_t all = ceil_div(d.M, 16), fill = all * p.column_blocks / 4096;
    p.tiles = (int)(fill < 1 ? 1 : fill > 4 ? 4 : fill);
    p.row_groups = (int)ceil_div(all, p.tiles);
    const int64_t workgroups = ceil_div((int64_t)p.column_blocks * p.row_groups * p.slots, 4);
    if (!grid_ok(workgroups, 256)) return MKQ_ERR_UNSUPPORTED;
    with_elem(w_dtype, [&](auto w) {
        with_elem(out_dtype, [&](auto o) {
            using W = decltype(w);
            using O = decltype(o);
            const int blocks = (int)ceil_div(d.rank, 32) * Parts<W>::N;  // of 8 KiB a wave
            if (p.tiles > 1 && blocks <= 2) expand_kernel<W, O, true><<<(unsigned)workgroups, 256, blocks * 4 * 8192, st>>>(p);
            else expand_kernel<W, O, false><<<(unsigned)workgroups, 256, 0, st>>>(p);
        });
    });
    return launch_status();
}

// Rows of a piece: about 2000 waves in all
static int piece_rows(const AdapterShape &d)
{
    const int64_t columns = ceil_div(d.K, 128) + ceil_div(d.N, 128), n = ceil_div(ceil_div(d.M * columns, 2048), 64) * 64;
    return (int)(n < 64 ? 64 : n > 2048 ? 2048 : n);
}

static int pitch_of(int rank) { return (rank + 7) / 8 * 8; }

struct AdapterWorkspace {
    size_t t, u, order, starts, tasks, down, up, total;
    int splits, piece;
    int64_t tasks_most;
};
static AdapterWorkspace forward_workspace(const AdapterShape &d)
{
    AdapterWorkspace w = {};
    w.splits = splits_of(d, d.K);
    w.total = (size_t)w.splits * d.M * pitch_of(d.rank) * sizeof(float);
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
    const size_t hidden = (size_t)d.M * pitch_of(d.rank) * sizeof(float), parts = d.M > w.piece ? 2 * (size_t)(d.M / w.piece) + 2 : 0;
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

static int launch_outer(const AdapterShape &d, OuterParams p, int x_dtype, int dy_dtype, hipStream_t st)
{
    const int tiles = d.rank <= 16 ? 1 : 2;
    p.rank_chunks = (int)ceil_div(d.rank, 16 * tiles);
    const int64_t workgroups = ceil_div((int64_t)p.plan.tasks_most * (p.side[0].column_blocks + p.side[1].column_blocks) * p.rank_chunks, 4);
    const int64_t joins = d.R * ceil_div((int64_t)d.rank * ((p.side[0].column_blocks ? d.K : 0) + (p.side[1].column_blocks ? d.N : 0)), 256);
    if (!grid_ok(workgroups, 256) || !grid_ok(joins, 256)) return MKQ_ERR_UNSUPPORTED;
    with_rows(x_dtype, [&](auto x) {
        with_elem(dy_dtype, [&](auto y) {
            if (tiles == 1) outer_kernel<decltype(x), decltype(y), 1><<<(unsigned)workgroups, 256, 0, st>>>(p);
            else outer_kernel<decltype(x), decltype(y), 2><<<(unsigned)workgroups, 256, 0, st>>>(p);
        });
    });
    if (d.M > p.plan.piece) outer_join_kernel<<<(unsigned)joins, 256, 0, st>>>(p);
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
    if (ld_out > STRIDE_MOST || (base && ld_base > STRIDE_MOST)) return MKQ_ERR_UNSUPPORTED;
    if (base && !in_place_or_apart(base, out_dtype, ld_base, out, out_dtype, ld_out, M, N)) return MKQ_ERR_UNSUPPORTED;
    const AdapterWorkspace w = forward_workspace(d);
    if (!workspace || workspace_bytes < w.total) return MKQ_ERR_WORKSPACE;
    if (!aligned16(workspace)) return MKQ_ERR_ALIGN;
    const hipStream_t st = as_stream(stream);
    const AdapterParams a = {adapter, scales, M, (int)R, rank, pitch_of(rank), w.splits};
    float *t = static_cast<float *>(workspace);
    status = launch_shrink(d, shrink_params(d, a, x, ldx, down, K, false, t, w.splits == 1 ? hidden : nullptr), x_dtype, w_dtype, st);
    if (status != MKQ_OK) return status;
    ExpandParams e = {};
    e.a = a;
    e.t = t;
    e.w = up;
    e.base = base;
    e.out = out;
    e.ld_base = ld_base;
    e.ld_out = ld_out;
    e.N = (int)N;
    e.scaled = true;
    e.keep = w.splits > 1 ? hidden : nullptr;
    e.keep_pitch = rank;
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
        if (ld_dx > STRIDE_MOST || (dx_base && ld_dx_base > STRIDE_MOST)) return MKQ_ERR_UNSUPPORTED;
        if (dx_base && !in_place_or_apart(dx_base, dx_dtype, ld_dx_base, dx, dx_dtype, ld_dx, M, K)) return MKQ_ERR_UNSUPPORTED;
        // the batch's rows are read again behind dx
        if (!apart(dy, dy_dtype, ld_dy, N, dx, dx_dtype, ld_dx, K, M) || (d_down && !apart(x, x_dtype, pitch, K, dx, dx_dtype, ld_dx, K, M))) return MKQ_ERR_UNSUPPORTED;
    }
    AdapterWorkspace w = gradient_workspace(d);
    if (!workspace || workspace_bytes < w.total) return MKQ_ERR_WORKSPACE;
    if (!aligned16(workspace)) return MKQ_ERR_ALIGN;
    uint8_t *ws = static_cast<uint8_t *>(workspace);
    const hipStream_t st = as_stream(stream);
    const AdapterParams a = {adapter, scales, M, (int)R, rank, pitch_of(rank), dx && M > 0 ? w.splits : 1};
    float *u = reinterpret_cast<float *>(ws + w.u), *t = a.splits > 1 ? reinterpret_cast<float *>(ws + w.t) : u;
    const PlanParams plan = {w.piece, (int)w.tasks_most, reinterpret_cast<int32_t *>(ws + w.order), reinterpret_cast<int32_t *>(ws + w.starts),
                             reinterpret_cast<int4 *>(ws + w.tasks)};
    // one launch puts the rows in order and makes u
    const bool products = M > 0 && (dx || d_down);
    ShrinkParams shrink = shrink_params(d, a, products ? dy : nullptr, ld_dy, up, N, a.splits == 1, t, nullptr);
    shrink.plans = d_down || d_up ? (int)R : 0;
    shrink.plan = plan;
    if (products || shrink.plans) {
        status = launch_shrink(d, shrink, dy_dtype, w_dtype, st);
        if (status != MKQ_OK) return status;
    }
    if (dx && M > 0) {
        ExpandParams e = {};
        e.a = a;
        e.t = t;
        e.w = down;
        e.base = dx_base;
        e.out = dx;
        e.ld_base = ld_dx_base;
        e.ld_out = ld_dx;
        e.N = (int)K;
        e.scaled = e.keep_scaled = a.splits > 1;
        e.keep = a.splits > 1 ? u : nullptr;
        e.keep_pitch = a.pitch;
        status = launch_expand(d, e, w_dtype, dx_dtype, st);
        if (status != MKQ_OK) return status;
    }
    if (!d_down && !d_up) return MKQ_OK;
    OuterParams o = {};
    o.a = a;
    o.plan = plan;
    o.grad_dtype = grad_dtype;
    o.accumulate = accumulate != 0;
    if (d_down) {
        OuterSide &s = o.side[0];
        s.coeff = u;
        s.coeff_pitch = a.pitch;
        s.y = x;
        s.steps = x_steps;
        s.ld = pitch;
        s.N = (int)K;
        s.column_blocks = (int)ceil_div(K, 128);
        s.group_shift = x_group == 32 ? 5 : x_group == 64 ? 6 : 7;
        s.groups = kept ? (int)ceil_div(K, x_group) : 0;
        s.partials = reinterpret_cast<float *>(ws + w.down);
        s.grad = d_down;
    }
    if (d_up) {
        OuterSide &s = o.side[1];
        s.coeff = hidden;
        s.coeff_pitch = rank;
        s.y = dy;
        s.ld = ld_dy;
        s.N = (int)N;
        s.column_blocks = (int)ceil_div(N, 128);
        s.scaled = true;
        s.partials = reinterpret_cast<float *>(ws + w.up);
        s.grad = d_up;
    }
    return launch_outer(d, o, d_down ? x_dtype : MKQ_F32, dy_dtype, st);
}
