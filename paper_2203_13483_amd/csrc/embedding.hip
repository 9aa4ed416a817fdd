// Token rows: the lookup from a float table and from a group-scaled 4-bit one, and the table's gradient by sorted tokens.
//
//     out[i,:] = scale * table[t_i,:]              dT[v,:] = scale * sum_{i: t_i = v} dy[i,:]
//
// All are bound by bytes: the rows read and written, and for the gradient the whole of dT, whose rows without a token are
// zeros.  A lookup is one multiplication in binary32 and one rounding per value.  Gradients, us, a call among others (and its kernels, each
// traced by itself): 4096 binary16 tokens of 768 into binary32 [30522, 768] 28.5 (18 sorting beside the zeros, 5 sums, 6 joining),
// 65536 bfloat16 tokens of 1024 into [30522, 1024] 95 (35 in four launches that sort beside the zeros, 45 to 50 sums: 4.6 TB/s, 8 joining).
#include "elements.h"

namespace mkq {

constexpr uint32_t NO_ROW = 0xFFFFFFFFu;
// The table row of position i's token, or NO_ROW
__device__ __forceinline__ uint32_t token_row(const void *__restrict__ tokens, int bits, int64_t i, uint32_t V)
{
    const int64_t t = bits == 64 ? static_cast<const int64_t *>(tokens)[i] : (int64_t)static_cast<const int32_t *>(tokens)[i];
    return t >= 0 && t < (int64_t)V ? (uint32_t)t : NO_ROW;
}

// ---- lookup -------------------------------------------------------------------------------------------------------------
struct LookupParams {
    const void *tokens;
    const void *table;  // float rows, or rows of nibbles (ld_table in words)
    const float *s_w;   // [V, groups] of the nibbles
    void *out;
    int64_t M, ld_table, ld_out;
    uint32_t V;
    int D, groups, group_shift, token_bits, threads_per_row;
    float scale;
};

// Where a row's values come from: eight neighbours from d (a multiple of 8), as fetched, or one
template <class E>
struct FloatRow {
    struct alignas(16) Eight {
        typename E::raw v[8];
    };
    const typename E::raw *row;
    __device__ __forceinline__ void set(const LookupParams &p, uint32_t r) { row = static_cast<const typename E::raw *>(p.table) + (int64_t)r * p.ld_table; }
    __device__ __forceinline__ void fetch(const LookupParams &, int d, Eight &to) const
    {
#pragma unroll
        for (int w = 0; w < (int)sizeof(Eight) / 16; ++w) reinterpret_cast<uint4 *>(&to)[w] = reinterpret_cast<const uint4 *>(row + d)[w];
    }
    __device__ static __forceinline__ float get(const Eight &x, int i) { return E::get(x.v[i]); }
    __device__ __forceinline__ float one(const LookupParams &, int d) const { return E::get(row[d]); }
};
struct NibbleRow {
    struct Eight {
        uint32_t word;
        float step;
    };
    const uint32_t *row;
    const float *s;
    __device__ __forceinline__ void set(const LookupParams &p, uint32_t r)
    {
        row = static_cast<const uint32_t *>(p.table) + (int64_t)r * p.ld_table;
        s = p.s_w + (int64_t)r * p.groups;
    }
    __device__ __forceinline__ void fetch(const LookupParams &p, int d, Eight &to) const
    {
        to.word = row[d / 8];
        to.step = s[d >> p.group_shift];
    }
    __device__ static __forceinline__ float get(const Eight &x, int i) { return (float)((int)(x.word << (28 - 4 * i)) >> 28) * x.step; }
    __device__ __forceinline__ float one(const LookupParams &p, int d) const
    {
        return (float)((int)(row[d / 8] << (28 - 4 * (d % 8))) >> 28) * s[d >> p.group_shift];
    }
};

// threads_per_row neighbouring threads write a token's row, and ROWS of them at a time, so that as many tokens, then as many rows are
// on their way together.  Rows are written through the caches: past them 65536 binary16 rows of 1024 take 30 instead of 47 us, but with
// the LayerNorm that reads them 99 instead of 97, 32768 rows 55 instead of 47.  VEC: D is a multiple of 8 and all rows of 16 bytes, a
// thread has eight neighbouring values; otherwise eight that are threads_per_row apart.
template <class Row, class O, bool VEC, int ROWS>
__global__ __launch_bounds__(256) void lookup_kernel(const LookupParams p)
{
    const int rows = 256 / p.threads_per_row;
    const int r = threadIdx.x / p.threads_per_row, u = threadIdx.x - r * p.threads_per_row;
    if (r >= rows) return;
    for (int64_t i0 = (int64_t)blockIdx.x * rows * ROWS + r; i0 < p.M; i0 += (int64_t)gridDim.x * rows * ROWS) {
        Row row[ROWS];
        bool known[ROWS];
#pragma unroll
        for (int k = 0; k < ROWS; ++k) {
            const int64_t i = i0 + k * rows;
            const uint32_t t = i < p.M ? token_row(p.tokens, p.token_bits, i, p.V) : NO_ROW;
            known[k] = t != NO_ROW;
            row[k].set(p, known[k] ? t : 0);
        }
        if constexpr (VEC) {
            for (int d = u * 8; d < p.D; d += p.threads_per_row * 8) {
                typename Row::Eight x[ROWS];
#pragma unroll
                for (int k = 0; k < ROWS; ++k) row[k].fetch(p, d, x[k]);  // (row 0 exists where there is none to look up)
#pragma unroll
                for (int k = 0; k < ROWS; ++k) {
                    float v[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[e] = known[k] ? product(Row::get(x[k], e), p.scale) : 0.0f;
                    if (i0 + k * rows < p.M) put8<O>(static_cast<typename O::raw *>(p.out) + (i0 + k * rows) * p.ld_out + d, v);
                }
            }
        } else {
#pragma unroll
            for (int k = 0; k < ROWS; ++k) {
                if (i0 + k * rows >= p.M) break;
                typename O::raw *out = static_cast<typename O::raw *>(p.out) + (i0 + k * rows) * p.ld_out;
                for (int d0 = u; d0 < p.D; d0 += p.threads_per_row * 8) {
                    float v[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const int d = d0 + e * p.threads_per_row;
                        v[e] = known[k] && d < p.D ? product(row[k].one(p, d), p.scale) : 0.0f;
                    }
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const int d = d0 + e * p.threads_per_row;
                        if (d < p.D) out[d] = O::put(v[e]);
                    }
                }
            }
        }
    }
}

// ---- gradient: zeros ------------------------------------------------------------------------------------------------------
// The rows without a token take most of the bytes of a usual gradient, sorting the tokens is bound by latency: the launches
// that sort fill the table with zeros as well, each a share of it in workgroups behind the sorting ones.
struct ZeroParams {
    void *grad;
    int64_t ld, rows_from, rows_to;  // this launch's share
    int D, bytes, vec;               // of a value; vec: rows are multiples of 16 bytes
    unsigned first;                  // workgroup
};

__device__ __forceinline__ void zero_rows(const ZeroParams &z)
{
    const int64_t threads = (int64_t)(gridDim.x - z.first) * blockDim.x, t = (int64_t)(blockIdx.x - z.first) * blockDim.x + threadIdx.x;
    uint8_t *const base = static_cast<uint8_t *>(z.grad) + z.rows_from * z.ld * z.bytes;
    const int64_t rows = z.rows_to - z.rows_from;
    if (z.ld == z.D) {  // one piece of memory, whatever its rows: 16 bytes a store between its first and last multiple of 16
        const uintptr_t begin = reinterpret_cast<uintptr_t>(base), end = begin + (uintptr_t)(rows * z.D * z.bytes);
        const uintptr_t inner = (begin + 15) / 16 * 16, outer = end / 16 * 16;
        for (uintptr_t p = inner + 16 * (uintptr_t)t; p < outer; p += 16 * (uintptr_t)threads) *reinterpret_cast<uint4 *>(p) = make_uint4(0, 0, 0, 0);
        if (t < 16) {  // (two bytes each: up to seven before and seven behind, all of it where it is shorter)
            const uintptr_t head = begin + 2 * (uintptr_t)t, tail = (outer > begin ? outer : begin) + 2 * (uintptr_t)t;
            if (head < inner && head < end) *reinterpret_cast<uint16_t *>(head) = 0;
            if (tail < end) *reinterpret_cast<uint16_t *>(tail) = 0;
        }
        return;
    }
    const int per = z.vec ? 16 / z.bytes : 1, units = (z.D + per - 1) / per;
    for (int64_t i = t; i < rows * units; i += threads) {
        const int64_t row = i / units;
        const int d = (int)(i - row * units) * per;
        uint8_t *at = base + (row * z.ld + d) * z.bytes;
        if (z.vec && d + per <= z.D) {
            *reinterpret_cast<uint4 *>(at) = make_uint4(0, 0, 0, 0);
        } else {
            for (int e = 0; e < per && d + e < z.D; ++e) {
                if (z.bytes == 4) reinterpret_cast<uint32_t *>(at)[e] = 0;
                else reinterpret_cast<uint16_t *>(at)[e] = 0;
            }
        }
    }
}

__global__ __launch_bounds__(256) void zero_rows_kernel(const ZeroParams z) { zero_rows(z); }

// ---- gradient: sorting the tokens ---------------------------------------------------------------------------------------
// Positions are put in the order of their tokens, equal tokens in the order of the batch, so a row's sum does not depend on how
// the work fell.  Tokens that count for nothing (the padding token, ids outside the table) get the key V, behind all others.
// Short batches: a position's place is the number of positions before it, counted directly; longer ones: a stable radix sort
// (least significant digit first, up to nine bits a pass).  A gradient of V = 30522, D = 768, us: 12000 tokens 42.4 counted directly, 16384
// 56.8, sorted by digits 50.2.
constexpr int SORT_BINS = 512, SORT_THREADS = 1024, SORT_WAVES = 16, SORT_ROUNDS = 2, SORT_TILE = SORT_THREADS * SORT_ROUNDS, SORT_BLOCKS = 256;
constexpr int RANK_MAX = 12288, RANK_FEW = 4096, RANK_THREADS = 1024;

struct SortParams {
    const void *tokens;
    int64_t padding;
    int M, per_block, blocks;  // positions of a workgroup: a multiple of SORT_TILE
    uint32_t V;
    int shift, bits;
    const uint32_t *keys_in, *order_in;  // null in the first pass: keys come from the tokens
    uint32_t *keys_out, *order_out;
    uint32_t *counts;  // [blocks][SORT_BINS]
    ZeroParams zero;
};

template <class I, bool FIRST>
__device__ __forceinline__ uint32_t sort_key(const SortParams &p, int i)
{
    if (!FIRST) return p.keys_in[i];
    const int64_t t = (int64_t)static_cast<const I *>(p.tokens)[i];
    return t >= 0 && t < (int64_t)p.V && t != p.padding ? (uint32_t)t : p.V;
}

// KEYS positions a workgroup, whose 16 waves share all M keys, and in a wave 64 / KEYS lanes share a position's: two operations
// for a pair of keys.  Every workgroup reads all tokens, so few positions a workgroup suit short batches, which would leave most CUs
// without any, and many the longer ones.  16 | 64, a whole gradient of V = 2000, D = 768, us: 100 tokens 8.9 | 11.2, 2048 13.1 | 16.4,
// 4096 15.5 | 19.8, 12000 35.7 | 33.4; V = 30522, with the zeros of 27000 rows beside it: 4096 27.1 | 28.1, 6000 36.1 | 30.9,
// 12000 51.1 | 42.3.  Keys behind a workgroup's group of 64 count if they are smaller, keys before it also if they are equal.
template <class I, int KEYS>
__global__ __launch_bounds__(RANK_THREADS) void rank_kernel(const SortParams p)
{
    if (blockIdx.x >= p.zero.first) {
        zero_rows(p.zero);
        return;
    }
    __shared__ __attribute__((aligned(16))) uint32_t keys[RANK_MAX];
    __shared__ uint32_t part[RANK_THREADS / 64][64];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int groups = (p.M + 63) / 64, own = blockIdx.x * KEYS / 64;
    for (int i = tid; i < groups * 64; i += 4 * RANK_THREADS) {  // (four on their way at a time)
        uint32_t k[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) k[j] = i + j * RANK_THREADS < p.M ? sort_key<I, true>(p, i + j * RANK_THREADS) : 0xFFFFFFFFu;
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (i + j * RANK_THREADS < groups * 64) keys[i + j * RANK_THREADS] = k[j];
    }
    __syncthreads();
    const int mine = blockIdx.x * KEYS + lane % KEYS, sharer = lane / KEYS;
    const uint32_t key = keys[mine];
    uint32_t count = 0;
    for (int g = wave; g < groups; g += RANK_THREADS / 64) {
        const int first = g * 64 + sharer * KEYS;
        const uint4 *at = reinterpret_cast<const uint4 *>(keys + first);
        if (g == own) {
            for (int j = 0; j < KEYS; ++j) {
                const uint32_t k = keys[first + j];
                count += k < key || (k == key && first + j < mine);
            }
        } else {
            const uint32_t limit = g < own ? key + 1 : key;  // (keys are at most V < 2^31, but for the places behind M, which nobody asks for)
#pragma unroll
            for (int j = 0; j < KEYS / 4; ++j) {
                const uint4 k = at[j];
                count += k.x < limit;
                count += k.y < limit;
                count += k.z < limit;
                count += k.w < limit;
            }
        }
    }
    part[wave][lane] = count;
    __syncthreads();
    if (wave != 0) return;
#pragma unroll
    for (int w = 1; w < RANK_THREADS / 64; ++w) count += part[w][lane];
#pragma unroll
    for (int d = KEYS; d < 64; d *= 2) count += __shfl_xor(count, d, 64);
    if (sharer != 0 || mine >= p.M) return;
    p.keys_out[count] = key;
    p.order_out[count] = (uint32_t)mine;
}

template <class I, bool FIRST>
__global__ __launch_bounds__(SORT_THREADS) void sort_count_kernel(const SortParams p)
{
    if (blockIdx.x >= p.zero.first) {
        zero_rows(p.zero);
        return;
    }
    __shared__ uint32_t bins[SORT_BINS];
    if (threadIdx.x < SORT_BINS) bins[threadIdx.x] = 0;
    __syncthreads();
    const uint32_t mask = (1u << p.bits) - 1;
    const int64_t from = (int64_t)blockIdx.x * p.per_block;
    const int to = (int)(from + p.per_block < p.M ? from + p.per_block : p.M);
    for (int64_t tile = from; tile < to; tile += SORT_TILE) {
        uint32_t key[SORT_ROUNDS];
#pragma unroll
        for (int r = 0; r < SORT_ROUNDS; ++r) {
            const int64_t i = tile + r * SORT_THREADS + threadIdx.x;
            key[r] = i < to ? sort_key<I, FIRST>(p, (int)i) : 0;
        }
#pragma unroll
        for (int r = 0; r < SORT_ROUNDS; ++r)
            if (tile + r * SORT_THREADS + threadIdx.x < to) atomicAdd(&bins[(key[r] >> p.shift) & mask], 1u);
    }
    __syncthreads();
    if (threadIdx.x < SORT_BINS) p.counts[blockIdx.x * SORT_BINS + threadIdx.x] = bins[threadIdx.x];
}

// A workgroup finds where its share of every digit begins (all counts of smaller digits, and those of the digit in the
// workgroups before), then places its positions tile by tile.  Within a tile a wave's positions are neighbours: a position's
// place is the digit's start, plus the counts of the waves before, plus the lanes before it with the same digit (ballots).
// Few large workgroups: each reads all workgroups' counts, and 64 of them with 1024 positions each took 22 us for 65536 positions.
template <class I, bool FIRST>
__global__ __launch_bounds__(SORT_THREADS) void sort_place_kernel(const SortParams p)
{
    if (blockIdx.x >= p.zero.first) {
        zero_rows(p.zero);
        return;
    }
    __shared__ uint32_t start[SORT_BINS], count[SORT_WAVES][SORT_BINS], part[2][SORT_BINS], sums[SORT_BINS / 64];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const uint32_t mask = (1u << p.bits) - 1;
    const int64_t from = (int64_t)blockIdx.x * p.per_block;
    const int to = (int)(from + p.per_block < p.M ? from + p.per_block : p.M);
    uint32_t key[SORT_ROUNDS], ord[SORT_ROUNDS];
    auto fetch = [&](int64_t tile) {
#pragma unroll
        for (int r = 0; r < SORT_ROUNDS; ++r) {
            const int64_t i = tile + (wave * SORT_ROUNDS + r) * 64 + lane;
            key[r] = i < to ? sort_key<I, FIRST>(p, (int)i) : 0;
            ord[r] = FIRST ? (uint32_t)i : i < to ? p.order_in[i] : 0;
        }
    };
    fetch(from);
    {
        // digit tid % 2^bits, of every sharers-th workgroup: one round trip to memory for up to 8 sharers workgroups
        const int digits = 1 << p.bits, digit = tid & (digits - 1), share = tid >> p.bits, sharers = SORT_THREADS >> p.bits;
        if (tid < SORT_BINS) part[0][tid] = part[1][tid] = 0;
        uint32_t before = 0, all = 0;
        for (int b = share; b < p.blocks; b += 8 * sharers) {
            uint32_t c[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) c[i] = p.counts[(b + i * sharers < p.blocks ? b + i * sharers : b) * SORT_BINS + digit];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int from_block = b + i * sharers;
                all += from_block < p.blocks ? c[i] : 0;
                before += from_block < (int)blockIdx.x ? c[i] : 0;
            }
        }
        __syncthreads();
        atomicAdd(&part[0][digit], before);
        atomicAdd(&part[1][digit], all);
        __syncthreads();
        uint32_t upto = 0;
        if (tid < SORT_BINS) {  // sums over the digits: within a wave, then over the waves before
            before = part[0][tid];
            all = upto = part[1][tid];
#pragma unroll
            for (int off = 1; off < 64; off <<= 1) {
                const uint32_t v = __shfl_up(upto, off, 64);
                if (lane >= off) upto += v;
            }
            if (lane == 63) sums[wave] = upto;
        }
        __syncthreads();
        if (tid < SORT_BINS) {
            for (int w = 0; w < wave; ++w) upto += sums[w];
            start[tid] = upto - all + before;
        }
    }
    for (int64_t tile = from; tile < to; tile += SORT_TILE) {
        for (int b = tid; b < SORT_WAVES * SORT_BINS; b += SORT_THREADS) count[b / SORT_BINS][b % SORT_BINS] = 0;
        __syncthreads();
        uint32_t rank[SORT_ROUNDS];
        bool in[SORT_ROUNDS];
#pragma unroll
        for (int r = 0; r < SORT_ROUNDS; ++r) {
            in[r] = tile + (wave * SORT_ROUNDS + r) * 64 + lane < to;
            const uint32_t digit = (key[r] >> p.shift) & mask;
            uint64_t same = __ballot(in[r]);
            for (int b = 0; b < p.bits; ++b) {
                const uint64_t ones = __ballot((digit >> b) & 1);
                same &= (digit >> b) & 1 ? ones : ~ones;
            }
            const uint64_t below = same & ((1ull << lane) - 1);
            uint32_t seen = 0;
            if (in[r]) seen = __hip_atomic_load(&count[wave][digit], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
            __builtin_amdgcn_wave_barrier();
            if (in[r] && below == 0)
                __hip_atomic_store(&count[wave][digit], seen + (uint32_t)__popcll(same), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
            __builtin_amdgcn_wave_barrier();
            rank[r] = seen + (uint32_t)__popcll(below);
        }
        __syncthreads();
        if (tid < SORT_BINS) {  // counts -> starts of the waves, and of the next tile
            uint32_t at = start[tid];
#pragma unroll
            for (int w = 0; w < SORT_WAVES; ++w) {
                const uint32_t c = count[w][tid];
                count[w][tid] = at;
                at += c;
            }
            start[tid] = at;
        }
        __syncthreads();
#pragma unroll
        for (int r = 0; r < SORT_ROUNDS; ++r)
            if (in[r]) {
                const uint32_t to_at = count[wave][(key[r] >> p.shift) & mask] + rank[r];
                p.keys_out[to_at] = key[r];
                p.order_out[to_at] = ord[r];
            }
        if (tile + SORT_TILE < to) fetch(tile + SORT_TILE);
        __syncthreads();
    }
}

// ---- gradient: sums of runs of equal tokens -------------------------------------------------------------------------------
struct GradParams {
    const uint32_t *keys, *order;  // sorted
    const void *dy;
    void *grad;
    float *head, *tail;  // [chunks][pitch] sums of a chunk's first run, if it began before, and of its last, if it goes on
    int64_t ld_dy, ld_grad;
    int M, D, pitch, chunk, chunks;
    uint32_t V;
    float scale;
    int accumulate;
};

// Eight columns of a row of the gradient from d, of a row's sums
template <class O, bool VEC, bool ADD>
__device__ __forceinline__ void write_row8(const GradParams &p, uint32_t row, int d, const float (&sum)[8])
{
    typename O::raw *at = static_cast<typename O::raw *>(p.grad) + (int64_t)row * p.ld_grad + d;
    float v[8];
    if constexpr (VEC) {
        if (ADD) get8<O>(at, v);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = ADD ? __builtin_fmaf(sum[i], p.scale, v[i]) : product(sum[i], p.scale);
        put8<O>(at, v);
    } else {
        for (int i = 0; i < 8; ++i)
            if (d + i < p.D) at[i] = O::put(ADD ? __builtin_fmaf(sum[i], p.scale, O::get(at[i])) : product(sum[i], p.scale));
    }
}

// A workgroup sums the rows of `chunk` (at most 64) sorted positions.  The next rows are asked for before the sums at hand are written:
// loads and stores come back in one order, and a wave that asks behind its stores waits for both.  A run of one token that
// lies within the chunk goes straight to its row; the parts of one that crosses chunks are kept and joined by the next kernel, so
// that a token as frequent as the padding of a batch is spread over the chip like all others.
// VEC: D is a multiple of 8 and all rows of 16 bytes: a lane has eight neighbouring columns.  Otherwise a lane's eight columns are a
// workgroup's width apart, so that neighbouring lanes still ask for neighbouring values.
template <class E, class O, bool VEC, bool ADD>
__global__ __launch_bounds__(256) void sum_runs_kernel(const GradParams p)
{
    constexpr int AHEAD = VEC && E::BYTES == 2 ? 8 : 4;
    constexpr uint32_t NONE = 0xFFFFFFFFu;
    struct alignas(16) Eight {
        typename E::raw v[8];
    };
    const int c = blockIdx.x, tid = threadIdx.x, lane = tid & 63, width = blockDim.x;
    const int64_t from = (int64_t)c * p.chunk;
    const int to = (int)(from + p.chunk < p.M ? from + p.chunk : p.M);
    const bool in = from + lane < to;
    const uint32_t my_key = in ? p.keys[from + lane] : NONE, my_row = in ? p.order[from + lane] : 0;
    const uint32_t before = from > 0 ? p.keys[from - 1] : NONE, after = to < p.M ? p.keys[to] : NONE;
    const int n = __popcll(__ballot(my_key < p.V));  // (keys of V are behind all others)
    if (n == 0) return;
    // (all lanes stay in this loop, whether they have columns or not: the keys and rows that they hold are read across lanes)
    for (int base = 0; base < p.D; base += width * 8) {
        const int d = VEC ? base + tid * 8 : base + tid, stride = VEC ? 1 : width;
        float sum[8];
        uint32_t run = NONE;
        bool first = true;
        auto flush = [&](bool last) {
            const bool head = first && run == before;
            first = false;
            if (d >= p.D) return;
            if (head || (last && run == after)) {
                float *at = (head ? p.head : p.tail) + (int64_t)c * p.pitch + d;
                if constexpr (VEC) {
                    put8<ElemF32>(at, sum);
                } else {
                    for (int e = 0; e < 8; ++e)
                        if (d + e * stride < p.D) at[e * stride] = sum[e];
                }
            } else if constexpr (VEC) {
                write_row8<O, true, ADD>(p, run, d, sum);
            } else {
                typename O::raw *at = static_cast<typename O::raw *>(p.grad) + (int64_t)run * p.ld_grad + d;
                for (int e = 0; e < 8; ++e)
                    if (d + e * stride < p.D)
                        at[e * stride] = O::put(ADD ? __builtin_fmaf(sum[e], p.scale, O::get(at[e * stride])) : product(sum[e], p.scale));
            }
        };
        Eight rows[2][AHEAD];
        auto fetch = [&](int i, Eight(&to)[AHEAD]) {
            const typename E::raw *at[AHEAD];
#pragma unroll
            for (int a = 0; a < AHEAD; ++a) {
                const uint32_t r = (uint32_t)__builtin_amdgcn_readlane((int)my_row, i + a < n ? i + a : n - 1);
                at[a] = static_cast<const typename E::raw *>(p.dy) + (int64_t)r * p.ld_dy + d;
            }
            if (d < p.D) {
#pragma unroll
                for (int a = 0; a < AHEAD; ++a) {
                    if constexpr (VEC) {
#pragma unroll
                        for (int w = 0; w < (int)sizeof(Eight) / 16; ++w)
                            reinterpret_cast<uint4 *>(&to[a])[w] = reinterpret_cast<const uint4 *>(at[a])[w];
                    } else {
#pragma unroll
                        for (int e = 0; e < 8; ++e) to[a].v[e] = d + e * stride < p.D ? at[a][e * stride] : typename E::raw(0);
                    }
                }
            }
        };
        auto add = [&](int i, const Eight(&from)[AHEAD]) {
#pragma unroll
            for (int a = 0; a < AHEAD; ++a) {
                if (i + a >= n) break;
                const uint32_t key = (uint32_t)__builtin_amdgcn_readlane((int)my_key, i + a);
                if (key != run) {
                    if (run != NONE) flush(false);
                    run = key;
#pragma unroll
                    for (int e = 0; e < 8; ++e) sum[e] = E::get(from[a].v[e]);
                } else {
#pragma unroll
                    for (int e = 0; e < 8; ++e) sum[e] += E::get(from[a].v[e]);
                }
            }
        };
        fetch(0, rows[0]);
        for (int i = 0; i < n; i += 2 * AHEAD) {
            if (i + AHEAD < n) fetch(i + AHEAD, rows[1]);
            add(i, rows[0]);
            if (i + 2 * AHEAD < n) fetch(i + 2 * AHEAD, rows[0]);
            add(i + AHEAD, rows[1]);
        }
        flush(true);
    }
}

// Joins the parts of the runs that cross chunks.  Workgroup c of the first `chunks` - 1 has the run that begins in chunk c, if it goes
// on, but over fewer than JOIN_SHORT chunks more.  A longer one covers a boundary whose number is a multiple of JOIN_SHORT: the
// first such boundary's JOIN_SHARES workgroups have a share of its columns each.  (Workgroups for all shares of all chunks, of which
// nearly all found nothing to do, took 17 us for 1024 chunks; a binary search for a run's end 11 us of latencies.)  Threads that share
// columns take the chunks in turn, and their sums are added in a fixed order.
constexpr int JOIN_SHARES = 8, JOIN_SHORT = 16;
template <class O, bool VEC, bool ADD>
__global__ __launch_bounds__(256) void join_runs_kernel(const GradParams p)
{
    __shared__ __attribute__((aligned(16))) float part[256][8];
    __shared__ int ends;
    const int tid = threadIdx.x;
    // whether a run of this key crosses boundary k (the begin of chunk k, 0 < k < chunks)
    auto crosses = [&](int k, uint32_t run) { return p.keys[(int64_t)k * p.chunk - 1] == run && p.keys[(int64_t)k * p.chunk] == run; };
    int c, last, share = -1;
    uint32_t run;
    if ((int)blockIdx.x < p.chunks - 1) {
        c = blockIdx.x;
        run = p.keys[(int64_t)(c + 1) * p.chunk - 1];
        const uint32_t next = p.keys[(int64_t)(c + 1) * p.chunk], begun = c > 0 ? p.keys[(int64_t)c * p.chunk - 1] : 0xFFFFFFFFu;
        const int k = c + 2 + (tid & 63);  // (a wave has all it needs, and all waves find the same)
        const bool goes_on = (tid & 63) < JOIN_SHORT && k < p.chunks && p.keys[(int64_t)k * p.chunk] == run;
        if (run >= p.V || next != run || begun == run) return;  // (sorted: begun == run says that it began before)
        last = c + 1 + __builtin_ctzll(~__ballot(goes_on));
        if (last - c >= JOIN_SHORT) return;
    } else {
        const int job = blockIdx.x - (p.chunks - 1), m = (job / JOIN_SHARES + 1) * JOIN_SHORT;
        share = job % JOIN_SHARES;
        run = p.keys[(int64_t)m * p.chunk];
        if (run >= p.V || !crosses(m, run) || (m > JOIN_SHORT && crosses(m - JOIN_SHORT, run))) return;
        const int back = tid & 63;
        const bool longer = back < JOIN_SHORT && m - back > 0 && crosses(m - back, run);
        c = m - __builtin_ctzll(~__ballot(longer));  // (boundaries m, m - 1, .. are crossed: as many chunks back it begins)
        last = m;
        for (int base = m + 1; base < p.chunks; base += 256) {
            if (tid == 0) ends = 256;
            __syncthreads();
            const int k = base + tid;
            if (!(k < p.chunks && p.keys[(int64_t)k * p.chunk] == run)) atomicMin(&ends, tid);
            __syncthreads();
            const int e = ends;
            last = base + e - 1;
            __syncthreads();
            if (e < 256) break;
        }
        if (last - c < JOIN_SHORT) return;
    }
    const int units = p.pitch / 8;
    int u0 = 0, u1 = units;
    if (share >= 0) {
        const int per = (units + JOIN_SHARES - 1) / JOIN_SHARES;
        u0 = share * per;
        u1 = u0 + per < units ? u0 + per : units;
    }
    for (; u0 < u1; u0 += 256) {
        const int tx = u1 - u0 < 256 ? u1 - u0 : 256;
        int sharers = 256 / tx;  // (no more than there are chunks for, and their sums are added one by one: all 51 of 39 columns took 8 us more)
        sharers = sharers < 32 ? sharers : 32;
        sharers = sharers < last - c + 1 ? sharers : last - c + 1;
        const int r = tid / tx, u = u0 + tid - r * tx;
        float sum[8] = {};
        if (r < sharers) {
#pragma unroll 4
            for (int k = c + r; k <= last; k += sharers) {
                float v[8];
                load8<float>((k == c ? p.tail : p.head) + (int64_t)k * p.pitch + u * 8, v);
#pragma unroll
                for (int e = 0; e < 8; ++e) sum[e] += v[e];
            }
        }
        __syncthreads();
#pragma unroll
        for (int e = 0; e < 8; ++e) part[tid][e] = sum[e];
        __syncthreads();
        if (r == 0) {
            for (int s = 1; s < sharers; ++s)
#pragma unroll
                for (int e = 0; e < 8; ++e) sum[e] += part[s * tx + tid][e];
            write_row8<O, VEC, ADD>(p, run, u * 8, sum);
        }
    }
}

// ---- host side ------------------------------------------------------------------------------------------------------------
constexpr int64_t MAX_ROWS = 0x7FFFFFF0, MAX_COLUMNS = 0x7FFF0000;  // (columns are counted up in ints, past the last by up to 2048)

static bool finite(float v) { return v - v == 0.0f; }
static bool tokens_aligned(const void *p, int bits) { return reinterpret_cast<uintptr_t>(p) % (bits / 8) == 0; }
template <class F>
static void with_index(int bits, F &&f)
{
    if (bits == 64) f(int64_t());
    else f(int32_t());
}
template <class F>
static void with_bool(bool b, F &&f)
{
    if (b) f(std::true_type());
    else f(std::false_type());
}

template <class Row>
static int launch_lookup(LookupParams p, bool table_vec, int out_dtype, hipStream_t st)
{
    const int64_t units = ceil_div(p.D, 8);
    p.threads_per_row = (int)(units < 256 ? units : 256);
    const int rows = 256 / p.threads_per_row;
    // Four rows a thread where that still leaves a workgroup for every place on the chip, eight a CU.  One | four, us, binary16 rows of 768 from
    // as many: 2048 tokens 3.5 | 3.9, 4096 4.7 | 4.6, 8192 7.8 | 6.6, 16384 (from where four are taken) 12.0 | 9.3, 65536 47.6 | 38.1; from
    // nibbles 3.0 | 4.0, 3.9 | 4.5, 6.0 | 5.9, 9.6 | 8.1, 38.1 | 31.2; rows of 1001 8192 11.4 | 15.7, 16384 19.9 | 17.5, 65536 101 | 97.  binary32 rows
    // lose a little by it: of 768 16384 16.6 | 16.9, 65536 73.9 | 76.9, of 2056 32768 97 | 110, but from nibbles 60.5 | 57.4 and 84 | 80.
    const bool four = p.M >= (int64_t)rows * 4 * 2048;
    int64_t workgroups = ceil_div(p.M, rows * (four ? 4 : 1));
    if (workgroups > 1 << 20) workgroups = 1 << 20;
    with_elem(out_dtype, [&](auto o) {
        with_bool(table_vec && p.D % 8 == 0 && (p.ld_out * decltype(o)::BYTES) % 16 == 0, [&](auto v) {
            with_bool(four, [&](auto f) {
                lookup_kernel<Row, decltype(o), decltype(v)::value, decltype(f)::value ? 4 : 1><<<(unsigned)workgroups, 256, 0, st>>>(p);
            });
        });
    });
    return launch_status();
}

// Waves that sum a chunk, eight columns a lane
static int grad_waves(int64_t D) { return D > 1536 ? 4 : (int)ceil_div(D, 512); }
// Sorted positions of a chunk: 8 to 64, about 2000 waves of them.  (Half as many waves: 16453 bfloat16 rows of 429 20.5 instead of 13.2 us.)
static int grad_chunk(int64_t M, int64_t D)
{
    if (M <= 64) return 64;  // one, which needs no joining
    int chunk = 8;
    while (chunk < 64 && M * grad_waves(D) > (int64_t)chunk * 2048) chunk *= 2;
    return chunk;
}

struct GradWorkspace {
    size_t keys[2], order[2], counts, head, tail, total;
    int chunk, chunks, pitch;
};
static GradWorkspace grad_workspace(int64_t M, int64_t D)
{
    GradWorkspace w;
    size_t at = 0;
    auto take = [&](size_t bytes) {
        const size_t here = at;
        at += (bytes + 255) / 256 * 256;
        return here;
    };
    w.chunk = grad_chunk(M, D);
    w.chunks = (int)ceil_div(M, w.chunk);
    w.pitch = (int)(ceil_div(D, 8) * 8);
    for (int i = 0; i < 2; ++i) {
        w.keys[i] = take((size_t)M * 4);
        w.order[i] = take((size_t)M * 4);
    }
    w.counts = take((size_t)SORT_BLOCKS * SORT_BINS * 4);
    w.head = take((size_t)w.chunks * w.pitch * 4);
    w.tail = take((size_t)w.chunks * w.pitch * 4);
    w.total = at;
    return w;
}

}  // namespace mkq

using namespace mkq;

extern "C" int mkq_embedding(const void *tokens, int token_bits, int64_t M, const void *table, int table_dtype, int64_t V, int64_t D,
                             int64_t ld_table, float scale, void *out, int out_dtype, int64_t ld_out, void *stream)
{
    if (!is_float_dtype(table_dtype) || !is_float_dtype(out_dtype) || (token_bits != 32 && token_bits != 64)) return MKQ_ERR_DTYPE;
    if (M < 0 || V <= 0 || D <= 0 || ld_table < D || ld_out < D) return MKQ_ERR_SHAPE;
    if (!finite(scale)) return MKQ_ERR_SCALE;
    if (M == 0) return MKQ_OK;
    if (!tokens || !table || !out) return MKQ_ERR_NULL;
    if (!tokens_aligned(tokens, token_bits) || !aligned16(table) || !aligned16(out)) return MKQ_ERR_ALIGN;
    if (V > MAX_ROWS || D > MAX_COLUMNS) return MKQ_ERR_UNSUPPORTED;
    const LookupParams p = {tokens, table, nullptr, out, M, ld_table, ld_out, (uint32_t)V, (int)D, 0, 0, token_bits, 0, scale};
    const hipStream_t st = as_stream(stream);
    int status = MKQ_OK;
    with_elem(table_dtype, [&](auto e) { status = launch_lookup<FloatRow<decltype(e)>>(p, (ld_table * decltype(e)::BYTES) % 16 == 0, out_dtype, st); });
    return status;
}

extern "C" int mkq_embedding_int4_group(const void *tokens, int token_bits, int64_t M, const uint8_t *Wq, const float *s_w, int group,
                                        int64_t V, int64_t D, float scale, void *out, int out_dtype, int64_t ld_out, void *stream)
{
    if (!is_float_dtype(out_dtype) || (token_bits != 32 && token_bits != 64)) return MKQ_ERR_DTYPE;
    if (M < 0 || V <= 0 || D <= 0 || ld_out < D || (group != 32 && group != 64 && group != 128)) return MKQ_ERR_SHAPE;
    if (!finite(scale)) return MKQ_ERR_SCALE;
    if (M == 0) return MKQ_OK;
    if (!tokens || !Wq || !s_w || !out) return MKQ_ERR_NULL;
    if (!tokens_aligned(tokens, token_bits) || !aligned16(Wq) || !aligned4(s_w) || !aligned16(out)) return MKQ_ERR_ALIGN;
    if (V > MAX_ROWS || D > MAX_COLUMNS) return MKQ_ERR_UNSUPPORTED;
    const LookupParams p = {tokens, Wq, s_w, out, M, ceil_div(D, 32) * 4, ld_out, (uint32_t)V, (int)D, (int)ceil_div(D, group),
                            group == 32 ? 5 : group == 64 ? 6 : 7, token_bits, 0, scale};
    return launch_lookup<NibbleRow>(p, true, out_dtype, as_stream(stream));
}

extern "C" size_t mkq_embedding_gradient_workspace_bytes(int64_t M, int64_t D)
{
    if (M <= 0 || D <= 0 || M > MAX_ROWS || D > MAX_COLUMNS) return 0;
    return grad_workspace(M, D).total;
}

extern "C" int mkq_embedding_gradient(const void *tokens, int token_bits, int64_t M, const void *dy, int dy_dtype, int64_t ld_dy, int64_t V,
                                      int64_t D, float scale, int64_t padding_token, int accumulate, void *grad, int grad_dtype,
                                      int64_t ld_grad, void *workspace, size_t workspace_bytes, void *stream)
{
    if (!is_float_dtype(dy_dtype) || !is_float_dtype(grad_dtype) || (token_bits != 32 && token_bits != 64)) return MKQ_ERR_DTYPE;
    if (M < 0 || V <= 0 || D <= 0 || ld_dy < D || ld_grad < D) return MKQ_ERR_SHAPE;
    if (!finite(scale)) return MKQ_ERR_SCALE;
    if (!grad || (M > 0 && (!tokens || !dy))) return MKQ_ERR_NULL;
    if ((M > 0 && (!tokens_aligned(tokens, token_bits) || !aligned16(dy))) || !aligned16(grad)) return MKQ_ERR_ALIGN;
    if (M > MAX_ROWS || V > MAX_ROWS || D > MAX_COLUMNS) return MKQ_ERR_UNSUPPORTED;
    const hipStream_t st = as_stream(stream);
    GradParams g = {};
    g.dy = dy;
    g.grad = grad;
    g.ld_dy = ld_dy;
    g.ld_grad = ld_grad;
    g.M = (int)M;
    g.D = (int)D;
    g.V = (uint32_t)V;
    g.scale = scale;
    g.accumulate = accumulate != 0;
    const bool vec_grad = (ld_grad * dtype_bytes(grad_dtype)) % 16 == 0;
    GradWorkspace w = {};
    uint8_t *ws = static_cast<uint8_t *>(workspace);
    if (M > 0) {
        w = grad_workspace(M, D);
        if (!workspace || workspace_bytes < w.total) return MKQ_ERR_WORKSPACE;
        if (!aligned16(workspace)) return MKQ_ERR_ALIGN;
        if (!grid_ok((int64_t)w.chunks * 2, 256)) return MKQ_ERR_UNSUPPORTED;
    }
    // share i of n of the rows to fill with zeros, behind `first` workgroups; *workgroups: how many more for it
    auto zero_share = [&](int i, int n, unsigned first, int threads, unsigned *workgroups) {
        ZeroParams z = {grad, ld_grad, V * i / n, V * (i + 1) / n, (int)D, (int)dtype_bytes(grad_dtype), vec_grad, first};
        const int64_t vectors = (z.rows_to - z.rows_from) * ceil_div(D * z.bytes, 16), most = 262144 / threads;
        const int64_t need = ceil_div(vectors, threads);
        *workgroups = g.accumulate ? 0 : (unsigned)(need < most ? need : most);
        return z;
    };
    if (M == 0) {
        unsigned workgroups;
        const ZeroParams z = zero_share(0, 1, 0, 256, &workgroups);
        if (workgroups == 0) return MKQ_OK;
        zero_rows_kernel<<<workgroups, 256, 0, st>>>(z);
        return launch_status();
    }

    SortParams s = {};
    s.tokens = tokens;
    s.padding = padding_token;
    s.M = (int)M;
    s.V = (uint32_t)V;
    s.counts = reinterpret_cast<uint32_t *>(ws + w.counts);
    unsigned zeros;
    if (M <= RANK_MAX) {
        s.keys_out = reinterpret_cast<uint32_t *>(ws + w.keys[0]);
        s.order_out = reinterpret_cast<uint32_t *>(ws + w.order[0]);
        with_index(token_bits, [&](auto i) {
            auto rank = [&](auto keys) {
                constexpr int KEYS = decltype(keys)::value;
                const unsigned blocks = (unsigned)ceil_div(M, KEYS);
                s.zero = zero_share(0, 1, blocks, RANK_THREADS, &zeros);
                rank_kernel<decltype(i), KEYS><<<blocks + zeros, RANK_THREADS, 0, st>>>(s);
            };
            if (M <= RANK_FEW)
                rank(std::integral_constant<int, 16>());
            else
                rank(std::integral_constant<int, 64>());
        });
    } else {
        s.per_block = (int)(ceil_div(ceil_div(M, SORT_BLOCKS), SORT_TILE) * SORT_TILE);
        s.blocks = (int)ceil_div(M, s.per_block);
        int key_bits = 1;  // of 0 .. V
        while (((int64_t)1 << key_bits) <= V) ++key_bits;
        const int passes = (key_bits + 8) / 9;
        s.bits = (key_bits + passes - 1) / passes;
        for (int pass = 0; pass < passes; ++pass) {
            s.shift = pass * s.bits;
            s.keys_in = pass ? reinterpret_cast<uint32_t *>(ws + w.keys[(pass + 1) & 1]) : nullptr;
            s.order_in = pass ? reinterpret_cast<uint32_t *>(ws + w.order[(pass + 1) & 1]) : nullptr;
            s.keys_out = reinterpret_cast<uint32_t *>(ws + w.keys[pass & 1]);
            s.order_out = reinterpret_cast<uint32_t *>(ws + w.order[pass & 1]);
            with_index(token_bits, [&](auto i) {
                with_bool(pass == 0, [&](auto first) {
                    s.zero = zero_share(2 * pass, 2 * passes, s.blocks, SORT_THREADS, &zeros);
                    sort_count_kernel<decltype(i), decltype(first)::value><<<s.blocks + zeros, SORT_THREADS, 0, st>>>(s);
                    s.zero = zero_share(2 * pass + 1, 2 * passes, s.blocks, SORT_THREADS, &zeros);
                    sort_place_kernel<decltype(i), decltype(first)::value><<<s.blocks + zeros, SORT_THREADS, 0, st>>>(s);
                });
            });
            if (launch_status() != MKQ_OK) return MKQ_ERR_HIP;
        }
    }
    g.keys = s.keys_out;
    g.order = s.order_out;
    g.head = reinterpret_cast<float *>(ws + w.head);
    g.tail = reinterpret_cast<float *>(ws + w.tail);
    g.chunk = w.chunk;
    g.chunks = w.chunks;
    g.pitch = w.pitch;
    const unsigned join_workgroups = (unsigned)(g.chunks - 1 + (g.chunks - 1) / JOIN_SHORT * JOIN_SHARES);
    const int sum_threads = 64 * grad_waves(D);
    with_elem(dy_dtype, [&](auto e) {
        with_elem(grad_dtype, [&](auto o) {
            with_bool(vec_grad && (ld_dy * decltype(e)::BYTES) % 16 == 0 && D % 8 == 0, [&](auto v) {
                with_bool(g.accumulate, [&](auto add) {
                    constexpr bool VEC = decltype(v)::value, ADD = decltype(add)::value;
                    sum_runs_kernel<decltype(e), decltype(o), VEC, ADD><<<g.chunks, sum_threads, 0, st>>>(g);
                    if (g.chunks > 1) join_runs_kernel<decltype(o), VEC, ADD><<<join_workgroups, 256, 0, st>>>(g);
                });
            });
        });
    });
    return launch_status();
}
