// Token rows: the lookup from a float table and from a group-scaled 4-bit one, and the table's gradient by sorted tokens.
//
//     out[i,:] = scale * table[t_i,:]              dT[v,:] = scale * sum_{i: t_i = v} dy[i,:]
//
// All are bound by bytes: the rows read and written, and for the gradient the whole of dT, whose rows without a token are
// zeros.  A lookup is one multiplication in binary32 and one rounding per value.
#include "elements.h"

namespace mkq {

template <class I>
__device__ __forceinline__ uint32_t token_row(const I *__restrict__ tokens, int64_t i, uint32_t V)
{
    const int64_t t = (int64_t)tokens[i];
    return t >= 0 && t < (int64_t)V ? (uint32_t)t : 0xFFFFFFFFu;
}

// ---- lookup -------------------------------------------------------------------------------------------------------------
struct LookupParams {
    const void *tokens;
    const void *table;  // float rows, or rows of nibbles
    const float *s_w;   // [V, groups] of the nibbles
    void *out;
    int64_t M, ld_table, ld_out;
    uint32_t V;
    int D, groups, units, threads_per_row;
    float scale;
};

// Where a row's values come from: eight at position d (a multiple of 8), zeros from D on
template <class E, bool VEC>
struct FloatRow {
    const typename E::raw *row;
    __device__ __forceinline__ FloatRow(const LookupParams &p, uint32_t r) : row(static_cast<const typename E::raw *>(p.table) + (int64_t)r * p.ld_table) {}
    __device__ __forceinline__ void get(const LookupParams &p, int d, float (&v)[8]) const
    {
        if (VEC && d + 8 <= p.D) {
            get8<E>(row + d, v);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = d + i < p.D ? E::get(row[d + i]) : 0.0f;
        }
    }
};
template <int G>
struct NibbleRow {
    const uint32_t *row;
    const float *s;
    __device__ __forceinline__ NibbleRow(const LookupParams &p, uint32_t r)
        : row(static_cast<const uint32_t *>(p.table) + (int64_t)r * p.ld_table), s(p.s_w + (int64_t)r * p.groups) {}
    __device__ __forceinline__ void get(const LookupParams &, int d, float (&v)[8]) const
    {
        const uint32_t w = row[d / 8];
        const float step = s[d / G];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = (float)((int)(w << (28 - 4 * i)) >> 28) * step;
    }
};

// threads_per_row neighbouring threads write a token's row, eight values each at a time.
template <class Row, class O, class I, bool VEC_OUT>
__global__ __launch_bounds__(256) void lookup_kernel(const LookupParams p)
{
    const int rows = blockDim.x / p.threads_per_row;
    const int r = threadIdx.x / p.threads_per_row, u0 = threadIdx.x - r * p.threads_per_row;
    if (r >= rows) return;
    for (int64_t i = (int64_t)blockIdx.x * rows + r; i < p.M; i += (int64_t)gridDim.x * rows) {
        const uint32_t t = token_row(static_cast<const I *>(p.tokens), i, p.V);
        const bool known = t != 0xFFFFFFFFu;
        const Row row(p, known ? t : 0);
        typename O::raw *out = static_cast<typename O::raw *>(p.out) + i * p.ld_out;
        for (int u = u0; u < p.units; u += p.threads_per_row) {
            const int d = u * 8;
            float v[8];
            if (known) {
                row.get(p, d, v);
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] *= p.scale;
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = 0.0f;
            }
            if (VEC_OUT && d + 8 <= p.D) {
                put8<O>(out + d, v);
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (d + e < p.D) out[d + e] = O::put(v[e]);
            }
        }
    }
}

// ---- gradient: sorting the tokens ---------------------------------------------------------------------------------------
// Positions are put in the order of their tokens by a stable radix sort (least significant digit first, up to nine bits a
// pass), so equal tokens keep the order of the batch and a row's sum does not depend on how the work fell.  Tokens that
// count for nothing (the padding token, ids outside the table) get the key V, behind all others.
constexpr int SORT_BINS = 512, SORT_TILE = 1024, SORT_BLOCKS = 256;

struct SortParams {
    const void *tokens;
    int64_t padding;
    int M, per_block, blocks;  // positions of a workgroup: a multiple of SORT_TILE
    uint32_t V;
    int shift, bits;
    const uint32_t *keys_in, *order_in;  // null in the first pass: keys come from the tokens
    uint32_t *keys_out, *order_out;
    uint32_t *counts;  // [blocks][SORT_BINS]
};

template <class I, bool FIRST>
__device__ __forceinline__ uint32_t sort_key(const SortParams &p, int i)
{
    if (!FIRST) return p.keys_in[i];
    const int64_t t = (int64_t)static_cast<const I *>(p.tokens)[i];
    return t >= 0 && t < (int64_t)p.V && t != p.padding ? (uint32_t)t : p.V;
}

template <class I, bool FIRST>
__global__ __launch_bounds__(256) void sort_count_kernel(const SortParams p)
{
    __shared__ uint32_t bins[SORT_BINS];
    for (int b = threadIdx.x; b < SORT_BINS; b += 256) bins[b] = 0;
    __syncthreads();
    const uint32_t mask = (1u << p.bits) - 1;
    const int64_t from = (int64_t)blockIdx.x * p.per_block;
    const int to = (int)(from + p.per_block < p.M ? from + p.per_block : p.M);
    for (int i = (int)from + threadIdx.x; i < to; i += 256) atomicAdd(&bins[(sort_key<I, FIRST>(p, i) >> p.shift) & mask], 1u);
    __syncthreads();
    for (int b = threadIdx.x; b < SORT_BINS; b += 256) p.counts[blockIdx.x * SORT_BINS + b] = bins[b];
}

// A workgroup finds where its share of every digit begins (all counts of smaller digits, and those of the digit in the
// workgroups before), then places its positions tile by tile.  Within a tile every wave has 256 neighbours: a position's
// place is the digit's start, plus the counts of the waves before, plus the lanes before it with the same digit (ballots).
template <class I, bool FIRST>
__global__ __launch_bounds__(256) void sort_place_kernel(const SortParams p)
{
    __shared__ uint32_t start[SORT_BINS], count[4][SORT_BINS], part[256];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const uint32_t mask = (1u << p.bits) - 1;
    uint32_t before[2] = {0, 0}, all[2] = {0, 0};  // of digits 2 tid, 2 tid + 1
    for (int b = 0; b < p.blocks; ++b) {
        const uint2 c = *reinterpret_cast<const uint2 *>(p.counts + b * SORT_BINS + 2 * tid);
        all[0] += c.x;
        all[1] += c.y;
        if (b < (int)blockIdx.x) {
            before[0] += c.x;
            before[1] += c.y;
        }
    }
    part[tid] = all[0] + all[1];
    __syncthreads();
    for (int off = 1; off < 256; off <<= 1) {  // inclusive sums over the threads
        const uint32_t v = tid >= off ? part[tid - off] : 0;
        __syncthreads();
        part[tid] += v;
        __syncthreads();
    }
    const uint32_t base = part[tid] - all[0] - all[1];
    start[2 * tid] = base + before[0];
    start[2 * tid + 1] = base + all[0] + before[1];

    const int64_t from = (int64_t)blockIdx.x * p.per_block;
    const int to = (int)(from + p.per_block < p.M ? from + p.per_block : p.M);
    for (int64_t tile = from; tile < to; tile += SORT_TILE) {
        for (int b = tid; b < 4 * SORT_BINS; b += 256) count[b / SORT_BINS][b % SORT_BINS] = 0;
        __syncthreads();
        uint32_t key[4], ord[4], rank[4];
        bool in[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int64_t i = tile + wave * 256 + r * 64 + lane;
            in[r] = i < to;
            key[r] = in[r] ? sort_key<I, FIRST>(p, (int)i) : 0;
            ord[r] = FIRST ? (uint32_t)i : in[r] ? p.order_in[i] : 0;
        }
#pragma unroll
        for (int r = 0; r < 4; ++r) {
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
        for (int b = tid; b < SORT_BINS; b += 256) {  // counts -> starts of the waves, and of the next tile
            uint32_t at = start[b];
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                const uint32_t c = count[w][b];
                count[w][b] = at;
                at += c;
            }
            start[b] = at;
        }
        __syncthreads();
#pragma unroll
        for (int r = 0; r < 4; ++r)
            if (in[r]) {
                const uint32_t to_at = count[wave][(key[r] >> p.shift) & mask] + rank[r];
                p.keys_out[to_at] = key[r];
                p.order_out[to_at] = ord[r];
            }
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

template <class O, bool VEC>
__device__ __forceinline__ void write_row8(const GradParams &p, uint32_t row, int d, const float (&sum)[8])
{
    typename O::raw *at = static_cast<typename O::raw *>(p.grad) + (int64_t)row * p.ld_grad + d;
    float v[8];
    if (VEC && d + 8 <= p.D) {
        if (p.accumulate) get8<O>(at, v);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = p.accumulate ? __builtin_fmaf(sum[i], p.scale, v[i]) : sum[i] * p.scale;
        put8<O>(at, v);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (d + i < p.D) at[i] = O::put(p.accumulate ? __builtin_fmaf(sum[i], p.scale, O::get(at[i])) : sum[i] * p.scale);
    }
}

template <class O, bool VEC>
__global__ __launch_bounds__(256) void zero_rows_kernel(const GradParams p, int units)
{
    const int64_t total = (int64_t)p.V * units;
    for (int64_t w = (int64_t)blockIdx.x * 256 + threadIdx.x; w < total; w += (int64_t)gridDim.x * 256) {
        const int64_t row = w / units;
        const int d = (int)(w - row * units) * 8;
        typename O::raw *at = static_cast<typename O::raw *>(p.grad) + row * p.ld_grad + d;
        const float zero[8] = {};
        if (VEC && d + 8 <= p.D) {
            put8<O>(at, zero);
        } else {
            for (int i = 0; i < 8; ++i)
                if (d + i < p.D) at[i] = O::put(0.0f);
        }
    }
}

// A workgroup sums the rows of `chunk` sorted positions.  A run of one token that lies within the chunk goes straight to its
// row; the parts of one that crosses chunks are kept and joined by the next kernel, so that a token as frequent as the padding
// of a batch is spread over the chip like all others.
template <class E, class O, bool VEC>
__global__ __launch_bounds__(256) void sum_runs_kernel(const GradParams p)
{
    const int c = blockIdx.x;
    const int64_t from = (int64_t)c * p.chunk;
    const int to = (int)(from + p.chunk < p.M ? from + p.chunk : p.M);
    const uint32_t before = from > 0 ? p.keys[from - 1] : 0xFFFFFFFFu;
    const uint32_t after = to < p.M ? p.keys[to] : 0xFFFFFFFFu;
    for (int d = threadIdx.x * 8; d < p.D; d += 256 * 8) {
        float sum[8];
        uint32_t run = 0xFFFFFFFFu;
        bool first = true;
        auto flush = [&](bool last) {
            if (first && run == before) {
                float *at = p.head + (int64_t)c * p.pitch + d;
                reinterpret_cast<float4 *>(at)[0] = make_float4(sum[0], sum[1], sum[2], sum[3]);
                reinterpret_cast<float4 *>(at)[1] = make_float4(sum[4], sum[5], sum[6], sum[7]);
            } else if (last && run == after) {
                float *at = p.tail + (int64_t)c * p.pitch + d;
                reinterpret_cast<float4 *>(at)[0] = make_float4(sum[0], sum[1], sum[2], sum[3]);
                reinterpret_cast<float4 *>(at)[1] = make_float4(sum[4], sum[5], sum[6], sum[7]);
            } else {
                write_row8<O, VEC>(p, run, d, sum);
            }
            first = false;
        };
        for (int i = (int)from; i < to; ++i) {
            const uint32_t key = p.keys[i];
            if (key >= p.V) break;
            const typename E::raw *row = static_cast<const typename E::raw *>(p.dy) + (int64_t)p.order[i] * p.ld_dy + d;
            float v[8];
            if (VEC && d + 8 <= p.D) {
                get8<E>(row, v);
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = d + e < p.D ? E::get(row[e]) : 0.0f;
            }
            if (key != run) {
                if (run != 0xFFFFFFFFu) flush(false);
                run = key;
#pragma unroll
                for (int e = 0; e < 8; ++e) sum[e] = v[e];
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) sum[e] += v[e];
            }
        }
        if (run != 0xFFFFFFFFu) flush(true);
    }
}

// Joins the parts of the run that chunk blockIdx.x begins and does not end: 32 rows of 8 threads take the chunks it crosses in
// turn, 64 columns at a time, and their sums are added in a fixed order.
template <class O, bool VEC>
__global__ __launch_bounds__(256) void join_runs_kernel(const GradParams p)
{
    __shared__ float part[32][65];
    const int c = blockIdx.x;
    const int64_t from = (int64_t)c * p.chunk, to = from + p.chunk;
    if (to >= p.M) return;
    const uint32_t run = p.keys[to - 1];
    if (run >= p.V || p.keys[to] != run) return;
    if (from > 0 && p.keys[from] == run && p.keys[from - 1] == run) return;  // it began before
    int lo = (int)to, hi = p.M;  // the first position past the run
    while (lo < hi) {
        const int mid = lo + (hi - lo) / 2;
        if (p.keys[mid] <= run) lo = mid + 1;
        else hi = mid;
    }
    const int last = (lo - 1) / p.chunk;
    const int r = threadIdx.x >> 3, t = threadIdx.x & 7;
    const int d = blockIdx.y * 64 + t * 8;
    float sum[8] = {};
    if (d < p.D)
        for (int k = c + r; k <= last; k += 32) {
            const float *at = (k == c ? p.tail : p.head) + (int64_t)k * p.pitch + d;
            float v[8];
            load8<float>(at, v);
#pragma unroll
            for (int e = 0; e < 8; ++e) sum[e] += v[e];
        }
#pragma unroll
    for (int e = 0; e < 8; ++e) part[r][t * 8 + e] = sum[e];
    for (int half = 16; half > 0; half >>= 1) {
        __syncthreads();
        if (r < half)
#pragma unroll
            for (int e = 0; e < 8; ++e) part[r][t * 8 + e] += part[r + half][t * 8 + e];
    }
    if (r == 0 && d < p.D) {
#pragma unroll
        for (int e = 0; e < 8; ++e) sum[e] = part[0][t * 8 + e];
        write_row8<O, VEC>(p, run, d, sum);
    }
}

// ---- host side ------------------------------------------------------------------------------------------------------------
constexpr int64_t MAX_ROWS = 0x7FFFFFF0;

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

template <class Row, class O, class I>
static int launch_lookup(LookupParams p, hipStream_t st)
{
    p.units = (int)ceil_div(p.D, 8);
    p.threads_per_row = p.units < 256 ? p.units : 256;
    const int rows = 256 / p.threads_per_row;
    int64_t workgroups = ceil_div(p.M, rows);
    if (workgroups > 8192) workgroups = 8192;
    with_bool((p.ld_out * O::BYTES) % 16 == 0, [&](auto v) {
        lookup_kernel<Row, O, I, decltype(v)::value><<<(unsigned)workgroups, 256, 0, st>>>(p);
    });
    return launch_status();
}

// Chunks of sorted positions: about a thousand workgroups of them, 8 to 64 rows each
static int grad_chunk(int64_t M)
{
    int chunk = 8;
    while (chunk < 64 && M > (int64_t)chunk * 1024) chunk *= 2;
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
    w.chunk = grad_chunk(M);
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
    if (V > MAX_ROWS || D > MAX_ROWS) return MKQ_ERR_UNSUPPORTED;
    LookupParams p = {tokens, table, nullptr, out, M, ld_table, ld_out, (uint32_t)V, (int)D, 0, 0, 0, scale};
    const hipStream_t st = as_stream(stream);
    int status = MKQ_OK;
    with_elem(table_dtype, [&](auto e) {
        with_elem(out_dtype, [&](auto o) {
            with_index(token_bits, [&](auto i) {
                with_bool((ld_table * decltype(e)::BYTES) % 16 == 0, [&](auto v) {
                    status = launch_lookup<FloatRow<decltype(e), decltype(v)::value>, decltype(o), decltype(i)>(p, st);
                });
            });
        });
    });
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
    if (V > MAX_ROWS || D > MAX_ROWS) return MKQ_ERR_UNSUPPORTED;
    LookupParams p = {tokens, Wq, s_w, out, M, ceil_div(D, 32) * 4, ld_out, (uint32_t)V, (int)D, (int)ceil_div(D, group), 0, 0, scale};
    const hipStream_t st = as_stream(stream);
    int status = MKQ_OK;
    with_elem(out_dtype, [&](auto o) {
        with_index(token_bits, [&](auto i) {
            using O = decltype(o);
            using I = decltype(i);
            if (group == 32) status = launch_lookup<NibbleRow<32>, O, I>(p, st);
            else if (group == 64) status = launch_lookup<NibbleRow<64>, O, I>(p, st);
            else status = launch_lookup<NibbleRow<128>, O, I>(p, st);
        });
    });
    return status;
}

extern "C" size_t mkq_embedding_gradient_workspace_bytes(int64_t M, int64_t D)
{
    if (M <= 0 || D <= 0 || M > MAX_ROWS || D > MAX_ROWS) return 0;
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
    if (M > MAX_ROWS || V > MAX_ROWS || D > MAX_ROWS) return MKQ_ERR_UNSUPPORTED;
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
    const int units = (int)ceil_div(D, 8);
    GradWorkspace w = {};
    uint8_t *ws = static_cast<uint8_t *>(workspace);
    if (M > 0) {
        w = grad_workspace(M, D);
        if (!workspace || workspace_bytes < w.total) return MKQ_ERR_WORKSPACE;
        if (!aligned16(workspace)) return MKQ_ERR_ALIGN;
        if (!grid_ok(w.chunks, 256) || ceil_div(D, 64) > 65535 || !grid_ok(w.chunks * ceil_div(D, 64), 256)) return MKQ_ERR_UNSUPPORTED;
    }
    if (!g.accumulate) {
        int64_t workgroups = ceil_div(V * units, 256);
        if (workgroups > 8192) workgroups = 8192;
        with_elem(grad_dtype, [&](auto o) {
            with_bool(vec_grad, [&](auto v) {
                zero_rows_kernel<decltype(o), decltype(v)::value><<<(unsigned)workgroups, 256, 0, st>>>(g, units);
            });
        });
        if (launch_status() != MKQ_OK) return MKQ_ERR_HIP;
    }
    if (M == 0) return MKQ_OK;

    SortParams s = {};
    s.tokens = tokens;
    s.padding = padding_token;
    s.M = (int)M;
    s.V = (uint32_t)V;
    s.per_block = (int)(ceil_div(ceil_div(M, SORT_BLOCKS), SORT_TILE) * SORT_TILE);
    s.blocks = (int)ceil_div(M, s.per_block);
    s.counts = reinterpret_cast<uint32_t *>(ws + w.counts);
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
                sort_count_kernel<decltype(i), decltype(first)::value><<<s.blocks, 256, 0, st>>>(s);
                sort_place_kernel<decltype(i), decltype(first)::value><<<s.blocks, 256, 0, st>>>(s);
            });
        });
        if (launch_status() != MKQ_OK) return MKQ_ERR_HIP;
    }
    g.keys = s.keys_out;
    g.order = s.order_out;
    g.head = reinterpret_cast<float *>(ws + w.head);
    g.tail = reinterpret_cast<float *>(ws + w.tail);
    g.chunk = w.chunk;
    g.chunks = w.chunks;
    g.pitch = w.pitch;
    with_elem(dy_dtype, [&](auto e) {
        with_elem(grad_dtype, [&](auto o) {
            with_bool(vec_grad && (ld_dy * decltype(e)::BYTES) % 16 == 0, [&](auto v) {
                sum_runs_kernel<decltype(e), decltype(o), decltype(v)::value><<<g.chunks, 256, 0, st>>>(g);
                join_runs_kernel<decltype(o), decltype(v)::value><<<dim3(g.chunks, (unsigned)ceil_div(D, 64)), 256, 0, st>>>(g);
            });
        });
    });
    return launch_status();
}
