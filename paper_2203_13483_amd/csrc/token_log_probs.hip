// Log probabilities of given tokens, entropies and the most probable alternatives of every row of scores, and the gradient of
// the first two with respect to the scores:
//
//     log p_j = scale (x_j - max) - L,   L = log sum_j exp(scale (x_j - max)),   H = -sum_j p_j log p_j
//     dx_j = scale (g (delta_jt - p_j) - h p_j (log p_j + H))
//
// Bound by bytes: the scores are read once (and read once more and written for the gradient).  What a score costs beside its load is
// vector issue: a fused product, an exponential, two sums and a maximum.  Measured, us a call among others (where calls come
// one by one, as in a trace, large ones take up to a fifth more): 8192 binary16 rows of 30522 with 20 alternatives 115 (4.3 TB/s; vector issue alone 81),
// 2048 bfloat16 rows of 131072 122 (4.4 TB/s) and their gradient 169 (6.3 TB/s); the kernel of one binary32 row of 30522 11.7.
//
// Rows of any alignment: with `shift` = the place of a row's first score modulo eight, the row is cut at multiples of eight
// counted from shift places before it, so that all whole vectors of eight are aligned to 16 bytes whatever the row stride is.
#include "elements.h"
#include "gemm_common.h"

namespace mkq {

constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;
constexpr float NO_MASS = -16384.0f;  // an exponent (base 2) whose power is 0, to be multiplied by it
// Rows whose largest scaled score (to the base 2) is beyond are summed relative to that score, in a pass of their own.  Up to here c * most rounded
// to binary32 is off by 2^-4 at most, and so is the largest score's exponent relative to what is rounded up from it.
constexpr float FAR = 0x1p20f;
constexpr float RISE = 4.0f;          // (exponents above the reference cancel in the logarithms, with the rounding of their size)
constexpr int TOP_MOST = 64;
constexpr int SCORE_UNROLL = 4;
constexpr int STEP = 64 * SCORE_UNROLL;  // vectors of eight neighbouring scores that a wave takes at a time
constexpr int STEPS_MOST = 64;           // of a workgroup that chooses alternatives: a lane's largest score of a step is kept, 16 KiB of LDS
constexpr int PARTS_MOST = 1024;         // of a row: from 2^27 columns on they have more steps each, up to 128 KiB at 2^30

struct ScoreParams {
    const void *logits;
    const void *tokens;
    int64_t ld, M;
    int V, token_bits, top;
    int parts, steps_per_part;
    float c;  // scale * log2(e)
    float scale;
    float *normalizers, *log_probs, *entropies;
    int32_t *top_tokens;
    float *top_log_probs;
    float4 *partials;          // [M, parts]
    unsigned long long *keys;  // [M, parts, top]
};

// What is known of some of a row's scores: the largest, and relative to 2^ref (of scaled scores to the base 2) the sum of the powers and
// of the powers times their exponents.  ref is a whole number near the largest, not the largest itself, so that c x - ref is one fused
// operation with one rounding.  It is raised only when a score is 2^RISE above it.  Where the largest scaled score of a row is
// beyond FAR, sums are relative to it: `far` says so, and ref means nothing.
struct Mass {
    float most, ref, sum, weighted;
};
__device__ __forceinline__ bool is_far(float most, float c) { return !(fabsf(most * c) <= FAR); }
// The exponent's distance between two references, of which `to` is not the smaller
__device__ __forceinline__ float fall(float from, float to) { return fmaxf(from - to, NO_MASS); }
__device__ __forceinline__ void rebase(Mass &m, float by)
{
    const float f = __builtin_amdgcn_exp2f(by);
    m.weighted = __builtin_fmaf(m.sum, by, m.weighted) * f;
    m.sum *= f;
}

__device__ __forceinline__ int64_t given_token(const void *tokens, int bits, int64_t row)
{
    return bits == 64 ? static_cast<const int64_t *>(tokens)[row] : (int64_t)static_cast<const int32_t *>(tokens)[row];
}

// ---- the order of scores --------------------------------------------------------------------------------------------------
// A score and its place as one number: larger scores first, then lower places; -0 and 0 are equal, and a NaN is as low as -infinity.
// 0 is none.
typedef unsigned long long Key;
__device__ __forceinline__ uint32_t ordered(float v)
{
    const uint32_t b = __float_as_uint((v == v ? v : -__builtin_inff()) + 0.0f);
    return b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float from_ordered(uint32_t o) { return __uint_as_float(o & 0x80000000u ? o ^ 0x80000000u : ~o); }
__device__ __forceinline__ Key key_of(float v, uint32_t place) { return (Key)ordered(v) << 32 | (0xFFFFFFFFu - place); }
__device__ __forceinline__ uint32_t place_of(Key k) { return 0xFFFFFFFFu - (uint32_t)k; }

// The value of lane ^ OFF, by permutations of the vector unit
template <int OFF>
__device__ __forceinline__ uint32_t from_pair(uint32_t v)
{
    auto dpp = [](uint32_t u, auto perm) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)u, decltype(perm)::value, 0xF, 0xF, true); };
    if constexpr (OFF == 1) return dpp(v, IntC<0xB1>());
    else if constexpr (OFF == 2) return dpp(v, IntC<0x4E>());
    else if constexpr (OFF == 4) return dpp(dpp(v, IntC<0x141>()), IntC<0x1B>());  // of eight the last first, of four the last first
    else if constexpr (OFF == 8) return dpp(v, IntC<0x128>());
    else {
        const auto r = OFF == 32 ? __builtin_amdgcn_permlane32_swap(v, v, false, false) : __builtin_amdgcn_permlane16_swap(v, v, false, false);
        return (threadIdx.x & OFF) ? r[0] : r[1];
    }
}
template <int OFF>
__device__ __forceinline__ void compare_exchange(Key &k, bool keep_larger)
{
    const Key o = (Key)from_pair<OFF>((uint32_t)(k >> 32)) << 32 | from_pair<OFF>((uint32_t)k);
    k = (o > k) == keep_larger ? o : k;
}
// Stages OFF, OFF / 2 .. 1 of a bitonic network over the lanes; blocks of SIZE lanes run down and up in turn
template <int SIZE, int OFF>
__device__ __forceinline__ void bitonic(Key &k)
{
    const int lane = threadIdx.x & 63;
    compare_exchange<OFF>(k, ((lane & SIZE) == 0) == ((lane & OFF) == 0));
    if constexpr (OFF > 1) bitonic<SIZE, OFF / 2>(k);
}
__device__ __forceinline__ Key sorted_down(Key k)
{
    bitonic<2, 1>(k);
    bitonic<4, 2>(k);
    bitonic<8, 4>(k);
    bitonic<16, 8>(k);
    bitonic<32, 16>(k);
    bitonic<64, 32>(k);
    return k;
}
__device__ __forceinline__ Key lane_key(Key k, int lane)
{
    return (Key)(uint32_t)__builtin_amdgcn_readlane((int)(k >> 32), lane) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)k, lane);
}
// The 64 largest of two lists that run down
__device__ __forceinline__ Key merged(Key a, Key b)
{
    const int turned = 63 - (threadIdx.x & 63);
    const Key t = (Key)(uint32_t)__shfl((int)(b >> 32), turned, 64) << 32 | (uint32_t)__shfl((int)b, turned, 64);
    a = t > a ? t : a;
    bitonic<64, 32>(a);
    return a;
}

// A wave's largest keys, running down over the lanes: those given that are at least `least`.  (64 a time, through `room` of 128.)
struct Choice {
    Key best = 0, least;
    int waiting = 0, top;
    bool any = false;
    Key *room;
    __device__ __forceinline__ Choice(Key *room, int top, Key least) : least(least), top(top), room(room) {}
    __device__ __forceinline__ void take(Key batch)
    {
        batch = sorted_down(batch);
        best = any ? merged(best, batch) : batch;
        any = true;
        const Key last = lane_key(best, top - 1);
        least = last > least ? last : least;
    }
    // A key of each lane, 0 for none; all lanes come here together
    __device__ __forceinline__ void add(Key k)
    {
        const bool pass = k != 0 && k >= least;
        const uint64_t mask = __ballot(pass);
        if (!mask) return;
        const int before = __builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0u));
        if (pass) room[waiting + before] = k;
        waiting += __popcll(mask);
        wave_order();
        if (waiting >= 64) {
            const int lane = threadIdx.x & 63;
            const Key batch = room[lane], rest = room[64 + lane];
            wave_order();
            waiting -= 64;
            if (lane < waiting) room[lane] = rest;
            wave_order();
            take(batch);
        }
    }
    __device__ __forceinline__ Key finish()
    {
        const int lane = threadIdx.x & 63;
        if (waiting) take(lane < waiting ? room[lane] : 0);
        waiting = 0;
        return best;
    }
};

// The `top` largest of n keys: the top-th largest of the lanes' own largest is a bound that most keys do not reach
template <class F>
__device__ __forceinline__ Key choose(int n, int top, Key *room, F &&key)
{
    const int lane = threadIdx.x & 63;
    Key mine = 0;
#pragma unroll 4
    for (int i = lane; i < n; i += 64) {
        const Key k = key(i);
        mine = k > mine ? k : mine;
    }
    mine = sorted_down(mine);
    if (n <= 64) return mine;
    Choice choice(room, top, lane_key(mine, top - 1));
    for (int i = 0; i < n; i += 64) choice.add(i + lane < n ? key(i + lane) : 0);
    return choice.finish();
}

// ---- one pass over the scores ---------------------------------------------------------------------------------------------
// Eight neighbouring scores as they are in memory
template <class E>
struct Eight {
    uint4 w[E::BYTES == 4 ? 2 : 1];
    __device__ __forceinline__ void fetch(const typename E::raw *at)
    {
#pragma unroll
        for (int i = 0; i < (int)(sizeof(w) / 16); ++i) w[i] = reinterpret_cast<const uint4 *>(at)[i];
    }
    __device__ __forceinline__ float get(int i) const
    {
        const uint4 &v = w[E::BYTES == 4 ? i / 4 : 0];
        const int at = E::BYTES == 4 ? i % 4 : i / 2;
        const uint32_t x = at == 0 ? v.x : at == 1 ? v.y : at == 2 ? v.z : v.w;
        if constexpr (E::BYTES == 4) return __uint_as_float(x);
        else return E::get((uint16_t)(x >> (16 * (i % 2))));
    }
};
// The largest of a lane's vectors, a quiet NaN as -infinity.  (Binary16: two at a time, so that get() is only an operand of the fused product)
template <class E, int N>
__device__ __forceinline__ float largest_of(const Eight<E> (&x)[N])
{
    float v = -__builtin_inff();
    if constexpr (std::is_same<E, ElemF16>::value) {
        uint32_t two = 0xFC00FC00u;
        auto take = [&](uint32_t w) { asm("v_pk_max_f16 %0, %0, %1" : "+v"(two) : "v"(w)); };
#pragma unroll
        for (int u = 0; u < N; ++u) {
            take(x[u].w[0].x);
            take(x[u].w[0].y);
            take(x[u].w[0].z);
            take(x[u].w[0].w);
        }
        v = fmaxf(fmaxf(v, ElemF16::get((uint16_t)two)), ElemF16::get((uint16_t)(two >> 16)));
    } else {
#pragma unroll
        for (int u = 0; u < N; ++u)
#pragma unroll
            for (int e = 0; e < 8; ++e) v = fmaxf(v, x[u].get(e));
    }
    return v;
}

// A row, or a part of it, seen as vectors of eight from `shift` places before its first score
template <class E>
struct ScoreRow {
    const typename E::raw *from;  // place 0 of the vectors: aligned
    int shift, end;               // places of the row: shift .. end - 1
    __device__ __forceinline__ ScoreRow(const ScoreParams &p, int64_t row)
    {
        const int64_t first = row * p.ld;
        shift = (int)(first & 7);
        from = static_cast<const typename E::raw *>(p.logits) + (first - shift);
        end = p.V + shift;
    }
    __device__ __forceinline__ bool whole(int v) const { return v * 8 >= shift && v * 8 + 8 <= end; }
    // places outside the row, and all if not `real`: -infinity
    __device__ __forceinline__ void get(int v, bool real, Eight<E> &x) const
    {
        if (real && whole(v)) return x.fetch(from + (int64_t)v * 8);
        constexpr uint32_t NONE = E::BYTES == 4 ? 0xFF800000u : std::is_same<E, ElemF16>::value ? 0xFC00u : 0xFF80u;
        uint32_t u[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            u[e] = NONE;
            if (real && v * 8 + e >= shift && v * 8 + e < end) {
                if constexpr (E::BYTES == 4) u[e] = __float_as_uint(from[v * 8 + e]);
                else u[e] = from[v * 8 + e];
            }
        }
        if constexpr (E::BYTES == 4) {
            x.w[0] = make_uint4(u[0], u[1], u[2], u[3]);
            x.w[1] = make_uint4(u[4], u[5], u[6], u[7]);
        } else {
            x.w[0] = make_uint4(u[0] | u[1] << 16, u[2] | u[3] << 16, u[4] | u[5] << 16, u[6] | u[7] << 16);
        }
    }
};

// N vectors of each lane, whose largest score is returned
template <class E, int N>
__device__ __forceinline__ float add_vectors(const ScoreParams &p, const Eight<E> (&x)[N], Mass &m)
{
    const float largest = largest_of(x);
    m.most = fmaxf(m.most, largest);
    const float up = m.most * p.c;
    if (up > m.ref + RISE) {
        const float ref = __builtin_ceilf(up);
        rebase(m, fall(m.ref, ref));
        m.ref = ref;
    }
#pragma unroll
    for (int u = 0; u < N; ++u)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float d = __builtin_fmaf(x[u].get(e), p.c, -m.ref), power = __builtin_amdgcn_exp2f(d);
            m.sum += power;
            m.weighted = __builtin_fmaf(power, fmaxf(d, NO_MASS), m.weighted);
        }
    return largest;
}

// The masses of all lanes of a wave, or of several waves, one after the other, in every lane
__device__ __forceinline__ Mass joined(Mass m)
{
    const float ref = wave_max(m.ref);
    rebase(m, fall(m.ref, ref));
    m.ref = ref;
    m.most = wave_max(m.most);
    m.sum = wave_sum(m.sum);
    m.weighted = wave_sum(m.weighted);
    return m;
}

// What a row's results are computed from: c x - ref, or (x - most) c in a far row
struct RowResult {
    float most, ref, c, scale, log_sum;  // log_sum: base 2, relative to ref
    bool far;
    __device__ __forceinline__ RowResult(const Mass &m, const ScoreParams &p, bool far)
        : most(m.most), ref(m.ref), c(p.c), scale(p.scale), log_sum(__log2f(m.sum)), far(far) {}
    __device__ __forceinline__ float log_prob(float x) const
    {
        if (x == -__builtin_inff() && log_sum == log_sum) return x;
        const float d = far ? (x - most) * c : __builtin_fmaf(x, c, -ref);
        float v = (d - log_sum) * LN2;
        if (fabsf(v) == __builtin_inff()) v = (x - most) * scale;  // the type's lowest value: to the base e it may be within binary32
        return v > 0.0f ? 0.0f : v;
    }
};

// The given token's score, asked for long before it is used
struct Given {
    bool inside;
    float score;
    template <class E>
    __device__ __forceinline__ void fetch(const ScoreParams &p, int64_t row, E)
    {
        const int64_t t = given_token(p.tokens, p.token_bits, row);
        inside = t >= 0 && t < p.V;
        score = E::get(static_cast<const typename E::raw *>(p.logits)[row * p.ld + (inside ? t : 0)]);
    }
};

__device__ __forceinline__ void write_row(const ScoreParams &p, int64_t row, const Given &given, const Mass &m, bool far, Key best)
{
    const RowResult r(m, p, far);
    const int lane = threadIdx.x & 63;
    if (lane < p.top) {
        p.top_tokens[row * p.top + lane] = (int32_t)place_of(best);
        p.top_log_probs[row * p.top + lane] = r.log_prob(from_ordered((uint32_t)(best >> 32)));
    }
    if (lane != 0) return;
    const bool empty = m.most == -__builtin_inff() && m.sum == 0.0f;
    p.log_probs[row] = given.inside ? r.log_prob(given.score) : 0.0f;
    const float entropy = (r.log_sum - m.weighted / m.sum) * LN2;
    p.entropies[row] = empty || entropy < 0.0f ? 0.0f : entropy;
    const float above = far ? 0.0f : __builtin_fmaf(m.most, p.c, -m.ref);
    *reinterpret_cast<float2 *>(p.normalizers + 2 * row) = make_float2(m.most, empty ? -__builtin_inff() : (r.log_sum - above) * LN2);
}

// A workgroup has a part of a row; rows of one part are done here, others are joined by the next kernel
template <class E, bool TOP, int THREADS>
__global__ __launch_bounds__(THREADS) void token_mass_kernel(const ScoreParams p)
{
    constexpr int WAVES = THREADS / 64;
    __shared__ Mass masses[WAVES];
    __shared__ Key room[TOP ? 128 : 1];
    __shared__ int chosen[TOP ? TOP_MOST : 1];
    extern __shared__ float largest[];
    const int64_t row = blockIdx.x / (unsigned)p.parts;
    const int part = (int)(blockIdx.x - (unsigned)row * (unsigned)p.parts);
    const ScoreRow<E> r(p, row);
    Given given;
    if (p.parts == 1 && threadIdx.x < 64) given.fetch(p, row, E());
    const int all_steps = (r.end + STEP * 8 - 1) / (STEP * 8);
    const int step0 = part * p.steps_per_part < all_steps ? part * p.steps_per_part : all_steps;
    const int steps = all_steps - step0 < p.steps_per_part ? all_steps - step0 : p.steps_per_part;
    const int v0 = step0 * STEP, v1 = v0 + steps * STEP;

    // A wave has STEP neighbouring vectors at a time.  Only where the row begins or ends among them they are looked at one by one.
    // (Rows a power of two apart that all began at the same place would ask the same memory channels: each begins at another.)
    Mass m = {-__builtin_inff(), -FAR, 0.0f, 0.0f};
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int mine = (steps - wave + WAVES - 1) / WAVES;
    int turn = mine > 0 ? (int)(blockIdx.x % (unsigned)mine) : 0;
    for (int i = 0; i < mine; ++i, turn = turn + 1 < mine ? turn + 1 : 0) {
        const int step = turn * WAVES + wave, v = v0 + step * STEP;
        float most;
        if (v * 8 >= r.shift && (v + STEP) * 8 <= r.end) {
            Eight<E> x[SCORE_UNROLL];
#pragma unroll
            for (int u = 0; u < SCORE_UNROLL; ++u) x[u].fetch(r.from + (int64_t)(v + u * 64 + lane) * 8);
            most = add_vectors(p, x, m);
        } else {
            most = -__builtin_inff();
#pragma unroll 1
            for (int w = v; w < v + STEP && w * 8 < r.end; w += 64) {
                Eight<E> x[1];
                r.get(w + lane, true, x[0]);
                most = fmaxf(most, add_vectors(p, x, m));
            }
        }
        if constexpr (TOP) largest[step * 64 + lane] = most;
    }
    // Beside a signalling NaN the unit's maximum is not the other value, but NaN, and the next maximum starts anew: a wave that has met any NaN looks
    // for its largest scores again by comparing them.  (In the loop above, this took half of the waves' registers: 8192 rows of 30522 in 150 instead of 122 us.)
    if (__builtin_expect(__ballot(m.sum != m.sum) != 0, 0)) {
#pragma unroll 1
        for (int step = wave; step < steps; step += WAVES) {
            const int v = v0 + step * STEP;
            float most = -__builtin_inff();
#pragma unroll 1
            for (int w = v; w < v + STEP && w * 8 < r.end; w += 64) {
                Eight<E> x;
                r.get(w + lane, true, x);
#pragma unroll
                for (int e = 0; e < 8; ++e) most = x.get(e) > most ? x.get(e) : most;
            }
            if constexpr (TOP) largest[step * 64 + lane] = most;
            m.most = fmaxf(m.most, most);
        }
    }
    m = joined(m);
    if ((threadIdx.x & 63) == 0) masses[threadIdx.x >> 6] = m;
    __syncthreads();
    float most = masses[0].most, ref = masses[0].ref;
#pragma unroll
    for (int w = 1; w < WAVES; ++w) {
        most = fmaxf(most, masses[w].most);
        ref = fmaxf(ref, masses[w].ref);
    }
    m = {most, ref, 0.0f, 0.0f};
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
        Mass o = masses[w];
        rebase(o, fall(o.ref, ref));
        m.sum += o.sum;
        m.weighted += o.weighted;
    }
    const bool far = is_far(most, p.c);
    if (far) {  // relative to the largest; without any, only a NaN counts
        Mass f = {most, 0.0f, 0.0f, 0.0f};
        for (int v = v0 + (int)threadIdx.x; v < v1; v += THREADS) {
            Eight<E> x;
            r.get(v, true, x);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const bool none = x.get(e) == -__builtin_inff();
                const float d = none ? NO_MASS : (x.get(e) - most) * p.c, power = __builtin_amdgcn_exp2f(d);
                f.sum += power;
                f.weighted = __builtin_fmaf(power, fmaxf(d, NO_MASS), f.weighted);
            }
        }
        f.sum = wave_sum(f.sum);
        f.weighted = wave_sum(f.weighted);
        __syncthreads();
        if ((threadIdx.x & 63) == 0) masses[threadIdx.x >> 6] = f;
        __syncthreads();
        m = {most, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            m.sum += masses[w].sum;
            m.weighted += masses[w].weighted;
        }
    }
    if (threadIdx.x >= 64) return;
    Key best = 0;
    if constexpr (TOP) {
        // A lane's scores of a step are a piece.  The top-th largest of the pieces' largest scores is a bound that only `top` pieces reach, or
        // more where scores are equal: the choice is among the scores of these that reach it.  Half a wave looks at a piece.
        const int pieces = steps * 64;
        const Key last = pieces < p.top ? 0 : lane_key(choose(pieces, p.top, room, [&](int i) { return key_of(largest[i], (uint32_t)i); }), p.top - 1);
        const uint32_t bound = (uint32_t)(last >> 32);
        Choice choice(room, p.top, (Key)bound << 32);
        auto look = [&](int n) {
            for (int i = 0; i < n; i += 16) {
                Key k[8];
#pragma unroll
                for (int u = 0; u < 8; ++u) {
                    const int which = i + 2 * u + lane / 32, piece = chosen[which < n ? which : 0];
                    const int place = (v0 + (piece >> 6) * STEP + (lane >> 3 & 3) * 64 + (piece & 63)) * 8 + (lane & 7);
                    const bool real = which < n && place >= r.shift && place < r.end;
                    k[u] = real ? key_of(E::get(r.from[place]), (uint32_t)(place - r.shift)) : 0;
                }
#pragma unroll
                for (int u = 0; u < 8; ++u)
                    if (i + 2 * u < n) choice.add(k[u]);
            }
        };
        int found = 0;
        for (int i = 0; i < pieces; i += 64) {
            const bool reaches = ordered(largest[i + lane]) >= bound;
            const uint64_t mask = __ballot(reaches);
            if (!mask) continue;
            const int n = __popcll(mask);
            if (found + n > TOP_MOST) {
                look(found);
                found = 0;
                wave_order();
            }
            const int before = __builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0u));
            if (reaches) chosen[found + before] = i + lane;
            found += n;
            wave_order();
        }
        look(found);
        best = choice.finish();
    }
    if (p.parts == 1) return write_row(p, row, given, m, far, best);
    const int64_t at = row * p.parts + part;
    if (lane == 0) p.partials[at] = make_float4(m.most, m.ref, m.sum, m.weighted);
    if (TOP && lane < p.top) p.keys[at * p.top + lane] = best;
}

// A wave joins the parts of a row
template <class E>
__global__ __launch_bounds__(64) void token_join_kernel(const ScoreParams p)
{
    __shared__ Key room[128];
    const int64_t row = blockIdx.x;
    const int lane = threadIdx.x;
    const float4 *parts = p.partials + row * p.parts;
    Given given;
    given.fetch(p, row, E());
    float most = -__builtin_inff(), ref = -FAR;
    for (int i = lane; i < p.parts; i += 64) {
        most = fmaxf(most, parts[i].x);
        if (!is_far(parts[i].x, p.c)) ref = fmaxf(ref, parts[i].y);
    }
    most = wave_max(most);
    ref = wave_max(ref);
    const bool far = is_far(most, p.c);
    Mass m = {most, ref, 0.0f, 0.0f};
    for (int i = lane; i < p.parts; i += 64) {
        Mass o = {parts[i].x, parts[i].y, parts[i].z, parts[i].w};
        const bool far_part = is_far(o.most, p.c);
        // a far part is relative to its largest score, another to its reference; and so is the row
        float by = far ? __builtin_fmaf(-most, p.c, o.ref) : o.ref - ref;
        if (far_part) by = !far ? __builtin_fmaf(o.most, p.c, -ref) : o.most == most ? 0.0f : (o.most - most) * p.c;
        rebase(o, fmaxf(by, NO_MASS));
        m.sum += o.sum;
        m.weighted += o.weighted;
    }
    m.sum = wave_sum(m.sum);
    m.weighted = wave_sum(m.weighted);
    Key best = 0;
    if (p.top > 0) {
        const Key *keys = p.keys + row * p.parts * p.top;
        best = choose(p.parts * p.top, p.top, room, [&](int i) { return keys[i]; });
    }
    write_row(p, row, given, m, far, best);
}

// ---- gradient -------------------------------------------------------------------------------------------------------------
struct ScoreGradParams {
    ScoreParams s;
    const float *d_log_probs, *d_entropies;
    void *grad;
    int64_t ld_grad;
    int chunks;  // workgroups of a row
};
constexpr int GRAD_CHUNK = 256 * 8 * SCORE_UNROLL;

// VEC: rows of scores and of the gradient begin at the same place modulo eight
template <class E, class O, bool ENTROPY, bool VEC>
__global__ __launch_bounds__(256) void token_gradient_kernel(const ScoreGradParams g)
{
    const ScoreParams &p = g.s;
    const int64_t row = blockIdx.x / (unsigned)g.chunks;
    const int chunk = (int)(blockIdx.x - (unsigned)row * (unsigned)g.chunks);
    const ScoreRow<E> r(p, row);
    typename O::raw *out = static_cast<typename O::raw *>(g.grad) + (row * g.ld_grad - r.shift);
    const float2 norm = *reinterpret_cast<const float2 *>(p.normalizers + 2 * row);
    const float most = norm.x, log_sum = norm.y * LOG2E;
    const int64_t t = given_token(p.tokens, p.token_bits, row);
    const bool given = t >= 0 && t < p.V;
    const float d = given ? g.d_log_probs[row] : 0.0f;
    float a = p.scale * d, b = 0.0f, h = 0.0f;
    if constexpr (ENTROPY) {
        h = g.d_entropies[row];
        a = p.scale * __builtin_fmaf(h, p.entropies[row], d);
        b = p.scale * h * LN2;
    }
    const bool zeros = norm.y == -__builtin_inff() || (d == 0.0f && h == 0.0f);  // a row without a score, or one that counts for nothing
    const float more = p.scale * d;
    const int token_place = given ? (int)t + r.shift : -1;
    auto value = [&](float x, int place) {
        const float e = __builtin_fmaf(x - most, p.c, -log_sum), power = __builtin_amdgcn_exp2f(e);
        float v = a;
        if constexpr (ENTROPY) v = __builtin_fmaf(b, fmaxf(e, NO_MASS), a);
        v = in_binary32(__builtin_fmaf(-power, v, place == token_place ? more : 0.0f));
        return zeros ? 0.0f : v;
    };
    const int v0 = chunk * (GRAD_CHUNK / 8) + (int)threadIdx.x;
    if constexpr (VEC) {
        Eight<E> x[SCORE_UNROLL];
#pragma unroll
        for (int u = 0; u < SCORE_UNROLL; ++u)
            if (v0 + u * 256 < (r.end + 7) / 8) r.get(v0 + u * 256, true, x[u]);
#pragma unroll
        for (int u = 0; u < SCORE_UNROLL; ++u) {
            const int v = v0 + u * 256;
            if (v >= (r.end + 7) / 8) break;
            float y[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) y[e] = value(x[u].get(e), v * 8 + e);
            if (r.whole(v)) {
                put8<O>(out + (int64_t)v * 8, y);
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (v * 8 + e >= r.shift && v * 8 + e < r.end) out[v * 8 + e] = O::put(y[e]);
            }
        }
    } else {
        const int from = chunk * GRAD_CHUNK;
        for (int i = from + (int)threadIdx.x; i < from + GRAD_CHUNK && i < r.end; i += 256)
            if (i >= r.shift) out[i] = O::put(value(E::get(r.from[i]), i));
    }
}

// ---- host side ------------------------------------------------------------------------------------------------------------
constexpr int64_t SCORES_MOST = (int64_t)1 << 30;  // columns, rows: places are counted in 32 bits, past a row's end too

// Parts of a row: so many that what is kept of each fits LDS, and more where there are few rows for 256 CUs
static int row_parts(int64_t M, int64_t V, int top)
{
    const int64_t steps = ceil_div(V + 7, STEP * 8);
    int64_t parts = top > 0 ? ceil_div(steps, STEPS_MOST) : 1;
    const int64_t wanted = ceil_div(512, M);        // workgroups for the chip
    const int64_t useful = ceil_div(steps, 32);     // two steps for each wave of a large workgroup
    const int64_t more = wanted < useful ? wanted : useful;
    if (more > parts) parts = more;
    return (int)(parts < PARTS_MOST ? parts : PARTS_MOST);
}

static bool score_scale_ok(float s) { return s >= 0x1p-100f && s <= 0x1p100f; }

template <class E, bool TOP, int THREADS>
static void launch_mass(const ScoreParams &p, hipStream_t st)
{
    const int lds = TOP ? p.steps_per_part * 64 * (int)sizeof(float) : 0;
    token_mass_kernel<E, TOP, THREADS><<<(unsigned)(p.M * p.parts), THREADS, lds, st>>>(p);
}

}  // namespace mkq

using namespace mkq;

extern "C" size_t mkq_token_log_probs_workspace_bytes(int64_t M, int64_t V, int top)
{
    if (M <= 0 || V <= 0 || top < 0 || top > TOP_MOST || M > SCORES_MOST || V > SCORES_MOST) return 0;
    const int parts = row_parts(M, V, top);
    return parts == 1 ? 0 : (size_t)M * parts * (sizeof(float4) + (size_t)top * sizeof(Key));
}

extern "C" int mkq_token_log_probs(const void *logits, int dtype, int64_t ld, int64_t M, int64_t V, float scale, const void *tokens,
                                   int token_bits, float *normalizers, float *log_probs, float *entropies, int top, int32_t *top_tokens,
                                   float *top_log_probs, void *workspace, size_t workspace_bytes, void *stream)
{
    if (!is_float_dtype(dtype) || (token_bits != 32 && token_bits != 64)) return MKQ_ERR_DTYPE;
    if (M < 0 || V <= 0 || ld < V || top < 0 || top > V) return MKQ_ERR_SHAPE;
    if (!score_scale_ok(scale)) return MKQ_ERR_SCALE;
    if (top > TOP_MOST) return MKQ_ERR_UNSUPPORTED;
    if (M == 0) return MKQ_OK;
    if (!logits || !tokens || !normalizers || !log_probs || !entropies || (top > 0 && (!top_tokens || !top_log_probs))) return MKQ_ERR_NULL;
    if (!aligned16(logits) || reinterpret_cast<uintptr_t>(tokens) % (token_bits / 8) || reinterpret_cast<uintptr_t>(normalizers) % 8 ||
        !aligned4(log_probs) || !aligned4(entropies) || (top > 0 && (!aligned4(top_tokens) || !aligned4(top_log_probs))))
        return MKQ_ERR_ALIGN;
    if (M > SCORES_MOST || V > SCORES_MOST) return MKQ_ERR_UNSUPPORTED;
    ScoreParams p = {};
    p.logits = logits;
    p.tokens = tokens;
    p.ld = ld;
    p.M = M;
    p.V = (int)V;
    p.token_bits = token_bits;
    p.top = top;
    p.parts = row_parts(M, V, top);
    p.steps_per_part = (int)ceil_div(ceil_div(V + 7, STEP * 8), p.parts);
    p.scale = scale;
    p.c = scale * LOG2E;
    p.normalizers = normalizers;
    p.log_probs = log_probs;
    p.entropies = entropies;
    p.top_tokens = top_tokens;
    p.top_log_probs = top_log_probs;
    const bool large = M * p.parts < 512;
    if (!grid_ok(M * p.parts, large ? 1024 : 256)) return MKQ_ERR_UNSUPPORTED;
    if (p.parts > 1) {
        if (!workspace || workspace_bytes < mkq_token_log_probs_workspace_bytes(M, V, top)) return MKQ_ERR_WORKSPACE;
        if (!aligned16(workspace)) return MKQ_ERR_ALIGN;
        p.partials = static_cast<float4 *>(workspace);
        p.keys = reinterpret_cast<Key *>(p.partials + M * p.parts);
    }
    const hipStream_t st = as_stream(stream);
    with_elem(dtype, [&](auto e) {
        using E = decltype(e);
        if (top > 0) {
            if (large) launch_mass<E, true, 1024>(p, st);
            else launch_mass<E, true, 256>(p, st);
        } else {
            if (large) launch_mass<E, false, 1024>(p, st);
            else launch_mass<E, false, 256>(p, st);
        }
        if (p.parts > 1) token_join_kernel<E><<<(unsigned)M, 64, 0, st>>>(p);
    });
    return launch_status();
}

extern "C" int mkq_token_log_probs_gradient(const void *logits, int dtype, int64_t ld, int64_t M, int64_t V, float scale, const void *tokens,
                                            int token_bits, const float *normalizers, const float *entropies, const float *d_log_probs,
                                            const float *d_entropies, void *grad, int grad_dtype, int64_t ld_grad, void *stream)
{
    if (!is_float_dtype(dtype) || !is_float_dtype(grad_dtype) || (token_bits != 32 && token_bits != 64)) return MKQ_ERR_DTYPE;
    if (M < 0 || V <= 0 || ld < V || ld_grad < V) return MKQ_ERR_SHAPE;
    if (!score_scale_ok(scale)) return MKQ_ERR_SCALE;
    if (M == 0) return MKQ_OK;
    if (!logits || !tokens || !normalizers || !d_log_probs || !grad || (d_entropies && !entropies)) return MKQ_ERR_NULL;
    if (!aligned16(logits) || !aligned16(grad) || reinterpret_cast<uintptr_t>(tokens) % (token_bits / 8) ||
        reinterpret_cast<uintptr_t>(normalizers) % 8 || !aligned4(d_log_probs) || !aligned4(d_entropies) || !aligned4(entropies))
        return MKQ_ERR_ALIGN;
    if (M > SCORES_MOST || V > SCORES_MOST) return MKQ_ERR_UNSUPPORTED;
    if (!in_place_or_apart(logits, dtype, ld, grad, grad_dtype, ld_grad, M, V)) return MKQ_ERR_UNSUPPORTED;
    ScoreGradParams g = {};
    g.s.logits = logits;
    g.s.tokens = tokens;
    g.s.ld = ld;
    g.s.M = M;
    g.s.V = (int)V;
    g.s.token_bits = token_bits;
    g.s.scale = scale;
    g.s.c = scale * LOG2E;
    g.s.normalizers = const_cast<float *>(normalizers);
    g.s.entropies = const_cast<float *>(entropies);
    g.d_log_probs = d_log_probs;
    g.d_entropies = d_entropies;
    g.grad = grad;
    g.ld_grad = ld_grad;
    g.chunks = (int)ceil_div(V + 7, GRAD_CHUNK);
    if (!grid_ok(M * g.chunks, 256)) return MKQ_ERR_UNSUPPORTED;
    const bool vec = M <= 1 || (ld - ld_grad) % 8 == 0;
    const unsigned workgroups = (unsigned)(M * g.chunks);
    const hipStream_t st = as_stream(stream);
    auto with_bool = [](bool b, auto &&f) {
        if (b) f(std::true_type());
        else f(std::false_type());
    };
    with_elem(dtype, [&](auto e) {
        with_elem(grad_dtype, [&](auto o) {
            with_bool(d_entropies != nullptr, [&](auto h) {
                with_bool(vec, [&](auto v) {
                    token_gradient_kernel<decltype(e), decltype(o), decltype(h)::value, decltype(v)::value><<<workgroups, 256, 0, st>>>(g);
                });
            });
        });
    });
    return launch_status();
}
