// Linears of few tokens with 4-bit weights that have a step for every group of 32, 64 or 128 neighbours of a row, and
// float activations.
//
//     y[m,n] = sum_g s[n,g] ( sum_{k in g} x[m,k] c[n,k] ) + bias[n]
//
// Codes are whole numbers in [-8, 7], exact in binary16 and in bfloat16, so the matrix instruction multiplies the codes
// themselves and a group's sum is scaled once, in binary32, behind its last product: no rounding of c * s to 16 bits.
// Activations enter exactly too: binary16 and bfloat16 ones as they are, binary32 ones as the sum of three bfloat16 parts
// (8 + 8 + 8 bits).
//
// Bound: the weights' bytes for few tokens (each is read once), the matrix pipe from about 100 tokens on.
#include <type_traits>

#include "elements.h"

namespace mkq {

typedef float v4f __attribute__((ext_vector_type(4)));
typedef _Float16 v8h __attribute__((ext_vector_type(8)));
typedef __bf16 v8b __attribute__((ext_vector_type(8)));

// ---- preparation of the weights ---------------------------------------------------------------------------------------
// One lane per eight codes (a word), G / 8 neighbouring lanes per group: the group's abs-max by lane exchanges, then Eq. 1
// for the lane's eight values.  Bound by the read of W.  grid.x: 256 words of a row at a time.
template <class E, int G>
__global__ __launch_bounds__(256) void pack_group_kernel(const typename E::raw *__restrict__ W, int64_t K, int64_t ldw, int vec,
                                                         const float *__restrict__ s_in, float *__restrict__ s_out,
                                                         uint32_t *__restrict__ q, int words, int groups, int blocks_per_row)
{
    const int64_t n = blockIdx.x / blocks_per_row;
    const int word = (int)(blockIdx.x % blocks_per_row) * 256 + threadIdx.x;
    const int64_t k = (int64_t)word * 8;
    const typename E::raw *row = W + n * ldw;
    float v[8];
    if (vec && k + 8 <= K) {
        get8<E>(row + k, v);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = k + i < K ? E::get(row[k + i]) : 0.0f;
    }
    float mx = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) mx = fmaxf(mx, fabsf(v[i]));  // (passes over NaN, whose code is 0)
    if constexpr (G >= 128) mx = fmaxf(mx, __shfl_xor(mx, 8, 64));
    if constexpr (G >= 64) mx = fmaxf(mx, __shfl_xor(mx, 4, 64));
    mx = fmaxf(mx, __shfl_xor(mx, 2, 64));
    mx = fmaxf(mx, __shfl_xor(mx, 1, 64));
    const int g = word / (G / 8);
    if (g >= groups) return;
    float s = mx > 0.0f ? mx / (float)QMAX : 1.0f;
    if (s_in) s = s_in[n * groups + g];
    if (word % (G / 8) == 0) s_out[n * groups + g] = s;
    if (word >= words) return;
    uint32_t packed = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) packed |= ((uint32_t)(k + i < K ? quantize_code(v[i], s) : 0) & 0xFu) << (4 * i);
    q[n * words + word] = packed;
}

// ---- the linear ---------------------------------------------------------------------------------------------------------
struct Group4Params {
    const void *x;
    int64_t ldx;
    const uint8_t *W;  // rows of pieces * 16 bytes
    const float *s_w;  // [N, groups]
    const float *bias;
    const void *residual;
    void *out;
    int residual_dtype, out_dtype, act;
    int M, N, K, pieces, groups;  // pieces: of 32 codes
    int tiles;                    // workgroups along N
    int ks;                       // waves of a workgroup that share a tile's k loop
};

// Eight codes of a word as the matrix instruction takes them.
// binary16: u + 1024 = 0x6400 | u with u = c ^ 8 in [0, 15] (two's complement with its sign bit flipped), and 1024 + 16 u for
// the nibble above it, so one shift and four three-operand logic operations place all eight, and one packed operation per
// pair takes the bias off exactly.  Order of the values: 0 4 1 5 2 6 3 7; the activations are put in the same order.
// bfloat16: the conversion gives c / 16 in binary32, whose upper half holds all of it; the 16 comes back on the step.
__device__ __forceinline__ v8h codes_f16(uint32_t w)
{
    typedef _Float16 h2 __attribute__((ext_vector_type(2)));
    const h2 off = {(_Float16)-1032.0f, (_Float16)-1032.0f};
    const h2 low = {(_Float16)0.0625f, (_Float16)0.0625f}, offl = {(_Float16)-72.0f, (_Float16)-72.0f};
    const uint32_t w8 = w >> 8;
    const uint32_t a = (w & 0x000F000Fu) ^ 0x64086408u, b = (w & 0x00F000F0u) ^ 0x64806480u;
    const uint32_t c = (w8 & 0x000F000Fu) ^ 0x64086408u, d = (w8 & 0x00F000F0u) ^ 0x64806480u;
    const h2 r[4] = {__builtin_bit_cast(h2, a) + off, __builtin_elementwise_fma(__builtin_bit_cast(h2, b), low, offl),
                     __builtin_bit_cast(h2, c) + off, __builtin_elementwise_fma(__builtin_bit_cast(h2, d), low, offl)};
    return __builtin_bit_cast(v8h, r);
}

__device__ __forceinline__ v8b codes_bf16(uint32_t w)
{
    uint32_t r[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float a = __builtin_amdgcn_cvt_off_f32_i4((int)(w >> (8 * i)));
        const float b = __builtin_amdgcn_cvt_off_f32_i4((int)(w >> (8 * i + 4)));
        r[i] = __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302u);
    }
    return __builtin_bit_cast(v8b, r);
}

// Eight neighbouring activations as matrix operands
template <class E>
struct XParts;
template <>
struct XParts<ElemF16> {
    static constexpr int PARTS = 1;
    v8h p[1];
    __device__ __forceinline__ void set(uint4 a, uint4)
    {
        const uint32_t r[4] = {__builtin_amdgcn_perm(a.z, a.x, 0x05040100u), __builtin_amdgcn_perm(a.z, a.x, 0x07060302u),
                               __builtin_amdgcn_perm(a.w, a.y, 0x05040100u), __builtin_amdgcn_perm(a.w, a.y, 0x07060302u)};
        p[0] = __builtin_bit_cast(v8h, r);
    }
    using Codes = v8h;
    __device__ static __forceinline__ Codes codes(uint32_t w) { return codes_f16(w); }
    __device__ __forceinline__ v4f mul_codes(Codes b, v4f c) const { return __builtin_amdgcn_mfma_f32_16x16x32_f16(p[0], b, c, 0, 0, 0); }
    static constexpr float UNIT = 1.0f;
};
template <>
struct XParts<ElemBF16> {
    static constexpr int PARTS = 1;
    v8b p[1];
    __device__ __forceinline__ void set(uint4 a, uint4) { p[0] = __builtin_bit_cast(v8b, a); }
    using Codes = v8b;
    __device__ static __forceinline__ Codes codes(uint32_t w) { return codes_bf16(w); }
    __device__ __forceinline__ v4f mul_codes(Codes b, v4f c) const { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(p[0], b, c, 0, 0, 0); }
    static constexpr float UNIT = 16.0f;
};
// x = hi + mid + lo: each part is the upper half of what is left (its first 8 bits), and what is left is exact, down to the
// smallest normal number; nothing is left of an infinity, and a NaN stays one.
template <>
struct XParts<ElemF32> {
    static constexpr int PARTS = 3;
    v8b p[3];
    __device__ __forceinline__ void set(uint4 a, uint4 b)
    {
        uint32_t u[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w}, mid[8], lo[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float x = __uint_as_float(u[i]);
            const bool finite = fabsf(x) < __builtin_inff();
            const float r = finite ? x - __uint_as_float(u[i] & 0xFFFF0000u) : 0.0f;
            if (x != x) u[i] = 0x7FC00000u;
            mid[i] = __float_as_uint(r);
            lo[i] = __float_as_uint(r - __uint_as_float(mid[i] & 0xFFFF0000u));
        }
        uint32_t h[4], m[4], l[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            h[i] = __builtin_amdgcn_perm(u[2 * i + 1], u[2 * i], 0x07060302u);
            m[i] = __builtin_amdgcn_perm(mid[2 * i + 1], mid[2 * i], 0x07060302u);
            l[i] = __builtin_amdgcn_perm(lo[2 * i + 1], lo[2 * i], 0x07060302u);
        }
        p[0] = __builtin_bit_cast(v8b, l);
        p[1] = __builtin_bit_cast(v8b, m);
        p[2] = __builtin_bit_cast(v8b, h);
    }
    using Codes = v8b;
    __device__ static __forceinline__ Codes codes(uint32_t w) { return codes_bf16(w); }
    __device__ __forceinline__ v4f mul_codes(Codes b, v4f c) const
    {
#pragma unroll
        for (int i = 0; i < 3; ++i) c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(p[i], b, c, 0, 0, 0);
        return c;
    }
    static constexpr float UNIT = 16.0f;
};

// Words of four lane quarters, transposed: word r of quarter q becomes word q of quarter r
__device__ __forceinline__ void transpose4(uint32_t (&w)[4])
{
    auto s32 = [](uint32_t &a, uint32_t &b) {
        const auto r = __builtin_amdgcn_permlane32_swap(a, b, false, false);
        a = r[0];
        b = r[1];
    };
    auto s16 = [](uint32_t &a, uint32_t &b) {
        const auto r = __builtin_amdgcn_permlane16_swap(a, b, false, false);
        a = r[0];
        b = r[1];
    };
    s32(w[0], w[2]);
    s32(w[1], w[3]);
    s16(w[0], w[1]);
    s16(w[2], w[3]);
}

__device__ __forceinline__ float load_dtype(const void *p, int dtype, int64_t i)
{
    if (dtype == MKQ_F32) return static_cast<const float *>(p)[i];
    const uint16_t h = static_cast<const uint16_t *>(p)[i];
    return dtype == MKQ_F16 ? ElemF16::get(h) : ElemBF16::get(h);
}

// A wave owns 16 channels and up to 16 * MT tokens; with ks > 1 the ks waves of a workgroup share the tile and take the
// steps of 128 codes in turn.  In a step a lane fetches 16 bytes (32 codes) of channel lane % 16; the words of the four lanes
// that share a channel are then exchanged (transpose4), so that each of the four products of a step covers 32 neighbouring
// codes and lies within one group, whatever its size.  A product's result has channel lane % 16, tokens 4 (lane / 16) + 0..3,
// so a lane needs one step per group.
template <class E, int G, int MT, bool VEC>
__global__ __launch_bounds__(256) void group4_few_kernel(const Group4Params p)
{
    using X = XParts<E>;
    __shared__ float part[4][MT * 4][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int nl = lane & 15, kq = lane >> 4;
    const int slice = wave % p.ks;
    const int tile = (int)(blockIdx.x % (unsigned)p.tiles) * (4 / p.ks) + wave / p.ks;
    const int m0 = (int)(blockIdx.x / (unsigned)p.tiles) * 16 * MT;
    const int n = tile * 16 + nl, nc = n < p.N ? n : p.N - 1;  // channels past the end are computed and not stored
    const uint8_t *wrow = p.W + (size_t)nc * ((size_t)p.pieces * 16);
    const float *srow = p.s_w + (size_t)nc * p.groups;
    const typename E::raw *xrow[MT];
    bool token[MT];
#pragma unroll
    for (int t = 0; t < MT; ++t) {
        const int m = m0 + 16 * t + nl;
        token[t] = m < p.M;
        xrow[t] = static_cast<const typename E::raw *>(p.x) + (int64_t)(token[t] ? m : 0) * p.ldx;
    }
    v4f total[MT];
#pragma unroll
    for (int t = 0; t < MT; ++t) total[t] = v4f{0.0f, 0.0f, 0.0f, 0.0f};

    const int steps = (p.pieces + 3) / 4;
    for (int step = slice; step < steps; step += p.ks) {
        const int piece = step * 4 + kq;
        const uint4 raw = *reinterpret_cast<const uint4 *>(wrow + (size_t)(piece < p.pieces ? piece : p.pieces - 1) * 16);
        uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
        transpose4(w);
        v4f sum[MT];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int g = (step * 128 + 32 * j) / G;
            if (32 * j % G == 0) {
#pragma unroll
                for (int t = 0; t < MT; ++t) sum[t] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
            }
            const int k = step * 128 + 32 * j + 8 * kq;
            const typename X::Codes codes = X::codes(w[j]);
#pragma unroll
            for (int t = 0; t < MT; ++t) {
                uint4 a = make_uint4(0, 0, 0, 0), b = a;
                if (token[t]) {  // past K the activations are zeros, whatever the weights hold there
                    if (VEC && k + 8 <= p.K) {
                        const uint4 *at = reinterpret_cast<const uint4 *>(xrow[t] + k);
                        a = at[0];
                        if (E::BYTES == 4) b = at[1];
                    } else if (k < p.K) {
                        typename E::raw v[8];
#pragma unroll
                        for (int i = 0; i < 8; ++i) v[i] = k + i < p.K ? xrow[t][k + i] : typename E::raw(0);
                        __builtin_memcpy(&a, v, 16);
                        if (E::BYTES == 4) __builtin_memcpy(&b, reinterpret_cast<const char *>(v) + 8 * E::BYTES - 16, 16);
                    }
                }
                X xp;
                xp.set(a, b);
                sum[t] = xp.mul_codes(codes, sum[t]);
            }
            if (32 * (j + 1) % G == 0) {
                // (a group past the last one has sums of zero; its step is not read)
                const float s = g < p.groups ? srow[g] * X::UNIT : 0.0f;
#pragma unroll
                for (int t = 0; t < MT; ++t)
#pragma unroll
                    for (int i = 0; i < 4; ++i) total[t][i] = __builtin_fmaf(sum[t][i], s, total[t][i]);
            }
        }
    }
    if (p.ks > 1) {
#pragma unroll
        for (int t = 0; t < MT; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) part[wave][t * 4 + i][lane] = total[t][i];
        __syncthreads();
        if (slice != 0) return;
        for (int s = 1; s < p.ks; ++s)
#pragma unroll
            for (int t = 0; t < MT; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i) total[t][i] += part[wave + s][t * 4 + i][lane];
    }
    if (n >= p.N) return;
    const float bias = p.bias ? p.bias[n] : 0.0f;
#pragma unroll
    for (int t = 0; t < MT; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int m = m0 + 16 * t + 4 * kq + i;
            if (m >= p.M) continue;
            const int64_t at = (int64_t)m * p.N + n;
            float y = total[t][i] + bias;
            if (p.residual) y += load_dtype(p.residual, p.residual_dtype, at);
            if (p.act == MKQ_ACT_GELU) y = p.out_dtype == MKQ_F16 ? gelu_erf(y) : gelu_erf_tail(y);
            if (p.out_dtype == MKQ_F32) static_cast<float *>(p.out)[at] = y;
            else static_cast<uint16_t *>(p.out)[at] = p.out_dtype == MKQ_F16 ? ElemF16::put(y) : ElemBF16::put(y);
        }
}

static bool group_ok(int group) { return group == 32 || group == 64 || group == 128; }

template <class F>
static void with_group(int group, F &&f)
{
    if (group == 32) f(std::integral_constant<int, 32>());
    else if (group == 64) f(std::integral_constant<int, 64>());
    else f(std::integral_constant<int, 128>());
}

}  // namespace mkq

using namespace mkq;

extern "C" size_t mkq_group_weight_bytes(int64_t N, int64_t K)
{
    if (N <= 0 || K <= 0 || N > 0x7FFFFFFF || K > 0x7FFFFFFF - 128) return 0;
    return (size_t)N * (size_t)(ceil_div(K, 32) * 16);
}

extern "C" int mkq_pack_weights_int4_group(const void *W, int w_dtype, int64_t N, int64_t K, int64_t ldw, int group,
                                           const float *s_w_in, float *s_w_out, uint8_t *Wq_out, void *stream)
{
    if (!is_float_dtype(w_dtype)) return MKQ_ERR_DTYPE;
    if (N < 0 || K <= 0 || ldw < K || !group_ok(group)) return MKQ_ERR_SHAPE;
    if (N == 0) return MKQ_OK;
    if (!W || !s_w_out || !Wq_out) return MKQ_ERR_NULL;
    if (!aligned16(W) || !aligned16(Wq_out) || !aligned4(s_w_out) || !aligned4(s_w_in)) return MKQ_ERR_ALIGN;
    if (N > 0x7FFFFFFF || K > 0x7FFFFFFF - 128) return MKQ_ERR_UNSUPPORTED;
    const int words = (int)(ceil_div(K, 32) * 4), groups = (int)ceil_div(K, group);
    const int64_t blocks_per_row = ceil_div(words, 256);
    if (!grid_ok(N * blocks_per_row, 256)) return MKQ_ERR_UNSUPPORTED;
    const int vec = rows_aligned16(W, ldw, w_dtype);
    const hipStream_t st = as_stream(stream);
    with_elem(w_dtype, [&](auto e) {
        using E = decltype(e);
        with_group(group, [&](auto g) {
            pack_group_kernel<E, decltype(g)::value><<<(unsigned)(N * blocks_per_row), 256, 0, st>>>(
                static_cast<const typename E::raw *>(W), K, ldw, vec, s_w_in, s_w_out, reinterpret_cast<uint32_t *>(Wq_out), words,
                groups, (int)blocks_per_row);
        });
    });
    return launch_status();
}

extern "C" int mkq_linear_int4_group(const void *x, int x_dtype, int64_t ldx, const uint8_t *Wq, const float *s_w, int group,
                                     const float *bias, int64_t M, int64_t N, int64_t K, void *out, int out_dtype,
                                     const mkq_epilogue *epi, void *stream)
{
    if (!is_float_dtype(x_dtype) || !is_float_dtype(out_dtype)) return MKQ_ERR_DTYPE;
    if (epi) {
        if (epi->act != MKQ_ACT_NONE && epi->act != MKQ_ACT_GELU) return MKQ_ERR_DTYPE;
        if (epi->residual && !is_float_dtype(epi->residual_dtype)) return MKQ_ERR_DTYPE;
        if (epi->q_out || epi->acc_out || epi->q_pitch) return MKQ_ERR_UNSUPPORTED;
    }
    if (M < 0 || N <= 0 || K <= 0 || ldx < K || !group_ok(group)) return MKQ_ERR_SHAPE;
    if (M == 0) return MKQ_OK;
    if (!x || !Wq || !s_w || !out) return MKQ_ERR_NULL;
    if (!aligned16(x) || !aligned16(Wq) || !aligned4(s_w) || !aligned16(out) || !aligned4(bias) || (epi && !aligned16(epi->residual)))
        return MKQ_ERR_ALIGN;
    if (M > 0x7FFFFFFF - 64 || N > 0x7FFFFFFF - 64 || K > 0x7FFFFFFF - 128) return MKQ_ERR_UNSUPPORTED;
    Group4Params p = {};
    p.x = x;
    p.ldx = ldx;
    p.W = Wq;
    p.s_w = s_w;
    p.bias = bias;
    p.residual = epi ? epi->residual : nullptr;
    p.residual_dtype = epi ? epi->residual_dtype : MKQ_F32;
    p.act = epi ? epi->act : MKQ_ACT_NONE;
    p.out = out;
    p.out_dtype = out_dtype;
    p.M = (int)M;
    p.N = (int)N;
    p.K = (int)K;
    p.pieces = (int)ceil_div(K, 32);
    p.groups = (int)ceil_div(K, group);
    p.ks = 4;
    p.tiles = (int)ceil_div(ceil_div(N, 16), 4 / p.ks);
    const int mt = M <= 16 ? 1 : M <= 32 ? 2 : 4;
    const int64_t workgroups = (int64_t)p.tiles * ceil_div(M, 16 * mt);
    if (!grid_ok(workgroups, 256)) return MKQ_ERR_UNSUPPORTED;
    const bool vec = rows_aligned16(x, ldx, x_dtype);
    const hipStream_t st = as_stream(stream);
    with_elem(x_dtype, [&](auto e) {
        using E = decltype(e);
        with_group(group, [&](auto g) {
            constexpr int G = decltype(g)::value;
            auto launch = [&](auto t, auto v) {
                group4_few_kernel<E, G, decltype(t)::value, decltype(v)::value><<<(unsigned)workgroups, 256, 0, st>>>(p);
            };
            auto tokens = [&](auto t) {
                if (vec) launch(t, std::true_type());
                else launch(t, std::false_type());
            };
            if (mt == 1) tokens(std::integral_constant<int, 1>());
            else if (mt == 2) tokens(std::integral_constant<int, 2>());
            else tokens(std::integral_constant<int, 4>());
        });
    });
    return launch_status();
}
