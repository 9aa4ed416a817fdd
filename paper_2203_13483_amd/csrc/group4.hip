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
// Bound: the weights' bytes for few tokens; from about ten on by waits between the loads, the barriers of the chunks and the
// instructions that turn codes into operands, none of which is busy all the time.  Of the SIMDs' cycles, vector issue and the matrix
// pipe take 58 % and 10 % for 16 bfloat16 tokens, K = 8192, N = 28672, 46 % and 25 % for 120 binary16 tokens, K = 1024, N = 30522, and
// waves wait 47 % and 43 % of theirs.  Measured in a graph, binary16, us: one token, K = 768, N = 30522, groups of 64 6.3 (2.1 TB/s; 7.0 under
// a trace, by itself); K = 8192, N = 28672, groups of 128: 1 token 27 (4.6 TB/s; the same loads with the arithmetic left out 23.5),
// 16 tokens 32 (4.0), 32 tokens 43, 64 tokens 54 (557 TFLOP/s); 120 tokens, K = 1024, N = 30522 15.3 (490 TFLOP/s).
#include <type_traits>

#include "elements.h"
#include "gemm_common.h"

namespace mkq {

typedef float v4f __attribute__((ext_vector_type(4)));
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
    int blocks_n;                 // workgroups along N
    int x_vec;                    // rows of x are multiples of 16 bytes, K of 8
    int lds_rows;                 // rows of x that a workgroup keeps: min(M, its tokens)
    bool setup_only;              // host side only: do the kernel's once-per-device setup, launch nothing
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

// c / 16 of the code in the low nibble of byte BYTE.  (The byte is picked by the instruction itself; the compiler shifts first, for
// seven of eight codes: 16 bfloat16 tokens, K = 8192, N = 28672 38 -> 36.5 us.)
template <int BYTE>
__device__ __forceinline__ float code_of_byte(uint32_t w)
{
    float r;
    if constexpr (BYTE == 0) asm("v_cvt_off_f32_i4_e32 %0, %1" : "=v"(r) : "v"(w));
    if constexpr (BYTE == 1) asm("v_cvt_off_f32_i4_sdwa %0, %1 dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:BYTE_1" : "=v"(r) : "v"(w));
    if constexpr (BYTE == 2) asm("v_cvt_off_f32_i4_sdwa %0, %1 dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:BYTE_2" : "=v"(r) : "v"(w));
    if constexpr (BYTE == 3) asm("v_cvt_off_f32_i4_sdwa %0, %1 dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:BYTE_3" : "=v"(r) : "v"(w));
    return r;
}
__device__ __forceinline__ v8b codes_bf16(uint32_t w)
{
    const uint32_t odd = w >> 4;
    auto pair = [](float a, float b) { return __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302u); };
    const uint32_t r[4] = {pair(code_of_byte<0>(w), code_of_byte<0>(odd)), pair(code_of_byte<1>(w), code_of_byte<1>(odd)),
                           pair(code_of_byte<2>(w), code_of_byte<2>(odd)), pair(code_of_byte<3>(w), code_of_byte<3>(odd))};
    return __builtin_bit_cast(v8b, r);
}

// The types of the products for one type of activations, and eight neighbouring activations as they enter them: PARTS
// vectors of eight 16-bit values whose sum they are
template <class E>
struct Product;
template <>
struct Product<ElemF16> {
    using V = v8h;
    static constexpr int PARTS = 1;
    static constexpr float UNIT = 1.0f;  // what a code of 1 stands for is 1 / UNIT
    __device__ static __forceinline__ V codes(uint32_t w) { return codes_f16(w); }
    __device__ static __forceinline__ void parts(uint4 a, uint4, uint4 (&p)[1])
    {
        p[0] = make_uint4(__builtin_amdgcn_perm(a.z, a.x, 0x05040100u), __builtin_amdgcn_perm(a.z, a.x, 0x07060302u),
                          __builtin_amdgcn_perm(a.w, a.y, 0x05040100u), __builtin_amdgcn_perm(a.w, a.y, 0x07060302u));
    }
    __device__ static __forceinline__ v4f mul(V x, V c, v4f s) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(x, c, s, 0, 0, 0); }
    __device__ static __forceinline__ v16f mul(V x, V c, v16f s) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(x, c, s, 0, 0, 0); }
};
template <>
struct Product<ElemBF16> {
    using V = v8b;
    static constexpr int PARTS = 1;
    static constexpr float UNIT = 16.0f;
    __device__ static __forceinline__ V codes(uint32_t w) { return codes_bf16(w); }
    __device__ static __forceinline__ void parts(uint4 a, uint4, uint4 (&p)[1]) { p[0] = a; }
    __device__ static __forceinline__ v4f mul(V x, V c, v4f s) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, c, s, 0, 0, 0); }
    __device__ static __forceinline__ v16f mul(V x, V c, v16f s) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(x, c, s, 0, 0, 0); }
};
// x = hi + mid + lo: each part is the upper half of what is left (its first 8 bits), and what is left is exact, down to multiples of
// 2^-133, bfloat16's smallest number (the matrix instruction takes those below its normal ones as they are); nothing is left of an
// infinity, and a NaN stays one.  The smallest part is multiplied first.
template <>
struct Product<ElemF32> : Product<ElemBF16> {
    static constexpr int PARTS = 3;
    __device__ static __forceinline__ void parts(uint4 a, uint4 b, uint4 (&p)[3])
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
        auto upper = [](const uint32_t (&v)[8]) {
            return make_uint4(__builtin_amdgcn_perm(v[1], v[0], 0x07060302u), __builtin_amdgcn_perm(v[3], v[2], 0x07060302u),
                              __builtin_amdgcn_perm(v[5], v[4], 0x07060302u), __builtin_amdgcn_perm(v[7], v[6], 0x07060302u));
        };
        p[0] = upper(lo);
        p[1] = upper(mid);
        p[2] = upper(u);
    }
};

__device__ __forceinline__ void swap32(uint32_t &a, uint32_t &b)
{
    const auto r = __builtin_amdgcn_permlane32_swap(a, b, false, false);
    a = r[0];
    b = r[1];
}
__device__ __forceinline__ void swap16(uint32_t &a, uint32_t &b)
{
    const auto r = __builtin_amdgcn_permlane16_swap(a, b, false, false);
    a = r[0];
    b = r[1];
}

// first[lane + 8 of 16] <-> second[lane]: of two registers, the upper halves of the first's rows of 16 lanes for the lower
// halves of the second's
__device__ __forceinline__ void swap8(uint32_t &a, uint32_t &b)
{
    const int t = (int)a;
    a = (uint32_t)__builtin_amdgcn_update_dpp(t, (int)b, 0x128, 0xF, 0xC, false);
    b = (uint32_t)__builtin_amdgcn_update_dpp((int)b, t, 0x128, 0xF, 0x3, false);
}

// A tile of TN channels and TN tokens: 16, products of KM = 32 codes a time, or 32, products of 16.  A wave fetches STEPS * 128
// codes of each channel at a time, 16 bytes (a piece, 32 codes) a lane and load; lane (c, q) has c = lane % TN, q = lane / TN.
// own() gives the words of the lane's own channel c: of 128 codes, piece q (32: also q + 2), of the next 128 likewise;
// operands() exchanges the words of the lanes that share a channel so that operand j of 128 codes has, in lane (c, q), the
// eight codes j * KM + 8 q ..: every product covers KM neighbours and lies within one group, whatever its size.
template <int TN>
struct Tile;
// Eight rows of 128 bytes with every load, so that a line of memory is asked for once.  Fetched as 16 rows of 64 bytes, what a
// lane needs at once, the other half of a line comes too late for the L1 where many waves stream: one token, K = 28672, N = 8192
// 54 -> 38 us.  Load i of lane (c, q) has row 8 i + c % 8, piece 4 (c / 8) + q; six exchanges for 128 codes put that right.
template <>
struct Tile<16> {
    using Acc = v4f;
    static constexpr int ACC = 4, KM = 32, STEPS = 2;
    __device__ static __forceinline__ int row(int i, int c) { return 8 * i + c % 8; }
    __device__ static __forceinline__ int piece(int, int c, int q) { return 4 * (c / 8) + q; }
    __device__ static __forceinline__ void own(uint32_t (&w)[8])
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) swap8(w[i], w[4 + i]);
    }
    __device__ static __forceinline__ void operands(uint32_t *w)
    {
        swap32(w[0], w[2]);
        swap32(w[1], w[3]);
        swap16(w[0], w[1]);
        swap16(w[2], w[3]);
    }
    __device__ static __forceinline__ int token(int i, int q) { return 4 * q + i; }
};
// 32 rows of 32 bytes with every load: many tokens are bound by the products and what is issued beside them, and the
// exchanges cost more than the lines (64 tokens, K = 8192, N = 28672 62 -> 76 us)
template <>
struct Tile<32> {
    using Acc = v16f;
    static constexpr int ACC = 16, KM = 16, STEPS = 1;
    __device__ static __forceinline__ int row(int, int c) { return c; }
    __device__ static __forceinline__ int piece(int i, int, int q) { return 2 * i + q; }
    __device__ static __forceinline__ void own(uint32_t (&)[8]) {}
    __device__ static __forceinline__ void operands(uint32_t *w)
    {
#pragma unroll
        for (int i = 0; i < 8; i += 4) {
            swap32(w[i], w[i + 1]);
            swap32(w[i + 2], w[i + 3]);
            const uint32_t t = w[i + 1];
            w[i + 1] = w[i + 2];
            w[i + 2] = t;
        }
    }
    __device__ static __forceinline__ int token(int i, int q) { return (i & 3) + 8 * (i >> 2) + 4 * q; }
};

// A lane's results: bias, residual, activation, one rounding
template <int TN, int MT>
__device__ __forceinline__ void store_tile(const Group4Params &p, typename Tile<TN>::Acc (&y)[MT], int n, int m0, int rows, int q)
{
    using T = Tile<TN>;
    if (n >= p.N) return;
    // f(result, its place) for the tokens that exist
    auto each = [&](auto &&f) {
#pragma unroll
        for (int t = 0; t < MT; ++t)
#pragma unroll
            for (int i = 0; i < T::ACC; ++i) {
                const int m = t * TN + T::token(i, q);
                if (m < rows) {
                    float v = y[t][i];
                    f(v, (int64_t)(m0 + m) * p.N + n);
                    y[t][i] = v;
                }
            }
    };
    auto add = [&](auto e) {
        const auto *r = static_cast<const typename decltype(e)::raw *>(p.residual);
        each([&](float &v, int64_t at) { v += decltype(e)::get(r[at]); });
    };
    auto write = [&](auto e) {
        auto *o = static_cast<typename decltype(e)::raw *>(p.out);
        each([&](float &v, int64_t at) { o[at] = decltype(e)::put(v); });
    };
    if (p.bias) {
        const float bias = p.bias[n];
        each([&](float &v, int64_t) { v += bias; });
    }
    if (p.residual) {
        if (p.residual_dtype == MKQ_F32) add(ElemF32());
        else if (p.residual_dtype == MKQ_F16) add(ElemF16());
        else add(ElemBF16());
    }
    if (p.act == MKQ_ACT_GELU) {
        if (p.out_dtype == MKQ_F16) each([&](float &v, int64_t) { v = gelu_erf<true>(v); });
        else each([&](float &v, int64_t) { v = gelu_erf_tail<true>(v); });
    }
    if (p.out_dtype == MKQ_F32) write(ElemF32());
    else if (p.out_dtype == MKQ_F16) write(ElemF16());
    else write(ElemBF16());
}

// Steps of 128 codes between two hand-overs of activations: four where the workgroup's x then takes 64 KiB of LDS, else two, at most
// eight vectors a thread.  Two steps take more than that in <32, 2, 8, 2>, <32, 1, 8, 4> and <16, 1, 16, 8> (135 to 141 KiB with the weights'
// steps) and in binary32's <16, 1, 8, 2> (101 to 104): one workgroup a CU there and in <16, 1, 16, 2> with groups of 32 (82), two with
// the others (51 to 75).  A call of fewer tokens than a tile's takes less.
template <class E, int G, int TN, int MT, int WAVES, int KS>
struct Shape {
    static constexpr int PARTS = Product<E>::PARTS, ROWS = TN * MT;
    static constexpr int FIT = 65536 / (512 * KS * ROWS * PARTS);
    static constexpr int U = FIT >= 4 ? 4 : 2;
    static constexpr int KC = 128 * U, PITCH = KC * 2 + 16;  // (bytes; 16 more than a multiple of 128: no bank conflicts among rows)
    static constexpr int VECTORS = (ROWS * (KC / 8) * KS + 64 * WAVES - 1) / (64 * WAVES);
    // steps of a wave's channels for a chunk, and where they are in LDS: rows of an odd number of words (no bank conflicts)
    static constexpr int SCALES = KC / G, SPITCH = SCALES | 1, SCALE_BYTES = WAVES * TN * SPITCH * 4;
    static constexpr size_t lds(int rows)
    {
        const size_t x = SCALE_BYTES + (size_t)2 * KS * PARTS * rows * PITCH, sums = KS > 1 ? (size_t)64 * WAVES * MT * Tile<TN>::ACC * 4 : 0;
        return x > sums ? x : sums;
    }
};

// KS of the WAVES waves share the k loop of a tile (chunks of KC codes in turn) and their sums meet in LDS at the end; the
// WAVES / KS tiles of the workgroup are neighbours and share the activations, which come through LDS, converted once, two
// chunks in turn: one is multiplied while the next is on its way in registers.  Weights and steps go from memory to registers,
// one chunk ahead.
template <class E, int G, int TN, int MT, int WAVES, int KS>
__global__ __launch_bounds__(64 * WAVES, TN == 16 ? (WAVES >= 8 || KS == 1 ? 4 : 3) : 2) void group4_kernel(const Group4Params p)
{
    using S = Shape<E, G, TN, MT, WAVES, KS>;
    using T = Tile<TN>;
    using P = Product<E>;
    using Acc = typename T::Acc;
    constexpr int U = S::U, KC = S::KC, ACC = T::ACC, CG = WAVES / KS, XT = 64 * WAVES / KS, THREADS = 64 * WAVES;
    extern __shared__ __attribute__((aligned(16))) uint8_t smem[];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int nl = lane % TN, q = lane / TN;
    const int slice = wave / CG, st = tid % XT;
    const int n = ((int)(blockIdx.x % (unsigned)p.blocks_n) * CG + wave % CG) * TN + nl;
    const int m0 = (int)(blockIdx.x / (unsigned)p.blocks_n) * S::ROWS;
    const int rows = p.M - m0 < S::ROWS ? p.M - m0 : S::ROWS;
    const int part_bytes = p.lds_rows * S::PITCH, buffer_bytes = S::PARTS * part_bytes;
    uint8_t *const xs = smem + S::SCALE_BYTES + slice * 2 * buffer_bytes;
    float *const scales = reinterpret_cast<float *>(smem) + wave * (TN * S::SPITCH);

    // activations of chunk c: vectors of eight, zeros past K
    uint4 xa[S::VECTORS], xb[E::BYTES == 4 ? S::VECTORS : 1];
    auto fetch_x = [&](int c) {
        const typename E::raw *const base = static_cast<const typename E::raw *>(p.x) + (int64_t)m0 * p.ldx;
        if (p.x_vec) {  // vectors are whole or past the end
#pragma unroll
            for (int v = 0; v < S::VECTORS; ++v) {
                const int i = v * XT + st, r = i / (KC / 8), k = c * KC + i % (KC / 8) * 8;
                uint4 a = make_uint4(0, 0, 0, 0), b = a;
                if (r < rows && k < p.K) {
                    const uint4 *at = reinterpret_cast<const uint4 *>(base + (int64_t)r * p.ldx + k);
                    a = at[0];
                    if constexpr (E::BYTES == 4) b = at[1];
                }
                xa[v] = a;
                if constexpr (E::BYTES == 4) xb[v] = b;
            }
        } else {
#pragma unroll
            for (int v = 0; v < S::VECTORS; ++v) {
                const int i = v * XT + st, r = i / (KC / 8), k = c * KC + i % (KC / 8) * 8;
                typename E::raw e[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) e[j] = r < rows && k + j < p.K ? base[(int64_t)r * p.ldx + k + j] : typename E::raw(0);
                __builtin_memcpy(&xa[v], e, 16);
                if constexpr (E::BYTES == 4) __builtin_memcpy(&xb[v], e + 4, 16);
            }
        }
    };
    auto store_x = [&](int buffer) {
#pragma unroll
        for (int v = 0; v < S::VECTORS; ++v) {
            const int i = v * XT + st, r = i / (KC / 8);
            if (r < rows) {
                uint4 parts[S::PARTS];
                P::parts(xa[v], E::BYTES == 4 ? xb[v] : xa[v], parts);
                uint8_t *to = xs + buffer * buffer_bytes + r * S::PITCH + i % (KC / 8) * 16;
#pragma unroll
                for (int k = 0; k < S::PARTS; ++k) *reinterpret_cast<uint4 *>(to + k * part_bytes) = parts[k];
            }
        }
    };
    // weights of STEPS steps of 128 codes from step s; past the end the last ones, whose activations are zeros
    constexpr int STEPS = T::STEPS;
    uint4 W[U / STEPS][2];
    const uint8_t *wrow[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int r = n - nl + T::row(i, nl);  // channels past the end: the last one's weights, never stored
        wrow[i] = p.W + (size_t)(r < p.N ? r : p.N - 1) * ((size_t)p.pieces * 16);
    }
    auto fetch_w = [&](int h, int s) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int piece = 4 * s + T::piece(i, nl, q);
            W[h][i] = *reinterpret_cast<const uint4 *>(wrow[i] + (size_t)(piece < p.pieces ? piece : p.pieces - 1) * 16);
        }
    };
    // steps of chunk c for the wave's channels: PER neighbours of a row a lane
    constexpr int PER = (TN * S::SCALES + 63) / 64, LPR = S::SCALES / PER;
    const int srow = lane / LPR, sg = lane % LPR * PER;
    const int sn = n - nl + srow < p.N ? n - nl + srow : p.N - 1;
    float sreg[PER];
    auto fetch_s = [&](int c) {
        const int g = c * S::SCALES + sg;
        const float *at = p.s_w + (size_t)sn * p.groups;
        if (srow < TN) {
            if (g + PER <= p.groups) {
#pragma unroll
                for (int i = 0; i < PER; ++i) sreg[i] = at[g + i];
            } else {
#pragma unroll
                for (int i = 0; i < PER; ++i) sreg[i] = at[g + i < p.groups ? g + i : p.groups - 1];
            }
        }
    };
    auto store_s = [&]() {  // (only this wave reads them)
        if (srow < TN)
#pragma unroll
            for (int i = 0; i < PER; ++i) scales[srow * S::SPITCH + sg + i] = sreg[i] * P::UNIT;
    };

    Acc total[MT];
#pragma unroll
    for (int t = 0; t < MT; ++t)
#pragma unroll
        for (int i = 0; i < ACC; ++i) total[t][i] = 0.0f;
    int xrow[MT];
#pragma unroll
    for (int t = 0; t < MT; ++t) {
        const int r = t * TN + nl;
        xrow[t] = (r < p.lds_rows ? r : p.lds_rows - 1) * S::PITCH + q * 16;
    }

    const int steps = (p.K + 127) / 128, chunks = (p.K + KC - 1) / KC, rounds = (chunks + KS - 1) / KS;
    // The i-th chunk of this workgroup: neighbours begin a chunk further on.  Rows are often a power of two of bytes apart, and
    // workgroups that walk k side by side would all ask the same few memory channels (the loads alone, rows of 4 KB, 24.2 -> 20.2 us).
    const int turn = (int)(blockIdx.x % (unsigned)chunks);
    auto chunk_at = [&](int i) { return i >= chunks ? chunks : i + turn < chunks ? i + turn : i + turn - chunks; };
    fetch_x(chunk_at(slice));
#pragma unroll
    for (int h = 0; h < U / STEPS; ++h) fetch_w(h, chunk_at(slice) * U + STEPS * h);
    fetch_s(chunk_at(slice));
    store_x(0);
    store_s();
    lds_barrier();
    for (int round = 0; round < rounds; ++round) {
        const int chunk = chunk_at(slice + round * KS), next = chunk_at(slice + (round + 1) * KS);
        const bool more = round + 1 < rounds;
        if (more) fetch_x(next);
        if (more) fetch_s(next);
        const uint8_t *xbuf = xs + (round & 1) * buffer_bytes;
        uint32_t words[8];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (u % STEPS == 0) {
                __builtin_memcpy(words, W[u / STEPS], sizeof(words));
                T::own(words);
                fetch_w(u / STEPS, next * U + u);  // (also behind the last chunk: under a branch they would all be waited for at its end)
            }
            if (chunk * U + u >= steps) continue;
            uint32_t *const word = words + u % STEPS * 4;
            float sc[128 / G];
#pragma unroll
            for (int i = 0; i < 128 / G; ++i) sc[i] = scales[nl * S::SPITCH + u * (128 / G) + i];
            T::operands(word);
            Acc sum[MT];
#pragma unroll
            for (int j = 0; j < 128 / T::KM; ++j) {
                if (j * T::KM % G == 0)
#pragma unroll
                    for (int t = 0; t < MT; ++t)
#pragma unroll
                        for (int i = 0; i < ACC; ++i) sum[t][i] = 0.0f;
                const typename P::V codes = P::codes(word[j]);
#pragma unroll
                for (int t = 0; t < MT; ++t)
#pragma unroll
                    for (int k = 0; k < S::PARTS; ++k) {
                        const uint4 x = *reinterpret_cast<const uint4 *>(xbuf + xrow[t] + k * part_bytes + (u * 128 + j * T::KM) * 2);
                        sum[t] = P::mul(__builtin_bit_cast(typename P::V, x), codes, sum[t]);
                    }
                if ((j + 1) * T::KM % G == 0)
#pragma unroll
                    for (int t = 0; t < MT; ++t)
#pragma unroll
                        for (int i = 0; i < ACC; ++i) total[t][i] = __builtin_fmaf(sum[t][i], sc[j * T::KM / G], total[t][i]);
            }
            // (else the compiler keeps the sums of all groups until the last product of the chunk, in registers that it lacks)
#pragma unroll
            for (int t = 0; t < MT; ++t) asm volatile("" : "+v"(total[t]));
        }
        if (more) {
            store_x((round + 1) & 1);
            store_s();
            lds_barrier();
        }
    }

    if constexpr (KS > 1) {
        float *const part = reinterpret_cast<float *>(smem);
        lds_barrier();  // the last chunk has been read
#pragma unroll
        for (int t = 0; t < MT; ++t)
#pragma unroll
            for (int i = 0; i < ACC; ++i) part[(t * ACC + i) * THREADS + tid] = total[t][i];
        lds_barrier();
        if (slice != 0) return;
#pragma unroll
        for (int s = 1; s < KS; ++s)
#pragma unroll
            for (int t = 0; t < MT; ++t)
#pragma unroll
                for (int i = 0; i < ACC; ++i) total[t][i] += part[(t * ACC + i) * THREADS + tid + s * XT];
    }
    store_tile<TN, MT>(p, total, n, m0, rows, q);
}

template <class E, int G, int TN, int MT, int WAVES, int KS>
static int launch_group4(Group4Params p, hipStream_t st)
{
    using S = Shape<E, G, TN, MT, WAVES, KS>;
    static_assert(S::lds(S::ROWS) <= 160 * 1024, "LDS is 160 KiB per CU");
    p.lds_rows = p.M < S::ROWS ? p.M : S::ROWS;
    p.blocks_n = (int)ceil_div(p.N, TN * (WAVES / KS));
    const int64_t workgroups = (int64_t)p.blocks_n * ceil_div(p.M, S::ROWS);
    if (!p.setup_only && !grid_ok(workgroups, 64 * WAVES)) return MKQ_ERR_UNSUPPORTED;
    static PerDeviceOnce once;  // (more than 64 KB of LDS have to be asked for)
    if (once.get([]() -> int {
            return hipFuncSetAttribute(reinterpret_cast<const void *>(&group4_kernel<E, G, TN, MT, WAVES, KS>), hipFuncAttributeMaxDynamicSharedMemorySize,
                                       (int)S::lds(S::ROWS)) == hipSuccess ? 1 : -1;
        }) <= 0)
        return MKQ_ERR_HIP;
    if (p.setup_only) return MKQ_OK;
    group4_kernel<E, G, TN, MT, WAVES, KS><<<(unsigned)workgroups, 64 * WAVES, S::lds(p.lds_rows), st>>>(p);
    return launch_status();
}

// Which tile, and how many of a workgroup's waves (eight) share its k loop: the largest tile whose workgroups fill the chip, since a tile
// of more tokens converts a code for more of them, and channels that share a workgroup read x once.  us, binary16, tokens of a tile and
// sharing waves: 120 tokens, K = 1024, N = 30522 15.3 (64, 1), 19.9 (64, 2), 21.3 (32, 2); 64 tokens, K = 8192, N = 28672 77.4 (64, 1), 54.8
// (64, 2), 68.7 (32, 2), 99.5 (16, 2); 128 tokens, K = 4096, N = 8192 25.9 (64, 2), 19.5 (32, 2), 25.0 (32, 4), K = 1024, N = 4096
// 9.1, 7.2, 6.2; 64 tokens, K = N = 4096 23.9 (64, 2), 12.6 (32, 4), 10.6 (16, 2), 11.2 (16, 4); one token, K = 768, N = 30522 6.3
// (16, 2), 7.6 (16, 4), K = 4096, N = 16384 10.2 and 9.7.  Sixteen waves where x is much of what is read: K = 8192, N = 28672 16 tokens 32.3
// instead of 34.1, 8 tokens 29.7 instead of 30.5, but one token 28.4 instead of 26.5; and eight of them on one k loop where that is
// long: one token, K = 28672, N = 8192 30.8 instead of 37.9, K = N = 8192 10.4 instead of 11.3, but K = 4096, N = 16384 12.2 instead of 9.7.
// Workgroups of four waves where even the last leave CUs idle, whatever K is; four | eight | sixteen with eight on a k loop, N = 768, one
// token, groups of 64: K = 768 3.4 | 3.7 | 4.2, 1200 4.2 | 4.3 | 4.1, 4096 6.1 | 6.4 | 6.1, 8192 9.9 | 10.2 | 8.9, 16384 17.7 | 17.8 | 14.6; 16
// tokens: 3.8 | 3.9 | 4.4, 4.8 | 4.7 | 4.5, 7.0 | 7.2 | 6.8, 11.4 | 11.6 | 10.3, 20.4 | 20.7 | 17.3: from K = 8192 on the sixteen would be better here, too.
// binary32 has 16 tokens a tile: its three parts leave larger tiles short chunks.  One | two waves on a k loop, groups of 64: 48 tokens,
// N = 30522, K = 768 16.4 | 32.0, K = 8192 147 | 209; 16 tokens, N = 8192, K = 768 7.2 | 6.3, K = 8192 53.5 | 34.8; between those, where two share
// a loop but take more than one round of the CUs, one would be better: 16 tokens, N = 30522, K = 768 8.0 | 11.9, K = 8192 56 | 71, 48 tokens,
// N = 16384, K = 768 10.6 | 16.3, N = 8192 7.5 | 11.2.
template <class E, int G>
static int choose_group4(const Group4Params &p, hipStream_t st)
{
    auto workgroups = [&](int tokens, int channels) { return ceil_div(p.N, channels) * ceil_div(p.M, tokens); };
    if constexpr (E::BYTES == 4) {
        return workgroups(16, 128) >= 400 ? launch_group4<E, G, 16, 1, 8, 1>(p, st) : launch_group4<E, G, 16, 1, 8, 2>(p, st);
    } else {
        if (p.M > 32 && workgroups(64, 256) >= 200) return launch_group4<E, G, 32, 2, 8, 1>(p, st);
        if (p.M > 32 && workgroups(64, 128) >= 200) return launch_group4<E, G, 32, 2, 8, 2>(p, st);
        if (p.M > 16 && workgroups(32, 128) >= 200) return launch_group4<E, G, 32, 1, 8, 2>(p, st);
        if (p.M > 16 && workgroups(32, 64) >= 200) return launch_group4<E, G, 32, 1, 8, 4>(p, st);
        if (p.M > 4 && workgroups(16, 128) >= 200) return launch_group4<E, G, 16, 1, 16, 2>(p, st);
        if (workgroups(16, 64) >= 400) return launch_group4<E, G, 16, 1, 8, 2>(p, st);
        if (workgroups(16, 32) >= 200) return p.K >= 8192 ? launch_group4<E, G, 16, 1, 16, 8>(p, st) : launch_group4<E, G, 16, 1, 8, 4>(p, st);
        return launch_group4<E, G, 16, 1, 4, 4>(p, st);
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

// Once-per-device setup of every tile (mkq_init)
int setup_group4()
{
    Group4Params p = {};
    p.M = p.N = p.K = 1;
    p.setup_only = true;
    int rc = MKQ_OK;
    auto all = [&](auto... statuses) { ((rc = rc == MKQ_OK ? statuses : rc), ...); };
    for (int dtype : {MKQ_F32, MKQ_F16, MKQ_BF16})
        for (int group : {32, 64, 128})
            with_elem(dtype, [&](auto e) {
                with_group(group, [&](auto g) {
                    using E = decltype(e);
                    constexpr int G = decltype(g)::value;
                    if constexpr (E::BYTES == 4)
                        all(launch_group4<E, G, 16, 1, 8, 1>(p, nullptr), launch_group4<E, G, 16, 1, 8, 2>(p, nullptr));
                    else
                        all(launch_group4<E, G, 32, 2, 8, 1>(p, nullptr), launch_group4<E, G, 32, 2, 8, 2>(p, nullptr),
                            launch_group4<E, G, 32, 1, 8, 2>(p, nullptr), launch_group4<E, G, 32, 1, 8, 4>(p, nullptr),
                            launch_group4<E, G, 16, 1, 16, 2>(p, nullptr), launch_group4<E, G, 16, 1, 8, 2>(p, nullptr),
                            launch_group4<E, G, 16, 1, 16, 8>(p, nullptr), launch_group4<E, G, 16, 1, 8, 4>(p, nullptr),
                            launch_group4<E, G, 16, 1, 4, 4>(p, nullptr));
                });
            });
    return rc;
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
    if (M > 0x7FFFFF00 || N > 0x7FFFFF00 || K > 0x7FFFF000) return MKQ_ERR_UNSUPPORTED;
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
    p.x_vec = rows_aligned16(x, ldx, x_dtype) && K % 8 == 0;
    const hipStream_t st = as_stream(stream);
    int status = MKQ_OK;
    with_elem(x_dtype, [&](auto e) {
        with_group(group, [&](auto g) { status = choose_group4<decltype(e), decltype(g)::value>(p, st); });
    });
    return status;
}
