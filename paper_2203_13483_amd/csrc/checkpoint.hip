// Activations kept in 8 bits from the forward pass to the backward: a step for every `group` neighbours of a row.
//
//     step = max|x| / 127 (binary32),  code = round(x / step)  to the nearest, ties to even, decided exactly
//     x' = code * step,   gelu(x') again,   dx = dy (Phi(x') + x' phi(x'))
//
// All are bound by bytes: each value is read once and written once.  A thread has eight neighbours, 4 to 16 lanes a group.  Measured, 16384 x 4096
// bfloat16, us among other calls (a trace's fastest; its medians, of calls one by one, are 43, 56 and 72): kept 38 (5.3 TB/s; vector issue 29), GELU again 45
// (4.5 TB/s; vector issue 44), GELU's gradient 66 (5.1 TB/s; vector issue 52).
#include "gemm_common.h"
#include "neighbours.h"

namespace mkq {

struct CheckpointParams {
    const void *x;         // what is kept, or dy
    int8_t *codes;         // rows of pitch bytes
    float *steps;          // [M, groups]
    void *out;
    int64_t M, ldx, ld_out;
    int K, pitch, groups;
    int chunks;            // of eight values in a row (checkpoint_kernel: whole groups of them)
    int group_shift;       // log2 of a group's values
    float chunk_part;      // 1 / chunks
    bool edge;             // K is no multiple of eight
};

// The u-th chunk of a thread: row and first value.  (The quotient of numbers below 2^20 by a reciprocal, from the middle of its step.)
struct ChunkAt {
    int64_t row;
    int k;
    __device__ __forceinline__ ChunkAt(const CheckpointParams &p, int64_t row0, uint32_t chunk0, int u)
    {
        const uint32_t c = chunk0 + u * 256;
        const uint32_t down = p.chunks < 1024 ? (uint32_t)(((float)c + 0.5f) * p.chunk_part) : c >= (uint32_t)p.chunks ? 1u : 0u;
        row = row0 + down;
        k = (int)(c - down * (uint32_t)p.chunks) * 8;
    }
};

constexpr int CHECKPOINT_UNROLL = 4;
constexpr float STEP_MOST = 8454659.0f * 0x1p98f;  // the largest step of which 127 are within binary32

// The code of the lane's value v in LANES neighbouring lanes, whose maximum all of them get
template <int LANES>
__device__ __forceinline__ uint32_t lanes_max(uint32_t v)
{
    auto with = [&](auto perm) {
        const uint32_t o = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, decltype(perm)::value, 0xF, 0xF, true);
        v = v > o ? v : o;
    };
    with(IntC<0xB1>());                              // of four lanes: 1 0 3 2
    with(IntC<0x4E>());                              // 2 3 0 1
    if constexpr (LANES >= 8) with(IntC<0x141>());   // of eight, the last first
    if constexpr (LANES >= 16) with(IntC<0x140>());  // of sixteen
    return v;
}

// code = round(x / step), |x| <= 127 step up to rounding: in binary64, in which a quotient cannot be mistaken for a boundary (it is off one by 2^-33 of
// itself or more)
__device__ __forceinline__ uint2 codes_by_division(const float (&x)[8], float step)
{
    int c[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) c[e] = (int)__builtin_amdgcn_fmed3f((float)__builtin_rint((double)x[e] / (double)step), -127.0f, 127.0f);
    return bytes8(c);
}

// Binary32 values: fma(x, 1 / step, 128) is off by less than 5e-5 (its own rounding 2^-17, two of the quotient's 2^-24 times 127); where it
// lies nearer than that to a boundary the eight are divided.
template <class E>
__device__ __forceinline__ uint2 checkpoint_codes(const Neighbours<E, true> &n, float step, float)
{
    float x[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = n.get(e);
    if constexpr (E::BYTES == 4) {
        const float rs = 1.0f / step;
        uint32_t w[2] = {0, 0};
        bool near = false;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float v = __builtin_fmaf(x[e], rs, 128.0f), r = __builtin_rintf(v);
            near |= !(fabsf(v - r) <= 0.5f - 5e-5f);
            w[e >> 2] = __builtin_amdgcn_cvt_pk_u8_f32(__builtin_amdgcn_fmed3f(r, 1.0f, 255.0f), e & 3, w[e >> 2]);
        }
        if (__builtin_expect(near, 0)) return codes_by_division(x, step);
        return make_uint2(w[0] ^ 0x80808080u, w[1] ^ 0x80808080u);
    }
}
// Values of 16 bits have significands of at most 11: 127 x / max|x| is a boundary k + 1/2 exactly, as it often is, or off it by 1 / (254 * 2^11)
// = 1.9e-6 of itself or more.  x / step differs from that quotient by the step's rounding, less than 6e-8, whose sign alone decides on the exact ones: a
// factor 1 / step moved by 3e-7 against it rounds all values as they have to be (its own roundings are 1.2e-7), in one fused
// addition of 1.5 * 2^23, which leaves the code in the low byte.  Steps that are exact, or not the quotient, divide.
template <class E>
__device__ __forceinline__ uint2 checkpoint_codes_16(const Neighbours<E, true> &n, float step, float most)
{
    const float off = __builtin_fmaf(step, 127.0f, -most);  // the step's rounding, with its sign
    if (__builtin_expect(off == 0.0f || step <= 0x1p-126f || step >= STEP_MOST || most == 0.0f, 0)) {
        float x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = n.get(e);
        return codes_by_division(x, step);
    }
    const float rs = (1.0f / step) * (off > 0.0f ? 1.0f - 3e-7f : 1.0f + 3e-7f);
    uint32_t v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = __float_as_uint(__builtin_fmaf(n.get(e), rs, 12582912.0f));
    auto four = [](uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
        return __builtin_amdgcn_perm(__builtin_amdgcn_perm(d, c, 0x0C0C0400u), __builtin_amdgcn_perm(b, a, 0x0C0C0400u), 0x05040100u);
    };
    return make_uint2(four(v[0], v[1], v[2], v[3]), four(v[4], v[5], v[6], v[7]));
}

// The largest |x| of eight as bits: those of infinities and NaN are above all others'
template <class E>
__device__ __forceinline__ uint32_t largest_bits(const Neighbours<E, true> &n)
{
    uint32_t most = 0;
    if constexpr (E::BYTES == 4) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const uint32_t b = n.w[e / 4][e % 4] & 0x7FFFFFFFu;
            most = most > b ? most : b;
        }
    } else {
        typedef unsigned short us2 __attribute__((ext_vector_type(2)));
        us2 two = {0, 0};
#pragma unroll
        for (int i = 0; i < 4; ++i) two = __builtin_elementwise_max(two, __builtin_bit_cast(us2, (uint32_t)(n.w[0][i] & 0x7FFF7FFFu)));
        most = two[0] > two[1] ? two[0] : two[1];
    }
    return most;
}

template <class E, int LANES>
__global__ __launch_bounds__(256) void checkpoint_kernel(const CheckpointParams p)
{
    const int64_t first = (int64_t)blockIdx.x * (256 * CHECKPOINT_UNROLL), row0 = first / p.chunks;
    const uint32_t chunk0 = (uint32_t)(first - row0 * p.chunks) + threadIdx.x;
    Neighbours<E, true> x[CHECKPOINT_UNROLL];
#pragma unroll
    for (int u = 0; u < CHECKPOINT_UNROLL; ++u) {
        const ChunkAt at(p, row0, chunk0, u);
        x[u].clear();
        if (at.row < p.M && at.k < p.K) x[u].fetch(static_cast<const typename E::raw *>(p.x) + at.row * p.ldx, at.k, p.K, p.edge);
    }
#pragma unroll
    for (int u = 0; u < CHECKPOINT_UNROLL; ++u) {
        const ChunkAt at(p, row0, chunk0, u);
        const uint32_t bits = lanes_max<LANES>(largest_bits(x[u]));
        float most;
        bool fine;
        if constexpr (E::BYTES == 4) {
            most = __uint_as_float(bits);
            fine = bits < 0x7F800000u;
        } else {
            most = E::get((uint16_t)bits);
            fine = bits < (std::is_same<E, ElemF16>::value ? 0x7C00u : 0x7F80u);
        }
        const float step = most == 0.0f ? 1.0f : __builtin_amdgcn_fmed3f(most / 127.0f, 0x1p-126f, STEP_MOST);
        if (at.row >= p.M) continue;
        uint2 codes = make_uint2(0u, 0u);
        if (fine) {
            if constexpr (E::BYTES == 4) codes = checkpoint_codes(x[u], step, most);
            else codes = checkpoint_codes_16(x[u], step, most);
        }
        if (at.k < p.pitch) *reinterpret_cast<uint2 *>(p.codes + at.row * p.pitch + at.k) = codes;
        if ((threadIdx.x & (LANES - 1)) == 0) p.steps[at.row * p.groups + (at.k >> p.group_shift)] = fine ? step : __uint_as_float(0x7FC00000u);
    }
}

enum CheckpointUse { USE_VALUE, USE_GELU, USE_GELU_GRADIENT };

// Phi(x) + x phi(x).  With a = |x|: w = Phi(-a) - a phi(a) = phi(a) (R(a) - a), R the ratio Phi(-a) / phi(a) as a polynomial in t = 1 / (1 + 0.28 a) (a
// minimax fit, linear program, our own, of the error of phi R, 1e-8); w for x < 0, else 1 - w.  Evaluated in binary32 against binary64: largest error
// 2.3e-7, most of it the rounding of values near 1; relative 2e-5 for x in [-12, -2].
__device__ __forceinline__ float gelu_slope(float x)
{
    const float ax = fabsf(x), t = __builtin_amdgcn_rcpf(__builtin_fmaf(0.28f, ax, 1.0f));
    float h = __builtin_fmaf(-0.26522333066030684f, t, 0.9772749130935714f);
    h = __builtin_fmaf(h, t, -0.5940637376271297f);
    h = __builtin_fmaf(h, t, 0.6740651936573456f);
    h = __builtin_fmaf(h, t, 0.16918633104212444f);
    h = __builtin_fmaf(h, t, 0.29207474454413423f);
    h = __builtin_fmaf(h, t, -ax);
    const float w = h * (0.3989422804014327f * __builtin_amdgcn_exp2f(-0.7213475204444817f * ax * ax));
    return x < 0.0f ? w : 1.0f - w;
}

// D: the type of dy (USE_GELU_GRADIENT)
template <class D, class O, int USE>
__global__ __launch_bounds__(256) void checkpoint_use_kernel(const CheckpointParams p)
{
    const int64_t first = (int64_t)blockIdx.x * (256 * CHECKPOINT_UNROLL), row0 = first / p.chunks;
    const uint32_t chunk0 = (uint32_t)(first - row0 * p.chunks) + threadIdx.x;
    uint2 codes[CHECKPOINT_UNROLL];
    float step[CHECKPOINT_UNROLL];
    Neighbours<D, true> dy[CHECKPOINT_UNROLL];
#pragma unroll
    for (int u = 0; u < CHECKPOINT_UNROLL; ++u) {
        const ChunkAt at(p, row0, chunk0, u);
        if (at.row >= p.M) continue;
        codes[u] = *reinterpret_cast<const uint2 *>(p.codes + at.row * p.pitch + at.k);
        step[u] = p.steps[at.row * p.groups + (at.k >> p.group_shift)];
        if constexpr (USE == USE_GELU_GRADIENT) dy[u].fetch(static_cast<const typename D::raw *>(p.x) + at.row * p.ldx, at.k, p.K, p.edge);
    }
#pragma unroll
    for (int u = 0; u < CHECKPOINT_UNROLL; ++u) {
        const ChunkAt at(p, row0, chunk0, u);
        if (at.row >= p.M) continue;
        float y[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float x = product((float)(int8_t)((e < 4 ? codes[u].x : codes[u].y) >> (8 * (e & 3))), step[u]);
            if constexpr (USE == USE_VALUE) y[e] = x;
            else if constexpr (USE == USE_GELU) y[e] = std::is_same<O, ElemF16>::value ? gelu_erf(x) : gelu_erf_tail(x);
            else y[e] = dy[u].get(e) * gelu_slope(x);
        }
        put_neighbours<O>(static_cast<typename O::raw *>(p.out) + at.row * p.ld_out, 0, at.k, p.K, p.edge, y);
    }
}

// ---- host side ------------------------------------------------------------------------------------------------------------
constexpr int64_t CHECKPOINT_MOST = 0x7FFFFF00, COLUMNS_MOST = (int64_t)1 << 29;  // rows; a row's bytes are counted in 32 bits

static bool group_ok(int group) { return group == 32 || group == 64 || group == 128; }

static int checkpoint_grid(const CheckpointParams &p, unsigned *workgroups)
{
    const int64_t n = ceil_div(p.M * p.chunks, 256 * CHECKPOINT_UNROLL);  // (M and chunks are below 2^31 and 2^28)
    if (!grid_ok(n, 256)) return MKQ_ERR_UNSUPPORTED;
    *workgroups = (unsigned)n;
    return MKQ_OK;
}

template <int USE>
static int launch_use(const CheckpointParams &p, int dy_dtype, int out_dtype, hipStream_t st)
{
    unsigned workgroups;
    const int status = checkpoint_grid(p, &workgroups);
    if (status != MKQ_OK) return status;
    with_elem(out_dtype, [&](auto o) {
        if constexpr (USE == USE_GELU_GRADIENT)
            with_elem(dy_dtype, [&](auto d) { checkpoint_use_kernel<decltype(d), decltype(o), USE><<<workgroups, 256, 0, st>>>(p); });
        else
            checkpoint_use_kernel<ElemF32, decltype(o), USE><<<workgroups, 256, 0, st>>>(p);
    });
    return launch_status();
}

static CheckpointParams checkpoint_params(const int8_t *codes, const float *steps, int group, int64_t M, int64_t K)
{
    CheckpointParams p = {};
    p.codes = const_cast<int8_t *>(codes);
    p.steps = const_cast<float *>(steps);
    p.M = M;
    p.K = (int)K;
    p.pitch = (int)(ceil_div(K, 32) * 32);
    p.groups = (int)ceil_div(K, group);
    p.chunks = (int)ceil_div(K, 8);
    p.group_shift = group == 32 ? 5 : group == 64 ? 6 : 7;
    p.chunk_part = 1.0f / (float)p.chunks;
    p.edge = K % 8 != 0;
    return p;
}

// Whether rows [M, K] lie apart from what is kept of them
static bool apart_from_kept(const CheckpointParams &p, const void *rows, int dtype, int64_t ld)
{
    return apart(rows, dtype, ld, p.K, p.codes, MKQ_I8, p.pitch, p.pitch, p.M) && apart(rows, dtype, ld, p.K, p.steps, MKQ_F32, p.groups, p.groups, p.M);
}

}  // namespace mkq

using namespace mkq;

extern "C" size_t mkq_checkpoint_bytes(int64_t M, int64_t K)
{
    return M <= 0 || K <= 0 || M > CHECKPOINT_MOST || K > COLUMNS_MOST ? 0 : (size_t)M * (size_t)(ceil_div(K, 32) * 32);
}

extern "C" int mkq_checkpoint_int8(const void *x, int x_dtype, int64_t M, int64_t K, int64_t ldx, int group, int8_t *codes, float *steps,
                                   void *stream)
{
    if (!is_float_dtype(x_dtype)) return MKQ_ERR_DTYPE;
    if (M < 0 || K <= 0 || ldx < K || !group_ok(group)) return MKQ_ERR_SHAPE;
    if (M == 0) return MKQ_OK;
    if (!x || !codes || !steps) return MKQ_ERR_NULL;
    if (!aligned16(x) || !aligned16(codes) || !aligned4(steps)) return MKQ_ERR_ALIGN;
    if (M > CHECKPOINT_MOST || K > COLUMNS_MOST) return MKQ_ERR_UNSUPPORTED;
    CheckpointParams p = checkpoint_params(codes, steps, group, M, K);
    if (!apart_from_kept(p, x, x_dtype, ldx) || !apart(codes, MKQ_I8, p.pitch, p.pitch, steps, MKQ_F32, p.groups, p.groups, M)) return MKQ_ERR_UNSUPPORTED;
    p.x = x;
    p.ldx = ldx;
    p.chunks = p.groups * (group / 8);
    p.chunk_part = 1.0f / (float)p.chunks;
    unsigned workgroups;
    const int status = checkpoint_grid(p, &workgroups);
    if (status != MKQ_OK) return status;
    const hipStream_t st = as_stream(stream);
    with_elem(x_dtype, [&](auto e) {
        if (group == 32) checkpoint_kernel<decltype(e), 4><<<workgroups, 256, 0, st>>>(p);
        else if (group == 64) checkpoint_kernel<decltype(e), 8><<<workgroups, 256, 0, st>>>(p);
        else checkpoint_kernel<decltype(e), 16><<<workgroups, 256, 0, st>>>(p);
    });
    return launch_status();
}

extern "C" int mkq_checkpoint_restore(const int8_t *codes, const float *steps, int group, int64_t M, int64_t K, int act, void *out,
                                      int out_dtype, int64_t ld_out, void *stream)
{
    if (!is_float_dtype(out_dtype) || (act != MKQ_ACT_NONE && act != MKQ_ACT_GELU)) return MKQ_ERR_DTYPE;
    if (M < 0 || K <= 0 || ld_out < K || !group_ok(group)) return MKQ_ERR_SHAPE;
    if (M == 0) return MKQ_OK;
    if (!codes || !steps || !out) return MKQ_ERR_NULL;
    if (!aligned16(codes) || !aligned4(steps) || !aligned16(out)) return MKQ_ERR_ALIGN;
    if (M > CHECKPOINT_MOST || K > COLUMNS_MOST) return MKQ_ERR_UNSUPPORTED;
    CheckpointParams p = checkpoint_params(codes, steps, group, M, K);
    if (!apart_from_kept(p, out, out_dtype, ld_out)) return MKQ_ERR_UNSUPPORTED;
    p.out = out;
    p.ld_out = ld_out;
    return act == MKQ_ACT_GELU ? launch_use<USE_GELU>(p, MKQ_F32, out_dtype, as_stream(stream))
                               : launch_use<USE_VALUE>(p, MKQ_F32, out_dtype, as_stream(stream));
}

extern "C" int mkq_checkpoint_gelu_gradient(const int8_t *codes, const float *steps, int group, int64_t M, int64_t K, const void *dy,
                                            int dy_dtype, int64_t ld_dy, void *dx, int dx_dtype, int64_t ld_dx, void *stream)
{
    if (!is_float_dtype(dy_dtype) || !is_float_dtype(dx_dtype)) return MKQ_ERR_DTYPE;
    if (M < 0 || K <= 0 || ld_dy < K || ld_dx < K || !group_ok(group)) return MKQ_ERR_SHAPE;
    if (M == 0) return MKQ_OK;
    if (!codes || !steps || !dy || !dx) return MKQ_ERR_NULL;
    if (!aligned16(codes) || !aligned4(steps) || !aligned16(dy) || !aligned16(dx)) return MKQ_ERR_ALIGN;
    if (M > CHECKPOINT_MOST || K > COLUMNS_MOST) return MKQ_ERR_UNSUPPORTED;
    if (!in_place_or_apart(dy, dy_dtype, ld_dy, dx, dx_dtype, ld_dx, M, K)) return MKQ_ERR_UNSUPPORTED;
    CheckpointParams p = checkpoint_params(codes, steps, group, M, K);
    if (!apart_from_kept(p, dx, dx_dtype, ld_dx)) return MKQ_ERR_UNSUPPORTED;
    p.x = dy;
    p.ldx = ld_dy;
    p.out = dx;
    p.ld_out = ld_dx;
    return launch_use<USE_GELU_GRADIENT>(p, dy_dtype, dx_dtype, as_stream(stream));
}
