// Activations kept in 8 bits from the forward pass to the backward: a step for every `group` neighbours of a row.
//
//     step = max|x| / 127 (binary32),  code = round(x / step)  to the nearest, ties to even, decided exactly
//     x' = code * step,   gelu(x') again,   dx = dy (Phi(x') + x' phi(x'))
//
// All are bound by bytes: each value is read once and written once.  A thread has eight neighbours, 4 to 16 lanes a group.
#include "elements.h"
#include "gemm_common.h"

namespace mkq {

struct CheckpointParams {
    const void *x;         // what is kept, or dy
    int8_t *codes;         // rows of pitch bytes
    float *steps;          // [M, groups]
    void *out;
    int64_t M, ldx, ld_out;
    int K, pitch, groups;
    int chunks;            // of eight values in a row, whole groups of them
    int group_shift;       // log2 of chunks in a group
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

// code = round(x / step) with |x| <= 127 step up to rounding.  fma(x, 1 / step, 128) is off by less than 5e-5 (its own rounding 2^-17,
// two of the quotient's 2^-24 times 127): where it lies nearer than that to a boundary the quotient is taken in binary64, in which
// it cannot be mistaken for one (x / step - (k + 1/2) is a multiple of 2^-32 of the quotient or more).
__device__ __forceinline__ uint2 checkpoint_codes(const float (&x)[8], float step)
{
    const float rs = 1.0f / step;
    uint32_t w[2] = {0, 0};
    bool near = false;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float v = __builtin_fmaf(x[e], rs, 128.0f), r = __builtin_rintf(v);
        near |= !(fabsf(v - r) <= 0.5f - 5e-5f);
        w[e >> 2] = __builtin_amdgcn_cvt_pk_u8_f32(__builtin_amdgcn_fmed3f(r, 1.0f, 255.0f), e & 3, w[e >> 2]);
    }
    if (__builtin_expect(near, 0)) {
        int c[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) c[e] = (int)__builtin_amdgcn_fmed3f((float)__builtin_rint((double)x[e] / (double)step), -127.0f, 127.0f);
        return bytes8(c);
    }
    return make_uint2(w[0] ^ 0x80808080u, w[1] ^ 0x80808080u);
}

// VEC: K is a multiple of 8 and all rows of x of 16 bytes
template <class E, int LANES, bool VEC>
__global__ __launch_bounds__(256) void checkpoint_kernel(const CheckpointParams p)
{
    const int64_t first = (int64_t)blockIdx.x * (256 * CHECKPOINT_UNROLL);
    const int64_t row0 = first / p.chunks;
    const uint32_t chunk0 = (uint32_t)(first - row0 * p.chunks) + threadIdx.x;
    float x[CHECKPOINT_UNROLL][8];
    int64_t row[CHECKPOINT_UNROLL];
    int k[CHECKPOINT_UNROLL];
#pragma unroll
    for (int u = 0; u < CHECKPOINT_UNROLL; ++u) {
        const uint32_t c = chunk0 + u * 256, down = c / (uint32_t)p.chunks;
        row[u] = row0 + down;
        k[u] = (int)(c - down * p.chunks) * 8;
#pragma unroll
        for (int e = 0; e < 8; ++e) x[u][e] = 0.0f;
        if (row[u] >= p.M) continue;
        const typename E::raw *at = static_cast<const typename E::raw *>(p.x) + row[u] * p.ldx + k[u];
        if constexpr (VEC) {
            if (k[u] < p.K) get8<E>(at, x[u]);
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (k[u] + e < p.K) x[u][e] = E::get(at[e]);
        }
    }
#pragma unroll
    for (int u = 0; u < CHECKPOINT_UNROLL; ++u) {
        uint32_t most = 0;  // bits of |x|: those of infinities and NaN are above all others'
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const uint32_t b = __float_as_uint(x[u][e]) & 0x7FFFFFFFu;
            most = most > b ? most : b;
        }
        most = lanes_max<LANES>(most);
        float step = __uint_as_float(most) / 127.0f;
        step = most == 0 ? 1.0f : __builtin_amdgcn_fmed3f(step, 0x1p-126f, STEP_MOST);
        const bool fine = most < 0x7F800000u;
        if (row[u] >= p.M) continue;
        const uint2 codes = fine ? checkpoint_codes(x[u], step) : make_uint2(0u, 0u);
        if (k[u] < p.pitch) *reinterpret_cast<uint2 *>(p.codes + row[u] * p.pitch + k[u]) = codes;
        if ((threadIdx.x & (LANES - 1)) == 0) p.steps[row[u] * p.groups + k[u] / (8 * LANES)] = fine ? step : __uint_as_float(0x7FC00000u);
    }
}

enum CheckpointUse { USE_VALUE, USE_GELU, USE_GELU_GRADIENT };

// Phi(x) + x phi(x).  With a = |x|: Phi(-a) from the polynomial of gelu_erf_tail, w = Phi(-a) - a phi(a); w for x < 0, else 1 - w.
__device__ __forceinline__ float gelu_slope(float x)
{
    const float ax = fabsf(x);
    float l = __builtin_fmaf(-6.406064857618525e-11f, ax, 3.993946363502951e-09f);
    l = __builtin_fmaf(l, ax, -1.0693068087399058e-07f);
    l = __builtin_fmaf(l, ax, 1.6153275431240008e-06f);
    l = __builtin_fmaf(l, ax, -1.517171398074849e-05f);
    l = __builtin_fmaf(l, ax, 9.05153156689754e-05f);
    l = __builtin_fmaf(l, ax, -3.076529474177308e-04f);
    l = __builtin_fmaf(l, ax, 3.0761933375104446e-05f);
    l = __builtin_fmaf(l, ax, 6.93251821915039e-03f);
    l = __builtin_fmaf(l, ax, -5.244305172617609e-02f);
    l = __builtin_fmaf(l, ax, -4.5921737336664303e-01f);
    l = __builtin_fmaf(l, ax, -1.1511048507359467f);
    l = __builtin_fmaf(l, ax, -1.0f);
    // (beyond 2^60 the density is 0 long since, and its square would be infinite)
    const float a = __builtin_amdgcn_fmed3f(ax, 0.0f, 0x1p60f);
    const float density = 0.3989422804014327f * __builtin_amdgcn_exp2f(-0.7213475204444817f * a * a);
    const float w = __builtin_fmaf(-ax, density, __builtin_amdgcn_exp2f(l));
    return x < 0.0f ? w : 1.0f - w;
}

// D: the type of dy (USE_GELU_GRADIENT); VEC: K is a multiple of 8 and all rows of dy and out of 16 bytes
template <class D, class O, int USE, bool VEC>
__global__ __launch_bounds__(256) void checkpoint_use_kernel(const CheckpointParams p)
{
    const int64_t first = (int64_t)blockIdx.x * (256 * CHECKPOINT_UNROLL);
    const int64_t row0 = first / p.chunks;
    const uint32_t chunk0 = (uint32_t)(first - row0 * p.chunks) + threadIdx.x;
    uint2 codes[CHECKPOINT_UNROLL];
    float step[CHECKPOINT_UNROLL], dy[CHECKPOINT_UNROLL][8];
    int64_t row[CHECKPOINT_UNROLL];
    int k[CHECKPOINT_UNROLL];
#pragma unroll
    for (int u = 0; u < CHECKPOINT_UNROLL; ++u) {
        const uint32_t c = chunk0 + u * 256, down = c / (uint32_t)p.chunks;
        row[u] = row0 + down;
        k[u] = (int)(c - down * p.chunks) * 8;
        if (row[u] >= p.M) continue;
        codes[u] = *reinterpret_cast<const uint2 *>(p.codes + row[u] * p.pitch + k[u]);
        step[u] = p.steps[row[u] * p.groups + (k[u] >> p.group_shift)];
        if constexpr (USE == USE_GELU_GRADIENT) {
            const typename D::raw *at = static_cast<const typename D::raw *>(p.x) + row[u] * p.ldx + k[u];
            if constexpr (VEC) {
                get8<D>(at, dy[u]);
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) dy[u][e] = k[u] + e < p.K ? D::get(at[e]) : 0.0f;
            }
        }
    }
#pragma unroll
    for (int u = 0; u < CHECKPOINT_UNROLL; ++u) {
        if (row[u] >= p.M) continue;
        float y[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const uint32_t w = e < 4 ? codes[u].x : codes[u].y;
            const float x = product((float)(int8_t)(w >> (8 * (e & 3))), step[u]);
            if constexpr (USE == USE_VALUE) y[e] = x;
            else if constexpr (USE == USE_GELU) y[e] = in_binary32(std::is_same<O, ElemF16>::value ? gelu_erf(x) : gelu_erf_tail(x));
            else y[e] = product(dy[u][e], gelu_slope(x));
        }
        typename O::raw *out = static_cast<typename O::raw *>(p.out) + row[u] * p.ld_out + k[u];
        if constexpr (VEC) {
            put8<O>(out, y);
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (k[u] + e < p.K) out[e] = O::put(y[e]);
        }
    }
}

// ---- host side ------------------------------------------------------------------------------------------------------------
constexpr int64_t CHECKPOINT_MOST = 0x7FFFFF00;  // columns, rows

static bool group_ok(int group) { return group == 32 || group == 64 || group == 128; }

static int checkpoint_grid(const CheckpointParams &p, unsigned *workgroups)
{
    const int64_t n = ceil_div(p.M * p.chunks, 256 * CHECKPOINT_UNROLL);  // (M and chunks are below 2^31 and 2^28)
    if (!grid_ok(n, 256)) return MKQ_ERR_UNSUPPORTED;
    *workgroups = (unsigned)n;
    return MKQ_OK;
}

// f(VEC)
template <class F>
static void with_vec(bool vec, F &&f)
{
    if (vec) f(std::true_type());
    else f(std::false_type());
}

template <int USE>
static int launch_use(const CheckpointParams &p, int dy_dtype, int out_dtype, hipStream_t st)
{
    unsigned workgroups;
    const int status = checkpoint_grid(p, &workgroups);
    if (status != MKQ_OK) return status;
    const bool vec = p.K % 8 == 0 && rows_aligned16(p.out, p.ld_out, out_dtype) &&
                     (USE != USE_GELU_GRADIENT || rows_aligned16(p.x, p.ldx, dy_dtype));
    with_elem(out_dtype, [&](auto o) {
        with_vec(vec, [&](auto v) {
            if constexpr (USE == USE_GELU_GRADIENT)
                with_elem(dy_dtype, [&](auto d) {
                    checkpoint_use_kernel<decltype(d), decltype(o), USE, decltype(v)::value><<<workgroups, 256, 0, st>>>(p);
                });
            else
                checkpoint_use_kernel<ElemF32, decltype(o), USE, decltype(v)::value><<<workgroups, 256, 0, st>>>(p);
        });
    });
    return launch_status();
}

static int log2_of(int group) { return group == 32 ? 5 : group == 64 ? 6 : 7; }

}  // namespace mkq

using namespace mkq;

extern "C" size_t mkq_checkpoint_bytes(int64_t M, int64_t K)
{
    return M <= 0 || K <= 0 || M > CHECKPOINT_MOST || K > CHECKPOINT_MOST ? 0 : (size_t)M * (size_t)(ceil_div(K, 32) * 32);
}

extern "C" int mkq_checkpoint_int8(const void *x, int x_dtype, int64_t M, int64_t K, int64_t ldx, int group, int8_t *codes, float *steps,
                                   void *stream)
{
    if (!is_float_dtype(x_dtype)) return MKQ_ERR_DTYPE;
    if (M < 0 || K <= 0 || ldx < K || !group_ok(group)) return MKQ_ERR_SHAPE;
    if (M == 0) return MKQ_OK;
    if (!x || !codes || !steps) return MKQ_ERR_NULL;
    if (!aligned16(x) || !aligned16(codes) || !aligned4(steps)) return MKQ_ERR_ALIGN;
    if (M > CHECKPOINT_MOST || K > CHECKPOINT_MOST) return MKQ_ERR_UNSUPPORTED;
    const int groups = (int)ceil_div(K, group), lanes = group / 8;
    const CheckpointParams p = {x, codes, steps, nullptr, M, ldx, 0, (int)K, (int)(ceil_div(K, 32) * 32), groups, groups * lanes, 0};
    unsigned workgroups;
    const int status = checkpoint_grid(p, &workgroups);
    if (status != MKQ_OK) return status;
    const hipStream_t st = as_stream(stream);
    with_elem(x_dtype, [&](auto e) {
        with_vec(K % 8 == 0 && rows_aligned16(x, ldx, x_dtype), [&](auto v) {
            constexpr bool VEC = decltype(v)::value;
            if (lanes == 4) checkpoint_kernel<decltype(e), 4, VEC><<<workgroups, 256, 0, st>>>(p);
            else if (lanes == 8) checkpoint_kernel<decltype(e), 8, VEC><<<workgroups, 256, 0, st>>>(p);
            else checkpoint_kernel<decltype(e), 16, VEC><<<workgroups, 256, 0, st>>>(p);
        });
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
    if (M > CHECKPOINT_MOST || K > CHECKPOINT_MOST) return MKQ_ERR_UNSUPPORTED;
    const CheckpointParams p = {nullptr, const_cast<int8_t *>(codes), const_cast<float *>(steps), out, M, 0, ld_out, (int)K,
                                (int)(ceil_div(K, 32) * 32), (int)ceil_div(K, group), (int)ceil_div(K, 8), log2_of(group)};
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
    if (M > CHECKPOINT_MOST || K > CHECKPOINT_MOST) return MKQ_ERR_UNSUPPORTED;
    if (!in_place_or_apart(dy, dy_dtype, ld_dy, dx, dx_dtype, ld_dx, M, K)) return MKQ_ERR_UNSUPPORTED;
    const CheckpointParams p = {dy, const_cast<int8_t *>(codes), const_cast<float *>(steps), dx, M, ld_dy, ld_dx, (int)K,
                                (int)(ceil_div(K, 32) * 32), (int)ceil_div(K, group), (int)ceil_div(K, 8), log2_of(group)};
    return launch_use<USE_GELU_GRADIENT>(p, dy_dtype, dx_dtype, as_stream(stream));
}
