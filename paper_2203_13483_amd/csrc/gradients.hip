// The norm over the gradients of many tensors, and their clipping:
//
//     norm = sqrt( sum_t sum_i g_t[i]^2 ),   out_t[i] = min(1, max_norm / (norm + 1e-6)) g_t[i]
//
// Bound by HBM: every value is read once for the norm and once more, behind it, to be scaled and written.  Squares and their
// sums are binary64, in an order that does not depend on which workgroup is done first, so the norm of gradients beyond
// 1e19 does not overflow and equal inputs give equal bits.  Measured: 81 million binary32 values 157 us (6.2 TB/s), 13 million 31 us.
#include <algorithm>
#include <memory>
#include <new>

#include "elements.h"
#include "gemm_common.h"

namespace mkq {

// Tensors of one launch travel in the kernel's arguments, whose room is 4 KiB
constexpr int TENSORS = 100;
constexpr int PIECE = 8192;            // values that a workgroup takes at a time
constexpr int NORM_WORKGROUPS = 2048;  // partial sums of a launch
struct TensorList {
    const void *grad[TENSORS];
    void *out[TENSORS];
    int64_t count[TENSORS];
    int32_t first_piece[TENSORS + 1];
    int8_t dtype[TENSORS];
    int32_t n;
};
static_assert(sizeof(TensorList) <= 3800, "kernel arguments");

// f(tensor, first value, values) for the pieces of this workgroup
template <bool BACKWARDS, class F>
__device__ __forceinline__ void for_each_piece(const TensorList &l, F &&f)
{
    const int pieces = l.first_piece[l.n];
    for (int i = blockIdx.x; i < pieces; i += gridDim.x) {
        const int piece = BACKWARDS ? pieces - 1 - i : i;
        int lo = 0, hi = l.n;  // the last tensor whose first piece is at most this one
        while (hi - lo > 1) {
            const int mid = (lo + hi) / 2;
            if (l.first_piece[mid] <= piece) lo = mid;
            else hi = mid;
        }
        const int64_t from = (int64_t)(piece - l.first_piece[lo]) * PIECE;
        const int64_t left = l.count[lo] - from;
        f(lo, from, (int)(left < PIECE ? left : PIECE));
    }
}

// Sum over a workgroup of 256, the same bits in every thread
__device__ __forceinline__ double workgroup_sum(double v, double *part)
{
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) v += __shfl_xor(v, off, 64);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
    __syncthreads();
    return (part[0] + part[1]) + (part[2] + part[3]);
}

// The values of 16 bytes
template <class E>
struct Vector {
    static constexpr int N = 16 / E::BYTES;
    uint4 raw;
    __device__ __forceinline__ float get(int i) const
    {
        const uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
        if constexpr (E::BYTES == 4) return __uint_as_float(w[i]);
        else return E::get((uint16_t)(w[i / 2] >> (16 * (i % 2))));
    }
    __device__ __forceinline__ void scale(float c)
    {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (E::BYTES == 4) w[i] = __float_as_uint(get(i) * c);
            else w[i] = std::is_same<E, ElemF16>::value ? pack2_f16(product(get(2 * i), c), product(get(2 * i + 1), c))
                                                        : pack2_bf16(product(get(2 * i), c), product(get(2 * i + 1), c));
        }
        raw = make_uint4(w[0], w[1], w[2], w[3]);
    }
};

// f(number of vectors, the first) and g(a value's place) for the values of a piece: whole pieces as neighbouring vectors of 16 bytes
// a thread, all of them asked for before the first is used; what is left, or not aligned to vectors, value by value
template <class E, class F, class G>
__device__ __forceinline__ void each_vector(uintptr_t aligned, int values, F &&f, G &&g)
{
    constexpr int N = Vector<E>::N;
    int from = 0;
    if (aligned % 16 == 0) {
        if (values == PIECE) return f(IntC<PIECE / 256 / N>(), threadIdx.x);
        const int vectors = values / N;
        for (int v = threadIdx.x; v < vectors; v += 256) f(IntC<1>(), v);
        from = vectors * N;
    }
    for (int i = from + threadIdx.x; i < values; i += 256) g(i);
}

template <class E>
__device__ __forceinline__ double sum_squares(const void *p, int64_t at, int values)
{
    const typename E::raw *g = static_cast<const typename E::raw *>(p) + at;
    double sum = 0.0;
    auto add = [&](float v) { sum = __builtin_fma((double)v, (double)v, sum); };
    each_vector<E>(
        reinterpret_cast<uintptr_t>(g), values,
        [&](auto n, int v) {
            Vector<E> x[decltype(n)::value];
#pragma unroll
            for (int k = 0; k < decltype(n)::value; ++k) x[k].raw = reinterpret_cast<const uint4 *>(g)[v + k * 256];
#pragma unroll
            for (int k = 0; k < decltype(n)::value; ++k)
#pragma unroll
                for (int i = 0; i < Vector<E>::N; ++i) add(x[k].get(i));
        },
        [&](int i) { add(E::get(g[i])); });
    return sum;
}

__global__ __launch_bounds__(256) void norm_partials_kernel(const TensorList l, double *__restrict__ partials)
{
    __shared__ double part[4];
    double sum = 0.0;
    for_each_piece<false>(l, [&](int t, int64_t from, int values) {
        if (l.dtype[t] == MKQ_F32) sum += sum_squares<ElemF32>(l.grad[t], from, values);
        else if (l.dtype[t] == MKQ_F16) sum += sum_squares<ElemF16>(l.grad[t], from, values);
        else sum += sum_squares<ElemBF16>(l.grad[t], from, values);
    });
    sum = workgroup_sum(sum, part);
    if (threadIdx.x == 0) partials[blockIdx.x] = sum;
}

__device__ __forceinline__ double norm_of(const double *__restrict__ partials, int count, double *part)
{
    double sum = 0.0;
    for (int i = threadIdx.x; i < count; i += 256) sum += partials[i];
    return sqrt(workgroup_sum(sum, part));
}

__global__ __launch_bounds__(256) void norm_kernel(const double *__restrict__ partials, int count, float *__restrict__ norm_out)
{
    __shared__ double part[4];
    const double norm = norm_of(partials, count, part);
    if (threadIdx.x == 0) *norm_out = (float)norm;
}

// Results go past the caches: left dirty there, they are written back under the next pass over as many bytes (81 million binary32
// values clipped 189 -> 157 us, with an update that reads them behind it 352 -> 335; 13 million 31 and 31, 63 -> 59).
template <class E>
__device__ __forceinline__ void scale_values(const void *p, void *q, int64_t at, int values, float c)
{
    const typename E::raw *g = static_cast<const typename E::raw *>(p) + at;
    typename E::raw *out = static_cast<typename E::raw *>(q) + at;
    each_vector<E>(
        reinterpret_cast<uintptr_t>(g) | reinterpret_cast<uintptr_t>(out), values,
        [&](auto n, int v) {
            Vector<E> x[decltype(n)::value];
#pragma unroll
            for (int k = 0; k < decltype(n)::value; ++k) x[k].raw = reinterpret_cast<const uint4 *>(g)[v + k * 256];
#pragma unroll
            for (int k = 0; k < decltype(n)::value; ++k) {
                x[k].scale(c);
                store16<true>(reinterpret_cast<uint4 *>(out) + v + k * 256, x[k].raw);
            }
        },
        [&](int i) { out[i] = E::put(product(E::get(g[i]), c)); });
}

// The same for a factor below binary32's normal numbers, which has few bits there or none: the product is binary64, rounded to binary32
// and to the type.  (Norms near the end of binary32's range under a small limit; value by value, nothing else is bound by it.)
template <class E>
__device__ __forceinline__ void scale_values_small(const void *p, void *q, int64_t at, int values, double c)
{
    const typename E::raw *g = static_cast<const typename E::raw *>(p) + at;
    typename E::raw *out = static_cast<typename E::raw *>(q) + at;
    for (int i = threadIdx.x; i < values; i += 256) out[i] = E::put((float)((double)E::get(g[i]) * c));
}

// Every workgroup adds up the partial sums itself (up to 16 KB out of the L2 for every hundred tensors), which spares a launch between
// the two passes.
// Last pieces first: they were read last, and what the memory-side cache still holds of them need not come from HBM again.
// A factor of 1 leaves gradients that are clipped in place as they are.  Without a limit (max_norm = infinity) it is 1 whatever the
// norm: infinity over an infinite norm would make every finite gradient a NaN.
__global__ __launch_bounds__(256) void clip_kernel(const TensorList l, const double *__restrict__ partials, int count, float max_norm,
                                                   float *__restrict__ norm_out)
{
    __shared__ double part[4];
    const double norm = norm_of(partials, count, part);
    if (norm_out && blockIdx.x == 0 && threadIdx.x == 0) *norm_out = (float)norm;
    const double q = max_norm == __builtin_inff() ? 1.0 : (double)max_norm / (norm + 1e-6);
    const float c = q < 1.0 || q != q ? (float)q : 1.0f;
    for_each_piece<true>(l, [&](int t, int64_t from, int values) {
        if (c == 1.0f && l.out[t] == l.grad[t]) return;
        if (q > 0.0 && q < 0x1p-126) {
            if (l.dtype[t] == MKQ_F32) scale_values_small<ElemF32>(l.grad[t], l.out[t], from, values, q);
            else if (l.dtype[t] == MKQ_F16) scale_values_small<ElemF16>(l.grad[t], l.out[t], from, values, q);
            else scale_values_small<ElemBF16>(l.grad[t], l.out[t], from, values, q);
            return;
        }
        if (l.dtype[t] == MKQ_F32) scale_values<ElemF32>(l.grad[t], l.out[t], from, values, c);
        else if (l.dtype[t] == MKQ_F16) scale_values<ElemF16>(l.grad[t], l.out[t], from, values, c);
        else scale_values<ElemBF16>(l.grad[t], l.out[t], from, values, c);
    });
}

// The lists of the launches that n tensors take, one after the other: f(list, workgroups)
template <class F>
static int for_each_list(int64_t n, const void *const *grads, void *const *outs, const int64_t *counts, const int32_t *dtypes, F &&f)
{
    for (int64_t t = 0; t < n;) {
        TensorList l;
        l.n = 0;
        l.first_piece[0] = 0;
        for (; t < n && l.n < TENSORS; ++t) {
            if (counts[t] == 0) continue;
            l.grad[l.n] = grads[t];
            l.out[l.n] = outs ? outs[t] : const_cast<void *>(grads[t]);
            l.count[l.n] = counts[t];
            l.dtype[l.n] = (int8_t)dtypes[t];
            l.first_piece[l.n + 1] = l.first_piece[l.n] + (int32_t)ceil_div(counts[t], PIECE);
            ++l.n;
        }
        if (l.n == 0) break;
        const int pieces = l.first_piece[l.n];
        f(l, pieces < NORM_WORKGROUPS ? pieces : NORM_WORKGROUPS);
        if (launch_status() != MKQ_OK) return MKQ_ERR_HIP;
    }
    return MKQ_OK;
}

static int check_tensors(int64_t n, const void *const *grads, void *const *outs, const int64_t *counts, const int32_t *dtypes,
                         const void *workspace, size_t workspace_bytes)
{
    if (n < 0) return MKQ_ERR_SHAPE;
    if (n > 0 && (!grads || !counts || !dtypes)) return MKQ_ERR_NULL;
    int64_t pieces = 0;
    for (int64_t t = 0; t < n; ++t) {
        if (!is_float_dtype(dtypes[t])) return MKQ_ERR_DTYPE;
        if (counts[t] < 0) return MKQ_ERR_SHAPE;
        if (counts[t] == 0) continue;
        if (!grads[t] || (outs && !outs[t])) return MKQ_ERR_NULL;
        const uintptr_t low = reinterpret_cast<uintptr_t>(grads[t]) | (outs ? reinterpret_cast<uintptr_t>(outs[t]) : 0);
        if (low % dtype_bytes(dtypes[t])) return MKQ_ERR_ALIGN;
        pieces += (counts[t] - 1) / PIECE + 1;
        if (pieces > 0x7FFFFFFF) return MKQ_ERR_UNSUPPORTED;
    }
    if (!workspace || workspace_bytes < mkq_gradient_norm_workspace_bytes(n)) return MKQ_ERR_WORKSPACE;
    if (!aligned16(workspace)) return MKQ_ERR_ALIGN;
    return MKQ_OK;
}

// Whether no result lies over another one or over a gradient other than the one it is clipped from in place: a launch's workgroups
// would read what others have scaled already.  In the order of their addresses every piece of memory has only to begin behind what was
// written before it, and a result behind what was read, too.  (Two gradients may share memory.  Sorting takes 2.9 us for 50 tensors
// with results of their own in any order, nothing for those of one allocation after the other.)
struct Piece {
    uintptr_t begin, end;
    bool written;
};
static bool results_apart(Piece *pieces, int64_t n, const void *const *grads, void *const *outs, const int64_t *counts, const int32_t *dtypes)
{
    int64_t m = 0;
    for (int64_t t = 0; t < n; ++t) {
        if (counts[t] == 0) continue;
        const uintptr_t bytes = (uintptr_t)(counts[t] * dtype_bytes(dtypes[t])), at = reinterpret_cast<uintptr_t>(outs[t]);
        pieces[m++] = {at, at + bytes, true};
        if (outs[t] != grads[t]) pieces[m++] = {reinterpret_cast<uintptr_t>(grads[t]), reinterpret_cast<uintptr_t>(grads[t]) + bytes, false};
    }
    const auto before = [](const Piece &a, const Piece &b) { return a.begin < b.begin; };
    if (!std::is_sorted(pieces, pieces + m, before)) std::sort(pieces, pieces + m, before);
    uintptr_t written = 0, read = 0;  // where they end
    for (int64_t i = 0; i < m; ++i) {
        const Piece &p = pieces[i];
        if (p.begin < written || (p.written && p.begin < read)) return false;
        uintptr_t &last = p.written ? written : read;
        last = p.end > last ? p.end : last;
    }
    return true;
}

static int check_results_apart(int64_t n, const void *const *grads, void *const *outs, const int64_t *counts, const int32_t *dtypes)
{
    constexpr int64_t FEW = 256;
    Piece few[2 * FEW];
    if (n <= FEW) return results_apart(few, n, grads, outs, counts, dtypes) ? MKQ_OK : MKQ_ERR_UNSUPPORTED;
    const std::unique_ptr<Piece[]> many(new (std::nothrow) Piece[2 * n]);
    return many && results_apart(many.get(), n, grads, outs, counts, dtypes) ? MKQ_OK : MKQ_ERR_UNSUPPORTED;
}

// Launches the partial sums of all tensors; *count: how many there are
static int launch_partials(int64_t n, const void *const *grads, const int64_t *counts, const int32_t *dtypes, double *partials, int *count,
                           hipStream_t st)
{
    *count = 0;
    return for_each_list(n, grads, nullptr, counts, dtypes, [&](const TensorList &l, int workgroups) {
        norm_partials_kernel<<<workgroups, 256, 0, st>>>(l, partials + *count);
        *count += workgroups;
    });
}

}  // namespace mkq

using namespace mkq;

extern "C" size_t mkq_gradient_norm_workspace_bytes(int64_t n)
{
    return n < 0 ? 0 : (size_t)(n / TENSORS + 1) * NORM_WORKGROUPS * sizeof(double);
}

extern "C" int mkq_gradient_norm(int64_t n, const void *const *grads_host, const int64_t *counts_host, const int32_t *dtypes_host,
                                 float *norm_out, void *workspace, size_t workspace_bytes, void *stream)
{
    if (!norm_out) return MKQ_ERR_NULL;
    if (!aligned4(norm_out)) return MKQ_ERR_ALIGN;
    int status = check_tensors(n, grads_host, nullptr, counts_host, dtypes_host, workspace, workspace_bytes);
    if (status != MKQ_OK) return status;
    const hipStream_t st = as_stream(stream);
    double *partials = static_cast<double *>(workspace);
    int count;
    status = launch_partials(n, grads_host, counts_host, dtypes_host, partials, &count, st);
    if (status != MKQ_OK) return status;
    norm_kernel<<<1, 256, 0, st>>>(partials, count, norm_out);
    return launch_status();
}

extern "C" int mkq_clip_gradients(int64_t n, const void *const *grads_host, void *const *outs_host, const int64_t *counts_host,
                                  const int32_t *dtypes_host, float max_norm, float *norm_out, void *workspace, size_t workspace_bytes,
                                  void *stream)
{
    if (!norm_out || (n > 0 && !outs_host)) return MKQ_ERR_NULL;
    if (!aligned4(norm_out)) return MKQ_ERR_ALIGN;
    if (!(max_norm > 0.0f)) return MKQ_ERR_SCALE;
    int status = check_tensors(n, grads_host, outs_host, counts_host, dtypes_host, workspace, workspace_bytes);
    if (status == MKQ_OK) status = check_results_apart(n, grads_host, outs_host, counts_host, dtypes_host);
    if (status != MKQ_OK) return status;
    const hipStream_t st = as_stream(stream);
    double *partials = static_cast<double *>(workspace);
    int count;
    status = launch_partials(n, grads_host, counts_host, dtypes_host, partials, &count, st);
    if (status != MKQ_OK) return status;
    if (count == 0) {
        norm_kernel<<<1, 256, 0, st>>>(partials, 0, norm_out);
        return launch_status();
    }
    float *norm_at = norm_out;  // written by the first of the launches
    return for_each_list(n, grads_host, outs_host, counts_host, dtypes_host, [&](const TensorList &l, int workgroups) {
        clip_kernel<<<workgroups, 256, 0, st>>>(l, partials, count, max_norm, norm_at);
        norm_at = nullptr;
    });
}
