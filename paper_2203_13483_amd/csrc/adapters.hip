// Low-rank adapters of many requests beside a shared projection, and their gradients.  Row m has the adapter a = adapter[m]:
//
//     t[m] = down_a x[m]        out[m] = base[m] + s_a up_a^T t[m]                  (down_a [rank, K], up_a [rank, N])
//     u[m] = s_a up_a dy[m]     dx[m]  = base[m] + down_a^T u[m]
//     d_down_a = sum_m u[m] x[m]^T,   d_up_a = s_a sum_m t[m] dy[m]^T
//
// Both matrices of an adapter have their long side in rows, so three kernels do all of it: `shrink` (t, u: products along rows),
// `expand` (out, dx: sums of the adapter's rows) and `outer` (sums of the batch's rows).  Bound by the bytes of x, dy, base and out; products
// are the matrix unit's.  Measured, 8192 bfloat16 rows of 1024 and 4096, rank 16, us (medians of a trace): shrink of x 9.3, of dy 18 (3.7 TB/s), expand to out with its base 31 (4.4
// TB/s), to dx 9.5, outer of both (x in 8 bits) 23, its join 5.7.  All binary32: shrink of dy 55, expand to dx 18, outer 38, its join 6.
//
// Operands enter the products exactly: binary16 and bfloat16 as they are where both sides are the same, otherwise a number is the sum of
// one to three bfloat16 parts (binary32 three, binary16 two), each the nearest to what is left.  Of a product only that of a second part with a third, and
// of thirds, are left out: 2^-24 of it at most, of either sign.  Sums are binary32.  A tile of rows may hold any adapters: it is gone through once for each of them, results are taken for the rows
// that have it, so a request's infinities and NaN stay in its rows.
#include "adapters.h"

namespace mkq {

constexpr int64_t ADAPTERS_MOST = 0x3FFFFF, SIDES_MOST = 0x7FFFFF00;
constexpr int RANK_MOST = 256;
constexpr int64_t STRIDE_MOST = (int64_t)1 << 25;  // elements between rows: 16 of them are addressed in 32 bits
constexpr int64_t PLANNED_MOST = (int64_t)1 << 40;  // adapters times rows, which the plan reads: about 1e12 of them a second
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
// Workgroups that share the places of a row: about 512 of them in all, four steps each at least
static int splits_of(const AdapterShape &d, int64_t side)
{
    const int64_t steps = ceil_div(side, 64), groups = ceil_div(d.M, 16) * slots_of(d) * ceil_div(d.rank, 16 * rank_tiles(d.rank));
    int64_t n = groups == 0 || groups >= 512 ? 1 : 512 / groups;
    if (n > ceil_div(steps, 4)) n = ceil_div(steps, 4);
    if (n > 16) n = 16;
    return (int)ceil_div(steps, ceil_div(steps, n));
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
// Workgroups of the launches; a call whose grids do not fit is refused before the first of them
static int64_t shrink_workgroups(const AdapterShape &d, int splits) { return ceil_div(d.M, 16) * slots_of(d) * splits * ceil_div(d.rank, 16 * rank_tiles(d.rank)); }
static int64_t expand_workgroups(const AdapterShape &d, int64_t side) { return ColumnTask::workgroups(ceil_div(d.M, 16) * slots_of(d), ceil_div(side, 128)); }
static int64_t outer_workgroups(const AdapterShape &d, int64_t tasks, int64_t blocks) { return ColumnTask::workgroups(tasks * ceil_div(d.rank, 16 * outer_tiles(d.rank)), blocks); }
static int64_t join_workgroups(const AdapterShape &d, int64_t sides) { return d.R * ceil_div((int64_t)d.rank * sides, 256); }

static int launch_shrink(const AdapterShape &d, const ShrinkParams &p, int x_dtype, int w_dtype, hipStream_t st)
{
    const int64_t workgroups = (p.x ? shrink_workgroups(d, p.a.splits) : 0) + p.plans;
    launch_shrink_kernel(p, x_dtype, w_dtype, (unsigned)workgroups, st);
    return launch_status();
}

static int launch_expand(const AdapterShape &d, ExpandParams p, int w_dtype, int out_dtype, hipStream_t st)
{
    p.column_blocks = (int)ceil_div(p.N, 128);
    p.slots = slots_of(d);
    p.row_groups = (int)ceil_div(d.M, 16);
    const int64_t workgroups = expand_workgroups(d, p.N);
    launch_expand_kernel(p, w_dtype, out_dtype, (unsigned)workgroups, st);
    return launch_status();
}

// Rows of a piece: about 3000 waves in all.  (8192 rows, 1024 and 4096 columns, rank 16, us of the call with 1000, 1500, 3000 and 6000 waves: x in 8 bits 65,
// 61, 58, 62; bfloat16 50, 53, 55, 59; 437 rows of 312 and 1200 all 30.)
static int piece_rows(const AdapterShape &d)
{
    const int64_t columns = ceil_div(d.K, 128) + ceil_div(d.N, 128), n = ceil_div(ceil_div(d.M * columns, 3000), 64) * 64;
    return (int)(n < 64 ? 64 : n > 2048 ? 2048 : n);
}

static int pitch_of(int rank) { return (rank + 7) / 8 * 8; }

// Few rows of short sides go in one launch: at most 64 rows, one tile of the rank, and what every workgroup reads again is 64 KiB at most (of 2 bytes)
static bool few_rows(const AdapterShape &d) { return d.M <= 64 && d.rank <= 16 && d.K <= 1024; }

struct AdapterWorkspace {
    size_t t, u, order, starts, tasks, down, up, total;
    int splits, piece;
    int64_t tasks_most;
};
static AdapterWorkspace forward_workspace(const AdapterShape &d)
{
    AdapterWorkspace w = {};
    w.splits = few_rows(d) ? 1 : splits_of(d, d.K);
    if (!few_rows(d)) w.total = (size_t)w.splits * d.M * pitch_of(d.rank) * sizeof(float);
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

// Memory from an address on
struct Extent {
    uintptr_t from, to;
    Extent(const void *p, int64_t rows, int64_t ld, int64_t cols, int dtype)
        : from(reinterpret_cast<uintptr_t>(p)),
          to(p && rows > 0 ? from + (uintptr_t)(((unsigned __int128)(rows - 1) * (uint64_t)ld + (uint64_t)cols) * (uint64_t)(is_float_dtype(dtype) ? dtype_bytes(dtype) : 1)) : from) {}
    bool apart(const Extent &o) const { return from == to || o.from == o.to || to <= o.from || o.to <= from; }
};

static int launch_outer(const AdapterShape &d, OuterParams p, int x_dtype, int dy_dtype, hipStream_t st)
{
    p.rank_chunks = (int)ceil_div(d.rank, 16 * outer_tiles(d.rank));
    const int64_t workgroups = outer_workgroups(d, p.plan.tasks_most, p.side[0].column_blocks + p.side[1].column_blocks);
    const int64_t joins = join_workgroups(d, (p.side[0].column_blocks ? d.K : 0) + (p.side[1].column_blocks ? d.N : 0));
    launch_outer_kernel(p, x_dtype, dy_dtype, (unsigned)workgroups, st);
    if (d.M > p.plan.piece) launch_outer_join_kernel(p, (unsigned)joins, st);
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
    // few rows' workgroups read whole rows of x beside others' writes
    if (!apart_or_beside(x, x_dtype, ldx, K, out, out_dtype, ld_out, N, M)) return MKQ_ERR_UNSUPPORTED;
    if (hidden && (!apart(x, x_dtype, ldx, K, hidden, MKQ_F32, rank, rank, M) || !apart(out, out_dtype, ld_out, N, hidden, MKQ_F32, rank, rank, M)))
        return MKQ_ERR_UNSUPPORTED;
    const AdapterWorkspace w = forward_workspace(d);
    if (!grid_ok(shrink_workgroups(d, w.splits), 256) || !grid_ok(expand_workgroups(d, N), 256)) return MKQ_ERR_UNSUPPORTED;
    if (w.total > 0 && (!workspace || workspace_bytes < w.total)) return MKQ_ERR_WORKSPACE;
    if (!aligned16(workspace)) return MKQ_ERR_ALIGN;
    const hipStream_t st = as_stream(stream);
    const AdapterParams a = {adapter, scales, M, (int)R, rank, pitch_of(rank), w.splits};
    float *t = static_cast<float *>(workspace);
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
    if (few_rows(d)) {  // (no workspace)
        e.column_blocks = (int)ceil_div(N, 128);
        e.slots = slots_of(d);
        launch_few_kernel(shrink_params(d, a, x, ldx, down, K, false, nullptr, hidden), e, x_dtype, w_dtype, out_dtype,
                          (unsigned)(ceil_div(M, 16) * e.slots * ceil_div(e.column_blocks, 4)), st);
        return launch_status();
    }
    status = launch_shrink(d, shrink_params(d, a, x, ldx, down, K, false, t, w.splits == 1 ? hidden : nullptr), x_dtype, w_dtype, st);
    return status == MKQ_OK ? launch_expand(d, e, w_dtype, out_dtype, st) : status;
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
    if ((d_down || d_up) && M * R > PLANNED_MOST) return MKQ_ERR_UNSUPPORTED;  // (below 2^31 and 2^22)
    const AdapterWorkspace w = gradient_workspace(d);
    if (!grid_ok(shrink_workgroups(d, w.splits) + R, 256) || (dx && M > 0 && !grid_ok(expand_workgroups(d, K), 256)) ||
        !grid_ok(outer_workgroups(d, w.tasks_most, ceil_div(K, 128) + ceil_div(N, 128)), 256) || !grid_ok(join_workgroups(d, K + N), 256))
        return MKQ_ERR_UNSUPPORTED;
    if (!workspace || workspace_bytes < w.total) return MKQ_ERR_WORKSPACE;
    if (!aligned16(workspace)) return MKQ_ERR_ALIGN;
    {  // the rows, hidden values and other results are read or written beside the gradients, and hidden values behind dx
        const int64_t groups = d_down && kept ? ceil_div(K, x_group) : 0;
        const Extent to_down(d_down, R * rank, K, K, grad_dtype), to_up(d_up, R * rank, N, N, grad_dtype), to_dx(dx, M, ld_dx, K, dx_dtype);
        const Extent read[] = {{dy, M, ld_dy, N, dy_dtype}, {d_down ? x : nullptr, M, pitch, K, x_dtype}, {d_down && kept ? x_steps : nullptr, M, groups, groups, MKQ_F32},
                               {d_up ? hidden : nullptr, M, rank, rank, MKQ_F32}};
        bool fine = to_down.apart(to_up) && to_down.apart(to_dx) && to_up.apart(to_dx) && to_dx.apart(read[3]);
        for (const Extent &r : read) fine = fine && to_down.apart(r) && to_up.apart(r);
        if (!fine) return MKQ_ERR_UNSUPPORTED;
    }
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
