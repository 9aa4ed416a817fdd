// Products along rows: t = down_a x, u = s_a up_a dy; and the batch's rows put in the order of their adapters beside them.
#include "adapters.h"

namespace mkq {

// A workgroup of 256 has an adapter: each thread looks through neighbouring rows for those of the adapter and those of smaller ones.  That reads R M
// numbers, most of them from the caches, in the launch that is there anyway: 8192 rows take as long with 1000 adapters as with 32, with 10000 80 us
// more, with 100000 700.
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
    // Tiles of an XCD begin at steps of their own: rows a power of two apart would all ask the same memory channels at a time
    const int n = to - from, turn = n > 0 ? (int)((m0 / 128 * 4) % n) : 0;
    auto step = [&](int i) { return from + (i + turn < n ? i + turn : i + turn - n); };
    XRows xs;
    auto fetch_x = [&](int s) __attribute__((always_inline)) {
        auto each = [&](auto edge) __attribute__((always_inline)) {
#pragma unroll
            for (int i = 0; i < XRows::N; ++i) xs.v[i] = fetch16<X, false>(x[i], 0, s * STEP + XRows::piece_of() * (16 / X::BYTES), p.K, edge);
        };
        if ((s + 1) * STEP > p.K) each(std::true_type());
        else each(std::false_type());
    };
    // the first of x do not wait for the rows' adapters
    bool ahead = wave < n;
    if (ahead) fetch_x(step(wave));
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
        WRows ws[RT];
        auto fetch_w = [&](int s) __attribute__((always_inline)) {
            auto each = [&](auto edge) __attribute__((always_inline)) {
#pragma unroll
                for (int r = 0; r < RT; ++r)
#pragma unroll
                    for (int i = 0; i < WRows::N; ++i) {
                        const int at = (chunk * RT + r) * 16 + WRows::row_of(i);
                        ws[r].v[i] = fetch16<W, false>(w, (uint32_t)(at < p.a.rank ? at : p.a.rank - 1) * ((uint32_t)p.K * W::BYTES),
                                                       s * STEP + WRows::piece_of() * (16 / W::BYTES), p.K, edge);
                    }
            };
            if ((s + 1) * STEP > p.K) each(std::true_type());
            else each(std::false_type());
        };
        if (wave < n) {
            fetch_w(step(wave));
            if (!ahead) fetch_x(step(wave));
            ahead = false;
        }
        for (int i = wave; i < n; i += 4) {
            xs.put(lds_x);
#pragma unroll
            for (int r = 0; r < RT; ++r) ws[r].put(lds_w + r * WRows::BYTES);
            if (i + 4 < n) {
                fetch_x(step(i + 4));
                fetch_w(step(i + 4));
            }
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

void launch_shrink_kernel(const ShrinkParams &p, int x_dtype, int w_dtype, unsigned workgroups, hipStream_t st)
{
    with_elem(x_dtype, [&](auto x) {
        with_elem(w_dtype, [&](auto w) {
            using X = decltype(x);
            using W = decltype(w);
            const int tiles = rank_tiles(p.a.rank);
            if (tiles == 1) shrink_kernel<X, W, 1><<<workgroups, 256, 0, st>>>(p);
            else if (tiles == 2) shrink_kernel<X, W, 2><<<workgroups, 256, 0, st>>>(p);
            else shrink_kernel<X, W, 4><<<workgroups, 256, 0, st>>>(p);
        });
    });
}

}  // namespace mkq
