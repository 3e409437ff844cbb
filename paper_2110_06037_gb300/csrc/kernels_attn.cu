// Attention of new tokens over a paged cache (sn_attend in include/sn.h): the choice between the forms for few
// queries (attn_few.cuh) and for many (attn_prompt.cuh), how the work is cut, and the join of split items.
#include <algorithm>

#include "attn_few.cuh"
#include "attn_prompt.cuh"

namespace sn {
namespace k {

namespace {

constexpr float LOG2E = 1.4426950408889634f;

// ------------------------------------------------------------------- join
// The items are counted again, and WPR warps take a row of one: its parts in turn, a lane eight values, and the
// warps' sums in order.  used: rows of an item that there can be.  (Four warps where an item has many parts, one where
// there are many items: for 64 sequences of 8 heads, from cold caches, one warp a row takes 10.5 us, four take 15.5.
// 64 registers: two blocks of it then fit beside the three of the kernel before, and count the items while that one ends:
// that case takes 186 us; with 72, of which one fits, 197.)
template <typename T, int WPR>
__global__ void __launch_bounds__(128, 8) attend_join_kernel(const __grid_constant__ AttnP p, int used) {
    constexpr int W = 4;
    __shared__ float so[W][256], sm[W], sl[W];
    griddep_launch();
    griddep_wait();
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, sub = warp % WPR, d = p.c.head_dim;
    const int64_t id = (int64_t)blockIdx.x * (W / WPR) + warp / WPR, item = id / used;
    const int r = (int)(id - item * used);
    int b = -1;
    int64_t all = 0, before = 0, items = 0, mine = 0;  // units of all; before b's; items before b's; of this item among them
    for (int b0 = 0; b0 < p.q.batch; b0 += 32) {
        const Past s = past_of(p, min(b0 + lane, p.q.batch - 1));
        const int64_t n = b0 + lane < p.q.batch ? (int64_t)s.tiles * p.c.heads : 0;
        int64_t up = n, units = n * s.units;
#pragma unroll
        for (int o = 1; o < 32; o *= 2) {
            const int64_t v = __shfl_up_sync(0xffffffffu, up, o), u = __shfl_up_sync(0xffffffffu, units, o);
            if (lane >= o) up += v, units += u;
        }
        const uint32_t in = __ballot_sync(0xffffffffu, item < items + up);
        if (b < 0 && in) {
            const int k = __ffs(in) - 1;
            b = b0 + k;
            mine = item - items - __shfl_sync(0xffffffffu, up - n, k);
            before = all + __shfl_sync(0xffffffffu, units - n * s.units, k);
        }
        items += __shfl_sync(0xffffffffu, up, 31);
        all += __shfl_sync(0xffffffffu, units, 31);
    }
    if (b < 0) return;
    const Past past = past_of(p, b);
    const int head = (int)(mine / past.tiles), tile = (int)(mine - (int64_t)head * past.tiles);
    const int64_t row = (int64_t)tile * p.rows + r;
    if (row >= (int64_t)past.s.len * p.group) return;
    const int64_t t = past.s.first + row / p.group;
    const int qh = head * p.group + (int)(row % p.group);
    const int64_t n = share_of(p, all), u0 = before + mine * past.units, u1 = u0 + past.units;
    const int c0 = (int)(u0 / n), c1 = (int)((u1 - 1) / n);
    if (c0 == c1) return;  // one block had all of it
    auto part = [&](int c) { return part_of_slot(p, 2 * c + (c == c0 && u0 != c0 * n)); };
    float m = -INFINITY, l = 0.0f;
    for (int c = c0 + sub * 32 + lane; c <= c1; c += 32 * WPR) {
        const float *f = part(c) + (int64_t)p.rows * d + r;
        const float up = fmaxf(m, f[0]), base = up == -INFINITY ? 0.0f : up;
        l = fmaf(l, ex2(m - base), f[p.rows] * ex2(f[0] - base));
        m = up;
    }
    float top = m;
#pragma unroll
    for (int o = 16; o; o /= 2) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    if constexpr (WPR > 1) {
        if (lane == 0) sm[warp] = top;
        __syncthreads();
        top = fmaxf(fmaxf(sm[0], sm[1]), fmaxf(sm[2], sm[3]));
    }
    const float base = top == -INFINITY ? 0.0f : top;
    l *= ex2(m - base);
#pragma unroll
    for (int o = 16; o; o /= 2) l += __shfl_xor_sync(0xffffffffu, l, o);
    if constexpr (WPR > 1) {
        if (lane == 0) sl[warp] = l;
        __syncthreads();
        l = (sl[0] + sl[1]) + (sl[2] + sl[3]);
    }
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;
    float o[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) o[i] = 0.0f;
#pragma unroll 4
    for (int c = c0 + sub; c <= c1; c += WPR) {
        const float *f = part(c);
        const float w = ex2(f[(int64_t)p.rows * d + r] - base) * inv;  // (so that no sum is beyond the largest value)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int e = 4 * lane + 128 * i;
            if (e < d) {
                const float4 v = *reinterpret_cast<const float4 *>(f + r * d + e);
                o[4 * i] = fmaf(v.x, w, o[4 * i]), o[4 * i + 1] = fmaf(v.y, w, o[4 * i + 1]);
                o[4 * i + 2] = fmaf(v.z, w, o[4 * i + 2]), o[4 * i + 3] = fmaf(v.w, w, o[4 * i + 3]);
            }
        }
    }
    if constexpr (WPR > 1) {
#pragma unroll
        for (int i = 0; i < 2; ++i) *reinterpret_cast<float4 *>(&so[warp][4 * lane + 128 * i]) = make_float4(o[4 * i], o[4 * i + 1], o[4 * i + 2], o[4 * i + 3]);
        __syncthreads();
        if (warp) return;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int e = 4 * lane + 128 * (i / 4) + i % 4;
            o[i] = (so[0][e] + so[1][e]) + (so[2][e] + so[3][e]);
        }
    }
    T *y = static_cast<T *>(p.h.y) + t * p.h.ldy + (int64_t)qh * p.h.hy;
    bool infinite = false;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int e = 4 * lane + 128 * (i / 4) + i % 4;
        if (e >= d) continue;
        stf(y + e, l == 0.0f ? 0.0f : o[i]);
        infinite |= fabsf(o[i]) == INFINITY;
    }
    if (!infinite) return;
    // by rounding, where no part is: the largest value
#pragma unroll 1
    for (int i = 0; i < 8; ++i) {
        const int e = 4 * lane + 128 * (i / 4) + i % 4;
        if (e >= d) continue;
        const float now = ldf(y + e);
        if (fabsf(now) < INFINITY) continue;
        bool any = false;
        for (int c = c0; c <= c1; ++c) any |= !(fabsf(part(c)[r * d + e]) < INFINITY);
        if (!any && now == now) stf(y + e, copysignf(largest_of<T>(), now));
    }
}

// ------------------------------------------------------------------ choice

struct Plan {
    AttnP p;
    int64_t grid;
    int64_t items;  // at most
    int used;       // rows of an item at most
};
// How the sequences of more than lo and up to hi tokens are cut into items of `rows` rows and units of `keys` keys
// for a grid of up to `room` blocks at once: split, unless every item is short or there are items for `waves` waves.
// (A prompt's items have their diagonals in different places, which a split into equal numbers of units does not see.)
// A split costs the join's launch (2 us); `least` units of a block are worth as much.
Plan plan_of(const sn_kv_cache &c, const AttendArgs &a, int lo, int hi, int rows, int keys, int room, int least, int waves) {
    Plan r{};
    AttnP &p = r.p;
    p.q = a.q, p.c = c, p.t = a.t;
    p.q_heads = a.h.heads, p.group = a.h.heads / c.heads;
    p.max_ctx = (int32_t)a.max_context;
    p.scale = a.scale * LOG2E;
    p.h = a.h;
    p.lo = lo, p.hi = hi, p.rows = rows, p.keys = keys, p.least = least;
    p.err = device_error_word();
    // items at most: a sequence's last one may be cut off
    const int64_t seqs = lo ? std::min<int64_t>(a.q.batch, a.q.tokens / (lo + 1)) : a.q.batch;
    const int64_t most = std::min<int64_t>(a.q.max_len, hi);
    const int64_t items = c.heads * std::min(seqs * ((most * p.group + rows - 1) / rows), a.q.tokens * p.group / rows + seqs);
    const int64_t units = std::max<int64_t>(1, (a.max_context + keys - 1) / keys);
    r.grid = r.items = items;
    r.used = (int)std::min<int64_t>(rows, most * p.group);
    if (items && units > 2 * least && items < waves * (int64_t)room) {  // (without items: grid 0, nothing is launched)
        p.blocks = (int32_t)std::max<int64_t>(1, std::min<int64_t>(room, (items * units + least - 1) / least));
        r.grid = p.blocks;
    }
    return r;
}
size_t part_bytes(const Plan &r) { return (size_t)r.p.blocks * 2 * r.p.rows * (r.p.c.head_dim + 2) * 4; }

struct Few {
    few::Shape (*shape)(int, int64_t);
    cudaError_t (*launch)(const AttnP &, int64_t, cudaStream_t);
};
Few few_of(int dt, int cache) {
    if (cache == SN_QI8)
        return dt == SN_F16 ? Few{few_shape_f16_q8, attend_few_f16_q8} : dt == SN_BF16 ? Few{few_shape_bf16_q8, attend_few_bf16_q8}
                                                                                 : Few{few_shape_f32_q8, attend_few_f32_q8};
    return dt == SN_F32 ? Few{few_shape_f32, attend_few_f32} : dt == SN_F16 ? Few{few_shape_f16, attend_few_f16} : Few{few_shape_bf16, attend_few_bf16};
}

// the launches of a call: sequences of few tokens, the others; either may have nothing to do (grid 0)
struct Plans {
    Few few;
    Plan a, b;
};
Plans plans_of(const sn_kv_cache &c, int dt, const AttendArgs &a) {
    Plans r{few_of(dt, c.dtype), Plan{}, Plan{}};
    const int group = a.h.heads / c.heads, sms = num_sms();
    const bool tensor = dt != SN_F32 && c.dtype != SN_QI8;
    // sequences of up to 64 rows go to the form for few queries
    const int n = tensor ? std::max(1, 64 / group) : INT32_MAX;
    // Items of as many rows as there can be, for then the cache is read once; of 8 beside prompts, whose single tokens these
    // are, and where there is so little to do that more blocks matter more.  Both, us by 8 rows and by as many as there can be:
    // 5 sequences of up to 8 drafted tokens, 6 heads of 80 over 2 in fp32, 2500 keys, 28 and 42; 2 of 4 tokens, 16 heads of 128 over 2
    // in bf16, 3000 keys, 23 and 38; 4 of 8 tokens, 32 over 8, 600 keys, 20 and 40; a prompt of 60 tokens over codes 6.7 and
    // 13.8; beside a prompt of 2048 tokens, 32 single tokens with 3000 keys each 143 and 242, 3 sequences of 4 tokens 123 and
    // 149, but one of 16 tokens with 60000 keys 339 and 286 (the rule sees the longest sequence alone).  Where the bound
    // chooses the other: 16 tokens with 60000 keys, 8 heads over 2, 84 and 80, with 20000 40 and 51; 8 sequences of 5 tokens over
    // codes, 32 heads over 8, 4000 keys, 69 and 94.
    int64_t rows = std::min<int64_t>(a.q.max_len, n) * group;
    const int64_t units = std::max<int64_t>(1, a.max_context / few::UNIT);
    if ((tensor && a.q.max_len > n) || a.q.tokens * group / 8 * c.heads * units < 16 * sms) rows = std::min<int64_t>(rows, std::max(group, 8));
    const few::Shape s = r.few.shape(c.head_dim, rows);
    r.a = plan_of(c, a, 0, n, s.rows, few::UNIT, s.blocks * sms, dt == SN_F32 && c.dtype != SN_QI8 ? 1 : 4, 16);
    if (!a.q.offsets && a.q.max_len > n) r.a.grid = 0;  // (its scratch counts all the same: that is asked for without offsets)
    if (a.q.max_len > n) {
        // two tiles of rows a block, unless one each makes more blocks busy (heads beyond 128 values: one)
        const int keys = c.head_dim > 128 ? 64 : 128;
        r.b = plan_of(c, a, n, INT32_MAX, 256, keys, sms, 4, 1);
        if (c.head_dim > 128 || r.b.p.blocks) r.b = plan_of(c, a, n, INT32_MAX, 128, keys, sms, 4, 1);
    }
    return r;
}

template <typename T>
cudaError_t join(const Plan &r, cudaStream_t st) {
    if (!r.p.blocks) return cudaSuccess;
    const int64_t rows = r.items * r.used;
    if (r.p.blocks > 8 * r.items) return launch_pdl(attend_join_kernel<T, 4>, dim3((unsigned)rows), dim3(128), 0, st, r.p, r.used);
    return launch_pdl(attend_join_kernel<T, 1>, dim3((unsigned)((rows + 3) / 4)), dim3(128), 0, st, r.p, r.used);
}

}  // namespace

size_t attend_workspace(const sn_kv_cache &c, int dt, const AttendArgs &a) {
    const Plans r = plans_of(c, dt, a);
    return std::max(part_bytes(r.a), part_bytes(r.b));
}

cudaError_t attend(const sn_kv_cache &c, int dt, const AttendArgs &a, void *work, cudaStream_t st) {
    Plans r = plans_of(c, dt, a);
    r.a.p.part = r.b.p.part = static_cast<float *>(work);  // (one after the other)
    SN_DT_SWITCH(dt, T, {
        if (r.a.grid) {
            if (const cudaError_t e = r.few.launch(r.a.p, r.a.grid, st)) return e;
            if (const cudaError_t e = join<T>(r.a, st)) return e;
        }
        if (r.b.grid) {
            if (const cudaError_t e = (dt == SN_F16 ? attend_prompt_f16 : attend_prompt_bf16)(r.b.p, r.b.grid, st)) return e;
            if (const cudaError_t e = join<T>(r.b, st)) return e;
        }
    })
    return cudaSuccess;
}

}  // namespace k
}  // namespace sn
