// Attention of new tokens over a paged cache (sn_attend in include/sn.h): the form for every type by
// multiply-adds in fp32, the join of split items, and the choice between the forms.
//
// A unit is 64 keys: scores of ROWS queries against them, their running maximum and sum, and the weighted
// values, all in fp32; keys and values lie in shared memory as fp32 (codes times their scales).
#include <algorithm>

#include "attn_few.cuh"
#include "attn_prompt.cuh"

namespace sn {
namespace k {

namespace {

constexpr int KEYS = 64;
constexpr float LOG2E = 1.4426950408889634f;

// four neighbours of a row of the cache
template <typename C>
__device__ __forceinline__ float4 row4(const C *p) {
    if constexpr (sizeof(C) == 4) {
        return *reinterpret_cast<const float4 *>(p);
    } else if constexpr (sizeof(C) == 2) {
        alignas(8) C t[4];
        *reinterpret_cast<uint2 *>(t) = *reinterpret_cast<const uint2 *>(p);
        return make_float4(ldf(t), ldf(t + 1), ldf(t + 2), ldf(t + 3));
    } else {
        const char4 c = *reinterpret_cast<const char4 *>(p);
        return make_float4((float)c.x, (float)c.y, (float)c.z, (float)c.w);
    }
}

// thread (tr, tc) of 16 x 16 has rows tr + 16 i, keys tc + 16 j and values 4 tc + 64 j of a row
template <typename T, typename C, int RPT, int DV>
__global__ void __launch_bounds__(256) attend_kernel(const __grid_constant__ AttnP p) {
    constexpr int ROWS = 16 * RPT;
    extern __shared__ __align__(16) float sm[];
    __shared__ int64_t sh[4];
    const int d = p.c.head_dim, ld = d + 4, tid = threadIdx.x, tr = tid / 16, tc = tid % 16;
    float *qs = sm, *ks = qs + ROWS * ld, *vs = ks + KEYS * ld, *ps = vs + KEYS * d;
    __shared__ uint8_t there[KEYS];
    griddep_launch();
    griddep_wait();
    Pieces pieces;
    pieces.start(p, sh);
    for (Piece w; pieces.next(p, w);) {
        const Seq &s = w.past.s;
        const int64_t row0 = (int64_t)w.tile * ROWS, all = (int64_t)s.len * p.group;
        __syncthreads();
        for (int i = tid; i < ROWS * d / 4; i += 256) {
            const int r = i / (d / 4), e = i % (d / 4) * 4;
            float4 f = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
            if (row0 + r < all) {
                const T *x = static_cast<const T *>(p.h.x) + (s.first + (row0 + r) / p.group) * p.h.ldx +
                             ((int64_t)w.head * p.group + (row0 + r) % p.group) * p.h.hx + e;
                f = make_float4(ldf(x), ldf(x + 1), ldf(x + 2), ldf(x + 3));
            }
            *reinterpret_cast<float4 *>(qs + r * ld + e) = f;
        }
        int last[RPT];
        float m[RPT], l[RPT], o[RPT][4 * DV];
#pragma unroll
        for (int i = 0; i < RPT; ++i) {
            const int64_t row = row0 + tr + 16 * i;
            last[i] = row < all ? last_key(p, w.past, row) : -1;
            m[i] = -INFINITY, l[i] = 0.0f;
#pragma unroll
            for (int j = 0; j < 4 * DV; ++j) o[i][j] = 0.0f;
        }
        const int end = last_key(p, w.past, min(row0 + ROWS, all) - 1);
        const int u1 = min(w.u1, end / KEYS + 1);
        for (int u = w.u0; u < u1; ++u) {
            __syncthreads();
            for (int i = tid; i < KEYS * d / 4; i += 256) {
                const int r = i / (d / 4), e = i % (d / 4) * 4, key = u * KEYS + r;
                const int64_t place = key < w.past.ctx ? place_in(p.c, p.t, s.slot, key) : -1;
                float4 f = make_float4(0.0f, 0.0f, 0.0f, 0.0f), g = f;
                if (place >= 0) {
                    const int64_t row = row_in(p.c, place, w.head), at = row * d + e;
                    f = row4(static_cast<const C *>(p.c.k) + at), g = row4(static_cast<const C *>(p.c.v) + at);
                    if constexpr (sizeof(C) == 1) {
                        const float a = p.c.k_scale[row], b = p.c.v_scale[row];
                        f.x *= a, f.y *= a, f.z *= a, f.w *= a;
                        g.x *= b, g.y *= b, g.z *= b, g.w *= b;
                    }
                }
                *reinterpret_cast<float4 *>(ks + r * ld + e) = f;
                *reinterpret_cast<float4 *>(vs + r * d + e) = g;
                if (e == 0) there[r] = place >= 0;
            }
            __syncthreads();
            float a[RPT][4];
#pragma unroll
            for (int i = 0; i < RPT; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) a[i][j] = 0.0f;
#pragma unroll 2
            for (int e = 0; e < d; e += 4) {
                float4 x[RPT], y[4];
#pragma unroll
                for (int i = 0; i < RPT; ++i) x[i] = *reinterpret_cast<const float4 *>(qs + (tr + 16 * i) * ld + e);
#pragma unroll
                for (int j = 0; j < 4; ++j) y[j] = *reinterpret_cast<const float4 *>(ks + (tc + 16 * j) * ld + e);
#pragma unroll
                for (int i = 0; i < RPT; ++i)
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        a[i][j] = fmaf(x[i].w, y[j].w, fmaf(x[i].z, y[j].z, fmaf(x[i].y, y[j].y, fmaf(x[i].x, y[j].x, a[i][j]))));
            }
#pragma unroll
            for (int i = 0; i < RPT; ++i) {
                float up = m[i];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int k = tc + 16 * j;
                    a[i][j] = there[k] && u * KEYS + k <= last[i] ? a[i][j] * p.scale : -INFINITY;
                    up = fmaxf(up, a[i][j]);
                }
#pragma unroll
                for (int k = 8; k; k /= 2) up = fmaxf(up, __shfl_xor_sync(0xffffffffu, up, k));
                const float base = up == -INFINITY ? 0.0f : up, old = exp2f(m[i] - base);
                m[i] = up;
                float sum = 0.0f;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float e = exp2f(a[i][j] - base);
                    sum += e;
                    ps[(tr + 16 * i) * (KEYS + 4) + tc + 16 * j] = e;
                }
#pragma unroll
                for (int k = 8; k; k /= 2) sum += __shfl_xor_sync(0xffffffffu, sum, k);
                l[i] = fmaf(l[i], old, sum);
#pragma unroll
                for (int j = 0; j < 4 * DV; ++j) o[i][j] *= old;
            }
            __syncwarp();  // (a row's weights are written and read by the same half of a warp)
            for (int k = 0; k < KEYS; k += 4) {
                float4 x[RPT];
#pragma unroll
                for (int i = 0; i < RPT; ++i) x[i] = *reinterpret_cast<const float4 *>(ps + (tr + 16 * i) * (KEYS + 4) + k);
#pragma unroll
                for (int j = 0; j < DV; ++j) {
                    const int e = 4 * tc + 64 * j;
                    if (e >= d) break;
                    float4 y[4];
#pragma unroll
                    for (int n = 0; n < 4; ++n) y[n] = *reinterpret_cast<const float4 *>(vs + (k + n) * d + e);
#pragma unroll
                    for (int i = 0; i < RPT; ++i) {
                        float *f = o[i] + 4 * j;
                        f[0] = fmaf(x[i].w, y[3].x, fmaf(x[i].z, y[2].x, fmaf(x[i].y, y[1].x, fmaf(x[i].x, y[0].x, f[0]))));
                        f[1] = fmaf(x[i].w, y[3].y, fmaf(x[i].z, y[2].y, fmaf(x[i].y, y[1].y, fmaf(x[i].x, y[0].y, f[1]))));
                        f[2] = fmaf(x[i].w, y[3].z, fmaf(x[i].z, y[2].z, fmaf(x[i].y, y[1].z, fmaf(x[i].x, y[0].z, f[2]))));
                        f[3] = fmaf(x[i].w, y[3].w, fmaf(x[i].z, y[2].w, fmaf(x[i].y, y[1].w, fmaf(x[i].x, y[0].w, f[3]))));
                    }
                }
            }
        }
        uint32_t again = 0;  // rows of this thread's that are not finite
#pragma unroll
        for (int i = 0; i < RPT; ++i) {
            const int64_t row = row0 + tr + 16 * i;
            if (w.slot >= 0) {
                float *part = part_of_slot(p, w.slot);
                const int r = tr + 16 * i;
#pragma unroll
                for (int j = 0; j < DV; ++j) {
                    const int e = 4 * tc + 64 * j;
                    if (e < d) *reinterpret_cast<float4 *>(part + r * d + e) = make_float4(o[i][4 * j], o[i][4 * j + 1], o[i][4 * j + 2], o[i][4 * j + 3]);
                }
                if (tc == 0) part[ROWS * d + r] = m[i], part[ROWS * d + ROWS + r] = l[i];
            } else if (row < all) {
                T *y = static_cast<T *>(p.h.y) + (s.first + row / p.group) * p.h.ldy + ((int64_t)w.head * p.group + row % p.group) * p.h.hy;
                const float f = l[i] == 0.0f ? 0.0f : 1.0f / l[i];
#pragma unroll
                for (int j = 0; j < DV; ++j)
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const int e = 4 * tc + 64 * j + k;
                        const float v = l[i] == 0.0f ? 0.0f : o[i][4 * j + k] * f;
                        if (e < d) stf(y + e, v);
                        if (!(fabsf(v) < INFINITY)) again |= 1u << i;
                    }
            }
        }
        if (w.slot < 0 && s.len > 1) {
#pragma unroll
            for (int i = 0; i < RPT; ++i) {
                const uint32_t bad = __ballot_sync(0xffffffffu, again >> i & 1u);
                for (int half = 0; half < 2; ++half)
                    if (bad >> (16 * half) & 0xffffu) attend_again<T>(p, w.b, w.head, row0 + tid / 32 * 2 + half + 16 * i);
            }
        }
    }
}

// ------------------------------------------------------------------- join
// The items are counted again, and WPR warps take a row of one: its parts in turn, a lane eight values, and the
// warps' sums in order.  used: rows of an item that there can be.  (Four warps where an item has many parts, one where
// there are many items: 64 sequences of 8 heads by one warp a row 5 us, by four 9.)
template <typename T, int WPR>
__global__ void __launch_bounds__(128) attend_join_kernel(const __grid_constant__ AttnP p, int used) {
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
    float m = -INFINITY;
    for (int c = c0 + sub * 32 + lane; c <= c1; c += 32 * WPR) m = fmaxf(m, part(c)[(int64_t)p.rows * d + r]);
#pragma unroll
    for (int o = 16; o; o /= 2) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
    if constexpr (WPR > 1) {
        if (lane == 0) sm[warp] = m;
        __syncthreads();
        m = fmaxf(fmaxf(sm[0], sm[1]), fmaxf(sm[2], sm[3]));
    }
    const float base = m == -INFINITY ? 0.0f : m;
    float o[8], l = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) o[i] = 0.0f;
#pragma unroll 4
    for (int c = c0 + sub; c <= c1; c += WPR) {
        const float *f = part(c);
        const float w = exp2f(f[(int64_t)p.rows * d + r] - base);
        l = fmaf(f[(int64_t)p.rows * d + p.rows + r], w, l);
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
        if (lane == 0) sl[warp] = l;
        __syncthreads();
        if (warp) return;
        l = (sl[0] + sl[1]) + (sl[2] + sl[3]);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int e = 4 * lane + 128 * (i / 4) + i % 4;
            o[i] = (so[0][e] + so[1][e]) + (so[2][e] + so[3][e]);
        }
    }
    const float f = l == 0.0f ? 0.0f : 1.0f / l;
    T *y = static_cast<T *>(p.h.y) + t * p.h.ldy + (int64_t)qh * p.h.hy;
    bool bad = false;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int e = 4 * lane + 128 * (i / 4) + i % 4;
        if (e >= d) continue;
        const float v = l == 0.0f ? 0.0f : o[i] * f;
        stf(y + e, v);
        bad |= !(fabsf(v) < INFINITY);
    }
    if (past.s.len > 1 && __any_sync(0xffffffffu, bad)) attend_again<T>(p, b, head, row);
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
    if (units > 2 * least && items < waves * (int64_t)room) {
        p.blocks = (int32_t)std::max<int64_t>(1, std::min<int64_t>(room, (items * units + least - 1) / least));
        r.grid = p.blocks;
    }
    return r;
}
size_t part_bytes(const Plan &r) { return (size_t)r.p.blocks * 2 * r.p.rows * (r.p.c.head_dim + 2) * 4; }

// sequences of up to this many tokens go to the form for few queries
int few_tokens(int group) { return std::max(1, 64 / group); }

struct Few {
    few::Shape (*shape)(int, int64_t);
    cudaError_t (*launch)(const AttnP &, int64_t, cudaStream_t);
};
Few few_of(int dt, int cache) {
    if (cache == SN_QI8)
        return dt == SN_F16 ? Few{few_shape_f16_q8, attend_few_f16_q8} : dt == SN_BF16 ? Few{few_shape_bf16_q8, attend_few_bf16_q8}
                                                                                 : Few{few_shape_f32_q8, attend_few_f32_q8};
    if (dt == SN_F32) return Few{nullptr, nullptr};
    return dt == SN_F16 ? Few{few_shape_f16, attend_few_f16} : Few{few_shape_bf16, attend_few_bf16};
}

// the launches of a call: sequences of few tokens, the others; either may have nothing to do (grid 0)
struct Plans {
    Few few;
    bool tensor;  // b by attn_prompt.cuh
    Plan a, b;
};
Plans plans_of(const sn_kv_cache &c, int dt, const AttendArgs &a) {
    Plans r{few_of(dt, c.dtype), dt != SN_F32 && c.dtype != SN_QI8, Plan{}, Plan{}};
    const int group = a.h.heads / c.heads, n = !r.few.launch ? 0 : r.tensor ? few_tokens(group) : INT32_MAX;
    if (n) {
        const few::Shape s = r.few.shape(c.head_dim, std::min<int64_t>(a.q.max_len, n) * group);
        r.a = plan_of(c, a, 0, n, s.rows, few::UNIT, s.blocks * num_sms(), 4, 16);
        if (!a.q.offsets && a.q.max_len > n) r.a.grid = 0;
    }
    if (a.q.max_len > n && r.tensor) {
        // two tiles of rows a block, unless one each makes more blocks busy (heads beyond 128 values: one)
        const int keys = c.head_dim > 128 ? 64 : 128, sms = num_sms();
        r.b = plan_of(c, a, n, INT32_MAX, 256, keys, sms, 4, 1);
        if (c.head_dim > 128 || r.b.p.blocks) r.b = plan_of(c, a, n, INT32_MAX, 128, keys, sms, 4, 1);
    } else if (a.q.max_len > n) {
        r.b = plan_of(c, a, n, INT32_MAX, a.q.max_len * group <= 16 ? 16 : 64, KEYS, 2 * num_sms(), 2, 1);
    }
    return r;
}

template <typename T, typename C, int RPT, int DV>
cudaError_t launch_simple(const Plan &r, cudaStream_t st) {
    const int d = r.p.c.head_dim;
    const size_t bytes = 4 * (size_t)(16 * RPT * (d + 4) + KEYS * (d + 4) + KEYS * d + 16 * RPT * (KEYS + 4));
    static PerDevice set;
    if (const cudaError_t e = allow_smem(set, attend_kernel<T, C, RPT, DV>, 224 * 1024)) return e;
    return launch_pdl(attend_kernel<T, C, RPT, DV>, dim3((unsigned)r.grid), dim3(256), bytes, st, r.p);
}
template <typename T, typename C>
cudaError_t simple_of(const Plan &r, cudaStream_t st) {
    const int dv = (r.p.c.head_dim + 63) / 64;
    if (r.p.rows == 16) {
        if (dv == 1) return launch_simple<T, C, 1, 1>(r, st);
        if (dv == 2) return launch_simple<T, C, 1, 2>(r, st);
        return launch_simple<T, C, 1, 4>(r, st);
    }
    if (dv == 1) return launch_simple<T, C, 4, 1>(r, st);
    if (dv == 2) return launch_simple<T, C, 4, 2>(r, st);
    return launch_simple<T, C, 4, 4>(r, st);
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
            if (const cudaError_t e = r.tensor ? (dt == SN_F16 ? attend_prompt_f16 : attend_prompt_bf16)(r.b.p, r.b.grid, st) : simple_of<float, float>(r.b, st))
                return e;
            if (const cudaError_t e = join<T>(r.b, st)) return e;
        }
    })
    return cudaSuccess;
}

}  // namespace k
}  // namespace sn
