// Pieces that the kernels of the attention layer's operators share.
#pragma once

#include "ssm_common.cuh"
#include "tc_common.cuh"

namespace sn {
namespace k {

// the sequence that token t lies in, -1: none (of empty sequences the one behind them)
__device__ __forceinline__ int sequence_at(const SeqArgs &q, int64_t t) {
    if (!q.offsets) {
        const int64_t b = q.max_len > 0 ? t / q.max_len : q.batch;
        return b < q.batch ? (int)b : -1;
    }
    int lo = 0, hi = q.batch;  // the last b with offsets[b] <= t is lo - 1 or in [lo, hi)
    while (lo < hi) {
        const int mid = (lo + hi) / 2;
        if (q.offsets[mid] <= t) lo = mid + 1;
        else hi = mid;
    }
    return lo > 0 && t < q.offsets[lo] ? lo - 1 : -1;
}

// where position `at` of slot's sequence lies: its page times the page's length plus its place there, -1: nowhere
__device__ __forceinline__ int64_t place_in(const sn_kv_cache &c, const TableArgs &t, int slot, int64_t at) {
    if (slot < 0 || at < 0) return -1;
    const int shift = 31 - __clz(c.page);
    const int64_t n = at >> shift;
    if (n >= t.width) return -1;
    const int page = t.at[(int64_t)slot * t.width + n];
    if (page < 0 || page >= c.pages) return -1;
    return ((int64_t)page << shift) + (at & (c.page - 1));
}
// the cache's row of a head at such a place
__device__ __forceinline__ int64_t row_in(const sn_kv_cache &c, int64_t place, int head) {
    const int shift = 31 - __clz(c.page);
    return (((place >> shift) * c.heads + head) << shift) + (place & (c.page - 1));
}

// ------------------------------------------------------------- attention
// What is to be done is cut into items, the rows of one sequence's queries that read one head of the
// cache, ROWS at a time (row r: token r / group, head r % group of those that share it); an item goes
// through its keys in units of KEYS.  Either a block takes an item (whole), or the units of all items
// lie end to end and each block takes as many of them (split): an item cut that way leaves its parts'
// sums in scratch, two slots a block, and attend_join_kernel joins them in the blocks' order.
struct AttnP {
    SeqArgs q;
    sn_kv_cache c;
    TableArgs t;
    int32_t q_heads, group;
    int32_t max_ctx;
    float scale;           // times log2 e
    HeadsArgs h;
    int32_t lo, hi;        // takes the sequences of more than lo and up to hi tokens
    int32_t rows, keys;    // of an item, of a unit
    int32_t blocks, least; // split: blocks of the grid, units each takes at least; blocks 0: whole
    float *part;           // [blocks][2]: [rows][head_dim] sums of weighted values, [rows] largest scores, [rows] sums of weights
    int *err;
};

struct Past {  // a sequence, the keys it has, its items a head and units an item
    Seq s;
    int32_t ctx, tiles, units;
};
__device__ __forceinline__ Past past_of(const AttnP &p, int b) {
    Past r;
    r.s = sequence(p.q, b);
    if (r.s.len > p.q.max_len) r.s.len = (int32_t)p.q.max_len;
    int64_t ctx = r.s.pos + r.s.len;
    const int64_t room = (int64_t)p.t.width * p.c.page;
    ctx = ctx < p.max_ctx ? ctx : p.max_ctx;
    ctx = ctx < room ? ctx : room;
    r.ctx = r.s.slot >= 0 ? (int32_t)ctx : 0;
    const bool mine = r.s.len > p.lo && r.s.len <= p.hi;
    r.tiles = mine ? (int32_t)(((int64_t)r.s.len * p.group + p.rows - 1) / p.rows) : 0;
    r.units = max(1, (r.ctx - 1) / p.keys + 1);  // (a sum would leave 32 bits)
    return r;
}
// units of a sequence (whole: its items)
__device__ __forceinline__ int64_t units_of(const AttnP &p, const Past &r) {
    return (int64_t)r.tiles * p.c.heads * (p.blocks ? r.units : 1);
}

// by one whole warp: the units of all sequences, and the sequence in which unit `at` lies (at >= 0; b < 0: none) and
// those before it
struct Span {
    int64_t all, before;
    int b;
};
__device__ __forceinline__ Span span_of(const AttnP &p, int64_t at) {
    const int lane = threadIdx.x % 32;
    Span r{0, 0, -1};
    for (int b0 = 0; b0 < p.q.batch; b0 += 32) {
        const int64_t n = b0 + lane < p.q.batch ? units_of(p, past_of(p, b0 + lane)) : 0;
        int64_t up = n;
#pragma unroll
        for (int o = 1; o < 32; o *= 2) {
            const int64_t v = __shfl_up_sync(0xffffffffu, up, o);
            if (lane >= o) up += v;
        }
        if (at >= 0 && r.b < 0) {
            const uint32_t in = __ballot_sync(0xffffffffu, at < r.all + up);
            if (in) {
                const int k = __ffs(in) - 1;
                r.b = b0 + k;
                r.before = r.all + __shfl_sync(0xffffffffu, up - n, k);
            }
        }
        r.all += __shfl_sync(0xffffffffu, up, 31);
    }
    return r;
}
// units that each block of a split takes
__device__ __forceinline__ int64_t share_of(const AttnP &p, int64_t all) {
    const int64_t n = (all + p.blocks - 1) / p.blocks;
    return n > p.least ? n : p.least;
}

// one piece of work: units [u0, u1) of an item
struct Piece {
    int b, head, tile, u0, u1;
    int slot;  // of the scratch that its sums go to, -1: it is the whole item
    Past past;
};
// the pieces of a block, one after the other
struct Pieces {
    int64_t at, end, before;  // units of this block; units before the sequence
    int b;
    bool first;
    // by every thread of the block (a barrier inside; sh: four numbers of shared memory)
    __device__ __forceinline__ void start(const AttnP &p, int64_t *sh) {
        if (threadIdx.x < 32) {
            Span s{0, 0, -1};
            int64_t from = blockIdx.x, to = from + 1;
            if (p.blocks) {
                s = span_of(p, -1);
                const int64_t n = share_of(p, s.all);
                from = min(n * (int64_t)blockIdx.x, s.all), to = min(from + n, s.all);
            }
            if (from < to) s = span_of(p, from);
            if (s.b < 0) to = from;
            if (threadIdx.x == 0) sh[0] = from, sh[1] = to, sh[2] = s.before, sh[3] = s.b;
        }
        __syncthreads();
        rewind(sh);
    }
    __device__ __forceinline__ void rewind(const int64_t *sh) {
        at = sh[0], end = sh[1], before = sh[2], b = (int)sh[3];
        first = true;
    }
    __device__ __forceinline__ bool next(const AttnP &p, Piece &r) {
        if (at >= end) return false;
        r.past = past_of(p, b);
        while (at >= before + units_of(p, r.past)) {
            before += units_of(p, r.past);
            r.past = past_of(p, ++b);
        }
        const int64_t i = at - before;
        r.b = b;
        if (p.blocks) {
            const int64_t item = i / r.past.units;
            r.u0 = (int)(i - item * r.past.units);
            r.u1 = (int)min((int64_t)r.past.units, r.u0 + (end - at));
            r.tile = (int)(item % r.past.tiles);
            r.head = (int)(item / r.past.tiles);
            // slot 0 is the block's first piece, slot 1 a later one (which begins its item)
            r.slot = r.u0 == 0 && r.u1 == r.past.units ? -1 : 2 * (int)blockIdx.x + !first;
            at += r.u1 - r.u0;
        } else {  // (the last tiles, with the most keys, first)
            r.head = (int)(i % p.c.heads);
            r.tile = r.past.tiles - 1 - (int)(i / p.c.heads);
            r.u0 = 0, r.u1 = r.past.units, r.slot = -1;
            ++at;
        }
        first = false;
        return true;
    }
};
// log2 of the weight of the largest score (fp16 products: so that small weights are within its range)
template <typename T, bool CODES>
constexpr float top_weight() { return CODES || std::is_same<T, __half>::value ? 14.0f : 0.0f; }
__device__ __forceinline__ float *part_of_slot(const AttnP &p, int slot) {
    return p.part + (int64_t)slot * p.rows * (p.c.head_dim + 2);
}

// the last key that row r sees (it sees all up to it), -1: none
__device__ __forceinline__ int last_key(const AttnP &p, const Past &s, int64_t row) {
    const int64_t at = s.s.pos + row / p.group;
    return (int)(at < s.ctx ? at : s.ctx - 1);
}

// A result that is not finite may have met values that its query does not see (0 times infinity), or infinities that
// it sees but that came to the products in two parts (infinity less infinity), or codes with scales beyond the products'
// range: it is then computed again from what it sees, by one whole warp, in fp32.  Of a cut item that is the part that has
// met them: its average, with a sum of weights of 1 (and its largest score changed accordingly).
// Keys go ONCE at a time, a lane pairs of a head's values, all loads before what needs them (for they are what it waits
// for), and the sums stay divided by that of the weights and within their type, so that roundings make no infinity.  A row ends
// where what is not finite has become NaN, which nothing changes any more.
// It is slow: a prompt of 4096 tokens, 32 heads of 128 over 8, all of whose rows see an infinite value from the start, takes
// 57 ms for 0.19 in bf16, 91 for 1.1 over codes, 165 for 5.1 in fp32; with a NaN in its place 0.9, 1.4 and 5.7, with
// one in the middle half of the infinity's; one token over 131072 keys 3.4 ms for 0.10, with a NaN 0.12.
template <typename C>
struct Pair {  // two neighbours as they lie in memory
    using Raw = typename std::conditional<sizeof(C) == 4, float2, typename std::conditional<sizeof(C) == 2, uint32_t, char2>::type>::type;
    static __device__ __forceinline__ Raw load(const void *p, int64_t at) { return *reinterpret_cast<const Raw *>(static_cast<const C *>(p) + at); }
    static __device__ __forceinline__ float2 floats(Raw v) {
        if constexpr (sizeof(C) == 4) return v;
        else if constexpr (sizeof(C) == 2) return tc::unpack2<C>(v);
        else return make_float2((float)v.x, (float)v.y);
    }
};
template <typename T>
constexpr float largest_of() { return std::is_same<T, __nv_bfloat16>::value ? 3.38953138925e38f : 3.40282346639e38f; }
template <typename T, typename C, int ONCE>
__device__ __forceinline__ void compute_again(const AttnP &p, const Past &past, int head, int tile, int r, int u0, int u1, float *part) {
    constexpr bool CODES = sizeof(C) == 1;
    const int lane = threadIdx.x % 32, d = p.c.head_dim;
    const int64_t row = (int64_t)tile * p.rows + r, token = past.s.first + row / p.group, qh = (int64_t)head * p.group + row % p.group;
    const T *x = static_cast<const T *>(p.h.x) + token * p.h.ldx + qh * p.h.hx;
    T *y = static_cast<T *>(p.h.y) + token * p.h.ldy + qh * p.h.hy;
    const int last = (int)min((int64_t)last_key(p, past, row), (int64_t)u1 * p.keys - 1);
    float q[8], o[8], m = -INFINITY, l = 0.0f;
    uint32_t need = 0, infinite = 0;  // of this lane's values: not finite; averages of an infinity
    __syncwarp();  // (others may have written them)
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int e = 64 * (i / 2) + 2 * lane + i % 2;
        o[i] = 0.0f;
        q[i] = e < d ? ldf(x + e) : 0.0f;
        if (e < d && !(fabsf(part ? part[r * d + e] : ldf(y + e)) < INFINITY)) need |= 1u << i;
    }
    if (!__any_sync(0xffffffffu, need)) return;
    bool open = true;
#pragma unroll 1
    for (int64_t j0 = (int64_t)u0 * p.keys; open && j0 <= last; j0 += 32) {
        int64_t mine = -1;  // the row of key j0 + lane
        if (j0 + lane <= last) {
            const int64_t place = place_in(p.c, p.t, past.s.slot, j0 + lane);
            if (place >= 0) mine = row_in(p.c, place, head);
        }
        float ks = 1.0f, vs = 1.0f;
        if (CODES && mine >= 0) ks = p.c.k_scale[mine], vs = p.c.v_scale[mine];
#pragma unroll 1
        for (int g = 0; open && g < 32 && j0 + g <= last; g += ONCE) {
            float s[ONCE];
#pragma unroll
            for (int k = 0; k < ONCE; ++k) s[k] = 0.0f;
#pragma unroll
            for (int i = 0; i < 8; i += 2) {
                const int e = 32 * i + 2 * lane;
                if (32 * i >= d) break;
                typename Pair<C>::Raw v[ONCE];
#pragma unroll
                for (int k = 0; k < ONCE; ++k) {
                    const int64_t r = __shfl_sync(0xffffffffu, mine, g + k);
                    v[k] = Pair<C>::load(p.c.k, (r < 0 ? 0 : r) * d + (e < d ? e : 0));
                }
#pragma unroll
                for (int k = 0; k < ONCE; ++k) {
                    const float2 f = Pair<C>::floats(v[k]);
                    const float z = CODES ? __shfl_sync(0xffffffffu, ks, g + k) : 1.0f;
                    if (e < d) s[k] = fmaf(q[i], CODES ? f.x * z : f.x, fmaf(q[i + 1], CODES ? f.y * z : f.y, s[k]));
                }
            }
            float up = m;
#pragma unroll
            for (int k = 0; k < ONCE; ++k) {
#pragma unroll
                for (int n = 16; n; n /= 2) s[k] += __shfl_xor_sync(0xffffffffu, s[k], n);
                s[k] = __shfl_sync(0xffffffffu, (int)(mine < 0), g + k) ? -INFINITY : s[k] * p.scale;
                up = fmaxf(up, s[k]);
            }
            const float base = up == -INFINITY ? 0.0f : up;
            const float before = l * exp2f(m - base);
            m = up, l = before;
#pragma unroll
            for (int k = 0; k < ONCE; ++k) {
                s[k] = exp2f(s[k] - base);
                l += s[k];
            }
            const float inv = l == 0.0f ? 0.0f : 1.0f / l, keep = before * inv;
            bool any = false;
#pragma unroll
            for (int i = 0; i < 8; i += 2) {
                const int e = 32 * i + 2 * lane;
                if (32 * i >= d) break;
                typename Pair<C>::Raw v[ONCE];
#pragma unroll
                for (int k = 0; k < ONCE; ++k) {
                    const int64_t r = __shfl_sync(0xffffffffu, mine, g + k);
                    v[k] = Pair<C>::load(p.c.v, (r < 0 ? 0 : r) * d + (e < d ? e : 0));
                }
                o[i] *= keep, o[i + 1] *= keep;
#pragma unroll
                for (int k = 0; k < ONCE; ++k) {
                    float2 f = Pair<C>::floats(v[k]);
                    const float z = CODES ? __shfl_sync(0xffffffffu, vs, g + k) : 1.0f;
                    if (CODES) f.x *= z, f.y *= z;
                    if (__shfl_sync(0xffffffffu, (int)(mine < 0), g + k)) f.x = f.y = 0.0f;
                    o[i] = fmaf(s[k] * inv, f.x, o[i]), o[i + 1] = fmaf(s[k] * inv, f.y, o[i + 1]);
                    infinite |= (uint32_t)(fabsf(f.x) == INFINITY) << i | (uint32_t)(fabsf(f.y) == INFINITY) << (i + 1);
                }
#pragma unroll
                for (int h = i; h < i + 2; ++h) {
                    if (fabsf(o[h]) == INFINITY && !(infinite >> h & 1u)) o[h] = copysignf(largest_of<T>(), o[h]);
                    any |= (need >> h & 1u) && o[h] == o[h];
                }
            }
            open = l == l && (l == 0.0f || __any_sync(0xffffffffu, any));
        }
    }
    const float bad = l != l ? l : 0.0f;
    const bool all = part && (open || l != l);  // (a part's other values get its new factor, but beside NaN they stay)
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int e = 64 * (i / 2) + 2 * lane + i % 2;
        if (e >= d || !(all || (need >> i & 1u))) continue;
        const float v = l > 0.0f ? o[i] : bad;
        if (part) part[r * d + e] = v;
        else stf(y + e, v);
    }
    if (all && lane == 0) {
        part[(int64_t)p.rows * d + r] = l > 0.0f ? m + log2f(l) + top_weight<T, CODES>() : m;
        part[(int64_t)p.rows * d + p.rows + r] = l > 0.0f ? 1.0f : bad;
    }
}
// row r of a piece of work
template <typename T, int ONCE>
__device__ __noinline__ void attend_again(const AttnP &p, int b, int head, int tile, int r, int u0, int u1, int slot) {
    const Past past = past_of(p, b);
    float *part = slot >= 0 ? part_of_slot(p, slot) : nullptr;
    if (p.c.dtype == SN_QI8) compute_again<T, int8_t, ONCE>(p, past, head, tile, r, u0, u1, part);
    else compute_again<T, T, ONCE>(p, past, head, tile, r, u0, u1, part);
}

}  // namespace k
}  // namespace sn
