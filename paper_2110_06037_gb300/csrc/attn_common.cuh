// Pieces that the kernels of the attention layer's operators share.
#pragma once

#include "ssm_common.cuh"

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
    r.units = max(1, (r.ctx + p.keys - 1) / p.keys);
    return r;
}
// units of a sequence (whole: its items)
__device__ __forceinline__ int64_t units_of(const AttnP &p, const Past &r) {
    return (int64_t)r.tiles * p.c.heads * (p.blocks ? r.units : 1);
}

// by one whole warp: the units of all sequences, those before sequence `b` (b >= 0), or the sequence in
// which unit `at` lies (at >= 0) and those before it
struct Span {
    int64_t all, before;
    int b;
};
__device__ __forceinline__ Span span_of(const AttnP &p, int b, int64_t at) {
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
        if (b >= b0 && b < b0 + 32) r.before = r.all + __shfl_sync(0xffffffffu, up - n, b - b0);
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
                s = span_of(p, -1, -1);
                const int64_t n = share_of(p, s.all);
                from = min(n * (int64_t)blockIdx.x, s.all), to = min(from + n, s.all);
            }
            if (from < to) s = span_of(p, -1, from);
            if (s.b < 0) to = from;
            if (threadIdx.x == 0) sh[0] = from, sh[1] = to, sh[2] = s.before, sh[3] = s.b;
        }
        __syncthreads();
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
__device__ __forceinline__ float *part_of_slot(const AttnP &p, int slot) {
    return p.part + (int64_t)slot * p.rows * (p.c.head_dim + 2);
}

// the last key that row r sees (it sees all up to it), -1: none
__device__ __forceinline__ int last_key(const AttnP &p, const Past &s, int64_t row) {
    const int64_t at = s.s.pos + row / p.group;
    return (int)(at < s.ctx ? at : s.ctx - 1);
}

// An output that is not finite may have met values that its query does not see (0 times infinity), or infinities that
// it sees but that came to the products in two parts (infinity less infinity), or codes with scales beyond the products'
// range: it is then computed again from what it sees, by one whole warp, in fp32.
template <typename T>
__device__ __noinline__ void attend_again(const AttnP &p, int b, int head, int64_t row) {
    const int lane = threadIdx.x % 32, d = p.c.head_dim;
    const Past past = past_of(p, b);
    const int64_t token = past.s.first + row / p.group, qh = (int64_t)head * p.group + row % p.group;
    const int last = last_key(p, past, row);
    float q[8], o[8], m = -INFINITY, l = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        o[i] = 0.0f;
        q[i] = lane + 32 * i < d ? ldf(static_cast<const T *>(p.h.x) + token * p.h.ldx + qh * p.h.hx + lane + 32 * i) : 0.0f;
    }
    for (int j = 0; j <= last; ++j) {
        const int64_t place = place_in(p.c, p.t, past.s.slot, j);
        if (place < 0) continue;
        const int64_t r = row_in(p.c, place, head);
        float s = 0.0f, v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int e = lane + 32 * i;
            v[i] = 0.0f;
            if (e >= d) continue;
            if (p.c.dtype == SN_QI8) {
                s = fmaf(q[i], (float)static_cast<const int8_t *>(p.c.k)[r * d + e], s);
                v[i] = p.c.v_scale[r] * (float)static_cast<const int8_t *>(p.c.v)[r * d + e];
            } else {
                s = fmaf(q[i], ldf(static_cast<const T *>(p.c.k) + r * d + e), s);
                v[i] = ldf(static_cast<const T *>(p.c.v) + r * d + e);
            }
        }
#pragma unroll
        for (int k = 16; k; k /= 2) s += __shfl_xor_sync(0xffffffffu, s, k);
        s *= p.scale;
        if (p.c.dtype == SN_QI8) s *= p.c.k_scale[r];
        const float up = fmaxf(m, s), base = up == -INFINITY ? 0.0f : up;
        const float old = exp2f(m - base), w = exp2f(s - base);
        m = up;
        l = fmaf(l, old, w);
#pragma unroll
        for (int i = 0; i < 8; ++i) o[i] = fmaf(o[i], old, w * v[i]);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (lane + 32 * i < d)
            stf(static_cast<T *>(p.h.y) + token * p.h.ldy + qh * p.h.hy + lane + 32 * i, l == 0.0f ? 0.0f : o[i] / l);
}

}  // namespace k
}  // namespace sn
