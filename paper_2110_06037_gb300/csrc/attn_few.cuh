// Attention of few queries over a long cache of 16-bit values or 8-bit codes (sn_attend in include/sn.h).
//
// What bounds it is the cache, read once.  A block's warps take 16 keys each in turn, with a ring of their own in
// shared memory (cp.async: keys and values of the next tiles are on their way while one is worked on) and sums of their
// own in registers; no warp waits for another before the end of an item, where their sums are joined.  A tile is two
// products by mma.sync of 16 queries (the heads that share the cache's head, and a sequence's few tokens):
//   S = Q K^T (16 x 16),   O += P V (16 x D),   P = 2^(S - m).
// tcgen05 has no form below 64 rows, of which a token's few heads would use a tenth, and its operands go through
// barriers of the whole block; with 16 rows the tensor pipe is at a quarter of its rate where memory is at its own.
// P goes in as two 16-bit parts, so that no weight is rounded to less than 16 bits; with fp16 the largest is brought
// to 2^14, so that a weight is off by 2^-22 of itself or 2^-39 of the largest.
//
// Codes: q and codes go in as fp16 (codes exact; q times a power of two that brings a row's largest to 2^10, what is
// below 2^-34 of that is lost; fp32 queries as two parts).  The keys' scales are factors of the scores.  A value's scale
// is 2^e f, f in [1, 2): e goes into the exponent and f into the weight,
//   P_j = 2^(s_j + e_j - m) f_j,   sum of weights += 2^(s_j + e_j - m) 2^-e_j,
// so that P is within fp16's range whatever the scales are.
#pragma once

#include <algorithm>

#include "attn_common.cuh"
#include "tc_common.cuh"

namespace sn {
namespace k {
namespace few {

constexpr int WARPS = 4, TILE = 16, UNIT = 64;  // keys of a warp's tile and of a unit of work

__device__ __forceinline__ void cp16(uint32_t dst, const void *src, bool there) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(there ? 16 : 0) : "memory");
}
__device__ __forceinline__ void ldsm4(uint32_t (&r)[4], uint32_t at) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
                 : "r"(at)
                 : "memory");
}
__device__ __forceinline__ void ldsm4_t(uint32_t (&r)[4], uint32_t at) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
                 : "r"(at)
                 : "memory");
}
template <typename M>
__device__ __forceinline__ void mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    if constexpr (std::is_same<M, __half>::value)
        asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
            : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
            : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
    else
        asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
            : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
            : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// two codes in offset binary (bytes lo and hi of x) as fp16: 1024 + c + 128 - 1152
__device__ __forceinline__ uint32_t codes_f16(uint32_t x, uint32_t select) {
    const uint32_t v = __byte_perm(x, 0x64646464u, select);
    const __half2 h = __hsub2(*reinterpret_cast<const __half2 *>(&v), __half2half2(__ushort_as_half(0x6480)));
    return *reinterpret_cast<const uint32_t *>(&h);
}

// T: queries; C: cache (T, or int8_t); DT: head_dim at most; MT: 16-row tiles of an item
template <typename T, typename C, int DT, int MT>
struct Form {
    static constexpr bool CODES = sizeof(C) == 1;
    using M = typename std::conditional<CODES, __half, T>::type;  // the products' type
    static constexpr int QP = CODES && sizeof(T) == 4 ? 2 : 1;      // parts of a query
    static constexpr bool QREG = DT * MT * QP <= 128;               // queries in registers
    static constexpr float TOP = std::is_same<M, __half>::value ? 14.0f : 0.0f;  // log2 of the largest weight
    static constexpr int STAGES = CODES ? 5 : 3;
    static constexpr int ROWS = 16 * MT;
    // bytes of a row of the tile (its number of 16 bytes odd, so that eight rows are in different banks)
    __host__ __device__ static constexpr int stride(int d) { return CODES ? (d / 16 % 2 ? d + 32 : d + 16) : 2 * d + 16; }
    __host__ __device__ static constexpr int stage(int d) { return 2 * TILE * stride(d) + (CODES ? 2 * TILE * 4 : 0); }
    // a warp's ring, which at the end holds its sums
    __host__ __device__ static constexpr int ring(int d) {
        const int a = STAGES * stage(d), b = ROWS * d * 4;
        return a > b ? a : b;
    }
    __host__ __device__ static constexpr int bytes(int d) { return WARPS * ring(d) + QP * ROWS * (2 * d + 16) + ROWS * 4; }
};

template <typename T, typename C, int DT, int MT>
__global__ void __launch_bounds__(32 * WARPS) attend_few_kernel(const __grid_constant__ AttnP p) {
    using F = Form<T, C, DT, MT>;
    using M = typename F::M;
    constexpr bool CODES = F::CODES;
    constexpr int ROWS = F::ROWS, S = F::STAGES, QP = F::QP;
    extern __shared__ __align__(128) uint8_t sm[];
    __shared__ int64_t sh[4];
    __shared__ float sh_m[WARPS][ROWS], sh_l[WARPS][ROWS];
    const int d = p.c.head_dim, tid = threadIdx.x, warp = tid / 32, lane = tid % 32, g = lane / 4, t4 = lane % 4;
    const int stride = F::stride(d), stage = F::stage(d), ring_bytes = F::ring(d);
    uint8_t *ring = sm + warp * ring_bytes;
    const uint32_t ring_at = tc::su32(ring);
    M *qs = reinterpret_cast<M *>(sm + WARPS * ring_bytes);
    const int qld = d + 8;
    float *rf = reinterpret_cast<float *>(qs + QP * ROWS * qld);  // codes: factors of the queries' rows
    // 16-byte pieces of a tile: they lie end to end in the cache, and 16 or 32 bytes further a row in the ring
    const int per_row = d * (int)sizeof(C) / 16, pieces = TILE * per_row;
    const uint32_t inv = 65536u / (uint32_t)per_row + 1;  // (exact for numbers below 512 and rows of up to 32)
    griddep_launch();
    griddep_wait();
    Pieces work;
    work.start(p, sh);
    for (Piece w; work.next(p, w);) {
        const Seq &s = w.past.s;
        const int64_t row0 = (int64_t)w.tile * ROWS, all = (int64_t)s.len * p.group;
        const int rows = (int)min((int64_t)ROWS, all - row0);
        const int first = last_key(p, w.past, row0), end = last_key(p, w.past, row0 + rows - 1);  // keys seen by all; by any
        const int tile1 = min(w.u1 * (UNIT / TILE), end / TILE + (end >= 0));
        int next = w.u0 * (UNIT / TILE) + warp;  // the next tile to load
        const int32_t *pages = p.t.at + (int64_t)max(s.slot, 0) * p.t.width;
        const int shift = 31 - __clz(p.c.page);
        uint32_t there = 0;  // of the tiles under way, by their number in the ring: do they have a page
        int page = next < tile1 ? pages[next * TILE >> shift] : -1;
        int at = 0;          // place in the ring of the next tile
        auto load = [&]() {
            if (next < tile1) {
                const bool ok = page >= 0 && page < p.c.pages;
                const int64_t row = ok ? ((((int64_t)page * p.c.heads + w.head) << shift) + ((next * TILE) & (p.c.page - 1))) : 0;
                there = (there & ~(1u << at)) | ((uint32_t)ok << at);
                const int keep = ok ? min(TILE, w.past.ctx - next * TILE) : 0;  // (keys behind the sequence are zeros)
                const char *kp = static_cast<const char *>(p.c.k) + row * d * (int)sizeof(C), *vp = static_cast<const char *>(p.c.v) + row * d * (int)sizeof(C);
                const uint32_t to = ring_at + at * stage;
                for (int i = lane; i < pieces; i += 32) {
                    const int r = (int)((uint32_t)i * inv >> 16);
                    const uint32_t o = to + r * stride + (i - r * per_row) * 16;
                    cp16(o, kp + i * 16, r < keep);
                    cp16(o + TILE * stride, vp + i * 16, r < keep);
                }
                if constexpr (CODES) {
                    if (lane < 8) cp16(to + 2 * TILE * stride + lane * 16, (lane < 4 ? p.c.k_scale : p.c.v_scale) + row + lane % 4 * 4, ok);
                }
                next += WARPS;
                if (next < tile1) page = pages[next * TILE >> shift];
            }
            at = at + 1 == S ? 0 : at + 1;
            asm volatile("cp.async.commit_group;" ::: "memory");
        };
#pragma unroll
        for (int i = 0; i < S - 1; ++i) load();
        // the queries
        if constexpr (CODES) {
            for (int r = warp; r < ROWS; r += WARPS) {
                const T *x = static_cast<const T *>(p.h.x) + (s.first + (row0 + r) / p.group) * p.h.ldx + ((int64_t)w.head * p.group + (row0 + r) % p.group) * p.h.hx;
                float v[DT / 32], top = 0.0f;
#pragma unroll
                for (int i = 0; i < DT / 32; ++i) {
                    v[i] = r < rows && lane + 32 * i < d ? ldf(x + lane + 32 * i) : 0.0f;
                    top = fmaxf(top, fabsf(v[i]));
                }
#pragma unroll
                for (int o = 16; o; o /= 2) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
                const int e = min(max(137 + 127 - (int)(__float_as_uint(top) >> 23), 1), 227);  // the factor's exponent, of 127 + 10 - (e - 127)
                const float f = __uint_as_float((uint32_t)e << 23);
                if (lane == 0) rf[r] = __uint_as_float((uint32_t)(254 - e) << 23);
#pragma unroll
                for (int i = 0; i < DT / 32; ++i) {
                    if (lane + 32 * i >= d) continue;
                    const float x0 = v[i] * f;
                    const __half hi = __float2half_rn(x0);
                    qs[r * qld + lane + 32 * i] = hi;
                    if constexpr (QP == 2) qs[(ROWS + r) * qld + lane + 32 * i] = __float2half_rn(x0 - __half2float(hi));
                }
            }
        } else {
            for (int i = tid; i < ROWS * d; i += 32 * WARPS) {
                const int r = i / d, e = i - r * d;
                qs[r * qld + e] = r < rows ? static_cast<const T *>(p.h.x)[(s.first + (row0 + r) / p.group) * p.h.ldx +
                                                                           ((int64_t)w.head * p.group + (row0 + r) % p.group) * p.h.hx + e]
                                           : cvt<T>(0.0f);
            }
        }
        __syncthreads();
        // a step of 16 dims of the queries: as ldmatrix lays them out, or for codes with a lane's four neighbours of a row
        // (dims 4 t .. 4 t + 3) in its two registers, as the codes' bytes come
        auto query = [&](uint32_t (&a)[4], int part, int mt, int k) {
            const M *q = qs + (part * ROWS + 16 * mt) * qld + 16 * k;
            if constexpr (CODES) {
                const uint2 x = *reinterpret_cast<const uint2 *>(q + g * qld + 4 * t4), y = *reinterpret_cast<const uint2 *>(q + (g + 8) * qld + 4 * t4);
                a[0] = x.x, a[2] = x.y, a[1] = y.x, a[3] = y.y;
            } else {
                ldsm4(a, tc::su32(q + (lane % 16) * qld + lane / 16 * 8));
            }
        };
        constexpr int KS = DT / 16;
        uint32_t qa[F::QREG ? QP * MT * KS : 1][4];
        if constexpr (F::QREG) {
#pragma unroll
            for (int i = 0; i < QP * MT; ++i)
#pragma unroll
                for (int k = 0; k < KS; ++k)
                    if (16 * k < d) query(qa[i * KS + k], i / MT, i % MT, k);
        }
        float factor[2 * MT];
        int last[2 * MT];
#pragma unroll
        for (int i = 0; i < 2 * MT; ++i) {
            const int r = 8 * i + g;
            factor[i] = p.scale * (CODES ? rf[r] : 1.0f);
            last[i] = r < rows ? last_key(p, w.past, row0 + r) : -1;
        }
        float m[2 * MT], l[2 * MT], o[MT][DT / 8][4];
#pragma unroll
        for (int i = 0; i < 2 * MT; ++i) m[i] = -INFINITY, l[i] = 0.0f;
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int j = 0; j < DT / 8; ++j)
#pragma unroll
                for (int k = 0; k < 4; ++k) o[i][j][k] = 0.0f;
        int now = 0;  // place in the ring of the tile worked on
        for (int tile = w.u0 * (UNIT / TILE) + warp; tile < tile1; tile += WARPS) {
            asm volatile("cp.async.wait_group %0;" ::"n"(S - 2) : "memory");
            __syncwarp();
            const bool ok = there >> now & 1u;
            load();
            const uint8_t *st = ring + now * stage;
            const uint32_t sa = ring_at + now * stage, va = sa + TILE * stride;
            now = now + 1 == S ? 0 : now + 1;
            float c[MT][2][4];
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
                for (int j = 0; j < 8; ++j) c[i][j / 4][j % 4] = 0.0f;
            if constexpr (CODES) {
#pragma unroll
                for (int k = 0; k < KS; k += 2) {
                    if (16 * k >= d) break;
                    uint32_t b[4];
                    ldsm4(b, sa + (lane / 16 * 8 + lane % 8) * stride + 16 * k + lane / 8 % 2 * 16);
#pragma unroll
                    for (int e = 0; e < 4; ++e) b[e] ^= 0x80808080u;
#pragma unroll
                    for (int e = 0; e < 2; ++e) {  // (of the last 16 dims alone, half is behind the row)
                        if (16 * (k + e) >= d) break;
                        const uint32_t b00 = codes_f16(b[e], 0x4140), b01 = codes_f16(b[e], 0x4342);
                        const uint32_t b10 = codes_f16(b[e + 2], 0x4140), b11 = codes_f16(b[e + 2], 0x4342);
#pragma unroll
                        for (int i = 0; i < QP * MT; ++i) {
                            uint32_t a[4];
                            if constexpr (F::QREG) {
#pragma unroll
                                for (int x = 0; x < 4; ++x) a[x] = qa[i * KS + k + e][x];
                            } else {
                                query(a, i / MT, i % MT, k + e);
                            }
                            mma<M>(c[i % MT][0], a, b00, b01);
                            mma<M>(c[i % MT][1], a, b10, b11);
                        }
                    }
                }
            } else {
#pragma unroll
                for (int k = 0; k < KS; ++k) {
                    if (16 * k >= d) break;
                    uint32_t b[4];
                    ldsm4(b, sa + (lane / 16 * 8 + lane % 8) * stride + 32 * k + lane / 8 % 2 * 16);
#pragma unroll
                    for (int i = 0; i < MT; ++i) {
                        uint32_t a[4];
                        if constexpr (F::QREG) {
#pragma unroll
                            for (int x = 0; x < 4; ++x) a[x] = qa[i * KS + k][x];
                        } else {
                            query(a, 0, i, k);
                        }
                        mma<M>(c[i][0], a, b[0], b[1]);
                        mma<M>(c[i][1], a, b[2], b[3]);
                    }
                }
            }
            // this lane's four keys: 2 t, 2 t + 1, 8 + 2 t, 9 + 2 t; scales, and of the values' the power of two, its inverse, the rest
            float ks[4], ve[4], vi[4], vf[4];
            if constexpr (CODES) {
                const float *f = reinterpret_cast<const float *>(st + 2 * TILE * stride);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int key = 8 * (j / 2) + 2 * t4 + j % 2;
                    ks[j] = f[key];
                    const uint32_t u = __float_as_uint(f[TILE + key]), e = u >> 23 & 255u;
                    // (below the normal range: 2^-126 and what is left; not finite: NaN)
                    ve[j] = (float)((int)(e ? e : 1u) - 127);
                    vi[j] = __uint_as_float((254u - min(max(e, 1u), 253u)) << 23);
                    vf[j] = e == 255u ? __int_as_float(0x7fc00000) : e ? __uint_as_float((u & 0x807fffffu) | 0x3f800000u)
                                                                     : f[TILE + key] * 8.507059173023462e37f;
                }
            }
            const bool whole = ok && tile * TILE + TILE - 1 <= first;
            uint32_t hi[MT][4], lo[MT][4];
#pragma unroll
            for (int i = 0; i < MT; ++i) {
                float old[2];
                bool grew = false;
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    const int n = 2 * i + r;
                    float x[4], up = m[n];
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        x[j] = c[i][j / 2][2 * r + j % 2] * factor[n];
                        if constexpr (CODES) x[j] = fmaf(x[j], ks[j], ve[j]);
                        if (!whole && !(ok && tile * TILE + 8 * (j / 2) + 2 * t4 + j % 2 <= last[n])) x[j] = -INFINITY;
                        up = fmaxf(up, x[j]);
                    }
                    up = fmaxf(up, __shfl_xor_sync(0xffffffffu, up, 1));
                    up = fmaxf(up, __shfl_xor_sync(0xffffffffu, up, 2));
                    const float base = up == -INFINITY ? 0.0f : up, low = base - F::TOP;
                    grew |= up > m[n];
                    old[r] = ex2(m[n] - base);
                    m[n] = up;
                    float sum = 0.0f;
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        x[j] = ex2(x[j] - low);
                        if constexpr (CODES) {
                            sum = fmaf(x[j], vi[j], sum);
                            x[j] *= x[j] == 0.0f && !whole ? 0.0f : vf[j];  // (a key that is not seen counts nothing, whatever its scale)
                        } else {
                            sum += x[j];
                        }
                    }
                    l[n] = fmaf(l[n], old[r], sum);
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        const uint32_t h = tc::pack2<M>(x[2 * j], x[2 * j + 1]);
                        const float2 f = tc::unpack2<M>(h);
                        hi[i][2 * j + r] = h;
                        lo[i][2 * j + r] = tc::pack2<M>(x[2 * j] - f.x, x[2 * j + 1] - f.y);
                    }
                }
                if (__any_sync(0xffffffffu, grew)) {
#pragma unroll
                    for (int j = 0; j < DT / 8; ++j) o[i][j][0] *= old[0], o[i][j][1] *= old[0], o[i][j][2] *= old[1], o[i][j][3] *= old[1];
                }
            }
            if constexpr (CODES) {
                // a block of 32 dims: the n-th column of its j-th product is dim 4 n + j
                const uint8_t *v = st + TILE * stride + 2 * t4 * stride + 4 * g;
#pragma unroll
                for (int k = 0; k < DT / 32; ++k) {
                    if (32 * k >= d) break;
                    uint32_t u[4];
#pragma unroll
                    for (int j = 0; j < 4; ++j) u[j] = *reinterpret_cast<const uint32_t *>(v + (8 * (j / 2) + j % 2) * stride + 32 * k) ^ 0x80808080u;
                    uint32_t y[4];  // dims 0 and 1, 2 and 3 of keys 0 and 1; of keys 8 and 9
                    y[0] = __byte_perm(u[0], u[1], 0x5140), y[1] = __byte_perm(u[0], u[1], 0x7362);
                    y[2] = __byte_perm(u[2], u[3], 0x5140), y[3] = __byte_perm(u[2], u[3], 0x7362);
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const uint32_t select = j % 2 ? 0x4342 : 0x4140;
                        const uint32_t b0 = codes_f16(y[j / 2], select), b1 = codes_f16(y[2 + j / 2], select);
#pragma unroll
                        for (int i = 0; i < MT; ++i) {
                            mma<M>(o[i][4 * k + j], hi[i], b0, b1);
                            mma<M>(o[i][4 * k + j], lo[i], b0, b1);
                        }
                    }
                }
            } else {
#pragma unroll
                for (int k = 0; k < KS; ++k) {
                    if (16 * k >= d) break;
                    uint32_t b[4];
                    ldsm4_t(b, va + (lane % 16) * stride + 32 * k + lane / 16 * 16);
#pragma unroll
                    for (int i = 0; i < MT; ++i) {
                        mma<M>(o[i][2 * k], hi[i], b[0], b[1]);
                        mma<M>(o[i][2 * k + 1], hi[i], b[2], b[3]);
                        mma<M>(o[i][2 * k], lo[i], b[0], b[1]);
                        mma<M>(o[i][2 * k + 1], lo[i], b[2], b[3]);
                    }
                }
            }
        }
        asm volatile("cp.async.wait_group 0;" ::: "memory");
        __syncwarp();
        // the warps' sums, through their rings
        float *mine = reinterpret_cast<float *>(ring);
#pragma unroll
        for (int n = 0; n < 2 * MT; ++n) {
            const int r = 8 * n + g;
            l[n] += __shfl_xor_sync(0xffffffffu, l[n], 1);
            l[n] += __shfl_xor_sync(0xffffffffu, l[n], 2);
            if (t4 == 0) sh_m[warp][r] = m[n], sh_l[warp][r] = l[n];
            if (r >= rows) continue;
#pragma unroll
            for (int j = 0; j < DT / 8; ++j) {
                const float a = o[n / 2][j][2 * (n % 2)], b = o[n / 2][j][2 * (n % 2) + 1];
                if constexpr (CODES) {
                    const int e = 32 * (j / 4) + 8 * t4 + j % 4;
                    if (e < d) mine[r * d + e] = a;
                    if (e + 4 < d) mine[r * d + e + 4] = b;
                } else {
                    if (8 * j < d) *reinterpret_cast<float2 *>(mine + r * d + 8 * j + 2 * t4) = make_float2(a, b);
                }
            }
        }
        __syncthreads();
        for (int r = warp; r < rows; r += WARPS) {
            float top = -INFINITY, f[WARPS], sum = 0.0f;
#pragma unroll
            for (int i = 0; i < WARPS; ++i) top = fmaxf(top, sh_m[i][r]);
            const float base = top == -INFINITY ? 0.0f : top;
#pragma unroll
            for (int i = 0; i < WARPS; ++i) {
                f[i] = ex2(sh_m[i][r] - base);
                sum = fmaf(sh_l[i][r], f[i], sum);
            }
            float *part = w.slot >= 0 ? part_of_slot(p, w.slot) : nullptr;
            T *y = static_cast<T *>(p.h.y) + (s.first + (row0 + r) / p.group) * p.h.ldy + ((int64_t)w.head * p.group + (row0 + r) % p.group) * p.h.hy;
            const float inv_l = sum == 0.0f ? 0.0f : 1.0f / sum;
            bool bad = false;
            for (int e = lane; e < d; e += 32) {
                float v = 0.0f;
#pragma unroll
                for (int i = 0; i < WARPS; ++i) v = fmaf(reinterpret_cast<const float *>(sm + i * ring_bytes)[r * d + e], f[i], v);
                if (part) {
                    part[r * d + e] = v;
                } else {
                    v = sum == 0.0f ? 0.0f : v * inv_l;
                    stf(y + e, v);
                    bad |= !(fabsf(v) < INFINITY);
                }
            }
            if (part && lane == 0) part[ROWS * d + r] = top, part[ROWS * d + ROWS + r] = sum;
            if (!part && s.len > 1 && __any_sync(0xffffffffu, bad)) attend_again<T>(p, w.b, w.head, row0 + r);
        }
        __syncthreads();  // the rings and the queries are free
    }
}

template <typename T, typename C, int DT, int MT>
cudaError_t launch(const AttnP &p, int64_t grid, cudaStream_t st) {
    static PerDevice set;
    const size_t bytes = Form<T, C, DT, MT>::bytes(p.c.head_dim);
    if (const cudaError_t e = allow_smem(set, attend_few_kernel<T, C, DT, MT>, Form<T, C, DT, MT>::bytes(DT))) return e;
    return launch_pdl(attend_few_kernel<T, C, DT, MT>, dim3((unsigned)grid), dim3(32 * WARPS), bytes, st, p);
}
// blocks of an SM at once: by shared memory, and two by registers
template <typename T, typename C>
int blocks_of(int d, int rows) {
    const bool two = rows > 16;
    const int bytes = d <= 64 ? (two ? Form<T, C, 64, 2>::bytes(d) : Form<T, C, 64, 1>::bytes(d))
                      : d <= 128 ? (two ? Form<T, C, 128, 2>::bytes(d) : Form<T, C, 128, 1>::bytes(d))
                                 : Form<T, C, 256, 1>::bytes(d);
    return std::max(1, std::min(d <= 64 && !two ? 3 : 2, 225 * 1024 / (bytes + 2048)));
}
template <typename T, typename C>
cudaError_t launch_any(const AttnP &p, int64_t grid, cudaStream_t st) {
    const int d = p.c.head_dim;
    if (d > 128) return launch<T, C, 256, 1>(p, grid, st);
    if (p.rows > 16) return d <= 64 ? launch<T, C, 64, 2>(p, grid, st) : launch<T, C, 128, 2>(p, grid, st);
    return d <= 64 ? launch<T, C, 64, 1>(p, grid, st) : launch<T, C, 128, 1>(p, grid, st);
}

// how a launch is cut: rows of an item, blocks of an SM at once
struct Shape {
    int rows, blocks;
};
template <typename T, typename C>
Shape shape_any(int d, int64_t rows) {
    const int n = rows > 16 && d <= 128 ? 32 : 16;
    return Shape{n, blocks_of<T, C>(d, n)};
}

}  // namespace few

// in files of their own, for the compiler's sake: queries of each type over its own values and over codes
few::Shape few_shape_f16(int d, int64_t rows);
cudaError_t attend_few_f16(const AttnP &p, int64_t grid, cudaStream_t st);
few::Shape few_shape_bf16(int d, int64_t rows);
cudaError_t attend_few_bf16(const AttnP &p, int64_t grid, cudaStream_t st);
few::Shape few_shape_f16_q8(int d, int64_t rows);
cudaError_t attend_few_f16_q8(const AttnP &p, int64_t grid, cudaStream_t st);
few::Shape few_shape_bf16_q8(int d, int64_t rows);
cudaError_t attend_few_bf16_q8(const AttnP &p, int64_t grid, cudaStream_t st);
few::Shape few_shape_f32_q8(int d, int64_t rows);
cudaError_t attend_few_f32_q8(const AttnP &p, int64_t grid, cudaStream_t st);

}  // namespace k
}  // namespace sn
