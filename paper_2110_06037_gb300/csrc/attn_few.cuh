// Attention of few queries over a long cache, and of fp32 queries in any number (sn_attend in include/sn.h).
//
// What bounds it is the cache, read once.  A block's warps take 16 keys each in turn, with a ring of their own in
// shared memory (cp.async: keys and values of the next tiles are on their way while one is worked on) and sums of their
// own in registers; no warp waits for another before the end of an item, where their sums are joined.  A tile is two
// products by mma.sync, with keys and dims as the rows and 8 queries (the heads that share the cache's head, and a
// sequence's few tokens) as the columns, so that a token's few heads fill the product:
//   S = K Q^T (16 x 8),   O += V^T P (D x 8),   P = 2^(S - m).
// (tcgen05 has no form below 64 rows, its operands go through barriers of the whole block.)  m is the largest
// score so far only up to a factor of 2^THR: one vote a tile says whether it has to grow, and the maximum across
// lanes and the sums' scaling are rare.  P is transposed from the first product's layout to the second's by movmatrix.
// 16-bit values: P goes in as two 16-bit parts, so that no weight is rounded to less than 16 bits; with fp16 the largest
// is brought to 2^14, so that a weight is off by 2^-22 of itself or 2^-39 of the largest.
//
// Codes: q and codes go in as fp16 (codes exact; q times a power of two that brings a row's largest to 2^10, what is
// below 2^-34 of that is lost, up to a power of 120; fp32 queries as two parts).  The keys' scales are factors of the scores.  A value's scale
// is 2^e f, f in [1, 2): e goes into the exponent and f into the weight,
//   P_j = 2^(s_j + e_j - m) f_j,   sum of weights += 2^(s_j + e_j - m) 2^-e_j,
// so that P is within fp16's range.  With e from -76 to 24 no sum of weights is infinite, and what 2^(s_j + e_j - m) loses
// below fp32's range is below 2^-40 of them; a key whose value has another scale makes the row NaN, and
// attend_again computes it.  For bf16 queries P is one part, off by 2^-11 of itself, an eighth of the output's rounding.
// What bounds codes is the issue of instructions: some 800 a tile of 16 keys, heads of 128 and 8 queries, of which some 200 load
// the codes and make fp16 of them (20 for 32 dims of keys, 24 of values, and 16 loads of these).
//
// fp32 values: products in tf32 of two parts each, hi hi + hi lo + lo hi: off by 2^-21 of a product.  With fp32 queries
// the products of 16 dims, or of a tile's keys, are summed apart and added to the sums in fp32: the tensor cores truncate what they add
// to, which over a row of 10000 keys is 3e-6 of it.
#pragma once

#include <algorithm>

#include "attn_common.cuh"
#include "tc_common.cuh"

namespace sn {
namespace k {
namespace few {

constexpr int TILE = 16, UNIT = 64;  // keys of a warp's tile and of a unit of work

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
    else if constexpr (std::is_same<M, __nv_bfloat16>::value)
        asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
            : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
            : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
    else
        asm("mma.sync.aligned.m16n8k8.row.col.f32.tf32.tf32.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
            : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
            : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// an 8 x 8 matrix of 16-bit values, a lane's two neighbours of row lane / 4: the same of its transpose
__device__ __forceinline__ uint32_t transposed(uint32_t v) {
    uint32_t r;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
    return r;
}
// the tf32 part of a value, to nearest, and the rest
__device__ __forceinline__ void split(uint32_t &hi, uint32_t &lo, float v) {
    asm("cvt.rna.tf32.f32 %0, %1;" : "=r"(hi) : "f"(v));
    lo = __float_as_uint(v - __uint_as_float(hi));
}
// two codes in offset binary (bytes lo and hi of x) as fp16: 1024 + c + 128 - 1152
__device__ __forceinline__ uint32_t codes_f16(uint32_t x, uint32_t select) {
    const uint32_t v = __byte_perm(x, 0x64646464u, select);
    const __half2 h = __hsub2(*reinterpret_cast<const __half2 *>(&v), __half2half2(__ushort_as_half(0x6480)));
    return *reinterpret_cast<const uint32_t *>(&h);
}

// T: queries; C: cache (T, or int8_t); DT: head_dim at most; NB: blocks of 8 queries of an item
template <typename T, typename C, int DT, int NB>
struct Form {
    static constexpr bool CODES = sizeof(C) == 1, WIDE = sizeof(C) == 4;
    using M = typename std::conditional<CODES, __half, T>::type;  // the products' type
    static constexpr bool HALF = std::is_same<M, __half>::value;
    static constexpr int QP = CODES && sizeof(T) == 4 ? 2 : 1;    // parts of a query in shared memory
    static constexpr bool LO = !(CODES && std::is_same<T, __nv_bfloat16>::value);  // weights in two parts
    static constexpr int STEP = WIDE ? 8 : 16;                    // dims of a product
    static constexpr int QR = WIDE ? 4 : 2 * QP;                  // registers of 8 queries of a step
    static constexpr bool QREG = NB * (DT / STEP) * QR <= 64 && NB * DT <= 256;  // queries in registers
    // log2 of the largest weight when m is the largest score, and how far a score may be above m
    // (codes: times the values' f, below 2)
    static constexpr float TOP = top_weight<T, CODES>(), THR = HALF ? (CODES ? 0.95f : 1.5f) : 8.0f;
    static constexpr int STAGES = 3;
    static constexpr int ROWS = 8 * NB;
    static constexpr int WARPS = WIDE && DT > 128 ? 2 : 4;
    // blocks of an SM, by registers
    static constexpr int BLOCKS = DT * NB <= 128 ? (WIDE ? 2 : 4) : DT * NB <= 256 ? 2 : 1;
    // bytes of a row of a tile.  16-bit and codes: its number of 16 bytes odd, so that eight rows are in different
    // banks.  fp32: keys are read two rows, 64 bytes each, at a time; values four rows 2 t, 32 bytes each
    __host__ __device__ static constexpr int pad(int n, int to) { return n + (to - n % 128 + 128) % 128; }
    __host__ __device__ static constexpr int k_row(int d) { return CODES ? (d / 16 % 2 ? d + 32 : d + 16) : WIDE ? pad(4 * d, 64) : 2 * d + 16; }
    __host__ __device__ static constexpr int v_row(int d) { return WIDE ? pad(4 * d, 16) : k_row(d); }
    __host__ __device__ static constexpr int stage(int d) { return TILE * (k_row(d) + v_row(d)) + (CODES ? 2 * TILE * 4 : 0); }
    // a warp's ring, which at the end holds its sums
    __host__ __device__ static constexpr int ring(int d) {
        const int a = STAGES * stage(d), b = ROWS * d * 4;
        return a > b ? a : b;
    }
    __host__ __device__ static constexpr int q_row(int d) { return WIDE ? k_row(d) : 2 * d + 16; }
    __host__ __device__ static constexpr int bytes(int d) { return WARPS * ring(d) + QP * ROWS * q_row(d) + ROWS * 4; }
};

template <typename T, typename C, int DT, int NB>
__global__ void __launch_bounds__(32 * Form<T, C, DT, NB>::WARPS, Form<T, C, DT, NB>::BLOCKS) attend_few_kernel(const __grid_constant__ AttnP p) {
    using F = Form<T, C, DT, NB>;
    using M = typename F::M;
    constexpr bool CODES = F::CODES, WIDE = F::WIDE;
    constexpr int ROWS = F::ROWS, S = F::STAGES, QP = F::QP, WARPS = F::WARPS, KS = DT / F::STEP;
    extern __shared__ __align__(128) uint8_t sm[];
    __shared__ int64_t sh[4];
    __shared__ float sh_m[WARPS][ROWS], sh_l[WARPS][ROWS];
    const int d = p.c.head_dim, tid = threadIdx.x, warp = tid / 32, lane = tid % 32, g = lane / 4, t4 = lane % 4;
    const int k_row = F::k_row(d), v_row = F::v_row(d), stage = F::stage(d), ring_bytes = F::ring(d), q_row = F::q_row(d);
    uint8_t *ring = sm + warp * ring_bytes, *qs = sm + WARPS * ring_bytes;
    const uint32_t ring_at = tc::su32(ring);
    float *rf = reinterpret_cast<float *>(qs + QP * ROWS * q_row);  // codes: factors of the queries
    // 16-byte pieces of a tile: they lie end to end in the cache
    const int per_row = d * (int)sizeof(C) / 16, pieces = TILE * per_row;
    const uint32_t inv = 65536u / (uint32_t)per_row + 1;  // (exact for numbers up to 1024 and rows of up to 64: checked for all)
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
                    const int r = (int)((uint32_t)i * inv >> 16), x = (i - r * per_row) * 16;
                    cp16(to + r * k_row + x, kp + i * 16, r < keep);
                    cp16(to + TILE * k_row + r * v_row + x, vp + i * 16, r < keep);
                }
                if constexpr (CODES) {
                    if (lane < 8) cp16(to + TILE * (k_row + v_row) + lane * 16, (lane < 4 ? p.c.k_scale : p.c.v_scale) + row + lane % 4 * 4, ok);
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
                const int e = min(max(137 + 127 - (int)(__float_as_uint(top) >> 23), 1), 247);  // the factor's exponent, of 127 + 10 - (e - 127)
                const float f = __uint_as_float((uint32_t)e << 23);
                if (lane == 0) rf[r] = __uint_as_float((uint32_t)(254 - e) << 23);
#pragma unroll
                for (int i = 0; i < DT / 32; ++i) {
                    if (lane + 32 * i >= d) continue;
                    const float x0 = v[i] * f;
                    const __half hi = __float2half_rn(x0);
                    reinterpret_cast<__half *>(qs + r * q_row)[lane + 32 * i] = hi;
                    if constexpr (QP == 2) reinterpret_cast<__half *>(qs + (ROWS + r) * q_row)[lane + 32 * i] = __float2half_rn(x0 - __half2float(hi));
                }
            }
        } else {
            for (int r = warp; r < ROWS; r += WARPS) {
                const T *x = static_cast<const T *>(p.h.x) + (s.first + (row0 + r) / p.group) * p.h.ldx + ((int64_t)w.head * p.group + (row0 + r) % p.group) * p.h.hx;
                for (int e = lane; e < d; e += 32) reinterpret_cast<T *>(qs + r * q_row)[e] = r < rows ? x[e] : cvt<T>(0.0f);
            }
        }
        __syncthreads();
        // a step's 16 (8) dims of 8 queries, as the product's columns.  The order of dims is that of the keys' registers: for
        // codes and fp32 a lane's four neighbours, as they come from one load
        auto query = [&](uint32_t (&b)[F::QR], int n, int k) {
            const uint8_t *q = qs + (8 * n + g) * q_row;
            if constexpr (WIDE) {
                const float2 x = *reinterpret_cast<const float2 *>(q + 64 * (k / 2) + 16 * t4 + 8 * (k % 2));
                split(b[0], b[2], x.x), split(b[1], b[3], x.y);
            } else if constexpr (CODES) {
#pragma unroll
                for (int i = 0; i < QP; ++i) {
                    const uint2 x = *reinterpret_cast<const uint2 *>(q + i * ROWS * q_row + 32 * k + 8 * t4);
                    b[2 * i] = x.x, b[2 * i + 1] = x.y;
                }
            } else {
                b[0] = *reinterpret_cast<const uint32_t *>(q + 32 * k + 4 * t4), b[1] = *reinterpret_cast<const uint32_t *>(q + 32 * k + 4 * t4 + 16);
            }
        };
        uint32_t qa[F::QREG ? NB * KS : 1][F::QR];
        if constexpr (F::QREG) {
#pragma unroll
            for (int n = 0; n < NB; ++n)
#pragma unroll
                for (int k = 0; k < KS; ++k)
                    if (F::STEP * k < d) query(qa[n * KS + k], n, k);
        }
        // a lane's queries: 8 n + 2 t and the next
        float factor[NB][2], m[NB][2], l[NB][2], o[NB][DT / 16][4];
        int last[NB][2];
#pragma unroll
        for (int n = 0; n < NB; ++n) {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int r = 8 * n + 2 * t4 + i;
                factor[n][i] = p.scale * (CODES ? rf[r] : 1.0f);
                last[n][i] = r < rows ? last_key(p, w.past, row0 + r) : INT32_MAX;  // (behind the queries: zeros, written nowhere)
                m[n][i] = -INFINITY, l[n][i] = 0.0f;
            }
#pragma unroll
            for (int j = 0; j < DT / 16; ++j)
#pragma unroll
                for (int k = 0; k < 4; ++k) o[n][j][k] = 0.0f;
        }
        int now = 0;  // place in the ring of the tile worked on
#pragma unroll 1
        for (int tile = w.u0 * (UNIT / TILE) + warp; tile < tile1; tile += WARPS) {
            asm volatile("cp.async.wait_group %0;" ::"n"(S - 2) : "memory");
            __syncwarp();
            const bool ok = there >> now & 1u;
            load();
            const uint8_t *kt = ring + now * stage, *vt = kt + TILE * k_row;
            const uint32_t ka = ring_at + now * stage, va = ka + TILE * k_row;
            now = now + 1 == S ? 0 : now + 1;
            // scores of keys g (0, 1) and g + 8 (2, 3)
            float c[NB][4];
#pragma unroll
            for (int n = 0; n < NB; ++n)
#pragma unroll
                for (int j = 0; j < 4; ++j) c[n][j] = 0.0f;
            auto with_query = [&](int n, int k, auto body) {
                if constexpr (F::QREG) {
                    body(qa[n * KS + k]);
                } else {
                    uint32_t b[F::QR];
                    query(b, n, k);
                    body(b);
                }
            };
            if constexpr (WIDE) {
#pragma unroll
                for (int k = 0; k < DT / 16; ++k) {
                    if (16 * k >= d) break;
                    const float4 x = *reinterpret_cast<const float4 *>(kt + g * k_row + 64 * k + 16 * t4);
                    const float4 y = *reinterpret_cast<const float4 *>(kt + (g + 8) * k_row + 64 * k + 16 * t4);
                    uint32_t hi[2][4], lo[2][4];
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        split(hi[e][0], lo[e][0], e ? x.z : x.x), split(hi[e][1], lo[e][1], e ? y.z : y.x);
                        split(hi[e][2], lo[e][2], e ? x.w : x.y), split(hi[e][3], lo[e][3], e ? y.w : y.y);
                    }
#pragma unroll
                    for (int n = 0; n < NB; ++n) {
                        float some[4] = {0.0f, 0.0f, 0.0f, 0.0f};
                        with_query(n, 2 * k, [&](const uint32_t (&b)[F::QR]) {
                            with_query(n, 2 * k + 1, [&](const uint32_t (&b1)[F::QR]) {
                                mma<float>(some, lo[0], b[0], b[1]);
                                mma<float>(some, hi[0], b[2 % F::QR], b[3 % F::QR]);
                                mma<float>(some, lo[1], b1[0], b1[1]);
                                mma<float>(some, hi[1], b1[2 % F::QR], b1[3 % F::QR]);
                                mma<float>(some, hi[0], b[0], b[1]);
                                mma<float>(some, hi[1], b1[0], b1[1]);
                            });
                        });
#pragma unroll
                        for (int j = 0; j < 4; ++j) c[n][j] += some[j];
                    }
                }
            } else if constexpr (CODES) {
#pragma unroll
                for (int k = 0; k < KS; k += 2) {
                    if (16 * k >= d) break;
                    uint32_t u[4];  // rows g, g + 8 of 16 dims, and of the next 16
                    ldsm4(u, ka + (lane % 16) * k_row + 16 * k + lane / 16 * 16);
#pragma unroll
                    for (int e = 0; e < 4; ++e) u[e] ^= 0x80808080u;
#pragma unroll
                    for (int e = 0; e < 2; ++e) {  // (of the last 16 dims alone, half is behind the row)
                        if (16 * (k + e) >= d) break;
                        const uint32_t a[4] = {codes_f16(u[2 * e], 0x4140), codes_f16(u[2 * e + 1], 0x4140), codes_f16(u[2 * e], 0x4342),
                                               codes_f16(u[2 * e + 1], 0x4342)};
#pragma unroll
                        for (int n = 0; n < NB; ++n)
                            with_query(n, k + e, [&](const uint32_t (&b)[F::QR]) {
                                if constexpr (QP == 2) {
                                    float some[4] = {0.0f, 0.0f, 0.0f, 0.0f};
                                    mma<M>(some, a, b[2], b[3]);
                                    mma<M>(some, a, b[0], b[1]);
#pragma unroll
                                    for (int j = 0; j < 4; ++j) c[n][j] += some[j];
                                } else {
                                    mma<M>(c[n], a, b[0], b[1]);
                                }
                            });
                    }
                }
            } else {
#pragma unroll
                for (int k = 0; k < KS; ++k) {
                    if (16 * k >= d) break;
                    uint32_t a[4];
                    ldsm4(a, ka + (lane % 16) * k_row + 32 * k + lane / 16 * 16);
#pragma unroll
                    for (int n = 0; n < NB; ++n) with_query(n, k, [&](const uint32_t (&b)[F::QR]) { mma<M>(c[n], a, b[0], b[1]); });
                }
            }
            // the scales of this lane's two keys; of the values' the power of two, its inverse, the rest
            float ks[2], ve[2], vi[2], vf[2];
            if constexpr (CODES) {
                const float *f = reinterpret_cast<const float *>(vt + TILE * v_row);
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    ks[j] = f[g + 8 * j];
                    const uint32_t u = __float_as_uint(f[TILE + g + 8 * j]), e = u >> 23 & 255u;
                    const bool far = e - (127u - 76u) > 100u;  // (not finite too)
                    const uint32_t n = far ? 127u : e;
                    ve[j] = (float)((int)n - 127);
                    vi[j] = __uint_as_float((254u - n) << 23);
                    vf[j] = far ? __int_as_float(0x7fc00000) : __uint_as_float((u & 0x807fffffu) | 0x3f800000u);
                }
            }
            const bool whole = ok && tile * TILE + TILE - 1 <= first;
            bool grew = false;
#pragma unroll
            for (int n = 0; n < NB; ++n)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    float &x = c[n][j];
                    x *= factor[n][j % 2];
                    if constexpr (CODES) x = fmaf(x, ks[j / 2], ve[j / 2]);
                    if (!whole && !(ok && tile * TILE + 8 * (j / 2) + g <= last[n][j % 2])) x = -INFINITY;
                    grew |= x > m[n][j % 2] + F::THR;
                }
            if (__any_sync(0xffffffffu, grew)) {
#pragma unroll
                for (int n = 0; n < NB; ++n)
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        float up = fmaxf(c[n][i], c[n][i + 2]);
#pragma unroll
                        for (int k = 4; k < 32; k *= 2) up = fmaxf(up, __shfl_xor_sync(0xffffffffu, up, k));
                        up = fmaxf(up, m[n][i]);
                        const float old = up == -INFINITY ? 1.0f : ex2(m[n][i] - up);
                        m[n][i] = up;
                        l[n][i] *= old;
#pragma unroll
                        for (int j = 0; j < DT / 16; ++j) o[n][j][i] *= old, o[n][j][i + 2] *= old;
                    }
            }
            // the weights, as columns of the second product: keys 2 t, 2 t + 1 (b[0]) and 8 further (b[1]) of query g; small parts
            uint32_t hi[NB][WIDE ? 4 : 2], lo[NB][WIDE ? 4 : 2];
#pragma unroll
            for (int n = 0; n < NB; ++n) {
                float x[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float base = m[n][j % 2];
                    x[j] = ex2(c[n][j] + (F::TOP - (base == -INFINITY ? 0.0f : base)));
                    if constexpr (CODES) {
                        l[n][j % 2] = fmaf(x[j], vi[j / 2], l[n][j % 2]);
                        x[j] *= x[j] == 0.0f && !whole ? 0.0f : vf[j / 2];  // (a key that is not seen counts nothing, whatever its scale)
                    } else {
                        l[n][j % 2] += x[j];
                    }
                }
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const float a = x[2 * h], b = x[2 * h + 1];
                    if constexpr (WIDE) {
                        const uint32_t low = transposed(__byte_perm(__float_as_uint(a), __float_as_uint(b), 0x5410));
                        const uint32_t high = transposed(__byte_perm(__float_as_uint(a), __float_as_uint(b), 0x7632));
                        split(hi[n][2 * h], lo[n][2 * h], __uint_as_float(__byte_perm(low, high, 0x5410)));
                        split(hi[n][2 * h + 1], lo[n][2 * h + 1], __uint_as_float(__byte_perm(low, high, 0x7632)));
                    } else {
                        const uint32_t u = tc::pack2<M>(a, b);
                        hi[n][h] = transposed(u);
                        if constexpr (F::LO) {
                            const float2 f = tc::unpack2<M>(u);
                            lo[n][h] = transposed(tc::pack2<M>(a - f.x, b - f.y));
                        }
                    }
                }
            }
            if constexpr (WIDE) {
                // a block of 32 dims: rows g and g + 8 of its product i are dims 4 g + 2 i and the next
                const uint8_t *v = vt + 2 * t4 * v_row + 16 * g;
#pragma unroll
                for (int k = 0; k < DT / 32; ++k) {
                    if (32 * k >= d) break;
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        uint32_t ah[2][4], al[2][4];
#pragma unroll
                        for (int h = 0; h < 2; ++h) {  // keys 8 h + 2 t, and the next
                            const float2 x = *reinterpret_cast<const float2 *>(v + 8 * h * v_row + 128 * k + 8 * i);
                            const float2 y = *reinterpret_cast<const float2 *>(v + (8 * h + 1) * v_row + 128 * k + 8 * i);
                            split(ah[h][0], al[h][0], x.x), split(ah[h][1], al[h][1], x.y);
                            split(ah[h][2], al[h][2], y.x), split(ah[h][3], al[h][3], y.y);
                        }
#pragma unroll
                        for (int n = 0; n < NB; ++n) {
                            float some[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                            for (int h = 0; h < 2; ++h) {
                                mma<float>(some, al[h], hi[n][2 * h], hi[n][2 * h + 1]);
                                mma<float>(some, ah[h], lo[n][2 * h], lo[n][2 * h + 1]);
                            }
#pragma unroll
                            for (int h = 0; h < 2; ++h) mma<float>(some, ah[h], hi[n][2 * h], hi[n][2 * h + 1]);
#pragma unroll
                            for (int j = 0; j < 4; ++j) o[n][2 * k + i][j] += some[j];
                        }
                    }
                }
            } else if constexpr (CODES) {
                // a block of 32 dims: as for fp32
                const uint8_t *v = vt + 2 * t4 * v_row + 4 * g;
#pragma unroll
                for (int k = 0; k < DT / 32; ++k) {
                    if (32 * k >= d) break;
                    uint32_t u[4];
#pragma unroll
                    for (int j = 0; j < 4; ++j) u[j] = *reinterpret_cast<const uint32_t *>(v + (8 * (j / 2) + j % 2) * v_row + 32 * k) ^ 0x80808080u;
#pragma unroll
                    for (int i = 0; i < 2; ++i) {  // dims 2 i and 2 i + 1 of keys 0 and 1; of keys 8 and 9
                        const uint32_t y0 = __byte_perm(u[0], u[1], i ? 0x7362 : 0x5140), y1 = __byte_perm(u[2], u[3], i ? 0x7362 : 0x5140);
                        const uint32_t a[4] = {codes_f16(y0, 0x4140), codes_f16(y0, 0x4342), codes_f16(y1, 0x4140), codes_f16(y1, 0x4342)};
#pragma unroll
                        for (int n = 0; n < NB; ++n) {
                            if constexpr (F::LO) {
                                float some[4] = {0.0f, 0.0f, 0.0f, 0.0f};
                                mma<M>(some, a, lo[n][0], lo[n][1]);
                                mma<M>(some, a, hi[n][0], hi[n][1]);
#pragma unroll
                                for (int j = 0; j < 4; ++j) o[n][2 * k + i][j] += some[j];
                            } else {
                                mma<M>(o[n][2 * k + i], a, hi[n][0], hi[n][1]);
                            }
                        }
                    }
                }
            } else {
#pragma unroll
                for (int k = 0; k < DT / 16; ++k) {
                    if (16 * k >= d) break;
                    uint32_t a[4];
                    ldsm4_t(a, va + (lane / 16 * 8 + lane % 8) * v_row + 32 * k + lane / 8 % 2 * 16);
#pragma unroll
                    for (int n = 0; n < NB; ++n) {
                        mma<M>(o[n][k], a, hi[n][0], hi[n][1]);
                        mma<M>(o[n][k], a, lo[n][0], lo[n][1]);
                    }
                }
            }
        }
        asm volatile("cp.async.wait_group 0;" ::: "memory");
        __syncwarp();
        // the warps' sums, through their rings
        float *mine = reinterpret_cast<float *>(ring);
#pragma unroll
        for (int n = 0; n < NB; ++n)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int r = 8 * n + 2 * t4 + i;
#pragma unroll
                for (int k = 4; k < 32; k *= 2) l[n][i] += __shfl_xor_sync(0xffffffffu, l[n][i], k);
                if (g == 0) sh_m[warp][r] = m[n][i], sh_l[warp][r] = l[n][i];
                if (r >= rows) continue;
#pragma unroll
                for (int j = 0; j < DT / 16; ++j) {
                    // the dims of rows g and g + 8
                    const int e = CODES || WIDE ? 32 * (j / 2) + 4 * g + 2 * (j % 2) : 16 * j + g, f = CODES || WIDE ? e + 1 : e + 8;
                    if (e < d) mine[r * d + e] = o[n][j][i];
                    if (f < d) mine[r * d + f] = o[n][j][i + 2];
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
                }
                bad |= !(fabsf(v) < INFINITY);
            }
            if (part && lane == 0) part[ROWS * d + r] = top, part[ROWS * d + ROWS + r] = sum;
            if (__any_sync(0xffffffffu, bad)) attend_again<T, 4>(p, w.b, w.head, w.tile, r, w.u0, w.u1, w.slot);
        }
        __syncthreads();  // the rings and the queries are free
    }
}

template <typename T, typename C, int DT, int NB>
cudaError_t launch(const AttnP &p, int64_t grid, cudaStream_t st) {
    using F = Form<T, C, DT, NB>;
    static PerDevice set;
    const size_t bytes = F::bytes(p.c.head_dim);
    if (const cudaError_t e = allow_smem(set, attend_few_kernel<T, C, DT, NB>, F::bytes(DT))) return e;
    return launch_pdl(attend_few_kernel<T, C, DT, NB>, dim3((unsigned)grid), dim3(32 * F::WARPS), bytes, st, p);
}
// how a launch is cut: rows of an item, blocks of an SM at once
struct Shape {
    int rows, blocks;
};
template <typename F>
Shape shape_of(int d) {
    return Shape{F::ROWS, std::max(1, std::min(F::BLOCKS, 226 * 1024 / (F::bytes(d) + 2048)))};
}
// the form for heads of d values and items of `rows` rows: body(its Form, its launch)
template <typename T, typename C, typename Body>
auto with_form(int d, int64_t rows, Body body) {
#define SN_FEW(DT, NB) return body(Form<T, C, DT, NB>{}, launch<T, C, DT, NB>)
    if (d > 128) {
        if constexpr (sizeof(C) < 4)  // (fp32: their products are the bound, and 16 queries' sums fill the registers)
            if (rows > 8) SN_FEW(256, 2);
        SN_FEW(256, 1);
    }
    if (d > 64) {
        if (rows <= 8) SN_FEW(128, 1);
        if (rows <= 16) SN_FEW(128, 2);
        SN_FEW(128, 4);
    }
    if (rows <= 8) SN_FEW(64, 1);
    if (rows <= 16) SN_FEW(64, 2);
    SN_FEW(64, 4);
#undef SN_FEW
}
template <typename T, typename C>
cudaError_t launch_any(const AttnP &p, int64_t grid, cudaStream_t st) {
    return with_form<T, C>(p.c.head_dim, p.rows, [&](auto, auto launch) { return launch(p, grid, st); });
}
template <typename T, typename C>
Shape shape_any(int d, int64_t rows) {
    return with_form<T, C>(d, rows, [&](auto form, auto) { return shape_of<decltype(form)>(d); });
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
few::Shape few_shape_f32(int d, int64_t rows);
cudaError_t attend_few_f32(const AttnP &p, int64_t grid, cudaStream_t st);
few::Shape few_shape_f32_q8(int d, int64_t rows);
cudaError_t attend_few_f32_q8(const AttnP &p, int64_t grid, cudaStream_t st);

}  // namespace k
}  // namespace sn
