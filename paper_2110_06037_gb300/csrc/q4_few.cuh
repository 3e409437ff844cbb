// The product of 4-bit weights with few rows of x (sn_q4_dense in include/sn.h; layout
// in q4_common.cuh): the kernel template and its launch, one translation unit a type of
// x (kernels_q4_f32.cu, kernels_q4_f16.cu, kernels_q4_bf16.cu).
#pragma once

#include <algorithm>
#include <climits>

#include "q4_common.cuh"

namespace sn {
namespace k {

namespace {

// Bound by reading the weights (half a byte a product and row): 16 x 8 x 16
// products on the tensor cores with the codes as the A operand, x as columns of B
// (rows of fp32 x as three bf16 columns each), one fp32 multiply-add a group to
// scale its sum.  A warp runs along k over one 16-row tile, its weights straight
// from global memory to registers in the operand's layout, eight tiles in flight; the
// block's part of x lies in shared memory.  k is split over the WK warps of a
// block that share a tile and over the S blocks of a cluster, whose sums meet in a
// fixed order.  One bf16 row, 25088 -> 4096: 17 us, 3200 GB/s; then bound by its 256
// equal blocks, of which 104 multiprocessors have two and 48 one, and by the
// instructions that unpack the codes.
constexpr int WARPS = 8;

// d = a b (first) or d += a b
template <typename T, bool FIRST>
__device__ __forceinline__ void mma16816(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
#define SN_MMA(TYPE)                                                                                                                  \
    if constexpr (FIRST)                                                                                                              \
        asm("mma.sync.aligned.m16n8k16.row.col.f32." TYPE "." TYPE ".f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %10, %10, %10};" \
            : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])                                                                         \
            : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(0.0f));                                               \
    else                                                                                                                              \
        asm("mma.sync.aligned.m16n8k16.row.col.f32." TYPE "." TYPE ".f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};" \
            : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])                                                                         \
            : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1))
    if constexpr (std::is_same<T, __half>::value) {
        SN_MMA("f16");
    } else {
        SN_MMA("bf16");
    }
#undef SN_MMA
}
__device__ __forceinline__ float ld_cluster_f32(uint32_t caddr) {
    float v;
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(caddr) : "memory");
    return v;
}
__device__ __forceinline__ uint4 ld_stream(const uint4 *p) {
    uint4 v;
    asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];"
                 : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
                 : "l"(p));
    return v;
}

struct FewP {
    Q4P q;
    int32_t rows, wk, s, phase;  // warps along k, blocks a cluster, tiles along k in shared memory at once
    int32_t vec;                 // x's rows begin at 16 bytes
    int64_t ldx, ldy;
};

// T: the operands' type, X: x's and y's, NC: groups of 8 columns, GLOG: log2 of the group, SB: scales are bf16 (not fp16)
template <typename T, typename X, int NC, int GLOG, bool SB>
__global__ void __launch_bounds__(WARPS * 32) q4_few_kernel(const __grid_constant__ FewP p, const X *__restrict__ x,
                                                            X *__restrict__ y) {
    constexpr int PL = std::is_same<X, float>::value ? 3 : 1, COLS = NC * 8, U = 4;
    constexpr bool G32 = GLOG == 5;
    extern __shared__ __align__(16) unsigned char smem[];
    float *red = reinterpret_cast<float *>(smem);                  // [WARPS][16][COLS]
    T *xs = reinterpret_cast<T *>(smem + WARPS * 16 * COLS * 4);   // [rows * PL][phase * 64 + 32]
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, g = lane / 4, t = lane % 4;
    const int rank = (int)(blockIdx.x % (unsigned)p.s), wn = WARPS / p.wk;
    const int nt0 = (int)(blockIdx.x / (unsigned)p.s) * wn, nt = nt0 + warp / p.wk, wki = warp % p.wk;
    const int b0 = (int)((int64_t)p.q.kb * rank / p.s), b1 = (int)((int64_t)p.q.kb * (rank + 1) / p.s);
    const bool live = nt < p.q.nt;
    const int ldxs = p.phase * 64 + 32;  // (columns of x half a bank row apart)
    float acc[NC][4];
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[c][i] = 0.0f;
    griddep_launch();

    // the warp's tiles along k, U to a batch, two batches in flight
    struct Batch {
        uint4 codes[U];
        uint32_t scales[U][G32 ? 2 : 1];
    };
    const uint4 *codes = p.q.codes + (int64_t)(live ? nt : 0) * p.q.kb * 32 + lane;
    const uint32_t *scales = p.q.scales + (int64_t)(live ? nt : 0) * p.q.kg * 8 + g;
    auto fetch = [&](Batch &f, int at, int end) {
        const uint4 *cp = codes + (int64_t)at * 32;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (at + u < end) {
                f.codes[u] = ld_stream(cp + u * 32);
                if constexpr (G32) {
                    f.scales[u][0] = __ldg(scales + (2 * (at + u)) * 8);
                    f.scales[u][1] = __ldg(scales + (2 * (at + u) + 1) * 8);
                } else {
                    f.scales[u][0] = __ldg(scales + ((at + u) >> (GLOG - 6 > 0 ? GLOG - 6 : 0)) * 8);
                }
            }
        }
    };
    // lane (g, t) reads columns g, g + 8, ... of B; behind the last column there is the
    // last one again (its products land in columns that nobody reads)
    const T *xcol[NC];
#pragma unroll
    for (int c = 0; c < NC; ++c) xcol[c] = xs + min(c * 8 + g, p.rows * PL - 1) * ldxs + 8 * t;
    // TI tiles side by side, from tile u of a batch on: their chains of dependent products
    // take turns (one after the other: 24.8 us instead of 18.1; the loads alone take
    // 11.1).  off: the first tile's columns in the phase
    constexpr int TI = NC == 1 ? 4 : NC == 2 ? 2 : 1;
    auto products = [&](const Batch &f, int u, int off) {
        float d[TI][NC][4];
        uint4 xv[TI][NC];
#pragma unroll
        for (int h = 0; h < 2; ++h) {  // halves of the tiles' columns
#pragma unroll
            for (int j = 0; j < TI; ++j)
#pragma unroll
                for (int c = 0; c < NC; ++c) xv[j][c] = *reinterpret_cast<const uint4 *>(xcol[c] + off + j * 64 + h * 32);
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int j = 0; j < TI; ++j) {
                    const uint4 &cw = f.codes[u + j];
                    const uint32_t w = h ? (i ? cw.w : cw.z) : (i ? cw.y : cw.x);
                    const uint32_t a[4] = {code_pair<T>(w, 0), code_pair<T>(w, 1), code_pair<T>(w, 2), code_pair<T>(w, 3)};
#pragma unroll
                    for (int c = 0; c < NC; ++c) {
                        if (i == 0 && (G32 || h == 0)) mma16816<T, true>(d[j][c], a, xv[j][c].x, xv[j][c].y);
                        else mma16816<T, false>(d[j][c], a, i ? xv[j][c].z : xv[j][c].x, i ? xv[j][c].w : xv[j][c].y);
                    }
                }
            if (G32 || h == 1) {
#pragma unroll
                for (int j = 0; j < TI; ++j) {
                    const float2 s = scale_pair(f.scales[u + j][G32 ? h : 0], SB);
#pragma unroll
                    for (int c = 0; c < NC; ++c) {
                        acc[c][0] = fmaf(d[j][c][0], s.x, acc[c][0]), acc[c][1] = fmaf(d[j][c][1], s.x, acc[c][1]);
                        acc[c][2] = fmaf(d[j][c][2], s.y, acc[c][2]), acc[c][3] = fmaf(d[j][c][3], s.y, acc[c][3]);
                    }
                }
            }
        }
    };
    auto one = [&](const Batch &f, int u, int off) {  // a single tile, where no TI are left
        float d[NC][4];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const uint4 &cw = f.codes[u];
            uint32_t a[2][4];
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) a[i][j] = code_pair<T>(h ? (i ? cw.w : cw.z) : (i ? cw.y : cw.x), j);
            const float2 s = scale_pair(f.scales[u][G32 ? h : 0], SB);
#pragma unroll
            for (int c = 0; c < NC; ++c) {
                const uint4 xv = *reinterpret_cast<const uint4 *>(xcol[c] + off + h * 32);
                if (G32 || h == 0) mma16816<T, true>(d[c], a[0], xv.x, xv.y);
                else mma16816<T, false>(d[c], a[0], xv.x, xv.y);
                mma16816<T, false>(d[c], a[1], xv.z, xv.w);
                if (G32 || h == 1) {
                    acc[c][0] = fmaf(d[c][0], s.x, acc[c][0]), acc[c][1] = fmaf(d[c][1], s.x, acc[c][1]);
                    acc[c][2] = fmaf(d[c][2], s.y, acc[c][2]), acc[c][3] = fmaf(d[c][3], s.y, acc[c][3]);
                }
            }
        }
    };
    bool first = true;
    for (int ph = b0; ph < b1; ph += p.phase) {
        const int pe = min(ph + p.phase, b1);
        const int w0 = ph + (pe - ph) * wki / p.wk, w1 = live ? ph + (pe - ph) * (wki + 1) / p.wk : w0;
        Batch f0, f1;  // (the weights do not depend on the kernel before)
        fetch(f0, w0, w1);
        fetch(f1, w0 + U, w1);
        if (first) griddep_wait();
        else __syncthreads();
        first = false;
        // the phase's columns of x, padded with zeros, eight at a time
        const int chunks = (pe - ph) * 8;
        for (int m = 0; m < p.rows; ++m) {
            const X *xr = x + m * p.ldx + (int64_t)ph * 64;
            if (PL == 1 && p.vec) {  // asynchronous copies, all in flight at once; zeros behind the row's end
                for (int c = threadIdx.x * 8; c < chunks * 8; c += WARPS * 32 * 8) {
                    const int left = max(0, min(8, p.q.k - ph * 64 - c));
                    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(tc::su32(xs + m * ldxs + c)),
                                 "l"(left ? xr + c : x), "r"(left * 2)
                                 : "memory");
                }
                continue;
            }
            for (int c = threadIdx.x * 8; c < chunks * 8; c += WARPS * 32 * 8) {
                const int left = p.q.k - ph * 64 - c;  // columns there are
                struct alignas(16) {
                    X v[8];
                } in;
                if (p.vec && left >= 8) {
                    const uint4 *src = reinterpret_cast<const uint4 *>(xr + c);
                    uint4 *dst = reinterpret_cast<uint4 *>(&in);
#pragma unroll
                    for (int i = 0; i < (int)sizeof(in) / 16; ++i) dst[i] = __ldg(src + i);
                } else {
#pragma unroll
                    for (int i = 0; i < 8; ++i) in.v[i] = i < left ? xr[c + i] : cvt<X>(0.0f);
                }
                if constexpr (PL == 3) {
                    struct alignas(16) {
                        T v[3][8];
                    } out;
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const Planes pl = planes_of(in.v[i]);
                        out.v[0][i] = pl.v[0], out.v[1][i] = pl.v[1], out.v[2][i] = pl.v[2];
                    }
#pragma unroll
                    for (int i = 0; i < 3; ++i)
                        *reinterpret_cast<uint4 *>(xs + (m * 3 + i) * ldxs + c) = reinterpret_cast<const uint4 *>(&out)[i];
                } else {
                    *reinterpret_cast<uint4 *>(xs + m * ldxs + c) = *reinterpret_cast<const uint4 *>(&in);
                }
            }
        }
        asm volatile("cp.async.wait_all;" ::: "memory");
        __syncthreads();
        int at = w0, off = (w0 - ph) * 64;
        for (; at + 4 * U <= w1; at += 2 * U, off += 2 * U * 64) {  // whole batches, whole batches ahead
#pragma unroll
            for (int u = 0; u < U; u += TI) products(f0, u, off + u * 64);
            fetch(f0, at + 2 * U, INT_MAX);
#pragma unroll
            for (int u = 0; u < U; u += TI) products(f1, u, off + (U + u) * 64);
            fetch(f1, at + 3 * U, INT_MAX);
        }
        for (; at < w1; at += 2 * U, off += 2 * U * 64) {
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (at + u < w1) one(f0, u, off + u * 64);
            fetch(f0, at + 2 * U, w1);
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (at + U + u < w1) one(f1, u, off + (U + u) * 64);
            fetch(f1, at + 3 * U, w1);
        }
    }
    if (first) griddep_wait();  // a block without columns of its own still may not leave early
    // the sums of the WK warps of a tile, then of the S blocks, in order
    float *mine = red + warp * 16 * COLS;
#pragma unroll
    for (int c = 0; c < NC; ++c) {
        *reinterpret_cast<float2 *>(mine + g * COLS + c * 8 + 2 * t) = make_float2(acc[c][0], acc[c][1]);
        *reinterpret_cast<float2 *>(mine + (g + 8) * COLS + c * 8 + 2 * t) = make_float2(acc[c][2], acc[c][3]);
    }
    __syncthreads();
    const int outs = wn * 16 * p.rows;  // output o: row o % 16 of tile o / 16 % wn, row of x o / (16 wn)
    auto block_sum = [&](int o) {
        const int r = o % 16, tile = o / 16 % wn, m = o / (16 * wn);
        float v = 0.0f;
        for (int i = 0; i < p.wk; ++i)
#pragma unroll
            for (int pl = PL - 1; pl >= 0; --pl) v += red[((tile * p.wk + i) * 16 + r) * COLS + m * PL + pl];
        return v;
    };
    auto finish = [&](int o, float v) {
        const int j = (nt0 + o / 16 % wn) * 16 + o % 16, m = o / (16 * wn);
        if (j < p.q.n) stf(y + m * p.ldy + j, q4_act(v + (p.q.bias ? p.q.bias[j] : 0.0f), p.q.act));
    };
    if (p.s == 1) {
        for (int o = threadIdx.x; o < outs; o += WARPS * 32) finish(o, block_sum(o));
        return;
    }
    float *part = reinterpret_cast<float *>(xs);  // the block's sums; x is done with
    for (int o = threadIdx.x; o < outs; o += WARPS * 32) part[o] = block_sum(o);
    tc::cluster_sync_all();
    for (int o = threadIdx.x * p.s + rank; o < outs; o += WARPS * 32 * p.s) {
        float v = 0.0f;
        for (int r = 0; r < p.s; ++r) v += ld_cluster_f32(tc::mapa(tc::su32(part + o), (uint32_t)r));
        finish(o, v);
    }
    tc::cluster_sync_all();  // peers may still be reading this block's sums
}

constexpr size_t X_SMEM = 64 << 10;  // shared memory for x

template <typename T, typename X, int NC, int GLOG, bool SB>
cudaError_t launch_few(const Q4P &q, int rows, const X *x, int64_t ldx, X *y, int64_t ldy, cudaStream_t st) {
    constexpr int PL = std::is_same<X, float>::value ? 3 : 1;
    // warps along k until there are about 12 a multiprocessor, at least 4 tiles each (two
    // blocks fit a multiprocessor: 25088 -> 4096 for one row in one wave 18.1 us, in two 22)
    FewP p{q, rows, 1, 1, 0, 0, ldx, ldy};
    p.vec = reinterpret_cast<uintptr_t>(x) % 16 == 0 && ldx * (int64_t)sizeof(X) % 16 == 0;
    const int64_t want = 12LL * num_sms();
    while (p.wk < WARPS && (int64_t)q.nt * p.wk < want && q.kb >= 8 * p.wk) p.wk *= 2;
    while (p.s < 8 && (int64_t)q.nt * p.wk * p.s < want && q.kb >= 8 * p.wk * p.s) p.s *= 2;
    const int fit = (int)(X_SMEM / (rows * PL * 128)) - 1;  // tiles along k that fit
    while (p.s < 8 && (q.kb + p.s - 1) / p.s > fit && q.kb >= 2 * p.s) p.s *= 2;
    p.phase = std::min((q.kb + p.s - 1) / p.s, fit);
    size_t smem = (size_t)WARPS * 16 * NC * 8 * 4;
    smem += std::max((size_t)rows * PL * (p.phase * 64 + 32) * 2, (size_t)WARPS / p.wk * 16 * rows * 4);
    auto kern = q4_few_kernel<T, X, NC, GLOG, SB>;
    static PerDevice set;
    if (const cudaError_t e = allow_smem(set, kern, X_SMEM + WARPS * 16 * NC * 8 * 4 + 1024)) return e;
    const int wn = WARPS / p.wk;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)((q.nt + wn - 1) / wn * p.s));
    cfg.blockDim = dim3(WARPS * 32);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)p.s;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = p.s > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, kern, p, x, y);
}

template <typename T, typename X, int GLOG, bool SB>
cudaError_t few_cols(const Q4P &q, int rows, const X *x, int64_t ldx, X *y, int64_t ldy, cudaStream_t st) {
    constexpr int PL = std::is_same<X, float>::value ? 3 : 1;
    switch ((rows * PL + 7) / 8) {
    case 1: return launch_few<T, X, 1, GLOG, SB>(q, rows, x, ldx, y, ldy, st);
    case 2: return launch_few<T, X, 2, GLOG, SB>(q, rows, x, ldx, y, ldy, st);
    case 3: return launch_few<T, X, 3, GLOG, SB>(q, rows, x, ldx, y, ldy, st);
    default: return launch_few<T, X, 4, GLOG, SB>(q, rows, x, ldx, y, ldy, st);
    }
}

template <typename T, typename X>
cudaError_t q4_few(const Q4P &q, int rows, const X *x, int64_t ldx, X *y, int64_t ldy, cudaStream_t st) {
    switch (q.glog) {
#define SN_GROUP(G)                                                                           \
    return q.scale_bf16 ? few_cols<T, X, G, true>(q, rows, x, ldx, y, ldy, st) : few_cols<T, X, G, false>(q, rows, x, ldx, y, ldy, st)
    case 5: SN_GROUP(5);
    case 6: SN_GROUP(6);
    default: SN_GROUP(7);
#undef SN_GROUP
    }
}

}  // namespace

}  // namespace k
}  // namespace sn
