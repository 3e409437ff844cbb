// 4-bit weights: quantisation, layout, and the product with few rows of x
// (sn_q4_quantize, sn_q4_pack, sn_q4_dense in include/sn.h; layout in q4_common.cuh).
#include <algorithm>
#include <climits>

#include "q4_common.cuh"

namespace sn {
namespace k {

namespace {

// -------------------------------------------------------- codes and scales
__device__ __forceinline__ float round_scale(float s, int bf16) {
    return bf16 ? __bfloat162float(__float2bfloat16_rn(s)) : __half2float(__float2half_rn(s));
}

// a warp a group of a row; group <= 128, so a lane has at most 4 weights, neighbours in pairs
template <typename T>
__global__ void __launch_bounds__(128) q4_quantize_kernel(const T *__restrict__ w, int64_t n, int64_t k, int group, int bf16,
                                                          uint8_t *__restrict__ codes, void *__restrict__ scales) {
    const int64_t kg = (k + group - 1) / group, id = (int64_t)blockIdx.x * 4 + threadIdx.x / 32;
    if (id >= n * kg) return;
    const int64_t row = id / kg, k0 = id % kg * group;
    const int lane = threadIdx.x % 32, len = (int)min((int64_t)group, k - k0);
    float v[2][2], m = 0.0f;
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int e = i * 64 + lane * 2 + j;
            v[i][j] = e < len ? ldf(w + row * k + k0 + e) : 0.0f;
            m = fmaxf(m, fabsf(v[i][j]));
        }
    for (int o = 16; o; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
    float s = round_scale(fminf(__fdiv_rn(m, 7.0f), bf16 ? 3.3895314e38f : 65504.0f), bf16);  // (the types' largest)
    if (!(s > 0.0f)) s = 1.0f;
    if (lane == 0) {
        if (bf16) static_cast<__nv_bfloat16 *>(scales)[id] = __float2bfloat16_rn(s);
        else static_cast<__half *>(scales)[id] = __float2half_rn(s);
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int e = i * 64 + lane * 2;
        if (e >= len) continue;
        int b = 0;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int q = max(-8, min(7, __float2int_rn(__fdiv_rn(v[i][j], s))));
            b |= (e + j < len ? q & 15 : 0) << (4 * j);
        }
        codes[row * ((k + 1) / 2) + (k0 + e) / 2] = (uint8_t)b;
    }
}

__device__ __forceinline__ uint32_t code_at(const uint8_t *codes, int64_t row, int64_t c, int64_t n, int64_t k) {
    if (row >= n || c >= k) return 8;
    return ((codes[row * ((k + 1) / 2) + c / 2] >> (4 * (c % 2))) & 15) ^ 8;
}

__global__ void __launch_bounds__(256) q4_pack_kernel(const uint8_t *__restrict__ codes, int64_t n, int64_t k, int64_t kb,
                                                      int64_t total, uint4 *__restrict__ out) {
    const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (id >= total) return;
    const int lane = (int)(id % 32), g = lane / 4, t = lane % 4;
    const int64_t tile = id / 32, row = tile / kb * 16 + g, c0 = tile % kb * 64 + 8 * t;
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        w[i] = 0;
        const int64_t c = c0 + 32 * (i / 2) + 4 * (i % 2);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int nib = (e / 2) * 2 + (e % 2) * 4;
            w[i] |= code_at(codes, row, c + e, n, k) << (4 * nib);
            w[i] |= code_at(codes, row + 8, c + e, n, k) << (4 * (nib + 1));
        }
    }
    out[id] = make_uint4(w[0], w[1], w[2], w[3]);
}

// a warp a row: its scales into place, and its power of two
__global__ void __launch_bounds__(128) q4_pack_scales_kernel(const uint16_t *__restrict__ scales, int bf16, int64_t n,
                                                             int64_t groups, int64_t kg, int64_t nt,
                                                             uint16_t *__restrict__ out, float *__restrict__ row_pow) {
    const int64_t row = (int64_t)blockIdx.x * 4 + threadIdx.x / 32;
    const int lane = threadIdx.x % 32, r = (int)(row % 16);
    if (row >= nt * 16) return;
    float m = 0.0f;
    for (int64_t i = lane; i < kg; i += 32) {
        const uint16_t s = row < n && i < groups ? scales[row * groups + i] : 0;
        out[(row / 16 * kg + i) * 16 + (r % 8) * 2 + r / 8] = s;
        const float v = bf16 ? __uint_as_float((uint32_t)s << 16) : __half2float(*reinterpret_cast<const __half *>(&s));
        m = fmaxf(m, fabsf(v));
    }
    for (int o = 16; o; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
    if (lane == 0) {
        int e = 0;
        if (m > 0.0f && m < INFINITY) frexpf(m, &e);
        row_pow[row] = ldexpf(1.0f, max(-126, min(126, e)));
    }
}

// ------------------------------------------------------------ few rows of x
// Bound by reading the weights (half a byte a product and row): 16 x 8 x 16
// products on the tensor cores with the codes as the A operand, x as columns of B
// (rows of fp32 x as three bf16 columns each), one fp32 multiply-add a group to
// scale its sum.  A warp runs along k over one 16-row tile, its weights straight
// from global memory to registers in the operand's layout, eight tiles in flight; the
// block's part of x lies in shared memory.  k is split over the WK warps of a
// block that share a tile and over the S blocks of a cluster, whose sums meet in a
// fixed order.
constexpr int WARPS = 8;

__device__ __forceinline__ void mma16816(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1, __half) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma16816(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1, __nv_bfloat16) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
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

// T: the operands' type, X: x's and y's, NC: groups of 8 columns, G32: two scales a tile
template <typename T, typename X, int NC, bool G32>
__global__ void __launch_bounds__(WARPS * 32) q4_few_kernel(const __grid_constant__ FewP p, const X *__restrict__ x,
                                                            X *__restrict__ y) {
    constexpr int PL = std::is_same<X, float>::value ? 3 : 1, COLS = NC * 8, U = 4;
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
                    f.scales[u][0] = __ldg(scales + ((at + u) >> (p.q.glog - 6)) * 8);
                }
            }
        }
    };
    // lane (g, t) reads columns g, g + 8, ... of B; behind the last column there is the
    // last one again (its products land in columns that nobody reads)
    const T *xcol[NC];
#pragma unroll
    for (int c = 0; c < NC; ++c) xcol[c] = xs + min(c * 8 + g, p.rows * PL - 1) * ldxs + 8 * t;
    auto products = [&](const Batch &f, int u, int off) {  // off: the tile's columns in the phase
        const uint32_t w[4] = {f.codes[u].x, f.codes[u].y, f.codes[u].z, f.codes[u].w};
        uint32_t a[4][4];
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) a[i][j] = code_pair<T>(w[i], j);
        const float2 s0 = scale_pair(f.scales[u][0], p.q.scale_bf16);
        const float2 s1 = G32 ? scale_pair(f.scales[u][G32 ? 1 : 0], p.q.scale_bf16) : s0;
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            const uint4 lo = *reinterpret_cast<const uint4 *>(xcol[c] + off), hi = *reinterpret_cast<const uint4 *>(xcol[c] + off + 32);
            float d[4] = {0.0f, 0.0f, 0.0f, 0.0f};
            mma16816(d, a[0], lo.x, lo.y, T{});
            mma16816(d, a[1], lo.z, lo.w, T{});
            if constexpr (G32) {
                acc[c][0] = fmaf(d[0], s0.x, acc[c][0]), acc[c][1] = fmaf(d[1], s0.x, acc[c][1]);
                acc[c][2] = fmaf(d[2], s0.y, acc[c][2]), acc[c][3] = fmaf(d[3], s0.y, acc[c][3]);
                d[0] = d[1] = d[2] = d[3] = 0.0f;
            }
            mma16816(d, a[2], hi.x, hi.y, T{});
            mma16816(d, a[3], hi.z, hi.w, T{});
            acc[c][0] = fmaf(d[0], s1.x, acc[c][0]), acc[c][1] = fmaf(d[1], s1.x, acc[c][1]);
            acc[c][2] = fmaf(d[2], s1.y, acc[c][2]), acc[c][3] = fmaf(d[3], s1.y, acc[c][3]);
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
            for (int u = 0; u < U; ++u) products(f0, u, off + u * 64);
            fetch(f0, at + 2 * U, INT_MAX);
#pragma unroll
            for (int u = 0; u < U; ++u) products(f1, u, off + (U + u) * 64);
            fetch(f1, at + 3 * U, INT_MAX);
        }
        for (; at < w1; at += 2 * U, off += 2 * U * 64) {
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (at + u < w1) products(f0, u, off + u * 64);
            fetch(f0, at + 2 * U, w1);
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (at + U + u < w1) products(f1, u, off + (U + u) * 64);
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
        if (j < p.q.n) stf(y + m * p.ldy + j, act_apply(v + (p.q.bias ? p.q.bias[j] : 0.0f), p.q.act));
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

constexpr int FEW_COLS = 32;       // columns of B that the kernel has
constexpr size_t X_SMEM = 64 << 10;  // shared memory for x

template <typename T, typename X, int NC, bool G32>
cudaError_t launch_few(const Q4P &q, int rows, const X *x, int64_t ldx, X *y, int64_t ldy, cudaStream_t st) {
    constexpr int PL = std::is_same<X, float>::value ? 3 : 1;
    // warps along k until there are about 16 a multiprocessor, at least 4 tiles each
    FewP p{q, rows, 1, 1, 0, 0, ldx, ldy};
    p.vec = reinterpret_cast<uintptr_t>(x) % 16 == 0 && ldx * (int64_t)sizeof(X) % 16 == 0;
    const int64_t want = 16LL * num_sms();
    while (p.wk < WARPS && (int64_t)q.nt * p.wk < want && q.kb >= 8 * p.wk) p.wk *= 2;
    while (p.s < 8 && (int64_t)q.nt * p.wk * p.s < want && q.kb >= 8 * p.wk * p.s) p.s *= 2;
    const int fit = (int)(X_SMEM / (rows * PL * 128)) - 1;  // tiles along k that fit
    while (p.s < 8 && (q.kb + p.s - 1) / p.s > fit && q.kb >= 2 * p.s) p.s *= 2;
    p.phase = std::min((q.kb + p.s - 1) / p.s, fit);
    size_t smem = (size_t)WARPS * 16 * NC * 8 * 4;
    smem += std::max((size_t)rows * PL * (p.phase * 64 + 32) * 2, (size_t)WARPS / p.wk * 16 * rows * 4);
    auto kern = q4_few_kernel<T, X, NC, G32>;
    static bool set = false;  // (idempotent)
    if (!set) {
        cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                             (int)(X_SMEM + WARPS * 16 * NC * 8 * 4 + 1024));
        if (e != cudaSuccess) return e;
        set = true;
    }
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

template <typename T, typename X, bool G32>
cudaError_t few_cols(const Q4P &q, int rows, const X *x, int64_t ldx, X *y, int64_t ldy, cudaStream_t st) {
    constexpr int PL = std::is_same<X, float>::value ? 3 : 1;
    switch ((rows * PL + 7) / 8) {
    case 1: return launch_few<T, X, 1, G32>(q, rows, x, ldx, y, ldy, st);
    case 2: return launch_few<T, X, 2, G32>(q, rows, x, ldx, y, ldy, st);
    case 3: return launch_few<T, X, 3, G32>(q, rows, x, ldx, y, ldy, st);
    default: return launch_few<T, X, 4, G32>(q, rows, x, ldx, y, ldy, st);
    }
}

template <typename T, typename X>
cudaError_t q4_few(const Q4P &q, int rows, const X *x, int64_t ldx, X *y, int64_t ldy, cudaStream_t st) {
    return q.glog == 5 ? few_cols<T, X, true>(q, rows, x, ldx, y, ldy, st) : few_cols<T, X, false>(q, rows, x, ldx, y, ldy, st);
}

// rows that fill the columns of the few-row kernel; more go to the tensor-core tiles
int few_rows(int dt) { return dt == SN_F32 ? FEW_COLS / 3 : FEW_COLS; }

}  // namespace

size_t q4_bytes(int64_t n, int64_t k, int group) { return (size_t)q4_layout(n, k, group).bytes; }

cudaError_t q4_quantize(const void *w, int dt, int64_t n, int64_t k, int group, int scale_dt, uint8_t *codes, void *scales,
                        cudaStream_t st) {
    const int64_t groups = n * ((k + group - 1) / group);
    const dim3 grid((unsigned)((groups + 3) / 4));
    SN_DT_SWITCH(dt, T, q4_quantize_kernel<T><<<grid, 128, 0, st>>>(static_cast<const T *>(w), n, k, group,
                                                                    scale_dt == SN_BF16, codes, scales))
    return cudaGetLastError();
}

cudaError_t q4_pack(const uint8_t *codes, const void *scales, const sn_q4_weights &w, cudaStream_t st) {
    const Q4Layout l = q4_layout(w.n, w.k, w.group);
    char *out = static_cast<char *>(w.packed);
    const int64_t total = l.nt * l.kb * 32, groups = (w.k + w.group - 1) / w.group;
    q4_pack_kernel<<<(unsigned)((total + 255) / 256), 256, 0, st>>>(codes, w.n, w.k, l.kb, total, reinterpret_cast<uint4 *>(out));
    cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return e;
    q4_pack_scales_kernel<<<(unsigned)(l.nt * 4), 128, 0, st>>>(static_cast<const uint16_t *>(scales), w.scale_dtype == SN_BF16,
                                                                w.n, groups, l.kg, l.nt,
                                                                reinterpret_cast<uint16_t *>(out + l.scales_at),
                                                                reinterpret_cast<float *>(out + l.pow_at));
    e = cudaGetLastError();
    return e != cudaSuccess ? e : cudaStreamSynchronize(st);
}

size_t q4_workspace(const sn_q4_weights &w, int dt, int64_t rows, const void *x, int64_t ldx) {
    return rows <= few_rows(dt) ? 0 : q4_prompt_workspace(w, dt, rows, x, ldx);
}

cudaError_t q4_dense(const sn_q4_weights &w, int dt, int64_t rows, const void *x, int64_t ldx, void *y, int64_t ldy,
                     void *work, cudaStream_t st) {
    if (rows > few_rows(dt)) return q4_prompt(w, dt, rows, x, ldx, y, ldy, work, st);
    const Q4P q = q4_params(w);
    const int m = (int)rows;
    if (dt == SN_F32)
        return q4_few<__nv_bfloat16, float>(q, m, static_cast<const float *>(x), ldx, static_cast<float *>(y), ldy, st);
    if (dt == SN_F16)
        return q4_few<__half, __half>(q, m, static_cast<const __half *>(x), ldx, static_cast<__half *>(y), ldy, st);
    return q4_few<__nv_bfloat16, __nv_bfloat16>(q, m, static_cast<const __nv_bfloat16 *>(x), ldx,
                                                static_cast<__nv_bfloat16 *>(y), ldy, st);
}

}  // namespace k
}  // namespace sn
