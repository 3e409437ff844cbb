// The norms behind and before a block, fused with the block's gate, its residual
// scale and the sum into the residual stream (sn_block_norm in include/sn.h):
//   t = post(y g) or g post(y),  sum = residual + scale t,  normed = pre(sum).
//
// Bound by memory: y, gate and residual are read once, sum and normed written
// once.  A row stays in registers between its statistics, its sum and its second
// statistics, so nothing is read twice; mean and variance are two reductions over
// the registers (the variance of v - mean, not a difference of squares).
//
// Three kernels.  Many rows of up to 4096 aligned values: persistent blocks, a
// thread's weights in its registers; the next rows come by bulk copies into a ring
// of shared memory while one is worked on.  Few or
// unaligned rows, or up to 8192 values: a block (or a warp) a row, straight from
// global memory.  Longer rows: a block a row, the row read again for each statistic.
// 8190 x 4096, bf16 with an fp32 residual: the block a row took 208 us (the loads of
// a block wait while it reduces, and the weights go through L1 for every row), the ring
// takes 82: 5700 GB/s, 84% of a copy's.
#include <algorithm>

#include "tc_common.cuh"

namespace sn {
namespace k {

namespace {

constexpr int PIECE = 8;  // elements a thread handles together: 16 bytes of a 16-bit type

struct NormP {
    NormArgs a;
    const float *post, *post_b, *pre, *pre_b, *scale;
    int32_t d, kind, gate, after, vec;
    float eps;
};

template <typename T>
__device__ __forceinline__ void load_piece(float (&v)[PIECE], const T *row, int at, int d, bool vec) {
    if (vec && at + PIECE <= d) {
        if constexpr (sizeof(T) == 4) {
            const float4 a = *reinterpret_cast<const float4 *>(row + at), b = *reinterpret_cast<const float4 *>(row + at + 4);
            v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w, v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
        } else {
            uint4 u = *reinterpret_cast<const uint4 *>(row + at);
            const T *e = reinterpret_cast<const T *>(&u);
#pragma unroll
            for (int i = 0; i < PIECE; ++i) v[i] = ldf(e + i);
        }
    } else {
#pragma unroll
        for (int i = 0; i < PIECE; ++i) v[i] = at + i < d ? ldf(row + at + i) : 0.0f;
    }
}
template <typename T>
__device__ __forceinline__ void store_piece(T *row, const float (&v)[PIECE], int at, int d, bool vec) {
    if (vec && at + PIECE <= d) {
        if constexpr (sizeof(T) == 4) {
            *reinterpret_cast<float4 *>(row + at) = make_float4(v[0], v[1], v[2], v[3]);
            *reinterpret_cast<float4 *>(row + at + 4) = make_float4(v[4], v[5], v[6], v[7]);
        } else {
            uint4 u;
            T *e = reinterpret_cast<T *>(&u);
#pragma unroll
            for (int i = 0; i < PIECE; ++i) e[i] = cvt<T>(v[i]);
            *reinterpret_cast<uint4 *>(row + at) = u;
        }
    } else {
#pragma unroll
        for (int i = 0; i < PIECE; ++i)
            if (at + i < d) stf(row + at + i, v[i]);
    }
}

__device__ __forceinline__ float gate_value(float g, int kind) {
    if (kind == SN_GATE_LINEAR) return g;
    // by the approximate exponential and division, 2 ulp each (a denominator beyond 2^126 gives 0)
    return __fdividef(kind == SN_GATE_SIGMOID ? 1.0f : g, 1.0f + __expf(-g));
}

// the sum over the row's TPR threads, the same in each of them
template <int TPR>
__device__ __forceinline__ float row_sum(float v, float *sh) {
#pragma unroll
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    if constexpr (TPR > 32) {
        const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
        __syncthreads();  // the previous sum has been read
        if (lane == 0) sh[warp] = v;
        __syncthreads();
        v = lane < TPR / 32 ? sh[lane] : 0.0f;
#pragma unroll
        for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    }
    return v;
}

// norm of the values in registers, in place; entries behind the row's end are zero before and ignored after
template <int TPR, int NP>
__device__ __forceinline__ void norm_row(float (&v)[NP][PIECE], const NormP &p, const float *w, const float *b, int t,
                                         float *sh) {
    const float inv_d = 1.0f / (float)p.d;
    if (p.kind == SN_NORM_LAYER) {
        float s = 0.0f;
#pragma unroll
        for (int i = 0; i < NP; ++i)
#pragma unroll
            for (int j = 0; j < PIECE; ++j) s += v[i][j];
        const float mean = row_sum<TPR>(s, sh) * inv_d;
#pragma unroll
        for (int i = 0; i < NP; ++i)
#pragma unroll
            for (int j = 0; j < PIECE; ++j) v[i][j] = (t + i * TPR) * PIECE + j < p.d ? v[i][j] - mean : 0.0f;
    }
    float s = 0.0f;
#pragma unroll
    for (int i = 0; i < NP; ++i)
#pragma unroll
        for (int j = 0; j < PIECE; ++j) s = fmaf(v[i][j], v[i][j], s);
    const float r = rsqrtf(row_sum<TPR>(s, sh) * inv_d + p.eps);
#pragma unroll
    for (int i = 0; i < NP; ++i) {
        const int at = (t + i * TPR) * PIECE;
        if (at >= p.d) break;
        float wv[PIECE], bv[PIECE];
        load_piece(wv, w, at, p.d, p.vec);
        if (b) load_piece(bv, b, at, p.d, p.vec);
#pragma unroll
        for (int j = 0; j < PIECE; ++j) v[i][j] = b ? fmaf(v[i][j] * r, wv[j], bv[j]) : v[i][j] * r * wv[j];
    }
}

template <typename T, typename R, int TPR, int NP>
__global__ void __launch_bounds__(TPR < 128 ? 128 : TPR) block_norm_kernel(const __grid_constant__ NormP p) {
    constexpr int RPB = TPR < 128 ? 128 / TPR : 1;
    __shared__ float sh[32];
    const int t = threadIdx.x % TPR;
    const int64_t row = (int64_t)blockIdx.x * RPB + threadIdx.x / TPR;
    griddep_launch();
    griddep_wait();
    if (row >= p.a.rows) return;  // whole warps: TPR is 32 where a block has several rows
    const T *y = static_cast<const T *>(p.a.y), *gate = static_cast<const T *>(p.a.gate);
    const R *res = static_cast<const R *>(p.a.res);
    float v[NP][PIECE], g[NP][PIECE], r[NP][PIECE];
#pragma unroll
    for (int i = 0; i < NP; ++i) {
        const int at = (t + i * TPR) * PIECE;
        if (y) load_piece(v[i], y + row * p.a.ldy, at, p.d, p.vec);
        if (gate) load_piece(g[i], gate + (row / p.a.per_gate) * p.a.ldg, at, p.d, p.vec);
        if (res) load_piece(r[i], res + row * p.a.ldr, at, p.d, p.vec);
    }
    if (y) {
        if (gate) {
#pragma unroll
            for (int i = 0; i < NP; ++i)
#pragma unroll
                for (int j = 0; j < PIECE; ++j) {
                    // (a gate behind the row's end multiplies a zero)
                    g[i][j] = (t + i * TPR) * PIECE + j < p.d ? gate_value(g[i][j], p.gate) : 1.0f;
                    if (!p.after) v[i][j] *= g[i][j];
                }
        }
        if (p.post) norm_row<TPR, NP>(v, p, p.post, p.post_b, t, sh);
        if (gate && p.after) {
#pragma unroll
            for (int i = 0; i < NP; ++i)
#pragma unroll
                for (int j = 0; j < PIECE; ++j) v[i][j] *= g[i][j];
        }
        if (p.scale) {
#pragma unroll
            for (int i = 0; i < NP; ++i) {
                const int at = (t + i * TPR) * PIECE;
                if (at >= p.d) break;
                float s[PIECE];
                load_piece(s, p.scale, at, p.d, p.vec);
#pragma unroll
                for (int j = 0; j < PIECE; ++j) v[i][j] *= s[j];
            }
        }
        if (res) {
#pragma unroll
            for (int i = 0; i < NP; ++i)
#pragma unroll
                for (int j = 0; j < PIECE; ++j) v[i][j] += r[i][j];
        }
    } else {
#pragma unroll
        for (int i = 0; i < NP; ++i)
#pragma unroll
            for (int j = 0; j < PIECE; ++j) v[i][j] = r[i][j];
    }
    if (p.a.sum) {
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            const int at = (t + i * TPR) * PIECE;
            if (res) store_piece(static_cast<R *>(p.a.sum) + row * p.a.lds, v[i], at, p.d, p.vec);
            else store_piece(static_cast<T *>(p.a.sum) + row * p.a.lds, v[i], at, p.d, p.vec);
        }
    }
    if (p.pre) {
        // what lies behind the row's end is zero again: the post norm's and scale's loops stop there, and sums of zeros are zero
        norm_row<TPR, NP>(v, p, p.pre, p.pre_b, t, sh);
#pragma unroll
        for (int i = 0; i < NP; ++i)
            store_piece(static_cast<T *>(p.a.normed) + row * p.a.ldn, v[i], (t + i * TPR) * PIECE, p.d, p.vec);
    }
}

// Rows too long for registers: a block a row, each statistic a pass over it (the
// later ones from L2), the values formed again in each pass.
template <typename T, typename R>
__global__ void __launch_bounds__(1024) block_norm_long_kernel(const __grid_constant__ NormP p) {
    __shared__ float sh[32];
    const int64_t row = blockIdx.x;
    griddep_launch();
    griddep_wait();
    const T *y = p.a.y ? static_cast<const T *>(p.a.y) + row * p.a.ldy : nullptr;
    const T *gate = p.a.gate ? static_cast<const T *>(p.a.gate) + (row / p.a.per_gate) * p.a.ldg : nullptr;
    const R *res = p.a.res ? static_cast<const R *>(p.a.res) + row * p.a.ldr : nullptr;
    const float inv_d = 1.0f / (float)p.d;
    float m1 = 0.0f, r1 = 1.0f, m2 = 0.0f, r2 = 1.0f;
    auto inner = [&](int i) {
        float v = ldf(y + i);
        return gate && !p.after ? v * gate_value(ldf(gate + i), p.gate) : v;
    };
    auto outer = [&](int i) {
        float v = 0.0f;
        if (y) {
            v = inner(i);
            if (p.post) v = fmaf((v - m1) * r1, p.post[i], p.post_b ? p.post_b[i] : 0.0f);
            if (gate && p.after) v *= gate_value(ldf(gate + i), p.gate);
            if (p.scale) v *= p.scale[i];
        }
        return res ? v + ldf(res + i) : v;
    };
    auto stats = [&](auto value, float &m, float &r) {
        if (p.kind == SN_NORM_LAYER) {
            float s = 0.0f;
            for (int i = threadIdx.x; i < p.d; i += blockDim.x) s += value(i);
            m = row_sum<1024>(s, sh) * inv_d;
        }
        float s = 0.0f;
        for (int i = threadIdx.x; i < p.d; i += blockDim.x) {
            const float c = value(i) - m;
            s = fmaf(c, c, s);
        }
        r = rsqrtf(row_sum<1024>(s, sh) * inv_d + p.eps);
    };
    if (y && p.post) stats(inner, m1, r1);
    if (p.pre) stats(outer, m2, r2);
    for (int i = threadIdx.x; i < p.d; i += blockDim.x) {  // (an output may be an input: each element is read before it is written)
        const float v = outer(i);
        if (p.a.sum) {
            if (res) stf(static_cast<R *>(p.a.sum) + row * p.a.lds + i, v);
            else stf(static_cast<T *>(p.a.sum) + row * p.a.lds + i, v);
        }
        if (p.pre)
            stf(static_cast<T *>(p.a.normed) + row * p.a.ldn + i, fmaf((v - m2) * r2, p.pre[i], p.pre_b ? p.pre_b[i] : 0.0f));
    }
}

// Many rows: block b takes the rows b, b + gridDim, ...; row i of the block lies in
// stage i % stages, filled by one thread's bulk copies of y, gate and residual.
constexpr int RING_MAX = 8;
struct RingP {
    NormP n;
    int32_t stages, stage_bytes, gate_at, res_at;  // offsets of the parts of a stage
    int *err;
};
__device__ __forceinline__ void bulk_load(uint32_t dst, const void *src, uint32_t bytes, uint64_t *bar) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst),
                 "l"(reinterpret_cast<uint64_t>(src)), "r"(bytes), "r"(tc::su32(bar))
                 : "memory");
}
// the sum over the block; sums take turns with the two halves of sh, so that one barrier each is enough
__device__ __forceinline__ float block_sum(float v, float *sh, int &turn) {
#pragma unroll
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    const int lane = threadIdx.x % 32;
    float *half = sh + 32 * (turn ^= 1);
    if (lane == 0) half[threadIdx.x / 32] = v;
    __syncthreads();
    v = lane < (int)blockDim.x / 32 ? half[lane] : 0.0f;
#pragma unroll
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

template <typename T>
__device__ __forceinline__ void load4(float *v, const T *src) {
    if constexpr (sizeof(T) == 4) {
        const float4 a = *reinterpret_cast<const float4 *>(src);
        v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w;
    } else {
        const uint2 a = *reinterpret_cast<const uint2 *>(src);
        const float2 x = tc::unpack2<T>(a.x), y = tc::unpack2<T>(a.y);
        v[0] = x.x, v[1] = x.y, v[2] = y.x, v[3] = y.y;
    }
}
template <typename T>
__device__ __forceinline__ void store4(T *dst, const float *v) {
    if constexpr (sizeof(T) == 4) *reinterpret_cast<float4 *>(dst) = make_float4(v[0], v[1], v[2], v[3]);
    else *reinterpret_cast<uint2 *>(dst) = make_uint2(tc::pack2<T>(v[0], v[1]), tc::pack2<T>(v[2], v[3]));
}

template <typename T, typename R, int NP>
__global__ void __launch_bounds__(256, 2) block_norm_ring_kernel(const __grid_constant__ RingP q) {
    constexpr int V = 4 * NP;
    extern __shared__ __align__(128) uint8_t ring[];
    __shared__ __align__(8) uint64_t full[RING_MAX];
    __shared__ float sh[64];
    __shared__ int stop_sh;
    const NormP &p = q.n;
    // a thread's values: four neighbours every blockDim fours, so that a warp's
    // accesses to fp32 rows are as contiguous as those to 16-bit ones
    const int at = threadIdx.x * 4, hop = blockDim.x * 4;
    const int64_t step = gridDim.x;
    if (threadIdx.x == 0) {
        for (int i = 0; i < q.stages; ++i) tc::mbar_init(&full[i], 1);
        stop_sh = 0;
        tc::fence_mbar_init();
    }
    __syncthreads();
    griddep_launch();
    griddep_wait();
    const uint32_t tb = (uint32_t)p.d * sizeof(T), rb = (uint32_t)p.d * sizeof(R);
    int64_t ahead = blockIdx.x;  // the next row to load, and its stage
    int s_ahead = 0;
    auto issue = [&]() {
        const int64_t row = ahead;
        const int s = s_ahead;
        ahead += step;
        s_ahead = s + 1 == q.stages ? 0 : s + 1;
        const uint32_t dst = tc::su32(ring) + (uint32_t)(s * q.stage_bytes);
        tc::mbar_expect_tx(&full[s], (p.a.y ? tb : 0u) + (p.a.gate ? tb : 0u) + (p.a.res ? rb : 0u));
        if (p.a.y) bulk_load(dst, static_cast<const T *>(p.a.y) + row * p.a.ldy, tb, &full[s]);
        if (p.a.gate)
            bulk_load(dst + q.gate_at, static_cast<const T *>(p.a.gate) + (p.a.per_gate == 1 ? row : row / p.a.per_gate) * p.a.ldg, tb,
                      &full[s]);
        if (p.a.res) bulk_load(dst + q.res_at, static_cast<const R *>(p.a.res) + row * p.a.ldr, rb, &full[s]);
    };
    if (threadIdx.x == 0)
        for (int i = 0; i < q.stages && ahead < p.a.rows; ++i) issue();
    // this thread's weights: the post norm's times the scale, and the pre norm's (zero
    // behind the row's end, so that nothing there counts; biases are read in place)
    float w[V], u[V];
#pragma unroll
    for (int i = 0; i < NP; ++i) {
        const int c = at + i * hop;
#pragma unroll
        for (int j = 0; j < 4; ++j) w[4 * i + j] = u[4 * i + j] = c < p.d ? 1.0f : 0.0f;
        if (c >= p.d) continue;
        if (p.post) load4(w + 4 * i, p.post + c);
        if (p.scale) {
            float f[4];
            load4(f, p.scale + c);
#pragma unroll
            for (int j = 0; j < 4; ++j) w[4 * i + j] *= f[j];
        }
        if (p.pre) load4(u + 4 * i, p.pre + c);
    }
    const float inv_d = 1.0f / (float)p.d;
    int turn = 0;
    // v centred (layer), and its factor 1 / sqrt(mean square + eps)
    auto stats = [&](float (&v)[V]) {
        if (p.kind == SN_NORM_LAYER) {
            float s = 0.0f;
#pragma unroll
            for (int j = 0; j < V; ++j) s += v[j];
            const float mean = block_sum(s, sh, turn) * inv_d;
#pragma unroll
            for (int i = 0; i < NP; ++i)
                if (at + i * hop < p.d) {
#pragma unroll
                    for (int j = 0; j < 4; ++j) v[4 * i + j] -= mean;
                }
        }
        float s[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int j = 0; j < V; ++j) s[j % 4] = fmaf(v[j], v[j], s[j % 4]);
        return rsqrtf(block_sum((s[0] + s[1]) + (s[2] + s[3]), sh, turn) * inv_d + p.eps);
    };
    // += bias (times scale), of the row's values there are
    auto add_bias = [&](float (&v)[V], const float *b, const float *scale) {
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            const int c = at + i * hop;
            if (c >= p.d) break;
            float f[4], g[4] = {1.0f, 1.0f, 1.0f, 1.0f};
            load4(f, b + c);
            if (scale) load4(g, scale + c);
#pragma unroll
            for (int j = 0; j < 4; ++j) v[4 * i + j] = fmaf(f[j], g[j], v[4 * i + j]);
        }
    };
    int s = 0;
    uint32_t par = 0;
    for (int64_t row = blockIdx.x; row < p.a.rows; row += step) {
        if (!tc::mbar_wait(&full[s], par)) stop_sh = 1;
        const uint8_t *st = ring + s * q.stage_bytes;
        float v[V], g[V], r[V];
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            const int c = at + i * hop;
            const bool in = c < p.d;
#pragma unroll
            for (int j = 0; j < 4; ++j) v[4 * i + j] = g[4 * i + j] = r[4 * i + j] = 0.0f;
            if (in && p.a.y) load4(v + 4 * i, reinterpret_cast<const T *>(st) + c);
            if (in && p.a.gate) load4(g + 4 * i, reinterpret_cast<const T *>(st + q.gate_at) + c);
            if (in && p.a.res) load4(r + 4 * i, reinterpret_cast<const R *>(st + q.res_at) + c);
        }
        __syncthreads();  // the stage has been read
        if (stop_sh) break;
        if (threadIdx.x == 0 && ahead < p.a.rows) issue();
        if (p.a.y) {
            if (p.a.gate) {
                if (p.gate != SN_GATE_LINEAR) {
                    const bool sig = p.gate == SN_GATE_SIGMOID;
#pragma unroll
                    for (int j = 0; j < V; ++j) g[j] = __fdividef(sig ? 1.0f : g[j], 1.0f + __expf(-g[j]));
                }
                if (!p.after) {
#pragma unroll
                    for (int j = 0; j < V; ++j) v[j] *= g[j];
                }
            }
            if (p.post) {
                const float f = stats(v);
#pragma unroll
                for (int j = 0; j < V; ++j) v[j] *= f * w[j];
                if (p.post_b) add_bias(v, p.post_b, p.scale);
            } else if (p.scale) {
#pragma unroll
                for (int j = 0; j < V; ++j) v[j] *= w[j];
            }
            if (p.a.gate && p.after) {
#pragma unroll
                for (int j = 0; j < V; ++j) r[j] = fmaf(v[j], g[j], r[j]);
            } else {
#pragma unroll
                for (int j = 0; j < V; ++j) r[j] += v[j];
            }
        }
        if (p.a.sum) {
            if (p.a.res) {
                R *o = static_cast<R *>(p.a.sum) + row * p.a.lds;
#pragma unroll
                for (int i = 0; i < NP; ++i)
                    if (at + i * hop < p.d) store4(o + at + i * hop, r + 4 * i);
            } else {
                T *o = static_cast<T *>(p.a.sum) + row * p.a.lds;
#pragma unroll
                for (int i = 0; i < NP; ++i)
                    if (at + i * hop < p.d) store4(o + at + i * hop, r + 4 * i);
            }
        }
        if (p.pre) {
            const float f = stats(r);
#pragma unroll
            for (int j = 0; j < V; ++j) r[j] *= f * u[j];
            if (p.pre_b) add_bias(r, p.pre_b, nullptr);
            T *o = static_cast<T *>(p.a.normed) + row * p.a.ldn;
#pragma unroll
            for (int i = 0; i < NP; ++i)
                if (at + i * hop < p.d) store4(o + at + i * hop, r + 4 * i);
        }
        if (++s == q.stages) {
            s = 0;
            par ^= 1u;
        }
    }
    if (threadIdx.x == 0 && stop_sh) {  // a wait gave up: record it, and let the copies in flight land (bounded)
        atomicOr(q.err, tc::ERR_TMA_WAIT);
        const long long t0 = clock64();
        for (int i = 0; i < q.stages; ++i)
            while (!tc::mbar_try(&full[(s + i) % q.stages], (s + i < q.stages) ? par : par ^ 1u) &&
                   clock64() - t0 < tc::WAIT_LIMIT) {
            }
    }
}

template <typename T, typename R, int NP>
cudaError_t launch_ring_np(const RingP &q, int threads, cudaStream_t st) {
    const int per_sm = 512 / threads, room = 220 * 1024 / per_sm;  // blocks a multiprocessor, shared memory of each
    static PerDevice set;
    if (const cudaError_t e = allow_smem(set, block_norm_ring_kernel<T, R, NP>, 110 * 1024)) return e;
    RingP p = q;
    p.stages = std::min(RING_MAX, room / q.stage_bytes);
    const int64_t blocks = std::min<int64_t>(q.n.a.rows, (int64_t)per_sm * num_sms());
    return launch_pdl(block_norm_ring_kernel<T, R, NP>, dim3((unsigned)blocks), dim3((unsigned)threads),
                      (size_t)(p.stages * p.stage_bytes), st, p);
}

template <typename T, typename R>
cudaError_t launch_ring(const NormP &p, cudaStream_t st) {
    RingP q{p, 0, 0, 0, 0, device_error_word()};
    auto up = [](int64_t b) { return (int32_t)((b + 127) / 128 * 128); };
    const int32_t tb = up((int64_t)p.d * sizeof(T)), rb = up((int64_t)p.d * sizeof(R));
    q.gate_at = p.a.y ? tb : 0;
    q.res_at = q.gate_at + (p.a.gate ? tb : 0);
    q.stage_bytes = q.res_at + (p.a.res ? rb : 0);
    if (p.d > 2048) return launch_ring_np<T, R, 4>(q, 256, st);
    if (p.d > 1024) return launch_ring_np<T, R, 2>(q, 256, st);
    return launch_ring_np<T, R, 2>(q, 128, st);
}

template <typename T, typename R, int TPR, int NP>
cudaError_t launch_rows(const NormP &p, cudaStream_t st) {
    constexpr int RPB = TPR < 128 ? 128 / TPR : 1;
    return launch_pdl(block_norm_kernel<T, R, TPR, NP>, dim3((unsigned)((p.a.rows + RPB - 1) / RPB)),
                      dim3(TPR < 128 ? 128 : TPR), 0, st, p);
}

template <typename T, typename R>
cudaError_t launch_norm(const NormP &p, cudaStream_t st) {
    const int pieces = (p.d + PIECE - 1) / PIECE;
    // the ring pays from the second row of a block on, and for rows that fill a block's warps
    if (p.vec && p.d % PIECE == 0 && p.d >= 512 && p.d <= 4096 && p.a.rows >= 4 * num_sms()) return launch_ring<T, R>(p, st);
    if (pieces <= 32) return launch_rows<T, R, 32, 1>(p, st);
    if (pieces <= 64) return launch_rows<T, R, 32, 2>(p, st);
    if (pieces <= 128) return launch_rows<T, R, 128, 1>(p, st);
    if (pieces <= 256) return launch_rows<T, R, 128, 2>(p, st);
    if (pieces <= 512) return launch_rows<T, R, 256, 2>(p, st);
    if (pieces <= 1024) return launch_rows<T, R, 512, 2>(p, st);
    return launch_pdl(block_norm_long_kernel<T, R>, dim3((unsigned)p.a.rows), dim3(1024), 0, st, p);
}

}  // namespace

cudaError_t block_norm(const sn_norm_params &q, int dt, int res_dt, const NormArgs &a, cudaStream_t st) {
    NormP p{a, q.post, q.post_bias, q.pre, q.pre_bias, q.scale, q.dim, q.kind, q.gate, q.gate_after, 0, q.eps};
    const int64_t es = dt == SN_F32 ? 4 : 2, rs = a.res ? (res_dt == SN_F32 ? 4 : 2) : es;
    auto ok = [](const void *ptr, int64_t stride_bytes) {
        return !ptr || (reinterpret_cast<uintptr_t>(ptr) % 16 == 0 && stride_bytes % 16 == 0);
    };
    p.vec = ok(a.y, a.ldy * es) && ok(a.gate, a.ldg * es) && ok(a.res, a.ldr * rs) && ok(a.sum, a.lds * rs) &&
            ok(a.normed, a.ldn * es) && ok(q.post, 0) && ok(q.post_bias, 0) && ok(q.pre, 0) && ok(q.pre_bias, 0) &&
            ok(q.scale, 0);
    if (dt == SN_F32) return launch_norm<float, float>(p, st);
    if (dt == SN_F16) return res_dt == SN_F32 ? launch_norm<__half, float>(p, st) : launch_norm<__half, __half>(p, st);
    return res_dt == SN_F32 ? launch_norm<__nv_bfloat16, float>(p, st) : launch_norm<__nv_bfloat16, __nv_bfloat16>(p, st);
}

}  // namespace k
}  // namespace sn
