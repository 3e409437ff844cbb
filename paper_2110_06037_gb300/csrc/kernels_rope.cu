// Norms of queries and keys for each head with the position rotation, one pass
// (sn_head_rope in include/sn.h).
//
//   v' = norm(v) * w over the head;  (a, b) -> (a cos t - b sin t, a sin t + b cos t),  t = pos f
//
// Angles: f / 2 pi is kept as a 64-bit fraction, and pos times it modulo 2^64 is the angle modulo one
// turn, exactly but for the fraction's own 2^-65 a position.  Its nearest quarter turn is taken off in
// integers; the rest, below an eighth of a turn, is exact to 2^-25 of itself in fp32 and goes to sincospif.
//
// A head is cut into slots of two values: a pair that turns, or two neighbours behind the pairs.  A lane
// has W slots in a row (two loads of W values) NC times, LPH lanes a head, 32 / LPH heads a warp, so that
// a pair's two values meet in one lane, its angle is computed once a lane and token and serves all heads
// that the lane sees, and only the norm's sums cross lanes.
#include <algorithm>

#include "kern_common.cuh"

namespace sn {
namespace k {

namespace {

struct RopeP {
    HeadsArgs h[2];
    int64_t tokens;
    const int32_t *pos, *axis;
    const uint64_t *turns;
    int32_t d, pairs, axes, norm, interleaved;
    int32_t split;  // warps a token
    float eps;
};

template <typename T, int W>
__device__ __forceinline__ void load_w(float *v, const T *p) {
    constexpr int B = W * sizeof(T);
    if constexpr (B == 16 || B == 8 || B == 4) {
        using U = typename std::conditional<B == 16, uint4, typename std::conditional<B == 8, uint2, uint32_t>::type>::type;
        U u = *reinterpret_cast<const U *>(p);
        const T *t = reinterpret_cast<const T *>(&u);
#pragma unroll
        for (int i = 0; i < W; ++i) v[i] = ldf(t + i);
    } else {
#pragma unroll
        for (int i = 0; i < W; ++i) v[i] = ldf(p + i);
    }
}
template <typename T, int W>
__device__ __forceinline__ void store_w(T *p, const float *v) {
    constexpr int B = W * sizeof(T);
    if constexpr (B == 16 || B == 8 || B == 4) {
        using U = typename std::conditional<B == 16, uint4, typename std::conditional<B == 8, uint2, uint32_t>::type>::type;
        U u;
        T *t = reinterpret_cast<T *>(&u);
#pragma unroll
        for (int i = 0; i < W; ++i) stf(t + i, v[i]);
        *reinterpret_cast<U *>(p) = u;
    } else {
#pragma unroll
        for (int i = 0; i < W; ++i) stf(p + i, v[i]);
    }
}

__device__ __forceinline__ void turn(uint64_t angle, float &c, float &s) {
    const uint32_t u = (uint32_t)(angle >> 32);
    const uint32_t quarter = (u + (1u << 29)) >> 30;
    const float r = (float)(int32_t)(u - (quarter << 30)) * (1.0f / 2147483648.0f);  // half turns
    float sn, cs;
    sincospif(r, &sn, &cs);
    const bool swap = quarter & 1u;
    c = swap ? sn : cs, s = swap ? cs : sn;
    if (((quarter + 1u) & 2u) != 0) c = -c;
    if ((quarter & 2u) != 0) s = -s;
}

template <typename T, int W, int NC>
__global__ void __launch_bounds__(256) head_rope_kernel(const __grid_constant__ RopeP p, int lph) {
    constexpr int V = 2 * W * NC;
    griddep_launch();
    griddep_wait();
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, sub = lane % lph, per = 32 / lph;
    const int64_t id = (int64_t)blockIdx.x * 8 + warp;
    const int64_t t = id / p.split;
    if (t >= p.tokens) return;
    const int part = (int)(id - t * p.split);
    // this lane's slots: where their values lie, and their turns
    int at[NC], bt[NC];
    float cs[NC * W], sn[NC * W];
    bool in[NC];
#pragma unroll
    for (int i = 0; i < NC; ++i) {
        const int c = (sub + i * lph) * W;
        in[i] = c < p.d / 2;
        const bool turns = c < p.pairs;
        at[i] = turns && !p.interleaved ? c : 2 * c;
        bt[i] = turns && !p.interleaved ? c + p.pairs : 2 * c + W;
#pragma unroll
        for (int j = 0; j < W; ++j) {
            cs[i * W + j] = 1.0f, sn[i * W + j] = 0.0f;
            if (!in[i] || !turns) continue;
            int axis = p.axis ? p.axis[c + j] : 0;
            if (axis < 0 || axis >= p.axes) axis = 0;
            turn((uint64_t)(int64_t)p.pos[t * p.axes + axis] * p.turns[c + j], cs[i * W + j], sn[i * W + j]);
        }
    }
    const float inv_d = 1.0f / (float)p.d;
    const uint32_t group = lph == 32 ? 0xffffffffu : ((1u << lph) - 1u) << (lane / lph * lph);
#pragma unroll 1
    for (int which = 0; which < 2; ++which) {
        const HeadsArgs &h = p.h[which];
        const int heads = h.heads;
        if (heads == 0) continue;
        float w[V];
#pragma unroll
        for (int i = 0; i < V; ++i) w[i] = 1.0f;
        if (h.weight) {
#pragma unroll
            for (int i = 0; i < NC; ++i)
                if (in[i]) {
#pragma unroll
                    for (int j = 0; j < W; ++j) w[2 * W * i + j] = h.weight[at[i] + j], w[2 * W * i + W + j] = h.weight[bt[i] + j];
                }
        }
        const T *x = static_cast<const T *>(h.x) + t * h.ldx;
        T *y = static_cast<T *>(h.y) + t * h.ldy;
        for (int n = part * per + lane / lph; n < heads; n += p.split * per) {
            const T *xh = x + n * h.hx;
            T *yh = y + n * h.hy;
            float v[V];
#pragma unroll
            for (int i = 0; i < NC; ++i) {
#pragma unroll
                for (int j = 0; j < 2 * W; ++j) v[2 * W * i + j] = 0.0f;
                if (in[i]) {
                    load_w<T, W>(v + 2 * W * i, xh + at[i]);
                    load_w<T, W>(v + 2 * W * i + W, xh + bt[i]);
                }
            }
            if (p.norm != SN_HEADS_NONE) {
                if (p.norm == SN_HEADS_LAYER) {
                    float s = 0.0f;
#pragma unroll
                    for (int j = 0; j < V; ++j) s += v[j];
                    for (int o = lph / 2; o; o /= 2) s += __shfl_xor_sync(group, s, o);
                    s *= inv_d;
#pragma unroll
                    for (int i = 0; i < NC; ++i)
                        if (in[i]) {
#pragma unroll
                            for (int j = 0; j < 2 * W; ++j) v[2 * W * i + j] -= s;
                        }
                }
                float s = 0.0f;
#pragma unroll
                for (int j = 0; j < V; ++j) s = fmaf(v[j], v[j], s);
                for (int o = lph / 2; o; o /= 2) s += __shfl_xor_sync(group, s, o);
                s = rsqrtf(s * inv_d + p.eps);
#pragma unroll
                for (int j = 0; j < V; ++j) v[j] *= s * w[j];
            }
#pragma unroll
            for (int i = 0; i < NC; ++i) {
                if (!in[i]) continue;
                float *a = v + 2 * W * i;
                if ((sub + i * lph) * W < p.pairs) {
                    if (p.interleaved) {
#pragma unroll
                        for (int j = 0; j < W; ++j) {
                            const float c = cs[i * W + j], s = sn[i * W + j], e = a[2 * j], f = a[2 * j + 1];
                            a[2 * j] = e * c - f * s, a[2 * j + 1] = e * s + f * c;
                        }
                    } else {
#pragma unroll
                        for (int j = 0; j < W; ++j) {
                            const float c = cs[i * W + j], s = sn[i * W + j], e = a[j], f = a[W + j];
                            a[j] = e * c - f * s, a[W + j] = e * s + f * c;
                        }
                    }
                }
                store_w<T, W>(yh + at[i], a);
                store_w<T, W>(yh + bt[i], a + W);
            }
        }
    }
}

template <typename T, int W, int NC>
cudaError_t launch_rope(RopeP p, cudaStream_t st) {
    int lph = 1;
    while (lph * W * NC < p.d / 2) lph *= 2;
    const int per = 32 / lph, most = std::max(p.h[0].heads, p.h[1].heads);
    // a warp takes a token's heads one after the other, unless there are too few tokens to fill the card:
    // then several share them
    const int64_t want = (int64_t)num_sms() * 32;
    p.split = (int32_t)std::clamp<int64_t>(want / std::max<int64_t>(p.tokens, 1), 1, (most + per - 1) / per);
    const int64_t warps = p.tokens * p.split;
    return launch_pdl(head_rope_kernel<T, W, NC>, dim3((unsigned)((warps + 7) / 8)), dim3(256), 0, st, p, lph);
}

template <typename T>
cudaError_t rope_of(const RopeP &p, cudaStream_t st) {
    // the widest loads that all of it allows
    auto fits = [&](int w) {
        if (p.pairs % w || p.d / 2 % w) return false;
        const int64_t bytes = (int64_t)w * sizeof(T);
        for (const HeadsArgs &h : p.h) {
            if (h.heads == 0) continue;
            if (reinterpret_cast<uintptr_t>(h.x) % bytes || reinterpret_cast<uintptr_t>(h.y) % bytes) return false;
            for (int64_t s : {h.ldx, h.hx, h.ldy, h.hy})
                if (s % w) return false;
        }
        return true;
    };
    if constexpr (sizeof(T) == 2)
        if (fits(8)) return launch_rope<T, 8, 1>(p, st);
    if (fits(4)) return launch_rope<T, 4, 1>(p, st);
    if (fits(2)) return launch_rope<T, 2, 2>(p, st);
    return launch_rope<T, 1, 4>(p, st);
}

}  // namespace

cudaError_t head_rope(const sn_rope_params &q, int dt, int64_t tokens, const HeadsArgs &hq, const HeadsArgs &hk, const int32_t *pos,
                      cudaStream_t st) {
    const RopeP p{{hq, hk}, tokens, pos, q.axis, q.turns, q.head_dim, q.pairs, q.axes, q.norm, q.interleaved, 1, q.eps};
    SN_DT_SWITCH(dt, T, return rope_of<T>(p, st))
    return cudaSuccess;
}

}  // namespace k
}  // namespace sn
