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
//
// What bounds a prompt is the issue of instructions and their latency, next to memory: 8192 tokens of 40 heads of 128 in bf16
// take 40 us (4.1 TB/s, 61 % of a copy's rate) with pairs of values in one instruction and the next two heads
// under way, 62 us without either.  A lane that shares its slots with others computes a part of their turns.
#include <algorithm>

#include "kern_common.cuh"
#include "tc_common.cuh"

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

// W values as they lie in memory, and pairs of them
template <typename T, int W>
struct alignas(W * sizeof(T) <= 16 ? W * sizeof(T) : 16) Raw {
    T v[W];
    __device__ __forceinline__ F2 two(int j) const {
        if constexpr (W == 1) {
            return f2(ldf(v), 0.0f);
        } else if constexpr (sizeof(T) == 4) {
            return f2(v[2 * j], v[2 * j + 1]);
        } else {
            const float2 f = tc::unpack2<T>(*reinterpret_cast<const uint32_t *>(v + 2 * j));
            return f2(f.x, f.y);
        }
    }
    __device__ __forceinline__ void set(int j, F2 x) {
        const float2 f = floats(x);
        if constexpr (W == 1) stf(v, f.x);
        else if constexpr (sizeof(T) == 4) v[2 * j] = f.x, v[2 * j + 1] = f.y;
        else *reinterpret_cast<uint32_t *>(v + 2 * j) = tc::pack2<T>(f.x, f.y);
    }
};

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
__global__ void __launch_bounds__(256, 3) head_rope_kernel(const __grid_constant__ RopeP p, int lph) {
    constexpr int AHEAD = 2, P = (W + 1) / 2;  // W = 1: the upper half of each F2 is idle
    __shared__ __align__(16) float weights[2][256];  // (1 without)
    griddep_launch();
    griddep_wait();
    for (int i = threadIdx.x; i < p.d; i += 256) {
        weights[0][i] = p.h[0].weight ? p.h[0].weight[i] : 1.0f;
        weights[1][i] = p.h[1].weight ? p.h[1].weight[i] : 1.0f;
    }
    __syncthreads();
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, sub = lane % lph, per = 32 / lph;
    const int64_t id = (int64_t)blockIdx.x * 8 + warp;
    const int64_t t = id / p.split;
    if (t >= p.tokens) return;
    const int part = (int)(id - t * p.split);
    // this lane's slots: where their values lie, and their turns
    int at[NC], bt[NC];
    F2 cs[NC * P], sn[NC * P];
    bool in[NC];
#pragma unroll
    for (int i = 0; i < NC; ++i) {
        const int c = (sub + i * lph) * W;
        in[i] = c < p.d / 2;
        const bool turns = c < p.pairs;
        at[i] = turns && !p.interleaved ? c : 2 * c;
        bt[i] = turns && !p.interleaved ? c + p.pairs : 2 * c + W;
        // (of the lanes that share a slot, each computes every per-th turn of it)
        float mc[W], ms[W];
#pragma unroll
        for (int j = 0; j < W; ++j) {
            mc[j] = 1.0f, ms[j] = 0.0f;
            const int mine = j * per + lane / lph % min(per, W);
            if (j * per >= W || !in[i] || !turns) continue;
            int axis = p.axis ? p.axis[c + mine] : 0;
            if (axis < 0 || axis >= p.axes) axis = 0;
            turn((uint64_t)(int64_t)p.pos[t * p.axes + axis] * p.turns[c + mine], mc[j], ms[j]);
        }
        float own_c[W], own_s[W];
#pragma unroll
        for (int j = 0; j < W; ++j) own_c[j] = mc[j], own_s[j] = ms[j];
#pragma unroll
        for (int j = 0; j < W; ++j) {
            const int from = sub + (j & (per - 1)) * lph, which = j / per;
            float c1 = own_c[0], s1 = own_s[0];
#pragma unroll
            for (int k = 1; k < W; ++k)
                if (k == which) c1 = own_c[k], s1 = own_s[k];
            mc[j] = __shfl_sync(0xffffffffu, c1, from);
            ms[j] = __shfl_sync(0xffffffffu, s1, from);
        }
#pragma unroll
        for (int j = 0; j < P; ++j) cs[i * P + j] = f2(mc[2 * j], W > 1 ? mc[2 * j + 1 < W ? 2 * j + 1 : 0] : 0.0f), sn[i * P + j] = f2(ms[2 * j], W > 1 ? ms[2 * j + 1 < W ? 2 * j + 1 : 0] : 0.0f);
    }
    const float inv_d = 1.0f / (float)p.d;
    auto both = [](F2 v) {
        const float2 f = floats(v);
        return f.x + f.y;
    };
    auto all = [&](float s) {  // (by whole warps: lanes without a head take part with what they have)
        for (int o = lph / 2; o; o /= 2) s += __shfl_xor_sync(0xffffffffu, s, o);
        return s;
    };
#pragma unroll 1
    for (int which = 0; which < 2; ++which) {
        const HeadsArgs &h = p.h[which];
        const int heads = h.heads, step = p.split * per;
        int n = part * per + lane / lph;
        const int turns = (heads - part * per + step - 1) / step;  // of the warp
        const T *x = static_cast<const T *>(h.x) + t * h.ldx + n * h.hx;
        T *y = static_cast<T *>(h.y) + t * h.ldy + n * h.hy;
        const int64_t dx = step * h.hx, dy = step * h.hy;
        const bool scaled = h.weight != nullptr;
        // (the next AHEAD heads are on their way while one is worked on)
        Raw<T, W> raw[AHEAD][2 * NC] = {};
        int next = n;
        auto load = [&](Raw<T, W> (&r)[2 * NC]) {
#pragma unroll
            for (int i = 0; i < NC; ++i)
                if (in[i] && next < heads) {
                    r[2 * i] = *reinterpret_cast<const Raw<T, W> *>(x + at[i]);
                    r[2 * i + 1] = *reinterpret_cast<const Raw<T, W> *>(x + bt[i]);
                }
            next += step, x += dx;
        };
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) load(raw[k]);
#pragma unroll 1
        for (int i0 = 0; i0 < turns; i0 += AHEAD)
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) {
                if (i0 + k >= turns) break;
                F2 v[NC][2][P];  // both values of this lane's slots
#pragma unroll
                for (int i = 0; i < NC; ++i)
#pragma unroll
                    for (int j = 0; j < 2 * P; ++j) v[i][j / P][j % P] = raw[k][2 * i + j / P].two(j % P);
                load(raw[k]);
                if (p.norm != SN_HEADS_NONE) {
                    if (p.norm == SN_HEADS_LAYER) {
                        F2 s2 = f2(0.0f, 0.0f);
#pragma unroll
                        for (int i = 0; i < NC; ++i)
#pragma unroll
                            for (int j = 0; j < 2 * P; ++j) s2 = add_2(s2, v[i][j / P][j % P]);
                        const float m = -all(both(s2)) * inv_d;
#pragma unroll
                        for (int i = 0; i < NC; ++i)
                            if (in[i]) {
#pragma unroll
                                for (int j = 0; j < 2 * P; ++j) v[i][j / P][j % P] = add_2(v[i][j / P][j % P], f2(m, W > 1 ? m : 0.0f));
                            }
                    }
                    F2 s2 = f2(0.0f, 0.0f);
#pragma unroll
                    for (int i = 0; i < NC; ++i)
#pragma unroll
                        for (int j = 0; j < 2 * P; ++j) s2 = fma_2(v[i][j / P][j % P], v[i][j / P][j % P], s2);
                    const float s = rsqrtf(all(both(s2)) * inv_d + p.eps);
#pragma unroll
                    for (int i = 0; i < NC; ++i)
#pragma unroll
                        for (int j = 0; j < 2 * P; ++j) v[i][j / P][j % P] = mul_2(v[i][j / P][j % P], f2(s, s));
                    if (scaled) {
#pragma unroll
                        for (int i = 0; i < NC; ++i) {
                            if (!in[i]) continue;
                            const Raw<float, W> wa = *reinterpret_cast<const Raw<float, W> *>(&weights[which][at[i]]);
                            const Raw<float, W> wb = *reinterpret_cast<const Raw<float, W> *>(&weights[which][bt[i]]);
#pragma unroll
                            for (int j = 0; j < P; ++j) v[i][0][j] = mul_2(v[i][0][j], wa.two(j)), v[i][1][j] = mul_2(v[i][1][j], wb.two(j));
                        }
                    }
                }
#pragma unroll
                for (int i = 0; i < NC; ++i) {
                    if ((sub + i * lph) * W < p.pairs) {
                        if (!p.interleaved || W == 1) {  // (one value of each: neighbours and halves are the same)
#pragma unroll
                            for (int j = 0; j < P; ++j) {
                                const F2 c = cs[i * P + j], z = sn[i * P + j], a = v[i][0][j], b = v[i][1][j];
                                v[i][0][j] = fma_2(a, c, mul_2(b, mul_2(z, f2(-1.0f, -1.0f))));
                                v[i][1][j] = fma_2(a, z, mul_2(b, c));
                            }
                        } else {
#pragma unroll
                            for (int j = 0; j < W; ++j) {
                                const float2 c = floats(cs[i * P + j / 2]), z = floats(sn[i * P + j / 2]), e = floats(v[i][j / P][j % P]);
                                const float cj = j % 2 ? c.y : c.x, zj = j % 2 ? z.y : z.x;
                                v[i][j / P][j % P] = fma_2(f2(e.x, e.x), f2(cj, zj), mul_2(f2(e.y, e.y), f2(-zj, cj)));
                            }
                        }
                    }
                    if (!in[i] || n >= heads) continue;
#pragma unroll
                    for (int half = 0; half < 2; ++half) {
                        Raw<T, W> r;
#pragma unroll
                        for (int j = 0; j < P; ++j) r.set(j, v[i][half][j]);
                        *reinterpret_cast<Raw<T, W> *>(y + (half ? bt[i] : at[i])) = r;
                    }
                }
                n += step, y += dy;
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
