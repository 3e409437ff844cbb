// Pieces that the scan's kernels share.
#pragma once

#include "kern_common.cuh"

namespace sn {
namespace k {

struct Seq {  // one sequence of the batch
    int64_t first, pos;  // its first token row, that token's position
    int32_t len, slot;
};
__device__ __forceinline__ Seq sequence(const SeqArgs &q, int b) {
    Seq s;
    if (q.offsets) {  // (clipped to the rows there are, so that bad offsets read nothing else)
        const int64_t n = q.tokens;
        const int64_t i = q.offsets[b], j = q.offsets[b + 1];
        s.first = i < 0 ? 0 : i > n ? n : i;
        const int64_t e = j < s.first ? s.first : j > n ? n : j;
        s.len = (int32_t)(e - s.first);
    } else {
        s.first = (int64_t)b * q.max_len;
        s.len = (int32_t)q.max_len;
    }
    const int slot = q.slots ? q.slots[b] : b;
    s.slot = slot >= 0 && slot < q.n_slots ? slot : -1;
    s.pos = q.pos ? q.pos[b] : 0;
    if (s.pos < 0) s.pos = 0;
    return s;
}

// What block `id` of a scan works on: each sequence has `own(length)` segments, each
// segment `blocks` blocks.  The blocks that have work so are the first of the grid and
// spread over the multiprocessors evenly.  Called by whole warps; alike: every sequence
// has own(its length) = own(max_len).
struct Place {
    int b, seg, block;  // b < 0: nothing
};
template <typename Own>
__device__ __forceinline__ Place place_of(const SeqArgs &q, bool alike, Own own, int blocks, int id) {
    const int lane = threadIdx.x % 32;
    int rest = id / blocks;  // the segment's number among all
    if (!q.offsets || alike) {
        const int n = own((int)q.max_len);
        return n > 0 && rest / n < q.batch ? Place{rest / n, rest % n, id % blocks} : Place{-1, 0, 0};
    }
    for (int b0 = 0; b0 < q.batch; b0 += 32) {
        const int n = b0 + lane < q.batch ? own(sequence(q, b0 + lane).len) : 0;
        int up = n;
#pragma unroll
        for (int o = 1; o < 32; o *= 2) {
            const int v = __shfl_up_sync(0xffffffffu, up, o);
            if (lane >= o) up += v;
        }
        const uint32_t in = __ballot_sync(0xffffffffu, rest < up);
        if (in) {
            const int k = __ffs(in) - 1;
            return Place{b0 + k, rest - (__shfl_sync(0xffffffffu, up, k) - __shfl_sync(0xffffffffu, n, k)), id % blocks};
        }
        rest -= __shfl_sync(0xffffffffu, up, 31);
    }
    return Place{-1, 0, 0};
}

__device__ __forceinline__ float ex2(float v) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
    return r;
}
// by the approximate exponential and division (2 ulp each; a denominator beyond 2^126 gives 0)
__device__ __forceinline__ float silu(float v) { return __fdividef(v, 1.0f + __expf(-v)); }
// the same of two values
__device__ __forceinline__ F2 silu_2(F2 v) {
    constexpr float LOG2E = 1.4426950408889634f;
    const float2 t = floats(mul_2(v, f2(-LOG2E, -LOG2E)));
    const float2 d = floats(add_2(f2(ex2(t.x), ex2(t.y)), f2(1.0f, 1.0f)));
    float a, b;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(a) : "f"(d.x));
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(b) : "f"(d.y));
    return mul_2(v, f2(a, b));
}
// log(1 + e^v) without overflow, and exact where e^v is small
__device__ __forceinline__ float softplus(float v) { return fmaxf(v, 0.0f) + log1pf(expf(-fabsf(v))); }

struct SsmP {
    SeqArgs q;
    int32_t H, P, G, N, W;
    const float *a, *d, *dt_bias, *conv_w, *conv_b;
    int64_t ldx, lddt, ldy;
    const float *s_in;
    float *s_out;
};

// the scan of bf16 tokens by matrix products (kernels_ssm_tc.cu)
bool ssm_tc_applies(const SsmP &p, const void *xbc, const void *y);
size_t ssm_tc_workspace(const SsmP &p);
cudaError_t ssm_tc_scan(const SsmP &p, const __nv_bfloat16 *xbc, const __nv_bfloat16 *dtv, __nv_bfloat16 *y, void *work,
                        cudaStream_t st);

}  // namespace k
}  // namespace sn
