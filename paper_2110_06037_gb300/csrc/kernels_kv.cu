// New tokens' keys and values into a paged cache and back, as they are or as 8-bit codes with a
// scale a token and head (sn_kv_write, sn_kv_read in include/sn.h).
//
// A lane has eight neighbours of a head (16 bytes of 16-bit values, 8 bytes of codes), the lanes of a
// head are neighbours, and a warp takes the heads of one token one after the other, keys and values
// alike, so that the token's sequence, page and place are found once.
#include <algorithm>

#include "attn_common.cuh"

namespace sn {
namespace k {

namespace {

struct KvP {
    sn_kv_cache c;
    SeqArgs q;
    TableArgs t;
    HeadsArgs k, v;
    int32_t lph, split;  // lanes a head; warps a token
};

template <typename T>
__device__ __forceinline__ void load8(float *v, const T *p, bool vec) {
    if (vec) {
        alignas(16) T t[8];
        *reinterpret_cast<uint4 *>(t) = *reinterpret_cast<const uint4 *>(p);
        if constexpr (sizeof(T) == 4) *reinterpret_cast<uint4 *>(t + 4) = *reinterpret_cast<const uint4 *>(p + 4);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = ldf(t + i);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = ldf(p + i);
    }
}
template <typename T>
__device__ __forceinline__ void store8(T *p, const float *v, bool vec) {
    if (vec) {
        alignas(16) T t[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) stf(t + i, v[i]);
        *reinterpret_cast<uint4 *>(p) = *reinterpret_cast<const uint4 *>(t);
        if constexpr (sizeof(T) == 4) *reinterpret_cast<uint4 *>(p + 4) = *reinterpret_cast<const uint4 *>(t + 4);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) stf(p + i, v[i]);
    }
}

template <typename T, bool CODES, bool WRITE>
__global__ void __launch_bounds__(256) kv_kernel(const __grid_constant__ KvP p, int vec) {
    griddep_launch();
    griddep_wait();
    const int lane = threadIdx.x % 32, sub = lane % p.lph, per = 32 / p.lph;
    const int64_t id = (int64_t)blockIdx.x * 8 + threadIdx.x / 32;
    const int64_t t = id / p.split;
    const int part = (int)(id - t * p.split);
    if (t >= p.q.tokens) return;
    const int b = sequence_of(p.q, t);
    if (b < 0) return;  // (a row behind the last sequence)
    const Seq s = sequence(p.q, b);
    const int64_t place = place_in(p.c, p.t, s.slot, s.pos + (t - s.first));
    if (WRITE && place < 0) return;
    const int d = p.c.head_dim;
    const bool in = sub * 8 < d;
    const uint32_t group = p.lph == 32 ? 0xffffffffu : ((1u << p.lph) - 1u) << (lane / p.lph * p.lph);
    for (int n = part * per + lane / p.lph; n < 2 * p.c.heads; n += p.split * per) {
        const int head = n / 2, which = n % 2;
        const HeadsArgs &h = which ? p.v : p.k;
        const int64_t row = place < 0 ? 0 : row_in(p.c, place, head), at = row * d + sub * 8;
        void *kept = which ? p.c.v : p.c.k;
        float *scales = which ? p.c.v_scale : p.c.k_scale;
        float v[8];
        if constexpr (WRITE) {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = 0.0f;
            if (in) load8<T>(v, static_cast<const T *>(h.x) + t * h.ldx + head * h.hx + sub * 8, vec);
            if constexpr (CODES) {
                float top = 0.0f;
                bool bad = false;
#pragma unroll
                for (int i = 0; i < 8; ++i) top = fmaxf(top, fabsf(v[i])), bad |= !(fabsf(v[i]) < INFINITY);
                for (int o = p.lph / 2; o; o /= 2) top = fmaxf(top, __shfl_xor_sync(group, top, o));
                bad = (__ballot_sync(group, bad) & group) != 0;
                float f = top > 0.0f ? fmaxf(__fdiv_rn(top, 127.0f), 1.401298464e-45f) : 1.0f;
                alignas(8) int8_t code[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) code[i] = bad ? 0 : (int8_t)fminf(fmaxf(rintf(__fdiv_rn(v[i], f)), -127.0f), 127.0f);
                if (bad) f = __int_as_float(0x7fc00000);
                if (in) *reinterpret_cast<uint2 *>(static_cast<int8_t *>(kept) + at) = *reinterpret_cast<const uint2 *>(code);
                if (sub == 0) scales[row] = f;
            } else {
                if (in) store8<T>(static_cast<T *>(kept) + at, v, true);
            }
        } else {
            if (!in) continue;
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = 0.0f;
            if (place >= 0) {
                if constexpr (CODES) {
                    const float f = scales[row];
                    alignas(8) int8_t code[8];
                    *reinterpret_cast<uint2 *>(code) = *reinterpret_cast<const uint2 *>(static_cast<const int8_t *>(kept) + at);
#pragma unroll
                    for (int i = 0; i < 8; ++i) v[i] = f * (float)code[i];
                } else {
                    load8<T>(v, static_cast<const T *>(kept) + at, true);
                }
            }
            store8<T>(static_cast<T *>(h.y) + t * h.ldy + head * h.hy + sub * 8, v, vec);
        }
    }
}

template <bool WRITE>
cudaError_t launch_kv(const sn_kv_cache &c, int dt, const SeqArgs &q, const TableArgs &t, const HeadsArgs &k, const HeadsArgs &v,
                      cudaStream_t st) {
    KvP p{c, q, t, k, v, 1, 1};
    while (p.lph * 8 < c.head_dim) p.lph *= 2;
    const int per = 32 / p.lph;
    // as many warps a token as fill the card, up to one for each turn of its heads
    p.split = (int32_t)std::clamp<int64_t>((int64_t)num_sms() * 32 / q.tokens, 1, (2 * (int64_t)c.heads + per - 1) / per);
    const int64_t es = dt == SN_F32 ? 4 : 2;
    int vec = 1;
    for (const HeadsArgs *h : {&k, &v}) {
        const void *ptr = WRITE ? h->x : h->y;
        const int64_t ld = WRITE ? h->ldx : h->ldy, hd = WRITE ? h->hx : h->hy;
        if (reinterpret_cast<uintptr_t>(ptr) % 16 || ld * es % 16 || hd * es % 16) vec = 0;
    }
    const dim3 grid((unsigned)((q.tokens * p.split + 7) / 8));
    SN_DT_SWITCH(dt, T, {
        if (c.dtype == SN_QI8) return launch_pdl(kv_kernel<T, true, WRITE>, grid, dim3(256), 0, st, p, vec);
        return launch_pdl(kv_kernel<T, false, WRITE>, grid, dim3(256), 0, st, p, vec);
    })
    return cudaSuccess;
}

}  // namespace

cudaError_t kv_write(const sn_kv_cache &c, int dt, const SeqArgs &q, const TableArgs &t, const HeadsArgs &k, const HeadsArgs &v,
                     cudaStream_t st) {
    return launch_kv<true>(c, dt, q, t, k, v, st);
}
cudaError_t kv_read(const sn_kv_cache &c, int dt, const SeqArgs &q, const TableArgs &t, const HeadsArgs &k, const HeadsArgs &v,
                    cudaStream_t st) {
    return launch_kv<false>(c, dt, q, t, k, v, st);
}

}  // namespace k
}  // namespace sn
