// New tokens' keys and values into a paged cache and back, as they are or as 8-bit codes with a
// scale a token and head (sn_kv_write, sn_kv_read in include/sn.h).
//
// What bounds it is memory, and next to it the chain of four loads from a token to its page.  A lane has 16
// neighbours of a head, the lanes of a head are neighbours, and a warp has as many heads of a token at once (a turn;
// keys and values alike).  A block of four warps takes a few tokens, finds their places at once, a lane each, and its
// warps take the turns, two of them loaded before the first is worked on.  8333 tokens of 8 heads of 128, bf16 into codes
// and back: 33 us (18 and 15, each 52 MB); with a warp a token and a division a value 50.
// Codes: the largest |v| by integers (above those of finite values there are infinities and NaN), v / s by the
// reciprocal, rounded by adding 1.5 * 2^23, whose low byte then is the code.
#include <algorithm>
#include <type_traits>

#include "attn_common.cuh"
#include "tc_common.cuh"

namespace sn {
namespace k {

namespace {

constexpr int TURNS = 2, WARPS = 4;

struct KvP {
    sn_kv_cache c;
    SeqArgs q;
    TableArgs t;
    HeadsArgs k, v;
    int32_t lph, tokens;  // lanes a head; tokens a block
    FastDiv turns;        // of a token
};

template <typename T>
struct alignas(16) Raw {
    T v[16];
};
template <typename T>
__device__ __forceinline__ void load16(Raw<T> &r, const T *p, bool vec) {
    if (vec) {
#pragma unroll
        for (int i = 0; i < (int)sizeof(T); ++i) reinterpret_cast<uint4 *>(r.v)[i] = reinterpret_cast<const uint4 *>(p)[i];
    } else {
#pragma unroll
        for (int i = 0; i < 16; ++i) r.v[i] = p[i];
    }
}
template <typename T>
__device__ __forceinline__ void store16(T *p, const Raw<T> &r, bool vec) {
    if (vec) {
#pragma unroll
        for (int i = 0; i < (int)sizeof(T); ++i) reinterpret_cast<uint4 *>(p)[i] = reinterpret_cast<const uint4 *>(r.v)[i];
    } else {
#pragma unroll
        for (int i = 0; i < 16; ++i) p[i] = r.v[i];
    }
}
// the bits of the largest |v| as fp32
template <typename T>
__device__ __forceinline__ uint32_t largest(const Raw<T> &r) {
    const uint32_t *u = reinterpret_cast<const uint32_t *>(r.v);
    if constexpr (sizeof(T) == 4) {
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < 16; ++i) top = max(top, u[i] & 0x7fffffffu);
        return top;
    } else {
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) top = __vmaxu2(top, u[i] & 0x7fff7fffu);
        top = max(top & 0xffffu, top >> 16);
        if constexpr (std::is_same<T, __half>::value) return __float_as_uint(__half2float(__ushort_as_half((unsigned short)top)));
        else return top << 16;
    }
}
template <typename T>
__device__ __forceinline__ F2 two(const Raw<T> &r, int j) {
    if constexpr (sizeof(T) == 4) {
        return f2(r.v[2 * j], r.v[2 * j + 1]);
    } else {
        const float2 f = tc::unpack2<T>(reinterpret_cast<const uint32_t *>(r.v)[j]);
        return f2(f.x, f.y);
    }
}

template <typename T, bool CODES, bool WRITE>
__global__ void __launch_bounds__(32 * WARPS) kv_kernel(const __grid_constant__ KvP p, int vec) {
    using In = typename std::conditional<CODES && !WRITE, int8_t, T>::type;  // what is loaded
    griddep_launch();
    griddep_wait();
    const int lane = threadIdx.x % 32, sub = lane % p.lph, per = 32 / p.lph, d = p.c.head_dim, turns = (int)p.turns.d;
    const bool in = sub * 16 < d;
    // the places of the block's tokens, a lane each
    const int64_t first = (int64_t)blockIdx.x * p.tokens;
    const int count = (int)min((int64_t)p.tokens, p.q.tokens - first);
    int64_t place = -2;  // -1: nowhere; -2: a row behind the last sequence
    if (lane < count) {
        const int b = sequence_at(p.q, first + lane);
        if (b >= 0) {
            const Seq s = sequence(p.q, b);
            place = place_in(p.c, p.t, s.slot, s.pos + (first + lane - s.first));
        }
    }
#pragma unroll 1
    for (int u0 = threadIdx.x / 32 * TURNS; u0 < count * turns; u0 += WARPS * TURNS) {
        Raw<In> raw[TURNS];
        float scale[TURNS];
        int64_t row[TURNS], at[TURNS];  // of the cache (-1: nothing to do), and where the head lies outside
        int which[TURNS];
#pragma unroll
        for (int i = 0; i < TURNS; ++i) {
            const int tok = (int)fdiv((uint32_t)(u0 + i), p.turns), n = (u0 + i - tok * turns) * per + lane / p.lph;
            const int head = n >> 1;
            which[i] = n & 1;
            const int64_t spot = __shfl_sync(0xffffffffu, place, tok & 31);
            const bool use = tok < count && n < 2 * p.c.heads && spot >= (WRITE ? 0 : -1);
            row[i] = use ? spot < 0 ? 0 : row_in(p.c, spot, head) : -1;
            const int64_t ld = which[i] ? (WRITE ? p.v.ldx : p.v.ldy) : (WRITE ? p.k.ldx : p.k.ldy);
            const int64_t hd = which[i] ? (WRITE ? p.v.hx : p.v.hy) : (WRITE ? p.k.hx : p.k.hy);
            at[i] = (first + tok) * ld + head * hd + sub * 16;
            scale[i] = 0.0f;
            raw[i] = Raw<In>{};
            if (WRITE) {
                if (use && in) load16(raw[i], static_cast<const In *>(which[i] ? p.v.x : p.k.x) + at[i], vec);
            } else if (use && spot >= 0) {
                if (in) load16(raw[i], static_cast<const In *>(which[i] ? p.c.v : p.c.k) + row[i] * d + sub * 16, true);
                if constexpr (CODES) scale[i] = (which[i] ? p.c.v_scale : p.c.k_scale)[row[i]];
            }
        }
#pragma unroll
        for (int i = 0; i < TURNS; ++i) {
            const bool use = row[i] >= 0 && in;
            const int64_t kept = row[i] * d + sub * 16;
            if constexpr (!CODES) {
                if (!use) continue;
                if (WRITE) store16(static_cast<T *>(which[i] ? p.c.v : p.c.k) + kept, raw[i], true);
                else store16(static_cast<T *>(which[i] ? p.v.y : p.k.y) + at[i], raw[i], vec);
            } else if constexpr (WRITE) {
                uint32_t bits = largest<T>(raw[i]);
                for (int o = p.lph / 2; o; o /= 2) bits = max(bits, __shfl_xor_sync(0xffffffffu, bits, o));
                const bool bad = bits >= 0x7f800000u;
                float f = bits ? fmaxf(__fdiv_rn(__uint_as_float(bits), 127.0f), 1.401298464e-45f) : 1.0f;
                // v / f rounded to nearest: a quotient off by less than one unit of the last place, corrected by its
                // remainder, which is exact, and the correctly rounded reciprocal (Markstein); where nothing underflows
                const float r = __frcp_rn(f);
                const F2 r2 = f2(r, r), f_2 = f2(-f, -f);
                alignas(16) uint32_t code[4];
                if (f > 8e-28f && f < 1e36f) {
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        uint32_t c[2];
#pragma unroll
                        for (int k = 0; k < 2; ++k) {
                            const F2 v = two<T>(raw[i], 2 * j + k);
                            F2 q = mul_2(v, r2);
                            q = fma_2(fma_2(q, f_2, v), r2, q);
                            q = fma_2(fma_2(q, f_2, v), r2, q);
                            const float2 e = floats(add_2(q, f2(12582912.0f, 12582912.0f)));
                            c[k] = __byte_perm(__float_as_uint(e.x), __float_as_uint(e.y), 0x0040);
                        }
                        code[j] = __byte_perm(c[0], c[1], 0x5410);
                    }
                } else {
                    int8_t *c = reinterpret_cast<int8_t *>(code);
#pragma unroll
                    for (int j = 0; j < 16; ++j) c[j] = (int8_t)fminf(fmaxf(rintf(__fdiv_rn(ldf(raw[i].v + j), f)), -127.0f), 127.0f);
                }
                if (bad) {
                    f = __int_as_float(0x7fc00000);
                    code[0] = code[1] = code[2] = code[3] = 0;
                }
                if (use) *reinterpret_cast<uint4 *>(static_cast<int8_t *>(which[i] ? p.c.v : p.c.k) + kept) = *reinterpret_cast<const uint4 *>(code);
                if (use && sub == 0) (which[i] ? p.c.v_scale : p.c.k_scale)[row[i]] = f;
            } else {
                if (!use) continue;
                const uint32_t *c = reinterpret_cast<const uint32_t *>(raw[i].v);
                Raw<T> o;
#pragma unroll
                for (int j = 0; j < 8; ++j) {  // a code's byte, shifted by 128, behind the exponent of 2^23
                    const uint32_t x = c[j / 2] ^ 0x80808080u;
                    const F2 v = add_2(f2(__uint_as_float(__byte_perm(x, 0x4b000000u, 0x7440 + j % 2 * 2)), __uint_as_float(__byte_perm(x, 0x4b000000u, 0x7441 + j % 2 * 2))),
                                       f2(-8388736.0f, -8388736.0f));
                    const float2 g = floats(mul_2(v, f2(scale[i], scale[i])));
                    if constexpr (sizeof(T) == 4) o.v[2 * j] = g.x, o.v[2 * j + 1] = g.y;
                    else reinterpret_cast<uint32_t *>(o.v)[j] = tc::pack2<T>(g.x, g.y);
                }
                store16(static_cast<T *>(which[i] ? p.v.y : p.k.y) + at[i], o, vec);
            }
        }
    }
}

template <bool WRITE>
cudaError_t launch_kv(const sn_kv_cache &c, int dt, const SeqArgs &q, const TableArgs &t, const HeadsArgs &k, const HeadsArgs &v,
                      cudaStream_t st) {
    KvP p{c, q, t, k, v, 1, 1, {}};
    while (p.lph * 16 < c.head_dim) p.lph *= 2;
    const int per = 32 / p.lph;
    p.turns = make_fastdiv((uint32_t)((2 * c.heads + per - 1) / per));
    // as many tokens a block as leave eight blocks a multiprocessor, up to a warp's lanes
    p.tokens = (int32_t)std::clamp<int64_t>((q.tokens + 8 * num_sms() - 1) / (8 * num_sms()), 1, 32);
    const int64_t es = dt == SN_F32 ? 4 : 2;
    int vec = 1;
    for (const HeadsArgs *h : {&k, &v}) {
        const void *ptr = WRITE ? h->x : h->y;
        const int64_t ld = WRITE ? h->ldx : h->ldy, hd = WRITE ? h->hx : h->hy;
        if (reinterpret_cast<uintptr_t>(ptr) % 16 || ld * es % 16 || hd * es % 16) vec = 0;
    }
    const dim3 grid((unsigned)((q.tokens + p.tokens - 1) / p.tokens));
    SN_DT_SWITCH(dt, T, {
        if (c.dtype == SN_QI8) return launch_pdl(kv_kernel<T, true, WRITE>, grid, dim3(32 * WARPS), 0, st, p, vec);
        return launch_pdl(kv_kernel<T, false, WRITE>, grid, dim3(32 * WARPS), 0, st, p, vec);
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
