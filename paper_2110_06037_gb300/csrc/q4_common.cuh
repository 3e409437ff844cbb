// Layout of 4-bit weights shared by their kernels.
//
// Weights [n][k] are cut into tiles of 16 rows x 64 columns, 512 bytes each, tile
// after tile along k, then along n; rows and columns behind the end are zero
// weights.  A tile is laid out for a warp: lane l = 4 g + t (g 0..7, t 0..3) has 16
// consecutive bytes, word i of them holding the codes of rows g and g + 8 at the
// columns c = 32 (i / 2) + 8 t + 4 (i % 2) + 0..3: nibbles 0, 4 are row g at c,
// c + 1; nibbles 2, 6 row g at c + 2, c + 3; nibbles 1, 5 and 3, 7 the same of row
// g + 8.  So (word >> 4 j) & 0x000f000f is register j of the A operand of an
// m16n8k16 product over 16 columns of one half of the tile (a group is at least a
// half), and a lane's columns in a half are 8 neighbours, 16 bytes of x.  A nibble
// holds q + 8.
//
// Scales follow: for each 16 rows and each group of columns 16 values, row g and
// g + 8 next to each other.
#pragma once

#include "tc_common.cuh"

namespace sn {
namespace k {

struct Q4P {
    const uint4 *codes;       // [nt][kb][32]
    const uint32_t *scales;   // [nt][kg][8] pairs
    int32_t n, k, nt, kb, kg, glog;  // tiles of 16 rows, tiles of 64 columns, groups a row, log2 of the group
    int32_t scale_bf16, act;
    const float *bias;
};

struct Q4Layout {
    int64_t nt, kb, kg, scales_at, bytes;
};
inline Q4Layout q4_layout(int64_t n, int64_t k, int group) {
    Q4Layout l;
    l.nt = (n + 15) / 16;
    l.kb = (k + 63) / 64;
    l.kg = (l.kb * 64 + group - 1) / group;
    auto up = [](int64_t v) { return (v + 255) / 256 * 256; };
    l.scales_at = up(l.nt * l.kb * 512);
    l.bytes = l.scales_at + up(l.nt * l.kg * 32);
    return l;
}
inline Q4P q4_params(const sn_q4_weights &w) {
    const Q4Layout l = q4_layout(w.n, w.k, w.group);
    const char *p = static_cast<const char *>(w.packed);
    return Q4P{reinterpret_cast<const uint4 *>(p), reinterpret_cast<const uint32_t *>(p + l.scales_at),
               w.n, w.k, (int32_t)l.nt, (int32_t)l.kb, (int32_t)l.kg,
               w.group == 32 ? 5 : w.group == 64 ? 6 : 7, w.scale_dtype == SN_BF16, w.act, w.bias};
}

// the two scales of a pair (row g, row g + 8)
__device__ __forceinline__ float2 scale_pair(uint32_t v, int bf16) {
    return bf16 ? make_float2(__uint_as_float(v << 16), __uint_as_float(v & 0xffff0000u)) : tc::unpack2<__half>(v);
}

// register j of the A operand from a word of codes: two weights' codes as exact
// 16-bit values.  0x4300 + c is 128 + c in bf16 and 0x6400 + c is 1024 + c in fp16
// for c < 16; the difference to 136 or 1032 is exact.
template <typename T>
__device__ __forceinline__ uint32_t code_pair(uint32_t w, int j);
template <>
__device__ __forceinline__ uint32_t code_pair<__nv_bfloat16>(uint32_t w, int j) {
    const uint32_t v = ((w >> (4 * j)) & 0x000f000fu) | 0x43004300u, o = 0x43084308u;
    const __nv_bfloat162 d = __hsub2(*reinterpret_cast<const __nv_bfloat162 *>(&v), *reinterpret_cast<const __nv_bfloat162 *>(&o));
    return *reinterpret_cast<const uint32_t *>(&d);
}
template <>
__device__ __forceinline__ uint32_t code_pair<__half>(uint32_t w, int j) {
    const uint32_t v = ((w >> (4 * j)) & 0x000f000fu) | 0x64006400u, o = 0x64086408u;
    const __half2 d = __hsub2(*reinterpret_cast<const __half2 *>(&v), *reinterpret_cast<const __half2 *>(&o));
    return *reinterpret_cast<const uint32_t *>(&d);
}

// A layer's activation of one of its sums; a sum that is NaN stays so (max and min alone would hide it).
__device__ __forceinline__ float q4_act(float v, int act) { return v != v ? v : act_apply(v, act); }

// Three bf16 values that sum to an fp32 one (8 + 8 + 8 bits; the first rounded
// towards zero, so that it cannot overflow; what is not finite stays in the first).
struct Planes {
    __nv_bfloat16 v[3];
};
__device__ __forceinline__ Planes planes_of(float x) {
    Planes p;
    p.v[0] = __float2bfloat16_rz(x);
    const float r = x - __bfloat162float(p.v[0]);
    const bool fin = fabsf(x) <= 3.4028234664e38f;
    p.v[1] = __float2bfloat16_rn(fin ? r : 0.0f);
    p.v[2] = __float2bfloat16_rn(fin ? r - __bfloat162float(p.v[1]) : 0.0f);
    return p;
}

// few rows, at most FEW_COLS columns of B (fp32 x takes three a row)
constexpr int FEW_COLS = 32;
cudaError_t q4_few_f32(const Q4P &q, int rows, const float *x, int64_t ldx, float *y, int64_t ldy, cudaStream_t st);
cudaError_t q4_few_f16(const Q4P &q, int rows, const __half *x, int64_t ldx, __half *y, int64_t ldy, cudaStream_t st);
cudaError_t q4_few_bf16(const Q4P &q, int rows, const __nv_bfloat16 *x, int64_t ldx, __nv_bfloat16 *y, int64_t ldy, cudaStream_t st);
// many rows, on the tensor cores
size_t q4_prompt_workspace(const sn_q4_weights &w, int dt, int64_t rows, const void *x, int64_t ldx);
cudaError_t q4_prompt(const sn_q4_weights &w, int dt, int64_t rows, const void *x, int64_t ldx, void *y, int64_t ldy,
                      void *work, cudaStream_t st);

}  // namespace k
}  // namespace sn
