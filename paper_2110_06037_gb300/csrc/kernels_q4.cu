// 4-bit weights: quantisation, layout, and which kernel a product takes
// (sn_q4_quantize, sn_q4_pack, sn_q4_dense in include/sn.h; layout in q4_common.cuh).
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

// the scales into place, a value a thread; zeros behind the last row and group
__global__ void __launch_bounds__(256) q4_pack_scales_kernel(const uint16_t *__restrict__ scales, int64_t n, int64_t groups,
                                                             int64_t kg, int64_t total, uint16_t *__restrict__ out) {
    const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (id >= total) return;
    const int64_t grp = id / 16 % kg, row = id / 16 / kg * 16 + id % 16 / 2 + id % 2 * 8;
    out[id] = row < n && grp < groups ? scales[row * groups + grp] : 0;
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
    const int64_t values = l.nt * l.kg * 16;
    q4_pack_scales_kernel<<<(unsigned)((values + 255) / 256), 256, 0, st>>>(static_cast<const uint16_t *>(scales), w.n, groups, l.kg,
                                                                            values, reinterpret_cast<uint16_t *>(out + l.scales_at));
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
    if (dt == SN_F32) return q4_few_f32(q, m, static_cast<const float *>(x), ldx, static_cast<float *>(y), ldy, st);
    if (dt == SN_F16) return q4_few_f16(q, m, static_cast<const __half *>(x), ldx, static_cast<__half *>(y), ldy, st);
    return q4_few_bf16(q, m, static_cast<const __nv_bfloat16 *>(x), ldx, static_cast<__nv_bfloat16 *>(y), ldy, st);
}

}  // namespace k
}  // namespace sn
