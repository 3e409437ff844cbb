// 4-bit weights with many rows of x, on the 5th-generation tensor cores
// (sn_q4_dense in include/sn.h; layout in q4_common.cuh).
//
//   D[m, j] = sum_k x[m, k] * w[j, k],  w = q * scale rounded to the operand type
//
// A tile is 128 G rows of x by BN outputs, accumulated in TMEM over steps of 64
// columns.  x, codes and scales come by TMA; the weights are expanded in the kernel:
// a warp reads 16 x 64 tiles of codes from shared memory, makes codes exact 16-bit
// values, multiplies by the group's scale in packed 16-bit arithmetic, one rounding,
// and writes the operand's 128-byte-swizzled rows into the stage.  Codes are a
// quarter of the bytes that 16-bit weights would move, and an SM expands only the
// BN / G rows it stages.  (Codes loaded straight into registers, some steps ahead,
// were waited for by every step's proxy fence: 338 us for 2048 rows, 4096 -> 8448.)
// G = 2: a CTA pair shares a tile of 256 rows; each stages 128 rows of x and half
// of the weights, which halves what a tile reads through L2 and expands per MMA.
//
// fp16 operands: scales are divided by their row's power of two (and multiplied by
// 2^12), so that a product neither overflows nor, for groups within 2^-26 of the
// row's largest scale, loses bits; the epilogue multiplies it back.
// Scales that are not values of the operand type go in as two parts (a product
// with the small one, a fused multiply-add with the large one).
// fp32 x: three bf16 planes of x (written to scratch by a first kernel) times two
// bf16 parts of w, which hold q * scale exactly; of the six products the smallest
// (2^-25 and less) is left out.  One k step then is five.  (A fourth plane is the
// first with zeros for what is not finite: the second part of w is often 0.)
// The tensor cores' sums are truncated, by some 1.4e-8 of them an MMA (4.6e-5 in all for
// 8192 columns), so they run over one column block, 20 MMAs with the four of the large
// product last; the epilogue's warps add those sums in fp32 to one that they keep in TMEM.
// (2.2e-7 then; over two blocks 4.8e-7, and 855 us for 2048 rows, 4096 -> 8448, against 897.)
//
// Warps: 0 loads x and allocates TMEM, 1 issues the MMAs (of the pair's leader), 2
// loads codes and scales, 4 to 7 drain the accumulators (two, so that a tile's
// epilogue overlaps the next tile's products), 8 to 19 expand weights, three groups
// of four that fill stages in turn (a fill takes a group about 1100 cycles, mostly
// latencies, the MMAs of a stage 450).  Waits are bounded; one that expires
// records its cause in the library's error word and stops the pair.
//
// 2048 bf16 rows, 4096 -> 8448: 115 us, 1230 TFLOP/s, 63% of a plain matrix product's
// measured rate; bound by the expanding warps.
#include <algorithm>

#include "q4_common.cuh"

namespace sn {
namespace k {

namespace {

using namespace tc;

constexpr int Q4_STAGES = 5, Q4_THREADS = 640;
constexpr int Q4_EXPAND = 4, Q4_TURNS = 3;            // warps that expand a column block; groups of them taking turns
constexpr int Q4_CSTAGES = 6;                         // column blocks of codes and scales in flight
constexpr uint32_t Q4_CBYTES = 8 * 512, Q4_CSTAGE = Q4_CBYTES + 8 * 64;  // eight tiles: codes; up to two groups' scales
constexpr uint32_t Q4_A_BYTES = BM * BK * 2, Q4_B_BYTES = 128 * BK * 2, Q4_STAGE = Q4_A_BYTES + Q4_B_BYTES;
constexpr uint32_t Q4_OUT_ROW = 128 + 16;  // staged output row: 32 values, and 16 bytes against bank conflicts
constexpr size_t Q4_SMEM = Q4_STAGES * (size_t)Q4_STAGE + Q4_CSTAGES * (size_t)Q4_CSTAGE + 4 * 32 * Q4_OUT_ROW + 1024;

constexpr int Q4_F32_BN = 160;  // fp32: the widest tile (two accumulators and the sum fit TMEM)

struct PromptP {
    Q4P q;
    int64_t rows, ldy;
    int32_t bn, mtiles, ntiles, steps;  // outputs a tile, tiles, k steps (five a column block for fp32)
    int32_t run;                        // k steps summed by the tensor cores
    int32_t plane_rows;                 // fp32: rows of a plane of x
    int32_t parts;                      // scales in two parts
    int32_t vec_out;
    int *err;
    long long wait_limit;
};

template <typename T>
__device__ __forceinline__ uint32_t mul2(uint32_t a, uint32_t b);
template <>
__device__ __forceinline__ uint32_t mul2<__half>(uint32_t a, uint32_t b) {
    const __half2 r = __hmul2(*reinterpret_cast<__half2 *>(&a), *reinterpret_cast<__half2 *>(&b));
    return *reinterpret_cast<const uint32_t *>(&r);
}
template <>
__device__ __forceinline__ uint32_t mul2<__nv_bfloat16>(uint32_t a, uint32_t b) {
    const __nv_bfloat162 r = __hmul2(*reinterpret_cast<__nv_bfloat162 *>(&a), *reinterpret_cast<__nv_bfloat162 *>(&b));
    return *reinterpret_cast<const uint32_t *>(&r);
}
template <typename T>
__device__ __forceinline__ uint32_t fma2(uint32_t a, uint32_t b, uint32_t c);
template <>
__device__ __forceinline__ uint32_t fma2<__half>(uint32_t a, uint32_t b, uint32_t c) {
    const __half2 r = __hfma2(*reinterpret_cast<__half2 *>(&a), *reinterpret_cast<__half2 *>(&b), *reinterpret_cast<__half2 *>(&c));
    return *reinterpret_cast<const uint32_t *>(&r);
}
template <>
__device__ __forceinline__ uint32_t fma2<__nv_bfloat16>(uint32_t a, uint32_t b, uint32_t c) {
    const __nv_bfloat162 r = __hfma2(*reinterpret_cast<__nv_bfloat162 *>(&a), *reinterpret_cast<__nv_bfloat162 *>(&b),
                                     *reinterpret_cast<__nv_bfloat162 *>(&c));
    return *reinterpret_cast<const uint32_t *>(&r);
}

// a scale as two parts of the operand type, each twice in a register
struct Scale2 {
    uint32_t hi, lo;
};
template <typename T>
__device__ __forceinline__ Scale2 scale_parts(float s) {
    Scale2 r;
    r.hi = pack2<T>(s, s);
    const float rest = s - unpack2<T>(r.hi).x;
    r.lo = pack2<T>(rest, rest);
    return r;
}
// code * scale in one rounding (parts: of a scale in two parts)
template <typename T>
__device__ __forceinline__ uint32_t expand(uint32_t c, const Scale2 &s, bool parts) {
    return parts ? fma2<T>(c, s.hi, mul2<T>(c, s.lo)) : mul2<T>(c, s.hi);
}
// what that rounding dropped: exact in bf16 (the scale has at most 11 bits, the code 4)
__device__ __forceinline__ uint32_t expand_rest(uint32_t c, const Scale2 &s, uint32_t w) {
    const uint32_t neg = w ^ 0x80008000u;
    return fma2<__nv_bfloat16>(c, s.lo, fma2<__nv_bfloat16>(c, s.hi, neg));
}

// Expanded weights are for the MMAs that the pair's leader issues: what this warp has
// written to shared memory, made visible to the async proxy, before the arrival at the
// leader's barrier.  The release is restricted to shared memory: the usual one at
// cluster scope took about 1000 cycles (223 us in all, against 167).
__device__ __forceinline__ void arrive_expanded(uint32_t caddr) {
    asm volatile("fence.release.sync_restrict::shared::cta.cluster;\n\t"
                 "mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(caddr)
                 : "memory");
}

// T: the operands' type; X: x's and y's
template <typename T, typename X, int G>
__global__ void __launch_bounds__(Q4_THREADS, 1)
    q4_prompt_kernel(const __grid_constant__ CUtensorMap mX, const __grid_constant__ CUtensorMap mC,
                     const __grid_constant__ CUtensorMap mS, const __grid_constant__ PromptP p, X *__restrict__ y) {
    constexpr bool F32 = std::is_same<X, float>::value;
    constexpr int COMBOS = F32 ? 5 : 1;
    constexpr uint32_t TMEM_COLS = G == 2 || F32 ? 512 : 256, ACC = F32 ? Q4_F32_BN : TMEM_COLS / 2;
    extern __shared__ uint8_t smem_raw[];
    __shared__ __align__(8) uint64_t full_bar[Q4_STAGES], empty_bar[Q4_STAGES], accf_bar[2], acce_bar[2];
    __shared__ __align__(8) uint64_t cfull_bar[Q4_CSTAGES], cempty_bar[Q4_CSTAGES];
    __shared__ __align__(16) float bias_sh[4][32], pow_sh[4][32];
    __shared__ uint32_t tmem_sh;
    __shared__ volatile int abort_sh;
    __shared__ int issued_sh, cissued_sh, consumed_sh;
    uint8_t *smem = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    uint8_t *cst = smem + Q4_STAGES * Q4_STAGE, *stg = cst + Q4_CSTAGES * Q4_CSTAGE;
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const uint32_t rank = G == 2 ? cluster_rank() : 0u;
    const bool leader = rank == 0;
    const int cid = (int)(blockIdx.x / G), ncl = (int)(gridDim.x / G);
    const int total = p.mtiles * p.ntiles;
    auto set_abort = [&]() {
        abort_sh = 1;
        if (G == 2) st_cluster_u32(mapa(su32((const void *)&abort_sh), rank ^ 1u), 1u);
    };
    if (warp == 0) {
        tmem_alloc<G>(&tmem_sh, TMEM_COLS);
    } else if (warp == 1) {
        if (lane < Q4_STAGES) {
            mbar_init(&full_bar[lane], 1 + G * Q4_EXPAND);  // the (leader's) loader, every expanding warp
            mbar_init(&empty_bar[lane], 1);
        }
        if (lane >= 8 && lane < 10) {
            mbar_init(&accf_bar[lane - 8], 1);
            mbar_init(&acce_bar[lane - 8], G * 4);
        }
        if (lane == 10) {
            abort_sh = 0;
            issued_sh = cissued_sh = consumed_sh = 0;
        }
        if (lane >= 16 && lane < 16 + Q4_CSTAGES) {
            mbar_init(&cfull_bar[lane - 16], 1);
            mbar_init(&cempty_bar[lane - 16], F32 ? Q4_TURNS * Q4_EXPAND : Q4_EXPAND);  // (fp32: every group reads a block)
        }
        fence_mbar_init();
    } else if (warp == 2 && lane < 3) {
        const CUtensorMap *m = lane == 0 ? &mX : lane == 1 ? &mC : &mS;
        asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(m)) : "memory");
    }
    if (G == 2) cluster_sync_all();
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = __shfl_sync(0xffffffffu, tmem_sh, 0);
    griddep_launch();  // (behind the allocation: see tmem_alloc)

    if (warp == 0) {
        if (lane == 0) {  // ---------------- loader of x
            int s = 0, g = 0;
            uint32_t par = 0;
            bool stop = false;
            griddep_wait();
            for (int t = cid; t < total && !stop; t += ncl) {
                const int m0 = (t / p.ntiles * G + (int)rank) * BM;
                for (int it = 0; it < p.steps; ++it, ++g) {
                    if (!mbar_wait(&empty_bar[s], par ^ 1u, p.wait_limit)) {
                        atomicOr(p.err, ERR_TMA_WAIT);
                        set_abort();
                    }
                    if (abort_sh) {
                        stop = true;
                        break;
                    }
                    if (leader) mbar_expect_tx(&full_bar[s], G * Q4_A_BYTES);
                    const uint32_t bar = G == 2 ? mapa(su32(&full_bar[s]), 0u) : su32(&full_bar[s]);
                    const int kb = F32 ? it / COMBOS : it, c = F32 ? it - kb * COMBOS : 0;
                    const int plane = F32 ? (c < 3 ? c + 1 : c == 3 ? 1 : 0) : 0;
                    tma_2d<G>(su32(smem + s * Q4_STAGE), &mX, bar, kb * BK, m0 + plane * p.plane_rows);
                    if (++s == Q4_STAGES) {
                        s = 0;
                        par ^= 1u;
                    }
                }
            }
            issued_sh = g;
        }
    } else if (warp == 1) {
        if (leader) {  // ---------------- MMA issuer: the whole warp, one lane of which issues
            const uint32_t one = elect_one();
            const uint32_t idesc = idesc_f16<T>(BM * G, p.bn);
            const uint64_t desc0 = sdesc_sw128(su32(smem));
            int g = 0, lt = 0, s = 0, i0 = 0;
            uint32_t par = 0;
            bool stop = false;
            for (int t = cid; t < total && !stop; ++lt) {  // run lt: steps i0 to i1 of tile t
                const int b = lt & 1, i1 = min(i0 + p.run, p.steps);
                const uint32_t aph = (uint32_t)(lt >> 1) & 1u;
                if (!__all_sync(0xffffffffu, G == 2 ? mbar_wait_cluster(&acce_bar[b], aph ^ 1u, p.wait_limit)
                                                    : mbar_wait(&acce_bar[b], aph ^ 1u, p.wait_limit))) {
                    if (lane == 0) {
                        atomicOr(p.err, ERR_EPI_WAIT);
                        set_abort();
                    }
                    break;
                }
                tc_fence_after();
                const uint32_t d = tmem + (uint32_t)b * ACC;
                for (int it = i0; it < i1; ++it, ++g) {
                    if (!__all_sync(0xffffffffu, G == 2 ? mbar_wait_cluster(&full_bar[s], par, p.wait_limit)
                                                        : mbar_wait(&full_bar[s], par, p.wait_limit))) {
                        if (lane == 0) {
                            atomicOr(p.err, ERR_MMA_WAIT);
                            set_abort();
                        }
                        stop = true;
                        break;
                    }
                    tc_fence_after();
                    const uint64_t da = desc0 + (uint64_t)((s * Q4_STAGE) >> 4), db = da + (Q4_A_BYTES >> 4);
#pragma unroll
                    for (int k = 0; k < BK / 16; ++k) umma_one<G>(one, d, da + 2 * k, db + 2 * k, idesc, (it > i0 || k > 0) ? 1u : 0u);
                    commit_one<G>(one, &empty_bar[s]);
                    if (++s == Q4_STAGES) {
                        s = 0;
                        par ^= 1u;
                    }
                }
                if (!stop) commit_one<G>(one, &accf_bar[b]);
                i0 = i1;
                if (i0 == p.steps) i0 = 0, t += ncl;
            }
            if (lane == 0) consumed_sh = g;
        }
    } else if (warp >= 4 && warp < 8) {  // ---------------- epilogue: 32 rows a warp
        const int q = warp - 4;
        uint8_t *out = stg + q * 32 * Q4_OUT_ROW;
        griddep_wait();
        int lt = 0, i0 = 0;
        for (int t = cid; t < total; ++lt) {
            const int b = lt & 1;
            const bool first = i0 == 0;
            i0 += p.run;
            const bool last = i0 >= p.steps;
            const int64_t r0 = (int64_t)(t / p.ntiles * G + (int)rank) * BM + q * 32;
            const int n0 = t % p.ntiles * p.bn;
            if (!mbar_wait(&accf_bar[b], (uint32_t)(lt >> 1) & 1u, p.wait_limit)) {
                if (lane == 0) {
                    atomicOr(p.err, ERR_ACC_WAIT);
                    set_abort();
                }
                break;
            }
            tc_fence_after();
            if (r0 < p.rows) {
#pragma unroll 1
                for (int c0 = 0; c0 < p.bn && n0 + c0 < p.q.n; c0 += 32) {
                    const int j0 = n0 + c0;
                    uint32_t v[32];
                    const uint32_t acc = tmem + ((uint32_t)(q * 32) << 16) + (uint32_t)c0;
                    __syncwarp();
                    tmem_ld32(acc + (uint32_t)b * ACC, v);
                    if constexpr (F32) {
                        if (!first) {
                            uint32_t sum[32];
                            tmem_ld32(acc + 2 * ACC, sum);
#pragma unroll
                            for (int i = 0; i < 32; ++i) v[i] = __float_as_uint(__uint_as_float(v[i]) + __uint_as_float(sum[i]));
                        }
                        if (!last) {
                            tmem_st32(acc + 2 * ACC, v);
                            continue;
                        }
                    }
                    bias_sh[q][lane] = p.q.bias && j0 + lane < p.q.n ? p.q.bias[j0 + lane] : 0.0f;
                    if constexpr (std::is_same<X, __half>::value)
                        pow_sh[q][lane] = j0 + lane < p.q.n ? p.q.row_pow[j0 + lane] * 0x1p-12f : 0.0f;
                    __syncwarp();
                    X *mine = reinterpret_cast<X *>(out + lane * Q4_OUT_ROW);
                    constexpr int V = 16 / sizeof(X);  // values in 16 bytes
#pragma unroll
                    for (int i = 0; i < 32; i += V) {
                        struct alignas(16) {
                            X v[V];
                        } piece;
#pragma unroll
                        for (int e = 0; e < V; ++e) {
                            float f = __uint_as_float(v[i + e]);
                            if constexpr (std::is_same<X, __half>::value) f *= pow_sh[q][i + e];
                            piece.v[e] = cvt<X>(act_apply(f + bias_sh[q][i + e], p.q.act));
                        }
                        *reinterpret_cast<uint4 *>(mine + i) = *reinterpret_cast<const uint4 *>(&piece);
                    }
                    __syncwarp();
                    const int live = (int)min((int64_t)32, p.rows - r0), cols = min(32, p.q.n - j0);
                    if (p.vec_out && cols == 32) {
                        constexpr int LPR = 32 / V;  // lanes a row
#pragma unroll
                        for (int r = 0; r < 32; r += 32 / LPR) {
                            const int row = r + lane / LPR;
                            if (row < live)
                                *reinterpret_cast<uint4 *>(y + (r0 + row) * p.ldy + j0 + lane % LPR * V) =
                                    *reinterpret_cast<const uint4 *>(out + row * Q4_OUT_ROW + lane % LPR * 16);
                        }
                    } else if (lane < cols) {
                        for (int r = 0; r < live; ++r)
                            y[(r0 + r) * p.ldy + j0 + lane] = reinterpret_cast<const X *>(out + r * Q4_OUT_ROW)[lane];
                    }
                }
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) {
                if (G == 2) mbar_arrive_cluster(mapa(su32(&acce_bar[b]), 0u));
                else mbar_arrive(&acce_bar[b]);
            }
            if (last) i0 = 0, t += ncl;
        }
    } else if (warp == 2) {
        if (lane == 0) {  // ---------------- loader of codes and scales (not written by the kernel before)
            const int own = p.bn / G, halves = p.q.glog == 5 ? 2 : 1;
            const uint32_t bytes = (uint32_t)(own / 16) * (512 + 32 * halves);
            int s = 0, g = 0;
            uint32_t par = 0;
            bool stop = false;
            for (int t = cid; t < total && !stop; t += ncl) {
                const int tile = (t % p.ntiles * p.bn + (int)rank * own) / 16;
                for (int kb = 0; kb < p.q.kb; ++kb, ++g) {
                    if (!mbar_wait(&cempty_bar[s], par ^ 1u, p.wait_limit)) {
                        atomicOr(p.err, ERR_TMA_WAIT);
                        set_abort();
                    }
                    if (abort_sh) {
                        stop = true;
                        break;
                    }
                    const uint32_t dst = su32(cst + s * Q4_CSTAGE), bar = su32(&cfull_bar[s]);
                    mbar_expect_tx(&cfull_bar[s], bytes);
                    tma_3d<1>(dst, &mC, bar, 0, kb, tile);
                    tma_3d<1>(dst + Q4_CBYTES, &mS, bar, 0, halves == 2 ? 2 * kb : kb >> (p.q.glog - 6), tile);
                    if (++s == Q4_CSTAGES) {
                        s = 0;
                        par ^= 1u;
                    }
                }
            }
            cissued_sh = g;
        }
    } else if (warp >= 8) {  // ---------------- weights: this CTA's rows, two 16-row tiles a warp
        const int grp = (warp - 8) / Q4_EXPAND, dw = (warp - 8) % Q4_EXPAND;
        // a lane takes the tile's row pair g and columns t4 of each half such that eight
        // lanes' 16-byte pieces, four of row g and four of row g + 4, cover all banks
        const int g = lane / 8 + 4 * (lane % 8 / 4), t4 = lane % 4;
        const int tiles = p.bn / G / 16, halves = p.q.glog == 5 ? 2 : 1;
        const uint32_t at[2] = {(uint32_t)g * 128 + ((uint32_t)(t4 ^ g) << 4), (uint32_t)g * 128 + ((uint32_t)((4 + t4) ^ g) << 4)};
        const uint32_t full0 = G == 2 ? mapa(su32(full_bar), 0u) : su32(full_bar);
        // Stages are filled by the groups in turn.  A group's fill f waits until fill f - 5
        // has been read; it last waited for fill f - 8, so the barrier it looks at is never
        // two phases behind what it waits for, which parities could not tell apart.
        static_assert(Q4_TURNS < Q4_STAGES, "a group waits in every round of the stages");
        int s = 0, cs = 0, turn = 0;  // stage of the operands, stage of the codes, whose fill it is
        uint32_t par = 0, cpar = 0;
        bool stop = false;  // (an aborting pair's barriers stand still, so the waits here end by themselves)
        auto give_up = [&]() {
            if (lane == 0) {
                atomicOr(p.err, ERR_TMA_WAIT);
                set_abort();
            }
            stop = true;
        };
        for (int t = cid; t < total && !stop; t += ncl) {
            float rp[2][2];
            if constexpr (std::is_same<T, __half>::value) {
                const int tile = (t % p.ntiles * p.bn + (int)rank * (p.bn / G)) / 16 + dw;
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int r = 0; r < 2; ++r)
                        rp[i][r] = 0x1p12f / __ldg(p.q.row_pow + min(tile + i * Q4_EXPAND, p.q.nt - 1) * 16 + g + 8 * r);
            }
            for (int kb = 0; kb < p.q.kb && !stop; ++kb) {
                uint4 cw[2];
                Scale2 sc[2][2][2];  // [tile][row g, row g + 8][half]
                if (F32 || turn == grp) {
                    if (!__all_sync(0xffffffffu, mbar_wait(&cfull_bar[cs], cpar, p.wait_limit))) {
                        give_up();
                        break;
                    }
                    const uint8_t *cb = cst + cs * Q4_CSTAGE;
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const int tile = dw + i * Q4_EXPAND;  // (behind the last: whatever lies there)
                        cw[i] = *reinterpret_cast<const uint4 *>(cb + tile * 512 + (4 * g + t4) * 16);
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            if (h < halves) {
                                const uint32_t sw =
                                    *reinterpret_cast<const uint32_t *>(cb + Q4_CBYTES + (tile * halves + h) * 32 + g * 4);
                                if (std::is_same<T, __nv_bfloat16>::value && p.q.scale_bf16) {
                                    sc[i][0][h] = Scale2{__byte_perm(sw, sw, 0x1010), 0u};  // the scale is its own large part
                                    sc[i][1][h] = Scale2{__byte_perm(sw, sw, 0x3232), 0u};
                                } else {
                                    float2 f = scale_pair(sw, p.q.scale_bf16);
                                    if constexpr (std::is_same<T, __half>::value) f = make_float2(f.x * rp[i][0], f.y * rp[i][1]);
                                    sc[i][0][h] = scale_parts<T>(f.x);
                                    sc[i][1][h] = scale_parts<T>(f.y);
                                }
                            } else {
                                sc[i][0][h] = sc[i][0][0];
                                sc[i][1][h] = sc[i][1][0];
                            }
                        }
                    }
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&cempty_bar[cs]);
                }
#pragma unroll 1
                for (int c = 0; c < COMBOS; ++c) {
                    if (turn == grp) {
                        if (!__all_sync(0xffffffffu, mbar_wait(&empty_bar[s], par ^ 1u, p.wait_limit))) {
                            give_up();
                            break;
                        }
                        uint8_t *b = smem + s * Q4_STAGE + Q4_A_BYTES;
                        auto tile_rows = [&](auto parts) {
#pragma unroll
                            for (int i = 0; i < 2; ++i) {
                                const int tile = dw + i * Q4_EXPAND;
                                if (tile >= tiles) break;
                                const uint32_t w[4] = {cw[i].x, cw[i].y, cw[i].z, cw[i].w};
#pragma unroll
                                for (int r = 0; r < 2; ++r)
#pragma unroll
                                    for (int h = 0; h < 2; ++h) {
                                        uint32_t v[4];
#pragma unroll
                                        for (int e = 0; e < 4; ++e) {
                                            const uint32_t code = code_pair<T>(w[2 * h + e / 2], r + 2 * (e % 2));
                                            v[e] = expand<T>(code, sc[i][r][h], parts.value);
                                            if (F32 && (c == 2 || c == 3)) v[e] = expand_rest(code, sc[i][r][h], v[e]);
                                        }
                                        *reinterpret_cast<uint4 *>(b + tile * 2048 + r * 1024 + at[h]) = make_uint4(v[0], v[1], v[2], v[3]);
                                    }
                            }
                        };
                        if (F32 || p.parts) tile_rows(std::true_type{});
                        else tile_rows(std::false_type{});
                        fence_proxy_async_smem();
                        __syncwarp();
                        if (lane == 0) {
                            if (G == 2 && rank) arrive_expanded(full0 + 8 * s);
                            else mbar_arrive(&full_bar[s]);
                        }
                    }
                    if (++turn == Q4_TURNS) turn = 0;
                    if (++s == Q4_STAGES) {
                        s = 0;
                        par ^= 1u;
                    }
                }
                if (++cs == Q4_CSTAGES) {
                    cs = 0;
                    cpar ^= 1u;
                }
            }
        }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 0) {
        if (abort_sh && lane == 0) {
            // let the copies and MMAs in flight land before the memory goes away
            // (one deadline; a stage whose weights never came completes no phase)
            const long long t0 = clock64();
            if (leader)
                for (int g = consumed_sh; g < issued_sh; ++g)
                    while (!mbar_try(&full_bar[g % Q4_STAGES], (uint32_t)(g / Q4_STAGES) & 1u) && clock64() - t0 < WAIT_LIMIT) {
                    }
            for (int g = cissued_sh > Q4_CSTAGES ? cissued_sh - Q4_CSTAGES : 0; g < cissued_sh; ++g)
                while (!mbar_try(&cfull_bar[g % Q4_CSTAGES], (uint32_t)(g / Q4_CSTAGES) & 1u) && clock64() - t0 < WAIT_LIMIT) {
                }
            if (leader && consumed_sh > 0) {
                const int g = consumed_sh - 1;
                while (!mbar_try(&empty_bar[g % Q4_STAGES], (uint32_t)(g / Q4_STAGES) & 1u) && clock64() - t0 < WAIT_LIMIT) {
                }
            }
        }
        __syncwarp();
    }
    if (G == 2) cluster_sync_all();
    else __syncthreads();
    if (warp == 0) {
        tc_fence_after();
        tmem_dealloc<G>(tmem, TMEM_COLS);
    }
}

// x where TMA cannot read it in place: 16-bit rows copied to rows of `kp` values, fp32
// rows cut into bf16 planes of plane_rows rows
template <typename X>
__global__ void __launch_bounds__(256) q4_planes_kernel(const X *__restrict__ x, int64_t ldx, int64_t rows, int k, int kp,
                                                        int64_t plane_rows, void *__restrict__ out) {
    griddep_launch();
    griddep_wait();
    const int64_t row = blockIdx.x;
    for (int c = threadIdx.x; c < kp; c += 256) {
        const X v = c < k ? x[row * ldx + c] : cvt<X>(0.0f);
        if constexpr (std::is_same<X, float>::value) {
            const Planes pl = planes_of(v);
#pragma unroll
            for (int i = 0; i < 4; ++i)
                static_cast<__nv_bfloat16 *>(out)[(plane_rows * i + row) * kp + c] =
                    i < 3 ? pl.v[i] : fabsf(v) <= 3.4028234664e38f ? pl.v[0] : __float2bfloat16_rn(0.0f);
        } else {
            static_cast<X *>(out)[row * kp + c] = v;
        }
    }
}

bool in_place(int dt, const void *x, int64_t ldx) {
    return dt != SN_F32 && reinterpret_cast<uintptr_t>(x) % 16 == 0 && ldx % 8 == 0;
}

// Rows of x and outputs a tile: the pair of CTAs or the single one, and the width,
// whose rounds of tiles over the SMs times the time of a tile are least.  A step
// takes 2 BN cycles of the tensor core and at least about 256 for its weights; a
// tile some 1500 more to fill and drain.
struct Shape4 {
    int g, bn;
};
Shape4 choose(int64_t rows, int n, int64_t steps, int widest) {
    Shape4 best{1, 32};
    double least = 1e300;
    for (int g = 1; g <= 2; ++g)
        for (int bn = 32; bn <= std::min(widest, 128 * g); bn += 32) {
            const int64_t tiles = ((rows + 128 * g - 1) / (128 * g)) * ((n + bn - 1) / bn);
            const int64_t slots = num_sms() / g, rounds = (tiles + slots - 1) / slots;
            const double cost = (double)rounds * ((double)std::max(2 * bn, 256) * (double)steps + 1500.0);
            if (cost < least) {
                least = cost;
                best = Shape4{g, bn};
            }
        }
    return best;
}

template <typename T, typename X, int G>
cudaError_t launch_prompt(const CUtensorMap &mX, PromptP &p, X *y, cudaStream_t st) {
    auto kern = q4_prompt_kernel<T, X, G>;
    static PerDevice set;
    if (const cudaError_t e = allow_smem(set, kern, Q4_SMEM)) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.blockDim = dim3(Q4_THREADS);
    cfg.dynamicSmemBytes = Q4_SMEM;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = G;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = G == 2 ? 2 : 1;
    const int64_t total = (int64_t)p.mtiles * p.ntiles;
    if (total > INT32_MAX) return cudaErrorInvalidValue;
    cfg.gridDim = dim3((unsigned)(G * std::min<int64_t>(total, num_sms() / G)));
    // codes as [nt][kb][256 halfwords], scales as [nt][kg][16]: a box is this CTA's tiles of one column block
    CUtensorMap mC, mS;
    const uint64_t cdims[3] = {256, (uint64_t)p.q.kb, (uint64_t)p.q.nt}, cstr[2] = {512, (uint64_t)p.q.kb * 512};
    const uint64_t sdims[3] = {16, (uint64_t)p.q.kg, (uint64_t)p.q.nt}, sstr[2] = {32, (uint64_t)p.q.kg * 32};
    const uint32_t tiles = (uint32_t)(p.bn / G / 16), cbox[3] = {256, 1, tiles}, sbox[3] = {16, p.q.glog == 5 ? 2u : 1u, tiles};
    if (!tma_encode(&mC, SN_F16, 3, p.q.codes, cdims, cstr, cbox, CU_TENSOR_MAP_SWIZZLE_NONE) ||
        !tma_encode(&mS, SN_F16, 3, p.q.scales, sdims, sstr, sbox, CU_TENSOR_MAP_SWIZZLE_NONE))
        return cudaErrorInvalidValue;
    return cudaLaunchKernelEx(&cfg, kern, mX, mC, mS, p, y);
}

template <typename T, typename X>
cudaError_t prompt(const sn_q4_weights &w, int dt, int64_t rows, const X *x, int64_t ldx, X *y, int64_t ldy, void *work,
                   cudaStream_t st) {
    constexpr bool F32 = std::is_same<X, float>::value;
    PromptP p{};
    p.q = q4_params(w);
    p.rows = rows;
    p.ldy = ldy;
    p.steps = p.q.kb * (F32 ? 5 : 1);
    const Shape4 sh = choose(rows, w.n, p.steps, F32 ? Q4_F32_BN : 256);
    p.run = F32 ? 5 : p.steps;
    p.bn = sh.bn;
    const int64_t mtiles = (rows + 128 * sh.g - 1) / (128 * sh.g);
    p.mtiles = (int32_t)mtiles;
    p.ntiles = (w.n + sh.bn - 1) / sh.bn;
    p.parts = F32 || !(std::is_same<T, __nv_bfloat16>::value && w.scale_dtype == SN_BF16);
    p.vec_out = reinterpret_cast<uintptr_t>(y) % 16 == 0 && (ldy * (int64_t)sizeof(X)) % 16 == 0;
    p.err = device_error_word();
    p.wait_limit = WAIT_LIMIT;
    const void *base = x;
    int64_t ld = ldx;
    uint64_t dims[2] = {(uint64_t)w.k, (uint64_t)rows};
    if (!in_place(dt, x, ldx)) {
        const int kp = p.q.kb * 64;
        const int64_t plane_rows = (rows + 255) / 256 * 256;
        const cudaError_t e = launch_pdl(q4_planes_kernel<X>, dim3((unsigned)rows), dim3(256), 0, st, x, ldx, rows, (int)w.k, kp,
                                         plane_rows, work);
        if (e != cudaSuccess) return e;
        base = work;
        ld = kp;
        dims[0] = (uint64_t)kp;
        if (F32) {
            p.plane_rows = (int32_t)plane_rows;
            dims[1] = (uint64_t)(4 * plane_rows);
        }
    }
    if (dims[1] > INT32_MAX) return cudaErrorInvalidValue;
    const uint64_t strides[1] = {(uint64_t)ld * 2};
    const uint32_t box[2] = {BK, BM};
    CUtensorMap mX;
    if (!tma_encode(&mX, std::is_same<T, __half>::value ? SN_F16 : SN_BF16, 2, base, dims, strides, box, CU_TENSOR_MAP_SWIZZLE_128B))
        return cudaErrorInvalidValue;
    return sh.g == 2 ? launch_prompt<T, X, 2>(mX, p, y, st) : launch_prompt<T, X, 1>(mX, p, y, st);
}

}  // namespace

size_t q4_prompt_workspace(const sn_q4_weights &w, int dt, int64_t rows, const void *x, int64_t ldx) {
    if (in_place(dt, x, ldx)) return 0;
    const int64_t kp = ((int64_t)w.k + 63) / 64 * 64;
    return (size_t)((rows + 255) / 256 * 256 * kp * 2 * (dt == SN_F32 ? 4 : 1));
}

cudaError_t q4_prompt(const sn_q4_weights &w, int dt, int64_t rows, const void *x, int64_t ldx, void *y, int64_t ldy, void *work,
                      cudaStream_t st) {
    if (dt == SN_F32)
        return prompt<__nv_bfloat16, float>(w, dt, rows, static_cast<const float *>(x), ldx, static_cast<float *>(y), ldy, work, st);
    if (dt == SN_F16)
        return prompt<__half, __half>(w, dt, rows, static_cast<const __half *>(x), ldx, static_cast<__half *>(y), ldy, work, st);
    return prompt<__nv_bfloat16, __nv_bfloat16>(w, dt, rows, static_cast<const __nv_bfloat16 *>(x), ldx,
                                                static_cast<__nv_bfloat16 *>(y), ldy, work, st);
}

}  // namespace k
}  // namespace sn
