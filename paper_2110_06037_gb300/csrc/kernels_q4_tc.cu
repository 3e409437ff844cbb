// 4-bit weights with many rows of x, on the 5th-generation tensor cores
// (sn_q4_dense in include/sn.h; layout in q4_common.cuh).
//
//   D[j, m] = sum over groups g of scale[j, g] * (sum over the group's k of q[j, k] * x[m, k])
//
// The codes themselves are the operand: in x's 16-bit type they are exact, and so is every
// product.  A group's sum is made in TMEM; the epilogue's warps read it, multiply it by the
// group's scale in fp32 and add it to sums that they keep in registers.  (Scaled weights
// as the operand would be rounded to x's type, or take two products.)
// fp32 x: three bf16 planes of x (written to scratch by a first kernel) times the codes,
// the smallest plane first: exact products again, three steps a column block.
// The tensor cores' sums are truncated, by some 1.4e-8 of them an MMA; here they run
// over one group, 24 MMAs at most.
//
// A tile is 128 outputs by BN rows of x, over pairs of column blocks (128 columns).  An
// output is a lane of TMEM, so that a group's scale is one value a thread.  x and codes
// come by TMA.  A thread expands the codes of one output and stores them into TMEM, from
// where the tensor core takes its left operand (shared memory keeps x alone).
//
// Warps: 0 loads x and allocates TMEM, 1 issues the MMAs, 3 waits for it, 2 loads codes, 4 to
// 11 take the groups' sums (two warps 32 outputs, half of the rows each) and write the
// outputs, 12 to 19 expand codes, two groups of four that fill stages in turn.  The sums
// take the registers that the other warps give up.  Waits are bounded; one that expires
// records its cause in the library's error word and stops the block.
//
// 4096 -> 8448, 2048 bf16 rows: 155 us with groups of 128 (917 TFLOP/s, 47% of a plain
// matrix product's measured rate), 227 with groups of 64, 389 with groups of 32; fp32 rows
// 417 (weights scaled in two bf16 parts took five products for the three: 895).  Bound by
// the hand-overs: a wait, an arrival and their instructions take a warp some 200 cycles
// each, and a pair of column blocks 1370 cycles (groups of 64: 2000, of 32: 3430), whatever BN
// is, where the tensor core takes 512.  With no sums read, no codes expanded and half
// of the MMAs it is 1200 (3000 of 32).  (One column block a stage: 268 us.  x's rows as the lanes,
// so that every column has a scale of its own: 256.)
#include <algorithm>

#include "q4_common.cuh"

namespace sn {
namespace k {

namespace {

using namespace tc;

// A stage is a pair of column blocks.
constexpr int Q4_XSTAGES = 5, Q4_WSTAGES = 2, Q4_CSTAGES = 4;  // of x, of expanded weights, of codes
constexpr int Q4_EPI = 8;                              // warps that take the groups' sums
constexpr int Q4_EXPAND = 4, Q4_TURNS = 2;             // warps that expand a stage; groups of them taking turns
constexpr int Q4_THREADS = (4 + Q4_EPI + Q4_EXPAND * Q4_TURNS) * 32;
constexpr int Q4_BN = 128;                             // most rows of x a tile
constexpr int Q4_BATCH = 4;                            // groups whose scales an epilogue thread asks for at once
constexpr uint32_t Q4_XBLOCK = Q4_BN * BK * 2, Q4_XSTAGE = 2 * Q4_XBLOCK, Q4_CSTAGE = 2 * 8 * 512;  // (eight tiles of codes, twice)
constexpr int Q4_OUT_ROW = 36;                         // staged outputs of a warp: 16 rows of 32 values and four against bank conflicts
constexpr uint32_t Q4_OUT = 16 * Q4_OUT_ROW * 4;
constexpr size_t Q4_SMEM = Q4_XSTAGES * (size_t)Q4_XSTAGE + Q4_CSTAGES * (size_t)Q4_CSTAGE + Q4_EPI * (size_t)Q4_OUT + 1024;
static_assert(Q4_SMEM <= 226 * 1024, "shared memory of a block");
// TMEM columns: accumulators, then the expanded weights (two a column)
constexpr int Q4_ACC = 3;
constexpr uint32_t Q4_WCOL = Q4_ACC * Q4_BN, Q4_WCOLS = 2 * BK / 2;
static_assert(Q4_WCOL + Q4_WSTAGES * Q4_WCOLS <= 512, "tensor memory of a block");
// Registers a thread: 96 at the launch (640 threads), then these (the issuer's and loaders' 48 or the
// expanding warps' 80 spill: 178 and 164 us for 155)
constexpr int Q4_REGS = 96, Q4_REGS_ISSUE = 56, Q4_REGS_EPI = 120, Q4_REGS_EXPAND = 88;
static_assert(4 * Q4_REGS_ISSUE + Q4_EPI * Q4_REGS_EPI + Q4_EXPAND * Q4_TURNS * Q4_REGS_EXPAND <= Q4_THREADS / 32 * Q4_REGS,
              "a share beyond what the block was launched with would be waited for without end");

struct PromptP {
    Q4P q;
    int64_t rows, ldy;
    int32_t mtiles, ntiles;  // tiles of outputs, of rows of x
    int32_t plane_rows;      // fp32: rows of a plane of x
    int32_t vec_out;         // y's rows begin at 16 bytes
    int *err;
};

template <int N>
__device__ __forceinline__ void regs_up() {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N));
}
template <int N>
__device__ __forceinline__ void regs_down() {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N));
}
// 16 columns on their way; they are there behind the wait, which names them
__device__ __forceinline__ void tmem_ask16(uint32_t ta, float (&a)[16]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
        : "=f"(a[0]), "=f"(a[1]), "=f"(a[2]), "=f"(a[3]), "=f"(a[4]), "=f"(a[5]), "=f"(a[6]), "=f"(a[7]), "=f"(a[8]), "=f"(a[9]),
          "=f"(a[10]), "=f"(a[11]), "=f"(a[12]), "=f"(a[13]), "=f"(a[14]), "=f"(a[15])
        : "r"(ta)
        : "memory");
}
__device__ __forceinline__ void tmem_have16(float (&a)[16]) {
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+f"(a[0]), "+f"(a[1]), "+f"(a[2]), "+f"(a[3]), "+f"(a[4]), "+f"(a[5]), "+f"(a[6]), "+f"(a[7]), "+f"(a[8]), "+f"(a[9]),
                   "+f"(a[10]), "+f"(a[11]), "+f"(a[12]), "+f"(a[13]), "+f"(a[14]), "+f"(a[15])::"memory");
}

// T: the operands' type; X: x's and y's; BN: rows of x a tile
template <typename T, typename X, int BN>
__global__ void __launch_bounds__(Q4_THREADS, 1)
    q4_prompt_kernel(const __grid_constant__ CUtensorMap mX, const __grid_constant__ CUtensorMap mC,
                     const __grid_constant__ PromptP p, X *__restrict__ y) {
    constexpr int PLANES = std::is_same<X, float>::value ? 3 : 1;
    extern __shared__ uint8_t smem_raw[];
    __shared__ __align__(8) uint64_t xfull_bar[Q4_XSTAGES], xempty_bar[Q4_XSTAGES], wfull_bar[Q4_WSTAGES], wempty_bar[Q4_WSTAGES];
    __shared__ __align__(8) uint64_t cfull_bar[Q4_CSTAGES], cempty_bar[Q4_CSTAGES], accf_bar[Q4_ACC], acce_bar[Q4_ACC], drain_bar;
    __shared__ uint32_t tmem_sh;
    __shared__ volatile int abort_sh;
    __shared__ int issued_sh, cissued_sh, consumed_sh;  // stages of x loaded, of codes loaded, of x multiplied
    uint8_t *smem = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    uint8_t *cst = smem + Q4_XSTAGES * Q4_XSTAGE, *stg = cst + Q4_CSTAGES * Q4_CSTAGE;
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const int total = p.mtiles * p.ntiles, pairs = (p.q.kb + 1) / 2;
    if (warp == 0) {
        tmem_alloc<1>(&tmem_sh, 512);
    } else if (warp == 1) {
        if (lane < Q4_XSTAGES) {
            mbar_init(&xfull_bar[lane], 1);
            mbar_init(&xempty_bar[lane], 1);
        }
        if (lane < Q4_WSTAGES) {
            mbar_init(&wfull_bar[lane], Q4_EXPAND);
            mbar_init(&wempty_bar[lane], 1);
        }
        if (lane < Q4_CSTAGES) {
            mbar_init(&cfull_bar[lane], 1);
            mbar_init(&cempty_bar[lane], Q4_EXPAND);
        }
        if (lane < Q4_ACC) {
            mbar_init(&accf_bar[lane], 1);
            mbar_init(&acce_bar[lane], Q4_EPI);
        }
        if (lane == 31) {
            mbar_init(&drain_bar, 1);
            abort_sh = 0;
            issued_sh = cissued_sh = consumed_sh = 0;
        }
        fence_mbar_init();
    } else if (warp == 2 && lane < 2) {
        const CUtensorMap *m = lane == 0 ? &mX : &mC;
        asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(m)) : "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = __shfl_sync(0xffffffffu, tmem_sh, 0);
    griddep_launch();  // (behind the allocation: see tmem_alloc)
    auto gave_up = [&](int code) {
        atomicOr(p.err, code);
        abort_sh = 1;
    };

    if (warp < 4) {
        regs_down<Q4_REGS_ISSUE>();
        if (warp == 0) {
            if (lane == 0) {  // ---------------- loader of x
                int s = 0, g = 0;
                uint32_t par = 0;
                griddep_wait();
                bool ok = true;  // (a block that gives up stands still, so the wait here ends by itself)
                for (int t = blockIdx.x; t < total && ok; t += gridDim.x) {
                    const int row = t % p.ntiles * BN;
                    for (int i = 0; i < pairs && ok; ++i) {
#pragma unroll
                        for (int plane = PLANES - 1; plane >= 0; --plane) {
                            if (!mbar_wait(&xempty_bar[s], par ^ 1u)) {
                                gave_up(ERR_TMA_WAIT);
                                ok = false;
                                break;
                            }
                            const uint32_t dst = su32(smem + s * Q4_XSTAGE), bar = su32(&xfull_bar[s]);
                            mbar_expect_tx(&xfull_bar[s], 2 * BN * BK * 2);  // (a block behind the last reads as zeros)
                            tma_2d<1>(dst, &mX, bar, 2 * i * BK, row + plane * p.plane_rows);
                            tma_2d<1>(dst + Q4_XBLOCK, &mX, bar, (2 * i + 1) * BK, row + plane * p.plane_rows);
                            ++g;
                            if (++s == Q4_XSTAGES) {
                                s = 0;
                                par ^= 1u;
                            }
                        }
                    }
                }
                issued_sh = g;
            }
        } else if (warp == 1 || warp == 3) {
            // ---------------- MMA issuer (warp 1: all of it runs, one lane issues) and its waiter (warp 3)
            // A wait of the issuing warp's own would queue behind the tensor core's operand reads, 250
            // cycles each; so the waiter waits, a step ahead, and the two meet at a hardware barrier.
            const bool issuer = warp == 1;
            const uint32_t one = elect_one();
            const uint32_t idesc = idesc_f16<T>(BM, BN);
            const uint64_t desc0 = sdesc_sw128(su32(smem));
            // A group's sum is one run, of a pair's 8 products 8, 4 or 2 (group 128, 64, 32) for each plane
            const int runs_all = 128 >> p.q.glog;
            int g = 0, s = 0, ws = 0, b = 0;
            uint32_t par = 0, wpar = 0, aph = 0;
            bool ok = true;
            for (int t = blockIdx.x; t < total && ok; t += gridDim.x) {
                for (int i = 0; i < pairs && ok; ++i) {
                    const int runs = 2 * i + 1 < p.q.kb ? runs_all : max(1, runs_all / 2);  // (the last pair may be half)
                    const uint32_t a = tmem + Q4_WCOL + (uint32_t)ws * Q4_WCOLS;
                    for (int r = 0; r < runs; ++r) {
                        if (!issuer) {  // all that the run needs at once, a barrier a lane
                            const int sl = s + lane < Q4_XSTAGES ? s + lane : s + lane - Q4_XSTAGES;
                            uint64_t *bar = lane < PLANES ? &xfull_bar[sl] : lane == PLANES ? &wfull_bar[ws] : &acce_bar[b];
                            const uint32_t parity = lane < PLANES ? par ^ (sl < s ? 1u : 0u) : lane == PLANES ? wpar : aph ^ 1u;
                            const bool need = lane == PLANES + 1 || (lane <= PLANES && r == 0);
                            ok = __all_sync(0xffffffffu, !need || mbar_wait(bar, parity));
                            if (!ok && lane == 0) gave_up(ERR_MMA_WAIT);
                        }
                        if (bar_red_or(BAR_MMA, 64, !ok)) {
                            ok = false;
                            break;
                        }
                        if (issuer) {
                            tc_fence_after();
                            const uint32_t d = tmem + (uint32_t)(b * Q4_BN);
#pragma unroll
                            for (int c = 0; c < PLANES; ++c) {
                                const int sc = s + c < Q4_XSTAGES ? s + c : s + c - Q4_XSTAGES;
                                const uint64_t db = desc0 + (uint64_t)((sc * Q4_XSTAGE) >> 4);
                                auto product = [&](int k, bool begins) {
                                    umma_ts_one(one, d, a + 8 * k, db + (uint64_t)(k / 4 * (Q4_XBLOCK >> 4) + k % 4 * 2), idesc, begins ? 0u : 1u);
                                };
                                if (runs_all == 1) {
#pragma unroll
                                    for (int k = 0; k < 8; ++k) product(k, c == 0 && k == 0);
                                } else if (runs_all == 2) {
#pragma unroll
                                    for (int k = 0; k < 4; ++k) product(4 * r + k, c == 0 && k == 0);
                                } else {
                                    product(2 * r, c == 0);
                                    product(2 * r + 1, false);
                                }
                            }
                            commit_one<1>(one, &accf_bar[b]);
                            if (r + 1 == runs) {
                                commit_one<1>(one, &wempty_bar[ws]);
#pragma unroll
                                for (int c = 0; c < PLANES; ++c) commit_one<1>(one, &xempty_bar[s + c < Q4_XSTAGES ? s + c : s + c - Q4_XSTAGES]);
                            }
                        }
                        if (++b == Q4_ACC) {
                            b = 0;
                            aph ^= 1u;
                        }
                    }
                    if (!ok) break;
                    g += PLANES;
                    if ((s += PLANES) >= Q4_XSTAGES) {
                        s -= Q4_XSTAGES;
                        par ^= 1u;
                    }
                    if (++ws == Q4_WSTAGES) {
                        ws = 0;
                        wpar ^= 1u;
                    }
                }
            }
            if (issuer && !ok) {  // the MMAs in flight end before the memory that they read and write goes away
                commit_one<1>(one, &drain_bar);
                mbar_wait(&drain_bar, 0u);
            }
            if (issuer && lane == 0) consumed_sh = g;
        } else if (warp == 2) {
            if (lane == 0) {  // ---------------- loader of codes (not written by the kernel before)
                int s = 0, g = 0;
                uint32_t par = 0;
                bool ok = true;
                for (int t = blockIdx.x; t < total && ok; t += gridDim.x) {
                    const int tile = t / p.ntiles * (BM / 16);
                    for (int i = 0; i < pairs; ++i, ++g) {
                        if (!mbar_wait(&cempty_bar[s], par ^ 1u)) {
                            gave_up(ERR_TMA_WAIT);
                            ok = false;
                            break;
                        }
                        mbar_expect_tx(&cfull_bar[s], Q4_CSTAGE);
                        tma_4d<1>(su32(cst + s * Q4_CSTAGE), &mC, su32(&cfull_bar[s]), 0, 0, 2 * i, tile);
                        if (++s == Q4_CSTAGES) {
                            s = 0;
                            par ^= 1u;
                        }
                    }
                }
                cissued_sh = g;
            }
        }
    } else if (warp < 4 + Q4_EPI) {  // ---------------- epilogue: 32 outputs and half of the rows a warp
        regs_up<Q4_REGS_EPI>();
        constexpr int COLS = BN / 2, LOADS = COLS / 16;
        const int q = warp % 4, half = (warp - 4) / 4;
        // This lane's scales, Q4_BATCH groups at once, the next ones on their way meanwhile (one group at
        // a time, passed on from register to register, each run waited for the load before)
        uint32_t now[Q4_BATCH], next[Q4_BATCH];
        auto ask = [&](int t, int g0) {
            const int j = t / p.ntiles * BM + q * 32 + lane;
            const uint16_t *from = reinterpret_cast<const uint16_t *>(p.q.scales) + ((int64_t)(j / 16) * p.q.kg + g0) * 16 + j % 8 * 2 + j / 8 % 2;
#pragma unroll
            for (int i = 0; i < Q4_BATCH; ++i) next[i] = j < p.q.n && g0 + i < p.q.kg ? __ldg(from + 16 * i) : 0;
        };
        if ((int)blockIdx.x < total) ask(blockIdx.x, 0);
        int b = 0;
        uint32_t ph = 0;
        bool ok = true;
        griddep_wait();
        for (int t = blockIdx.x; t < total; t += gridDim.x) {
            F2 acc[COLS / 2];
#pragma unroll
            for (int i = 0; i < COLS / 2; ++i) acc[i] = f2(0.0f, 0.0f);
#pragma unroll 1
            for (int g = 0; g < p.q.kg; ++g) {
                if (g % Q4_BATCH == 0) {
#pragma unroll
                    for (int i = 0; i < Q4_BATCH; ++i) now[i] = next[i];
                    if (g + Q4_BATCH < p.q.kg) ask(t, g + Q4_BATCH);
                    else if (t + (int)gridDim.x < total) ask(t + gridDim.x, 0);
                }
                const float own = scale_pair(now[0], p.q.scale_bf16).x;
                const F2 scale = f2(own, own);
#pragma unroll
                for (int i = 0; i + 1 < Q4_BATCH; ++i) now[i] = now[i + 1];
                if (!__all_sync(0xffffffffu, mbar_wait(&accf_bar[b], ph))) {
                    if (lane == 0) gave_up(ERR_ACC_WAIT);
                    ok = false;
                    break;
                }
                tc_fence_after();
                const uint32_t from = tmem + ((uint32_t)(q * 32) << 16) + (uint32_t)(b * Q4_BN + half * COLS);
#pragma unroll
                for (int i0 = 0; i0 < LOADS; i0 += 2) {  // 32 columns at once
                    constexpr int N = LOADS < 2 ? 1 : 2;
                    float v[N][16];
#pragma unroll
                    for (int i = 0; i < N; ++i) tmem_ask16(from + 16 * (i0 + i), v[i]);
#pragma unroll
                    for (int i = 0; i < N; ++i) tmem_have16(v[i]);
                    if (i0 + N == LOADS) {  // all of it has been read
                        tc_fence_before();
                        __syncwarp();
                        if (lane == 0) mbar_arrive(&acce_bar[b]);
                    }
#pragma unroll
                    for (int i = 0; i < N; ++i)
#pragma unroll
                        for (int j = 0; j < 16; j += 2) {
                            F2 &sum = acc[8 * (i0 + i) + j / 2];
                            sum = fma_2(f2(v[i][j], v[i][j + 1]), scale, sum);
                        }
                }
                if (++b == Q4_ACC) {
                    b = 0;
                    ph ^= 1u;
                }
            }
            if (!ok) break;
            // The outputs, 16 rows at a time through shared memory, one rolled loop for all of them: there a
            // lane takes eight neighbours of a row, or, where y's rows are not aligned or end, one of each row
            const int j0 = t / p.ntiles * BM + q * 32, j = j0 + lane;
            const int64_t r0 = (int64_t)(t % p.ntiles) * BN + half * COLS;
            const int live = (int)max((int64_t)0, min((int64_t)COLS, p.rows - r0));
            float *mine = reinterpret_cast<float *>(stg + (warp - 4) * Q4_OUT);
            const bool wide = p.vec_out && j0 + 32 <= p.q.n;
            float bias[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int je = wide ? j0 + lane % 4 * 8 + e : j;
                bias[e] = p.q.bias && je < p.q.n ? __ldg(p.q.bias + je) : 0.0f;
            }
#pragma unroll 1
            for (int c = 0; c < live; c += 16) {
#pragma unroll
                for (int i = 0; i < LOADS; ++i)
                    if (16 * i == c)
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            const float2 a = floats(acc[8 * i + e]);
                            mine[2 * e * Q4_OUT_ROW + lane] = a.x, mine[(2 * e + 1) * Q4_OUT_ROW + lane] = a.y;
                        }
                __syncwarp();
                auto put = [&](auto act) {
                    if (wide) {
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            const int row = 8 * e + lane / 4;
                            const float4 *from = reinterpret_cast<const float4 *>(mine + row * Q4_OUT_ROW + lane % 4 * 8);
                            const float4 a = from[0], b = from[1];
                            struct alignas(16) {
                                X v[8];
                            } piece;
                            piece.v[0] = cvt<X>(act(a.x + bias[0])), piece.v[1] = cvt<X>(act(a.y + bias[1]));
                            piece.v[2] = cvt<X>(act(a.z + bias[2])), piece.v[3] = cvt<X>(act(a.w + bias[3]));
                            piece.v[4] = cvt<X>(act(b.x + bias[4])), piece.v[5] = cvt<X>(act(b.y + bias[5]));
                            piece.v[6] = cvt<X>(act(b.z + bias[6])), piece.v[7] = cvt<X>(act(b.w + bias[7]));
                            uint4 *to = reinterpret_cast<uint4 *>(y + (r0 + c + row) * p.ldy + j0 + lane % 4 * 8);
                            if (c + row < live)
#pragma unroll
                                for (int k = 0; k < (int)sizeof(piece) / 16; ++k) to[k] = reinterpret_cast<const uint4 *>(&piece)[k];
                        }
                    } else if (j < p.q.n) {
                        X *to = y + (r0 + c) * p.ldy + j;
#pragma unroll 4
                        for (int e = 0; e < 16; ++e) {
                            const X v = cvt<X>(act(mine[e * Q4_OUT_ROW + lane] + bias[0]));
                            if (c + e < live) to[e * p.ldy] = v;
                        }
                    }
                };
                if (p.q.act == SN_ACT_NONE) put([](float v) { return v; });
                else put([&](float v) { return q4_act(v, p.q.act); });
                __syncwarp();
            }
        }
    } else {  // ---------------- weights: a thread expands two column blocks of one output
        regs_down<Q4_REGS_EXPAND>();
        const int grp = (warp - 4 - Q4_EPI) / Q4_EXPAND, q = warp % 4;  // (the lanes of TMEM that a warp reaches: by its number)
        // A row of 64 codes lies in four pieces of 16 bytes, piece i of the tile's row pair at i ^ (pair / 2)
        // (the copy's 64-byte swizzle: eight lanes' pieces cover all banks)
        const uint32_t at = (uint32_t)((2 * q + lane / 16) * 1024 + lane % 8 * 64), swz = (uint32_t)(lane % 8 / 2) << 4;
        const uint32_t shift = lane % 16 / 8 * 4;  // the pair's second row: the odd nibbles
        static_assert(Q4_WSTAGES % Q4_TURNS == 0 && Q4_CSTAGES % Q4_TURNS == 0, "a stage has one group, which sees all of its phases");
        const int64_t fills = (int)blockIdx.x < total ? (int64_t)((total - 1 - (int)blockIdx.x) / (int)gridDim.x + 1) * pairs : 0;
        int s = grp % Q4_WSTAGES, cs = grp % Q4_CSTAGES;
        uint32_t par = 0, cpar = 0;
        uint4 c[8];
        auto load = [&]() {  // the codes of the next fill
            if (!__all_sync(0xffffffffu, mbar_wait(&cfull_bar[cs], cpar))) return false;
            const uint8_t *cb = cst + cs * Q4_CSTAGE + at;
#pragma unroll
            for (int i = 0; i < 8; ++i) c[i] = *reinterpret_cast<const uint4 *>(cb + i / 4 * 512 + ((uint32_t)(16 * (i % 4)) ^ swz));
            __syncwarp();
            if (lane == 0) mbar_arrive(&cempty_bar[cs]);
            if ((cs += Q4_TURNS) >= Q4_CSTAGES) {
                cs -= Q4_CSTAGES;
                cpar ^= 1u;
            }
            return true;
        };
        uint32_t v[32];
        auto expand = [&](int block) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint4 &p = c[4 * block + i];
                const uint32_t w[4] = {p.x >> shift, p.y >> shift, p.z >> shift, p.w >> shift};
#pragma unroll
                for (int e = 0; e < 4; ++e) {  // word e of piece i: columns 32 (e / 2) + 8 i + 4 (e % 2) + 0..3 of its block
                    v[16 * (e / 2) + 4 * i + 2 * (e % 2)] = code_pair<T>(w[e], 0);
                    v[16 * (e / 2) + 4 * i + 2 * (e % 2) + 1] = code_pair<T>(w[e], 2);
                }
            }
        };
        bool ok = grp >= fills || load();
        for (int64_t f = grp; f < fills && ok; f += Q4_TURNS) {
            expand(0);
            if (!__all_sync(0xffffffffu, mbar_wait(&wempty_bar[s], par ^ 1u))) {
                ok = false;
                break;
            }
            tc_fence_after();
            const uint32_t to = tmem + ((uint32_t)(q * 32) << 16) + Q4_WCOL + (uint32_t)s * Q4_WCOLS;
            tmem_st32(to, v);
            expand(1);
            tmem_st32(to + 32, v);
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(&wfull_bar[s]);
            if ((s += Q4_TURNS) >= Q4_WSTAGES) {
                s -= Q4_WSTAGES;
                par ^= 1u;
            }
            if (f + Q4_TURNS < fills) ok = load();
        }
        if (!ok && lane == 0) gave_up(ERR_TMA_WAIT);
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 0) {
        if (abort_sh && lane == 0) {
            // let the copies in flight land before the memory goes away (one deadline)
            const long long t0 = clock64();
            for (int g = consumed_sh; g < issued_sh; ++g)
                while (!mbar_try(&xfull_bar[g % Q4_XSTAGES], (uint32_t)(g / Q4_XSTAGES) & 1u) && clock64() - t0 < WAIT_LIMIT) {
                }
            for (int g = cissued_sh > Q4_CSTAGES ? cissued_sh - Q4_CSTAGES : 0; g < cissued_sh; ++g)
                while (!mbar_try(&cfull_bar[g % Q4_CSTAGES], (uint32_t)(g / Q4_CSTAGES) & 1u) && clock64() - t0 < WAIT_LIMIT) {
                }
        }
        __syncwarp();
    }
    __syncthreads();
    if (warp == 0) {
        tc_fence_after();
        tmem_dealloc<1>(tmem, 512);
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
            for (int i = 0; i < 3; ++i) static_cast<__nv_bfloat16 *>(out)[(plane_rows * i + row) * kp + c] = pl.v[i];
        } else {
            static_cast<X *>(out)[row * kp + c] = v;
        }
    }
}

bool in_place(int dt, const void *x, int64_t ldx) {
    return dt != SN_F32 && reinterpret_cast<uintptr_t>(x) % 16 == 0 && ldx % 8 == 0;
}

// Rows of x a tile: the fewest with which the tiles take the least rounds over the SMs.
// A round's time does not depend on the rows (64 rows, 4096 -> 4096: 21.8 us in tiles of
// 32, 22.0 of 64, 23.6 of 128, one round each; 1024 rows, 2048 -> 2048: 61, 33 and 20 us
// in four, two and one).
int choose(int64_t rows, int n) {
    int best = 32;
    int64_t least = INT64_MAX;
    for (int bn = 32; bn <= Q4_BN; bn *= 2) {
        const int64_t tiles = (int64_t)((n + BM - 1) / BM) * ((rows + bn - 1) / bn), rounds = (tiles + num_sms() - 1) / num_sms();
        if (rounds < least) {
            least = rounds;
            best = bn;
        }
    }
    return best;
}

template <typename T, typename X, int BN>
cudaError_t launch_prompt(const CUtensorMap &mX, const PromptP &p, X *y, cudaStream_t st) {
    auto kern = q4_prompt_kernel<T, X, BN>;
    static PerDevice set;
    if (const cudaError_t e = allow_smem(set, kern, Q4_SMEM)) return e;
    const int64_t total = (int64_t)p.mtiles * p.ntiles;
    if (total > INT32_MAX / 2) return cudaErrorInvalidValue;  // (a block's next tile is counted in 32 bits)
    // codes as [nt][kb][8 row pairs][32 halfwords]: a box is eight tiles of two column blocks
    CUtensorMap mC;
    const uint64_t dims[4] = {32, 8, (uint64_t)p.q.kb, (uint64_t)p.q.nt}, strides[3] = {64, 512, (uint64_t)p.q.kb * 512};
    const uint32_t box[4] = {32, 8, 2, BM / 16};
    if (!tma_encode(&mC, SN_F16, 4, p.q.codes, dims, strides, box, CU_TENSOR_MAP_SWIZZLE_64B)) return cudaErrorInvalidValue;
    return launch_pdl(kern, dim3((unsigned)std::min<int64_t>(total, num_sms())), dim3(Q4_THREADS), Q4_SMEM, st, mX, mC, p, y);
}

template <typename T, typename X>
cudaError_t prompt(const sn_q4_weights &w, int dt, int64_t rows, const X *x, int64_t ldx, X *y, int64_t ldy, void *work,
                   cudaStream_t st) {
    constexpr bool F32 = std::is_same<X, float>::value;
    PromptP p{};
    p.q = q4_params(w);
    p.rows = rows;
    p.ldy = ldy;
    const int bn = choose(rows, w.n);
    p.mtiles = (w.n + BM - 1) / BM;
    p.ntiles = (int32_t)((rows + bn - 1) / bn);
    p.err = device_error_word();
    p.vec_out = reinterpret_cast<uintptr_t>(y) % 16 == 0 && ldy * (int64_t)sizeof(X) % 16 == 0;
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
            dims[1] = (uint64_t)(3 * plane_rows);
        }
    }
    if (dims[1] > INT32_MAX) return cudaErrorInvalidValue;
    const uint64_t strides[1] = {(uint64_t)ld * 2};
    const uint32_t box[2] = {BK, (uint32_t)bn};
    CUtensorMap mX;
    if (!tma_encode(&mX, std::is_same<T, __half>::value ? SN_F16 : SN_BF16, 2, base, dims, strides, box, CU_TENSOR_MAP_SWIZZLE_128B))
        return cudaErrorInvalidValue;
    if (bn == 32) return launch_prompt<T, X, 32>(mX, p, y, st);
    if (bn == 64) return launch_prompt<T, X, 64>(mX, p, y, st);
    return launch_prompt<T, X, 128>(mX, p, y, st);
}

}  // namespace

size_t q4_prompt_workspace(const sn_q4_weights &w, int dt, int64_t rows, const void *x, int64_t ldx) {
    if (in_place(dt, x, ldx)) return 0;
    const int64_t kp = ((int64_t)w.k + 63) / 64 * 64;
    return (size_t)((rows + 255) / 256 * 256 * kp * 2 * (dt == SN_F32 ? 3 : 1));
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
