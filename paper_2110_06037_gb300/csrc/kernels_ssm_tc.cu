// Selective scan of bf16 tokens by matrix products on the 5th-generation tensor
// cores (sn_ssm_scan in include/sn.h).
//
// A chunk of 128 tokens of one head, S the state before it, a_i = d_i a, and
// A_t = a_0 + .. + a_t:
//   Y   = e^{A_t} C S^T  +  (C B^T o e^{A_t - A_s} d_s [s <= t]) X
//   S'  = e^{A_127} S  +  (e^{A_127 - A_s} d_s X)^T B
// so the recurrence runs from chunk to chunk, and a chunk is four products:
//   pairs   C B^T       128 x 128, K = N       both as they lie in xbc
//   carried C S^T       128 x P,   K = N       S in two bf16 parts
//   inside  P X         128 x P,   K = 128     P (the pairs, weighted) in two parts, from TMEM
//   made    B^T X'      N x P,     K = 128     X' = weighted X in three parts
// x, B and C are bf16, exact operands; what is computed goes in as bf16 parts: two for
// the outputs, which are bf16 (2^-18 of a factor is lost, and by the decays 2^-24 of sums of
// 16 steps, see TABLE), three for the state, which goes on in
// fp32 (off by 9e-8 of itself; with two parts 2.4e-6, and 9 us less for 8192 tokens).
// It stays in registers: each chunk's product is added by an fp32 multiply-add, since
// the tensor core's own sums do not round to nearest.
//
// Work: a block of one SM takes one head, 64 of its channels and a segment of a
// sequence's chunks.  With few heads the sequence is cut into segments: a first pass
// makes the states of (finer) segments from nothing, the last product alone, and the
// second starts each segment from the joined ones.  A small kernel before both turns
// time steps into sums of a and weights, once per token and head.
//
// Each product has warps of its own for what goes into and comes out of it, so that
// only the state's one multiply-add a chunk runs from chunk to chunk: in one order, two
// blocks an SM, a chunk took a block 17.9 thousand cycles of waiting for one step after
// the other: 198 us for 8192 tokens of 64 heads (64 channels, N = 128).  So: 159 us, of
// which 7 are the time steps, 32 the first pass, 118 the second, 7300 cycles a chunk.
// The tensor cores are busy in 38% of them, schedulers issue in 49%; what
// bounds it is the way from the pairs to P and to the next pairs.  (Tried and no faster: the next
// chunk's pairs ahead, in TMEM of their own, 163; X' by the state's warps, 163; P's
// columns 32 at a time, 165.)
// Non-finite x: 0 * NaN would reach tokens before it, so such an x goes into the
// product as 0 and makes its channel NaN from its token on; into the state it goes as
// it is.  Waits are bounded.
#include <algorithm>

#include "ssm_common.cuh"
#include "tc_common.cuh"

namespace sn {
namespace k {

namespace {

using namespace tc;

constexpr int Q = 128;          // tokens a chunk
constexpr int PB = 64;          // channels a block
constexpr float LOG2E = 1.4426950408889634f;

// Per chunk and head, in units of log 2, v_t = d_t a: A_t, the sum of v from the chunk's start to t;
// weights for the state d_s e^{A_127 - A_s}; and for the pairs' weights, by blocks of 16 tokens:
// R_t, the sum from the block's start to t; log2 d_s - R_s; d; what lies between blocks.  A pair's decay is
// R_t - R_s and the sums of the blocks from s's to t's: a difference of sums of 16 steps, those
// below -126 as -126 (nothing passes them).  It is off by 2^-24 of such sums; a difference A_t - A_s is by
// that of a chunk's, 1e-3 where steps with a = -16 are 20, and the diagonal's weight, d_t, with it.
constexpr int TAB_W = Q, TAB_F = 2 * Q, TAB_R = 3 * Q, TAB_D = 4 * Q, TAB_S = 5 * Q, TABLE = 5 * Q + 64;

struct TcP {
    SsmP s;
    int32_t segs, step;      // segments a sequence at most; chunks of a segment at least
    int32_t fine;            // finer ones of the first pass in each
    float *table, *total;    // [chunks][H][TABLE], [chunks][H]: A_127
    float *part;             // [tokens / Q / step * fine][H][p blocks][64][N]: state before the first, then after fine segment j
    int32_t pblocks;
    int *err;
};

// index of a chunk's table: unique for chunk c of sequence b, since each sequence
// before it has at most its tokens / Q + 1 chunks
__device__ __forceinline__ int64_t chunk_at(const Seq &s, int b, int c) { return s.first / Q + b + c; }
// segments of one sequence; one of two and more has as many as it has steps, or fewer, so that the
// states of sequences before it end where its own begin, at first / Q / step
__device__ __forceinline__ int own_segments(int len, const TcP &p) { return max(1, min(p.segs, len / Q / p.step)); }
// segment g of a sequence: chunks [first, last)
__device__ __forceinline__ int2 segment(int len, int segs, int g) {
    const int chunks = (len + Q - 1) / Q;
    return make_int2((int)((int64_t)chunks * g / segs), (int)((int64_t)chunks * (g + 1) / segs));
}

// ------------------------------------------------------------ time steps
// a block takes eight heads of a chunk, a warp one of them
__global__ void __launch_bounds__(256) ssm_steps_kernel(const __grid_constant__ TcP p, const __nv_bfloat16 *__restrict__ dtv, int vec) {
    __shared__ float sh[8][Q + 1];
    griddep_launch();
    griddep_wait();
    const int b = blockIdx.z, c = blockIdx.x, h0 = blockIdx.y * 8, nh = min(8, p.s.H - h0);
    const Seq s = sequence(p.s.q, b);
    if ((int64_t)c * Q >= s.len) return;
    const int n = min(Q, s.len - c * Q), warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    if (vec) {
        const int t = threadIdx.x;
        if (t < n) {
            const uint4 u = *reinterpret_cast<const uint4 *>(dtv + (s.first + c * Q + t) * p.s.lddt + h0);
            const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float2 f = unpack2<__nv_bfloat16>(w[i]);
                sh[2 * i][t] = f.x, sh[2 * i + 1][t] = f.y;
            }
        }
    } else {
        for (int e = threadIdx.x; e < Q * 8; e += 256)
            if (e / 8 < n && e % 8 < nh) sh[e % 8][e / 8] = ldf(dtv + (s.first + c * Q + e / 8) * p.s.lddt + h0 + e % 8);
    }
    __syncthreads();
    const int hh = warp;
    if (hh < nh) {
        const int head = h0 + hh;
        const float a = p.s.a[head] * LOG2E, bias = p.s.dt_bias ? p.s.dt_bias[head] : 0.0f;
        // a lane's four tokens; sums up to them and from behind them
        float d[4], v[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int t = 4 * lane + i;
            d[i] = t < n ? softplus(sh[hh][t] + bias) : 0.0f;
            v[i] = d[i] * a;
            if (!(d[i] > 0.0f) && !(d[i] != d[i])) v[i] = 0.0f;  // (a step of 0 with any a)
        }
        const float mine = (v[0] + v[1]) + (v[2] + v[3]);
        float up = mine, down = mine;
#pragma unroll
        for (int o = 1; o < 32; o *= 2) {
            const float x = __shfl_up_sync(0xffffffffu, up, o), y = __shfl_down_sync(0xffffffffu, down, o);
            if (lane >= o) up += x;
            if (lane + o < 32) down += y;
        }
        float before = __shfl_up_sync(0xffffffffu, up, 1), behind = __shfl_down_sync(0xffffffffu, down, 1);
        if (lane == 0) before = 0.0f;
        if (lane == 31) behind = 0.0f;
        float4 A, W;
        A.x = before + v[0], A.y = A.x + v[1], A.z = A.y + v[2], A.w = A.z + v[3];
        float r = behind;
        W.w = d[3] * exp2f(r), r += v[3];
        W.z = d[2] * exp2f(r), r += v[2];
        W.y = d[1] * exp2f(r), r += v[1];
        W.x = d[0] * exp2f(r);
        // the sums inside blocks of 16 tokens, four lanes each
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = v[i] < -126.0f ? -126.0f : v[i];  // (NaN stays)
        const float low = (v[0] + v[1]) + (v[2] + v[3]);
        up = low;
#pragma unroll
        for (int o = 1; o < 4; o *= 2) {
            const float x = __shfl_up_sync(0xffffffffu, up, o, 4);
            if (lane % 4 >= o) up += x;
        }
        before = __shfl_up_sync(0xffffffffu, up, 1, 4);
        if (lane % 4 == 0) before = 0.0f;
        float4 R;
        R.x = before + v[0], R.y = R.x + v[1], R.z = R.y + v[2], R.w = R.z + v[3];
        const int64_t at = chunk_at(s, b, c) * p.s.H + head;
        float *tab = p.table + at * TABLE;
        auto put = [&](int which, const float4 &f) { *reinterpret_cast<float4 *>(tab + which + 4 * lane) = f; };
        put(0, A);
        put(TAB_W, W);
        put(TAB_F, make_float4(log2f(d[0]) - R.x, log2f(d[1]) - R.y, log2f(d[2]) - R.z, log2f(d[3]) - R.w));
        put(TAB_R, R);
        put(TAB_D, make_float4(d[0], d[1], d[2], d[3]));
        // the sums of the blocks from kb to t's, for t in block e / 8 and the four kb of each half of P's warps
        float between[2] = {0.0f, 0.0f};
#pragma unroll
        for (int k = 0; k < Q / 16; ++k) {
            const float sum = __shfl_sync(0xffffffffu, R.w, 4 * k + 3);
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int e = lane + 32 * i, kb = 4 * (e % 4 / 2) + 2 * (e / 4 % 2) + e % 2;
                between[i] += k >= kb && k < e / 8 ? sum : 0.0f;
            }
        }
        tab[TAB_S + lane] = between[0], tab[TAB_S + 32 + lane] = between[1];
        if (lane == 31) p.total[at] = A.w;
    }
}

// ------------------------------------------------------------- PTX pieces
// an MN-major operand: rows of 128 bytes are 64 values of the M or N axis at one k,
// 128-byte swizzled; groups of 8 k 1024 bytes apart, blocks of 64 values `block` bytes
__device__ __forceinline__ uint64_t sdesc_mn(uint32_t saddr, uint32_t block) {
    uint64_t d = 0;
    d |= (uint64_t)((saddr & 0x3FFFFu) >> 4);
    d |= (uint64_t)(block >> 4) << 16;
    d |= (uint64_t)(1024 >> 4) << 32;
    d |= (uint64_t)1 << 46;
    d |= (uint64_t)2 << 61;
    return d;
}
constexpr uint32_t A_MN = 1u << 15, B_MN = 1u << 16;  // instruction descriptor: operand is MN-major
__device__ __forceinline__ void tmem_st8(uint32_t taddr, const uint32_t (&v)[8]) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"r"(taddr), "r"(v[0]), "r"(v[1]),
                 "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7])
                 : "memory");
}
// 16 columns, at one, two or three addresses (the wait in the same statement: nothing of them is used before it)
__device__ __forceinline__ void tmem_ld16(uint32_t ta, float (&a)[16]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];\n\t"
        "tcgen05.wait::ld.sync.aligned;"
        : "=f"(a[0]), "=f"(a[1]), "=f"(a[2]), "=f"(a[3]), "=f"(a[4]), "=f"(a[5]), "=f"(a[6]), "=f"(a[7]), "=f"(a[8]), "=f"(a[9]),
          "=f"(a[10]), "=f"(a[11]), "=f"(a[12]), "=f"(a[13]), "=f"(a[14]), "=f"(a[15])
        : "r"(ta)
        : "memory");
}
__device__ __forceinline__ void tmem_ld16x2(uint32_t ta, float (&a)[16], uint32_t tb, float (&b)[16]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%32];\n\t"
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%33];\n\t"
        "tcgen05.wait::ld.sync.aligned;"
        : "=f"(a[0]), "=f"(a[1]), "=f"(a[2]), "=f"(a[3]), "=f"(a[4]), "=f"(a[5]), "=f"(a[6]), "=f"(a[7]),
          "=f"(a[8]), "=f"(a[9]), "=f"(a[10]), "=f"(a[11]), "=f"(a[12]), "=f"(a[13]), "=f"(a[14]), "=f"(a[15]),
          "=f"(b[0]), "=f"(b[1]), "=f"(b[2]), "=f"(b[3]), "=f"(b[4]), "=f"(b[5]), "=f"(b[6]), "=f"(b[7]),
          "=f"(b[8]), "=f"(b[9]), "=f"(b[10]), "=f"(b[11]), "=f"(b[12]), "=f"(b[13]), "=f"(b[14]), "=f"(b[15])
        : "r"(ta), "r"(tb)
        : "memory");
}
__device__ __forceinline__ void tmem_ld16x3(uint32_t ta, float (&a)[16], uint32_t tb, float (&b)[16], uint32_t tc_, float (&c)[16]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%48];\n\t"
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%49];\n\t"
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%32, %33, %34, %35, %36, %37, %38, %39, %40, %41, %42, %43, %44, %45, %46, %47}, [%50];\n\t"
        "tcgen05.wait::ld.sync.aligned;"
        : "=f"(a[0]), "=f"(a[1]), "=f"(a[2]), "=f"(a[3]), "=f"(a[4]), "=f"(a[5]), "=f"(a[6]), "=f"(a[7]), "=f"(a[8]), "=f"(a[9]), "=f"(a[10]), "=f"(a[11]), "=f"(a[12]), "=f"(a[13]), "=f"(a[14]), "=f"(a[15]),
          "=f"(b[0]), "=f"(b[1]), "=f"(b[2]), "=f"(b[3]), "=f"(b[4]), "=f"(b[5]), "=f"(b[6]), "=f"(b[7]), "=f"(b[8]), "=f"(b[9]), "=f"(b[10]), "=f"(b[11]), "=f"(b[12]), "=f"(b[13]), "=f"(b[14]), "=f"(b[15]),
          "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3]), "=f"(c[4]), "=f"(c[5]), "=f"(c[6]), "=f"(c[7]), "=f"(c[8]), "=f"(c[9]), "=f"(c[10]), "=f"(c[11]), "=f"(c[12]), "=f"(c[13]), "=f"(c[14]), "=f"(c[15])
        : "r"(ta), "r"(tb), "r"(tc_)
        : "memory");
}
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
// the large bf16 parts of two values, which keep the rest
__device__ __forceinline__ uint32_t part_of(F2 &v) {
    const float2 f = floats(v);
    const uint32_t p = pack2<__nv_bfloat16>(f.x, f.y);
    const float2 h = unpack2<__nv_bfloat16>(p);
    v = fma_2(f2(h.x, h.y), f2(-1.0f, -1.0f), v);
    return p;
}
__device__ __forceinline__ uint32_t rounded(F2 v) {
    const float2 f = floats(v);
    return pack2<__nv_bfloat16>(f.x, f.y);
}
// ------------------------------------------------------------------- scan
constexpr uint32_t TILE64 = Q * 128;  // 128 rows of 64 bf16 values
// C (two tiles) and x twice, X's and the state's first two parts once; B's two tiles, the
// third part of X' and a tile of zeros once.  The pass for states alone has B and X'
// twice, in the places of C and the state.
constexpr uint32_t OFF_B = 0, OFF_C = 4 * TILE64, OFF_X = 8 * TILE64, OFF_XW = 10 * TILE64, OFF_H = 12 * TILE64, OFF_SHARED = 14 * TILE64;
constexpr size_t SCAN_SMEM = OFF_SHARED + 2048;
static_assert(SCAN_SMEM <= 227 * 1024, "shared memory of a block");
// Barriers, one phase a chunk, or (two of a kind) a phase every other chunk.  F_*:
// copies landed; E_*: MMAs have read the tile; M_*: MMAs done; A_*: arrivals of the
// warps that have written or read what the name says.
enum Bar {
    F_B, F_C = F_B + 2, F_X = F_C + 2, E_B = F_X + 2, E_C = E_B + 2, E_X = E_C + 2,
    M_PAIRS = E_X + 2, M_CARRIED, M_INSIDE, M_MADE, A_XW = M_MADE + 2, A_MADE = A_XW + 2, A_STATE = A_MADE + 2, A_P, A_OUT, BARS
};
struct Work {  // what a block works on: a sequence (b < 0: none), its segment's chunks, the place of its states
    int first, len, slot, b, seg, segs, chunk0, chunks, part0;
};
struct Shared {
    alignas(16) float fs[2][Q];  // TAB_F of a chunk
    uint64_t bar[BARS];
    uint32_t tmem;
    int abort, any_bad[2];
    Work w;
    int bad[2][PB];              // first token of a chunk whose x is not finite, by channel
};
static_assert(sizeof(Shared) <= 2048, "behind the tiles");
// TMEM columns: pairs, and P's large parts in their place; carried and made with their
// large and small parts' products apart; inside; P's small parts
constexpr uint32_t T_S = 0, T_Y0 = 128, T_D = 256, T_Y1 = 384, T_LO = 448;

// Warps: 0 copies, 1 issues the MMAs; FULL: 2 to 9 make P and the next chunk's X' (two
// threads a row), 10 to 17 carry the state (half of the columns each four), 18 to 21
// take the outputs; otherwise 2 to 17 make X' (four threads a row), 18 to 25 carry the state.
constexpr int FULL_THREADS = 22 * 32, STATE_THREADS = 26 * 32;

// FULL: the outputs; otherwise a segment's state from nothing (segment 0: from s_in).
// The MMAs' order, chunk i: inside(i), pairs(i + 1), carried(i), made(i + 1).  The two
// that the next P waits for come first; X'(i + 1) is made meanwhile, and the state goes
// from made(i) to carried(i + 1) beside all of them.
template <bool FULL>
__global__ void __launch_bounds__(FULL ? FULL_THREADS : STATE_THREADS, 1)
    ssm_scan_tc_kernel(const __grid_constant__ CUtensorMap mX, const __grid_constant__ CUtensorMap mB,
                       const __grid_constant__ CUtensorMap mC, const __grid_constant__ TcP p, __nv_bfloat16 *__restrict__ y) {
    extern __shared__ __align__(1024) uint8_t smem[];
    Shared &sh = *reinterpret_cast<Shared *>(smem + OFF_SHARED);
    constexpr int XT = FULL ? 2 : 4, STATE0 = 2 + 4 * XT;  // threads a row of X'; the state's first warp
    constexpr int STAGES1 = FULL ? 1 : 2;  // of B, X' and the products with it
    constexpr uint32_t OFF_XW3 = FULL ? 2 * TILE64 : OFF_C;  // the third part of X', and zeros
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const int pb = blockIdx.x % p.pblocks, head = blockIdx.x / p.pblocks;  // (blockIdx.x: head * p.pblocks + pb)
    if (su32(smem) & 1023) {  // (the swizzled tiles need it; uniform over the block)
        if (threadIdx.x == 0) atomicOr(p.err, ERR_TMA_WAIT);
        return;
    }
    if (warp == 0) {
        tmem_alloc<1>(&sh.tmem, 512);
    } else if (warp == 1) {
        if (lane < BARS) mbar_init(&sh.bar[lane], lane < A_XW ? 1 : lane < A_MADE ? 4 * XT : lane == A_OUT ? 4 : 8);
        if (lane == 31) sh.abort = sh.any_bad[0] = sh.any_bad[1] = 0;
        fence_mbar_init();
    } else if (warp >= 2 && warp < 6) {
        (&sh.bad[0][0])[threadIdx.x - 64] = Q;
    }
    static_assert(BARS < 31, "one lane a barrier");
    for (uint32_t e = threadIdx.x; e < TILE64 / 16; e += blockDim.x)
#pragma unroll
        for (int i = 0; i < STAGES1; ++i)
            reinterpret_cast<uint4 *>(smem + OFF_XW3 + (2 * i + 1) * TILE64)[e] = make_uint4(0u, 0u, 0u, 0u);
    fence_proxy_async_smem();
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = __shfl_sync(0xffffffffu, sh.tmem, 0);
    griddep_launch();  // (behind the allocation: see tmem_alloc)
    griddep_wait();
    const SsmP &q = p.s;
    if (warp == 0) {  // what the block works on
        const Place place = place_of(q.q, p.segs == 1, [&](int len) { return FULL ? own_segments(len, p) : (own_segments(len, p) - 1) * p.fine; },
                                     1, (int)(blockIdx.y + blockIdx.z * gridDim.y));
        const Seq s = sequence(q.q, max(place.b, 0));
        const int segs = own_segments(s.len, p);
        const int2 chunks = place.b >= 0 ? segment(s.len, FULL ? segs : segs * p.fine, place.seg) : make_int2(0, 0);
        if (lane == 0)
            sh.w = Work{(int)s.first, s.len, s.slot, place.b, place.seg, segs, chunks.x, chunks.y - chunks.x, (int)(s.first / Q / p.step) * p.fine};
    }
    __syncthreads();
    // (by a reduction: in uniform registers, of which there are enough; as loaded, 165 us for 159)
    auto uniform = [](int v) { return __reduce_max_sync(0xffffffffu, v); };
    const bool used = uniform(sh.w.b) >= 0;
    Seq s;
    s.first = uniform(sh.w.first), s.len = uniform(sh.w.len), s.slot = uniform(sh.w.slot);
    const int b = max(uniform(sh.w.b), 0), seg = uniform(sh.w.seg), segs = uniform(sh.w.segs), part0 = uniform(sh.w.part0);
    const int chunk0 = uniform(sh.w.chunk0), nc = uniform(sh.w.chunks), grp = head / (q.H / q.G);
    const int p0 = pb * PB, np = min(PB, q.P - p0);
    const uint32_t base = su32(smem);
    const int row = (warp % 4) * 32 + lane;  // token t, or n of the state, by the warp's TMEM lanes
    const uint32_t lanes = (uint32_t)((warp % 4) * 32) << 16;
    const int64_t tab0 = chunk_at(s, b, chunk0) * q.H + head;
    auto table = [&](int c) { return p.table + (tab0 + (int64_t)c * q.H) * TABLE; };
    bool ok = true;
    auto gave_up = [&](int code) {
        atomicOr(p.err, code);
        *reinterpret_cast<volatile int *>(&sh.abort) = 1;
    };
    auto must = [&](int i, uint32_t par) {  // a whole warp's wait; after one that gave up, no further ones
        if (ok && !__all_sync(0xffffffffu, mbar_wait(&sh.bar[i], par))) {
            if (lane == 0) gave_up(ERR_EPI_WAIT);
            ok = false;
        }
        return ok;
    };
    auto arrive = [&](int i) {
        __syncwarp();
        if (lane == 0) mbar_arrive(&sh.bar[i]);
    };

    if (warp == 0) {
        if (lane == 0) {  // ---------------- copies
            auto load = [&](const CUtensorMap *m, int bar, uint32_t off, int c, int boxes, int x0, int g) {
                mbar_expect_tx(&sh.bar[bar], boxes * TILE64);
                for (int i = 0; i < boxes; ++i)
                    tma_3d<1>(base + off + i * TILE64, m, su32(&sh.bar[bar]), x0 + 64 * i, g, (int)(s.first + (int64_t)(chunk0 + c) * Q));
            };
            auto freed = [&](int i, int n) {  // the n-th chunk in a stage waits until the one before has been read
                if (ok && n > 0 && !mbar_wait(&sh.bar[i], (uint32_t)(n - 1) & 1u)) {
                    gave_up(ERR_TMA_WAIT);
                    ok = false;
                }
                return ok;
            };
            for (int c = 0; c < nc && ok; ++c) {
                const int st = c & 1, bs = c % STAGES1;
                if (FULL) {
                    if (!freed(E_C + st, c >> 1)) break;
                    load(&mC, F_C + st, OFF_C + st * 2 * TILE64, c, 2, 0, grp);
                }
                if (!freed(E_X + st, c >> 1)) break;
                load(&mX, F_X + st, OFF_X + st * TILE64, c, 1, p0, head);
                if (!freed(E_B + bs, c / STAGES1)) break;
                load(&mB, F_B + bs, OFF_B + bs * 2 * TILE64, c, 2, 0, grp);
            }
        }
        __syncwarp();
    } else if (warp == 1) {
        {  // ---------------- MMAs: the whole warp, so that descriptors stay in uniform registers; one lane issues
            const uint32_t one = elect_one();
            constexpr uint32_t FMT = (1u << 4) | (1u << 7) | (1u << 10) | ((128u >> 4) << 24);  // fp32 sums of bf16, M = 128
            constexpr uint32_t N128 = (128u >> 3) << 17, N64 = ((uint32_t)PB >> 3) << 17;
            const int nblk = q.N > 64 ? 2 : 1;  // blocks of 64 of the state's axis (zeros behind N)
            auto need = [&](int i, uint32_t par) {
                if (ok && !__all_sync(0xffffffffu, mbar_wait(&sh.bar[i], par))) {
                    if (lane == 0) gave_up(ERR_MMA_WAIT);
                    ok = false;
                }
                return ok;
            };
            // operands' descriptors at step 0; a step of 16 adds 32 bytes of a tile's 64 columns
            // (K-major) or 16 rows (MN-major).  The steps are unrolled: one thread issues all MMAs,
            // and forming a descriptor for each took it 150 cycles, an MMA takes the tensor core 64.
            const uint64_t b_k = sdesc_sw128(base + OFF_B), c_k = sdesc_sw128(base + OFF_C);
            const uint64_t b_mn = sdesc_mn(base + OFF_B, TILE64), x_mn = sdesc_mn(base + OFF_X, TILE64);
            const uint64_t xw_mn = sdesc_mn(base + OFF_XW, TILE64), xw3_mn = sdesc_mn(base + OFF_XW3, TILE64), h_mn = sdesc_mn(base + OFF_H, TILE64);
            constexpr uint64_t STAGE2 = 2 * TILE64 >> 4, STAGE1 = TILE64 >> 4;
            auto mn_major = [](int k) { return (uint64_t)(k * (2048 >> 4)); };
            auto pairs = [&](int c) {
                const uint32_t st = c & 1, half = (uint32_t)(c >> 1) & 1u;
                // (they take the place of the chunk before's P: only MMAs on one accumulator keep their order by themselves)
                if (!need(F_B, c & 1) || !need(F_C + st, half) || (c > 0 && !need(M_INSIDE, (c - 1) & 1))) return;
                tc_fence_after();
                const uint64_t dc = c_k + st * STAGE2;
#pragma unroll 1
                for (int blk = 0; blk < nblk; ++blk) {
                    const uint64_t o = blk * STAGE1;
#pragma unroll
                    for (int k = 0; k < 4; ++k) umma_one<1>(one, tmem + T_S, dc + o + 2 * k, b_k + o + 2 * k, FMT | N128, blk > 0 || k > 0);
                }
                commit_one<1>(one, &sh.bar[M_PAIRS]);
            };
            auto inside = [&](int c) {
                const uint32_t st = c & 1, par = c & 1;
                if (!need(A_P, par) || (c > 0 && !need(A_OUT, par ^ 1u))) return;
                tc_fence_after();
                const uint64_t dx = x_mn + st * STAGE1;
#pragma unroll
                for (int part = 0; part < 2; ++part)
#pragma unroll
                    for (int k = 0; k < Q / 16; ++k)
                        umma_ts_one(one, tmem + T_Y1, tmem + (part ? T_LO + k * 8 : T_S + k * 16), dx + mn_major(k),
                                    FMT | N64 | B_MN, part > 0 || k > 0);
                commit_one<1>(one, &sh.bar[M_INSIDE]);
                commit_one<1>(one, &sh.bar[E_X + st]);
            };
            auto carried = [&](int c) {
                const uint32_t st = c & 1;
                if (!need(A_STATE, c & 1)) return;
                tc_fence_after();
                const uint64_t dc = c_k + st * STAGE2;
#pragma unroll 1
                for (int blk = 0; blk < nblk; ++blk)
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        umma_one<1>(one, tmem + T_Y0, dc + blk * STAGE1 + 2 * k, h_mn + mn_major(4 * blk + k), FMT | N128 | B_MN, blk > 0 || k > 0);
                commit_one<1>(one, &sh.bar[M_CARRIED]);
                commit_one<1>(one, &sh.bar[E_C + st]);
            };
            auto made = [&](int c) {
                const uint32_t bs = c % STAGES1;
                const uint32_t n = c / STAGES1;
                if (!need(F_B + bs, n & 1u) || !need(A_XW + bs, n & 1u) || (n > 0 && !need(A_MADE + bs, (n - 1) & 1u))) return;
                tc_fence_after();
                const uint64_t db = b_mn + bs * STAGE2, xw = xw_mn + bs * STAGE2, xw3 = xw3_mn + bs * STAGE2;
                const uint32_t d = tmem + T_D + bs * 128;
                // (N = 128: the products with two parts of X' side by side.  The third part, beside
                // zeros, comes first, while the sums are small: they are truncated at every MMA)
#pragma unroll
                for (int k = 0; k < Q / 16; ++k)
                    umma_one<1>(one, d, db + mn_major(k), xw3 + mn_major(k), FMT | N128 | A_MN | B_MN, k > 0);
#pragma unroll
                for (int k = 0; k < Q / 16; ++k)
                    umma_one<1>(one, d, db + mn_major(k), xw + mn_major(k), FMT | N128 | A_MN | B_MN, 1);
                commit_one<1>(one, &sh.bar[M_MADE + bs]);
                commit_one<1>(one, &sh.bar[E_B + bs]);
                if (!FULL) commit_one<1>(one, &sh.bar[E_X + (c & 1)]);
            };
#pragma unroll 1
            for (int c = -1; c < nc && ok; ++c) {
                if (FULL && c >= 0) inside(c);
                if (FULL && c + 1 < nc && ok) pairs(c + 1);
                if (FULL && c >= 0 && ok) carried(c);
                if (c + 1 < nc && ok) made(c + 1);
            }
        }
        __syncwarp();
    } else if (warp < STATE0) {
        // ---------------- X', XT threads a row
        const int tid = threadIdx.x - 64, t = tid / XT, j0 = 8 / XT * (tid % XT);
        float w_next = nc > 0 ? __ldg(table(0) + TAB_W + t) : 0.0f;
        auto weigh = [&](int c) {
            const int st = c & 1, bs = c % STAGES1, valid = min(Q, s.len - (chunk0 + c) * Q);  // tokens there are
            const float w = w_next;
            if (c + 1 < nc) w_next = __ldg(table(c + 1) + TAB_W + t);
            must(F_X + st, (uint32_t)(c >> 1) & 1u);
            const uint32_t n = c / STAGES1;
            if (n > 0) must(M_MADE + bs, (n - 1) & 1u);  // the X' before has been read
            if (valid < Q) {
                must(F_B + bs, n & 1u);
                if (FULL) must(M_PAIRS, c & 1);
            }
            if (!ok) return;
            uint8_t *xr = smem + OFF_X + st * TILE64 + t * 128, *wr = smem + OFF_XW + bs * 2 * TILE64 + t * 128;
            uint8_t *w3 = smem + OFF_XW3 + bs * 2 * TILE64 + t * 128;
#pragma unroll 1  // (two at a time: 4 us more for 8192 tokens)
            for (int i = 0; i < 8 / XT; ++i) {
                const uint32_t at = (uint32_t)((j0 + i) ^ (t & 7)) << 4;
                uint4 xv = *reinterpret_cast<const uint4 *>(xr + at);
                if (t >= valid) {  // rows of another sequence: nothing of them may count
                    xv = make_uint4(0u, 0u, 0u, 0u);
                    *reinterpret_cast<uint4 *>(xr + at) = xv;
                    uint8_t *br = smem + OFF_B + bs * 2 * TILE64 + t * 128 + at;
                    *reinterpret_cast<uint4 *>(br) = xv;
                    *reinterpret_cast<uint4 *>(br + TILE64) = xv;
                }
                const uint32_t u[4] = {xv.x, xv.y, xv.z, xv.w};
                uint32_t hi[4], lo[4], lo2[4], odd = 0u;  // odd: a value's exponent is all ones
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float2 f = unpack2<__nv_bfloat16>(u[e]);
                    odd |= ((u[e] & 0x7f807f80u) + 0x00800080u) & 0x80008000u;
                    F2 v = mul_2(f2(f.x, f.y), f2(w, w));
                    hi[e] = part_of(v), lo[e] = part_of(v), lo2[e] = rounded(v);
                }
                *reinterpret_cast<uint4 *>(wr + at) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
                *reinterpret_cast<uint4 *>(wr + TILE64 + at) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
                *reinterpret_cast<uint4 *>(w3 + at) = make_uint4(lo2[0], lo2[1], lo2[2], lo2[3]);
                if (odd) {
#pragma unroll 1
                    for (int e = 0; e < 8; ++e) {
                        uint16_t *xe = reinterpret_cast<uint16_t *>(xr + at) + e;
                        if ((*xe & 0x7f80u) != 0x7f80u) continue;
                        reinterpret_cast<uint16_t *>(wr + TILE64 + at)[e] = reinterpret_cast<uint16_t *>(w3 + at)[e] = 0;  // into the state as it is
                        if (FULL) {  // out of the product inside the chunk; its channel is NaN from here on
                            *xe = 0;
                            atomicMin(&sh.bad[st][8 * (j0 + i) + e], t);
                            sh.any_bad[st] = 1;
                        }
                    }
                }
            }
            fence_proxy_async_smem();
            arrive(A_XW + bs);
        };
        if constexpr (!FULL) {
            for (int c = 0; c < nc && ok; ++c) weigh(c);
        } else {
            // ---------------- P from the pairs: 32 x 32 blocks, this warp's two of its rows' four; D,
            // the factor of x itself, joins the diagonal.  After it the next chunk's X'
            const int quarter = warp % 4, half = (warp - 2) / 4;
            const float skip = q.d ? q.d[head] : 0.0f;
            // of the next chunk: this row's TAB_R and TAB_D; TAB_F of token tid (tid < 128)
            float r_next = 0.0f, d_next = 0.0f, f_next = 0.0f;
            auto fetch = [&](int c) {
                if (c >= nc) return;
                const float *tab = table(c);
                r_next = __ldg(tab + TAB_R + row), d_next = __ldg(tab + TAB_D + row);
                if (tid < Q) f_next = __ldg(tab + TAB_F + tid);
            };
            fetch(0);
#pragma unroll 1
            for (int c = -1; c < nc; ++c) {
                if (c >= 0) {
                    const uint32_t par = c & 1;
                    const float dt = d_next;
                    // R_t and what lies between, for the four times 16 columns at hand
                    float4 base = __ldg(reinterpret_cast<const float4 *>(table(c) + TAB_S) + row / 16 * 2 + half);
                    base.x += r_next, base.y += r_next, base.z += r_next, base.w += r_next;
                    if (tid < Q) sh.fs[par][tid] = f_next;  // (its last readers, two chunks ago, have passed the barrier since)
                    fetch(c + 1);
                    if (bar_red_or(1, 256, !ok)) break;  // (the group leaves together)
                    if (!must(M_PAIRS, par)) continue;
                    tc_fence_after();
                    // 16 columns at a time in a rolled loop (all 64 unrolled, as every role's loop was,
                    // the warps waited for instructions: some 14 cycles for each)
#pragma unroll 1
                    for (int i = 0; i < 4; ++i) {
                        const int blk = 2 * (i / 2) + half, c0 = 32 * blk + 16 * (i % 2);
                        uint32_t hi[8], lo[8];
                        __syncwarp();
                        if (blk <= quarter) {
                            float f[16];
                            F2 v[8];
                            tmem_ld16(tmem + lanes + T_S + c0, f);
                            const float from = i == 0 ? base.x : i == 1 ? base.y : i == 2 ? base.z : base.w;
#pragma unroll
                            for (int j = 0; j < 4; ++j) {
                                const float4 t = *reinterpret_cast<const float4 *>(&sh.fs[par][c0 + 4 * j]);
                                const float2 a = floats(add_2(f2(t.x, t.y), f2(from, from)));
                                const float2 b = floats(add_2(f2(t.z, t.w), f2(from, from)));
                                v[2 * j] = mul_2(f2(f[4 * j], f[4 * j + 1]), f2(ex2(a.x), ex2(a.y)));
                                v[2 * j + 1] = mul_2(f2(f[4 * j + 2], f[4 * j + 3]), f2(ex2(b.x), ex2(b.y)));
                            }
                            if (blk == quarter) {
                                const int own = row - c0;  // the diagonal's place among these columns: its weight is d
#pragma unroll
                                for (int j = 0; j < 8; ++j) {
                                    const float2 m = floats(v[j]);
                                    v[j] = f2(2 * j < own ? m.x : 2 * j == own ? fmaf(f[2 * j], dt, skip) : 0.0f,
                                              2 * j + 1 < own ? m.y : 2 * j + 1 == own ? fmaf(f[2 * j + 1], dt, skip) : 0.0f);
                                }
                            }
#pragma unroll
                            for (int j = 0; j < 8; ++j) {
                                hi[j] = part_of(v[j]);
                                lo[j] = rounded(v[j]);
                            }
                        } else {
#pragma unroll
                            for (int j = 0; j < 8; ++j) hi[j] = lo[j] = 0u;
                        }
                        __syncwarp();
                        tmem_st8(tmem + lanes + T_S + c0, hi);  // (these columns' pairs have been read)
                        tmem_st8(tmem + lanes + T_LO + c0 / 2, lo);
                    }
                    tmem_wait_st();
                    tc_fence_before();
                    if (c > 0) must(A_OUT, par ^ 1u);  // (what the next X' says of values that are not finite takes the place of what the outputs have read)
                    arrive(A_P);
                }
                if (c + 1 < nc && ok) weigh(c + 1);
            }
        }
    } else if (warp < STATE0 + 8) {
        // ---------------- the state, [p][n] with lane n, in fp32: columns c0 to c0 + 31
        constexpr int HC = PB / 2;
        F2 h[HC / 2];
        const int c0 = (warp - STATE0) / 4 * HC;
        const int64_t srow = s.slot >= 0 ? (((int64_t)s.slot * q.H + head) * q.P + p0 + c0) * q.N + row : -1;
        auto live = [&](int i) { return c0 + i < np && row < q.N; };
        auto part = [&](int j) { return p.part + (((int64_t)(part0 + j) * q.H * p.pblocks + blockIdx.x) * PB + c0) * q.N + row; };  // before segment 0, after fine segment j - 1
        auto load = [&](const float *from) {
#pragma unroll
            for (int i = 0; i < HC; i += 2)
                h[i / 2] = f2(live(i) ? from[(int64_t)i * q.N] : 0.0f, live(i + 1) ? from[(int64_t)(i + 1) * q.N] : 0.0f);
        };
        auto store = [&](float *to) {
#pragma unroll
            for (int i = 0; i < HC; i += 2) {
                const float2 v = floats(h[i / 2]);
                if (live(i)) to[(int64_t)i * q.N] = v.x;
                if (live(i + 1)) to[(int64_t)(i + 1) * q.N] = v.y;
            }
        };
#pragma unroll
        for (int i = 0; i < HC / 2; ++i) h[i] = f2(0.0f, 0.0f);
        if (used && FULL && segs > 1) load(part(seg > 0 ? 1 : 0));
        else if (used && seg == 0 && q.s_in && srow >= 0) load(q.s_in + srow);
        if (!used) {
        } else if (FULL) {
            for (int j = 1; j < seg * p.fine; ++j) {
                const int2 ch = segment(s.len, segs * p.fine, j);
                float sum = 0.0f;
                for (int c = ch.x; c < ch.y; ++c) sum += p.total[chunk_at(s, b, c) * q.H + head];
                const float e = exp2f(sum), *next = part(j + 1);
#pragma unroll
                for (int i = 0; i < HC; i += 2)
                    h[i / 2] = fma_2(h[i / 2], f2(e, e), f2(live(i) ? next[(int64_t)i * q.N] : 0.0f, live(i + 1) ? next[(int64_t)(i + 1) * q.N] : 0.0f));
            }
        } else if (seg == 0) {  // the second pass may store over s_in: it reads this copy
            store(part(0));
        }
        auto put_state = [&]() {  // its two bf16 parts as an operand: rows n, 64 p
            uint8_t *hr = smem + OFF_H + row * 128;
#pragma unroll
            for (int i = 0; i < HC / 8; ++i) {
                uint32_t hi[4], lo[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    // (an infinite state's small part is NaN, as its sums over B's signs are)
                    F2 v = h[4 * i + e];
                    hi[e] = part_of(v), lo[e] = rounded(v);
                }
                const uint32_t at = (uint32_t)((c0 / 8 + i) ^ (row & 7)) << 4;
                *reinterpret_cast<uint4 *>(hr + at) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
                *reinterpret_cast<uint4 *>(hr + TILE64 + at) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
            }
            fence_proxy_async_smem();
            arrive(A_STATE);
        };
        float total_next = nc > 0 ? __ldg(p.total + tab0) : 0.0f;
#pragma unroll 1
        for (int c = 0; c < nc; ++c) {
            if (FULL) {
                if (c > 0 && !must(M_CARRIED, (c - 1) & 1)) break;  // the operand before has been read
                put_state();
            }
            const float e = exp2f(total_next);
            if (c + 1 < nc) total_next = __ldg(p.total + tab0 + (int64_t)(c + 1) * q.H);
            const uint32_t bs = c % STAGES1, d = tmem + lanes + T_D + bs * 128 + c0;
            if (!must(M_MADE + bs, (uint32_t)(c / STAGES1) & 1u)) break;
            tc_fence_after();
#pragma unroll
            for (int i = 0; i < HC; i += 16) {
                float u[16], v[16];
                __syncwarp();
                tmem_ld16x2(d + i, u, d + PB + i, v);
#pragma unroll
                for (int j = 0; j < 16; j += 2)
                    h[(i + j) / 2] = fma_2(h[(i + j) / 2], f2(e, e), add_2(f2(u[j], u[j + 1]), f2(v[j], v[j + 1])));
            }
            tc_fence_before();
            arrive(A_MADE + bs);
        }
        float *out = !used ? nullptr : !FULL ? part(seg + 1) : seg == segs - 1 && q.s_out && srow >= 0 ? q.s_out + srow : nullptr;
        if (ok && out) store(out);
    } else {
        // ---------------- the outputs
        const int t = threadIdx.x - (STATE0 + 8) * 32;
        float at_next = nc > 0 ? __ldg(table(0) + row) : 0.0f;
#pragma unroll 1
        for (int c = 0; c < nc; ++c) {
            const float et = ex2(at_next);
            if (c + 1 < nc) at_next = __ldg(table(c + 1) + row);
            const int st = c & 1, valid = min(Q, s.len - (chunk0 + c) * Q);
            must(M_INSIDE, c & 1);
            must(M_CARRIED, c & 1);
            if (bar_red_or(2, 128, !ok)) break;  // (the group leaves together)
            tc_fence_after();
            const bool bad = *reinterpret_cast<volatile int *>(&sh.any_bad[st]);
            __nv_bfloat16 *yr = y + (s.first + (int64_t)(chunk0 + c) * Q + row) * q.ldy + (int64_t)head * q.P + p0;
#pragma unroll 1
            for (int i = 0; i < PB; i += 16) {
                float u[16], v[16], in[16];
                __syncwarp();
                tmem_ld16x3(tmem + lanes + T_Y0 + i, u, tmem + lanes + T_Y0 + PB + i, v, tmem + lanes + T_Y1 + i, in);
#pragma unroll
                for (int j = 0; j < 16; j += 8) {
                    uint32_t o[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int n = j + 2 * e;
                        F2 f = fma_2(add_2(f2(u[n], u[n + 1]), f2(v[n], v[n + 1])), f2(et, et), f2(in[n], in[n + 1]));
                        if (bad) {
                            const float2 g = floats(f);
                            f = f2(row >= sh.bad[st][i + n] ? NAN : g.x, row >= sh.bad[st][i + n + 1] ? NAN : g.y);
                        }
                        o[e] = rounded(f);
                    }
                    if (row < valid && i + j < np) *reinterpret_cast<uint4 *>(yr + i + j) = make_uint4(o[0], o[1], o[2], o[3]);
                }
            }
            if (bad) {  // (the same in the group's every warp)
                asm volatile("bar.sync 3, 128;" ::: "memory");
                if (t < PB) sh.bad[st][t] = Q;
                if (t == 0) sh.any_bad[st] = 0;
                asm volatile("bar.sync 3, 128;" ::: "memory");
            }
            tc_fence_before();
            arrive(A_OUT);
        }
    }
    tc_fence_before();
    __syncthreads();
    if (threadIdx.x == 0 && sh.abort) {  // copies in flight land before the block's memory goes away (bounded)
        const long long t0 = clock64();
        while (clock64() - t0 < WAIT_LIMIT / 1000) {
        }
    }
    __syncthreads();
    if (warp == 0) {
        tc_fence_after();
        tmem_dealloc<1>(tmem, 512);
    }
}

// Segments that a sequence is cut into: as many as fill the SMs, of four chunks at
// least; and the first pass's, which leaves the last segment out
struct Cut {
    int segs, step, fine;
};
Cut cut_of(const SsmP &p) {
    const int64_t full = (p.q.tokens + p.q.max_len - 1) / std::max<int64_t>(p.q.max_len, 1);  // sequences, counted by length
    const int64_t blocks = std::max<int64_t>(full * p.H * ((p.P + PB - 1) / PB), 1), chunks = (p.q.max_len + Q - 1) / Q;
    Cut c;
    c.segs = (int)std::max<int64_t>(1, std::min<int64_t>({num_sms() / blocks, 64, chunks / 4}));
    c.step = (int)std::max<int64_t>(4, p.q.max_len / Q / c.segs);
    c.fine = c.segs == 1 ? 1 : (int)std::max<int64_t>(1, std::min<int64_t>(num_sms() / (blocks * (c.segs - 1)), chunks / c.segs / 2));
    return c;
}
struct TcWork {
    int64_t chunks, table, total, part, bytes;  // offsets
};
TcWork work_of(const SsmP &p) {
    TcWork w;
    auto up = [](int64_t v) { return (v + 255) / 256 * 256; };
    w.chunks = p.q.tokens / Q + p.q.batch + 1;
    w.table = 0;
    w.total = w.table + up(w.chunks * p.H * TABLE * 4);
    w.part = w.total + up(w.chunks * p.H * 4);
    const Cut c = cut_of(p);
    w.bytes = w.part + (c.segs > 1 ? up(p.q.tokens / Q / c.step * c.fine * p.H * ((p.P + PB - 1) / PB) * PB * p.N * 4) : 0);
    return w;
}

}  // namespace

// bf16 tokens whose rows TMA can read: 16-byte aligned, whole 16-byte pieces of every head and group
bool ssm_tc_applies(const SsmP &p, const void *xbc, const void *y) {
    return p.N <= 128 && p.N % 8 == 0 && p.P % 8 == 0 && p.ldx % 8 == 0 && p.ldy % 8 == 0 && reinterpret_cast<uintptr_t>(xbc) % 16 == 0 &&
           reinterpret_cast<uintptr_t>(y) % 16 == 0 && p.q.max_len >= 16;
}

size_t ssm_tc_workspace(const SsmP &p) { return (size_t)work_of(p).bytes; }

cudaError_t ssm_tc_scan(const SsmP &s, const __nv_bfloat16 *xbc, const __nv_bfloat16 *dtv, __nv_bfloat16 *y, void *work,
                        cudaStream_t st) {
    const TcWork w = work_of(s);
    char *base = static_cast<char *>(work);
    const Cut cut = cut_of(s);
    TcP p{s, cut.segs, cut.step, cut.fine, reinterpret_cast<float *>(base + w.table), reinterpret_cast<float *>(base + w.total),
          reinterpret_cast<float *>(base + w.part), (s.P + PB - 1) / PB, device_error_word()};
    // xbc's rows as [heads][P] of x and [groups][N] of B and C: what lies behind a head's or group's end reads as 0
    CUtensorMap mX, mB, mC;
    const uint64_t str_x[2] = {(uint64_t)s.P * 2, (uint64_t)s.ldx * 2}, str_b[2] = {(uint64_t)s.N * 2, (uint64_t)s.ldx * 2};
    const uint64_t dim_x[3] = {(uint64_t)s.P, (uint64_t)s.H, (uint64_t)s.q.tokens}, dim_b[3] = {(uint64_t)s.N, (uint64_t)s.G, (uint64_t)s.q.tokens};
    const uint32_t box[3] = {64, 1, Q};
    const __nv_bfloat16 *xb = xbc + (int64_t)s.H * s.P, *xc = xb + (int64_t)s.G * s.N;
    if (!tma_encode(&mX, SN_BF16, 3, xbc, dim_x, str_x, box, CU_TENSOR_MAP_SWIZZLE_128B) ||
        !tma_encode(&mB, SN_BF16, 3, xb, dim_b, str_b, box, CU_TENSOR_MAP_SWIZZLE_128B) ||
        !tma_encode(&mC, SN_BF16, 3, xc, dim_b, str_b, box, CU_TENSOR_MAP_SWIZZLE_128B))
        return cudaErrorInvalidValue;
    static PerDevice set_full, set_states;
    if (const cudaError_t e = allow_smem(set_full, ssm_scan_tc_kernel<true>, SCAN_SMEM)) return e;
    if (const cudaError_t e = allow_smem(set_states, ssm_scan_tc_kernel<false>, SCAN_SMEM)) return e;
    const unsigned chunks = (unsigned)((s.q.max_len + Q - 1) / Q);
    const int vec = s.H % 8 == 0 && s.lddt % 8 == 0 && reinterpret_cast<uintptr_t>(dtv) % 16 == 0;
    cudaError_t e = launch_pdl(ssm_steps_kernel, dim3(chunks, (unsigned)((s.H + 7) / 8), (unsigned)s.q.batch), dim3(256), 0, st, p, dtv, vec);
    if (e != cudaSuccess) return e;
    // segments that there can be: one of each sequence, and one more for each step
    const int64_t heads = (int64_t)s.H * p.pblocks, steps = s.q.tokens / Q / p.step, batch = s.q.batch;
    const int64_t most = std::min(batch * p.segs, batch + steps), states = std::min(batch * (p.segs - 1), steps) * p.fine;
    if (std::max(most, states) > INT32_MAX) return cudaErrorInvalidValue;
    auto grid = [&](int64_t n) {  // head and channels, segment's number
        const int64_t z = (n + 65534) / 65535;
        return dim3((unsigned)heads, (unsigned)((n + z - 1) / z), (unsigned)z);
    };
    if (states > 0) {
        e = launch_pdl(ssm_scan_tc_kernel<false>, grid(states), dim3(STATE_THREADS), SCAN_SMEM, st, mX, mB, mC, p, y);
        if (e != cudaSuccess) return e;
    }
    return launch_pdl(ssm_scan_tc_kernel<true>, grid(most), dim3(FULL_THREADS), SCAN_SMEM, st, mX, mB, mC, p, y);
}

}  // namespace k
}  // namespace sn
