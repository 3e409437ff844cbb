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
//   made    B^T X'      N x P,     K = 128     X' = weighted X in two parts
// x, B and C are bf16, exact operands; what is computed goes in as two bf16 parts
// (2^-18 of it is lost, as much as a few fp32 roundings).  The state stays in
// registers in fp32: each chunk's product is added by an fp32 multiply-add, since the
// tensor core's own sums do not round to nearest.
//
// Work: a block takes one head, 64 of its channels and a segment of a sequence's
// chunks, two blocks an SM.  With few heads the sequence is cut into segments: a first
// pass makes each segment's state from nothing (the last product alone), and the
// second starts each segment from the joined ones.  A small kernel before both turns
// time steps into sums of a and weights, once per token and head.
//
// Eight warps: warp w has TMEM lanes 32 (w % 4) + 0..31 (tokens t, or the state's n)
// and half w / 4 of the columns; one lane of warps 0 to 4 each also issues one of the
// products, or the copies, behind a barrier of the block (a ninth warp for that would
// take a quarter of the registers).
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
constexpr int SCAN_THREADS = 256;
constexpr float LOG2E = 1.4426950408889634f;

// per chunk and head: A_t (inclusive, in units of log 2), A_s - log2 d_s, weights d_s e^{A_127 - A_s}
constexpr int TABLE = 3 * Q;

struct TcP {
    SsmP s;
    int32_t segs;            // segments a sequence
    float *table, *total;    // [chunks][H][TABLE], [chunks][H]: A_127
    float *part;             // [batch][H][p blocks][segs][64][N]: state before segment 0, then after segment j
    int32_t pblocks;
    int *err;
};

// index of a chunk's table: unique for chunk c of sequence b, since each sequence
// before it has at most its tokens / Q + 1 chunks
__device__ __forceinline__ int64_t chunk_at(const Seq &s, int b, int c) { return s.first / Q + b + c; }
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
        float4 A, B, W;
        A.x = before + v[0], A.y = A.x + v[1], A.z = A.y + v[2], A.w = A.z + v[3];
        B = make_float4(A.x - log2f(d[0]), A.y - log2f(d[1]), A.z - log2f(d[2]), A.w - log2f(d[3]));
        float r = behind;
        W.w = d[3] * exp2f(r), r += v[3];
        W.z = d[2] * exp2f(r), r += v[2];
        W.y = d[1] * exp2f(r), r += v[1];
        W.x = d[0] * exp2f(r);
        const int64_t at = chunk_at(s, b, c) * p.s.H + head;
        float4 *out = reinterpret_cast<float4 *>(p.table + at * TABLE);
        out[lane] = A;
        out[Q / 4 + lane] = B;
        out[Q / 2 + lane] = W;
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
// A from TMEM: a lane's row, two bf16 values a column
__device__ __forceinline__ void umma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t acc) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d),
        "r"(a), "l"(b), "r"(idesc), "r"(acc)
        : "memory");
}
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t (&v)[16]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};" ::"r"(
            taddr),
        "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]), "r"(v[9]), "r"(v[10]),
        "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15])
        : "memory");
}
// 16 columns at each of two addresses (the wait in the same statement: nothing of them is used before it)
__device__ __forceinline__ void tmem_ld16x2(uint32_t ta, uint32_t (&a)[16], uint32_t tb, uint32_t (&b)[16]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%32];\n\t"
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%33];\n\t"
        "tcgen05.wait::ld.sync.aligned;"
        : "=r"(a[0]), "=r"(a[1]), "=r"(a[2]), "=r"(a[3]), "=r"(a[4]), "=r"(a[5]), "=r"(a[6]), "=r"(a[7]),
          "=r"(a[8]), "=r"(a[9]), "=r"(a[10]), "=r"(a[11]), "=r"(a[12]), "=r"(a[13]), "=r"(a[14]), "=r"(a[15]),
          "=r"(b[0]), "=r"(b[1]), "=r"(b[2]), "=r"(b[3]), "=r"(b[4]), "=r"(b[5]), "=r"(b[6]), "=r"(b[7]),
          "=r"(b[8]), "=r"(b[9]), "=r"(b[10]), "=r"(b[11]), "=r"(b[12]), "=r"(b[13]), "=r"(b[14]), "=r"(b[15])
        : "r"(ta), "r"(tb)
        : "memory");
}
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ float ex2(float v) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
    return r;
}
// two values as the large and small bf16 parts of each
struct Parts2 {
    uint32_t hi, lo;
};
__device__ __forceinline__ Parts2 parts2(float a, float b) {
    Parts2 r;
    r.hi = pack2<__nv_bfloat16>(a, b);
    const float2 h = unpack2<__nv_bfloat16>(r.hi);
    r.lo = pack2<__nv_bfloat16>(a - h.x, b - h.y);
    return r;
}
// ------------------------------------------------------------------- scan
constexpr uint32_t TILE64 = Q * 128;  // 128 rows of 64 bf16 values
constexpr uint32_t OFF_B = 0, OFF_C = 2 * TILE64, OFF_X = 4 * TILE64, OFF_H = 5 * TILE64, OFF_BARS = 7 * TILE64;
constexpr size_t SCAN_SMEM = OFF_BARS + 1024;  // twice this and 1 KB each is all that an SM has
// barriers (F_*: copies landed, M_*: MMAs done), one phase a chunk (F_B, F_B1: every other one without outputs)
enum Bar { F_B, F_B1, F_C, F_X, M_PAIRS, M_CARRIED, M_MADE, M_INSIDE, BARS };
struct Shared {
    uint64_t bar[BARS];
    uint32_t tmem;
    int abort, any_bad;
    int bad[PB];  // first token of the chunk whose x is not finite, by channel
    alignas(16) float as[Q];  // the chunk's A_s - log2 d_s
};
static_assert(sizeof(Shared) <= 1024, "behind the tiles");

// FULL: the outputs; otherwise a segment's state from nothing (segment 0: from s_in).
// A wait that gives up leaves the warp's later ones and all further issues out; the
// barriers of the block are passed by every warp in any case.
template <bool FULL>
__global__ void __launch_bounds__(SCAN_THREADS, 2)
    ssm_scan_tc_kernel(const __grid_constant__ CUtensorMap mX, const __grid_constant__ CUtensorMap mB,
                       const __grid_constant__ CUtensorMap mC, const __grid_constant__ TcP p, __nv_bfloat16 *__restrict__ y) {
    extern __shared__ __align__(1024) uint8_t smem[];
    Shared &sh = *reinterpret_cast<Shared *>(smem + OFF_BARS);
    constexpr uint32_t COLS = FULL ? 256 : 64;
    constexpr uint32_t T_S = 0, T_Y0 = 128, T_D = FULL ? 192 : 0;  // pairs and P; carried; made and inside
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const int pb = blockIdx.x % p.pblocks, head = blockIdx.x / p.pblocks, seg = blockIdx.y, b = blockIdx.z;
    if (su32(smem) & 1023) {  // (the swizzled tiles need it; uniform over the block)
        if (threadIdx.x == 0) atomicOr(p.err, ERR_TMA_WAIT);
        return;
    }
    if (warp == 0) {
        tmem_alloc<1>(&sh.tmem, COLS);
    } else if (warp == 1 && lane == 0) {
        for (int i = 0; i < BARS; ++i) mbar_init(&sh.bar[i], 1);
        sh.abort = sh.any_bad = 0;
        fence_mbar_init();
    } else if (warp >= 6) {
        sh.bad[threadIdx.x - 192] = Q;
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = sh.tmem;
    griddep_launch();  // (behind the allocation: see tmem_alloc)
    griddep_wait();
    const SsmP &q = p.s;
    const Seq s = sequence(q.q, b);
    const int2 chunks = segment(s.len, p.segs, seg);
    const int nc = chunks.y - chunks.x, grp = head / (q.H / q.G);
    const int p0 = pb * PB, np = min(PB, q.P - p0);
    const int64_t part0 = (((int64_t)b * q.H + head) * p.pblocks + pb) * p.segs * PB * q.N;
    const uint32_t base = su32(smem);
    const int quarter = warp % 4, half = warp / 4, row = quarter * 32 + lane;  // token, or n of the state
    const uint32_t lanes = (uint32_t)(quarter * 32) << 16;
    bool ok = true;
    auto must = [&](int i, uint32_t par) {  // the whole warp
        if (ok && !__all_sync(0xffffffffu, mbar_wait(&sh.bar[i], par))) {
            if (lane == 0) {
                atomicOr(p.err, ERR_EPI_WAIT);
                *reinterpret_cast<volatile int *>(&sh.abort) = 1;
            }
            ok = false;
        }
    };
    auto may = [&]() { return ok && !*reinterpret_cast<volatile int *>(&sh.abort); };
    // ---- what single lanes issue
    auto load = [&](const CUtensorMap *m, int bar, uint32_t off, int c, int boxes, int x0, int g) {
        if (lane != 0 || c >= nc || !may()) return;
        mbar_expect_tx(&sh.bar[bar], boxes * TILE64);
        for (int i = 0; i < boxes; ++i)
            tma_3d<1>(base + off + i * TILE64, m, su32(&sh.bar[bar]), x0 + 64 * i, g, (int)(s.first + (int64_t)(chunks.x + c) * Q));
    };
    // (without outputs the C tile's place takes every other B)
    auto b_bar = [&](int c) { return FULL || !(c & 1) ? F_B : F_B1; };
    auto b_par = [&](int c) { return FULL ? (uint32_t)c & 1u : (uint32_t)(c >> 1) & 1u; };
    auto b_off = [&](int c) { return FULL || !(c & 1) ? OFF_B : OFF_C; };
    auto load_b = [&](int c) { load(&mB, b_bar(c), b_off(c), c, 2, 0, grp); };
    auto load_c = [&](int c) { load(&mC, F_C, OFF_C, c, 2, 0, grp); };
    auto load_x = [&](int c) { load(&mX, F_X, OFF_X, c, 1, p0, head); };
    constexpr uint32_t FMT = (1u << 4) | (1u << 7) | (1u << 10) | ((128u >> 4) << 24);  // fp32 sums of bf16, M = 128
    constexpr uint32_t N128 = (128u >> 3) << 17, N64 = ((uint32_t)PB >> 3) << 17;
    const int nk = (q.N + 15) / 16;
    auto issue_carried = [&](int c) {  // warp 1
        must(F_C, c & 1);
        if (lane != 0 || !may()) return;
        tc_fence_after();
        for (int part = 0; part < 2; ++part)
            for (int k = 0; k < nk; ++k)
                umma<1>(tmem + T_Y0, sdesc_sw128(base + OFF_C + (uint32_t)(k / 4) * TILE64 + (uint32_t)(k % 4) * 32),
                        sdesc_mn(base + OFF_H + part * TILE64 + k * 2048, TILE64), FMT | N64 | B_MN, part > 0 || k > 0);
        umma_commit<1>(&sh.bar[M_CARRIED]);
    };
    auto issue_pairs = [&](int c) {  // warp 0
        must(F_B, c & 1);
        must(F_C, c & 1);
        if (lane != 0 || !may()) return;
        tc_fence_after();
        for (int k = 0; k < nk; ++k) {
            const uint32_t o = (uint32_t)(k / 4) * TILE64 + (uint32_t)(k % 4) * 32;
            umma<1>(tmem + T_S, sdesc_sw128(base + OFF_C + o), sdesc_sw128(base + OFF_B + o), FMT | N128, k > 0);
        }
        umma_commit<1>(&sh.bar[M_PAIRS]);
    };
    auto issue_made = [&](int c) {  // warp 2
        must(b_bar(c), b_par(c));
        if (lane != 0 || !may()) return;
        tc_fence_after();
        for (int k = 0; k < Q / 16; ++k)
            for (int part = 0; part < 2; ++part)
                umma<1>(tmem + T_D, sdesc_mn(base + b_off(c) + k * 2048, TILE64), sdesc_mn(base + OFF_H + part * TILE64 + k * 2048, TILE64),
                        FMT | N64 | A_MN | B_MN, part > 0 || k > 0);
        umma_commit<1>(&sh.bar[M_MADE]);
    };
    auto issue_inside = [&]() {  // warp 3
        if (lane != 0 || !may()) return;
        tc_fence_after();
        for (int part = 0; part < 2; ++part)
            for (int k = 0; k < Q / 16; ++k)
                umma_ts(tmem + T_D, tmem + T_S + (k / 2) * 32 + (k % 2) * 8 + part * 16, sdesc_mn(base + OFF_X + k * 2048, TILE64), FMT | N64 | B_MN,
                        part > 0 || k > 0);
        umma_commit<1>(&sh.bar[M_INSIDE]);
    };
    if (warp == 4) {
        load_b(0);
        if (FULL) load_c(0);
        load_x(0);
        if (!FULL) load_b(1);
        __syncwarp();
    }
    // the state before the segment, [p][n] with lane n: from s_in, or from the segments' parts joined
    float h[32];
    const int64_t srow = s.slot >= 0 ? (((int64_t)s.slot * q.H + head) * q.P + p0) * q.N : -1;
#pragma unroll
    for (int i = 0; i < 32; ++i) {
        const int pc = half * 32 + i;
        h[i] = 0.0f;
        if (pc >= np || row >= q.N) continue;
        if (p.segs > 1 && FULL) h[i] = p.part[part0 + ((int64_t)(seg > 0 ? 1 : 0) * PB + pc) * q.N + row];
        else if (seg == 0 && q.s_in && srow >= 0) h[i] = q.s_in[srow + (int64_t)pc * q.N + row];
    }
    if (FULL) {
        for (int j = 1; j < seg; ++j) {
            const int2 ch = segment(s.len, p.segs, j);
            float sum = 0.0f;
            for (int c = ch.x; c < ch.y; ++c) sum += p.total[chunk_at(s, b, c) * q.H + head];
            const float e = exp2f(sum);
#pragma unroll
            for (int i = 0; i < 32; ++i) {
                const int pc = half * 32 + i;
                if (pc < np && row < q.N) h[i] = fmaf(h[i], e, p.part[part0 + ((int64_t)(j + 1) * PB + pc) * q.N + row]);
            }
        }
    } else if (seg == 0) {  // the second pass may store over s_in: it reads this copy
#pragma unroll
        for (int i = 0; i < 32; ++i) {
            const int pc = half * 32 + i;
            if (pc < np && row < q.N) p.part[part0 + (int64_t)pc * q.N + row] = h[i];
        }
    }
    auto put_state = [&]() {  // its two bf16 parts as an operand: rows n, 64 p
        uint8_t *hr = smem + OFF_H + row * 128;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            uint32_t hi[4], lo[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const Parts2 v = parts2(h[8 * i + 2 * e], h[8 * i + 2 * e + 1]);  // (an infinite state's small part is NaN, as its sums over B's signs are)
                hi[e] = v.hi, lo[e] = v.lo;
            }
            const uint32_t at = (uint32_t)((4 * half + i) ^ (row & 7)) << 4;
            *reinterpret_cast<uint4 *>(hr + at) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
            *reinterpret_cast<uint4 *>(hr + TILE64 + at) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
        }
        fence_proxy_async_smem();
    };
    if (FULL) put_state();
    // what this thread needs of a chunk's table, loaded a chunk ahead
    struct {
        float at, as, w, total;  // A of its row, A_s - log2 d_s (threads 0 to 127: of token s), the weight of its token, A_127
    } now, next{};
    const int64_t tab0 = chunk_at(s, b, chunks.x) * q.H + head;
    auto fetch = [&](int c) {
        if (c >= nc) return;
        const float *table = p.table + (tab0 + (int64_t)c * q.H) * TABLE;
        if (FULL) {
            next.at = __ldg(table + row);
            next.as = __ldg(table + Q + (threadIdx.x & (Q - 1)));
        }
        next.w = __ldg(table + 2 * Q + threadIdx.x / 2);
        next.total = __ldg(p.total + tab0 + (int64_t)c * q.H);
    };
    fetch(0);
    const float skip = FULL && q.d ? q.d[head] : 0.0f;
    for (int c = 0; c < nc; ++c) {
        const uint32_t par = c & 1;
        const int valid = min(Q, s.len - (chunks.x + c) * Q);  // tokens there are
        now = next;
        fetch(c + 1);
        if constexpr (FULL) {
            if (threadIdx.x < Q) sh.as[threadIdx.x] = now.as;  // (last read before the barrier ahead of the products inside)
            // ---- the state's parts are written, the chunk before has been read everywhere
            tc_fence_before();
            __syncthreads();
            if (warp == 1) issue_carried(c);
            if (warp == 0) issue_pairs(c);
            __syncwarp();
            must(M_CARRIED, par);  // X' takes the place of the state's parts
        }
        // ---- X': half a row a thread
        must(F_X, par);
        if (valid < Q) {
            must(b_bar(c), b_par(c));
            if (FULL) must(M_PAIRS, par);
        }
        {
            const int t = threadIdx.x / 2, j0 = 4 * (threadIdx.x & 1);
            const float w = now.w;
            uint8_t *xr = smem + OFF_X + t * 128, *hr = smem + OFF_H + t * 128;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t at = (uint32_t)((j0 + i) ^ (t & 7)) << 4;
                uint4 xv = *reinterpret_cast<const uint4 *>(xr + at);
                if (t >= valid) {  // rows of another sequence: nothing of them may count
                    xv = make_uint4(0u, 0u, 0u, 0u);
                    *reinterpret_cast<uint4 *>(xr + at) = xv;
                    uint8_t *br = smem + b_off(c) + t * 128 + at;
                    *reinterpret_cast<uint4 *>(br) = xv;
                    *reinterpret_cast<uint4 *>(br + TILE64) = xv;
                }
                uint32_t u[4] = {xv.x, xv.y, xv.z, xv.w}, hi[4], lo[4], odd = 0u;  // odd: a value's exponent is all ones
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float2 f = unpack2<__nv_bfloat16>(u[e]);
                    odd |= ((u[e] & 0x7f807f80u) + 0x00800080u) & 0x80008000u;
                    const Parts2 v = parts2(f.x * w, f.y * w);
                    hi[e] = v.hi, lo[e] = v.lo;
                }
                if (odd) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const uint32_t shift = 16 * (e % 2);
                        if ((u[e / 2] >> shift & 0x7f80u) != 0x7f80u) continue;
                        lo[e / 2] &= ~(0xffffu << shift);  // into the state as it is
                        if (FULL) {  // out of the product inside the chunk; its channel is NaN from here on
                            u[e / 2] &= ~(0xffffu << shift);
                            atomicMin(&sh.bad[8 * (j0 + i) + e], t);
                            sh.any_bad = 1;
                        }
                    }
                    if (FULL) *reinterpret_cast<uint4 *>(xr + at) = make_uint4(u[0], u[1], u[2], u[3]);
                }
                *reinterpret_cast<uint4 *>(hr + at) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
                *reinterpret_cast<uint4 *>(hr + TILE64 + at) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
            }
        }
        fence_proxy_async_smem();
        __syncthreads();
        if (warp == 2) issue_made(c);
        if (!FULL && warp == 4) load_x(c + 1);
        __syncwarp();
        if constexpr (FULL) {
            // ---- P from the pairs: 32 x 32 blocks, this warp's two of its rows' four; D, the
            // factor of x itself, joins the diagonal
            const float At = now.at;
            must(M_PAIRS, par);
            tc_fence_after();
            if (warp == 4) load_c(c + 1);  // (both of its products are done)
#pragma unroll
            for (int step = 0; step < 2; ++step) {
                // a block's two parts, 16 columns each, take the place of its pairs
                const int blk = 2 * step + half;
                uint32_t hi[16], lo[16];
                __syncwarp();
                if (blk <= quarter) {
                    uint32_t v[32];
                    tmem_ld32(tmem + lanes + T_S + 32 * blk, v);
                    auto weigh = [&](auto diagonal) {
#pragma unroll
                        for (int j = 0; j < 8; ++j) {
                            const float4 As = *reinterpret_cast<const float4 *>(&sh.as[32 * blk + 4 * j]);
                            const float as[4] = {As.x, As.y, As.z, As.w};
                            float f[4];
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                f[e] = __uint_as_float(v[4 * j + e]) * ex2(At - as[e]);
                                if (diagonal.value) f[e] = 4 * j + e < lane ? f[e] : 4 * j + e == lane ? f[e] + skip : 0.0f;
                            }
                            const Parts2 a = parts2(f[0], f[1]), bb = parts2(f[2], f[3]);
                            hi[2 * j] = a.hi, hi[2 * j + 1] = bb.hi, lo[2 * j] = a.lo, lo[2 * j + 1] = bb.lo;
                        }
                    };
                    if (blk == quarter) weigh(std::true_type{});
                    else weigh(std::false_type{});
                } else {
#pragma unroll
                    for (int j = 0; j < 16; ++j) hi[j] = lo[j] = 0u;
                }
                __syncwarp();
                tmem_st16(tmem + lanes + T_S + 32 * blk, hi);
                tmem_st16(tmem + lanes + T_S + 32 * blk + 16, lo);
            }
            tmem_wait_st();
        }
        // ---- the state behind the chunk
        must(M_MADE, par);
        tc_fence_after();
        {
            const float e = exp2f(now.total);
            uint32_t v[32];
            __syncwarp();
            tmem_ld32(tmem + lanes + T_D + 32 * half, v);
#pragma unroll
            for (int i = 0; i < 32; ++i) h[i] = fmaf(h[i], e, __uint_as_float(v[i]));
        }
        tc_fence_before();
        if constexpr (FULL) {
            __syncthreads();  // P is written, the made state has been read
            if (warp == 3) issue_inside();
            if (warp == 4) load_b(c + 1);
            __syncwarp();
            put_state();
            // ---- the chunk's outputs
            const float et = ex2(now.at);
            must(M_INSIDE, par);
            if (warp == 4) load_x(c + 1);
            __syncwarp();
            tc_fence_after();
            const bool bad = *reinterpret_cast<volatile int *>(&sh.any_bad);
            __nv_bfloat16 *yr = y + (s.first + (int64_t)(chunks.x + c) * Q + row) * q.ldy + (int64_t)head * q.P + p0 + 32 * half;
#pragma unroll
            for (int i2 = 0; i2 < 2; ++i2) {
                uint32_t y0[16], y1[16];
                __syncwarp();
                tmem_ld16x2(tmem + lanes + T_Y0 + 32 * half + 16 * i2, y0, tmem + lanes + T_D + 32 * half + 16 * i2, y1);
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const int i = 2 * i2 + j;
                    uint32_t o[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        float f0 = fmaf(__uint_as_float(y0[8 * j + 2 * e]), et, __uint_as_float(y1[8 * j + 2 * e]));
                        float f1 = fmaf(__uint_as_float(y0[8 * j + 2 * e + 1]), et, __uint_as_float(y1[8 * j + 2 * e + 1]));
                        if (bad) {
                            if (row >= sh.bad[32 * half + 8 * i + 2 * e]) f0 = NAN;
                            if (row >= sh.bad[32 * half + 8 * i + 2 * e + 1]) f1 = NAN;
                        }
                        o[e] = pack2<__nv_bfloat16>(f0, f1);
                    }
                    if (row < valid && 32 * half + 8 * i < np) *reinterpret_cast<uint4 *>(yr + 8 * i) = make_uint4(o[0], o[1], o[2], o[3]);
                }
            }
            if (bad) {  // (the same in every warp: it was set before the barrier behind X')
                __syncthreads();
                if (threadIdx.x < PB) sh.bad[threadIdx.x] = Q;
                if (threadIdx.x == 0) sh.any_bad = 0;
            }
        } else {
            // (the next chunk's X' is written behind this wait: its place has been read)
            if (warp == 4) load_b(c + 2);
            __syncwarp();
        }
    }
    // the state behind the segment
    if (may()) {
        float *out = FULL ? (seg == p.segs - 1 && q.s_out && srow >= 0 ? q.s_out + srow : nullptr)
                          : p.part + part0 + (int64_t)(seg + 1) * PB * q.N;
        if (out) {
#pragma unroll
            for (int i = 0; i < 32; ++i) {
                const int pc = half * 32 + i;
                if (pc < np && row < q.N) out[(int64_t)pc * q.N + row] = h[i];
            }
        }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 4 && lane == 0 && sh.abort) {  // copies in flight land before the block's memory goes away (bounded)
        const long long t0 = clock64();
        while (clock64() - t0 < WAIT_LIMIT / 1000) {
        }
    }
    __syncthreads();
    if (warp == 0) {
        tc_fence_after();
        tmem_dealloc<1>(tmem, COLS);
    }
}

// Segments that a sequence is cut into: as many as fill two blocks an SM, of four chunks at least
int segments_of(const SsmP &p) {
    const int64_t full = (p.q.tokens + p.q.max_len - 1) / std::max<int64_t>(p.q.max_len, 1);  // sequences, counted by length
    const int64_t blocks = full * p.H * ((p.P + PB - 1) / PB), chunks = (p.q.max_len + Q - 1) / Q;
    const int64_t want = 2LL * num_sms() / std::max<int64_t>(blocks, 1);
    return (int)std::max<int64_t>(1, std::min<int64_t>(std::min<int64_t>(want, 64), chunks / 4));
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
    const int segs = segments_of(p);
    w.bytes = w.part + (segs > 1 ? up((int64_t)p.q.batch * p.H * ((p.P + PB - 1) / PB) * segs * PB * p.N * 4) : 0);
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
    TcP p{s, segments_of(s), reinterpret_cast<float *>(base + w.table), reinterpret_cast<float *>(base + w.total),
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
    static bool set = false;  // (idempotent)
    if (!set) {
        cudaError_t e = cudaFuncSetAttribute(ssm_scan_tc_kernel<true>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)SCAN_SMEM);
        if (e == cudaSuccess)
            e = cudaFuncSetAttribute(ssm_scan_tc_kernel<false>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)SCAN_SMEM);
        if (e != cudaSuccess) return e;
        set = true;
    }
    const unsigned chunks = (unsigned)((s.q.max_len + Q - 1) / Q), heads = (unsigned)(s.H * p.pblocks);
    const int vec = s.H % 8 == 0 && s.lddt % 8 == 0 && reinterpret_cast<uintptr_t>(dtv) % 16 == 0;
    cudaError_t e = launch_pdl(ssm_steps_kernel, dim3(chunks, (unsigned)((s.H + 7) / 8), (unsigned)s.q.batch), dim3(256), 0, st, p, dtv, vec);
    if (e != cudaSuccess) return e;
    if (p.segs > 1) {
        e = launch_pdl(ssm_scan_tc_kernel<false>, dim3(heads, (unsigned)(p.segs - 1), (unsigned)s.q.batch), dim3(SCAN_THREADS), SCAN_SMEM, st,
                       mX, mB, mC, p, y);
        if (e != cudaSuccess) return e;
    }
    return launch_pdl(ssm_scan_tc_kernel<true>, dim3(heads, (unsigned)p.segs, (unsigned)s.q.batch), dim3(SCAN_THREADS), SCAN_SMEM, st, mX, mB,
                      mC, p, y);
}

}  // namespace k
}  // namespace sn
