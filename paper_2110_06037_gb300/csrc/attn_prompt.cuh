// Attention of many queries (prompts) over a cache of 16-bit values on the 5th-generation tensor cores
// (sn_attend in include/sn.h).
//
//   S = Q K^T,   P = 2^(c S - m),   O += P V,   l += sum of P,   y = O / l
// What bounds it is the tensor pipe: 4 D operations a query and key, and one exponential.  A block of one SM takes NT tiles of
// 128 rows (a row: a token's query head; the heads that share the cache's head are neighbours) and goes through
// their keys KT at a time.  TMEM holds S of two tiles and O; P, in the queries' type, takes the place of its S and
// is the next product's operand from there, so that scores never leave the SM.  Warps, each for one thing:
//   4 NT  softmax: a thread has a row, so that no row's maximum or sum crosses threads
//   1     copies: keys and values of whole pages (or KT of their tokens) by TMA, in a ring
//   1     issues the products
//   1     waits for the copies on behalf of the one before (its own accesses to shared memory would queue behind
//         the products' operand reads), and clears values behind a sequence's end
// Two tiles (NT = 2) take turns: while one's softmax works, the other's products run.  One tile (few rows, or heads
// beyond 128 values, whose O fills the columns) has two S in turn, the next one's product ahead of its softmax.
// m is the largest score so far only up to a factor: O and l are scaled again when it grows beyond 2^THR, which
// O, in fp32, and P, of its type's range, allow, and which random scores do once or twice a row.
// A weight is rounded once, to the queries' type: off by half a step of the output's type, and independent from
// key to key.  (fp16: the largest weight is between 2^14 and 2^15, so that one is off by 2^-11 of itself or 2^-39 of the largest.)
// Products on different accumulators do not keep their order, so the S that takes P's place waits until P has been read.
// A wait by parity holds only where the phase before is known to be over and the one after is not: see attn_order.h.
// Prompts of 4096 and 777 tokens, 32 heads of 128 over 8, bf16: 187 us a call, 820 TFLOP/s, of which this kernel takes 164 (profiled) and
// the launches for few rows before it, which find nothing to do there, the rest.  A pair of tiles of rows and a tile of keys take
// some 4900 cycles of a multiprocessor, the tensor cores busy 46 % of them: a tile goes from S through its softmax to the
// products before its next S, and two of them side by side do not fill that.  The instances with two tiles spill 164
// bytes a thread: a row's 128 scores are live at once.
#pragma once

#include "attn_common.cuh"
#include "attn_order.h"
#include "tc_common.cuh"

namespace sn {
namespace k {
namespace prompt {

using namespace tc;

template <int DT, int NT>
struct Form {
    static constexpr int KT = DT > 128 ? 64 : 128;  // keys of a tile
    static constexpr int LA = NT == 1 ? 2 : 1;      // S are this many tiles ahead of their P
    static constexpr uint32_t Q_BYTES = 128 * DT * 2, STAGE = KT * DT * 2;
    static constexpr uint32_t R = DT == 64 ? 8 : NT == 1 && DT == 128 ? 6 : 5;  // tiles of keys or values in the ring
    static constexpr uint32_t OFF_RING = NT * Q_BYTES, OFF_SH = OFF_RING + R * STAGE;
    static constexpr size_t BYTES = OFF_SH + 1024;
    static constexpr int THREADS = NT * 128 + 128;  // (the last warp has nothing to do)
    // registers a thread: at the launch, and of two tiles' softmax and the others then
    static constexpr int REGS = 168, REGS_SOFT = 216, REGS_REST = 72;
    static_assert(NT == 1 || 2 * REGS_SOFT + REGS_REST <= 3 * REGS, "a share beyond what the block was launched with would be waited for without end");
    static constexpr uint32_t T_S = KT, T_O = 256;  // columns of an S; first of O (tile t: 128 t further)
    static_assert(BYTES <= 227 * 1024, "shared memory of a block");
};
struct Shared {
    uint64_t full[8], empty[8], s[2], pv[2];
    int64_t start[4];
    uint32_t tmem;
    int abort, again;  // a wait gave up; a result is not finite
};
static_assert(sizeof(Shared) <= 1024, "behind the ring");

// an MN-major operand: rows of 128 bytes are 64 values of the N axis at one k, 128-byte swizzled; groups of
// 8 k 1024 bytes apart, blocks of 64 values `block` bytes
__device__ __forceinline__ uint64_t sdesc_mn(uint32_t saddr, uint32_t block) {
    return (uint64_t)((saddr & 0x3FFFFu) >> 4) | (uint64_t)(block >> 4) << 16 | (uint64_t)(1024 >> 4) << 32 | (uint64_t)1 << 46 | (uint64_t)2 << 61;
}
constexpr uint32_t B_MN = 1u << 16;  // instruction descriptor: B is MN-major

// 32 columns asked for; what was asked for is there (N: registers of it)
template <int B, int N>
__device__ __forceinline__ void tmem_ask32(uint32_t ta, uint32_t (&v)[N]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
        : "=r"(v[B + 0]), "=r"(v[B + 1]), "=r"(v[B + 2]), "=r"(v[B + 3]), "=r"(v[B + 4]), "=r"(v[B + 5]), "=r"(v[B + 6]), "=r"(v[B + 7]),
          "=r"(v[B + 8]), "=r"(v[B + 9]), "=r"(v[B + 10]), "=r"(v[B + 11]), "=r"(v[B + 12]), "=r"(v[B + 13]), "=r"(v[B + 14]), "=r"(v[B + 15]),
          "=r"(v[B + 16]), "=r"(v[B + 17]), "=r"(v[B + 18]), "=r"(v[B + 19]), "=r"(v[B + 20]), "=r"(v[B + 21]), "=r"(v[B + 22]), "=r"(v[B + 23]),
          "=r"(v[B + 24]), "=r"(v[B + 25]), "=r"(v[B + 26]), "=r"(v[B + 27]), "=r"(v[B + 28]), "=r"(v[B + 29]), "=r"(v[B + 30]), "=r"(v[B + 31])
        : "r"(ta)
        : "memory");
}
template <int B, int N>
__device__ __forceinline__ void tmem_have32(uint32_t (&v)[N]) {
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+r"(v[B + 0]), "+r"(v[B + 1]), "+r"(v[B + 2]), "+r"(v[B + 3]), "+r"(v[B + 4]), "+r"(v[B + 5]), "+r"(v[B + 6]), "+r"(v[B + 7]),
                   "+r"(v[B + 8]), "+r"(v[B + 9]), "+r"(v[B + 10]), "+r"(v[B + 11]), "+r"(v[B + 12]), "+r"(v[B + 13]), "+r"(v[B + 14]), "+r"(v[B + 15]),
                   "+r"(v[B + 16]), "+r"(v[B + 17]), "+r"(v[B + 18]), "+r"(v[B + 19]), "+r"(v[B + 20]), "+r"(v[B + 21]), "+r"(v[B + 22]), "+r"(v[B + 23]),
                   "+r"(v[B + 24]), "+r"(v[B + 25]), "+r"(v[B + 26]), "+r"(v[B + 27]), "+r"(v[B + 28]), "+r"(v[B + 29]), "+r"(v[B + 30]), "+r"(v[B + 31])
                 :
                 : "memory");
}
template <int N>
__device__ __forceinline__ void tmem_put32(uint32_t ta, const uint32_t (&v)[N]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], "
        "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, "
        "%17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32};" ::"r"(ta),
        "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]), "r"(v[9]), "r"(v[10]), "r"(v[11]),
        "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15]), "r"(v[16]), "r"(v[17]), "r"(v[18]), "r"(v[19]), "r"(v[20]), "r"(v[21]), "r"(v[22]),
        "r"(v[23]), "r"(v[24]), "r"(v[25]), "r"(v[26]), "r"(v[27]), "r"(v[28]), "r"(v[29]), "r"(v[30]), "r"(v[31])
        : "memory");
}
__device__ __forceinline__ void tmem_put16(uint32_t ta, const uint32_t (&v)[16]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};" ::"r"(ta), "r"(v[0]),
        "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]), "r"(v[9]), "r"(v[10]), "r"(v[11]), "r"(v[12]),
        "r"(v[13]), "r"(v[14]), "r"(v[15])
        : "memory");
}
template <int N>
__device__ __forceinline__ void regs_up() {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N));
}
template <int N>
__device__ __forceinline__ void regs_down() {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N));
}
__device__ __forceinline__ void tmem_stored() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void bar_arrive(uint32_t id, uint32_t count) { asm volatile("bar.arrive %0, %1;" ::"r"(id), "r"(count) : "memory"); }
__device__ __forceinline__ void bar_wait(uint32_t id, uint32_t count) { asm volatile("bar.sync %0, %1;" ::"r"(id), "r"(count) : "memory"); }

// what a piece of work is to the warps: rows and tiles of keys of each tile of rows
template <int NT, int KT>
struct Part {
    int rows[NT], n[NT], most, user;  // user: the tile of rows that is the last to use a tile of keys
    __device__ __forceinline__ Part(const AttnP &p, const Piece &w) {
        const int64_t row0 = (int64_t)w.tile * (128 * NT), all = (int64_t)w.past.s.len * p.group;
        most = user = 0;
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            rows[t] = (int)max((int64_t)0, min((int64_t)128, all - row0 - 128 * t));
            const int end = rows[t] ? last_key(p, w.past, row0 + 128 * t + rows[t] - 1) : -1;
            n[t] = end < 0 ? 0 : max(0, min(w.u1, end / KT + 1) - w.u0);
            if (n[t]) user = t;
            most = max(most, n[t]);
        }
    }
};

template <typename T, int DT, int NT>
__global__ void __launch_bounds__(Form<DT, NT>::THREADS, 1)
    attend_prompt_kernel(const __grid_constant__ CUtensorMap mK, const __grid_constant__ CUtensorMap mV, const __grid_constant__ AttnP p) {
    using F = Form<DT, NT>;
    constexpr int KT = F::KT, LA = F::LA, GATE = 128 + 64;  // threads that meet at a named barrier: a tile's softmax, two warps
    constexpr uint32_t R = F::R;
    constexpr float TOP = top_weight<T, false>(), THR = std::is_same<T, __half>::value ? 1.0f : 8.0f;
    extern __shared__ __align__(1024) uint8_t smem[];
    Shared &sh = *reinterpret_cast<Shared *>(smem + F::OFF_SH);
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const int d = p.c.head_dim;
    if (su32(smem) & 1023) {  // (the swizzled tiles need it; uniform over the block)
        if (threadIdx.x == 0) atomicOr(p.err, ERR_TMA_WAIT);
        return;
    }
    if (warp == 0) {
        tmem_alloc<1>(&sh.tmem, 512);
    } else if (warp == 1) {
        if (lane < 20) mbar_init(&sh.full[0] + lane, 1);
        if (lane == 31) sh.abort = sh.again = 0;
        fence_mbar_init();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = __shfl_sync(0xffffffffu, sh.tmem, 0);
    griddep_launch();  // (behind the allocation: see tmem_alloc)
    griddep_wait();
    Pieces pieces;
    pieces.start(p, sh.start);
    const uint32_t base = su32(smem), ring = base + F::OFF_RING;
    const int nb = KT / min(p.c.page, KT), shift = 31 - __clz(p.c.page);  // pages of a tile (or 1: a part of one)
    bool ok = true;
    auto must = [&](uint64_t *bar, uint32_t par, int code) {  // a whole warp's wait; after one that gave up, no further ones
        if (ok && !__all_sync(0xffffffffu, mbar_wait(bar, par))) {
            if (lane == 0) {
                atomicOr(p.err, code);
                *reinterpret_cast<volatile int *>(&sh.abort) = 1;
            }
            ok = false;
        }
        return ok;
    };
    // the page of this lane's part of a tile of keys, `of` keys, -1: none
    auto page_of = [&](const Piece &w, int j, int of) {
        if (lane * of >= KT) return -1;
        const int key = (w.u0 + j) * KT + lane * of;
        if (key >= w.past.ctx) return -1;
        const int n = p.t.at[(int64_t)w.past.s.slot * p.t.width + (key >> shift)];
        return n >= 0 && n < p.c.pages ? n : -1;
    };

    if (NT == 2 && warp >= 4 * NT) regs_down<F::REGS_REST>();
    if (warp == 4 * NT) {  // ---------------- copies
        uint32_t at = 0;
        const int chunks = (d + 63) / 64, bp = min(p.c.page, KT);
        for (Piece w; ok && pieces.next(p, w);) {
            const Part<NT, KT> part(p, w);
            int page = part.most ? page_of(w, 0, bp) : -1;
            for (int j = 0; j < part.most && ok; ++j) {
                const int now = page >= 0 ? page : p.c.pages;  // (behind the last page: reads as zeros)
                const int in = ((w.u0 + j) * KT) & (p.c.page - 1);
                if (j + 1 < part.most) page = page_of(w, j + 1, bp);
#pragma unroll 1
                for (int which = 0; which < 2; ++which, ++at) {
                    const uint32_t st = at % R;
                    if (at >= R && !must(&sh.empty[st], (at / R - 1) & 1u, ERR_TMA_WAIT)) break;
                    const uint32_t bar = su32(&sh.full[st]);
                    if (lane == 0) mbar_expect_tx(&sh.full[st], chunks * KT * 128);
                    __syncwarp();
                    if (lane < nb)
                        for (int c = 0; c < chunks; ++c)
                            tma_4d<1>(ring + st * F::STAGE + c * (KT * 128) + lane * bp * 128, which ? &mV : &mK, bar, 64 * c, in, w.head, now);
                }
            }
        }
    } else if (warp == 4 * NT + 1) {  // ---------------- products: the whole warp, so that descriptors stay in uniform registers
        const uint32_t one = elect_one();
        constexpr uint32_t FMT = (1u << 4) | (std::is_same<T, __half>::value ? 0u : (1u << 7) | (1u << 10)) | ((128u >> 4) << 24);
        const uint32_t NS = FMT | ((uint32_t)KT >> 3) << 17, NO = FMT | B_MN | ((uint32_t)d >> 3) << 17;
        const int ks = d / 16;
        uint32_t at = 0, tiles = 0, gate = 0;  // positions of the ring, S and meetings so far (of the pieces before)
        uint32_t read[2] = {0, 0};             // products with P of each tile
        for (Piece w; pieces.next(p, w);) {
            const Part<NT, KT> part(p, w);
            auto meet = [&](int t) {
                bar_wait(NT == 2 ? 2 + t : 2 + (gate++ & 1u), GATE);
                tc_fence_after();
            };
            auto scores = [&](int t, int j) {
                const uint32_t st = (at + 2 * j) % R, b = NT == 2 ? t : (tiles + j) & 1u;
                const uint64_t a = sdesc_sw128(base + t * F::Q_BYTES), k = sdesc_sw128(ring + st * F::STAGE);
#pragma unroll
                for (int i = 0; i < DT / 16; ++i)
                    if (i < ks)
                        umma_one<1>(one, tmem + b * F::T_S, a + (i / 4 * (128 * 128 >> 4) + i % 4 * 2), k + (i / 4 * (KT * 128 >> 4) + i % 4 * 2), NS, i > 0);
                commit_one<1>(one, &sh.s[b]);
                if (t == part.user) commit_one<1>(one, &sh.empty[st]);
            };
            auto values = [&](int t, int j) {
                const uint32_t st = (at + 2 * j + 1) % R, b = NT == 2 ? t : (tiles + j) & 1u;
                const uint64_t v = sdesc_mn(ring + st * F::STAGE, KT * 128);
#pragma unroll
                for (int i = 0; i < KT / 16; ++i)
                    umma_ts_one(one, tmem + F::T_O + t * 128, tmem + b * F::T_S + 8 * i, v + i * (2048 >> 4), NO, i > 0 || j > 0);
                commit_one<1>(one, &sh.pv[t]);
                if (t == part.user) commit_one<1>(one, &sh.empty[st]);
            };
#pragma unroll
            for (int t = 0; t < NT; ++t)
                if (part.n[t]) {
                    meet(t);
                    for (int i = 0; i < min(LA, part.n[t]); ++i) scores(t, i);
                }
#pragma unroll 1
            for (int j = 0; j < part.most; ++j)
#pragma unroll
                for (int t = 0; t < NT; ++t)
                    if (j < part.n[t]) {
                        meet(t);
                        values(t, j);
                        const uint32_t par = read[t]++ & 1u;
                        if (j + LA < part.n[t]) {
                            must(&sh.pv[t], par, ERR_MMA_WAIT);
                            tc_fence_after();
                            scores(t, j + LA);
                        }
                    }
            at += 2 * part.most, tiles += part.most;
        }
    } else if (warp == 4 * NT + 2) {  // ---------------- waits for the copies
        uint32_t at = 0, gate = 0;
        for (Piece w; pieces.next(p, w);) {
            const Part<NT, KT> part(p, w);
            auto have = [&](int i) { must(&sh.full[(at + i) % R], (at + i) / R & 1u, ERR_MMA_WAIT); };
            auto meet = [&](int t) {
                __syncwarp();  // (it stays until the others have come too: two arrivals ahead would count for them)
                bar_wait(NT == 2 ? 2 + t : 2 + (gate++ & 1u), GATE);
            };
#pragma unroll
            for (int t = 0; t < NT; ++t)
                if (part.n[t]) {
                    for (int i = 0; i < min(LA, part.n[t]); ++i) have(2 * i);
                    meet(t);
                }
            bool cleared = false;
#pragma unroll 1
            for (int j = 0; j < part.most; ++j)
#pragma unroll
                for (int t = 0; t < NT; ++t)
                    if (j < part.n[t]) {
                        have(2 * j + 1);
                        // values behind the sequence: anything may be there, and 0 times infinity is not 0
                        const int left = w.past.ctx - (w.u0 + j) * KT;
                        if (left < KT && !cleared && ok) {
                            cleared = true;
                            uint8_t *v = smem + F::OFF_RING + (at + 2 * j + 1) % R * F::STAGE;
                            for (int i = left * 8 + lane; i < KT * 8; i += 32)
                                for (int c = 0; c < (d + 63) / 64; ++c) *reinterpret_cast<uint4 *>(v + c * (KT * 128) + i * 16) = make_uint4(0u, 0u, 0u, 0u);
                            fence_proxy_async_smem();
                        }
                        if (j + LA < part.n[t]) have(2 * (j + LA));
                        meet(t);
                    }
            at += 2 * part.most;
        }
    } else if (warp < 4 * NT) {  // ---------------- softmax: a thread's row
        if (NT == 2) regs_up<F::REGS_SOFT>();
        const int t = warp / 4, r = threadIdx.x % 128;
        const uint32_t lanes = (uint32_t)((warp % 4) * 32) << 16, o_at = tmem + lanes + F::T_O + t * 128;
        const float c = p.scale == 0.0f ? 1.0f : fabsf(p.scale);
        const uint32_t flip = p.scale < 0.0f ? 0x80008000u : 0u, keep = p.scale == 0.0f ? 0u : 0xffffffffu;
        const bool vec_x = (reinterpret_cast<uintptr_t>(p.h.x) | (uintptr_t)(p.h.ldx * 2) | (uintptr_t)(p.h.hx * 2)) % 16 == 0;
        const bool vec_y = (reinterpret_cast<uintptr_t>(p.h.y) | (uintptr_t)(p.h.ldy * 2) | (uintptr_t)(p.h.hy * 2)) % 16 == 0;
        uint32_t tiles = 0, sums = 0, gate = 0;  // S and P V so far (of the pieces before)
        for (Piece w; pieces.next(p, w);) {
            const Part<NT, KT> part(p, w);
            const int n = part.n[NT == 2 ? t : 0], rows = part.rows[NT == 2 ? t : 0];
            const Seq &s = w.past.s;
            const int64_t row = (int64_t)w.tile * (128 * NT) + 128 * t + r;
            const bool mine = r < rows;
            auto meet = [&]() { bar_arrive(NT == 2 ? 2 + t : 2 + (gate++ & 1u), GATE); };
            if (n) {  // this row of the queries
                const T *x = static_cast<const T *>(p.h.x) + (s.first + row / p.group) * p.h.ldx + ((int64_t)w.head * p.group + row % p.group) * p.h.hx;
                uint8_t *q = smem + t * F::Q_BYTES + r * 128;
                for (int i = 0; i < d / 8; ++i) {
                    uint4 u = make_uint4(0u, 0u, 0u, 0u);
                    if (mine) {
                        if (vec_x) {
                            u = *reinterpret_cast<const uint4 *>(x + 8 * i);
                        } else {
                            const uint16_t *h = reinterpret_cast<const uint16_t *>(x + 8 * i);
                            u = make_uint4(h[0] | (uint32_t)h[1] << 16, h[2] | (uint32_t)h[3] << 16, h[4] | (uint32_t)h[5] << 16, h[6] | (uint32_t)h[7] << 16);
                        }
                    }
                    u.x = (u.x ^ flip) & keep, u.y = (u.y ^ flip) & keep, u.z = (u.z ^ flip) & keep, u.w = (u.w ^ flip) & keep;
                    *reinterpret_cast<uint4 *>(q + i / 8 * (128 * 128) + ((i % 8) ^ (r & 7)) * 16) = u;
                }
                fence_proxy_async_smem();
                tc_fence_before();
                meet();
            }
            const int last = mine ? last_key(p, w.past, row) : INT32_MAX;  // (rows behind the queries: zeros, written nowhere)
            float m = -INFINITY;
            F2 l2 = f2(0.0f, 0.0f);
            int page = n ? page_of(w, 0, 16) : -1;
#pragma unroll 1
            for (int j = 0; j < n; ++j) {
                const uint32_t there = __ballot_sync(0xffffffffu, page >= 0);
                if (j + 1 < n) page = page_of(w, j + 1, 16);
                const uint32_t b = NT == 2 ? t : (tiles + j) & 1u, par = NT == 2 ? (tiles + j) & 1u : (tiles + j) >> 1 & 1u;
                const uint32_t s_at = tmem + lanes + b * F::T_S;
                must(&sh.s[b], par, ERR_EPI_WAIT);
                tc_fence_after();
                uint32_t x[KT];
                tmem_ask32<0>(s_at, x);
                tmem_ask32<32>(s_at + 32, x);
                if constexpr (KT == 128) {
                    tmem_ask32<64>(s_at + 64, x);
                    tmem_ask32<96>(s_at + 96, x);
                    tmem_have32<96>(x);
                    tmem_have32<64>(x);
                }
                tmem_have32<32>(x);
                tmem_have32<0>(x);
                const int seen = last - (w.u0 + j) * KT;  // (of a row behind the queries: all)
                if (!__all_sync(0xffffffffu, seen >= KT - 1)) {
#pragma unroll
                    for (int i = 0; i < KT; ++i)
                        if (i > seen) x[i] = 0xff800000u;
                }
                if (there != (1u << KT / 16) - 1u) {
#pragma unroll
                    for (int i = 0; i < KT; ++i)
                        if (!(there >> i / 16 & 1u)) x[i] = 0xff800000u;
                }
                float up = -INFINITY, up1 = -INFINITY;
#pragma unroll
                for (int i = 0; i < KT; i += 4) {
                    up = fmaxf(fmaxf(up, __uint_as_float(x[i])), __uint_as_float(x[i + 1]));
                    up1 = fmaxf(fmaxf(up1, __uint_as_float(x[i + 2])), __uint_as_float(x[i + 3]));
                }
                up = fmaxf(up, up1) * c;
                float f = 1.0f;
                const bool grew = up > m + THR;
                if (grew) f = ex2(m - up), m = up;
                if (__any_sync(0xffffffffu, grew)) {
                    l2 = mul_2(l2, f2(f, f));
                    if (j > 0) {  // (the product before that one is over: these scores were asked for behind it)
                        must(&sh.pv[t], (sums + j - 1) & 1u, ERR_EPI_WAIT);
                        tc_fence_after();
#pragma unroll 1
                        for (int e = 0; e < d; e += 32) {
                            uint32_t o[32];
                            tmem_ask32<0>(o_at + e, o);
                            tmem_have32<0>(o);
#pragma unroll
                            for (int i = 0; i < 32; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * f);
                            tmem_put32(o_at + e, o);
                        }
                    }
                }
                const float low = TOP - (m == -INFINITY ? 0.0f : m);
                const F2 c2 = f2(c, c), low2 = f2(low, low);
                F2 sum[2] = {l2, f2(0.0f, 0.0f)};
#pragma unroll
                for (int h = 0; h < KT / 32; ++h) {
                    uint32_t u[16];
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const float2 e = floats(fma_2(f2(__uint_as_float(x[32 * h + 2 * i]), __uint_as_float(x[32 * h + 2 * i + 1])), c2, low2));
                        const float a = ex2(e.x), b1 = ex2(e.y);
                        sum[i % 2] = add_2(sum[i % 2], f2(a, b1));
                        u[i] = pack2<T>(a, b1);
                    }
                    tmem_put16(s_at + 16 * h, u);
                }
                l2 = add_2(sum[0], sum[1]);
                tmem_stored();
                if (waits_before_weights(j, n, LA)) must(&sh.pv[t], (sums + j - 1) & 1u, ERR_EPI_WAIT);
                tc_fence_before();
                meet();
            }
            if (n) {
                must(&sh.pv[t], (sums + n - 1) & 1u, ERR_EPI_WAIT);
                tc_fence_after();
            }
            tiles += n, sums += n;
            const float2 lf = floats(l2);
            const float l = lf.x + lf.y, inv = l == 0.0f ? 0.0f : 1.0f / l;
            bool bad = false;
            T *y = static_cast<T *>(p.h.y) + (s.first + row / p.group) * p.h.ldy + ((int64_t)w.head * p.group + row % p.group) * p.h.hy;
            float *part_at = w.slot >= 0 ? part_of_slot(p, w.slot) : nullptr;
            const int pr = 128 * t + r;
            if (part_at && mine) part_at[(int64_t)p.rows * d + pr] = m, part_at[(int64_t)p.rows * d + p.rows + pr] = l;
#pragma unroll 1
            for (int e = 0; e < d; e += 32) {
                uint32_t o[32];
                if (n) {
                    tmem_ask32<0>(o_at + e, o);
                    tmem_have32<0>(o);
                }
#pragma unroll
                for (int i = 0; i < 32; i += 8) {
                    if (e + i >= d || !mine) continue;
                    float f[8];
#pragma unroll
                    for (int k = 0; k < 8; ++k) f[k] = l == 0.0f ? 0.0f : __uint_as_float(o[i + k]) * (part_at ? 1.0f : inv);
#pragma unroll
                    for (int k = 0; k < 8; ++k) bad |= !(fabsf(f[k]) < INFINITY);
                    if (part_at) {
                        float4 *q = reinterpret_cast<float4 *>(part_at + (int64_t)pr * d + e + i);
                        q[0] = make_float4(f[0], f[1], f[2], f[3]), q[1] = make_float4(f[4], f[5], f[6], f[7]);
                    } else if (vec_y) {
                        *reinterpret_cast<uint4 *>(y + e + i) = make_uint4(pack2<T>(f[0], f[1]), pack2<T>(f[2], f[3]), pack2<T>(f[4], f[5]), pack2<T>(f[6], f[7]));
                    } else {
#pragma unroll
                        for (int k = 0; k < 8; ++k) stf(y + e + i + k, f[k]);
                    }
                }
            }
            if (bad) *reinterpret_cast<volatile int *>(&sh.again) = 1;
        }
        // such rows, when every piece of the block is done: no other warp waits for these then
        bar_wait(1, 128 * NT);
        if (*reinterpret_cast<volatile int *>(&sh.again) && ok) {
            pieces.rewind(sh.start);
            for (Piece w; pieces.next(p, w);) {
                const int rows = (int)min((int64_t)128 * NT, (int64_t)w.past.s.len * p.group - (int64_t)w.tile * (128 * NT));
                for (int i = warp; i < rows; i += 4 * NT) attend_again<T, 16>(p, w.b, w.head, w.tile, i, w.u0, w.u1, w.slot);
            }
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

template <typename T, int DT, int NT>
cudaError_t launch(const AttnP &p, int dt, int64_t grid, cudaStream_t st) {
    using F = Form<DT, NT>;
    const int d = p.c.head_dim;
    CUtensorMap m[2];
    const uint64_t dims[4] = {(uint64_t)d, (uint64_t)p.c.page, (uint64_t)p.c.heads, (uint64_t)p.c.pages};
    const uint64_t strides[3] = {(uint64_t)d * 2, dims[1] * d * 2, dims[2] * dims[1] * d * 2};
    const uint32_t box[4] = {64, (uint32_t)(p.c.page < F::KT ? p.c.page : F::KT), 1, 1};
    for (int i = 0; i < 2; ++i)
        if (!tma_encode(&m[i], dt, 4, i ? p.c.v : p.c.k, dims, strides, box, CU_TENSOR_MAP_SWIZZLE_128B)) return cudaErrorInvalidValue;
    static PerDevice set;
    if (const cudaError_t e = allow_smem(set, attend_prompt_kernel<T, DT, NT>, F::BYTES)) return e;
    return launch_pdl(attend_prompt_kernel<T, DT, NT>, dim3((unsigned)grid), dim3(F::THREADS), F::BYTES, st, m[0], m[1], p);
}
template <typename T>
cudaError_t launch_any(const AttnP &p, int dt, int64_t grid, cudaStream_t st) {
    const int d = p.c.head_dim;
    if (d > 128) return launch<T, 256, 1>(p, dt, grid, st);
    if (p.rows == 128) return d <= 64 ? launch<T, 64, 1>(p, dt, grid, st) : launch<T, 128, 1>(p, dt, grid, st);
    return d <= 64 ? launch<T, 64, 2>(p, dt, grid, st) : launch<T, 128, 2>(p, dt, grid, st);
}

}  // namespace prompt

cudaError_t attend_prompt_f16(const AttnP &p, int64_t grid, cudaStream_t st);
cudaError_t attend_prompt_bf16(const AttnP &p, int64_t grid, cudaStream_t st);

}  // namespace k
}  // namespace sn
