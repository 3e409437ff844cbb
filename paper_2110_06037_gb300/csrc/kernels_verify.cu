// Verification of drafted tokens (sn_verify_draft in include/sn.h).
//
// A cluster of 1 to 8 blocks takes a sequence.  Each block finds the first token that is not accepted
// (a load of two probabilities a token); the row behind it is cut into the blocks' and their warps'
// contiguous pieces, whose weights are summed in units of 2^-60, in integers: exact, so that neither the
// cut nor the order matters.  With every block's and warp's sum known, one warp's piece holds the drawn
// index, and that warp's block goes through it once more (from L2): the warps' sums of its parts, and one warp's
// running sums.  64 sequences over 128000 tokens: 26 us (2.4 TB/s): a chain of five dependent reads before the rows,
// two meetings of a cluster behind them.
#include <algorithm>

#include "attn_common.cuh"
#include "tc_common.cuh"

namespace sn {
namespace k {

namespace {

constexpr int WARPS = 8;
using U64 = unsigned long long;

struct VerifyP {
    VerifyArgs a;
    int32_t vocab, piece;  // values a warp's piece, a multiple of 128
    int32_t blocks;        // of a cluster
};

__device__ __forceinline__ uint32_t left(uint32_t v, int n) {  // (shifts by 32 and more, or less than 0: nothing is left)
    uint32_t r;
    asm("shl.b32 %0, %1, %2;" : "=r"(r) : "r"(v), "r"(n));
    return r;
}
__device__ __forceinline__ uint32_t right(uint32_t v, int n) {
    uint32_t r;
    asm("shr.u32 %0, %1, %2;" : "=r"(r) : "r"(v), "r"(n));
    return r;
}
// in whole units of 2^-60; outside [0, 1] the nearer end, NaN 0.  By shifts of the significand, 14 integer operations:
// the conversion to 64 bits is a rare unit's, and two of them an element took 47 us for 64 rows of 128000 pairs.
__device__ __forceinline__ U64 fixed(float v) {
    const uint32_t u = __float_as_uint(fminf(fmaxf(v, 0.0f), 1.0f));
    const uint32_t m = (u & 0x7fffffu) | 0x800000u;
    const int n = (int)(u >> 23) - 90;  // v = m 2^n units (below the normal range: less than one)
    return (U64)(left(m, n - 32) | right(m, 32 - n)) << 32 | (left(m, n) | right(m, -n));
}
__device__ __forceinline__ U64 weight(U64 p, U64 q) { return p > q ? p - q : 0; }
__device__ __forceinline__ U64 sum_warp(U64 v) {
#pragma unroll
    for (int o = 16; o; o /= 2) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

// a lane's E neighbours of both rows from i on (beyond `end`: zeros), as they lie there and their weights
template <typename T, int E>
struct alignas(E * sizeof(T)) Some {
    T v[E];
};
template <typename T, int E>
__device__ __forceinline__ Some<T, E> load_some(const T *p, int i, int end) {
    if (i + E <= end) return *reinterpret_cast<const Some<T, E> *>(p + i);
    Some<T, E> r;
#pragma unroll
    for (int j = 0; j < E; ++j) r.v[j] = i + j < end ? p[i + j] : cvt<T>(0.0f);
    return r;
}
template <typename T, int E>
__device__ __forceinline__ U64 sum_some(const Some<T, E> &x, const Some<T, E> &z, bool pair, U64 (&w)[E]) {
    U64 sum = 0;
#pragma unroll
    for (int j = 0; j < E; ++j) {
        w[j] = fixed(ldf(x.v + j));
        if (pair) w[j] = weight(w[j], fixed(ldf(z.v + j)));
        sum += w[j];
    }
    return sum;
}
// a lane's weights of [begin, end), the warp's next to one another; ONCE loads of each under way
template <typename T, int E>
__device__ __forceinline__ U64 sum_range(const T *p, const T *q, int begin, int end, int lane) {
    constexpr int STEP = 32 * E, ONCE = E == 8 ? 2 : 4;
    U64 sum = 0, w[E];
    int i = begin;
#pragma unroll 1
    for (; i + ONCE * STEP <= end; i += ONCE * STEP) {
        Some<T, E> x[ONCE], z[ONCE];
#pragma unroll
        for (int k = 0; k < ONCE; ++k) {
            x[k] = *reinterpret_cast<const Some<T, E> *>(p + i + k * STEP + lane * E);
            if (q) z[k] = *reinterpret_cast<const Some<T, E> *>(q + i + k * STEP + lane * E);
        }
#pragma unroll
        for (int k = 0; k < ONCE; ++k) sum += sum_some<T, E>(x[k], z[k], q != nullptr, w);
    }
#pragma unroll 1
    for (; i < end; i += STEP) {
        const Some<T, E> x = load_some<T, E>(p, i + lane * E, end), z = q ? load_some<T, E>(q, i + lane * E, end) : x;
        sum += sum_some<T, E>(x, z, q != nullptr, w);
    }
    return sum;
}

template <typename T, int E>  // E: values of a 16-byte load, 1 where rows are not aligned to it
__global__ void __launch_bounds__(32 * WARPS) verify_kernel(const __grid_constant__ VerifyP p) {
    __shared__ U64 sums[WARPS], parts[WARPS], total_sh, all_sh[8];
    __shared__ int first_sh;
    griddep_launch();
    griddep_wait();
    const int rank = blockIdx.x % p.blocks, b = blockIdx.x / p.blocks;
    const int tid = threadIdx.x, lane = tid % 32, warp = tid / 32;
    const VerifyArgs &a = p.a;
    const Seq s = sequence(a.q, b);
    const int n = (int)min((int64_t)s.len, a.q.max_len);
    const T *target = static_cast<const T *>(a.target) + (s.first + b) * a.ldt;
    const T *draft = static_cast<const T *>(a.draft) + s.first * a.ldd;
    if (tid == 0) first_sh = n;
    __syncthreads();
    for (int i = tid; i < n; i += 32 * WARPS) {
        const int x = a.drafted[s.first + i];
        bool ok = false;
        if (x >= 0 && x < p.vocab) {
            // the product of two fp32 values is exact in fp64
            const float pt = fminf(fmaxf(ldf(target + i * a.ldt + x), 0.0f), 1.0f), pd = fminf(fmaxf(ldf(draft + i * a.ldd + x), 0.0f), 1.0f);
            ok = (double)a.accept[s.first + i] * (double)pd < (double)pt;
        }
        if (!ok) atomicMin(&first_sh, i);
    }
    __syncthreads();
    const int count = first_sh;
    int32_t *out = a.out + (int64_t)b * (a.q.max_len + 1);
    if (rank == 0) {
        for (int64_t i = tid; i <= a.q.max_len; i += 32 * WARPS)
            if (i != count) out[i] = i < count ? a.drafted[s.first + i] : -1;
        if (tid == 0) a.count[b] = count;
    }
    const T *pr = target + count * a.ldt, *qr = count < n ? draft + count * a.ldd : nullptr;
    const int64_t from = ((int64_t)rank * WARPS + warp) * p.piece;
    const int begin = (int)min(from, (int64_t)p.vocab), end = (int)min(from + p.piece, (int64_t)p.vocab);
    constexpr int STEP = 32 * E;
    U64 all;
    while (true) {
        const U64 mine = sum_warp(sum_range<T, E>(pr, qr, begin, end, lane));
        if (lane == 0) sums[warp] = mine;
        __syncthreads();
        if (warp == 0) {
            const U64 t = sum_warp(lane < WARPS ? sums[lane] : 0);
            if (lane == 0) total_sh = t;
        }
        if (p.blocks > 1) {
            tc::cluster_sync_all();
            if (tid < p.blocks) {
                U64 v;
                asm volatile("ld.shared::cluster.u64 %0, [%1];" : "=l"(v) : "r"(tc::mapa(tc::su32(&total_sh), tid)) : "memory");
                all_sh[tid] = v;
            }
            tc::cluster_sync_all();  // (every block has read the others' sums)
        } else {
            if (tid == 0) all_sh[0] = total_sh;
            __syncthreads();
        }
        all = 0;
        for (int i = 0; i < p.blocks; ++i) all += all_sh[i];
        if (all || !qr) break;
        qr = nullptr;  // p >= q nowhere beyond: the target's own row
        __syncthreads();
    }
    // floor(sample * all): the first cumulative sum beyond it.  Its 64 bits of fraction are all of sample
    // from 2^-40 on
    const float u = a.sample[b];
    const U64 frac = u > 0.0f ? (u < 1.0f ? __float2ull_rd(u * 18446744073709551616.0f) : ~0ull) : 0ull;
    const U64 bar = u < 1.0f || !(u == u) ? __umul64hi(frac, all) : all;
    U64 before = 0;
    for (int i = 0; i < rank; ++i) before += all_sh[i];
    if (all <= bar) {  // nothing exceeds it (all weights zero, or sample 1 and more)
        if (rank == 0 && tid == 0) out[count] = p.vocab - 1;
        return;
    }
    if (bar < before || bar - before >= all_sh[rank]) return;
    // the warp whose piece holds it, and its piece in parts for all of the block's
    int has = 0;
    while (has < WARPS - 1 && bar - before >= sums[has]) before += sums[has++];
    const int64_t start = ((int64_t)rank * WARPS + has) * p.piece;
    const int e0 = (int)min(start + p.piece, (int64_t)p.vocab), step = ((p.piece + WARPS - 1) / WARPS + STEP - 1) / STEP * STEP;
    const int b1 = (int)min(start + (int64_t)warp * step, (int64_t)e0), e1 = min(b1 + step, e0);
    const U64 mine = sum_warp(sum_range<T, E>(pr, qr, b1, e1, lane));
    if (lane == 0) parts[warp] = mine;
    __syncthreads();
    for (int i = 0; i < warp; ++i) before += parts[i];
    if (bar < before || bar - before >= parts[warp]) return;
    for (int i = b1; i < e1; i += STEP) {
        const Some<T, E> x = load_some<T, E>(pr, i + lane * E, e1), z = qr ? load_some<T, E>(qr, i + lane * E, e1) : x;
        U64 w[E];
        const U64 own = sum_some<T, E>(x, z, qr != nullptr, w);
        U64 up = own;
#pragma unroll
        for (int o = 1; o < 32; o *= 2) {
            const U64 v = __shfl_up_sync(0xffffffffu, up, o);
            if (lane >= o) up += v;
        }
        const uint32_t beyond = __ballot_sync(0xffffffffu, before + up > bar);
        if (beyond) {
            if (lane == __ffs(beyond) - 1) {
                U64 c = before + up - own;
                int at = 0;
#pragma unroll
                for (int j = 0; j < E; ++j) {
                    c += w[j];
                    at += c <= bar;
                }
                out[count] = i + lane * E + at;
            }
            return;
        }
        before += __shfl_sync(0xffffffffu, up, 31);
    }
}

template <typename T, int E>
cudaError_t launch_verify(VerifyP &p, cudaStream_t st) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(p.a.q.batch * p.blocks));
    cfg.blockDim = dim3(32 * WARPS);
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)p.blocks, attr[1].val.clusterDim.y = 1, attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, verify_kernel<T, E>, p);
}

}  // namespace

cudaError_t verify_draft(int dt, int vocab, const VerifyArgs &a, cudaStream_t st) {
    VerifyP p{a, vocab, 0, 1};
    // as many blocks a sequence as keep a piece of 128 values and more a warp, and the card one to two waves
    while (p.blocks < 8 && p.blocks * WARPS * 128 < vocab && (int64_t)a.q.batch * p.blocks < 4LL * num_sms()) p.blocks *= 2;
    const int warps = p.blocks * WARPS;
    p.piece = ((vocab + warps - 1) / warps + 127) / 128 * 128;
    const int64_t es = dt == SN_F32 ? 4 : 2;
    const bool vec = reinterpret_cast<uintptr_t>(a.target) % 16 == 0 && reinterpret_cast<uintptr_t>(a.draft) % 16 == 0 &&
                     a.ldt * es % 16 == 0 && a.ldd * es % 16 == 0;
    SN_DT_SWITCH(dt, T, {
        if (vec) return launch_verify<T, 16 / sizeof(T)>(p, st);
        return launch_verify<T, 1>(p, st);
    })
    return cudaSuccess;
}

}  // namespace k
}  // namespace sn
