// Verification of drafted tokens (sn_verify_draft in include/sn.h).
//
// A cluster of 1 to 8 blocks takes a sequence.  Each block finds the first token that is not accepted
// (a load of two probabilities a token); the row behind it is cut into the blocks' and their warps'
// contiguous pieces, whose weights are summed in units of 2^-60, in integers: exact, so that neither the
// cut nor the order matters.  With every block's and warp's sum known, one warp's piece holds the drawn
// index, and that warp goes through it once more (from L2) with running sums.
#include <algorithm>

#include "attn_common.cuh"
#include "tc_common.cuh"

namespace sn {
namespace k {

namespace {

constexpr int WARPS = 16;
using U64 = unsigned long long;

struct VerifyP {
    VerifyArgs a;
    int32_t vocab, piece;  // values a warp's piece, a multiple of 128
    int32_t blocks;        // of a cluster
};

// in units of 2^-60; outside [0, 1] the nearer end, NaN 0
__device__ __forceinline__ U64 fixed(float v) { return __float2ull_rn(fminf(fmaxf(v, 0.0f), 1.0f) * 1152921504606846976.0f); }
__device__ __forceinline__ U64 weight(U64 p, U64 q) { return p > q ? p - q : 0; }
__device__ __forceinline__ U64 sum_warp(U64 v) {
#pragma unroll
    for (int o = 16; o; o /= 2) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

// a lane's E neighbours of both rows from i on (beyond `end`: zeros)
template <typename T, int E>
__device__ __forceinline__ void load_pair(U64 (&w)[E], const T *p, const T *q, int i, int end) {
    alignas(16) T x[E], z[E];
    if constexpr (E * sizeof(T) == 16) {
        if (i + E <= end) {
            *reinterpret_cast<uint4 *>(x) = *reinterpret_cast<const uint4 *>(p + i);
            if (q) *reinterpret_cast<uint4 *>(z) = *reinterpret_cast<const uint4 *>(q + i);
#pragma unroll
            for (int j = 0; j < E; ++j) w[j] = q ? weight(fixed(ldf(x + j)), fixed(ldf(z + j))) : fixed(ldf(x + j));
            return;
        }
    }
#pragma unroll
    for (int j = 0; j < E; ++j)
        w[j] = i + j >= end ? 0 : q ? weight(fixed(ldf(p + i + j)), fixed(ldf(q + i + j))) : fixed(ldf(p + i + j));
}

template <typename T, int E>  // E: values of a 16-byte load, 1 where rows are not aligned to it
__global__ void __launch_bounds__(32 * WARPS) verify_kernel(const __grid_constant__ VerifyP p) {
    __shared__ U64 sums[WARPS], total_sh, all_sh[8];
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
        U64 mine = 0;
#pragma unroll 4
        for (int i = begin; i < end; i += STEP) {
            U64 w[E];
            load_pair<T, E>(w, pr, qr, i + lane * E, end);
#pragma unroll
            for (int j = 0; j < E; ++j) mine += w[j];
        }
        mine = sum_warp(mine);
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
    for (int i = 0; i < warp; ++i) before += sums[i];
    if (bar < before || bar - before >= sums[warp]) return;
    // this warp's piece holds it
    for (int i = begin; i < end; i += STEP) {
        U64 w[E], mine = 0;
        load_pair<T, E>(w, pr, qr, i + lane * E, end);
#pragma unroll
        for (int j = 0; j < E; ++j) mine += w[j];
        U64 up = mine;
#pragma unroll
        for (int o = 1; o < 32; o *= 2) {
            const U64 v = __shfl_up_sync(0xffffffffu, up, o);
            if (lane >= o) up += v;
        }
        const uint32_t beyond = __ballot_sync(0xffffffffu, before + up > bar);
        if (beyond) {
            if (lane == __ffs(beyond) - 1) {
                U64 c = before + up - mine;
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
