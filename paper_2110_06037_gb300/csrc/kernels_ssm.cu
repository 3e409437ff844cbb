// Causal convolution, selective scan and token step of a state-space block
// (sn_causal_conv, sn_ssm_scan, sn_ssm_step in include/sn.h).
#include <algorithm>

#include "ssm_common.cuh"

namespace sn {
namespace k {

namespace {

constexpr int MAX_W = 8;

// ------------------------------------------------------------- convolution
// A thread takes V neighbouring channels (four where rows and weights allow)
// over a run of tokens, its weights and the last W - 1 inputs in registers: each
// input is read once, and the W - 1 before the run once more (from L2).  The run is
// as long as one wave of blocks needs it to be, so that weights are loaded once for
// as many tokens as can be.  Bound by memory: 8192 x 4352 bf16, width 4, silu: 26 us,
// 5500 GB/s (81% of a copy's).
constexpr int CONV_THREADS = 128, CONV_BLOCKS = 5;  // blocks on a multiprocessor (4: 32 us, 6: 29)
template <typename T, int W, int V>
__global__ void __launch_bounds__(CONV_THREADS, CONV_BLOCKS)
    causal_conv_kernel(SeqArgs q, const T *__restrict__ x, int64_t ldx, T *__restrict__ y, int64_t ldy, T *kept,
                       const float *__restrict__ w, const float *__restrict__ bias, int C, int act, int len) {
    griddep_launch();
    griddep_wait();
    const uint32_t cg = (uint32_t)(C / V), id = blockIdx.x * CONV_THREADS + threadIdx.x;  // (V divides C)
    const uint32_t run = id / cg;
    const int c0 = (int)(id - run * cg) * V;
    const Seq s = sequence(q, blockIdx.y);
    const int64_t t0 = (int64_t)run * len;
    if (t0 >= s.len) return;
    struct alignas(sizeof(T) * V) Piece {
        T v[V];
    };
    // Two channels a register pair where there are two (arithmetic of single values: 41 us)
    constexpr bool PAIRS = V % 2 == 0;
    using L = typename std::conditional<PAIRS, F2, float>::type;
    constexpr int VL = PAIRS ? V / 2 : V;
    float wt[V * W], b[V];
    L h[W][VL];  // h[j]: the input j + 1 - W tokens from the present one
    auto unpack = [](const Piece &p, L(&to)[VL], bool have) {
#pragma unroll
        for (int v = 0; v < VL; ++v) {
            if constexpr (PAIRS) to[v] = have ? f2(ldf(p.v + 2 * v), ldf(p.v + 2 * v + 1)) : f2(0.0f, 0.0f);
            else to[v] = have ? ldf(p.v + v) : 0.0f;
        }
    };
    if constexpr (V % 4 == 0) {
#pragma unroll
        for (int i = 0; i < V * W / 4; ++i)
            *reinterpret_cast<float4 *>(wt + 4 * i) = __ldg(reinterpret_cast<const float4 *>(w + (int64_t)c0 * W) + i);
#pragma unroll
        for (int i = 0; i < V / 4; ++i)
            *reinterpret_cast<float4 *>(b + 4 * i) =
                bias ? __ldg(reinterpret_cast<const float4 *>(bias + c0) + i) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    } else {
#pragma unroll
        for (int i = 0; i < V * W; ++i) wt[i] = w[(int64_t)c0 * W + i];
#pragma unroll
        for (int v = 0; v < V; ++v) b[v] = bias ? bias[c0 + v] : 0.0f;
    }
    L wl[VL][W], bl[VL];
#pragma unroll
    for (int v = 0; v < VL; ++v) {
        if constexpr (PAIRS) bl[v] = f2(b[2 * v], b[2 * v + 1]);
        else bl[v] = b[v];
#pragma unroll
        for (int j = 0; j < W; ++j) {
            if constexpr (PAIRS) wl[v][j] = f2(wt[2 * v * W + j], wt[(2 * v + 1) * W + j]);
            else wl[v][j] = wt[v * W + j];
        }
    }
    const T *xr = x + (s.first + t0) * ldx + c0;
    T *yr = y + (s.first + t0) * ldy + c0;
    T *kp = kept && s.slot >= 0 ? kept + (int64_t)s.slot * W * C + c0 : nullptr;
#pragma unroll
    for (int j = 1; j < W; ++j) {  // inputs before the run
        const int back = W - j;
        Piece p;
        bool have = true;
        if (t0 >= back) p = *reinterpret_cast<const Piece *>(xr - back * ldx);
        else if (kp && s.pos + t0 >= back) p = *reinterpret_cast<const Piece *>(kp + (int64_t)((s.pos + t0 - back) % W) * C);
        else have = false;
        unpack(p, h[j], have);
    }
    const int n = (int)min((int64_t)len, s.len - t0);
    // Four tokens at once.  The inputs of the eight next are on their way into the
    // thread's own places of shared memory (pieces of 8 or 16 bytes, else registers,
    // which let fewer threads run: 39 us; sixteen ahead 27).
    constexpr int U = 4;
    constexpr bool RING = sizeof(Piece) >= 8;
    constexpr int D = 2 * U;
    __shared__ Piece ring[RING ? D : 1][CONV_THREADS];
    Piece raw[2][U];
    auto ahead = [&](Piece(&in)[U], int t) {  // tokens t to t + 3, at xr
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (t + u < n) {
                if constexpr (RING) {
                    const uint32_t to = (uint32_t)__cvta_generic_to_shared(&ring[(t + u) % D][threadIdx.x]);
                    asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(to), "l"(xr + u * ldx), "n"(sizeof(Piece)) : "memory");
                } else {
                    in[u] = *reinterpret_cast<const Piece *>(xr + u * ldx);
                }
            }
        }
        if constexpr (RING) asm volatile("cp.async.commit_group;" ::: "memory");
        xr += U * ldx;
    };
#pragma unroll
    for (int t = 0; t < D; t += U) ahead(raw[t / U % 2], t);
    auto tokens = [&](Piece(&in)[U], int t) {
        if constexpr (RING) {
            asm volatile("cp.async.wait_group %0;" ::"n"(D / U - 1) : "memory");
#pragma unroll
            for (int u = 0; u < U; ++u) in[u] = ring[(t + u) % D][threadIdx.x];
        }
        L win[W - 1 + U][VL];  // inputs t + 1 - W to t + U - 1
#pragma unroll
        for (int j = 0; j + 1 < W; ++j)
#pragma unroll
            for (int v = 0; v < VL; ++v) win[j][v] = h[j + 1][v];
#pragma unroll
        for (int u = 0; u < U; ++u) unpack(in[u], win[W - 1 + u], true);
        ahead(in, t + D);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (t + u < n) {
                L a[VL];
#pragma unroll
                for (int v = 0; v < VL; ++v) {
                    a[v] = bl[v];
#pragma unroll
                    for (int j = 0; j < W; ++j) {
                        if constexpr (PAIRS) a[v] = fma_2(wl[v][j], win[u + j][v], a[v]);
                        else a[v] = fmaf(wl[v][j], win[u + j][v], a[v]);
                    }
                }
                if (act) {
#pragma unroll
                    for (int v = 0; v < VL; ++v) {
                        if constexpr (PAIRS) a[v] = silu_2(a[v]);
                        else a[v] = silu(a[v]);
                    }
                }
                Piece out;
#pragma unroll
                for (int v = 0; v < VL; ++v) {
                    if constexpr (PAIRS) {
                        const float2 f = floats(a[v]);
                        out.v[2 * v] = cvt<T>(f.x), out.v[2 * v + 1] = cvt<T>(f.y);
                    } else {
                        out.v[v] = cvt<T>(a[v]);
                    }
                }
                *reinterpret_cast<Piece *>(yr) = out;
            }
            yr += ldy;
        }
#pragma unroll
        for (int j = 1; j < W; ++j)
#pragma unroll
            for (int v = 0; v < VL; ++v) h[j][v] = win[U - 1 + j][v];
    };
    for (int t = 0; t < n; t += 2 * U) {
        tokens(raw[0], t);
        tokens(raw[1], t + U);
    }
    // The thread of the first run also leaves the last W inputs behind: it alone
    // has read the kept ones of its channels.
    if (t0 == 0 && kp) {
        for (int t = max(0, s.len - W); t < s.len; ++t)
            *reinterpret_cast<Piece *>(kp + (int64_t)((s.pos + t) % W) * C) =
                *reinterpret_cast<const Piece *>(x + (s.first + t) * ldx + c0);
    }
}

template <typename T, int W>
cudaError_t launch_conv(const SeqArgs &q, const T *x, int64_t ldx, T *y, int64_t ldy, T *kept, const float *w,
                        const float *bias, int C, int act, cudaStream_t st) {
    constexpr int V = 4;  // (eight 16-bit channels would need twice the registers)
    auto at = [](const void *p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; };
    constexpr size_t n = V * sizeof(T);
    const bool vec = C % V == 0 && ldx % V == 0 && ldy % V == 0 && at(x, n) && at(y, n) && at(kept, n) && at(w, 16) && at(bias, 16);
    // Runs of 8 to 256 tokens (a run's start has up to W - 1 = 7 tokens before it in
    // its sequence), as long as the blocks fill one wave.
    const int64_t groups = vec ? C / V : C, threads = (int64_t)num_sms() * CONV_BLOCKS * CONV_THREADS;
    int64_t len = (q.tokens * groups + threads - 1) / threads;
    len = len < 8 ? 8 : len > 256 ? 256 : (len + 3) / 4 * 4;
    const int64_t blocks = ((q.max_len + len - 1) / len * groups + CONV_THREADS - 1) / CONV_THREADS;
    if (blocks > (int64_t)UINT32_MAX / CONV_THREADS) return cudaErrorInvalidValue;
    const dim3 grid((unsigned)blocks, (unsigned)q.batch);
    if (vec)
        return launch_pdl(causal_conv_kernel<T, W, V>, grid, dim3(CONV_THREADS), 0, st, q, x, ldx, y, ldy, kept, w, bias, C, act, (int)len);
    return launch_pdl(causal_conv_kernel<T, W, 1>, grid, dim3(CONV_THREADS), 0, st, q, x, ldx, y, ldy, kept, w, bias, C, act, (int)len);
}

template <typename T>
cudaError_t conv_width(int W, const SeqArgs &q, const T *x, int64_t ldx, T *y, int64_t ldy, T *kept, const float *w,
                       const float *bias, int C, int act, cudaStream_t st) {
    switch (W) {
#define SN_CASE(N) case N: return launch_conv<T, N>(q, x, ldx, y, ldy, kept, w, bias, C, act, st);
        SN_CASE(1) SN_CASE(2) SN_CASE(3) SN_CASE(4) SN_CASE(5) SN_CASE(6) SN_CASE(7) SN_CASE(8)
#undef SN_CASE
    }
    return cudaErrorInvalidValue;
}

// --------------------------------------------------------------------- scan
// The recurrence itself in fp32.  A block takes 32 rows of one head's state and a
// segment of one sequence; 8 lanes share a row, each with NL of its values in
// registers, lane l the float4s l, l + 8, ... of the row.  Inputs come in runs of RT
// tokens through shared memory, the next run's loads in flight meanwhile; four
// tokens' sums are exchanged together.  What bounds it is the chain of a row's
// tokens, so few rows are spread over segments of the sequence: a first pass makes
// every segment's state from nothing, the second starts from the joined ones.
// Six sequences, 1030 tokens the longest, 6 heads of 48 x 40: in one piece 256 us, cut
// all alike 45, each by its own length 36, the blocks with work first 33; the two
// passes' latencies are what is left.  (Segments of 32 tokens: 31, but 98 for 61 for one
// sequence of 2048 tokens and 4 heads of 64 x 128, whose segments are joined longer.)
constexpr int RT = 16, SEG_MIN = 64;  // tokens of a run, and of a segment at least

struct RecP {
    SsmP s;
    int32_t segs, step;   // segments of a sequence at most, tokens of a segment at least
    float *part, *total;  // [tokens / step][H][P][N] states: before segment 0, then after segment j; [tokens / step][H]: sums of d a
};
// segments of one sequence, and the place of the first of their states: a sequence of two and more
// has as many as it has steps, or fewer, so that those of the sequences before it end there
__device__ __forceinline__ int rec_own(int len, int most, int step) { return max(1, min(most, len / step)); }
__device__ __forceinline__ int64_t rec_first(const Seq &s, int step) { return s.first / step; }
__device__ __forceinline__ int2 rec_segment(int len, int segs, int g) {  // tokens [first, last), whole runs
    const int runs = (len + RT - 1) / RT;
    return make_int2(min(len, (int)((int64_t)runs * g / segs) * RT), min(len, (int)((int64_t)runs * (g + 1) / segs) * RT));
}

// FULL: the outputs; otherwise a segment's state from nothing (segment 0: from s_in)
template <typename T, int NL, bool FULL>
__global__ void __launch_bounds__(256) ssm_scan_rec_kernel(const __grid_constant__ RecP p, const T *__restrict__ xbc,
                                                           const T *__restrict__ dtv, T *__restrict__ y) {
    constexpr int NPAD = NL * 8, E = RT * NPAD / 256, EX = RT * 32 / 256;  // values of B (and C), and of x, a thread loads
    __shared__ __align__(16) float sb[RT][NPAD], sc[FULL ? RT : 1][NPAD];
    __shared__ float sx[RT][32], sy[FULL ? RT : 1][32], sd[RT], sda[RT];
    griddep_launch();
    griddep_wait();
    const SsmP &q = p.s;
    const int pblocks = (q.P + 31) / 32, blocks = q.H * pblocks, tid = threadIdx.x, l = tid % 8;
    const Place at = place_of(q.q, p.segs == 1, [&](int len) { return rec_own(len, p.segs, p.step) - (FULL ? 0 : 1); }, blocks, blockIdx.x);
    if (at.b < 0) return;
    const int b = at.b, seg = at.seg, head = at.block / pblocks, p0 = at.block % pblocks * 32, row = p0 + tid / 8;
    const Seq s = sequence(q.q, b);
    const int segs = rec_own(s.len, p.segs, p.step);
    const int2 tok = rec_segment(s.len, segs, seg);
    const int grp = head / (q.H / q.G), np = min(32, q.P - p0);
    const float a = q.a[head], dskip = q.d ? q.d[head] : 0.0f, dtb = q.dt_bias ? q.dt_bias[head] : 0.0f;
    const int64_t part0 = rec_first(s, p.step) * q.H + head, srow = s.slot >= 0 ? (((int64_t)s.slot * q.H + head) * q.P + row) * q.N : -1;
    auto state_at = [&](int j) { return p.part + ((part0 + (int64_t)j * q.H) * q.P + row) * q.N; };
    float st[NL];
    auto value = [&](int i) { return ((i / 4) * 8 + l) * 4 + i % 4; };
#pragma unroll
    for (int i = 0; i < NL; ++i) {
        const int n = value(i);
        st[i] = 0.0f;
        if (row >= q.P || n >= q.N) continue;
        if (FULL && segs > 1) st[i] = state_at(seg > 0 ? 1 : 0)[n];
        else if (seg == 0 && q.s_in && srow >= 0) st[i] = q.s_in[srow + n];
    }
    if (FULL) {
#pragma unroll 4
        for (int j = 1; j < seg; ++j) {
            const float e = expf(p.total[part0 + (int64_t)j * q.H]);
#pragma unroll
            for (int i = 0; i < NL; ++i)
                if (row < q.P && value(i) < q.N) st[i] = fmaf(st[i], e, state_at(j + 1)[value(i)]);
        }
    } else if (seg == 0) {  // the second pass may store over s_in: it reads this copy
#pragma unroll
        for (int i = 0; i < NL; ++i)
            if (row < q.P && value(i) < q.N) state_at(0)[value(i)] = st[i];
    }
    // a run's inputs, in registers until the run before has been worked on
    T nb[E], ncv[FULL ? E : 1], nx[EX];
    float nd = 0.0f, sum = 0.0f;  // (threads 0 to RT - 1: a token's step; sum of steps)
    auto fetch = [&](int t0) {
        const int nt = min(RT, tok.y - t0);
        if (nt <= 0) return;
        const T *r0 = xbc + (s.first + t0) * q.ldx;
#pragma unroll
        for (int i = 0; i < E; ++i) {
            const int e = tid + i * 256, t = e / NPAD, n = e % NPAD;
            if (t < nt && n < q.N) {
                const T *r = r0 + (int64_t)t * q.ldx + q.H * q.P + grp * q.N + n;
                nb[i] = *r;
                if (FULL) ncv[i] = r[q.G * q.N];
            }
        }
#pragma unroll
        for (int i = 0; i < EX; ++i) {
            const int e = tid + i * 256, t = e / 32, c = e % 32;
            if (t < nt && c < np) nx[i] = r0[(int64_t)t * q.ldx + head * q.P + p0 + c];
        }
        if (tid < nt) nd = softplus(ldf(dtv + (s.first + t0 + tid) * q.lddt + head) + dtb);
    };
    fetch(tok.x);
    for (int t0 = tok.x; t0 < tok.y; t0 += RT) {
        const int nt = min(RT, tok.y - t0);
        __syncthreads();
#pragma unroll
        for (int i = 0; i < E; ++i) {
            const int e = tid + i * 256, t = e / NPAD, n = e % NPAD;
            const bool in = t < nt && n < q.N;
            sb[t][n] = in ? ldf(nb + i) : 0.0f;
            if (FULL) sc[t][n] = in ? ldf(ncv + i) : 0.0f;
        }
#pragma unroll
        for (int i = 0; i < EX; ++i) {
            const int e = tid + i * 256, t = e / 32, c = e % 32;
            sx[t][c] = t < nt && c < np ? ldf(nx + i) : 0.0f;
        }
        if (tid < RT) {  // (behind the segment's end: a step of 0)
            sd[tid] = tid < nt ? nd : 0.0f;
            sda[tid] = tid < nt ? expf(nd * a) : 1.0f;
            sum += tid < nt ? nd * a : 0.0f;
        }
        __syncthreads();
        fetch(t0 + RT);
        for (int t = 0; t < nt; t += 4) {  // (RT is a multiple of 4: what lies behind the end changes nothing)
            float acc[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const float da = sda[t + u], dx = sd[t + u] * sx[t + u][tid / 8];
                float4 c4 = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
                for (int i = 0; i < NL / 4; ++i) {
                    const float4 bv = *reinterpret_cast<const float4 *>(&sb[t + u][(i * 8 + l) * 4]);
                    st[4 * i] = fmaf(st[4 * i], da, dx * bv.x);
                    st[4 * i + 1] = fmaf(st[4 * i + 1], da, dx * bv.y);
                    st[4 * i + 2] = fmaf(st[4 * i + 2], da, dx * bv.z);
                    st[4 * i + 3] = fmaf(st[4 * i + 3], da, dx * bv.w);
                    if (FULL) {
                        const float4 cv = *reinterpret_cast<const float4 *>(&sc[t + u][(i * 8 + l) * 4]);
                        c4.x = fmaf(st[4 * i], cv.x, c4.x), c4.y = fmaf(st[4 * i + 1], cv.y, c4.y);
                        c4.z = fmaf(st[4 * i + 2], cv.z, c4.z), c4.w = fmaf(st[4 * i + 3], cv.w, c4.w);
                    }
                }
                acc[u] = (c4.x + c4.y) + (c4.z + c4.w);
            }
            if (FULL) {
                // four tokens' sums over eight lanes in four exchanges: lanes 0 and 1 of each pair end with one token's
                const bool up = l & 4, up2 = l & 2;
                float a0 = up ? acc[2] : acc[0], a1 = up ? acc[3] : acc[1];
                a0 += __shfl_xor_sync(0xffffffffu, up ? acc[0] : acc[2], 4);
                a1 += __shfl_xor_sync(0xffffffffu, up ? acc[1] : acc[3], 4);
                float v = up2 ? a1 : a0;
                v += __shfl_xor_sync(0xffffffffu, up2 ? a0 : a1, 2);
                v += __shfl_xor_sync(0xffffffffu, v, 1);
                const int tt = t + l / 2;
                if (l % 2 == 0) sy[tt][tid / 8] = fmaf(dskip, sx[tt][tid / 8], v);
            }
        }
        if (FULL) {
            __syncthreads();
#pragma unroll
            for (int i = 0; i < EX; ++i) {
                const int e = tid + i * 256, t = e / 32, c = e % 32;
                if (t < nt && c < np) stf(y + (s.first + t0 + t) * q.ldy + head * q.P + p0 + c, sy[t][c]);
            }
        }
    }
    float *out = FULL ? (seg == segs - 1 && q.s_out && srow >= 0 ? q.s_out + srow : nullptr) : state_at(seg + 1);
    if (out && row < q.P) {
#pragma unroll
        for (int i = 0; i < NL; ++i)
            if (value(i) < q.N) out[value(i)] = st[i];
    }
    if (!FULL && p0 == 0 && tid < 32) {  // threads 0 to RT - 1 hold the parts of the sum
        if (tid >= RT) sum = 0.0f;
#pragma unroll
        for (int o = RT / 2; o; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
        if (tid == 0) p.total[part0 + (int64_t)seg * q.H] = sum;
    }
}

// Segments: as many as give three blocks an SM for the tokens there are, of SEG_MIN tokens at least
int rec_segments(const SsmP &p) {
    const int64_t full = (p.q.tokens + p.q.max_len - 1) / std::max<int64_t>(p.q.max_len, 1);  // sequences, counted by length
    const int64_t blocks = std::max<int64_t>(full * p.H * ((p.P + 31) / 32), 1);
    return (int)std::max<int64_t>(1, std::min<int64_t>({3LL * num_sms() / blocks, 64, p.q.max_len / SEG_MIN}));
}
int64_t rec_step(const SsmP &p, int64_t segs) { return std::max<int64_t>(SEG_MIN, p.q.max_len / segs); }
int64_t rec_workspace(const SsmP &p) {
    const int64_t segs = rec_segments(p);
    return segs > 1 ? (p.q.tokens / rec_step(p, segs) * p.H * ((int64_t)p.P * p.N + 1) * 4 + 255) / 256 * 256 : 0;
}

template <typename T, int NL>
cudaError_t launch_rec(const RecP &p, const T *xbc, const T *dtv, T *y, cudaStream_t st) {
    const int64_t heads = (int64_t)p.s.H * ((p.s.P + 31) / 32), steps = p.s.q.tokens / p.step, batch = p.s.q.batch;
    // segments that there can be: one of each sequence, and one more for each step
    const int64_t most = std::min(batch * p.segs, batch + steps), states = std::min(batch * (p.segs - 1), steps);
    if (heads * most > INT32_MAX) return cudaErrorInvalidValue;
    if (states > 0) {
        const cudaError_t e = launch_pdl(ssm_scan_rec_kernel<T, NL, false>, dim3((unsigned)(heads * states)), dim3(256), 0, st, p, xbc, dtv, y);
        if (e != cudaSuccess) return e;
    }
    return launch_pdl(ssm_scan_rec_kernel<T, NL, true>, dim3((unsigned)(heads * most)), dim3(256), 0, st, p, xbc, dtv, y);
}

template <typename T>
cudaError_t launch_scan(const SsmP &s, const T *xbc, const T *dtv, T *y, void *work, cudaStream_t st) {
    RecP p{s, s.q.tokens ? rec_segments(s) : 1, 0, static_cast<float *>(work), nullptr};
    p.step = (int32_t)rec_step(s, p.segs);
    p.total = p.part + s.q.tokens / p.step * s.H * s.P * s.N;
    if (s.N <= 32) return launch_rec<T, 4>(p, xbc, dtv, y, st);
    if (s.N <= 64) return launch_rec<T, 8>(p, xbc, dtv, y, st);
    if (s.N <= 128) return launch_rec<T, 16>(p, xbc, dtv, y, st);
    return launch_rec<T, 32>(p, xbc, dtv, y, st);
}

// --------------------------------------------------------------------- step
// One token: the state is read, updated and written once.  The state's rows of the
// heads of a group lie one behind the other and share B and C: a block takes `rows`
// of them.  A warp's lanes lie along a row (VEC values a piece, VPL pieces a lane,
// `lpr` lanes a row), RU rows per lane at once and the next RU in flight.  The
// convolution of the block's own channels and of the group's B and C is done again
// by every block of the group (its inputs come from L2); each channel's new input is
// stored by one of them, at a place none of them reads.  Bound by memory: 128 sequences
// of 64 heads of 64 x 128: 89 us, 6100 GB/s, 90% of a copy's (eight rows a lane at once were a fifth slower).
constexpr int STEP_ROWS = 256;  // most rows of a block
// W: the convolution's width, or 0: p.W
template <typename T, int VEC, int VPL, int W>
__global__ void __launch_bounds__(256) ssm_step_kernel(const __grid_constant__ SsmP p, const T *__restrict__ xbc,
                                                       const T *__restrict__ dtv, T *kept, T *__restrict__ y, int rows,
                                                       int lpr) {
    __shared__ __align__(16) float sx[STEP_ROWS], sbc[2][256];  // x of the block's rows; B, C
    __shared__ float2 sd[STEP_ROWS];                            // of the block's rows: time step, decay
    constexpr int RU = VPL * VEC >= 8 ? 2 : 4;
    griddep_launch();
    griddep_wait();
    const int b = blockIdx.z, grp = blockIdx.y, tid = threadIdx.x, hpg = p.H / p.G;
    const int r0 = grp * hpg * p.P + blockIdx.x * rows, nr = min(rows, hpg * p.P - (int)blockIdx.x * rows);
    const int slot = p.q.slots ? p.q.slots[b] : b;
    T *yr = y + (int64_t)b * p.ldy + r0;
    if (slot < 0 || slot >= p.q.n_slots) {  // no slot: nothing to continue
        for (int i = tid; i < nr; i += 256) stf(yr + i, 0.0f);
        return;
    }
    const int pos = max(p.q.pos ? p.q.pos[b] : 0, 0);
    const int sub = tid % lpr, first = tid / lpr, rpb = 256 / lpr;  // rows that the block handles at once
    const int64_t base = ((int64_t)slot * p.H * p.P + r0) * p.N + sub * VEC;
    const int nv = p.N / VEC;  // (VEC divides N)
    struct alignas(4 * VEC) Piece {
        float v[VEC];
    };
    Piece h[RU][VPL];
    auto load = [&](Piece(&d)[RU][VPL], int r) {
#pragma unroll
        for (int u = 0; u < RU; ++u)
#pragma unroll
            for (int i = 0; i < VPL; ++i) {
                if (p.s_in && r + u * rpb < nr && sub + i * lpr < nv)
                    d[u][i] = *reinterpret_cast<const Piece *>(p.s_in + base + (int64_t)(r + u * rpb) * p.N + i * lpr * VEC);
                else
#pragma unroll
                    for (int e = 0; e < VEC; ++e) d[u][i].v[e] = 0.0f;
            }
    };
    load(h, first);  // in flight before the convolution
    for (int i = tid; i < nr; i += 256) {
        const int head = (r0 + i) / p.P;
        const float d = softplus(ldf(dtv + (int64_t)b * p.lddt + head) + (p.dt_bias ? p.dt_bias[head] : 0.0f));
        sd[i] = make_float2(d, expf(d * p.a[head]));
    }
    const int C = p.H * p.P + 2 * p.G * p.N, width = W ? W : p.W;
    const T *xr = xbc + (int64_t)b * p.ldx;
    T *kb = kept + (int64_t)slot * width * C;
    int64_t at[W ? W : MAX_W];  // of tap j's kept input; -1: before the sequence's first
#pragma unroll
    for (int j = 0; j < (W ? W : MAX_W); ++j) {
        const int back = width - 1 - j;
        at[j] = back >= 0 && pos >= back ? (int64_t)((pos - back) % width) * C : -1;
    }
    const int64_t at_new = (int64_t)(pos % width) * C;
    for (int e = tid; e < nr + 2 * p.N; e += 256) {
        const int n = e - nr;
        const int c = n < 0 ? r0 + e : p.H * p.P + (n < p.N ? grp * p.N + n : (p.G + grp - 1) * p.N + n);
        const float *w = p.conv_w + (int64_t)c * width;
        const T now = xr[c];
        T old[W ? W : MAX_W];
#pragma unroll
        for (int j = 0; j < (W ? W : MAX_W) - 1; ++j)
            if (at[j] >= 0 && j + 1 < width) old[j] = kb[at[j] + c];
        float acc = p.conv_b ? p.conv_b[c] : 0.0f;
#pragma unroll
        for (int j = 0; j < (W ? W : MAX_W) - 1; ++j)
            if (at[j] >= 0 && j + 1 < width) acc = fmaf(w[j], ldf(old + j), acc);
        acc = silu(fmaf(w[width - 1], ldf(&now), acc));
        if (n < 0) sx[e] = acc;
        else sbc[n >= p.N][n >= p.N ? n - p.N : n] = acc;
        if (n < 0 || blockIdx.x == 0) kb[at_new + c] = now;
    }
    __syncthreads();
    Piece bv[VPL], cv[VPL];
#pragma unroll
    for (int i = 0; i < VPL; ++i)
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
            const int n = (sub + i * lpr) * VEC + e;
            bv[i].v[e] = n < p.N ? sbc[0][n] : 0.0f;
            cv[i].v[e] = n < p.N ? sbc[1][n] : 0.0f;
        }
    for (int at_row = first; at_row - first < nr; at_row += RU * rpb) {  // (the same trips for every thread)
        Piece nx[RU][VPL];
        load(nx, at_row + RU * rpb);
        float acc[RU];
#pragma unroll
        for (int u = 0; u < RU; ++u) {
            const int r = at_row + u * rpb;
            const bool in = r < nr;
            const float2 dd = in ? sd[r] : make_float2(0.0f, 0.0f);
            const float dx = in ? dd.x * sx[r] : 0.0f;
            acc[u] = 0.0f;
#pragma unroll
            for (int i = 0; i < VPL; ++i) {
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    h[u][i].v[e] = fmaf(h[u][i].v[e], dd.y, dx * bv[i].v[e]);
                    acc[u] = fmaf(h[u][i].v[e], cv[i].v[e], acc[u]);
                }
                if (p.s_out && in && sub + i * lpr < nv)
                    *reinterpret_cast<Piece *>(p.s_out + base + (int64_t)r * p.N + i * lpr * VEC) = h[u][i];
            }
        }
        auto skip = [&](int r) { return p.d ? p.d[(r0 + r) / p.P] * sx[r] : 0.0f; };
        if (RU == 4 && lpr == 32) {
            // four rows' sums in six exchanges: lanes of each quarter end with one row's
            const bool up = sub & 16, up2 = sub & 8;
            float a0 = up ? acc[2 % RU] : acc[0], a1 = up ? acc[3 % RU] : acc[1 % RU];
            a0 += __shfl_xor_sync(0xffffffffu, up ? acc[0] : acc[2 % RU], 16);
            a1 += __shfl_xor_sync(0xffffffffu, up ? acc[1 % RU] : acc[3 % RU], 16);
            float v = up2 ? a1 : a0;
            v += __shfl_xor_sync(0xffffffffu, up2 ? a0 : a1, 8);
            v += __shfl_xor_sync(0xffffffffu, v, 4);
            v += __shfl_xor_sync(0xffffffffu, v, 2);
            v += __shfl_xor_sync(0xffffffffu, v, 1);
            const int r = at_row + (sub / 8) * rpb;
            if (sub % 8 == 0 && r < nr) stf(yr + r, v + skip(r));
        } else {
#pragma unroll
            for (int u = 0; u < RU; ++u) {
                for (int o = lpr / 2; o; o >>= 1) acc[u] += __shfl_xor_sync(0xffffffffu, acc[u], o);
                const int r = at_row + u * rpb;
                if (sub == 0 && r < nr) stf(yr + r, acc[u] + skip(r));
            }
        }
#pragma unroll
        for (int u = 0; u < RU; ++u)
#pragma unroll
            for (int i = 0; i < VPL; ++i) h[u][i] = nx[u][i];
    }
}

template <typename T>
cudaError_t launch_step(const SsmP &p, const T *xbc, const T *dtv, T *kept, T *y, cudaStream_t st) {
    // up to 256 rows a block, fewer (8 at least) until there are two blocks a multiprocessor
    const int grp_rows = p.H / p.G * p.P;
    int rows = STEP_ROWS;
    while (rows > 8 && (int64_t)p.q.batch * p.G * ((grp_rows + rows - 1) / rows) < 2 * num_sms()) rows /= 2;
    const dim3 grid((unsigned)((grp_rows + rows - 1) / rows), (unsigned)p.G, (unsigned)p.q.batch);
    const bool vec = p.N % 4 == 0 && reinterpret_cast<uintptr_t>(p.s_in) % 16 == 0 && reinterpret_cast<uintptr_t>(p.s_out) % 16 == 0;
    const int nv = vec ? p.N / 4 : p.N;
    int lpr = 1;
    while (lpr < 32 && lpr < nv) lpr *= 2;
    const int vpl = (nv + lpr - 1) / lpr;
#define SN_STEP(VEC, VPL)                                                                                              \
    return p.W == 4 ? launch_pdl(ssm_step_kernel<T, VEC, VPL, 4>, grid, dim3(256), 0, st, p, xbc, dtv, kept, y, rows, lpr) \
                    : launch_pdl(ssm_step_kernel<T, VEC, VPL, 0>, grid, dim3(256), 0, st, p, xbc, dtv, kept, y, rows, lpr)
    if (vec) {
        if (vpl == 1) SN_STEP(4, 1);
        SN_STEP(4, 2);
    }
    if (vpl == 1) SN_STEP(1, 1);
    if (vpl <= 4) SN_STEP(1, 4);
    SN_STEP(1, 8);
#undef SN_STEP
}

SsmP ssm_params(const sn_ssm_params &c, const SeqArgs &q, int64_t ldx, int64_t lddt, const float *s_in, float *s_out,
                int64_t ldy) {
    return SsmP{q, c.heads, c.head_dim, c.groups, c.state, c.width, c.a, c.d, c.dt_bias, c.conv_w, c.conv_b,
                ldx, lddt, ldy, s_in, s_out};
}

}  // namespace

cudaError_t causal_conv(int dt, int channels, int width, int act, const float *w, const float *bias, const SeqArgs &q,
                        const void *x, int64_t ldx, void *y, int64_t ldy, void *kept, cudaStream_t st) {
    SN_DT_SWITCH(dt, T, return conv_width<T>(width, q, static_cast<const T *>(x), ldx, static_cast<T *>(y), ldy,
                                             static_cast<T *>(kept), w, bias, channels, act, st))
}

size_t ssm_workspace(const sn_ssm_params &c, int dt, const SeqArgs &q) {
    const SsmP p = ssm_params(c, q, 0, 0, nullptr, nullptr, 0);  // (which of the two it is depends on alignments too)
    const size_t rec = (size_t)rec_workspace(p);
    return dt == SN_BF16 && c.state <= 128 ? std::max(rec, ssm_tc_workspace(p)) : rec;
}

cudaError_t ssm_scan(const sn_ssm_params &c, int dt, const SeqArgs &q, const void *xbc, int64_t ldx, const void *dtv,
                     int64_t lddt, const float *s_in, float *s_out, void *y, int64_t ldy, void *work, cudaStream_t st) {
    const SsmP p = ssm_params(c, q, ldx, lddt, s_in, s_out, ldy);
    if (dt == SN_BF16 && q.tokens && ssm_tc_applies(p, xbc, y))
        return ssm_tc_scan(p, static_cast<const __nv_bfloat16 *>(xbc), static_cast<const __nv_bfloat16 *>(dtv),
                           static_cast<__nv_bfloat16 *>(y), work, st);
    SN_DT_SWITCH(dt, T, return launch_scan<T>(p, static_cast<const T *>(xbc), static_cast<const T *>(dtv),
                                              static_cast<T *>(y), work, st))
}

cudaError_t ssm_step(const sn_ssm_params &c, int dt, const SeqArgs &q, const void *xbc, int64_t ldx, const void *dtv,
                     int64_t lddt, void *kept, const float *s_in, float *s_out, void *y, int64_t ldy, cudaStream_t st) {
    const SsmP p = ssm_params(c, q, ldx, lddt, s_in, s_out, ldy);
    SN_DT_SWITCH(dt, T, return launch_step<T>(p, static_cast<const T *>(xbc), static_cast<const T *>(dtv),
                                              static_cast<T *>(kept), static_cast<T *>(y), st))
}

}  // namespace k
}  // namespace sn
