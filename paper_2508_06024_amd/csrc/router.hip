// Training operators of the router, for gfx950: the load balance loss with its per-expert counts and
// gradient, and the backward pass of the group gate.
#include "device_common.h"
#include "router.h"

#include <algorithm>

namespace ec2moe {
namespace {

constexpr int kMaxExperts = 256;
constexpr int kMaxGroups = 160;

// names of the timing record (launches outside the layer step)
constexpr const char *kBalanceName = "balance_loss", *kBalanceFinishName = "balance_finish",
                     *kLogitGradName = "gate_logit_grad", *kProductsName = "gate_products",
                     *kDwSumName = "gate_dw_sum";

// ------------------------------------------------------------------ load balance loss
//
// Column sums of probs over the valid tokens and a histogram of the selected experts, by chunks of
// tokens (a workgroup each); a second launch adds the chunks in order, a workgroup per 32 experts, and the last of its
// workgroups to arrive adds their shares of the loss in order. With one chunk the first launch finishes by itself.
// Integer counts are added with LDS atomics: their order changes nothing. Memory-bound (probs once) for long batches;
// short ones are two launches.
constexpr int kBalThreads = 512;
constexpr int kBalMaxChunks = 512;
constexpr int kBalRows = 8;   // rows of a float32 sum, loaded together
constexpr int kBalCols = 32;  // experts of a workgroup of the second launch

int balance_chunks(int n_tokens, int n_experts) {
    const int64_t values = static_cast<int64_t>(n_tokens) * n_experts;
    return static_cast<int>(std::max<int64_t>(1, std::min<int64_t>(kBalMaxChunks, (values + 8191) / 8192)));
}

struct BalancePart {
    double* loss;    // [kMaxExperts / kBalCols] shares of the second launch's workgroups
    uint32_t* done;  // its workgroups that have finished (cleared by the first launch)
    float* p;        // [chunks][M]
    int32_t* c;      // [chunks][M]
    int32_t* n;      // [chunks] valid tokens
};

__host__ __device__ inline BalancePart balance_part(void* ws, int chunks, int M) {
    double* loss = static_cast<double*>(ws);
    uint32_t* done = reinterpret_cast<uint32_t*>(loss + kMaxExperts / kBalCols);
    float* p = reinterpret_cast<float*>(done + 2);
    int32_t* c = reinterpret_cast<int32_t*>(p + static_cast<size_t>(chunks) * M);
    return {loss, done, p, c, c + static_cast<size_t>(chunks) * M};
}

// Expert e of the sum of probabilities p and count c over n valid tokens: writes its outputs, returns its share of the loss.
__device__ __forceinline__ double balance_expert(const BalanceArgs& a, int e, double p, int c, int n) {
    double d = 0.0;
    if (n > 0) d = static_cast<double>(a.coef) * a.n_experts * c / (static_cast<double>(a.top_k) * n * n);
    if (a.counts) a.counts[e] = c;
    if (a.d_probs) a.d_probs[e] = static_cast<float>(d);
    return n > 0 ? d * p : 0.0;
}

// V: consecutive experts a thread loads together
template <int V>
__global__ __launch_bounds__(kBalThreads) void balance_kernel(BalanceArgs a, int chunk) {
    __shared__ double s_sum[kBalThreads * V];
    __shared__ int s_cnt[kMaxExperts];
    __shared__ int s_n;
    __shared__ double s_loss[kMaxExperts];
    const int tid = threadIdx.x, M = a.n_experts, k = a.top_k;
    const int L = (M + V - 1) / V;         // threads per row
    const int RP = kBalThreads / L;        // rows per pass
    const int64_t t0 = static_cast<int64_t>(blockIdx.x) * chunk;
    const int nt = static_cast<int>(max(static_cast<int64_t>(0), min(static_cast<int64_t>(chunk), a.n_tokens - t0)));
    const float* probs = a.probs + t0 * M;
    const int32_t* idx = a.topk_idx + t0 * k;
    const uint8_t* valid = a.valid ? a.valid + t0 : nullptr;
    for (int i = tid; i < kMaxExperts; i += kBalThreads) s_cnt[i] = 0;
    if (tid == 0) s_n = 0;
    __syncthreads();
    const int rs = tid / L, c = (tid % L) * V;
    double sum[V];
#pragma unroll
    for (int v = 0; v < V; ++v) sum[v] = 0.0;
    if (rs < RP) {
        // Eight rows are summed in float32, these sums in float64, so that the error does not grow with the batch. (A token
        // that does not count adds zero, not its value times zero.)
        auto add = [&](int t, float (&run)[V]) {
            const bool ok = !valid || valid[t];
            if constexpr (V == 4) {
                const f32x4 v = *reinterpret_cast<const f32x4*>(probs + static_cast<int64_t>(t) * M + c);
#pragma unroll
                for (int i = 0; i < 4; ++i) run[i] += ok ? v[i] : 0.f;
            } else {
                const float v = probs[static_cast<int64_t>(t) * M + c];
                run[0] += ok ? v : 0.f;
            }
        };
        int t = rs;
        for (; t + (kBalRows - 1) * RP < nt; t += kBalRows * RP) {
            float run[V] = {};
#pragma unroll
            for (int u = 0; u < kBalRows; ++u) add(t + u * RP, run);
#pragma unroll
            for (int v = 0; v < V; ++v) sum[v] += run[v];
        }
        float run[V] = {};
        for (; t < nt; t += RP) add(t, run);
#pragma unroll
        for (int v = 0; v < V; ++v) sum[v] += run[v];
    }
    // a thread keeps its slot of the token: kBalThreads / k tokens a pass
    const int tp = kBalThreads / k, slot = tid % k;
#pragma unroll 4
    for (int t = tid / k; t < nt; t += tp) {
        if (tid / k >= tp) break;
        const int e = idx[static_cast<int64_t>(t) * k + slot];
        if ((!valid || valid[t]) && e >= 0 && e < M) atomicAdd(&s_cnt[e], 1);
    }
    int n = 0;
    if (valid) {
        for (int t = tid; t < nt; t += kBalThreads) n += valid[t] ? 1 : 0;
        if (n) atomicAdd(&s_n, n);
    } else if (tid == 0) {
        s_n = nt;
    }
    if (rs < RP)
#pragma unroll
        for (int v = 0; v < V; ++v) s_sum[rs * L * V + c + v] = sum[v];
    __syncthreads();
    double p = 0.0;
    if (tid < M) {
        double q[4] = {0.0, 0.0, 0.0, 0.0};  // four sums side by side: a float64 addition's latency each
        int r = 0;
        for (; r + 4 <= RP; r += 4)
#pragma unroll
            for (int u = 0; u < 4; ++u) q[u] += s_sum[(r + u) * L * V + tid];
        for (; r < RP; ++r) q[0] += s_sum[r * L * V + tid];
        p = (q[0] + q[1]) + (q[2] + q[3]);
    }
    if (gridDim.x == 1) {
        if (tid < M) s_loss[tid] = balance_expert(a, tid, p, s_cnt[tid], s_n);
        __syncthreads();
        if (tid == 0) {
            double loss = 0.0;
            for (int i = 0; i < M; ++i) loss += s_loss[i];
            a.loss[0] = static_cast<float>(loss);
        }
        return;
    }
    const BalancePart part = balance_part(a.ws, gridDim.x, M);
    if (tid < M) {
        part.p[static_cast<int64_t>(blockIdx.x) * M + tid] = static_cast<float>(p);  // half the traffic of the second launch
        part.c[static_cast<int64_t>(blockIdx.x) * M + tid] = s_cnt[tid];
    }
    if (tid == 0) {
        part.n[blockIdx.x] = s_n;
        if (blockIdx.x == 0) part.done[0] = 0;
    }
}

__global__ __launch_bounds__(1024) void balance_finish_kernel(BalanceArgs a, int chunks) {
    constexpr int SLOTS = 1024 / kBalCols;
    __shared__ double s_p[SLOTS][kBalCols];
    __shared__ int s_c[SLOTS][kBalCols];
    __shared__ int s_n;
    __shared__ double s_loss[kBalCols];
    const int tid = threadIdx.x, M = a.n_experts;
    const int col = tid % kBalCols, slot = tid / kBalCols, e = blockIdx.x * kBalCols + col;
    const BalancePart part = balance_part(a.ws, chunks, M);
    if (tid == 0) s_n = 0;
    __syncthreads();
    double p = 0.0;
    int c = 0, n = 0;
    if (e < M)
#pragma unroll 8
        for (int j = slot; j < chunks; j += SLOTS) {
            p += part.p[static_cast<int64_t>(j) * M + e];
            c += part.c[static_cast<int64_t>(j) * M + e];
        }
    for (int j = tid; j < chunks; j += 1024) n += part.n[j];
    if (n) atomicAdd(&s_n, n);
    s_p[slot][col] = p;
    s_c[slot][col] = c;
    __syncthreads();
    if (slot == 0) {
        for (int j = 1; j < SLOTS; ++j) {
            p += s_p[j][col];
            c += s_c[j][col];
        }
        s_loss[col] = e < M ? balance_expert(a, e, p, c, s_n) : 0.0;
    }
    __syncthreads();
    if (tid != 0) return;
    double loss = 0.0;
    for (int i = 0; i < kBalCols; ++i) loss += s_loss[i];
    if (gridDim.x > 1) {
        __hip_atomic_store(part.loss + blockIdx.x, loss, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        const uint32_t before = __hip_atomic_fetch_add(part.done, 1u, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT);
        if (before + 1 != gridDim.x) return;
        loss = 0.0;
        for (unsigned i = 0; i < gridDim.x; ++i)
            loss += __hip_atomic_load(part.loss + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    a.loss[0] = static_cast<float>(loss);
}

// ------------------------------------------------------------------ gate backward
//
// The gradient D [T][M + K] of the logits (columns: M local, then K group logits) from the probabilities, then
// two products around it: d_x = D W and d_W = D^T X, with the column sums of D for the biases. Both have long
// sides T and d and a short one R = M + K, and move X and d_x once: memory-bound, if the matrix cores are fast
// enough. Float32 ones are not (4 T R d operations: 8192 x 2048, 72 rows: 31 us at their peak, against 13 us for the
// 70 MB), so D is kept as three bfloat16 planes, D = hi + mid + lo up to 2^-24 |D|, whose products with bfloat16 X
// and W are exact and summed in float32. d_x in bfloat16 takes two planes (2^-16 of each term, against 2^-8 for its
// rounding). Float32 X and W are split the same way, and the pairs of planes below 2^-24 left out.
// Contractions run down the rows of X, W and D: the gfx950 transposing LDS read gathers a lane's 4 values.
constexpr int kGbWaves = 4;      // waves per workgroup, everywhere
constexpr int kDxBlocks = 2;     // blocks of 16 tokens of a wave's step of d_x
constexpr int kDwStage = 64;     // tokens per LDS stage of d_W
constexpr int kDwCols = 128;     // columns of a d_W workgroup

typedef short i16x4 __attribute__((ext_vector_type(4)));

// In each group of 16 lanes, lane i reads the 8 bytes at its address (elements S[i][0..3]) and receives
// S[4 e + i / 4][i % 4] in element e: with lane i at row i / 4 and columns 4 (i % 4) .. + 3 of a row-major tile, the 4
// rows of column i.
__device__ __forceinline__ uint2 read_tr(const char* p) {
    return __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                                         (__attribute__((address_space(3))) i16x4*)(const_cast<char*>(p))));
}
__device__ __forceinline__ bf16x8 frag16(uint2 lo, uint2 hi) {
    return __builtin_bit_cast(bf16x8, make_uint4(lo.x, lo.y, hi.x, hi.y));
}

// v = plane 0 + plane 1 + plane 2
__device__ __forceinline__ void split3(float v, uint16_t (&pl)[3]) {
#pragma unroll
    for (int i = 0; i < 3; ++i) {
        pl[i] = f32_to_bf16(v);
        v -= bf16_to_f32(pl[i]);
    }
}

template <typename T>
constexpr int kPlanes = sizeof(T) == 4 ? 3 : 1;  // of X and W
template <typename T>
constexpr int kDwRowBlocks = sizeof(T) == 4 ? 3 : 5;  // blocks of 16 logits of one d_W workgroup (registers)

inline int logit_steps(int R) {  // contraction steps of 32 logits of d_x
    const int n = (R + 31) / 32;
    return n <= 1 ? 1 : n <= 3 ? 3 : n <= 5 ? 5 : 10;
}

// Sums over aligned runs of 2, 4, 8 or 16 lanes, which all lanes of the run receive (a lane's row is 16 lanes).
template <int CTRL>
__device__ __forceinline__ float dpp_add(float v) {
    return v + __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(v), CTRL, 0xf, 0xf, true));
}
// width: a power of two, 1 to 64, uniform
__device__ __forceinline__ float run_sum(float v, int width) {
    typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
    if (width > 1) v = dpp_add<0xB1>(v);   // lanes 1 0 3 2 of a quad
    if (width > 2) v = dpp_add<0x4E>(v);   // lanes 2 3 0 1
    if (width > 4) v = dpp_add<0x141>(v);  // mirrored within 8
    if (width > 8) v = dpp_add<0x140>(v);  // mirrored within 16
    if (width > 16) {
        const u32x2 r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        v = __uint_as_float(r[0]) + __uint_as_float(r[1]);
    }
    if (width > 32) {
        const u32x2 r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        v = __uint_as_float(r[0]) + __uint_as_float(r[1]);
    }
    return v;
}

// One wave per token, `tokens` of them in turn; lane l holds experts l, l + 64, ... Writes the planes of D ([3][T][ldd],
// zeros past M + K) and the workgroup's column sums. RUNS: equal groups of a power of two up to 64 experts lie in
// aligned runs of lanes, which sum over them in registers; else one lane sums a group from LDS.
// Bound by the chain of a token's steps, so a wave takes few tokens (see the launch).
template <int E, bool RUNS>
__global__ __launch_bounds__(64 * kGbWaves) void gate_logit_grad_kernel(GateBackwardArgs a, uint16_t* D, int ldd, int tokens,
                                                                        float* bpart) {
    constexpr int KQ = RUNS ? 0 : (kMaxGroups + 63) / 64;
    __shared__ float s_g[kGbWaves][64 * E], s_gd[RUNS ? 1 : kGbWaves][64 * E];
    __shared__ float s_a[RUNS ? 1 : kGbWaves][kMaxGroups], s_p[RUNS ? 1 : kGbWaves][kMaxGroups];
    __shared__ uint8_t s_grp[64 * E];
    __shared__ float s_sum[kGbWaves][64 * E + kMaxGroups];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int M = a.n_experts, K = a.n_groups, k = a.top_k;
    int g0[KQ + 1], g1[KQ + 1];  // experts of the lane's groups
    if constexpr (!RUNS) {
        for (int kk = threadIdx.x; kk < K; kk += 64 * kGbWaves)
            for (int i = a.goff[kk]; i < a.goff[kk + 1]; ++i) s_grp[i] = static_cast<uint8_t>(kk);
#pragma unroll
        for (int q = 0; q < KQ; ++q) {
            const int kk = lane + 64 * q;
            g0[q] = kk < K ? a.goff[kk] : 0;
            g1[q] = kk < K ? a.goff[kk + 1] : 0;
        }
        __syncthreads();
    }
    const int mk = a.group_size;
    float bal[E], suml[E], sumg[RUNS ? E : KQ];
#pragma unroll
    for (int j = 0; j < E; ++j) {
        bal[j] = a.d_balance && lane + 64 * j < M ? a.d_balance[lane + 64 * j] : 0.f;
        suml[j] = 0.f;
    }
#pragma unroll
    for (int q = 0; q < (RUNS ? E : KQ); ++q) sumg[q] = 0.f;
    float* sg = s_g[wave];
    float* sgd = s_gd[RUNS ? 0 : wave];
    const int64_t plane = static_cast<int64_t>(a.n_tokens) * ldd;
    const int64_t t0 = (static_cast<int64_t>(blockIdx.x) * kGbWaves + wave) * tokens;
    // Only this wave's LDS is shared below: its lanes run together, a wait for the LDS counter orders them.
    auto settle = [&]() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); };
    for (int u = 0; u < tokens; ++u) {
        const int64_t t = t0 + u;
        if (t >= a.n_tokens) break;  // uniform in the wave
        const bool live = !a.valid || a.valid[t];
        float g[E], dg[E];
#pragma unroll
        for (int j = 0; j < E; ++j) {
            const int i = lane + 64 * j;
            const bool in = live && i < M;
            g[j] = in ? a.probs[t * M + i] : 0.f;
            dg[j] = (in ? bal[j] : 0.f) + (in && a.d_probs ? a.d_probs[t * M + i] : 0.f);
            sg[i] = g[j];
        }
        int e = -1;
        float dw = 0.f;
        if (a.d_topk_w && live && lane < k) {
            e = a.topk_idx[t * k + lane];
            dw = a.d_topk_w[t * k + lane];
        }
        settle();
        if (a.d_topk_w && live) {  // uniform in the wave
            if (e < 0 || e >= M) e = -1;
            const float gs = e >= 0 ? sg[e] : 0.f;
            if (a.renormalize) {
                // w_j = g_j / S: dg_j = (dw_j - sum w dw) / S
                const float S = run_sum(gs, 16);
                const float m = run_sum(lane < k ? gs / S * dw : 0.f, 16);
                dw = (dw - m) / S;
            }
            for (int j = 0; j < k; ++j) {
                const int ej = __builtin_amdgcn_readlane(e, j);
                const float dj = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(dw), j));
#pragma unroll
                for (int q = 0; q < E; ++q)
                    if (lane + 64 * q == ej) dg[q] += dj;
            }
        }
        uint16_t* row = D + t * ldd;
        auto put = [&](int c, float v) {
            uint16_t pl[3];
            split3(v, pl);
#pragma unroll
            for (int i = 0; i < 3; ++i) row[i * plane + c] = pl[i];
        };
        // a group without mass (no candidate, or underflow) has g = 0 throughout
        auto local = [&](float gd, float gj, float A, float P) { return P > 0.f ? gd - gj / P * A : gd; };
        if constexpr (RUNS) {
            float gd[E], tot = 0.f;
#pragma unroll
            for (int j = 0; j < E; ++j) {
                gd[j] = g[j] * dg[j];
                tot += gd[j];
            }
            tot = run_sum(tot, 64);
#pragma unroll
            for (int j = 0; j < E; ++j) {
                const int i = lane + 64 * j;
                const float A = run_sum(gd[j], mk), P = run_sum(g[j], mk);
                if (i >= M) continue;
                const float v = local(gd[j], g[j], A, P);
                suml[j] += v;
                put(i, v);
                if ((i & (mk - 1)) == 0) {  // the group's first lane: its group logit
                    const float w = A - P * tot;
                    sumg[j] += w;
                    put(M + i / mk, w);
                }
            }
        } else {
#pragma unroll
            for (int j = 0; j < E; ++j) sgd[lane + 64 * j] = g[j] * dg[j];
            settle();
            float A[KQ + 1], P[KQ + 1], tot = 0.f;
#pragma unroll
            for (int q = 0; q < KQ; ++q) {
                A[q] = P[q] = 0.f;
                for (int i = g0[q]; i < g1[q]; ++i) {
                    A[q] += sgd[i];
                    P[q] += sg[i];
                }
                if (lane + 64 * q < K) {
                    s_a[wave][lane + 64 * q] = A[q];
                    s_p[wave][lane + 64 * q] = P[q];
                }
                tot += A[q];
            }
            tot = run_sum(tot, 64);
            settle();
#pragma unroll
            for (int j = 0; j < E; ++j) {
                const int i = lane + 64 * j;
                if (i >= M) continue;
                const int kk = s_grp[i];
                const float v = local(sgd[i], g[j], s_a[wave][kk], s_p[wave][kk]);
                suml[j] += v;
                put(i, v);
            }
#pragma unroll
            for (int q = 0; q < KQ; ++q) {
                if (lane + 64 * q >= K) continue;
                const float v = A[q] - P[q] * tot;
                sumg[q] += v;
                put(M + lane + 64 * q, v);
            }
        }
        for (int i = M + K + lane; i < ldd; i += 64) put(i, 0.f);
    }
#pragma unroll
    for (int j = 0; j < E; ++j) {
        const int i = lane + 64 * j;
        if (i < M) s_sum[wave][i] = suml[j];
        if (RUNS && i < M && (i & (mk - 1)) == 0) s_sum[wave][M + i / mk] = sumg[RUNS ? j : 0];
    }
#pragma unroll
    for (int q = 0; q < KQ; ++q)
        if (lane + 64 * q < K) s_sum[wave][M + lane + 64 * q] = sumg[q];
    __syncthreads();
    for (int r = threadIdx.x; r < M + K; r += 64 * kGbWaves) {
        float v = s_sum[0][r];
#pragma unroll
        for (int w = 1; w < kGbWaves; ++w) v += s_sum[w][r];
        bpart[static_cast<int64_t>(blockIdx.x) * (M + K) + r] = v;
    }
}

// row r of the stacked gate weights (local rows, then group rows)
template <typename T>
__device__ __forceinline__ const T* gate_row(const GateBackwardArgs& a, int r) {
    return r < a.n_experts ? static_cast<const T*>(a.w_local) + static_cast<int64_t>(r) * a.d
                           : static_cast<const T*>(a.w_global) + static_cast<int64_t>(r - a.n_experts) * a.d;
}

// 16 bytes as loaded (8 bfloat16 or 4 float32 values) into the planes of a staged tile, at byte offset off of a bfloat16
// plane (float32 values take 8 bytes there)
__device__ __forceinline__ void stage16(char* tile, int, int off, uint4 v, bf16_t) {
    *reinterpret_cast<uint4*>(tile + off) = v;
}
__device__ __forceinline__ void stage16(char* tile, int plane_bytes, int off, uint4 v, float) {
    const float f[4] = {__uint_as_float(v.x), __uint_as_float(v.y), __uint_as_float(v.z), __uint_as_float(v.w)};
    uint16_t pl[4][3];
#pragma unroll
    for (int i = 0; i < 4; ++i) split3(f[i], pl[i]);
#pragma unroll
    for (int p = 0; p < 3; ++p)
        *reinterpret_cast<uint2*>(tile + p * plane_bytes + off) =
            make_uint2(pl[0][p] | static_cast<uint32_t>(pl[1][p]) << 16, pl[2][p] | static_cast<uint32_t>(pl[3][p]) << 16);
}

// Column tile and token chunk of a workgroup: the column tiles of a chunk run on one XCD (workgroups go round-robin over
// the eight), so that its rows of D are fetched into that XCD's L2 once. Chunks at or past `chunks` have no work.
__device__ __forceinline__ int2 col_chunk(int block, int cols, int chunks) {
    const int j = block / 8;
    return make_int2(j % cols, j / cols * 8 + block % 8);
}
inline unsigned col_chunk_grid(int cols, int chunks) { return static_cast<unsigned>(cols) * ((chunks + 7) / 8) * 8; }

// d_x [T][d] = D W. A workgroup holds the whole W [R][COLS] of its columns in LDS (the 32-byte chunk c of row r at c ^
// (r % chunks), so that the 4 rows of a transposing read lie in different banks); its waves walk the tokens, 32 each at
// a time, over all the columns. The fragments of D come straight from memory (a lane's 8 consecutive logits), a set
// ahead. Finished rows are turned in LDS (each wave its own 4 KB) so that a store covers whole 256-byte rows: stores of
// 8 bytes a lane, 32 bytes of a row, took 26 us in place of 18 (8192 tokens of 2048, 72 logits).
template <typename T, int KS>
struct DxLds {
    static constexpr int kCols = kPlanes<T> == 1 ? 128 : 64;
    static constexpr int kTurn = kPlanes<T> * KS * 32 * kCols * 2;  // offset of the waves' rows
    static constexpr int kBytes = kTurn + kGbWaves * 16 * 256;
};
template <typename T, int KS>
__device__ __forceinline__ void gate_dx(const GateBackwardArgs& a, const uint16_t* D, int tokens, int chunks, int block, char* lds) {
    constexpr int PX = kPlanes<T>, PD = PX == 1 ? 2 : 3;
    constexpr int COLS = DxLds<T, KS>::kCols, CB = COLS / 16;  // column blocks of 16
    constexpr int ROWB = COLS * 2, CH = ROWB / 32, PLANE = KS * 32 * ROWB;
    constexpr int LDD = KS * 32;
    constexpr int MB = kDxBlocks;         // token blocks of a step
    constexpr int NK = KS <= 3 ? KS : 1;  // contraction steps loaded together, one set ahead
    constexpr int EPC = Elem<T>::kPerChunk;
    constexpr int STEP = 16 * MB * kGbWaves;  // tokens of the workgroup's step
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int l16 = lane & 15, lg = lane >> 4;
    char* w = lds;
    char* turn = lds + DxLds<T, KS>::kTurn + wave * 16 * 256;
    const int R = a.n_experts + a.n_groups;
    const int2 at = col_chunk(block, a.d / COLS, chunks);
    if (at.y >= chunks) return;
    const int c0 = at.x * COLS;
    const int64_t tb = static_cast<int64_t>(at.y) * tokens;
    const int64_t te = min(tb + tokens, static_cast<int64_t>(a.n_tokens));
    const int64_t plane = static_cast<int64_t>(a.n_tokens) * LDD;
    // the fragments of D of NK steps of the 16 MB tokens from t0
    auto load = [&](int64_t t0, int ks0, uint4 (&dv)[NK][MB][PD]) {
#pragma unroll
        for (int m = 0; m < MB; ++m) {
            const uint16_t* drow = D + min(t0 + m * 16 + l16, te - 1) * LDD + 8 * lg;
#pragma unroll
            for (int ks = 0; ks < NK; ++ks)
#pragma unroll
                for (int p = 0; p < PD; ++p) dv[ks][m][p] = ldg16(drow + p * plane + (ks0 + ks) * 32);
        }
    };
    uint4 dv[NK][MB][PD], nx[NK][MB][PD];
    int64_t t0 = tb + wave * 16 * MB;
    load(t0, 0, nx);
    constexpr int PER_ROW = COLS / EPC;
    for (int i = tid; i < KS * 32 * PER_ROW; i += 64 * kGbWaves) {
        const int r = i / PER_ROW, e = (i % PER_ROW) * EPC;
        const uint4 v = r < R ? ldg16(gate_row<T>(a, r) + c0 + e) : make_uint4(0, 0, 0, 0);
        stage16(w, PLANE, r * ROWB + (((e / 16) ^ (r % CH)) * 32) + (e % 16) * 2, v, T{});
    }
    __syncthreads();
    for (; t0 < te; t0 += STEP) {
        f32x4 acc[CB][MB];
#pragma unroll
        for (int c = 0; c < CB; ++c)
#pragma unroll
            for (int m = 0; m < MB; ++m) acc[c][m] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int ks0 = 0; ks0 < KS; ks0 += NK) {
            __builtin_memcpy(dv, nx, sizeof dv);
            if (ks0 + NK < KS) load(t0, ks0 + NK, nx);
            else if (t0 + STEP < te) load(t0 + STEP, 0, nx);
#pragma unroll
            for (int kk = 0; kk < NK; ++kk) {
                const int r = (ks0 + kk) * 32 + 8 * lg + (l16 >> 2);
#pragma unroll
                for (int c = 0; c < CB; ++c) {
                    bf16x8 wv[PX];
#pragma unroll
                    for (int p = 0; p < PX; ++p) {
                        const char* base = w + p * PLANE + (l16 & 3) * 8;
                        wv[p] = frag16(read_tr(base + r * ROWB + (c ^ (r % CH)) * 32),
                                       read_tr(base + (r + 4) * ROWB + (c ^ ((r + 4) % CH)) * 32));
                    }
#pragma unroll
                    for (int m = 0; m < MB; ++m)
#pragma unroll
                        for (int pd = PD - 1; pd >= 0; --pd)
#pragma unroll
                            for (int px = PX - 1; px >= 0; --px)
                                if (pd + px <= 2)
                                    acc[c][m] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                                        wv[px], __builtin_bit_cast(bf16x8, dv[kk][m][pd]), acc[c][m], 0, 0, 0);
                }
            }
        }
        // 16 rows of 256 bytes: the 16-byte chunk x of row r at x ^ r
#pragma unroll
        for (int m = 0; m < MB; ++m) {
            char* row = turn + l16 * 256;
#pragma unroll
            for (int c = 0; c < CB; ++c) {
                if constexpr (PX == 1) {
                    uint2 o;
                    o.x = static_cast<uint32_t>(f32_to_bf16(acc[c][m][0])) | static_cast<uint32_t>(f32_to_bf16(acc[c][m][1])) << 16;
                    o.y = static_cast<uint32_t>(f32_to_bf16(acc[c][m][2])) | static_cast<uint32_t>(f32_to_bf16(acc[c][m][3])) << 16;
                    *reinterpret_cast<uint2*>(row + (((2 * c + (lg >> 1)) ^ l16) * 16) + (lg & 1) * 8) = o;
                } else {
                    *reinterpret_cast<f32x4*>(row + (((4 * c + lg) ^ l16) * 16)) = acc[c][m];
                }
            }
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // the wave's own rows
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int r = 4 * i + lg;
                const int64_t t = t0 + m * 16 + r;
                const uint4 v = *reinterpret_cast<const uint4*>(turn + r * 256 + ((l16 ^ r) * 16));
                if (t < te) stg16(static_cast<T*>(a.d_x) + t * a.d + c0 + l16 * EPC, v);
            }
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // read before the next rows land
        }
    }
}

// part[chunk][r][c] = sum over the chunk's tokens of D[t][r] X[t][c], for NRB blocks of 16 logits from row group
// `group` and 128 columns. Stages of 64 tokens: X as [token][128] (32-byte chunk c of row t at c ^ (t % 8)) and the
// logits' columns of D as [token][16 NRB], per plane. Two waves take the column halves of the first 32 tokens of a
// stage, two those of the others; their sums meet in LDS at the end. Padding tokens' rows of X count as zeros, whatever
// they hold.
template <typename T, int NRB>
struct DwLds {
    static constexpr int kStage = kPlanes<T> * kDwStage * kDwCols * 2 + 3 * kDwStage * NRB * 32;
    static constexpr int kSums = 2 * NRB * 4 * 64 * 16;  // two waves' sums
    static constexpr int kBytes = kStage > kSums ? kStage : kSums;
};
template <typename T, int NRB>
__device__ __forceinline__ void gate_dw(const GateBackwardArgs& a, const uint16_t* D, int ldd, int chunk, int chunks, float* part,
                                        int block, int group, char* lds) {
    constexpr int PX = kPlanes<T>;
    constexpr int EPC = Elem<T>::kPerChunk;
    constexpr int XROW = kDwCols * 2, XPLANE = kDwStage * XROW;
    constexpr int DROW = NRB * 32, DPLANE = kDwStage * DROW;
    constexpr int XL = kDwStage * kDwCols / EPC / 256;            // 16-byte loads a thread
    constexpr int DI = 3 * kDwStage * DROW / 16;                  // 16-byte pieces of a stage of D
    constexpr int DL = (DI + 255) / 256;
    char* xs = lds;
    char* ds = lds + PX * XPLANE;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int l16 = lane & 15, lg = lane >> 4;
    const int ch = wave & 1, th = wave >> 1;
    const int2 at = col_chunk(block, a.d / kDwCols, chunks);
    if (at.y >= chunks) return;
    const int c0 = at.x * kDwCols;
    const int r0 = group * kDwRowBlocks<T> * 16;
    const int64_t tb = static_cast<int64_t>(at.y) * chunk;
    const int64_t te = min(tb + chunk, static_cast<int64_t>(a.n_tokens));
    const int64_t plane = static_cast<int64_t>(a.n_tokens) * ldd;
    uint4 xv[XL], dv[DL];
    auto load = [&](int64_t t0) {
#pragma unroll
        for (int i = 0; i < XL; ++i) {
            const int item = tid + 256 * i, row = item / (kDwCols / EPC), e = item % (kDwCols / EPC) * EPC;
            const int64_t t = t0 + row;
            const bool in = t < te && (!a.valid || a.valid[t]);
            xv[i] = in ? ldg16(static_cast<const T*>(a.x) + t * a.d + c0 + e) : make_uint4(0, 0, 0, 0);
        }
#pragma unroll
        for (int i = 0; i < DL; ++i) {
            const int item = tid + 256 * i, p = item / (DI / 3), q = item % (DI / 3);
            const int64_t t = t0 + q / (DROW / 16);
            const int c = r0 + q % (DROW / 16) * 8;
            dv[i] = item < DI && t < te && c < ldd ? ldg16(D + p * plane + t * ldd + c) : make_uint4(0, 0, 0, 0);
        }
    };
    f32x4 acc[NRB][4];
#pragma unroll
    for (int b = 0; b < NRB; ++b)
#pragma unroll
        for (int c = 0; c < 4; ++c) acc[b][c] = f32x4{0.f, 0.f, 0.f, 0.f};
    load(tb);
    for (int64_t t0 = tb; t0 < te; t0 += kDwStage) {
        __syncthreads();  // every wave is done with the stage before
#pragma unroll
        for (int i = 0; i < XL; ++i) {
            const int item = tid + 256 * i, row = item / (kDwCols / EPC), e = item % (kDwCols / EPC) * EPC;
            stage16(xs, XPLANE, row * XROW + (((e / 16) ^ (row & 7)) * 32) + (e % 16) * 2, xv[i], T{});
        }
#pragma unroll
        for (int i = 0; i < DL; ++i) {
            const int item = tid + 256 * i;
            if (item < DI) *reinterpret_cast<uint4*>(ds + item * 16) = dv[i];
        }
        __syncthreads();
        if (t0 + kDwStage < te) load(t0 + kDwStage);
        const int row = th * 32 + 8 * lg + (l16 >> 2);
        bf16x8 xf[4][PX];
#pragma unroll
        for (int c = 0; c < 4; ++c)
#pragma unroll
            for (int p = 0; p < PX; ++p) {
                const char* base = xs + p * XPLANE + (l16 & 3) * 8;
                const int cc = ch * 4 + c;
                xf[c][p] = frag16(read_tr(base + row * XROW + (cc ^ (row & 7)) * 32),
                                  read_tr(base + (row + 4) * XROW + (cc ^ ((row + 4) & 7)) * 32));
            }
#pragma unroll
        for (int b = 0; b < NRB; ++b) {
            bf16x8 df[3];
#pragma unroll
            for (int p = 0; p < 3; ++p) {
                const char* base = ds + p * DPLANE + b * 32 + (l16 & 3) * 8;
                df[p] = frag16(read_tr(base + row * DROW), read_tr(base + (row + 4) * DROW));
            }
#pragma unroll
            for (int c = 0; c < 4; ++c)
#pragma unroll
                for (int pd = 2; pd >= 0; --pd)
#pragma unroll
                    for (int px = PX - 1; px >= 0; --px)
                        if (pd + px <= 2)
                            acc[b][c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(xf[c][px], df[pd], acc[b][c], 0, 0, 0);
        }
    }
    __syncthreads();
    f32x4* sums = reinterpret_cast<f32x4*>(lds) + ch * NRB * 4 * 64 + lane;
    if (th == 1)
#pragma unroll
        for (int b = 0; b < NRB; ++b)
#pragma unroll
            for (int c = 0; c < 4; ++c) sums[(b * 4 + c) * 64] = acc[b][c];
    __syncthreads();
    if (th == 1) return;
    const int R = a.n_experts + a.n_groups;
    float* out = part + static_cast<int64_t>(at.y) * R * a.d + c0 + ch * 64 + 4 * lg;
#pragma unroll
    for (int b = 0; b < NRB; ++b) {
        const int r = r0 + b * 16 + l16;
        if (r >= R) continue;
#pragma unroll
        for (int c = 0; c < 4; ++c)
            *reinterpret_cast<f32x4*>(out + static_cast<int64_t>(r) * a.d + 16 * c) = acc[b][c] + sums[(b * 4 + c) * 64];
    }
}

// Both products in one launch: the first dw_blocks workgroups of each of the dw_groups row groups d_W, the rest d_x. They
// wait for memory at different times: 37 -> 31 us for 8192 tokens of 2048, 72 logits, 28 in long runs (67 MB of X and d_x; 4.7 MB of
// planes, which every column tile reads from the L2s).
struct GateProducts {
    const uint16_t* D;
    int ldd, chunk, chunks, dw_blocks, dw_groups;
    int dx_tokens, dx_chunks;
    float* part;
};
template <typename T, int KS, int NRB>
__global__ __launch_bounds__(64 * kGbWaves, 2) void gate_products_kernel(GateBackwardArgs a, GateProducts g) {
    constexpr int kDx = DxLds<T, KS>::kBytes, kDw = DwLds<T, NRB>::kBytes;
    __shared__ __attribute__((aligned(16))) char lds[kDx > kDw ? kDx : kDw];
    const int b = blockIdx.x;
    if (b < g.dw_blocks * g.dw_groups)
        gate_dw<T, NRB>(a, g.D, g.ldd, g.chunk, g.chunks, g.part, b % g.dw_blocks, b / g.dw_blocks, lds);
    else
        gate_dx<T, KS>(a, g.D, g.dx_tokens, g.dx_chunks, b - g.dw_blocks * g.dw_groups, lds);
}

// The chunks' sums in order: 4 columns of a row a thread; the first workgroups add the biases' partial sums instead, a
// logit each (in float64, strided over the threads, then down a tree).
__global__ __launch_bounds__(256) void gate_dw_sum_kernel(GateBackwardArgs a, const float* part, int chunks,
                                                          const float* bpart, int bparts, int bias_groups) {
    const int M = a.n_experts, R = M + a.n_groups;
    if (static_cast<int>(blockIdx.x) < bias_groups) {
        __shared__ double s[256];
        const int r = blockIdx.x;
        double v = 0.0;
        for (int j = threadIdx.x; j < bparts; j += 256) v += bpart[static_cast<int64_t>(j) * R + r];
        s[threadIdx.x] = v;
        __syncthreads();
        for (int h = 128; h > 0; h >>= 1) {
            if (static_cast<int>(threadIdx.x) < h) s[threadIdx.x] += s[threadIdx.x + h];
            __syncthreads();
        }
        float* dst = r < M ? a.d_b_local : a.d_b_global;
        if (threadIdx.x == 0 && dst) dst[r < M ? r : r - M] = static_cast<float>(s[0]);
        return;
    }
    const int64_t i = static_cast<int64_t>(blockIdx.x - bias_groups) * 256 + threadIdx.x;
    if (i >= static_cast<int64_t>(R) * (a.d / 4)) return;
    const int r = static_cast<int>(i / (a.d / 4));
    const int c = static_cast<int>(i % (a.d / 4)) * 4;
    f32x4 v = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
    for (int j = 0; j < chunks; ++j)
        v += *reinterpret_cast<const f32x4*>(part + (static_cast<int64_t>(j) * R + r) * a.d + c);
    float* dst = r < M ? a.d_w_local + static_cast<int64_t>(r) * a.d : a.d_w_global + static_cast<int64_t>(r - M) * a.d;
    *reinterpret_cast<f32x4*>(dst + c) = v;
}

// Token chunks of d_W, whole stages each: a workgroup a CU over the column tiles and row groups, those of d_x beside it (two
// a CU: 19 in place of 9 MB of partial sums, 43.8 us against 42.9 for 8192 tokens of 2048, 72 logits).
int dw_chunk(int n_tokens, int d, int R, int row_blocks) {
    const int nrb = (R + 15) / 16;
    const int tiles = (d / kDwCols) * ((nrb + row_blocks - 1) / row_blocks);
    const int want = std::max(1, 256 / tiles);
    const int per = (n_tokens + want - 1) / want;
    return std::max(kDwStage, (per + kDwStage - 1) / kDwStage * kDwStage);
}

struct GateBackwardWs {
    size_t D, part, bpart, total;
    int ldd, chunk, chunks, tokens, bparts;
};

template <typename T>
GateBackwardWs gate_backward_ws(int n_tokens, int d, int R) {
    auto up = [](size_t n) { return (n + 255) / 256 * 256; };
    GateBackwardWs w{};
    w.ldd = 32 * logit_steps(R);
    w.chunk = dw_chunk(n_tokens, d, R, kDwRowBlocks<T>);
    w.chunks = (n_tokens + w.chunk - 1) / w.chunk;
    // a token a wave up to four workgroups a CU; more only lengthen the list of the biases' partial sums
    w.tokens = std::max(1, std::min(16, n_tokens / (1024 * kGbWaves)));
    w.bparts = (n_tokens + kGbWaves * w.tokens - 1) / (kGbWaves * w.tokens);
    size_t o = 0;
    w.D = o; o += up(static_cast<size_t>(n_tokens) * w.ldd * 2 * 3);
    w.part = o; o += up(static_cast<size_t>(w.chunks) * R * d * 4);
    w.bpart = o; o += up(static_cast<size_t>(w.bparts) * R * 4);
    w.total = o;
    return w;
}

template <typename T>
hipError_t gate_backward(const GateBackwardArgs& a, hipStream_t s) {
    const int R = a.n_experts + a.n_groups;
    const GateBackwardWs w = gate_backward_ws<T>(a.n_tokens, a.d, R);
    char* base = static_cast<char*>(a.ws);
    uint16_t* D = reinterpret_cast<uint16_t*>(base + w.D);
    float* part = reinterpret_cast<float*>(base + w.part);
    float* bpart = reinterpret_cast<float*>(base + w.bpart);
    const dim3 threads(64 * kGbWaves);
    hipError_t e = hipSuccess;
    if (a.n_tokens) {
        ProfileScope prof(kLogitGradName, s);
        auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(w.bparts), threads, 0, s, a, D, w.ldd, w.tokens, bpart); };
        const int mk = a.group_size;
        const bool runs = mk > 0 && mk <= 64 && (mk & (mk - 1)) == 0;
        if (a.n_experts <= 64) runs ? go(gate_logit_grad_kernel<1, true>) : go(gate_logit_grad_kernel<1, false>);
        else if (a.n_experts <= 128) runs ? go(gate_logit_grad_kernel<2, true>) : go(gate_logit_grad_kernel<2, false>);
        else runs ? go(gate_logit_grad_kernel<4, true>) : go(gate_logit_grad_kernel<4, false>);
        e = hipGetLastError();
    }
    if (e == hipSuccess && a.n_tokens && (a.d_x || a.d_w_local)) {
        ProfileScope prof(kProductsName, s);
        GateProducts g{};
        g.D = D;
        g.ldd = w.ldd;
        g.part = part;
        const int nrb = (R + 15) / 16;
        if (a.d_w_local) {
            g.chunk = w.chunk;
            g.chunks = w.chunks;
            g.dw_blocks = static_cast<int>(col_chunk_grid(a.d / kDwCols, w.chunks));
            g.dw_groups = (nrb + kDwRowBlocks<T> - 1) / kDwRowBlocks<T>;
        }
        unsigned dx_blocks = 0;
        if (a.d_x) {
            const int cols = kPlanes<T> == 1 ? 128 : 64;
            // about six workgroups a CU in turn, whole steps each
            const int want = std::max(1, 1536 / (a.d / cols));
            const int step = 16 * kDxBlocks * kGbWaves;
            g.dx_tokens = std::max(step, ((a.n_tokens + want - 1) / want + step - 1) / step * step);
            g.dx_chunks = (a.n_tokens + g.dx_tokens - 1) / g.dx_tokens;
            dx_blocks = col_chunk_grid(a.d / cols, g.dx_chunks);
        }
        auto go = [&](auto kernel) {
            hipLaunchKernelGGL(kernel, dim3(g.dw_blocks * g.dw_groups + dx_blocks), threads, 0, s, a, g);
        };
        if (nrb <= 1) go(gate_products_kernel<T, 1, 1>);
        else if (nrb <= 2) go(gate_products_kernel<T, 1, 2>);
        else if (nrb <= 3) go(gate_products_kernel<T, 3, 3>);
        else if (nrb <= 6) go(gate_products_kernel<T, 3, kDwRowBlocks<T>>);
        else if (nrb <= 10) go(gate_products_kernel<T, 5, kDwRowBlocks<T>>);
        else go(gate_products_kernel<T, 10, kDwRowBlocks<T>>);
        e = hipGetLastError();
    }
    if (!a.d_w_local && !a.d_b_local && !a.d_b_global) return e;
    if (e == hipSuccess) {
        ProfileScope prof(kDwSumName, s);
        const int bias = a.d_b_local || a.d_b_global ? R : 0;
        const int64_t quads = a.d_w_local ? static_cast<int64_t>(R) * (a.d / 4) : 0;
        hipLaunchKernelGGL(gate_dw_sum_kernel, dim3(static_cast<unsigned>(bias + (quads + 255) / 256)), dim3(256), 0, s, a, part,
                           w.chunks, bpart, w.bparts, bias);
        e = hipGetLastError();
    }
    return e;
}

}  // namespace

size_t balance_ws_bytes(int n_tokens, int n_experts) {
    const size_t chunks = balance_chunks(n_tokens, n_experts);
    return chunks == 1 ? 0 : (kMaxExperts / kBalCols) * 8 + 8 + chunks * (2 * static_cast<size_t>(n_experts) + 1) * 4;
}

hipError_t launch_balance(const BalanceArgs& a, hipStream_t s) {
    const int chunks0 = balance_chunks(a.n_tokens, a.n_experts);
    const int chunk = std::max(1, static_cast<int>((static_cast<int64_t>(a.n_tokens) + chunks0 - 1) / chunks0));
    const int chunks = chunks0;  // trailing ones may be empty
    {
        ProfileScope prof(kBalanceName, s);
        if (a.n_experts % 4 == 0)
            hipLaunchKernelGGL(balance_kernel<4>, dim3(chunks), dim3(kBalThreads), 0, s, a, chunk);
        else
            hipLaunchKernelGGL(balance_kernel<1>, dim3(chunks), dim3(kBalThreads), 0, s, a, chunk);
    }
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || chunks == 1) return e;
    ProfileScope prof(kBalanceFinishName, s);
    hipLaunchKernelGGL(balance_finish_kernel, dim3((a.n_experts + kBalCols - 1) / kBalCols), dim3(1024), 0, s, a, chunks);
    return hipGetLastError();
}

size_t gate_backward_ws_bytes(DType dt, int n_tokens, int d, int n_experts, int n_groups) {
    const int R = n_experts + n_groups;
    return dt == DType::BF16 ? gate_backward_ws<bf16_t>(n_tokens, d, R).total : gate_backward_ws<float>(n_tokens, d, R).total;
}

hipError_t launch_gate_backward(DType dt, const GateBackwardArgs& a, hipStream_t s) {
    return dt == DType::BF16 ? gate_backward<bf16_t>(a, s) : gate_backward<float>(a, s);
}

}  // namespace ec2moe
