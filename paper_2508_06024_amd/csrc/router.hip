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
                     *kLogitGradName = "gate_logit_grad", *kDxName = "gate_dx", *kDwName = "gate_dw",
                     *kDbName = "gate_db", *kDwSumName = "gate_dw_sum";

// ------------------------------------------------------------------ load balance loss
//
// Column sums of probs over the valid tokens and a histogram of the selected experts, by chunks of
// tokens (a workgroup each); a second launch adds the chunks in order. With one chunk the first
// launch finishes by itself. Integer counts are added with LDS atomics: their order changes nothing.
constexpr int kBalThreads = 256;
constexpr int kBalMaxChunks = 512;

int balance_chunks(int n_tokens, int n_experts) {
    const int64_t values = static_cast<int64_t>(n_tokens) * n_experts;
    return static_cast<int>(std::max<int64_t>(1, std::min<int64_t>(kBalMaxChunks, (values + 8191) / 8192)));
}

struct BalancePart {
    float* p;    // [chunks][M]
    int32_t* c;  // [chunks][M]
    int32_t* n;  // [chunks] valid tokens
};

__host__ __device__ inline BalancePart balance_part(void* ws, int chunks, int M) {
    float* p = static_cast<float*>(ws);
    int32_t* c = reinterpret_cast<int32_t*>(p + static_cast<size_t>(chunks) * M);
    return {p, c, c + static_cast<size_t>(chunks) * M};
}

// Thread e < M of a workgroup holds expert e's sum of probabilities and count, n the valid tokens: writes
// the outputs. sm: kMaxExperts doubles.
__device__ __forceinline__ void balance_outputs(const BalanceArgs& a, int e, double p, int c, int n, double* sm) {
    const int M = a.n_experts;
    double d = 0.0;
    if (e < M) {
        if (n > 0) d = static_cast<double>(a.coef) * M * c / (static_cast<double>(a.top_k) * n * n);
        if (a.counts) a.counts[e] = c;
        if (a.d_probs) a.d_probs[e] = static_cast<float>(d);
        sm[e] = n > 0 ? d * p : 0.0;
    }
    __syncthreads();
    if (e == 0) {
        double loss = 0.0;
        for (int i = 0; i < M; ++i) loss += sm[i];
        a.loss[0] = static_cast<float>(loss);
    }
}

// V: consecutive experts a thread loads together
template <int V>
__global__ __launch_bounds__(kBalThreads) void balance_kernel(BalanceArgs a, int chunk) {
    __shared__ float s_sum[kBalThreads * V];
    __shared__ int s_cnt[kMaxExperts];
    __shared__ int s_n;
    __shared__ double s_loss[kMaxExperts];
    const int tid = threadIdx.x, M = a.n_experts;
    const int L = (M + V - 1) / V;         // threads per row
    const int RP = kBalThreads / L;        // rows per pass
    const int64_t t0 = static_cast<int64_t>(blockIdx.x) * chunk;
    const int64_t t1 = min(t0 + chunk, static_cast<int64_t>(a.n_tokens));
    for (int i = tid; i < kMaxExperts; i += kBalThreads) s_cnt[i] = 0;
    if (tid == 0) s_n = 0;
    __syncthreads();
    const int rs = tid / L, c = (tid % L) * V;
    float sum[V];
#pragma unroll
    for (int v = 0; v < V; ++v) sum[v] = 0.f;
    if (rs < RP) {
#pragma unroll 8
        for (int64_t t = t0 + rs; t < t1; t += RP) {
            const bool ok = !a.valid || a.valid[t];
            if constexpr (V == 4) {
                const f32x4 v = *reinterpret_cast<const f32x4*>(a.probs + t * M + c);
#pragma unroll
                for (int i = 0; i < 4; ++i) sum[i] += ok ? v[i] : 0.f;
            } else {
                sum[0] += ok ? a.probs[t * M + c] : 0.f;
            }
        }
    }
    for (int64_t i = t0 * a.top_k + tid; i < t1 * a.top_k; i += kBalThreads) {
        const int e = a.topk_idx[i];
        if ((!a.valid || a.valid[i / a.top_k]) && e >= 0 && e < M) atomicAdd(&s_cnt[e], 1);
    }
    int n = 0;
    for (int64_t t = t0 + tid; t < t1; t += kBalThreads) n += !a.valid || a.valid[t] ? 1 : 0;
    if (n) atomicAdd(&s_n, n);
    if (rs < RP)
#pragma unroll
        for (int v = 0; v < V; ++v) s_sum[rs * L * V + c + v] = sum[v];
    __syncthreads();
    float p = 0.f;
    if (tid < M)
        for (int r = 0; r < RP; ++r) p += s_sum[r * L * V + tid];
    if (gridDim.x == 1) {
        balance_outputs(a, tid, p, tid < M ? s_cnt[tid] : 0, s_n, s_loss);
        return;
    }
    const BalancePart part = balance_part(a.ws, gridDim.x, M);
    if (tid < M) {
        part.p[static_cast<int64_t>(blockIdx.x) * M + tid] = p;
        part.c[static_cast<int64_t>(blockIdx.x) * M + tid] = s_cnt[tid];
    }
    if (tid == 0) part.n[blockIdx.x] = s_n;
}

__global__ __launch_bounds__(1024) void balance_finish_kernel(BalanceArgs a, int chunks) {
    __shared__ double s_p[1024];
    __shared__ int s_c[1024];
    __shared__ int s_n;
    __shared__ double s_loss[kMaxExperts];
    const int tid = threadIdx.x, M = a.n_experts;
    const int slots = 1024 / M;
    const int e = tid % M, slot = tid / M;
    const BalancePart part = balance_part(a.ws, chunks, M);
    if (tid == 0) s_n = 0;
    __syncthreads();
    double p = 0.0;
    int c = 0, n = 0;
    if (slot < slots)
#pragma unroll 8
        for (int j = slot; j < chunks; j += slots) {
            p += part.p[static_cast<int64_t>(j) * M + e];
            c += part.c[static_cast<int64_t>(j) * M + e];
        }
    for (int j = tid; j < chunks; j += 1024) n += part.n[j];
    if (n) atomicAdd(&s_n, n);
    s_p[tid] = p;
    s_c[tid] = c;
    __syncthreads();
    p = 0.0;
    c = 0;
    if (tid < M)
        for (int j = 0; j < slots; ++j) {
            p += s_p[j * M + tid];
            c += s_c[j * M + tid];
        }
    balance_outputs(a, tid, p, c, s_n, s_loss);
}

// ------------------------------------------------------------------ gate backward
//
// Three products around the gradient of the logits D [T][M + K] (columns: M local, then K group
// logits): D itself from the probabilities, d_x = D W, and d_W = D^T X with the column sums of D.
constexpr int kGbTok = 4;  // tokens (waves) per workgroup of the first launch

inline int padded_rows(int R) { return (R + 15) / 16 * 16; }

// One wave per token; lane l holds experts l, l + 64, ... D [T][ldd], zeros past M + K.
__global__ __launch_bounds__(64 * kGbTok) void gate_logit_grad_kernel(GateBackwardArgs a, float* D, int ldd) {
    constexpr int E = kMaxExperts / 64;
    __shared__ float s_g[kGbTok][kMaxExperts], s_gd[kGbTok][kMaxExperts];
    __shared__ float s_a[kGbTok][kMaxGroups], s_p[kGbTok][kMaxGroups];
    __shared__ uint8_t s_grp[kMaxExperts];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int M = a.n_experts, K = a.n_groups, k = a.top_k;
    for (int kk = threadIdx.x; kk < K; kk += 64 * kGbTok)
        for (int i = a.goff[kk]; i < a.goff[kk + 1]; ++i) s_grp[i] = static_cast<uint8_t>(kk);
    const int64_t t = static_cast<int64_t>(blockIdx.x) * kGbTok + wave;
    const bool live = t < a.n_tokens && (!a.valid || a.valid[t]);
    float* sg = s_g[wave];
    float* sgd = s_gd[wave];
    float g[E], dg[E];
#pragma unroll
    for (int j = 0; j < E; ++j) {
        const int i = lane + 64 * j;
        const bool in = live && i < M;
        g[j] = in ? a.probs[t * M + i] : 0.f;
        dg[j] = (in && a.d_balance ? a.d_balance[i] : 0.f) + (in && a.d_probs ? a.d_probs[t * M + i] : 0.f);
        if (i < M) sg[i] = g[j];
    }
    __syncthreads();
    if (a.d_topk_w && live) {  // uniform in the wave
        int e = -1;
        float dw = 0.f, gs = 0.f;
        if (lane < k) {
            e = a.topk_idx[t * k + lane];
            if (e < 0 || e >= M) e = -1;
            dw = a.d_topk_w[t * k + lane];
            gs = e >= 0 ? sg[e] : 0.f;
        }
        if (a.renormalize) {
            // w_j = g_j / S: dg_j = (dw_j - sum w dw) / S
            float S = gs;
#pragma unroll
            for (int off = 1; off < 16; off <<= 1) S += __shfl_xor(S, off);
            const float w = gs / S;
            float m = lane < k ? w * dw : 0.f;
#pragma unroll
            for (int off = 1; off < 16; off <<= 1) m += __shfl_xor(m, off);
            dw = (dw - m) / S;
        }
        for (int j = 0; j < k; ++j) {
            const int ej = __shfl(e, j);
            const float dj = __shfl(dw, j);
#pragma unroll
            for (int q = 0; q < E; ++q)
                if (lane + 64 * q == ej) dg[q] += dj;
        }
    }
#pragma unroll
    for (int j = 0; j < E; ++j) {
        const int i = lane + 64 * j;
        if (i < M) sgd[i] = g[j] * dg[j];
    }
    __syncthreads();
    float tot = 0.f;
    for (int kk = lane; kk < K; kk += 64) {
        float A = 0.f, P = 0.f;
        for (int i = a.goff[kk]; i < a.goff[kk + 1]; ++i) {
            A += sgd[i];
            P += sg[i];
        }
        s_a[wave][kk] = A;
        s_p[wave][kk] = P;
        tot += A;
    }
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) tot += __shfl_xor(tot, off);
    __syncthreads();
    if (t >= a.n_tokens) return;
    float* row = D + t * ldd;
#pragma unroll
    for (int j = 0; j < E; ++j) {
        const int i = lane + 64 * j;
        if (i >= M) continue;
        const int kk = s_grp[i];
        const float P = s_p[wave][kk];
        // a group without mass (no candidate, or underflow) has g = 0 throughout
        row[i] = P > 0.f ? sgd[i] - g[j] / P * s_a[wave][kk] : sgd[i];
    }
    for (int i = M + lane; i < ldd; i += 64) row[i] = i < M + K ? s_a[wave][i - M] - s_p[wave][i - M] * tot : 0.f;
}

// value r of column c of the stacked gate weights (local rows, then group rows)
template <typename T>
__device__ __forceinline__ const T* gate_row(const GateBackwardArgs& a, int r) {
    return r < a.n_experts ? static_cast<const T*>(a.w_local) + static_cast<int64_t>(r) * a.d
                           : static_cast<const T*>(a.w_global) + static_cast<int64_t>(r - a.n_experts) * a.d;
}

// d_x [T][d] = D W: 16 tokens x 64 columns a wave, 4 waves side by side
template <typename T>
__global__ __launch_bounds__(256) void gate_dx_kernel(GateBackwardArgs a, const float* D, int ldd) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int l16 = lane & 15, lg = lane >> 4;
    const int R = a.n_experts + a.n_groups;
    const int c0 = (blockIdx.y * 4 + wave) * 64;
    if (c0 >= a.d) return;
    const int64_t t = static_cast<int64_t>(blockIdx.x) * 16 + l16;
    const float* drow = D + min(t, static_cast<int64_t>(a.n_tokens) - 1) * ldd;
    f32x4 acc[4];
#pragma unroll
    for (int b = 0; b < 4; ++b) acc[b] = f32x4{0.f, 0.f, 0.f, 0.f};
    for (int r0 = 0; r0 < R; r0 += 4) {
        const int r = r0 + lg;
        const float dv = drow[r];  // ldd is a multiple of 16: zeros past R
        const T* w = gate_row<T>(a, min(r, R - 1)) + c0 + l16;
#pragma unroll
        for (int b = 0; b < 4; ++b)
            acc[b] = __builtin_amdgcn_mfma_f32_16x16x4f32(r < R ? Elem<T>::to_f32(w[16 * b]) : 0.f, dv, acc[b], 0, 0, 0);
    }
    if (t >= a.n_tokens) return;
    T* out = static_cast<T*>(a.d_x) + t * a.d + c0 + 4 * lg;
#pragma unroll
    for (int b = 0; b < 4; ++b)
#pragma unroll
        for (int i = 0; i < 4; ++i) out[16 * b + i] = Elem<T>::from_f32(acc[b][i]);
}

// part[chunk][r][c] = sum over the chunk's tokens of D[t][r] X[t][c]: 16 columns and every r a wave
template <typename T, int NRB>
__global__ __launch_bounds__(256) void gate_dw_kernel(GateBackwardArgs a, const float* D, int ldd, int chunk, float* part) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int l16 = lane & 15, lg = lane >> 4;
    const int c0 = (blockIdx.x * 4 + wave) * 16;
    const int64_t t0 = static_cast<int64_t>(blockIdx.y) * chunk;
    const int64_t t1 = min(t0 + chunk, static_cast<int64_t>(a.n_tokens));
    const T* x = static_cast<const T*>(a.x) + c0 + l16;
    f32x4 acc[NRB];
#pragma unroll
    for (int b = 0; b < NRB; ++b) acc[b] = f32x4{0.f, 0.f, 0.f, 0.f};
    for (int64_t t = t0; t < t1; t += 4) {
        const int64_t tt = t + lg;
        const bool in = tt < t1;
        const int64_t tc = in ? tt : t1 - 1;
        const float xv = in ? Elem<T>::to_f32(x[tc * a.d]) : 0.f;
        const float* drow = D + tc * ldd + l16;
#pragma unroll
        for (int b = 0; b < NRB; ++b)
            if (16 * b < ldd) acc[b] = __builtin_amdgcn_mfma_f32_16x16x4f32(xv, in ? drow[16 * b] : 0.f, acc[b], 0, 0, 0);
    }
    float* out = part + static_cast<int64_t>(blockIdx.y) * ldd * a.d;
#pragma unroll
    for (int b = 0; b < NRB; ++b)
        if (16 * b < ldd) *reinterpret_cast<f32x4*>(out + static_cast<int64_t>(16 * b + l16) * a.d + c0 + 4 * lg) = acc[b];
}

// column sums of D over the chunk's tokens
__global__ __launch_bounds__(320) void gate_db_kernel(const float* D, int ldd, int n_tokens, int chunk, float* part) {
    const int r = threadIdx.x;
    if (r >= ldd) return;
    const int64_t t0 = static_cast<int64_t>(blockIdx.x) * chunk, t1 = min(t0 + chunk, static_cast<int64_t>(n_tokens));
    float s = 0.f;
#pragma unroll 8
    for (int64_t t = t0; t < t1; ++t) s += D[t * ldd + r];
    part[static_cast<int64_t>(blockIdx.x) * ldd + r] = s;
}

// the chunks' sums in order: rows r of 4 columns a thread, then the biases
__global__ __launch_bounds__(256) void gate_dw_sum_kernel(GateBackwardArgs a, const float* part, const float* bpart,
                                                          int ldd, int chunks) {
    const int M = a.n_experts, R = M + a.n_groups;
    const int64_t quads = static_cast<int64_t>(R) * (a.d / 4);
    const int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
    if (a.d_w_local && i < quads) {
        const int r = static_cast<int>(i / (a.d / 4));
        const int c = static_cast<int>(i % (a.d / 4)) * 4;
        f32x4 s = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
        for (int j = 0; j < chunks; ++j)
            s += *reinterpret_cast<const f32x4*>(part + (static_cast<int64_t>(j) * ldd + r) * a.d + c);
        float* dst = r < M ? a.d_w_local + static_cast<int64_t>(r) * a.d : a.d_w_global + static_cast<int64_t>(r - M) * a.d;
        *reinterpret_cast<f32x4*>(dst + c) = s;
    }
    if (blockIdx.x == 0)
        for (int r = threadIdx.x; r < R; r += 256) {
            double s = 0.0;
            for (int j = 0; j < chunks; ++j) s += bpart[static_cast<int64_t>(j) * ldd + r];
            float* dst = r < M ? a.d_b_local : a.d_b_global;
            if (dst) dst[r < M ? r : r - M] = static_cast<float>(s);
        }
}

// Token chunks of d_W: about two workgroups a CU over the column tiles, 64 tokens or more each
int dw_chunks(int n_tokens, int d) {
    const int want = std::max(1, 512 / std::max(1, d / 64));
    return std::max(1, std::min(want, (n_tokens + 63) / 64));
}

struct GateBackwardWs {
    size_t D, part, bpart, total;
};

GateBackwardWs gate_backward_ws(int n_tokens, int d, int R) {
    const size_t ldd = padded_rows(R), ch = dw_chunks(n_tokens, d);
    auto up = [](size_t n) { return (n + 255) / 256 * 256; };
    GateBackwardWs w{};
    size_t o = 0;
    w.D = o; o += up(static_cast<size_t>(n_tokens) * ldd * 4);
    w.part = o; o += up(ch * ldd * d * 4);
    w.bpart = o; o += up(ch * ldd * 4);
    w.total = o;
    return w;
}

template <typename T>
hipError_t gate_backward(const GateBackwardArgs& a, hipStream_t s) {
    const int R = a.n_experts + a.n_groups, ldd = padded_rows(R);
    const GateBackwardWs w = gate_backward_ws(a.n_tokens, a.d, R);
    char* base = static_cast<char*>(a.ws);
    float* D = reinterpret_cast<float*>(base + w.D);
    float* part = reinterpret_cast<float*>(base + w.part);
    float* bpart = reinterpret_cast<float*>(base + w.bpart);
    const int chunks = a.n_tokens ? dw_chunks(a.n_tokens, a.d) : 0;
    const int chunk = chunks ? (a.n_tokens + chunks - 1) / chunks : 0;
    hipError_t e = hipSuccess;
    if (a.n_tokens) {
        ProfileScope prof(kLogitGradName, s);
        hipLaunchKernelGGL(gate_logit_grad_kernel, dim3((a.n_tokens + kGbTok - 1) / kGbTok), dim3(64 * kGbTok), 0, s, a, D, ldd);
        e = hipGetLastError();
    }
    if (e == hipSuccess && a.n_tokens && a.d_x) {
        ProfileScope prof(kDxName, s);
        hipLaunchKernelGGL(gate_dx_kernel<T>, dim3((a.n_tokens + 15) / 16, (a.d + 255) / 256), dim3(256), 0, s, a, D, ldd);
        e = hipGetLastError();
    }
    if (!a.d_w_local && !a.d_b_local && !a.d_b_global) return e;
    if (e == hipSuccess && a.n_tokens && a.d_w_local) {
        ProfileScope prof(kDwName, s);
        auto go = [&](auto kernel) {
            hipLaunchKernelGGL(kernel, dim3(a.d / 64, chunks), dim3(256), 0, s, a, D, ldd, chunk, part);
        };
        const int nrb = ldd / 16;
        if (nrb <= 1) go(gate_dw_kernel<T, 1>);
        else if (nrb <= 2) go(gate_dw_kernel<T, 2>);
        else if (nrb <= 5) go(gate_dw_kernel<T, 5>);
        else if (nrb <= 10) go(gate_dw_kernel<T, 10>);
        else go(gate_dw_kernel<T, 20>);
        e = hipGetLastError();
    }
    if (e == hipSuccess && a.n_tokens) {
        ProfileScope prof(kDbName, s);
        hipLaunchKernelGGL(gate_db_kernel, dim3(chunks), dim3(320), 0, s, D, ldd, a.n_tokens, chunk, bpart);
        e = hipGetLastError();
    }
    if (e == hipSuccess) {
        ProfileScope prof(kDwSumName, s);
        const int64_t quads = a.d_w_local ? static_cast<int64_t>(R) * (a.d / 4) : 1;
        hipLaunchKernelGGL(gate_dw_sum_kernel, dim3(static_cast<unsigned>((quads + 255) / 256)), dim3(256), 0, s, a, part,
                           bpart, ldd, chunks);
        e = hipGetLastError();
    }
    return e;
}

}  // namespace

size_t balance_ws_bytes(int n_tokens, int n_experts) {
    const size_t chunks = balance_chunks(n_tokens, n_experts);
    return chunks == 1 ? 0 : chunks * (2 * static_cast<size_t>(n_experts) + 1) * 4;
}

hipError_t launch_balance(const BalanceArgs& a, hipStream_t s) {
    const int chunks0 = balance_chunks(a.n_tokens, a.n_experts);
    const int chunk = std::max(1, (a.n_tokens + chunks0 - 1) / chunks0);
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
    hipLaunchKernelGGL(balance_finish_kernel, dim3(1), dim3(1024), 0, s, a, chunks);
    return hipGetLastError();
}

size_t gate_backward_ws_bytes(DType, int n_tokens, int d, int n_experts, int n_groups) {
    return gate_backward_ws(n_tokens, d, n_experts + n_groups).total;
}

hipError_t launch_gate_backward(DType dt, const GateBackwardArgs& a, hipStream_t s) {
    return dt == DType::BF16 ? gate_backward<bf16_t>(a, s) : gate_backward<float>(a, s);
}

}  // namespace ec2moe
