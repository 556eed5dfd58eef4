// Weighted combine of the 8-bit experts' output rows, Eq. 1, for gfx950:
//   y[t] = sum_{j<k} w[t][j] * row[inv_perm[t*k + j]]
// The rows come in float32 (few rows an expert, where their traffic is nothing beside the weights') or, from the 256 x
// 256 tiles, as float16 with a power-of-two scale for each 128 columns of a row: 11 bits in the bytes of bfloat16, whose 8
// would round every row before the sum (1.2e-3 of the result, beside 1.7e-3 for its own rounding to bfloat16).
// Accumulated in float32 in slot order and rounded once; a slot without a row (position -1: its expert id was out of
// range) adds nothing. One wave per token, 8 columns a lane; few tokens also split
// the row over blockIdx.y. Memory-bound: 8192 tokens of 2048, 6 slots, 37 us.
#include "device_common.h"
#include "fp8.h"

namespace ec2moe {
namespace {

constexpr int kTokens = 4;  // waves of a workgroup, a token each

// KMAX slots, all of them in use up to 8 (MORE: top_k of them, between 9 and 16). NT: the streaming cache policy.
template <bool HALF, int KMAX, int B, bool NT, bool MORE>
__global__ __launch_bounds__(64 * kTokens) void fp8_combine_kernel(const void* __restrict__ rows, const float* __restrict__ scale,
                                                                   const int32_t* __restrict__ inv_perm,
                                                                   const float* __restrict__ w, int n_tokens, int top_k, int d,
                                                                   bf16_t* __restrict__ y) {
    constexpr int W = HALF ? 1 : 2;  // 16-byte loads of 8 columns
    const int lane = threadIdx.x & 63;
    const int t = blockIdx.x * kTokens + (threadIdx.x >> 6);
    if (t >= n_tokens) return;
    int my_pos = 0;
    float my_w = 0.f;
    if (lane < top_k) {
        my_pos = inv_perm[static_cast<int64_t>(t) * top_k + lane];
        my_w = w[static_cast<int64_t>(t) * top_k + lane];
    }
    int pos[KMAX];
    float wt[KMAX];
#pragma unroll
    for (int j = 0; j < KMAX; ++j) {
        pos[j] = __builtin_amdgcn_readlane(my_pos, j);
        wt[j] = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(my_w), j));
    }
    const int chunks = d / 8, per = chunks / gridDim.y;  // gridDim.y divides chunks
    const int cbeg = blockIdx.y * per, cend = cbeg + per;
    for (int c0 = cbeg + lane; c0 < cend; c0 += 64 * B) {
        uint4 v[B][KMAX][W];
        float s[B][KMAX];
#pragma unroll
        for (int b = 0; b < B; ++b) {
            const int c = std::min(c0 + 64 * b, cend - 1);
#pragma unroll
            for (int j = 0; j < KMAX; ++j) {
                if (MORE && j >= top_k) continue;
                const int64_t row = std::max(pos[j], 0);
                if constexpr (HALF) {
                    const uint16_t* src = static_cast<const uint16_t*>(rows) + row * d + c * 8;
                    v[b][j][0] = NT ? ldg16_nt(src) : ldg16(src);
                    s[b][j] = scale[row * (d / kFp8Block) + c / (kFp8Block / 8)];
                } else {
#pragma unroll
                    for (int q = 0; q < W; ++q) v[b][j][q] = ldg16(static_cast<const float*>(rows) + row * d + c * 8 + 4 * q);
                }
            }
        }
#pragma unroll
        for (int b = 0; b < B; ++b) {
            const int c = c0 + 64 * b;
            if (c >= cend) break;
            float acc[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) acc[i] = 0.f;
#pragma unroll
            for (int j = 0; j < KMAX; ++j) {
                if ((MORE && j >= top_k) || pos[j] < 0) continue;  // uniform
                if constexpr (HALF) {
                    const _Float16* h = reinterpret_cast<const _Float16*>(&v[b][j][0]);
                    const float f = wt[j] * s[b][j];  // s a power of two
#pragma unroll
                    for (int i = 0; i < 8; ++i) acc[i] = fmaf(f, static_cast<float>(h[i]), acc[i]);
                } else {
                    const float* f = reinterpret_cast<const float*>(&v[b][j][0]);
#pragma unroll
                    for (int i = 0; i < 8; ++i) acc[i] = fmaf(wt[j], f[i], acc[i]);
                }
            }
            uint32_t o[4];
#pragma unroll
            for (int i = 0; i < 4; ++i)
                o[i] = static_cast<uint32_t>(f32_to_bf16(acc[2 * i])) | static_cast<uint32_t>(f32_to_bf16(acc[2 * i + 1])) << 16;
            bf16_t* dst = y + static_cast<int64_t>(t) * d + c * 8;
            if (NT) stg16_nt(dst, make_uint4(o[0], o[1], o[2], o[3]));
            else stg16(dst, make_uint4(o[0], o[1], o[2], o[3]));
        }
    }
}

template <bool HALF>
void run(const void* rows, const float* scale, const int32_t* inv_perm, const float* w, int n_tokens, int top_k, int d, void* y,
         hipStream_t s) {
    // row ranges of at least 64 chunks while the token waves number fewer than 1024
    const int chunks = d / 8;
    int split = 1;
    while (n_tokens * split * 2 <= 1024 && chunks % (split * 2) == 0 && chunks / (split * 2) >= 64) split *= 2;
    auto go = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, dim3((n_tokens + kTokens - 1) / kTokens, split), dim3(64 * kTokens), 0, s, rows, scale, inv_perm,
                           w, n_tokens, top_k, d, static_cast<bf16_t*>(y));
    };
    switch (top_k) {
        case 1: go(fp8_combine_kernel<HALF, 1, 4, false, false>); break;
        case 2: go(fp8_combine_kernel<HALF, 2, 2, false, false>); break;
        case 3: go(fp8_combine_kernel<HALF, 3, 1, false, false>); break;
        case 4: go(fp8_combine_kernel<HALF, 4, 1, false, false>); break;
        case 5: go(fp8_combine_kernel<HALF, 5, 1, true, false>); break;
        case 6: go(fp8_combine_kernel<HALF, 6, 1, true, false>); break;
        case 7: go(fp8_combine_kernel<HALF, 7, 1, true, false>); break;
        case 8: go(fp8_combine_kernel<HALF, 8, 1, true, false>); break;
        default: go(fp8_combine_kernel<HALF, 16, 1, true, true>);
    }
}

}  // namespace

hipError_t launch_fp8_combine(const void* rows, const float* scale, const int32_t* inv_perm, const float* w, int n_tokens,
                              int top_k, int d, void* y, hipStream_t s) {
    if (n_tokens == 0) return hipSuccess;
    ProfileScope prof("fp8_combine", s);
    if (scale) run<true>(rows, scale, inv_perm, w, n_tokens, top_k, d, y, s);
    else run<false>(rows, scale, inv_perm, w, n_tokens, top_k, d, y, s);
    return hipGetLastError();
}

}  // namespace ec2moe
