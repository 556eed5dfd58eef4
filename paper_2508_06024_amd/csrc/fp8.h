// Interface of the 8-bit (e4m3) quantisation and products (fp8_quant.hip, fp8_gemm.hip).
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "gemm.h"
#include "host_common.h"

namespace ec2moe {

constexpr int kFp8Block = 128;  // values that share a scale

// x [n_mats][rows][cols] -> q, scale per block_rows (1 or 128) x 128 block
hipError_t launch_fp8_quantize(DType dt, const void* x, int n_mats, int rows, int cols, int block_rows, void* q,
                               float* scale, hipStream_t s);

// launch_permute and the quantisation of x [rows][cols] by rows, in one launch where the permutation takes one
hipError_t launch_fp8_permute(const int32_t* topk_idx, int64_t n_assign, int top_k, int n_experts, int32_t* chunk_counts,
                              int32_t* seg_offsets, int32_t* perm_src, int32_t* inv_perm, DType dt, const void* x, int rows,
                              int cols, void* q, float* scale, hipStream_t s);

// out[p][n] = sum_k a[row(p)][k] w_e[n][k] for every row p of group e on the scaled values, row(p) =
// row_index ? row_index[p] : p.
struct Fp8GemmArgs {
    const uint8_t* a;         // [src_rows][K]
    const float* a_scale;     // [src_rows][K / 128]
    const int32_t* row_index; // gather map or null
    const int32_t* seg;       // [groups+1] device segment offsets, or null (dense: one group)
    int n_groups;
    int64_t rows;             // total rows (upper bound for grouped; exact for dense)
    int64_t src_rows;         // rows of a
    const uint8_t* b;         // [groups][b_rows][K]
    const float* b_scale;     // [groups][ceil(b_rows / 128)][K / 128]
    int b_rows;
    int K, N;
    void* out;                // [rows][N]
    float* out_scale;         // [rows][N / 128] (hidden rows, float16 rows)
    float* part;              // fp8_split_scratch_bytes() of scratch, or null: the last round is not split along K
    const char* name;         // kernel name for the timing record
};
// Whether a launch can hold the product's tiles, and 32 bits their offsets: larger ones are refused.
bool fp8_gemm_fits(const Fp8GemmArgs& a);
// out of out_type. Float32 outputs and few rows a group: exact products (through bfloat16); else those of the 8-bit matrix
// core (fp8_device.h).
hipError_t launch_fp8_gemm(DType out_type, const Fp8GemmArgs& a, hipStream_t s);

// Hidden rows of the experts: SwiGLU (weight rows 0..N-1 are the gate branch and N..2N-1 the up branch), silu(gate)
// * up, or ReLU, max(sum, 0); N and K multiples of 128. Quantised by rows from their float32 values to out and
// out_scale, by way of scratch (fp8_hidden_scratch_bytes) where the product's tiles do not hold whole blocks. exact: sums of
// exact products for any number of rows, as of launch_fp8_gemm with float32 outputs.
hipError_t launch_fp8_hidden(Epilogue epi, const Fp8GemmArgs& a, bool exact, float* scratch, hipStream_t s);

// Rows for launch_fp8_combine (N a multiple of 128): float16 with a scale per 128 columns in out_scale where
// fp8_rows_half(), else float32.
bool fp8_rows_half(const Fp8GemmArgs& a);
hipError_t launch_fp8_rows(const Fp8GemmArgs& a, hipStream_t s);
// y[t] (bfloat16) = sum over k slots of w times the rows, which have scales or are float32 (scale null)
hipError_t launch_fp8_combine(const void* rows, const float* scale, const int32_t* inv_perm, const float* w, int n_tokens,
                              int top_k, int d, void* y, hipStream_t s);

// Scratch of a product, from the shape fields of its arguments and whether they have seg and row_index.
size_t fp8_hidden_scratch_bytes(Epilogue epi, const Fp8GemmArgs& a, bool exact);
size_t fp8_split_scratch_bytes(Epilogue epi, const Fp8GemmArgs& a);

}  // namespace ec2moe
