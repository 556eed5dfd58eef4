// Quantisation to 8-bit floating point (e4m3) with a float32 scale for each block of 128 columns of
// a row, or of 128 x 128 values of a weight matrix, for gfx950.
//
//   amax = max(max |x|, 2^-100), scale = amax / 448, q = e4m3(448 x / amax)
//
// (the rounding itself: fp8_device.h). Memory-bound: one pass, every block's values stay in registers between its maximum
// and its rounding; 1.1 GB of weights 206 us, 5.4 TB/s.
#include "device_common.h"
#include "fp8.h"
#include "fp8_device.h"

namespace ec2moe {
namespace {

template <typename T, int U>
__global__ __launch_bounds__(256) void quantize_rows_kernel(const T* __restrict__ x, int64_t n_blocks,
                                                            uint8_t* __restrict__ q, float* __restrict__ scale) {
    quantize_rows<T, U>(x, n_blocks, q, scale, static_cast<int64_t>(blockIdx.x) * 4 + (threadIdx.x >> 6));
}

// A scale per 128 x 128 block: a workgroup per block, 16 lanes a row, 16 rows a pass.
template <typename T>
__global__ __launch_bounds__(256) void quantize_blocks_kernel(const T* __restrict__ x, int rows, int cols, int col_blocks,
                                                              int row_blocks, uint8_t* __restrict__ q,
                                                              float* __restrict__ scale) {
    __shared__ uint32_t s_max[4];
    const int64_t blk = blockIdx.x;  // (matrix, row block, column block)
    const int cb = static_cast<int>(blk % col_blocks);
    const int64_t mr = blk / col_blocks;
    const int rb = static_cast<int>(mr % row_blocks);
    const int64_t mat = mr / row_blocks;
    const int tid = threadIdx.x;
    const int r0 = rb * kFp8Block + tid / 16;
    const int64_t base = (mat * rows + r0) * cols + cb * kFp8Block + (tid & 15) * 8;
    Eight<T> in[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        if (r0 + 16 * i < rows) in[i].load(x + base + static_cast<int64_t>(16 * i) * cols);
        else in[i].clear();
    }
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        float v[8];
        in[i].values(v);
        m = max(m, magnitude_max(v));
    }
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) m = max(m, static_cast<uint32_t>(__shfl_xor(static_cast<int>(m), off)));
    if ((tid & 63) == 0) s_max[tid >> 6] = m;
    __syncthreads();
    m = max(max(s_max[0], s_max[1]), max(s_max[2], s_max[3]));
    const BlockScale bs = block_scale(m);
    if (tid == 0) scale[blk] = bs.scale;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        if (r0 + 16 * i >= rows) break;
        float v[8];
        in[i].values(v);
        *reinterpret_cast<uint2*>(q + base + static_cast<int64_t>(16 * i) * cols) =
            make_uint2(quantize4(v, bs), quantize4(v + 4, bs));
    }
}

template <typename T>
hipError_t run(const T* x, int n_mats, int rows, int cols, int block_rows, uint8_t* q, float* scale, hipStream_t s) {
    const int cb = cols / kFp8Block;
    if (block_rows == 1) {
        const int64_t n = static_cast<int64_t>(n_mats) * rows * cb;
        constexpr int U = 4;
        const int64_t grid = (n + 16 * U - 1) / (16 * U);
        hipLaunchKernelGGL((quantize_rows_kernel<T, U>), dim3(static_cast<unsigned>(grid)), dim3(256), 0, s, x, n, q, scale);
    } else {
        const int rb = (rows + kFp8Block - 1) / kFp8Block;
        const int64_t grid = static_cast<int64_t>(n_mats) * rb * cb;
        hipLaunchKernelGGL((quantize_blocks_kernel<T>), dim3(static_cast<unsigned>(grid)), dim3(256), 0, s, x, rows, cols, cb,
                           rb, q, scale);
    }
    return hipGetLastError();
}

}  // namespace

hipError_t launch_fp8_quantize(DType dt, const void* x, int n_mats, int rows, int cols, int block_rows, void* q,
                               float* scale, hipStream_t s) {
    if (n_mats == 0 || rows == 0) return hipSuccess;
    const char* blocks = "fp8_quantize_blocks";  // weights: outside the layer step
    ProfileScope prof(block_rows != 1 ? blocks : "fp8_quantize_rows", s);
    uint8_t* q8 = static_cast<uint8_t*>(q);
    if (dt == DType::BF16) return run(static_cast<const bf16_t*>(x), n_mats, rows, cols, block_rows, q8, scale, s);
    return run(static_cast<const float*>(x), n_mats, rows, cols, block_rows, q8, scale, s);
}

}  // namespace ec2moe
