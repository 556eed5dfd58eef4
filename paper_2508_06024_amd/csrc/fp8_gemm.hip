// Grouped and dense products of 8-bit (e4m3) matrices with a float32 scale per 128 values, on the
// gfx950 matrix cores:
//
//   out[p][n] = sum_kb sa[row(p)][kb] sb_e[n / 128][kb] sum_{k in kb} a[row(p)][k] w_e[n][k]
//
// for every row p of group e. v_mfma_f32_16x16x128_f8f6f4 contracts one block of 128 in one
// instruction, so its result is scaled by sa sb and added to the float32 accumulators by four
// fused multiply-adds a lane. Weight rows feed the A operand and token rows the B operand: a lane ends
// with 4 consecutive output columns of one token row. Both operands give lane group g of a wave the
// bytes 16 g .. + 15 and 64 + 16 g .. + 15 of the block; any assignment that both share covers it.
#include "device_common.h"
#include "fp8.h"
#include "gemm_tiles.h"

namespace ec2moe {
namespace {

typedef int i32x8 __attribute__((ext_vector_type(8)));

__device__ __forceinline__ i32x8 frag(uint4 lo, uint4 hi) {
    return i32x8{static_cast<int>(lo.x), static_cast<int>(lo.y), static_cast<int>(lo.z), static_cast<int>(lo.w),
                 static_cast<int>(hi.x), static_cast<int>(hi.y), static_cast<int>(hi.z), static_cast<int>(hi.w)};
}

__device__ __forceinline__ f32x4 mfma8(i32x8 a, i32x8 b) {
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, f32x4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0, 0, 0, 0);
}

template <typename TO>
__device__ __forceinline__ void store_run(TO* dst, f32x4 v, int left, bool whole) {
    if (whole) {  // four columns, the run aligned
        if constexpr (sizeof(TO) == 4) {
            *reinterpret_cast<f32x4*>(dst) = v;
        } else {
            uint2 o;
            o.x = static_cast<uint32_t>(f32_to_bf16(v[0])) | (static_cast<uint32_t>(f32_to_bf16(v[1])) << 16);
            o.y = static_cast<uint32_t>(f32_to_bf16(v[2])) | (static_cast<uint32_t>(f32_to_bf16(v[3])) << 16);
            *reinterpret_cast<uint2*>(dst) = o;
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (i < left) dst[i] = Elem<TO>::from_f32(v[i]);
}

// A tile of 16 MT token rows and 16 NT weight rows (SwiGLU: NT gate and NT up blocks) by WAVES waves that
// take every WAVES-th block of K, fragments straight from memory; their sums meet in LDS and are added
// in wave order.
template <typename TO, int MT, int NT, int WAVES, Epilogue EPI>
__global__ __launch_bounds__(64 * WAVES) void fp8_skinny_kernel(Fp8GemmArgs p) {
    constexpr bool SWIGLU = EPI == Epilogue::SwiGLU;
    constexpr int NB = SWIGLU ? 2 * NT : NT;  // weight blocks
    constexpr int TM = 16 * MT, TN = 16 * NT;
    __shared__ f32x4 red[WAVES][NB * MT][64];
    TileInfo ti;
    const int ntn = (p.N + TN - 1) / TN;
    if (!find_tile<TM>(p, ntn, ti)) return;
    const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
    const int l16 = lane & 15, lg = lane >> 4;
    const int nkb = p.K / kFp8Block;
    const int n0 = ti.nt * TN;

    const uint8_t* wrow[NB];
    const float* wscale[NB];
    const uint8_t* wg = p.b + static_cast<int64_t>(ti.group) * p.b_rows * p.K;
    const float* sg = p.b_scale + static_cast<int64_t>(ti.group) * ((p.b_rows + kFp8Block - 1) / kFp8Block) * nkb;
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
        const int r0 = SWIGLU && nb >= NT ? p.N + n0 + (nb - NT) * 16 : n0 + nb * 16;
        const int last = p.b_rows - 1;
        wrow[nb] = wg + static_cast<int64_t>(min(r0 + l16, last)) * p.K + lg * 16;
        wscale[nb] = sg + static_cast<int64_t>(min(r0, last) / kFp8Block) * nkb;
    }
    const uint8_t* trow[MT];
    const float* tscale[MT];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
        const int64_t pos = ti.row0 + min(mt * 16 + l16, ti.valid - 1);
        const int64_t src = p.row_index ? p.row_index[pos] : pos;
        trow[mt] = p.a + src * p.K + lg * 16;
        tscale[mt] = p.a_scale + src * nkb;
    }
    f32x4 acc[NB][MT];
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) acc[nb][mt] = f32x4{0.f, 0.f, 0.f, 0.f};

    for (int kb = wave; kb < nkb; kb += WAVES) {
        const int64_t off = static_cast<int64_t>(kb) * kFp8Block;
        i32x8 fw[NB], ft[MT];
        float sw[NB], st[MT];
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
            fw[nb] = frag(ldg16(wrow[nb] + off), ldg16(wrow[nb] + off + 64));
            sw[nb] = wscale[nb][kb];
        }
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
            ft[mt] = frag(ldg16(trow[mt] + off), ldg16(trow[mt] + off + 64));
            st[mt] = tscale[mt][kb];
        }
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) {
                const f32x4 part = mfma8(fw[nb], ft[mt]);
                const float s = sw[nb] * st[mt];
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[nb][mt][i] = fmaf(part[i], s, acc[nb][mt][i]);
            }
    }
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) red[wave][nb * MT + mt][lane] = acc[nb][mt];
    __syncthreads();
    auto total = [&](int blk) {
        f32x4 v = red[0][blk][lane];
#pragma unroll
        for (int w = 1; w < WAVES; ++w) v += red[w][blk][lane];
        return v;
    };
    TO* out = static_cast<TO*>(p.out);
    for (int blk = wave; blk < NT * MT; blk += WAVES) {
        const int nb = blk / MT, mt = blk % MT;
        f32x4 v = total(blk);
        if constexpr (SWIGLU) {
            const f32x4 u = total(NT * MT + blk);
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = silu(v[i]) * u[i];
        } else if constexpr (EPI == Epilogue::ReLU) {
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = v[i] < 0.f ? 0.f : v[i];
        }
        const int r = mt * 16 + l16, c = n0 + nb * 16 + 4 * lg;
        if (r < ti.valid && c < p.N)
            store_run(out + (ti.row0 + r) * p.N + c, v, p.N - c, c + 4 <= p.N && p.N % 4 == 0);
    }
}

// Tiles of a launch at most: a group of r rows has ceil(r / TM) <= r / TM + 1 of them per column tile.
int64_t max_tiles(const Fp8GemmArgs& a, int tm, int tn) {
    const int64_t mt = a.seg ? a.rows / tm + std::min<int64_t>(a.rows, a.n_groups) : (a.rows + tm - 1) / tm;
    return mt * ((a.N + tn - 1) / tn);
}

template <typename TO, int MT, int NT, int WAVES, Epilogue EPI>
hipError_t run_skinny(const Fp8GemmArgs& a, hipStream_t s) {
    const int64_t grid = (max_tiles(a, 16 * MT, 16 * NT) + kXcds - 1) / kXcds * kXcds;
    if (grid == 0) return hipSuccess;
    ProfileScope prof(a.name, s);
    hipLaunchKernelGGL((fp8_skinny_kernel<TO, MT, NT, WAVES, EPI>), dim3(static_cast<unsigned>(grid)), dim3(64 * WAVES), 0, s,
                       a);
    return hipGetLastError();
}

template <typename TO, Epilogue EPI>
hipError_t dispatch(const Fp8GemmArgs& a, hipStream_t s) {
    constexpr int NT = EPI == Epilogue::SwiGLU ? 2 : 4;
    if (a.rows / std::max(1, a.n_groups) >= 16) return run_skinny<TO, 4, NT, 4, EPI>(a, s);
    return run_skinny<TO, 1, NT, 4, EPI>(a, s);
}

}  // namespace

bool fp8_gemm_fits(int64_t rows, int n_groups, int64_t n) {
    Fp8GemmArgs a{};
    a.rows = rows;
    a.n_groups = n_groups;
    a.N = static_cast<int>(n);
    int seg = 0;
    a.seg = &seg;
    return max_tiles(a, 16, 32) < (int64_t(1) << 23);  // workgroups of 256 threads of a launch: 2^32 threads at most
}

hipError_t launch_fp8_gemm(Epilogue epi, DType out_type, const Fp8GemmArgs& a, hipStream_t s) {
    const bool f32 = out_type == DType::F32;
    switch (epi) {
        case Epilogue::SwiGLU: return dispatch<float, Epilogue::SwiGLU>(a, s);
        case Epilogue::ReLU: return dispatch<float, Epilogue::ReLU>(a, s);
        default: return f32 ? dispatch<float, Epilogue::Store>(a, s) : dispatch<bf16_t, Epilogue::Store>(a, s);
    }
}

}  // namespace ec2moe
