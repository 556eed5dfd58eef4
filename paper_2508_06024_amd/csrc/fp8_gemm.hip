// Grouped and dense products of 8-bit (e4m3) matrices with a float32 scale per 128 values, on the
// gfx950 matrix cores:
//
//   out[p][n] = sum_kb sa[row(p)][kb] sb_e[n / 128][kb] sum_{k in kb} a[row(p)][k] w_e[n][k]
//
// for every row p of group e. A block of 128 is contracted into fresh accumulators, which four fused
// multiply-adds a lane scale by sa sb and add to the float32 sums. Weight rows feed the A operand and
// token rows the B operand: a lane ends with 4 consecutive output columns of one token row.
//
// Three kernels:
//   * fp8_skinny_kernel (few rows a group): a stream of the weights, straight from memory to registers;
//   * fp8_ring_kernel (32- to 128-row tiles): operands through a ring of LDS slabs;
//   * fp8_pp_kernel (256 x 256 tiles, bfloat16 outputs and hidden rows): two groups of waves that alternate between
//     products and memory.
// The first, the ring's 32-row tiles, float32 outputs and a float32 layer's hidden rows multiply exactly, through bfloat16
// (with few rows a group memory is the bound); the others use the 8-bit matrix core, at twice the rate, whose sums are cut
// off as fp8_device.h says.
//
// Measured (means of passes in a row): one row of 4096 x 4096 weights 5.8 us (2.9 TB/s of weights, a launch's length); 32
// tokens through 40 of 64 experts of 4096 -> 1536, 8 a token, 88 us (5.7 TB/s) and 51 (4.9); 8 experts of 4096 -> 14336, 8192
// rows, 978 and 484 us, 2.0 PFLOP/s in and out, the matrix cores busy 57% of the cycles at 1.89 GHz; 49152 rows over 48
// experts of 2048 -> 1408, 346 and 197 us, 1.6 and 1.4 PFLOP/s: 5 to 9 us of every 16 or 11 slabs' round go into the tile's
// end, whose stores all workgroups make at once.
#include "device_common.h"
#include "fp8_device.h"
#include "gemm_tiles.h"

#include <cmath>
#include <cstdio>
#include <type_traits>

namespace ec2moe {
namespace {

typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(4))) float cfloat;  // constant memory
constexpr int kSplitSlots = 256;                         // workgroups of the 256 x 256 kernel, one per CU

__device__ __forceinline__ float relu(float v) { return v < 0.f ? 0.f : v; }  // NaN stays

__device__ __forceinline__ int scale_rows(const Fp8GemmArgs& p) { return (p.b_rows + kFp8Block - 1) / kFp8Block; }

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

// out[mi] of every lane = v of lane 16 mi + lane % 16 (MI 2: the upper half of the wave holds the lower one's values)
template <int MI>
__device__ __forceinline__ void spread(float v, float (&out)[MI]) {
    static_assert(MI == 2 || MI == 4, "a row of the wave per block of 16");
    typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
    const uint32_t u = __float_as_uint(v);
    const u32x2 r = __builtin_amdgcn_permlane16_swap(u, u, false, false);  // rows 0 0 2 2, 1 1 3 3
    if constexpr (MI == 2) {
        out[0] = __uint_as_float(r[0]);
        out[1] = __uint_as_float(r[1]);
    } else {
        const u32x2 e = __builtin_amdgcn_permlane32_swap(r[0], r[0], false, false);  // rows 0 0 0 0, 2 2 2 2
        const u32x2 o = __builtin_amdgcn_permlane32_swap(r[1], r[1], false, false);
        out[0] = __uint_as_float(e[0]);
        out[1] = __uint_as_float(o[0]);
        out[2] = __uint_as_float(e[1]);
        out[3] = __uint_as_float(o[1]);
    }
}

// ------------------------------------------------------------------ few rows
//
// A tile of 16 token rows and 16 output columns (SwiGLU: their gate and up rows) by kFewWaves waves that take every
// kFewWaves-th block of K, fragments straight from memory, kFewDepth blocks of each in flight; their sums meet in LDS and
// are added in wave order.
constexpr int kFewWaves = 8, kFewDepth = 4;
template <typename TO, Epilogue EPI>
__global__ __launch_bounds__(64 * kFewWaves) void fp8_skinny_kernel(Fp8GemmArgs p) {
    constexpr bool SWIGLU = EPI == Epilogue::SwiGLU;
    constexpr int NB = SWIGLU ? 2 : 1;  // weight blocks of 16 rows
    __shared__ f32x4 red[kFewWaves][NB][64];
    TileInfo ti;
    const int ntn = (p.N + 15) / 16;
    if (!find_tile<16>(p, ntn, ti)) return;
    const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
    const int l16 = lane & 15, lg = lane >> 4;
    const int nkb = p.K / kFp8Block;
    const int n0 = ti.nt * 16;

    const uint8_t* wrow[NB];
    const float* wscale[NB];
    const uint8_t* wg = p.b + static_cast<int64_t>(ti.group) * p.b_rows * p.K;
    const float* sg = p.b_scale + static_cast<int64_t>(ti.group) * scale_rows(p) * nkb;
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
        const int r0 = nb * p.N + n0;
        const int last = p.b_rows - 1;
        wrow[nb] = wg + static_cast<int64_t>(min(r0 + l16, last)) * p.K + lg * 16;
        wscale[nb] = sg + static_cast<int64_t>(min(r0, last) / kFp8Block) * nkb;
    }
    const int64_t pos = ti.row0 + min(l16, ti.valid - 1);
    const int64_t src = p.row_index ? p.row_index[pos] : pos;
    const uint8_t* trow = p.a + src * p.K + lg * 16;
    const float* tscale = p.a_scale + src * nkb;
    f32x4 acc[NB];
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) acc[nb] = f32x4{0.f, 0.f, 0.f, 0.f};

    // blocks past the end repeat the last one and are not counted
    for (int kb0 = wave; kb0 < nkb; kb0 += kFewWaves * kFewDepth) {
        i32x8 fw[kFewDepth][NB], ft[kFewDepth];
        float sw[kFewDepth][NB], st[kFewDepth];
#pragma unroll
        for (int u = 0; u < kFewDepth; ++u) {
            const int kb = min(kb0 + u * kFewWaves, nkb - 1);
            const int64_t off = static_cast<int64_t>(kb) * kFp8Block;
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) {
                fw[u][nb] = frag8(ldg16_nt(wrow[nb] + off), ldg16_nt(wrow[nb] + off + 64));
                sw[u][nb] = wscale[nb][kb];
            }
            ft[u] = frag8(ldg16(trow + off), ldg16(trow + off + 64));
            st[u] = tscale[kb];
        }
#pragma unroll
        for (int u = 0; u < kFewDepth; ++u) {
            if (kb0 + u * kFewWaves >= nkb) break;  // uniform
            const Wide wt = widen(ft[u]);
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) {
                const f32x4 part = mfma_wide(widen(fw[u][nb]), wt);
                const float s = sw[u][nb] * st[u];
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[nb][i] = fmaf(part[i], s, acc[nb][i]);
            }
        }
    }
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) red[wave][nb][lane] = acc[nb];
    __syncthreads();
    if (wave > 0) return;
    auto total = [&](int nb) {
        f32x4 v = red[0][nb][lane];
#pragma unroll
        for (int w = 1; w < kFewWaves; ++w) v += red[w][nb][lane];
        return v;
    };
    f32x4 v = total(0);
    if constexpr (SWIGLU) {
        const f32x4 u = total(1);
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = silu(v[i]) * u[i];
    } else if constexpr (EPI == Epilogue::ReLU) {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = relu(v[i]);
    }
    const int c = n0 + 4 * lg;
    if (l16 < ti.valid && c < p.N)
        store_run(static_cast<TO*>(p.out) + (ti.row0 + l16) * p.N + c, v, p.N - c, c + 4 <= p.N && p.N % 4 == 0);
}

// Weight row (within the group's matrix) of tile row n: SwiGLU tiles hold TN/2 gate rows, then the matching up
// rows; rows past the matrix repeat its last one (their columns are not stored).
template <int TN, bool SWIGLU>
__device__ __forceinline__ int weight_row(const Fp8GemmArgs& p, int nt, int n) {
    if (SWIGLU) return n < TN / 2 ? nt * (TN / 2) + n : p.N + nt * (TN / 2) + (n - TN / 2);
    return std::min(nt * TN + n, p.b_rows - 1);
}

// ------------------------------------------------------------------ 32- to 128-row tiles through a ring
//
// Tiles of TM x 128 over the whole K: slabs of one block of 128 (128-byte pieces of each row) go through
// a ring of RING LDS stages filled by buffer_load ... lds, RING - 1 of them in flight behind counted waits
// and one barrier per slab. Four waves of TM x 32, or of 64 x 64 of 128 rows. Chunk c of staged row R sits at c ^ ((R >> 1) & 7).
// STREAM: the weights pass the caches by (each is read once).
// EXACT: products through bfloat16, bound by the conversions (96 a wave a slab for 32 products at 64 rows, 128 for 64 at 128;
// about as long as a product each): 3000 rows in 12 segments, 2048 -> 2001, float32: 52 us with 64 rows, 46 with 128 (0.53
// PFLOP/s). Else the 8-bit core: 8 groups of 400 rows, 2048 -> 2048, 25 us (1.1 PFLOP/s).
template <typename TO, int TM, int RING, Epilogue EPI, bool STREAM, bool EXACT>
__global__ __launch_bounds__(256, 2) void fp8_ring_kernel(Fp8GemmArgs p) {
    constexpr bool SWIGLU = EPI == Epilogue::SwiGLU;
    constexpr int TN = 128;
    constexpr int NLD = (TM + TN) / 32;  // load instructions (8 rows) per wave per slab
    constexpr int WM = TM > 64 ? 2 : 1, WN = 4 / WM;  // waves
    constexpr int MI = TM / WM / 16, NI = TN / WN / 16;
    constexpr int NBK = SWIGLU ? NI / 2 : NI;  // blocks of 16 output columns of a wave
    constexpr int NOUT = SWIGLU ? TN / 2 : TN;
    constexpr int STAGE = (TM + TN) * kFp8Block;
    static_assert((TM + TN) % 32 == 0 && TM % 16 == 0, "whole load instructions");
    static_assert(RING >= 2 && RING <= 4, "ring of 2 to 4 slabs");
    __shared__ __attribute__((aligned(1024))) char lds0[STAGE];
    __shared__ __attribute__((aligned(1024))) char lds1[STAGE];
    __shared__ __attribute__((aligned(1024))) char lds2[RING > 2 ? STAGE : 16];
    __shared__ __attribute__((aligned(1024))) char lds3[RING > 3 ? STAGE : 16];

    const int ntn = (p.N + NOUT - 1) / NOUT;
    TileInfo ti;
    if (!find_tile<TM>(p, ntn, ti)) return;
    int tid = threadIdx.x;
    asm volatile("" : "+v"(tid));
    const int lane = tid & 63, wave = uniform(tid >> 6);
    const int l16 = lane & 15, lg = lane >> 4;
    const int wm = wave % WM, wn = wave / WM;
    const int K = p.K, nkb = K / kFp8Block;

    auto swz = [](int R) { return (R >> 1) & 7; };
    // contiguous token rows: the descriptor starts at the tile, so that offsets stay within 32 bits
    const uint8_t* abase = p.row_index ? p.a : p.a + ti.row0 * K;
    const i32x4 rtok = buffer_rsrc(abase, static_cast<uint32_t>(p.row_index ? p.src_rows * K : static_cast<int64_t>(ti.valid) * K));
    const i32x4 rw = buffer_rsrc(p.b + static_cast<int64_t>(ti.group) * p.b_rows * K,
                                 static_cast<uint32_t>(static_cast<int64_t>(p.b_rows) * K));
    uint32_t voff[NLD];
#pragma unroll
    for (int j = 0; j < NLD; ++j) {
        const int R = 8 * (NLD * wave + j) + lane / 8;
        uint32_t src;
        if (R < TM) {
            const int r = std::min(R, ti.valid - 1);
            src = p.row_index ? static_cast<uint32_t>(p.row_index[ti.row0 + r]) : static_cast<uint32_t>(r);
        } else {
            src = static_cast<uint32_t>(weight_row<TN, SWIGLU>(p, ti.nt, R - TM));
        }
        voff[j] = src * static_cast<uint32_t>(K) + static_cast<uint32_t>(((lane % 8) ^ swz(R)) * 16);
    }
    auto issue = [&](int st, char* slot) {
#pragma unroll
        for (int j = 0; j < NLD; ++j) {
            const bool tok = 8 * (NLD * wave + j) < TM;  // uniform
            lds_void* dst = reinterpret_cast<lds_void*>(reinterpret_cast<uintptr_t>(slot + 1024 * (NLD * wave + j)));
            if (tok) raw_buffer_load_lds(rtok, dst, 16, static_cast<int>(voff[j]), st * kFp8Block, 0, 0);
            else raw_buffer_load_lds(rw, dst, 16, static_cast<int>(voff[j]), st * kFp8Block, 0, STREAM ? 2 : 0);
        }
    };

    // scales: a lane loads the one of token row `lane` of the tile, a slab ahead; one (SwiGLU: two) of the weights for the
    // tile, through the scalar cache
    uint32_t tso;
    {
        const int64_t pos = ti.row0 + std::min(wm * (TM / WM) + lane % (TM / WM), ti.valid - 1);
        tso = static_cast<uint32_t>(p.row_index ? p.row_index[pos] : pos) * static_cast<uint32_t>(4 * nkb);
    }
    const float* sg = p.b_scale + static_cast<int64_t>(ti.group) * scale_rows(p) * nkb;
    const cfloat* wsc0 = (const cfloat*)(sg + static_cast<int64_t>(uniform(weight_row<TN, SWIGLU>(p, ti.nt, 0) / kFp8Block)) * nkb);
    const cfloat* wsc1 =
        (const cfloat*)(sg + static_cast<int64_t>(uniform(weight_row<TN, SWIGLU>(p, ti.nt, TN / 2) / kFp8Block)) * nkb);

    const int soff = (lg ^ swz(l16)) * 16, soff4 = ((4 + lg) ^ swz(l16)) * 16;  // blocks start at multiples of 16 rows
    int foff_t[MI], foff_w[NI];
#pragma unroll
    for (int mi = 0; mi < MI; ++mi) foff_t[mi] = (wm * (TM / WM) + mi * 16 + l16) * kFp8Block;
#pragma unroll
    for (int ni = 0; ni < NI; ++ni)
        foff_w[ni] = (TM + (SWIGLU ? ni / NBK * (TN / 2) : 0) + (wn * NBK + ni % NBK) * 16 + l16) * kFp8Block;
    f32x4 acc[NI][MI];
#pragma unroll
    for (int ni = 0; ni < NI; ++ni)
#pragma unroll
        for (int mi = 0; mi < MI; ++mi) acc[ni][mi] = f32x4{0.f, 0.f, 0.f, 0.f};

    float st_next, sw_next[2];
    auto load_scales = [&](int st) {
        st_next = *reinterpret_cast<const float*>(reinterpret_cast<const char*>(p.a_scale + st) + tso);
        sw_next[0] = wsc0[st];
        if (SWIGLU) sw_next[1] = wsc1[st];
    };
    auto step = [&](int st, const char* cur, char* refill) {
        if (st >= nkb) return;
        // slabs issued after this one stay in flight
        const int later = std::min(RING - 2, nkb - 1 - st);
        if (RING > 3 && later >= 2) __builtin_amdgcn_s_waitcnt(vmcnt_imm(2 * NLD));
        else if (RING > 2 && later >= 1) __builtin_amdgcn_s_waitcnt(vmcnt_imm(NLD));
        else __builtin_amdgcn_s_waitcnt(vmcnt_imm(0));
        // every wave's loads of this slab have landed, and every wave is done with the previous
        // slab, whose slot is refilled next
        __builtin_amdgcn_sched_barrier(0);
        asm volatile("s_barrier" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
        float s[SWIGLU ? 2 : 1][MI];
        spread(st_next * sw_next[0], s[0]);
        if (SWIGLU) spread(st_next * sw_next[1], s[SWIGLU ? 1 : 0]);
        if (st + 1 < nkb) load_scales(st + 1);
        if (st + RING - 1 < nkb) issue(st + RING - 1, refill);
        i32x8 ft[MI], fw[NI];
#pragma unroll
        for (int ni = 0; ni < NI; ++ni)
            fw[ni] = frag8(*reinterpret_cast<const uint4*>(cur + foff_w[ni] + soff),
                           *reinterpret_cast<const uint4*>(cur + foff_w[ni] + soff4));
#pragma unroll
        for (int mi = 0; mi < MI; ++mi)
            ft[mi] = frag8(*reinterpret_cast<const uint4*>(cur + foff_t[mi] + soff),
                           *reinterpret_cast<const uint4*>(cur + foff_t[mi] + soff4));
        auto add = [&](int ni, int mi, f32x4 part) {
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[ni][mi][i] = fmaf(part[i], s[ni / NBK][mi], acc[ni][mi][i]);
        };
        // the products of a token block in NI chains side by side, then the multiply-adds of the block before
        Wide ww[NI];
        if constexpr (EXACT)
#pragma unroll
            for (int ni = 0; ni < NI; ++ni) ww[ni] = widen(fw[ni]);
        f32x4 part[2][NI];
#pragma unroll
        for (int mi = 0; mi <= MI; ++mi) {
            if (mi < MI) {
                const i32x8 t = ft[mi < MI ? mi : 0];
                if constexpr (EXACT) {
                    const Wide wt = widen(t);
#pragma unroll
                    for (int ni = 0; ni < NI; ++ni) part[mi & 1][ni] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int i = 0; i < 4; ++i)
#pragma unroll
                        for (int ni = 0; ni < NI; ++ni)
                            part[mi & 1][ni] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ww[ni].v[i], wt.v[i], part[mi & 1][ni], 0, 0, 0);
                } else {
#pragma unroll
                    for (int ni = 0; ni < NI; ++ni) part[mi & 1][ni] = mfma8(fw[ni], t);
                }
            }
            if (mi > 0)
#pragma unroll
                for (int ni = 0; ni < NI; ++ni) add(ni, mi - 1, part[(mi - 1) & 1][ni]);
        }
    };
    load_scales(0);
    issue(0, lds0);
    if (RING > 2 && nkb > 1) issue(1, lds1);
    if (RING > 3 && nkb > 2) issue(2, lds2);
    for (int st = 0; st < nkb; st += RING) {
        if constexpr (RING == 2) {
            step(st, lds0, lds1);
            step(st + 1, lds1, lds0);
        } else if constexpr (RING == 3) {
            step(st, lds0, lds2);
            step(st + 1, lds1, lds0);
            step(st + 2, lds2, lds1);
        } else {
            step(st, lds0, lds3);
            step(st + 1, lds1, lds0);
            step(st + 2, lds2, lds1);
            step(st + 3, lds3, lds2);
        }
    }
    TO* out = static_cast<TO*>(p.out);
    const bool runs = p.N % 4 == 0;
#pragma unroll
    for (int mi = 0; mi < MI; ++mi) {
        const int r = wm * (TM / WM) + mi * 16 + l16;
        if (r >= ti.valid) continue;
        TO* orow = out + (ti.row0 + r) * p.N;
#pragma unroll
        for (int ni = 0; ni < NBK; ++ni) {
            const int c = ti.nt * NOUT + (wn * NBK + ni) * 16 + 4 * lg;
            f32x4 v = acc[ni][mi];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (SWIGLU) v[i] = silu(v[i]) * acc[SWIGLU ? ni + NBK : ni][mi][i];
                else if (EPI == Epilogue::ReLU) v[i] = relu(v[i]);
            }
            if (c < p.N) store_run(orow + c, v, p.N - c, c + 4 <= p.N && runs);
        }
    }
}

// ------------------------------------------------------------------ 256 x 256 tiles
//
// Waves 0-3 (group 0, token loaders) and waves 4-7 (group 1, weight loaders) sit one per SIMD each; the
// groups alternate between a compute phase (the 32 products of one slab of 128 k, at raised priority) and a
// memory phase (fragment reads of the next slab, buffer loads), with a workgroup barrier between phases, so on
// every SIMD one wave issues products while the other waits on memory.
//   group 0, slab s: issue token rows of slab s+1 | read slab s | barrier | products of slab s |
//                    wait own loads | barrier
//   group 1, slab s: products of slab s-1 | barrier | issue weight rows of slab s+2 into the slot of
//                    slab s-1, read slab s | wait loads of slab s+1 | barrier
// Token rows sit in two 32 KB slots and weight rows in three, so that every slot is refilled only after a
// barrier that follows the last read of it by any wave. A wave holds 4 x 8 blocks of 16 x 16 (128 float32
// sums). The memory phase reads the token fragments and the first weight blocks' fragments; a weight
// block's 32 bytes a lane are read AHEAD blocks of products ahead, behind the same barriers. Scales are loaded a slab
// ahead and before the slab loads of the phase, so that its counted waits cover them. The 128
// scaling multiply-adds of a slab issue under its products (16 of every 32 cycles).
// EPI Store writes bfloat16 rows, or (HALF) float16 rows with a power-of-two scale for each 128 columns, a wave's. SwiGLU
// and ReLU quantise: a tile holds one (ReLU: two) whole blocks of 128 hidden columns of each row, whose largest value
// meets across the lanes and, with SwiGLU, the two waves of the row.
template <Epilogue EPI, bool HALF = false>
__global__ __launch_bounds__(512, 1) void fp8_pp_kernel(Fp8GemmArgs p) {
    constexpr bool SWIGLU = EPI == Epilogue::SwiGLU;
    constexpr bool QUANT = EPI != Epilogue::Store;
    constexpr int TM = 256, TN = 256, WM = 4, WN = 2, NW = 8;
    constexpr int MI = TM / WM / 16;           // 4 token blocks of 16 per wave
    constexpr int NI = TN / WN / 16;           // 8 weight blocks of 16 per wave
    constexpr int NOUT = SWIGLU ? TN / 2 : TN;
    constexpr int RB = kFp8Block;
    constexpr int SLOT = TM * RB;              // 32 KB: the token rows, or the weight rows, of one slab
    constexpr int WROWS = (TM + TN) / NW;      // 64 rows a wave loads
    constexpr int LOADS = WROWS / 8;           // 8
    constexpr int WTOK = TM / WM;

    __shared__ __attribute__((aligned(1024))) char t0[SLOT];
    __shared__ __attribute__((aligned(1024))) char t1[SLOT];
    __shared__ __attribute__((aligned(1024))) char w0[SLOT];
    __shared__ __attribute__((aligned(1024))) char w1[SLOT];
    __shared__ __attribute__((aligned(1024))) char w2[SLOT];

    const int ntn = (p.N + NOUT - 1) / NOUT;
    const int K = p.K, nk_all = K / kFp8Block;
    constexpr int P = kSplitSlots;   // workgroups, one per CU
    constexpr int XW = P / kXcds;
    const SplitPlan sp = split_plan(count_tiles<TM>(p, ntn), P, p.part ? kMaxSplitChunks : 1, nk_all);
    const int rounds = sp.full / P;
    const int wg = blockIdx.x;

    // whole rounds first, each XCD's workgroups stepping through consecutive tiles; then the tail
    for (int it = 0; it <= rounds; ++it) {
    int bid, chunk = 0;
    bool split = false;
    if (it < rounds) {
        bid = (wg % kXcds) * (rounds * XW) + it * XW + wg / kXcds;
    } else {
        if (wg >= sp.tail * sp.S) break;
        bid = sp.full + wg / sp.S;
        chunk = wg % sp.S;
        split = sp.S > 1;
    }
    TileInfo ti;
    if (!tile_of<TM>(p, ntn, bid, ti)) break;
    const int kb = split ? chunk * sp.chunk_slabs : 0;  // first slab of this unit
    const int nk = split ? std::min(nk_all, kb + sp.chunk_slabs) - kb : nk_all;

    int tid = threadIdx.x;
    asm volatile("" : "+v"(tid));
    const int lane = tid & 63;
    const int wave = uniform(tid >> 6);
    const int wm = wave % WM;
    const int wn = wave / WM;                 // also the group
    const bool tok_wave = wave * WROWS < TM;  // group 0
    const uint8_t* abase = p.row_index ? p.a : p.a + ti.row0 * K;
    const uint8_t* bbase = p.b + static_cast<int64_t>(ti.group) * p.b_rows * K;
    const i32x4 rs = tok_wave ? buffer_rsrc(abase, static_cast<uint32_t>(p.row_index ? p.src_rows * K : static_cast<int64_t>(ti.valid) * K))
                              : buffer_rsrc(bbase, static_cast<uint32_t>(static_cast<int64_t>(p.b_rows) * K));
    uint32_t voff[LOADS];
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
        const int row = wave * WROWS + i * 8 + (lane >> 3);
        uint32_t src;
        if (tok_wave) {
            const int r = std::min(row, ti.valid - 1);
            src = p.row_index ? static_cast<uint32_t>(p.row_index[ti.row0 + r]) : static_cast<uint32_t>(r);
        } else {
            src = static_cast<uint32_t>(weight_row<TN, SWIGLU>(p, ti.nt, row - TM));
        }
        voff[i] = src * static_cast<uint32_t>(K) + static_cast<uint32_t>(((lane & 7) ^ ((row >> 1) & 7)) * 16);
        asm volatile("" : "+v"(voff[i]));  // kept as it is: the compiler would hold the 64-bit product
    }
    // this wave's rows of a slab into a token or weight slot (rows 64 (wave & 3) .. + 63 of it)
    auto issue_slab = [&](int ks, char* slot) {
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            lds_void* dst = reinterpret_cast<lds_void*>(
                reinterpret_cast<uintptr_t>(slot + ((wave & 3) * WROWS + i * 8) * RB));
            raw_buffer_load_lds(rs, dst, 16, static_cast<int>(voff[i]), (kb + ks) * RB, 0, 0);
        }
    };

    const int l16 = lane & 15;
    const int lg = lane >> 4;
    const int sw = (l16 >> 1) & 7;
    constexpr int WW = SWIGLU ? TN / 2 / WN : TN / WN;
    const int c0 = (lg ^ sw) * 16, c1 = ((4 + lg) ^ sw) * 16;
    const int off_t = (wm * WTOK + l16) * RB;  // in a token slot
    const int off_w = (wn * WW + l16) * RB;    // in a weight slot
    auto wblk = [](int ni) constexpr {
        if (SWIGLU) {
            return (ni < NI / 2 ? 0 : TN / 2) + (ni % (NI / 2)) * 16;
        }
        return ni * 16;
    };

    // Scales: a lane loads the one of row `lane` of the wave's 64 token rows, a slab ahead; those of the wave's
    // weight block (SwiGLU: gate and up) are uniform and come through the scalar cache (written by no kernel that
    // runs now).
    uint32_t tso;
    {
        const int64_t pos = ti.row0 + std::min(wm * WTOK + lane, ti.valid - 1);
        tso = static_cast<uint32_t>(p.row_index ? p.row_index[pos] : pos) * static_cast<uint32_t>(4 * nk_all);
        asm volatile("" : "+v"(tso));
    }
    const float* sg = p.b_scale + static_cast<int64_t>(ti.group) * scale_rows(p) * nk_all;
    const cfloat* ws0 = (const cfloat*)(sg + static_cast<int64_t>(uniform(weight_row<TN, SWIGLU>(p, ti.nt, wn * WW) / kFp8Block)) * nk_all + kb);
    const cfloat* ws1 =
        (const cfloat*)(sg + static_cast<int64_t>(uniform(weight_row<TN, SWIGLU>(p, ti.nt, TN / 2 + wn * WW) / kFp8Block)) * nk_all + kb);
    struct Scales {
        float t, w0, w1;
    };
    auto load_scales = [&](int ks) {
        Scales s;
        s.t = *reinterpret_cast<const float*>(reinterpret_cast<const char*>(p.a_scale + kb + ks) + tso);
        s.w0 = ws0[ks];
        s.w1 = SWIGLU ? ws1[ks] : 0.f;
        return s;
    };
    f32x4 acc[NI][MI];
#pragma unroll
    for (int ni = 0; ni < NI; ++ni)
#pragma unroll
        for (int mi = 0; mi < MI; ++mi) acc[ni][mi] = f32x4{0.f, 0.f, 0.f, 0.f};

    constexpr int AHEAD = 2;
    struct Frags {
        i32x8 a[AHEAD], b[MI];
    };
    auto read_w = [&](const char* wslot, int ni) {
        return frag8(*reinterpret_cast<const uint4*>(wslot + off_w + c0 + wblk(ni) * RB),
                     *reinterpret_cast<const uint4*>(wslot + off_w + c1 + wblk(ni) * RB));
    };
    auto read_slab = [&](const char* tslot, const char* wslot, Frags& f) {
#pragma unroll
        for (int ni = 0; ni < AHEAD; ++ni) f.a[ni] = read_w(wslot, ni);
#pragma unroll
        for (int mi = 0; mi < MI; ++mi)
            f.b[mi] = frag8(*reinterpret_cast<const uint4*>(tslot + off_t + c0 + mi * 16 * RB),
                           *reinterpret_cast<const uint4*>(tslot + off_t + c1 + mi * 16 * RB));
    };
    auto mma_slab = [&](const char* wslot, Frags& f, const Scales& s) {
        __builtin_amdgcn_s_setprio(1);
        float sc[SWIGLU ? 2 : 1][MI];
        spread(s.t * s.w0, sc[0]);
        if (SWIGLU) spread(s.t * s.w1, sc[SWIGLU ? 1 : 0]);
        // two products, then the multiply-adds of the two before, in this order: left alone the scheduler
        // raises all products of the slab above them and spills
        constexpr int NP = NI * MI / 2;
        f32x4 part[2][2];
        auto add = [&](int q) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int ni = q * 2 / MI, mi = q * 2 % MI + h;
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    acc[ni][mi][i] = fmaf(part[q & 1][h][i], sc[SWIGLU && ni >= NI / 2 ? 1 : 0][mi], acc[ni][mi][i]);
            }
        };
#pragma unroll
        for (int q = 0; q < NP; ++q) {
            const int ni = q * 2 / MI;
#pragma unroll
            for (int h = 0; h < 2; ++h) part[q & 1][h] = mfma8(f.a[ni % AHEAD], f.b[q * 2 % MI + h]);
            if (q * 2 % MI == MI - 2 && ni + AHEAD < NI) f.a[ni % AHEAD] = read_w(wslot, ni + AHEAD);
            if (q > 0) add(q - 1);
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x002, 4, 0);
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x002, 4, 0);
            __builtin_amdgcn_sched_barrier(0);
        }
        add(NP - 1);
        // the sums are wanted here: the compiler otherwise sinks the multiply-adds past the barrier, into the next
        // phase, and spills the products
#pragma unroll
        for (int ni = 0; ni < NI; ++ni)
#pragma unroll
            for (int mi = 0; mi < MI; ++mi) asm volatile("" : "+v"(acc[ni][mi]));
        __builtin_amdgcn_s_setprio(0);
    };
    auto barrier = [&]() {
        __builtin_amdgcn_sched_barrier(0);
        asm volatile("s_barrier" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
    };

    // slab s: tokens in slot s % 2, weights in slot s % 3 (the loops run six slabs a turn)
    if (nk <= 0) {
        // a chunk past the end of K (whole pairs of slabs a chunk): zeros
    } else if (tok_wave) {
        Scales nxt = load_scales(0);
        issue_slab(0, t0);
        __builtin_amdgcn_s_waitcnt(vmcnt_imm(0));
        barrier();
        auto slab0 = [&](const char* tcur, char* tnxt, const char* wcur, int s) {
            Frags f;
            const Scales sc = nxt;
            nxt = load_scales(std::min(s + 1, nk - 1));
            __builtin_amdgcn_sched_barrier(0);
            if (s + 1 < nk) issue_slab(s + 1, tnxt);
            read_slab(tcur, wcur, f);
            __builtin_amdgcn_s_waitcnt(0xC07F);  // lgkmcnt(0)
            barrier();
            mma_slab(wcur, f, sc);
            __builtin_amdgcn_sched_barrier(0);
            __builtin_amdgcn_s_waitcnt(0x0070);  // token rows of slab s+1 landed
            barrier();
        };
        int s = 0;
        for (; s + 6 <= nk; s += 6) {
            slab0(t0, t1, w0, s);
            slab0(t1, t0, w1, s + 1);
            slab0(t0, t1, w2, s + 2);
            slab0(t1, t0, w0, s + 3);
            slab0(t0, t1, w1, s + 4);
            slab0(t1, t0, w2, s + 5);
        }
        if (s < nk) slab0(t0, t1, w0, s);
        if (s + 1 < nk) slab0(t1, t0, w1, s + 1);
        if (s + 2 < nk) slab0(t0, t1, w2, s + 2);
        if (s + 3 < nk) slab0(t1, t0, w0, s + 3);
        if (s + 4 < nk) slab0(t0, t1, w1, s + 4);
    } else {
        Scales sc, nxt = load_scales(0);
        Frags f;
        __builtin_amdgcn_sched_barrier(0);
        issue_slab(0, w0);
        if (nk > 1) issue_slab(1, w1);
        if (nk > 1) __builtin_amdgcn_s_waitcnt(vmcnt_imm(LOADS));  // own rows of slab 0 landed
        else __builtin_amdgcn_s_waitcnt(vmcnt_imm(0));
        barrier();
        // Memory phase of slab s. The slot refilled in it holds slab s - 1, whose last reads (this group's) were
        // done before the barrier ahead of it: no wave can still be reading it.
        auto fetch = [&](const char* tcur, const char* wcur, char* wfree, int s) {
            barrier();
            sc = nxt;
            if (s + 2 < nk) issue_slab(s + 2, wfree);
            __builtin_amdgcn_sched_barrier(0);
            // after the slab loads: the wait below then leaves it in flight (a load's latency a slab otherwise:
            // gate-up of the layer of 8 experts 1007 us, 967 so)
            nxt = load_scales(std::min(s + 1, nk - 1));
            __builtin_amdgcn_sched_barrier(0);
            read_slab(tcur, wcur, f);
            __builtin_amdgcn_s_waitcnt(0xC07F);  // lgkmcnt(0)
            // weight rows of slab s+1 landed
            if (s + 2 < nk) __builtin_amdgcn_s_waitcnt(vmcnt_imm(LOADS + 1));
            else __builtin_amdgcn_s_waitcnt(vmcnt_imm(1));
            barrier();
        };
        auto slab1 = [&](const char* tcur, const char* wcur, char* wfree, int s) {
            mma_slab(wfree, f, sc);  // slab s - 1, whose weights sit in the slot refilled next
            fetch(tcur, wcur, wfree, s);
        };
        fetch(t0, w0, w2, 0);
        int s = 1;
        for (; s + 6 <= nk; s += 6) {
            slab1(t1, w1, w0, s);
            slab1(t0, w2, w1, s + 1);
            slab1(t1, w0, w2, s + 2);
            slab1(t0, w1, w0, s + 3);
            slab1(t1, w2, w1, s + 4);
            slab1(t0, w0, w2, s + 5);
        }
        if (s < nk) slab1(t1, w1, w0, s);
        if (s + 1 < nk) slab1(t0, w2, w1, s + 1);
        if (s + 2 < nk) slab1(t1, w0, w2, s + 2);
        if (s + 3 < nk) slab1(t0, w1, w0, s + 3);
        if (s + 4 < nk) slab1(t1, w2, w1, s + 4);
        const int last = (nk - 1) % 3;
        mma_slab(last == 0 ? w0 : last == 1 ? w1 : w2, f, sc);
    }

    if (split) {
        // float32 sums [TM][TN] (weight rows in tile order) of this chunk of K; lane l holds, per block, weight rows
        // 4 (l / 16) .. + 3 of token row l % 16
        float* part = p.part + static_cast<int64_t>(wg) * TM * TN;
#pragma unroll
        for (int mi = 0; mi < MI; ++mi) {
            const int trow = wm * WTOK + mi * 16 + l16;
#pragma unroll
            for (int ni = 0; ni < NI; ++ni)
                *reinterpret_cast<f32x4*>(part + trow * TN + wn * WW + wblk(ni) + 4 * lg) = acc[ni][mi];
        }
        break;  // the last unit of the workgroup
    }
    // The finished tile is staged in LDS so that the global stores are whole rows: 16 bytes per lane. Token
    // slots are free after the last slab; weight slots once the weight loaders' last products are done.
    if constexpr (QUANT) {
        // Staged row r (NOUT bytes) holds its 16-byte chunk c at c ^ (r % OCH).
        constexpr int OCH = NOUT / 16;
        constexpr int NB = SWIGLU ? NI / 2 : NI;
        uint32_t mx[MI];
#pragma unroll
        for (int mi = 0; mi < MI; ++mi) {
            mx[mi] = 0;
#pragma unroll
            for (int ni = 0; ni < NB; ++ni)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float v = SWIGLU ? silu(acc[ni][mi][e]) * acc[SWIGLU ? ni + NB : ni][mi][e] : relu(acc[ni][mi][e]);
                    acc[ni][mi][e] = v;
                    mx[mi] = max(mx[mi], magnitude(v));
                }
            mx[mi] = max(mx[mi], static_cast<uint32_t>(__shfl_xor(static_cast<int>(mx[mi]), 16)));
            mx[mi] = max(mx[mi], static_cast<uint32_t>(__shfl_xor(static_cast<int>(mx[mi]), 32)));
        }
        if constexpr (SWIGLU) {
            uint32_t* rowmax = reinterpret_cast<uint32_t*>(t1);  // [2][256]
            if (lg == 0)
#pragma unroll
                for (int mi = 0; mi < MI; ++mi) rowmax[wn * TM + wm * WTOK + mi * 16 + l16] = mx[mi];
            __builtin_amdgcn_s_waitcnt(0xC07F);  // lgkmcnt(0)
            barrier();
#pragma unroll
            for (int mi = 0; mi < MI; ++mi) mx[mi] = max(mx[mi], rowmax[(1 - wn) * TM + wm * WTOK + mi * 16 + l16]);
        }
        const int nsb = p.N / kFp8Block;
        const int blk = ti.nt * (NOUT / kFp8Block) + (SWIGLU ? 0 : wn);
#pragma unroll
        for (int mi = 0; mi < MI; ++mi) {
            const int r = wm * WTOK + mi * 16 + l16;
            const BlockScale bs = block_scale(mx[mi]);
            if ((SWIGLU ? wn == 0 : true) && lg == 0 && r < ti.valid && blk < nsb)
                p.out_scale[(ti.row0 + r) * nsb + blk] = bs.scale;
            char* row = (SWIGLU || r < 128 ? t0 : t1) + (SWIGLU ? r : r & 127) * NOUT;
#pragma unroll
            for (int ni = 0; ni < NB; ++ni) {
                float v[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = acc[ni][mi][e];
                const int ch = (wn * (NOUT / WN / 16) + ni) ^ (r % OCH);
                *reinterpret_cast<uint32_t*>(row + ch * 16 + 4 * lg) = quantize4(v, bs);
            }
        }
        __builtin_amdgcn_s_waitcnt(0xC07F);  // lgkmcnt(0)
        barrier();
        constexpr int RPI = 64 / OCH;
        uint8_t* out = static_cast<uint8_t*>(p.out);
#pragma unroll
        for (int j = 0; j < TM / NW / RPI; ++j) {
            const int r = wave * (TM / NW) + j * RPI + lane / OCH;
            const int c = lane % OCH;
            const char* src = (SWIGLU || r < 128 ? t0 : t1) + (SWIGLU ? r : r & 127) * NOUT + ((c ^ (r % OCH)) * 16);
            const uint4 v = *reinterpret_cast<const uint4*>(src);
            const int col = ti.nt * NOUT + c * 16;
            if (r < ti.valid && col < p.N) *reinterpret_cast<uint4*>(out + (ti.row0 + r) * p.N + col) = v;
        }
    } else {
        constexpr int OROW = NOUT * 2;   // bytes per staged row
        constexpr int OCH = OROW / 16;   // 16-byte chunks per row
        constexpr int RPS = SLOT / OROW;  // rows per 32 KB slot: 64
        static_assert(TM <= 4 * RPS && WTOK <= RPS && RPS % WTOK == 0, "staged tile fits four slots");
        auto ost = [&](int i) -> char* { return i == 0 ? t0 : i == 1 ? t1 : i == 2 ? w0 : w1; };
        char* wst = ost(wm * WTOK / RPS) + (wm * WTOK % RPS) * OROW;
        barrier();  // the weight loaders' last products read a weight slot
#pragma unroll
        for (int mi = 0; mi < MI; ++mi) {
            const int r = mi * 16 + l16;
            const int sr = wm * WTOK + r;
            HalfScale hs{1.f, 1.f};
            if constexpr (HALF) {
                uint32_t m = 0;
#pragma unroll
                for (int ni = 0; ni < NI; ++ni)
#pragma unroll
                    for (int e = 0; e < 4; ++e) m = max(m, magnitude(acc[ni][mi][e]));
                if (__any(m >= 0x7f800000u)) {  // rare: an infinity or a NaN in one of the wave's rows
                    m = 0;
#pragma unroll
                    for (int ni = 0; ni < NI; ++ni)
#pragma unroll
                        for (int e = 0; e < 4; ++e) m = max(m, finite_magnitude(acc[ni][mi][e]));
                }
                m = max(m, static_cast<uint32_t>(__shfl_xor(static_cast<int>(m), 16)));
                m = max(m, static_cast<uint32_t>(__shfl_xor(static_cast<int>(m), 32)));
                hs = half_scale(m);
                const int blk = ti.nt * WN + wn;
                if (lg == 0 && sr < ti.valid && blk < p.N / kFp8Block)
                    p.out_scale[(ti.row0 + sr) * (p.N / kFp8Block) + blk] = hs.scale;
            }
#pragma unroll
            for (int ni = 0; ni < NI; ++ni) {
                uint2 o;
                if constexpr (HALF) {
                    f16x4 h;
#pragma unroll
                    for (int e = 0; e < 4; ++e) h[e] = static_cast<_Float16>(acc[ni][mi][e] * hs.inv);
                    o = __builtin_bit_cast(uint2, h);
                } else {
                    bf16x4 h;
#pragma unroll
                    for (int e = 0; e < 4; ++e) h[e] = static_cast<__bf16>(acc[ni][mi][e]);
                    o = __builtin_bit_cast(uint2, h);
                }
                const int col = wn * (NOUT / WN) + ni * 16 + 8 * (lg >> 1);
                const int ch = (col / 8) ^ (sr % OCH);
                *reinterpret_cast<uint2*>(wst + r * OROW + ch * 16 + (lg & 1) * 8) = o;
            }
        }
        __builtin_amdgcn_s_waitcnt(0xC07F);  // lgkmcnt(0)
        barrier();
        constexpr int RPI = 64 / OCH;
        bf16_t* out = static_cast<bf16_t*>(p.out);
#pragma unroll
        for (int j = 0; j < TM / NW / RPI; ++j) {
            const int r = wave * (TM / NW) + j * RPI + lane / OCH;
            const int c = lane % OCH;
            const char* src = ost(r / RPS) + (r % RPS) * OROW + ((c ^ (r % OCH)) * 16);
            const uint4 v = *reinterpret_cast<const uint4*>(src);
            const int col = ti.nt * NOUT + c * 8;
            if (r < ti.valid && col < p.N) *reinterpret_cast<uint4*>(out + (ti.row0 + r) * p.N + col) = v;
        }
    }
    __builtin_amdgcn_s_waitcnt(0xC07F);  // lgkmcnt(0): staged rows read before the slots refill
    barrier();
    }
}

// Sums the partial tiles of the split tail in chunk order and finishes them like the kernel above. One workgroup per (tail
// tile, 16 rows); a thread owns 4 output columns, 32 threads a block of 128 of a row.
template <Epilogue EPI, bool HALF>
__global__ __launch_bounds__(256) void fp8_split_reduce_kernel(Fp8GemmArgs p) {
    constexpr bool SWIGLU = EPI == Epilogue::SwiGLU;
    constexpr int TM = 256, TN = 256, NOUT = SWIGLU ? TN / 2 : TN, QUADS = NOUT / 4, ROWS = 16;
    const int ntn = (p.N + NOUT - 1) / NOUT;
    const SplitPlan sp = split_plan(count_tiles<TM>(p, ntn), kSplitSlots, kMaxSplitChunks, p.K / kFp8Block);
    const int t = blockIdx.x / (TM / ROWS);
    if (sp.S <= 1 || t >= sp.tail) return;
    TileInfo ti;
    if (!tile_of<TM>(p, ntn, sp.full + t, ti)) return;
    const float* tile = p.part + static_cast<int64_t>(t) * sp.S * TM * TN;
    const int r0 = (blockIdx.x % (TM / ROWS)) * ROWS;
    for (int i = threadIdx.x; i < ROWS * QUADS; i += 256) {
        const int r = r0 + i / QUADS, c = i % QUADS * 4;
        f32x4 v = f32x4{0.f, 0.f, 0.f, 0.f}, u = v;
#pragma unroll 4
        for (int k = 0; k < sp.S; ++k) {
            const float* src = tile + (static_cast<int64_t>(k) * TM + r) * TN + c;
            v += *reinterpret_cast<const f32x4*>(src);
            if (SWIGLU) u += *reinterpret_cast<const f32x4*>(src + TN / 2);
        }
        const int col = ti.nt * NOUT + c;
        const bool keep = r < ti.valid && col < p.N;
        if constexpr (HALF) {
            uint32_t m = 0;
#pragma unroll
            for (int e = 0; e < 4; ++e) m = max(m, finite_magnitude(v[e]));
#pragma unroll
            for (int off = 1; off < 32; off <<= 1) m = max(m, static_cast<uint32_t>(__shfl_xor(static_cast<int>(m), off)));
            const HalfScale hs = half_scale(m);
            f16x4 h;
#pragma unroll
            for (int e = 0; e < 4; ++e) h[e] = static_cast<_Float16>(v[e] * hs.inv);
            if (!keep) continue;
            *reinterpret_cast<f16x4*>(static_cast<_Float16*>(p.out) + (ti.row0 + r) * p.N + col) = h;
            if (c % kFp8Block == 0) p.out_scale[(ti.row0 + r) * (p.N / kFp8Block) + col / kFp8Block] = hs.scale;
        } else if constexpr (EPI == Epilogue::Store) {
            if (keep) store_run(static_cast<bf16_t*>(p.out) + (ti.row0 + r) * p.N + col, v, 4, true);
        } else {
            uint32_t m = 0;
            float f[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                f[e] = SWIGLU ? silu(v[e]) * u[e] : relu(v[e]);
                m = max(m, magnitude(f[e]));
            }
#pragma unroll
            for (int off = 1; off < 32; off <<= 1) m = max(m, static_cast<uint32_t>(__shfl_xor(static_cast<int>(m), off)));
            const BlockScale bs = block_scale(m);
            const uint32_t q = quantize4(f, bs);
            if (!keep) continue;
            *reinterpret_cast<uint32_t*>(static_cast<uint8_t*>(p.out) + (ti.row0 + r) * p.N + col) = q;
            if (c % kFp8Block == 0) p.out_scale[(ti.row0 + r) * (p.N / kFp8Block) + col / kFp8Block] = bs.scale;
        }
    }
}

// ------------------------------------------------------------------ dispatch

// Tiles of a launch at most: a group of r rows has ceil(r / TM) <= r / TM + 1 of them per column tile.
int64_t max_tiles(const Fp8GemmArgs& a, int tm, int tn) {
    const int64_t mt = a.seg ? a.rows / tm + std::min<int64_t>(a.rows, a.n_groups) : (a.rows + tm - 1) / tm;
    return mt * ((a.N + tn - 1) / tn);
}

unsigned tile_grid(const Fp8GemmArgs& a, int tm, int tn) {
    return static_cast<unsigned>((max_tiles(a, tm, tn) + kXcds - 1) / kXcds * kXcds);
}

template <typename TO, Epilogue EPI>
hipError_t run_skinny(const Fp8GemmArgs& a, hipStream_t s) {
    ProfileScope prof(a.name, s);
    hipLaunchKernelGGL((fp8_skinny_kernel<TO, EPI>), dim3(tile_grid(a, 16, 16)), dim3(64 * kFewWaves), 0, s, a);
    return hipGetLastError();
}

template <typename TO, int TM, int RING, Epilogue EPI, bool STREAM, bool EXACT>
hipError_t run_ring(const Fp8GemmArgs& a, hipStream_t s) {
    ProfileScope prof(a.name, s);
    hipLaunchKernelGGL((fp8_ring_kernel<TO, TM, RING, EPI, STREAM, EXACT>), dim3(tile_grid(a, TM, EPI == Epilogue::SwiGLU ? 64 : 128)),
                       dim3(256), 0, s, a);
    return hipGetLastError();
}

template <Epilogue EPI, bool HALF = false>
hipError_t run_pp(const Fp8GemmArgs& a, hipStream_t s) {
    {
        ProfileScope prof(a.name, s);
        hipLaunchKernelGGL((fp8_pp_kernel<EPI, HALF>), dim3(kSplitSlots), dim3(512), 0, s, a);
    }
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || !a.part) return e;
    // a tail is split into two chunks or more: at most half a round of tiles
    char name[48];  // of the timing record; no allocation, which could throw
    std::snprintf(name, sizeof name, "%s_tail", a.name);
    ProfileScope prof(name, s);
    hipLaunchKernelGGL((fp8_split_reduce_kernel<EPI, HALF>), dim3(kSplitSlots / 2 * 16), dim3(256), 0, s, a);
    return hipGetLastError();
}

int64_t avg_rows(const Fp8GemmArgs& a) { return a.rows / std::max(1, a.n_groups); }

// 32-bit byte offsets of gathered token rows and of scale rows
bool offsets32(const Fp8GemmArgs& a) {
    return (!a.row_index || a.src_rows * a.K < (int64_t(1) << 32)) && a.src_rows * (a.K / kFp8Block) * 4 < (int64_t(1) << 32);
}

// Tiles of tm x tn expected of a launch: the segments' lengths are on the device, so a group with rows is taken to have the
// mean of them and a quarter of a tile more, one tile at least.
double expected_tiles(const Fp8GemmArgs& a, int tm, int tn) {
    const double active = static_cast<double>(std::min<int64_t>(a.rows, a.n_groups));
    const double mt = a.seg ? active * std::max(1.0, a.rows / active / tm + 0.25) : std::ceil(static_cast<double>(a.rows) / tm);
    return mt * ((a.N + tn - 1) / tn);
}
// Whether the last round of the 256 x 256 tiles may be worth splitting along K: long K, and rounds few enough that it weighs.
// (Whether it is split, and into how many chunks, follows from the number of tiles, on the device.) Measured, whole and split
// (us): one matrix 2048 wide with 8448 rows, K 1024 36 and 40, 1536 47 and 47, 2048 58 and 54, 4096 99 and 86; 4096 wide with
// 8448 rows, 2.1 rounds, K 2048 85 and 85, 4096 153 and 148, with 4400 rows and K 2048 55 and 63 (the sums of a round's eighth);
// 8192 wide with 16640 rows, 8.1 rounds, K 2048 291 and 301, 4096 523 and 515; 17 rounds 524 and 525; without a part of a
// round, 8 groups of 1056 rows, K 2048, 157 and 166 (the launch that finds no sums).
bool may_split(const Fp8GemmArgs& a, bool swiglu) {
    return a.K >= 16 * kFp8Block && expected_tiles(a, 256, swiglu ? 128 : 256) <= 8 * kSplitSlots;
}

// Which tiles a product takes: those whose rounds are expected to take least time. A round is a workgroup a CU; two of the
// ring's run together. Each takes a time per block of K and one at its end, fitted (us) to dense products of 512 to 4096 rows
// and 1024 to 4096 wide:
//   8-bit core, 64 rows: 0.50 n + 3.3 alone, 0.72 n + 4.5 the pair; 128 rows: 0.74 n + 3.6 and 1.07 n + 6.0;
//   256 x 256: 1.59 n + 8.1, a split last round its share of the blocks, its end, and 6 + 0.055 a partial tile for the sums;
//   exact, 64 rows: 0.73 n + 1.3 and 1.09 n + 3.8; 128 rows: 1.02 n + 2.5 and 1.78 n + 5.3.
// Measured, 64 rows, 128 rows and 256 x 256 (8-bit core, whole call): one matrix 4096 x 4096 with 512 rows 25, 33, 43 us, 2048
// rows 57, 45, 57, 4096 rows 112, 85, 64, 4400 rows 133, 107, 96, 512 rows of 14336 73, 93, 54; 8 groups 2048 -> 2048 of 100
// rows 16, 20, 26, 400 rows 33, 25, 50, 600 rows 48, 41, 34; 64 groups 2048 -> 1408 of 32 rows 39, 42, 57, 100 rows 53, 47, 59,
// 200 rows 86, 71, 83, 500 rows 221, 171, 133. Exact, 64 and 128 rows: one matrix with 512 rows 33, 42, 1024 rows 45, 45, 4096
// rows 159, 129; 8 groups of 100 rows 19, 24, 400 rows 44, 36.
struct RingCost {
    double slab1, end1, slab2, end2;  // a workgroup alone, a pair
};
constexpr RingCost kRing64{0.50, 3.3, 0.72, 4.5}, kRing128{0.74, 3.6, 1.07, 6.0};
constexpr RingCost kExact64{0.73, 1.3, 1.09, 3.8}, kExact128{1.02, 2.5, 1.78, 5.3};

double ring_cost(const Fp8GemmArgs& a, int tm, int tn, const RingCost& c) {
    const double nkb = a.K / kFp8Block;
    // (an expected number barely past a round is as likely below it)
    const int wgs = std::max(1, static_cast<int>(std::ceil(expected_tiles(a, tm, tn) / 256 - 0.02)));
    return wgs / 2 * (c.slab2 * nkb + c.end2) + wgs % 2 * (c.slab1 * nkb + c.end1);
}

double pp_cost(const Fp8GemmArgs& a, bool swiglu) {
    const double nkb = a.K / kFp8Block, slab = 1.59, end = 8.1;
    const double tiles = std::max(1.0, expected_tiles(a, 256, swiglu ? 128 : 256));
    const double full = std::floor(tiles / kSplitSlots + 0.02), tail = tiles - full * kSplitSlots;
    double t = full * (slab * nkb + end);
    if (tail > 0.02 * kSplitSlots || full == 0) {
        const int chunks = may_split(a, swiglu) ? std::max(1, static_cast<int>(std::min(kSplitSlots / tail, nkb / 2))) : 1;
        t += slab * nkb / chunks + end + (chunks > 1 ? 6.0 + 0.055 * chunks * tail : 0.0);
    }
    return t;
}

bool use_pp(const Fp8GemmArgs& a, Epilogue epi) {
    // Few rows are a stream of the weights, which the other kernels follow: 64 groups of 24 rows, 2048 -> 2048, 71 us here and
    // 49 in the ring, 48 rows 74 and 61; 16 groups of 24 rows, 4096 -> 4096, 75 and 62.
    if (!offsets32(a) || a.K < 2 * kFp8Block || avg_rows(a) < 32) return false;
    const bool swiglu = epi == Epilogue::SwiGLU;
    const int tn = swiglu ? 64 : 128;
    // hidden rows of the ring pass through memory in float32 and a launch of their own
    const double extra = epi == Epilogue::Store ? 0.0 : 4.5 + static_cast<double>(a.rows) * a.N * 8 / 4.5e6;
    return pp_cost(a, swiglu) <= extra + std::min(ring_cost(a, 64, tn, kRing64), ring_cost(a, 128, tn, kRing128));
}

// The smaller tiles. Measured (us; few-row kernel, ring of 32, 64 and 128 rows):
//   fewer than 32 rows a group and fewer 32-row tiles than CUs: the few-row kernel, whose 16 x 16 tiles are eight times as
//   many. 1 row, 4096 -> 4096 (32 tiles), 7.0, 27, 22, -; 2 groups of 8 rows, 14336 -> 4096 (64), 34, 88, 92, -; 4 groups of 4,
//   4096 -> 4096 (128), 19, 30, 31, -; 8 groups of 4, 2048 -> 2048 (144), 11, 16, 13, -; behind the limit 16 rows, 2048 -> 32768
//   (256), 25, 18, 19, -; 8 groups of 4, 2048 -> 4096 (288), 19, 18, 19, -; 64 groups of 2, 2048 -> 1024 (544), 34, 24, 27, -.
//   fewer than 16 rows a group: the ring of 32, a stream of weights with exact products. 64 groups, 2048 -> 2048, of 8 rows 68,
//   46, 54, 56, of 24 rows 156, 49, 57, 60, of 48 rows 230, 85, 61, 64; with Zipf's lengths a mean of 8 rows 79, 43, 49, 51, 16
//   rows 119, 58, 63, 60, 28 rows 169, 68, 66, 69; 1024 -> 4096, 16 rows 149, 63, 66, 66, 24 rows 192, 75, 68, 73; 16 groups,
//   4096 -> 4096, 12 rows 97, 83, 69, 71. Equal lengths favour it up to 32 rows, unequal ones up to 12 to 24.
//   else 64 or 128 rows by their cost.
template <typename TO, Epilogue EPI, bool EXACT>
hipError_t dispatch_small(const Fp8GemmArgs& a, hipStream_t s) {
    const int tn = EPI == Epilogue::SwiGLU ? 64 : 128;
    if (!offsets32(a) || (avg_rows(a) < 32 && max_tiles(a, 32, tn) < 256)) return run_skinny<TO, EPI>(a, s);
    if (avg_rows(a) < 16) return run_ring<TO, 32, 4, EPI, true, true>(a, s);
    if (ring_cost(a, 128, tn, EXACT ? kExact128 : kRing128) < ring_cost(a, 64, tn, EXACT ? kExact64 : kRing64))
        return run_ring<TO, 128, 2, EPI, false, EXACT>(a, s);
    return run_ring<TO, 64, 3, EPI, false, EXACT>(a, s);
}

}  // namespace

bool fp8_gemm_fits(const Fp8GemmArgs& a) {
    // a launch holds fewer than 2^32 threads: 512 a tile of the few-row kernel, 256 a tile of the ring (32 x 64 at least)
    if (max_tiles(a, 32, 64) >= (int64_t(1) << 24) - kXcds || (!offsets32(a) && max_tiles(a, 16, 16) >= (int64_t(1) << 23) - kXcds))
        return false;
    return a.K < 1 << 24;  // 32-bit byte offsets of the 256 rows of a tile
}

hipError_t launch_fp8_gemm(DType out_type, const Fp8GemmArgs& a, hipStream_t s) {
    if (a.rows == 0) return hipSuccess;
    if (out_type == DType::F32) return dispatch_small<float, Epilogue::Store, true>(a, s);
    if (use_pp(a, Epilogue::Store) && a.N % 8 == 0) return run_pp<Epilogue::Store>(a, s);
    return dispatch_small<bf16_t, Epilogue::Store, false>(a, s);
}

bool fp8_rows_half(const Fp8GemmArgs& a) { return use_pp(a, Epilogue::Store); }

hipError_t launch_fp8_rows(const Fp8GemmArgs& a, hipStream_t s) {
    if (a.rows == 0) return hipSuccess;
    return fp8_rows_half(a) ? run_pp<Epilogue::Store, true>(a, s) : dispatch_small<float, Epilogue::Store, false>(a, s);
}

size_t fp8_split_scratch_bytes(Epilogue epi, const Fp8GemmArgs& a) {
    const bool swiglu = epi == Epilogue::SwiGLU;
    return use_pp(a, epi) && may_split(a, swiglu) ? static_cast<size_t>(kSplitSlots) * 256 * 256 * sizeof(float) : 0;
}

size_t fp8_hidden_scratch_bytes(Epilogue epi, const Fp8GemmArgs& a, bool exact) {
    return !exact && use_pp(a, epi) ? 0 : static_cast<size_t>(a.rows) * a.N * sizeof(float);
}

hipError_t launch_fp8_hidden(Epilogue epi, const Fp8GemmArgs& a, bool exact, float* scratch, hipStream_t s) {
    if (a.rows == 0) return hipSuccess;
    const bool swiglu = epi == Epilogue::SwiGLU;
    if (!exact && use_pp(a, epi)) return swiglu ? run_pp<Epilogue::SwiGLU>(a, s) : run_pp<Epilogue::ReLU>(a, s);
    Fp8GemmArgs g = a;
    g.out = scratch;
    auto go = [&](auto ex) {
        return swiglu ? dispatch_small<float, Epilogue::SwiGLU, ex.value>(g, s) : dispatch_small<float, Epilogue::ReLU, ex.value>(g, s);
    };
    const hipError_t e = exact ? go(std::true_type{}) : go(std::false_type{});
    if (e != hipSuccess) return e;
    return launch_fp8_quantize(DType::F32, scratch, 1, static_cast<int>(a.rows), a.N, 1, a.out, a.out_scale, s);
}

}  // namespace ec2moe
