// Work decomposition shared by the matrix-core GEMMs of this library: tiles of row segments whose
// lengths stay on the device, their order over the XCDs, the split of the last round along K,
// and the buffer loads that write LDS directly. The argument structs (A) carry
//   const int32_t* seg;  [groups+1] device segment offsets, or null (dense: one group)
//   int n_groups;  int64_t rows;
#pragma once

#include <algorithm>

#include "device_common.h"

namespace ec2moe {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) void lds_void;

// buffer_load_dwordx4 ... lds: each lane's 16 bytes land at M0 + 16 * lane
__device__ void raw_buffer_load_lds(i32x4 rsrc, lds_void* lds, int size, int voffset, int soffset, int offset,
                                    int aux) __asm("llvm.amdgcn.raw.buffer.load.lds");

namespace {

constexpr int kXcds = 8;
constexpr int kMaxSplitChunks = 32;  // K chunks of a split tail tile

struct TileInfo {
    int group;
    int64_t row0;  // first row of the tile (position in the permuted order)
    int valid;     // rows of the tile inside the group
    int nt;        // n-tile index
    int mtiles;    // token tiles of the group
};

__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }

// s_waitcnt immediate for vmcnt(n), lgkmcnt(0) and no expcnt wait: n <= 63 (vmcnt bits 3:0 and 15:14)
constexpr int vmcnt_imm(int n) { return 0x0070 | (n & 15) | ((n >> 4) << 14); }

// Number of real tiles (uniform): sum over groups of ceil(rows_e / TM) * ntn.
template <int TM, typename A>
__device__ __forceinline__ int count_tiles(const A& a, int ntn) {
    if (a.seg == nullptr) return uniform(static_cast<int>((a.rows + TM - 1) / TM) * ntn);
    const int lane = threadIdx.x & 63;
    int t = 0;
    for (int e0 = 0; e0 < a.n_groups; e0 += 64) {
        const int e = e0 + lane;
        int cnt = 0;
        if (e < a.n_groups) cnt = ((a.seg[e + 1] - a.seg[e] + TM - 1) / TM) * ntn;
#pragma unroll
        for (int off = 32; off >= 1; off >>= 1) cnt += __shfl_xor(cnt, off);
        t += cnt;
    }
    return uniform(t);
}

// Position of tile `local` within one group of mtiles x ntn tiles: m-tiles go in
// ceil(mtiles / 8) bands of near-equal size (4 to 8 m-tiles when there are enough); a
// band's n-tiles run in order with the band's m-tiles adjacent. A run of 32 consecutive
// tiles (one XCD's workgroups) then covers b m-tiles x 32/b n-tiles, which share
// b + 32/b slabs (11 to 12 of 64) in that XCD's L2.
__device__ __forceinline__ void band_decode(int local, int mtiles, int ntn, int& mt, int& nt) {
    const int nbands = (mtiles + 7) / 8;
    const int bsz = (mtiles + nbands - 1) / nbands;
    const int band = local / (bsz * ntn);
    const int m0 = band * bsz;
    const int bm = std::min(bsz, mtiles - m0);  // m-tiles in this band
    const int r = local - band * bsz * ntn;
    nt = r / bm;
    mt = m0 + (r - nt * bm);
}

// Tile with logical index bid (groups in order; within a group, banded as above).
template <int TM, typename A>
__device__ __forceinline__ bool tile_of(const A& a, int ntn, int bid, TileInfo& ti) {
    if (a.seg == nullptr) {
        const int mtiles = static_cast<int>((a.rows + TM - 1) / TM);
        int mt, nt;
        band_decode(bid, mtiles, ntn, mt, nt);
        ti.group = 0;
        ti.nt = nt;
        ti.mtiles = mtiles;
        ti.row0 = static_cast<int64_t>(mt) * TM;
        ti.valid = static_cast<int>(std::min<int64_t>(TM, a.rows - ti.row0));
        return true;
    }
    const int lane = threadIdx.x & 63;
    int base = 0;
    for (int e0 = 0; e0 < a.n_groups; e0 += 64) {
        const int e = e0 + lane;
        int lo = 0, hi = 0, cnt = 0;
        if (e < a.n_groups) {
            lo = a.seg[e];
            hi = a.seg[e + 1];
            cnt = ((hi - lo + TM - 1) / TM) * ntn;
        }
        int inc = cnt;
#pragma unroll
        for (int off = 1; off < 64; off <<= 1) {
            const int v = __shfl_up(inc, off);
            if (lane >= off) inc += v;
        }
        const bool hit = e < a.n_groups && cnt > 0 && bid >= base + inc - cnt && bid < base + inc;
        const uint64_t hits = __ballot(hit);
        if (hits) {
            const int src = __ffsll(static_cast<long long>(hits)) - 1;
            const int first = base + __shfl(inc - cnt, src);
            const int glo = uniform(__shfl(lo, src));
            const int ghi = uniform(__shfl(hi, src));
            const int mtiles = (ghi - glo + TM - 1) / TM;
            const int local = uniform(bid - first);
            ti.group = uniform(e0 + src);
            int mt, nt;
            band_decode(local, mtiles, ntn, mt, nt);
            ti.nt = nt;
            ti.mtiles = mtiles;
            ti.row0 = glo + static_cast<int64_t>(mt) * TM;
            ti.valid = std::min(TM, ghi - static_cast<int>(ti.row0));
            return true;
        }
        base += __shfl(inc, 63);
    }
    return false;
}

// XCD-aware order: workgroup p of a launch of `units` whole tiles runs logical tile
// (p % 8) * ceil(units / 8) + p / 8; -1 if p has no tile.
__device__ __forceinline__ int xcd_remap(int p, int units) {
    const int per_xcd = (units + kXcds - 1) / kXcds;
    const int j = p / kXcds;
    const int bid = (p % kXcds) * per_xcd + j;
    return (j >= per_xcd || bid >= units) ? -1 : bid;
}

// Finds the tile of this workgroup (whole tiles only); false if it has none.
template <int TM, typename A>
__device__ __forceinline__ bool find_tile(const A& a, int ntn, TileInfo& ti) {
    const int bid = xcd_remap(blockIdx.x, count_tiles<TM>(a, ntn));
    return bid >= 0 && tile_of<TM>(a, ntn, bid, ti);
}

// Split plan of a launch with `total` tiles and `slots` workgroups resident at once: the
// tiles that fill whole rounds run whole; the tail (fewer than one round) is split into
// S chunks along K so the last round is about as wide as the machine. Chunks hold an even
// number of 64-wide slabs.
struct SplitPlan {
    int full, tail, S, chunk_slabs;
};

__host__ __device__ __forceinline__ SplitPlan split_plan(int total, int slots, int max_split, int nk) {
    SplitPlan sp;
    sp.full = slots > 0 ? total / slots * slots : total;
    sp.tail = total - sp.full;
    int S = 1;
    if (sp.tail > 0 && max_split > 1)
        // at most one split workgroup per CU: more (two 128x128 tiles fit a CU) only adds
        // partial-sum traffic (the fine-grained encoder's X V: 18.0 against 21.7 us)
        S = std::max(1, std::min(std::min(std::min(max_split, kMaxSplitChunks), std::min(slots, 256) / sp.tail),
                                 nk / 2));
    sp.S = S;
    sp.chunk_slabs = ((nk + S - 1) / S + 1) / 2 * 2;
    return sp;
}

// silu(g) = g / (1 + e^-g) with the hardware 2^x and reciprocal (each within about 1 ulp),
// e^-g = 2^(-g log2 e); a very negative g gives e^-g = inf and a zero reciprocal.
__device__ __forceinline__ float silu(float g) {
    const float e = __builtin_amdgcn_exp2f(-g * 1.4426950408889634f);
    return g * __builtin_amdgcn_rcpf(1.0f + e);
}

__device__ __forceinline__ i32x4 buffer_rsrc(const void* base, uint32_t bytes) {
    const uint64_t p = reinterpret_cast<uint64_t>(base);
    i32x4 r;
    r[0] = uniform(static_cast<int>(static_cast<uint32_t>(p)));
    r[1] = uniform(static_cast<int>(static_cast<uint32_t>(p >> 32)));
    r[2] = uniform(static_cast<int>(bytes));
    r[3] = 0x00020000;  // raw (untyped, unswizzled) buffer of the gfx9 family
    return r;
}

}  // namespace
}  // namespace ec2moe
