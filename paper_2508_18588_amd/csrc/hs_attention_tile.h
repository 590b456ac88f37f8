// What the attention kernels have in common: a tile of 32 query rows, a row per lane of either half of a wavefront, and the
// partial result of a row for a partition of the keys.
#pragma once
#include "hs_gemm_common.h"   // fragment types
#include "hs_internal.h"

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));

__device__ inline float fast_exp2(float x) { return __builtin_amdgcn_exp2f(x); }

// A 32-key sub-tile (two pages) in LDS: K as 32 rows of HD elements, then V^T as two pages of HD rows of 16 tokens, both
// without padding, so that a page's K or V^T block is one contiguous run that a load into LDS can fill.  16-byte chunks are
// permuted instead: within a row of K, so that 16 consecutive rows read at the same chunk cover the 64 banks once; of 16 rows of
// V^T first the first halves, then the second ones, so that an operand is two 8-byte pieces a constant distance apart.  (32 lanes
// read the same half of their chunks, so two of them meet on each bank: the counters show LDS busy 50 % of the cycles, 20 of
// them conflicts, where single 16-byte pieces had 23 % and none; a 14B step with trees 1388 -> 1391 us.)
template <int HD>
struct sub_tile {
    static constexpr int PAGE = 32 * HD, V = 2 * PAGE, BYTES = 4 * PAGE;   // a page's K (or V^T) block, V^T's place, all
    static __device__ __forceinline__ int k_at(int key, int chunk) {
        return key * 2 * HD + ((chunk ^ (HD == 128 ? key & 15 : (key >> 1) & 7)) << 4);
    }
    // what 1 KB further on changes in the permutation
    static constexpr int k_step(int i) { return (HD == 128 ? 4 * i & 15 : 4 * i & 7) << 4; }
    static constexpr int V_HALF = 256;   // from a row's first to its second half
    static __device__ __forceinline__ int v_at(int dim, int chunk) { return (dim >> 4) * 512 + chunk * V_HALF + (dim & 15) * 16; }
    // where in a page's V^T block the 16 bytes that belong at 16 c of it in LDS come from
    static __device__ __forceinline__ int v_from(int c) { return ((c >> 5) * 16 + (c & 15)) * 32 + ((c >> 4) & 1) * 16; }
};

// Query fragments (B operand of S^T) and ancestor mask of the lane's row; rows beyond R read as zero.
template <int HD>
__device__ inline void load_query_tile(const bf16_t* q, const uint64_t* anc_mask, int r0, int rt, int R, int G,
                                       int hq, int j, int half, int l32, bf16x8 (&qf)[HD / 16], uint64_t& anc) {
    int rho = rt * 32 + l32;
    bool ok = rho < R;
    int node = ok ? rho / G : 0;
    int g = ok ? rho - node * G : 0;
    anc = (ok && anc_mask) ? anc_mask[r0 + node] : 0ull;
    const bf16_t* qp = q + ((size_t)(r0 + node) * hq + j * G + g) * HD;
#pragma unroll
    for (int ks = 0; ks < HD / 16; ks++) {
        if (ok) {
            qf[ks] = *reinterpret_cast<const bf16x8*>(qp + ks * 16 + half * 8);
        } else {
#pragma unroll
            for (int e = 0; e < 8; e++) qf[ks][e] = (__bf16)0.f;
        }
    }
}

// Partial result of one partition for the lane's row: running max (log2 domain) and sum in fp32, and the partition's
// own normalised output O / l in fp16 -- a convex combination of V rows, so within fp16's range whenever V is, and
// rounded 8 times finer than the bf16 result of the merge.  Half the bytes of an fp32 partial: the partial results
// are the one write stream of the launch, and writes in the middle of the K/V read stream are dear.
typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));

template <int HD>
__device__ inline void store_partial(const f32x16 (&o)[HD / 32], float m_run, float l_run, _Float16* part_o,
                                     float* part_ml, int r0, int rt, int R, int G, int hq, int j, int max_parts,
                                     int part, int half, int l32) {
    int rho = rt * 32 + l32;
    if (rho >= R) return;
    int node = rho / G, g = rho - node * G;
    size_t prow = ((size_t)(r0 + node) * hq + j * G + g) * max_parts + part;
    _Float16* po = part_o + prow * HD;
    const float inv = l_run > 0.f ? 1.f / l_run : 0.f;   // a partition in which the row sees no key: all zero
#pragma unroll
    for (int dt = 0; dt < HD / 32; dt++)
#pragma unroll
        for (int g4 = 0; g4 < 4; g4++) {
            f16x4 v = {(_Float16)(o[dt][4 * g4] * inv), (_Float16)(o[dt][4 * g4 + 1] * inv),
                       (_Float16)(o[dt][4 * g4 + 2] * inv), (_Float16)(o[dt][4 * g4 + 3] * inv)};
            *reinterpret_cast<f16x4*>(po + dt * 32 + 8 * g4 + 4 * half) = v;
        }
    if (half == 0) {
        part_ml[prow * 2] = m_run;
        part_ml[prow * 2 + 1] = l_run;
    }
}
