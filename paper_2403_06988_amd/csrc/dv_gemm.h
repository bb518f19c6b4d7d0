// Tiled bf16 matrix product C[i][j] = sum_k A[i][k] B[j][k] with fp32 sums,
// the core of the head loss (dv_head.hip).  Both operands are stored with k
// contiguous, rows on 16-byte boundaries, k a multiple of 64.
#pragma once

#include "dv_internal.h"

namespace dv {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(4))) float f32x4;

// One operand: rows of `ld` elements; row indices past `rows` read the last
// row (the epilogue drops what comes of them).  An fp32 operand is held as
// three bf16 planes, `plane` elements apart, that add up to it exactly.
struct GemmOperand {
    const __bf16 *p;
    int64_t ld;
    int64_t plane;
    int rows;
};

struct GemmShape {
    GemmOperand a, b;
    int k;         // elements of one pass over k, a multiple of 64
    int segments;  // 1: bf16 operands; 6: fp32 ones, the pairs of planes whose product counts (below)
};

// fp32 operands x = x0 + x1 + x2, w = w0 + w1 + w2 (each plane at most 2^-8 of
// the one before): the products x0w0, x0w1, x1w0, x0w2, x1w1 and x2w0; the
// three left out are below 2^-22 of the whole.
constexpr int kGemmSegments = 6;
__device__ __forceinline__ int segment_plane_a(int s) { return (0x012010 >> (4 * (5 - s))) & 15; }
__device__ __forceinline__ int segment_plane_b(int s) { return (0x210100 >> (4 * (5 - s))) & 15; }

// The waves of a block split its BM x BN tile into WM x WN parts.
//
// A stage holds 32 k of both tiles in LDS as groups of 16 rows x 64 bytes
// (1 KiB, what one wave's direct-to-LDS load writes).  In a group the 16-byte
// piece c of row r sits at place 4 r + (c ^ f(r)), f(r) = (r / 2 mod 4) ^ (r / 8),
// so that the lanes of a fragment read (row l mod 16, piece l / 16) meet
// distinct banks.  kStages stages are in flight or in use: while the matrix
// instructions work on the registers of stage k, stage k + 1 goes from LDS to
// registers and stage k + 3 from memory to LDS.
constexpr int kGemmStages = 4;
constexpr int kGemmStageK = 32;

template <int BM, int BN, int WM, int WN>
struct Gemm {
    static constexpr int kWaves = WM * WN;
    static constexpr int kThreads = kWaves * kWave;
    static constexpr int kTm = BM / WM / 16;  // 16-row fragments of a wave
    static constexpr int kTn = BN / WN / 16;
    static constexpr int kGroupsA = BM / 16;
    static constexpr int kGroups = (BM + BN) / 16;
    static constexpr int kLoads = kGroups / kWaves;  // of one wave per stage
    static constexpr int kStageBytes = kGroups * 1024;
    static constexpr int kLdsBytes = kGemmStages * kStageBytes;
    static_assert(kGroups % kWaves == 0, "whole groups per wave");

    using Lds = __attribute__((address_space(3))) void *;

    struct Fragments {
        bf16x8 a[kTm], b[kTn];
    };

    static __device__ __forceinline__ int swizzle(int r) { return ((r >> 1) & 3) ^ (r >> 3); }

    static __device__ __forceinline__ void read(Fragments &f, const char *stage, int wm, int wn, int place)
    {
#pragma unroll
        for (int i = 0; i < kTn; ++i)
            f.b[i] = *reinterpret_cast<const bf16x8 *>(stage + (kGroupsA + wn * kTn + i) * 1024 + place);
#pragma unroll
        for (int i = 0; i < kTm; ++i)
            f.a[i] = *reinterpret_cast<const bf16x8 *>(stage + (wm * kTm + i) * 1024 + place);
    }

    static __device__ __forceinline__ void multiply(f32x4 (&acc)[kTm][kTn], const Fragments &f)
    {
#pragma unroll
        for (int i = 0; i < kTm; ++i)
#pragma unroll
            for (int j = 0; j < kTn; ++j)
                acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f.a[i], f.b[j], acc[i][j], 0, 0, 0);
    }

    // vmcnt: at most n of this wave's loads still on the way
    template <int N>
    static __device__ __forceinline__ void wait_loads()
    {
        static_assert(N < 64, "six bits of the count");
        __builtin_amdgcn_s_waitcnt(0x0F70 | (N & 15) | (N >> 4) << 14);
    }

    // acc += the tile at rows i0 of A and j0 of B.  lane l of a wave ends
    // with acc[ti][tj][e] = C[i0 + wm BM/WM + 16 ti + 4 (l / 16) + e][j0 + wn BN/WN + 16 tj + l mod 16].
    // `from`, `stages`: this block's part of the 32-k steps (both even).
    static __device__ __forceinline__ void run(f32x4 (&acc)[kTm][kTn], const GemmShape &g, int i0, int j0, int from,
                                               int stages, char *lds)
    {
        const int lane = threadIdx.x & (kWave - 1);
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
        const int wm = wave / WN, wn = wave % WN;
        const int lr = lane >> 2, lc = (lane & 3) ^ swizzle(lr);
        int voff[kLoads];
        bool is_a[kLoads];
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int group = wave * kLoads + i;
            is_a[i] = group < kGroupsA;
            const GemmOperand &o = is_a[i] ? g.a : g.b;
            const int r0 = is_a[i] ? i0 : j0;
            int r = (is_a[i] ? group : group - kGroupsA) * 16 + lr;
            r = r < o.rows - r0 ? r : o.rows - 1 - r0;
            voff[i] = r * (int)(o.ld * 2) + lc * 16;
        }
        const char *pa = reinterpret_cast<const char *>(g.a.p + (int64_t)i0 * g.a.ld);
        const char *pb = reinterpret_cast<const char *>(g.b.p + (int64_t)j0 * g.b.ld);
        const int per_segment = g.k / kGemmStageK;
        int segment = from / per_segment;
        int at = (from - segment * per_segment) * (kGemmStageK * 2);  // bytes along k

        auto load = [&](int slot) {
            const char *qa = pa, *qb = pb;
            if (g.segments > 1) {
                qa += (int64_t)segment_plane_a(segment) * g.a.plane * 2;
                qb += (int64_t)segment_plane_b(segment) * g.b.plane * 2;
            }
            auto ra = __builtin_amdgcn_make_buffer_rsrc(const_cast<char *>(qa), 0, 0x7FFFFFFF, 0x00027000);
            auto rb = __builtin_amdgcn_make_buffer_rsrc(const_cast<char *>(qb), 0, 0x7FFFFFFF, 0x00027000);
            char *dst = lds + slot * kStageBytes + wave * kLoads * 1024;
#pragma unroll
            for (int i = 0; i < kLoads; ++i)
                __builtin_amdgcn_raw_ptr_buffer_load_lds(is_a[i] ? ra : rb, (Lds)(dst + i * 1024), 16, voff[i], at, 0, 0);
            at += kGemmStageK * 2;
            if (at == g.k * 2) {
                at = 0;
                ++segment;
            }
        };

        const int place = ((lane & 15) * 4 + ((lane >> 4) ^ swizzle(lane & 15))) * 16;
        Fragments f[2];
        load(0);
        load(1);
        if (stages > 2) {
            load(2);
            wait_loads<2 * kLoads>();
        } else {
            wait_loads<kLoads>();
        }
        __builtin_amdgcn_s_barrier();
        read(f[0], lds, wm, wn, place);
        auto step = [&](int k, const Fragments &cur, Fragments &next) {
            if (k + 1 < stages) {
                if (k + 2 < stages)
                    wait_loads<kLoads>();
                else
                    wait_loads<0>();
                __builtin_amdgcn_s_barrier();
                asm volatile("" ::: "memory");
                if (k + 3 < stages)
                    load((k + 3) & (kGemmStages - 1));
                read(next, lds + ((k + 1) & (kGemmStages - 1)) * kStageBytes, wm, wn, place);
                __builtin_amdgcn_sched_barrier(0);
            }
            multiply(acc, cur);
        };
        for (int k = 0; k < stages; k += 2) {
            step(k, f[0], f[1]);
            step(k + 1, f[1], f[0]);
        }
    }
};

// The tile of a block, so that blocks that run at the same time on one XCD
// (the hardware deals blocks out to the 8 XCDs in turn) share their operands'
// rows in its L2: each XCD takes one run of the tiles, ordered in bands of
// kBand tiles along i.
constexpr int kXcds = 8;
constexpr int kBand = 8;

__device__ __forceinline__ void tile_of_block(int block, int tiles_i, int tiles_j, int &ti, int &tj)
{
    const int n = tiles_i * tiles_j;
    const int x = block % kXcds, q = n / kXcds, r = n % kXcds;
    const int t = x * q + (x < r ? x : r) + block / kXcds;
    const int per_band = kBand * tiles_j;
    const int band = t / per_band;
    const int height = tiles_i - band * kBand < kBand ? tiles_i - band * kBand : kBand;
    const int in = t - band * per_band;
    ti = band * kBand + in % height;
    tj = in / height;
}

}  // namespace dv
