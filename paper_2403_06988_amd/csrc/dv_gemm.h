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
// A stage holds 64 k of both tiles in LDS as groups of 8 rows x 128 bytes
// (1 KiB, what one wave's direct-to-LDS load writes; whole lines of memory: with 32 k
// stages the same product ran 15 to 20 % slower on twice the requests).  In a
// tile the 16-byte piece c of row r sits at place c ^ (r / 2 mod 8) of its row,
// so that the lanes of a fragment read (row l mod 16, piece l / 16) meet
// distinct banks.  Two stages: while the matrix instructions work on one half of a
// stage's k in registers, its other half (then the next stage's first) goes
// from LDS to registers, and the stage after it from memory to LDS.  One barrier
// a stage: past it every wave has the stage's fragments in registers, so its
// buffer is free, and the next stage has arrived.
//
// What it reaches with 256 x 256 tiles: 16384 x 8192 x 4096 1.31 PFLOP/s, 4096 x
// 8192 x 16384 1.26 (the library 1.55 and 1.57); 128 x 128 tiles 1.10 and 1.06,
// 64 x 64 tiles 0.71 and 0.69.
constexpr int kGemmStageK = 64;

template <int BM, int BN, int WM, int WN>
struct Gemm {
    static constexpr int kWaves = WM * WN;
    static constexpr int kTm = BM / WM / 16;  // 16-row fragments of a wave
    static constexpr int kTn = BN / WN / 16;
    static constexpr int kGroupsA = BM / 8;
    static constexpr int kGroups = (BM + BN) / 8;
    static constexpr int kLoads = kGroups / kWaves;  // of one wave per stage
    static constexpr int kStageBytes = kGroups * 1024;
    static constexpr int kLdsBytes = 2 * kStageBytes;
    static_assert(kGroups % kWaves == 0, "whole groups per wave");

    using Lds = __attribute__((address_space(3))) void *;

    struct Fragments {
        bf16x8 a[kTm], b[kTn];
    };

    static __device__ __forceinline__ void read(Fragments &f, const char *stage, int wm, int wn, int place)
    {
#pragma unroll
        for (int i = 0; i < kTn; ++i)
            f.b[i] = *reinterpret_cast<const bf16x8 *>(stage + kGroupsA * 1024 + (wn * kTn + i) * 2048 + place);
#pragma unroll
        for (int i = 0; i < kTm; ++i)
            f.a[i] = *reinterpret_cast<const bf16x8 *>(stage + (wm * kTm + i) * 2048 + place);
    }

    // acc += a b^T, with the LDS reads issued just before dealt out between
    // the matrix instructions.
    static __device__ __forceinline__ void multiply(f32x4 (&acc)[kTm][kTn], const Fragments &f)
    {
#pragma unroll
        for (int i = 0; i < kTm; ++i)
#pragma unroll
            for (int j = 0; j < kTn; ++j)
                acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f.a[i], f.b[j], acc[i][j], 0, 0, 0);
#pragma unroll
        for (int i = 0; i < kTm + kTn; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);  // a matrix instruction
            __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);  // an LDS read
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        }
        __builtin_amdgcn_sched_barrier(0);
    }

    // s_waitcnt: at most N of this wave's loads on the way; LDS reads done too with 0
    template <int N>
    static __device__ __forceinline__ void wait_loads()
    {
        static_assert(N < 64, "six bits of the count");
        __builtin_amdgcn_s_waitcnt((N ? 0x0F70 : 0x0070) | (N & 15) | (N >> 4) << 14);
    }

    // acc += the tile at rows i0 of A and j0 of B.  Lane l of a wave ends
    // with acc[ti][tj][e] = C[i0 + wm BM/WM + 16 ti + 4 (l / 16) + e][j0 + wn BN/WN + 16 tj + l mod 16].
    // `from`, `stages` (at least 1): this block's part of the 64-k stages.
    static __device__ __forceinline__ void run(f32x4 (&acc)[kTm][kTn], const GemmShape &g, int i0, int j0, int from,
                                               int stages, char *lds)
    {
        const int lane = threadIdx.x & (kWave - 1);
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
        const int wm = wave / WN, wn = wave % WN;
        int voff[kLoads];
        bool is_a[kLoads];
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int group = wave * kLoads + i;
            is_a[i] = group < kGroupsA;
            const GemmOperand &o = is_a[i] ? g.a : g.b;
            const int r0 = is_a[i] ? i0 : j0;
            int r = (is_a[i] ? group : group - kGroupsA) * 8 + (lane >> 3);
            const int c = (lane & 7) ^ ((r >> 1) & 7);
            r = r < o.rows - r0 ? r : o.rows - 1 - r0;
            voff[i] = r * (int)(o.ld * 2) + c * 16;
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

        const int r = lane & 15;
        const int place0 = r * 128 + ((lane >> 4) ^ (r >> 1)) * 16;        // first half of a stage's k
        const int place1 = r * 128 + ((4 + (lane >> 4)) ^ (r >> 1)) * 16;  // second half
        Fragments f0, f1;
        load(0);
        if (stages > 1) {
            load(1);
            wait_loads<kLoads>();
        } else {
            wait_loads<0>();
        }
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        read(f0, lds, wm, wn, place0);
        for (int s = 0; s < stages; ++s) {
            read(f1, lds + (s & 1) * kStageBytes, wm, wn, place1);
            multiply(acc, f0);
            if (s + 1 < stages) {
                wait_loads<0>();
                __builtin_amdgcn_s_barrier();
                asm volatile("" ::: "memory");
                if (s + 2 < stages)
                    load(s & 1);
                read(f0, lds + ((s + 1) & 1) * kStageBytes, wm, wn, place0);
            }
            multiply(acc, f1);
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
