// Tiled bf16 matrix product C[i][j] = sum_k A(i, k) B(j, k) with fp32 sums,
// the core of the head loss (dv_head.hip).  Each operand is stored with k
// along its rows ("rows": i by k) or with k from row to row ("columns": k by i);
// row starts are on 16-byte boundaries and k is a multiple of 64.
#pragma once

#include "dv_internal.h"

namespace dv {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(4))) float f32x4;

// One operand, rows of `ld` elements.  Stored by rows: `n` rows (indices past
// them read the last one).  Stored by columns: rows of `n` elements, n a
// multiple of 8 (pieces past them read the last one), of which k_rows exist (past
// them the last one is read again: the other operand holds zeros there).  What
// comes of indices past n is dropped by the epilogue.  An fp32 operand is held
// as three bf16 planes, `plane` elements apart, that add up to it exactly.
struct GemmOperand {
    const __bf16 *p;
    int64_t ld;
    int64_t plane;
    int n;
    int k_rows;
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

// The waves of a block split its BM x BN tile into WM x WN parts; COLS_A and
// COLS_B say which operands are stored by columns.
//
// A stage holds 64 k of both tiles in LDS, laid out in groups of 1 KiB (what
// one wave's direct-to-LDS load writes; whole lines of memory: with 32 k stages
// the same product ran 15 to 20 % slower on twice the requests).
//
// By rows: 8 rows x 128 bytes a group; the 16-byte piece c of row r sits at
// place c ^ (r / 2 mod 8) of its row, so that the lanes of a fragment read (row
// l mod 16, piece l / 16) meet distinct banks.
//
// By columns: a group is 1024 / (2 BM) rows of k, each the tile's BM columns.  A
// fragment is read by transposing 8-byte loads: 16 lanes give the places of 4
// rows x 16 columns, and lane c receives column c's four values of k.  What is read
// at once are the rows that differ in bits 0, 1 and 3 of k; a group therefore
// takes rows that differ in the other bits (2, then 4, then 5), and groups are 32
// bytes more than their size apart: distinct banks again.
//
// Two stages: while the matrix instructions work on one half of a stage's k in
// registers, its other half (then the next stage's first) goes from LDS to
// registers, and the stage after it from memory to LDS.  One barrier a stage: past
// it every wave has the stage's fragments in registers, so its buffer is free,
// and the next stage has arrived.
//
// What it reaches by rows with 256 x 256 tiles: 16384 x 8192 x 4096 1.31 PFLOP/s,
// 4096 x 8192 x 16384 1.26 (the library 1.55 and 1.57); 128 x 128 tiles 1.10 and
// 1.06, 64 x 64 tiles 0.71 and 0.69.
constexpr int kGemmStageK = 64;

// One side's tile in LDS: B rows or columns, of which a wave takes F fragments.
template <int B, bool COLS>
struct GemmSide {
    static constexpr int kGroups = B / 8;
    static constexpr int kPitch = COLS ? 1024 + 32 : 1024;
    static constexpr int kBytes = kGroups * kPitch;
    static constexpr int kRowsPerGroup = 1024 / (2 * B);  // by columns: 2, 4 or 8
    static_assert(!COLS || (B >= 64 && B <= 256), "a group holds 2, 4 or 8 rows of k");

    // By columns, row `r` of a stage's 64: its group and its place in the group.
    // Bits 0, 1, 3 of r (and of 4, 5 what the place does not take) make the group.
    static constexpr __host__ __device__ int row_of(int group, int slot)
    {
        int r = (group & 3) | (group >> 2 & 1) << 3 | (slot & 1) << 2;
        if (kRowsPerGroup == 2)
            r |= (group >> 3 & 1) << 4 | (group >> 4 & 1) << 5;
        else if (kRowsPerGroup == 4)
            r |= (slot >> 1 & 1) << 4 | (group >> 3 & 1) << 5;
        else
            r |= (slot >> 1 & 1) << 4 | (slot >> 2 & 1) << 5;
        return r;
    }

    // What lane `lane` loads for group `group`, of the tile from `i0` on:
    // byte offset from the stage's start in memory; `k_left` rows of k are left.
    static __device__ __forceinline__ int source(const GemmOperand &o, int i0, int group, int lane, int k_left)
    {
        if constexpr (COLS) {
            constexpr int kPieces = B / 8;
            int r = row_of(group, lane / kPieces);
            int c = (lane % kPieces) * 8;
            r = r < k_left ? r : k_left - 1;
            c = c < o.n - i0 ? c : o.n - 8 - i0;
            return r * (int)(o.ld * 2) + c * 2;
        } else {
            int r = group * 8 + (lane >> 3);
            const int c = (lane & 7) ^ ((r >> 1) & 7);
            r = r < o.n - i0 ? r : o.n - 1 - i0;
            return r * (int)(o.ld * 2) + c * 16;
        }
    }

    // A lane's place in the tile for its part of a wave's fragments, and the
    // distance of fragment i and of half h of the stage's k from it.
    static __device__ __forceinline__ int place(int lane, int h)
    {
        const int r = lane & 15, b = lane >> 4;
        if constexpr (COLS) {
            const int group = r >> 2 | (b & 1) << 2;
            int at = group * kPitch + (lane & 3) * 8;
            if (kRowsPerGroup == 2)
                at += (b >> 1) * 8 * kPitch + h * 16 * kPitch;
            else if (kRowsPerGroup == 4)
                at += (b >> 1) * 2 * (2 * B) + h * 8 * kPitch;
            else
                at += (b >> 1) * 2 * (2 * B) + h * 4 * (2 * B);
            return at;
        } else {
            return r * 128 + ((h * 4 + b) ^ (r >> 1)) * 16;
        }
    }

    static constexpr __device__ __forceinline__ int fragment_step() { return COLS ? 32 : 2048; }

    static __device__ __forceinline__ bf16x8 fragment(const char *tile, int at, int i)
    {
        if constexpr (COLS) {
            typedef __attribute__((ext_vector_type(4))) short s16x4;
            using Ptr = __attribute__((address_space(3))) s16x4 *;
            union {
                s16x4 half[2];
                bf16x8 v;
            } f;
            f.half[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Ptr)(tile + at + i * fragment_step()));
            f.half[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Ptr)(tile + at + i * fragment_step() + 2 * B));
            return f.v;
        } else {
            return *reinterpret_cast<const bf16x8 *>(tile + at + i * fragment_step());
        }
    }
};

template <int BM, int BN, int WM, int WN, bool COLS_A = false, bool COLS_B = false>
struct Gemm {
    using A = GemmSide<BM, COLS_A>;
    using B = GemmSide<BN, COLS_B>;
    static constexpr int kWaves = WM * WN;
    static constexpr int kTm = BM / WM / 16;  // 16-row fragments of a wave
    static constexpr int kTn = BN / WN / 16;
    static constexpr int kGroups = A::kGroups + B::kGroups;
    static constexpr int kLoads = kGroups / kWaves;  // of one wave per stage
    static constexpr int kStageBytes = A::kBytes + B::kBytes;
    static constexpr int kLdsBytes = 2 * kStageBytes;
    static_assert(kGroups % kWaves == 0 && A::kGroups % kLoads == 0, "a wave loads whole groups of one side");

    using Lds = __attribute__((address_space(3))) void *;

    struct Fragments {
        bf16x8 a[kTm], b[kTn];
    };

    static __device__ __forceinline__ void read(Fragments &f, const char *stage, int at_a, int at_b)
    {
#pragma unroll
        for (int i = 0; i < kTn; ++i)
            f.b[i] = B::fragment(stage + A::kBytes, at_b, i);
#pragma unroll
        for (int i = 0; i < kTm; ++i)
            f.a[i] = A::fragment(stage, at_a, i);
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
        constexpr int kReads = kTm * (COLS_A ? 2 : 1) + kTn * (COLS_B ? 2 : 1);
        static_assert(kReads <= 2 * kTm * kTn, "at least one matrix instruction to two reads");
        constexpr int kPer = kReads > kTm * kTn ? 2 : 1;
#pragma unroll
        for (int i = 0; i < kReads / kPer; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);     // a matrix instruction
            __builtin_amdgcn_sched_group_barrier(0x100, kPer, 0);  // LDS reads
            if (2 * kReads <= kTm * kTn)
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

    // 16 bytes a lane from base + offset to LDS, lane after lane from `dst` on.
    // In assembly, because the compiler takes any later transposing read for a
    // read of what is on its way and waits for it; it writes no register, and
    // the waits and the barrier of `run` order it.  (m0 is never held over a
    // statement: the compiler sets it where it needs it.)
    static __device__ __forceinline__ void load_to_lds(const char *base, int offset, uint32_t dst)
    {
        typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
        const uint64_t p = reinterpret_cast<uint64_t>(base);
        const u32x4 rsrc = {(uint32_t)p, (uint32_t)(p >> 32) & 0xFFFFu, 0x7FFFFFFFu, 0x00027000u};
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds"
                     :
                     : "s"(dst), "v"(offset), "s"(rsrc)
                     : "memory");
    }

    // acc += the tile at i0 of A and j0 of B.  Lane l of a wave ends with
    // acc[ti][tj][e] = C[i0 + wm BM/WM + 16 ti + 4 (l / 16) + e][j0 + wn BN/WN + 16 tj + l mod 16].
    // `from`, `stages` (at least 1): this block's part of the 64-k stages.
    static __device__ __forceinline__ void run(f32x4 (&acc)[kTm][kTn], const GemmShape &g, int i0, int j0, int from,
                                               int stages, char *lds)
    {
        const int lane = threadIdx.x & (kWave - 1);
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
        const int wm = wave / WN, wn = wave % WN;

        // this wave's loads: kLoads groups of one side, whose next stage begins at `next`
        const int group = wave * kLoads;
        const bool side_a = group < A::kGroups;
        const GemmOperand &o = side_a ? g.a : g.b;
        const bool cols = side_a ? COLS_A : COLS_B;
        const int first = side_a ? i0 : j0;
        const int64_t stage_step = (cols ? kGemmStageK * o.ld : kGemmStageK) * 2;
        const char *const start = reinterpret_cast<const char *>(o.p + (cols ? first : first * o.ld));
        int voff[kLoads];
        const auto place_loads = [&](int k_left) {
#pragma unroll
            for (int i = 0; i < kLoads; ++i)
                voff[i] = side_a ? A::source(o, first, group + i, lane, k_left)
                                 : B::source(o, first, group - A::kGroups + i, lane, k_left);
        };
        place_loads(kGemmStageK);
        const int per_segment = g.k / kGemmStageK;
        int segment = from / per_segment;
        int stage = from - segment * per_segment;
        const int slot_base = side_a ? group * A::kPitch : A::kBytes + (group - A::kGroups) * B::kPitch;
        const int pitch = side_a ? A::kPitch : B::kPitch;
        const bool ragged = cols && o.k_rows < g.k;  // k's last stage has rows that do not exist

        const auto load = [&](int slot) {
            const char *q = start + stage * stage_step;
            if (g.segments > 1)
                q += (int64_t)(side_a ? segment_plane_a(segment) : segment_plane_b(segment)) * o.plane * 2;
            if (ragged && stage == per_segment - 1)
                place_loads(o.k_rows - stage * kGemmStageK);
            const uint32_t dst = (uint32_t)(uintptr_t)(Lds)(lds + slot * kStageBytes + slot_base);
#pragma unroll
            for (int i = 0; i < kLoads; ++i)
                load_to_lds(q, voff[i], dst + i * pitch);
            if (++stage == per_segment) {
                stage = 0;
                ++segment;
                if (ragged)
                    place_loads(kGemmStageK);
            }
        };

        const int a0 = A::place(lane, 0) + wm * (A::fragment_step() * kTm), a1 = A::place(lane, 1) + wm * (A::fragment_step() * kTm);
        const int b0 = B::place(lane, 0) + wn * (B::fragment_step() * kTn), b1 = B::place(lane, 1) + wn * (B::fragment_step() * kTn);
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
        read(f0, lds, a0, b0);
        for (int s = 0; s < stages; ++s) {
            read(f1, lds + (s & 1) * kStageBytes, a1, b1);
            multiply(acc, f0);
            if (s + 1 < stages) {
                wait_loads<0>();
                __builtin_amdgcn_s_barrier();
                asm volatile("" ::: "memory");
                if (s + 2 < stages)
                    load(s & 1);
                read(f0, lds + ((s + 1) & 1) * kStageBytes, a0, b0);
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
