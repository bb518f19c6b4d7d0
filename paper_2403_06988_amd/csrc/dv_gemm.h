// Tiled matrix product C[i][j] = sum_k A(i, k) B(j, k) of bf16 or fp32 operands with
// fp32 sums, the core of the head loss (dv_head.hip).  Each operand is stored with
// k along its rows ("rows": i by k) or with k from row to row ("columns": k by i);
// row starts are on 16-byte boundaries.  B may be a bf16 operand in two parts.
#pragma once

#include "dv_internal.h"

namespace dv {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(4))) float f32x4;

// One operand, rows of `ld` elements.  Stored by rows: `n` rows (indices past
// them read the last one).  Stored by columns: rows of `n` elements, n a
// multiple of 8 (pieces past them read the last one), of which k_rows exist (past
// them the last one is read again: the other operand holds zeros there).  What
// comes of indices past n is dropped by the epilogue.
struct GemmOperand {
    const void *p;
    int64_t ld;
    int n;
    int k_rows;
};

struct GemmShape {
    GemmOperand a, b;
    int k;  // whole stages: a multiple of 64 (bf16) or 32 (fp32); two parts: of both together
};

// The place of column c in a row of an operand in two bf16 parts, the sum of which is the
// operand: 32 columns of the first part, the same 32 of the second, and so on.
constexpr int kPartColumns = 32;
__host__ __device__ constexpr int64_t part_column(int64_t c) { return (c / kPartColumns * 2) * kPartColumns + c % kPartColumns; }

// The waves of a block split its BM x BN tile into WM x WN parts; COLS_A and
// COLS_B say which operands are stored by columns.
//
// A stage holds 64 (bf16) or 32 (fp32) k of both tiles in LDS, laid out in groups
// of 1 KiB (what one wave's direct-to-LDS load writes; whole lines of memory: with
// half the k a stage the same product ran 15 to 20 % slower on twice the requests).
//
// By rows: 8 rows x 128 bytes a group; the 16-byte piece c of row r sits at
// place c ^ (r / 2 mod 8) of its row, so that the lanes of a fragment read (row
// l mod 16, piece l / 16) meet distinct banks.
//
// bf16 by columns: a group is 1024 / (2 BM) rows of k, each the tile's BM columns.
// A fragment is read by transposing 8-byte loads: 16 lanes give the places of 4
// rows x 16 columns, and lane c receives column c's four values of k.  What is read
// at once are the rows that differ in bits 0, 1 and 3 of k; a group therefore
// takes rows that differ in the other bits (2, then 4, then 5), and groups are 32
// bytes more than their size apart: distinct banks again.  fp32 by columns: a lane
// reads its column's eight values of k one by one; read at once are rows 8
// apart, which groups of 1024 / (4 BM) rows, 64 bytes more than their size apart,
// keep in distinct banks.
//
// B in two parts (bf16; A by columns): a stage holds 32 k of A, and of B those 32 of the
// first part, then of the second: one half of its k each, both multiplied by the same
// fragments of A.  By rows that is how B lies; by columns a lane loads its row's parts.
//
// bf16: while the matrix instructions work on one half of a stage's k in
// registers, its other half (then the next stage's first) goes from LDS to
// registers, and the stage after it from memory to LDS.  One barrier a stage: past
// it every wave has the stage's fragments in registers, so its buffer is free,
// and the next stage has arrived.
//
// fp32: a fragment is split in registers into three bf16 parts, each the rest
// rounded to nearest (their sum is exact, 24 bits), and six products are added:
// a0b0, a0b1, a1b0, a0b2, a1b1, a2b0.  The three left out are below 2^-22 of the
// whole.  Six bf16 matrix instructions do what sixteen fp32 ones would, at 6/16
// of their time.  (Finite elements below bf16's largest: infinities come out as NaN.)
//
// What it reaches: see the figures at its kernels in dv_head.hip.
template <typename E>
struct GemmStage {
    static constexpr int kK = 128 / (int)sizeof(E);  // k of a stage
};

// One side's tile in LDS: B rows or columns, of which a wave takes F fragments.  HALF: 32 k
// of an operand by columns, for both halves of a stage; PARTS: an operand in two parts.
template <typename E, int B, bool COLS, bool HALF = false, bool PARTS = false>
struct GemmSide {
    static constexpr bool kBf16 = sizeof(E) == 2;
    static constexpr int kStageK = GemmStage<E>::kK;
    static constexpr int kGroups = HALF ? B / 16 : B / 8;
    // of a stage, by columns: rows of k in memory
    static constexpr int kStageRows = HALF || PARTS ? kStageK / 2 : kStageK;
    static_assert(!HALF || (COLS && kBf16), "half a stage is of bf16 by columns");
    static_assert(!PARTS || (kBf16 && !HALF), "parts are bf16");
    static constexpr int kPitch = !COLS ? 1024 : kBf16 ? 1024 + 32 : 1024 + 64;
    static constexpr int kBytes = kGroups * kPitch;
    static constexpr int kRowBytes = B * (int)sizeof(E);      // by columns: of a row of k
    static constexpr int kRowsPerGroup = 1024 / kRowBytes;    // by columns
    static_assert(!COLS || (B >= 64 && B <= 256), "a group holds whole rows of k");

    // By columns, the row of k at place `slot` of a group.  bf16: bits 0, 1, 3
    // of r (and of 4, 5 what the place does not take) make the group.  fp32: bits
    // 3, 4 (and of 0 to 2 what the place does not take).  Half a stage of 64 columns has four
    // groups: bit 3 makes the place's first bit, half of the banks apart.
    static __device__ __forceinline__ int row_of(int group, int slot)
    {
        if constexpr (HALF) {
            if (kRowsPerGroup == 8)
                return (group & 3) | (slot & 1) << 3 | (slot >> 1 & 1) << 2 | (slot >> 2 & 1) << 4;
            int r = (group & 3) | (group >> 2 & 1) << 3 | (slot & 1) << 2;
            r |= (kRowsPerGroup == 2 ? group >> 3 & 1 : slot >> 1 & 1) << 4;
            return r;
        } else if constexpr (kBf16) {
            int r = (group & 3) | (group >> 2 & 1) << 3 | (slot & 1) << 2;
            if (kRowsPerGroup == 2)
                r |= (group >> 3 & 1) << 4 | (group >> 4 & 1) << 5;
            else if (kRowsPerGroup == 4)
                r |= (slot >> 1 & 1) << 4 | (group >> 3 & 1) << 5;
            else
                r |= (slot >> 1 & 1) << 4 | (slot >> 2 & 1) << 5;
            return r;
        } else {
            return (group & 3) * 8 + (group >> 2) * kRowsPerGroup + slot;
        }
    }

    // What lane `lane` loads for group `group`, of the tile from `i0` on: byte
    // offset from the stage's start in memory; `k_left` rows of k are left.
    static __device__ __forceinline__ int source(const GemmOperand &o, int i0, int group, int lane, int k_left)
    {
        constexpr int kElt = (int)sizeof(E);
        if constexpr (COLS) {
            constexpr int kPieces = kRowBytes / 16;
            int r = row_of(group, lane / kPieces);
            int c = (lane % kPieces) * (16 / kElt);
            c = c < o.n - i0 ? c : o.n - 16 / kElt - i0;
            if constexpr (PARTS) {
                c = (int)part_column(c) + r / kStageRows * kPartColumns;
                r %= kStageRows;
            }
            r = r < k_left ? r : k_left - 1;
            return r * (int)(o.ld * kElt) + c * kElt;
        } else {
            int r = group * 8 + (lane >> 3);
            const int c = (lane & 7) ^ ((r >> 1) & 7);
            r = r < o.n - i0 ? r : o.n - 1 - i0;
            return r * (int)(o.ld * kElt) + c * 16;
        }
    }

    static constexpr int kFragmentStep = !COLS ? 2048 : kBf16 ? 32 : 64;  // bytes between fragments

    // A lane's place in the tile for its part of a wave's fragments; bf16: of
    // half h of the stage's k.  fp32 by rows has a second place, for the
    // lane's second four k.
    static __device__ __forceinline__ int place(int lane, int h)
    {
        const int r = lane & 15, b = lane >> 4;
        if constexpr (HALF) {
            if (kRowsPerGroup == 8)
                return (r >> 2) * kPitch + (lane & 3) * 8 + (b & 1) * kRowBytes + (b >> 1) * 4 * kRowBytes;
            const int group = r >> 2 | (b & 1) << 2;
            return group * kPitch + (lane & 3) * 8 + (b >> 1) * (kRowsPerGroup == 2 ? 8 * kPitch : 2 * kRowBytes);
        } else if constexpr (COLS && kBf16) {
            const int group = r >> 2 | (b & 1) << 2;
            int at = group * kPitch + (lane & 3) * 8;
            if (kRowsPerGroup == 2)
                at += (b >> 1) * 8 * kPitch + h * 16 * kPitch;
            else if (kRowsPerGroup == 4)
                at += (b >> 1) * 2 * kRowBytes + h * 8 * kPitch;
            else
                at += (b >> 1) * 2 * kRowBytes + h * 4 * kRowBytes;
            return at;
        } else if constexpr (COLS) {
            return b * kPitch + r * 4;
        } else if constexpr (kBf16) {
            return r * 128 + ((h * 4 + b) ^ (r >> 1)) * 16;
        } else {
            return r * 128 + ((2 * b + h) ^ (r >> 1)) * 16;
        }
    }

    static __device__ __forceinline__ bf16x8 fragment(const char *tile, int at, int i)
    {
        static_assert(kBf16, "fp32 fragments are read raw");
        if constexpr (COLS) {
            typedef __attribute__((ext_vector_type(4))) short s16x4;
            using Ptr = __attribute__((address_space(3))) s16x4 *;
            union {
                s16x4 half[2];
                bf16x8 v;
            } f;
            constexpr int kNext = HALF && kRowsPerGroup == 8 ? 2 * kRowBytes : kRowBytes;  // bit 2 of k
            f.half[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Ptr)(tile + at + i * kFragmentStep));
            f.half[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Ptr)(tile + at + i * kFragmentStep + kNext));
            return f.v;
        } else {
            return *reinterpret_cast<const bf16x8 *>(tile + at + i * kFragmentStep);
        }
    }

    // A lane's eight fp32 values of fragment i; at0 and at1 its two places.
    static __device__ __forceinline__ void raw(float (&x)[8], const char *tile, int at0, int at1, int i)
    {
        if constexpr (COLS) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                constexpr int R = kRowsPerGroup;
                x[e] = *reinterpret_cast<const float *>(tile + at0 + i * kFragmentStep + (e / R) * 4 * kPitch +
                                                        (e % R) * kRowBytes);
            }
        } else {
            const f32x4 lo = *reinterpret_cast<const f32x4 *>(tile + at0 + i * kFragmentStep);
            const f32x4 hi = *reinterpret_cast<const f32x4 *>(tile + at1 + i * kFragmentStep);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                x[e] = lo[e];
                x[4 + e] = hi[e];
            }
        }
    }
};

// Eight fp32 values as three bf16 fragments that add up to them.
struct SplitFragment {
    bf16x8 part[3];
    __device__ __forceinline__ void set(float (&x)[8])
    {
#pragma unroll
        for (int p = 0; p < 3; ++p)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                part[p][e] = (__bf16)x[e];
                x[e] -= (float)part[p][e];
            }
    }
};

template <typename E, int BM, int BN, int WM, int WN, bool COLS_A = false, bool COLS_B = false, bool PARTS = false>
struct Gemm {
    using A = GemmSide<E, BM, COLS_A, PARTS>;
    using B = GemmSide<E, BN, COLS_B, false, PARTS>;
    static constexpr int kStageK = GemmStage<E>::kK;
    static constexpr int kWaves = WM * WN;
    static constexpr int kTm = BM / WM / 16;  // 16-row fragments of a wave
    static constexpr int kTn = BN / WN / 16;
    static constexpr int kGroups = A::kGroups + B::kGroups;
    static constexpr int kLoads = kGroups / kWaves;  // of one wave per stage
    static constexpr int kStageBytes = A::kBytes + B::kBytes;
    static constexpr int kLdsBytes = 2 * kStageBytes;
    static_assert(kGroups % kWaves == 0, "a wave loads whole groups");

    using Lds = __attribute__((address_space(3))) void *;

    struct Fragments {
        bf16x8 a[kTm], b[kTn];
    };

    template <bool BOTH = true>
    static __device__ __forceinline__ void read(Fragments &f, const char *stage, int at_a, int at_b)
    {
#pragma unroll
        for (int i = 0; i < kTn; ++i)
            f.b[i] = B::fragment(stage + A::kBytes, at_b, i);
        if constexpr (BOTH)
#pragma unroll
            for (int i = 0; i < kTm; ++i)
                f.a[i] = A::fragment(stage, at_a, i);
    }

    // acc += a b^T, with the LDS reads issued just before (of both sides, or of B)
    // dealt out between the matrix instructions.
    template <bool BOTH = true>
    static __device__ __forceinline__ void multiply(f32x4 (&acc)[kTm][kTn], const Fragments &f)
    {
#pragma unroll
        for (int i = 0; i < kTm; ++i)
#pragma unroll
            for (int j = 0; j < kTn; ++j)
                acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f.a[i], f.b[j], acc[i][j], 0, 0, 0);
        constexpr int kReads = (BOTH ? kTm * (COLS_A ? 2 : 1) : 0) + kTn * (COLS_B ? 2 : 1);
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

    static __device__ __forceinline__ void barrier()
    {
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    }

    // 16 bytes a lane from base + offset to LDS, lane after lane from `dst` on.
    // In assembly, because the compiler takes any later transposing read for a
    // read of what is on its way and waits for it; it writes no register, and
    // the waits and the barrier of `run` order it.  m0, which it sets, is named as
    // written: the compiler keeps nothing there across it.
    static __device__ __forceinline__ void load_to_lds(const char *base, int offset, uint32_t dst)
    {
        typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
        const uint64_t p = reinterpret_cast<uint64_t>(base);
        const u32x4 rsrc = {(uint32_t)p, (uint32_t)(p >> 32) & 0xFFFFu, 0x7FFFFFFFu, 0x00027000u};
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"  // m0 is reserved: not preserved, as meant
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds"
                     :
                     : "s"(dst), "v"(offset), "s"(rsrc)
                     : "memory", "m0");
#pragma clang diagnostic pop
    }

    // Tiles of few fragments have registers to spare and are those of few rows, whose
    // results stand for themselves: their sums run in kChains accumulators, joined at the
    // end.  bf16: each half of a stage of each parity its own, a quarter of the additions one
    // after the other.  fp32: the leading products of each parity, and the five small ones, which
    // then round nothing of the large sum.
    static constexpr bool kSplitSums = kTm * kTn <= 4;
    static constexpr int kChains = !kSplitSums ? 1 : sizeof(E) == 2 ? 4 : 3;

    // acc += the tile at i0 of A and j0 of B.  Lane l of a wave ends with
    // acc[ti][tj][e] = C[i0 + wm BM/WM + 16 ti + 4 (l / 16) + e][j0 + wn BN/WN + 16 tj + l mod 16].
    // `from`, `stages` (at least 1): this block's part of the stages of k.
    static __device__ __forceinline__ void run(f32x4 (&acc)[kTm][kTn], const GemmShape &g, int i0, int j0, int from,
                                               int stages, char *lds)
    {
        const int lane = threadIdx.x & (kWave - 1);
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
        const int wm = wave / WN, wn = wave % WN;

        // this wave's loads: kLoads groups, of one side (or, in tiles of uneven
        // sides, of both)
        const int group = wave * kLoads;
        const auto side_a = [&](int i) {
            constexpr bool kMixed = A::kGroups % kLoads != 0;
            return group + (kMixed ? i : 0) < A::kGroups;
        };
        const auto start = [&](const GemmOperand &o, bool cols, bool parts, int first) {
            return reinterpret_cast<const char *>(static_cast<const E *>(o.p) +
                                                  (!cols ? first * o.ld : parts ? part_column(first) : first));
        };
        const auto step = [&](const GemmOperand &o, bool cols, int rows) {
            return (cols ? rows * o.ld : kStageK) * (int64_t)sizeof(E);
        };
        const char *const start_a = start(g.a, COLS_A, false, i0), *const start_b = start(g.b, COLS_B, PARTS, j0);
        const int64_t step_a = step(g.a, COLS_A, A::kStageRows), step_b = step(g.b, COLS_B, B::kStageRows);
        int voff[kLoads];
        const auto place_loads = [&](int left_a, int left_b) {
#pragma unroll
            for (int i = 0; i < kLoads; ++i)
                voff[i] = side_a(i) ? A::source(g.a, i0, group + i, lane, left_a)
                                    : B::source(g.b, j0, group + i - A::kGroups, lane, left_b);
        };
        place_loads(A::kStageRows, B::kStageRows);
        int stage = from;

        const auto load = [&](int slot) {
            // rows of k that do not exist, by columns: the last one again
            const auto left = [&](const GemmOperand &o, bool cols, int rows) {
                return cols ? o.k_rows - stage * rows : rows;
            };
            const auto place = [&](const char *start, int64_t step, const GemmOperand &o, int left) {
                return left > 0 ? start + stage * step : start + (int64_t)(o.k_rows - 1) * o.ld * (int64_t)sizeof(E);
            };
            const int left_a = left(g.a, COLS_A, A::kStageRows), left_b = left(g.b, COLS_B, B::kStageRows);
            if (left_a < A::kStageRows || left_b < B::kStageRows)
                place_loads(left_a > 0 ? left_a : 1, left_b > 0 ? left_b : 1);
            const char *const qa = place(start_a, step_a, g.a, left_a), *const qb = place(start_b, step_b, g.b, left_b);
            const uint32_t dst = (uint32_t)(uintptr_t)(Lds)(lds + slot * kStageBytes);
#pragma unroll
            for (int i = 0; i < kLoads; ++i) {
                const int at = group + i;
                load_to_lds(side_a(i) ? qa : qb, voff[i],
                            dst + (side_a(i) ? at * A::kPitch : A::kBytes + (at - A::kGroups) * B::kPitch));
            }
            ++stage;
        };

        const int at_a = wm * (A::kFragmentStep * kTm), at_b = wn * (B::kFragmentStep * kTn);
        const int a0 = at_a + A::place(lane, 0), a1 = at_a + A::place(lane, 1);
        const int b0 = at_b + B::place(lane, 0), b1 = at_b + B::place(lane, 1);
        load(0);
        if (stages > 1) {
            load(1);
            wait_loads<kLoads>();
        } else {
            wait_loads<0>();
        }
        barrier();
        f32x4 more[kChains > 1 ? kChains - 1 : 1][kTm][kTn] = {};  // the chains beside acc
        if constexpr (sizeof(E) == 2) {
            Fragments f0, f1;
            read(f0, lds, a0, b0);
            const auto work = [&](int s, f32x4 (&first)[kTm][kTn], f32x4 (&second)[kTm][kTn]) {
                read<!PARTS>(f1, lds + (s & 1) * kStageBytes, a1, b1);
                if constexpr (PARTS)
#pragma unroll
                    for (int i = 0; i < kTm; ++i)
                        f1.a[i] = f0.a[i];
                multiply<!PARTS>(first, f0);
                if (s + 1 < stages) {
                    wait_loads<0>();
                    barrier();
                    if (s + 2 < stages)
                        load(s & 1);
                    read(f0, lds + ((s + 1) & 1) * kStageBytes, a0, b0);
                }
                multiply(second, f1);
            };
            if constexpr (kSplitSums) {
                for (int s = 0; s < stages; s += 2) {
                    work(s, acc, more[0]);
                    if (s + 1 < stages)
                        work(s + 1, more[1], more[2]);
                }
            } else {
                for (int s = 0; s < stages; ++s)
                    work(s, acc, acc);
            }
        } else {
            const auto work = [&](int s, f32x4 (&large)[kTm][kTn], f32x4 (&small)[kTm][kTn]) {
                const char *tile = lds + (s & 1) * kStageBytes;
                float x[8];
                SplitFragment b[kTn];
#pragma unroll
                for (int j = 0; j < kTn; ++j) {
                    B::raw(x, tile + A::kBytes, b0, b1, j);
                    b[j].set(x);
                }
                float next[8];
                A::raw(next, tile, a0, a1, 0);
#pragma unroll
                for (int i = 0; i < kTm; ++i) {
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        x[e] = next[e];
                    if (i + 1 < kTm)
                        A::raw(next, tile, a0, a1, i + 1);
                    SplitFragment a;
                    a.set(x);
                    constexpr int kPairs[6][2] = {{0, 2}, {1, 1}, {2, 0}, {0, 1}, {1, 0}, {0, 0}};
#pragma unroll
                    for (int p = 0; p < 6; ++p)
#pragma unroll
                        for (int j = 0; j < kTn; ++j) {
                            f32x4 &sum = p < 5 ? small[i][j] : large[i][j];
                            sum = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.part[kPairs[p][0]], b[j].part[kPairs[p][1]], sum, 0,
                                                                          0, 0);
                        }
                }
                if (s + 1 < stages) {
                    wait_loads<0>();
                    barrier();
                    if (s + 2 < stages)
                        load(s & 1);
                }
            };
            if constexpr (kSplitSums) {
                for (int s = 0; s < stages; s += 2) {
                    work(s, acc, more[0]);
                    if (s + 1 < stages)
                        work(s + 1, more[1], more[0]);
                }
            } else {
                for (int s = 0; s < stages; ++s)
                    work(s, acc, acc);
            }
        }
        if constexpr (kSplitSums) {
#pragma unroll
            for (int i = 0; i < kTm; ++i)
#pragma unroll
                for (int j = 0; j < kTn; ++j) {
                    if constexpr (sizeof(E) == 2)
                        acc[i][j] = (acc[i][j] + more[0][i][j]) + (more[1][i][j] + more[2][i][j]);
                    else
                        acc[i][j] = (acc[i][j] + more[1][i][j]) + more[0][i][j];
                }
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
