// Products of e4m3 operands with block scales:
//
//     out[m][n] = sum over blocks kb of 128 k:  sa[kb][m] sb(kb, n) sum_{k in kb} a[m][k] b[n][k]
//
// sb is one number for 128 n (tiles), or one for each n.  A block's sum of 128 products leaves
// the matrix instruction (16 x 16 x 128) in fp32 and is added to the result's sum under
// its scale.
//
// Operands stand in LDS as the bf16 ones of dv_gemm.h do: a stage is 128 bytes of every row,
// here 128 k.  b (whose index n runs along a row of the result) is the instruction's first
// operand, so that a lane holds four neighbouring n of one m: sa is one number a lane and
// fragment, and sb, for tiles, one of the wave.
#include <type_traits>

#include "dv_gemm.h"
#include "dv_logits.h"

namespace dv {
namespace {

typedef __attribute__((ext_vector_type(8))) int i32x8;

struct ProductShape {
    GemmOperand b, a;  // in units of two bytes, as dv_gemm.h takes them
    const float *sa, *sb;
    int rows, cols;
    int blocks;        // of 128 k
};

// A lane's 32 e4m3 values of a fragment (16 rows of 128 k), as the 8-bit matrix instruction
// takes them, or (EXACT) as bf16, which holds each of them.
template <bool EXACT>
struct Fragment8 {
    i32x8 v;
    __device__ __forceinline__ void set(i32x8 x) { v = x; }
    static __device__ __forceinline__ f32x4 multiply(const Fragment8 &a, const Fragment8 &b)
    {
        return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a.v, b.v, f32x4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0, 0, 0, 0);
    }
};
template <>
struct Fragment8<true> {
    bf16x8 part[4];
    __device__ __forceinline__ void set(i32x8 x)
    {
        typedef __attribute__((ext_vector_type(2))) __bf16 Pair;
#pragma unroll
        for (int w = 0; w < 8; ++w) {
            const Pair lo = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((unsigned)x[w], 1.f, false);
            const Pair hi = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((unsigned)x[w], 1.f, true);
            part[w / 2][w % 2 * 4] = lo[0];
            part[w / 2][w % 2 * 4 + 1] = lo[1];
            part[w / 2][w % 2 * 4 + 2] = hi[0];
            part[w / 2][w % 2 * 4 + 3] = hi[1];
        }
    }
    static __device__ __forceinline__ f32x4 multiply(const Fragment8 &a, const Fragment8 &b)
    {
        f32x4 p = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int h = 0; h < 4; ++h)
            p = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.part[h], b.part[h], p, 0, 0, 0);
        return p;
    }
};

template <int BM, int BN, int WM, int WN, bool TILES, bool EXACT>
struct Product8 {
    using G = Gemm<__bf16, BM, BN, WM, WN>;
    using A = typename G::A;
    using B = typename G::B;
    using Fragment = Fragment8<EXACT>;
    static constexpr int kTm = G::kTm, kTn = G::kTn, kLoads = G::kLoads, kWaves = G::kWaves;
    // by rows, b's scales of a stage stand in LDS behind the operands
    static constexpr int kScaleBytes = TILES ? 0 : BM * 4;
    static constexpr int kStageBytes = G::kStageBytes + kScaleBytes;
    static constexpr int kLdsBytes = 2 * kStageBytes;
    static_assert(!TILES || BM / WM <= kScaleBlock, "one scale of b a wave");
    static_assert(TILES || BM / kWave <= kWaves, "a wave loads 64 scales at most");

    template <typename S>
    static __device__ __forceinline__ i32x8 raw(const char *tile, int at0, int at1, int i)
    {
        union {
            bf16x8 half[2];
            i32x8 v;
        } f;
        f.half[0] = S::fragment(tile, at0, i);
        f.half[1] = S::fragment(tile, at1, i);
        return f.v;
    }

    // acc += the tile at i0 of b and j0 of a, over `stages` blocks of 128 k from `from` on.
    static __device__ __forceinline__ void run(f32x4 (&acc)[kTm][kTn], const ProductShape &g, int i0, int j0, int from,
                                               int stages, char *lds)
    {
        const int lane = threadIdx.x & (kWave - 1);
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
        const int wm = wave / WN, wn = wave % WN;
        const int group = wave * kLoads;
        const auto side_a = [&](int i) {
            constexpr bool kMixed = A::kGroups % kLoads != 0;
            return group + (kMixed ? i : 0) < A::kGroups;
        };
        const char *const start_a = static_cast<const char *>(g.b.p) + (int64_t)i0 * g.b.ld * 2;
        const char *const start_b = static_cast<const char *>(g.a.p) + (int64_t)j0 * g.a.ld * 2;
        int voff[kLoads];
#pragma unroll
        for (int i = 0; i < kLoads; ++i)
            voff[i] = side_a(i) ? A::source(g.b, i0, group + i, lane, 0) : B::source(g.a, j0, group + i - A::kGroups, lane, 0);
        const bool loads_scales = !TILES && wave < BM / kWave;
        const int scale_at = i0 + wave * kWave + lane < g.cols ? i0 + wave * kWave + lane : g.cols - 1;
        int stage = from;
        const auto load = [&](int slot) {
            const uint32_t dst = (uint32_t)(uintptr_t)(typename G::Lds)(lds + slot * kStageBytes);
            const int64_t at = (int64_t)stage * kScaleBlock;
            if constexpr (!TILES)
                if (loads_scales)
                    load_word_to_lds(g.sb + (int64_t)stage * g.cols, scale_at * 4, dst + G::kStageBytes + wave * kWave * 4);
#pragma unroll
            for (int i = 0; i < kLoads; ++i) {
                const int p = group + i;
                G::load_to_lds((side_a(i) ? start_a : start_b) + at, voff[i],
                               dst + (side_a(i) ? p * A::kPitch : A::kBytes + (p - A::kGroups) * B::kPitch));
            }
            ++stage;
        };
        const int at_a = wm * (A::kFragmentStep * kTm), at_b = wn * (B::kFragmentStep * kTn);
        const int a0 = at_a + A::place(lane, 0), a1 = at_a + A::place(lane, 1);
        const int b0 = at_b + B::place(lane, 0), b1 = at_b + B::place(lane, 1);
        const int at_scales = G::kStageBytes + (wm * (BM / WM) + (lane >> 4) * 4) * 4;

        // the scales of a: rows past the end read the last one
        int at_sa[kTn];
#pragma unroll
        for (int j = 0; j < kTn; ++j) {
            const int c = j0 + wn * (BN / WN) + j * 16 + (lane & 15);
            at_sa[j] = c < g.rows ? c : g.rows - 1;
        }
        const int iw = i0 + wm * (BM / WM);
        const float *sb_tile = g.sb + (int64_t)((iw < g.cols ? iw : g.cols - 1) / kScaleBlock) * g.blocks;
        float scale[kTn], next_scale[kTn], next_sb = 1.f;
        const auto load_scales = [&](int kb) {
            const float *p = g.sa + (int64_t)kb * g.rows;
#pragma unroll
            for (int j = 0; j < kTn; ++j)
                next_scale[j] = p[at_sa[j]];
            if constexpr (TILES)
                next_sb = sb_tile[kb];
        };

        load_scales(from);
        load(0);
        if (stages > 1)
            load(1);
        if (stages > 1 && TILES)
            G::template wait_loads<kLoads>();
        else
            G::template wait_loads<0>();
        G::barrier();
        Fragment fa, fb[kTn];
        f32x4 p[2];
        i32x8 next = raw<A>(lds, a0, a1, 0);
#pragma unroll
        for (int j = 0; j < kTn; ++j)
            fb[j].set(raw<B>(lds + A::kBytes, b0, b1, j));
        for (int s = 0; s < stages; ++s) {
            const char *tile = lds + (s & 1) * kStageBytes;
            f32x4 sb[2];
            // a finished product, under its scales
            const auto add = [&](int i, int j) {
                const f32x4 x = p[(i * kTn + j) & 1];
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    acc[i][j][e] = __builtin_fmaf(TILES ? x[e] : x[e] * sb[i & 1][e], scale[j], acc[i][j][e]);
                // here, not where the compiler would sink it to: that takes registers for every product
                asm volatile("" : "+v"(acc[i][j]));
            };
#pragma unroll
            for (int j = 0; j < kTn; ++j)
                scale[j] = TILES ? next_scale[j] * next_sb : next_scale[j];
            if (s + 1 < stages)
                load_scales(from + s + 1);
#pragma unroll
            for (int i = 0; i < kTm; ++i) {
                fa.set(next);
                if constexpr (!TILES)
                    sb[i & 1] = *reinterpret_cast<const f32x4 *>(tile + at_scales + i * 64);
                if (i + 1 < kTm) {
                    next = raw<A>(tile, a0, a1, i + 1);
                } else if (s + 1 < stages) {
                    G::template wait_loads<0>();  // and this wave's reads of the stage
                    G::barrier();
                    if (s + 2 < stages)
                        load(s & 1);
                    next = raw<A>(lds + ((s + 1) & 1) * kStageBytes, a0, a1, 0);
                }
                // a product at a time, the one before it added while it runs
#pragma unroll
                for (int j = 0; j < kTn; ++j) {
                    p[(i * kTn + j) & 1] = Fragment::multiply(fa, fb[j]);
                    if (i + j)
                        add(j ? i : i - 1, j ? j - 1 : kTn - 1);
                    __builtin_amdgcn_sched_barrier(0);
                    if (i + 1 == kTm && s + 1 < stages)
                        fb[j].set(raw<B>(lds + ((s + 1) & 1) * kStageBytes + A::kBytes, b0, b1, j));
                }
            }
            add(kTm - 1, kTn - 1);
        }
    }

    // 4 bytes a lane from base + offset to LDS, as Gemm::load_to_lds
    static __device__ __forceinline__ void load_word_to_lds(const float *base, int offset, uint32_t dst)
    {
        typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
        const uint64_t p = reinterpret_cast<uint64_t>(base);
        const u32x4 rsrc = {(uint32_t)p, (uint32_t)(p >> 32) & 0xFFFFu, 0x7FFFFFFFu, 0x00027000u};
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"  // m0 is reserved: not preserved, as meant
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dword %1, %2, 0 offen lds"
                     :
                     : "s"(dst), "v"(offset), "s"(rsrc)
                     : "memory", "m0");
#pragma clang diagnostic pop
    }
};

// Few rows of a (at most 16 KN): bound by b, which passes once, from memory to registers.
//
// A wave takes 16 n, a block WAVES of them.  D blocks of 128 k of b are on their way to a wave's
// registers at any time: each is asked for as soon as the one whose place it takes has been
// multiplied.  a's rows are shared through LDS, C blocks of k at a time in two buffers,
// as bf16 (turned once a block, not once a wave), with the chunk's scales.  An a row's 16-byte unit u stands
// at place u ^ (row mod 16): the 16 rows that are read at once meet distinct banks.
template <typename T, int KN, int WAVES, int C, int D, bool TILES>
__global__ __launch_bounds__(WAVES *kWave, 4) void stream8_kernel(ProductShape g, T *out, int64_t ld, int64_t split_stride,
                                                               int split_blocks)
{
    static_assert(D % C == 0, "a turn of b's places is whole chunks of a");
    constexpr int kRows = 16 * KN, kThreads = WAVES * kWave, kCols = WAVES * 16;
    constexpr int kPitch = C * kScaleBlock * 2, kA = kRows * kPitch;
    constexpr int kScales = C * (kRows + (TILES ? 0 : kCols));  // of a chunk: a's, then b's by rows
    constexpr int kBuffer = kA + kScales * 4;
    constexpr int kPieces = kRows * C * 8;                      // of 16 e4m3 values, in a chunk of a
    constexpr int kMine = (kPieces + kThreads - 1) / kThreads;
    constexpr int kMyScales = (kScales + kThreads - 1) / kThreads;
    constexpr int kOutPitch = kCols * (int)sizeof(T) + 16;
    constexpr int kOut = kRows * kOutPitch;
    __shared__ __attribute__((aligned(16))) char lds[2 * kBuffer > kOut ? 2 * kBuffer : kOut];
    const int lane = threadIdx.x & (kWave - 1);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int n0 = blockIdx.x * kCols, nw = n0 + wave * 16;
    const int from = blockIdx.y * split_blocks;
    const int blocks = g.blocks - from < split_blocks ? g.blocks - from : split_blocks;
    const int n = nw + (lane & 15) < g.cols ? nw + (lane & 15) : g.cols - 1;
    const char *const b = static_cast<const char *>(g.b.p) + (int64_t)n * g.b.ld * 2 + (int64_t)from * kScaleBlock + (lane >> 4) * 16;
    const char *const a = static_cast<const char *>(g.a.p) + (int64_t)from * kScaleBlock;
    const float *const sb_tile = g.sb + (int64_t)((nw < g.cols ? nw : g.cols - 1) / kScaleBlock) * g.blocks + from;

    const auto load_b = [&](int kb) {
        const char *p = b + (int64_t)kb * kScaleBlock;
        union {
            Words half[2];
            i32x8 v;
        } f;
        f.half[0] = *reinterpret_cast<const Words *>(p);
        f.half[1] = *reinterpret_cast<const Words *>(p + 64);
        return f.v;
    };
    Words pieces[kMine];
    float scales[kMyScales];
    const auto load_a = [&](int chunk) {
        const auto block = [&](int i) { return chunk * C + i < blocks ? chunk * C + i : blocks - 1; };
#pragma unroll
        for (int m = 0; m < kMine; ++m) {
            const int at = m * kThreads + threadIdx.x;
            if (kPieces % kThreads && at >= kPieces)
                break;
            const int row = at / (C * 8), piece = at % (C * 8);
            pieces[m] = *reinterpret_cast<const Words *>(a + (int64_t)(row < g.rows ? row : g.rows - 1) * g.a.ld * 2 +
                                                         block(piece / 8) * kScaleBlock + piece % 8 * 16);
        }
#pragma unroll
        for (int m = 0; m < kMyScales; ++m) {
            const int at = m * kThreads + threadIdx.x;
            if (at >= kScales)
                break;
            if (at < C * kRows) {
                const int r = at % kRows;
                scales[m] = g.sa[(int64_t)(from + block(at / kRows)) * g.rows + (r < g.rows ? r : g.rows - 1)];
            } else {
                const int c = n0 + (at - C * kRows) % kCols;
                scales[m] = g.sb[(int64_t)(from + block((at - C * kRows) / kCols)) * g.cols + (c < g.cols ? c : g.cols - 1)];
            }
        }
    };
    const auto keep_a = [&](char *buffer) {
        typedef __attribute__((ext_vector_type(2))) __bf16 Pair;
#pragma unroll
        for (int m = 0; m < kMine; ++m) {
            const int at = m * kThreads + threadIdx.x;
            if (kPieces % kThreads && at >= kPieces)
                break;
            const int row = at / (C * 8), piece = at % (C * 8);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                union {
                    Pair p[4];
                    Words w;
                } y;
#pragma unroll
                for (int w = 0; w < 2; ++w) {
                    y.p[2 * w] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(pieces[m][2 * h + w], 1.f, false);
                    y.p[2 * w + 1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(pieces[m][2 * h + w], 1.f, true);
                }
                *reinterpret_cast<Words *>(buffer + row * kPitch + (((piece * 2 + h) ^ (row & 15)) * 16)) = y.w;
            }
        }
#pragma unroll
        for (int m = 0; m < kMyScales; ++m) {
            const int at = m * kThreads + threadIdx.x;
            if (at < kScales)
                reinterpret_cast<float *>(buffer + kA)[at] = scales[m];
        }
    };
    const auto barrier = [&] {  // LDS is written and read; loads stay on their way
        __builtin_amdgcn_s_waitcnt(0xC07F);
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };

    f32x4 acc[KN] = {};
    i32x8 x[D];
    load_a(0);
#pragma unroll
    for (int i = 0; i < D; ++i)
        x[i] = load_b(i < blocks ? i : blocks - 1);
    keep_a(lds);
    barrier();
    for (int base = 0; base < blocks; base += D) {
#pragma unroll
        for (int i = 0; i < D; ++i) {
            const int kb = base + i;
            if (kb >= blocks)
                break;
            const int chunk = kb / C;
            const bool more = (chunk + 1) * C < blocks;
            if (i % C == 0 && more)
                load_a(chunk + 1);
            const char *const buffer = lds + (chunk & 1) * kBuffer;
            const float *const sc = reinterpret_cast<const float *>(buffer + kA);
            Fragment8<true> fb;
            fb.set(x[i]);
            if (kb + D < blocks)
                x[i] = load_b(kb + D);
            const float tile_scale = TILES ? sb_tile[kb] : 1.f;
            f32x4 sb = {1.f, 1.f, 1.f, 1.f};
            if constexpr (!TILES)
                sb = *reinterpret_cast<const f32x4 *>(sc + C * kRows + i % C * kCols + wave * 16 + (lane >> 4) * 4);
#pragma unroll
            for (int j = 0; j < KN; ++j) {
                f32x4 p = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int h = 0; h < 4; ++h) {
                    const int unit = i % C * 16 + ((lane >> 4) + (h >> 1) * 4) * 2 + (h & 1);
                    const bf16x8 fa = *reinterpret_cast<const bf16x8 *>(buffer + (j * 16 + (lane & 15)) * kPitch +
                                                                        ((unit ^ (lane & 15)) * 16));
                    p = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fb.part[h], fa, p, 0, 0, 0);
                }
                const float sa = sc[i % C * kRows + j * 16 + (lane & 15)] * tile_scale;
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    acc[j][e] = __builtin_fmaf(TILES ? p[e] : p[e] * sb[e], sa, acc[j][e]);
            }
            if (i % C == C - 1 && more) {
                keep_a(lds + ((chunk + 1) & 1) * kBuffer);
                barrier();
            }
        }
    }
    barrier();
    // whole lines of the result's rows leave through LDS
#pragma unroll
    for (int j = 0; j < KN; ++j) {
        T y[4];
#pragma unroll
        for (int e = 0; e < 4; ++e)
            y[e] = (T)acc[j][e];
        __builtin_memcpy(lds + (j * 16 + (lane & 15)) * kOutPitch + (wave * 16 + (lane >> 4) * 4) * (int)sizeof(T), y, sizeof y);
    }
    __syncthreads();
    constexpr int kN = 16 / (int)sizeof(T), kPerRow = kCols / kN;
    out += blockIdx.y * split_stride;
    for (int at = threadIdx.x; at < kRows * kPerRow; at += kThreads) {
        const int row = at / kPerRow, col = at % kPerRow * kN;
        if (row >= g.rows)
            break;
        const Words y = *reinterpret_cast<const Words *>(lds + row * kOutPitch + col * (int)sizeof(T));
        T *to = out + row * ld + n0 + col;
        const int left = g.cols - n0 - col;
        if (left >= kN) {
            store_words(to, y);
        } else {
#pragma unroll
            for (int e = 0; e < kN; ++e)
                if (e < left)
                    to[e] = element<T>(y, e);
        }
    }
}

template <typename T, int BM, int BN, int WM, int WN, bool TILES, bool EXACT>
__global__ __launch_bounds__(WM *WN *kWave, 2) void product8_kernel(ProductShape g, T *out, int64_t ld, int64_t split_stride,
                                                                    int split_stages, int tiles_i, int tiles_j)
{
    using P = Product8<BM, BN, WM, WN, TILES, EXACT>;
    __shared__ __attribute__((aligned(1024))) char lds[P::kLdsBytes];
    int ti, tj;
    tile_of_block(blockIdx.x, tiles_i, tiles_j, ti, tj);
    const int from = blockIdx.y * split_stages;
    const int stages = g.blocks - from < split_stages ? g.blocks - from : split_stages;
    f32x4 acc[P::kTm][P::kTn] = {};
    P::run(acc, g, ti * BM, tj * BN, from, stages, lds);
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
    const int wm = wave / WN, wn = wave % WN;
    out += blockIdx.y * split_stride;
    // results leave through LDS in whole lines, 16 rows of them a time
    using Rows = RowStage<T, BM / WM>;
    static_assert(WM * WN * Rows::kBytes <= P::kLdsBytes, "every wave has its rows");
    char *mine = lds + wave * Rows::kBytes;
    __builtin_amdgcn_s_waitcnt(0xC07F);
    P::G::barrier();  // the last stage is read
    const int c0 = ti * BM + wm * (BM / WM);
#pragma unroll
    for (int j = 0; j < P::kTn; ++j) {
        const int r0 = tj * BN + wn * (BN / WN) + j * 16;
        if (r0 >= g.rows)
            break;
#pragma unroll
        for (int i = 0; i < P::kTm; ++i) {
            T y[4];
#pragma unroll
            for (int e = 0; e < 4; ++e)
                y[e] = (T)acc[i][j][e];
            Rows::put(mine, lane, i, y);
        }
        Rows::each(mine, lane, [&](int row, int col, Words y) {
            T *to = out + (int64_t)(r0 + row) * ld + c0 + col;
            const int left = r0 + row < g.rows ? g.cols - c0 - col : 0;
            if (left >= Rows::kN) {
                store_words(to, y);
            } else {
#pragma unroll
                for (int e = 0; e < Rows::kN; ++e)
                    if (e < left)
                        to[e] = element<T>(y, e);
            }
        });
    }
}

}  // namespace

size_t product_f8_workspace_bytes(int, int, int) { return 0; }

hipError_t launch_product_f8(const ProductArgs &a, void *, hipStream_t stream_)
{
    const ProductShape g{{a.b, a.ld_b / 2, a.cols, 0}, {a.a, a.ld_a / 2, a.rows, 0}, a.a_scales, a.b_scales,
                         a.rows, a.cols, a.depth / kScaleBlock};
    const auto go = [&](auto kernel, auto zero, int side_i, int side_j, int threads) {
        using T = decltype(zero);
        const int ti = (a.cols + side_i - 1) / side_i, tj = (a.rows + side_j - 1) / side_j;
        kernel<<<dim3((unsigned)(ti * tj)), threads, 0, stream_>>>(g, static_cast<T *>(a.out), a.ld_out, 0, g.blocks, ti, tj);
    };
    const auto sides = [&](auto tiles, auto zero, auto exact) {
        using T = decltype(zero);
        constexpr bool kTiles = decltype(tiles)::value, kExact = decltype(exact)::value;
        const auto stream = [&](auto kernel, int waves) {
            kernel<<<dim3((unsigned)((a.cols + waves * 16 - 1) / (waves * 16))), waves * kWave, 0, stream_>>>(
                g, static_cast<T *>(a.out), a.ld_out, 0, g.blocks);
        };
        if constexpr (kExact) {
            if (a.rows <= 16)
                return stream(stream8_kernel<T, 1, 4, 2, 4, kTiles>, 4);
            if (a.rows <= 32)
                return stream(stream8_kernel<T, 2, 4, 2, 4, kTiles>, 4);
            if (a.rows <= 64)
                return stream(stream8_kernel<T, 4, 8, 2, 2, kTiles>, 8);
        }
        if constexpr (!kExact)
            if (a.rows > 256)
                return go(product8_kernel<T, 256, 256, 2, 4, kTiles, kExact>, zero, 256, 256, 512);
        go(product8_kernel<T, 128, 128, 2, 2, kTiles, kExact>, zero, 128, 128, 256);
    };
    const auto types = [&](auto tiles) {
        if (a.dtype == 1)
            a.rows > 256 ? sides(tiles, __bf16{}, std::false_type{}) : sides(tiles, __bf16{}, std::true_type{});
        else
            sides(tiles, float{}, std::true_type{});
    };
    a.tiles ? types(std::true_type{}) : types(std::false_type{});
    return last_launch();
}

}  // namespace dv
