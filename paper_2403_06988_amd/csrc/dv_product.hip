// Products of e4m3 operands with block scales:
//
//     out[m][n] = sum over blocks kb of 128 k:  sa[kb][m] sb(kb, n) sum_{k in kb} a[m][k] b[n][k]
//
// sb is one number for 128 n (tiles), or one for each n.  A block's sum of 128 products leaves
// the matrix instruction (16 x 16 x 128) in fp32 and is added to the result's sum under
// its scales; where these might leave fp32's range on the way and the result not, in more steps (Factors).
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

// Scales lie from 2^-109 to 2^119 (a caller's own anywhere): sa sb, or by rows a block's sum under
// sb, may be subnormal or past the largest where the result is neither.  Where no scale is such
// (is_far), which is nearly always, a tile is summed the short way:
//     tiles     sum * (sa sb), sa sb a normal number: one rounding
//     by rows   (sum * sb) * sa, sb from 2^-109 (a block of zeros' scale is above) to 2^103: a sum is
//               a multiple of 2^-18 and at most 2^25
// A block that has met one that is sums its tile again the long way (FAR): sa sb, or sa, in two factors, a
// power of two from 2^-100 to 2^95, under which a sum is exact, and the rest, which is at least 1/4
// (by rows 1) unless the power is the least: what leaves the range then is the result.
struct alignas(8) Factors {
    float power, rest;

    __device__ __forceinline__ Factors(float mantissa, int exponent)
    {
        const int e = exponent < -100 ? -100 : exponent > 95 ? 95 : exponent;
        const int left = exponent - e < 127 ? exponent - e : 127;  // past it every sum but 0 is infinite
        power = __builtin_ldexpf(1.f, e);
        rest = __builtin_ldexpf(mantissa, left);
    }
    static __device__ __forceinline__ Factors of(float s)
    {
        return Factors(2.f * __builtin_amdgcn_frexp_mantf(s), __builtin_amdgcn_frexp_expf(s) - 1);
    }
    static __device__ __forceinline__ Factors of(float s, float t)
    {
        return Factors(__builtin_amdgcn_frexp_mantf(s) * __builtin_amdgcn_frexp_mantf(t),
                       __builtin_amdgcn_frexp_expf(s) + __builtin_amdgcn_frexp_expf(t));
    }
};
// Whether a scale asks for the long way: sa sb by tiles, sb by rows.
template <bool TILES>
__device__ __forceinline__ bool is_far(float s)
{
    s = __builtin_fabsf(s);
    return TILES ? !(s >= 0x1p-126f && s <= 0x1.fffffep127f) : !(s >= 0x1p-109f && s < 0x1p103f);
}

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
    // Fragments of b on their way from LDS, and products on their way before one is added under
    // its scales: 8,192 x 32,000 x 4,096 (8-bit instructions) with 1 and 1 1.13 ms, 2 and 1 1.10,
    // 2 and 2 1.04.
    static constexpr int kAhead = EXACT ? 1 : 2, kLag = EXACT ? 1 : 2;
    // A stage's loads are asked for one after kPerLoad products, the first kEarly of them as soon as
    // the stage before the last has been read: all of a block's at once hold up every wave (the
    // same product: 1.10 ms; exact, 4,096 in each direction, all at once 127 us, one a product 126).
    static constexpr int kPerLoad = EXACT ? 1 : 2;
    static constexpr int kEarly = kAhead * kTn / kPerLoad < kLoads ? kAhead * kTn / kPerLoad : kLoads;
    static_assert(kLag < 4 && kTn % kPerLoad == 0, "four products are held");
    static_assert(kEarly + (kTm - kAhead) * (kTn / kPerLoad) >= kLoads, "every load has its place");
    static_assert(kTm % 4 == 0 && kTm % kAhead == 0 && kAhead <= 2, "a stage is whole turns of the fragments' and scales' places");
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

    // acc += the tile at i0 of b and j0 of a, over `stages` blocks of 128 k from `from` on.  Whether one of this
    // lane's scales asked for the long way.
    template <bool FAR>
    static __device__ __forceinline__ bool run(f32x4 (&acc)[kTm][kTn], const ProductShape &g, int i0, int j0, int from,
                                               int stages, char *lds)
    {
        bool far = false;
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
        // this wave's loads i0 to i1 of stage s
        const auto load = [&](int s, int i0, int i1) {
            const uint32_t dst = (uint32_t)(uintptr_t)(typename G::Lds)(lds + (s & 1) * kStageBytes);
            const int64_t at = (int64_t)(from + s) * kScaleBlock;
            if (!TILES && i0 == 0 && loads_scales)
                load_word_to_lds(g.sb + (int64_t)(from + s) * g.cols, scale_at * 4, dst + G::kStageBytes + wave * kWave * 4);
#pragma unroll
            for (int i = 0; i < kLoads; ++i) {
                if (i < i0 || i >= i1)
                    continue;
                const int p = group + i;
                G::load_to_lds((side_a(i) ? start_a : start_b) + at, voff[i],
                               dst + (side_a(i) ? p * A::kPitch : A::kBytes + (p - A::kGroups) * B::kPitch));
            }
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
        float scale[kTn], power[kTn], next_scale[kTn], next_sb = 1.f;
        // by rows: b's scales of the stage in this buffer, 64 of them a wave
        const auto check_sb = [&](const char *tile) {
            far |= is_far<false>(*reinterpret_cast<const float *>(tile + G::kStageBytes + (wave * kWave % BM + lane) * 4));
        };
        static_assert(TILES || (BM % kWave == 0 && BM / kWave <= kWaves), "the waves check all of them");
        const auto load_scales = [&](int kb) {
            const float *p = g.sa + (int64_t)kb * g.rows;
#pragma unroll
            for (int j = 0; j < kTn; ++j)
                next_scale[j] = p[at_sa[j]];
            if constexpr (TILES)
                next_sb = sb_tile[kb];
        };

        load_scales(from);
        load(0, 0, kLoads);
        G::template wait_loads<0>();
        G::barrier();
        if (stages > 1)
            load(1, 0, kEarly);
        Fragment fa, fb[kTn];
        f32x4 p[4];
        i32x8 next[kAhead];
        f32x4 sb[4];  // of the row before, this one and those ahead
        const auto read = [&](const char *tile, int i) {
            next[i % kAhead] = raw<A>(tile, a0, a1, i);
            if constexpr (!TILES)
                sb[i & 3] = *reinterpret_cast<const f32x4 *>(tile + at_scales + i * 64);
        };
#pragma unroll
        for (int i = 0; i < kAhead; ++i)
            read(lds, i);
#pragma unroll
        for (int j = 0; j < kTn; ++j)
            fb[j].set(raw<B>(lds + A::kBytes, b0, b1, j));
        for (int s = 0; s < stages; ++s) {
            const char *tile = lds + (s & 1) * kStageBytes;
            // a finished product, under its scales
            const auto add = [&](int i, int j) {
                const f32x4 x = p[(i * kTn + j) & 3];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float y = FAR ? x[e] * power[j] : x[e];
                    acc[i][j][e] = __builtin_fmaf(TILES ? y : y * sb[i & 3][e], scale[j], acc[i][j][e]);
                }
                // here, not where the compiler would sink it to: that takes registers for every product
                asm volatile("" : "+v"(acc[i][j]));
            };
#pragma unroll
            for (int j = 0; j < kTn; ++j) {
                if constexpr (FAR) {
                    const Factors f = TILES ? Factors::of(next_scale[j], next_sb) : Factors::of(next_scale[j]);
                    power[j] = f.power;
                    scale[j] = f.rest;
                } else {
                    scale[j] = TILES ? next_scale[j] * next_sb : next_scale[j];
                    if constexpr (TILES)
                        far |= is_far<true>(scale[j]);
                }
            }
            if constexpr (!FAR && !TILES)
                check_sb(tile);
            if (s + 1 < stages)
                load_scales(from + s + 1);
#pragma unroll
            for (int i = 0; i < kTm; ++i) {
                fa.set(next[i % kAhead]);
                if (i + kAhead < kTm) {
                    read(tile, i + kAhead);
                } else if (s + 1 < stages) {
                    if (i + kAhead == kTm) {
                        G::template wait_loads<0>();  // and this wave's reads of the stage
                        G::barrier();
                    }
                    read(lds + ((s + 1) & 1) * kStageBytes, i + kAhead - kTm);
                }
                // a product at a time, one before it added while it runs, and a load asked for
#pragma unroll
                for (int j = 0; j < kTn; ++j) {
                    const int at = i * kTn + j;
                    p[at & 3] = Fragment::multiply(fa, fb[j]);
                    if (at >= kLag)
                        add((at - kLag) / kTn, (at - kLag) % kTn);
                    if (j % kPerLoad == kPerLoad - 1) {
                        const int early = (i + kAhead - kTm) * (kTn / kPerLoad) + j / kPerLoad;
                        const int late = kEarly + i * (kTn / kPerLoad) + j / kPerLoad;
                        if (i + kAhead >= kTm && early < kEarly && s + 2 < stages)
                            load(s + 2, early, early + 1);
                        else if (late < kLoads && s + 1 < stages)
                            load(s + 1, late, late + 1);
                    }
                    __builtin_amdgcn_sched_barrier(0);
                    if (i + 1 == kTm && s + 1 < stages)
                        fb[j].set(raw<B>(lds + ((s + 1) & 1) * kStageBytes + A::kBytes, b0, b1, j));
                }
            }
#pragma unroll
            for (int l = kLag; l > 0; --l)
                add((kTm * kTn - l) / kTn, (kTm * kTn - l) % kTn);
        }
        return far;
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
// used.  a's rows are shared through LDS, C blocks of k at a time in two buffers, as
// bf16 (turned once a block, not once a wave), with the scales; a chunk is asked for two chunks
// ahead, so that what waits for it leaves the later blocks of b on their way.  An a row's 16-byte unit u stands
// at place u ^ (row mod 16): the 16 rows that are read at once meet distinct banks.
//
// Scales always go the long way (Factors): four multiplications more a fragment, in time that the loads take anyway.
//
// 128,256 x 4,096: 16 rows 101 us (5.3 TB/s; loads alone in this pattern 95), 32 rows 110, 64 rows
// 125 (4.3 TB/s); 1 x 1,024 x 32,000 9.0 us, most of them the call.
template <typename T, int KN, int WAVES, int C, int D, bool TILES>
__global__ __launch_bounds__(WAVES *kWave, KN == 1 ? 4 : 3)
    void stream8_kernel(ProductShape g, T *out, int64_t ld, int64_t split_stride, int split_blocks)
{
    static_assert(D % (2 * C) == 0, "a turn of b's places is a whole turn of the two chunks that are held");
    constexpr int kRows = 16 * KN, kThreads = WAVES * kWave, kCols = WAVES * 16;
    constexpr int kPitch = C * kScaleBlock * 2, kA = kRows * kPitch;
    constexpr int kScales = C * (kRows + (TILES ? 0 : kCols));  // of a chunk: a's, then b's by rows
    constexpr int kBuffer = kA + (kScales + C * kRows) * 4;     // a's in two factors
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
    static_assert(!TILES || kScaleBlock % kCols == 0, "a block of threads lies in one tile of b's scales");
    struct Held {
        Words pieces[kMine];
        float scales[kMyScales], tile_scales[TILES ? kMyScales : 1];
    };
    Held held[2];
    const auto load_a = [&](Held &to, int chunk) {
        Words (&pieces)[kMine] = to.pieces;
        float (&scales)[kMyScales] = to.scales;
        // (b's scales by tiles with a's: one read by itself for each block of k would wait for everything before it)
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
            const int at = m * kThreads + (int)threadIdx.x < kScales ? m * kThreads + (int)threadIdx.x : kScales - 1;
            if (TILES || at < C * kRows) {
                const int r = at % kRows;
                scales[m] = g.sa[(int64_t)(from + block(at / kRows)) * g.rows + (r < g.rows ? r : g.rows - 1)];
                if constexpr (TILES)
                    to.tile_scales[m] = g.sb[(int64_t)(n0 / kScaleBlock) * g.blocks + from + block(at / kRows)];
            } else {
                const int c = n0 + (at - C * kRows) % kCols;
                scales[m] = g.sb[(int64_t)(from + block((at - C * kRows) / kCols)) * g.cols + (c < g.cols ? c : g.cols - 1)];
            }
        }
    };
    const auto keep_a = [&](const Held &from, char *buffer) {
        const Words (&pieces)[kMine] = from.pieces;
        const float (&scales)[kMyScales] = from.scales;
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
            if (at < C * kRows)
                reinterpret_cast<Factors *>(buffer + kA)[at] =
                    TILES ? Factors::of(scales[m], from.tile_scales[TILES ? m : 0]) : Factors::of(scales[m]);
            else if (at < kScales)
                reinterpret_cast<float *>(buffer + kA)[C * kRows + at] = scales[m];
        }
    };
    const auto barrier = [&] {  // LDS is written and read; loads stay on their way
        __builtin_amdgcn_s_waitcnt(0xC07F);
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };

    f32x4 acc[KN] = {};
    i32x8 x[D];
    load_a(held[0], 0);
    if (C < blocks)
        load_a(held[1], 1);
#pragma unroll
    for (int i = 0; i < D; ++i)
        x[i] = load_b(i < blocks ? i : blocks - 1);
    keep_a(held[0], lds);
    barrier();
    // a lane's units of a fragment of a: h's sixteen bytes of its two pieces
    int place[4];
#pragma unroll
    for (int h = 0; h < 4; ++h)
        place[h] = (lane & 15) * kPitch + (((((lane >> 4) + (h >> 1) * 4) * 2 + (h & 1)) ^ (lane & 15)) * 16);
    // D blocks of k from `base` on.  ALL: as many follow, and nothing is conditional (a load that may not
    // have been asked for makes what waits for an earlier one wait for all: 16 x 128,256 x 4,096 108 us for 101).
    const auto turn = [&](int base, auto all) {
        constexpr bool ALL = decltype(all)::value;
#pragma unroll
        for (int i = 0; i < D; ++i) {
            const int kb = base + i;
            if (!ALL && kb >= blocks)
                break;
            if (i % C == 0 && (ALL || kb + 2 * C < blocks))
                load_a(held[i / C % 2], kb / C + 2);
            constexpr int kTurn = D / C;  // chunks: an even number, so that a chunk's buffer is known here
            static_assert(kTurn % 2 == 0, "two buffers");
            const char *const buffer = lds + i / C % 2 * kBuffer;
            const Factors *const sc = reinterpret_cast<const Factors *>(buffer + kA);
            Fragment8<true> fb;
            fb.set(x[i]);
            if (ALL || kb + D < blocks)
                x[i] = load_b(kb + D);
            f32x4 sb = {1.f, 1.f, 1.f, 1.f};
            if constexpr (!TILES)
                sb = *reinterpret_cast<const f32x4 *>(reinterpret_cast<const float *>(sc + C * kRows) + i % C * kCols + wave * 16 +
                                                      (lane >> 4) * 4);
#pragma unroll
            for (int j = 0; j < KN; ++j) {
                f32x4 p = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int h = 0; h < 4; ++h) {
                    const bf16x8 fa = *reinterpret_cast<const bf16x8 *>(buffer + j * 16 * kPitch + i % C * 256 + place[h]);
                    p = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fb.part[h], fa, p, 0, 0, 0);
                }
                const Factors sa = sc[i % C * kRows + j * 16 + (lane & 15)];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float y = p[e] * sa.power;
                    acc[j][e] = __builtin_fmaf(TILES ? y : y * sb[e], sa.rest, acc[j][e]);
                }
                if constexpr (KN > 2)
                    asm volatile("" : "+v"(acc[j]));  // added here, as in Product8
            }
            if (i % C == C - 1 && (ALL || kb + 1 < blocks)) {
                keep_a(held[(i / C + 1) % 2], lds + (i / C + 1) % 2 * kBuffer);
                barrier();
            }
            __builtin_amdgcn_sched_barrier(0);  // a block of k after the other: registers
        }
    };
    int base = 0;
    for (; base + 2 * D <= blocks; base += D)
        turn(base, std::true_type{});
    for (; base < blocks; base += D)
        turn(base, std::false_type{});
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

// 8-bit instructions: 8,192 x 32,000 x 4,096 1.04 ms (2.06 PFLOP/s), 8,192 x 4,096 x 32,000 0.98 (2.19), b by rows
// 32,000 x 4,096 x 8,192 1.19; bound by the matrix instructions and the adds under the scales, which hardly overlap (without
// the adds 2.85 PFLOP/s).  Exact: 4,096 in each direction 126 us (1.09 PFLOP/s).
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
    if (__syncthreads_or(P::template run<false>(acc, g, ti * BM, tj * BN, from, stages, lds))) {
#pragma unroll
        for (int i = 0; i < P::kTm; ++i)
#pragma unroll
            for (int j = 0; j < P::kTn; ++j)
                acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
        P::template run<true>(acc, g, ti * BM, tj * BN, from, stages, lds);
    }
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

// The sum of the splits' parts [rows][cols], four elements a lane, as rows of the result.
template <typename T>
__global__ __launch_bounds__(256) void join8_kernel(const float *parts, int splits, int rows, int cols, T *out, int64_t ld)
{
    const int vecs = (cols + 3) / 4;
    const int64_t total = (int64_t)rows * vecs, step = (int64_t)rows * cols;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
        const int64_t row = i / vecs;
        const int c = (int)(i - row * vecs) * 4;
        const float *p = parts + row * cols + c;
        T *to = out + row * ld + c;
        f32x4 s = {0.f, 0.f, 0.f, 0.f};
        if (c + 4 <= cols) {
            for (int k = 0; k < splits; ++k)
                s += __builtin_bit_cast(f32x4, load_words(p + k * step));
            const T y[4] = {(T)s[0], (T)s[1], (T)s[2], (T)s[3]};
            __builtin_memcpy(to, y, sizeof y);
        } else {
            for (int e = 0; c + e < cols; ++e) {
                float x = 0.f;
                for (int k = 0; k < splits; ++k)
                    x += p[k * step + e];
                to[e] = (T)x;
            }
        }
    }
}

// ------------------------------------------------------------------- the plan

// How a product is cut: the kernel (few rows, or tiles of a side), and the splits of its
// blocks of 128 k, none of them empty.
struct Plan8 {
    bool exact;
    int side;    // of a tile; 0: the kernel of at most 64 rows
    int waves;   // of one of its blocks
    int splits, blocks;
};

constexpr int kFewRows = 64, kMostSplits = 16;

// The 8-bit matrix instruction cuts eight neighbouring products to 13 bits below the largest of
// them before it adds them up in fp32: at most 7 * 2^-13 of the magnitudes, 1.4e-5 of a sum of
// normal values (measured), where a bf16 result's own rounding is 1.7e-3.  fp32
// results take the products of the same values as bf16, which lose nothing (half the rate: 4,096 in each direction
// 126 us against 63), and so does a call that asks for it.  So do bf16 results of at most 256 rows, a decode step's,
// whose tokens are chosen by differences of logits.  That is for the sums' sake, at a price (x 128,256 x 4,096):
// 65 to 128 rows 161-164 us, by 8-bit instructions 142-150; 129 to 256 rows 283-289, by these 162-172.
bool exact_sums(int rows, int dtype, bool asked) { return asked || dtype == 0 || rows <= 256; }

Plan8 plan_f8(int rows, int cols, int depth, bool exact)
{
    const int blocks = depth / kScaleBlock;
    Plan8 best{exact, 0, 0, 1, blocks};
    if (rows <= kFewRows) {
        best.waves = rows <= 32 ? 4 : 8;
        const int64_t n = (cols + best.waves * 16 - 1) / (best.waves * 16);
        int64_t want = n >= 384 ? 1 : 512 / n;
        want = want < blocks / 4 ? want : blocks / 4;
        want = want < kMostSplits ? want : kMostSplits;
        best.blocks = want > 1 ? (int)((blocks + want - 1) / want) : blocks;
        best.splits = (blocks + best.blocks - 1) / best.blocks;
        return best;
    }
    // By the time that each choice would take: a block of k of all the tiles that a compute unit
    // holds takes `us`, one tile alone two fifths of that and more; a tile costs `around` blocks
    // of k to start and end; splits write and read their sums.
    struct Side {
        int side, per_unit, around;
        double us;
    };
    constexpr Side kFast[] = {{256, 1, 3, 1.85}, {128, 2, 5, 1.2}}, kExact[] = {{128, 2, 4, 1.85}};
    constexpr int kUnits = 256;
    double least = 1e30;
    const auto consider = [&](const Side &s) {
        const int64_t tiles = (int64_t)((rows + s.side - 1) / s.side) * ((cols + s.side - 1) / s.side);
        if (tiles > (int64_t)1 << 22 && s.side < 256 && !best.exact)
            return;
        for (int want = 1; want <= kMostSplits && want <= blocks; ++want) {
            const int per = (blocks + want - 1) / want, used = (blocks + per - 1) / per;
            const int64_t n = tiles * used, slots = (int64_t)kUnits * s.per_unit, rest = n % slots;
            const auto round = [&](int64_t per_unit) {
                return (per + s.around) * s.us * (0.4 + 0.6 * (double)per_unit / s.per_unit);
            };
            const double us = (double)(n / slots) * round(s.per_unit) + (rest ? round((rest + kUnits - 1) / kUnits) : 0) +
                              (used > 1 ? (double)used * rows * cols * 2e-6 + 5 : 0);
            if (us < least) {
                least = us;
                best.side = s.side;
                best.splits = used;
                best.blocks = per;
            }
        }
    };
    if (best.exact)
        for (const Side &s : kExact)
            consider(s);
    else
        for (const Side &s : kFast)
            consider(s);
    return best;
}

size_t parts_bytes(const Plan8 &p, int rows, int cols)
{
    return p.splits > 1 ? align_up((size_t)p.splits * (size_t)rows * (size_t)cols * 4, 256) : 0;
}

template <typename T>
hipError_t launch_product(const ProductArgs &a, const Plan8 &plan, void *workspace, hipStream_t stream)
{
    const ProductShape g{{a.b, a.ld_b / 2, a.cols, 0}, {a.a, a.ld_a / 2, a.rows, 0}, a.a_scales, a.b_scales,
                         a.rows, a.cols, a.depth / kScaleBlock};
    const unsigned splits = (unsigned)plan.splits;
    const auto run = [&](auto tiles, auto *out, int64_t ld, int64_t stride) {
        using O = std::remove_pointer_t<decltype(out)>;
        constexpr bool kTiles = decltype(tiles)::value;
        const auto few = [&](auto kernel) {
            const int n = plan.waves * 16;
            kernel<<<dim3((unsigned)((a.cols + n - 1) / n), splits), plan.waves * kWave, 0, stream>>>(g, out, ld, stride, plan.blocks);
        };
        const auto tiled = [&](auto kernel, int threads) {
            const int ti = (a.cols + plan.side - 1) / plan.side, tj = (a.rows + plan.side - 1) / plan.side;
            kernel<<<dim3((unsigned)(ti * tj), splits), threads, 0, stream>>>(g, out, ld, stride, plan.blocks, ti, tj);
        };
        if (!plan.side) {
            if (a.rows <= 16)
                few(stream8_kernel<O, 1, 4, 2, 4, kTiles>);
            else if (a.rows <= 32)
                few(stream8_kernel<O, 2, 4, 2, 4, kTiles>);
            else
                few(stream8_kernel<O, 4, 8, 2, 4, kTiles>);
        } else if (plan.exact) {
            tiled(product8_kernel<O, 128, 128, 2, 2, kTiles, true>, 256);
        } else if (plan.side == 256) {
            tiled(product8_kernel<O, 256, 256, 2, 4, kTiles, false>, 512);
        } else {
            tiled(product8_kernel<O, 128, 128, 2, 2, kTiles, false>, 256);
        }
    };
    const auto types = [&](auto *out, int64_t ld, int64_t stride) {
        a.tiles ? run(std::true_type{}, out, ld, stride) : run(std::false_type{}, out, ld, stride);
    };
    T *const out = static_cast<T *>(a.out);
    if (splits == 1) {
        types(out, a.ld_out, 0);
    } else {
        float *const parts = static_cast<float *>(workspace);
        types(parts, a.cols, (int64_t)a.rows * a.cols);
        const int64_t blocks = ((int64_t)a.rows * ((a.cols + 3) / 4) + 255) / 256;
        join8_kernel<<<(unsigned)(blocks < 4096 ? blocks : 4096), 256, 0, stream>>>(parts, plan.splits, a.rows, a.cols, out, a.ld_out);
    }
    return last_launch();
}

}  // namespace

size_t product_f8_workspace_bytes(int rows, int cols, int depth)
{
    const size_t exact = parts_bytes(plan_f8(rows, cols, depth, true), rows, cols);
    const size_t cut = exact_sums(rows, 1, false) ? 0 : parts_bytes(plan_f8(rows, cols, depth, false), rows, cols);
    return exact > cut ? exact : cut;
}

// The most of any call of up to `rows` rows.  Between two multiples of 128 rows (32 and 64 below that) only the
// cost of the parts' sums changes with the rows, so that the splits only fall: the first row's, for all of them.
size_t product_f8_workspace_bytes_up_to(int rows, int cols, int depth)
{
    size_t most = 0;
    for (int64_t first = 1, last; first <= rows; first = last + 1) {
        last = first <= 32 ? 32 : first <= kFewRows ? kFewRows : up_block(first);
        const int end = (int)(last < rows ? last : rows);
        for (bool exact : {true, exact_sums((int)first, 1, false)}) {
            const size_t bytes = parts_bytes(plan_f8((int)first, cols, depth, exact), end, cols);
            most = bytes > most ? bytes : most;
        }
    }
    return most;
}

hipError_t launch_product_f8(const ProductArgs &a, void *workspace, hipStream_t stream)
{
    const Plan8 plan = plan_f8(a.rows, a.cols, a.depth, exact_sums(a.rows, a.dtype, a.exact));
    return a.dtype == 1 ? launch_product<__bf16>(a, plan, workspace, stream) : launch_product<float>(a, plan, workspace, stream);
}

}  // namespace dv
