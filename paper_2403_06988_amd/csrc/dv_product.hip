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
typedef __attribute__((ext_vector_type(4))) int i32x4;

__device__ __forceinline__ f32x4 mfma8(i32x8 a, i32x8 b)
{
    const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, zero, 0, 0, 0, 0, 0, 0);
}

struct ProductShape {
    GemmOperand b, a;  // in units of two bytes, as dv_gemm.h takes them
    const float *sa, *sb;
    int rows, cols;
    int blocks;        // of 128 k
};

template <int BM, int BN, int WM, int WN, bool TILES>
struct Product8 {
    using G = Gemm<__bf16, BM, BN, WM, WN>;
    using A = typename G::A;
    using B = typename G::B;
    static constexpr int kTm = G::kTm, kTn = G::kTn, kLoads = G::kLoads;
    static constexpr int kLdsBytes = G::kLdsBytes;
    static_assert(!TILES || BM / WM <= kScaleBlock, "one scale of b a wave");

    template <typename S>
    static __device__ __forceinline__ i32x8 fragment(const char *tile, int at0, int at1, int i)
    {
        union {
            bf16x8 half[2];
            i32x8 v;
        } f;
        f.half[0] = S::fragment(tile, at0, i);
        f.half[1] = S::fragment(tile, at1, i);
        return f.v;
    }

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
        int stage = from;
        const auto load = [&](int slot) {
            const uint32_t dst = (uint32_t)(uintptr_t)(typename G::Lds)(lds + slot * G::kStageBytes);
            const int64_t at = (int64_t)stage * 128;
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

        // the scales' places: columns past the end read the last one
        int jcol[kTn];
#pragma unroll
        for (int j = 0; j < kTn; ++j) {
            const int c = j0 + wn * (BN / WN) + j * 16 + (lane & 15);
            jcol[j] = c < g.rows ? c : g.rows - 1;
        }
        const int iw = i0 + wm * (BM / WM);
        const float *sb_tile = g.sb + (int64_t)((iw < g.cols ? iw : g.cols - 1) / kScaleBlock) * g.blocks;

        load(0);
        if (stages > 1)
            load(1);
        for (int s = 0; s < stages; ++s) {
            const int kb = from + s;
            float sa[kTn];
#pragma unroll
            for (int j = 0; j < kTn; ++j)
                sa[j] = g.sa[(int64_t)kb * g.rows + jcol[j]];
            if constexpr (TILES) {
                const float sb = sb_tile[kb];
#pragma unroll
                for (int j = 0; j < kTn; ++j)
                    sa[j] *= sb;
            }
            if (s + 1 < stages)
                G::template wait_loads<kLoads>();
            else
                G::template wait_loads<0>();
            G::barrier();
            const char *tile = lds + (s & 1) * G::kStageBytes;
            i32x8 fb[kTn];
#pragma unroll
            for (int j = 0; j < kTn; ++j)
                fb[j] = fragment<B>(tile + A::kBytes, b0, b1, j);
#pragma unroll
            for (int i = 0; i < kTm; ++i) {
                const i32x8 fa = fragment<A>(tile, a0, a1, i);
                f32x4 sb = {1.f, 1.f, 1.f, 1.f};
                if constexpr (!TILES)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int c = iw + i * 16 + (lane >> 4) * 4 + e;
                        sb[e] = g.sb[(int64_t)kb * g.cols + (c < g.cols ? c : g.cols - 1)];
                    }
#pragma unroll
                for (int j = 0; j < kTn; ++j) {
                    const f32x4 p = mfma8(fa, fb[j]);
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        acc[i][j][e] = __builtin_fmaf(TILES ? p[e] : p[e] * sb[e], sa[j], acc[i][j][e]);
                }
            }
            __builtin_amdgcn_s_waitcnt(0xC07F);  // this wave's reads from LDS are done
            G::barrier();                        // and every wave's are
            if (s + 2 < stages)
                load(s & 1);
        }
    }
};

template <typename T, int BM, int BN, int WM, int WN, bool TILES>
__global__ __launch_bounds__(WM *WN *kWave, 2) void product8_kernel(ProductShape g, T *out, int64_t ld, int64_t split_stride,
                                                                    int split_stages, int tiles_i, int tiles_j)
{
    using P = Product8<BM, BN, WM, WN, TILES>;
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
#pragma unroll
    for (int j = 0; j < P::kTn; ++j) {
        const int r = tj * BN + wn * (BN / WN) + j * 16 + (lane & 15);
        if (r >= g.rows)
            continue;
#pragma unroll
        for (int i = 0; i < P::kTm; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int c = ti * BM + wm * (BM / WM) + i * 16 + (lane >> 4) * 4 + e;
                if (c < g.cols)
                    out[r * ld + c] = (T)acc[i][j][e];
            }
    }
}

}  // namespace

size_t product_f8_workspace_bytes(int, int, int) { return 0; }

hipError_t launch_product_f8(const ProductArgs &a, void *, hipStream_t stream)
{
    const ProductShape g{{a.b, a.ld_b / 2, a.cols, 0}, {a.a, a.ld_a / 2, a.rows, 0}, a.a_scales, a.b_scales,
                         a.rows, a.cols, a.depth / kScaleBlock};
    const auto go = [&](auto tiles, auto zero) {
        using T = decltype(zero);
        constexpr int kSide = 128;
        const int ti = (a.cols + kSide - 1) / kSide, tj = (a.rows + kSide - 1) / kSide;
        product8_kernel<T, kSide, kSide, 2, 2, decltype(tiles)::value>
            <<<dim3((unsigned)(ti * tj)), 256, 0, stream>>>(g, static_cast<T *>(a.out), a.ld_out, 0, g.blocks, ti, tj);
    };
    if (a.dtype == 1)
        a.tiles ? go(std::true_type{}, __bf16{}) : go(std::false_type{}, __bf16{});
    else
        a.tiles ? go(std::true_type{}, float{}) : go(std::false_type{}, float{});
    return last_launch();
}

}  // namespace dv
