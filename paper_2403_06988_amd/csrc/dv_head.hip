// Head loss: softmax cross entropy over the allowed tokens, from hidden
// states x [N][D] and head weights w [V][D], in pieces of the vocabulary.
//
//     z_nv = <x_n, w_v>,  lse_n = ln sum over allowed v of exp(z_nv),
//     loss_n = lse_n - z_nt                (t the target; 0 where it is not allowed)
//     G_nv = g_n (exp(z_nv - lse_n) - [v = t]) over allowed v, 0 elsewhere
//     dx = G w,  dw = G^T x.
//
// The logits (4 N V bytes) never reach memory.  Forward: a tile of logits stays
// in the registers of the product that made it and leaves as each row's
// maximum and sum of exponentials over the tile, the target's apart; a second kernel
// joins the tiles.  Backward: a piece of the vocabulary at a time, the same product again,
// its tiles leaving as G, and from the piece's G the two other products.
// Four products of 2 N D V operations against six N D V that cannot be avoided:
// the price of not keeping the logits.
//
// For bf16 operands G leaves as two bf16 parts, 16 bits together, and each of the two
// products runs over both (8,192 x 4,096 x 128,256, loss and gradients: 37.5 ms, with G rounded
// to one part 26.0).  One part costs an error of the size of the results' own rounding: gradients
// off by 0.0024 to 0.0027 of their norm, where that rounding alone makes 0.0017.
//
// All products are the one of dv_gemm.h, which takes operands with k along their
// rows or from row to row: x, w and G are used as they lie.
#include <type_traits>

#include "dv_gemm.h"
#include "dv_head_plan.h"

namespace dv {
namespace {

// ------------------------------------------------------------- preparation

// src [rows][cols] (row stride ld) to rows of out_cols (a multiple of 64), zeros
// past cols: a lane copies 16 bytes, from any element's alignment.
template <typename T>
__global__ __launch_bounds__(256) void pack_kernel(const T *src, int64_t ld, int rows, int cols, int out_cols, T *dst)
{
    constexpr int N = 16 / (int)sizeof(T);
    const int vecs = out_cols / N;
    const int64_t total = (int64_t)rows * vecs;
    for (int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; i < total; i += (int64_t)gridDim.x * blockDim.x) {
        const int64_t row = i / vecs;
        const int col = (int)(i - row * vecs) * N;
        const T *p = src + row * ld + col;
        Words x;
        if (col + N <= cols) {
            x = load_words(p);
        } else {
            union {
                T t[N];
                Words w;
            } part;
#pragma unroll
            for (int e = 0; e < N; ++e)
                part.t[e] = col + e < cols ? p[e] : T(0);
            x = part.w;
        }
        *reinterpret_cast<Words *>(dst + row * out_cols + col) = x;
    }
}

// A wave's results on their way out: 16 rows (index j of the product, one a lane of
// each 16) of COLS columns (index i, four a lane) go through LDS, so that they
// leave as 16-byte pieces of whole lines (8-byte stores of 16 rows at a time,
// straight from the registers, wrote 1 GB at 1.3 TB/s).
template <typename T, int COLS>
struct RowStage {
    static constexpr int kPitch = COLS * (int)sizeof(T) + 16;
    static constexpr int kBytes = 16 * kPitch;
    static constexpr int kN = 16 / (int)sizeof(T);        // elements of a piece
    static constexpr int kLanesPerRow = COLS / kN;
    static constexpr int kRowsAtOnce = kWave / kLanesPerRow;
    static_assert(kLanesPerRow <= kWave && kWave % kLanesPerRow == 0, "whole rows at once");

    // four elements of fragment a, from lane `lane`
    static __device__ __forceinline__ void put(char *lds, int lane, int a, const T (&y)[4])
    {
        __builtin_memcpy(lds + (lane & 15) * kPitch + (a * 16 + (lane >> 4) * 4) * (int)sizeof(T), y, sizeof y);
    }
    // f(row of the 16, first column, piece) for each of this lane's pieces
    template <typename F>
    static __device__ __forceinline__ void each(const char *lds, int lane, F &&f)
    {
        wave_lds_sync();
#pragma unroll
        for (int r = 0; r < 16; r += kRowsAtOnce) {
            const int row = r + lane / kLanesPerRow, piece = lane % kLanesPerRow;
            f(row, piece * kN, *reinterpret_cast<const Words *>(lds + row * kPitch + piece * 16));
        }
        wave_lds_sync();
    }
};

// Parts of an element of G in the operands' type.
template <typename E>
constexpr int parts_of()
{
    return sizeof(E) == 2 ? 2 : 1;
}

// --------------------------------------------------------------- the logits

// Per row and tile: maximum and sum of exponentials of the allowed logits but the
// target's; the target's logit.  i runs over the piece's tokens, j over rows.
// Bound by the matrix instructions: 8,192 x 4,096 x 128,256 bf16 in 6.3 ms, 1.36 PFLOP/s
// (a library product that stores the logits: 5.9 ms); 1 x 1,024 x 32,000 in 13.0 us, by the
// weights' 65 MB; fp32 1,024 x 512 x 32,000 in 200 us, 168
// TFLOP/s (a library product: 249 us).
template <typename E, int BM, int BN, int WM, int WN>
__global__ __launch_bounds__(WM *WN *kWave, 2) void stats_kernel(GemmShape g, int v0, int V, int rows, Masks masks,
                                                                 const int32_t *targets, Softmax *parts,
                                                                 float *target_logit, int tiles_i, int tiles_j)
{
    using G = Gemm<E, BM, BN, WM, WN>;
    __shared__ __attribute__((aligned(1024))) char lds[G::kLdsBytes];
    int ti, tj;
    tile_of_block(blockIdx.x, tiles_i, tiles_j, ti, tj);
    f32x4 acc[G::kTm][G::kTn] = {};
    G::run(acc, g, ti * BM, tj * BN, 0, g.k / G::kStageK, lds);

    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
    const int wm = wave / WN, wn = wave % WN;
    const int vw = v0 + ti * BM + wm * (BM / WM);  // the wave's first token
    const int quarter = lane >> 4;
    constexpr int kWords = BM / WM / 32;
#pragma unroll
    for (int b = 0; b < G::kTn; ++b) {
        const int n = tj * BN + wn * (BN / WN) + b * 16 + (lane & 15);
        const bool live = n < rows;
        const RowMask m(masks, V, live ? n : 0);
        const int t = live ? targets[n] - vw : -1;
        uint32_t word[kWords];
#pragma unroll
        for (int i = 0; i < kWords; ++i)
            word[i] = (m.word((vw >> 5) + i) & ~(t >> 5 == i ? 1u << (t & 31) : 0u)) >> (quarter * 4);
        float top = -INFINITY;
#pragma unroll
        for (int a = 0; a < G::kTm; ++a)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const bool in = word[a >> 1] >> ((a & 1) * 16 + e) & 1u;
                const float z = in ? acc[a][b][e] : -INFINITY;
                top = fmaxf(top, z);
            }
        top = fmaxf(top, __shfl_xor(top, 16));
        top = fmaxf(top, __shfl_xor(top, 32));
        const float base = top == -INFINITY ? 0.f : top;
        float sum = 0.f;
#pragma unroll
        for (int a = 0; a < G::kTm; ++a)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const bool in = word[a >> 1] >> ((a & 1) * 16 + e) & 1u;
                sum += in ? softmax_term(acc[a][b][e], base, kLog2e) : 0.f;
            }
        sum += __shfl_xor(sum, 16);
        sum += __shfl_xor(sum, 32);
        if (live && quarter == 0)
            parts[(size_t)(vw / (BM / WM)) * rows + n] = {top, sum};
        const bool here = (uint32_t)t < (uint32_t)(BM / WM) && ((t >> 2) & 3) == quarter;
        if (__ballot(here)) {
            float z = 0.f;
#pragma unroll
            for (int a = 0; a < G::kTm; ++a)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    z = t == a * 16 + quarter * 4 + e ? acc[a][b][e] : z;
            if (here)
                target_logit[n] = z;
        }
    }
}

// Joins the tiles of each row: blocks of 256 threads take 256 / slices rows.
__global__ __launch_bounds__(256) void finish_kernel(const Softmax *parts, int nparts, int rows, int V, Masks masks,
                                                      const int32_t *targets, const float *target_logit, float *loss,
                                                      float *lse, int slices)
{
    __shared__ Softmax sh[256];
    const int per_block = 256 / slices;
    const int slice = threadIdx.x / per_block;
    const int n = blockIdx.x * per_block + threadIdx.x % per_block;
    Softmax s{-INFINITY, 0.f};
    if (n < rows) {
#pragma unroll 4
        for (int p = slice; p < nparts; p += slices)
            s = softmax_join(s, parts[(size_t)p * rows + n], kLog2e);
    }
    sh[threadIdx.x] = s;
    for (int half = slices / 2; half; half /= 2) {
        __syncthreads();
        if (slice < half)
            sh[threadIdx.x] = softmax_join(sh[threadIdx.x], sh[threadIdx.x + half * per_block], kLog2e);
    }
    if (slice || n >= rows)
        return;
    s = sh[threadIdx.x];
    const int t = targets[n];
    const RowMask m(masks, V, n);
    // s holds every allowed token but the target.  Where the target is the largest, the
    // loss is ln(1 + the others' share of it), to the last bits also where that is small.
    if (!m.has(t)) {
        lse[n] = s.empty() ? -INFINITY : s.max + logf(s.sum);
        loss[n] = 0.f;
        return;
    }
    const float z = target_logit[n];
    if (z >= s.max) {
        const float l = log1pf(s.empty() ? 0.f : s.sum * softmax_term(s.max, z, kLog2e)) + (z - z);  // NaN if z is infinite
        lse[n] = z + l;
        loss[n] = l;
    } else {
        const float lns = logf(s.sum + softmax_term(z, s.max, kLog2e));
        lse[n] = s.max + lns;
        loss[n] = (s.max - z) + lns;
    }
}

// The weight of each row's gradient: grad_loss where the target is allowed, else 0.
__global__ void weights_kernel(int rows, int V, Masks masks, const int32_t *targets, const float *grad_loss, float *weight)
{
    const int n = blockIdx.x * blockDim.x + threadIdx.x;
    if (n < rows)
        weight[n] = RowMask(masks, V, n).has(targets[n]) ? grad_loss[n] : 0.f;
}

// A piece of G: rows of `cols` tokens in fp32, or in two bf16 parts (part_column), zeros from
// the piece's end up to the next multiple of 64 tokens and from the last row up to the next
// whole stage of rows.  8,192 x 4,096 x 16,128 tokens bf16: 910 us, 1.19 PFLOP/s with 528 MB of stores.
template <typename E, int BM, int BN, int WM, int WN>
__global__ __launch_bounds__(WM *WN *kWave, 2) void grad_kernel(GemmShape g, int v0, int V, int rows, Masks masks,
                                                                const int32_t *targets, const float *lse,
                                                                const float *weight, E *out, int cols, int tiles_i,
                                                                int tiles_j)
{
    using G = Gemm<E, BM, BN, WM, WN>;
    __shared__ __attribute__((aligned(1024))) char lds[G::kLdsBytes];
    int ti, tj;
    tile_of_block(blockIdx.x, tiles_i, tiles_j, ti, tj);
    f32x4 acc[G::kTm][G::kTn] = {};
    G::run(acc, g, ti * BM, tj * BN, 0, g.k / G::kStageK, lds);

    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
    const int wm = wave / WN, wn = wave % WN;
    const int lw = ti * BM + wm * (BM / WM);  // the wave's first token in the piece
    const int vw = v0 + lw;
    const int quarter = lane >> 4;
    constexpr int kParts = parts_of<E>();
    const int rows_k = gradient_rows(rows);
    using Rows = RowStage<E, BM / WM>;
    static_assert(WM * WN * Rows::kBytes <= G::kLdsBytes, "every wave has its rows");
    char *mine = lds + wave * Rows::kBytes;
    G::barrier();  // the last stage is read
#pragma unroll
    for (int b = 0; b < G::kTn; ++b) {
        const int n0 = tj * BN + wn * (BN / WN) + b * 16;
        if (n0 >= rows_k)
            break;
        const int n = n0 + (lane & 15);
        const bool live = n < rows;
        const RowMask m(masks, V, live ? n : 0);
        const float w = live ? weight[n] : 0.f;
        const float base = w != 0.f ? lse[n] : 0.f;
        const int t = live ? targets[n] - vw : -1;
#pragma unroll
        for (int a = 0; a < G::kTm; ++a) {
            const uint32_t bits = m.word((vw >> 5) + (a >> 1)) >> (quarter * 4 + (a & 1) * 16);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                float p = (bits >> e & 1u) && w != 0.f ? softmax_term(acc[a][b][e], base, kLog2e) : 0.f;
                p -= t == a * 16 + quarter * 4 + e ? 1.f : 0.f;
                acc[a][b][e] = p * w;
            }
        }
#pragma unroll
        for (int part = 0; part < kParts; ++part) {
#pragma unroll
            for (int a = 0; a < G::kTm; ++a) {
                E y[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    y[e] = (E)acc[a][b][e];
                    acc[a][b][e] -= (float)y[e];  // the rest
                }
                Rows::put(mine, lane, a, y);
            }
            Rows::each(mine, lane, [&](int row, int col, Words y) {
                if (lw + col >= cols)  // 64 divides cols
                    return;
                E *to = out + (int64_t)(n0 + row) * kParts * cols;
                store_words(to + (kParts == 2 ? part_column(lw + col) + part * kPartColumns : lw + col), y);
            });
        }
    }
}

// ------------------------------------------------------- the other products

enum class Out { kStore, kPartial, kPartialAdd };

// C[j][i] of a product as `out_rows` rows of `cols` elements: in T, or in fp32
// as (or on top of) the partial sums of this block's share of k.  A is stored by
// columns, B (G, in two parts if bf16) by columns with COLS_B.  8,192 x 4,096 x 16,128
// tokens bf16: dx 1.43 ms, dw 1.51 over both parts, 1.51 and 1.43 PFLOP/s, bound by the matrix
// instructions.
template <typename E, int BM, int BN, int WM, int WN, bool COLS_B, typename T, Out OUT>
__global__ __launch_bounds__(WM *WN *kWave, 2) void product_kernel(GemmShape g, T *out, int out_rows, int cols,
                                                                   int64_t split_stride, int split_stages, int tiles_i,
                                                                   int tiles_j)
{
    using G = Gemm<E, BM, BN, WM, WN, true, COLS_B, parts_of<E>() == 2>;
    __shared__ __attribute__((aligned(1024))) char lds[G::kLdsBytes];
    int ti, tj;
    tile_of_block(blockIdx.x, tiles_i, tiles_j, ti, tj);
    const int total = g.k / G::kStageK;
    const int from = blockIdx.y * split_stages;
    const int stages = total - from < split_stages ? total - from : split_stages;
    f32x4 acc[G::kTm][G::kTn] = {};
    G::run(acc, g, ti * BM, tj * BN, from, stages, lds);
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
    const int wm = wave / WN, wn = wave % WN;
    out += blockIdx.y * split_stride;
    using Rows = RowStage<T, BM / WM>;
    static_assert(WM * WN * Rows::kBytes <= G::kLdsBytes, "every wave has its rows");
    char *mine = lds + wave * Rows::kBytes;
    G::barrier();  // the last stage is read
    const int c0 = ti * BM + wm * (BM / WM);
#pragma unroll
    for (int b = 0; b < G::kTn; ++b) {
        const int r0 = tj * BN + wn * (BN / WN) + b * 16;
        if (r0 >= out_rows)
            break;
#pragma unroll
        for (int a = 0; a < G::kTm; ++a) {
            T y[4];
#pragma unroll
            for (int e = 0; e < 4; ++e)
                y[e] = (T)acc[a][b][e];
            Rows::put(mine, lane, a, y);
        }
        Rows::each(mine, lane, [&](int row, int col, Words y) {
            T *p = out + (int64_t)(r0 + row) * cols + c0 + col;
            const int left = r0 + row < out_rows ? cols - c0 - col : 0;
            if constexpr (OUT == Out::kPartialAdd) {
                f32x4 before = {};
                if (left >= Rows::kN) {
                    before = __builtin_bit_cast(f32x4, load_words(p));
                } else {
#pragma unroll
                    for (int e = 0; e < Rows::kN; ++e)
                        before[e] = e < left ? p[e] : 0.f;
                }
                y = __builtin_bit_cast(Words, before + __builtin_bit_cast(f32x4, y));
            }
            if (left >= Rows::kN) {
                // the weight's gradient is large and read by nobody here (64 rows x 2048 x
                // 128,256 bf16 with one part of G: 129 us for it, with ordinary stores 217)
                if (COLS_B && OUT == Out::kStore)
                    stream_words(p, y);
                else
                    store_words(p, y);
            } else {
#pragma unroll
                for (int e = 0; e < Rows::kN; ++e)
                    if (e < left)
                        p[e] = element<T>(y, e);
            }
        });
    }
}

// The sum of the splits' parts, n elements each (a lane four of them at a time), in T.
template <typename T>
__global__ __launch_bounds__(256) void join_splits_kernel(const float *parts, int splits, int64_t n, T *out)
{
    const int64_t first = ((int64_t)blockIdx.x * blockDim.x + threadIdx.x) * 4;
    for (int64_t i = first; i < n; i += (int64_t)gridDim.x * blockDim.x * 4) {
        const int left = (int)(n - i < 4 ? n - i : 4);
        f32x4 s = {};
        for (int k = 0; k < splits; ++k) {
            f32x4 x = {};
            if (left == 4)
                x = __builtin_bit_cast(f32x4, load_words(parts + k * n + i));
            else
                for (int e = 0; e < left; ++e)
                    x[e] = parts[k * n + i + e];
            s += x;
        }
        const T y[4] = {(T)s[0], (T)s[1], (T)s[2], (T)s[3]};
        if (left == 4)
            __builtin_memcpy(out + i, y, sizeof y);
        else
            for (int e = 0; e < left; ++e)
                out[i + e] = y[e];
    }
}

template <typename T>
__global__ void zero_kernel(T *p, int64_t n)
{
    for (int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; i < n; i += (int64_t)gridDim.x * blockDim.x)
        p[i] = (T)0.f;
}

// --------------------------------------------------------------- the launches

// An operand as the products need it: in place, or packed into `buffer`.
hipError_t operand(const void *p, int64_t ld, int dtype, int rows, int hidden, bool here, int64_t k, void *buffer,
                   GemmOperand &out, hipStream_t s)
{
    if (here) {
        out = {p, ld, rows, 0};
        return hipSuccess;
    }
    out = {buffer, k, rows, 0};
    const int64_t vecs = (int64_t)rows * (k / (dtype == 1 ? 8 : 4));
    const int64_t blocks = (vecs + 255) / 256;
    const unsigned grid = (unsigned)(blocks < 8192 ? blocks : 8192);
    if (dtype == 1)
        pack_kernel<uint16_t><<<grid, 256, 0, s>>>(static_cast<const uint16_t *>(p), ld, rows, hidden, (int)k,
                                                   static_cast<uint16_t *>(buffer));
    else
        pack_kernel<float><<<grid, 256, 0, s>>>(static_cast<const float *>(p), ld, rows, hidden, (int)k,
                                                static_cast<float *>(buffer));
    return last_launch();
}

#define DV_TRY(call)                   \
    do {                               \
        const hipError_t e_ = (call);  \
        if (e_ != hipSuccess)          \
            return e_;                 \
    } while (0)

template <int BM, int BN, int WN>
struct Tile {
    static constexpr int kM = BM, kN = BN, kWn = WN;
    static constexpr int kThreads = 2 * WN * kWave;
};

// f with the tile of a plan's side; NARROW: whether that may be the 64 x 32 one.
template <bool NARROW, typename F>
hipError_t with_tile(int side, F &&f)
{
    if (side == 256)
        f(Tile<256, 256, 4>{});
    else if (side == 128)
        f(Tile<128, 128, 2>{});
    else if (side == 64)
        f(Tile<64, 64, 2>{});
    else if constexpr (NARROW)
        f(Tile<64, kNarrow, 1>{});
    return last_launch();
}

// An operand stored by rows, seen as one stored by columns: `k` elements a row.
GemmOperand by_columns(const GemmOperand &o, int64_t k)
{
    return {o.p, o.ld, (int)k, o.n};
}

template <typename E, bool COLS_B, typename T, Out OUT>
hipError_t product(const GemmShape &g, const Plan &plan, T *out, int out_rows, int cols, int64_t split_stride, hipStream_t s)
{
    return with_tile<!COLS_B && sizeof(E) == 4>(plan.side, [&](auto tile) {
        using X = decltype(tile);
        const int ti = (cols + X::kM - 1) / X::kM, tj = (out_rows + X::kN - 1) / X::kN;
        const dim3 grid(ti * tj, plan.splits);
        product_kernel<E, X::kM, X::kN, 2, X::kWn, COLS_B, T, OUT><<<grid, X::kThreads, 0, s>>>(
            g, out, out_rows, cols, split_stride, plan.stages, ti, tj);
    });
}

template <typename T>
hipError_t zero(T *p, int64_t n, hipStream_t s)
{
    if (n == 0)
        return hipSuccess;
    const int64_t blocks = (n + 255) / 256;
    zero_kernel<T><<<(unsigned)(blocks < 4096 ? blocks : 4096), 256, 0, s>>>(p, n);
    return last_launch();
}

template <typename T>
hipError_t join_splits(const float *parts, int splits, int64_t n, T *out, hipStream_t s)
{
    const int64_t blocks = (n + 1023) / 1024, most = (int64_t)1 << 23;  // a grid has fewer than 2^32 threads
    join_splits_kernel<T><<<(unsigned)(blocks < most ? blocks : most), 256, 0, s>>>(parts, splits, n, out);
    return last_launch();
}

const void *weight_rows(const HeadArgs &a, int v0)
{
    return static_cast<const char *>(a.weight) + (int64_t)v0 * a.ld_w * (a.dtype == 1 ? 2 : 4);
}

template <typename T>
hipError_t backward(const HeadArgs &a, const float *lse, const float *grad_loss, T *grad_x, T *grad_weight, char *ws,
                    hipStream_t s)
{
    const BackwardLayout l = backward_layout(a.rows, a.hidden, a.V, a.dtype, in_place(a));
    constexpr int kParts = parts_of<T>();
    const int rows_k = gradient_rows(a.rows);
    float *weight = reinterpret_cast<float *>(ws + l.weight), *dx = reinterpret_cast<float *>(ws + l.dx);
    T *g_piece = reinterpret_cast<T *>(ws + l.g);
    constexpr bool kBf16 = sizeof(T) == 2;
    GemmOperand x;
    DV_TRY(operand(a.x, a.ld_x, a.dtype, a.rows, a.hidden, l.here.x, l.k, ws + l.x, x, s));
    weights_kernel<<<(a.rows + 255) / 256, 256, 0, s>>>(a.rows, a.V, a.masks, a.targets, grad_loss, weight);
    DV_TRY(last_launch());
    int splits = 1;
    for (int piece = 0; piece < l.pieces; ++piece) {
        const int v0 = piece * l.piece;
        const int n = a.V - v0 < l.piece ? a.V - v0 : l.piece;
        const int64_t n64 = up64(n);
        GemmOperand w;
        DV_TRY(operand(weight_rows(a, v0), a.ld_w, a.dtype, n, a.hidden, l.here.w, l.k, ws + l.w, w, s));
        const GemmShape logits{w, x, (int)l.k};
        const GemmOperand g{g_piece, kParts * n64, a.rows, 0};
        DV_TRY(with_tile<!kBf16>(logits_side(l, a.rows, n, kBf16), [&](auto tile) {
            using X = decltype(tile);
            const int ti = (n + X::kM - 1) / X::kM, tj = (a.rows + X::kN - 1) / X::kN;
            grad_kernel<T, X::kM, X::kN, 2, X::kWn><<<ti * tj, X::kThreads, 0, s>>>(
                logits, v0, a.V, a.rows, a.masks, a.targets, lse, weight, g_piece, (int)n64, ti, tj);
        }));
        if (grad_x) {
            const GemmShape shape{by_columns(w, l.k), g, (int)(kParts * n64)};
            const int64_t stride = (int64_t)a.rows * a.hidden;
            if (piece == 0) {
                splits = l.dx_plan.splits;
                if (l.pieces == 1 && splits == 1)
                    DV_TRY((product<T, false, T, Out::kStore>(shape, l.dx_plan, grad_x, a.rows, a.hidden, 0, s)));
                else
                    DV_TRY((product<T, false, float, Out::kPartial>(shape, l.dx_plan, dx, a.rows, a.hidden, stride, s)));
            } else {
                // the last piece's k is no longer than the first one's: its splits are no more
                const int stages = (int)(n64 / kGradientStage);
                Plan plan = l.dx_plan;
                plan.splits = (stages + plan.stages - 1) / plan.stages;
                DV_TRY((product<T, false, float, Out::kPartialAdd>(shape, plan, dx, a.rows, a.hidden, stride, s)));
            }
        }
        if (grad_weight) {
            GemmOperand g_t = by_columns(g, n64);
            g_t.k_rows = rows_k;
            const GemmShape shape{by_columns(x, l.k), g_t, kParts * rows_k};
            const Plan plan = dw_plan(l, a.rows, n, kBf16);
            T *out = grad_weight + (int64_t)v0 * a.hidden;
            if (plan.splits == 1) {
                DV_TRY((product<T, true, T, Out::kStore>(shape, plan, out, n, a.hidden, 0, s)));
            } else {
                const int64_t size = (int64_t)n * a.hidden;
                float *dw = reinterpret_cast<float *>(ws + l.dw);
                DV_TRY((product<T, true, float, Out::kPartial>(shape, plan, dw, n, a.hidden, size, s)));
                DV_TRY(join_splits(dw, plan.splits, size, out, s));
            }
        }
    }
    if (grad_x && !(l.pieces == 1 && splits == 1)) {
        DV_TRY(join_splits(dx, splits, (int64_t)a.rows * a.hidden, grad_x, s));
    }
    return hipSuccess;
}

}  // namespace

size_t head_workspace_bytes(const HeadArgs &a)
{
    return forward_layout(a.rows, a.hidden, a.V, a.dtype, in_place(a)).bytes;
}

size_t head_backward_workspace_bytes(const HeadArgs &a)
{
    return backward_layout(a.rows, a.hidden, a.V, a.dtype, in_place(a)).bytes;
}

// For operands of any stride and alignment.
size_t head_workspace_bytes(int rows, int hidden, int V, int dtype)
{
    size_t most = 0;
    for (const InPlace here : {InPlace{false, false}, InPlace{false, true}}) {
        const size_t n = forward_layout(rows, hidden, V, dtype, here).bytes;
        most = n > most ? n : most;
    }
    return most;
}

size_t head_backward_workspace_bytes(int rows, int hidden, int V, int dtype)
{
    size_t most = 0;
    for (const InPlace here : {InPlace{false, false}, InPlace{false, true}}) {
        const size_t n = backward_layout(rows, hidden, V, dtype, here).bytes;
        most = n > most ? n : most;
    }
    return most;
}

hipError_t launch_head_loss(const HeadArgs &a, float *loss, float *lse, void *workspace, hipStream_t s)
{
    const ForwardLayout l = forward_layout(a.rows, a.hidden, a.V, a.dtype, in_place(a));
    char *ws = static_cast<char *>(workspace);
    Softmax *parts = reinterpret_cast<Softmax *>(ws + l.parts);
    float *target_logit = reinterpret_cast<float *>(ws + l.target_logit);
    GemmOperand x;
    DV_TRY(operand(a.x, a.ld_x, a.dtype, a.rows, a.hidden, l.here.x, l.k, ws + l.x, x, s));
    for (int v0 = 0; v0 < a.V; v0 += l.step) {
        const int n = a.V - v0 < l.step ? a.V - v0 : l.step;
        GemmOperand w;
        DV_TRY(operand(weight_rows(a, v0), a.ld_w, a.dtype, n, a.hidden, l.here.w, l.k, ws + l.w, w, s));
        const GemmShape g{w, x, (int)l.k};
        const auto run = [&](auto zero) {
            using E = decltype(zero);
            return with_tile<sizeof(E) == 4>(l.side, [&](auto tile) {
                using X = decltype(tile);
                const int ti = (n + X::kM - 1) / X::kM, tj = (a.rows + X::kN - 1) / X::kN;
                stats_kernel<E, X::kM, X::kN, 2, X::kWn><<<ti * tj, X::kThreads, 0, s>>>(
                    g, v0, a.V, a.rows, a.masks, a.targets, parts, target_logit, ti, tj);
            });
        };
        DV_TRY(a.dtype == 1 ? run((__bf16)0.f) : run(0.f));
    }
    // a thread's share of the parts: about 16, more of them only for many rows
    int slices = 16;
    while (slices < (a.rows < 64 ? 256 : 64) && slices * 16 < l.nparts)
        slices *= 2;
    const int per_block = 256 / slices;
    finish_kernel<<<(a.rows + per_block - 1) / per_block, 256, 0, s>>>(parts, l.nparts, a.rows, a.V, a.masks, a.targets,
                                                                      target_logit, loss, lse, slices);
    return last_launch();
}

hipError_t launch_head_loss_backward(const HeadArgs &a, const float *lse, const float *grad_loss, void *grad_x,
                                     void *grad_weight, void *workspace, hipStream_t s)
{
    if (a.rows == 0) {
        const int64_t n = (int64_t)a.V * a.hidden;
        if (!grad_weight)
            return hipSuccess;
        return a.dtype == 1 ? zero(static_cast<__bf16 *>(grad_weight), n, s) : zero(static_cast<float *>(grad_weight), n, s);
    }
    char *ws = static_cast<char *>(workspace);
    if (a.dtype == 1)
        return backward(a, lse, grad_loss, static_cast<__bf16 *>(grad_x), static_cast<__bf16 *>(grad_weight), ws, s);
    return backward(a, lse, grad_loss, static_cast<float *>(grad_x), static_cast<float *>(grad_weight), ws, s);
}

}  // namespace dv
