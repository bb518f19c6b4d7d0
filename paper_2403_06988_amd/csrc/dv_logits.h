// Internal declarations of the operators between a model's last layer and its
// next token: RMS norm (dv_norm.hip), quantization in blocks (dv_quantize.hip),
// products of 8-bit operands (dv_product.hip) and adjusted logits (dv_adjust.hip).
#pragma once

#include "dv_train.h"

namespace dv {

constexpr int kScaleBlock = 128;  // columns, or rows and columns, of a scale
constexpr int64_t up_block(int64_t n) { return (n + kScaleBlock - 1) / kScaleBlock * kScaleBlock; }

// ------------------------------------------------------------- e4m3 values
//
// A block's scale takes its largest magnitude to e4m3's largest, 448; magnitudes
// below 2^-100 count as that, so that a scale and its reciprocal are normal
// numbers.  An infinity or a NaN in a block makes NaN of all of it.
struct BlockScale {
    float scale, inv;  // both NaN where the block is

    BlockScale() = default;
    __device__ __forceinline__ BlockScale(float scale, float inv) : scale(scale), inv(inv) {}
    // `largest`: the bits of the largest magnitude (as whole numbers they order as the
    // values do, infinity and then NaN above the rest)
    __device__ __forceinline__ explicit BlockScale(uint32_t largest)
    {
        scale = largest >= 0x7F800000u ? __uint_as_float(0x7FC00000u) : fmaxf(__uint_as_float(largest), 0x1p-100f) / 448.f;
        inv = 1.f / scale;
    }
    // x / scale correctly rounded: one Newton step on the product with the correctly rounded
    // reciprocal.  Quotients of bf16 values often lie on the border between two
    // e4m3 values (448 = 7 * 64), where a product alone would fall to either side.
    // The step makes +0 of -0.
    __device__ __forceinline__ float quotient(float x) const
    {
        const float t = x * inv;
        return __builtin_fmaf(__builtin_fmaf(-t, scale, x), inv, t);
    }
};

__device__ __forceinline__ uint32_t magnitude(float x) { return __float_as_uint(x) & 0x7FFFFFFFu; }
__device__ __forceinline__ uint32_t larger(uint32_t a, uint32_t b) { return a > b ? a : b; }

// Four e4m3 values in a word, the first lowest; to nearest, ties to even.
__device__ __forceinline__ uint32_t to_e4m3(float a, float b, float c, float d)
{
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
}

// Eight values of a block in e4m3.
__device__ __forceinline__ uint2 quantize8(const float (&x)[8], const BlockScale &s)
{
    float t[8];
#pragma unroll
    for (int e = 0; e < 8; ++e)
        t[e] = s.quotient(x[e]);
    const bool bad = s.inv != s.inv;
    return {bad ? 0x7F7F7F7Fu : to_e4m3(t[0], t[1], t[2], t[3]), bad ? 0x7F7F7F7Fu : to_e4m3(t[4], t[5], t[6], t[7])};
}

// Largest of 16 lanes' values (lanes 0-15, 16-31, ...), in each of them.
__device__ __forceinline__ uint32_t largest16(uint32_t v)
{
    v = larger(v, dpp_move<kDppQuadSwap1>(v));
    v = larger(v, dpp_move<kDppQuadSwap2>(v));
    v = larger(v, dpp_move<kDppRowHalfMirror>(v));
    return larger(v, dpp_move<kDppRowMirror>(v));
}

// Eight consecutive elements of a row of n, from column c on (zeros past n), as they lie:
// asked for here, turned to fp32 where they are needed, so that several are on their way at once.
template <typename T>
struct Raw8 {
    Words w[sizeof(T) / 2];

    __device__ __forceinline__ void load(const T *row, int c, int n)
    {
        constexpr int kN = 16 / (int)sizeof(T);
        if (c + 8 <= n) {
#pragma unroll
            for (int i = 0; i < (int)sizeof(T) / 2; ++i)
                w[i] = load_words(row + c + i * kN);
        } else {
            T t[8];
#pragma unroll
            for (int e = 0; e < 8; ++e)
                t[e] = c + e < n ? row[c + e] : T(0);
            __builtin_memcpy(w, t, sizeof t);
        }
    }
    __device__ __forceinline__ void zero()
    {
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i)
            w[i] = Words{0, 0, 0, 0};
    }
    __device__ __forceinline__ void to(float (&x)[8]) const
    {
        if constexpr (sizeof(T) == 2) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                x[2 * e] = __uint_as_float(w[0][e] << 16);
                x[2 * e + 1] = __uint_as_float(w[0][e] & 0xFFFF0000u);
            }
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                x[e] = __uint_as_float(w[e / 4][e % 4]);
        }
    }
};

// The same to memory, rounded once to T (uint16_t: bf16).
template <typename T>
__device__ __forceinline__ void store8(T *row, int c, int n, const float (&x)[8])
{
    if (c + 8 <= n) {
        if constexpr (sizeof(T) == 2) {
            store_words(row + c, Words{narrow_pair(x[0], x[1]), narrow_pair(x[2], x[3]), narrow_pair(x[4], x[5]),
                                       narrow_pair(x[6], x[7])});
        } else {
            store_words(row + c, Words{__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3])});
            store_words(row + c + 4, Words{__float_as_uint(x[4]), __float_as_uint(x[5]), __float_as_uint(x[6]), __float_as_uint(x[7])});
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (c + e < n) {
                if constexpr (sizeof(T) == 2)
                    row[c + e] = narrow(x[e]);
                else
                    row[c + e] = x[e];
            }
    }
}

// ------------------------------------------------------------------ RMS norm
struct NormArgs {
    const void *x;
    int64_t ld_x;
    const void *residual;  // NULL: the norm is of x itself
    int64_t ld_residual;
    const void *weight;
    int dtype, rows, hidden;
    float eps;
    void *total;  // x + residual, or NULL
    void *out;    // NULL, or the result in the inputs' type
    float *rstd;  // NULL, or a row's 1 / rms
    uint8_t *q;   // NULL, or the result in e4m3, rows of up_block(hidden)
    float *scales;
};
hipError_t launch_rms_norm(const NormArgs &a, hipStream_t stream);

struct NormGradArgs {
    const void *grad_out;
    int64_t ld_grad_out;
    const void *total;
    int64_t ld_total;
    const void *weight;
    const float *rstd;
    const void *grad_total;  // NULL: zeros
    int64_t ld_grad_total;
    int dtype, rows, hidden;
    void *grad_x, *grad_weight;  // either may be NULL
};
size_t rms_norm_backward_workspace_bytes(int rows, int hidden);
hipError_t launch_rms_norm_backward(const NormGradArgs &a, void *workspace, hipStream_t stream);

// -------------------------------------------------------------- quantization
struct QuantizeArgs {
    const void *x;
    int64_t ld_x;
    int dtype, rows, cols;
    bool tiles;  // a scale for 128 x 128, else for 128 columns of a row (of the transposed: 128 rows of a column)
    uint8_t *q;
    float *scales;
    uint8_t *qt;
    float *t_scales;
};
hipError_t launch_quantize_f8(const QuantizeArgs &a, hipStream_t stream);

// ------------------------------------------------------------------ products
struct ProductArgs {
    const uint8_t *a;
    int64_t ld_a;
    const float *a_scales;  // [depth / 128][rows]
    const uint8_t *b;
    int64_t ld_b;
    const float *b_scales;  // tiles: [cols / 128][depth / 128], else [depth / 128][cols]
    bool tiles;
    int rows, cols, depth;
    int dtype;  // of the result
    bool exact; // exact sums, whatever the type and rows
    void *out;
    int64_t ld_out;
};
size_t product_f8_workspace_bytes(int rows, int cols, int depth);
size_t product_f8_workspace_bytes_up_to(int rows, int cols, int depth);
hipError_t launch_product_f8(const ProductArgs &a, void *workspace, hipStream_t stream);

// ----------------------------------------------------------- adjusted logits
struct AdjustArgs {
    const void *logits;
    int64_t ld;
    int dtype, rows, V;
    const int32_t *history;
    int64_t ld_history;
    int max_history;
    const int32_t *lengths, *prompt_lengths;
    const float *repetition, *presence, *frequency;
    const int32_t *bias_ids;
    const float *bias;
    int num_bias;
    Masks masks;
    void *out;
    int64_t ld_out;
};
hipError_t launch_adjust_logits(const AdjustArgs &a, hipStream_t stream);

}  // namespace dv
