// Quantization to e4m3 with a scale for every 128 columns of a row, or for every
// 128 x 128: of a matrix as it lies, transposed, or both in one read.
//
//     scale = max(largest magnitude of the block, 2^-100) / 448
//     q     = e4m3(x / scale)          to nearest of the quotient in fp32
//
// One block of 256 threads takes a 128 x 128 tile: 16 lanes cover a row with 8
// columns each, a thread holds 8 rows of them in registers.  A row's largest value
// is that of 16 lanes; a column's that of a thread's 8 rows, then of the 16
// threads that share its columns, through LDS.  The transposed tile goes through LDS, 8
// bytes (8 rows of a column) a thread and column, and leaves in whole lines.
#include "dv_logits.h"

namespace dv {
namespace {

constexpr int kB = kScaleBlock;

template <typename T, bool TILES, bool ROWS, bool COLUMNS>
__global__ __launch_bounds__(256) void quantize_kernel(const T *x, int64_t ld, int rows, int cols, int tiles_c,
                                                        uint8_t *q, float *scales, uint8_t *qt, float *t_scales)
{
    constexpr int kPitch = kB + 16;  // of a transposed row in LDS
    __shared__ __attribute__((aligned(16))) uint8_t turned[COLUMNS ? kB * kPitch : 16];
    __shared__ uint32_t shared_largest[COLUMNS && !TILES ? 16 * kB : 4];
    const int64_t tile = blockIdx.x;
    const int tr = (int)(tile / tiles_c), tc = (int)(tile % tiles_c);
    const int lane = threadIdx.x & 15, group = threadIdx.x >> 4;
    const int c = tc * kB + lane * 8;          // this thread's 8 columns
    const int r0 = tr * kB + group * 8;        // and its 8 rows
    float v[8][8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        if (r0 + i < rows) {
            load8(v[i], x + (int64_t)(r0 + i) * ld, c, cols);
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                v[i][e] = 0.f;
        }
    }
    uint32_t whole = 0;
    if constexpr (TILES) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
            for (int e = 0; e < 8; ++e)
                whole = larger(whole, magnitude(v[i][e]));
        whole = wave_reduce<true>(whole);
        if ((threadIdx.x & (kWave - 1)) == 0)
            shared_largest[threadIdx.x / kWave] = whole;
        __syncthreads();
        whole = larger(larger(shared_largest[0], shared_largest[1]), larger(shared_largest[2], shared_largest[3]));
    }
    const BlockScale tile_scale(whole);
    const int64_t depth = (int64_t)tiles_c * kB;                 // of a row of q
    const int64_t t_depth = up_block(rows), tiles_r = t_depth / kB;
    if constexpr (TILES) {
        if (threadIdx.x == 0) {
            if constexpr (ROWS)
                scales[tile] = tile_scale.scale;
            if constexpr (COLUMNS)
                t_scales[tc * tiles_r + tr] = tile_scale.scale;
        }
    }
    if constexpr (ROWS) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            uint32_t m = 0;
            if constexpr (!TILES) {
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    m = larger(m, magnitude(v[i][e]));
                m = largest16(m);
            }
            const BlockScale s = TILES ? tile_scale : BlockScale(m);
            if (r0 + i < rows) {
                *reinterpret_cast<uint2 *>(q + (r0 + i) * depth + c) = quantize8(v[i], s);
                if (!TILES && lane == 0)
                    scales[(int64_t)tc * rows + r0 + i] = s.scale;
            }
        }
    }
    if constexpr (COLUMNS) {
        if constexpr (!TILES) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                uint32_t m = 0;
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    m = larger(m, magnitude(v[i][e]));
                shared_largest[group * kB + lane * 8 + e] = m;
            }
            __syncthreads();
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            float column[8];
#pragma unroll
            for (int i = 0; i < 8; ++i)
                column[i] = v[i][e];
            uint32_t m = whole;
            if constexpr (!TILES)
#pragma unroll
                for (int g = 0; g < 16; ++g)
                    m = larger(m, shared_largest[g * kB + lane * 8 + e]);
            const BlockScale s = TILES ? tile_scale : BlockScale(m);
            *reinterpret_cast<uint2 *>(turned + (lane * 8 + e) * kPitch + group * 8) = quantize8(column, s);
            if (!TILES && group == 0 && c + e < cols)
                t_scales[(int64_t)tr * cols + c + e] = s.scale;
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int piece = i * 256 + threadIdx.x;
            const int column = piece / 8, at = piece % 8 * 16;
            if (tc * kB + column < cols)
                *reinterpret_cast<Words *>(qt + (int64_t)(tc * kB + column) * t_depth + (int64_t)tr * kB + at) =
                    *reinterpret_cast<const Words *>(turned + column * kPitch + at);
        }
    }
}

template <typename T, bool TILES>
hipError_t launch(const QuantizeArgs &a, hipStream_t stream)
{
    const int tiles_c = (int)(up_block(a.cols) / kB);
    const unsigned tiles = (unsigned)(up_block(a.rows) / kB * tiles_c);
    const T *x = static_cast<const T *>(a.x);
    const auto go = [&](auto kernel) {
        kernel<<<tiles, 256, 0, stream>>>(x, a.ld_x, a.rows, a.cols, tiles_c, a.q, a.scales, a.qt, a.t_scales);
    };
    if (a.q && a.qt)
        go(quantize_kernel<T, TILES, true, true>);
    else if (a.q)
        go(quantize_kernel<T, TILES, true, false>);
    else
        go(quantize_kernel<T, TILES, false, true>);
    return last_launch();
}

}  // namespace

hipError_t launch_quantize_f8(const QuantizeArgs &a, hipStream_t stream)
{
    if (a.dtype == 1)
        return a.tiles ? launch<uint16_t, true>(a, stream) : launch<uint16_t, false>(a, stream);
    return a.tiles ? launch<float, true>(a, stream) : launch<float, false>(a, stream);
}

}  // namespace dv
