// Quantization to e4m3 with a scale for every 128 columns of a row, or for every
// 128 x 128: of a matrix as it lies, transposed, or both in one read.
//
//     scale = max(largest magnitude of the block, 2^-100) / 448
//     q     = e4m3(x / scale)          to nearest of the quotient in fp32
//
// One block of 256 threads takes a 128 x 128 tile: 16 lanes cover a row with 8
// columns each, a thread holds 8 rows of them in registers.  A row's largest value
// is that of 16 lanes, a column's that of a thread's 8 rows, then of 16 threads through LDS.
// A scale and its reciprocal (two divisions) are worked out once, by one lane of the 16 or one
// thread of the block, and read by the others.  The transposed tile goes through LDS, 8
// bytes (8 rows of a column) a thread and column, and leaves in whole lines.
//
// Memory-bound: 8,192 x 32,000 bf16 by rows 151 us (5.2 TB/s), transposed 177, both 241 (4.35 TB/s,
// the quotients of both hold three waves a SIMD); by tiles both 222.
#include <type_traits>

#include "dv_logits.h"

namespace dv {
namespace {

constexpr int kB = kScaleBlock;

// The value of lane K of each 16.
template <int K>
__device__ __forceinline__ uint32_t lane_of_16(uint32_t v)
{
    return dpp_move<0x150 + K>(v);  // row_newbcast
}

// The scales of a thread's 8 rows, by their largest magnitudes (the same in all 16 lanes): lane k
// works out row k mod 8's, and returns it.
__device__ __forceinline__ float row_scales(BlockScale (&s)[8], const uint32_t (&m)[8], int lane)
{
    uint32_t mine = m[0];
#pragma unroll
    for (int i = 1; i < 8; ++i)
        mine = (lane & 7) == i ? m[i] : mine;
    const BlockScale b(mine);
    const auto take = [&](auto k) {
        constexpr int K = decltype(k)::value;
        s[K] = BlockScale(__uint_as_float(lane_of_16<K>(__float_as_uint(b.scale))),
                          __uint_as_float(lane_of_16<K>(__float_as_uint(b.inv))));
    };
    take(std::integral_constant<int, 0>{}), take(std::integral_constant<int, 1>{});
    take(std::integral_constant<int, 2>{}), take(std::integral_constant<int, 3>{});
    take(std::integral_constant<int, 4>{}), take(std::integral_constant<int, 5>{});
    take(std::integral_constant<int, 6>{}), take(std::integral_constant<int, 7>{});
    return b.scale;
}

template <typename T, bool TILES, bool ROWS, bool COLUMNS>
__global__ __launch_bounds__(256) void quantize_kernel(const T *x, int64_t ld, int rows, int cols, int tiles_c,
                                                        uint8_t *q, float *scales, uint8_t *qt, float *t_scales)
{
    // A column's 16-byte piece p (16 rows) stands at place p ^ (column / 8 mod 8): what is
    // written at once, 16 columns 8 apart, meets distinct banks.
    __shared__ __attribute__((aligned(16))) uint8_t turned[COLUMNS ? kB * kB : 16];
    __shared__ __attribute__((aligned(16))) uint32_t shared_largest[COLUMNS && !TILES ? 16 * kB : 4];
    __shared__ __attribute__((aligned(16))) float column_scale[COLUMNS && !TILES ? 2 : 1][kB];
    const int64_t tile = blockIdx.x;
    const int tr = (int)(tile / tiles_c), tc = (int)(tile % tiles_c);
    const int lane = threadIdx.x & 15, group = threadIdx.x >> 4;
    const int c = tc * kB + lane * 8;          // this thread's 8 columns
    const int r0 = tr * kB + group * 8;        // and its 8 rows
    Raw8<T> raw[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        if (r0 + i < rows)
            raw[i].load(x + (int64_t)(r0 + i) * ld, c, cols);
        else
            raw[i].zero();
    }
    float v[8][8];
#pragma unroll
    for (int i = 0; i < 8; ++i)
        raw[i].to(v[i]);
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
    if constexpr (COLUMNS && !TILES) {
        uint4 m[2] = {};
        uint32_t *const largest = reinterpret_cast<uint32_t *>(m);
#pragma unroll
        for (int e = 0; e < 8; ++e)
#pragma unroll
            for (int i = 0; i < 8; ++i)
                largest[e] = larger(largest[e], magnitude(v[i][e]));
        uint4 *const to = reinterpret_cast<uint4 *>(shared_largest + group * kB + lane * 8);
        to[0] = m[0];
        to[1] = m[1];
        __syncthreads();
        if (threadIdx.x < kB) {
            uint32_t k = 0;
#pragma unroll
            for (int g = 0; g < 16; ++g)
                k = larger(k, shared_largest[g * kB + threadIdx.x]);
            const BlockScale s(k);
            column_scale[0][threadIdx.x] = s.scale;
            column_scale[1][threadIdx.x] = s.inv;
            if (tc * kB + (int)threadIdx.x < cols)
                t_scales[(int64_t)tr * cols + tc * kB + threadIdx.x] = s.scale;
        }
    }
    if constexpr (ROWS) {
        BlockScale s[8];
        if constexpr (TILES) {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                s[i] = tile_scale;
        } else {
            uint32_t m[8] = {};
#pragma unroll
            for (int i = 0; i < 8; ++i) {
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    m[i] = larger(m[i], magnitude(v[i][e]));
                m[i] = largest16(m[i]);
            }
            const float mine = row_scales(s, m, lane);
            if (lane < 8 && r0 + lane < rows)
                scales[(int64_t)tc * rows + r0 + lane] = mine;
        }
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (r0 + i < rows)
                *reinterpret_cast<uint2 *>(q + (r0 + i) * depth + c) = quantize8(v[i], s[i]);
    }
    if constexpr (COLUMNS) {
        if constexpr (!TILES)
            __syncthreads();
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            float column[8];
#pragma unroll
            for (int i = 0; i < 8; ++i)
                column[i] = v[i][e];
            const BlockScale s = TILES ? tile_scale : BlockScale(column_scale[0][lane * 8 + e], column_scale[COLUMNS && !TILES][lane * 8 + e]);
            *reinterpret_cast<uint2 *>(turned + (lane * 8 + e) * kB + (((group >> 1) ^ (lane & 7)) * 16) + (group & 1) * 8) =
                quantize8(column, s);
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int piece = i * 256 + threadIdx.x;
            const int column = piece / 8, at = piece % 8;
            if (tc * kB + column < cols)
                *reinterpret_cast<Words *>(qt + (int64_t)(tc * kB + column) * t_depth + (int64_t)tr * kB + at * 16) =
                    *reinterpret_cast<const Words *>(turned + column * kB + ((at ^ (column >> 3 & 7)) * 16));
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
