// Root-mean-square norm with the residual's addition, and its gradients.
//
//     h = x + residual, rounded to the inputs' type (what the next layer adds to)
//     r = 1 / sqrt(mean of h^2 + eps),   y = h r w
//     u = h r,   dh = r (g w - u / D  sum of (g w u)) + dtotal,   dw = sum over rows of g u
//
// y leaves in the inputs' type, or in e4m3 with a scale for every 128 columns, which is
// how the 8-bit head product reads it.
//
// Memory-bound: each row is read once and held in registers, 8 columns a lane and
// vector, by one wave (up to 1,024 columns) or one block; a row's loads are all asked for before the first
// is needed.  Gradients of more than 16,384 columns have no registers for that: rows are read twice for dh and a
// third time for dw (512 x 65,536 bf16 65 us).  8,192 x 4,096 bf16 with a residual 43 us (6.3 TB/s), its gradients 46 (5.8
// TB/s) and 6 to join the weight's; 2,304 x 4,096 to e4m3 13 us; 1 x 1,024 2.7.
#include "dv_logits.h"

namespace dv {
namespace {

// Sum over the threads of a row: a wave, or a block through LDS.  `sums` is free again
// for what comes after the block's next barrier.
template <int THREADS>
__device__ __forceinline__ float row_sum(float v, float *sums)
{
    v = wave_sum(v);
    if constexpr (THREADS > kWave) {
        constexpr int kWaves = THREADS / kWave;
        if ((threadIdx.x & (kWave - 1)) == 0)
            sums[threadIdx.x / kWave] = v;
        __syncthreads();
        v = 0.f;
#pragma unroll
        for (int i = 0; i < kWaves; ++i)
            v += sums[i];
    }
    return v;
}

// The bits of the largest magnitude over the threads of a row, likewise.
template <int THREADS>
__device__ __forceinline__ uint32_t row_largest(uint32_t v, float *sums)
{
    v = wave_reduce<true>(v);
    if constexpr (THREADS > kWave) {
        if ((threadIdx.x & (kWave - 1)) == 0)
            sums[threadIdx.x / kWave] = __uint_as_float(v);
        __syncthreads();
#pragma unroll
        for (int i = 0; i < THREADS / kWave; ++i)
            v = larger(v, __float_as_uint(sums[i]));
    }
    return v;
}

// THREADS take a row, NV vectors of 8 columns each; blocks hold a row, or four of a wave each.
template <typename T, int THREADS, int NV>
__global__ __launch_bounds__(THREADS == kWave ? 256 : THREADS) void norm_kernel(const T *x, int64_t ld_x, const T *residual,
                                                                             int64_t ld_residual, const T *weight,
                                                                             int rows, int hidden, float eps, T *total,
                                                                             T *out, float *rstd, uint8_t *q, float *scales)
{
    constexpr int kRows = THREADS == kWave ? 256 / THREADS : 1;  // of a block
    __shared__ float sums[3][kRows == 1 ? THREADS / kWave : 1];
    const int t = threadIdx.x % THREADS;
    const int64_t row = (int64_t)blockIdx.x * kRows + threadIdx.x / THREADS;
    if (kRows > 1 && row >= rows)  // whole waves
        return;
    // all of a row's vectors at once, but for the longest rows, whose registers hold one after the other
    constexpr int kAtOnce = NV <= 4 ? NV : 1;
    Raw8<T> raw[kAtOnce], raw_residual[kAtOnce], raw_weight[kAtOnce];
    const auto load = [&](int v) {
        const int c = (v * THREADS + t) * 8;
        raw[v % kAtOnce].load(x + row * ld_x, c, hidden);
        if (residual)
            raw_residual[v % kAtOnce].load(residual + row * ld_residual, c, hidden);
    };
    const auto load_weight = [&](int v) { raw_weight[v % kAtOnce].load(weight, (v * THREADS + t) * 8, hidden); };
    if constexpr (kAtOnce == NV) {
#pragma unroll
        for (int v = 0; v < NV; ++v)
            load(v);
#pragma unroll
        for (int v = 0; v < NV; ++v)
            load_weight(v);
    }
    float h[NV][8];
    float sum = 0.f;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        const int c = (v * THREADS + t) * 8;
        if constexpr (kAtOnce != NV)
            load(v);
        raw[v % kAtOnce].to(h[v]);
        if (residual) {
            float y[8];
            raw_residual[v % kAtOnce].to(y);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                h[v][e] += y[e];
                if constexpr (sizeof(T) == 2)
                    h[v][e] = widen(narrow(h[v][e]));
            }
        }
        if (total)
            store8(total + row * hidden, c, hidden, h[v]);
#pragma unroll
        for (int e = 0; e < 8; ++e)
            sum = __builtin_fmaf(h[v][e], h[v][e], sum);
    }
    sum = row_sum<THREADS>(sum, sums[0]);
    float mean = sum / (float)hidden + eps, unit = 1.f;
    if (!(mean >= 0x1p-90f && sum <= 0x1p120f)) {
        // squares out of range: the same of h times a power of two, if the row is finite
        uint32_t m = 0;
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
            for (int e = 0; e < 8; ++e)
                m = larger(m, magnitude(h[v][e]));
        m = row_largest<THREADS>(m, sums[1]);
        if (m && m < 0x7F800000u) {
            const int up = 127 - (int)(m >> 23);
            unit = __builtin_ldexpf(1.f, up < 100 ? up : 100);
            sum = 0.f;
#pragma unroll
            for (int v = 0; v < NV; ++v)
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    h[v][e] *= unit;
                    sum = __builtin_fmaf(h[v][e], h[v][e], sum);
                }
            sum = row_sum<THREADS>(sum, sums[2]);
            mean = sum / (float)hidden + eps * unit * unit;
        }
    }
    const float r = 1.f / sqrtf(mean);
    if (rstd && t == 0)
        rstd[row] = r * unit;
    const int64_t depth = up_block(hidden);
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        const int c = (v * THREADS + t) * 8;
        float w[8];
        if constexpr (kAtOnce != NV)
            load_weight(v);
        raw_weight[v % kAtOnce].to(w);
#pragma unroll
        for (int e = 0; e < 8; ++e)
            h[v][e] = h[v][e] * r * w[e];
        if (out)
            store8(out + row * hidden, c, hidden, h[v]);
        if (q) {  // 16 lanes hold a block; lanes past the depth take part with zeros
            uint32_t m = 0;
#pragma unroll
            for (int e = 0; e < 8; ++e)
                m = larger(m, magnitude(h[v][e]));
            const BlockScale s(largest16(m));
            if (c < depth) {
                *reinterpret_cast<uint2 *>(q + row * depth + c) = quantize8(h[v], s);
                if ((t & 15) == 0)
                    scales[(int64_t)(c / kScaleBlock) * rows + row] = s.scale;
            }
        }
    }
}

template <typename T>
__device__ __forceinline__ void read8(float (&x)[8], const T *row, int c, int n)
{
    Raw8<T> raw;
    raw.load(row, c, n);
    raw.to(x);
}

// Blocks take every gridDim.x-th row.  HELD: a row's h and g stay in registers and the block's
// share of dw goes to `partial` [gridDim.x][hidden]; else (the longest rows, whose share of dw has no
// registers left either: norm_weight_part_kernel) they are read again.
template <typename T, int THREADS, int NV, bool HELD>
__global__ __launch_bounds__(THREADS) void norm_grad_kernel(const T *grad_out, int64_t ld_g, const T *total, int64_t ld_h,
                                                            const T *weight, const float *rstd, const T *grad_total,
                                                            int64_t ld_gt, int rows, int hidden, T *grad_x, float *partial)
{
    constexpr int kHeld = HELD ? NV : 1;
    __shared__ float sums[2][THREADS / kWave];
    float dw[kHeld][8];
#pragma unroll
    for (int v = 0; v < kHeld; ++v)
#pragma unroll
        for (int e = 0; e < 8; ++e)
            dw[v][e] = 0.f;
    const auto column = [](int v) { return (v * THREADS + (int)threadIdx.x) * 8; };
    int half = 0;
    for (int64_t row = blockIdx.x; row < rows; row += gridDim.x) {
        const T *gr = grad_out + row * ld_g, *hr = total + row * ld_h;
        const T *const dr = grad_total ? grad_total + row * ld_gt : nullptr;
        const float r = rstd[row];
        Raw8<T> raw_h[kHeld], raw_g[kHeld], raw_d[kHeld];
        float h[kHeld][8], g[kHeld][8];
        // h r and g w of vector v
        const auto take = [&](int v, int at) {
            float w[8];
            read8(w, weight, column(v), hidden);
            raw_h[at].to(h[at]);
            raw_g[at].to(g[at]);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                h[at][e] *= r;
                if constexpr (HELD)
                    dw[at][e] = __builtin_fmaf(g[at][e], h[at][e], dw[at][e]);
                g[at][e] *= w[e];
            }
        };
        const auto finish = [&](int v, int at, float k) {
            float d[8];
            if (dr) {
                raw_d[at].to(d);
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    d[e] = 0.f;
            }
#pragma unroll
            for (int e = 0; e < 8; ++e)
                d[e] = __builtin_fmaf(r, g[at][e] - h[at][e] * k, d[e]);
            store8(grad_x + row * hidden, column(v), hidden, d);
        };
        float sum = 0.f;
        if constexpr (HELD) {
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                raw_h[v].load(hr, column(v), hidden);
                raw_g[v].load(gr, column(v), hidden);
            }
            if (dr && grad_x)
#pragma unroll
                for (int v = 0; v < NV; ++v)
                    raw_d[v].load(dr, column(v), hidden);
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                take(v, v);
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    sum = __builtin_fmaf(g[v][e], h[v][e], sum);
            }
        } else {
#pragma unroll 1
            for (int v = 0; v < NV; ++v) {
                raw_h[0].load(hr, column(v), hidden);
                raw_g[0].load(gr, column(v), hidden);
                take(v, 0);
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    sum = __builtin_fmaf(g[0][e], h[0][e], sum);
            }
        }
        if (!grad_x)
            continue;
        sum = row_sum<THREADS>(sum, sums[half]);
        half ^= 1;  // the next row's sums meet elsewhere: its barrier comes after everyone has read these
        const float k = sum / (float)hidden;
        if constexpr (HELD) {
#pragma unroll
            for (int v = 0; v < NV; ++v)
                finish(v, v, k);
        } else {
#pragma unroll 1
            for (int v = 0; v < NV; ++v) {
                raw_h[0].load(hr, column(v), hidden);
                raw_g[0].load(gr, column(v), hidden);
                if (dr)
                    raw_d[0].load(dr, column(v), hidden);
                take(v, 0);
                finish(v, 0, k);
            }
        }
    }
    if constexpr (HELD)
        if (partial)
#pragma unroll
            for (int v = 0; v < NV; ++v)
                store8(partial + (int64_t)blockIdx.x * hidden, column(v), hidden, dw[v]);
}

// The shares of dw of the longest rows: a block takes 2,048 columns of every gridDim.y-th row, four of
// them at a time, and leaves its share as norm_grad_kernel's blocks do.
template <typename T>
__global__ __launch_bounds__(256) void norm_weight_part_kernel(const T *grad_out, int64_t ld_g, const T *total, int64_t ld_h,
                                                               const float *rstd, int rows, int hidden, float *partial)
{
    constexpr int kAtOnce = 4;
    const int c = (blockIdx.x * 256 + (int)threadIdx.x) * 8;
    float dw[8] = {};
    for (int64_t from = blockIdx.y; from < rows; from += (int64_t)gridDim.y * kAtOnce) {
        Raw8<T> raw_h[kAtOnce], raw_g[kAtOnce];
        float r[kAtOnce];
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k) {
            const int64_t row = from + (int64_t)k * gridDim.y;
            r[k] = 0.f;
            raw_h[k].zero();
            raw_g[k].zero();
            if (row < rows) {
                raw_h[k].load(total + row * ld_h, c, hidden);
                raw_g[k].load(grad_out + row * ld_g, c, hidden);
                r[k] = rstd[row];
            }
        }
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k) {
            float h[8], g[8];
            raw_h[k].to(h);
            raw_g[k].to(g);
#pragma unroll
            for (int e = 0; e < 8; ++e)
                dw[e] = __builtin_fmaf(g[e], h[e] * r[k], dw[e]);
        }
    }
    store8(partial + (int64_t)blockIdx.y * hidden, c, hidden, dw);
}

// dw: the blocks' shares added.  A block takes 64 columns, 16 lanes a share with 4 of them each
// (the columns past the end are not there: 16 bytes are read where they lie in the row), its 64
// groups every 64th share, 8 of them asked for at a time; then the groups' sums, through LDS.
template <typename T>
__global__ __launch_bounds__(1024) void norm_weight_kernel(const float *partial, int parts, int hidden, T *grad_weight)
{
    constexpr int kGroups = 64, kColumns = 64, kAtOnce = 8;
    __shared__ float sh[kGroups][kColumns];
    const int lane = threadIdx.x % 16, group = threadIdx.x / 16;
    const int c = blockIdx.x * kColumns + lane * 4;
    const int left = hidden - c;
    float s[4] = {0.f, 0.f, 0.f, 0.f};
    for (int from = group; from < parts; from += kGroups * kAtOnce) {
        float x[kAtOnce][4];
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k) {
            const int p = from + k * kGroups;
            const float *row = partial + (int64_t)p * hidden + c;
            if (p < parts && left >= 4) {
                const Words w = load_words(row);
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    x[k][e] = __uint_as_float(w[e]);
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    x[k][e] = p < parts && e < left ? row[e] : 0.f;
            }
        }
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k)
#pragma unroll
            for (int e = 0; e < 4; ++e)
                s[e] += x[k][e];
    }
#pragma unroll
    for (int e = 0; e < 4; ++e)
        sh[group][lane * 4 + e] = s[e];
    __syncthreads();
    // 16 threads a column, 4 groups each, of one wave's quarter
    const int column = threadIdx.x / 16, part = threadIdx.x % 16;
    float sum = 0.f;
#pragma unroll
    for (int k = 0; k < kGroups / 16; ++k)
        sum += sh[part * (kGroups / 16) + k][column];
#pragma unroll
    for (int d = 8; d; d >>= 1)
        sum += __shfl_xor(sum, d);
    const int at = blockIdx.x * kColumns + column;
    if (part == 0 && at < hidden) {
        if constexpr (sizeof(T) == 2)
            grad_weight[at] = narrow(sum);
        else
            grad_weight[at] = sum;
    }
}

template <typename T>
hipError_t launch_norm(const NormArgs &a, hipStream_t stream)
{
    const auto go = [&](auto kernel, int threads) {
        const int per_block = threads == kWave ? 256 / threads : 1;
        const unsigned grid = (unsigned)((a.rows + per_block - 1) / per_block);
        kernel<<<grid, threads == kWave ? 256 : threads, 0, stream>>>(
            static_cast<const T *>(a.x), a.ld_x, static_cast<const T *>(a.residual), a.ld_residual,
            static_cast<const T *>(a.weight), a.rows, a.hidden, a.eps, static_cast<T *>(a.total), static_cast<T *>(a.out),
            a.rstd, a.q, a.scales);
    };
    const int64_t depth = up_block(a.hidden);
    if (depth <= 512)
        go(norm_kernel<T, 64, 1>, 64);
    else if (depth <= 1024)
        go(norm_kernel<T, 64, 2>, 64);
    else if (depth <= 2048)
        go(norm_kernel<T, 256, 1>, 256);
    else if (depth <= 4096)
        go(norm_kernel<T, 256, 2>, 256);
    else if (depth <= 8192)
        go(norm_kernel<T, 256, 4>, 256);
    else if (depth <= 16384)
        go(norm_kernel<T, 1024, 2>, 1024);
    else if (depth <= 32768)
        go(norm_kernel<T, 1024, 4>, 1024);
    else
        go(norm_kernel<T, 1024, 8>, 1024);
    return last_launch();
}

// Blocks of the backward pass: each leaves a share of dw, so no more than fill the card.
int grad_blocks(int rows, int hidden)
{
    const int most = hidden <= 8192 ? 1024 : 256;
    return rows < most ? rows : most;
}

template <typename T>
hipError_t launch_grad(const NormGradArgs &a, float *partial, hipStream_t stream)
{
    const int blocks = grad_blocks(a.rows, a.hidden);
    const auto go = [&](auto kernel, int threads) {
        kernel<<<(unsigned)blocks, threads, 0, stream>>>(
            static_cast<const T *>(a.grad_out), a.ld_grad_out, static_cast<const T *>(a.total), a.ld_total,
            static_cast<const T *>(a.weight), a.rstd, static_cast<const T *>(a.grad_total), a.ld_grad_total, a.rows,
            a.hidden, static_cast<T *>(a.grad_x), a.grad_weight ? partial : nullptr);
    };
    if (a.rows > 0) {
        if (a.hidden <= 512)
            go(norm_grad_kernel<T, 64, 1, true>, 64);
        else if (a.hidden <= 1024)
            go(norm_grad_kernel<T, 128, 1, true>, 128);
        else if (a.hidden <= 2048)
            go(norm_grad_kernel<T, 256, 1, true>, 256);
        else if (a.hidden <= 4096)
            go(norm_grad_kernel<T, 256, 2, true>, 256);
        else if (a.hidden <= 8192)
            go(norm_grad_kernel<T, 512, 2, true>, 512);
        else if (a.hidden <= 16384)
            go(norm_grad_kernel<T, 1024, 2, true>, 1024);
        else {
            if (a.grad_x)
                a.hidden <= 32768 ? go(norm_grad_kernel<T, 1024, 4, false>, 1024) : go(norm_grad_kernel<T, 1024, 8, false>, 1024);
            if (a.grad_weight)
                norm_weight_part_kernel<T><<<dim3((unsigned)((a.hidden + 2047) / 2048), (unsigned)blocks), 256, 0, stream>>>(
                    static_cast<const T *>(a.grad_out), a.ld_grad_out, static_cast<const T *>(a.total), a.ld_total, a.rstd,
                    a.rows, a.hidden, partial);
        }
    }
    if (a.grad_weight)
        norm_weight_kernel<T><<<(unsigned)((a.hidden + 63) / 64), 1024, 0, stream>>>(
            partial, blocks, a.hidden, static_cast<T *>(a.grad_weight));
    return last_launch();
}

}  // namespace

hipError_t launch_rms_norm(const NormArgs &a, hipStream_t stream)
{
    return a.dtype == 1 ? launch_norm<uint16_t>(a, stream) : launch_norm<float>(a, stream);
}

size_t rms_norm_backward_workspace_bytes(int rows, int hidden)
{
    const int blocks = grad_blocks(rows, hidden);
    return align_up((size_t)(blocks > 0 ? blocks : 1) * (size_t)hidden * 4, 256);
}

hipError_t launch_rms_norm_backward(const NormGradArgs &a, void *workspace, hipStream_t stream)
{
    float *partial = static_cast<float *>(workspace);
    return a.dtype == 1 ? launch_grad<uint16_t>(a, partial, stream) : launch_grad<float>(a, partial, stream);
}

}  // namespace dv
