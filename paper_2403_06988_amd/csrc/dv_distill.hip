// Distillation from a teacher's top logits over the allowed tokens.
//
// Per row, with the allowed tokens A of the row's state, c = 1/T, and the
// listed teacher entries L = {k : id_k in A, top_k > -inf}:
//     q_k = exp(c (top_k - max)) / sum over L,   p_v = exp(c (z_v - m)) / s,
//     loss = sum_L q_k (ln q_k - ln p_{id_k}),
//     dloss/dz_v = c (p_v - sum of q_k with id_k = v)   on A, 0 elsewhere.
//
// The loss needs one read of the row, loss and gradient one read and one
// write of it: both are bound by memory.  The gradient kernel keeps the row in no
// wider place than the caches between its two passes: a row is 0.25 to 1 MB.
#include <type_traits>

#include "dv_train.h"

namespace dv {
namespace {

constexpr int kThreads = 512;
constexpr int kWaves = kThreads / kWave;
constexpr int kMaxTop = 1024;

// Vectors of 16 bytes at any element's alignment.  The gradient's are stored
// past the caches: what a row's second pass is to find there is its logits (2,048 x
// 128,256 bf16: 264 us, with ordinary stores 307).
template <typename T>
struct Vec;
template <>
struct Vec<float> {
    static constexpr int kN = 4;
    float x[4];
    static __device__ __forceinline__ Vec load(const float *p)
    {
        Vec v;
        __builtin_memcpy(v.x, p, 16);
        return v;
    }
    __device__ __forceinline__ float get(int i) const { return x[i]; }
    // elements whose bit is clear become -infinity
    __device__ __forceinline__ void keep(uint32_t bits)
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t m = (uint32_t)((int32_t)(bits << (31 - i)) >> 31);
            x[i] = __uint_as_float((__float_as_uint(x[i]) & m) | (0xFF800000u & ~m));
        }
    }
    static __device__ __forceinline__ void store(float *p, const float (&y)[4])
    {
        typedef __attribute__((ext_vector_type(4), aligned(4))) float Four;
        __builtin_nontemporal_store(Four{y[0], y[1], y[2], y[3]}, reinterpret_cast<Four *>(p));
    }
    static __device__ __forceinline__ float one(const float *p) { return *p; }
    static __device__ __forceinline__ void put(float *p, float y) { *p = y; }
};
template <>
struct Vec<uint16_t> {
    static constexpr int kN = 8;
    uint32_t x[4];
    static __device__ __forceinline__ Vec load(const uint16_t *p)
    {
        Vec v;
        __builtin_memcpy(v.x, p, 16);
        return v;
    }
    __device__ __forceinline__ float get(int i) const
    {
        return __uint_as_float(i & 1 ? x[i >> 1] & 0xFFFF0000u : x[i >> 1] << 16);
    }
    __device__ __forceinline__ void keep(uint32_t bits)
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t lo = (uint32_t)((int32_t)(bits << (31 - 2 * i)) >> 31);
            const uint32_t hi = (uint32_t)((int32_t)(bits << (30 - 2 * i)) >> 31);
            const uint32_t m = (lo & 0xFFFFu) | (hi & 0xFFFF0000u);
            x[i] = (x[i] & m) | (0xFF80FF80u & ~m);
        }
    }
    static __device__ __forceinline__ void store(uint16_t *p, const float (&y)[8])
    {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i)
            w[i] = narrow_pair(y[2 * i], y[2 * i + 1]);
        typedef __attribute__((ext_vector_type(4), aligned(2))) uint32_t Four;
        __builtin_nontemporal_store(Four{w[0], w[1], w[2], w[3]}, reinterpret_cast<Four *>(p));
    }
    static __device__ __forceinline__ float one(const uint16_t *p) { return widen(*p); }
    static __device__ __forceinline__ void put(uint16_t *p, float y) { *p = narrow(y); }
};

struct Shared {
    float wave_a[kWaves], wave_b[kWaves];
    int id[kMaxTop];
    float q[kMaxTop];
    float z[kMaxTop];
};

// Over the block's waves, in every lane.
__device__ __forceinline__ float block_sum(float v, Shared &sh)
{
    v = wave_sum(v);
    __syncthreads();
    if ((threadIdx.x & (kWave - 1)) == 0)
        sh.wave_a[threadIdx.x / kWave] = v;
    __syncthreads();
    float t = 0.f;
#pragma unroll
    for (int i = 0; i < kWaves; ++i)
        t += sh.wave_a[i];
    return t;
}

__device__ __forceinline__ Softmax block_join(Softmax v, float c2, Shared &sh)
{
    const float top = wave_max(v.max);
    const float sum = wave_sum(v.max == -INFINITY ? v.sum : v.sum * softmax_term(v.max, top, c2));
    __syncthreads();
    if ((threadIdx.x & (kWave - 1)) == 0) {
        sh.wave_a[threadIdx.x / kWave] = top;
        sh.wave_b[threadIdx.x / kWave] = sum;
    }
    __syncthreads();
    Softmax t{-INFINITY, 0.f};
#pragma unroll
    for (int i = 0; i < kWaves; ++i)
        t.max = fmaxf(t.max, sh.wave_a[i]);
#pragma unroll
    for (int i = 0; i < kWaves; ++i)
        t.sum += sh.wave_a[i] == -INFINITY ? sh.wave_b[i] : sh.wave_b[i] * softmax_term(sh.wave_a[i], t.max, c2);
    return t;
}

// The teacher's entries of a row: ids (-1 where an entry takes no part) and
// probabilities in LDS; returns the maximum and the sum of exp(c (top - max)).
__device__ __forceinline__ Softmax teacher(const DistillArgs &a, const RowMask &m, int row, float c2, Shared &sh)
{
    Softmax own{-INFINITY, 0.f};
    for (int k = threadIdx.x; k < a.K; k += kThreads) {
        const int id = a.ids[(size_t)row * a.K + k];
        const float t = a.top[(size_t)row * a.K + k];
        const bool in = m.has(id) && t != -INFINITY;
        sh.id[k] = in ? id : -1;
        sh.q[k] = t;
        if (in)
            own = softmax_join(own, {t, 1.f}, c2);
    }
    const Softmax all = block_join(own, c2, sh);
    for (int k = threadIdx.x; k < a.K; k += kThreads)
        sh.q[k] = sh.id[k] < 0 ? 0.f : softmax_term(sh.q[k], all.max, c2) / all.sum;
    return all;
}

// Vectors [j0, j1) of a row, kBatch a lane at a time: f(vectors, first, whole) has
// vector first + u kThreads + lane in place u; masked elements read as -infinity, and
// so do vectors past j1 (only where `whole` is false).  A batch's start is in
// scalar registers, a lane's offset from it 32 bits.
constexpr int kBatch = 4;

template <typename T, bool MASK, bool WHOLE>
__device__ __forceinline__ void load_batch(Vec<T> (&v)[kBatch], const T *z, const RowMask &m, int first, int j1)
{
    constexpr int N = Vec<T>::kN;
    uint32_t bits[kBatch];
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
        const int at = first + u * kThreads;  // uniform
        const int left = j1 - at;
        const bool in = WHOLE || (int)threadIdx.x < left;
        const int base = WHOLE || left > 0 ? at : first;
        const uint32_t lane = in ? threadIdx.x : 0;
        v[u] = Vec<T>::load(reinterpret_cast<const T *>(reinterpret_cast<const char *>(z) + (size_t)base * 16 + lane * 16u));
        if (MASK) {
            const uint8_t *bytes = reinterpret_cast<const uint8_t *>(m.words) + base / (8 / N);
            bits[u] = N == 8 ? bytes[lane] : (uint32_t)bytes[lane >> 1] >> ((lane & 1) * 4);
            bits[u] = in ? bits[u] : 0u;
        } else {
            bits[u] = in ? 0xFFu : 0u;
        }
    }
#pragma unroll
    for (int u = 0; u < kBatch; ++u)
        if (MASK || (!WHOLE && !bits[u]))
            v[u].keep(bits[u]);
}

template <typename T, bool MASK, typename F>
__device__ __forceinline__ void for_batches(const T *z, const RowMask &m, int j0, int j1, F &&f)
{
    constexpr int kStep = kThreads * kBatch;
    Vec<T> v[kBatch];
    int first = j0;
    for (; first + kStep <= j1; first += kStep) {
        load_batch<T, MASK, true>(v, z, m, first, j1);
        f(v, first, std::true_type{});
    }
    if (first < j1) {
        load_batch<T, MASK, false>(v, z, m, first, j1);
        f(v, first, std::false_type{});
    }
}

// exp(c (x - max)) as exp2(x c2 - shift), shift = max c2 rounded: one operation and
// one rounding; `correction` is the factor 2^(shift - max c2) that the rounding of
// the shift leaves.  Only where max c2 is of ordinary size: else (a row of
// nothing but the type's lowest value, say) differences are scaled.
struct Shift {
    float max, c2, shift, correction;
    bool plain;
    __device__ __forceinline__ Shift(float max_, float c2_) : max(max_ == -INFINITY ? 0.f : max_), c2(c2_)
    {
        shift = max * c2;
        plain = fabsf(shift) < 1048576.f;
        correction = plain ? 1.f - __builtin_fmaf(max, c2, -shift) * 0.69314718f : 1.f;
    }
    template <bool PLAIN>
    __device__ __forceinline__ float term(float x) const
    {
        return exp2_fast(PLAIN ? __builtin_fmaf(x, c2, -shift) : (x - max) * c2);
    }
};

// The softmax state of tokens [from, to) of a row (from a multiple of 8).
template <typename T, bool MASK>
__device__ __forceinline__ Softmax row_stats(const T *z, const RowMask &m, int from, int to, float c2)
{
    using V = Vec<T>;
    constexpr int N = V::kN;
    Softmax own{-INFINITY, 0.f};
    for_batches<T, MASK>(z, m, from / N, to / N, [&](const V (&v)[kBatch], int, auto) {
        float top = own.max;
#pragma unroll
        for (int u = 0; u < kBatch; ++u)
#pragma unroll
            for (int i = 0; i < N; i += 2)
                top = fmaxf(fmaxf(top, v[u].get(i)), v[u].get(i + 1));
        const Shift t(top, c2);
        float sum = 0.f;
        if (__all(t.plain)) {
#pragma unroll
            for (int u = 0; u < kBatch; ++u)
#pragma unroll
                for (int i = 0; i < N; ++i)
                    sum += t.template term<true>(v[u].get(i));
            sum *= t.correction;
        } else {
#pragma unroll
            for (int u = 0; u < kBatch; ++u)
#pragma unroll
                for (int i = 0; i < N; ++i)
                    sum += t.template term<false>(v[u].get(i));
        }
        const float before = own.max == -INFINITY ? own.sum : own.sum * softmax_term(own.max, t.max, c2);
        own = {top, before + sum};
    });
    for (int i = to / N * N + threadIdx.x; i < to; i += kThreads)
        if (m.has(i)) {
            const float x = V::one(z + i);
            own = x == -INFINITY ? own : softmax_join(own, {x, 1.f}, c2);
        }
    return own;
}

// The row's part of the loss: needs sh.id, sh.q and sh.z.
__device__ __forceinline__ float row_loss(const DistillArgs &a, int row, Softmax t, Softmax s, Shared &sh)
{
    const float c = a.inv_temperature;
    const float lnt = logf(t.sum), lns = logf(s.sum);
    float sum = 0.f;
    for (int k = threadIdx.x; k < a.K; k += kThreads) {
        const float q = sh.q[k];
        if (!(q == 0.f))  // NaN counts
            sum += q * (((a.top[(size_t)row * a.K + k] - t.max) * c - lnt) - ((sh.z[k] - s.max) * c - lns));
    }
    return block_sum(sum, sh);
}

// The gradient of the listed tokens in [from, to), once the block's other stores
// there are done: an id listed more than once takes the sum of its entries, in
// their order, from each of them.
template <typename T>
__device__ __forceinline__ void listed_grad(T *grad, int from, int to, float c2, float max, float scale, float w, int K,
                                            Shared &sh)
{
    __syncthreads();
    for (int k = threadIdx.x; k < K; k += kThreads) {
        const int id = sh.id[k];
        if (id < from || id >= to)
            continue;
        float q = 0.f;
        for (int i = 0; i < K; ++i)
            q += sh.id[i] == id ? sh.q[i] : 0.f;
        Vec<T>::put(grad + id, softmax_term(sh.z[k], max, c2) * scale - w * q);
    }
}

// Writes the gradient of tokens [from, to): w (p - q).  `part` false: zeros.
template <typename T, bool MASK>
__device__ __forceinline__ void row_grad(const T *z, T *grad, const RowMask &m, int from, int to, float c2, Softmax s,
                                         float w, bool part, int K, Shared &sh)
{
    using V = Vec<T>;
    constexpr int N = V::kN;
    const int j0 = from / N, j1 = to / N;
    if (!part) {
        const float zeros[N] = {};
        for (int j = j0 + threadIdx.x; j < j1; j += kThreads)
            V::store(grad + (size_t)j * N, zeros);
        for (int i = j1 * N + threadIdx.x; i < to; i += kThreads)
            V::put(grad + i, 0.f);
        return;
    }
    const Shift t(s.max, c2);
    const float scale = w / s.sum;
    const auto write = [&](auto plain) {
        constexpr bool PLAIN = decltype(plain)::value;
        const float by = PLAIN ? scale * t.correction : scale;
        for_batches<T, MASK>(z, m, j0, j1, [&](const V (&v)[kBatch], int first, auto whole) {
#pragma unroll
            for (int u = 0; u < kBatch; ++u) {
                float y[N];
#pragma unroll
                for (int i = 0; i < N; ++i)
                    y[i] = t.template term<PLAIN>(v[u].get(i)) * by;
                const int at = first + u * kThreads;
                if (decltype(whole)::value || at + (int)threadIdx.x < j1)
                    V::store(reinterpret_cast<T *>(reinterpret_cast<char *>(grad) + (size_t)at * 16 + threadIdx.x * 16u), y);
            }
        });
    };
    if (t.plain)
        write(std::true_type{});
    else
        write(std::false_type{});
    for (int i = j1 * N + threadIdx.x; i < to; i += kThreads)
        V::put(grad + i, m.has(i) ? softmax_term(V::one(z + i), s.max, c2) * scale : 0.f);
    listed_grad(grad, from, to, c2, s.max, scale, w, K, sh);
}

// One block per row: the row's softmax, the loss, and with GRAD the gradient
// from a second pass over the row, which its first pass left in the caches.
template <typename T, bool MASK, bool GRAD>
__global__ __launch_bounds__(kThreads) void distill_row_kernel(DistillArgs a, const float *grad_loss, float *loss,
                                                                T *grad, int64_t ld_grad)
{
    __shared__ Shared sh;
    const int row = blockIdx.x;
    const float c2 = a.inv_temperature * kLog2e;
    const RowMask m(a.masks, a.V, row);
    const T *z = static_cast<const T *>(a.logits) + (size_t)row * a.ld;
    const Softmax t = teacher(a, m, row, c2, sh);
    for (int k = threadIdx.x; k < a.K; k += kThreads)
        sh.z[k] = sh.id[k] < 0 ? 0.f : Vec<T>::one(z + sh.id[k]);
    Softmax s{-INFINITY, 0.f};
    bool part = !m.dead && !t.empty();
    if (part)
        s = block_join(row_stats<T, MASK>(z, m, 0, a.V, c2), c2, sh);
    part = part && !s.empty();
    if (loss) {
        const float l = part ? row_loss(a, row, t, s, sh) : 0.f;
        if (threadIdx.x == 0)
            loss[row] = l;
    }
    if (GRAD)
        row_grad<T, MASK>(z, grad + (size_t)row * ld_grad, m, 0, a.V, c2, s, part ? grad_loss[row] * a.inv_temperature : 0.f,
                 part, a.K, sh);
}

// Rows split over blocks (few rows): the chunks' softmax states, and the
// logits of the listed tokens (the gradient may overwrite the logits) ...
template <typename T, bool MASK>
__global__ __launch_bounds__(kThreads) void distill_stats_kernel(DistillArgs a, int chunk, Softmax *part, float *listed)
{
    __shared__ Shared sh;
    const int row = blockIdx.y, c = blockIdx.x;
    const float c2 = a.inv_temperature * kLog2e;
    const RowMask m(a.masks, a.V, row);
    const T *z = static_cast<const T *>(a.logits) + (size_t)row * a.ld;
    const int from = c * chunk, to = a.V - from < chunk ? a.V : from + chunk;
    if (c == 0)
        for (int k = threadIdx.x; k < a.K; k += kThreads) {
            const int id = a.ids[(size_t)row * a.K + k];
            listed[(size_t)row * a.K + k] = m.has(id) ? Vec<T>::one(z + id) : 0.f;
        }
    Softmax s{-INFINITY, 0.f};
    if (!m.dead)
        s = block_join(row_stats<T, MASK>(z, m, from, to, c2), c2, sh);
    if (threadIdx.x == 0)
        part[(size_t)row * gridDim.x + c] = s;
}

// ... and then the loss (chunk 0's block) and each chunk's gradient.
template <typename T, bool MASK, bool GRAD>
__global__ __launch_bounds__(kThreads) void distill_finish_kernel(DistillArgs a, int chunk, int chunks,
                                                                   const Softmax *parts, const float *listed,
                                                                   const float *grad_loss, float *loss, T *grad,
                                                                   int64_t ld_grad)
{
    __shared__ Shared sh;
    const int row = blockIdx.y, c = blockIdx.x;
    const float c2 = a.inv_temperature * kLog2e;
    const RowMask m(a.masks, a.V, row);
    const Softmax t = teacher(a, m, row, c2, sh);
    for (int k = threadIdx.x; k < a.K; k += kThreads)
        sh.z[k] = listed[(size_t)row * a.K + k];
    Softmax s{-INFINITY, 0.f};
    for (int i = threadIdx.x; i < chunks; i += kThreads)
        s = softmax_join(s, parts[(size_t)row * chunks + i], c2);
    s = block_join(s, c2, sh);
    const bool part = !t.empty() && !s.empty();
    if (loss && c == 0) {
        const float l = part ? row_loss(a, row, t, s, sh) : 0.f;
        if (threadIdx.x == 0)
            loss[row] = l;
    }
    if (GRAD) {
        const int from = c * chunk, to = a.V - from < chunk ? a.V : from + chunk;
        const T *z = static_cast<const T *>(a.logits) + (size_t)row * a.ld;
        row_grad<T, MASK>(z, grad + (size_t)row * ld_grad, m, from, to, c2, s, part ? grad_loss[row] * a.inv_temperature : 0.f,
                 part, a.K, sh);
    }
}

struct Split {
    int chunk, chunks;  // tokens of a chunk (a multiple of 8), chunks of a row
};

// A row is one block's when rows are many or short: a split row costs a second
// launch and the chunks' meeting (us a call, whole rows and split ones, loss and
// gradient: 40 x 64,000 bf16 12.6 and 14.4, 40 x 128,256 18.5 and 14.3, 100 x 128,256
// 20.9 and 17.3, 200 x 128,256 29.1 and 31.1; the loss alone: 40 x 128,256 10.8 and
// 12.7, 8 x 256,000 16.7 and 12.5).  Else rows are split until the launch has two
// blocks a compute unit, each with at least one pass of its lanes' vectors.
constexpr int kSplitBlocks = 512;
constexpr int kWholeRows = 160;

Split split_of(int rows, int V, int dtype, bool grad)
{
    const int64_t row_bytes = (int64_t)V * (dtype == 1 ? 2 : 4);
    const int pass = kThreads * (dtype == 1 ? 8 : 4);
    int want = kSplitBlocks / (rows > 0 ? rows : 1);
    if (rows >= kWholeRows || row_bytes <= (grad ? 131072 : 262144))
        want = 1;
    const int most = V / pass > 1 ? V / pass : 1;
    want = want < most ? want : most;
    int chunk = (int)align_up((size_t)(V + want - 1) / want, 8);
    return {chunk, (V + chunk - 1) / chunk};
}

template <typename T, bool MASK>
hipError_t launch(const DistillArgs &a, const float *grad_loss, float *loss, T *grad, int64_t ld_grad, void *workspace,
                  hipStream_t stream)
{
    const Split s = split_of(a.rows, a.V, a.dtype, grad != nullptr);
    if (s.chunks == 1) {
        if (grad)
            distill_row_kernel<T, MASK, true><<<a.rows, kThreads, 0, stream>>>(a, grad_loss, loss, grad, ld_grad);
        else
            distill_row_kernel<T, MASK, false><<<a.rows, kThreads, 0, stream>>>(a, nullptr, loss, nullptr, 0);
        return last_launch();
    }
    Softmax *parts = static_cast<Softmax *>(workspace);
    float *listed = reinterpret_cast<float *>(parts + (size_t)a.rows * s.chunks);
    const dim3 grid(s.chunks, a.rows);
    distill_stats_kernel<T, MASK><<<grid, kThreads, 0, stream>>>(a, s.chunk, parts, listed);
    hipError_t e = last_launch();
    if (e != hipSuccess)
        return e;
    if (grad)
        distill_finish_kernel<T, MASK, true><<<grid, kThreads, 0, stream>>>(a, s.chunk, s.chunks, parts, listed,
                                                                            grad_loss, loss, grad, ld_grad);
    else
        distill_finish_kernel<T, MASK, false><<<dim3(1, a.rows), kThreads, 0, stream>>>(a, s.chunk, s.chunks, parts,
                                                                                        listed, nullptr, loss, nullptr, 0);
    return last_launch();
}

}  // namespace

// At most 512 chunks in all, of rows that are split (fewer than kWholeRows).
size_t distill_workspace_bytes(int rows, int V, int K)
{
    (void)V;
    const int split = rows < kWholeRows ? rows : kWholeRows - 1;
    return align_up((size_t)kSplitBlocks * sizeof(Softmax) + (size_t)split * (size_t)K * 4, 256);
}

hipError_t launch_distill(const DistillArgs &a, const float *grad_loss, float *loss, void *grad, int64_t ld_grad,
                          void *workspace, hipStream_t stream)
{
    const auto run = [&](auto *out) {
        using T = std::remove_pointer_t<decltype(out)>;
        if (a.masks.allow)
            return launch<T, true>(a, grad_loss, loss, out, ld_grad, workspace, stream);
        return launch<T, false>(a, grad_loss, loss, out, ld_grad, workspace, stream);
    };
    return a.dtype == 1 ? run(static_cast<uint16_t *>(grad)) : run(static_cast<float *>(grad));
}

}  // namespace dv
