// Distillation from a teacher's top logits over the allowed tokens.
//
// Per row, with the allowed tokens A of the row's state, c = 1/T, and the
// listed teacher entries L = {k : id_k in A, top_k > -inf}:
//     q_k = exp(c (top_k - max)) / sum over L,   p_v = exp(c (z_v - m)) / s,
//     loss = sum_L q_k (ln q_k - ln p_{id_k}),
//     dloss/dz_v = c (p_v - sum of q_k with id_k = v)   on A, 0 elsewhere.
//
// The loss needs one read of the row, loss and gradient one read and one write of
// it: both are bound by memory.  The gradient's second pass finds the row in the
// caches, or in the block's registers.  Loss and gradient of 2,048 rows of 128,256 bf16 logits take 245 us (4.3
// TB/s of the 4.9 that a copy reaches), of 8,000 rows of 4,000 fp32 50 us (5.1);
// the loss alone 93 us and 24 us (5.6 and 5.3 TB/s).
//
// Few or short rows are bound by latency instead: a row's chain is its loads, a join
// over the block, and the stores.  So the teacher's entries are loaded first, their
// logits are on the way while the row streams, and one barrier joins both softmaxes.
#include <type_traits>

#include "dv_train.h"

namespace dv {
namespace {

constexpr int kThreads = 512;  // of blocks that share a row, and of those with a long one
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

constexpr int kMostThreads = 1024;  // of a block that holds a long row, or has a unit to itself
struct Shared {
    Softmax row[kMostThreads / kWave], top[kMostThreads / kWave];  // of each wave
    float loss[kMostThreads / kWave];
    int id[kMaxTop];
    float q[kMaxTop];
    float z[kMaxTop];
};

__device__ __forceinline__ Softmax wave_join(Softmax v, float c2)
{
    const float top = wave_max(v.max);
    return {top, wave_sum(v.max == -INFINITY ? v.sum : v.sum * softmax_term(v.max, top, c2))};
}

template <int THREADS>
__device__ __forceinline__ Softmax join_waves(const Softmax *of_wave, float c2)
{
    constexpr int kWaves = THREADS / kWave;
    Softmax t{-INFINITY, 0.f};
#pragma unroll
    for (int i = 0; i < kWaves; ++i)
        t.max = fmaxf(t.max, of_wave[i].max);
#pragma unroll
    for (int i = 0; i < kWaves; ++i)
        t.sum += of_wave[i].max == -INFINITY ? of_wave[i].sum : of_wave[i].sum * softmax_term(of_wave[i].max, t.max, c2);
    return t;
}

// A row's entries of the teacher, spread over a block's lanes.
template <int THREADS>
struct Teacher {
    static constexpr int kN = kMaxTop / THREADS;  // of a lane at most
    int id[kN];  // -1 where an entry takes no part
    float top[kN], z[kN];

    __device__ __forceinline__ void load(const DistillArgs &a, int row)
    {
#pragma unroll
        for (int e = 0; e < kN; ++e) {
            const int k = e * THREADS + threadIdx.x;
            id[e] = -1;
            top[e] = -INFINITY;
            z[e] = 0.f;
            if (k < a.K) {
                id[e] = a.ids[(size_t)row * a.K + k];
                top[e] = a.top[(size_t)row * a.K + k];
            }
        }
    }
    // logit(k, id): the model's logit of an entry that takes part
    template <typename F>
    __device__ __forceinline__ Softmax admit(const RowMask &m, float c2, F &&logit)
    {
        Softmax own{-INFINITY, 0.f};
#pragma unroll
        for (int e = 0; e < kN; ++e) {
            if (!m.has(id[e]) || top[e] == -INFINITY) {
                id[e] = -1;
            } else {
                z[e] = logit(e * THREADS + (int)threadIdx.x, id[e]);
                own = softmax_join(own, {top[e], 1.f}, c2);
            }
        }
        return own;
    }
    // Probabilities, ids and logits to LDS, and this lane's part of the loss.
    __device__ __forceinline__ float publish(int K, Softmax t, Softmax s, float c, float c2, Shared &sh) const
    {
        const float lnt = logf(t.sum), lns = logf(s.sum);
        float loss = 0.f;
#pragma unroll
        for (int e = 0; e < kN; ++e) {
            const int k = e * THREADS + threadIdx.x;
            const float q = id[e] < 0 ? 0.f : softmax_term(top[e], t.max, c2) / t.sum;
            if (k < K) {
                sh.id[k] = id[e];
                sh.q[k] = q;
                sh.z[k] = z[e];
            }
            if (!(q == 0.f)) {  // NaN counts
                // q c (z - max): c (z - max) of a logit near the type's lowest may pass its range
                const float below = z[e] - s.max;
                loss += q * (((top[e] - t.max) * c - lnt) + lns) - (below == -INFINITY ? below : q * c * below);
            }
        }
        return loss;
    }
};

// Vectors [j0, j1) of a row, kBatch a lane at a time: f(vectors, first, whole) has
// vector first + u THREADS + lane in place u; masked elements read as -infinity, and
// so do vectors past j1 (only where `whole` is false).  A batch's start is in
// scalar registers, a lane's offset from it 32 bits.
constexpr int kBatch = 4;

template <typename T, int THREADS, bool MASK, bool WHOLE>
__device__ __forceinline__ void load_batch(Vec<T> (&v)[kBatch], const T *z, const RowMask &m, int first, int j1)
{
    constexpr int N = Vec<T>::kN;
    uint32_t bits[kBatch];
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
        const int at = first + u * THREADS;  // uniform
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

template <typename T, int THREADS, bool MASK, typename F>
__device__ __forceinline__ void for_batches(const T *z, const RowMask &m, int j0, int j1, F &&f)
{
    constexpr int kStep = THREADS * kBatch;
    Vec<T> v[kBatch];
    int first = j0;
    for (; first + kStep <= j1; first += kStep) {
        load_batch<T, THREADS, MASK, true>(v, z, m, first, j1);
        f(v, first, std::true_type{});
    }
    if (first < j1) {
        load_batch<T, THREADS, MASK, false>(v, z, m, first, j1);
        f(v, first, std::false_type{});
    }
}

// exp(c (x - max)) as exp2(x c2 - shift), shift = max c2 rounded: one operation and
// one rounding; `correction` is the factor 2^(shift - max c2) that the rounding of
// the shift leaves: an exponential of its own, once a batch, because at logits of 500,000
// its first-order form 1 - d ln 2 is off by 2.4e-4.  Only where max c2 is of ordinary size:
// else (a row of nothing but the type's lowest value, say) differences are scaled.
struct Shift {
    float max, c2, shift, correction;
    bool plain;
    __device__ __forceinline__ Shift(float max_, float c2_) : max(max_ == -INFINITY ? 0.f : max_), c2(c2_)
    {
        shift = max * c2;
        plain = fabsf(shift) < 1048576.f;
        correction = plain ? exp2_fast(-__builtin_fmaf(max, c2, -shift)) : 1.f;
    }
    template <bool PLAIN>
    __device__ __forceinline__ float term(float x) const
    {
        return exp2_fast(PLAIN ? __builtin_fmaf(x, c2, -shift) : (x - max) * c2);
    }
};

// The softmax state of tokens [from, to) of a row (from a multiple of 8).
template <typename T, int THREADS, bool MASK>
__device__ __forceinline__ Softmax row_stats(const T *z, const RowMask &m, int from, int to, float c2)
{
    using V = Vec<T>;
    constexpr int N = V::kN;
    Softmax own{-INFINITY, 0.f};
    for_batches<T, THREADS, MASK>(z, m, from / N, to / N, [&](const V (&v)[kBatch], int, auto) {
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
    for (int i = to / N * N + threadIdx.x; i < to; i += THREADS)
        if (m.has(i)) {
            const float x = V::one(z + i);
            own = x == -INFINITY ? own : softmax_join(own, {x, 1.f}, c2);
        }
    return own;
}

// The gradient of the listed tokens in [from, to), once the block's other stores
// there are done: an id listed more than once takes the sum of its entries, in
// their order, from each of them.
template <typename T, int THREADS>
__device__ __forceinline__ void listed_grad(T *grad, int from, int to, float c2, float max, float scale, float w, int K,
                                            Shared &sh)
{
    for (int k = threadIdx.x; k < K; k += THREADS) {
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
template <typename T, int THREADS, bool MASK>
__device__ __forceinline__ void row_grad(const T *z, T *grad, const RowMask &m, int from, int to, float c2, Softmax s,
                                         float w, bool part)
{
    using V = Vec<T>;
    constexpr int N = V::kN;
    const int j0 = from / N, j1 = to / N;
    if (!part) {
        const float zeros[N] = {};
        for (int j = j0 + threadIdx.x; j < j1; j += THREADS)
            V::store(grad + (size_t)j * N, zeros);
        for (int i = j1 * N + threadIdx.x; i < to; i += THREADS)
            V::put(grad + i, 0.f);
        return;
    }
    const Shift t(s.max, c2);
    const float scale = w / s.sum;
    const auto write = [&](auto plain) {
        constexpr bool PLAIN = decltype(plain)::value;
        const float by = PLAIN ? scale * t.correction : scale;
        for_batches<T, THREADS, MASK>(z, m, j0, j1, [&](const V (&v)[kBatch], int first, auto whole) {
#pragma unroll
            for (int u = 0; u < kBatch; ++u) {
                float y[N];
#pragma unroll
                for (int i = 0; i < N; ++i)
                    y[i] = t.template term<PLAIN>(v[u].get(i)) * by;
                const int at = first + u * THREADS;
                if (decltype(whole)::value || at + (int)threadIdx.x < j1)
                    V::store(reinterpret_cast<T *>(reinterpret_cast<char *>(grad) + (size_t)at * 16 + threadIdx.x * 16u), y);
            }
        });
    };
    if (t.plain)
        write(std::true_type{});
    else
        write(std::false_type{});
    for (int i = j1 * N + threadIdx.x; i < to; i += THREADS)
        V::put(grad + i, m.has(i) ? softmax_term(V::one(z + i), s.max, c2) * scale : 0.f);
}

// What follows a row's (or chunk's) statistics `own` and the teacher's `entries`:
// the block's lanes join both, then the loss (if wanted) and the gradient of
// tokens [from, to): write(softmax, weight, part), then the listed tokens.  Two
// barriers: the joined statistics, and the listed tokens after the other stores.
template <typename T, int THREADS, bool GRAD, typename F>
__device__ __forceinline__ void finish_row(const DistillArgs &a, int row, int from, int to, Softmax own,
                                           Teacher<THREADS> &entries, Softmax own_top, const float *grad_loss, float *loss,
                                           T *grad, Shared &sh, F &&write)
{
    const float c = a.inv_temperature, c2 = c * kLog2e;
    const bool first_lane = (threadIdx.x & (kWave - 1)) == 0;
    const int wave = threadIdx.x / kWave;
    own = wave_join(own, c2);
    own_top = wave_join(own_top, c2);
    if (first_lane) {
        sh.row[wave] = own;
        sh.top[wave] = own_top;
    }
    __syncthreads();
    const Softmax s = join_waves<THREADS>(sh.row, c2), t = join_waves<THREADS>(sh.top, c2);
    const bool part = !s.empty() && !t.empty();
    if (part) {
        const float l = wave_sum(entries.publish(a.K, t, s, c, c2, sh));
        if (first_lane)
            sh.loss[wave] = l;
    }
    const float w = GRAD && part ? grad_loss[row] * c : 0.f;
    if (GRAD)
        write(s, w, part);
    __syncthreads();
    if (loss && threadIdx.x == 0) {
        float l = 0.f;
#pragma unroll
        for (int i = 0; i < THREADS / kWave; ++i)
            l += part ? sh.loss[i] : 0.f;
        loss[row] = l;
    }
    if (GRAD && part)
        listed_grad<T, THREADS>(grad, from, to, c2, s.max, w / s.sum, w, a.K, sh);
}

// One block per row: the row's softmax, the loss, and with GRAD the gradient
// from a second pass over the row, which its first pass left in the caches.
template <typename T, int THREADS, bool MASK, bool GRAD>
__global__ __launch_bounds__(THREADS) void distill_row_kernel(DistillArgs a, const float *grad_loss, float *loss, T *grad,
                                                              int64_t ld_grad)
{
    __shared__ Shared sh;
    const int row = blockIdx.x;
    const float c2 = a.inv_temperature * kLog2e;
    Teacher<THREADS> entries;
    entries.load(a, row);
    const RowMask m(a.masks, a.V, row);
    const T *z = static_cast<const T *>(a.logits) + (size_t)row * a.ld;
    const Softmax top = entries.admit(m, c2, [&](int, int id) { return Vec<T>::one(z + id); });
    Softmax own{-INFINITY, 0.f};
    if (!m.dead)
        own = row_stats<T, THREADS, MASK>(z, m, 0, a.V, c2);
    T *const out = GRAD ? grad + (size_t)row * ld_grad : nullptr;
    finish_row<T, THREADS, GRAD>(a, row, 0, a.V, own, entries, top, grad_loss, loss, out, sh,
                                 [&](Softmax s, float w, bool part) {
                                     row_grad<T, THREADS, MASK>(z, out, m, 0, a.V, c2, s, w, part);
                                 });
}

// Loss and gradient with the row held in the block's registers, VECS vectors a lane
// (at most THREADS VECS in all): it is read once, and every load is on its way
// before the first is used.
template <typename T, int THREADS, int VECS, bool MASK>
__global__ __launch_bounds__(THREADS, 4) void distill_held_kernel(DistillArgs a, const float *grad_loss, float *loss, T *grad,
                                                               int64_t ld_grad)
{
    using V = Vec<T>;
    constexpr int N = V::kN;
    __shared__ Shared sh;
    const int row = blockIdx.x;
    const float c2 = a.inv_temperature * kLog2e;
    Teacher<THREADS> entries;
    entries.load(a, row);
    const RowMask m(a.masks, a.V, row);
    const T *z = static_cast<const T *>(a.logits) + (size_t)row * a.ld;
    T *const out = grad + (size_t)row * ld_grad;
    const int vecs = a.V / N;
    V v[VECS];
    uint32_t bits[VECS];
    const uint8_t *bytes = reinterpret_cast<const uint8_t *>(m.words);
#pragma unroll
    for (int u = 0; u < VECS; ++u) {
        const int left = vecs - u * THREADS;  // uniform
        bits[u] = 0;
        if (left > 0 && !m.dead) {
            const bool in = (int)threadIdx.x < left;
            const uint32_t lane = in ? threadIdx.x : 0;
            v[u] = V::load(reinterpret_cast<const T *>(reinterpret_cast<const char *>(z) + (size_t)(u * THREADS) * 16 + lane * 16u));
            bits[u] = in ? 0xFFu : 0u;
            if (MASK) {
                const uint8_t *at = bytes + (size_t)(u * THREADS) / (8 / N);
                bits[u] &= N == 8 ? at[lane] : (uint32_t)at[lane >> 1] >> ((lane & 1) * 4);
            }
        }
    }
    const Softmax top = entries.admit(m, c2, [&](int, int id) { return V::one(z + id); });
    float most = -INFINITY;
#pragma unroll
    for (int u = 0; u < VECS; ++u) {
        v[u].keep(bits[u]);
#pragma unroll
        for (int i = 0; i < N; i += 2)
            most = fmaxf(fmaxf(most, v[u].get(i)), v[u].get(i + 1));
    }
    // the compiler would keep the widened elements from one pass to the next
    const auto narrow_again = [&] {
#pragma unroll
        for (int u = 0; u < VECS; ++u)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                asm("" : "+v"(v[u].x[i]));
    };
    narrow_again();
    const Shift t(most, c2);
    float sum = 0.f;
    if (__all(t.plain)) {
#pragma unroll
        for (int u = 0; u < VECS; ++u)
#pragma unroll
            for (int i = 0; i < N; ++i)
                sum += t.template term<true>(v[u].get(i));
        sum *= t.correction;
    } else {
#pragma unroll
        for (int u = 0; u < VECS; ++u)
#pragma unroll
            for (int i = 0; i < N; ++i)
                sum += t.template term<false>(v[u].get(i));
    }
    Softmax own{most, sum};
    const int rest = vecs * N + (int)threadIdx.x;  // of the row's end, an element a lane
    const bool has_rest = rest < a.V && m.has(rest);
    const float x_rest = has_rest ? V::one(z + rest) : -INFINITY;
    if (has_rest && x_rest != -INFINITY)
        own = softmax_join(own, {x_rest, 1.f}, c2);
    finish_row<T, THREADS, true>(a, row, 0, a.V, own, entries, top, grad_loss, loss, out, sh,
                                 [&](Softmax s, float w, bool part) {
        narrow_again();
        const Shift t(s.max, c2);
        const float scale = part ? w / s.sum : 0.f;
        const auto write = [&](auto plain) {
            constexpr bool PLAIN = decltype(plain)::value;
            const float by = PLAIN ? scale * t.correction : scale;
#pragma unroll
            for (int u = 0; u < VECS; ++u) {
                const int j = u * THREADS + (int)threadIdx.x;
                float y[N];
#pragma unroll
                for (int i = 0; i < N; ++i)
                    y[i] = part ? t.template term<PLAIN>(v[u].get(i)) * by : 0.f;
                if (j < vecs)
                    V::store(reinterpret_cast<T *>(reinterpret_cast<char *>(out) + (size_t)(u * THREADS) * 16 + threadIdx.x * 16u), y);
            }
        };
        if (t.plain)
            write(std::true_type{});
        else
            write(std::false_type{});
        if (rest < a.V)
            V::put(out + rest, part && has_rest ? softmax_term(x_rest, s.max, c2) * scale : 0.f);
    });
}

// Rows split over blocks (few rows): the chunks' softmax states, and the
// logits of the listed tokens (the gradient may overwrite the logits) ...
template <typename T, bool MASK>
__global__ __launch_bounds__(kThreads) void distill_stats_kernel(DistillArgs a, int chunk, Softmax *part, float *listed)
{
    __shared__ Softmax of_wave[kThreads / kWave];
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
        s = row_stats<T, kThreads, MASK>(z, m, from, to, c2);
    s = wave_join(s, c2);
    if ((threadIdx.x & (kWave - 1)) == 0)
        of_wave[threadIdx.x / kWave] = s;
    __syncthreads();
    if (threadIdx.x == 0)
        part[(size_t)row * gridDim.x + c] = join_waves<kThreads>(of_wave, c2);
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
    Teacher<kThreads> entries;
    entries.load(a, row);
    const RowMask m(a.masks, a.V, row);
    Softmax own{-INFINITY, 0.f};
    for (int i = threadIdx.x; i < chunks; i += kThreads)
        own = softmax_join(own, parts[(size_t)row * chunks + i], c2);
    const Softmax top = entries.admit(m, c2, [&](int k, int) { return listed[(size_t)row * a.K + k]; });
    const int from = c * chunk, to = a.V - from < chunk ? a.V : from + chunk;
    const T *z = static_cast<const T *>(a.logits) + (size_t)row * a.ld;
    T *const out = GRAD ? grad + (size_t)row * ld_grad : nullptr;
    finish_row<T, kThreads, GRAD>(a, row, from, to, own, entries, top, grad_loss, c == 0 ? loss : nullptr, out, sh,
                                  [&](Softmax s, float w, bool part) {
                                      row_grad<T, kThreads, MASK>(z, out, m, from, to, c2, s, w, part);
                                  });
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

// Blocks of 512 lanes leave most of them idle in a short row, and fewer rows under
// way on a compute unit.  Loss and gradient with 512, 256 and 128 lanes (us):
//     8,192 x 1,000 fp32 (250 vectors)     57  32  27
//     8,000 x 4,000 bf16 (500)             81  45  37
//     8,000 x 4,000 fp32 (1,000)           77  58  65
//     8,000 x 8,000 bf16 (1,000)           92  59  63
//     4,000 x 8,000 fp32 (2,000)           53  60   -
//     4,000 x 16,000 bf16 (2,000)          60  61   -
// and the loss alone 42 23 16, 57 30 21, 40 24 24, 54 31 28, 24 22, 31 26.
constexpr int kShortRow = 512;    // vectors of a row for blocks of 128 lanes
constexpr int kMiddleRow = 2048;  // and of 256, without the gradient
constexpr int kMiddleRowGrad = 1536;

// The lanes of a block that holds a row of `vecs` vectors of n elements, or 0 for the
// two passes.  Logits that fit the L2s (32 MB) are read twice at little cost; past
// them holding pays (loss and gradient, two passes and held, us):
//     8,192 x 1,000 fp32 (128 lanes x 4 vectors)   28  27     4,000 x 16,000 fp32 (512 x 8)  110  89
//     8,000 x 4,000 bf16 (128 x 4)                 38  36     2,000 x 32,003 bf16 (512 x 8)   69  62
//     8,000 x 4,000 fp32 (256 x 4)                 53  50     2,000 x 32,000 fp32 (512 x 16) 116  90
//     4,000 x 8,000 fp32 (256 x 8)                 52  47     1,500 x 50,257 bf16 (512 x 16)  83  71
//     4,000 x 16,000 bf16 (256 x 8)                61  52     1,000 x 65,000 fp32 (1024 x 16) 122 107
// and below 400 x 32,000 bf16 16.0 16.8, 250 x 60,000 bf16 18.3 19.3.  Blocks of 16 vectors a lane
// fill a compute unit by two (512 lanes) or alone (1,024): the last round of them must
// not be nearly empty (520 x 50,257 fp32: 57.5 and 59.3).  Alone, bf16 rows' exponentials
// are not hidden behind another block's loads (2,048 x 128,256: 243 and 263): two passes.
constexpr int64_t kL2Bytes = (int64_t)32 << 20;

int held_lanes(int64_t rows, int vecs, int n)
{
    if (rows * vecs * 16 < kL2Bytes || vecs > (n == 4 ? 16384 : 8192))
        return 0;
    if (vecs <= 512)
        return 128;
    if (vecs <= 2048)
        return 256;
    if (vecs <= 4096)
        return 512;
    const int lanes = vecs <= 8192 ? 512 : 1024;
    const int64_t slots = vecs <= 8192 ? 512 : 256;
    const int64_t rounds = (rows + slots - 1) / slots;
    return rounds * slots * 10 <= rows * 13 ? lanes : 0;
}

template <typename T, int THREADS, int VECS, bool MASK>
hipError_t launch_held(const DistillArgs &a, const float *grad_loss, float *loss, T *grad, int64_t ld_grad,
                       hipStream_t stream)
{
    distill_held_kernel<T, THREADS, VECS, MASK><<<a.rows, THREADS, 0, stream>>>(a, grad_loss, loss, grad, ld_grad);
    return last_launch();
}

// The second pass over rows past the L2s finds them in the memory-side cache (256 MB) if the
// rows under way fit there.  Four blocks a compute unit of rows over 200 KB do not: LDS
// that a block asks for and does not use leaves room for two, or for one of twice the
// lanes (loss and gradient with four, two, one, and one of 1,024 lanes, us):
//     1,000 x 150,000 bf16 147 143 158   -     1,000 x 256,000 bf16 276 256 251 243
//     1,000 x 200,000 bf16 201 196 201   -     2,000 x 256,000 bf16 560 506 494 479
//     1,000 x 100,000 fp32 205 192 192   -       600 x 128,256 fp32 161 162 149 144
//     2,000 x  80,000 fp32 312 304 299   -     1,000 x 256,000 fp32 599 601 502 487
// (2,048 x 128,256 bf16, three instead of four: 243 242.)
constexpr size_t kRowsUnderWay = (size_t)208 << 20;
constexpr unsigned kRoomForTwo = 50 << 10, kRoomForOne = 100 << 10;  // of 160 KB; a block uses 13

bool too_many(int64_t blocks_per_unit, size_t row_bytes) { return blocks_per_unit * 256 * row_bytes > kRowsUnderWay; }

template <typename T, int THREADS, bool MASK>
hipError_t launch_rows(const DistillArgs &a, const float *grad_loss, float *loss, T *grad, int64_t ld_grad,
                       hipStream_t stream, unsigned idle_lds = 0)
{
    if (grad)
        distill_row_kernel<T, THREADS, MASK, true>
            <<<a.rows, THREADS, idle_lds, stream>>>(a, grad_loss, loss, grad, ld_grad);
    else
        distill_row_kernel<T, THREADS, MASK, false><<<a.rows, THREADS, 0, stream>>>(a, nullptr, loss, nullptr, 0);
    return last_launch();
}

template <typename T, bool MASK>
hipError_t launch(const DistillArgs &a, const float *grad_loss, float *loss, T *grad, int64_t ld_grad, void *workspace,
                  hipStream_t stream)
{
    const Split s = split_of(a.rows, a.V, a.dtype, grad != nullptr);
    if (s.chunks == 1) {
        const int vecs = a.V / Vec<T>::kN;
        const int held = grad ? held_lanes(a.rows, vecs, Vec<T>::kN) : 0;
        if (held == 128)
            return launch_held<T, 128, 4, MASK>(a, grad_loss, loss, grad, ld_grad, stream);
        if (held == 256 && vecs <= 1024)
            return launch_held<T, 256, 4, MASK>(a, grad_loss, loss, grad, ld_grad, stream);
        if (held == 256)
            return launch_held<T, 256, 8, MASK>(a, grad_loss, loss, grad, ld_grad, stream);
        if (held == 512 && vecs <= 4096)
            return launch_held<T, 512, 8, MASK>(a, grad_loss, loss, grad, ld_grad, stream);
        if (held == 512)
            return launch_held<T, 512, 16, MASK>(a, grad_loss, loss, grad, ld_grad, stream);
        if constexpr (Vec<T>::kN == 4)
            if (held)
                return launch_held<T, 1024, 16, MASK>(a, grad_loss, loss, grad, ld_grad, stream);
        if (vecs <= kShortRow)
            return launch_rows<T, 128, MASK>(a, grad_loss, loss, grad, ld_grad, stream);
        if (vecs <= (grad ? kMiddleRowGrad : kMiddleRow))
            return launch_rows<T, 256, MASK>(a, grad_loss, loss, grad, ld_grad, stream);
        const size_t row_bytes = (size_t)a.V * sizeof(T);
        if (grad && too_many(2, row_bytes)) {
            distill_row_kernel<T, kMostThreads, MASK, true>
                <<<a.rows, kMostThreads, kRoomForOne, stream>>>(a, grad_loss, loss, grad, ld_grad);
            return last_launch();
        }
        return launch_rows<T, kThreads, MASK>(a, grad_loss, loss, grad, ld_grad, stream,
                                              too_many(3, row_bytes) ? kRoomForTwo : 0);
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
