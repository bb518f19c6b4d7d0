// Logits with each sequence's penalties, biases and grammar mask applied.
//
//     z' = z / rho (z > 0) or z rho (else)     for tokens of the prompt or the output
//     z' -= c frequency, - presence (c > 0)    c: how often the token stands in the output
//     z' += the sum of its biases
//     z' = -infinity                           where the row's state does not allow it
//
// A block takes a window of one row's vocabulary.  Its logits are on their way to registers
// while the block counts the window's tokens of the history in LDS, one word a token: how
// often it stands in the output, whether it was seen at all, and the number of its
// bias.  Where the word is zero a logit leaves as it came.  In place and without a mask only
// the tokens of the history and of the biases are touched, each by whoever takes its word first.
//
// 256 x 128,256 bf16 with histories of up to 2,048, 32 biases and a mask: 36 us (reading and writing
// all of it once: 26 at a copy's rate); windows of 8,192 tokens (fewer blocks at once) 58 us
// before the loads came first, of 4,096 45.  A mask alone on 64 x 128,256: 7.1 us.
#include <type_traits>

#include "../../include/dv.h"
#include "dv_logits.h"

namespace dv {
namespace {

constexpr uint32_t kCountMask = (1u << 20) - 1;  // occurrences in the output
constexpr uint32_t kPrompt = 1u << 20;           // seen in the prompt
constexpr int kBiasShift = 21;                   // 0: none, else DV_MAX_BIAS less its first entry's place
static_assert(DV_MAX_HISTORY <= (int)kCountMask && DV_MAX_BIAS < (1 << (32 - kBiasShift)), "a word holds them");

constexpr int kWindow = 4096;

struct Request {
    float rho, presence, frequency;
};

template <typename T>
__device__ __forceinline__ float as_float(T x)
{
    if constexpr (sizeof(T) == 2)
        return widen(x);
    else
        return x;
}
template <typename T>
__device__ __forceinline__ T as_logit(float x)
{
    if constexpr (sizeof(T) == 2)
        return narrow(x);
    else
        return x;
}

// bias_of(i): the bias of the token whose first entry is i
template <typename F>
__device__ __forceinline__ float adjusted(float z, uint32_t word, const Request &r, F &&bias_of)
{
    if (word & (kPrompt | kCountMask))
        z = z > 0.f ? z / r.rho : z * r.rho;
    if (const uint32_t c = word & kCountMask)
        z = z - (float)c * r.frequency - r.presence;
    if (const uint32_t k = word >> kBiasShift)
        z += bias_of(DV_MAX_BIAS - (int)k);
    return z;
}

// NAMED: the call has histories or biases.  Everything that it reads at known places is asked for
// at once, before the first of it is needed: a block is mostly one wait for memory.
// Dynamic LDS: the window's words, then the biases' entries.
template <typename T, int THREADS, bool SPARSE, bool NAMED>
__global__ __launch_bounds__(THREADS) void adjust_kernel(AdjustArgs a, int windows)
{
    constexpr int kN = 16 / (int)sizeof(T), kV = kWindow / THREADS / kN;  // logits of a vector, vectors of a thread
    extern __shared__ __attribute__((aligned(16))) uint32_t words[];
    struct Entry {
        int at;        // the token's place in the window (past it: another window's, or none)
        float total;   // its bias; of a token's first entry the sum of all of them
        int again;     // of a first entry: there are others
    };
    Entry *const entries = reinterpret_cast<Entry *>(words + kWindow);
    const int row = blockIdx.x / windows;
    const int v0 = (int)(blockIdx.x % windows) * kWindow;
    const int n = a.V - v0 < kWindow ? a.V - v0 : kWindow;
    const T *in = static_cast<const T *>(a.logits) + (int64_t)row * a.ld + v0;
    T *out = static_cast<T *>(a.out) + (int64_t)row * a.ld_out + v0;
    const auto place = [&](int i) { return (i * THREADS + (int)threadIdx.x) * kN; };  // of vector i in the window

    constexpr int kAtOnce = 8;
    const int32_t *const history = NAMED && a.history ? a.history + (int64_t)row * a.ld_history : nullptr;
    const int32_t *const bias_ids = a.bias_ids + (int64_t)row * a.num_bias;
    const float *const bias = a.bias + (int64_t)row * a.num_bias;
    int first_ids[kAtOnce], length = 0, prompt = 0, my_id = 0;
    float my_bias = 0.f;
    Request r{1.f, 0.f, 0.f};
    if constexpr (NAMED) {
        if (history) {
#pragma unroll
            for (int k = 0; k < kAtOnce; ++k) {
                const int i = k * THREADS + (int)threadIdx.x;
                first_ids[k] = i < a.max_history ? history[i] : -1;
            }
            length = a.lengths[row];
            prompt = a.prompt_lengths ? a.prompt_lengths[row] : 0;
            r.rho = a.repetition ? a.repetition[row] : 1.f;
            r.presence = a.presence ? a.presence[row] : 0.f;
            r.frequency = a.frequency ? a.frequency[row] : 0.f;
        }
        if ((int)threadIdx.x < a.num_bias) {
            my_id = bias_ids[threadIdx.x];
            my_bias = bias[threadIdx.x];
        }
    }

    // the window's logits; what the mask leaves nothing of is not read
    const RowMask mask(a.masks, a.V, row);
    Words x[kV];
    uint32_t may[kV];
    if constexpr (!SPARSE) {
#pragma unroll
        for (int i = 0; i < kV; ++i) {
            const int at = place(i);
            may[i] = at < n ? a.masks.allow ? mask.word((v0 + at) >> 5) >> (at & 31) & ((1u << kN) - 1u) : (1u << kN) - 1u : 0u;
            if (at + kN <= n) {
                if (may[i])
                    x[i] = load_words(in + at);
            } else {
                T t[kN];
#pragma unroll
                for (int e = 0; e < kN; ++e)
                    t[e] = at + e < n ? in[at + e] : T(0);
                __builtin_memcpy(&x[i], t, sizeof t);
            }
        }
    }

    if constexpr (NAMED) {
        for (int i = threadIdx.x; i < kWindow / 4; i += THREADS)
            reinterpret_cast<uint4 *>(words)[i] = uint4{0, 0, 0, 0};
        for (int i = threadIdx.x; i < a.num_bias; i += THREADS) {
            const bool first = i < THREADS;
            entries[i] = {(int)((uint32_t)(first ? my_id : bias_ids[i]) - (uint32_t)v0), first ? my_bias : bias[i], 0};
        }
        __syncthreads();
        if (a.num_bias) {
            // the word's upper bits take the token's first entry
            for (int i = threadIdx.x; i < a.num_bias; i += THREADS)
                if ((uint32_t)entries[i].at < (uint32_t)n)
                    atomicMax(&words[entries[i].at], (uint32_t)(DV_MAX_BIAS - i) << kBiasShift);
            __syncthreads();
            int others = 0;
            for (int i = threadIdx.x; i < a.num_bias; i += THREADS)
                if ((uint32_t)entries[i].at < (uint32_t)n) {
                    const int first = DV_MAX_BIAS - (int)(words[entries[i].at] >> kBiasShift);
                    if (first != i)
                        entries[first].again = others = 1;
                }
            if (__syncthreads_or(others)) {
                // a token listed twice: a wave adds up its entries, in their order
                const int lane = threadIdx.x & (kWave - 1);
                for (int base = threadIdx.x - lane; base < a.num_bias; base += THREADS) {
                    uint64_t marked = __ballot(base + lane < a.num_bias && entries[base + lane].again);
                    for (; marked; marked &= marked - 1) {
                        const int i = base + __builtin_ctzll(marked), at = entries[i].at;
                        float sum = 0.f;
                        for (int from = i - i % kWave; from < a.num_bias; from += kWave) {
                            uint64_t same = __ballot(from + lane < a.num_bias && entries[from + lane].at == at);
                            for (; same; same &= same - 1)
                                sum += entries[from + __builtin_ctzll(same)].total;
                        }
                        entries[i].total = sum;  // (no other wave reads this token's)
                    }
                }
            }
        }
        if (history) {
            length = length < 0 ? 0 : length > a.max_history ? a.max_history : length;
            const auto count = [&](int i, int id) {
                const uint32_t at = (uint32_t)id - (uint32_t)v0;
                if (i < length && at < (uint32_t)n) {
                    if (i >= prompt)
                        atomicAdd(&words[at], 1u);
                    else
                        atomicOr(&words[at], kPrompt);
                }
            };
#pragma unroll
            for (int k = 0; k < kAtOnce; ++k)
                count(k * THREADS + (int)threadIdx.x, first_ids[k]);
            for (int from = kAtOnce * THREADS; from < length; from += kAtOnce * THREADS) {
                int id[kAtOnce];
#pragma unroll
                for (int k = 0; k < kAtOnce; ++k) {
                    const int i = from + k * THREADS + (int)threadIdx.x;
                    id[k] = i < length ? history[i] : -1;
                }
#pragma unroll
                for (int k = 0; k < kAtOnce; ++k)
                    count(from + k * THREADS + (int)threadIdx.x, id[k]);
            }
        }
        __syncthreads();
    }
    const auto bias_of = [&](int i) { return entries[i].total; };
    if constexpr (SPARSE) {
        const auto touch = [&](uint32_t at) {
            if (at < (uint32_t)n) {
                const uint32_t word = atomicExch(&words[at], 0u);
                if (word)
                    out[at] = as_logit<T>(adjusted(as_float(in[at]), word, r, bias_of));
            }
        };
        for (int i = threadIdx.x; i < length; i += THREADS)
            touch((uint32_t)history[i] - (uint32_t)v0);
        for (int i = threadIdx.x; i < a.num_bias; i += THREADS)
            touch((uint32_t)entries[i].at);
    } else {
#pragma unroll
        for (int i = 0; i < kV; ++i) {
            const int at = place(i);
            if (at >= n)
                break;
            T y[kN];
            __builtin_memcpy(y, &x[i], sizeof y);
            if constexpr (NAMED) {
                uint32_t w[kN], any = 0;
#pragma unroll
                for (int e = 0; e < kN; e += 4) {
                    const uint4 four = *reinterpret_cast<const uint4 *>(words + at + e);
                    w[e] = four.x, w[e + 1] = four.y, w[e + 2] = four.z, w[e + 3] = four.w;
                    any |= four.x | four.y | four.z | four.w;
                }
                if (any && may[i])
#pragma unroll
                    for (int e = 0; e < kN; ++e)
                        if (w[e])
                            y[e] = as_logit<T>(adjusted(as_float(y[e]), w[e], r, bias_of));
            }
#pragma unroll
            for (int e = 0; e < kN; ++e)
                y[e] = may[i] >> e & 1u ? y[e] : as_logit<T>(-INFINITY);
            if (at + kN <= n) {
                Words w;
                __builtin_memcpy(&w, y, sizeof w);
                store_words(out + at, w);
            } else {
#pragma unroll
                for (int e = 0; e < kN; ++e)
                    if (at + e < n)
                        out[at + e] = y[e];
            }
        }
    }
}

}  // namespace

hipError_t launch_adjust_logits(const AdjustArgs &a, hipStream_t stream)
{
    const bool sparse = a.out == a.logits && !a.masks.allow, named = a.history || a.num_bias;
    if (sparse && !named)
        return hipSuccess;
    const int windows = (a.V + kWindow - 1) / kWindow;
    const unsigned grid = (unsigned)((int64_t)a.rows * windows);
    const size_t lds = named ? kWindow * 4 + (size_t)a.num_bias * 12 : 0;
    // Blocks of 512 threads where all of them run at once: a history is counted in half the time
    // (77 x 50,257 fp32, histories of up to 16,384 tokens: 14.0 us, in blocks of 256 17.2; 1 x 32,000 4.8
    // and 5.9).  Of 256 where they take turns (256 x 128,256 bf16 36 us, in blocks of 512 44).
    const auto types = [&](auto zero, auto threads) {
        using T = decltype(zero);
        constexpr int kThreads = decltype(threads)::value;
        const auto go = [&](auto kernel) { kernel<<<grid, kThreads, lds, stream>>>(a, windows); };
        if (sparse)
            go(adjust_kernel<T, kThreads, true, true>);
        else if (named)
            go(adjust_kernel<T, kThreads, false, true>);
        else if constexpr (kThreads == 256)
            go(adjust_kernel<T, kThreads, false, false>);
    };
    const auto blocks = [&](auto threads) { a.dtype == 1 ? types(uint16_t{}, threads) : types(float{}, threads); };
    if (named && grid <= 1024)
        blocks(std::integral_constant<int, 512>{});
    else
        blocks(std::integral_constant<int, 256>{});
    return last_launch();
}

}  // namespace dv
