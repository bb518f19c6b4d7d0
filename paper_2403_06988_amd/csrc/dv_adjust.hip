// Logits with each sequence's penalties, biases and grammar mask applied.
//
//     z' = z / rho (z > 0) or z rho (else)     for tokens of the prompt or the output
//     z' -= c frequency, - presence (c > 0)    c: how often the token stands in the output
//     z' += the sum of its biases
//     z' = -infinity                           where the row's state does not allow it
//
// A block takes a window of one row's vocabulary.  It counts the window's tokens of the
// history in LDS, one word a token: the count, whether it was seen at all, and the
// number of its bias.  Then the window's logits pass through once; where the word is
// zero a logit is copied as it is.  In place and without a mask only the tokens of the
// history and of the biases are touched, each by whoever takes its word first.
#include "../../include/dv.h"
#include "dv_logits.h"

namespace dv {
namespace {

constexpr uint32_t kCountMask = (1u << 20) - 1;  // occurrences in the output
constexpr uint32_t kSeen = 1u << 20;
constexpr int kBiasShift = 21;                   // 0: none, else its place + 1
static_assert(DV_MAX_HISTORY <= (int)kCountMask && DV_MAX_BIAS < (1 << (32 - kBiasShift)), "a word holds them");

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

__device__ __forceinline__ float adjusted(float z, uint32_t word, const Request &r, const float *totals)
{
    if (word & kSeen)
        z = z > 0.f ? z / r.rho : z * r.rho;
    if (const uint32_t c = word & kCountMask)
        z = z - (float)c * r.frequency - r.presence;
    if (const uint32_t k = word >> kBiasShift)
        z += totals[k - 1];
    return z;
}

template <typename T, int WINDOW, bool SPARSE>
__global__ __launch_bounds__(256) void adjust_kernel(AdjustArgs a, int windows)
{
    __shared__ __attribute__((aligned(16))) uint32_t words[WINDOW];
    __shared__ float totals[DV_MAX_BIAS];
    const int row = blockIdx.x / windows;
    const int v0 = (int)(blockIdx.x % windows) * WINDOW;
    const int n = a.V - v0 < WINDOW ? a.V - v0 : WINDOW;
    const T *in = static_cast<const T *>(a.logits) + (int64_t)row * a.ld + v0;
    T *out = static_cast<T *>(a.out) + (int64_t)row * a.ld_out + v0;

    for (int i = threadIdx.x; i < WINDOW; i += 256)
        words[i] = 0;
    __syncthreads();
    Request r{1.f, 0.f, 0.f};
    int length = 0;
    const int32_t *history = nullptr;
    if (a.history) {
        length = a.lengths[row];
        length = length < 0 ? 0 : length > a.max_history ? a.max_history : length;
        const int prompt = a.prompt_lengths ? a.prompt_lengths[row] : 0;
        history = a.history + (int64_t)row * a.ld_history;
        r.rho = a.repetition ? a.repetition[row] : 1.f;
        r.presence = a.presence ? a.presence[row] : 0.f;
        r.frequency = a.frequency ? a.frequency[row] : 0.f;
        for (int i = threadIdx.x; i < length; i += 256) {
            const uint32_t at = (uint32_t)history[i] - (uint32_t)v0;
            if (at < (uint32_t)n) {
                atomicOr(&words[at], kSeen);
                if (i >= prompt)
                    atomicAdd(&words[at], 1u);
            }
        }
    }
    const int32_t *ids = a.num_bias ? a.bias_ids + (int64_t)row * a.num_bias : nullptr;
    const float *bias = a.num_bias ? a.bias + (int64_t)row * a.num_bias : nullptr;
    for (int i = threadIdx.x; i < a.num_bias; i += 256) {
        const int id = ids[i];
        const uint32_t at = (uint32_t)id - (uint32_t)v0;
        if (at >= (uint32_t)n)
            continue;
        bool first = true;  // the first entry of a token adds up all of them, in their order
        for (int k = 0; k < i && first; ++k)
            first = ids[k] != id;
        if (!first)
            continue;
        float sum = bias[i];
        for (int k = i + 1; k < a.num_bias; ++k)
            if (ids[k] == id)
                sum += bias[k];
        totals[i] = sum;
        atomicOr(&words[at], (uint32_t)(i + 1) << kBiasShift);
    }
    __syncthreads();
    if constexpr (SPARSE) {
        const auto touch = [&](int id) {
            const uint32_t at = (uint32_t)id - (uint32_t)v0;
            if (at < (uint32_t)n) {
                const uint32_t word = atomicExch(&words[at], 0u);
                if (word)
                    out[at] = as_logit<T>(adjusted(as_float(in[at]), word, r, totals));
            }
        };
        for (int i = threadIdx.x; i < length; i += 256)
            touch(history[i]);
        for (int i = threadIdx.x; i < a.num_bias; i += 256)
            touch(ids[i]);
    } else {
        const RowMask mask(a.masks, a.V, row);
        for (int i = threadIdx.x; i < n; i += 256) {
            const uint32_t word = words[i];
            T z = in[i];
            if (word)
                z = as_logit<T>(adjusted(as_float(z), word, r, totals));
            out[i] = !a.masks.allow || mask.has(v0 + i) ? z : as_logit<T>(-INFINITY);
        }
    }
}

}  // namespace

hipError_t launch_adjust_logits(const AdjustArgs &a, hipStream_t stream)
{
    constexpr int kWindow = 8192;
    const bool sparse = a.out == a.logits && !a.masks.allow;
    const int windows = (a.V + kWindow - 1) / kWindow;
    const unsigned grid = (unsigned)((int64_t)a.rows * windows);
    const auto go = [&](auto kernel) { kernel<<<grid, 256, 0, stream>>>(a, windows); };
    if (a.dtype == 1)
        sparse ? go(adjust_kernel<uint16_t, kWindow, true>) : go(adjust_kernel<uint16_t, kWindow, false>);
    else
        sparse ? go(adjust_kernel<float, kWindow, true>) : go(adjust_kernel<float, kWindow, false>);
    return last_launch();
}

}  // namespace dv
