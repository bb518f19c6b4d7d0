// Internal declarations of the training operators: the head loss
// (dv_head.hip), distillation (dv_distill.hip) and the embedding
// (dv_embed.hip).
#pragma once

#include "dv_internal.h"

namespace dv {

// The allowed tokens of a call's rows: allow[S][ceil(V/32)] and each row's
// state, or allow = NULL where every token is allowed.
struct Masks {
    const uint32_t *allow;
    const int32_t *states;
    int S;
};

// One row's allowed tokens, 32 a word, tokens past V never among them.
struct RowMask {
    const uint32_t *words;  // NULL: every token, or none of a dead row
    int V;
    bool dead;

    __device__ __forceinline__ RowMask(const Masks &m, int V, int row) : words(nullptr), V(V), dead(false)
    {
        if (m.allow) {
            const int s = m.states[row];
            dead = (uint32_t)s >= (uint32_t)m.S;
            words = dead ? nullptr : m.allow + (size_t)s * (((size_t)V + 31) / 32);
        }
    }
    __device__ __forceinline__ uint32_t word(int i) const
    {
        const int left = V - i * 32;
        if (dead || left <= 0)
            return 0;
        const uint32_t w = words ? words[i] : 0xFFFFFFFFu;
        return left >= 32 ? w : w & ((1u << left) - 1u);
    }
    __device__ __forceinline__ bool has(int v) const
    {
        return !dead && (uint32_t)v < (uint32_t)V && (!words || ((words[v >> 5] >> (v & 31)) & 1u));
    }
};

constexpr float kLog2e = 1.4426950408889634f;

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// Sum and maximum over the 64 lanes of a wave, the same value in every lane.
__device__ __forceinline__ float wave_sum(float v)
{
#pragma unroll
    for (int d = 32; d; d >>= 1)
        v += __shfl_xor(v, d);
    return v;
}
__device__ __forceinline__ float wave_max(float v)
{
#pragma unroll
    for (int d = 32; d; d >>= 1)
        v = fmaxf(v, __shfl_xor(v, d));
    return v;
}

// The running state of a softmax's sum: `sum` of exp((x - max) scale) over
// what has been seen.  Nothing seen, or only -infinity: max = -infinity and
// sum = 0; a NaN seen makes the sum NaN.  Differences are taken before they
// are scaled, so that values near the type's lowest stay in range.
struct Softmax {
    float max, sum;
    __device__ __forceinline__ bool empty() const { return sum == 0.f; }
};
__device__ __forceinline__ float softmax_term(float x, float max, float scale_log2e)
{
    return exp2_fast((x - max) * scale_log2e);
}
__device__ __forceinline__ Softmax softmax_join(Softmax a, Softmax b, float scale_log2e)
{
    const float m = fmaxf(a.max, b.max);
    const float sa = a.max == -INFINITY ? a.sum : a.sum * softmax_term(a.max, m, scale_log2e);
    const float sb = b.max == -INFINITY ? b.sum : b.sum * softmax_term(b.max, m, scale_log2e);
    return {m, sa + sb};
}

// bf16 conversions: the widening is exact, the narrowing rounds to nearest
// even (NaN stays NaN).
__device__ __forceinline__ float widen(uint16_t b) { return __uint_as_float((uint32_t)b << 16); }
__device__ __forceinline__ uint16_t narrow(float x)
{
    union {
        __bf16 b;
        uint16_t u;
    } c;
    c.b = (__bf16)x;
    return c.u;
}

// Two at once, the first in the low half.
__device__ __forceinline__ uint32_t narrow_pair(float lo, float hi)
{
    typedef __attribute__((ext_vector_type(2))) __bf16 Pair;
    union {
        Pair b;
        uint32_t u;
    } c;
    c.b = Pair{(__bf16)lo, (__bf16)hi};
    return c.u;
}

// 16 bytes from and to any element's alignment, as one access (arrays of
// elements copied with memcpy come apart into smaller ones).
typedef __attribute__((ext_vector_type(4))) uint32_t Words;
typedef __attribute__((ext_vector_type(4), aligned(2))) uint32_t AnyWords;
__device__ __forceinline__ Words load_words(const void *p) { return *static_cast<const AnyWords *>(p); }
__device__ __forceinline__ void store_words(void *p, Words w) { *static_cast<AnyWords *>(p) = w; }
// the same, past the caches: for what this call does not read again
__device__ __forceinline__ void stream_words(void *p, Words w)
{
    __builtin_nontemporal_store(static_cast<AnyWords>(w), static_cast<AnyWords *>(p));
}
// Element i of 16 bytes of T.
template <typename T>
__device__ __forceinline__ T element(const Words &w, int i)
{
    union {
        Words w;
        T t[16 / sizeof(T)];
    } u;
    u.w = w;
    return u.t[i];
}

inline hipError_t last_launch() { return hipGetLastError(); }

// --------------------------------------------------------------- head loss
struct HeadArgs {
    const void *x;
    int64_t ld_x;
    const void *weight;
    int64_t ld_w;
    int dtype;
    int rows, hidden, V;
    const int32_t *targets;
    Masks masks;
};
// For a call's own operands (x, weight, their strides, type and sizes), and for any operands.
size_t head_workspace_bytes(const HeadArgs &a);
size_t head_workspace_bytes(int rows, int hidden, int V, int dtype);
hipError_t launch_head_loss(const HeadArgs &a, float *loss, float *lse, void *workspace, hipStream_t stream);
size_t head_backward_workspace_bytes(const HeadArgs &a);
size_t head_backward_workspace_bytes(int rows, int hidden, int V, int dtype);
hipError_t launch_head_loss_backward(const HeadArgs &a, const float *lse, const float *grad_loss, void *grad_x,
                                     void *grad_weight, void *workspace, hipStream_t stream);

// ------------------------------------------------------------ distillation
struct DistillArgs {
    const void *logits;
    int64_t ld;
    int dtype;
    int rows, V;
    const int32_t *ids;
    const float *top;
    int K;
    float inv_temperature;
    Masks masks;
};
size_t distill_workspace_bytes(int rows, int V, int K);
// grad = NULL: the loss alone; loss may be NULL with grad.
hipError_t launch_distill(const DistillArgs &a, const float *grad_loss, float *loss, void *grad, int64_t ld_grad,
                          void *workspace, hipStream_t stream);

// --------------------------------------------------------------- embedding
hipError_t launch_embed(const void *weight, int64_t ld_w, int dtype, int V, int hidden, const int32_t *ids, int rows,
                        float scale, void *out, hipStream_t stream);
size_t embed_backward_workspace_bytes(int rows, int hidden, int V);
hipError_t launch_embed_backward(const void *grad_out, int64_t ld, int dtype, int rows, int hidden,
                                 const int32_t *ids, int V, float scale, bool accumulate, void *grad_weight,
                                 void *workspace, hipStream_t stream);

}  // namespace dv
