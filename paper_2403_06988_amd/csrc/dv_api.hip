// C ABI of libdv.so (declared in include/dv.h): argument checks, then the
// launches.  Every check runs on the host before any HIP call, so a rejected
// call enqueues nothing and touches no device state.
#include <stdarg.h>
#include <stdio.h>

#include <atomic>
#include <mutex>

#include "../../include/dv.h"
#include "dv_internal.h"
#include "dv_logits.h"
#include "dv_sample.h"
#include "dv_train.h"

namespace {

thread_local char g_error[512] = "";

dv_status fail(dv_status st, const char *fmt, ...)
{
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(g_error, sizeof g_error, fmt, ap);
    va_end(ap);
    return st;
}

// Byte range [p, p + n) of a device pointer, for overlap checks.
struct Range {
    uintptr_t lo, hi;
};
Range range_of(const void *p, size_t n) { return {reinterpret_cast<uintptr_t>(p), reinterpret_cast<uintptr_t>(p) + n}; }
bool overlap(Range a, Range b) { return a.lo < b.hi && b.lo < a.hi && a.lo != a.hi && b.lo != b.hi; }

dv_status hip_status(hipError_t e, const char *what)
{
    if (e == hipSuccess)
        return DV_OK;
    return fail(DV_ERR_HIP, "%s: %s", what, hipGetErrorString(e));
}

}  // namespace

extern "C" {

int32_t dv_version(void) { return 100; }

const char *dv_status_string(int32_t status)
{
    switch (status) {
    case DV_OK: return "DV_OK";
    case DV_ERR_INVALID_ARG: return "DV_ERR_INVALID_ARG";
    case DV_ERR_SHAPE: return "DV_ERR_SHAPE";
    case DV_ERR_DTYPE: return "DV_ERR_DTYPE";
    case DV_ERR_ALIAS: return "DV_ERR_ALIAS";
    case DV_ERR_WORKSPACE: return "DV_ERR_WORKSPACE";
    case DV_ERR_HIP: return "DV_ERR_HIP";
    default: return "DV_ERR_UNKNOWN";
    }
}

const char *dv_last_error(void) { return g_error; }

size_t dv_align_workspace_bytes(int32_t num_states, int32_t num_tokens)
{
    if (num_states < 1 || num_states > DV_MAX_STATES || num_tokens < 1 || num_tokens > DV_MAX_TOKENS)
        return 0;
    return dv::align_workspace_bytes(num_states, num_tokens);
}

static dv_status align_common(const char *name, const int32_t *trans, int32_t num_states,
                              const int32_t *offsets, const uint8_t *bytes, int32_t num_tokens,
                              const uint8_t *accepting, int32_t eos_token, int32_t *next_state,
                              uint32_t *allow, void *workspace, size_t workspace_bytes, void *stream)
{
    g_error[0] = '\0';
    if (!trans || !offsets || !next_state || !allow)
        return fail(DV_ERR_INVALID_ARG, "%s: trans, offsets, next_state and allow must be non-NULL", name);
    if (num_states < 1 || num_states > DV_MAX_STATES)
        return fail(DV_ERR_SHAPE, "%s: num_states=%d outside [1, %d]", name, num_states, DV_MAX_STATES);
    if (num_tokens < 1 || num_tokens > DV_MAX_TOKENS)
        return fail(DV_ERR_SHAPE, "%s: num_tokens=%d outside [1, %d]", name, num_tokens, DV_MAX_TOKENS);
    if (eos_token < -1 || eos_token >= num_tokens)
        return fail(DV_ERR_SHAPE, "%s: eos_token=%d outside [0, %d)", name, eos_token, num_tokens);
    const size_t S = (size_t)num_states, V = (size_t)num_tokens, W = (V + 31) / 32;
    const Range r_ns = range_of(next_state, S * V * 4), r_al = range_of(allow, S * W * 4);
    const Range r_tr = range_of(trans, S * 256 * 4), r_off = range_of(offsets, (V + 1) * 4);
    const Range r_acc = range_of(accepting, accepting ? S : 0);
    if (overlap(r_ns, r_al) || overlap(r_ns, r_tr) || overlap(r_ns, r_off) || overlap(r_al, r_tr) ||
        overlap(r_al, r_off) || overlap(r_ns, r_acc) || overlap(r_al, r_acc))
        return fail(DV_ERR_ALIAS, "%s: next_state / allow overlap each other or an input", name);
    const size_t need = dv::align_workspace_bytes(num_states, num_tokens);
    if (!workspace || workspace_bytes < need)
        return fail(DV_ERR_WORKSPACE, "%s: workspace of %zu bytes given, %zu needed", name, workspace_bytes, need);
    if (reinterpret_cast<uintptr_t>(workspace) & 255)
        return fail(DV_ERR_WORKSPACE, "%s: workspace must be 256-byte aligned", name);
    const Range r_ws = range_of(workspace, need);
    if (overlap(r_ws, r_ns) || overlap(r_ws, r_al) || overlap(r_ws, r_tr) || overlap(r_ws, r_off) ||
        overlap(r_ws, r_acc))
        return fail(DV_ERR_ALIAS, "%s: workspace overlaps an input or output", name);
    // bytes == NULL is accepted; the kernels read it only for non-empty tokens.
    return hip_status(dv::launch_align(trans, num_states, offsets, bytes, num_tokens, accepting, eos_token,
                                       next_state, allow, workspace, static_cast<hipStream_t>(stream)),
                      "launch");
}

dv_status dv_align(const int32_t *trans, int32_t num_states, const int32_t *offsets,
                   const uint8_t *bytes, int32_t num_tokens, int32_t *next_state, uint32_t *allow,
                   void *workspace, size_t workspace_bytes, void *stream)
{
    return align_common("dv_align", trans, num_states, offsets, bytes, num_tokens, nullptr, -1, next_state,
                        allow, workspace, workspace_bytes, stream);
}

dv_status dv_align_eos(const int32_t *trans, int32_t num_states, const int32_t *offsets,
                       const uint8_t *bytes, int32_t num_tokens, const uint8_t *accepting,
                       int32_t eos_token, int32_t *next_state, uint32_t *allow, void *workspace,
                       size_t workspace_bytes, void *stream)
{
    if (eos_token < 0) {
        g_error[0] = '\0';
        return fail(DV_ERR_SHAPE, "dv_align_eos: eos_token=%d must be a token id", eos_token);
    }
    return align_common("dv_align_eos", trans, num_states, offsets, bytes, num_tokens, accepting, eos_token,
                        next_state, allow, workspace, workspace_bytes, stream);
}

dv_status dv_validate_vocab(const int32_t *offsets, int32_t num_tokens, int64_t num_bytes, int32_t *first_bad,
                            void *stream)
{
    g_error[0] = '\0';
    const char *name = "dv_validate_vocab";
    if (!offsets || !first_bad)
        return fail(DV_ERR_INVALID_ARG, "%s: offsets and first_bad must be non-NULL", name);
    if (num_tokens < 1 || num_tokens > DV_MAX_TOKENS)
        return fail(DV_ERR_SHAPE, "%s: num_tokens=%d outside [1, %d]", name, num_tokens, DV_MAX_TOKENS);
    if (num_bytes < 0)
        return fail(DV_ERR_SHAPE, "%s: num_bytes=%lld must be >= 0", name, (long long)num_bytes);
    if (overlap(range_of(first_bad, 4), range_of(offsets, ((size_t)num_tokens + 1) * 4)))
        return fail(DV_ERR_ALIAS, "%s: first_bad overlaps offsets", name);
    return hip_status(dv::launch_validate_vocab(offsets, num_tokens, num_bytes, first_bad,
                                                static_cast<hipStream_t>(stream)),
                      "dv_validate_vocab launch");
}

size_t dv_masked_step_workspace_bytes(int32_t batch, int32_t num_tokens)
{
    if (batch < 0 || batch > DV_MAX_BATCH || num_tokens < 1 || num_tokens > DV_MAX_TOKENS)
        return 0;
    return dv::step_workspace_bytes(batch, num_tokens);
}

// How a step call decodes: greedy, greedy with the check first, or sampled.
struct StepMode {
    int kind;  // 0 greedy, 1 opportunistic, 2 sampled, 3 argument checks only
    float inv_temperature;
    uint64_t seed, offset;
};

static dv_status step_common(const char *name, StepMode mode, const int32_t *next_state,
                             const uint32_t *allow, int32_t num_states, int32_t num_tokens, const int32_t *states,
                             const void *logits, int32_t dtype, int32_t batch, int64_t ld_logits, int32_t *token,
                             int32_t *new_state, void *workspace, size_t workspace_bytes, void *stream)
{
    g_error[0] = '\0';
    if (!next_state || !allow)
        return fail(DV_ERR_INVALID_ARG, "%s: next_state and allow must be non-NULL", name);
    if (batch > 0 && (!states || !logits || !token || !new_state))
        return fail(DV_ERR_INVALID_ARG, "%s: states, logits, token and new_state must be "
                                        "non-NULL when batch > 0", name);
    if (num_states < 1 || num_states > DV_MAX_STATES)
        return fail(DV_ERR_SHAPE, "%s: num_states=%d outside [1, %d]", name, num_states, DV_MAX_STATES);
    if (num_tokens < 1 || num_tokens > DV_MAX_TOKENS)
        return fail(DV_ERR_SHAPE, "%s: num_tokens=%d outside [1, %d]", name, num_tokens, DV_MAX_TOKENS);
    if (batch < 0 || batch > DV_MAX_BATCH)
        return fail(DV_ERR_SHAPE, "%s: batch=%d outside [0, %d]", name, batch, DV_MAX_BATCH);
    if (ld_logits < num_tokens || ld_logits > ((int64_t)1 << 40))
        return fail(DV_ERR_SHAPE, "%s: ld_logits=%lld must be >= num_tokens=%d", name,
                    (long long)ld_logits, num_tokens);
    if (dtype != DV_F32 && dtype != DV_BF16)
        return fail(DV_ERR_DTYPE, "%s: unknown dtype %d", name, dtype);
    if (mode.kind == 2 && !(mode.inv_temperature > 0.0f && mode.inv_temperature <= 3.0e38f))
        return fail(DV_ERR_SHAPE, "%s: inv_temperature=%g must be finite and > 0", name,
                    (double)mode.inv_temperature);
    if (batch == 0)
        return DV_OK;
    const size_t S = (size_t)num_states, V = (size_t)num_tokens, W = (V + 31) / 32, B = (size_t)batch;
    const size_t elt = dtype == DV_F32 ? 4 : 2;
    if (reinterpret_cast<uintptr_t>(logits) % elt)
        return fail(DV_ERR_INVALID_ARG, "%s: logits must be aligned to their element size (%zu bytes)", name, elt);
    const Range r_tok = range_of(token, B * 4), r_new = range_of(new_state, B * 4);
    const Range r_ns = range_of(next_state, S * V * 4), r_al = range_of(allow, S * W * 4);
    const Range r_st = range_of(states, B * 4);
    const Range r_lg = range_of(logits, ((B - 1) * (size_t)ld_logits + V) * elt);
    if (overlap(r_tok, r_new))
        return fail(DV_ERR_ALIAS, "%s: token and new_state overlap", name);
    for (Range out : {r_tok, r_new})
        if (overlap(out, r_ns) || overlap(out, r_al) || overlap(out, r_st) || overlap(out, r_lg))
            return fail(DV_ERR_ALIAS, "%s: an output overlaps an input "
                                      "(ping-pong two state buffers instead of updating in place)", name);
    if (mode.kind == 3)
        return DV_OK;  // argument checks only (the scratch-backed step checks before its set-up)
    const size_t need = mode.kind == 2 ? dv::sample_workspace_bytes(batch, num_tokens)
                                       : dv::step_workspace_bytes(batch, num_tokens);
    if (!workspace || workspace_bytes < need)
        return fail(DV_ERR_WORKSPACE, "%s: workspace of %zu bytes given, %zu needed", name, workspace_bytes,
                    need);
    if (reinterpret_cast<uintptr_t>(workspace) & 255)
        return fail(DV_ERR_WORKSPACE, "%s: workspace must be 256-byte aligned", name);
    const Range r_ws = range_of(workspace, need);
    for (Range r : {r_tok, r_new, r_ns, r_al, r_st, r_lg})
        if (overlap(r_ws, r))
            return fail(DV_ERR_ALIAS, "%s: workspace overlaps an input or output", name);
    const hipStream_t st = static_cast<hipStream_t>(stream);
    hipError_t e;
    if (mode.kind == 2)
        e = dv::launch_masked_sample(next_state, allow, num_states, num_tokens, states, logits, dtype, batch,
                                     ld_logits, mode.inv_temperature, mode.seed, mode.offset, token, new_state,
                                     workspace, st);
    else if (mode.kind == 1)
        e = dv::launch_masked_step_opportunistic(next_state, allow, num_states, num_tokens, states, logits, dtype,
                                                 batch, ld_logits, token, new_state, workspace, st);
    else
        e = dv::launch_masked_step(next_state, allow, num_states, num_tokens, states, logits, dtype, batch,
                                   ld_logits, token, new_state, workspace, st);
    return hip_status(e, "launch");
}

dv_status dv_masked_step(const int32_t *next_state, const uint32_t *allow, int32_t num_states,
                         int32_t num_tokens, const int32_t *states, const void *logits, int32_t dtype,
                         int32_t batch, int64_t ld_logits, int32_t *token, int32_t *new_state,
                         void *workspace, size_t workspace_bytes, void *stream)
{
    return step_common("dv_masked_step", StepMode{0, 1.0f, 0, 0}, next_state, allow, num_states, num_tokens, states, logits,
                       dtype, batch, ld_logits, token, new_state, workspace, workspace_bytes, stream);
}

// ------------------------------------------------ step without allocation
//
// dv_masked_step_noalloc meets split rows in `scratch`, a device array of
// the library, instead of a caller's workspace.  Its size covers
// DV_NOALLOC_MAX_BATCH rows that meet through a maximum and a count (12
// bytes a row); rows that meet in pairs need up to 24 bytes a row, but from
// 256 rows on only vocabularies beyond 516,096 tokens need more than 12, and
// the workspace check below refuses any call the array would not cover.
// Each GPU holds its own copy until the process ends.  Host code never uses
// the array's name as an address: the device address of each GPU's copy is
// looked up once per device and kept in g_scratch_ptr.
namespace {

constexpr size_t kScratchBytes = dv::row_meet_bytes(DV_NOALLOC_MAX_BATCH);
__device__ __align__(256) uint4 scratch[kScratchBytes / sizeof(uint4)];

constexpr int kMaxScratchDevices = 64;
std::atomic<void *> g_scratch_ptr[kMaxScratchDevices];
std::mutex g_scratch_mu;

__global__ void clear_scratch_kernel(uint4 *p, size_t n)
{
    for (size_t i = (size_t)blockIdx.x * blockDim.x + threadIdx.x; i < n; i += (size_t)gridDim.x * blockDim.x)
        p[i] = make_uint4(0, 0, 0, 0);
}

// The current device's scratch address; on a device's first call, looked up
// and cleared with a kernel on `stream` (a kernel, not a memset, so that a
// first call under graph capture records a plain kernel node).
dv_status scratch_for_current_device(const char *name, hipStream_t stream, void **out)
{
    int dev = -1;
    hipError_t e = hipGetDevice(&dev);
    if (e != hipSuccess)
        return fail(DV_ERR_HIP, "%s: hipGetDevice: %s", name, hipGetErrorString(e));
    if (dev < 0 || dev >= kMaxScratchDevices)
        return fail(DV_ERR_HIP, "%s: device %d beyond the %d devices the scratch table covers", name, dev,
                    kMaxScratchDevices);
    void *p = g_scratch_ptr[dev].load(std::memory_order_acquire);
    if (p) {
        *out = p;
        return DV_OK;
    }
    std::lock_guard<std::mutex> lock(g_scratch_mu);
    p = g_scratch_ptr[dev].load(std::memory_order_acquire);
    if (!p) {
        e = hipGetSymbolAddress(&p, HIP_SYMBOL(scratch));
        if (e != hipSuccess || !p)
            return fail(DV_ERR_HIP, "%s: hipGetSymbolAddress(scratch): %s", name, hipGetErrorString(e));
        const size_t n = kScratchBytes / sizeof(uint4);
        clear_scratch_kernel<<<(unsigned)((n + 255) / 256), 256, 0, stream>>>(static_cast<uint4 *>(p), n);
        e = hipGetLastError();
        if (e != hipSuccess)
            return fail(DV_ERR_HIP, "%s: clearing the scratch array: %s", name, hipGetErrorString(e));
        g_scratch_ptr[dev].store(p, std::memory_order_release);
    }
    *out = p;
    return DV_OK;
}

}  // namespace

dv_status dv_masked_step_noalloc(const int32_t *next_state, const uint32_t *allow, int32_t num_states,
                                 int32_t num_tokens, const int32_t *states, const void *logits, int32_t dtype,
                                 int32_t batch, int64_t ld_logits, int32_t *token, int32_t *new_state,
                                 void *stream)
{
    const char *name = "dv_masked_step_noalloc";
    g_error[0] = '\0';
    if (batch > DV_NOALLOC_MAX_BATCH)
        return fail(DV_ERR_SHAPE, "%s: batch=%d exceeds DV_NOALLOC_MAX_BATCH=%d (the scratch array's size); "
                                  "use dv_masked_step with a workspace", name, batch, DV_NOALLOC_MAX_BATCH);
    // The same checks as dv_masked_step, with a stand-in workspace address
    // (never dereferenced: a failed check enqueues nothing) so that no HIP
    // call happens before the arguments are known good.
    const dv_status pre = step_common(name, StepMode{3, 1.0f, 0, 0}, next_state, allow, num_states, num_tokens,
                                      states, logits, dtype, batch, ld_logits, token, new_state, nullptr, 0,
                                      stream);
    if (pre != DV_OK || batch == 0)
        return pre;
    void *ws = nullptr;
    const dv_status got = scratch_for_current_device(name, static_cast<hipStream_t>(stream), &ws);
    if (got != DV_OK)
        return got;
    return step_common(name, StepMode{0, 1.0f, 0, 0}, next_state, allow, num_states, num_tokens, states, logits,
                       dtype, batch, ld_logits, token, new_state, ws, kScratchBytes, stream);
}

dv_status dv_masked_step_opportunistic(const int32_t *next_state, const uint32_t *allow, int32_t num_states,
                                       int32_t num_tokens, const int32_t *states, const void *logits,
                                       int32_t dtype, int32_t batch, int64_t ld_logits, int32_t *token,
                                       int32_t *new_state, void *workspace, size_t workspace_bytes,
                                       void *stream)
{
    return step_common("dv_masked_step_opportunistic", StepMode{1, 1.0f, 0, 0}, next_state, allow, num_states, num_tokens, states,
                       logits, dtype, batch, ld_logits, token, new_state, workspace, workspace_bytes, stream);
}

size_t dv_masked_sample_workspace_bytes(int32_t batch, int32_t num_tokens)
{
    if (batch < 0 || batch > DV_MAX_BATCH || num_tokens < 1 || num_tokens > DV_MAX_TOKENS)
        return 0;
    return dv::sample_workspace_bytes(batch, num_tokens);
}

dv_status dv_masked_sample(const int32_t *next_state, const uint32_t *allow, int32_t num_states, int32_t num_tokens,
                           const int32_t *states, const void *logits, int32_t dtype, int32_t batch,
                           int64_t ld_logits, float inv_temperature, uint64_t seed, uint64_t offset,
                           int32_t *token, int32_t *new_state, void *workspace, size_t workspace_bytes,
                           void *stream)
{
    return step_common("dv_masked_sample", StepMode{2, inv_temperature, seed, offset}, next_state, allow,
                       num_states, num_tokens, states, logits, dtype, batch, ld_logits, token, new_state, workspace,
                       workspace_bytes, stream);
}

static dv_status spec_shape_checks(const char *name, int32_t num_states, int32_t num_tokens, int32_t batch,
                                   int32_t num_proposed, int64_t ld_proposals)
{
    if (num_states < 1 || num_states > DV_MAX_STATES)
        return fail(DV_ERR_SHAPE, "%s: num_states=%d outside [1, %d]", name, num_states, DV_MAX_STATES);
    if (num_tokens < 1 || num_tokens > DV_MAX_TOKENS)
        return fail(DV_ERR_SHAPE, "%s: num_tokens=%d outside [1, %d]", name, num_tokens, DV_MAX_TOKENS);
    if (batch < 0 || batch > DV_MAX_BATCH)
        return fail(DV_ERR_SHAPE, "%s: batch=%d outside [0, %d]", name, batch, DV_MAX_BATCH);
    if (num_proposed < 0 || num_proposed > DV_MAX_PROPOSED)
        return fail(DV_ERR_SHAPE, "%s: num_proposed=%d outside [0, %d]", name, num_proposed, DV_MAX_PROPOSED);
    if ((int64_t)batch * (num_proposed + 1) > DV_MAX_BATCH)
        return fail(DV_ERR_SHAPE, "%s: batch * (num_proposed + 1) = %lld exceeds %d", name,
                    (long long)batch * (num_proposed + 1), DV_MAX_BATCH);
    if (num_proposed > 0 && (ld_proposals < num_proposed || ld_proposals > ((int64_t)1 << 40)))
        return fail(DV_ERR_SHAPE, "%s: ld_proposals=%lld must be >= num_proposed=%d", name,
                    (long long)ld_proposals, num_proposed);
    return DV_OK;
}

dv_status dv_spec_walk(const int32_t *next_state, const uint32_t *allow, int32_t num_states, int32_t num_tokens,
                       const int32_t *states, const int32_t *proposals, int32_t num_proposed,
                       int64_t ld_proposals, int32_t batch, int32_t *accepted, int32_t *final_state, void *stream)
{
    g_error[0] = '\0';
    const char *name = "dv_spec_walk";
    if (!next_state || !allow)
        return fail(DV_ERR_INVALID_ARG, "%s: next_state and allow must be non-NULL", name);
    if (batch > 0 && (!states || !accepted || !final_state || (num_proposed > 0 && !proposals)))
        return fail(DV_ERR_INVALID_ARG, "%s: states, proposals, accepted and final_state must be non-NULL "
                                        "when batch > 0", name);
    const dv_status st = spec_shape_checks(name, num_states, num_tokens, batch, num_proposed, ld_proposals);
    if (st != DV_OK)
        return st;
    if (batch == 0)
        return DV_OK;
    const size_t S = (size_t)num_states, V = (size_t)num_tokens, W = (V + 31) / 32, B = (size_t)batch;
    const size_t np = (size_t)num_proposed;
    const Range r_acc = range_of(accepted, B * 4), r_fin = range_of(final_state, B * 4);
    const Range r_ns = range_of(next_state, S * V * 4), r_al = range_of(allow, S * W * 4);
    const Range r_st = range_of(states, B * 4);
    const Range r_pr = range_of(proposals, np ? ((B - 1) * (size_t)ld_proposals + np) * 4 : 0);
    if (overlap(r_acc, r_fin))
        return fail(DV_ERR_ALIAS, "%s: accepted and final_state overlap", name);
    for (Range out : {r_acc, r_fin})
        if (overlap(out, r_ns) || overlap(out, r_al) || overlap(out, r_st) || overlap(out, r_pr))
            return fail(DV_ERR_ALIAS, "%s: an output overlaps an input", name);
    return hip_status(dv::launch_spec_walk(next_state, allow, num_states, num_tokens, states, proposals,
                                           num_proposed, num_proposed ? ld_proposals : 0, batch, accepted,
                                           final_state, static_cast<hipStream_t>(stream)),
                      "dv_spec_walk launch");
}

size_t dv_spec_verify_workspace_bytes(int32_t batch, int32_t num_proposed, int32_t num_tokens)
{
    if (batch < 0 || batch > DV_MAX_BATCH || num_proposed < 0 || num_proposed > DV_MAX_PROPOSED ||
        (int64_t)batch * (num_proposed + 1) > DV_MAX_BATCH || num_tokens < 1 || num_tokens > DV_MAX_TOKENS)
        return 0;
    return dv::spec_workspace_bytes(batch, num_proposed, num_tokens);
}

dv_status dv_spec_verify(const int32_t *next_state, const uint32_t *allow, int32_t num_states,
                         int32_t num_tokens, const int32_t *states, const int32_t *proposals,
                         int32_t num_proposed, int64_t ld_proposals, const void *logits, int32_t dtype,
                         int64_t ld_row, int64_t ld_pos, int32_t batch, int32_t *token, int32_t *accepted,
                         int32_t *new_state, void *workspace, size_t workspace_bytes, void *stream)
{
    g_error[0] = '\0';
    const char *name = "dv_spec_verify";
    if (!next_state || !allow)
        return fail(DV_ERR_INVALID_ARG, "%s: next_state and allow must be non-NULL", name);
    if (batch > 0 && (!states || !logits || !token || !accepted || !new_state || (num_proposed > 0 && !proposals)))
        return fail(DV_ERR_INVALID_ARG, "%s: states, proposals, logits, token, accepted and new_state must be "
                                        "non-NULL when batch > 0", name);
    dv_status st = spec_shape_checks(name, num_states, num_tokens, batch, num_proposed, ld_proposals);
    if (st != DV_OK)
        return st;
    const int64_t kMaxStride = (int64_t)1 << 40;
    if (ld_row < 0 || ld_row > kMaxStride || ld_pos < 0 || ld_pos > kMaxStride)
        return fail(DV_ERR_SHAPE, "%s: ld_row=%lld and ld_pos=%lld must be in [0, 2^40]", name,
                    (long long)ld_row, (long long)ld_pos);
    if (dtype != DV_F32 && dtype != DV_BF16)
        return fail(DV_ERR_DTYPE, "%s: unknown dtype %d", name, dtype);
    if (batch == 0)
        return DV_OK;
    const size_t S = (size_t)num_states, V = (size_t)num_tokens, W = (V + 31) / 32, B = (size_t)batch;
    const size_t np = (size_t)num_proposed, P = np + 1;
    const size_t elt = dtype == DV_F32 ? 4 : 2;
    if (reinterpret_cast<uintptr_t>(logits) % elt)
        return fail(DV_ERR_INVALID_ARG, "%s: logits must be aligned to their element size (%zu bytes)", name, elt);
    const Range r_tok = range_of(token, B * P * 4), r_acc = range_of(accepted, B * 4),
                r_new = range_of(new_state, B * 4);
    const Range r_ns = range_of(next_state, S * V * 4), r_al = range_of(allow, S * W * 4);
    const Range r_st = range_of(states, B * 4);
    const Range r_pr = range_of(proposals, np ? ((B - 1) * (size_t)ld_proposals + np) * 4 : 0);
    const Range r_lg = range_of(logits, ((B - 1) * (size_t)ld_row + np * (size_t)ld_pos + V) * elt);
    if (overlap(r_tok, r_acc) || overlap(r_tok, r_new) || overlap(r_acc, r_new))
        return fail(DV_ERR_ALIAS, "%s: token, accepted and new_state overlap", name);
    for (Range out : {r_tok, r_acc, r_new})
        if (overlap(out, r_ns) || overlap(out, r_al) || overlap(out, r_st) || overlap(out, r_pr) ||
            overlap(out, r_lg))
            return fail(DV_ERR_ALIAS, "%s: an output overlaps an input", name);
    const size_t need = dv::spec_workspace_bytes(batch, num_proposed, num_tokens);
    if (!workspace || workspace_bytes < need)
        return fail(DV_ERR_WORKSPACE, "%s: workspace of %zu bytes given, %zu needed", name, workspace_bytes, need);
    if (reinterpret_cast<uintptr_t>(workspace) & 255)
        return fail(DV_ERR_WORKSPACE, "%s: workspace must be 256-byte aligned", name);
    const Range r_ws = range_of(workspace, need);
    for (Range r : {r_tok, r_acc, r_new, r_ns, r_al, r_st, r_pr, r_lg})
        if (overlap(r_ws, r))
            return fail(DV_ERR_ALIAS, "%s: workspace overlaps an input or output", name);
    return hip_status(dv::launch_spec_verify(next_state, allow, num_states, num_tokens, states, proposals,
                                             num_proposed, num_proposed ? ld_proposals : 0, logits, dtype, ld_row,
                                             ld_pos, batch, token, accepted, new_state, workspace,
                                             static_cast<hipStream_t>(stream)),
                      "dv_spec_verify launch");
}

}  // extern "C"

// ---------------------------------------------------------------- training

namespace {

constexpr int64_t kMaxRowStride = (int64_t)1 << 40;

size_t element_size(int32_t dtype) { return dtype == DV_F32 ? 4 : 2; }

// Bytes that `rows` rows of n elements take, ld elements apart.
Range rows_range(const void *p, int64_t rows, int64_t n, int64_t ld, size_t elt)
{
    return range_of(p, p && rows ? ((size_t)(rows - 1) * (size_t)ld + (size_t)n) * elt : 0);
}

struct TrainSizes {
    int32_t rows, num_tokens, dtype;
};

dv_status train_sizes(const char *name, TrainSizes s)
{
    if (s.num_tokens < 1 || s.num_tokens > DV_MAX_TOKENS)
        return fail(DV_ERR_SHAPE, "%s: num_tokens=%d outside [1, %d]", name, s.num_tokens, DV_MAX_TOKENS);
    if (s.rows < 0 || s.rows > DV_MAX_BATCH)
        return fail(DV_ERR_SHAPE, "%s: rows=%d outside [0, %d]", name, s.rows, DV_MAX_BATCH);
    if (s.dtype != DV_F32 && s.dtype != DV_BF16)
        return fail(DV_ERR_DTYPE, "%s: unknown dtype %d", name, s.dtype);
    return DV_OK;
}

dv_status hidden_size(const char *name, int32_t hidden)
{
    if (hidden < 1 || hidden > DV_MAX_HIDDEN)
        return fail(DV_ERR_SHAPE, "%s: hidden=%d outside [1, %d]", name, hidden, DV_MAX_HIDDEN);
    return DV_OK;
}

dv_status row_stride(const char *name, const char *what, int64_t ld, int64_t least)
{
    if (ld < least || ld > kMaxRowStride)
        return fail(DV_ERR_SHAPE, "%s: %s=%lld must be at least %lld", name, what, (long long)ld, (long long)least);
    return DV_OK;
}

dv_status aligned(const char *name, const char *what, const void *p, size_t elt)
{
    if (reinterpret_cast<uintptr_t>(p) % elt)
        return fail(DV_ERR_INVALID_ARG, "%s: %s must be aligned to its element size (%zu bytes)", name, what, elt);
    return DV_OK;
}

// The allowed tokens' arguments: all or none of them (states may be NULL with
// no rows).
dv_status mask_args(const char *name, const uint32_t *allow, int32_t num_states, const int32_t *states, int32_t rows)
{
    if ((allow && !states && rows > 0) || (!allow && states))
        return fail(DV_ERR_INVALID_ARG, "%s: allow and states must be given together", name);
    if (allow && (num_states < 1 || num_states > DV_MAX_STATES))
        return fail(DV_ERR_SHAPE, "%s: num_states=%d outside [1, %d]", name, num_states, DV_MAX_STATES);
    return DV_OK;
}

Range allow_range(const uint32_t *allow, int32_t num_states, int32_t num_tokens)
{
    return range_of(allow, allow ? (size_t)num_states * (((size_t)num_tokens + 31) / 32) * 4 : 0);
}

template <size_t OUT, size_t IN>
dv_status no_overlap(const char *name, const Range (&outs)[OUT], const Range (&ins)[IN])
{
    for (size_t i = 0; i < OUT; ++i) {
        for (size_t j = 0; j < i; ++j)
            if (overlap(outs[i], outs[j]))
                return fail(DV_ERR_ALIAS, "%s: two outputs, or an output and the workspace, overlap", name);
        for (const Range &in : ins)
            if (overlap(outs[i], in))
                return fail(DV_ERR_ALIAS, "%s: an output or the workspace overlaps an input", name);
    }
    return DV_OK;
}

dv_status workspace_args(const char *name, const void *workspace, size_t bytes, size_t need)
{
    if (!workspace || bytes < need)
        return fail(DV_ERR_WORKSPACE, "%s: workspace of %zu bytes given, %zu needed", name, bytes, need);
    if (reinterpret_cast<uintptr_t>(workspace) & 255)
        return fail(DV_ERR_WORKSPACE, "%s: workspace must be 256-byte aligned", name);
    return DV_OK;
}

bool head_sizes_ok(int32_t rows, int32_t hidden, int32_t num_tokens, int32_t dtype)
{
    return rows >= 0 && rows <= DV_MAX_BATCH && hidden >= 1 && hidden <= DV_MAX_HIDDEN && num_tokens >= 1 &&
           num_tokens <= DV_MAX_TOKENS && (dtype == DV_F32 || dtype == DV_BF16);
}

#define DV_CHECK(call)                \
    do {                              \
        const dv_status st_ = (call); \
        if (st_ != DV_OK)             \
            return st_;               \
    } while (0)

// The inputs that both head calls share.
dv_status head_args(const char *name, const void *x, int64_t ld_x, const void *weight, int64_t ld_weight,
                    int32_t dtype, int32_t rows, int32_t hidden, int32_t num_tokens, const int32_t *targets,
                    const uint32_t *allow, int32_t num_states, const int32_t *states)
{
    if (!weight || (rows > 0 && (!x || !targets)))
        return fail(DV_ERR_INVALID_ARG, "%s: weight must be non-NULL, x and targets when rows > 0", name);
    DV_CHECK(train_sizes(name, {rows, num_tokens, dtype}));
    DV_CHECK(hidden_size(name, hidden));
    DV_CHECK(row_stride(name, "ld_x", ld_x, hidden));
    DV_CHECK(row_stride(name, "ld_weight", ld_weight, hidden));
    DV_CHECK(mask_args(name, allow, num_states, states, rows));
    DV_CHECK(aligned(name, "x", x, element_size(dtype)));
    return aligned(name, "weight", weight, element_size(dtype));
}

}  // namespace

extern "C" {

size_t dv_head_loss_workspace_bytes(int32_t rows, int32_t hidden, int32_t num_tokens, int32_t dtype)
{
    return head_sizes_ok(rows, hidden, num_tokens, dtype) ? dv::head_workspace_bytes(rows, hidden, num_tokens, dtype) : 0;
}

size_t dv_head_loss_workspace_bytes_for(const void *x, int64_t ld_x, const void *weight, int64_t ld_weight, int32_t dtype,
                                        int32_t rows, int32_t hidden, int32_t num_tokens)
{
    if (!head_sizes_ok(rows, hidden, num_tokens, dtype))
        return 0;
    return dv::head_workspace_bytes({x, ld_x, weight, ld_weight, dtype, rows, hidden, num_tokens, nullptr, {}});
}

dv_status dv_head_loss(const void *x, int64_t ld_x, const void *weight, int64_t ld_weight, int32_t dtype, int32_t rows,
                       int32_t hidden, int32_t num_tokens, const int32_t *targets, const uint32_t *allow,
                       int32_t num_states, const int32_t *states, float *loss, float *lse, void *workspace,
                       size_t workspace_bytes, void *stream)
{
    g_error[0] = '\0';
    const char *name = "dv_head_loss";
    DV_CHECK(head_args(name, x, ld_x, weight, ld_weight, dtype, rows, hidden, num_tokens, targets, allow, num_states,
                       states));
    if (rows == 0)
        return DV_OK;
    if (!loss || !lse)
        return fail(DV_ERR_INVALID_ARG, "%s: loss and lse must be non-NULL when rows > 0", name);
    const dv::HeadArgs a{x, ld_x, weight, ld_weight, dtype, rows, hidden, num_tokens, targets, {allow, states, num_states}};
    const size_t elt = element_size(dtype), need = dv::head_workspace_bytes(a);
    DV_CHECK(workspace_args(name, workspace, workspace_bytes, need));
    const Range outs[] = {range_of(loss, (size_t)rows * 4), range_of(lse, (size_t)rows * 4), range_of(workspace, need)};
    const Range ins[] = {rows_range(x, rows, hidden, ld_x, elt), rows_range(weight, num_tokens, hidden, ld_weight, elt),
                         range_of(targets, (size_t)rows * 4), allow_range(allow, num_states, num_tokens),
                         range_of(states, states ? (size_t)rows * 4 : 0)};
    DV_CHECK(no_overlap(name, outs, ins));
    return hip_status(dv::launch_head_loss(a, loss, lse, workspace, static_cast<hipStream_t>(stream)),
                      "dv_head_loss launch");
}

size_t dv_head_loss_backward_workspace_bytes(int32_t rows, int32_t hidden, int32_t num_tokens, int32_t dtype)
{
    return head_sizes_ok(rows, hidden, num_tokens, dtype)
               ? dv::head_backward_workspace_bytes(rows, hidden, num_tokens, dtype)
               : 0;
}

size_t dv_head_loss_backward_workspace_bytes_for(const void *x, int64_t ld_x, const void *weight, int64_t ld_weight,
                                                 int32_t dtype, int32_t rows, int32_t hidden, int32_t num_tokens)
{
    if (!head_sizes_ok(rows, hidden, num_tokens, dtype))
        return 0;
    return dv::head_backward_workspace_bytes({x, ld_x, weight, ld_weight, dtype, rows, hidden, num_tokens, nullptr, {}});
}

dv_status dv_head_loss_backward(const void *x, int64_t ld_x, const void *weight, int64_t ld_weight, int32_t dtype,
                                int32_t rows, int32_t hidden, int32_t num_tokens, const int32_t *targets,
                                const uint32_t *allow, int32_t num_states, const int32_t *states, const float *lse,
                                const float *grad_loss, void *grad_x, void *grad_weight, void *workspace,
                                size_t workspace_bytes, void *stream)
{
    g_error[0] = '\0';
    const char *name = "dv_head_loss_backward";
    DV_CHECK(head_args(name, x, ld_x, weight, ld_weight, dtype, rows, hidden, num_tokens, targets, allow, num_states,
                       states));
    if (rows > 0 && (!lse || !grad_loss))
        return fail(DV_ERR_INVALID_ARG, "%s: lse and grad_loss must be non-NULL when rows > 0", name);
    if (!grad_weight && (rows == 0 || !grad_x))
        return rows == 0 ? DV_OK : fail(DV_ERR_INVALID_ARG, "%s: grad_x or grad_weight must be non-NULL", name);
    const size_t elt = element_size(dtype);
    DV_CHECK(aligned(name, "grad_x", grad_x, elt));
    DV_CHECK(aligned(name, "grad_weight", grad_weight, elt));
    const dv::HeadArgs a{x, ld_x, weight, ld_weight, dtype, rows, hidden, num_tokens, targets, {allow, states, num_states}};
    const size_t need = dv::head_backward_workspace_bytes(a);
    DV_CHECK(workspace_args(name, workspace, workspace_bytes, need));
    const Range outs[] = {rows_range(grad_x, rows, hidden, hidden, elt),
                          rows_range(grad_weight, num_tokens, hidden, hidden, elt), range_of(workspace, need)};
    const Range ins[] = {rows_range(x, rows, hidden, ld_x, elt), rows_range(weight, num_tokens, hidden, ld_weight, elt),
                         range_of(targets, (size_t)rows * 4), allow_range(allow, num_states, num_tokens),
                         range_of(states, states ? (size_t)rows * 4 : 0), range_of(lse, (size_t)rows * 4),
                         range_of(grad_loss, (size_t)rows * 4)};
    DV_CHECK(no_overlap(name, outs, ins));
    return hip_status(dv::launch_head_loss_backward(a, lse, grad_loss, grad_x, grad_weight, workspace,
                                                    static_cast<hipStream_t>(stream)),
                      "dv_head_loss_backward launch");
}

size_t dv_distill_loss_workspace_bytes(int32_t rows, int32_t num_tokens, int32_t num_top)
{
    if (rows < 0 || rows > DV_MAX_BATCH || num_tokens < 1 || num_tokens > DV_MAX_TOKENS || num_top < 1 ||
        num_top > DV_MAX_TOP)
        return 0;
    return dv::distill_workspace_bytes(rows, num_tokens, num_top);
}

namespace {

// The kernels take powers of two: inv_temperature log2(e) has to be finite.
constexpr float kMaxInvTemperature = 2.3e38f;

// Both distillation calls; `grad_wanted`: the backward one.
dv_status distill_common(const char *name, bool grad_wanted, const void *logits, int64_t ld_logits, int32_t dtype,
                         int32_t rows, int32_t num_tokens, const int32_t *teacher_ids, const float *teacher_logits,
                         int32_t num_top, float inv_temperature, const uint32_t *allow, int32_t num_states,
                         const int32_t *states, const float *grad_loss, float *loss, void *grad, int64_t ld_grad,
                         void *workspace, size_t workspace_bytes, void *stream)
{
    g_error[0] = '\0';
    if (rows > 0 && (!logits || !teacher_ids || !teacher_logits))
        return fail(DV_ERR_INVALID_ARG, "%s: logits, teacher_ids and teacher_logits must be non-NULL when rows > 0", name);
    DV_CHECK(train_sizes(name, {rows, num_tokens, dtype}));
    if (num_top < 1 || num_top > DV_MAX_TOP)
        return fail(DV_ERR_SHAPE, "%s: num_top=%d outside [1, %d]", name, num_top, DV_MAX_TOP);
    if (!(inv_temperature > 0.0f && inv_temperature <= kMaxInvTemperature))
        return fail(DV_ERR_SHAPE, "%s: inv_temperature=%g must be > 0 and at most %g", name, (double)inv_temperature,
                    (double)kMaxInvTemperature);
    DV_CHECK(row_stride(name, "ld_logits", ld_logits, num_tokens));
    if (grad_wanted)
        DV_CHECK(row_stride(name, "ld_grad", ld_grad, num_tokens));
    DV_CHECK(mask_args(name, allow, num_states, states, rows));
    const size_t elt = element_size(dtype);
    DV_CHECK(aligned(name, "logits", logits, elt));
    if (rows == 0)
        return DV_OK;
    if (grad_wanted ? !grad || !grad_loss : !loss)
        return fail(DV_ERR_INVALID_ARG, "%s: %s must be non-NULL when rows > 0", name,
                    grad_wanted ? "grad and grad_loss" : "loss");
    DV_CHECK(aligned(name, "grad", grad, elt));
    const size_t need = dv::distill_workspace_bytes(rows, num_tokens, num_top);
    DV_CHECK(workspace_args(name, workspace, workspace_bytes, need));
    const size_t entries = (size_t)rows * (size_t)num_top * 4;
    const Range r_logits = rows_range(logits, rows, num_tokens, ld_logits, elt);
    const bool in_place = grad == logits && ld_grad == ld_logits;
    const Range outs[] = {range_of(loss, loss ? (size_t)rows * 4 : 0), rows_range(grad, rows, num_tokens, ld_grad, elt),
                          range_of(workspace, need)};
    const Range ins[] = {in_place ? range_of(nullptr, 0) : r_logits, range_of(teacher_ids, entries),
                         range_of(teacher_logits, entries), allow_range(allow, num_states, num_tokens),
                         range_of(states, states ? (size_t)rows * 4 : 0),
                         range_of(grad_loss, grad_loss ? (size_t)rows * 4 : 0)};
    DV_CHECK(no_overlap(name, outs, ins));
    const dv::DistillArgs a{logits,         ld_logits, dtype,           rows, num_tokens, teacher_ids,
                            teacher_logits, num_top,   inv_temperature, {allow, states, num_states}};
    return hip_status(dv::launch_distill(a, grad_loss, loss, grad, ld_grad, workspace, static_cast<hipStream_t>(stream)),
                      name);
}

}  // namespace

dv_status dv_distill_loss(const void *logits, int64_t ld_logits, int32_t dtype, int32_t rows, int32_t num_tokens,
                          const int32_t *teacher_ids, const float *teacher_logits, int32_t num_top,
                          float inv_temperature, const uint32_t *allow, int32_t num_states, const int32_t *states,
                          float *loss, void *workspace, size_t workspace_bytes, void *stream)
{
    return distill_common("dv_distill_loss", false, logits, ld_logits, dtype, rows, num_tokens, teacher_ids,
                          teacher_logits, num_top, inv_temperature, allow, num_states, states, nullptr, loss, nullptr,
                          0, workspace, workspace_bytes, stream);
}

dv_status dv_distill_loss_backward(const void *logits, int64_t ld_logits, int32_t dtype, int32_t rows,
                                   int32_t num_tokens, const int32_t *teacher_ids, const float *teacher_logits,
                                   int32_t num_top, float inv_temperature, const uint32_t *allow, int32_t num_states,
                                   const int32_t *states, const float *grad_loss, float *loss, void *grad,
                                   int64_t ld_grad, void *workspace, size_t workspace_bytes, void *stream)
{
    return distill_common("dv_distill_loss_backward", true, logits, ld_logits, dtype, rows, num_tokens, teacher_ids,
                          teacher_logits, num_top, inv_temperature, allow, num_states, states, grad_loss, loss, grad,
                          ld_grad, workspace, workspace_bytes, stream);
}

namespace {

dv_status embed_args(const char *name, int32_t dtype, int32_t num_tokens, int32_t hidden, int32_t rows, float scale,
                     const char *stride_name, int64_t ld)
{
    DV_CHECK(train_sizes(name, {rows, num_tokens, dtype}));
    DV_CHECK(hidden_size(name, hidden));
    DV_CHECK(row_stride(name, stride_name, ld, hidden));
    if (!(scale >= -3.0e38f && scale <= 3.0e38f))
        return fail(DV_ERR_SHAPE, "%s: scale=%g must be finite", name, (double)scale);
    return DV_OK;
}

}  // namespace

dv_status dv_embed(const void *weight, int64_t ld_weight, int32_t dtype, int32_t num_tokens, int32_t hidden,
                   const int32_t *ids, int32_t rows, float scale, void *out, void *stream)
{
    g_error[0] = '\0';
    const char *name = "dv_embed";
    if (!weight || (rows > 0 && (!ids || !out)))
        return fail(DV_ERR_INVALID_ARG, "%s: weight must be non-NULL, ids and out when rows > 0", name);
    DV_CHECK(embed_args(name, dtype, num_tokens, hidden, rows, scale, "ld_weight", ld_weight));
    const size_t elt = element_size(dtype);
    DV_CHECK(aligned(name, "weight", weight, elt));
    DV_CHECK(aligned(name, "out", out, elt));
    if (rows == 0)
        return DV_OK;
    const Range outs[] = {rows_range(out, rows, hidden, hidden, elt)};
    const Range ins[] = {rows_range(weight, num_tokens, hidden, ld_weight, elt), range_of(ids, (size_t)rows * 4)};
    DV_CHECK(no_overlap(name, outs, ins));
    return hip_status(dv::launch_embed(weight, ld_weight, dtype, num_tokens, hidden, ids, rows, scale, out,
                                       static_cast<hipStream_t>(stream)),
                      "dv_embed launch");
}

size_t dv_embed_backward_workspace_bytes(int32_t rows, int32_t hidden, int32_t num_tokens)
{
    if (!head_sizes_ok(rows, hidden, num_tokens, DV_F32))
        return 0;
    return dv::embed_backward_workspace_bytes(rows, hidden, num_tokens);
}

dv_status dv_embed_backward(const void *grad_out, int64_t ld_grad_out, int32_t dtype, int32_t rows, int32_t hidden,
                            const int32_t *ids, int32_t num_tokens, float scale, int32_t accumulate, void *grad_weight,
                            void *workspace, size_t workspace_bytes, void *stream)
{
    g_error[0] = '\0';
    const char *name = "dv_embed_backward";
    if (!grad_weight || (rows > 0 && (!grad_out || !ids)))
        return fail(DV_ERR_INVALID_ARG, "%s: grad_weight must be non-NULL, grad_out and ids when rows > 0", name);
    DV_CHECK(embed_args(name, dtype, num_tokens, hidden, rows, scale, "ld_grad_out", ld_grad_out));
    const size_t elt = element_size(dtype);
    DV_CHECK(aligned(name, "grad_out", grad_out, elt));
    DV_CHECK(aligned(name, "grad_weight", grad_weight, elt));
    const size_t need = dv::embed_backward_workspace_bytes(rows, hidden, num_tokens);
    DV_CHECK(workspace_args(name, workspace, workspace_bytes, need));
    const Range outs[] = {rows_range(grad_weight, num_tokens, hidden, hidden, elt), range_of(workspace, need)};
    const Range ins[] = {rows_range(grad_out, rows, hidden, ld_grad_out, elt), range_of(ids, (size_t)rows * 4)};
    DV_CHECK(no_overlap(name, outs, ins));
    if (rows == 0 && accumulate)
        return DV_OK;
    return hip_status(dv::launch_embed_backward(grad_out, ld_grad_out, dtype, rows, hidden, ids, num_tokens, scale,
                                                accumulate != 0, grad_weight, workspace,
                                                static_cast<hipStream_t>(stream)),
                      "dv_embed_backward launch");
}

namespace {

dv_status rows_args(const char *name, int32_t rows, int32_t hidden, int32_t dtype)
{
    DV_CHECK(train_sizes(name, {rows, 1, dtype}));
    return hidden_size(name, hidden);
}

}  // namespace

dv_status dv_rms_norm(const void *x, int64_t ld_x, const void *residual, int64_t ld_residual, const void *weight,
                      int32_t dtype, int32_t rows, int32_t hidden, float eps, void *total, void *out, float *rstd, void *q,
                      float *scales, void *stream)
{
    g_error[0] = '\0';
    const char *name = "dv_rms_norm";
    if (!weight || (rows > 0 && !x))
        return fail(DV_ERR_INVALID_ARG, "%s: weight must be non-NULL, x when rows > 0", name);
    if (!q != !scales)
        return fail(DV_ERR_INVALID_ARG, "%s: q and scales must be given together", name);
    DV_CHECK(rows_args(name, rows, hidden, dtype));
    DV_CHECK(row_stride(name, "ld_x", ld_x, hidden));
    if (residual)
        DV_CHECK(row_stride(name, "ld_residual", ld_residual, hidden));
    if (!(eps >= 0.f && eps <= 3.0e38f))
        return fail(DV_ERR_SHAPE, "%s: eps=%g must be >= 0 and finite", name, (double)eps);
    const size_t elt = element_size(dtype);
    DV_CHECK(aligned(name, "x", x, elt));
    DV_CHECK(aligned(name, "residual", residual, elt));
    DV_CHECK(aligned(name, "weight", weight, elt));
    DV_CHECK(aligned(name, "total", total, elt));
    DV_CHECK(aligned(name, "out", out, elt));
    DV_CHECK(aligned(name, "rstd", rstd, 4));
    DV_CHECK(aligned(name, "q", q, 8));
    DV_CHECK(aligned(name, "scales", scales, 4));
    if (rows == 0)
        return DV_OK;
    if (!out && !q)
        return fail(DV_ERR_INVALID_ARG, "%s: out or q must be non-NULL when rows > 0", name);
    const size_t depth = (size_t)dv::up_block(hidden), n = (size_t)rows;
    const bool over_x = total && total == x && (ld_x == hidden || rows == 1);
    const bool over_residual = total && total == residual && (ld_residual == hidden || rows == 1);
    const Range none = range_of(nullptr, 0), r_total = rows_range(total, rows, hidden, hidden, elt);
    const Range outs[] = {rows_range(out, rows, hidden, hidden, elt), range_of(rstd, rstd ? n * 4 : 0),
                          range_of(q, q ? n * depth : 0), range_of(scales, scales ? depth / 128 * n * 4 : 0), r_total};
    const Range r_x = rows_range(x, rows, hidden, ld_x, elt), r_res = rows_range(residual, rows, hidden, ld_residual, elt);
    const Range ins[] = {range_of(weight, (size_t)hidden * elt)};
    DV_CHECK(no_overlap(name, outs, ins));
    for (const Range &o : outs) {
        const bool is_total = &o == &outs[4];
        if (overlap(o, is_total && over_x ? none : r_x) || overlap(o, is_total && over_residual ? none : r_res))
            return fail(DV_ERR_ALIAS, "%s: an output overlaps an input", name);
    }
    const dv::NormArgs a{x,    ld_x, residual, ld_residual, weight, dtype, rows, hidden, eps, total, out, rstd,
                         static_cast<uint8_t *>(q), scales};
    return hip_status(dv::launch_rms_norm(a, static_cast<hipStream_t>(stream)), "dv_rms_norm launch");
}

size_t dv_rms_norm_backward_workspace_bytes(int32_t rows, int32_t hidden)
{
    return head_sizes_ok(rows, hidden, 1, DV_F32) ? dv::rms_norm_backward_workspace_bytes(rows, hidden) : 0;
}

dv_status dv_rms_norm_backward(const void *grad_out, int64_t ld_grad_out, const void *total, int64_t ld_total,
                               const void *weight, const float *rstd, const void *grad_total, int64_t ld_grad_total,
                               int32_t dtype, int32_t rows, int32_t hidden, void *grad_x, void *grad_weight,
                               void *workspace, size_t workspace_bytes, void *stream)
{
    g_error[0] = '\0';
    const char *name = "dv_rms_norm_backward";
    if (!weight || (rows > 0 && (!grad_out || !total || !rstd)))
        return fail(DV_ERR_INVALID_ARG, "%s: weight must be non-NULL, grad_out, total and rstd when rows > 0", name);
    DV_CHECK(rows_args(name, rows, hidden, dtype));
    DV_CHECK(row_stride(name, "ld_grad_out", ld_grad_out, hidden));
    DV_CHECK(row_stride(name, "ld_total", ld_total, hidden));
    if (grad_total)
        DV_CHECK(row_stride(name, "ld_grad_total", ld_grad_total, hidden));
    if (!grad_weight && (rows == 0 || !grad_x))
        return rows == 0 ? DV_OK : fail(DV_ERR_INVALID_ARG, "%s: grad_x or grad_weight must be non-NULL", name);
    const size_t elt = element_size(dtype);
    DV_CHECK(aligned(name, "grad_out", grad_out, elt));
    DV_CHECK(aligned(name, "total", total, elt));
    DV_CHECK(aligned(name, "weight", weight, elt));
    DV_CHECK(aligned(name, "rstd", rstd, 4));
    DV_CHECK(aligned(name, "grad_total", grad_total, elt));
    DV_CHECK(aligned(name, "grad_x", grad_x, elt));
    DV_CHECK(aligned(name, "grad_weight", grad_weight, elt));
    const size_t need = dv::rms_norm_backward_workspace_bytes(rows, hidden);
    DV_CHECK(workspace_args(name, workspace, workspace_bytes, need));
    const Range outs[] = {rows_range(grad_x, rows, hidden, hidden, elt),
                          range_of(grad_weight, grad_weight ? (size_t)hidden * elt : 0), range_of(workspace, need)};
    const Range ins[] = {rows_range(grad_out, rows, hidden, ld_grad_out, elt), rows_range(total, rows, hidden, ld_total, elt),
                         range_of(weight, (size_t)hidden * elt), range_of(rstd, (size_t)rows * 4),
                         rows_range(grad_total, rows, hidden, ld_grad_total, elt)};
    DV_CHECK(no_overlap(name, outs, ins));
    const dv::NormGradArgs a{grad_out, ld_grad_out, total, ld_total, weight, rstd, grad_total, ld_grad_total,
                             dtype,    rows,        hidden, rows > 0 ? grad_x : nullptr, grad_weight};
    return hip_status(dv::launch_rms_norm_backward(a, workspace, static_cast<hipStream_t>(stream)),
                      "dv_rms_norm_backward launch");
}

namespace {

// By rows or by tiles.
dv_status tile_arg(const char *name, int32_t tile)
{
    if (tile != 1 && tile != DV_SCALE_BLOCK)
        return fail(DV_ERR_SHAPE, "%s: tile=%d must be 1 or %d", name, tile, DV_SCALE_BLOCK);
    return DV_OK;
}

// Bytes of the scales of an 8-bit operand.
size_t scale_bytes(int64_t n, int64_t depth, int32_t tile)
{
    return (size_t)(tile == 1 ? n : dv::up_block(n) / DV_SCALE_BLOCK) * (size_t)(depth / DV_SCALE_BLOCK) * 4;
}

}  // namespace

dv_status dv_quantize_f8(const void *x, int64_t ld_x, int32_t dtype, int32_t rows, int32_t cols, int32_t tile, void *q,
                         float *scales, void *t_q, float *t_scales, void *stream)
{
    g_error[0] = '\0';
    const char *name = "dv_quantize_f8";
    if (rows > 0 && !x)
        return fail(DV_ERR_INVALID_ARG, "%s: x must be non-NULL when rows > 0", name);
    if (!q != !scales || !t_q != !t_scales)
        return fail(DV_ERR_INVALID_ARG, "%s: q and scales, t_q and t_scales must be given together", name);
    DV_CHECK(train_sizes(name, {0, cols, dtype}));
    if (rows < 0 || rows > DV_MAX_TOKENS)
        return fail(DV_ERR_SHAPE, "%s: rows=%d outside [0, %d]", name, rows, DV_MAX_TOKENS);
    DV_CHECK(tile_arg(name, tile));
    DV_CHECK(row_stride(name, "ld_x", ld_x, cols));
    const int64_t depth = dv::up_block(cols), t_depth = dv::up_block(rows);
    if ((depth / 128) * (t_depth / 128) >= (int64_t)1 << 24)
        return fail(DV_ERR_SHAPE, "%s: %d x %d has 2^24 tiles or more", name, rows, cols);
    DV_CHECK(aligned(name, "x", x, element_size(dtype)));
    DV_CHECK(aligned(name, "q", q, 16));
    DV_CHECK(aligned(name, "t_q", t_q, 16));
    DV_CHECK(aligned(name, "scales", scales, 4));
    DV_CHECK(aligned(name, "t_scales", t_scales, 4));
    if (rows == 0)
        return DV_OK;
    if (!q && !t_q)
        return fail(DV_ERR_INVALID_ARG, "%s: q or t_q must be non-NULL when rows > 0", name);
    const Range outs[] = {range_of(q, q ? (size_t)rows * (size_t)depth : 0), range_of(scales, scales ? scale_bytes(rows, depth, tile) : 0),
                          range_of(t_q, t_q ? (size_t)cols * (size_t)t_depth : 0),
                          range_of(t_scales, t_scales ? scale_bytes(cols, t_depth, tile) : 0)};
    const Range ins[] = {rows_range(x, rows, cols, ld_x, element_size(dtype))};
    DV_CHECK(no_overlap(name, outs, ins));
    const dv::QuantizeArgs a{x, ld_x, dtype, rows, cols, tile != 1, static_cast<uint8_t *>(q), scales,
                             static_cast<uint8_t *>(t_q), t_scales};
    return hip_status(dv::launch_quantize_f8(a, static_cast<hipStream_t>(stream)), "dv_quantize_f8 launch");
}

namespace {

bool product_sizes_ok(int32_t rows, int32_t cols, int32_t depth)
{
    return rows >= 0 && rows <= DV_MAX_TOKENS && cols >= 1 && cols <= DV_MAX_TOKENS && depth >= DV_SCALE_BLOCK &&
           depth <= DV_MAX_DEPTH && depth % DV_SCALE_BLOCK == 0 && (int64_t)rows * cols < (int64_t)1 << 36;
}

}  // namespace

size_t dv_product_f8_workspace_bytes(int32_t rows, int32_t cols, int32_t depth)
{
    return product_sizes_ok(rows, cols, depth) ? dv::product_f8_workspace_bytes(rows, cols, depth) : 0;
}

size_t dv_product_f8_workspace_bytes_up_to(int32_t rows, int32_t cols, int32_t depth)
{
    return product_sizes_ok(rows, cols, depth) ? dv::product_f8_workspace_bytes_up_to(rows, cols, depth) : 0;
}

dv_status dv_product_f8(const void *a, int64_t ld_a, const float *a_scales, const void *b, int64_t ld_b,
                        const float *b_scales, int32_t tile, int32_t rows, int32_t cols, int32_t depth, int32_t dtype,
                        void *out, int64_t ld_out, void *workspace, size_t workspace_bytes, void *stream)
{
    g_error[0] = '\0';
    const char *name = "dv_product_f8";
    if (!b || !b_scales || (rows > 0 && (!a || !a_scales || !out)))
        return fail(DV_ERR_INVALID_ARG, "%s: b and b_scales must be non-NULL, a, a_scales and out when rows > 0", name);
    const bool exact = dtype >= 0 && (dtype & DV_EXACT_SUMS);
    if (exact)
        dtype -= DV_EXACT_SUMS;
    DV_CHECK(train_sizes(name, {0, 1, dtype}));
    DV_CHECK(tile_arg(name, tile));
    if (!product_sizes_ok(rows, cols, depth))
        return fail(DV_ERR_SHAPE, "%s: rows=%d in [0, %d], cols=%d in [1, %d], fewer than 2^36 results, depth=%d a multiple of 128 in [128, %d]",
                    name, rows, DV_MAX_TOKENS, cols, DV_MAX_TOKENS, depth, DV_MAX_DEPTH);
    DV_CHECK(row_stride(name, "ld_a", ld_a, depth));
    DV_CHECK(row_stride(name, "ld_b", ld_b, depth));
    if (ld_a % 16 || ld_b % 16 || ld_a > DV_MAX_DEPTH || ld_b > DV_MAX_DEPTH)
        return fail(DV_ERR_SHAPE, "%s: ld_a=%lld and ld_b=%lld must be multiples of 16 and at most %d", name, (long long)ld_a,
                    (long long)ld_b, DV_MAX_DEPTH);
    DV_CHECK(row_stride(name, "ld_out", ld_out, cols));
    const size_t elt = element_size(dtype);
    DV_CHECK(aligned(name, "a", a, 16));
    DV_CHECK(aligned(name, "b", b, 16));
    DV_CHECK(aligned(name, "a_scales", a_scales, 4));
    DV_CHECK(aligned(name, "b_scales", b_scales, 4));
    DV_CHECK(aligned(name, "out", out, elt));
    if (rows == 0)
        return DV_OK;
    const size_t need = dv::product_f8_workspace_bytes(rows, cols, depth);
    if (need)
        DV_CHECK(workspace_args(name, workspace, workspace_bytes, need));
    const Range outs[] = {rows_range(out, rows, cols, ld_out, elt), range_of(workspace, need)};
    const Range ins[] = {rows_range(a, rows, depth, ld_a, 1), rows_range(b, cols, depth, ld_b, 1),
                         range_of(a_scales, scale_bytes(rows, depth, 1)), range_of(b_scales, scale_bytes(cols, depth, tile))};
    DV_CHECK(no_overlap(name, outs, ins));
    const dv::ProductArgs p{static_cast<const uint8_t *>(a), ld_a, a_scales, static_cast<const uint8_t *>(b), ld_b, b_scales,
                            tile != 1, rows, cols, depth, dtype, exact, out, ld_out};
    return hip_status(dv::launch_product_f8(p, workspace, static_cast<hipStream_t>(stream)), "dv_product_f8 launch");
}

dv_status dv_adjust_logits(const void *logits, int64_t ld_logits, int32_t dtype, int32_t rows, int32_t num_tokens,
                           const int32_t *history, int64_t ld_history, int32_t max_history, const int32_t *lengths,
                           const int32_t *prompt_lengths, const float *repetition, const float *presence,
                           const float *frequency, const int32_t *bias_ids, const float *bias, int32_t num_bias,
                           const uint32_t *allow, int32_t num_states, const int32_t *states, void *out, int64_t ld_out,
                           void *stream)
{
    g_error[0] = '\0';
    const char *name = "dv_adjust_logits";
    if (rows > 0 && (!logits || !out))
        return fail(DV_ERR_INVALID_ARG, "%s: logits and out must be non-NULL when rows > 0", name);
    DV_CHECK(train_sizes(name, {rows, num_tokens, dtype}));
    if (max_history < 0 || max_history > DV_MAX_HISTORY)
        return fail(DV_ERR_SHAPE, "%s: max_history=%d outside [0, %d]", name, max_history, DV_MAX_HISTORY);
    if (num_bias < 0 || num_bias > DV_MAX_BIAS)
        return fail(DV_ERR_SHAPE, "%s: num_bias=%d outside [0, %d]", name, num_bias, DV_MAX_BIAS);
    if (rows > 0 && max_history > 0 && (!history || !lengths))
        return fail(DV_ERR_INVALID_ARG, "%s: history and lengths must be non-NULL with max_history > 0", name);
    if (rows > 0 && num_bias > 0 && (!bias_ids || !bias))
        return fail(DV_ERR_INVALID_ARG, "%s: bias_ids and bias must be non-NULL with num_bias > 0", name);
    if (max_history > 0)
        DV_CHECK(row_stride(name, "ld_history", ld_history, max_history));
    DV_CHECK(row_stride(name, "ld_logits", ld_logits, num_tokens));
    DV_CHECK(row_stride(name, "ld_out", ld_out, num_tokens));
    if ((int64_t)rows * (((int64_t)num_tokens + 4095) / 4096) >= (int64_t)1 << 24)
        return fail(DV_ERR_SHAPE, "%s: %d rows of %d tokens are too many", name, rows, num_tokens);
    DV_CHECK(mask_args(name, allow, num_states, states, rows));
    const size_t elt = element_size(dtype), n = (size_t)rows;
    DV_CHECK(aligned(name, "logits", logits, elt));
    DV_CHECK(aligned(name, "out", out, elt));
    const struct {
        const char *name;
        const void *p;
    } words[] = {{"history", history},       {"lengths", lengths},     {"prompt_lengths", prompt_lengths},
                 {"repetition", repetition}, {"presence", presence},   {"frequency", frequency},
                 {"bias_ids", bias_ids},     {"bias", bias},           {"allow", allow},
                 {"states", states}};
    for (const auto &w : words)
        DV_CHECK(aligned(name, w.name, w.p, 4));
    if (rows == 0)
        return DV_OK;
    const bool in_place = out == logits && (ld_out == ld_logits || rows == 1);
    const Range outs[] = {rows_range(out, rows, num_tokens, ld_out, elt)};
    const Range ins[] = {in_place ? range_of(nullptr, 0) : rows_range(logits, rows, num_tokens, ld_logits, elt),
                         max_history ? rows_range(history, rows, max_history, ld_history, 4) : range_of(nullptr, 0),
                         range_of(lengths, max_history ? n * 4 : 0), range_of(prompt_lengths, prompt_lengths ? n * 4 : 0),
                         range_of(repetition, repetition ? n * 4 : 0), range_of(presence, presence ? n * 4 : 0),
                         range_of(frequency, frequency ? n * 4 : 0), range_of(bias_ids, n * (size_t)num_bias * 4),
                         range_of(bias, n * (size_t)num_bias * 4), allow_range(allow, num_states, num_tokens),
                         range_of(states, states ? n * 4 : 0)};
    DV_CHECK(no_overlap(name, outs, ins));
    const dv::AdjustArgs a{logits,     ld_logits,  dtype,     rows,     num_tokens, max_history ? history : nullptr,
                           ld_history, max_history, lengths,  prompt_lengths, repetition, presence,
                           frequency,  bias_ids,   bias,      num_bias, {allow, states, num_states}, out, ld_out};
    return hip_status(dv::launch_adjust_logits(a, static_cast<hipStream_t>(stream)), "dv_adjust_logits launch");
}

}  // extern "C"
