// What the entry points of the other translation units share with tir_api.hip: error reports and the workspace a caller registered.
#pragma once
#include <hip/hip_runtime.h>
#include <memory>
#include <mutex>
#include "tir.h"

namespace tir {

// Records the message for tir_last_error and returns st.
tir_status host_error(tir_status st, const char* fmt, ...) __attribute__((format(printf, 2, 3)));

// The workspace registered for `stream` of the current device (tir_set_workspace): partial sums and zeroed arrival counters.  partial is
// null where there is none: what needs it runs unsplit then.  While the object lives, no other thread's call launches anything that uses this workspace: an operator may be several launches that
// pass results through it.
struct StreamWorkspace {
    void* partial;
    unsigned* count;
    int64_t bytes, counters;
    std::shared_ptr<std::mutex> mutex;
    std::unique_lock<std::mutex> turn;
};
StreamWorkspace stream_workspace(hipStream_t stream);

inline bool host_aligned(const void* p, uintptr_t a) { return ((uintptr_t)p % a) == 0; }

constexpr int64_t kMax31 = 2147483647LL;

// A launch's extent along x is counted in work items, in 32 bits.
inline bool grid_fits(int64_t groups, int64_t threads) { return groups <= 0xffffffffll / threads; }
// What a launcher that checks this returns, as the caller's error.
inline tir_status launch_error(const char* who, hipError_t e) {
    if (e == hipErrorInvalidConfiguration) return host_error(TIR_ERR_UNSUPPORTED, "%s: more workgroups than one launch can have", who);
    return host_error(TIR_ERR_LAUNCH, "%s: launch failed: %s", who, hipGetErrorString(e));
}

// Strides of rows that the decoder's attentions read or write 16 bytes at a time.
inline tir_status check_row_strides(const char* who, const char* what, int64_t bs, int64_t rs, int64_t hs) {
    if (bs < 0 || rs < 0 || hs < 0) return host_error(TIR_ERR_INVALID_ARG, "%s: negative stride of %s", who, what);
    if ((bs | rs | hs) & 7) return host_error(TIR_ERR_ALIGNMENT, "%s: the strides of %s must be multiples of 8 elements", who, what);
    // (a chunk of 64 rows is addressed with 31 bits, whole tensors with 64)
    if (bs > (1ll << 40) || hs > (1ll << 40) || rs > (1ll << 23)) return host_error(TIR_ERR_UNSUPPORTED, "%s: a stride of %s is beyond 2^23 (rows) or 2^40 elements", who, what);
    return TIR_OK;
}

// The kernels multiply by scale * log2(e), which has to be finite too.
inline tir_status check_scale(const char* who, float scale) {
    if (!(scale <= 0x1p127f && scale >= -0x1p127f)) return host_error(TIR_ERR_INVALID_ARG, "%s: scale must be finite and at most 2^127 in magnitude", who);
    return TIR_OK;
}

// Extents of the attention over another sequence's states, forward and backward.
inline tir_status check_cross(const char* who, int64_t batch, int64_t M, int64_t N, int64_t Hq, int64_t Hkv, int64_t d, float scale) {
    if (batch < 0 || M < 0 || N < 0 || Hq < 0 || Hkv < 1 || d < 0)
        return host_error(TIR_ERR_INVALID_ARG, "%s: negative extent or no key head (batch=%lld M=%lld N=%lld Hq=%lld Hkv=%lld d=%lld)", who, (long long)batch, (long long)M, (long long)N, (long long)Hq, (long long)Hkv, (long long)d);
    if (d != 64 && d != 128) return host_error(TIR_ERR_UNSUPPORTED, "%s: head dimension %lld (64 and 128 are compiled)", who, (long long)d);
    const tir_status st = check_scale(who, scale);
    if (st != TIR_OK) return st;
    if (Hq % Hkv) return host_error(TIR_ERR_INVALID_ARG, "%s: %lld key heads do not divide %lld query heads", who, (long long)Hkv, (long long)Hq);
    if (batch > kMax31 || M > kMax31 || N > kMax31 - 65535 || Hq > kMax31) return host_error(TIR_ERR_UNSUPPORTED, "extent beyond 2^31-1");
    if (batch == 0 || Hq == 0) return TIR_OK;
    // rows of a key head, and tiles of 32 rows resp. keys of all of them
    if (M > (kMax31 - 512) / (Hq / Hkv) || batch > kMax31 / Hkv || batch * Hkv > kMax31 / ((M * (Hq / Hkv) + 31) / 32 + 1) || batch * Hkv > kMax31 / ((N + 31) / 32 + 1))
        return host_error(TIR_ERR_UNSUPPORTED, "%s: too many tiles of queries or keys", who);
    return TIR_OK;
}

}  // namespace tir
