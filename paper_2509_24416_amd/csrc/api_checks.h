// Argument checks and launch bookkeeping shared by the entry points' source
// files (host only).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>
#include <stdlib.h>

#include <atomic>

#include "../../include/clq.h"

namespace clq {
namespace api {

constexpr int64_t kMaxK = 32768;
constexpr int64_t kMaxRows = 2147483647;

inline bool aligned(const void *p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }

inline clq_status check_block(int64_t K, int32_t block) {
    if (block != 32 && block != 64 && block != 128) return CLQ_ERR_BLOCK;
    if (K % block != 0) return CLQ_ERR_BLOCK;
    return CLQ_OK;
}

inline clq_status check_k(int64_t K) {
    if (K < 64 || K > kMaxK || K % 64 != 0) return CLQ_ERR_SHAPE;
    return CLQ_OK;
}

inline clq_status check_rows(int64_t R) {
    if (R < 1 || R > kMaxRows) return CLQ_ERR_SHAPE;
    return CLQ_OK;
}

// Debug knobs (process-wide host state).  CLQ_DEBUG_SYNC starts from the
// CLQ_SYNC environment variable.
inline std::atomic<int> debug_sync{-1};

inline bool sync_mode() {
    int v = debug_sync.load(std::memory_order_relaxed);
    if (v < 0) {
        const char *e = getenv("CLQ_SYNC");
        v = (e != nullptr && e[0] != '\0' && e[0] != '0') ? 1 : 0;
        int expect = -1;
        debug_sync.compare_exchange_strong(expect, v);
        v = debug_sync.load(std::memory_order_relaxed);
    }
    return v != 0;
}

// The status of an enqueued launch; in sync mode the stream is drained first,
// so that a kernel's own failure is reported by the call that launched it.
inline clq_status done(hipStream_t stream, hipError_t e) {
    if (e != hipSuccess) return CLQ_ERR_HIP;
    if (sync_mode()) {
        if (hipStreamSynchronize(stream) != hipSuccess) return CLQ_ERR_HIP;
        if (hipGetLastError() != hipSuccess) return CLQ_ERR_HIP;
    }
    return CLQ_OK;
}

}  // namespace api
}  // namespace clq
