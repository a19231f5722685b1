// What the two files behind hps_seq.h share.  Not part of the C ABI, and not exported.
#ifndef HPS_SEQ_COMMON_H
#define HPS_SEQ_COMMON_H

#include <hip/hip_runtime.h>

#include <cstdint>

#include "hps_seq.h"

// Stores the message of hps_seq_last_error() (no allocation, so nothing can be thrown) and returns `code`.
__attribute__((visibility("hidden"))) hps_status_t hps_seq_fail(hps_status_t code, const char *what, const char *more = "");

#define SEQ_TRY(expr)                                                                                                          \
    do {                                                                                                                       \
        hipError_t e_ = (expr);                                                                                                \
        if (e_ != hipSuccess)                                                                                                  \
            return hps_seq_fail(e_ == hipErrorOutOfMemory ? HPS_ERR_OOM : HPS_ERR_DEVICE, #expr ": ", hipGetErrorString(e_));  \
    } while (0)

#define SEQ_REQUIRE(cond, msg)                                      \
    do {                                                            \
        if (!(cond)) return hps_seq_fail(HPS_ERR_INVALID_ARG, msg); \
    } while (0)

// A launch has room for fewer than 2^32 threads.  launch(first, n) is called for each stretch of up to 2^23 work-groups, of up to 256 threads.
template <typename F> hipError_t seq_launches(uint64_t groups, F launch) {
    constexpr uint64_t kMost = 1ull << 23;             // a multiple of 8: the XCDs are dealt to as in one launch
    for (uint64_t first = 0; first < groups; first += kMost) {
        launch((uint32_t)first, (uint32_t)(groups - first < kMost ? groups - first : kMost));
        if (hipError_t e = hipGetLastError()) return e;
    }
    return hipSuccess;
}

inline bool seq_aligned(const void *p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }
inline bool seq_words(const void *p) { return p && seq_aligned(p, 4); }                  // an int32 array that is there
inline bool seq_block_size(uint32_t b) { return b != 0 && (b & (b - 1)) == 0 && b <= HPS_SEQ_MAX_BLOCK; }

#endif  // HPS_SEQ_COMMON_H
