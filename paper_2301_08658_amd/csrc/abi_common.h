// Internal: argument checks and launch timing of the C ABI, shared by its
// translation units (defined in abi.hip).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "errors.h"

namespace atp {
namespace abi {

// A row-major device matrix / a device vector argument (as every call checks them).
atp_status check_matrix(const void* p, int64_t rows, int64_t ld, int64_t cols, const char* name);
atp_status check_vector(const void* p, const char* name);
// Runs launch(arg) on s, with timing events around it when profiling is on.
atp_status run_timed(const char* name, double flops, double bytes, hipStream_t s,
                     hipError_t (*launch)(void*), void* arg);
template <class F>
atp_status run_timed(const char* name, double flops, double bytes, hipStream_t s, F&& launch) {
    return run_timed(name, flops, bytes, s,
                     [](void* f) { return (*static_cast<std::remove_reference_t<F>*>(f))(); },
                     &launch);
}

#define ATP_CHECK(expr)                                   \
    do {                                                  \
        atp_status _s = (expr);                           \
        if (_s != ATP_OK) return _s;                      \
    } while (0)

constexpr int64_t kMaxTokens = 1 << 24;
constexpr int64_t kMaxLd = 1 << 22;

// Bytes [0, extent) that a matrix of these rows takes from its first element.
inline int64_t extent(int64_t rows, int64_t ld, int64_t cols, int64_t size = 2) {
    return rows > 0 ? ((rows - 1) * ld + cols) * size : 0;
}
inline bool share_bytes(const void* a, int64_t na, const void* b, int64_t nb) {
    const uintptr_t a0 = reinterpret_cast<uintptr_t>(a), b0 = reinterpret_cast<uintptr_t>(b);
    return na > 0 && nb > 0 && a0 < b0 + (uintptr_t)nb && b0 < a0 + (uintptr_t)na;
}

inline atp_status check_heads(int64_t kv_heads, int32_t group) {
    if (kv_heads < 1 || group < 1)
        return set_error(ATP_ERR_INVALID_ARGUMENT, "kv_heads %lld and group %d must be positive",
                         (long long)kv_heads, group);
    if (group > ATP_MAX_QUERY_GROUP)
        return set_error(ATP_ERR_UNSUPPORTED, "group %d: at most %d query heads per key head",
                         group, ATP_MAX_QUERY_GROUP);
    if (kv_heads * (group + 2) * 128 > kMaxLd)
        return set_error(ATP_ERR_UNSUPPORTED, "%lld heads of group %d: rows above 4M elements",
                         (long long)kv_heads, group);
    return ATP_OK;
}

inline atp_status check_tokens(int64_t tokens) {
    if (tokens < 0) return set_error(ATP_ERR_INVALID_ARGUMENT, "negative number of tokens");
    if (tokens > kMaxTokens)
        return set_error(ATP_ERR_UNSUPPORTED, "%lld tokens: at most 2^24", (long long)tokens);
    return ATP_OK;
}

// Aligned like every vector; NULL allowed.
inline atp_status check_optional(const void* p, const char* name) {
    return p ? check_vector(p, name) : ATP_OK;
}

inline atp_status check_workspace(const void* ws, size_t have, size_t need) {
    if (need == 0) return ATP_OK;
    ATP_CHECK(check_vector(ws, "workspace"));
    if (have < need)
        return set_error(ATP_ERR_INVALID_ARGUMENT, "workspace of %zu bytes: needs %zu", have, need);
    return ATP_OK;
}

inline const uint16_t* bits(const void* p) { return static_cast<const uint16_t*>(p); }
inline uint16_t* bits(void* p) { return static_cast<uint16_t*>(p); }
inline hipStream_t stream_of(void* s) { return static_cast<hipStream_t>(s); }

}  // namespace abi
}  // namespace atp
