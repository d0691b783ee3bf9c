// What the entry points share: messages of failures, checks of arguments, the workspace's parts, shapes of launches.
#pragma once
#include <hip/hip_runtime.h>
#include <stdarg.h>
#include <stdio.h>
#include <type_traits>
#include "../../include/chicle_train.h"
#include "elements.hpp"
#include "layer_norm.hpp"

namespace chicle_train {

inline thread_local char last_error[256] = "";

inline int fail(int code, const char *format, ...)
{
    va_list args;
    va_start(args, format);
    vsnprintf(last_error, sizeof last_error, format, args);
    va_end(args);
    return code;
}

inline int launched(const char *what)
{
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? CHICLE_OK : fail(CHICLE_EDEVICE, "%s: %s", what, hipGetErrorString(e));
}

#define TRY(...)                               \
    do {                                       \
        const int rc_ = (__VA_ARGS__);         \
        if (rc_ != CHICLE_OK) return rc_;      \
    } while (0)

constexpr size_t ALIGN = 256;

// Hands out parts of the workspace; without one it only adds up.
struct Carver {
    char *base;
    size_t used = 0;
    explicit Carver(void *p) : base((char *)p) {}
    template <typename T> T *take(int64_t count)
    {
        used = (used + ALIGN - 1) / ALIGN * ALIGN;
        T *p = base ? (T *)(base + used) : nullptr;
        used += sizeof(T) * (size_t)count;
        return p;
    }
    size_t total() const { return used + ALIGN; }        // (the workspace itself may begin at any sixteen bytes)
};

inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
inline int64_t round_up(int64_t a, int64_t b) { return ceil_div(a, b) * b; }
inline int size_of(int32_t type) { return type == CHICLE_F32 ? 4 : 2; }
inline bool type_ok(int32_t type) { return type == CHICLE_F32 || type == CHICLE_BF16 || type == CHICLE_F16; }
inline bool placed(const void *p, int size) { return p && (uintptr_t)p % (uintptr_t)size == 0; }

inline int check_workspace(const void *workspace, size_t have, size_t need)
{
    if (have < need) return fail(CHICLE_ENOMEM, "workspace of %zu bytes where %zu are needed", have, need);
    if (need > 0 && !placed(workspace, 16)) return fail(CHICLE_EINVAL, "workspace must be 16-byte aligned");
    return CHICLE_OK;
}

// f(T()) with the element type
template <typename F>
inline int with_type(int32_t type, F f)
{
    return type == CHICLE_F32 ? f(float()) : type == CHICLE_BF16 ? f(bf16()) : f(f16());
}

inline int pow2_at_least(int64_t x, int most)
{
    int p = 1;
    while (p < x && p < most) p <<= 1;
    return p;
}

constexpr int CUS = 256;                                 // compute units

struct RowShape { int lanes, vectors, threads; };        // vectors 0: the row is not held

// Threads of a row and vectors of each: up to `first_values` values to a thread, then up to LN_MOST_THREADS threads, then up to `most_values`.
// With 16 values first, 65,536 x 4096 in 16 bits take 231 us forward and 295 backward, with 8 358 and 363; shorter rows do not care.
inline RowShape row_shape(int64_t d, int vec, int first_values, int most_values)
{
    const int64_t v = ceil_div(d, vec);
    const int most = most_values / vec;
    RowShape s;
    s.vectors = 1;
    s.lanes = pow2_at_least(v, 256);
    while ((int64_t)s.lanes * s.vectors < v && s.vectors < first_values / vec) s.vectors *= 2;
    while ((int64_t)s.lanes * s.vectors < v && s.lanes < LN_MOST_THREADS) s.lanes *= 2;
    while ((int64_t)s.lanes * s.vectors < v && s.vectors < most) s.vectors *= 2;
    if ((int64_t)s.lanes * s.vectors < v) s.vectors = 0;
    s.threads = s.lanes > 256 ? s.lanes : 256;
    return s;
}

// f(first row, rows, workgroups) for all n rows (or columns), `per` to a workgroup: a launch has fewer than 2^32 threads, of which a workgroup here has
// up to 2^10.
template <typename F>
inline int with_rows(int64_t n, int per, F f)
{
    const int64_t most = ((int64_t)1 << 21) * per;
    for (int64_t first = 0; first < n; first += most) {
        const int64_t many = n - first < most ? n - first : most;
        TRY(f(first, many, (unsigned)ceil_div(many, per)));
    }
    return CHICLE_OK;
}

template <typename F>
inline int with_vectors(int vectors, F f)
{
    switch (vectors) {
    case 1: return f(std::integral_constant<int, 1>());
    case 2: return f(std::integral_constant<int, 2>());
    case 4: return f(std::integral_constant<int, 4>());
    case 8: return f(std::integral_constant<int, 8>());
    default: return f(std::integral_constant<int, 0>());
    }
}

template <typename K>
inline int allow_lds(K kernel, int bytes)
{
    const hipError_t e = hipFuncSetAttribute((const void *)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
    return e == hipSuccess ? CHICLE_OK : fail(CHICLE_EDEVICE, "shared memory: %s", hipGetErrorString(e));
}

}  // namespace chicle_train
