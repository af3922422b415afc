// What the host sides of the student's operators share: checks of arguments, messages, the parts of a workspace.
#pragma once

#include <hip/hip_runtime.h>

#include <algorithm>
#include <atomic>
#include <cstdarg>
#include <cstdint>
#include <cstdio>
#include <numeric>
#include <string>

#include "dynlp_train.h"

namespace dynlp {

std::string& thread_error();  // what dynlp_last_error(NULL) returns; dynlp.hip

// Learning from a teacher's first classes with a head of up to DYNLP_MAX_CLASSES classes, arguments checked (dynlp_train.hip).
struct Teacher;
void distill_few_classes(const dynlp_matrix& h, const dynlp_matrix& weight, const float* bias, const Teacher& teacher, float grad_scale, float* loss,
                         const dynlp_matrix* dh, const dynlp_matrix* dweight, float* dbias, const dynlp_call* call);
int64_t distill_few_classes_workspace(int64_t rows, int32_t dim, int32_t classes, int32_t type);

namespace {

inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
inline int64_t round_up(int64_t a, int64_t b) { return ceil_div(a, b) * b; }

__attribute__((format(printf, 2, 3))) dynlp_status fail(dynlp_status status, const char* format, ...) {
    char text[256];
    va_list args;
    va_start(args, format);
    std::vsnprintf(text, sizeof text, format, args);
    va_end(args);
    try {
        thread_error() = text;
    } catch (...) {  // no memory for the message
    }
    return status;
}

#define REFUSE(...) return fail(DYNLP_ERR_INVALID_ARG, __VA_ARGS__)

dynlp_status launched() {
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? DYNLP_OK : fail(DYNLP_ERR_DEVICE, "kernel launch failed: %s", hipGetErrorString(e));
}

constexpr int64_t kMostRows = 0x7ffffffe;
constexpr int32_t kMostDim = 1 << 28;  // 32 bits hold the bytes of a row

int type_size(int32_t type) { return type == DYNLP_FLOAT32 ? 4 : 2; }

dynlp_status check_matrix(const dynlp_matrix* m, const char* name) {
    if (!m) REFUSE("%s is NULL", name);
    if (m->type < DYNLP_FLOAT32 || m->type > DYNLP_FLOAT16) REFUSE("%s: type %d is not a dynlp_type", name, m->type);
    if (m->rows < 0 || m->rows > kMostRows) REFUSE("%s: %lld rows", name, (long long)m->rows);
    if (m->dim < 1 || m->dim > kMostDim) REFUSE("%s: rows of %d elements", name, m->dim);
    if (m->stride < m->dim) REFUSE("%s: stride %lld is less than the %d elements of a row", name, (long long)m->stride, m->dim);
    if (m->stride > (int64_t(1) << 40)) REFUSE("%s: stride %lld", name, (long long)m->stride);
    if (m->rows > 0 && !m->data) REFUSE("%s: data is NULL", name);
    if (reinterpret_cast<uintptr_t>(m->data) % type_size(m->type)) REFUSE("%s: data is not aligned to its elements", name);
    return DYNLP_OK;
}

#define CHECK(call)                            \
    do {                                       \
        const dynlp_status s_ = (call);        \
        if (s_ != DYNLP_OK) return s_;         \
    } while (0)

dynlp_status check_workspace(const dynlp_call* call, int64_t bytes) {
    if (!call) REFUSE("call is NULL");
    if (bytes > 0 && (!call->workspace || call->workspace_bytes < bytes))
        REFUSE("workspace of %lld bytes: %lld are needed", (long long)(call->workspace ? call->workspace_bytes : 0), (long long)bytes);
    if (bytes > 0 && reinterpret_cast<uintptr_t>(call->workspace) % 256) REFUSE("workspace is not aligned to 256 bytes");
    return DYNLP_OK;
}

// Whether rows of a and rows of b share memory.  Rows of two matrices may take turns in one array; where their strides differ, matrices whose rows
// would meet if there were enough of them count as overlapping.
bool overlap(const dynlp_matrix& a, const dynlp_matrix& b) {
    using wide = __int128;  // rows times stride
    if (a.rows == 0 || b.rows == 0) return false;
    const wide width_a = (wide)a.dim * type_size(a.type), width_b = (wide)b.dim * type_size(b.type);
    wide step_a = (wide)a.stride * type_size(a.type), step_b = (wide)b.stride * type_size(b.type);
    const wide behind = (wide) reinterpret_cast<uintptr_t>(b.data) - (wide) reinterpret_cast<uintptr_t>(a.data);
    if (behind >= (a.rows - 1) * step_a + width_a || -behind >= (b.rows - 1) * step_b + width_b) return false;
    if (a.rows == 1) step_a = step_b;
    if (b.rows == 1) step_b = step_a;
    if (step_a != step_b) {
        const wide step = std::gcd((int64_t)step_a, (int64_t)step_b), at = (behind % step + step) % step;
        return at < width_a || at + width_b > step;
    }
    // row i of a and row i + k of b meet where -width_b < behind + k step < width_a
    auto down = [&](wide x) { return (x >= 0 ? x : x - step_a + 1) / step_a; };
    const wide least = -down(width_b - 1 + behind), most = down(width_a - 1 - behind);
    return std::max(least, (wide)(1 - a.rows)) <= std::min(most, (wide)(b.rows - 1));
}

// Hands out the parts of a workspace, or only measures them (base NULL).
struct Carve {
    char* base;
    int64_t used = 0;
    template <typename T>
    T* take(int64_t n) {
        T* p = base ? reinterpret_cast<T*>(base + used) : nullptr;
        used += round_up(n * (int64_t)sizeof(T), 256);
        return p;
    }
};

constexpr int64_t kSharedMemory = 160 * 1024;  // of a CU

// Shared memory beyond 64 KB is to be asked for, once per kernel and device; `done` has a bit per device (those from the 64th on are asked each time).
// bytes: without the kernel's own arrays.
template <typename F>
void allow_shared(F kernel, std::atomic<uint64_t>& done, int64_t bytes = kSharedMemory) {
    int device = 0;
    if (hipGetDevice(&device) != hipSuccess) return;  // the launch will say so
    const uint64_t bit = device < 64 ? uint64_t(1) << device : 0;
    if (done.load(std::memory_order_relaxed) & bit) return;
    if (hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes) == hipSuccess)
        done.fetch_or(bit, std::memory_order_relaxed);
    else
        (void)hipGetLastError();  // the launch will say so
}

}  // namespace
}  // namespace dynlp
