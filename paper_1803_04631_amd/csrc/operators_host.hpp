// What the operators' sources share on the host: refusals, launches, types, and what is checked of rows.
#pragma once
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "../../include/mlda.h"
#include "host_errors.hpp"
#include "vec_io.hpp"

namespace {

using mlda::Bf16;
using mlda::Fp16;
using mlda::set_error;

int refuse(const char* why) { return set_error(MLDA_EINVAL, why); }

int launched(const char* what) {
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? MLDA_OK : set_error(MLDA_EHIP, what, hipGetErrorString(e));
}

constexpr int32_t kMostCols = 1 << 30;        // columns and words are 32-bit in the kernels, with room for a tile past the end
constexpr int kCus = 256;
constexpr int64_t kMostGroups = 1 << 20;      // of a launch, which has fewer than 2^32 threads: what is beyond is taken in turn

bool known_type(int32_t t) { return t == MLDA_FP32 || t == MLDA_BF16 || t == MLDA_FP16; }
size_t type_bytes(int32_t t) { return t == MLDA_FP32 ? 4 : 2; }
bool aligned(const void* p, size_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

// Whether a call that reads and writes so many bytes leaves them out of the caches (256 MB on the way to memory): what is written then
// does not push out what is still to be read.  Below, the next call finds the results there.  The gradient of 1,024 x 102,000 bf16 logits 97 us,
// written past the caches 72, with the loss 122 and 109; layer norm's gradients of 30,011 x 1,537 bf16 75 and 62; but layer norm of 300,000 x 1,000
// 247 and 253; the gradient of 1,000 x 5,000 fp32, 40 MB in all, 15 either way.
bool passes_caches(double bytes) { return bytes > 192e6; }

// f(tag) for the type; the type is known.
template <class F>
int with_type(int32_t type, F&& f) {
    switch (type) {
    case MLDA_FP32: return f(float());
    case MLDA_BF16: return f(Bf16());
    default: return f(Fp16());
    }
}

int check_rows(const void* p, int64_t stride, int64_t rows, int64_t cols, int32_t type, const char* null, const char* bad) {
    if (!p) return refuse(null);
    if ((rows > 1 && stride < cols) || !aligned(p, type_bytes(type))) return refuse(bad);
    return MLDA_OK;
}

#define RC_TRY(expr)                    \
    do {                                \
        const int rc_ = (expr);         \
        if (rc_ != MLDA_OK) return rc_; \
    } while (0)

}  // namespace
