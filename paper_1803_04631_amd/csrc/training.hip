// What training steps need besides: dropout, and the policy loss.  Argument checks and launches; the kernels are in kernels_dropout.hpp and
// kernels_policy.hpp.
#include "operators_host.hpp"

#include <math.h>

#include "kernels_dropout.hpp"
#include "kernels_policy.hpp"

namespace {

// How the words of a policy loss are dealt out: one workgroup and one launch for few, neighbouring four to a thread beyond.
struct PolicyForm {
    int threads, each;
    unsigned groups;
};
PolicyForm policy_form(int64_t n) {
    if (n <= 4096) return {1024, n <= 1024 ? 1 : 4, 1};
    return {256, 4, (unsigned)std::min<int64_t>((n + 1023) / 1024, mlda::kPolicyGroups)};
}
constexpr size_t kPolicyBytes = (size_t)mlda::kPolicyGroups * 3 * 8;

bool overlap(const void* p, int64_t p_bytes, const void* q, int64_t q_bytes) {
    const char *const a = static_cast<const char*>(p), *const b = static_cast<const char*>(q);
    return p_bytes > 0 && q_bytes > 0 && a < b + q_bytes && b < a + p_bytes;
}

int check_tokens(int64_t n) {
    return n < 0 || n >= ((int64_t)1 << 31) ? refuse("policy loss: need 0 <= n_tokens < 2^31") : MLDA_OK;
}

}  // namespace

extern "C" {

int mlda_dropout(const void* x, int64_t x_stride, const void* residual, int64_t residual_stride, void* y, int64_t y_stride, int64_t rows,
                 int32_t cols, double p, uint64_t seed, uint32_t step, const int64_t* dev_step, int64_t first_row, int32_t type,
                 void* hip_stream) {
    if (rows < 0 || cols < 1 || cols > kMostCols) return refuse("dropout: need rows >= 0 and 1 <= cols <= 2^30");
    if (!known_type(type)) return refuse("dropout: unknown type");
    if (!(p >= 0.0 && p <= 1.0)) return refuse("dropout: need 0 <= p <= 1");
    if (first_row < 0 || first_row > ((int64_t)1 << 32) || rows > ((int64_t)1 << 32) - first_row)
        return refuse("dropout: need 0 <= first_row and first_row + rows <= 2^32");
    if (!aligned(dev_step, 8)) return refuse("dropout: dev_step is not aligned to its type");
    if (rows == 0) return MLDA_OK;
    RC_TRY(check_rows(x, x_stride, rows, cols, type, "dropout: x is null", "dropout: rows of x overlap or are not aligned to their type"));
    RC_TRY(check_rows(y, y_stride, rows, cols, type, "dropout: y is null", "dropout: rows of y overlap or are not aligned to their type"));
    if (residual) RC_TRY(check_rows(residual, residual_stride, rows, cols, type, "", "dropout: rows of residual overlap or are not aligned to their type"));
    if (((x == y && x_stride != y_stride) || (residual == y && residual_stride != y_stride)) && rows > 1)
        return refuse("dropout: y in the place of an input has its stride");
    const int64_t bytes = (int64_t)type_bytes(type), per_row = ((int64_t)cols + mlda::kDropCols - 1) / mlda::kDropCols;
    const int64_t most = std::max<int64_t>(1, ((int64_t)1 << 30) / per_row);
    const uint64_t threshold = (uint64_t)(p * 4294967296.0 + 0.5);
    const float scale = p < 1.0 ? (float)(1.0 / (1.0 - p)) : 0.0f;
    for (int64_t row = 0; row < rows; row += most) {
        const int64_t n = std::min(most, rows - row);
        const mlda::DropoutArgs a{static_cast<const char*>(x) + row * x_stride * bytes, x_stride,
                                  residual ? static_cast<const char*>(residual) + row * residual_stride * bytes : nullptr, residual_stride,
                                  static_cast<char*>(y) + row * y_stride * bytes, y_stride, (uint32_t)(n * per_row), cols,
                                  mlda::divisor((uint32_t)per_row), threshold, scale, (uint32_t)seed, (uint32_t)(seed >> 32), step,
                                  (uint32_t)(first_row + row), dev_step, passes_caches((residual ? 3.0 : 2.0) * rows * cols * bytes)};
        const dim3 grid((unsigned)((n * per_row + mlda::kDropThreads - 1) / mlda::kDropThreads));
        RC_TRY(with_type(type, [&](auto t) {
            typedef decltype(t) T;
            if (residual) hipLaunchKernelGGL((mlda::dropout_kernel<T, true>), grid, dim3(mlda::kDropThreads), 0, (hipStream_t)hip_stream, a);
            else hipLaunchKernelGGL((mlda::dropout_kernel<T, false>), grid, dim3(mlda::kDropThreads), 0, (hipStream_t)hip_stream, a);
            return launched("dropout_kernel");
        }));
    }
    return MLDA_OK;
}

int mlda_policy_loss_workspace_bytes(int64_t n_tokens, size_t* bytes) {
    if (!bytes) return refuse("bytes is null");
    RC_TRY(check_tokens(n_tokens));
    *bytes = policy_form(n_tokens).groups > 1 ? kPolicyBytes : 0;
    return MLDA_OK;
}

int mlda_policy_loss(const float* logprobs, const float* old_logprobs, const float* reference, const float* advantages, const float* weights,
                     const int64_t* row_ptr, int64_t rows, int64_t n_tokens, double low, double high, double kl, float* sums,
                     float* grad_logprobs, void* dev_workspace, size_t workspace_bytes, void* hip_stream) {
    RC_TRY(check_tokens(n_tokens));
    if (rows < 0 || (!row_ptr && rows != n_tokens)) return refuse("policy loss: need rows >= 0, and without row_ptr as many as words");
    if (!(low >= 0.0 && low <= 1.0) || !(high >= 0.0)) return refuse("policy loss: need 0 <= low <= 1 and high >= 0");
    if (!(fabs(kl) <= 3.4e38)) return refuse("policy loss: kl must be finite");
    if (kl != 0.0 && !reference && n_tokens > 0) return refuse("policy loss: a KL term needs the reference");
    if (!sums) return refuse("policy loss: sums are null");
    if (n_tokens > 0 && (!logprobs || !old_logprobs || !grad_logprobs || (rows > 0 && !advantages)))
        return refuse("policy loss: logprobs, old_logprobs, advantages or grad_logprobs are null");
    if (!aligned(logprobs, 4) || !aligned(old_logprobs, 4) || !aligned(reference, 4) || !aligned(advantages, 4) || !aligned(weights, 4) ||
        !aligned(row_ptr, 8) || !aligned(sums, 4) || !aligned(grad_logprobs, 4))
        return refuse("policy loss: an argument is not aligned to its type");
    const PolicyForm form = policy_form(n_tokens);
    const unsigned groups = form.groups;
    if (groups > 1) {
        if (!dev_workspace || !aligned(dev_workspace, 8)) return refuse("policy loss: the workspace is null or not aligned");
        if (workspace_bytes < kPolicyBytes)
            return set_error(MLDA_ENOMEM, "policy loss: the workspace is smaller than mlda_policy_loss_workspace_bytes");
    }
    // (a row's advantage is read for other words' gradients too, and its bounds)
    if (row_ptr && (overlap(grad_logprobs, n_tokens * 4, advantages, rows * 4) || overlap(grad_logprobs, n_tokens * 4, row_ptr, (rows + 1) * 8)))
        return refuse("policy loss: grad_logprobs cannot be in the place of rows' advantages or of row_ptr");
    const mlda::PolicyArgs a{logprobs, old_logprobs, reference, advantages, weights, row_ptr, rows, n_tokens, log1p(-low), log1p(high),
                             1.0 - low, 1.0 + high, kl, n_tokens ? 1.0 / (double)n_tokens : 0.0, grad_logprobs,
                             groups > 1 ? nullptr : sums, static_cast<double*>(dev_workspace),
                             passes_caches((double)n_tokens * (12 + (reference ? 4 : 0) + (row_ptr ? 0 : 4) + (weights ? 4 : 0)))};
    const hipStream_t stream = (hipStream_t)hip_stream;
    auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(groups), dim3(form.threads), 0, stream, a); };
    auto of = [&](auto with_reference) {
        constexpr bool kReference = decltype(with_reference)::value;
        if (form.threads == 1024) launch(form.each == 1 ? mlda::policy_kernel<1024, 1, kReference> : mlda::policy_kernel<1024, 4, kReference>);
        else launch(mlda::policy_kernel<256, 4, kReference>);
    };
    if (reference) of(std::true_type());
    else of(std::false_type());
    RC_TRY(launched("policy_kernel"));
    if (groups == 1) return MLDA_OK;
    hipLaunchKernelGGL(mlda::policy_sums_kernel, dim3(3), dim3(mlda::kPolicySumThreads), 0, stream, a.partial, (int32_t)groups, sums);
    return launched("policy_sums_kernel");
}

}  // extern "C"
