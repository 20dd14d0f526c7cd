// Entry points of the operators that train and serve heads: argument checks.
// Declarations and contracts: include/lipcache.h.
#include <cmath>
#include <type_traits>

#include "operators.cuh"

#define LC_API extern "C" __attribute__((visibility("default")))

namespace {

using lc::Error;

template <typename F>
lipcache_status guarded(F&& f) {
  return lc::run_guarded([](void* c) { (*static_cast<typename std::remove_reference<F>::type*>(c))(); }, &f);
}

bool known_type(int32_t t) { return t == LIPCACHE_F32 || t == LIPCACHE_BF16; }

#define LC_ARG(cond, msg) LC_REQUIRE(cond, LIPCACHE_E_INVALID, msg)

bool aligned(const void* p, int type) { return reinterpret_cast<uintptr_t>(p) % lc::ops::elem(type) == 0; }
// of arrays of 32-bit values whatever the operator's type
bool aligned4(const void* p) { return reinterpret_cast<uintptr_t>(p) % 4 == 0; }

void check_adapted_sizes(const lipcache_adapted* p) {
  LC_ARG(p != nullptr, "NULL operator description");
  LC_ARG(known_type(p->type), "unknown tensor type");
  LC_ARG(p->d >= 1 && p->d <= LIPCACHE_MAX_SIDE, "d must be in [1, LIPCACHE_MAX_SIDE]");
  LC_ARG(p->classes >= 1 && p->classes <= LIPCACHE_MAX_SIDE, "classes must be in [1, LIPCACHE_MAX_SIDE]");
  LC_ARG(p->adapters >= 0 && p->adapters <= LIPCACHE_MAX_ADAPTERS, "adapters must be in [0, LIPCACHE_MAX_ADAPTERS]");
  LC_ARG(p->adapters == 0 || (p->rank >= 1 && p->rank <= LIPCACHE_MAX_RANK),
         "rank must be in [1, LIPCACHE_MAX_RANK]");
  LC_ARG(p->reserved == 0, "reserved must be 0");
  LC_ARG(p->tokens >= 0 && p->tokens <= LIPCACHE_MAX_TOKENS, "tokens must be in [0, LIPCACHE_MAX_TOKENS]");
}

void check_workspace(void* ws, int64_t have, size_t need) {
  LC_ARG(have >= 0 && (size_t)have >= need, "the workspace is too small");
  LC_ARG(need == 0 || ws != nullptr, "NULL workspace");
  LC_ARG(reinterpret_cast<uintptr_t>(ws) % 256 == 0, "the workspace must be 256-byte aligned");
}

void check_adapted(const lipcache_adapted* p) {
  check_adapted_sizes(p);
  LC_ARG(p->ldx >= p->d && p->ldw >= p->d, "a row stride is smaller than the row");
  LC_ARG(p->tokens == 0 || (p->x && p->W), "NULL x or W");
  LC_ARG(p->tokens == 0 || p->adapters == 0 || (p->A && p->B && p->adapter), "NULL A, B or adapter");
  LC_ARG(aligned(p->x, p->type) && aligned(p->W, p->type) && aligned(p->A, p->type) && aligned(p->B, p->type) &&
             aligned4(p->adapter) && aligned4(p->scales),
         "a tensor is not aligned to its elements");
}

}  // namespace

LC_API int64_t lipcache_adapted_workspace(const lipcache_adapted* p, int32_t backward) {
  int64_t bytes = -1;
  guarded([&] {
    check_adapted_sizes(p);
    bytes = (int64_t)lc::ops::adapted_bytes(*p, backward != 0);
  });
  return bytes;
}

LC_API lipcache_status lipcache_adapted_logits(const lipcache_adapted* p, const float* bias, void* y, int64_t ldy,
                                               void* workspace, int64_t workspace_bytes, lipcache_stream_t stream) {
  return guarded([&] {
    check_adapted(p);
    if (p->tokens == 0) return;
    LC_ARG(y != nullptr && aligned(y, p->type), "y is NULL or not aligned to its elements");
    LC_ARG(aligned4(bias), "a tensor is not aligned to its elements");
    LC_ARG(ldy >= p->classes, "a row stride is smaller than the row");
    check_workspace(workspace, workspace_bytes, lc::ops::adapted_bytes(*p, false));
    lc::ops::adapted_logits(*p, bias, y, ldy, static_cast<unsigned char*>(workspace), stream);
  });
}

LC_API lipcache_status lipcache_adapted_logits_backward(const lipcache_adapted* p, const void* dy, int64_t lddy,
                                                        void* dx, int64_t lddx, void* dA, void* dB, void* workspace,
                                                        int64_t workspace_bytes, lipcache_stream_t stream) {
  return guarded([&] {
    check_adapted(p);
    LC_ARG(aligned(dy, p->type) && aligned(dx, p->type) && aligned(dA, p->type) && aligned(dB, p->type),
           "a tensor is not aligned to its elements");
    if (p->tokens > 0) {
      LC_ARG(dy != nullptr, "NULL dy");
      LC_ARG(lddy >= p->classes && (dx == nullptr || lddx >= p->d), "a row stride is smaller than the row");
    }
    check_workspace(workspace, workspace_bytes, lc::ops::adapted_bytes(*p, true));
    if (p->tokens == 0) {
      const size_t e = lc::ops::elem(p->type), n = (size_t)p->adapters * p->rank;
      if (dA && p->adapters) LC_CUDA(cudaMemsetAsync(dA, 0, n * p->d * e, stream));
      if (dB && p->adapters) LC_CUDA(cudaMemsetAsync(dB, 0, n * p->classes * e, stream));
      return;
    }
    lc::ops::adapted_backward(*p, dy, lddy, dx, lddx, dA, dB, static_cast<unsigned char*>(workspace), stream);
  });
}

LC_API lipcache_status lipcache_cross_entropy(int32_t type, const void* logits, int64_t ldz, int64_t tokens,
                                              int32_t classes, const int32_t* target, const float* weight, float* loss,
                                              void* dlogits, int64_t ldd, lipcache_stream_t stream) {
  return guarded([&] {
    LC_ARG(known_type(type), "unknown tensor type");
    LC_ARG(tokens >= 0 && tokens <= LIPCACHE_MAX_TOKENS, "tokens must be in [0, LIPCACHE_MAX_TOKENS]");
    LC_ARG(classes >= 1 && classes <= LIPCACHE_MAX_LOSS_CLASSES, "classes must be in [1, LIPCACHE_MAX_LOSS_CLASSES]");
    if (tokens == 0) return;
    LC_ARG(logits != nullptr && target != nullptr, "NULL logits or target");
    LC_ARG(ldz >= classes && (dlogits == nullptr || ldd >= classes), "a row stride is smaller than the row");
    LC_ARG(dlogits != logits || ldd == ldz, "gradients in place need the logits' row stride");
    LC_ARG(aligned(logits, type) && aligned(dlogits, type) && aligned4(target) && aligned4(weight) && aligned4(loss),
           "a tensor is not aligned to its elements");
    if (loss == nullptr && dlogits == nullptr) return;
    lc::ops::cross_entropy(type, logits, ldz, tokens, classes, target, weight, loss, dlogits, ldd, stream);
  });
}

namespace {

void check_ortho_sizes(int32_t type, int64_t batch, int32_t rows, int32_t cols) {
  LC_ARG(known_type(type), "unknown tensor type");
  LC_ARG(batch >= 0 && batch <= 65535, "batch must be in [0, 65535]");
  LC_ARG(rows >= 1 && rows <= LIPCACHE_MAX_SIDE && cols >= 1 && cols <= LIPCACHE_MAX_SIDE,
         "rows and cols must be in [1, LIPCACHE_MAX_SIDE]");
  LC_ARG(rows <= 16384 || cols <= 16384, "the smaller side must be at most 16384");
}

void check_ortho(int32_t steps, const double* coefficients, double eps) {
  LC_ARG(steps >= 1 && steps <= LIPCACHE_MAX_NS_STEPS, "steps must be in [1, LIPCACHE_MAX_NS_STEPS]");
  LC_ARG(coefficients != nullptr, "NULL coefficients");
  for (int i = 0; i < 3 * steps; ++i)
    LC_ARG(std::isfinite(coefficients[i]) && std::fabs(coefficients[i]) <= 64.0,
           "coefficients must be finite, at most 64 in magnitude");
  LC_ARG(eps >= 1e-30 && eps <= 1.0, "eps must be in [1e-30, 1]");
}

}  // namespace

LC_API int64_t lipcache_orthogonalize_workspace(int32_t type, int64_t batch, int32_t rows, int32_t cols) {
  int64_t bytes = -1;
  guarded([&] {
    check_ortho_sizes(type, batch, rows, cols);
    bytes = (int64_t)lc::ops::ortho_bytes(type, batch, rows, cols);
  });
  return bytes;
}

LC_API lipcache_status lipcache_orthogonalize(int32_t type, const void* G, int64_t ldg, int64_t batch, int32_t rows,
                                              int32_t cols, int32_t steps, const double* coefficients, double eps,
                                              void* out, void* workspace, int64_t workspace_bytes,
                                              lipcache_stream_t stream) {
  return guarded([&] {
    check_ortho_sizes(type, batch, rows, cols);
    check_ortho(steps, coefficients, eps);
    if (batch == 0) return;
    LC_ARG(G != nullptr && out != nullptr, "NULL G or out");
    LC_ARG(aligned(G, type) && aligned(out, type), "a tensor is not aligned to its elements");
    LC_ARG(ldg >= cols, "a row stride is smaller than the row");
    LC_ARG(G != out || ldg == cols, "an orthogonalisation in place needs a dense matrix");
    check_workspace(workspace, workspace_bytes, lc::ops::ortho_bytes(type, batch, rows, cols));
    lc::ops::orthogonalize(type, G, ldg, batch, rows, cols, steps, coefficients, eps, out, lc::ops::OrthoStep{},
                           static_cast<unsigned char*>(workspace), stream);
  });
}

LC_API lipcache_status lipcache_orthogonal_step(int32_t weight_type, int32_t grad_type, const void* weight,
                                                const void* grad, const float* momentum, void* out_weight,
                                                float* out_momentum, int64_t batch, int32_t rows, int32_t cols,
                                                double lr, double beta, int32_t nesterov, double weight_decay,
                                                int32_t steps, const double* coefficients, double eps, void* workspace,
                                                int64_t workspace_bytes, lipcache_stream_t stream) {
  return guarded([&] {
    check_ortho_sizes(weight_type, batch, rows, cols);
    LC_ARG(known_type(grad_type), "unknown tensor type");
    check_ortho(steps, coefficients, eps);
    LC_ARG(beta >= 0.0 && beta <= 1.0, "beta must be in [0, 1]");
    LC_ARG(std::isfinite(lr) && std::isfinite(weight_decay), "lr and weight_decay must be finite");
    if (batch == 0) return;
    LC_ARG(weight && grad && momentum && out_weight && out_momentum, "NULL weight, grad or momentum");
    LC_ARG(aligned(weight, weight_type) && aligned(out_weight, weight_type) && aligned(grad, grad_type) &&
               aligned(momentum, LIPCACHE_F32) && aligned(out_momentum, LIPCACHE_F32),
           "a tensor is not aligned to its elements");
    check_workspace(workspace, workspace_bytes, lc::ops::ortho_bytes(weight_type, batch, rows, cols));
    lc::ops::OrthoStep st;
    st.weight = weight;
    st.out_weight = out_weight;
    st.momentum = momentum;
    st.out_momentum = out_momentum;
    st.weight_type = weight_type;
    st.beta = (float)beta;
    st.fresh = (float)(1.0 - beta);
    st.keep = (float)(1.0 - lr * weight_decay);
    st.rate = (float)(lr * std::sqrt(std::fmax(1.0, (double)rows / cols)));
    st.nesterov = nesterov != 0;
    lc::ops::orthogonalize(grad_type, grad, cols, batch, rows, cols, steps, coefficients, eps, nullptr, st,
                           static_cast<unsigned char*>(workspace), stream);
  });
}

LC_API lipcache_status lipcache_operator_errors(int64_t* count, lipcache_stream_t stream) {
  return guarded([&] {
    LC_ARG(count != nullptr, "count is NULL");
    *count = (int64_t)lc::ops::operator_errors(stream);
  });
}
