// Calls whose arguments come as words in memory.
#include <cstring>
#include <utility>

#include "damoe.h"

namespace {

union Word {
  int64_t i;
  double f;
  void* p;
};

// Argument by argument, each as the type that the callee declares.
struct Args {
  const Word* w;
  template <class T>
  operator T*() const { return static_cast<T*>(w->p); }
  operator int32_t() const { return (int32_t)w->i; }
  operator int64_t() const { return w->i; }
  operator size_t() const { return (size_t)w->i; }
  operator float() const { return (float)w->f; }
};

template <class... A, size_t... I>
damoe_status apply(damoe_status (*f)(A...), const Word* w, std::index_sequence<I...>) {
  return f(static_cast<A>(Args{w + I})...);
}

template <class... A>
damoe_status call(damoe_status (*f)(A...), const void* words, size_t n) {
  Word w[sizeof...(A)];
  if (!words || n != sizeof...(A)) return DAMOE_ERR_INVALID_ARG;
  std::memcpy(w, words, sizeof w);
  return apply(f, w, std::index_sequence_for<A...>{});
}

}  // namespace

extern "C" damoe_status damoe_call_words(int32_t fn, const void* words, size_t n) {
  switch (fn) {
    case DAMOE_CALL_ROUTER_LOSS: return call(damoe_router_loss, words, n);
    case DAMOE_CALL_ROUTER_LOSS_GRAD: return call(damoe_router_loss_grad, words, n);
    case DAMOE_CALL_MXFP4_LINEAR: return call(damoe_mxfp4_linear, words, n);
    default: return DAMOE_ERR_INVALID_ARG;
  }
}
