// The operators beside the plans, called with their arguments as an array of
// 64-bit words: a binding packs them with one call, where it would convert up to
// sixteen of them one by one (a combination of one token from Python 5.7 -> 5.4
// us of the host, a dispatch 6.6 -> 6.0).
#include <cstring>
#include <limits>
#include <utility>

#include "op_common.h"

using namespace bfsop;

namespace {

// Word w as a parameter of type T; ok: whether it fits.
template <typename T>
T argument(int64_t w, bool &ok) {
  if constexpr (std::is_pointer_v<T>) {
    return reinterpret_cast<T>((uintptr_t)w);
  } else if constexpr (std::is_floating_point_v<T>) {
    static_assert(sizeof(T) == sizeof w, "a double by its bits");
    T x;
    std::memcpy(&x, &w, sizeof x);
    return x;
  } else {
    if constexpr (sizeof(T) < sizeof w)
      ok = ok && w >= (int64_t)std::numeric_limits<T>::min() && w <= (int64_t)std::numeric_limits<T>::max();
    return (T)w;
  }
}

template <typename... P, size_t... I>
bfs_status call(bfs_status (*f)(P...), const int64_t *words, std::index_sequence<I...>) {
  if (words[1] != (int64_t)sizeof...(P))
    return fail(BFS_E_INVALID, "call: " + std::to_string(sizeof...(P)) + " arguments needed");
  int64_t w[sizeof...(P)];
  std::memcpy(w, words + 2, sizeof w);
  bool ok = true;
  std::tuple<P...> args{argument<P>(w[I], ok)...};
  if (!ok) return fail(BFS_E_INVALID, "call: an integer does not fit its parameter");
  return f(std::get<I>(args)...);
}

template <typename... P>
bfs_status call(bfs_status (*f)(P...), const int64_t *words) {
  return call(f, words, std::index_sequence_for<P...>{});
}

}  // namespace

extern "C" bfs_status bfs_call(const int64_t *words) {
  return entry([&]() -> bfs_status {
    if (!words || (uintptr_t)words % sizeof(int64_t)) return fail(BFS_E_INVALID, "call: bad address");
    switch (words[0]) {
      case BFS_CALL_MOE_ROUTE: return call(bfs_moe_route, words);
      case BFS_CALL_MOE_ROUTE_GRAD: return call(bfs_moe_route_grad, words);
      case BFS_CALL_MOE_DISPATCH: return call(bfs_moe_dispatch, words);
      case BFS_CALL_MOE_COMBINE: return call(bfs_moe_combine, words);
      case BFS_CALL_MOE_COMBINE_GRAD: return call(bfs_moe_combine_grad, words);
      case BFS_CALL_GRAD_NORM: return call(bfs_grad_norm, words);
      case BFS_CALL_GRAD_CLIP: return call(bfs_grad_clip, words);
      default: return fail(BFS_E_INVALID, "call: unknown operator");
    }
  });
}
