// The mixture-of-experts calls with their arguments as words in memory.
#include "../../include/osdp.h"

#include <cstring>

namespace {
struct Word {
  int64_t v;
  template <typename T>
  operator T *() const { return reinterpret_cast<T *>((uintptr_t)v); }
  operator int64_t() const { return v; }
  operator size_t() const { return (size_t)v; }
  // an int that the word does not fit is none that any call takes
  operator int() const { return v < INT32_MIN || v > INT32_MAX ? INT32_MIN : (int)v; }
  operator double() const {
    double d;
    memcpy(&d, &v, 8);
    return d;
  }
};
}  // namespace

extern "C" int osdp_call(const void *words) {
  if (!words) return OSDP_ERR_NULL_POINTER;
  int64_t which, w[24];
  memcpy(&which, words, 8);
  static const int count[] = {16, 14, 7, 12, 10, 16, 21};      // arguments of each
  if (which < 0 || which >= (int64_t)(sizeof(count) / sizeof(count[0]))) return OSDP_ERR_UNSUPPORTED;
  memcpy(w, static_cast<const char *>(words) + 8, 8 * (size_t)count[which]);
  auto a = [&](int k) { return Word{w[k]}; };
  switch (which) {
    case OSDP_CALL_ROUTE_FWD:
      return osdp_route_fwd(a(0), a(1), a(2), a(3), a(4), a(5), a(6), a(7), a(8), a(9), a(10), a(11), a(12), a(13), a(14), a(15));
    case OSDP_CALL_ROUTE_BWD:
      return osdp_route_bwd(a(0), a(1), a(2), a(3), a(4), a(5), a(6), a(7), a(8), a(9), a(10), a(11), a(12), a(13));
    case OSDP_CALL_EXPERT_PLAN:
      return osdp_expert_plan(a(0), a(1), a(2), a(3), a(4), a(5), a(6));
    case OSDP_CALL_EXPERT_DISPATCH:
      return osdp_expert_dispatch(a(0), a(1), a(2), a(3), a(4), a(5), a(6), a(7), a(8), a(9), a(10), a(11));
    case OSDP_CALL_EXPERT_COMBINE:
      return osdp_expert_combine(a(0), a(1), a(2), a(3), a(4), a(5), a(6), a(7), a(8), a(9));
    case OSDP_CALL_EXPERT_LINEAR_FWD:
      return osdp_expert_linear_fwd(a(0), a(1), a(2), a(3), a(4), a(5), a(6), a(7), a(8), a(9), a(10), a(11), a(12), a(13), a(14), a(15));
    default:
      return osdp_expert_linear_bwd(a(0), a(1), a(2), a(3), a(4), a(5), a(6), a(7), a(8), a(9), a(10), a(11), a(12), a(13), a(14), a(15), a(16), a(17),
                                    a(18), a(19), a(20));
  }
}
