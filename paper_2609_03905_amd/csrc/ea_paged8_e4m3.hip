// ea_paged8_e4m3.hip -- attention over a paged cache of e4m3 codes.
#include "ea_paged8.h"

namespace ea {

hipError_t launch_paged8_e4m3(const PagedArgs& a, const PagedPass& sh, const PagedPass& own, int32_t d, int32_t dt,
                              hipStream_t s) {
  return run_code<false>(a, sh, own, d, dt, s);
}

}  // namespace ea
