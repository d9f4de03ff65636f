// Rounds of copies that a thread starts and sees land in the same order, and which of them are still to be waited for when it leaves.
#pragma once
#include <cstdint>

#ifdef __CUDACC__
#define GF_BOTH __host__ __device__ __forceinline__
#else
#define GF_BOTH inline
#endif

namespace gf {

struct Rounds {
  uint32_t started = 0, landed = 0;
  bool ok = true;  // no wait has given up
  GF_BOTH void start() { ++started; }
  // The next round in order has been waited for: only one that was there counts, and none behind one that was not.
  GF_BOTH void waited(bool there) {
    ok = ok && there;
    if (ok) ++landed;
  }
  GF_BOTH uint32_t on_the_way() const { return started - landed; }  // rounds landed .. started - 1
};

}  // namespace gf
