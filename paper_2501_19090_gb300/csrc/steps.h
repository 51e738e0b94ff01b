// steps.h -- arithmetic of steps that are dealt to workers (device, and the same on the host): there may be close to 2^31 of them.
#ifndef PIFA_STEPS_H_
#define PIFA_STEPS_H_

#ifdef __CUDACC__
#define PIFA_STEPS_HD __host__ __device__ __forceinline__
#else
#define PIFA_STEPS_HD inline
#endif

namespace pifa {

// A worker is at step `at` of its run, which ends at `stop`, and that is step s0 of a head's `steps`: where it ends in the head.
PIFA_STEPS_HD int segment_end(int steps, int s0, int at, int stop) {
  const int left = stop - at;  // (s0 + stop may be 2^31 and more)
  return left < steps - s0 ? s0 + left : steps;
}

}  // namespace pifa

#endif  // PIFA_STEPS_H_
