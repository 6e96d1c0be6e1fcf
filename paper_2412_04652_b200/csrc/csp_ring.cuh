// Which phase of a stage's barrier belongs to the last load that went into the stage.  Plain arithmetic, for device and host.
#pragma once
#include <stdint.h>

#ifdef __CUDACC__
#define CSP_HOST_DEVICE __host__ __device__ __forceinline__
#else
#define CSP_HOST_DEVICE inline
#endif

namespace csp {
namespace dev {

// Fills 0, 1, 2, ... go round a ring of `stages`: fill i is phase i / stages of stage i % stages.  Parity of the phase that
// the last of `issued` fills completes at stage s, or -1 if the stage has had none.  A wait for that parity ends when this fill
// is there; a wait for the other one ends at once, whatever is under way, because the phase before is complete.
CSP_HOST_DEVICE int last_fill_parity(uint32_t issued, uint32_t stages, uint32_t s) {
    return s < issued ? int(((issued - 1u - s) / stages) & 1u) : -1;
}

}  // namespace dev
}  // namespace csp
