// The Newton-Schulz steps on operands of two fp16 parts (22 digits).
#include <hip/hip_runtime.h>

#include "newton_schulz_steps.h"

namespace chunkft {

template int run_newton_schulz<2>(const OrthoProblem& p, const NsBuffers& b, hipStream_t st);

}  // namespace chunkft
