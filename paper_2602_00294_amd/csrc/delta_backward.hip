#include <hip/hip_runtime.h>
#include "kernels.hpp"
namespace sata {
size_t delta_backward_scratch(bool, int, int, int, int, int) { return 0; }
hipError_t launch_delta_backward(const DeltaArgs&, bool, void*, hipStream_t) { return hipErrorNotSupported; }
}  // namespace sata
