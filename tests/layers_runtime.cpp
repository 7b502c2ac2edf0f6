// The stand-in runtime of host_runtime.cpp with an MI355X's 256 compute units, by which the operators
// around a delivered product cut their work.
#define hipGetDevicePropertiesR0600 plain_properties
#include "host_runtime.cpp"
#undef hipGetDevicePropertiesR0600

extern "C" hipError_t hipGetDevicePropertiesR0600(hipDeviceProp_tR0600* p, int device) {
  const hipError_t e = plain_properties(p, device);
  p->multiProcessorCount = 256;
  return e;
}
