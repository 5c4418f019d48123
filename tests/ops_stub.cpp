// ops_stub.cpp -- hip_stub.cpp's recording HIP runtime with the current device's changes.
#include "hip_stub.cpp"

extern "C" hipError_t hipSetDevice(int d) {
  g_device = d;
  g_log += "device " + std::to_string(d) + "\n";
  return hipSuccess;
}
