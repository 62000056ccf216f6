// As much of the CUDA runtime as csrc/a2sgd_train.cu calls, for two devices that differ in their SMs and in what fits on one.
#include <cstddef>

extern "C" {
int current_device = 0, occupancy_questions = 0;

int cudaGetDevice(int *d) { return *d = current_device, 0; }
int cudaGetLastError() { return 0; }
int cudaDeviceGetAttribute(int *v, int, int d) { return *v = 100 + d, 0; }
int cudaFuncSetAttribute(const void *, int, int) { return 0; }
int cudaOccupancyMaxActiveBlocksPerMultiprocessor(int *n, const void *, int, size_t) { return ++occupancy_questions, *n = 2 + current_device, 0; }
}
