#include "ff_cross.cuh"
cudaError_t cx_backward_init() { return cudaSuccess; }
size_t cx_backward_bytes(const CrossDims&) { return 0; }
