// What a caller that keeps data between calls has to know of captured graphs: which capture a stream is in.
#include <cuda_runtime.h>

#include "b2gemm.h"

extern "C" int b2_graph_capture_id(void* cuda_stream, uint64_t* id) {
  if (!id) return -2;
  cudaStreamCaptureStatus status = cudaStreamCaptureStatusNone;
  unsigned long long number = 0;
  if (cudaStreamGetCaptureInfo((cudaStream_t)cuda_stream, &status, &number) != cudaSuccess) {
    (void)cudaGetLastError();
    return B2_ERR_LAUNCH;
  }
  *id = status == cudaStreamCaptureStatusNone ? 0 : number + 1;
  return B2_OK;
}
