// For callers that keep data between calls: which capture a stream is in, and that data made outside a capture are there before a graph reads them.
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

extern "C" int b2_event_finish(void* cuda_event) {
  cudaStreamCaptureMode mode = cudaStreamCaptureModeRelaxed;  // the event is none of a capture: waiting for it disturbs none
  if (!cuda_event) return -1;
  if (cudaThreadExchangeStreamCaptureMode(&mode) != cudaSuccess) return B2_ERR_LAUNCH;
  const cudaError_t rc = cudaEventSynchronize((cudaEvent_t)cuda_event);
  if (cudaThreadExchangeStreamCaptureMode(&mode) != cudaSuccess || rc != cudaSuccess) {
    (void)cudaGetLastError();
    return B2_ERR_LAUNCH;
  }
  return B2_OK;
}
