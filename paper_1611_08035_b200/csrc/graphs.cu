// For callers that keep data between calls: which capture a stream is in, that data made outside a capture are there before a graph reads them, and when the graph is gone that does.
#include <cuda_runtime.h>

#include <atomic>

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

// A watch is a place in a table, so that no call allocates.  The graph holds it through a user object, which CUDA's executable forms of the graph share: its callback comes when the last of
// them is destroyed and has run.
namespace {
constexpr int kWatches = 4096;
enum : int { kFree = 0, kWatched, kGone, kLeft };  // kLeft: the graph lives, nobody asks any more
std::atomic<int> g_watch[kWatches];
std::atomic<unsigned> g_next_watch{0};

void CUDART_CB graph_gone(void* place) {
  auto* w = static_cast<std::atomic<int>*>(place);
  int now = kWatched;
  if (!w->compare_exchange_strong(now, kGone)) w->store(kFree);
}
}  // namespace

extern "C" int b2_graph_watch(void* cuda_stream, int* watch) {
  if (!watch) return -2;
  cudaStreamCaptureStatus status = cudaStreamCaptureStatusNone;
  unsigned long long number = 0;
  cudaGraph_t graph = nullptr;
  if (cudaStreamGetCaptureInfo((cudaStream_t)cuda_stream, &status, &number, &graph) != cudaSuccess) {
    (void)cudaGetLastError();
    return B2_ERR_LAUNCH;
  }
  if (status != cudaStreamCaptureStatusActive) return -1;
  for (int i = 0; i < kWatches; ++i) {
    const unsigned at = g_next_watch.fetch_add(1) % kWatches;
    int now = kFree;
    if (!g_watch[at].compare_exchange_strong(now, kWatched)) continue;
    cudaUserObject_t object = nullptr;
    if (cudaUserObjectCreate(&object, &g_watch[at], graph_gone, 1, cudaUserObjectNoDestructorSync) != cudaSuccess) {
      (void)cudaGetLastError();
      g_watch[at].store(kFree);
      return B2_ERR_LAUNCH;
    }
    if (cudaGraphRetainUserObject(graph, object, 1, cudaGraphUserObjectMove) != cudaSuccess) {
      (void)cudaGetLastError();
      g_watch[at].store(kLeft);
      (void)cudaUserObjectRelease(object, 1);  // the callback frees the place
      return B2_ERR_LAUNCH;
    }
    *watch = (int)at;
    return B2_OK;
  }
  return B2_ERR_STATIC_LIMIT;
}

extern "C" int b2_graph_gone(int watch) { return watch >= 0 && watch < kWatches && g_watch[watch].load() == kGone; }

extern "C" int b2_graph_unwatch(int watch) {
  if (watch < 0 || watch >= kWatches) return -1;
  int now = kWatched;
  if (g_watch[watch].compare_exchange_strong(now, kLeft)) return B2_OK;
  now = kGone;
  return g_watch[watch].compare_exchange_strong(now, kFree) ? B2_OK : -1;
}
