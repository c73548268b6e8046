// fake_operators.cpp with streams that can be captured: what the runtime refuses
// during a capture, or afterwards of an event that was last recorded in one, counts.
#include <cuda_runtime.h>

#define cudaStreamIsCapturing plain_is_capturing
#define cudaEventQuery plain_event_query
#define cudaEventRecord plain_event_record
#define cudaEventSynchronize plain_event_synchronize
#define cudaStreamWaitEvent plain_stream_wait_event
#define cudaMalloc plain_malloc
#define cudaFree plain_free
#define cudaMemcpyAsync plain_memcpy_async
#define launch_blocks plain_launch_blocks
#define launch_norm_rope plain_launch_norm_rope
#define launch_norm_rope_grad plain_launch_norm_rope_grad
#define launch_decode plain_launch_decode
#define launch_prefill plain_launch_prefill
extern "C" {
cudaError_t plain_is_capturing(cudaStream_t, cudaStreamCaptureStatus*);
cudaError_t plain_event_query(cudaEvent_t);
cudaError_t plain_event_record(cudaEvent_t, cudaStream_t);
cudaError_t plain_event_synchronize(cudaEvent_t);
cudaError_t plain_stream_wait_event(cudaStream_t, cudaEvent_t, unsigned);
cudaError_t plain_malloc(void**, size_t);
cudaError_t plain_free(void*);
cudaError_t plain_memcpy_async(void*, const void*, size_t, cudaMemcpyKind, cudaStream_t);
}
#include "fake_operators.cpp"
#undef cudaStreamIsCapturing
#undef cudaEventQuery
#undef cudaEventRecord
#undef cudaEventSynchronize
#undef cudaStreamWaitEvent
#undef cudaMalloc
#undef cudaFree
#undef cudaMemcpyAsync
#undef launch_blocks
#undef launch_norm_rope
#undef launch_norm_rope_grad
#undef launch_decode
#undef launch_prefill

#include <set>

namespace {
void* g_capturing = nullptr;
int64_t g_wrong = 0, g_uploads = 0;
std::set<cudaEvent_t> g_captured;   // events last recorded in a capture
std::set<void*> g_freed;
cudaError_t wrong() { return ++g_wrong, cudaErrorStreamCaptureUnsupported; }
}  // namespace

// The buffers that the last launch of a kind was given (since a capture began).
static const void *g_plan, *g_parts, *g_places, *g_grad_part;
EXPORT void fake_capture(void* stream) {  // null: the capture ends
    g_capturing = stream;
    g_freed.clear();
    if (stream) g_plan = g_parts = g_places = g_grad_part = nullptr;
}
EXPORT int64_t fake_wrong() { return g_wrong; }
EXPORT int64_t fake_captured_uploads() { return g_uploads; }
EXPORT int fake_was_freed(void* p) { return (int)g_freed.count(p); }  // since the capture
EXPORT void fake_capture_reset() {
    g_capturing = nullptr;
    g_wrong = g_uploads = 0;
    g_captured.clear();
    g_freed.clear();
}

EXPORT void fake_given(const void** out) {
    out[0] = g_plan;
    out[1] = g_parts;
    out[2] = g_places;
    out[3] = g_grad_part;
}
namespace sq {
cudaError_t launch_blocks(const CUtensorMap& m, const CUtensorMap& q, const BlockShortArgs& a, int D, bool one,
                          cudaStream_t st) {
    g_plan = a.tiles;
    g_parts = a.part_o;
    return plain_launch_blocks(m, q, a, D, one, st);
}
cudaError_t launch_norm_rope(const NormRopeArgs& a, int D, bool store, cudaStream_t st) {
    g_places = a.places;
    return plain_launch_norm_rope(a, D, store, st);
}
cudaError_t launch_norm_rope_grad(const NormRopeGradArgs& a, int D, cudaStream_t st) {
    g_grad_part = a.part;
    return plain_launch_norm_rope_grad(a, D, st);
}
cudaError_t launch_decode(const CUtensorMap& m, const DecodeArgs& a, int n, int D, cudaStream_t st) {
    g_plan = a.segs;
    g_parts = a.part_o;
    return plain_launch_decode(m, a, n, D, st);
}
cudaError_t launch_prefill(const CUtensorMap& m, const CUtensorMap& q, const PrefillShortArgs& a, int D,
                           cudaStream_t st) {
    g_plan = a.tiles;
    g_parts = a.part_o;
    return plain_launch_prefill(m, q, a, D, st);
}
}  // namespace sq

extern "C" {

cudaError_t cudaStreamIsCapturing(cudaStream_t st, cudaStreamCaptureStatus* s) {
    *s = g_capturing && st == g_capturing ? cudaStreamCaptureStatusActive : cudaStreamCaptureStatusNone;
    return cudaSuccess;
}
cudaError_t cudaEventQuery(cudaEvent_t e) {
    if (g_capturing || g_captured.count(e)) return wrong();
    return cudaSuccess;  // (everything eager is complete)
}
cudaError_t cudaEventRecord(cudaEvent_t e, cudaStream_t st) {
    if (g_capturing && st == g_capturing) g_captured.insert(e);
    else g_captured.erase(e);
    return plain_event_record(e, st);
}
cudaError_t cudaEventSynchronize(cudaEvent_t e) {
    if (g_capturing || g_captured.count(e)) return wrong();
    return plain_event_synchronize(e);
}
cudaError_t cudaStreamWaitEvent(cudaStream_t st, cudaEvent_t e, unsigned f) {
    const bool inside = g_capturing && st == g_capturing;
    if (inside != (g_captured.count(e) > 0)) return wrong();
    return plain_stream_wait_event(st, e, f);
}
cudaError_t cudaMalloc(void** p, size_t n) {
    if (g_capturing) return wrong();
    return plain_malloc(p, n);
}
cudaError_t cudaFree(void* p) {
    if (g_capturing) return wrong();
    if (p) g_freed.insert(p);
    return plain_free(p);
}
cudaError_t cudaMemcpyAsync(void* d, const void* s, size_t n, cudaMemcpyKind k, cudaStream_t st) {
    if (g_capturing && st == g_capturing) ++g_uploads;  // (its source is reused before a replay)
    return plain_memcpy_async(d, s, n, k, st);
}

}  // extern "C"
