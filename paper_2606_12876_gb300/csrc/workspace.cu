// Workspaces for captured calls (aq_workspace_create, aq_workspace_destroy, aq_capture_id).
//
// A captured graph keeps the addresses that its calls were given and may be replayed on any stream, beside
// other graphs and eager calls, so a workspace that a call must have to itself has to belong to the capture.
// It is made while the capture is under way, when an allocation through a caching allocator would come from
// the graph's own pool, where a replay may write it before its use, and a zero-fill on the capturing stream
// would become a node that every replay repeats, clearing the status that the one before recorded. Memory
// made here belongs to no pool and is zero when the call returns.
#include "aq_internal.cuh"

namespace {

// Allocations and the like are refused while a thread captures, unless it declares that they are not part
// of what it captures.
class OutsideCapture {
public:
    OutsideCapture() { (void)cudaThreadExchangeStreamCaptureMode(&mode_); }
    ~OutsideCapture() { (void)cudaThreadExchangeStreamCaptureMode(&mode_); }

private:
    cudaStreamCaptureMode mode_ = cudaStreamCaptureModeRelaxed;
};

// Zero-fill that has finished when it returns, on a stream of its own.
aq_status fill_zero(void* p, size_t bytes) {
    cudaStream_t st;
    if (cudaError_t e = cudaStreamCreateWithFlags(&st, cudaStreamNonBlocking); e != cudaSuccess)
        return aq::cuda_fail(e, "cudaStreamCreateWithFlags");
    aq_status rc = aq::cuda_ok(cudaMemsetAsync(p, 0, bytes, st), "cudaMemsetAsync");
    if (rc == AQ_OK) rc = aq::cuda_ok(cudaStreamSynchronize(st), "cudaStreamSynchronize");
    (void)cudaStreamDestroy(st);
    return rc;
}

}  // namespace

extern "C" {

aq_status aq_workspace_create(size_t bytes, void** workspace) {
    if (!workspace) return AQ_ERR_INVALID_ARG;
    *workspace = nullptr;
    if (bytes == 0) return AQ_ERR_INVALID_ARG;
    OutsideCapture guard;
    void* p = nullptr;
    if (cudaError_t e = cudaMalloc(&p, bytes); e != cudaSuccess) return aq::cuda_fail(e, "cudaMalloc");
    if (aq_status rc = fill_zero(p, bytes); rc != AQ_OK) {
        (void)cudaFree(p);
        return rc;
    }
    *workspace = p;
    return AQ_OK;
}

aq_status aq_workspace_destroy(void* workspace) {
    if (!workspace) return AQ_OK;
    OutsideCapture guard;
    return aq::cuda_ok(cudaFree(workspace), "cudaFree");
}

aq_status aq_capture_id(void* stream, unsigned long long* id) {
    if (!id) return AQ_ERR_INVALID_ARG;
    *id = 0;
    cudaStreamCaptureStatus status = cudaStreamCaptureStatusNone;
    unsigned long long n = 0;
    if (cudaError_t e = cudaStreamGetCaptureInfo((cudaStream_t)stream, &status, &n); e != cudaSuccess)
        return aq::cuda_fail(e, "cudaStreamGetCaptureInfo");
    if (status == cudaStreamCaptureStatusActive) *id = n;
    return AQ_OK;
}

}  // extern "C"
