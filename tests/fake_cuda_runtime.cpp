// A CUDA runtime of the host's own memory, and launchers that launch nothing, for the host side of the library (test
// infrastructure).  Copies from host memory behave as the runtime's documentation allows for pageable memory: cudaMemcpy returns with
// the data staged, and it arrives at its destination when something waits for the stream.
#include <cuda_runtime.h>

#include <cstdlib>
#include <cstring>
#include <map>
#include <vector>

#include "dlm_gradients.h"
#include "dlm_internal.h"
#include "dlm_train.h"

namespace {
struct Staged {
    void* dst;
    std::vector<unsigned char> bytes;
};
std::vector<Staged> staged;
std::map<void*, size_t> blocks;
cudaError_t last = cudaSuccess;
int copies = 0, mallocs_left = -1, launches_fail = 0;

cudaError_t note(cudaError_t e) {
    if (e != cudaSuccess) last = e;
    return e;
}
void arrive() {
    for (const Staged& s : staged) std::memcpy(s.dst, s.bytes.data(), s.bytes.size());
    staged.clear();
}
int launch() {
    if (!launches_fail) return DLM_OK;
    note(cudaErrorInvalidValue);
    return DLM_ERR_CUDA;
}
}  // namespace

extern "C" {

cudaError_t cudaGetDeviceCount(int* n) { *n = 1; return cudaSuccess; }
cudaError_t cudaGetDevice(int* d) { *d = 0; return cudaSuccess; }
cudaError_t cudaDeviceGetAttribute(int* v, cudaDeviceAttr, int) { *v = 148; return cudaSuccess; }
cudaError_t cudaGetLastError(void) { cudaError_t e = last; last = cudaSuccess; return e; }
cudaError_t cudaMalloc(void** p, size_t bytes) {
    if (mallocs_left == 0) return note(cudaErrorMemoryAllocation);
    if (mallocs_left > 0) --mallocs_left;
    *p = std::malloc(bytes ? bytes : 1);
    blocks[*p] = bytes;
    return cudaSuccess;
}
cudaError_t cudaFree(void* p) {
    if (!blocks.erase(p)) return note(cudaErrorInvalidValue);
    std::free(p);
    return cudaSuccess;
}
cudaError_t cudaMemcpy(void* dst, const void* src, size_t bytes, cudaMemcpyKind kind) {
    if (kind != cudaMemcpyHostToDevice) return note(cudaErrorInvalidValue);
    const unsigned char* b = static_cast<const unsigned char*>(src);
    staged.push_back({dst, {b, b + bytes}});
    ++copies;
    return cudaSuccess;
}
cudaError_t cudaStreamSynchronize(cudaStream_t) { arrive(); return cudaSuccess; }
cudaError_t cudaDeviceSynchronize(void) { arrive(); return cudaSuccess; }

// what the tests look at and set
int fake_copies(void) { return copies; }
int fake_staged(void) { return (int)staged.size(); }
int fake_blocks(void) { return (int)blocks.size(); }
int fake_last_error(void) { return (int)last; }
void fake_mallocs_left(int n) { mallocs_left = n; }
void fake_launches_fail(int v) { launches_fail = v; }

}  // extern "C"

int dlm_launch_gradients(const dlm_gradients&, int, float, float*, void*, int, int64_t, void*) { return launch(); }
int dlm_norm_max_ctas(int, int64_t rows, int64_t) { return (int)(rows < 8 ? rows : 8); }
int dlm_launch_layer_norm(const dlm_norm_args&, void*) { return launch(); }
int dlm_launch_layer_norm_grad(const dlm_norm_args&, void*) { return launch(); }
int dlm_launch_policy_loss(const dlm_policy_args&, void*) { return launch(); }
int dlm_launch_shard_step(int, const dlm_shard_args&, void*) { return launch(); }
int dlm_launch_local_momentum(int, int64_t, int64_t, float*, float*, const void*, int, int64_t, float, float, void*) { return launch(); }
