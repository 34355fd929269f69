#include "paged.cuh"
namespace sc {
bool paged_decode_mma_supported(const PagedDecodeArgs&) { return false; }
cudaError_t launch_paged_decode_mma(const PagedDecodeArgs&, cudaStream_t) { return cudaErrorNotSupported; }
size_t paged_decode_mma_ws_bytes() { return 0; }
}
