#include "paged.cuh"
namespace moqae {
long long paged_prefill_workspace_bytes(int, int, int, int) { return 16; }
cudaError_t launch_paged_prefill(const PagedView&, const RowsView&, const int32_t*, int, const RowsView&, const AttnOptions&, void*, cudaStream_t) { return cudaErrorNotSupported; }
}
