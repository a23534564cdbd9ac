#include "shaped.cuh"
namespace pda {
bool prefill_tc_supports(const PrefillParams&) { return false; }
cudaError_t launch_prefill_tc(const PrefillParams&, cudaStream_t) { return cudaErrorNotSupported; }
int64_t prefill_workspace_bytes(int head_dim) { return 256; }
}  // namespace pda
