// The decode kernels whose sums are applied as an AdamW step: instances of their own, so that the others keep their registers and
// their code.
#include "nuq_decode_chains.cuh"

namespace nuq {

cudaError_t upload_adamw_token_tables() { return upload_tables(); }
cudaError_t launch_decode_adamw(const DecodeParamsOf<AdamwSum>& P, int sms, cudaStream_t stream) { return launch(P, sms, stream); }

}  // namespace nuq
