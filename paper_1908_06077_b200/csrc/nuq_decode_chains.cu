// The decode kernels whose sums are stored or applied as the step of Algorithm 1.
#include "nuq_decode_chains.cuh"

namespace nuq {

cudaError_t upload_token_tables() { return upload_tables(); }
cudaError_t launch_decode(const DecodeParams& P, int sms, cudaStream_t stream) { return launch(P, sms, stream); }

}  // namespace nuq
