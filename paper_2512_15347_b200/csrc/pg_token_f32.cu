// The kernels of pg_token.cuh for fp32 logits, in a file of their own so that the types are compiled side by side.
#include "pg_token.cuh"

namespace pg {

template int token_launch<float, kForward>(const TokenParams&, cudaStream_t);
template int token_launch<float, kBackward>(const TokenParams&, cudaStream_t);
template int token_launch<float, kBoth>(const TokenParams&, cudaStream_t);

}  // namespace pg
