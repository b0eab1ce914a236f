// The kernels of pg_token.cuh for fp16 logits, in a file of their own so that the types are compiled side by side.
#include "pg_token.cuh"

namespace pg {

template int token_launch<__half, kForward>(const TokenParams&, cudaStream_t);
template int token_launch<__half, kBackward>(const TokenParams&, cudaStream_t);
template int token_launch<__half, kBoth>(const TokenParams&, cudaStream_t);

}  // namespace pg
