// The kernels of pg_token.cuh for bf16 logits, in a file of their own so that the types are compiled side by side.
#include "pg_token.cuh"

namespace pg {

template int token_launch<__nv_bfloat16, kForward>(const TokenParams&, cudaStream_t);
template int token_launch<__nv_bfloat16, kBackward>(const TokenParams&, cudaStream_t);
template int token_launch<__nv_bfloat16, kBoth>(const TokenParams&, cudaStream_t);

}  // namespace pg
