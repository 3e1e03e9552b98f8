// y = x Q^T, tokens by the 16, bf16: the kernel for every width of code.
#include "tb_packed_few.cuh"

namespace tb {

tb_status packed_few_bf16_2(const PackedFew& p, cudaStream_t st) { return launch_few_bits<2, 1, __nv_bfloat16>(p, st); }
int packed_few_bf16_2_error_read_clear() { return few_tu_error_read_clear(); }

}  // namespace tb
