// y = x Q^T, tokens by the 8, float: the kernel for every width of code.
#include "tb_packed_few.cuh"

namespace tb {

tb_status packed_few_f32_1(const PackedFew& p, cudaStream_t st) { return launch_few_bits<1, 3, float>(p, st); }
int packed_few_f32_1_error_read_clear() { return few_tu_error_read_clear(); }

}  // namespace tb
