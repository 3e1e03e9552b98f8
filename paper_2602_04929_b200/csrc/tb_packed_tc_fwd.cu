// y = x Q^T on the tensor cores: the kernel for every width of code.
#include "tb_packed_tc.cuh"

namespace tb {

tb_status packed_tc_forward(const PackedTc& p, const CUtensorMap& xmap, const CUtensorMap& wmap, int pairs, cudaStream_t st) {
  return launch_packed_tc_bits<false>(p, xmap, wmap, pairs, st);
}

int packed_fwd_error_read_clear() { return packed_tc_error_read_clear(); }

}  // namespace tb
