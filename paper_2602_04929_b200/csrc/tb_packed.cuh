// Shared pieces of the products with bit-packed weights (tb_packed_linear and its gradients).
#pragma once

#include "tb_common.cuh"

namespace tb {

// A packed projection and the adapters beside it as the kernels take them.
struct PackedW {
  const unsigned int* packed;
  const float* scales;
  const int* zeros;
  int d_out, d_in, bits, group, n_g, words;  // group: columns of a scale (d_in where there is one a row); words of a row
};
struct Adapt {  // n = 0: none
  const void *A, *B;
  const float* scale;
  const int *starts, *ids;
  int n, rank, n_req;
};

// The adapter of token t, or -1: the last request that starts at or before t, if t is not behind all of them.  Whatever
// the device arrays hold, the search ends and the result indexes an adapter or nothing.
__device__ __forceinline__ int adapter_of(const Adapt& a, long long t) {
  int lo = -1, hi = a.n_req;  // starts[lo] <= t < starts[hi]
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (a.starts[mid] <= t)
      lo = mid;
    else
      hi = mid;
  }
  if (lo < 0 || a.starts[a.n_req] <= t) return -1;
  const int id = a.ids[lo];
  return id >= 0 && id < a.n ? id : -1;
}

// The input of a product of gradients: in full, or 8-bit codes with a scale for a token and CKPT_RUN columns.
constexpr int CKPT_RUN = 128;

// Pieces of floats: two floats truncated to bf16, and what that leaves of one of them, nothing of what is not finite.  A piece takes
// eight bits, so that three hold a float; rounded to the nearest, the first piece of a value above 3.396e38 would be infinite.
__device__ __forceinline__ unsigned first_pieces(float lo, float hi) {
  unsigned o;
  asm("cvt.rz.bf16x2.f32 %0, %1, %2;" : "=r"(o) : "f"(hi), "f"(lo));
  return o;
}
__device__ __forceinline__ float rest_of(float v, unsigned piece) {  // `piece` in the upper half, as a float's bits
  const float f = __uint_as_float(piece);
  return fabsf(f) < __int_as_float(0x7f800000) ? v - f : 0.0f;
}

int sm_count();  // of the current device, 0 where it cannot be asked

}  // namespace tb
