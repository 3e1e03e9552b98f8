// The tensor-core product with bit-packed weights as its host side sees it.
#pragma once

#include "tb_packed.cuh"
#include "tb_tma.cuh"

namespace tb {

enum {
  PT_BK = 64,
  PT_STAGES = 6,
  PT_A_BYTES = 128 * PT_BK * 2,
  PT_STAGE_BYTES = 2 * PT_A_BYTES,  // A, then B (at most 128 tokens)
  PT_THREADS = 512,
  PT_PART = 2048,  // contraction columns of one accumulation at most
  PT_SMEM = PT_STAGES * PT_STAGE_BYTES + 1024 + 512
};

// What a launch works on.
struct PackedTc {
  PackedW w;
  Adapt ad;
  const __nv_bfloat16* M;  // adapters' matrix of the result's columns, [adapter][rank][n_cols]
  const float* low;        // [n_tok][rank]
  const int4* runs;        // per token tile, from its first token's index on: first token, end, adapter
  const int* n_runs;       // per token tile
  __nv_bfloat16* out;      // [n_tok][n_cols]
  float* part;             // splits > 1: [split][n_tok][n_cols]
  unsigned long long group_inv;  // floor(2^38 / (group / 32)) + 1: j / group = (j / 32 * group_inv) >> 38 below 2^24 columns
  int n_tok, n_cols, n_sum, n_tile, m_tiles, t_tiles, splits, split_len;
};

struct TcPlan {
  int n_tile, m_tiles, t_tiles, splits, split_len, pairs;
};
TcPlan packed_tc_plan(int n_tok, int n_cols, int n_sum);
// Scratch of a product from `ws` on (nullptr: only its size).
size_t packed_tc_carve(const TcPlan& t, const Adapt& ad, int n_tok, int n_cols, char* ws, PackedTc* p);
tb_status packed_product_tc(const PackedW& w, const Adapt& ad, const __nv_bfloat16* in, long long n_tok, __nv_bfloat16* out,
                            const float* low, bool back, void* ws, cudaStream_t st);
tb_status packed_tc_forward(const PackedTc& p, const CUtensorMap& map, int pairs, cudaStream_t st);
tb_status packed_tc_backward(const PackedTc& p, const CUtensorMap& map, int pairs, cudaStream_t st);

}  // namespace tb
