// The tensor-core product with bit-packed weights as its host side sees it.
#pragma once

#include "tb_packed.cuh"
#include "tb_tma.cuh"

namespace tb {

enum {
  PT_BK = 64,
  PT_A_BYTES = 128 * PT_BK * 2,
  PT_STAGE_BYTES = 2 * PT_A_BYTES,  // A, then B (at most 128 tokens)
  PT_PART = 2048,  // contraction columns of one accumulation at most
  PT_SMEM = 226 * 1024 + 512       // stages, ring, 1024 bytes to align them, 512 of barriers
};

// What a launch works on.
struct PackedTc {
  PackedW w;
  Adapt ad;
  const __nv_bfloat16* M;  // adapters' matrix of the result's columns, [adapter][rank][n_cols]
  const float* low;        // [n_tok][rank]
  const float* st;         // forward: scales [n_g][rows_pad], zeros behind d_out
  const unsigned* zt;      // zero-points as the decoders take them, likewise; backward each followed by its scale's two bf16 pieces
  const unsigned* words;   // the packed rows, `pitch` words apart (a multiple of 16 bytes)
  int rows_pad, pitch;
  const int4* runs;        // per token tile, from its first token's index on: first token, end, adapter
  const int* n_runs;       // per token tile; nullptr: no adapters, or added with the splits' sums
  __nv_bfloat16* out;      // [n_tok][n_cols]
  float* part;             // [split][n_tok][n_cols] where the sums are joined afterwards, else nullptr
  int n_tok, n_cols, n_sum, n_tile, m_tiles, t_tiles, splits, split_len;
};

struct TcPlan {
  int n_tile, m_tiles, t_tiles, splits, split_len, pairs;
  bool joined;  // float sums, added with the adapters' share by a kernel of their own: with splits, or where runs are many
};
TcPlan packed_tc_plan(const Adapt& ad, int n_tok, int n_cols, int n_sum, bool back);
// Scratch of a product from `ws` on (nullptr: only its size).
size_t packed_tc_carve(const TcPlan& t, const PackedW& w, const Adapt& ad, int n_tok, int n_cols, bool back, char* ws, PackedTc* p);
// out = in Q^T or in Q, with the adapters' share; makes their low [n_tok][rank] = in M_i^T too.
tb_status packed_product_tc(const PackedW& w, const Adapt& ad, const __nv_bfloat16* in, long long n_tok, __nv_bfloat16* out,
                            float* low, bool back, void* ws, cudaStream_t st);
bool adapter_low_in_small_tiles(const Adapt& ad, int n_tok, int width);
tb_status adapter_low_bf16(const Adapt& ad, const __nv_bfloat16* in, const __nv_bfloat16* M, int n_tok, int width, float* low, bool late,
                           cudaStream_t st);
tb_status packed_tc_forward(const PackedTc& p, const CUtensorMap& xmap, const CUtensorMap& wmap, int pairs, cudaStream_t st);
tb_status packed_tc_backward(const PackedTc& p, const CUtensorMap& xmap, const CUtensorMap& wmap, int pairs, cudaStream_t st);

}  // namespace tb
