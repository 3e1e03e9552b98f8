// Host side of the tensor-core product with bit-packed weights: tiles and splits, the runs of tokens with one adapter, and the
// sum of the splits.
#include "tb_packed_plan.cuh"

namespace tb {

// The tokens of a tile in runs of one adapter.  Tokens without one are in no run.
__global__ void __launch_bounds__(256) k_adapter_runs(Adapt ad, int n_tok, int n_tile, int4* __restrict__ runs, int* __restrict__ n_runs) {
  __shared__ int own[257], count[8];
  const int t0 = blockIdx.x * n_tile, n = min(n_tile, n_tok - t0), i = threadIdx.x;
  own[i] = i < n ? adapter_of(ad, t0 + i) : -1;
  __syncthreads();
  const bool first = own[i] >= 0 && (i == 0 || own[i - 1] != own[i]);
  const unsigned m = __ballot_sync(0xffffffffu, first);
  if ((i & 31) == 0) count[i >> 5] = __popc(m);
  __syncthreads();
  int at = __popc(m & ((1u << (i & 31)) - 1u)), all = 0;
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    if (k < (i >> 5)) at += count[k];
    all += count[k];
  }
  if (first) {
    int e = i + 1;
    while (e < n && own[e] == own[i]) ++e;
    runs[t0 + at] = make_int4(t0 + i, t0 + e, own[i], 0);
  }
  if (i == 0) n_runs[blockIdx.x] = all;
}

// out = the splits' sums, added in their order, rounded once; four values a thread.
__global__ void __launch_bounds__(256) k_packed_join(const float4* __restrict__ part, uint2* __restrict__ out, long long n4, int splits) {
  for (long long i = blockIdx.x * 256ll + threadIdx.x; i < n4; i += gridDim.x * 256ll) {
    float4 s = __ldcs(part + i);
    for (int k = 1; k < splits; ++k) {
      const float4 v = __ldcs(part + k * n4 + i);
      s.x += v.x, s.y += v.y, s.z += v.z, s.w += v.w;
    }
    const __nv_bfloat162 a = __floats2bfloat162_rn(s.x, s.y), b = __floats2bfloat162_rn(s.z, s.w);
    out[i] = make_uint2(*reinterpret_cast<const unsigned*>(&a), *reinterpret_cast<const unsigned*>(&b));
  }
}

// Tile and splits by an estimate of the clocks: a stage costs what its MMAs take, 2 clocks a token of the tile, or its decoding,
// a tile about 3000 clocks more, and splits cost writing and adding their float sums.
TcPlan packed_tc_plan(int n_tok, int n_cols, int n_sum) {
  TcPlan best = {};
  double best_cost = 0.0;
  int sms = sm_count();
  if (sms < 2) sms = 148;  // a query where there is no device
  const int pairs = sms / 2, m_tiles = (n_cols + 255) / 256;
  const int top = n_tok >= 256 ? 256 : (n_tok + 31) / 32 * 32;
  for (int n_tile = 32; n_tile <= top; n_tile += 32) {
    const int t_tiles = (n_tok + n_tile - 1) / n_tile;
    for (int splits = 1; splits <= 16; ++splits) {
      const int len = ((n_sum + splits - 1) / splits + 63) / 64 * 64;
      if (splits > 1 && (len < 256 || (long long)len * (splits - 1) >= n_sum)) continue;
      const long long tiles = (long long)m_tiles * t_tiles * splits;
      if (tiles > 0x3fffffff) continue;
      const double waves = (double)((tiles + pairs - 1) / pairs);
      const double stage = 2.0 * n_tile > 200.0 ? 2.0 * n_tile : 200.0;
      double cost = waves * (len / 64 * stage + 1500.0 + 6.0 * n_tile);
      if (splits > 1) cost += 4000.0 + 8.0 * splits * (double)n_tok * n_cols / 2500.0;
      if (best.n_tile == 0 || cost < best_cost) {
        best_cost = cost;
        best.n_tile = n_tile, best.m_tiles = m_tiles, best.t_tiles = t_tiles, best.splits = splits, best.split_len = len;
        best.pairs = tiles < pairs ? (int)tiles : pairs;
      }
    }
  }
  return best;
}

size_t packed_tc_carve(const TcPlan& t, const Adapt& ad, int n_tok, int n_cols, char* ws, PackedTc* p) {
  Bump b(ws);
  p->runs = ad.n ? b.take<int4>(n_tok) : nullptr;
  p->n_runs = ad.n ? b.take<int>(t.t_tiles) : nullptr;
  p->part = t.splits > 1 ? b.take<float>((size_t)t.splits * n_tok * n_cols) : nullptr;
  return b.total();
}

tb_status packed_product_tc(const PackedW& w, const Adapt& ad, const __nv_bfloat16* in, long long n_tok, __nv_bfloat16* out,
                            const float* low, bool back, void* ws, cudaStream_t st) {
  PackedTc p = {};
  p.n_cols = back ? w.d_in : w.d_out, p.n_sum = back ? w.d_out : w.d_in, p.n_tok = (int)n_tok;
  const TcPlan t = packed_tc_plan(p.n_tok, p.n_cols, p.n_sum);
  packed_tc_carve(t, ad, p.n_tok, p.n_cols, static_cast<char*>(ws), &p);
  p.w = w, p.ad = ad, p.low = low, p.out = out;
  p.M = static_cast<const __nv_bfloat16*>(back ? ad.A : ad.B);
  p.n_tile = t.n_tile, p.m_tiles = t.m_tiles, p.t_tiles = t.t_tiles, p.splits = t.splits, p.split_len = t.split_len;
  p.group_inv = (1ull << 38) / (unsigned)(w.group / 32) + 1;
  CUtensorMap map;
  TB_TRY(make_map_2d(&map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, sizeof(__nv_bfloat16), in, (unsigned long long)p.n_sum,
                     (unsigned long long)p.n_tok, 64, (unsigned)(t.n_tile / 2), CU_TENSOR_MAP_SWIZZLE_128B));
  if (ad.n) {
    k_adapter_runs<<<t.t_tiles, 256, 0, st>>>(ad, p.n_tok, t.n_tile, const_cast<int4*>(p.runs), const_cast<int*>(p.n_runs));
    TB_LAUNCH_CHECK();
  }
  TB_TRY(back ? packed_tc_backward(p, map, t.pairs, st) : packed_tc_forward(p, map, t.pairs, st));
  if (t.splits > 1) {
    const long long n4 = (long long)p.n_tok * p.n_cols / 4;
    const long long nb = (n4 + 255) / 256;
    k_packed_join<<<(unsigned)(nb < 4096 ? nb : 4096), 256, 0, st>>>(reinterpret_cast<const float4*>(p.part), reinterpret_cast<uint2*>(out), n4, t.splits);
    TB_LAUNCH_CHECK();
  }
  return TB_OK;
}

}  // namespace tb
