// Host side of the tensor-core product with bit-packed weights: tiles and splits, the runs of tokens with one adapter, and the
// sum of the splits.  Preparing 8192 x 8192 with groups of 128 takes 5.5 us, joining 64 tokens x 4096 in splits about 4 us with rank 16
// adapters; both start ahead of their predecessor's end.
#include "tb_packed_decode.cuh"
#include "tb_packed_plan.cuh"

namespace tb {

// What the product kernel wants laid out otherwise, by three kinds of CTAs in one launch: scales and zero-points with the weight rows
// side by side (a CTA transposes 32 x 32 of them), packed rows on a pitch that TMA takes where theirs is none, and the tokens of
// every tile in runs of one adapter.
struct PrepP {
  PackedW w;
  Adapt ad;
  float* st;
  unsigned *zt, *copy;  // copy: nullptr where the rows are taken as they are
  int4* runs;
  int* n_runs;
  int rows_pad, pitch, n_tok, n_tile, sz_ctas, sz_across, copy_ctas;
};
__global__ void __launch_bounds__(256) k_packed_prep(const PrepP p) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  int b = blockIdx.x;
  pdl_trigger();  // the product's CTAs may take their places
  if (b < p.sz_ctas) {
    __shared__ float s[32][33];
    __shared__ unsigned z[32][33];
    const int r0 = (b / p.sz_across) * 32, g0 = (b % p.sz_across) * 32;
    for (int i = warp; i < 32; i += 8) {
      const int r = r0 + i, g = g0 + lane;
      const bool in = r < p.w.d_out && g < p.w.n_g;
      const long long at = (long long)r * p.w.n_g + g;
      const int zero = in ? p.w.zeros[at] : 0;
      s[i][lane] = in ? p.w.scales[at] : 0.0f;
      z[i][lane] = zero_word(zero, p.w.bits);
    }
    __syncthreads();
    for (int i = warp; i < 32; i += 8)
      if (g0 + i < p.w.n_g) {  // rows_pad is a multiple of 32
        const long long at = (long long)(g0 + i) * p.rows_pad + r0 + lane;
        if (p.st) {
          p.st[at] = s[lane][i];
          p.zt[at] = z[lane][i];
        } else {  // the scale's pieces: the first in the upper half
          const float v = s[lane][i], hi = __bfloat162float(__float2bfloat16(v));
          reinterpret_cast<uint2*>(p.zt)[at] = make_uint2(z[lane][i], bf2(__floats2bfloat162_rn(v - hi, hi)));
        }
      }
    pdl_wait();  // whoever waits for this kernel has waited for the one before it, beside which it may have run
    return;
  }
  b -= p.sz_ctas;
  if (b < p.copy_ctas) {
    const long long n = (long long)p.w.d_out * p.pitch;
    for (long long i = (long long)b * 1024 + tid; i < min(n, (long long)(b + 1) * 1024); i += 256) {
      const int r = (int)(i / p.pitch), k = (int)(i - (long long)r * p.pitch);
      p.copy[i] = k < p.w.words ? p.w.packed[(long long)r * p.w.words + k] : 0u;
    }
    pdl_wait();
    return;
  }
  b -= p.copy_ctas;
  __shared__ int own[257];
  __shared__ unsigned first[8], change[8];
  const int t0 = b * p.n_tile, n = min(p.n_tile, p.n_tok - t0);
  own[tid] = tid < n ? adapter_of(p.ad, t0 + tid) : -1;  // tokens without an adapter are in no run
  __syncthreads();
  const bool other = tid == 0 || own[tid - 1] != own[tid];
  const unsigned mf = __ballot_sync(0xffffffffu, other && own[tid] >= 0), mc = __ballot_sync(0xffffffffu, other);
  if (lane == 0) first[warp] = mf, change[warp] = mc;
  __syncthreads();
  int at = __popc(mf & ((1u << lane) - 1u)), all = 0;
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    if (k < warp) at += __popc(first[k]);
    all += __popc(first[k]);
  }
  if (other && own[tid] >= 0) {
    int e = n, k = warp;
    unsigned m = lane == 31 ? 0u : change[warp] & ~((2u << lane) - 1u);
    while (m == 0 && ++k < 8) m = change[k];
    if (m) e = min(n, 32 * k + __ffs(m) - 1);
    p.runs[t0 + at] = make_int4(t0 + tid, t0 + e, own[tid], 0);
  }
  if (tid == 0) p.n_runs[b] = all;
  pdl_wait();
}

// out = the splits' sums, added in their order, and the adapters' share of the token, rounded once; four columns a thread.
__global__ void __launch_bounds__(256) k_packed_join(const float4* part, uint2* out, long long n4, int cols4, int splits, const Adapt ad,
                                                     const float* low, const __nv_bfloat16* M) {
  pdl_wait();
  for (long long i = blockIdx.x * 256ll + threadIdx.x; i < n4; i += gridDim.x * 256ll) {
    float4 s = __ldcs(part + i);
    for (int k = 1; k < splits; ++k) {
      const float4 v = __ldcs(part + k * n4 + i);
      s.x += v.x, s.y += v.y, s.z += v.z, s.w += v.w;
    }
    if (ad.n) {
      const long long t = i / cols4;
      const int id = adapter_of(ad, t);
      if (id >= 0) {
        const uint2* m = reinterpret_cast<const uint2*>(M) + (long long)id * ad.rank * cols4 + (i - t * cols4);
        const float* l = low + t * ad.rank;
        float4 a = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll 8
        for (int r = 0; r < ad.rank; ++r) {
          const uint2 w = m[(long long)r * cols4];
          const float v = l[r];
          a.x = fmaf(v, __uint_as_float(w.x << 16), a.x), a.y = fmaf(v, __uint_as_float(w.x & 0xffff0000u), a.y);
          a.z = fmaf(v, __uint_as_float(w.y << 16), a.z), a.w = fmaf(v, __uint_as_float(w.y & 0xffff0000u), a.w);
        }
        const float f = ad.scale[id];
        s.x = fmaf(f, a.x, s.x), s.y = fmaf(f, a.y, s.y), s.z = fmaf(f, a.z, s.z), s.w = fmaf(f, a.w, s.w);
      }
    }
    const __nv_bfloat162 a = __floats2bfloat162_rn(s.x, s.y), b = __floats2bfloat162_rn(s.z, s.w);
    out[i] = make_uint2(*reinterpret_cast<const unsigned*>(&a), *reinterpret_cast<const unsigned*>(&b));
  }
}

// Tile and splits by an estimate of the clocks, fitted to sweeps of both (64 to 1999 tokens, widths of 1024 to 8192): a stage of 64
// columns (backward there are two, one a piece of the weights) costs its decoding, whatever the tile, and a little for every token, a
// tile 1500 clocks and what its results take, and splits cost writing and adding their float sums.  The adapters' share is further stages of the tile, four slots each (see the
// kernel), or joins the float sums: 64 tokens of 32 requests, rank 64, 8192 x 512, has 64 such stages and takes 70 us with them, 26 us
// joined.
TcPlan packed_tc_plan(const Adapt& ad, int n_tok, int n_cols, int n_sum, bool back) {
  TcPlan best = {};
  double best_cost = 0.0;
  int sms = sm_count();
  if (sms < 2) sms = 148;  // a query where there is no device
  const int pairs = sms / 2, m_tiles = (n_cols + 255) / 256;
  const int top = n_tok >= 256 ? 256 : (n_tok + 31) / 32 * 32;
  for (int n_tile = 32; n_tile <= top; n_tile += 32) {
    const int t_tiles = (n_tok + n_tile - 1) / n_tile;
    for (int splits = 1; splits <= 16; ++splits) {
      const int len = ((n_sum + splits - 1) / splits + 127) / 128 * 128;
      if (splits > 1 && (len < 256 || (long long)len * (splits - 1) >= n_sum)) continue;
      const long long tiles = (long long)m_tiles * t_tiles * splits;
      if (tiles > 0x3fffffff) continue;
      const double waves = (double)((tiles + pairs - 1) / pairs);
      const double stage = 600.0 + 0.4 * n_tile;
      const double plain = waves * (len / 64 * (back ? 2.0 : 1.0) * stage + 1500.0 + 6.0 * n_tile);
      for (int joined = splits > 1; joined <= (splits > 1 || ad.n); ++joined) {
        double cost = plain;
        if (joined) {
          cost += 4000.0 + 8.0 * splits * (double)n_tok * n_cols / 2500.0;
          if (ad.n) cost += 2000.0 + (double)n_tok * n_cols * ad.rank / 2600.0;
        } else if (ad.n) {
          const double runs = min((double)min(n_tile, ad.n_req), 1.0 + (double)ad.n_req * n_tile / n_tok);
          cost += waves * (3000.0 + 1600.0 * ceil(runs * ((ad.rank + 15) / 16) * 2.0 / 4.0));
        }
        if (best.n_tile == 0 || cost < best_cost) {
          best_cost = cost;
          best.n_tile = n_tile, best.m_tiles = m_tiles, best.t_tiles = t_tiles, best.splits = splits, best.split_len = len;
          best.pairs = tiles < pairs ? (int)tiles : pairs, best.joined = joined;
        }
      }
    }
  }
  return best;
}

size_t packed_tc_carve(const TcPlan& t, const PackedW& w, const Adapt& ad, int n_tok, int n_cols, bool back, char* ws, PackedTc* p) {
  Bump b(ws);
  p->rows_pad = (w.d_out + 255) / 256 * 256;  // whole tiles of a CTA pair
  p->pitch = (w.words + 3) / 4 * 4;
  p->st = back ? nullptr : b.take<float>((size_t)w.n_g * p->rows_pad);
  p->zt = b.take<unsigned>((size_t)w.n_g * p->rows_pad * (back ? 2 : 1));
  p->words = p->pitch != w.words ? b.take<unsigned>((size_t)w.d_out * p->pitch) : w.packed;
  p->runs = ad.n && !t.joined ? b.take<int4>(n_tok) : nullptr;
  p->n_runs = ad.n && !t.joined ? b.take<int>(t.t_tiles) : nullptr;
  p->part = t.joined ? b.take<float>((size_t)t.splits * n_tok * n_cols) : nullptr;
  return b.total();
}

// Rows of 32-bit words, `pitch` words apart.
static tb_status words_map(CUtensorMap* map, const unsigned* base, int words, int rows, int pitch, int box_words, int box_rows) {
  EncodeTiledFn enc = encode_tiled_fn();
  if (!enc) return TB_ERR_CUDA;
  const cuuint64_t dims[2] = {(cuuint64_t)words, (cuuint64_t)rows};
  const cuuint64_t strides[1] = {(cuuint64_t)pitch * 4};
  const cuuint32_t box[2] = {(cuuint32_t)box_words, (cuuint32_t)box_rows}, estr[2] = {1, 1};
  const CUtensorMapSwizzle sw = box_words == 8    ? CU_TENSOR_MAP_SWIZZLE_32B
                                : box_words == 16 ? CU_TENSOR_MAP_SWIZZLE_64B
                                : box_words == 32 ? CU_TENSOR_MAP_SWIZZLE_128B
                                                  : CU_TENSOR_MAP_SWIZZLE_NONE;
  return enc(map, CU_TENSOR_MAP_DATA_TYPE_UINT32, 2, const_cast<unsigned*>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, sw,
             CU_TENSOR_MAP_L2_PROMOTION_L2_128B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS
             ? TB_OK
             : TB_ERR_CUDA;
}

tb_status packed_product_tc(const PackedW& w, const Adapt& ad, const __nv_bfloat16* in, long long n_tok, __nv_bfloat16* out,
                            float* low, bool back, void* ws, cudaStream_t st) {
  PackedTc p = {};
  p.n_cols = back ? w.d_in : w.d_out, p.n_sum = back ? w.d_out : w.d_in, p.n_tok = (int)n_tok;
  const TcPlan t = packed_tc_plan(ad, p.n_tok, p.n_cols, p.n_sum, back);
  packed_tc_carve(t, w, ad, p.n_tok, p.n_cols, back, static_cast<char*>(ws), &p);
  p.w = w, p.ad = ad, p.low = low, p.out = out;
  p.M = static_cast<const __nv_bfloat16*>(back ? ad.A : ad.B);
  p.n_tile = t.n_tile, p.m_tiles = t.m_tiles, p.t_tiles = t.t_tiles, p.splits = t.splits, p.split_len = t.split_len;
  CUtensorMap xmap, wmap;
  TB_TRY(make_map_2d(&xmap, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, sizeof(__nv_bfloat16), in, (unsigned long long)p.n_sum,
                     (unsigned long long)p.n_tok, 64, (unsigned)(t.n_tile / 2), CU_TENSOR_MAP_SWIZZLE_128B));
  TB_TRY(words_map(&wmap, p.words, w.words, w.d_out, p.pitch, 4 * w.bits, back ? 64 : 128));
  PrepP q = {};
  q.w = w, q.ad = ad;
  q.st = const_cast<float*>(p.st), q.zt = const_cast<unsigned*>(p.zt);
  q.copy = p.words != w.packed ? const_cast<unsigned*>(p.words) : nullptr;
  q.runs = const_cast<int4*>(p.runs), q.n_runs = const_cast<int*>(p.n_runs);
  q.rows_pad = p.rows_pad, q.pitch = p.pitch, q.n_tok = p.n_tok, q.n_tile = t.n_tile;
  q.sz_across = (w.n_g + 31) / 32;
  q.sz_ctas = q.sz_across * (p.rows_pad / 32);
  q.copy_ctas = q.copy ? (int)(((long long)w.d_out * p.pitch + 1023) / 1024) : 0;
  const dim3 prep((unsigned)(q.sz_ctas + q.copy_ctas + (p.n_runs ? t.t_tiles : 0)));
  // x A^T: before the product, which adds the adapters' share itself where its sums are not joined; else beside it
  const __nv_bfloat16* lowM = static_cast<const __nv_bfloat16*>(back ? ad.B : ad.A);
  const bool late = ad.n && t.joined && adapter_low_in_small_tiles(ad, p.n_tok, p.n_sum);
  if (ad.n && !late) TB_TRY(adapter_low_bf16(ad, in, lowM, p.n_tok, p.n_sum, low, false, st));
  if (ad.n && !late)  // beside that kernel, which started when all before it had ended
    TB_CUDA_CHECK(launch_pdl(k_packed_prep, prep, dim3(256), 0, st, q));
  else
    k_packed_prep<<<prep, 256, 0, st>>>(q);
  TB_LAUNCH_CHECK();
  TB_TRY(back ? packed_tc_backward(p, xmap, wmap, t.pairs, st) : packed_tc_forward(p, xmap, wmap, t.pairs, st));
  if (late) TB_TRY(adapter_low_bf16(ad, in, lowM, p.n_tok, p.n_sum, low, true, st));
  if (t.joined) {
    const long long n4 = (long long)p.n_tok * p.n_cols / 4;
    const long long nb = (n4 + 255) / 256;
    TB_CUDA_CHECK(launch_pdl(k_packed_join, dim3((unsigned)(nb < 4096 ? nb : 4096)), dim3(256), 0, st, reinterpret_cast<const float4*>(p.part),
                             reinterpret_cast<uint2*>(out), n4, p.n_cols / 4, t.splits, ad, low, p.M));
    TB_LAUNCH_CHECK();
  }
  return TB_OK;
}

}  // namespace tb
