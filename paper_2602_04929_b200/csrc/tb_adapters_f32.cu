// The adapters of float activations on the FP32 pipe, with float products and sums: x A_i^T (or dy B_i^T) and the gradients.
#include "tb_packed.cuh"

namespace tb {

// low [n_tok][rank] = in M_i^T for the adapter i of every token (M [adapter][rank][width]), zero for a token without one.
// A CTA has LOW_TOK neighbouring tokens and 64 of the rank: a warp has eight rows of M, the warps that are left share the width.  A
// lane's sums run over its columns and are joined at the end, in a fixed order; for each further adapter among the tokens the
// CTA starts over, with the other tokens' rows left out.
enum { LOW_TOK = 4, LOW_ROWS = 8 };
__global__ void __launch_bounds__(256) k_low_f32(Adapt ad, const float* __restrict__ in, const float* __restrict__ M, long long n_tok,
                                                 int width, int row_warps, float* __restrict__ low) {
  __shared__ float part[8][LOW_TOK * LOW_ROWS];
  __shared__ int own[LOW_TOK];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int r0 = blockIdx.y * 64 + warp % row_warps * LOW_ROWS, along = 8 / row_warps, my = warp / row_warps;
  const long long t0 = (long long)blockIdx.x * LOW_TOK;
  if (threadIdx.x < LOW_TOK) own[threadIdx.x] = t0 + threadIdx.x < n_tok ? adapter_of(ad, t0 + threadIdx.x) : -2;
  __syncthreads();
  for (int a = 0; a < LOW_TOK; ++a) {
    const int id = own[a];
    bool first = id != -2;
    for (int b = 0; b < a; ++b) first = first && own[b] != id;
    if (!first) continue;  // the same in the whole CTA
    float acc[LOW_TOK][LOW_ROWS] = {};
    if (id >= 0 && r0 < ad.rank) {
      const float* m = M + ((long long)id * ad.rank + r0) * width;
      for (int k = 4 * (32 * my + lane); k < width; k += 128 * along) {
        float4 x[LOW_TOK];
#pragma unroll
        for (int i = 0; i < LOW_TOK; ++i)
          x[i] = own[i] == id ? *reinterpret_cast<const float4*>(in + (t0 + i) * width + k) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
        for (int r = 0; r < LOW_ROWS; ++r) {
          const float4 y = *reinterpret_cast<const float4*>(m + (long long)r * width + k);
#pragma unroll
          for (int i = 0; i < LOW_TOK; ++i)
            acc[i][r] = fmaf(x[i].w, y.w, fmaf(x[i].z, y.z, fmaf(x[i].y, y.y, fmaf(x[i].x, y.x, acc[i][r]))));
        }
      }
    }
#pragma unroll
    for (int i = 0; i < LOW_TOK; ++i)
#pragma unroll
      for (int r = 0; r < LOW_ROWS; ++r) {
        float v = acc[i][r];
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
        if (lane == i * LOW_ROWS + r) part[warp][lane] = v;
      }
    __syncthreads();
    const int i = lane / LOW_ROWS, r = r0 + lane % LOW_ROWS;
    if (my == 0 && r < ad.rank && own[i] == id) {
      float v = part[warp][lane];
      for (int o = 1; o < along; ++o) v += part[warp + o * row_warps][lane];
      low[(t0 + i) * ad.rank + r] = v;
    }
    __syncthreads();
  }
}

// G [adapter][rank][width] = scale_i sum over the tokens t of adapter i of low_t^T in_t; `in` in full or, where T is signed
// char, as 8-bit codes with their scales.  A CTA has 64 columns of one adapter; tokens of other adapters are skipped.
enum { G_TOK = 16 };
template <typename T>
__global__ void __launch_bounds__(256) k_grad_f32(Adapt ad, const T* __restrict__ in, const float* __restrict__ in_scales,
                                                           const float* __restrict__ low, long long n_tok, int width,
                                                           float* __restrict__ G) {
  __shared__ float ls[G_TOK][128], xs[G_TOK][64];
  const int id = blockIdx.y, c0 = blockIdx.x * 64;
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
  const int n_run = (width + CKPT_RUN - 1) / CKPT_RUN;
  float acc[8][4] = {};
  for (int j = 0; j < ad.n_req; ++j) {
    if (ad.ids[j] != id) continue;
    const long long b = max(0, ad.starts[j]), e = min(n_tok, (long long)ad.starts[j + 1]);
    for (long long t0 = b; t0 < e; t0 += G_TOK) {
      for (int q = threadIdx.x; q < G_TOK * ad.rank; q += 256) {
        const int t = q / ad.rank, r = q - t * ad.rank;
        ls[t][r] = t0 + t < e ? low[(t0 + t) * ad.rank + r] : 0.0f;
      }
      for (int q = threadIdx.x; q < G_TOK * 64; q += 256) {
        const int t = q >> 6, c = q & 63;
        float v = 0.0f;
        if (t0 + t < e && c0 + c < width) {
          if constexpr (sizeof(T) == 1)
            v = (float)in[(t0 + t) * width + c0 + c] * in_scales[(t0 + t) * n_run + (c0 + c) / CKPT_RUN];
          else
            v = in[(t0 + t) * width + c0 + c];
        }
        xs[t][c] = v;
      }
      __syncthreads();
#pragma unroll
      for (int t = 0; t < G_TOK; ++t) {
        float x[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = xs[t][4 * tx + i];
#pragma unroll
        for (int q = 0; q < 8; ++q) {
          const int r = ty + 16 * q;
          if (r < ad.rank) {
            const float l = ls[t][r];
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[q][i] = fmaf(l, x[i], acc[q][i]);
          }
        }
      }
      __syncthreads();
    }
  }
  const float sc = ad.scale[id];
#pragma unroll
  for (int q = 0; q < 8; ++q) {
    const int r = ty + 16 * q;
    if (r >= ad.rank) continue;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (c0 + 4 * tx + i < width) G[((long long)id * ad.rank + r) * width + c0 + 4 * tx + i] = sc * acc[q][i];
  }
}

tb_status adapter_low_f32(const Adapt& ad, const float* in, const float* M, long long n_tok, int width, float* low, cudaStream_t st) {
  int row_warps = 1;
  while (row_warps < 8 && row_warps * LOW_ROWS < ad.rank) row_warps *= 2;
  k_low_f32<<<dim3((unsigned)((n_tok + LOW_TOK - 1) / LOW_TOK), (unsigned)((ad.rank + 63) / 64)), 256, 0, st>>>(ad, in, M, n_tok, width,
                                                                                                             row_warps, low);
  TB_LAUNCH_CHECK();
  return TB_OK;
}

tb_status adapter_grad_f32(const Adapt& ad, const void* in, const float* in_scales, const float* low, long long n_tok, int width,
                            float* G, cudaStream_t st) {
  const dim3 grid((width + 63) / 64, ad.n);
  if (in_scales)
    k_grad_f32<<<grid, 256, 0, st>>>(ad, static_cast<const signed char*>(in), in_scales, low, n_tok, width, G);
  else
    k_grad_f32<<<grid, 256, 0, st>>>(ad, static_cast<const float*>(in), in_scales, low, n_tok, width, G);
  TB_LAUNCH_CHECK();
  return TB_OK;
}

}  // namespace tb
