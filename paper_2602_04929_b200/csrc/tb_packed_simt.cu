// Products with bit-packed weights on the FP32 pipe: every case of tb_packed_linear and its gradients, with float products
// and sums.  y = x Q^T and dx = dy Q are one kernel, a 64 x 64 tile of the result by 256 threads; the adapters' share is
// added to the finished sums, token by token, since neighbouring tokens may have different adapters.
#include "tb_packed.cuh"

namespace tb {

template <typename T>
__device__ __forceinline__ T from_float(float v) {
  return v;
}
template <>
__device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float v) {
  return __float2bfloat16(v);
}

enum { S_TILE = 64, S_BK = 32 };

// out [n_tok][n_cols] = in [n_tok][n_sum] times Q^T (forward: columns are Q's rows) or Q (BACK: columns are Q's columns), plus
// scale low M of the token's adapter, M [adapter][rank][n_cols].
template <typename T, bool BACK>
__global__ void __launch_bounds__(256) k_packed_simt(PackedW w, Adapt ad, const T* __restrict__ in, long long n_tok,
                                                     T* __restrict__ out, const float* __restrict__ low,
                                                     const T* __restrict__ M) {
  __shared__ float xs[S_BK][S_TILE + 4], ws[S_BK][S_TILE + 4];
  const int n_cols = BACK ? w.d_in : w.d_out, n_sum = BACK ? w.d_out : w.d_in;
  const int c0 = blockIdx.x * S_TILE;
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
  for (long long t0 = (long long)blockIdx.y * S_TILE; t0 < n_tok; t0 += (long long)gridDim.y * S_TILE) {
    float acc[4][4] = {};
    for (int k0 = 0; k0 < n_sum; k0 += S_BK) {
      for (int e = threadIdx.x; e < S_TILE * S_BK; e += 256) {
        const int k = e % S_BK, t = e / S_BK;
        xs[k][t] = t0 + t < n_tok && k0 + k < n_sum ? cvt<float>(in[(t0 + t) * n_sum + k0 + k]) : 0.0f;
      }
      {
        // 8 codes a thread: of one row, along the sum (forward) or along the columns (BACK)
        const int row = BACK ? k0 + threadIdx.x / 8 : c0 + threadIdx.x / 4;
        const int col = BACK ? c0 + 8 * (threadIdx.x % 8) : k0 + 8 * (threadIdx.x % 4);
        float v[8] = {};
        if (row < w.d_out && col < w.d_in) {
          unsigned c[8];
          unpack_codes(w.packed + (long long)row * w.words, w.words, col, w.bits, c);
          const long long g = (long long)row * w.n_g + col / w.group;
          const float s = w.scales[g];
          const int z = w.zeros[g];
#pragma unroll
          for (int i = 0; i < 8; ++i) v[i] = s * (float)((int)c[i] - z);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          if (BACK)
            ws[threadIdx.x / 8][8 * (threadIdx.x % 8) + i] = v[i];
          else
            ws[8 * (threadIdx.x % 4) + i][threadIdx.x / 4] = v[i];
        }
      }
      __syncthreads();
#pragma unroll
      for (int k = 0; k < S_BK; ++k) {
        float a[4], b[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) a[i] = xs[k][4 * ty + i], b[i] = ws[k][4 * tx + i];
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int j = 0; j < 4; ++j) acc[i][j] = fmaf(a[i], b[j], acc[i][j]);
      }
      __syncthreads();
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const long long t = t0 + 4 * ty + i;
      if (t >= n_tok) continue;
      const int id = ad.n ? adapter_of(ad, t) : -1;
      if (id >= 0) {
        const float sc = ad.scale[id];
        const T* m = M + (long long)id * ad.rank * n_cols;
        for (int r = 0; r < ad.rank; ++r) {
          const float v = sc * low[t * ad.rank + r];
#pragma unroll
          for (int j = 0; j < 4; ++j)
            if (c0 + 4 * tx + j < n_cols) acc[i][j] = fmaf(v, cvt<float>(m[(long long)r * n_cols + c0 + 4 * tx + j]), acc[i][j]);
        }
      }
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (c0 + 4 * tx + j < n_cols) out[t * n_cols + c0 + 4 * tx + j] = from_float<T>(acc[i][j]);
    }
  }
}

// low [n_tok][rank] = in M_i^T for the adapter i of every token (M [adapter][rank][width]), zero for a token without one.
// A CTA has a token: its warps share the rank's rows.
template <typename T>
__global__ void __launch_bounds__(256) k_low_simt(Adapt ad, const T* __restrict__ in, const T* __restrict__ M, long long n_tok,
                                                  int width, float* __restrict__ low) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  for (long long t = blockIdx.x; t < n_tok; t += gridDim.x) {
    const int id = adapter_of(ad, t);
    for (int r = warp; r < ad.rank; r += 8) {
      float s = 0.0f;
      if (id >= 0) {
        const T* m = M + ((long long)id * ad.rank + r) * width;
        for (int k = lane; k < width; k += 32) s = fmaf(cvt<float>(in[t * width + k]), cvt<float>(m[k]), s);
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
      }
      if (lane == 0) low[t * ad.rank + r] = s;
    }
  }
}

// G [adapter][rank][width] = scale_i sum over the tokens t of adapter i of low_t^T in_t; `in` in full (T) or, where T is signed
// char, as 8-bit codes with their scales.  A CTA has 64 columns of one adapter; tokens of other adapters are skipped.
enum { G_TOK = 16 };
template <typename T>
__global__ void __launch_bounds__(256) k_adapter_grad_simt(Adapt ad, const T* __restrict__ in, const float* __restrict__ in_scales,
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
            v = cvt<float>(in[(t0 + t) * width + c0 + c]);
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

template <typename T>
static tb_status product(const PackedW& w, const Adapt& ad, const T* in, long long n_tok, T* out, const float* low, bool back,
                         cudaStream_t st) {
  const int n_cols = back ? w.d_in : w.d_out;
  const long long rows = (n_tok + S_TILE - 1) / S_TILE;
  const dim3 grid((n_cols + S_TILE - 1) / S_TILE, (unsigned)(rows < 65535 ? rows : 65535));
  if (back)
    k_packed_simt<T, true><<<grid, 256, 0, st>>>(w, ad, in, n_tok, out, low, static_cast<const T*>(ad.A));
  else
    k_packed_simt<T, false><<<grid, 256, 0, st>>>(w, ad, in, n_tok, out, low, static_cast<const T*>(ad.B));
  TB_LAUNCH_CHECK();
  return TB_OK;
}

tb_status packed_product_simt(const PackedW& w, const Adapt& ad, const void* in, tb_dtype type, long long n_tok, void* out,
                              const float* low, bool back, cudaStream_t st) {
  if (type == TB_BF16)
    return product(w, ad, static_cast<const __nv_bfloat16*>(in), n_tok, static_cast<__nv_bfloat16*>(out), low, back, st);
  return product(w, ad, static_cast<const float*>(in), n_tok, static_cast<float*>(out), low, back, st);
}

tb_status adapter_low_simt(const Adapt& ad, const void* in, const void* M, tb_dtype type, long long n_tok, int width, float* low,
                           cudaStream_t st) {
  const unsigned nb = (unsigned)(n_tok < 65535 ? n_tok : 65535);
  if (type == TB_BF16)
    k_low_simt<<<nb, 256, 0, st>>>(ad, static_cast<const __nv_bfloat16*>(in), static_cast<const __nv_bfloat16*>(M), n_tok, width, low);
  else
    k_low_simt<<<nb, 256, 0, st>>>(ad, static_cast<const float*>(in), static_cast<const float*>(M), n_tok, width, low);
  TB_LAUNCH_CHECK();
  return TB_OK;
}

tb_status adapter_grad_simt(const Adapt& ad, const void* in, const float* in_scales, tb_dtype type, const float* low,
                            long long n_tok, int width, float* G, cudaStream_t st) {
  const dim3 grid((width + 63) / 64, ad.n);
  if (in_scales)
    k_adapter_grad_simt<<<grid, 256, 0, st>>>(ad, static_cast<const signed char*>(in), in_scales, low, n_tok, width, G);
  else if (type == TB_BF16)
    k_adapter_grad_simt<<<grid, 256, 0, st>>>(ad, static_cast<const __nv_bfloat16*>(in), in_scales, low, n_tok, width, G);
  else
    k_adapter_grad_simt<<<grid, 256, 0, st>>>(ad, static_cast<const float*>(in), in_scales, low, n_tok, width, G);
  TB_LAUNCH_CHECK();
  return TB_OK;
}

}  // namespace tb
