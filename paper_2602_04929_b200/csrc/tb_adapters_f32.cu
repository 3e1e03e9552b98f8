// The adapters of float activations on the FP32 pipe, with float products and sums: x A_i^T (or dy B_i^T) and the gradients.
// 1024 tokens x 8192, rank 64: 126 us the narrow product (8.5 TFLOP/s; the adapters' rows come from L2 once for every four tokens),
// 86 us a gradient (12 TFLOP/s; shared-memory reads).  30 tokens x 2048, rank 64: 14 and 7 us, latency.
#include "tb_packed.cuh"
#include "tb_pair.cuh"

namespace tb {

// low [n_tok][rank] = in M_i^T for the adapter i of every token (M [adapter][rank][width]), zero for a token without one.
// A CTA has LOW_TOK neighbouring tokens and 64 of the rank: a warp has eight rows of M, the warps that are left and the CTAs of a
// cluster share the width.  A lane's sums run over its columns and are joined at the end, in a fixed order; for each further adapter
// among the tokens the CTA starts over, with the other tokens' rows left out.
enum { LOW_TOK = 4, LOW_ROWS = 8, LOW_CTAS = 4 };  // LOW_CTAS: an SM's share of them to aim at
__global__ void __launch_bounds__(256) k_low_f32(Adapt ad, const float* __restrict__ in, const float* __restrict__ M, long long n_tok,
                                                 int width, int row_warps, float* __restrict__ low) {
  __shared__ float part[8][LOW_TOK * LOW_ROWS];
  __shared__ int own[LOW_TOK];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  uint32_t rank, cs;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
  asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(cs));
  const int r0 = blockIdx.y * 64 + warp % row_warps * LOW_ROWS, along = 8 / row_warps, my = warp / row_warps;
  const long long t0 = (long long)(blockIdx.x / cs) * LOW_TOK;
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
      for (int k = 4 * (32 * ((int)rank * along + my) + lane); k < width; k += 128 * along * (int)cs) {
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
    if (cs > 1)
      cluster_barrier();
    else
      __syncthreads();
    const int i = lane / LOW_ROWS, r = r0 + lane % LOW_ROWS;
    if (rank == 0 && my == 0 && r < ad.rank && own[i] == id) {
      float v = 0.0f;
      for (uint32_t c = 0; c < cs; ++c)
        for (int o = 0; o < along; ++o) {
          const float* at = &part[warp + o * row_warps][lane];
          float q = *at;
          if (c) asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(q) : "r"(map_to_rank(smem_u32(at), c)) : "memory");
          v = c || o ? v + q : q;
        }
      low[(t0 + i) * ad.rank + r] = v;
    }
    if (cs > 1)
      cluster_barrier();  // the sums are read before they are written again, or the CTA leaves
    else
      __syncthreads();
  }
}

// G [adapter][rank][width] = scale_i sum over the tokens t of adapter i of low_t^T in_t; `in` in full or, where T is signed
// char, as 8-bit codes with their scales.  A CTA has 64 columns of one adapter and, as one of a cluster, every cs-th piece of
// G_TOK tokens of its requests; the next piece's values are on their way while one is multiplied.  The CTAs' sums are added in a
// fixed order.
enum { G_TOK = 16, G_COLS = 64 };
template <typename T>
__global__ void __launch_bounds__(256, 2) k_grad_f32(Adapt ad, const T* __restrict__ in, const float* __restrict__ in_scales,
                                                  const float* __restrict__ low, long long n_tok, int width, float* __restrict__ G) {
  __shared__ __align__(16) float ls[G_TOK][128], xs[G_TOK][G_COLS], sums[128][G_COLS];
  uint32_t rank, cs;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
  asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(cs));
  const int id = blockIdx.y, c0 = (int)(blockIdx.x / cs) * G_COLS;
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
  const int n_run = (width + CKPT_RUN - 1) / CKPT_RUN;
  float acc[8][4] = {};
  float lv[8], xv[4];
  // the pieces that this CTA has, one after the other: request j, tokens t0 .. min(e, t0 + G_TOK) - 1
  int j = -1;
  long long t0 = 0, e = 0;
  uint32_t turn = 0;
  auto next = [&]() -> bool {  // the same in the whole CTA
    for (;;) {
      t0 += G_TOK;
      while (t0 >= e) {
        do {
          if (++j >= ad.n_req) return false;
        } while (ad.ids[j] != id);
        t0 = max(0, ad.starts[j]), e = min(n_tok, (long long)ad.starts[j + 1]);
      }
      const uint32_t at = turn;
      turn = turn + 1 == cs ? 0 : turn + 1;
      if (at == rank) return true;
    }
  };
  auto fetch = [&]() {
#pragma unroll
    for (int q = 0; q < 8; ++q) {  // a row of `low` at a time
      const int t = 2 * q + (int)(threadIdx.x >> 7), r = threadIdx.x & 127;
      lv[q] = t0 + t < e && r < ad.rank ? low[(t0 + t) * ad.rank + r] : 0.0f;
    }
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int t = 4 * q + (int)(threadIdx.x >> 6), c = c0 + (int)(threadIdx.x & 63);
      xv[q] = 0.0f;
      if (t0 + t < e && c < width) {
        if constexpr (sizeof(T) == 1)
          xv[q] = (float)in[(t0 + t) * width + c] * in_scales[(t0 + t) * n_run + c / CKPT_RUN];
        else
          xv[q] = in[(t0 + t) * width + c];
      }
    }
  };
  bool more = next();
  if (more) fetch();
  while (more) {
    __syncthreads();
#pragma unroll
    for (int q = 0; q < 8; ++q) ls[2 * q + (threadIdx.x >> 7)][threadIdx.x & 127] = lv[q];
#pragma unroll
    for (int q = 0; q < 4; ++q) xs[4 * q + (threadIdx.x >> 6)][threadIdx.x & 63] = xv[q];
    __syncthreads();
    more = next();
    if (more) fetch();
#pragma unroll
    for (int t = 0; t < G_TOK; ++t) {
      const float4 x = *reinterpret_cast<const float4*>(&xs[t][4 * tx]);
#pragma unroll
      for (int q = 0; q < 8; ++q) {
        if (16 * q >= ad.rank) break;  // ranks from there on are padding
        const float l = ls[t][ty + 16 * q];
        acc[q][0] = fmaf(l, x.x, acc[q][0]), acc[q][1] = fmaf(l, x.y, acc[q][1]);
        acc[q][2] = fmaf(l, x.z, acc[q][2]), acc[q][3] = fmaf(l, x.w, acc[q][3]);
      }
    }
  }
#pragma unroll
  for (int q = 0; q < 8; ++q) *reinterpret_cast<float4*>(&sums[ty + 16 * q][4 * tx]) = make_float4(acc[q][0], acc[q][1], acc[q][2], acc[q][3]);
  if (cs > 1)
    cluster_barrier();
  else
    __syncthreads();
  const float sc = ad.scale[id];
  for (int r = (int)rank * 16 + ty; r < ad.rank; r += 16 * (int)cs) {
    const float* at = &sums[r][4 * tx];
    float4 v = *reinterpret_cast<const float4*>(at);
    if (cs > 1) {
      const uint32_t addr = smem_u32(at);
      for (uint32_t o = 0; o < cs; ++o) {
        float4 q;
        asm volatile("ld.shared::cluster.v4.f32 {%0,%1,%2,%3}, [%4];" : "=f"(q.x), "=f"(q.y), "=f"(q.z), "=f"(q.w) : "r"(map_to_rank(addr, o)) : "memory");
        v.x = o ? v.x + q.x : q.x, v.y = o ? v.y + q.y : q.y, v.z = o ? v.z + q.z : q.z, v.w = o ? v.w + q.w : q.w;
      }
    }
    if (c0 + 4 * tx < width)
      *reinterpret_cast<float4*>(G + ((long long)id * ad.rank + r) * width + c0 + 4 * tx) = make_float4(sc * v.x, sc * v.y, sc * v.z, sc * v.w);
  }
  if (cs > 1) cluster_barrier();  // nobody leaves while its sums are read
}

static cudaLaunchConfig_t clusters(unsigned x, int y, int cs, cudaLaunchAttribute* attr, cudaStream_t st) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(x * cs, (unsigned)y);
  cfg.blockDim = dim3(256);
  cfg.stream = st;
  attr->id = cudaLaunchAttributeClusterDimension;
  attr->val.clusterDim.x = (unsigned)cs;
  attr->val.clusterDim.y = 1;
  attr->val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cfg;
}

tb_status adapter_low_f32(const Adapt& ad, const float* in, const float* M, long long n_tok, int width, float* low, cudaStream_t st) {
  int row_warps = 1;
  while (row_warps < 8 && row_warps * LOW_ROWS < ad.rank) row_warps *= 2;
  const long long tiles = (n_tok + LOW_TOK - 1) / LOW_TOK, zs = (ad.rank + 63) / 64;
  const int sms = sm_count() > 0 ? sm_count() : 148;
  int cs = 1;
  while (cs < 8 && tiles * zs * cs < LOW_CTAS * sms && width / (2 * cs) >= 128 * (8 / row_warps)) cs *= 2;
  cudaLaunchAttribute attr;
  const cudaLaunchConfig_t cfg = clusters((unsigned)tiles, (int)zs, cs, &attr, st);
  TB_CUDA_CHECK(cudaLaunchKernelEx(&cfg, k_low_f32, ad, in, M, n_tok, width, row_warps, low));
  TB_LAUNCH_CHECK();
  return TB_OK;
}

tb_status adapter_grad_f32(const Adapt& ad, const void* in, const float* in_scales, const float* low, long long n_tok, int width,
                            float* G, cudaStream_t st) {
  const int cols = (width + G_COLS - 1) / G_COLS, sms = sm_count() > 0 ? sm_count() : 148;
  int cs = 1;  // requests may have any length, all tokens among them
  while (cs < 8 && (long long)cols * ad.n * cs < 4 * sms && n_tok / (2 * cs) >= G_TOK) cs *= 2;
  cudaLaunchAttribute attr;
  const cudaLaunchConfig_t cfg = clusters((unsigned)cols, ad.n, cs, &attr, st);
  if (in_scales)
    TB_CUDA_CHECK(cudaLaunchKernelEx(&cfg, k_grad_f32<signed char>, ad, static_cast<const signed char*>(in), in_scales, low, n_tok, width, G));
  else
    TB_CUDA_CHECK(cudaLaunchKernelEx(&cfg, k_grad_f32<float>, ad, static_cast<const float*>(in), in_scales, low, n_tok, width, G));
  TB_LAUNCH_CHECK();
  return TB_OK;
}

}  // namespace tb
