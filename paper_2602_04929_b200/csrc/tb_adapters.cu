// Low-rank adapters of many requests, bf16 activations: the narrow products x A_i^T (k_adapter_low) and the gradients of the
// adapters' matrices (k_adapter_grad), both on mma.sync: a narrow product has a few dozen products for every value it reads, far
// below what the tensor cores need to be kept busy, so both are bound by reading the activations (or, with a token or two for an
// adapter, the adapters) once.
#include "tb_packed.cuh"
#include "tb_pair.cuh"

namespace tb {

__device__ __forceinline__ void mma_bf16(float (&c)[4], unsigned a0, unsigned a1, unsigned a2, unsigned a3, unsigned b0, unsigned b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
               : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ float ld_cluster(uint32_t addr) {
  float v;
  asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(addr) : "memory");
  return v;
}

// ------------------------------------------------------------------------------------------ x A_i^T
//
// A CTA has TT tokens (64, or 16 where there are few), one of the adapters that they have, up to 64 of its rank and, as one of a
// cluster, a share of the contraction; its warps split the tokens into MT x 16 and the contraction further.  Operands go from
// global memory straight into fragments: a lane loads 16 bytes of a row, eight neighbouring columns, and which columns a fragment
// calls k = 0 .. 15 does not matter as long as both operands agree.  Rows of other adapters are not read.  The warps' and the CTAs'
// sums are added in a fixed order.

template <int MT, int NT>
__global__ void __launch_bounds__(256) k_adapter_low(Adapt ad, const __nv_bfloat16* __restrict__ in, const __nv_bfloat16* __restrict__ M,
                                                     int n_tok, int width, float* __restrict__ low) {
  constexpr int TT = MT == 2 ? 64 : 16, WT = TT / (16 * MT), KG = 8 / WT, R = 8 * NT, PITCH = R + 1;
  __shared__ int own[TT], pick[3];
  __shared__ float sum[TT * PITCH];
  uint32_t rank, cs;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
  asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(cs));
  pdl_trigger();  // a product that only needs these sums at its end may start beside
  const int t0 = (blockIdx.x / cs) * TT, r0 = blockIdx.z * 64;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (threadIdx.x < TT) own[threadIdx.x] = t0 + (int)threadIdx.x < n_tok ? adapter_of(ad, t0 + threadIdx.x) : -2;
  if (threadIdx.x == 0) pick[0] = -1, pick[1] = 0;
  __syncthreads();
  // the blockIdx.y-th adapter among the tile's, by its first token
  if (threadIdx.x < 32) {
    int before = 0;
#pragma unroll
    for (int b = 0; b < TT; b += 32) {
      const int i = b + lane;
      bool first = i < TT && own[i < TT ? i : 0] >= 0;
      for (int k = 0; first && k < i; ++k) first = own[k] != own[i];
      const unsigned m = __ballot_sync(0xffffffffu, first);
      const int at = before + __popc(m & ((1u << lane) - 1u));
      if (first && at == (int)blockIdx.y) pick[0] = own[i];
      before += __popc(m);
    }
  }
  __syncthreads();
  if (blockIdx.y == 0 && rank == 0)  // tokens without an adapter
    for (int e = threadIdx.x; e < TT * R; e += 256) {
      const int t = e / R, r = r0 + e % R;
      if (own[t] == -1 && r < ad.rank) low[(long long)(t0 + t) * ad.rank + r] = 0.0f;
    }
  const int id = pick[0];
  if (id < 0) return;  // the same in every CTA of the cluster
  const int g = lane >> 2, q = lane & 3, tg = warp % WT, kg = warp / WT;
  const __nv_bfloat16* xr[2 * MT];
  const __nv_bfloat16* mr[NT];
#pragma unroll
  for (int i = 0; i < 2 * MT; ++i) {
    const int t = tg * 16 * MT + 8 * i + g;
    xr[i] = own[t] == id ? in + (long long)(t0 + t) * width : nullptr;
  }
#pragma unroll
  for (int n = 0; n < NT; ++n) mr[n] = r0 + 8 * n + g < ad.rank ? M + ((long long)id * ad.rank + r0 + 8 * n + g) * width : nullptr;
  float acc[MT][NT][4] = {};
  const int steps = (width + 31) / 32, per = (steps + (int)cs * KG - 1) / ((int)cs * KG);
  const int s0 = ((int)rank * KG + kg) * per, s1 = min(steps, s0 + per);
#pragma unroll 4
  for (int s = s0; s < s1; ++s) {
    const int k = 32 * s + 8 * q;
    const bool in_k = k < width;
    uint4 x[2 * MT], m[NT];
#pragma unroll
    for (int i = 0; i < 2 * MT; ++i) x[i] = in_k && xr[i] ? __ldg(reinterpret_cast<const uint4*>(xr[i] + k)) : make_uint4(0, 0, 0, 0);
#pragma unroll
    for (int n = 0; n < NT; ++n) m[n] = in_k && mr[n] ? __ldg(reinterpret_cast<const uint4*>(mr[n] + k)) : make_uint4(0, 0, 0, 0);
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        mma_bf16(acc[i][n], x[2 * i].x, x[2 * i + 1].x, x[2 * i].y, x[2 * i + 1].y, m[n].x, m[n].y);
        mma_bf16(acc[i][n], x[2 * i].z, x[2 * i + 1].z, x[2 * i].w, x[2 * i + 1].w, m[n].z, m[n].w);
      }
  }
  // the warps along the contraction, one after the other
  for (int k = 0; k < KG; ++k) {
    if (kg == k) {
#pragma unroll
      for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            float* o = sum + (tg * 16 * MT + 16 * i + g + 8 * (c >> 1)) * PITCH + 8 * n + 2 * q + (c & 1);
            *o = k ? *o + acc[i][n][c] : acc[i][n][c];
          }
    }
    __syncthreads();
  }
  if (cs > 1) cluster_barrier();
  const uint32_t mine = smem_u32(sum);
  for (int e = threadIdx.x + 256 * rank; e < TT * R; e += 256 * cs) {
    const int t = e / R, r = e % R;
    if (own[t] != id || r0 + r >= ad.rank) continue;
    float v = 0.0f;
    for (uint32_t c = 0; c < cs; ++c) {
      const float p = cs > 1 ? ld_cluster(map_to_rank(mine + 4u * (t * PITCH + r), c)) : sum[t * PITCH + r];
      v = c ? v + p : p;
    }
    low[(long long)(t0 + t) * ad.rank + r0 + r] = v;
  }
  if (cs > 1) cluster_barrier();  // nobody leaves while its sums are read
}

template <int MT, int NT>
static tb_status launch_low(const Adapt& ad, const __nv_bfloat16* in, const __nv_bfloat16* M, int n_tok, int width, float* low,
                            cudaStream_t st) {
  constexpr int TT = MT == 2 ? 64 : 16;
  const int tiles = (n_tok + TT - 1) / TT, zs = (ad.rank + 63) / 64;
  const int ys = min(TT, min(ad.n_req, ad.n));
  // clusters along the contraction until about two CTAs an SM: adapters are counted as if the requests were spread over the tiles
  const int sms = sm_count() > 0 ? sm_count() : 148;
  const long long ctas = (long long)zs * (tiles + min((long long)tiles * (ys - 1), (long long)ad.n_req));
  int cs = 1;
  while (cs < 8 && ctas * cs * 2 <= 2 * sms && width / (2 * cs) >= 512) cs *= 2;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(tiles * cs), (unsigned)ys, (unsigned)zs);
  cfg.blockDim = dim3(256);
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = (unsigned)cs;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  TB_CUDA_CHECK(cudaLaunchKernelEx(&cfg, k_adapter_low<MT, NT>, ad, in, M, n_tok, width, low));
  TB_LAUNCH_CHECK();
  return TB_OK;
}

// low [n_tok][rank] = in M_i^T for the adapter i of every token, zero for a token without one.
tb_status adapter_low_bf16(const Adapt& ad, const __nv_bfloat16* in, const __nv_bfloat16* M, int n_tok, int width, float* low,
                           cudaStream_t st) {
  // With 64 tokens a tile the adapters are read once for 64 tokens; with 16 there are more CTAs and less is computed for rows of
  // other adapters.
  const bool few = n_tok <= 512 || (long long)n_tok / ad.n_req < 48;
  if (ad.rank <= 8) return few ? launch_low<1, 1>(ad, in, M, n_tok, width, low, st) : launch_low<2, 1>(ad, in, M, n_tok, width, low, st);
  if (ad.rank <= 16) return few ? launch_low<1, 2>(ad, in, M, n_tok, width, low, st) : launch_low<2, 2>(ad, in, M, n_tok, width, low, st);
  if (ad.rank <= 32) return few ? launch_low<1, 4>(ad, in, M, n_tok, width, low, st) : launch_low<2, 4>(ad, in, M, n_tok, width, low, st);
  return few ? launch_low<1, 8>(ad, in, M, n_tok, width, low, st) : launch_low<2, 8>(ad, in, M, n_tok, width, low, st);
}

// ------------------------------------------------------------------------------------------ gradients
//
// G_i [rank][width] = scale_i sum over i's tokens of low_t^T in_t.  A CTA has 128 columns of one adapter and, as one of a cluster,
// every cs-th piece of 64 tokens; rows are the rank (M), columns N, tokens the contraction.  The input's tile goes to shared
// memory by cp.async (8-bit codes through registers, as bf16 integers) and is read with transposing loads; low is split into three
// bf16 pieces, all 24 bits of it, times the codes' scale of its token and these 128 columns.  The CTAs' sums are added in a fixed
// order through distributed shared memory.

enum { AG_TOK = 64, AG_COLS = 128, AG_PIECES = 3 };

__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src, bool in) {
  const int n = in ? 16 : 0;  // the rest is filled with zeros
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(n) : "memory");
}
__device__ __forceinline__ void ldsm4(uint32_t addr, unsigned (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldsm4_t(uint32_t addr, unsigned (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}

// RT: rows of the rank in sixteens.  Shared memory: two input tiles [64 tokens][128 columns] of bf16, the pieces of low
// [piece][16 RT][64 tokens], both in 16-byte units swizzled by their row.
template <int RT, bool EIGHT>
__global__ void __launch_bounds__(256) k_adapter_grad(Adapt ad, const void* __restrict__ in, const float* __restrict__ in_scales,
                                                      const float* __restrict__ low, int n_tok, int width, float* __restrict__ G) {
  constexpr int ROWS = 16 * RT;
  extern __shared__ __align__(128) unsigned char ag_smem[];
  __shared__ int2 piece[256];
  __shared__ int n_piece, wsum[8];
  const uint32_t xs = smem_u32(ag_smem), ls = xs + 2 * AG_TOK * AG_COLS * 2;
  float* sum = reinterpret_cast<float*>(ag_smem);  // after the last tile: [ROWS][128]
  uint32_t rank, cs;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
  asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(cs));
  const int c0 = (blockIdx.x / cs) * AG_COLS, id = blockIdx.y;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int n_run = (width + CKPT_RUN - 1) / CKPT_RUN;
  float acc[RT][2][4] = {};

  auto load_x = [&](int buf, int t, int n) {  // 64 tokens from t on, n of them inside
    const uint32_t dst = xs + buf * (AG_TOK * AG_COLS * 2);
    if constexpr (!EIGHT) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int e = tid + 256 * i, row = e >> 4, u = e & 15;
        const bool ok = row < n && c0 + 8 * u < width;
        const __nv_bfloat16* src = static_cast<const __nv_bfloat16*>(in) + (ok ? (long long)(t + row) * width + c0 + 8 * u : 0);
        cp_async16(dst + row * 256 + ((u ^ (row & 7)) << 4), src, ok);
      }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  uint4 codes[2];
  auto fetch_codes = [&](int t, int n) {
    if constexpr (EIGHT) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int e = tid + 256 * i, row = e >> 3, u = e & 7;
        const bool ok = row < n && c0 + 16 * u < width;
        codes[i] = ok ? __ldcs(reinterpret_cast<const uint4*>(static_cast<const signed char*>(in) + (long long)(t + row) * width + c0 + 16 * u))
                      : make_uint4(0, 0, 0, 0);
      }
    }
  };
  auto store_codes = [&](int buf) {
    if constexpr (EIGHT) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int e = tid + 256 * i, row = e >> 3, u = e & 7;
        const unsigned w[4] = {codes[i].x, codes[i].y, codes[i].z, codes[i].w};
        unsigned o[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const unsigned v = w[k >> 1] >> (16 * (k & 1));
          const __nv_bfloat162 b = __floats2bfloat162_rn((float)(signed char)(v & 0xffu), (float)(signed char)((v >> 8) & 0xffu));
          o[k] = *reinterpret_cast<const unsigned*>(&b);
        }
#pragma unroll
        for (int h = 0; h < 2; ++h)
          *reinterpret_cast<uint4*>(ag_smem + buf * (AG_TOK * AG_COLS * 2) + row * 256 + (((2 * u + h) ^ (row & 7)) << 4)) =
              make_uint4(o[4 * h], o[4 * h + 1], o[4 * h + 2], o[4 * h + 3]);
      }
    }
  };
  // a thread has a token and every fourth group of 4 of the rank
  const int lt = tid & 63, lq = tid >> 6;
  float4 lv[RT];
  auto fetch_low = [&](int t, int n) {
    const bool ok = lt < n;
    float f = 1.0f;
    if (EIGHT && ok) f = __ldg(in_scales + (long long)(t + lt) * n_run + c0 / CKPT_RUN);
#pragma unroll
    for (int k = 0; k < RT; ++k) {
      const int r = 16 * k + 4 * lq;
      float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
      if (ok && r < ad.rank) {
        v = *reinterpret_cast<const float4*>(low + (long long)(t + lt) * ad.rank + r);
        if (EIGHT) v.x *= f, v.y *= f, v.z *= f, v.w *= f;
      }
      lv[k] = v;
    }
  };
  auto store_low = [&]() {
#pragma unroll
    for (int k = 0; k < RT; ++k) {
      const float v[4] = {lv[k].x, lv[k].y, lv[k].z, lv[k].w};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int r = 16 * k + 4 * lq + i;
        float left = v[i];
#pragma unroll
        for (int p = 0; p < AG_PIECES; ++p) {
          const __nv_bfloat16 b = __float2bfloat16(left);
          const float f = __bfloat162float(b);
          left = fabsf(f) <= 3.3895e38f ? left - f : 0.0f;  // nothing is left of what is not finite
          *reinterpret_cast<__nv_bfloat16*>(ag_smem + 2 * AG_TOK * AG_COLS * 2 + ((p * ROWS + r) << 7) + (((lt >> 3) ^ (r & 7)) << 4) + 2 * (lt & 7)) = b;
        }
      }
    }
  };

  for (int j0 = 0; j0 < ad.n_req; j0 += 256) {
    // the adapter's requests among these 256, in their order
    int b = 0, e = 0;
    if (j0 + tid < ad.n_req && ad.ids[j0 + tid] == id) {
      b = max(0, ad.starts[j0 + tid]);
      e = min(n_tok, ad.starts[j0 + tid + 1]);
    }
    const unsigned m = __ballot_sync(0xffffffffu, e > b);
    if (lane == 0) wsum[warp] = __popc(m);
    __syncthreads();
    int at = __popc(m & ((1u << lane) - 1u)), all = 0;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      if (k < warp) at += wsum[k];
      all += wsum[k];
    }
    if (e > b) piece[at] = make_int2(b, e);
    if (tid == 0) n_piece = all;
    __syncthreads();
    // this CTA's pieces of 64 tokens: every cs-th, counted through these requests
    int rq = 0, t = 0;
    auto advance = [&](int n) {  // n pieces on from (rq, t)
      while (rq < n_piece) {
        const int have = (piece[rq].y - t + AG_TOK - 1) / AG_TOK;
        if (n < have) {
          t += n * AG_TOK;
          return;
        }
        n -= have;
        if (++rq < n_piece) t = piece[rq].x;
      }
    };
    if (n_piece > 0) t = piece[0].x;
    advance((int)rank);
    int buf = 0;
    if (rq < n_piece) {
      const int n = min(AG_TOK, piece[rq].y - t);
      load_x(0, t, n);
      fetch_codes(t, n);
      fetch_low(t, n);
    }
    while (rq < n_piece) {
      store_low();
      store_codes(buf);
      advance((int)cs);
      const bool more = rq < n_piece;
      const int n = more ? min(AG_TOK, piece[rq].y - t) : 0;
      if (more) {
        load_x(buf ^ 1, t, n);
        fetch_codes(t, n);
        fetch_low(t, n);
        asm volatile("cp.async.wait_group 1;" ::: "memory");
      } else {
        asm volatile("cp.async.wait_group 0;" ::: "memory");
      }
      __syncthreads();
      const uint32_t xb = xs + buf * (AG_TOK * AG_COLS * 2);
#pragma unroll
      for (int kk = 0; kk < AG_TOK / 16; ++kk) {
        unsigned x[4];  // b0, b1 of the warp's two column tiles
        {
          const int row = 16 * kk + (lane & 15), u = 2 * warp + (lane >> 4);
          ldsm4_t(xb + row * 256 + ((u ^ (row & 7)) << 4), x);
        }
#pragma unroll
        for (int p = 0; p < AG_PIECES; ++p)
#pragma unroll
          for (int k = 0; k < RT; ++k) {
            unsigned a[4];
            const int r = 16 * k + (lane & 7) + 8 * ((lane >> 3) & 1), u = 2 * kk + (lane >> 4);
            ldsm4(ls + ((p * ROWS + r) << 7) + ((u ^ (r & 7)) << 4), a);
            mma_bf16(acc[k][0], a[0], a[1], a[2], a[3], x[0], x[1]);
            mma_bf16(acc[k][1], a[0], a[1], a[2], a[3], x[2], x[3]);
          }
      }
      __syncthreads();
      buf ^= 1;
    }
  }
  // (every thread is past its last tile: the sums may take its place)
  const int g = lane >> 2, q = lane & 3;
#pragma unroll
  for (int k = 0; k < RT; ++k)
#pragma unroll
    for (int n = 0; n < 2; ++n)
#pragma unroll
      for (int c = 0; c < 4; ++c) sum[(16 * k + g + 8 * (c >> 1)) * AG_COLS + 16 * warp + 8 * n + 2 * q + (c & 1)] = acc[k][n][c];
  __syncthreads();
  if (cs > 1) cluster_barrier();
  const float sc = ad.scale[id];
  for (int e = tid + 256 * rank; e < ROWS * AG_COLS; e += 256 * cs) {
    const int r = e / AG_COLS, c = e % AG_COLS;
    if (r >= ad.rank || c0 + c >= width) continue;
    float v = 0.0f;
    for (uint32_t k = 0; k < cs; ++k) {
      const float p = cs > 1 ? ld_cluster(map_to_rank(xs + 4u * e, k)) : sum[e];
      v = k ? v + p : p;
    }
    G[((long long)id * ad.rank + r) * width + c0 + c] = sc * v;
  }
  if (cs > 1) cluster_barrier();
}

template <int RT, bool EIGHT>
static tb_status launch_grad(const Adapt& ad, const void* in, const float* in_scales, const float* low, int n_tok, int width, float* G,
                             cudaStream_t st) {
  constexpr int tiles_bytes = 2 * AG_TOK * AG_COLS * 2 + AG_PIECES * 16 * RT * AG_TOK * 2, sum_bytes = 16 * RT * AG_COLS * 4;
  constexpr int smem = tiles_bytes > sum_bytes ? tiles_bytes : sum_bytes;
  static bool configured[64] = {false};
  int dev = 0;
  TB_CUDA_CHECK(cudaGetDevice(&dev));
  if (dev < 0 || dev >= 64) return TB_ERR_CUDA;
  if (!configured[dev]) {
    TB_CUDA_CHECK(cudaFuncSetAttribute(k_adapter_grad<RT, EIGHT>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem));
    configured[dev] = true;
  }
  const int cols = (width + AG_COLS - 1) / AG_COLS, sms = sm_count() > 0 ? sm_count() : 148;
  int cs = 1;  // CTAs along the tokens until about two an SM
  while (cs < 8 && (long long)cols * ad.n * cs * 2 <= 2 * sms && n_tok / ad.n / (2 * cs) >= AG_TOK) cs *= 2;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(cols * cs), (unsigned)ad.n);
  cfg.blockDim = dim3(256);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = (unsigned)cs;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  TB_CUDA_CHECK(cudaLaunchKernelEx(&cfg, k_adapter_grad<RT, EIGHT>, ad, in, in_scales, low, n_tok, width, G));
  TB_LAUNCH_CHECK();
  return TB_OK;
}

template <bool EIGHT>
static tb_status grad_of_rank(const Adapt& ad, const void* in, const float* in_scales, const float* low, int n_tok, int width, float* G,
                              cudaStream_t st) {
  if (ad.rank <= 16) return launch_grad<1, EIGHT>(ad, in, in_scales, low, n_tok, width, G, st);
  if (ad.rank <= 32) return launch_grad<2, EIGHT>(ad, in, in_scales, low, n_tok, width, G, st);
  if (ad.rank <= 64) return launch_grad<4, EIGHT>(ad, in, in_scales, low, n_tok, width, G, st);
  return launch_grad<8, EIGHT>(ad, in, in_scales, low, n_tok, width, G, st);
}

// `in` bf16, or 8-bit codes where in_scales is given.
tb_status adapter_grad_bf16(const Adapt& ad, const void* in, const float* in_scales, const float* low, int n_tok, int width, float* G,
                            cudaStream_t st) {
  return in_scales ? grad_of_rank<true>(ad, in, in_scales, low, n_tok, width, G, st)
                   : grad_of_rank<false>(ad, in, in_scales, low, n_tok, width, G, st);
}

}  // namespace tb
