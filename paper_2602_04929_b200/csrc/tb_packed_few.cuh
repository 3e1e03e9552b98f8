// y = x Q^T for a few tokens (bf16), and for any number of them in float: mma.sync on weights decoded in registers.
//
// With few tokens the product is bound by reading the packed words and, at two to four bits, nearly as much by the
// instructions that decode them, so the words go from global memory straight into fragments.  A weight row is a row of operand A
// (16 rows a tile, MT tiles a CTA), tokens are operand B's columns (NT tiles of 8).  Which contraction columns a fragment calls
// k = 0 .. 15 does not matter as long as both operands agree: a lane takes 32 neighbouring codes of a row (BITS words), hence its
// quad 128 columns, and the same columns of x; eight codes decode to the four registers that two MMAs take.  c - z is exact in
// bf16; the scale of a row and of the 128 columns multiplies the sum.  The CTA's warps take every eighth block of 128 columns, the
// CTAs of a cluster (cs of them) every cs-th eight; sums are joined in a fixed order.  Float activations go through three bf16 pieces, all
// 24 bits.
//
// NARROW: scales of fewer than 128 columns, or a width that is no multiple of 128.  A lane then takes 8 codes of a run of 32.
#pragma once

#include "tb_packed_decode.cuh"
#include "tb_packed.cuh"
#include "tb_pair.cuh"

namespace tb {

struct PackedFew {
  PackedW w;
  Adapt ad;
  const void *x, *M;  // M: the adapters' [adapter][rank][d_out]
  const float* low;   // [n_tok][rank]
  void* out;
  int n_tok;
};

__device__ __forceinline__ void mma_few(float (&c)[4], unsigned a0, unsigned a1, unsigned a2, unsigned a3, unsigned b0, unsigned b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
               : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// Eight neighbouring activations as NP pieces of bf16 pairs.
template <int NP>
struct Acts {
  unsigned v[NP][4];
};
__device__ __forceinline__ void load_acts(const __nv_bfloat16* p, Acts<1>& a) {
  const uint4 q = *reinterpret_cast<const uint4*>(p);
  a.v[0][0] = q.x, a.v[0][1] = q.y, a.v[0][2] = q.z, a.v[0][3] = q.w;
}
__device__ __forceinline__ void load_acts(const float* p, Acts<3>& a) {
  const float4 q0 = reinterpret_cast<const float4*>(p)[0], q1 = reinterpret_cast<const float4*>(p)[1];
  float f[8] = {q0.x, q0.y, q0.z, q0.w, q1.x, q1.y, q1.z, q1.w};
#pragma unroll
  for (int n = 0; n < 3; ++n)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const __nv_bfloat162 b = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);
      a.v[n][i] = bf2(b);
      // what is left, nothing of what is not finite (or rounds to infinity)
      const float lo = __uint_as_float(a.v[n][i] << 16), hi = __uint_as_float(a.v[n][i] & 0xffff0000u);
      f[2 * i] = fabsf(lo) <= 3.3895e38f ? f[2 * i] - lo : 0.0f;
      f[2 * i + 1] = fabsf(hi) <= 3.3895e38f ? f[2 * i + 1] - hi : 0.0f;
    }
}

// Codes 8 C .. 8 C + 7 of both rows of a tile against every token tile.
template <int BITS, int C, int NT, int NP, int N>
__device__ __forceinline__ void few_step(const unsigned (&w0)[N], const unsigned (&w1)[N], unsigned z0, unsigned z1, const Acts<NP> (&x)[NT],
                                         float (&acc)[NT][4]) {
  unsigned a[4], b[4];
  decode8<BITS, 8 * C>(w0, z0, a);
  decode8<BITS, 8 * C>(w1, z1, b);
#pragma unroll
  for (int n = 0; n < NT; ++n)
#pragma unroll
    for (int p = 0; p < NP; ++p) {
      mma_few(acc[n], a[0], b[0], a[1], b[1], x[n].v[p][0], x[n].v[p][1]);
      mma_few(acc[n], a[2], b[2], a[3], b[3], x[n].v[p][2], x[n].v[p][3]);
    }
}

template <int BITS>
__device__ __forceinline__ void load_words(const unsigned* p, unsigned (&w)[BITS]) {  // on a multiple of BITS words
  if constexpr (BITS % 4 == 0) {
#pragma unroll
    for (int i = 0; i < BITS / 4; ++i) {
      const uint4 v = reinterpret_cast<const uint4*>(p)[i];
      w[4 * i] = v.x, w[4 * i + 1] = v.y, w[4 * i + 2] = v.z, w[4 * i + 3] = v.w;
    }
  } else if constexpr (BITS % 2 == 0) {
#pragma unroll
    for (int i = 0; i < BITS / 2; ++i) {
      const uint2 v = reinterpret_cast<const uint2*>(p)[i];
      w[2 * i] = v.x, w[2 * i + 1] = v.y;
    }
  } else {
#pragma unroll
    for (int i = 0; i < BITS; ++i) w[i] = p[i];
  }
}

template <int BITS, int MT, int NT, int NP, bool NARROW, typename T>
__global__ void __launch_bounds__(256, 2) k_packed_few(const PackedFew p) {
  constexpr int RC = 16 * MT, TB = 8 * NT, OUT = RC * TB;
  extern __shared__ float few_part[];  // [8 warps][token][row]
  __shared__ int own[TB];
  uint32_t rank, cs;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
  asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(cs));
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, q = lane & 3;
  const int r0 = (blockIdx.x / cs) * RC, t0 = blockIdx.y * TB;
  if (p.ad.n && threadIdx.x < TB) own[threadIdx.x] = t0 + (int)threadIdx.x < p.n_tok ? adapter_of(p.ad, t0 + threadIdx.x) : -1;
  const unsigned* row[2 * MT];
  long long sz[2 * MT];
#pragma unroll
  for (int i = 0; i < 2 * MT; ++i) {
    const int r = min(r0 + 8 * i + g, p.w.d_out - 1);  // rows behind the last are computed from it and not stored
    row[i] = p.w.packed + (long long)r * p.w.words;
    sz[i] = (long long)r * p.w.n_g;
  }
  const T* x[NT];
#pragma unroll
  for (int n = 0; n < NT; ++n) x[n] = static_cast<const T*>(p.x) + (long long)min(t0 + 8 * n + g, p.n_tok - 1) * p.w.d_in;
  float sum[MT][NT][4] = {};
  if constexpr (!NARROW) {
    const int blocks = p.w.d_in >> 7, per_group = p.w.group >> 7;
#pragma unroll 1
    for (int b = (int)rank * 8 + warp; b < blocks; b += 8 * (int)cs) {
      unsigned w[2 * MT][BITS];
      int z[2 * MT];
      float s[2 * MT];
      const int gi = b / per_group;
#pragma unroll
      for (int i = 0; i < 2 * MT; ++i) {
        load_words<BITS>(row[i] + (4 * b + q) * BITS, w[i]);
        z[i] = p.w.zeros[sz[i] + gi];
        s[i] = p.w.scales[sz[i] + gi];
      }
      float acc[MT][NT][4] = {};
#pragma unroll
      for (int i = 0; i < 2 * MT; ++i) z[i] = (int)zero_word(z[i], BITS);
#define TB_FEW_STEP(C)                                                                                                 \
  {                                                                                                                    \
    Acts<NP> a[NT];                                                                                                    \
    _Pragma("unroll") for (int n = 0; n < NT; ++n) load_acts(x[n] + 128 * b + 32 * q + 8 * C, a[n]);                    \
    _Pragma("unroll") for (int m = 0; m < MT; ++m)                                                                      \
        few_step<BITS, C, NT, NP>(w[2 * m], w[2 * m + 1], (unsigned)z[2 * m], (unsigned)z[2 * m + 1], a, acc[m]);       \
  }
      TB_FEW_STEP(0)
      TB_FEW_STEP(1)
      TB_FEW_STEP(2)
      TB_FEW_STEP(3)
#undef TB_FEW_STEP
#pragma unroll
      for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int c = 0; c < 4; ++c) sum[m][n][c] = fmaf(s[2 * m + (c >> 1)], acc[m][n][c], sum[m][n][c]);
    }
  } else {
    const int runs = p.w.d_in >> 5, per_group = p.w.group >> 5;
#pragma unroll 1
    for (int b = (int)rank * 8 + warp; b < runs; b += 8 * (int)cs) {
      // this lane's eight codes: BITS bytes from byte BITS q of the run's words on
      const int first = (BITS * q) >> 2, shift = 8 * ((BITS * q) & 3);
      Acts<NP> a[NT];
#pragma unroll
      for (int n = 0; n < NT; ++n) load_acts(x[n] + 32 * b + 8 * q, a[n]);
      const int gi = b / per_group;
#pragma unroll
      for (int m = 0; m < MT; ++m) {
        unsigned w[2][2], z[2];
        float s[2], acc[NT][4] = {};
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const unsigned* v = row[2 * m + i] + b * BITS;
          const unsigned v0 = v[first], v1 = v[min(first + 1, BITS - 1)];
          w[i][0] = __funnelshift_r(v0, v1, shift);
          w[i][1] = BITS > 4 ? __funnelshift_r(v1, v[min(first + 2, BITS - 1)], shift) : 0u;
          z[i] = zero_word(p.w.zeros[sz[2 * m + i] + gi], BITS);
          s[i] = p.w.scales[sz[2 * m + i] + gi];
        }
        few_step<BITS, 0, NT, NP>(w[0], w[1], z[0], z[1], a, acc);
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int c = 0; c < 4; ++c) sum[m][n][c] = fmaf(s[c >> 1], acc[n][c], sum[m][n][c]);
      }
    }
  }
#pragma unroll
  for (int m = 0; m < MT; ++m)
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int c = 0; c < 4; ++c) few_part[warp * OUT + (8 * n + 2 * q + (c & 1)) * RC + 16 * m + g + 8 * (c >> 1)] = sum[m][n][c];
  __syncthreads();
  for (int e = threadIdx.x; e < OUT; e += 256) {
    float v = few_part[e];
#pragma unroll
    for (int k = 1; k < 8; ++k) v += few_part[k * OUT + e];
    few_part[e] = v;
  }
  if (cs > 1)
    cluster_barrier();
  else
    __syncthreads();
  if (p.ad.n) pdl_wait();  // x A^T is another kernel's, which may still run
  const uint32_t mine = smem_u32(few_part);
  for (int e = threadIdx.x + 256 * (int)rank; e < OUT; e += 256 * (int)cs) {
    const int t = e / RC, r = r0 + e % RC;
    if (t0 + t >= p.n_tok || r >= p.w.d_out) continue;
    float v = few_part[e];
    if (cs > 1) {
      v = 0.0f;
      for (uint32_t k = 0; k < cs; ++k) {
        float u;
        asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(u) : "r"(map_to_rank(mine + 4u * e, k)) : "memory");
        v = k ? v + u : u;
      }
    }
    if (p.ad.n && own[t] >= 0) {
      const T* m = static_cast<const T*>(p.M) + (long long)own[t] * p.ad.rank * p.w.d_out + r;
      const float* l = p.low + (long long)(t0 + t) * p.ad.rank;
      float a = 0.0f;
#pragma unroll 8
      for (int k = 0; k < p.ad.rank; ++k) a = fmaf(l[k], cvt<float>(m[(long long)k * p.w.d_out]), a);
      v = fmaf(p.ad.scale[own[t]], a, v);
    }
    if constexpr (sizeof(T) == 2)
      static_cast<T*>(p.out)[(long long)(t0 + t) * p.w.d_out + r] = __float2bfloat16(v);
    else
      static_cast<T*>(p.out)[(long long)(t0 + t) * p.w.d_out + r] = v;
  }
  if (cs > 1) cluster_barrier();  // nobody leaves while its sums are read
}

template <int BITS, int NT, int NP, bool NARROW, typename T>
tb_status launch_few(const PackedFew& p, cudaStream_t st) {
  constexpr int MT = BITS <= 4 && NP * NT <= 3 ? 4 : 2, RC = 16 * MT, smem = 8 * RC * 8 * NT * 4;  // what 128 registers hold
  auto kern = k_packed_few<BITS, MT, NT, NP, NARROW, T>;
  static bool configured[64] = {false};
  int dev = 0;
  TB_CUDA_CHECK(cudaGetDevice(&dev));
  if (dev < 0 || dev >= 64) return TB_ERR_CUDA;
  if (!configured[dev]) {
    TB_CUDA_CHECK(cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, smem));
    configured[dev] = true;
  }
  const int tiles = (p.w.d_out + RC - 1) / RC, blocks = (p.n_tok + 8 * NT - 1) / (8 * NT);
  const int sms = sm_count() > 0 ? sm_count() : 148, units = p.w.d_in >> (NARROW ? 5 : 7);
  int cs = 1;  // CTAs along the contraction, up to two an SM, a block of columns for every warp
  while (cs < 8 && (long long)tiles * blocks * cs * 2 <= 2 * sms && 8 * cs < units) cs *= 2;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(tiles * cs), (unsigned)blocks);
  cfg.blockDim = dim3(256);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = (unsigned)cs;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = p.ad.n ? 2 : 1;  // beside the kernel that makes x A^T, which started when all before it had ended
  TB_CUDA_CHECK(cudaLaunchKernelEx(&cfg, kern, p));
  TB_LAUNCH_CHECK();
  return TB_OK;
}

template <int NT, int NP, typename T>
tb_status launch_few_bits(const PackedFew& p, cudaStream_t st) {
  const bool narrow = p.w.d_in % 128 != 0 || p.w.group % 128 != 0;
  switch (p.w.bits) {
    case 2: return narrow ? launch_few<2, NT, NP, true, T>(p, st) : launch_few<2, NT, NP, false, T>(p, st);
    case 3: return narrow ? launch_few<3, NT, NP, true, T>(p, st) : launch_few<3, NT, NP, false, T>(p, st);
    case 4: return narrow ? launch_few<4, NT, NP, true, T>(p, st) : launch_few<4, NT, NP, false, T>(p, st);
    case 5: return narrow ? launch_few<5, NT, NP, true, T>(p, st) : launch_few<5, NT, NP, false, T>(p, st);
    case 6: return narrow ? launch_few<6, NT, NP, true, T>(p, st) : launch_few<6, NT, NP, false, T>(p, st);
    case 7: return narrow ? launch_few<7, NT, NP, true, T>(p, st) : launch_few<7, NT, NP, false, T>(p, st);
    default: return narrow ? launch_few<8, NT, NP, true, T>(p, st) : launch_few<8, NT, NP, false, T>(p, st);
  }
}

}  // namespace tb
