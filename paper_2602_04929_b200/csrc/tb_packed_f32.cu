// Products of float activations with bit-packed weights where tokens are many, y = x Q^T and dx = dy Q: tiles of 64 tokens and 128
// columns on mma.sync.
//
// A float is the sum of three bf16 pieces (all 24 bits), and c - z is exact in bf16, so three products with float sums lose nothing
// that one in float would keep.  The scale is a row's and a run's of columns.  Forward, the contraction runs along the row: the sum of
// a step is scaled.  Backward it runs down the rows, so dy takes the scale before it is split, which needs a tile whose columns have
// one group: 32 columns (COLS) where groups are not multiples of 128.
//
// A step takes 32 of the contraction and its sum joins a float sum: the matrix instruction drops bits of its sum instead of rounding,
// so long sums in it are off by 2^-24 of their size a step, all to one side.  Activations are split and codes decoded once for the CTA,
// into shared memory (two buffers; rows padded so that ldmatrix meets no bank twice), while the step before is multiplied; the next
// step's words are on their way in registers.  A cluster (cs CTAs) shares the contraction where tiles are few, and its sums are joined
// in a fixed order.  Adapters join the finished sums on the FP32 pipe.
//
// 1024 tokens x 8192 x 8192, 4 bits: 2128 us forward, 194 TFLOP/s of bf16 products (a library's float product of that shape, without
// the dequantizing, takes 2.2 ms); 4096 x 4096, 603 us.  It is bound by the load/store unit: fragments, split activations and codes
// pass through shared memory, and every row's words come in 8-byte pieces.
#include "tb_packed_decode.cuh"
#include "tb_packed.cuh"
#include "tb_pair.cuh"

namespace tb {

enum { F_TOK = 64, F_K = 32, F_THREADS = 256 };

struct PackedF32 {
  PackedW w;
  Adapt ad;
  const float *in, *low, *M;  // M: the adapters' [adapter][rank][n_cols]
  float* out;
  int n_tok, n_cols, n_sum, col_tiles, per;  // per: steps of a CTA of the cluster
};

__device__ __forceinline__ void ldm(unsigned (&r)[4], uint32_t a) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(a) : "memory");
}
__device__ __forceinline__ void ldm_trans(unsigned (&r)[4], uint32_t a) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(a)
               : "memory");
}
__device__ __forceinline__ void mma_f(float (&c)[4], const unsigned (&a)[4], unsigned b0, unsigned b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

template <bool BACK, int COLS>
struct F32Tile {
  static constexpr int WN = COLS / 32 > 1 ? 4 : 2, WM = 8 / WN;  // warps along the columns, the tokens
  static constexpr int MF = F_TOK / 16 / WM, NF = COLS / 8 / WN;  // a warp's fragments
  static constexpr int A_PITCH = 2 * F_K + 16, B_PITCH = BACK ? 2 * COLS + 16 : 2 * F_K + 16;
  static constexpr int A_BYTES = F_TOK * A_PITCH, B_BYTES = (BACK ? F_K : COLS) * B_PITCH;
  static constexpr int BUFFER = 3 * A_BYTES + B_BYTES;
  static constexpr int S_PITCH = COLS + 4;  // floats of a row of finished sums
  static constexpr int SMEM = 2 * BUFFER > F_TOK * S_PITCH * 4 ? 2 * BUFFER : F_TOK * S_PITCH * 4;
};

template <bool BACK, int COLS>
__global__ void __launch_bounds__(F_THREADS, 2) k_packed_f32(PackedF32 p) {
  using L = F32Tile<BACK, COLS>;
  constexpr int MF = L::MF, NF = L::NF;
  extern __shared__ __align__(16) char smem[];
  const uint32_t base = smem_u32(smem);
  uint32_t part, cs;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(part));
  asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(cs));
  const PackedW& w = p.w;
  const int tile = blockIdx.x / cs, c0 = tile % p.col_tiles * COLS;
  const long long t0 = (long long)(tile / p.col_tiles) * F_TOK;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int steps = (p.n_sum + F_K - 1) / F_K, s0 = min(steps, (int)part * p.per), s1 = min(steps, s0 + p.per);

  // what a thread brings: 8 activations of a token, 16 codes of a row
  const long long tok = t0 + tid / 4;
  const float* x_row = tok < p.n_tok ? p.in + tok * p.n_sum : nullptr;
  constexpr int PER_ROW = (BACK ? COLS : F_K) / 16;  // threads of a row of codes
  const bool codes = tid < (BACK ? F_K : COLS) * PER_ROW;
  const int w_row = tid / PER_ROW, w_col = 16 * (tid % PER_ROW);
  const int group0 = BACK ? c0 / w.group : 0;
  float4 x[2];
  unsigned v[4] = {};
  float scale = 0.0f, zero = 0.0f;
  int shift = 0;
  bool valid = false;
  auto fetch = [&](int s) {
    const int k0 = s * F_K, k = k0 + 8 * (tid & 3);
#pragma unroll
    for (int i = 0; i < 2; ++i)
      x[i] = x_row && k + 4 * i < p.n_sum ? *reinterpret_cast<const float4*>(x_row + k + 4 * i) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    if (BACK) scale = k0 + lane < w.d_out ? w.scales[(long long)(k0 + lane) * w.n_g + group0] : 0.0f;
    if (!codes) return;
    const int row = BACK ? k0 + w_row : c0 + w_row, col = BACK ? c0 + w_col : k0 + w_col;
    valid = row < w.d_out && col < w.d_in;
    if (!valid) return;
    const long long bit = (long long)col * w.bits;
    const int word = (int)(bit >> 5);
    shift = (int)(bit & 31);
    const unsigned* r = w.packed + (long long)row * w.words + word;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (32 * i < shift + 16 * w.bits) v[i] = r[i];
    if (!BACK && s > s0 && k0 % w.group) return;  // the group's zero-point is at hand
    const int z = w.zeros[(long long)row * w.n_g + (BACK ? group0 : col / w.group)];
    zero = (float)z + 8388608.0f;
  };
  auto store = [&](int buffer) {
    char* a = smem + buffer * L::BUFFER;
    float f[8] = {x[0].x, x[0].y, x[0].z, x[0].w, x[1].x, x[1].y, x[1].z, x[1].w};
    if (BACK)
#pragma unroll
      for (int i = 0; i < 8; ++i) f[i] *= __shfl_sync(0xffffffffu, scale, 8 * (lane & 3) + i);
    // truncated, each piece takes eight bits; of what is not finite there is one piece
    float left = 0.0f;
    unsigned o[3][4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float lo = f[2 * i], hi = f[2 * i + 1];
#pragma unroll
      for (int n = 0; n < 3; ++n) {
        o[n][i] = __byte_perm(__float_as_uint(lo), __float_as_uint(hi), 0x7632);
        lo -= __uint_as_float(__float_as_uint(lo) & 0xffff0000u), hi -= __uint_as_float(__float_as_uint(hi) & 0xffff0000u);
      }
      left += lo + hi;  // 0, or not a number
    }
    if (left != 0.0f)
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (!(fabsf(f[i]) <= 3.4028235e38f)) {
          const unsigned keep = i & 1 ? 0x0000ffffu : 0xffff0000u, one = f[i] != f[i] ? 0x7fc0u : __float_as_uint(f[i]) >> 16;
          o[0][i / 2] = (o[0][i / 2] & keep) | (i & 1 ? one << 16 : one);
          o[1][i / 2] &= keep, o[2][i / 2] &= keep;
        }
#pragma unroll
    for (int n = 0; n < 3; ++n)
      *reinterpret_cast<uint4*>(a + n * L::A_BYTES + (tid >> 2) * L::A_PITCH + 16 * (tid & 3)) = make_uint4(o[n][0], o[n][1], o[n][2], o[n][3]);
    if (!codes) return;
    char* b = a + 3 * L::A_BYTES + w_row * L::B_PITCH + 2 * w_col;
    const unsigned long long lo = v[0] | (unsigned long long)v[1] << 32, hi = v[2] | (unsigned long long)v[3] << 32;
#pragma unroll
    for (int h = 0; h < 2; ++h) {  // 8 codes from bit `at` of the 128 on
      const int at = shift + 8 * h * w.bits;
      unsigned long long q = at >= 64 ? hi >> (at - 64) : at ? lo >> at | hi << (64 - at) : lo;
      unsigned d[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float c[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          c[j] = __uint_as_float(0x4B000000u | ((unsigned)q & ((1u << w.bits) - 1u))) - zero;
          q >>= w.bits;
        }
        d[i] = valid ? bf2(__floats2bfloat162_rn(c[0], c[1])) : 0u;
      }
      *reinterpret_cast<uint4*>(b + 16 * h) = make_uint4(d[0], d[1], d[2], d[3]);
    }
  };

  const int wm = warp / L::WN * (16 * MF), wn = warp % L::WN * (8 * NF);
  const int g = lane >> 2, q2 = 2 * (lane & 3);
  float acc[MF][NF][4], sum[MF][NF][4] = {}, row_scale[BACK ? 1 : NF][2];
  if (s0 < s1) fetch(s0), store(0);
  for (int s = s0; s < s1; ++s) {
    __syncthreads();  // this step's buffer is full, and nobody reads the other one
    if (s + 1 < s1) fetch(s + 1);
#pragma unroll
    for (int m = 0; m < MF; ++m)
#pragma unroll
      for (int f = 0; f < NF; ++f) acc[m][f][0] = acc[m][f][1] = acc[m][f][2] = acc[m][f][3] = 0.0f;
    if constexpr (!BACK)
      if (s == s0 || s * F_K % w.group == 0) {  // a group begins
#pragma unroll
        for (int f = 0; f < NF; ++f)
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            const int row = c0 + wn + 8 * f + q2 + j;
            row_scale[f][j] = row < w.d_out ? w.scales[(long long)row * w.n_g + s * F_K / w.group] : 0.0f;
          }
      }
    const uint32_t a = base + (s - s0 & 1) * L::BUFFER, b = a + 3 * L::A_BYTES;
#pragma unroll
    for (int kk = 0; kk < F_K; kk += 16) {
      unsigned bf[NF / 2][4];
#pragma unroll
      for (int n = 0; n < NF / 2; ++n) {
        const int half = lane >> 4, mid = lane >> 3 & 1;
        if (BACK)
          ldm_trans(bf[n], b + (kk + (lane & 7) + 8 * mid) * L::B_PITCH + 2 * (wn + 16 * n + 8 * half));
        else
          ldm(bf[n], b + (wn + 16 * n + (lane & 7) + 8 * half) * L::B_PITCH + 2 * (kk + 8 * mid));
      }
#pragma unroll
      for (int n = 0; n < 3; ++n)
#pragma unroll
        for (int m = 0; m < MF; ++m) {
          unsigned af[4];
          ldm(af, a + n * L::A_BYTES + (wm + 16 * m + (lane & 15)) * L::A_PITCH + 2 * (kk + 8 * (lane >> 4)));
#pragma unroll
          for (int f = 0; f < NF; ++f) mma_f(acc[m][f], af, bf[f / 2][2 * (f & 1)], bf[f / 2][2 * (f & 1) + 1]);
        }
    }
#pragma unroll
    for (int m = 0; m < MF; ++m)
#pragma unroll
      for (int f = 0; f < NF; ++f)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          if constexpr (BACK)
            sum[m][f][j] += acc[m][f][j];
          else
            sum[m][f][j] = fmaf(row_scale[f][j & 1], acc[m][f][j], sum[m][f][j]);
        }
    if (s + 1 < s1) store(s + 1 - s0 & 1);
  }
  __syncthreads();
  float* tile_sum = reinterpret_cast<float*>(smem);
#pragma unroll
  for (int m = 0; m < MF; ++m)
#pragma unroll
    for (int f = 0; f < NF; ++f)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        *reinterpret_cast<float2*>(tile_sum + (wm + 16 * m + g + 8 * h) * L::S_PITCH + wn + 8 * f + q2) = make_float2(sum[m][f][2 * h], sum[m][f][2 * h + 1]);
      }
  if (cs > 1)
    cluster_barrier();
  else
    __syncthreads();
  // the cluster's CTAs have a share of the tokens each; a thread has four columns of neighbouring tokens
  constexpr int LANES = COLS / 4, AT_ONCE = F_THREADS / LANES;
  const int mine = F_TOK / (int)cs, first = (int)part * mine, c = c0 + 4 * (tid % LANES);
  constexpr int RUN = 4;  // tokens that read an adapter's row together where it is the same
  for (int t1 = first + tid / LANES * RUN; t1 < first + mine; t1 += AT_ONCE * RUN) {
    float4 r[RUN];
    int id[RUN];
    bool same = true;
#pragma unroll
    for (int i = 0; i < RUN; ++i) {
      const float* at = tile_sum + (t1 + i) * L::S_PITCH + 4 * (tid % LANES);
      r[i] = *reinterpret_cast<const float4*>(at);
      if (cs > 1) {
        const uint32_t addr = smem_u32(at);
        for (uint32_t o = 0; o < cs; ++o) {
          float4 q;
          asm volatile("ld.shared::cluster.v4.f32 {%0,%1,%2,%3}, [%4];" : "=f"(q.x), "=f"(q.y), "=f"(q.z), "=f"(q.w) : "r"(map_to_rank(addr, o)) : "memory");
          r[i].x = o ? r[i].x + q.x : q.x, r[i].y = o ? r[i].y + q.y : q.y, r[i].z = o ? r[i].z + q.z : q.z, r[i].w = o ? r[i].w + q.w : q.w;
        }
      }
      id[i] = p.ad.n && t0 + t1 + i < p.n_tok ? adapter_of(p.ad, t0 + t1 + i) : -1;
      same = same && id[i] == id[0];
    }
    if (c >= p.n_cols) continue;
    auto add = [&](float4& y, long long t, int r_, float sc, const float4& m) {
      const float u = sc * p.low[t * p.ad.rank + r_];
      y.x = fmaf(u, m.x, y.x), y.y = fmaf(u, m.y, y.y), y.z = fmaf(u, m.z, y.z), y.w = fmaf(u, m.w, y.w);
    };
    if (same && id[0] >= 0) {
      const float sc = p.ad.scale[id[0]];
      const float* m = p.M + (long long)id[0] * p.ad.rank * p.n_cols + c;
#pragma unroll 4
      for (int k = 0; k < p.ad.rank; ++k) {
        const float4 mk = *reinterpret_cast<const float4*>(m + (long long)k * p.n_cols);
#pragma unroll
        for (int i = 0; i < RUN; ++i) add(r[i], t0 + t1 + i, k, sc, mk);
      }
    } else {
#pragma unroll
      for (int i = 0; i < RUN; ++i) {
        if (id[i] < 0) continue;
        const float sc = p.ad.scale[id[i]];
        const float* m = p.M + (long long)id[i] * p.ad.rank * p.n_cols + c;
        for (int k = 0; k < p.ad.rank; ++k) add(r[i], t0 + t1 + i, k, sc, *reinterpret_cast<const float4*>(m + (long long)k * p.n_cols));
      }
    }
#pragma unroll
    for (int i = 0; i < RUN; ++i)
      if (t0 + t1 + i < p.n_tok) *reinterpret_cast<float4*>(p.out + (t0 + t1 + i) * p.n_cols + c) = r[i];
  }
  if (cs > 1) cluster_barrier();  // nobody leaves while its sums are read
}

template <bool BACK, int COLS>
static tb_status launch(PackedF32& p, cudaStream_t st) {
  using L = F32Tile<BACK, COLS>;
  p.col_tiles = (p.n_cols + COLS - 1) / COLS;
  const long long tiles = (long long)p.col_tiles * ((p.n_tok + F_TOK - 1) / F_TOK);
  const int sms = sm_count() > 0 ? sm_count() : 148, steps = (p.n_sum + F_K - 1) / F_K;
  int cs = 1;
  while (cs < 8 && tiles * cs * 2 <= 2 * sms && steps / (2 * cs) >= 4) cs *= 2;
  p.per = (steps + cs - 1) / cs;
  TB_CUDA_CHECK(cudaFuncSetAttribute(k_packed_f32<BACK, COLS>, cudaFuncAttributeMaxDynamicSharedMemorySize, L::SMEM));
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(tiles * cs));
  cfg.blockDim = dim3(F_THREADS);
  cfg.dynamicSmemBytes = L::SMEM;
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = (unsigned)cs;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  TB_CUDA_CHECK(cudaLaunchKernelEx(&cfg, k_packed_f32<BACK, COLS>, p));
  TB_LAUNCH_CHECK();
  return TB_OK;
}

tb_status packed_product_f32(const PackedW& w, const Adapt& ad, const float* in, int n_tok, float* out, const float* low, bool back,
                             cudaStream_t st) {
  PackedF32 p = {};
  p.w = w, p.ad = ad, p.in = in, p.low = low, p.out = out, p.n_tok = n_tok;
  p.M = static_cast<const float*>(back ? ad.A : ad.B);
  p.n_cols = back ? w.d_in : w.d_out, p.n_sum = back ? w.d_out : w.d_in;
  if (!back) return launch<false, 128>(p, st);
  return w.group % 128 == 0 || w.n_g == 1 ? launch<true, 128>(p, st) : launch<true, 32>(p, st);
}

}  // namespace tb
