// y = x Q^T where tokens are few or the work is small: mma.sync on weights decoded in registers.
//
// With few tokens the product is bound by reading the packed words and, at two to four bits, as much by the instructions that decode
// them (logical operations go at half rate), so the words are decoded straight into fragments.  A weight row is a row of operand A (16
// rows a tile, MT tiles a CTA), tokens are operand B's columns (NT tiles of 8).  Which contraction columns a fragment calls k = 0 .. 15
// does not matter as long as both operands agree: a lane takes 32 neighbouring codes of a row (BITS words), hence its quad 128 columns,
// and the same columns of x; 16 codes decode to the eight registers that four MMAs take.  With two and four bits a pair of neighbours
// in a register is a code of a word's lower half and the one 16 bits above it, so that a mask extracts both, and it is x that is
// brought into that order, once for all MT tiles.  c - z is exact in bf16 (zero-points' second pieces, where a warp meets one, are further
// weights beside the same activations); the scale of a row and of the 128 columns multiplies the sum.  Float activations go through three
// bf16 pieces, all 24 bits.
//
// The words come by TMA, in stages of eight blocks of 128 columns (one for every warp), as many stages ahead as fit beside a second
// CTA: a warp that loads its own words has too few bytes in flight for the memory's latency.  A tile has the most rows (16 MT) that
// leave a CTA and a half for every SM; where even 16 rows do not, CTAs of a cluster (cs of them) have a range of blocks each.  The
// warps' and the CTAs' sums are joined in a fixed order.
//
// 1 token: 4096 x 4096, 4 bits, 6.0 us; 8192 x 8192, 2 bits, 12.9 us (17 MB of words and 4 MB of scales, 1.6 TB/s); 64 tokens x 2048 x
// 2048, 4 bits, 9.0 us.  Latency bounds it: nothing is saturated (ALU 44 %, issue 1.9 of 4, DRAM 15 %), about 3 us are launch and first
// loads, and of decoding, an instruction for every two codes at half rate, there are 1.8 us in the 12.9.
//
// NARROW: scales of fewer than 128 columns, or a width that is no multiple of 128.  A lane then takes 8 codes of a run of 32.
#pragma once

#include "tb_packed_decode.cuh"
#include "tb_packed.cuh"
#include "tb_pair.cuh"

namespace tb {

enum { FEW_STAGES_MAX = 8 };
static __device__ int g_few_error = 0;  // of this translation unit; tb_device_error_flag reads and clears all of them

struct PackedFew {
  PackedW w;
  Adapt ad;
  const void *x, *M;  // M: the adapters' [adapter][rank][d_out]
  const float* low;   // [n_tok][rank]
  void* out;
  int n_tok, stages;
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
      a.v[n][i] = first_pieces(f[2 * i], f[2 * i + 1]);
      f[2 * i] = rest_of(f[2 * i], a.v[n][i] << 16), f[2 * i + 1] = rest_of(f[2 * i + 1], a.v[n][i] & 0xffff0000u);
    }
}

// Codes 8 C .. 8 C + 7 of both rows of a tile against every token tile.
template <int BITS, int C, int NT, int NP, int N>
__device__ __forceinline__ void few_step(const unsigned (&w0)[N], const unsigned (&w1)[N], unsigned z0, unsigned z1, const Acts<NP> (&x)[NT],
                                         float (&acc)[NT][4]) {
  unsigned a[4], b[4];
  decode8<BITS, 8 * C>(w0, zero_first<BITS>(z0), a);
  decode8<BITS, 8 * C>(w1, zero_first<BITS>(z1), b);
  if constexpr (BITS < 8)  // the zero-points' second pieces: 0 mostly, but a vote and a branch cost more than adding them to eight codes
#pragma unroll
    for (int i = 0; i < 4; ++i)
      a[i] = bf2(__hadd2(bf2(a[i]), bf2(zero_second<BITS>(z0)))), b[i] = bf2(__hadd2(bf2(b[i]), bf2(zero_second<BITS>(z1))));
#pragma unroll
  for (int n = 0; n < NT; ++n)
#pragma unroll
    for (int p = 0; p < NP; ++p) {
      mma_few(acc[n], a[0], b[0], a[1], b[1], x[n].v[p][0], x[n].v[p][1]);
      mma_few(acc[n], a[2], b[2], a[3], b[3], x[n].v[p][2], x[n].v[p][3]);
    }
}

// The zero-points' second pieces, the same for every code of a row: as further weights beside the same activations.
template <int NP>
__device__ __forceinline__ void few_second(unsigned z0, unsigned z1, const unsigned (&x)[NP][8], float (&acc)[4]) {
#pragma unroll
  for (int p = 0; p < NP; ++p)
#pragma unroll
    for (int i = 0; i < 8; i += 2) mma_few(acc, z0, z1, z0, z1, x[p][i], x[p][i + 1]);
}

// Columns of register i of 16: the lower half's, the upper half's.
template <int BITS>
struct Pair {
  static __host__ __device__ constexpr int lo(int i) { return BITS == 2 ? i : BITS == 4 ? (i & 3) + 8 * (i >> 2) : 2 * i; }
  static __host__ __device__ constexpr int hi(int i) { return lo(i) + (BITS == 2 ? 8 : BITS == 4 ? 4 : 1); }
};
template <int NP>
struct Acts16 {
  unsigned v[NP][8];
};
// 16 neighbouring activations as they are loaded, and as pieces of bf16 pairs.
template <int NP>
struct Raw16 {
  uint4 v[NP == 1 ? 2 : 4];
  template <typename T>
  __device__ __forceinline__ void load(const T* p) {
#pragma unroll
    for (int i = 0; i < (NP == 1 ? 2 : 4); ++i) v[i] = reinterpret_cast<const uint4*>(p)[i];
  }
};
template <int BITS>
__device__ __forceinline__ void pieces16(const Raw16<1>& x, Acts16<1>& a) {
  const unsigned r[8] = {x.v[0].x, x.v[0].y, x.v[0].z, x.v[0].w, x.v[1].x, x.v[1].y, x.v[1].z, x.v[1].w};
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    if (BITS == 2 || BITS == 4)
      a.v[0][i] = __byte_perm(r[Pair<BITS>::lo(i) >> 1], r[Pair<BITS>::hi(i) >> 1], i & 1 ? 0x7632 : 0x5410);
    else
      a.v[0][i] = r[i];
  }
}
template <int BITS>
__device__ __forceinline__ void pieces16(const Raw16<3>& x, Acts16<3>& a) {
  float f[16];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    f[4 * i] = __uint_as_float(x.v[i].x), f[4 * i + 1] = __uint_as_float(x.v[i].y);
    f[4 * i + 2] = __uint_as_float(x.v[i].z), f[4 * i + 3] = __uint_as_float(x.v[i].w);
  }
#pragma unroll
  for (int n = 0; n < 3; ++n)
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      float &fl = f[Pair<BITS>::lo(i)], &fh = f[Pair<BITS>::hi(i)];
      a.v[n][i] = first_pieces(fl, fh);
      fl = rest_of(fl, a.v[n][i] << 16), fh = rest_of(fh, a.v[n][i] & 0xffff0000u);
    }
}

// Codes 16 H .. 16 H + 15 of a lane's words, in that order.  A code p bits up in the mantissa of 2^(7 - p) is 2^(7 - p) + c.
template <int BITS, int H>
__device__ __forceinline__ void decode16(const unsigned (&w)[BITS], unsigned z, unsigned (&o)[8]) {
  if constexpr (BITS == 2) {
    const __nv_bfloat162 z0 = bf2(z), z2 = __hadd2(z0, __float2bfloat162_rn(96.0f)), z4 = __hadd2(z0, __float2bfloat162_rn(120.0f));
    unsigned v = w[H];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if (i == 3 || i == 6) v >>= 6;
      if (i % 3 == 0) o[i] = bf2(__hadd2(bf2(masked(v, 0x00030003u, 0x43004300u)), z0));
      if (i % 3 == 1) o[i] = bf2(__hadd2(bf2(masked(v, 0x000c000cu, 0x42004200u)), z2));
      if (i % 3 == 2) o[i] = bf2(__hadd2(bf2(masked(v, 0x00300030u, 0x41004100u)), z4));
    }
  } else if constexpr (BITS == 4) {
#pragma unroll
    for (int i = 0; i < 8; ++i) o[i] = bf2(__hadd2(bf2(masked(w[2 * H + (i >> 2)] >> (4 * (i & 3)), 0x000f000fu, 0x43004300u)), bf2(z)));
  } else {
    unsigned a[4], b[4];
    decode8<BITS, 16 * H>(w, z, a);
    decode8<BITS, 16 * H + 8>(w, z, b);
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] = a[i], o[4 + i] = b[i];
  }
}
template <int BITS, int H, int NT, int NP>
__device__ __forceinline__ void few_step16(const unsigned (&w0)[BITS], const unsigned (&w1)[BITS], unsigned z0, unsigned z1,
                                           const Acts16<NP> (&x)[NT], float (&acc)[NT][4]) {
  unsigned a[8], b[8];
  decode16<BITS, H>(w0, z0, a);
  decode16<BITS, H>(w1, z1, b);
#pragma unroll
  for (int n = 0; n < NT; ++n)
#pragma unroll
    for (int p = 0; p < NP; ++p)
#pragma unroll
      for (int i = 0; i < 8; i += 2) mma_few(acc[n], a[i], b[i], a[i + 1], b[i + 1], x[n].v[p][i], x[n].v[p][i + 1]);
}

// A stage: 128-byte pieces of all rows, one after the other, in TMA's 128-byte swizzle.  A lane's BITS words from byte `at` of row r on.
template <int BITS, int RC>
__device__ __forceinline__ void load_words(const unsigned char* stage, int r, int at, unsigned (&w)[BITS]) {
  constexpr int STEP = BITS % 4 == 0 ? 4 : BITS % 2 == 0 ? 2 : 1;
#pragma unroll
  for (int i = 0; i < BITS; i += STEP) {
    const int b = at + 4 * i;
    const unsigned char* p = stage + (b >> 7) * (RC * 128) + r * 128 + (((((b & 127) >> 4) ^ (r & 7)) << 4) | (b & 15));
    if constexpr (STEP == 4) {
      const uint4 v = *reinterpret_cast<const uint4*>(p);
      w[i] = v.x, w[i + 1] = v.y, w[i + 2] = v.z, w[i + 3] = v.w;
    } else if constexpr (STEP == 2) {
      const uint2 v = *reinterpret_cast<const uint2*>(p);
      w[i] = v.x, w[i + 1] = v.y;
    } else {
      w[i] = *reinterpret_cast<const unsigned*>(p);
    }
  }
}

template <int BITS, int MT, int NT, int NP, bool NARROW, typename T>
__global__ void __launch_bounds__(256, NT * NP == 1 ? 2 : 1) k_packed_few(const __grid_constant__ PackedFew p, const __grid_constant__ CUtensorMap wmap) {
  constexpr int RC = 16 * MT, TB = 8 * NT, OUT = RC * TB;
  extern __shared__ __align__(128) float few_part[];  // a ring of the words' stages, then [8 warps][token][row]
  __shared__ int own[TB];
  __shared__ __align__(8) unsigned long long bars[FEW_STAGES_MAX];
  __shared__ int gave_up;
  if (!NARROW && threadIdx.x == 0) {
    for (int s = 0; s < FEW_STAGES_MAX; ++s) mbar_init(smem_u32(bars + s), 1);
    gave_up = 0;
    mbar_fence_init();
  }
  __syncthreads();
  uint32_t rank, cs;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
  asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(cs));
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, q = lane & 3;
  const int r0 = (blockIdx.x / cs) * RC, t0 = blockIdx.y * TB;
  // rows come eight at a time, d_out is a multiple of eight: those behind the last are taken to be the last eight and not stored
  const int eights = min(2 * MT, (p.w.d_out - r0) >> 3) - 1;
  const unsigned* row0 = p.w.packed + (long long)(r0 + g) * p.w.words;
  const long long sz0 = (long long)(r0 + g) * p.w.n_g;
  const T* x[NT];
#pragma unroll
  for (int n = 0; n < NT; ++n) x[n] = static_cast<const T*>(p.x) + (long long)min(t0 + 8 * n + g, p.n_tok - 1) * p.w.d_in;
  float sum[MT][NT][4] = {};
  if (p.ad.n && warp == 7) {
    // the tokens' adapters, and their rows towards this CTA's columns: the end of the kernel would wait for them
    if (lane < TB) own[lane] = t0 + lane < p.n_tok ? adapter_of(p.ad, t0 + lane) : -1;
    __syncwarp();
    for (int e = lane; e < TB * p.ad.rank; e += 32) {
      const int id = own[e / p.ad.rank];
      if (id >= 0) {
        const T* at = static_cast<const T*>(p.M) + ((long long)id * p.ad.rank + e % p.ad.rank) * p.w.d_out + r0;
        asm volatile("prefetch.global.L2 [%0];" ::"l"(at));
      }
    }
  }
  if constexpr (!NARROW) {
    constexpr int STAGE = RC * 128 * BITS;  // eight blocks of 16 BITS bytes a row: BITS pieces
    const int blocks = p.w.d_in >> 7, per_group = p.w.group >> 7;
    const int per = (blocks + (int)cs - 1) / (int)cs, b0 = (int)rank * per, b_end = min(blocks, b0 + per);
    const int n_st = b_end > b0 ? (b_end - b0 + 7) >> 3 : 0;
    // the dynamic part starts on a multiple of 1024 in the swizzle's eyes
    const uint32_t ring0 = (smem_u32(few_part) + 1023u) & ~1023u, bar0 = smem_u32(bars);
    const unsigned char* ring = reinterpret_cast<const unsigned char*>(few_part) + (ring0 - smem_u32(few_part));
    auto fill = [&](int st) {  // by one thread; what lies behind the columns or rows comes as zeros
      const int s = st % p.stages;
      mbar_expect_tx(bar0 + 8 * s, STAGE);
      for (int k = 0; k < BITS; ++k)
        tma_load_2d(ring0 + s * STAGE + k * (RC * 128), &wmap, (b0 + 8 * st) * 4 * BITS + 32 * k, r0, bar0 + 8 * s);
    };
    if (threadIdx.x == 0)
      for (int st = 0; st < min(n_st, p.stages); ++st) fill(st);
    // what a warp loads itself for a block, an iteration ahead: activations, zero-points, scales
    struct Own {
      Raw16<NP> x[2][NT];
      int z[2 * MT];
      float s[2 * MT];
    } next;
    const int* zeros = p.w.zeros + sz0;
    const float* scales = p.w.scales + sz0;
    auto fetch = [&](int b) {
      const int gi = per_group == 1 ? b : b / per_group;
#pragma unroll
      for (int i = 0; i < 2 * MT; ++i) {
        const int e = gi + 8 * min(i, eights) * p.w.n_g;
        next.z[i] = zeros[e], next.s[i] = scales[e];
      }
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int n = 0; n < NT; ++n) next.x[h][n].load(x[n] + 128 * b + 32 * q + 16 * h);
    };
    if (b0 + warp < b_end) fetch(b0 + warp);
    int s = 0;
    uint32_t phase = 0;
#pragma unroll 1
    for (int st = 0; st < n_st; ++st) {
      const int b = b0 + 8 * st + warp;
      const bool mine = b < b_end;
      Acts16<NP> a[2][NT];
      unsigned z[2 * MT];
      float sc[2 * MT];
      unsigned seconds = 0;
      if (mine) {
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int n = 0; n < NT; ++n) pieces16<BITS>(next.x[h][n], a[h][n]);
#pragma unroll
        for (int i = 0; i < 2 * MT; ++i) z[i] = zero_word(next.z[i], BITS), seconds |= z[i], sc[i] = next.s[i];
        if (b + 8 < b_end) fetch(b + 8);
      }
      const bool second = BITS < 8 && __any_sync(0xffffffffu, has_second<BITS>(seconds));
      const bool landed = __all_sync(0xffffffffu, mbar_wait(bar0 + 8 * s, phase, &gave_up, &g_few_error));
      if (mine && landed) {  // (a wait that gave up leaves its share out; nobody skips a barrier)
        const unsigned char* stage = ring + s * STAGE;
        const int at = (4 * warp + q) * 4 * BITS;
#pragma unroll
        for (int m = 0; m < MT; ++m) {
          unsigned w0[BITS], w1[BITS];
          load_words<BITS, RC>(stage, 16 * m + g, at, w0);
          load_words<BITS, RC>(stage, 16 * m + 8 + g, at, w1);
          float acc[NT][4] = {};
          const unsigned z0 = zero_first<BITS>(z[2 * m]), z1 = zero_first<BITS>(z[2 * m + 1]);
          few_step16<BITS, 0, NT, NP>(w0, w1, z0, z1, a[0], acc);
          few_step16<BITS, 1, NT, NP>(w0, w1, z0, z1, a[1], acc);
#pragma unroll
          for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int c = 0; c < 4; ++c) sum[m][n][c] = fmaf(sc[2 * m + (c >> 1)], acc[n][c], sum[m][n][c]);
        }
        if (second)
#pragma unroll
          for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int n = 0; n < NT; ++n) {
              float acc[4] = {};
              few_second<NP>(zero_second<BITS>(z[2 * m]), zero_second<BITS>(z[2 * m + 1]), a[0][n].v, acc);
              few_second<NP>(zero_second<BITS>(z[2 * m]), zero_second<BITS>(z[2 * m + 1]), a[1][n].v, acc);
#pragma unroll
              for (int c = 0; c < 4; ++c)  // rows without one are left alone: an infinite activation would make their 0 no number
                if (has_second<BITS>(z[2 * m + (c >> 1)])) sum[m][n][c] = fmaf(sc[2 * m + (c >> 1)], acc[c], sum[m][n][c]);
            }
      }
      if (st + p.stages < n_st) {
        __syncthreads();
        if (threadIdx.x == 0) fill(st + p.stages);
      }
      if (++s == p.stages) s = 0, phase ^= 1u;
    }
    settle(*(volatile int*)&gave_up);
    __syncthreads();  // the ring becomes the sums'
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
          const long long e = 8 * min(2 * m + i, eights);
          const unsigned* v = row0 + e * p.w.words + b * BITS;
          const unsigned v0 = v[first], v1 = v[min(first + 1, BITS - 1)];
          w[i][0] = __funnelshift_r(v0, v1, shift);
          w[i][1] = BITS > 4 ? __funnelshift_r(v1, v[min(first + 2, BITS - 1)], shift) : 0u;
          z[i] = zero_word(p.w.zeros[sz0 + e * p.w.n_g + gi], BITS);
          s[i] = p.w.scales[sz0 + e * p.w.n_g + gi];
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

template <int BITS, int MT, int NT, int NP, bool NARROW, typename T>
tb_status launch_few_rows(PackedFew p, cudaStream_t st) {
  constexpr int RC = 16 * MT;
  constexpr int sums = 8 * RC * 8 * NT * 4, stage = NARROW ? 1 : RC * 128 * BITS, room = (NT * NP == 1 ? 108 : 216) * 1024;
  auto kern = k_packed_few<BITS, MT, NT, NP, NARROW, T>;
  static bool configured[64] = {false};
  int dev = 0;
  TB_CUDA_CHECK(cudaGetDevice(&dev));
  if (dev < 0 || dev >= 64) return TB_ERR_CUDA;
  if (!configured[dev]) {
    TB_CUDA_CHECK(cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, room + 1024));
    configured[dev] = true;
  }
  const int tiles = (p.w.d_out + RC - 1) / RC, blocks = (p.n_tok + 8 * NT - 1) / (8 * NT);
  const int sms = sm_count() > 0 ? sm_count() : 148, units = p.w.d_in >> (NARROW ? 5 : 7);
  int cs = 1;  // CTAs along the contraction, up to two an SM, a block of columns for every warp
  while (cs < 8 && (long long)tiles * blocks * cs * 2 <= 2 * sms && 8 * cs < units) cs *= 2;
  // all of a CTA's stages at once where they fit
  const int n_st = ((units + cs - 1) / cs + 7) / 8, fit = room / stage;
  p.stages = NARROW ? 1 : n_st < fit ? n_st : fit;
  if (p.stages > FEW_STAGES_MAX) p.stages = FEW_STAGES_MAX;
  const int smem = NARROW ? sums : (p.stages * stage < sums ? sums : p.stages * stage) + 1024;
  CUtensorMap map = {};
  if (!NARROW)
    TB_TRY(make_map_2d(&map, CU_TENSOR_MAP_DATA_TYPE_UINT32, 4, p.w.packed, (unsigned long long)p.w.words, (unsigned long long)p.w.d_out, 32, RC,
                       CU_TENSOR_MAP_SWIZZLE_128B));
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(tiles * cs), (unsigned)blocks);
  cfg.blockDim = dim3(256);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  int n = 0;
  if (cs > 1) {
    attr[n].id = cudaLaunchAttributeClusterDimension;
    attr[n].val.clusterDim.x = (unsigned)cs;
    attr[n].val.clusterDim.y = 1;
    attr[n++].val.clusterDim.z = 1;
  }
  if (p.ad.n) {  // beside the kernel that makes x A^T, which started when all before it had ended
    attr[n].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[n++].val.programmaticStreamSerializationAllowed = 1;
  }
  cfg.attrs = attr;
  cfg.numAttrs = n;
  TB_CUDA_CHECK(cudaLaunchKernelEx(&cfg, kern, p, map));
  TB_LAUNCH_CHECK();
  return TB_OK;
}

template <int BITS, int NT, int NP, bool NARROW, typename T>
tb_status launch_few(const PackedFew& p, cudaStream_t st) {
  constexpr int TOP = BITS <= 4 && NP * NT <= 3 ? 4 : 2;  // what the registers hold
  const long long wanted = 3ll * (sm_count() > 0 ? sm_count() : 148) / 2, blocks = (p.n_tok + 8 * NT - 1) / (8 * NT);
  if (TOP == 4 && (p.w.d_out + 63) / 64 * blocks >= wanted) return launch_few_rows<BITS, TOP, NT, NP, NARROW, T>(p, st);
  if ((p.w.d_out + 31) / 32 * blocks >= wanted) return launch_few_rows<BITS, 2, NT, NP, NARROW, T>(p, st);
  return launch_few_rows<BITS, 1, NT, NP, NARROW, T>(p, st);
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

static int few_tu_error_read_clear() {
  int v = 0;
  if (cudaMemcpyFromSymbol(&v, g_few_error, sizeof(int)) != cudaSuccess) return -1;
  if (v) {
    int z = 0;
    cudaMemcpyToSymbol(g_few_error, &z, sizeof(int));
  }
  return v;
}

}  // namespace tb
