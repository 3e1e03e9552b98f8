// Products with bit-packed weights on the tensor cores, bf16 activations: the kernel and its launch.
//
// Forward (BACK = 0): out [tokens][d_out] = x Q^T, contraction over d_in.  Backward (BACK = 1): dx [tokens][d_in] = dy Q,
// contraction over d_out.  Either way the result's columns are the rows M of a tcgen05.mma tile and the tokens its columns N: a
// CTA pair (cta_group::2) has 256 columns x n_tile tokens, CTA r of it 128 of the columns (operand A) and half of the tokens
// (operand B).  B comes by TMA, A is decoded from the packed words into the swizzled tile by four warps while the tensor
// cores work on earlier stages: 8192 weights a stage and SM, about 3 instructions for two of them, against the 512 clocks that
// 256 x 256 x 64 takes.
//
// Scales.  Forward, a scale belongs to a row of the tile and a group of contraction columns, so it leaves the sum: the tile
// holds c - z, which bf16 has exactly, and the accumulator of a group (at most 2048 columns of it) is taken from one of two TMEM
// buffers, scaled and added to float registers by the epilogue warps while the other buffer fills.  The product so has no rounding
// but that of float sums.  Backward, a scale belongs to the contraction row: the weight s (c - z) is rounded to bf16 when it is
// decoded, and accumulators are added to the registers every 2048 rows.
//
// Adapters.  scale v M, v [tokens][rank] float, joins the sum as further contraction steps: slots of 16 for a run of tokens with one
// adapter, 16 of its rank and one of two bf16 pieces of scale v (2^-16 of it); tokens outside the run have zeros there.  What is not finite in M goes
// into the tile as zero and is added by the epilogue to the run's own tokens, so that it reaches no other token.
//
// Roles (512 threads): warp 0 TMA, warp 1 MMA (CTA 0 issues for the pair), warps 4-7 decode, warps 8-15 epilogue.  Registers are
// split 56 / 104 / 176 / 176 over the four warpgroups of a launch at 128 (the sums say no more than the launch has).  Every wait is
// bounded as in the Hessian kernels.
#pragma once

#include "tb_packed.cuh"
#include "tb_packed_plan.cuh"
#include "tb_pair.cuh"

namespace tb {

static __device__ int g_packed_error = 0;  // of this translation unit; tb_device_error_flag reads and clears all of them

__device__ __forceinline__ uint64_t smem_desc_k_sw128(uint32_t addr) {
  // K-major, 128-byte swizzle: rows of 64 bf16, 8 rows an atom of 1024 bytes
  uint64_t d = 0;
  d |= (uint64_t)((addr >> 4) & 0x3FFF);
  d |= (uint64_t)1 << 16;
  d |= (uint64_t)(1024 >> 4) << 32;
  d |= (uint64_t)1 << 46;
  d |= (uint64_t)2 << 61;
  return d;
}

// The contraction is taken in accumulations that end where a scale's columns end, or PT_PART columns after their beginning.
struct Parts {
  int group, part;
  __device__ __forceinline__ Parts(int g) : group(g) {
    const int n = (g + PT_PART - 1) / PT_PART;
    part = ((g + n - 1) / n + 31) & ~31;
  }
  __device__ __forceinline__ int end(int k, int k_end) const {  // of the accumulation that has column k
    const int g = k / group, at = k - g * group;
    int e = (at / part + 1) * part;
    if (e > group) e = group;
    return min(k_end, g * group + e);
  }
};

// Field of NB bits from bit POS of the words on.
template <int POS, int NB, int N>
__device__ __forceinline__ unsigned field(const unsigned (&w)[N]) {
  constexpr int i = POS >> 5, s = POS & 31;
  unsigned v;
  if constexpr (s + NB <= 32)
    v = w[i] >> s;
  else
    v = __funnelshift_r(w[i], w[i + 1], s);
  if constexpr (NB < 32) v &= (1u << NB) - 1u;
  return v;
}

__device__ __forceinline__ unsigned bf2(__nv_bfloat162 v) { return *reinterpret_cast<const unsigned*>(&v); }
__device__ __forceinline__ __nv_bfloat162 bf2(unsigned v) { return *reinterpret_cast<const __nv_bfloat162*>(&v); }

// A zero-point as the decoders take it.
struct Zero {
  __nv_bfloat162 up;  // -(128 + z), twice
  float f;            // 2^23 + z
  __device__ __forceinline__ void set(int z) {
    up = __float2bfloat162_rn((float)(-128 - z));
    f = (float)(8388608 + z);
  }
};

// Codes C0 .. C0 + 7 of a lane's words as four pairs of bf16 holding c - z.  A code placed in the low mantissa bits of 128.0
// is 128 + c (up to seven bits), and 128 + z is subtracted; to bring neighbours 16 bits apart, a field of codes (at most 16 bits)
// is joined with itself 16 - b bits higher.  Eight bits go through float.
template <int BITS, int N>
__device__ __forceinline__ unsigned apart(unsigned f) {  // f: N codes; a product where the two do not overlap, else an or
  if constexpr (N * BITS <= 16 - BITS)
    return f * (1u + (1u << (16 - BITS)));
  else
    return f | (f << (16 - BITS));
}
template <int BITS, int C0, int N>
__device__ __forceinline__ void decode8(const unsigned (&w)[N], const Zero& z, unsigned (&o)[4]) {
  if constexpr (BITS == 8) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const unsigned v = w[(C0 + 2 * i) >> 2] >> (8 * ((C0 + 2 * i) & 3));
      const float a = __uint_as_float(0x4B000000u | (v & 0xffu)) - z.f, b = __uint_as_float(0x4B000000u | ((v >> 8) & 0xffu)) - z.f;
      o[i] = bf2(__floats2bfloat162_rn(a, b));
    }
  } else if constexpr (BITS <= 4) {
    constexpr unsigned m = ((1u << BITS) - 1u) * 0x10001u;
    const unsigned y0 = apart<BITS, 4>(field<C0 * BITS, 4 * BITS>(w)), y1 = apart<BITS, 4>(field<(C0 + 4) * BITS, 4 * BITS>(w));
    o[0] = bf2(__hadd2(bf2((y0 & m) | 0x43004300u), z.up));
    o[1] = bf2(__hadd2(bf2(((y0 >> (2 * BITS)) & m) | 0x43004300u), z.up));
    o[2] = bf2(__hadd2(bf2((y1 & m) | 0x43004300u), z.up));
    o[3] = bf2(__hadd2(bf2(((y1 >> (2 * BITS)) & m) | 0x43004300u), z.up));
  } else {
    constexpr unsigned m = ((1u << BITS) - 1u) * 0x10001u;
    const unsigned y0 = apart<BITS, 2>(field<C0 * BITS, 2 * BITS>(w)), y1 = apart<BITS, 2>(field<(C0 + 2) * BITS, 2 * BITS>(w));
    const unsigned y2 = apart<BITS, 2>(field<(C0 + 4) * BITS, 2 * BITS>(w)), y3 = apart<BITS, 2>(field<(C0 + 6) * BITS, 2 * BITS>(w));
    o[0] = bf2(__hadd2(bf2((y0 & m) | 0x43004300u), z.up));
    o[1] = bf2(__hadd2(bf2((y1 & m) | 0x43004300u), z.up));
    o[2] = bf2(__hadd2(bf2((y2 & m) | 0x43004300u), z.up));
    o[3] = bf2(__hadd2(bf2((y3 & m) | 0x43004300u), z.up));
  }
}

// c - z, exact, times s, rounded to bf16 once
__device__ __forceinline__ void scale8(unsigned (&o)[4], float s) {
#pragma unroll
  for (int i = 0; i < 4; ++i)
    o[i] = bf2(__floats2bfloat162_rn(__uint_as_float(o[i] << 16) * s, __uint_as_float(o[i] & 0xffff0000u) * s));
}

__device__ __forceinline__ void sts16(uint32_t addr, const unsigned (&o)[4]) {
  asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(o[0]), "r"(o[1]), "r"(o[2]), "r"(o[3]) : "memory");
}

// A decoder thread's 64 codes of a stage: one row, 2 BITS words, and the zero-point and scale of either half.
template <int BITS>
struct Words {
  unsigned w[2 * BITS];
  int z[2];
  float s[2];
  __device__ __forceinline__ void load(const unsigned* p, int n, bool wide) {  // n words are inside the row
    if (wide && n == 2 * BITS) {
      if constexpr (BITS % 2 == 0) {
#pragma unroll
        for (int i = 0; i < BITS / 2; ++i) {
          const uint4 v = __ldg(reinterpret_cast<const uint4*>(p) + i);
          w[4 * i] = v.x, w[4 * i + 1] = v.y, w[4 * i + 2] = v.z, w[4 * i + 3] = v.w;
        }
      } else {
#pragma unroll
        for (int i = 0; i < BITS; ++i) {
          const uint2 v = __ldg(reinterpret_cast<const uint2*>(p) + i);
          w[2 * i] = v.x, w[2 * i + 1] = v.y;
        }
      }
    } else {
#pragma unroll
      for (int i = 0; i < 2 * BITS; ++i) w[i] = i < n ? __ldg(p + i) : 0u;
    }
  }
};

template <int BITS, int C, bool BACK>
__device__ __forceinline__ void decode_row(const unsigned (&w)[2 * BITS], const Zero (&z)[2], const float (&s)[2], uint32_t row_addr,
                                           uint32_t sw) {
  if constexpr (C < 8) {
    unsigned o[4];
    decode8<BITS, 8 * C>(w, z[C / 4], o);
    if constexpr (BACK) scale8(o, s[C / 4]);
    sts16(row_addr + ((C ^ sw) << 4), o);
    decode_row<BITS, C + 1, BACK>(w, z, s, row_addr, sw);
  }
}

__device__ __forceinline__ bool not_finite2(unsigned v) {
  return (v & 0x7f80u) == 0x7f80u || (v & 0x7f800000u) == 0x7f800000u;
}

// bf16 pieces of v: the value rounded, and what that leaves rounded (nothing where the value is not finite or rounds to infinity)
__device__ __forceinline__ unsigned short piece_of(float v, int piece) {
  const __nv_bfloat16 hi = __float2bfloat16(v);
  if (piece == 0) return *reinterpret_cast<const unsigned short*>(&hi);
  const float h = __bfloat162float(hi);
  const __nv_bfloat16 lo = __float2bfloat16(fabsf(h) <= 3.3895e38f ? v - h : 0.0f);
  return *reinterpret_cast<const unsigned short*>(&lo);
}

template <int BITS, bool BACK>
__global__ void __launch_bounds__(PT_THREADS, 1) k_packed_tc(const __grid_constant__ PackedTc p, const __grid_constant__ CUtensorMap xmap) {
  extern __shared__ unsigned char pt_smem_raw[];
  const uint32_t raw = smem_u32(pt_smem_raw);
  const uint32_t base = (raw + 1023u) & ~1023u;
  unsigned char* gen_base = pt_smem_raw + (base - raw);
  uint64_t* bars = reinterpret_cast<uint64_t*>(gen_base + PT_STAGES * PT_STAGE_BYTES);
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + 2 * PT_STAGES + 4);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  volatile int* odd_flag = reinterpret_cast<volatile int*>(tmem_slot + 2);  // adapters hold what is not finite (once seen, stays)
  const uint32_t bar0 = smem_u32(bars);
  // full: in CTA 0, its TMA warp and the decode warps of both CTAs arrive, and the bytes of both; empty, accf: in both, from the
  // commits of CTA 0; acce: in CTA 0, the epilogue warps of both
  auto full_bar = [&](int s) { return bar0 + 8u * s; };
  auto empty_bar = [&](int s) { return bar0 + 8u * (PT_STAGES + s); };
  auto accf_bar = [&](int b) { return bar0 + 8u * (2 * PT_STAGES + b); };
  auto acce_bar = [&](int b) { return bar0 + 8u * (2 * PT_STAGES + 2 + b); };

  uint32_t rank;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
  const int pair = blockIdx.x >> 1, n_pairs = gridDim.x >> 1;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    for (int s = 0; s < PT_STAGES; ++s) {
      mbar_init(full_bar(s), 1 + 8);
      mbar_init(empty_bar(s), 1);
    }
    for (int b = 0; b < 2; ++b) {
      mbar_init(accf_bar(b), 1);
      mbar_init(acce_bar(b), 16);
    }
    *abort_flag = 0;
    *odd_flag = 0;
    mbar_fence_init();
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(512u) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
  }
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  cluster_barrier();
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  const uint32_t tmem_base = *tmem_slot;
  const int half_n = p.n_tile >> 1;
  const int n_tiles = p.m_tiles * p.t_tiles * p.splits;
  const int group = BACK ? p.n_sum : p.w.group;
  const Parts parts(group);
  struct Tile {
    int m0, t0, split, k0, k1, n_runs, lora;
  };
  const int nb = (p.ad.rank + 15) >> 4;
  auto tile_of = [&](int t) {
    Tile r;
    const int mi = t % p.m_tiles, rest = t / p.m_tiles;
    const int ti = rest % p.t_tiles;
    r.split = rest / p.t_tiles;
    r.m0 = mi * 256 + 128 * (int)rank;
    r.t0 = ti * p.n_tile;
    r.k0 = r.split * p.split_len;
    r.k1 = min(p.n_sum, r.k0 + p.split_len);
    r.n_runs = p.ad.n && r.split == 0 ? p.n_runs[ti] : 0;
    r.lora = (r.n_runs * nb * 2 + 3) >> 2;  // stages of four slots
    return r;
  };

  if (warp < 4) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 56;");
    if (warp == 0 && lane == 0) {
      // ---------------- TMA producer: this CTA's half of the tokens ----------------
      uint32_t it = 0;
      bool ok = true;
      for (int t = pair; t < n_tiles && ok; t += n_pairs) {
        const Tile c = tile_of(t);
        const int n_st = (c.k1 - c.k0 + PT_BK - 1) / PT_BK;
        for (int st = 0; st < n_st + c.lora; ++st, ++it) {
          const int s = it % PT_STAGES;
          if (!mbar_poll(empty_bar(s), ((it / PT_STAGES) & 1u) ^ 1u, abort_flag, &g_packed_error)) {
            ok = false;
            break;
          }
          if (st < n_st) {
            if (rank == 0) mbar_expect_tx(full_bar(s), 2u * half_n * PT_BK * 2u);
            tma_load_2d_pair(base + s * PT_STAGE_BYTES + PT_A_BYTES, &xmap, c.k0 + st * PT_BK, c.t0 + (int)rank * half_n,
                             map_to_rank(full_bar(s), 0));
          } else if (rank == 0) {
            mbar_arrive(full_bar(s));
          }
        }
      }
    } else if (warp == 1 && rank == 0 && lane == 0) {
      // ---------------- MMA issuer (CTA 0) ----------------
      const uint32_t id_main = (1u << 4) | (1u << 7) | (1u << 10) | (BACK ? 1u << 15 : 0u) | ((uint32_t)(p.n_tile >> 3) << 17) | (16u << 24);
      const uint32_t id_lora = id_main | (1u << 15);  // the adapters' matrix is stored along M either way
      uint32_t it = 0, acc_it = 0;
      bool ok = true;
      for (int t = pair; t < n_tiles && ok; t += n_pairs) {
        const Tile c = tile_of(t);
        const int n_st = (c.k1 - c.k0 + PT_BK - 1) / PT_BK;
        int end = 0;  // of the accumulation under way
        for (int st = 0; st < n_st + c.lora && ok; ++st, ++it) {
          const int s = it % PT_STAGES;
          ok = mbar_poll_cluster(full_bar(s), (it / PT_STAGES) & 1u, abort_flag, &g_packed_error);
          if (!ok) break;
          asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
          const uint32_t sa = base + s * PT_STAGE_BYTES, sb = sa + PT_A_BYTES;
          const bool lora = st >= n_st;
#pragma unroll
          for (int kk = 0; kk < PT_BK / 16; ++kk) {
            const int k = c.k0 + st * PT_BK + kk * 16;
            if (!lora && k >= c.k1) break;
            const bool first = lora ? (st == n_st && kk == 0) : (k == c.k0 || k >= end);
            const uint32_t b = acc_it & 1u;
            if (first) {
              ok = mbar_poll_cluster(acce_bar(b), ((acc_it >> 1) & 1u) ^ 1u, abort_flag, &g_packed_error);
              if (!ok) break;
              asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
              if (!lora) end = parts.end(k, c.k1);
            }
            const uint64_t ad = BACK || lora ? smem_desc_mn_sw128(sa + kk * 2048) : smem_desc_k_sw128(sa + kk * 32);
            umma_bf16_pair(tmem_base + b * 256u, ad, smem_desc_k_sw128(sb + kk * 32), lora ? id_lora : id_main, first ? 0u : 1u);
            if (lora ? (st == n_st + c.lora - 1 && kk == PT_BK / 16 - 1) : k + 16 >= end) {
              umma_commit_pair(accf_bar(b));
              ++acc_it;
            }
          }
          if (ok) umma_commit_pair(empty_bar(s));
        }
      }
    }
  } else if (warp < 8) {
    // ---------------- decode: operand A of this CTA ----------------
    asm volatile("setmaxnreg.dec.sync.aligned.u32 104;");
    const int tid = threadIdx.x - 128;
    // forward: thread = tile row (a weight row), 64 contraction columns; backward: 64 weight rows x two halves of the columns
    const int my_row = BACK ? tid & 63 : tid;
    const uint32_t row_off = BACK ? (uint32_t)(tid >> 6) * 8192u + (uint32_t)my_row * 128u : (uint32_t)my_row * 128u;
    const uint32_t sw = (uint32_t)(my_row & 7);
    const bool wide = p.w.d_in % 64 == 0;
    uint32_t it = 0;
    bool ok = true;
    for (int t = pair; t < n_tiles && ok; t += n_pairs) {
      const Tile c = tile_of(t);
      const int n_st = (c.k1 - c.k0 + PT_BK - 1) / PT_BK;
      // first code of this thread at stage st: row r, column j
      auto place = [&](int st, int& r, int& j) {
        r = BACK ? c.k0 + st * PT_BK + my_row : c.m0 + my_row;
        j = BACK ? c.m0 + 64 * (tid >> 6) : c.k0 + st * PT_BK;
      };
      auto fetch = [&](int st, Words<BITS>& wd) {
        int r, j;
        place(st, r, j);
        const int left = r < p.w.d_out && st < n_st ? min(64, p.w.d_in - j) : 0;
        wd.load(p.w.packed + (long long)r * p.w.words + (j >> 5) * BITS, left > 0 ? left / 32 * BITS : 0, wide);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          // outside, the words are zeros: any zero-point gives finite values, which meet zeros or are not stored
          const bool in = left > 32 * h;
          const long long at = (long long)r * p.w.n_g + (int)(((unsigned long long)((j >> 5) + h) * p.group_inv) >> 38);
          wd.z[h] = in ? __ldg(p.w.zeros + at) : 0;
          wd.s[h] = BACK && in ? __ldg(p.w.scales + at) : 0.0f;
        }
      };
      Words<BITS> nxt;
      fetch(0, nxt);
      for (int st = 0; st < n_st && ok; ++st, ++it) {
        const int s = it % PT_STAGES;
        const Words<BITS> cur = nxt;
        fetch(st + 1, nxt);
        Zero z[2];
        z[0].set(cur.z[0]), z[1].set(cur.z[1]);
        int okw = 1;
        if (lane == 0) okw = mbar_poll(empty_bar(s), ((it / PT_STAGES) & 1u) ^ 1u, abort_flag, &g_packed_error) ? 1 : 0;
        ok = __shfl_sync(0xffffffffu, okw, 0) != 0;
        if (!ok) break;
        decode_row<BITS, 0, BACK>(cur.w, z, cur.s, base + s * PT_STAGE_BYTES + row_off, sw);
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
        if (lane == 0) mbar_arrive_remote(map_to_rank(full_bar(s), 0));
      }
      // the adapters: four slots a stage, slot = (run, 16 of the rank, piece)
      const int n_slots = c.n_runs * nb * 2;
      for (int st = 0; st < c.lora && ok; ++st, ++it) {
        const int s = it % PT_STAGES;
        int okw = 1;
        if (lane == 0) okw = mbar_poll(empty_bar(s), ((it / PT_STAGES) & 1u) ^ 1u, abort_flag, &g_packed_error) ? 1 : 0;
        ok = __shfl_sync(0xffffffffu, okw, 0) != 0;
        if (!ok) break;
        const uint32_t sa = base + s * PT_STAGE_BYTES, sb = sa + PT_A_BYTES;
        {
          // A: contraction row kk of 64 x two halves of 64 columns
          const int kk = tid & 63, hf = tid >> 6;
          const int slot = 4 * st + (kk >> 4);
          const int run = slot / (2 * nb), q = slot - run * 2 * nb, r = (q >> 1) * 16 + (kk & 15);
          const __nv_bfloat16* m = nullptr;
          if (slot < n_slots && r < p.ad.rank) m = p.M + ((long long)p.runs[c.t0 + run].z * p.ad.rank + r) * p.n_cols;
          bool odd = false;
#pragma unroll
          for (int ch = 0; ch < 8; ++ch) {
            const int col = c.m0 + 64 * hf + 8 * ch;
            unsigned o[4] = {0u, 0u, 0u, 0u};
            if (m && col < p.n_cols) {
              const uint4 v = __ldg(reinterpret_cast<const uint4*>(m + col));
              o[0] = v.x, o[1] = v.y, o[2] = v.z, o[3] = v.w;
#pragma unroll
              for (int i = 0; i < 4; ++i)
                if (not_finite2(o[i])) {
                  odd = true;
                  if ((o[i] & 0x7f80u) == 0x7f80u) o[i] &= 0xffff0000u;
                  if ((o[i] & 0x7f800000u) == 0x7f800000u) o[i] &= 0xffffu;
                }
            }
            sts16(sa + (uint32_t)hf * 8192u + (uint32_t)kk * 128u + (((uint32_t)ch ^ (uint32_t)(kk & 7)) << 4), o);
          }
          if (odd) *odd_flag = 1;
        }
        if (tid < half_n) {
          // B: a token's 64 slot columns
          const int tok = c.t0 + (int)rank * half_n + tid;
#pragma unroll
          for (int sl = 0; sl < 4; ++sl) {
            const int slot = 4 * st + sl, run = slot / (2 * nb), q = slot - run * 2 * nb;
            unsigned o[8] = {0u, 0u, 0u, 0u, 0u, 0u, 0u, 0u};
            if (slot < n_slots) {
              const int4 ru = p.runs[c.t0 + run];
              if (tok >= ru.x && tok < ru.y) {
                const float f = p.ad.scale[ru.z];
                const int r0 = (q >> 1) * 16;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                  const int r = r0 + 2 * i;
                  if (r < p.ad.rank) {  // rank is a multiple of 8
                    const float2 v = *reinterpret_cast<const float2*>(p.low + (long long)tok * p.ad.rank + r);
                    o[i] = (unsigned)piece_of(f * v.x, q & 1) | ((unsigned)piece_of(f * v.y, q & 1) << 16);
                  }
                }
              }
            }
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              const unsigned part[4] = {o[4 * h], o[4 * h + 1], o[4 * h + 2], o[4 * h + 3]};
              sts16(sb + (uint32_t)tid * 128u + (((uint32_t)(2 * sl + h) ^ (uint32_t)(tid & 7)) << 4), part);
            }
          }
        }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
        if (lane == 0) mbar_arrive_remote(map_to_rank(full_bar(s), 0));
      }
    }
  } else {
    // ---------------- epilogue: 128 columns (TMEM lanes), half of the tokens each ----------------
    asm volatile("setmaxnreg.inc.sync.aligned.u32 176;");
    const int q = warp & 3, hf = (warp - 8) >> 2;
    uint32_t acc_it = 0;
    bool ok = true;
    for (int t = pair; t < n_tiles && ok; t += n_pairs) {
      const Tile c = tile_of(t);
      const int col = c.m0 + q * 32 + lane;
      float run[128];
#pragma unroll
      for (int i = 0; i < 128; ++i) run[i] = 0.0f;
      const float* srow = p.w.scales + (long long)min(col, p.w.d_out - 1) * p.w.n_g;
      int k = c.k0;
      bool lora = false;
      while (ok) {
        if (k >= c.k1) {
          if (lora || c.lora == 0) break;
          lora = true;
        }
        float s = 1.0f;
        if (!BACK && !lora) s = __ldg(srow + k / group);
        const uint32_t b = acc_it & 1u;
        int okw = 1;
        if (lane == 0) okw = mbar_poll(accf_bar(b), (acc_it >> 1) & 1u, abort_flag, &g_packed_error) ? 1 : 0;
        ok = __shfl_sync(0xffffffffu, okw, 0) != 0;
        if (!ok) break;
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        const uint32_t taddr = tmem_base + ((uint32_t)(q * 32) << 16) + b * 256u + (uint32_t)(hf * half_n);
#pragma unroll
        for (int ch = 0; ch < 8; ++ch) {
          if (16 * ch < half_n) {
            uint32_t r[16];
            tmem_ld_32x16(taddr + ch * 16, r);
            asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
            for (int i = 0; i < 16; ++i) run[16 * ch + i] = fmaf(s, __uint_as_float(r[i]), run[16 * ch + i]);
          }
        }
        asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
        __syncwarp();
        if (lane == 0) mbar_arrive_remote(map_to_rank(acce_bar(b), 0));
        ++acc_it;
        if (!lora) k = parts.end(k, c.k1);
      }
      if (!ok) break;
      const int tok0 = c.t0 + hf * half_n;
      if (c.lora && *odd_flag) {
        // (set before the adapters' last stage was handed over, hence before its accumulation was complete)
        if (col < p.n_cols)
          for (int u = 0; u < c.n_runs; ++u) {
            const int4 ru = p.runs[c.t0 + u];
            const float f = p.ad.scale[ru.z];
            for (int r = 0; r < p.ad.rank; ++r) {
              const float m = __bfloat162float(p.M[((long long)ru.z * p.ad.rank + r) * p.n_cols + col]);
              if (fabsf(m) <= 3.4028234e38f) continue;
#pragma unroll
              for (int i = 0; i < 128; ++i) {
                const int tok = tok0 + i;
                if (i < half_n && tok >= ru.x && tok < ru.y) run[i] = fmaf(f * p.low[(long long)tok * p.ad.rank + r], m, run[i]);
              }
            }
          }
      }
      if (col < p.n_cols) {
        if (p.splits > 1) {
          float* o = p.part + ((long long)c.split * p.n_tok + tok0) * p.n_cols + col;
#pragma unroll
          for (int i = 0; i < 128; ++i)
            if (i < half_n && tok0 + i < p.n_tok) o[(long long)i * p.n_cols] = run[i];
        } else {
          __nv_bfloat16* o = p.out + (long long)tok0 * p.n_cols + col;
#pragma unroll
          for (int i = 0; i < 128; ++i)
            if (i < half_n && tok0 + i < p.n_tok) o[(long long)i * p.n_cols] = __float2bfloat16(run[i]);
        }
      }
    }
  }

  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  cluster_barrier();
  if (warp == 1) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(512u) : "memory");
}

}  // namespace tb

namespace tb {

template <int BITS, bool BACK>
tb_status launch_packed_tc(const PackedTc& p, const CUtensorMap& map, int pairs, cudaStream_t st) {
  static bool configured[64] = {false};
  int dev = 0;
  TB_CUDA_CHECK(cudaGetDevice(&dev));
  if (dev < 0 || dev >= 64) return TB_ERR_CUDA;
  if (!configured[dev]) {
    cudaFuncAttributes at;
    TB_CUDA_CHECK(cudaFuncGetAttributes(&at, k_packed_tc<BITS, BACK>));
    if (at.numRegs != 128) return TB_ERR_CUDA;  // the warpgroups' shares add up to what a launch at 128 registers a thread has
    TB_CUDA_CHECK(cudaFuncSetAttribute(k_packed_tc<BITS, BACK>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)PT_SMEM));
    configured[dev] = true;
  }
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(2 * pairs));
  cfg.blockDim = dim3(PT_THREADS);
  cfg.dynamicSmemBytes = PT_SMEM;
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = 2;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  TB_CUDA_CHECK(cudaLaunchKernelEx(&cfg, k_packed_tc<BITS, BACK>, p, map));
  TB_LAUNCH_CHECK();
  return TB_OK;
}

template <bool BACK>
tb_status launch_packed_tc_bits(const PackedTc& p, const CUtensorMap& map, int pairs, cudaStream_t st) {
  switch (p.w.bits) {
    case 2: return launch_packed_tc<2, BACK>(p, map, pairs, st);
    case 3: return launch_packed_tc<3, BACK>(p, map, pairs, st);
    case 4: return launch_packed_tc<4, BACK>(p, map, pairs, st);
    case 5: return launch_packed_tc<5, BACK>(p, map, pairs, st);
    case 6: return launch_packed_tc<6, BACK>(p, map, pairs, st);
    case 7: return launch_packed_tc<7, BACK>(p, map, pairs, st);
    default: return launch_packed_tc<8, BACK>(p, map, pairs, st);
  }
}

static int packed_tc_error_read_clear() {
  int v = 0;
  if (cudaMemcpyFromSymbol(&v, g_packed_error, sizeof(int)) != cudaSuccess) return -1;
  if (v) {
    int z = 0;
    cudaMemcpyToSymbol(g_packed_error, &z, sizeof(int));
  }
  return v;
}

}  // namespace tb
