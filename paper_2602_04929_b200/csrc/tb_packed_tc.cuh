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
// but that of float sums.  Backward, a scale belongs to the contraction row, so the weight s (c - z) itself is decoded, as two pieces
// of bf16 (scale8: 2^-17 of the weight in the mean, 2^-13.9 at most; a single piece would put as large an error on dx as its own rounding
// does).  Each piece is a stage of its own with the same tokens, twice the products of a single one.  Accumulations end after 2048
// rows here too: in one sum, 8192 rows put dx 1.5e-5 of its size off, 16384 3.3e-5, all to one side.
//
// Adapters.  scale v M, v [tokens][rank] float, joins the sum as further contraction steps: slots of 16 for a run of tokens with one
// adapter, 16 of its rank and one of two bf16 pieces of scale v (2^-16 of it); tokens outside the run have zeros there.  What is not finite in M goes
// into the tile as 2^-126 of its sign (an infinite v so comes to the infinity that it should) and is added by the epilogue to the run's own
// tokens, so that it reaches no other token.
//
// Roles: warp 0 TMA of the tokens, warp 1 MMA (CTA 0 issues for the pair), warp 2 TMA of the packed words with their zero-points and
// scales, then two warpgroups of decode warps, which take pairs of stages in turn, then eight warps of the epilogue.  The decode warps have
// no global loads of their own: fence.proxy.async, which hands a decoded stage to the tensor cores, waits for all that its thread has
// in flight, and loads of a row by every lane would take the load unit 32 clocks each.  Registers are split 40 / 56 / 56 / 160 / 160 over
// the five warpgroups of a launch at 96 (no more in sum than the launch has).
// Every wait is bounded as in the Hessian kernels.  The MMA warp goes through two stages at a time where it can: its instructions
// between the MMAs, on a scheduler shared with busy warps, are what limits it.
//
// 4096 tokens x 8192 x 8192, 2 bits: 430-440 us, 1.25-1.28 PFLOP/s (a library's bf16 product settles at 1.37 under the power cap);
// gradient, two products: 4099 tokens, 760-790 us, 1.45-1.39 PFLOP/s, where a single piece of the weights takes 390; 8192 tokens x 4096 x
// 4096, 4 bits, 371 us, 1.48 PFLOP/s (204).  Bound by the MMA warp's share of its scheduler and, in long runs, by the power cap.  Small work
// is bound by latency: 64 tokens x 4096 x 4096 takes 13 us, 3 of them the start, 3 until the first words are decoded.
#pragma once

#include "tb_packed.cuh"
#include "tb_packed_decode.cuh"
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

// The contraction is taken in accumulations that end where a scale's columns end, or PT_PART columns (a little less for groups that
// PT_PART does not divide) after their beginning: `end` of the one under way, `g` its group.
struct Parts {
  int group, part, g, group_end, end;
  __device__ __forceinline__ Parts(int gr) : group(gr) {
    const int n = (gr + PT_PART - 1) / PT_PART;
    part = ((gr + n - 1) / n + 31) & ~31;
  }
  __device__ __forceinline__ void start(int k) {  // at column k
    g = k / group;
    const int g0 = g * group;
    group_end = g0 + group;
    end = min(group_end, g0 + ((k - g0) / part + 1) * part);
  }
  __device__ __forceinline__ void next() {
    if (end == group_end) ++g, group_end += group;
    end = min(group_end, end + part);
  }
};

// c - z, exact, times s, as two pieces of bf16; s comes in two as well, hi and lo.  The first piece is (c - z) s less a little more than
// 2^-8 of it, half a step, rounded; the second is what that leaves, more than 0 and at most 2^-6.9 of the weight, so that both have the
// weight's sign and an infinite dy comes to the infinity that it should (a remainder of either sign would give infinity less infinity).
// (c - z) hi less the first piece is exact for codes of four bits, else rounded like the second piece itself: at most 2^-14.9 of the weight
// each, 2^-17 in the mean.
struct ScalePieces {
  unsigned hi, lo, less;  // twice each; less: lo less 1.0625 2^-8 of hi
  __device__ __forceinline__ void set(unsigned v) {
    hi = __byte_perm(v, 0, 0x3232), lo = __byte_perm(v, 0, 0x1010);
    less = bf2(__hfma2(bf2(hi), __float2bfloat162_rn(-0.004150390625f), bf2(lo)));
  }
};
__device__ __forceinline__ void scale8(unsigned (&o)[4], unsigned (&second)[4], const ScalePieces& s) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const __nv_bfloat162 q = bf2(o[i]), first = __hfma2(q, bf2(s.hi), __hmul2(q, bf2(s.less)));
    o[i] = bf2(first);
    second[i] = bf2(__hfma2(q, bf2(s.lo), __hfma2(q, bf2(s.hi), __hneg2(first))));
  }
}

__device__ __forceinline__ void sts16(uint32_t addr, const unsigned (&o)[4]) {
  asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(o[0]), "r"(o[1]), "r"(o[2]), "r"(o[3]) : "memory");
}

// The packed words on their way to the decode warps: 128 columns of the CTA's 128 weight rows (forward, two stages) or of 64 weight
// rows (backward, a stage for each piece), 16 BITS bytes a row, by TMA, then what belongs to their four runs of 32 columns: zero-points,
// backward each beside its scale.  A ring of STAGES such units.  Rows of 32, 64 and 128 bytes are swizzled, so that neighbouring threads' rows lie
// in different banks.
template <int BITS, bool BACK>
struct Raw {
  enum {
    ROWS = BACK ? 64 : 128,
    ROW = 16 * BITS,
    Z = ROWS * ROW,
    BYTES = Z + 4 * ROWS * (BACK ? 8 : 4),
    PAD = (BYTES + 1023) & ~1023,  // swizzled rows start on a multiple of their pattern
    MMA_STAGES = BITS <= 4 ? 6 : 4,  // even: the MMA warp takes two at a time
    ROOM = PT_SMEM - 1024 - 512 - MMA_STAGES * PT_STAGE_BYTES,
    FIT = ROOM / PAD < 8 ? ROOM / PAD : 8,
    // a whole number of turns of the two warpgroups, so that a slot is always the same one's: waits go by parity, and one that skipped a
    // phase of the barrier that it looks at would take the phase before for its own
    STAGES = FIT / 2 * 2
  };
  static_assert(STAGES >= 2, "the ring holds a unit for every turn");
  // 16-byte piece c of row r
  static __device__ __forceinline__ uint32_t piece(int r, int c) {
    if constexpr (ROW == 32) return r * ROW + ((c ^ ((r >> 2) & 1)) << 4);
    if constexpr (ROW == 64) return r * ROW + ((c ^ ((r >> 1) & 3)) << 4);
    if constexpr (ROW == 128) return r * ROW + ((c ^ (r & 7)) << 4);
    return r * ROW + (c << 4);
  }
};

__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src), "r"(bytes), "r"(bar)
               : "memory");
}

// 64 neighbouring codes of a row into the tile: c - z, or (SCALED) the pieces of s (c - z), the second into the stage behind.  FAR: with the
// zero-points' second pieces.
template <int BITS, int C, bool SCALED, bool FAR>
__device__ __forceinline__ void decode_codes(const unsigned (&w)[2 * BITS], const unsigned (&z)[2], const ScalePieces (&s)[2], uint32_t row_addr,
                                             uint32_t sw) {
  if constexpr (C < 8) {
    unsigned o[4];
    decode8<BITS, 8 * C>(w, zero_first<BITS>(z[C / 4]), o);
    if constexpr (FAR)
#pragma unroll
      for (int i = 0; i < 4; ++i) o[i] = bf2(__hadd2(bf2(o[i]), bf2(zero_second<BITS>(z[C / 4]))));
    if constexpr (SCALED) {
      unsigned second[4];
      scale8(o, second, s[C / 4]);
      sts16(row_addr + PT_STAGE_BYTES + ((C ^ sw) << 4), second);
    }
    sts16(row_addr + ((C ^ sw) << 4), o);
    decode_codes<BITS, C + 1, SCALED, FAR>(w, z, s, row_addr, sw);
  }
}
template <int BITS, bool SCALED>
__device__ __forceinline__ void decode_row(const unsigned (&w)[2 * BITS], const unsigned (&z)[2], const ScalePieces (&s)[2], uint32_t row_addr,
                                           uint32_t sw) {
  if (BITS < 8 && __any_sync(0xffffffffu, has_second<BITS>(z[0] | z[1])))
    decode_codes<BITS, 0, SCALED, BITS < 8>(w, z, s, row_addr, sw);
  else
    decode_codes<BITS, 0, SCALED, false>(w, z, s, row_addr, sw);
}

__device__ __forceinline__ bool not_finite2(unsigned v) {
  return (v & 0x7f80u) == 0x7f80u || (v & 0x7f800000u) == 0x7f800000u;
}

// A bf16 piece of two values: themselves rounded, or what that leaves rounded, nothing of what is not finite.  TOP: truncated, so that
// finite values above the largest bf16 stay finite.
template <bool TOP>
__device__ __forceinline__ unsigned pieces_of(float lo, float hi, int piece) {
  const unsigned p = TOP ? first_pieces(lo, hi) : bf2(__floats2bfloat162_rn(lo, hi));
  return piece == 0 ? p : bf2(__floats2bfloat162_rn(rest_of(lo, p << 16), rest_of(hi, p & 0xffff0000u)));
}

// Warpgroups that decode, epilogue warps, the first of these, threads.
struct R {
  enum { DECODE = 2, EPILOGUE = 8, EPI0 = 4 + 4 * DECODE, THREADS = 32 * (EPI0 + EPILOGUE) };
};

template <int BITS, bool BACK>
__global__ void __launch_bounds__(R::THREADS, 1) k_packed_tc(const __grid_constant__ PackedTc p, const __grid_constant__ CUtensorMap xmap, const __grid_constant__ CUtensorMap wmap) {
  using Ring = Raw<BITS, BACK>;
  constexpr int STAGES = Ring::MMA_STAGES;
  extern __shared__ unsigned char pt_smem_raw[];
  const uint32_t raw = smem_u32(pt_smem_raw);
  const uint32_t base = (raw + 1023u) & ~1023u;
  unsigned char* gen_base = pt_smem_raw + (base - raw);
  const uint32_t raw_base = base + STAGES * PT_STAGE_BYTES;
  uint64_t* bars = reinterpret_cast<uint64_t*>(gen_base + (PT_SMEM - 1024 - 512));
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + 2 * STAGES + 4 + 17);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  volatile int* odd_flag = reinterpret_cast<volatile int*>(tmem_slot + 2);  // adapters hold what is not finite (once seen, stays)
  const uint32_t bar0 = smem_u32(bars);
  // full: in CTA 0, the TMA warps and the decode warps of both CTAs (four a stage each) arrive, and the bytes of both; empty, accf: in
  // both, from the commits of CTA 0; acce: in CTA 0, the epilogue warps of both; tile: the decode warps, between tiles with adapters.
  // Waits go by parity, so a barrier must never be two phases from what a wait takes it for: whoever waits for a stage also fills it,
  // and has filled one at most STAGES before, or knows that all those of the tile before are filled.
  auto full_bar = [&](int s) { return bar0 + 8u * s; };
  auto empty_bar = [&](int s) { return bar0 + 8u * (STAGES + s); };
  auto accf_bar = [&](int b) { return bar0 + 8u * (2 * STAGES + b); };
  auto acce_bar = [&](int b) { return bar0 + 8u * (2 * STAGES + 2 + b); };
  auto raw_full = [&](int s) { return bar0 + 8u * (2 * STAGES + 4 + s); };   // a unit's bytes are in the ring
  const uint32_t tile_bar = bar0 + 8u * (2 * STAGES + 20);
  auto raw_empty = [&](int s) { return bar0 + 8u * (2 * STAGES + 12 + s); };  // the decode warps that it belongs to have read it

  uint32_t rank;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
  const int pair = blockIdx.x >> 1, n_pairs = gridDim.x >> 1;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    for (int s = 0; s < STAGES; ++s) {
      mbar_init(full_bar(s), 2 + 8);
      mbar_init(empty_bar(s), 1);
    }
    for (int s = 0; s < 8; ++s) {
      mbar_init(raw_full(s), 1);
      mbar_init(raw_empty(s), 4);
    }
    for (int b = 0; b < 2; ++b) {
      mbar_init(accf_bar(b), 1);
      mbar_init(acce_bar(b), 2 * R::EPILOGUE);
    }
    mbar_init(tile_bar, 4 * R::DECODE);
    *abort_flag = 0;
    *odd_flag = 0;
    mbar_fence_init();
  }
  if (threadIdx.x == 64) prefetch_map(&xmap), prefetch_map(&wmap);
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(512u) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
  }
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  cluster_barrier();
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  const uint32_t tmem_base = *tmem_slot;
  // from here on, what the preparing kernel (and the one that makes x A^T) wrote is read; the operands were there before both
  pdl_wait();
  pdl_trigger();
  const int half_n = p.n_tile >> 1;
  const int n_tiles = p.m_tiles * p.t_tiles * p.splits;
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
    r.n_runs = p.n_runs ? p.n_runs[ti] : 0;
    r.lora = ((r.n_runs * nb * 2 + 7) >> 3) * 2;  // stages of four slots, an even number of them
    return r;
  };
  // stages of a tile's product; backward two for every 64 rows of the contraction, so always an even number
  auto stages_of = [&](const Tile& c) { return (c.k1 - c.k0 + PT_BK - 1) / PT_BK * (BACK ? 2 : 1); };

  if (warp < 4) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 40;");
    if (warp == 0 && lane == 0) {
      // ---------------- TMA producer: this CTA's half of the tokens ----------------
      uint32_t it = 0;
      bool ok = true;
      for (int t = pair; t < n_tiles && ok; t += n_pairs) {
        const Tile c = tile_of(t);
        const int n_st = stages_of(c);
        for (int st = 0; st < n_st + c.lora; ++st, ++it) {
          const int s = it % STAGES;
          if (!mbar_wait(empty_bar(s), ((it / STAGES) & 1u) ^ 1u, abort_flag, &g_packed_error)) {
            ok = false;
            break;
          }
          if (st < n_st) {
            if (rank == 0)
              mbar_expect_tx(full_bar(s), 2u * half_n * PT_BK * 2u);
            else
              mbar_arrive_remote_cta(map_to_rank(full_bar(s), 0));
            tma_load_2d_pair(base + s * PT_STAGE_BYTES + PT_A_BYTES, &xmap, c.k0 + (BACK ? st >> 1 : st) * PT_BK, c.t0 + (int)rank * half_n,
                             map_to_rank(full_bar(s), 0));
          } else {
            mbar_arrive_remote_cta(map_to_rank(full_bar(s), 0));
          }
        }
      }
    } else if (warp == 1 && rank == 0) {
      // ---------------- MMA issuer (CTA 0): the warp goes through the stages together, one lane issues ----------------
      const uint32_t id_main = (1u << 4) | (1u << 7) | (1u << 10) | (BACK ? 1u << 15 : 0u) | ((uint32_t)(p.n_tile >> 3) << 17) | (16u << 24);
      const uint32_t id_lora = id_main | (1u << 15);  // the adapters' matrix is stored along M either way
      const bool one = elect_one();
      uint32_t s = 0, phase = 0, acc_it = 0;
      bool ok = true;
      // the constant halves of the descriptors; an operand's address goes into the low half, in units of 16 bytes
      const uint64_t a_main = BACK ? smem_desc_mn_sw128(base) : smem_desc_k_sw128(base), a_lora = smem_desc_mn_sw128(base);
      const uint64_t b_main = smem_desc_k_sw128(base + PT_A_BYTES);
      constexpr uint32_t a_step = (BACK ? 2048 : 32) >> 4, l_step = 2048 >> 4, b_step = 32 >> 4;
      Parts parts(p.w.group);
      auto wait = [&](uint32_t bar, uint32_t parity) { return mbar_wait_warp(bar, parity, abort_flag, &g_packed_error); };
      auto acc_free = [&]() {
        const bool got = wait(acce_bar(acc_it & 1u), ((acc_it >> 1) & 1u) ^ 1u);
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        return got;
      };
      auto four = [&](uint32_t d, uint64_t ad, uint64_t bd, uint32_t more) {
        umma_bf16_pair(d, ad, bd, id_main, more);
        umma_bf16_pair(d, ad + a_step, bd + b_step, id_main, 1);
        umma_bf16_pair(d, ad + 2 * a_step, bd + 2 * b_step, id_main, 1);
        umma_bf16_pair(d, ad + 3 * a_step, bd + 3 * b_step, id_main, 1);
      };
      for (int t = pair; t < n_tiles && ok; t += n_pairs) {
        const Tile c = tile_of(t);
        const int n_st = stages_of(c);
        int st = 0, left = 0;
        // accumulations of one length and of whole pairs of stages: nothing to keep but how many pairs are left.  Backward all are: a pair is
        // two pieces, and what lies behind the last row is zeros
        const int len = parts.part;
        const bool regular = BACK || (p.w.group % len == 0 && c.k0 % len == 0 && c.k1 % len == 0 && len % (2 * PT_BK) == 0 && s % 2 == 0);
        if (regular) {
          uint32_t d = 0, more = 0;
          for (; st < n_st; st += 2) {
            if (left == 0) {
              ok = acc_free();
              left = BACK ? min(PT_PART / PT_BK, (n_st - st) / 2) : len / (2 * PT_BK);
              d = tmem_base + (acc_it & 1u) * 256u;
              more = 0;
            }
            const uint32_t at = s * (PT_STAGE_BYTES >> 4);
            ok = ok && wait(full_bar(s), phase);
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            if (!ok) break;
            if (one) {
              four(d, a_main + at, b_main + at, more);
              umma_commit_pair(empty_bar(s));
            }
            __syncwarp();
            ok = wait(full_bar(s + 1), phase);
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            if (!ok) break;
            --left;
            if (one) {
              four(d, a_main + at + (PT_STAGE_BYTES >> 4), b_main + at + (PT_STAGE_BYTES >> 4), 1);
              umma_commit_pair(empty_bar(s + 1));
              if (left == 0) umma_commit_pair(accf_bar(acc_it & 1u));
            }
            __syncwarp();
            more = 1;
            if (left == 0) ++acc_it;
            s += 2;
            if (s == STAGES) s = 0, phase ^= 1u;
          }
        }
        int k = c.k0, todo = (c.k1 - c.k0 + 15) >> 4;  // column; steps of 16 left of the tile
        if (st < n_st) parts.start(c.k0);
        for (; st < n_st + c.lora && ok; ++st) {
          ok = wait(full_bar(s), phase);
          if (!ok) break;
          asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
          const uint32_t at = s * (PT_STAGE_BYTES >> 4);
          const uint64_t bd = b_main + at;
          if (!BACK && st < n_st) {
            const uint64_t ad = a_main + at;
            const int steps = min(4, todo);
            todo -= steps;
            for (int kk = 0; kk < steps; ++kk) {
              uint32_t more = 1;
              if (left == 0) {
                ok = acc_free();
                if (!ok) break;
                left = (min(parts.end, c.k1) - k + 15) >> 4;
                parts.next();
                more = 0;
              }
              --left;
              if (one) {
                umma_bf16_pair(tmem_base + (acc_it & 1u) * 256u, ad + kk * a_step, bd + kk * b_step, id_main, more);
                if (left == 0) umma_commit_pair(accf_bar(acc_it & 1u));
              }
              __syncwarp();
              k += 16;
              if (left == 0) ++acc_it;
            }
            if (!ok) break;
            if (one) umma_commit_pair(empty_bar(s));
            __syncwarp();
          } else {
            if (st == n_st) {  // an accumulation of their own: no scale applies to them
              ok = acc_free();
              if (!ok) break;
            }
            const bool last = st == n_st + c.lora - 1;
            if (one) {
#pragma unroll
              for (int kk = 0; kk < PT_BK / 16; ++kk)
                umma_bf16_pair(tmem_base + (acc_it & 1u) * 256u, a_lora + at + kk * l_step, bd + kk * b_step, id_lora,
                               st == n_st && kk == 0 ? 0u : 1u);
              umma_commit_pair(empty_bar(s));
              if (last) umma_commit_pair(accf_bar(acc_it & 1u));
            }
            __syncwarp();
            if (last) ++acc_it;
          }
          if (++s == STAGES) s = 0, phase ^= 1u;
        }
      }
    }
    if (warp == 2 && lane == 0) {
      // ---------------- TMA producer of the packed words, zero-points and scales ----------------
      const int G = p.w.group >> 5, last = (p.w.d_in >> 5) - 1;  // runs of 32 columns with one scale; the last run
      const int n_sz = p.w.group % 128 == 0 ? 1 : 4;             // one zero-point (and scale) for a unit's four runs, or each its own
      const uint32_t bytes = Ring::Z + n_sz * Ring::ROWS * (BACK ? 8u : 4u);
      uint32_t s = 0, phase = 1;
      bool ok = true;
      for (int t = pair; t < n_tiles && ok; t += n_pairs) {
        const Tile c = tile_of(t);
        const int n_u = BACK ? (c.k1 - c.k0 + 63) / 64 : (c.k1 - c.k0 + 127) / 128;
        int r = BACK ? c.k0 : c.m0, j = BACK ? c.m0 : c.k0;
        // (backward, the second CTA's columns may all lie behind the matrix: any zero-points will do for them)
        const int g = min(j >> 5, last) / G;
        int left = (g + 1) * G - (j >> 5);
        const unsigned* zt = p.zt + ((long long)g * p.rows_pad + r) * (BACK ? 2 : 1);  // of the unit's first run
        for (int u = 0; u < n_u; ++u) {
          ok = mbar_wait(raw_empty(s), phase, abort_flag, &g_packed_error);
          if (!ok) break;
          const uint32_t dst = raw_base + s * Ring::PAD, bar = raw_full(s);
          mbar_expect_tx(bar, bytes);
          tma_load_2d(dst, &wmap, (j >> 5) * BITS, r, bar);
          if (n_sz == 1) {
            bulk_load(dst + Ring::Z, zt, Ring::ROWS * (BACK ? 8 : 4), bar);
          } else {
            for (int h = 0; h < 4; ++h) {
              const long long at = (long long)(min((j >> 5) + h, last) / G) * p.rows_pad + r;
              bulk_load(dst + Ring::Z + h * Ring::ROWS * (BACK ? 8 : 4), p.zt + at * (BACK ? 2 : 1), Ring::ROWS * (BACK ? 8 : 4), bar);
            }
          }
          if (BACK) {
            r += 64;
            zt += 128;
          } else {
            j += 128;
            left -= 4;
            if (left == 0) left = G, zt += p.rows_pad;
          }
          if (++s == Ring::STAGES) s = 0, phase ^= 1u;
        }
      }
    }
  } else if (warp < R::EPI0) {
    // ---------------- decode: operand A of this CTA ----------------
    asm volatile("setmaxnreg.dec.sync.aligned.u32 56;");
    const int tid = (threadIdx.x - 128) & 127, turn = (warp - 4) >> 2;  // the warpgroups take turns at the units
    // forward: thread = tile row (a weight row), 64 contraction columns of a stage; backward: 64 weight rows x two halves
    const int my_row = BACK ? tid & 63 : tid;
    const uint32_t row_off = BACK ? (uint32_t)(tid >> 6) * 8192u + (uint32_t)my_row * 128u : (uint32_t)my_row * 128u;
    const uint32_t sw = (uint32_t)(my_row & 7);
    const bool one_sz = p.w.group % 128 == 0;
    constexpr int PER = 2;  // stages of a unit: its two halves, backward its two pieces
    uint32_t it = 0, unit = 0, tiles = 0;
    bool ok = true;
    for (int t = pair; t < n_tiles && ok; t += n_pairs) {
      const Tile c = tile_of(t);
      const int n_st = stages_of(c);
      if (p.n_runs && tiles > 0) {
        ok = mbar_wait_warp(tile_bar, (tiles - 1) & 1u, abort_flag, &g_packed_error);
        if (!ok) break;
      }
      ++tiles;
      for (int st = 0; st < n_st && ok; st += PER, ++unit) {
        const int here = min(PER, n_st - st);
        if ((int)(unit % R::DECODE) != turn) {
          it += here;
          continue;
        }
        const uint32_t rs = unit % Ring::STAGES;
        ok = mbar_wait_warp(raw_full(rs), (unit / Ring::STAGES) & 1u, abort_flag, &g_packed_error);
        if (!ok) break;
        const unsigned char* q = gen_base + (raw_base - base) + rs * Ring::PAD;
#pragma unroll
        for (int i = 0; i < (BACK ? 1 : PER); ++i) {
          if (i >= here) break;
          // outside the matrix the words are zeros and any zero-point gives finite values, which meet zeros or are not stored
          const int half = BACK ? tid >> 6 : i;  // of the unit's 128 columns
          unsigned w[2 * BITS], z[2];
          ScalePieces sc[2];
          if constexpr (BITS % 2 == 0) {
#pragma unroll
            for (int e = 0; e < BITS / 2; ++e) {
              const uint4 v = *reinterpret_cast<const uint4*>(q + Ring::piece(my_row, half * (BITS / 2) + e));
              w[4 * e] = v.x, w[4 * e + 1] = v.y, w[4 * e + 2] = v.z, w[4 * e + 3] = v.w;
            }
          } else {
#pragma unroll
            for (int e = 0; e < BITS; ++e) {
              const uint2 v = *reinterpret_cast<const uint2*>(q + my_row * Ring::ROW + half * 8 * BITS + 8 * e);
              w[2 * e] = v.x, w[2 * e + 1] = v.y;
            }
          }
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const int o = (one_sz ? 0 : 2 * half + h) * Ring::ROWS + my_row;
            if constexpr (BACK) {
              const uint2 v = reinterpret_cast<const uint2*>(q + Ring::Z)[o];
              z[h] = v.x;
              sc[h].set(v.y);
            } else {
              z[h] = reinterpret_cast<const unsigned*>(q + Ring::Z)[o];
            }
          }
          if (BACK || i == here - 1) {
            __syncwarp();
            if (lane == 0) mbar_arrive(raw_empty(rs));
          }
          const int s = it % STAGES;
          ok = mbar_wait_warp(empty_bar(s), ((it / STAGES) & 1u) ^ 1u, abort_flag, &g_packed_error);
          if (BACK && ok) ok = mbar_wait_warp(empty_bar(s + 1), ((it / STAGES) & 1u) ^ 1u, abort_flag, &g_packed_error);
          if (!ok) break;
          decode_row<BITS, BACK>(w, z, sc, base + s * PT_STAGE_BYTES + row_off, sw);
          asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
          __syncwarp();
          if (lane == 0) {
            mbar_arrive_remote_cta(map_to_rank(full_bar(s), 0));
            if (BACK) mbar_arrive_remote_cta(map_to_rank(full_bar(s + 1), 0));
          }
          it += BACK ? 2 : 1;
        }
      }
      // the adapters (where the sum is not split): four slots a stage, slot = (run, 16 of the rank, piece)
      const int n_slots = c.n_runs * nb * 2;
      for (int st = 0; st < c.lora && ok; ++st, ++it) {
        if ((int)((unit + st / PER) % R::DECODE) != turn) continue;  // as if they were further units
        const int s = it % STAGES;
        const uint32_t sa = base + s * PT_STAGE_BYTES, sb = sa + PT_A_BYTES;
        {
          // A: contraction row kk of 64 x two halves of 64 columns
          const int kk = tid & 63, hf = tid >> 6;
          const int slot = 4 * st + (kk >> 4);
          const int run = slot / (2 * nb), q = slot - run * 2 * nb, r = (q >> 1) * 16 + (kk & 15);
          const __nv_bfloat16* m = nullptr;
          if (slot < n_slots && r < p.ad.rank) m = p.M + ((long long)p.runs[c.t0 + run].z * p.ad.rank + r) * p.n_cols;
          uint4 v[8];
#pragma unroll
          for (int ch = 0; ch < 8; ++ch) {
            const int col = c.m0 + 64 * hf + 8 * ch;
            v[ch] = m && col < p.n_cols ? *reinterpret_cast<const uint4*>(m + col) : make_uint4(0u, 0u, 0u, 0u);
          }
          ok = mbar_wait_warp(empty_bar(s), ((it / STAGES) & 1u) ^ 1u, abort_flag, &g_packed_error);
          if (!ok) break;
          bool odd = false;
#pragma unroll
          for (int ch = 0; ch < 8; ++ch) {
            unsigned o[4] = {v[ch].x, v[ch].y, v[ch].z, v[ch].w};
#pragma unroll
            for (int i = 0; i < 4; ++i)
              if (not_finite2(o[i])) {
                odd = true;
                if ((o[i] & 0x7f80u) == 0x7f80u) o[i] = (o[i] & 0xffff8000u) | 0x0080u;
                if ((o[i] & 0x7f800000u) == 0x7f800000u) o[i] = (o[i] & 0x8000ffffu) | 0x00800000u;
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
                const float2* low = reinterpret_cast<const float2*>(p.low + (long long)tok * p.ad.rank + r0);
                float top = 0.0f;
#pragma unroll
                for (int i = 0; i < 8; ++i)
                  if (r0 + 2 * i < p.ad.rank) {  // rank is a multiple of 8
                    const float2 v = low[i];
                    const float a = f * v.x, b = f * v.y;
                    top = fmaxf(top, fmaxf(fabsf(a), fabsf(b)));
                    o[i] = pieces_of<false>(a, b, q & 1);
                  }
                if (top > 3.38953139e38f) {  // the largest bf16
#pragma unroll
                  for (int i = 0; i < 8; ++i)
                    if (r0 + 2 * i < p.ad.rank) o[i] = pieces_of<true>(f * low[i].x, f * low[i].y, q & 1);
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
        if (lane == 0) mbar_arrive_remote_cta(map_to_rank(full_bar(s), 0));
      }
      if (p.n_runs) {
        __syncwarp();
        if (lane == 0) mbar_arrive(tile_bar);
      }
    }
  } else {
    // ---------------- epilogue: 128 columns (TMEM lanes), half of the tokens each ----------------
    asm volatile("setmaxnreg.inc.sync.aligned.u32 160;");
    const int q = warp & 3, hf = (warp - R::EPI0) >> 2;
    Parts parts(p.w.group);
    uint32_t acc_it = 0;
    bool ok = true;
    for (int t = pair; t < n_tiles && ok; t += n_pairs) {
      const Tile c = tile_of(t);
      const int col = c.m0 + q * 32 + lane;
      const int tok0 = c.t0 + hf * half_n, n = min(half_n, p.n_tok - tok0);  // this warp's tokens
      const bool store = col < p.n_cols && n > 0;
      const long long at = (long long)tok0 * p.n_cols + col;
      float* fo = p.part + (long long)c.split * p.n_tok * p.n_cols + at;
      __nv_bfloat16* bo = p.out + at;
      const uint32_t tmem_row = tmem_base + ((uint32_t)(q * 32) << 16) + (uint32_t)(hf * half_n);
      auto acc_full = [&]() {
        ok = mbar_wait_warp(accf_bar(acc_it & 1u), (acc_it >> 1) & 1u, abort_flag, &g_packed_error);
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        return ok;
      };
      auto acc_read = [&]() {
        asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
        __syncwarp();
        if (lane == 0) mbar_arrive_remote_relaxed(map_to_rank(acce_bar(acc_it & 1u), 0));
        ++acc_it;
      };
      float run[128];
#pragma unroll
      for (int i = 0; i < 128; ++i) run[i] = 0.0f;
      if (!BACK) parts.start(c.k0);
      int k = c.k0;
      bool lora = false;
      while (true) {
        if (k >= c.k1) {
          if (lora || c.lora == 0) break;
          lora = true;
        }
        float s = 1.0f;
        if (!BACK && !lora) s = p.st[(long long)parts.g * p.rows_pad + col];
        if (!acc_full()) break;
        const uint32_t taddr = tmem_row + (acc_it & 1u) * 256u;
#pragma unroll
        for (int ch = 0; ch < 8; ++ch) {
          if (16 * ch >= half_n) break;
          uint32_t r[16];
          tmem_ld_32x16(taddr + ch * 16, r);
          asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
          for (int i = 0; i < 16; ++i) run[16 * ch + i] = fmaf(s, __uint_as_float(r[i]), run[16 * ch + i]);
        }
        acc_read();
        if (BACK)
          k += PT_PART;
        else if (!lora)
          k = parts.end, parts.next();
      }
      if (!ok) break;
      if (store) {  // (32 bits hold 127 rows of the 2^24 columns that a call may have)
        if (p.part) {
#pragma unroll
          for (int i = 0; i < 128; ++i)
            if (i < n) fo[i * p.n_cols] = run[i];
        } else {
#pragma unroll
          for (int i = 0; i < 128; ++i)
            if (i < n) bo[i * p.n_cols] = __float2bfloat16(run[i]);
        }
      }
      if (!store) continue;
      // what is not finite in the adapters' rows, to the tokens that it belongs to: whatever finite value was stored there stops
      // being one.  (The flag was set before the adapters' last stage was handed over, hence before its accumulation was complete.)
      if (c.lora && *odd_flag)
        for (int u = 0; u < c.n_runs; ++u) {
          const int4 ru = p.runs[c.t0 + u];
          const float f = p.ad.scale[ru.z];
          for (int r = 0; r < p.ad.rank; ++r) {
            const float m = __bfloat162float(p.M[((long long)ru.z * p.ad.rank + r) * p.n_cols + col]);
            if (fabsf(m) <= 3.4028234e38f) continue;
            for (int tok = max(ru.x, tok0); tok < min(ru.y, tok0 + n); ++tok) {
              const long long i = (long long)(tok - tok0) * p.n_cols;
              bo[i] = __float2bfloat16(__bfloat162float(bo[i]) + f * p.low[(long long)tok * p.ad.rank + r] * m);
            }
          }
        }
    }
  }

  settle(*abort_flag);
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  cluster_barrier();
  if (warp == 1) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(512u) : "memory");
}

}  // namespace tb

namespace tb {

template <int BITS, bool BACK>
tb_status launch_packed_tc(const PackedTc& p, const CUtensorMap& xmap, const CUtensorMap& wmap, int pairs, cudaStream_t st) {
  static bool configured[64] = {false};
  int dev = 0;
  TB_CUDA_CHECK(cudaGetDevice(&dev));
  if (dev < 0 || dev >= 64) return TB_ERR_CUDA;
  if (!configured[dev]) {
    cudaFuncAttributes at;
    TB_CUDA_CHECK(cudaFuncGetAttributes(&at, k_packed_tc<BITS, BACK>));
    if (at.numRegs != 96) return TB_ERR_CUDA;  // the warpgroups' shares add up to what a launch at 96 registers a thread has
    TB_CUDA_CHECK(cudaFuncSetAttribute(k_packed_tc<BITS, BACK>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)PT_SMEM));
    configured[dev] = true;
  }
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(2 * pairs));
  cfg.blockDim = dim3(R::THREADS);
  cfg.dynamicSmemBytes = PT_SMEM;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = 2;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  TB_CUDA_CHECK(cudaLaunchKernelEx(&cfg, k_packed_tc<BITS, BACK>, p, xmap, wmap));
  TB_LAUNCH_CHECK();
  return TB_OK;
}

template <bool BACK>
tb_status launch_packed_tc_bits(const PackedTc& p, const CUtensorMap& xmap, const CUtensorMap& wmap, int pairs, cudaStream_t st) {
  switch (p.w.bits) {
    case 2: return launch_packed_tc<2, BACK>(p, xmap, wmap, pairs, st);
    case 3: return launch_packed_tc<3, BACK>(p, xmap, wmap, pairs, st);
    case 4: return launch_packed_tc<4, BACK>(p, xmap, wmap, pairs, st);
    case 5: return launch_packed_tc<5, BACK>(p, xmap, wmap, pairs, st);
    case 6: return launch_packed_tc<6, BACK>(p, xmap, wmap, pairs, st);
    case 7: return launch_packed_tc<7, BACK>(p, xmap, wmap, pairs, st);
    default: return launch_packed_tc<8, BACK>(p, xmap, wmap, pairs, st);
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
