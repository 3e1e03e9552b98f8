// Low-rank adapters of many requests, bf16 activations: the narrow products x A_i^T (k_adapter_low) and the gradients of the
// adapters' matrices (k_adapter_grad).  A narrow product has a few dozen products for every value it reads, far below what keeps
// the tensor cores busy, so both are bound by reading the activations (or, with a token or two for an adapter, the adapters) once.
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

static __device__ int g_grad_error = 0;

// Columns of an accumulation of x A_i^T at most: every step of 16 may drop the last bits of the sum, always to one side.  In one sum,
// 8192 columns are 2.1e-6 off and 65536 are 1.9e-5; in sums of 512 added in float, 4.7e-7 and 5.2e-7.
enum { LOW_PART = 512 };

// ------------------------------------------------------------------------------------------ x A_i^T
//
// For few tokens, on mma.sync: a CTA has 16 tokens, one of the adapters that they have, up to 64 of its rank and, as one of a cluster,
// a share of the contraction, which its warps split further.  Operands go from global memory straight into fragments: a lane loads 16
// bytes of a row, eight neighbouring columns, and which columns a fragment calls k = 0 .. 15 does not matter as long as both operands
// agree.  Rows of other adapters are not read.  The warps' and the CTAs' sums are added in a fixed order.  8 tokens x 8192, rank 8: 5.7
// us, latency; 1999 x 4096, rank 32: 17 us (16 MB of x, 1.0 TB/s; the adapters come from L2 once for every 16 tokens).

template <int NT>
__global__ void __launch_bounds__(256) k_adapter_low(Adapt ad, const __nv_bfloat16* in, const __nv_bfloat16* M, int n_tok, int width,
                                                     float* low, int late) {
  constexpr int TT = 16, KG = 8, R = 8 * NT, PITCH = R + 1;
  __shared__ int own[TT], pick;
  __shared__ float sum[TT * PITCH];
  uint32_t rank, cs;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
  asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(cs));
  pdl_trigger();  // a product that only needs these sums at its end may start beside
  const int t0 = (blockIdx.x / cs) * TT, r0 = blockIdx.z * 64;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (threadIdx.x < TT) own[threadIdx.x] = t0 + (int)threadIdx.x < n_tok ? adapter_of(ad, t0 + threadIdx.x) : -2;
  if (threadIdx.x == 0) pick = -1;
  __syncthreads();
  // the blockIdx.y-th adapter among the tile's, by its first token
  if (threadIdx.x < 32) {
    bool first = lane < TT && own[lane & (TT - 1)] >= 0;
    for (int k = 0; first && k < lane; ++k) first = own[k] != own[lane];
    const unsigned m = __ballot_sync(0xffffffffu, first);
    if (first && __popc(m & ((1u << lane) - 1u)) == (int)blockIdx.y) pick = own[lane];
  }
  __syncthreads();
  if (blockIdx.y == 0 && rank == 0)  // tokens without an adapter
    for (int e = threadIdx.x; e < TT * R; e += 256) {
      const int t = e / R, r = r0 + e % R;
      if (own[t] == -1 && r < ad.rank) low[(long long)(t0 + t) * ad.rank + r] = 0.0f;
    }
  const int id = pick;
  if (id < 0 && late) pdl_wait();  // `late`: launched beside a product; whoever waits for this kernel waits for both
  if (id < 0) return;  // the same in every CTA of the cluster
  const int g = lane >> 2, q = lane & 3;
  const __nv_bfloat16* xr[2];
  const __nv_bfloat16* mr[NT];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int t = 8 * i + g;
    xr[i] = own[t] == id ? in + (long long)(t0 + t) * width : nullptr;
  }
#pragma unroll
  for (int n = 0; n < NT; ++n) mr[n] = r0 + 8 * n + g < ad.rank ? M + ((long long)id * ad.rank + r0 + 8 * n + g) * width : nullptr;
  float acc[NT][4] = {};
  const int steps = (width + 31) / 32, per = (steps + (int)cs * KG - 1) / ((int)cs * KG);
  const int s0 = ((int)rank * KG + warp) * per, s1 = min(steps, s0 + per);
  auto add = [&](float (&to)[NT][4], int from, int end) {
#pragma unroll 4
    for (int s = from; s < end; ++s) {
      const int k = 32 * s + 8 * q;
      const bool in_k = k < width;
      uint4 x[2], m[NT];
#pragma unroll
      for (int i = 0; i < 2; ++i) x[i] = in_k && xr[i] ? *reinterpret_cast<const uint4*>(xr[i] + k) : make_uint4(0, 0, 0, 0);
#pragma unroll
      for (int n = 0; n < NT; ++n) m[n] = in_k && mr[n] ? *reinterpret_cast<const uint4*>(mr[n] + k) : make_uint4(0, 0, 0, 0);
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        mma_bf16(to[n], x[0].x, x[1].x, x[0].y, x[1].y, m[n].x, m[n].y);
        mma_bf16(to[n], x[0].z, x[1].z, x[0].w, x[1].w, m[n].z, m[n].w);
      }
    }
  };
  constexpr int PART = LOW_PART / 32;
  add(acc, s0, min(s1, s0 + PART));  // most calls end here, without a second set of sums
  for (int p0 = s0 + PART; p0 < s1; p0 += PART) {
    float more[NT][4] = {};
    add(more, p0, min(s1, p0 + PART));
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int c = 0; c < 4; ++c) acc[n][c] += more[n][c];
  }
  // the warps along the contraction, one after the other
  for (int k = 0; k < KG; ++k) {
    if (warp == k) {
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          float* o = sum + (g + 8 * (c >> 1)) * PITCH + 8 * n + 2 * q + (c & 1);
          *o = k ? *o + acc[n][c] : acc[n][c];
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
  if (late) pdl_wait();
}

template <int NT>
static tb_status launch_low(const Adapt& ad, const __nv_bfloat16* in, const __nv_bfloat16* M, int n_tok, int width, float* low,
                            cudaStream_t st, bool late) {
  constexpr int TT = 16;
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
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = (unsigned)cs;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = late ? 2 : 1;
  TB_CUDA_CHECK(cudaLaunchKernelEx(&cfg, k_adapter_low<NT>, ad, in, M, n_tok, width, low, (int)late));
  TB_LAUNCH_CHECK();
  return TB_OK;
}

// The same for many tokens, on tcgen05: 128 tokens are the rows M of the tile, the rank its columns N, both operands by TMA as they
// are stored (K-major).  x so is read once, at HBM's rate, and an adapter once for 128 tokens.  A tile's adapters (AL_COLS / N of
// them, more in further CTAs) are gone through one after the other, each into columns of its own; rows of other adapters are computed and
// dropped.  CTAs of a cluster share the contraction; an accumulation ends after LOW_PART columns.  Where tensor memory has not room for all
// of them (the CTA then has one adapter), they are added to registers as often as it is full, and the products go on from its beginning.
//
// 8192 x 4096, rank 16: 22 us (67 MB at 3.0 TB/s); 4099 x 8192, rank 64: 33 us (67 MB at 2.0 TB/s).  A tile is loaded, multiplied and
// written by one CTA an SM in turn, so that neither end of it overlaps with another tile's loads.

enum { AL_TOK = 128, AL_BK = 64, AL_COLS = 512, AL_THREADS = 192, AL_ROOM = 200 * 1024 };

struct LowTc {
  Adapt ad;
  float* low;
  // n: the rank rounded up to 16; per: contraction columns of a CTA; part: stages of an accumulation, n_parts: those of an adapter that
  // tensor memory holds at a time
  int n_tok, width, n, stages, per, part, n_parts;
};

// ROUNDS: tensor memory fills more than once
template <bool ROUNDS>
__global__ void __launch_bounds__(AL_THREADS, 1)
    k_adapter_low_tc(const __grid_constant__ LowTc p, const __grid_constant__ CUtensorMap xmap, const __grid_constant__ CUtensorMap mmap) {
  extern __shared__ unsigned char al_raw[];
  __shared__ __align__(8) unsigned long long bars[2 * 16 + 2];
  __shared__ uint32_t tmem_slot;
  __shared__ int gave_up, own[AL_TOK], cand[AL_TOK], firsts[4], n_ids;
  const uint32_t base = (smem_u32(al_raw) + 1023u) & ~1023u;
  float* sums = reinterpret_cast<float*>(al_raw + (base - smem_u32(al_raw)));  // after the last stage: [128][n + 1]
  const uint32_t bar0 = smem_u32(bars), done_bar = bar0 + 8u * 32, read_bar = bar0 + 8u * 33;
  auto full_bar = [&](int s) { return bar0 + 8u * s; };
  auto empty_bar = [&](int s) { return bar0 + 8u * (16 + s); };
  uint32_t rank, cs;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
  asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(cs));
  const int t0 = (blockIdx.x / cs) * AL_TOK, tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  if (tid == 0) {
    for (int s = 0; s < p.stages; ++s) {
      mbar_init(full_bar(s), 1);
      mbar_init(empty_bar(s), 1);
    }
    mbar_init(done_bar, 1);
    mbar_init(read_bar, 4);
    gave_up = 0;
    mbar_fence_init();
  }
  if (tid == 160) prefetch_map(&xmap), prefetch_map(&mmap);
  if (tid < AL_TOK) own[tid] = t0 + tid < p.n_tok ? adapter_of(p.ad, t0 + tid) : -2;
  __syncthreads();
  {
    const bool first = tid < AL_TOK && own[tid] >= 0 && (tid == 0 || own[tid - 1] != own[tid]);
    const unsigned m = __ballot_sync(0xffffffffu, first);
    if (warp < 4 && lane == 0) firsts[warp] = __popc(m);
    __syncthreads();
    int at = __popc(m & ((1u << lane) - 1u));
    for (int k = 0; k < min(warp, 4); ++k) at += firsts[k];
    if (first) cand[at] = own[tid];
    __syncthreads();
    if (tid == 0) {  // each adapter once, in the order of their first tokens
      const int all = firsts[0] + firsts[1] + firsts[2] + firsts[3];
      int n = 0;
      for (int i = 0; i < all; ++i) {
        int k = 0;
        while (k < n && cand[k] != cand[i]) ++k;
        if (k == n) cand[n++] = cand[i];
      }
      n_ids = n;
    }
    __syncthreads();
  }
  const int room = AL_COLS / (p.n * p.n_parts), id0 = (int)blockIdx.y * room, ids = min(room, n_ids - id0);
  if (blockIdx.y == 0 && rank == 0)  // tokens without an adapter
    for (int t = warp; t < AL_TOK; t += AL_THREADS / 32)
      if (own[t] == -1)
        for (int r = lane; r < p.ad.rank; r += 32) p.low[(long long)(t0 + t) * p.ad.rank + r] = 0.0f;
  if (ids <= 0) return;  // the same in every CTA of the cluster
  if (warp == 5) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_slot)), "r"((uint32_t)AL_COLS) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  const uint32_t tmem = tmem_slot;
  const int stage_bytes = AL_TOK * 128 + p.n * 128;  // a multiple of 1024: n is one of 16, hence of 8 rows of 128 bytes
  const int k0 = (int)rank * p.per, k1 = min(p.width, k0 + p.per), n_st = k1 > k0 ? (k1 - k0 + AL_BK - 1) / AL_BK : 0;
  const int full = p.part * p.n_parts, rounds = ROUNDS && n_st > full ? (n_st + full - 1) / full : 1;  // stages that fill tensor memory
  float total[ROUNDS ? 128 : 1];  // warps 0 to 3: a token's sums of the rounds but the last
  if (ROUNDS && warp < 4) {
#pragma unroll
    for (int i = 0; i < (ROUNDS ? 128 : 1); ++i) total[i] = 0.0f;
    for (int round = 0; round + 1 < rounds; ++round) {
      if (!__all_sync(0xffffffffu, mbar_wait(done_bar, round & 1u, &gave_up, &g_grad_error))) break;
      asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
      for (int part = 0; part < p.n_parts; ++part)
#pragma unroll
        for (int c = 0; c < 128; c += 8) {
          if (c >= p.n) break;
          uint32_t r[8];
          tmem_ld_32x8(tmem + ((uint32_t)(warp * 32) << 16) + (uint32_t)(part * p.n + c), r);
          asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
          for (int i = 0; i < 8; ++i) total[ROUNDS ? c + i : 0] += __uint_as_float(r[i]);
        }
      asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
      __syncwarp();
      if (lane == 0) mbar_arrive(read_bar);
    }
  }
  if (warp == 4 && lane == 0) {
    int s = 0;
    uint32_t phase = 1;
    bool ok = true;
    for (int a = 0; a < ids && ok; ++a)
      for (int st = 0; st < n_st; ++st) {
        ok = mbar_wait(empty_bar(s), phase, &gave_up, &g_grad_error);
        if (!ok) break;
        const uint32_t dst = base + s * stage_bytes;
        mbar_expect_tx(full_bar(s), stage_bytes);
        tma_load_2d(dst, &xmap, k0 + st * AL_BK, t0, full_bar(s));
        tma_load_2d(dst + AL_TOK * 128, &mmap, k0 + st * AL_BK, cand[id0 + a] * p.ad.rank, full_bar(s));
        if (++s == p.stages) s = 0, phase ^= 1u;
      }
  } else if (warp == 5) {
    const uint32_t idesc = (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(p.n >> 3) << 17) | (8u << 24);
    const bool one = elect_one();
    const uint64_t desc = smem_desc_k(base, 16) & ~((uint64_t)0x3fff << 32) | ((uint64_t)(1024 >> 4) << 32) | ((uint64_t)2 << 61);
    int s = 0;
    uint32_t phase = 0;
    bool ok = true;
    for (int a = 0; a < ids && ok; ++a) {
      int in_part = 0, part = 0, round = 0;
      for (int st = 0; st < n_st; ++st) {
        ok = __all_sync(0xffffffffu, mbar_wait(full_bar(s), phase, &gave_up, &g_grad_error));
        if (!ok) break;
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        if (one) {
          const uint64_t x = desc + (uint64_t)(s * (stage_bytes >> 4)), m = x + (AL_TOK * 128 >> 4);
          const uint32_t d = tmem + (uint32_t)((a * p.n_parts + part) * p.n);
#pragma unroll
          for (int kk = 0; kk < 4; ++kk) umma_bf16(d, x + 2 * kk, m + 2 * kk, idesc, in_part > 0 || kk > 0 ? 1u : 0u);
          umma_commit(empty_bar(s));
        }
        __syncwarp();
        if (++in_part == p.part) in_part = 0, ++part;
        if (++s == p.stages) s = 0, phase ^= 1u;
        if (ROUNDS && part == p.n_parts && st + 1 < n_st) {  // full: from its beginning again, once these have been read
          if (one) umma_commit(done_bar);
          __syncwarp();
          ok = __all_sync(0xffffffffu, mbar_wait(read_bar, round & 1u, &gave_up, &g_grad_error));
          if (!ok) break;
          asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
          part = 0, ++round;
        }
      }
    }
    if (one) umma_commit(done_bar);
  }
  __syncthreads();
  bool ok = __all_sync(0xffffffffu, mbar_wait(done_bar, (rounds - 1) & 1u, &gave_up, &g_grad_error));
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  // a thread of the first four warps has a token, whose sums are in the columns of its adapter
  const uint32_t mine = smem_u32(sums);
  const int pitch = p.n + 1, parts_here = ok ? (n_st - (rounds - 1) * full + p.part - 1) / p.part : 0;
  if (warp < 4) {
    bool here = false;
    for (int a = 0; a < ids; ++a) {
      const bool own_row = own[tid] == cand[id0 + a];
      if (!__any_sync(0xffffffffu, own_row)) continue;
      here = here || own_row;
#pragma unroll(ROUNDS ? 4 : 1)
      for (int c = 0; c < 128; c += 32) {
        if (c >= p.n) break;
        float v[32];
#pragma unroll
        for (int i = 0; i < 32; ++i) v[i] = ROUNDS ? total[ROUNDS ? c + i : 0] : 0.0f;
        for (int part = 0; part < parts_here; ++part) {
          uint32_t r[4][8];
#pragma unroll
          for (int h = 0; h < 4; ++h)
            if (c + 8 * h < p.n) tmem_ld_32x8(tmem + ((uint32_t)(warp * 32) << 16) + (uint32_t)((a * p.n_parts + part) * p.n + c + 8 * h), r[h]);
          asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
          for (int h = 0; h < 4; ++h)
#pragma unroll
            for (int i = 0; i < 8; ++i)
              if (c + 8 * h < p.n) v[8 * h + i] += __uint_as_float(r[h][i]);
        }
        if (own_row)
#pragma unroll
          for (int i = 0; i < 32; ++i)
            if (c + i < p.n) sums[tid * pitch + c + i] = v[i];
      }
    }
    if (!here) own[tid] = -2;  // of another CTA's adapters, or none
  }
  if (cs > 1)
    cluster_barrier();
  else
    __syncthreads();
  for (int t = warp * (int)cs + (int)rank; t < AL_TOK; t += AL_THREADS / 32 * (int)cs) {  // a warp has a row
    if (own[t] < 0) continue;
    for (int r = lane; r < p.ad.rank; r += 32) {
      float u[8];
#pragma unroll
      for (uint32_t k = 0; k < 8; ++k)
        u[k] = k >= cs ? 0.0f : cs > 1 ? ld_cluster(map_to_rank(mine + 4u * (t * pitch + r), k)) : sums[t * pitch + r];
      float v = u[0];
#pragma unroll
      for (uint32_t k = 1; k < 8; ++k)
        if (k < cs) v += u[k];
      p.low[(long long)(t0 + t) * p.ad.rank + r] = v;
    }
  }
  if (cs > 1) cluster_barrier();  // nobody leaves while its sums are read
  settle(*(volatile int*)&gave_up);
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  if (warp == 5) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"((uint32_t)AL_COLS) : "memory");
}

template <bool ROUNDS>
static tb_status launch_low_tc(const LowTc& p, const CUtensorMap& xmap, const CUtensorMap& mmap, unsigned x, unsigned y, int cs, cudaStream_t st) {
  static bool configured[64] = {false};
  int dev = 0;
  TB_CUDA_CHECK(cudaGetDevice(&dev));
  if (dev < 0 || dev >= 64) return TB_ERR_CUDA;
  if (!configured[dev]) {
    TB_CUDA_CHECK(cudaFuncSetAttribute(k_adapter_low_tc<ROUNDS>, cudaFuncAttributeMaxDynamicSharedMemorySize, AL_ROOM + 1024));
    configured[dev] = true;
  }
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(x, y);
  cfg.blockDim = dim3(AL_THREADS);
  cfg.dynamicSmemBytes = AL_ROOM + 1024;  // no second CTA that would wait for tensor memory
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = (unsigned)cs;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  TB_CUDA_CHECK(cudaLaunchKernelEx(&cfg, k_adapter_low_tc<ROUNDS>, p, xmap, mmap));
  TB_LAUNCH_CHECK();
  return TB_OK;
}

static tb_status adapter_low_tc(const Adapt& ad, const __nv_bfloat16* in, const __nv_bfloat16* M, int n_tok, int width, float* low, cudaStream_t st) {
  const int tiles = (n_tok + AL_TOK - 1) / AL_TOK, sms = sm_count() > 0 ? sm_count() : 148;
  int cs = 1;  // CTAs along the contraction, up to one an SM
  while (cs < 8 && tiles * cs * 2 <= sms && width / (2 * cs) >= 256) cs *= 2;
  LowTc p;
  p.ad = ad, p.low = low, p.n_tok = n_tok, p.width = width;
  p.n = (ad.rank + 15) / 16 * 16;
  p.per = ((width + cs - 1) / cs + AL_BK - 1) / AL_BK * AL_BK;
  p.n_parts = min((p.per + LOW_PART - 1) / LOW_PART, AL_COLS / p.n);
  p.part = min(LOW_PART / AL_BK, (p.per / AL_BK + p.n_parts - 1) / p.n_parts);
  const int stage = AL_TOK * 128 + p.n * 128;
  p.stages = min(12, AL_ROOM / stage);
  const int ys = (min(AL_TOK, min(ad.n_req, ad.n)) + AL_COLS / (p.n * p.n_parts) - 1) / (AL_COLS / (p.n * p.n_parts));
  CUtensorMap xmap, mmap;
  TB_TRY(make_map_2d(&xmap, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, in, (unsigned long long)width, (unsigned long long)n_tok, AL_BK, AL_TOK,
                     CU_TENSOR_MAP_SWIZZLE_128B));
  TB_TRY(make_map_2d(&mmap, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, M, (unsigned long long)width, (unsigned long long)ad.n * ad.rank, AL_BK, p.n,
                     CU_TENSOR_MAP_SWIZZLE_128B));
  const unsigned x = (unsigned)(tiles * cs), y = (unsigned)ys;
  return p.per / AL_BK > p.part * p.n_parts ? launch_low_tc<true>(p, xmap, mmap, x, y, cs, st) : launch_low_tc<false>(p, xmap, mmap, x, y, cs, st);
}

// Tiles of 16 tokens start sooner and compute less for rows of other adapters, but read an adapter once for every 16 tokens.
// Measured, tiles of 16 / tcgen05 (us): rank 128, 4 requests, 512 x 256 7.6 / 23.7, 512 x 1024 10.2 / 16.0, 512 x 4096 25.7 / 16.2, 1024 x
// 4096 18.8 / 16.4; rank 64, 1024 x 1024 9.0 / 12.2, 2048 x 2048 15.1 / 18.5, 4096 x 1024 12.3 / 12.5, 1024 x 4096 17.2 / 13.3, 1024 x 8192
// 44 / 18; rank 16, 4096 x 4096 14.1 / 17.0.  Where requests are short, most rows of a tile of 128 are another adapter's.
enum { LOW_TC_WORK = 1 << 28 };  // tokens x rank x width
bool adapter_low_in_small_tiles(const Adapt& ad, int n_tok, int width) {
  return (long long)n_tok * ad.rank * width < LOW_TC_WORK || n_tok / ad.n_req < 48;  // n_tok < 2^30, rank <= 2^7, width <= 2^24
}

// low [n_tok][rank] = in M_i^T for the adapter i of every token, zero for a token without one.  `late` (small tiles only): the call
// before on the stream is a product that does not need it, and the one after waits for both.
tb_status adapter_low_bf16(const Adapt& ad, const __nv_bfloat16* in, const __nv_bfloat16* M, int n_tok, int width, float* low, bool late,
                           cudaStream_t st) {
  if (adapter_low_in_small_tiles(ad, n_tok, width)) {
    if (ad.rank <= 8) return launch_low<1>(ad, in, M, n_tok, width, low, st, late);
    if (ad.rank <= 16) return launch_low<2>(ad, in, M, n_tok, width, low, st, late);
    if (ad.rank <= 32) return launch_low<4>(ad, in, M, n_tok, width, low, st, late);
    return launch_low<8>(ad, in, M, n_tok, width, low, st, late);
  }
  return adapter_low_tc(ad, in, M, n_tok, width, low, st);
}

// ------------------------------------------------------------------------------------------ gradients
//
// G_i [rank][width] = scale_i sum over i's tokens of low_t^T in_t, on tcgen05: 128 columns of the input are the rows M of the tile,
// the rank its columns N, tokens the contraction, 64 of them a stage.  Both operands are written to shared memory by the producer
// warps, as they are stored (M- and N-major, 128-byte swizzle): the input as it is, or its 8-bit codes as bf16 integers; low as
// three bf16 pieces side by side (N = 3 RP), all 24 bits of it, times the codes' scale of its token and these 128 columns.  Tokens
// behind the end of a request are zeros in both, so nothing of another request gets in.  Full pieces of bf16 input come by TMA,
// ahead of the producers.  The kernel is bound by reading the input
// and, at high ranks, by making the pieces.  A CTA has one adapter's columns and, as one of a cluster, every cs-th piece of 64
// tokens; accumulations end after 256 tokens (every step of 16 may drop the last bit); the CTAs' sums are added in a fixed order through
// distributed shared memory.  8192 x 4096, rank 16: 25 us (67 MB at 2.7 TB/s); 4099 x 8192, rank 64: 50 us, from 8 bits 61 us, where the
// pieces of `low`, made again for every 128 columns, take the time.

enum { AG_TOK = 64, AG_COLS = 128, AG_PART = 4, AG_THREADS = 320 };  // AG_PART: stages of an accumulation

// RP: the rank, rounded up to 16, 32, 64 or 128.
template <int RP>
struct GradShape {
  enum {
    N = 3 * RP,
    BOXES = (N + 63) / 64,  // of 64 columns
    A_BYTES = AG_TOK * AG_COLS * 2,
    STAGE = A_BYTES + BOXES * AG_TOK * 128,
    STAGES = RP == 16 ? 4 : RP == 64 ? 2 : 3,
    TMEM = RP == 16 ? 64 : RP == 32 ? 128 : RP == 64 ? 256 : 512,
    SUMS = RP * AG_COLS * 4,
    SMEM = (STAGES * STAGE > SUMS ? STAGES * STAGE : SUMS) + 1024
  };
};

__device__ __forceinline__ void sts8(uint32_t addr, unsigned a, unsigned b) {
  asm volatile("st.shared.v2.b32 [%0], {%1, %2};" ::"r"(addr), "r"(a), "r"(b) : "memory");
}
__device__ __forceinline__ void sts16(uint32_t addr, uint4 v) {
  asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}
__device__ __forceinline__ unsigned pair_bf16(float a, float b) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<const unsigned*>(&v);
}

template <int RP, bool EIGHT>
__global__ void __launch_bounds__(AG_THREADS, RP == 128 ? 1 : 2)
    k_adapter_grad(Adapt ad, const void* __restrict__ in, const float* __restrict__ in_scales, const float* __restrict__ low, int n_tok,
                   int width, float* __restrict__ G, const __grid_constant__ CUtensorMap imap) {
  using S = GradShape<RP>;
  extern __shared__ unsigned char ag_raw[];
  __shared__ __align__(8) unsigned long long bars[2 * S::STAGES + 1];
  __shared__ uint32_t tmem_slot;
  __shared__ int gave_up;
  __shared__ int2 piece[256];
  __shared__ int n_piece, wsum[8];
  const uint32_t base = (smem_u32(ag_raw) + 1023u) & ~1023u;
  float* sums = reinterpret_cast<float*>(ag_raw + (base - smem_u32(ag_raw)));  // after the last stage: [RP][128]
  const uint32_t bar0 = smem_u32(bars);
  auto full_bar = [&](int s) { return bar0 + 8u * s; };
  auto empty_bar = [&](int s) { return bar0 + 8u * (S::STAGES + s); };
  const uint32_t done_bar = bar0 + 16u * S::STAGES;
  uint32_t rank, cs;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
  asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(cs));
  const int c0 = (blockIdx.x / cs) * AG_COLS, id = blockIdx.y;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  if (tid == 0) {
    for (int s = 0; s < S::STAGES; ++s) {
      mbar_init(full_bar(s), EIGHT ? 8 : 9);  // the producers', and that of the warp that fetches full pieces
      mbar_init(empty_bar(s), 1);
    }
    mbar_init(done_bar, 1);
    gave_up = 0;
    mbar_fence_init();
  }
  if (warp == 8) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_slot)), "r"((uint32_t)S::TMEM) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  const uint32_t tmem = tmem_slot;
  const int n_run = (width + CKPT_RUN - 1) / CKPT_RUN;

  // producers: a thread has 64 bytes of the input's tile (16-byte units e = tid + 256 i), and fours of low, neighbours side by side
  uint4 xv[EIGHT ? 2 : 4];
  float lv[RP / 4], fv[RP / 16];
  auto fetch = [&](int t, int n) {  // 64 tokens from t on, n of them inside
    if constexpr (EIGHT) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int e = tid + 256 * i, row = e >> 3, u = e & 7;
        const signed char* src = static_cast<const signed char*>(in) + (long long)(t + row) * width + c0 + 16 * u;
        xv[i] = row < n && c0 + 16 * u < width ? __ldcs(reinterpret_cast<const uint4*>(src)) : make_uint4(0, 0, 0, 0);
      }
    } else if (n < AG_TOK) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int e = tid + 256 * i, row = e >> 4, u = e & 15;
        const __nv_bfloat16* src = static_cast<const __nv_bfloat16*>(in) + (long long)(t + row) * width + c0 + 8 * u;
        xv[i] = row < n && c0 + 8 * u < width ? __ldcs(reinterpret_cast<const uint4*>(src)) : make_uint4(0, 0, 0, 0);
      }
    }
#pragma unroll
    for (int k = 0; k < RP / 16; ++k) {
      const int e = tid + 256 * k, lt = e / (RP / 4), r = 4 * (e % (RP / 4));
      const bool in4 = lt < n && r < ad.rank;
      float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
      if (in4) v = __ldg(reinterpret_cast<const float4*>(low + (long long)(t + lt) * ad.rank + r));
      if (EIGHT) fv[k] = in4 ? __ldg(in_scales + (long long)(t + lt) * n_run + c0 / CKPT_RUN) : 0.0f;
      lv[4 * k] = v.x, lv[4 * k + 1] = v.y, lv[4 * k + 2] = v.z, lv[4 * k + 3] = v.w;
    }
  };
  auto store = [&](uint32_t stage, int n) {
    if constexpr (EIGHT) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int e = tid + 256 * i, row = e >> 3, u = e & 7;
        const unsigned w[4] = {xv[i].x, xv[i].y, xv[i].z, xv[i].w};
        unsigned o[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          // codes as floats: the byte, its sign flipped, in the low mantissa bits of 2^23, less 2^23 + 128
          const unsigned v = (w[k >> 1] ^ 0x80808080u) >> (16 * (k & 1));
          const float a = __uint_as_float(__byte_perm(v, 0x4B000000u, 0x7540)) - 8388736.0f;
          const float b = __uint_as_float(__byte_perm(v, 0x4B000000u, 0x7541)) - 8388736.0f;
          o[k] = pair_bf16(a, b);
        }
        const uint32_t at = stage + (u >> 2) * 8192 + row * 128;
#pragma unroll
        for (int h = 0; h < 2; ++h)
          sts16(at + ((((u & 3) * 2 + h) ^ (row & 7)) << 4), make_uint4(o[4 * h], o[4 * h + 1], o[4 * h + 2], o[4 * h + 3]));
      }
    } else if (n < AG_TOK) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int e = tid + 256 * i, row = e >> 4, u = e & 15;
        sts16(stage + (u >> 3) * 8192 + row * 128 + (((u & 7) ^ (row & 7)) << 4), xv[i]);
      }
    }
#pragma unroll
    for (int k = 0; k < RP / 16; ++k) {
      const int e = tid + 256 * k, lt = e / (RP / 4), r = 4 * (e % (RP / 4));
      float v[4] = {lv[4 * k], lv[4 * k + 1], lv[4 * k + 2], lv[4 * k + 3]};
      if (EIGHT) v[0] *= fv[k], v[1] *= fv[k], v[2] *= fv[k], v[3] *= fv[k];
#pragma unroll
      for (int p = 0; p < 3; ++p) {
        const unsigned a = first_pieces(v[0], v[1]), b = first_pieces(v[2], v[3]);
        const int n = p * RP + r;
        sts8(stage + S::A_BYTES + (n >> 6) * 8192 + lt * 128 + ((((n & 63) >> 3) ^ (lt & 7)) << 4) + (n & 7) * 2, a, b);
        if (p < 2) {
          v[0] = rest_of(v[0], a << 16), v[1] = rest_of(v[1], a & 0xffff0000u);
          v[2] = rest_of(v[2], b << 16), v[3] = rest_of(v[3], b & 0xffff0000u);
        }
      }
    }
  };

  // the MMAs of a stage, and after the last of an accumulation its end: by warp 8
  const uint32_t idesc = idesc_bf16_mn(128, RP == 128 ? 192 : S::N);
  float acc[RP / 2];  // producers: lane's column of the input, half of the rank
#pragma unroll
  for (int i = 0; i < RP / 2; ++i) acc[i] = 0.0f;
  uint32_t it = 0, parts = 0;
  bool ok = true;
  auto drain = [&]() {  // the finished accumulation into the registers (warps 0-7)
    ok = __all_sync(0xffffffffu, mbar_wait(done_bar, parts & 1u, &gave_up, &g_grad_error));
    ++parts;
    if (!ok) return;
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
#pragma unroll
    for (int p = 2; p >= 0; --p)
#pragma unroll
      for (int c = 0; c < RP / 2; c += 8) {
        uint32_t r[8];
        tmem_ld_32x8(tmem + ((uint32_t)((warp & 3) * 32) << 16) + p * RP + (warp >> 2) * (RP / 2) + c, r);
        asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
        for (int i = 0; i < 8; ++i) acc[c + i] += __uint_as_float(r[i]);
      }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  };

  for (int j0 = 0; j0 < ad.n_req; j0 += 256) {
    // the adapter's requests among these 256, in their order
    int b = 0, e = 0;
    if (warp < 8) {
      if (j0 + tid < ad.n_req && ad.ids[j0 + tid] == id) {
        b = max(0, ad.starts[j0 + tid]);
        e = min(n_tok, ad.starts[j0 + tid + 1]);
      }
      const unsigned m = __ballot_sync(0xffffffffu, e > b);
      if (lane == 0) wsum[warp] = __popc(m);
      __syncwarp();
    }
    __syncthreads();
    if (warp < 8) {
      const unsigned m = __ballot_sync(0xffffffffu, e > b);
      int at = __popc(m & ((1u << lane) - 1u)), all = 0;
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        if (k < warp) at += wsum[k];
        all += wsum[k];
      }
      if (e > b) piece[at] = make_int2(b, e);
      if (tid == 0) n_piece = all;
    }
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
    if (warp < 8 && rq < n_piece) fetch(t, min(AG_TOK, piece[rq].y - t));
    uint32_t in_part = 0;
    while (rq < n_piece && ok) {
      const uint32_t s = it % S::STAGES, ph = (it / S::STAGES) & 1u;
      const uint32_t stage = base + s * S::STAGE;
      const int here = t, n_here = min(AG_TOK, piece[rq].y - t);
      advance((int)cs);
      const bool more = rq < n_piece, last = !more || in_part == AG_PART - 1;
      if (warp < 8) {
        ok = __all_sync(0xffffffffu, mbar_wait(empty_bar(s), ph ^ 1u, &gave_up, &g_grad_error));
        if (ok) {
          store(stage, n_here);
          asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
          __syncwarp();
          if (lane == 0) mbar_arrive(full_bar(s));
          // (loads after the fence: it waits for all that its thread has in flight)
          if (more) fetch(t, min(AG_TOK, piece[rq].y - t));
          if (last) drain();
        }
      } else if (warp == 9) {
        if (!EIGHT) {
          ok = __all_sync(0xffffffffu, mbar_wait(empty_bar(s), ph ^ 1u, &gave_up, &g_grad_error));
          if (ok && lane == 0) {
            if (n_here == AG_TOK) {
              mbar_expect_tx(full_bar(s), S::A_BYTES);
              tma_load_2d(stage, &imap, c0, here, full_bar(s));
              tma_load_2d(stage + 8192, &imap, c0 + 64, here, full_bar(s));
            } else {
              mbar_arrive(full_bar(s));
            }
          }
        }
      } else {
        ok = __all_sync(0xffffffffu, mbar_wait(full_bar(s), ph, &gave_up, &g_grad_error));
        if (ok && elect_one()) {
          asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
#pragma unroll
          for (int kk = 0; kk < AG_TOK / 16; ++kk) {
            const uint64_t a = smem_desc_mn_sw128(stage + kk * 2048);
            const uint32_t first = in_part > 0 || kk > 0 ? 1u : 0u;
            umma_bf16(tmem, a, smem_desc_mn_sw128(stage + S::A_BYTES + kk * 2048), idesc, first);
            if (RP == 128) umma_bf16(tmem + 192, a, smem_desc_mn_sw128(stage + S::A_BYTES + 3 * 8192 + kk * 2048), idesc, first);
          }
          umma_commit(empty_bar(s));
          if (last) umma_commit(done_bar);
        }
        __syncwarp();
      }
      in_part = last ? 0 : in_part + 1;
      ++it;
      // the next accumulation overwrites the drained one: its first stage is handed over by every producer after its drain
    }
    __syncthreads();
  }
  settle(*(volatile int*)&gave_up);
  __syncthreads();
  // (every MMA has been drained: the sums may take the stages' place)
  if (warp < 8) {
    const int c = (warp & 3) * 32 + lane;
#pragma unroll
    for (int i = 0; i < RP / 2; ++i) sums[((warp >> 2) * (RP / 2) + i) * AG_COLS + c] = acc[i];
  }
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  if (warp == 8) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"((uint32_t)S::TMEM) : "memory");
  if (cs > 1) cluster_barrier();
  const float sc = ad.scale[id];
  const uint32_t mine = smem_u32(sums);
  for (int e = tid + AG_THREADS * (int)rank; e < RP * AG_COLS; e += AG_THREADS * (int)cs) {
    const int r = e / AG_COLS, c = e % AG_COLS;
    if (r >= ad.rank || c0 + c >= width) continue;
    float v = 0.0f;
    for (uint32_t k = 0; k < cs; ++k) {
      const float p = cs > 1 ? ld_cluster(map_to_rank(mine + 4u * e, k)) : sums[e];
      v = k ? v + p : p;
    }
    G[((long long)id * ad.rank + r) * width + c0 + c] = sc * v;
  }
  if (cs > 1) cluster_barrier();
}

int adapter_grad_error_read_clear() {
  int v = 0;
  if (cudaMemcpyFromSymbol(&v, g_grad_error, sizeof(int)) != cudaSuccess) return -1;
  if (v) {
    int z = 0;
    cudaMemcpyToSymbol(g_grad_error, &z, sizeof(int));
  }
  return v;
}

template <int RP, bool EIGHT>
static tb_status launch_grad(const Adapt& ad, const void* in, const float* in_scales, const float* low, int n_tok, int width, float* G,
                             cudaStream_t st) {
  constexpr int smem = GradShape<RP>::SMEM;
  static bool configured[64] = {false};
  int dev = 0;
  TB_CUDA_CHECK(cudaGetDevice(&dev));
  if (dev < 0 || dev >= 64) return TB_ERR_CUDA;
  if (!configured[dev]) {
    TB_CUDA_CHECK(cudaFuncSetAttribute(k_adapter_grad<RP, EIGHT>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem));
    configured[dev] = true;
  }
  const int cols = (width + AG_COLS - 1) / AG_COLS, sms = sm_count() > 0 ? sm_count() : 148;
  // CTAs along the tokens until an adapter that had nearly all of them would fill the GPU, while an even share is a stage at least
  int cs = 1;
  while (cs < 8 && cols * cs * 2 <= 2 * sms && n_tok / ad.n / (2 * cs) >= AG_TOK) cs *= 2;
  CUtensorMap imap = {};
  if (!EIGHT)
    TB_TRY(make_map_2d(&imap, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, in, (unsigned long long)width, (unsigned long long)n_tok, 64, AG_TOK,
                       CU_TENSOR_MAP_SWIZZLE_128B));
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(cols * cs), (unsigned)ad.n);
  cfg.blockDim = dim3(AG_THREADS);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = (unsigned)cs;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  TB_CUDA_CHECK(cudaLaunchKernelEx(&cfg, k_adapter_grad<RP, EIGHT>, ad, in, in_scales, low, n_tok, width, G, imap));
  TB_LAUNCH_CHECK();
  return TB_OK;
}

template <bool EIGHT>
static tb_status grad_of_rank(const Adapt& ad, const void* in, const float* in_scales, const float* low, int n_tok, int width, float* G,
                              cudaStream_t st) {
  if (ad.rank <= 16) return launch_grad<16, EIGHT>(ad, in, in_scales, low, n_tok, width, G, st);
  if (ad.rank <= 32) return launch_grad<32, EIGHT>(ad, in, in_scales, low, n_tok, width, G, st);
  if (ad.rank <= 64) return launch_grad<64, EIGHT>(ad, in, in_scales, low, n_tok, width, G, st);
  return launch_grad<128, EIGHT>(ad, in, in_scales, low, n_tok, width, G, st);
}

// `in` bf16, or 8-bit codes where in_scales is given.
tb_status adapter_grad_bf16(const Adapt& ad, const void* in, const float* in_scales, const float* low, int n_tok, int width, float* G,
                            cudaStream_t st) {
  return in_scales ? grad_of_rank<true>(ad, in, in_scales, low, n_tok, width, G, st)
                   : grad_of_rank<false>(ad, in, in_scales, low, n_tok, width, G, st);
}

}  // namespace tb
