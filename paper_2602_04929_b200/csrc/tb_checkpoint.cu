// Activations kept in 8 bits: a scale max|x| / 127 for every token and run of 128 columns, codes rne(x / scale).
//
// Both kernels move data once and are bound by HBM.  Half a warp has a run: a lane holds 8 values (16 bytes of bf16, two
// 16-byte loads of float), so a run's maximum is four shuffles away and a warp stores 256 bytes of codes.  A lane has two
// such pieces in flight.
//
// Packing is bound by its instructions as much as by HBM, about nine a value.  bf16 magnitudes are compared two at a time.  The scale's
// division is a product with 1 / 127 and a correction by its remainder, two fused steps (P. Markstein, Computation of elementary functions
// on the IBM RISC System/6000 processor, 1990); where nothing underflows it rounds correctly, for every mantissa (tested).  16384 x 8192, bf16: packing 93 us (4.4 TB/s), unpacking 64.5 us
// (6.4 TB/s, the rate of a copy).
//
// The codes are those of the true quotient.  y = x * (1 / scale) is off by less than 2^-14 where |y| <= 127, so rounding it decides
// unless it lies that close to the middle between two codes.  Only such a value is looked at further: the sign of x - (q +- 1/2) scale,
// which one fused multiply-add gives exactly, says whether q is the nearest, and a tie (the sum is 0) goes to the even one.  Rounding
// is one fused step: 1.5 * 2^23 + y has the code in its low bits.
#include "tb_packed.cuh"

namespace tb {

// Eight neighbouring values as they are stored; the largest magnitude of half a warp's as the bits of a float, which order like the
// values, with what is not finite on top.
template <typename T>
struct Words8;
template <>
struct Words8<__nv_bfloat16> {
  unsigned w[4];
  static __device__ __forceinline__ unsigned max2(unsigned a, unsigned b) {  // what is no number wins
    unsigned o;
    asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(o) : "r"(a), "r"(b));
    return o;
  }
  __device__ __forceinline__ void zero() { w[0] = w[1] = w[2] = w[3] = 0; }
  __device__ __forceinline__ void load(const __nv_bfloat16* p) {
    const uint4 q = __ldcs(reinterpret_cast<const uint4*>(p));
    w[0] = q.x, w[1] = q.y, w[2] = q.z, w[3] = q.w;
  }
  __device__ __forceinline__ unsigned half_warp_top() const {
    unsigned m = max2(max2(w[0] & 0x7fff7fffu, w[1] & 0x7fff7fffu), max2(w[2] & 0x7fff7fffu, w[3] & 0x7fff7fffu));
    m = max2(m, __byte_perm(m, 0, 0x1032));  // both halves, so that one shuffle carries the same twice
#pragma unroll
    for (int o = 1; o < 16; o <<= 1) m = max2(m, __shfl_xor_sync(0xffffffffu, m, o));
    return m & 0xffff0000u;
  }
  __device__ __forceinline__ void values(float (&v)[8]) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[2 * i] = __uint_as_float(w[i] << 16), v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
  }
};
template <>
struct Words8<float> {
  float f[8];
  __device__ __forceinline__ void zero() {
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = 0.0f;
  }
  __device__ __forceinline__ void load(const float* p) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const float4 q = __ldcs(reinterpret_cast<const float4*>(p) + h);
      f[4 * h] = q.x, f[4 * h + 1] = q.y, f[4 * h + 2] = q.z, f[4 * h + 3] = q.w;
    }
  }
  __device__ __forceinline__ unsigned half_warp_top() const {
    unsigned m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(f[i]) & 0x7fffffffu);
#pragma unroll
    for (int o = 1; o < 16; o <<= 1) m = max(m, __shfl_xor_sync(0xffffffffu, m, o));
    return m;
  }
  __device__ __forceinline__ void values(float (&v)[8]) const {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = f[i];
  }
};
__device__ __forceinline__ void store8(__nv_bfloat16* p, const float (&v)[8]) {
  unsigned w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const __nv_bfloat162 b = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
    w[i] = *reinterpret_cast<const unsigned*>(&b);
  }
  *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ void store8(float* p, const float (&v)[8]) {
  reinterpret_cast<float4*>(p)[0] = make_float4(v[0], v[1], v[2], v[3]);
  reinterpret_cast<float4*>(p)[1] = make_float4(v[4], v[5], v[6], v[7]);
}

// rne(x / s) for finite x, |x| <= 127 s up to the rounding of s, s > 0; inv is about 1 / s
__device__ __forceinline__ int nearest_code(float x, float s, float inv) {
  float q = rintf(x * inv);
  q = fminf(fmaxf(q, -127.0f), 127.0f);
  const float up = fmaf(-(q + 0.5f), s, x), down = fmaf(-(q - 0.5f), s, x);
  const bool odd = ((int)q) & 1;
  if (up > 0.0f || (up == 0.0f && odd))
    q += 1.0f;
  else if (down < 0.0f || (down == 0.0f && odd))
    q -= 1.0f;
  return (int)fminf(fmaxf(q, -127.0f), 127.0f);
}

constexpr int CKPT_PER = 2;  // runs that a lane has in flight

// run -> token and column; per_inv: 2^64 / n_g rounded up, 0 for one run a token
__device__ __forceinline__ void place_of(long long run, int n_g, unsigned long long per_inv, int l, long long& t, int& col) {
  t = per_inv ? (long long)__umul64hi((unsigned long long)run, per_inv) : run;
  col = (int)(run - t * n_g) * CKPT_RUN + 8 * l;
}

template <typename T>
__global__ void __launch_bounds__(256) k_checkpoint_pack(const T* __restrict__ x, signed char* __restrict__ codes,
                                                         float* __restrict__ scales, long long n_runs, int d, int n_g,
                                                         unsigned long long per_inv) {
  const int half = threadIdx.x >> 4, l = threadIdx.x & 15;
  const long long r0 = (long long)blockIdx.x * (16 * CKPT_PER) + half;
  Words8<T> raw[CKPT_PER];
  bool in[CKPT_PER];
  long long at[CKPT_PER];
#pragma unroll
  for (int k = 0; k < CKPT_PER; ++k) {
    const long long run = r0 + 16 * k;
    long long t;
    int col;
    place_of(run, n_g, per_inv, l, t, col);
    in[k] = run < n_runs && col < d;
    at[k] = t * d + col;
    raw[k].zero();
    if (in[k]) raw[k].load(x + at[k]);
  }
#pragma unroll
  for (int k = 0; k < CKPT_PER; ++k) {
    const unsigned top = raw[k].half_warp_top();
    const bool finite = top < 0x7f800000u;
    float s;
    if (top >= 0x10000000u) {  // 2^-95 and more
      constexpr float i127 = 1.0f / 127.0f;
      const float t = __uint_as_float(top), q = t * i127;
      s = finite ? fmaf(fmaf(-q, 127.0f, t), i127, q) : __uint_as_float(0x7fffffffu);
    } else {
      s = __fdiv_rn(__uint_as_float(top), 127.0f);
    }
    float inv;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(inv) : "f"(s));
    float v[8];
    raw[k].values(v);
    unsigned w[2] = {0, 0};
    if (finite && s >= 7.9e-31f) {  // 2^-100: no product below underflows
      constexpr float magic = 12582912.0f;
      unsigned q[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float r = fmaf(v[i], inv, magic);
        q[i] = __float_as_uint(r);
        // value by value: half of a bf16 run's maximum is a tie, so that nearly every second warp has one among its 256
        const float near = r - magic, d = fmaf(v[i], inv, -near);
        if (fabsf(d) > 0.5f - 6.1035156e-5f) {  // near or its neighbour on d's side: whose side of the middle is x on?
          const float half = copysignf(0.5f, d), e = fmaf(-(near + half), s, v[i]) * half;
          if (e > 0.0f || (e == 0.0f && (q[i] & 1u))) q[i] += half > 0.0f ? 1u : 0xffffffffu;
        }
      }
#pragma unroll
      for (int h = 0; h < 2; ++h)
        w[h] = __byte_perm(__byte_perm(q[4 * h], q[4 * h + 1], 0x0040), __byte_perm(q[4 * h + 2], q[4 * h + 3], 0x0040), 0x5410);
    } else if (finite && s > 0.0f) {
      // a smaller scale is scaled up by 2^64 first, and so is x
      constexpr float up = 18446744073709551616.0f;
      const float su = s * up, iu = 1.0f / su;
#pragma unroll
      for (int i = 0; i < 8; ++i) w[i >> 2] |= ((unsigned)nearest_code(v[i] * up, su, iu) & 0xffu) << (8 * (i & 3));
    }
    if (in[k]) *reinterpret_cast<uint2*>(codes + at[k]) = make_uint2(w[0], w[1]);
    if (l == 0 && r0 + 16 * k < n_runs) scales[r0 + 16 * k] = s;
  }
}

template <typename T>
__global__ void __launch_bounds__(256) k_checkpoint_unpack(const signed char* __restrict__ codes,
                                                           const float* __restrict__ scales, T* __restrict__ x,
                                                           long long n_runs, int d, int n_g, unsigned long long per_inv) {
  const int half = threadIdx.x >> 4, l = threadIdx.x & 15;
  uint2 w[CKPT_PER];
  float s[CKPT_PER];
  long long at[CKPT_PER];
#pragma unroll
  for (int k = 0; k < CKPT_PER; ++k) {
    const long long run = (long long)blockIdx.x * (16 * CKPT_PER) + 16 * k + half;
    long long t;
    int col;
    place_of(run, n_g, per_inv, l, t, col);
    at[k] = run < n_runs && col < d ? t * d + col : -1;
    if (at[k] >= 0) {
      w[k] = __ldcs(reinterpret_cast<const uint2*>(codes + at[k]));
      s[k] = __ldg(scales + run);
    }
  }
#pragma unroll
  for (int k = 0; k < CKPT_PER; ++k) {
    if (at[k] < 0) continue;
    float v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = (float)(signed char)((i < 4 ? w[k].x : w[k].y) >> (8 * (i & 3))) * s[k];
    store8(x + at[k], v);
  }
}

}  // namespace tb

using namespace tb;

static tb_status checkpoint_shape(tb_dtype type, long long n_tok, int d, const void* x, const void* codes,
                                  const void* scales, long long* n_runs, unsigned* blocks, unsigned long long* per_inv) {
  if ((type != TB_F32 && type != TB_BF16) || n_tok < 0 || d <= 0) return TB_ERR_INVALID_ARG;
  if (d % 32 || n_tok > 0x7fffffffll) return TB_ERR_UNSUPPORTED;
  const long long n_g = ((long long)d + CKPT_RUN - 1) / CKPT_RUN;  // d may be 2^31 - 32
  *n_runs = n_tok * n_g;
  *per_inv = n_g > 1 ? ~0ull / (unsigned long long)n_g + 1 : 0;
  const long long nb = (*n_runs + 16 * CKPT_PER - 1) / (16 * CKPT_PER);
  if (nb > 0x7fffffffll) return TB_ERR_UNSUPPORTED;
  *blocks = (unsigned)nb;
  if (n_tok == 0) return TB_OK;
  if (!x || !codes || !scales) return TB_ERR_INVALID_ARG;
  if (!aligned(x, 16) || !aligned(codes, 16) || !aligned(scales, 4)) return TB_ERR_INVALID_ARG;
  return TB_OK;
}

extern "C" tb_status tb_checkpoint_pack(const void* x, tb_dtype x_type, long long n_tok, int d, signed char* codes,
                                        float* scales, void* stream) {
  long long n_runs;
  unsigned nb;
  unsigned long long per_inv;
  TB_TRY(checkpoint_shape(x_type, n_tok, d, x, codes, scales, &n_runs, &nb, &per_inv));
  if (nb == 0) return TB_OK;
  const int n_g = (int)(((long long)d + CKPT_RUN - 1) / CKPT_RUN);
  if (x_type == TB_BF16)
    k_checkpoint_pack<<<nb, 256, 0, as_stream(stream)>>>(static_cast<const __nv_bfloat16*>(x), codes, scales, n_runs, d, n_g, per_inv);
  else
    k_checkpoint_pack<<<nb, 256, 0, as_stream(stream)>>>(static_cast<const float*>(x), codes, scales, n_runs, d, n_g, per_inv);
  TB_LAUNCH_CHECK();
  return TB_OK;
}

extern "C" tb_status tb_checkpoint_unpack(const signed char* codes, const float* scales, long long n_tok, int d,
                                          tb_dtype x_type, void* x, void* stream) {
  long long n_runs;
  unsigned nb;
  unsigned long long per_inv;
  TB_TRY(checkpoint_shape(x_type, n_tok, d, x, codes, scales, &n_runs, &nb, &per_inv));
  if (nb == 0) return TB_OK;
  const int n_g = (int)(((long long)d + CKPT_RUN - 1) / CKPT_RUN);
  if (x_type == TB_BF16)
    k_checkpoint_unpack<<<nb, 256, 0, as_stream(stream)>>>(codes, scales, static_cast<__nv_bfloat16*>(x), n_runs, d, n_g, per_inv);
  else
    k_checkpoint_unpack<<<nb, 256, 0, as_stream(stream)>>>(codes, scales, static_cast<float*>(x), n_runs, d, n_g, per_inv);
  TB_LAUNCH_CHECK();
  return TB_OK;
}
