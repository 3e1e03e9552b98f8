// Products with bit-packed weights, low-rank adapters of many requests beside them, and their gradients: the entry points.
#include "tb_packed_few.cuh"
#include "tb_packed_plan.cuh"

namespace tb {

int sm_count() {
  static int count[64] = {0};
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return 0;
  if (!count[dev]) {
    int n = 0;
    if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) return 0;
    count[dev] = n;
  }
  return count[dev];
}

tb_status packed_product_f32(const PackedW& w, const Adapt& ad, const float* in, int n_tok, float* out, const float* low, bool back,
                             cudaStream_t st);
tb_status adapter_low_f32(const Adapt& ad, const float* in, const float* M, long long n_tok, int width, float* low, cudaStream_t st);
tb_status adapter_grad_f32(const Adapt& ad, const void* in, const float* in_scales, const float* low, long long n_tok, int width,
                           float* G, cudaStream_t st);

tb_status adapter_grad_bf16(const Adapt& ad, const void* in, const float* in_scales, const float* low, int n_tok, int width, float* G,
                            cudaStream_t st);

static tb_status adapter_low(const Adapt& ad, const void* in, const void* M, tb_dtype type, long long n_tok, int width, float* low,
                             cudaStream_t st) {
  if (type == TB_BF16)
    return adapter_low_bf16(ad, static_cast<const __nv_bfloat16*>(in), static_cast<const __nv_bfloat16*>(M), (int)n_tok, width, low, false, st);
  return adapter_low_f32(ad, static_cast<const float*>(in), static_cast<const float*>(M), n_tok, width, low, st);
}
// of an input in `type`, or of 8-bit codes where their scales are given
static tb_status adapter_grad(const Adapt& ad, const void* in, const float* in_scales, tb_dtype type, const float* low, long long n_tok,
                              int width, float* G, cudaStream_t st) {
  if (type == TB_BF16) return adapter_grad_bf16(ad, in, in_scales, low, (int)n_tok, width, G, st);
  return adapter_grad_f32(ad, in, in_scales, low, n_tok, width, G, st);
}

// Shapes first (so that the workspace queries can use them), pointers with `with_data`.
static tb_status checked(const tb_packed_weight* w, const tb_adapters* a, tb_dtype type, long long n_tok, bool with_data,
                         PackedW* pw, Adapt* ad) {
  if (!w || (type != TB_F32 && type != TB_BF16) || n_tok < 0) return TB_ERR_INVALID_ARG;
  if (w->d_out <= 0 || w->d_in <= 0 || w->bits < 2 || w->bits > 8 || w->quant_group < 0) return TB_ERR_INVALID_ARG;
  if (w->quant_group > 0 && w->d_in % w->quant_group) return TB_ERR_INVALID_ARG;
  if (a && (a->n_adapters < 1 || a->rank < 1 || a->n_requests < 1)) return TB_ERR_INVALID_ARG;
  if (w->d_in % 32 || w->d_out % 8 || w->quant_group % 32) return TB_ERR_UNSUPPORTED;
  if (n_tok > 0x7fffffffll / 2 || w->d_out > (1 << 24) || w->d_in > (1 << 24)) return TB_ERR_UNSUPPORTED;
  if (a && (a->rank % 8 || a->rank > 128 || a->n_adapters > 65535)) return TB_ERR_UNSUPPORTED;
  if (with_data) {
    if (!w->packed || !w->scales || !w->zeros) return TB_ERR_INVALID_ARG;
    if (!aligned(w->packed, 16) || !aligned(w->scales, 4) || !aligned(w->zeros, 4)) return TB_ERR_INVALID_ARG;
    if (a && (!a->A || !a->B || !a->scale || !a->starts || !a->ids)) return TB_ERR_INVALID_ARG;
    if (a && (!aligned(a->A, 16) || !aligned(a->B, 16) || !aligned(a->scale, 4) || !aligned(a->starts, 4) || !aligned(a->ids, 4)))
      return TB_ERR_INVALID_ARG;
  }
  pw->packed = w->packed, pw->scales = w->scales, pw->zeros = w->zeros;
  pw->d_out = w->d_out, pw->d_in = w->d_in, pw->bits = w->bits;
  pw->group = w->quant_group ? w->quant_group : w->d_in;
  pw->n_g = w->d_in / pw->group;
  pw->words = w->d_in / 32 * w->bits;
  *ad = Adapt{};
  if (a) {
    ad->A = a->A, ad->B = a->B, ad->scale = a->scale, ad->starts = a->starts, ad->ids = a->ids;
    ad->n = a->n_adapters, ad->rank = a->rank, ad->n_req = a->n_requests;
  }
  return TB_OK;
}

tb_status packed_few_bf16_1(const PackedFew& p, cudaStream_t st);
tb_status packed_few_bf16_2(const PackedFew& p, cudaStream_t st);
tb_status packed_few_f32_1(const PackedFew& p, cudaStream_t st);
tb_status packed_few_f32_2(const PackedFew& p, cudaStream_t st);

// Which product: where tokens are few or the work small, the weights go into registers (one launch instead of two or three); else bf16
// goes to tcgen05 tiles, whose smallest has 32 tokens, and float, like the gradient of float inputs, to mma.sync tiles of 64.
// Measured on 4096 x 4096, 4 bits / 8192 x 8192, 2 bits (us), registers / tiles: 24 tokens 13.9 / 17.1, 31.5 / 31.1; 32 tokens
// 14.4 / 17.1, 32.2 / 31.2; 48 tokens 20.5 / 17.5, 46.7 / 32.0.  Smaller weights, 4 bits (us in a graph): 2048 x 2048, 64 tokens
// 9.1 / 12.5, 96 tokens 12.8 / 12.7; 1024 x 4096, 64 tokens 11.1 / 12.9, 96 tokens 15.9 / 12.6; 1024 x 1024, 128 tokens 6.9 / 10.9,
// 256 tokens 9.3 / 11.8; 2048 x 512, 128 tokens 7.9 / 9.7, 256 tokens 14.5 / 10.3; 512 x 512, 512 tokens 7.9 / 9.5, 1023 tokens 14.3 /
// 10.2.  The adapters' share is computed per 16 tokens here, from rows that each of its outputs reads, so that tokens x columns x rank decides
// from nine tokens on (4 bits, requests of a token each): 4096 x 4096, 16 tokens, rank 64 23.0 / 29.3, rank 128 39.3 / 35.0; 32 tokens,
// rank 16 24.0 / 23.2, rank 64 36.7 / 30.5, rank 128 50.7 / 36.2; 8192 x 512, 32 tokens, rank 16 16.7 / 17.3, rank 128 51.6 / 39.5; 8192 x 8192,
// 2 bits, 32 tokens, rank 128 82 / 58; 1024 x 1024, 32 tokens, rank 128 22.6 / 24.8; with eight tokens 8192 x 8192, rank 128 30.8 / 50.9,
// 512 x 8192 21.2 / 27.4.  Work of more tokens: rank 16, 1024 x 1024, 256 tokens 18.4 / 20.5; rank 64, 512 x 512, 128
// tokens 19.1 / 44, 512 tokens 35.7 / 32.6; rank 128, 512 x 512, 64 tokens 14.7 / 33.4, 256 tokens 36.0 / 32.7, 8192 x 512, 64 tokens
// 100 / 35.
// Float, 4 bits, registers / tiles: 4096 x 4096, 64 tokens 61 / 85, 128 tokens 104 / 85, 1024 tokens 784 / 603; 8192 x 8192, 128 tokens
// 350 / 309, 1024 tokens 2740 / 2128; 1024 x 4096, 128 tokens 32 / 46, 256 tokens 60 / 48.
enum { FEW_TOKENS = 32, FEW_TOKENS_F32 = 96, FEW_OUTPUTS = 1 << 18, FEW_WORK = 1 << 28 };
static bool takes_few(const PackedW& w, const Adapt& ad, tb_dtype type, long long n_tok, bool back) {
  if (back) return false;
  if (type == TB_F32) return n_tok <= FEW_TOKENS_F32;
  const long long outputs = n_tok * w.d_out, ranks = ad.n && ad.rank > 16 ? ad.rank : 16;  // n_tok < 2^30, d_out <= 2^24
  if (n_tok <= 8 || (n_tok <= FEW_TOKENS && !ad.n)) return true;
  return outputs * ranks <= FEW_OUTPUTS * 16ll && (n_tok <= FEW_TOKENS || outputs * w.d_in <= FEW_WORK);
}

// Scratch of a call: the product's own, and for the backward pass u = dy B^T of every token, not scaled.
struct Scratch {
  float* u;
  char* product;
  size_t bytes;
};
static Scratch carve(const PackedW& w, const Adapt& ad, tb_dtype type, long long n_tok, bool back, void* ws) {
  Scratch s;
  Bump b(ws);
  s.u = back && ad.n ? b.take<float>((size_t)n_tok * ad.rank) : nullptr;
  size_t n = 0;
  if (type == TB_BF16 && !takes_few(w, ad, type, n_tok, back)) {
    PackedTc p;
    const int cols = back ? w.d_in : w.d_out;
    n = packed_tc_carve(packed_tc_plan(ad, (int)n_tok, cols, back ? w.d_out : w.d_in, back), w, ad, (int)n_tok, cols, back, nullptr, &p);
  }
  s.product = b.take<char>(n);
  s.bytes = (back && ad.n) || n ? b.total() : 0;
  return s;
}

// in Q^T or in Q and the adapters' share, with their low = in M_i^T
static tb_status product(const PackedW& w, const Adapt& ad, const void* in, tb_dtype type, long long n_tok, void* out, float* low,
                         bool back, void* ws, cudaStream_t st) {
  if (type == TB_BF16 && !takes_few(w, ad, type, n_tok, back))
    return packed_product_tc(w, ad, static_cast<const __nv_bfloat16*>(in), n_tok, static_cast<__nv_bfloat16*>(out), low, back, ws, st);
  if (ad.n) TB_TRY(adapter_low(ad, in, back ? ad.B : ad.A, type, n_tok, back ? w.d_out : w.d_in, low, st));
  if (takes_few(w, ad, type, n_tok, back)) {
    PackedFew p;
    p.w = w, p.ad = ad, p.x = in, p.M = ad.B, p.low = low, p.out = out, p.n_tok = (int)n_tok;
    if (type == TB_BF16) return n_tok <= 8 ? packed_few_bf16_1(p, st) : packed_few_bf16_2(p, st);
    return n_tok <= 8 ? packed_few_f32_1(p, st) : packed_few_f32_2(p, st);
  }
  return packed_product_f32(w, ad, static_cast<const float*>(in), (int)n_tok, static_cast<float*>(out), low, back, st);
}

}  // namespace tb

using namespace tb;

extern "C" size_t tb_packed_linear_workspace(const tb_packed_weight* w, const tb_adapters* adapters, tb_dtype x_type,
                                             long long n_tok) {
  PackedW pw;
  Adapt ad;
  if (checked(w, adapters, x_type, n_tok, false, &pw, &ad) != TB_OK || n_tok == 0) return 0;
  return carve(pw, ad, x_type, n_tok, false, nullptr).bytes;
}

extern "C" tb_status tb_packed_linear(const tb_packed_weight* w, const tb_adapters* adapters, const void* x, tb_dtype x_type,
                                      long long n_tok, void* y, float* xa, void* ws, size_t ws_bytes, void* stream) {
  PackedW pw;
  Adapt ad;
  TB_TRY(checked(w, adapters, x_type, n_tok, true, &pw, &ad));
  if (n_tok == 0) return TB_OK;
  if (!x || !y || (ad.n && !xa)) return TB_ERR_INVALID_ARG;
  if (!aligned(x, 16) || !aligned(y, 16) || !aligned(xa, 16)) return TB_ERR_INVALID_ARG;
  const Scratch sc = carve(pw, ad, x_type, n_tok, false, ws);
  if (sc.bytes && (!ws || !aligned(ws, 256) || ws_bytes < sc.bytes)) return TB_ERR_WORKSPACE;
  cudaStream_t st = as_stream(stream);
  return product(pw, ad, x, x_type, n_tok, y, xa, false, sc.product, st);
}

extern "C" size_t tb_packed_linear_backward_workspace(const tb_packed_weight* w, const tb_adapters* adapters, tb_dtype x_type,
                                                      long long n_tok) {
  PackedW pw;
  Adapt ad;
  if (checked(w, adapters, x_type, n_tok, false, &pw, &ad) != TB_OK || n_tok == 0) return 0;
  return carve(pw, ad, x_type, n_tok, true, nullptr).bytes;
}

extern "C" tb_status tb_packed_linear_backward(const tb_packed_weight* w, const tb_adapters* adapters, const void* dy,
                                               tb_dtype x_type, long long n_tok, const void* x, const signed char* x_codes,
                                               const float* x_scales, const float* xa, void* dx, float* dA, float* dB, void* ws,
                                               size_t ws_bytes, void* stream) {
  PackedW pw;
  Adapt ad;
  TB_TRY(checked(w, adapters, x_type, n_tok, true, &pw, &ad));
  if ((dA == nullptr) != (dB == nullptr) || (dA && !ad.n) || (!dx && !dA && n_tok > 0)) return TB_ERR_INVALID_ARG;
  if (!aligned(dA, 16) || !aligned(dB, 16)) return TB_ERR_INVALID_ARG;
  cudaStream_t st = as_stream(stream);
  if (n_tok == 0) {
    if (dA) {
      TB_CUDA_CHECK(cudaMemsetAsync(dA, 0, (size_t)ad.n * ad.rank * pw.d_in * sizeof(float), st));
      TB_CUDA_CHECK(cudaMemsetAsync(dB, 0, (size_t)ad.n * ad.rank * pw.d_out * sizeof(float), st));
    }
    return TB_OK;
  }
  if (!dy || !aligned(dy, 16) || !aligned(dx, 16)) return TB_ERR_INVALID_ARG;
  if (dA) {  // the input in one of its two forms
    if (!xa || (x != nullptr) == (x_codes != nullptr) || (x_codes != nullptr) != (x_scales != nullptr)) return TB_ERR_INVALID_ARG;
    if (!aligned(x, 16) || !aligned(x_codes, 16) || !aligned(x_scales, 4) || !aligned(xa, 16)) return TB_ERR_INVALID_ARG;
  }
  const Scratch sc = carve(pw, ad, x_type, n_tok, true, ws);
  if (sc.bytes && (!ws || !aligned(ws, 256) || ws_bytes < sc.bytes)) return TB_ERR_WORKSPACE;
  float* u = sc.u;
  if (dx)
    TB_TRY(product(pw, ad, dy, x_type, n_tok, dx, u, true, sc.product, st));
  else
    TB_TRY(adapter_low(ad, dy, ad.B, x_type, n_tok, pw.d_out, u, st));
  if (dA) {
    TB_TRY(adapter_grad(ad, x_codes ? (const void*)x_codes : x, x_scales, x_type, u, n_tok, pw.d_in, dA, st));
    TB_TRY(adapter_grad(ad, dy, nullptr, x_type, xa, n_tok, pw.d_out, dB, st));
  }
  return TB_OK;
}
