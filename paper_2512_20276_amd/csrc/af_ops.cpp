// Entry points of the 8-bit operators and the sampler: argument checks on the host, then one launch.
// None of them allocates, waits or keeps anything between calls.
#include "af_fp8.h"

using namespace af;

namespace {

bool aligned(const void* p, size_t n) { return (uintptr_t)p % n == 0; }

af_status invalid(const char* what, const char* why) {
  set_error("%s: %s", what, why);
  return AF_ERR_INVALID_ARG;
}

af_status too_large(const char* what, const char* of, int64_t n, int64_t limit) {
  set_error("%s: %lld %s, a launch takes fewer than %lld", what, (long long)n, of, (long long)limit);
  return AF_ERR_UNSUPPORTED;
}

}  // namespace

extern "C" af_status af_op_add_rmsnorm_fp8(int32_t dtype, const void* x, const void* resid, const void* g,
                                           void* resid_out, void* q, float* scales, int32_t M, int32_t D, float eps,
                                           void* hip_stream) {
  clear_error();
  const char* me = "af_op_add_rmsnorm_fp8";
  if (dtype != AF_BF16 && dtype != AF_F32) return invalid(me, "dtype must be AF_BF16 or AF_F32");
  if (!x || !g || !q || !scales) return invalid(me, "x, g, q and scales must be non-NULL");
  if (!resid != !resid_out) return invalid(me, "resid and resid_out go together: both or neither");
  if (M <= 0 || D <= 0) return invalid(me, "M and D must be positive");
  if (M >= 1 << 23) return too_large(me, "rows", M, 1 << 23);  // a launch has fewer than 2^32 work-items
  const size_t t = dtype_size(dtype);
  if (!aligned(x, t) || !aligned(resid, t) || !aligned(g, t) || !aligned(resid_out, t) || !aligned(scales, 4))
    return invalid(me, "a pointer is not aligned to its element type");
  AF_HIP(launch_add_rmsnorm_fp8(dtype, x, resid, g, resid_out, q, scales, M, D, eps, (hipStream_t)hip_stream));
  return AF_OK;
}

extern "C" af_status af_op_quantize_fp8(int32_t dtype, const void* x, void* q, float* scales, int32_t M, int32_t K,
                                        int32_t block_rows, void* hip_stream) {
  clear_error();
  const char* me = "af_op_quantize_fp8";
  if (dtype != AF_BF16 && dtype != AF_F32) return invalid(me, "dtype must be AF_BF16 or AF_F32");
  if (!x || !q || !scales) return invalid(me, "x, q and scales must be non-NULL");
  if (M <= 0 || K <= 0) return invalid(me, "M and K must be positive");
  if (block_rows != 1 && block_rows != FP8_BLOCK) return invalid(me, "block_rows must be 1 or 128");
  if (!aligned(x, dtype_size(dtype)) || !aligned(scales, 4))
    return invalid(me, "a pointer is not aligned to its element type");
  const int64_t blocks = (int64_t)(block_rows == 1 ? M : fp8_blocks(M)) * fp8_blocks(K);
  const int64_t most = block_rows == 1 ? (1 << 28) - 15 : 1 << 24;  // 16 blocks, or one, to 256 work-items
  if (blocks >= most) return too_large(me, "blocks", blocks, most);
  AF_HIP(launch_quantize_fp8(dtype, x, q, scales, M, K, block_rows, (hipStream_t)hip_stream));
  return AF_OK;
}

extern "C" af_status af_op_linear_fp8(const void* xq, const float* xs, const void* wq, const float* ws, void* y,
                                      int32_t out_dtype, int32_t M, int32_t N, int32_t K, void* hip_stream) {
  clear_error();
  const char* me = "af_op_linear_fp8";
  if (out_dtype != AF_BF16 && out_dtype != AF_F32) return invalid(me, "out_dtype must be AF_BF16 or AF_F32");
  if (!xq || !xs || !wq || !ws || !y) return invalid(me, "xq, xs, wq, ws and y must be non-NULL");
  if (M <= 0 || N <= 0 || K <= 0) return invalid(me, "M, N and K must be positive");
  if (!aligned(xs, 4) || !aligned(ws, 4) || !aligned(y, dtype_size(out_dtype)))
    return invalid(me, "a pointer is not aligned to its element type");
  if (K % 16 != 0 || !aligned(xq, 16) || !aligned(wq, 16)) {
    set_error("%s: need K %% 16 == 0 and 16-byte aligned xq and wq", me);
    return AF_ERR_UNSUPPORTED;
  }
  const int64_t tiles = (((int64_t)M + 15) / 16) * (((int64_t)N + 15) / 16);
  if (K > FP8_MAX_K) return too_large(me, "columns", K, FP8_MAX_K + 1);
  if (tiles >= 1 << 23) return too_large(me, "tiles of 16 x 16", tiles, 1 << 23);  // of up to 512 work-items each
  const Fp8GemmArgs a{xq, xs, wq, ws, y, M, N, K, fp8_blocks(K)};
  AF_HIP(launch_gemm_fp8(out_dtype, a, (hipStream_t)hip_stream));
  return AF_OK;
}

extern "C" af_status af_op_sample(int32_t dtype, const void* logits, int32_t n_rows, int32_t vocab,
                                  const float* temperature, const int32_t* top_k, const float* top_p,
                                  const float* min_p, const float* uniforms, int32_t* tokens, void* hip_stream) {
  clear_error();
  const char* me = "af_op_sample";
  if (dtype != AF_BF16 && dtype != AF_F32) return invalid(me, "dtype must be AF_BF16 or AF_F32");
  if (!logits || !uniforms || !tokens) return invalid(me, "logits, uniforms and tokens must be non-NULL");
  if (n_rows <= 0 || vocab <= 0) return invalid(me, "n_rows and vocab must be positive");
  if (!aligned(logits, dtype_size(dtype)) || !aligned(temperature, 4) || !aligned(top_k, 4) || !aligned(top_p, 4) ||
      !aligned(min_p, 4) || !aligned(uniforms, 4) || !aligned(tokens, 4))
    return invalid(me, "a pointer is not aligned to its element type");
  if (vocab > SAMPLE_MAX_V) return too_large(me, "tokens", vocab, SAMPLE_MAX_V + 1);
  if (n_rows >= 1 << 22) return too_large(me, "rows", n_rows, 1 << 22);
  const SampleArgs a{logits, vocab, temperature, top_k, top_p, min_p, uniforms, tokens};
  AF_HIP(launch_sample(dtype, a, n_rows, (hipStream_t)hip_stream));
  return AF_OK;
}
