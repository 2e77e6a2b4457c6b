// Writing rows into an 8-bit K/V cache and reading them back:
//   focus_quantize_kv    scale = max|x| / Q over the head_dim elements of one token and KV head, code = the format's
//                        number nearest to x / scale;
//   focus_dequantize_kv  x = code * scale.
// Both are bound by HBM: per element size(T) + 1 bytes move, with a handful of operations.  A row (64 or 128 elements)
// belongs to 8 to 32 neighbouring lanes, sixteen bytes of the wide side each, so every access is a full sector and the
// maximum is a butterfly over those lanes.  Rows of one KV head are neighbours in the grid: their codes and scales
// are neighbours in the cache.
#include <float.h>

#include "focus_common.cuh"

namespace {

constexpr int QK_THREADS = 256;
constexpr float FLUSH_BELOW = 8.271806125530277e-25f;   // 2^-80: rows smaller than this are stored as zeros

template <typename F> __device__ __forceinline__ constexpr float fmt_max() { return sizeof(F) == 1 ? 448.f : 0.f; }
template <> __device__ __forceinline__ constexpr float fmt_max<int8_t>() { return 127.f; }

// The quotient is a true division (one rounding): a code must not depend on how a reciprocal was rounded.
__device__ __forceinline__ uint32_t encode(float x, float scale, int8_t) {
  if (x != x || scale == 0.f) return 0u;
  const float q = rintf(__fdiv_rn(x, scale));
  return (uint32_t)(int)fminf(fmaxf(q, -127.f), 127.f) & 0xffu;
}
__device__ __forceinline__ uint32_t encode(float x, float scale, __nv_fp8_e4m3) {
  if (x != x || scale == 0.f) return 0u;
  return (uint32_t)__nv_cvt_float_to_fp8(__fdiv_rn(x, scale), __NV_SATFINITE, __NV_E4M3);
}

struct RowArgs {
  long long wide_stride_row, wide_stride_head;    // of the rows written from / read into
  long long kv_stride_tok, kv_stride_head, scale_stride;
  int L, Hkv, pos_base, max_rows;
  const int32_t* rows;
  const int32_t* n_rows;
  int32_t* status;
};

// position of row r, or -1 (reported by the caller's lane 0 of the row)
__device__ __forceinline__ int row_position(const RowArgs& a, int r, bool ascending) {
  if (!a.rows) return a.pos_base + r;
  const int pos = a.rows[r];
  if (pos < 0 || pos >= a.L) return -1;
  if (ascending && r > 0 && a.rows[r - 1] >= pos) return -1;
  return pos;
}

template <typename T>
__device__ __forceinline__ void unpack16(const uint4& raw, float (&x)[16 / sizeof(T)]) {
  if constexpr (sizeof(T) == 2) {
    const __nv_bfloat162* p2 = reinterpret_cast<const __nv_bfloat162*>(&raw);
#pragma unroll
    for (int e = 0; e < 4; ++e) { const float2 f = __bfloat1622float2(p2[e]); x[2 * e] = f.x; x[2 * e + 1] = f.y; }
  } else {
    x[0] = __uint_as_float(raw.x); x[1] = __uint_as_float(raw.y);
    x[2] = __uint_as_float(raw.z); x[3] = __uint_as_float(raw.w);
  }
}

// grid (row groups, Hkv, 2): z = 0 keys, 1 values; LPR lanes per row
template <typename T, typename F, int D>
__global__ void __launch_bounds__(QK_THREADS)
quantize_rows_kernel(const T* __restrict__ Kn, const T* __restrict__ Vn, uint8_t* __restrict__ Kc,
                     uint8_t* __restrict__ Vc, float* __restrict__ Ks, float* __restrict__ Vs, const RowArgs a) {
  constexpr int EPC = 16 / sizeof(T), LPR = D / EPC;
  const bool val = blockIdx.z != 0;
  const T* src = val ? Vn : Kn;
  if (!src) return;
  const int g = blockIdx.y, c = threadIdx.x % LPR;
  const int r = blockIdx.x * (QK_THREADS / LPR) + threadIdx.x / LPR;
  const int n = a.rows ? min(max(*a.n_rows, 0), a.max_rows) : a.max_rows;
  int pos = -1;
  if (r < n) {
    pos = row_position(a, r, true);
    if (pos < 0 && c == 0) set_status(a.status, FOCUS_ERR_INVALID_ARG);
  }
  float x[EPC];
  float m = 0.f;
  if (pos >= 0) {
    const uint4 raw = __ldg(reinterpret_cast<const uint4*>(src + (long long)r * a.wide_stride_row +
                                                           (long long)g * a.wide_stride_head + c * EPC));
    unpack16<T>(raw, x);
#pragma unroll
    for (int e = 0; e < EPC; ++e) {
      const float v = fabsf(x[e]);
      m = fmaxf(m, v <= FLT_MAX ? v : 0.f);                  // NaN and infinities do not enter the scale
    }
  }
#pragma unroll
  for (int o = LPR / 2; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
  if (pos < 0) return;
  const float scale = m < FLUSH_BELOW ? 0.f : __fdiv_rn(m, fmt_max<F>());
  uint32_t w[EPC / 4];
#pragma unroll
  for (int i = 0; i < EPC / 4; ++i) {
    w[i] = 0u;
#pragma unroll
    for (int e = 0; e < 4; ++e) w[i] |= encode(x[4 * i + e], scale, F()) << (8 * e);
  }
  uint8_t* dst = (val ? Vc : Kc) + (long long)g * a.kv_stride_head + (long long)pos * a.kv_stride_tok + c * EPC;
  if constexpr (EPC == 8) *reinterpret_cast<uint2*>(dst) = make_uint2(w[0], w[1]);
  else *reinterpret_cast<uint32_t*>(dst) = w[0];
  if (c == 0) (val ? Vs : Ks)[(long long)g * a.scale_stride + pos] = scale;
  publish_outputs();
}

// grid (row groups, Hkv, 2); a lane reads EPC codes and writes sixteen bytes
template <typename T, typename F, int D>
__global__ void __launch_bounds__(QK_THREADS)
dequantize_rows_kernel(const uint8_t* __restrict__ Kc, const uint8_t* __restrict__ Vc, const float* __restrict__ Ks,
                       const float* __restrict__ Vs, T* __restrict__ Ko, T* __restrict__ Vo, const RowArgs a) {
  constexpr int EPC = 16 / sizeof(T), LPR = D / EPC;
  const bool val = blockIdx.z != 0;
  T* out = val ? Vo : Ko;
  if (!out) return;
  const int g = blockIdx.y, c = threadIdx.x % LPR;
  const int r = blockIdx.x * (QK_THREADS / LPR) + threadIdx.x / LPR;
  const int n = a.rows ? min(max(*a.n_rows, 0), a.max_rows) : a.max_rows;
  if (r >= n) return;
  const int pos = row_position(a, r, false);
  if (pos < 0) {
    if (c == 0) set_status(a.status, FOCUS_ERR_INVALID_ARG);
    return;
  }
  const uint8_t* src = (val ? Vc : Kc) + (long long)g * a.kv_stride_head + (long long)pos * a.kv_stride_tok + c * EPC;
  const float scale = __ldg((val ? Vs : Ks) + (long long)g * a.scale_stride + pos);
  uint32_t w[EPC / 4];
  if constexpr (EPC == 8) {
    const uint2 v = __ldg(reinterpret_cast<const uint2*>(src));
    w[0] = v.x; w[1] = v.y;
  } else {
    w[0] = __ldg(reinterpret_cast<const uint32_t*>(src));
  }
  uint32_t o[4];
#pragma unroll
  for (int i = 0; i < EPC / 4; ++i) {
    float f[4];
    codes_to_float(w[i], F(), f);
    if constexpr (sizeof(T) == 2) {
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const __nv_bfloat162 b = __floats2bfloat162_rn(f[2 * e] * scale, f[2 * e + 1] * scale);
        o[2 * i + e] = *reinterpret_cast<const uint32_t*>(&b);
      }
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] = __float_as_uint(f[e] * scale);
    }
  }
  *reinterpret_cast<uint4*>(out + (long long)r * a.wide_stride_row + (long long)g * a.wide_stride_head + c * EPC) =
      make_uint4(o[0], o[1], o[2], o[3]);
  publish_outputs();
}

// arguments both calls share; `wide` are the row tensors in shape->dtype
focus_status row_args(focus_ctx* ctx, const focus_shape* shape, const focus_quant_cache* cache, const void* wide_k,
                      const void* wide_v, long long stride_row, long long stride_head, int pos_base, const int32_t* rows,
                      const int32_t* n_rows, int max_rows, RowArgs& a) {
  if (!ctx || !quant_cache_ok(shape, cache, wide_k != nullptr, wide_v != nullptr)) return FOCUS_ERR_INVALID_ARG;
  if (!wide_k && !wide_v) return FOCUS_ERR_INVALID_ARG;
  if (!all_aligned16(wide_k, wide_v)) return FOCUS_ERR_INVALID_ARG;
  if (stride_row < shape->head_dim || stride_head < shape->head_dim || ((stride_row | stride_head) & 7))
    return FOCUS_ERR_INVALID_ARG;
  if ((rows == nullptr) != (n_rows == nullptr) || max_rows < 0) return FOCUS_ERR_INVALID_ARG;
  if (!rows && (pos_base < 0 || pos_base > shape->L || max_rows > shape->L - pos_base)) return FOCUS_ERR_INVALID_ARG;
  if (!shape_supported(shape) || shape->n_kv_heads > 65535) return FOCUS_ERR_UNSUPPORTED;
  a.wide_stride_row = stride_row; a.wide_stride_head = stride_head;
  a.kv_stride_tok = shape->kv_stride_tok; a.kv_stride_head = shape->kv_stride_head;
  a.scale_stride = quant_scale_stride(cache, shape);
  a.L = shape->L; a.Hkv = shape->n_kv_heads; a.pos_base = pos_base; a.max_rows = max_rows;
  a.rows = rows; a.n_rows = n_rows; a.status = ctx->d_status;
  return FOCUS_OK;
}

// one instantiation per (dtype, format, head dim); LPR as in the kernels
#define FOCUS_QK_DISPATCH(LAUNCH)                                                          \
  do {                                                                                     \
    const bool bf = shape->dtype == FOCUS_BF16, i8 = cache->format == FOCUS_KV_INT8;       \
    if (shape->head_dim == 128) {                                                          \
      if (bf) { if (i8) LAUNCH(__nv_bfloat16, int8_t, 128); else LAUNCH(__nv_bfloat16, __nv_fp8_e4m3, 128); } \
      else { if (i8) LAUNCH(float, int8_t, 128); else LAUNCH(float, __nv_fp8_e4m3, 128); } \
    } else {                                                                               \
      if (bf) { if (i8) LAUNCH(__nv_bfloat16, int8_t, 64); else LAUNCH(__nv_bfloat16, __nv_fp8_e4m3, 64); }   \
      else { if (i8) LAUNCH(float, int8_t, 64); else LAUNCH(float, __nv_fp8_e4m3, 64); }   \
    }                                                                                      \
  } while (0)

inline dim3 row_grid(const focus_shape* s, int max_rows) {
  const int lpr = s->head_dim * (s->dtype == FOCUS_BF16 ? 2 : 4) / 16, per = QK_THREADS / lpr;
  return dim3((max_rows + per - 1) / per, s->n_kv_heads, 2);
}

}  // namespace

extern "C" focus_status focus_quantize_kv(focus_ctx* ctx, const focus_shape* shape, const void* K_new, const void* V_new,
                                          int64_t new_stride_row, int64_t new_stride_head, int32_t pos_base,
                                          const int32_t* rows, const int32_t* n_rows, int32_t max_rows,
                                          const focus_quant_cache* cache, focus_stream stream) {
  FOCUS_STAGE("focus_quantize_kv");
  RowArgs a;
  const focus_status s = row_args(ctx, shape, cache, K_new, V_new, new_stride_row, new_stride_head, pos_base, rows, n_rows,
                                  max_rows, a);
  if (s != FOCUS_OK) return s;
  if (max_rows == 0) return FOCUS_OK;
#define LAUNCH(T, F, D)                                                                                          \
  quantize_rows_kernel<T, F, D><<<row_grid(shape, max_rows), QK_THREADS, 0, stream>>>(                           \
      (const T*)K_new, (const T*)V_new, (uint8_t*)cache->K, (uint8_t*)cache->V, cache->K_scale, cache->V_scale, a)
  FOCUS_QK_DISPATCH(LAUNCH);
#undef LAUNCH
  FOCUS_CHECK_LAUNCH();
  return FOCUS_OK;
}

extern "C" focus_status focus_dequantize_kv(focus_ctx* ctx, const focus_shape* shape, const focus_quant_cache* cache,
                                            int32_t pos_base, const int32_t* rows, const int32_t* n_rows,
                                            int32_t max_rows, void* K_out, void* V_out, int64_t out_stride_row,
                                            int64_t out_stride_head, focus_stream stream) {
  FOCUS_STAGE("focus_dequantize_kv");
  RowArgs a;
  const focus_status s = row_args(ctx, shape, cache, K_out, V_out, out_stride_row, out_stride_head, pos_base, rows, n_rows,
                                  max_rows, a);
  if (s != FOCUS_OK) return s;
  if (max_rows == 0) return FOCUS_OK;
#define LAUNCH(T, F, D)                                                                                          \
  dequantize_rows_kernel<T, F, D><<<row_grid(shape, max_rows), QK_THREADS, 0, stream>>>(                         \
      (const uint8_t*)cache->K, (const uint8_t*)cache->V, cache->K_scale, cache->V_scale, (T*)K_out, (T*)V_out, a)
  FOCUS_QK_DISPATCH(LAUNCH);
#undef LAUNCH
  FOCUS_CHECK_LAUNCH();
  return FOCUS_OK;
}
