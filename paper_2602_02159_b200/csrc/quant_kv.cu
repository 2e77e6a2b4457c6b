// Writing rows into an 8-bit K/V cache and reading them back:
//   focus_quantize_kv    scale = max|x| / Q over the head_dim elements of one token and KV head, code = the format's
//                        number nearest to x / scale;
//   focus_dequantize_kv  x = code * scale, the product in fp32, which bf16 outputs round once more (one product instead of
//                        an exact one of 32 bits: 2^-24 of the element beside the 2^-8 that bf16 costs anyway).
// Both are bound by HBM: per element size(T) + 1 bytes move.  A row (64 or 128 elements) belongs to neighbouring lanes,
// sixteen bytes of the wide side at a time (one such vector per lane when reading back, two when writing, so that the
// row's two divisions are shared by more elements), so every access covers full sectors and the maximum is a butterfly
// over those lanes.  Rows of one KV head are neighbours in the grid: their codes and scales are neighbours in the cache.
// A thread has one row in flight where there are few (latency counts), else two (writing) or four (reading back):
// 32768 keys of 32 heads of 128 read back into bf16 in 66 us with four (6.2 TB/s), 139 us with one.  Writing is held by
// its instructions before HBM: 16384 positions of 4 heads of 128, keys and values from bf16 to e4m3, take 14.4 us
// (3.5 TB/s; the fixed cost of a launch is about 3), against 25 to 33 us with a library division and conversion per
// element; blocks of 128 threads, because the fence at a block's end then holds up fewer of them (int8 16.2 -> 14.7 us).
#include <float.h>

#include "focus_common.cuh"

namespace {

constexpr int QK_THREADS = 128;
constexpr int QK_VECS = 2;                              // sixteen-byte vectors per lane when writing
constexpr float FLUSH_BELOW = 8.271806125530277e-25f;   // 2^-80: rows smaller than this are stored as zeros

template <typename F> __device__ __forceinline__ constexpr float fmt_max() { return sizeof(F) == 1 ? 448.f : 0.f; }
template <> __device__ __forceinline__ constexpr float fmt_max<int8_t>() { return 127.f; }

// A code must not depend on how a reciprocal was rounded: the quotient is the correctly rounded x / scale.  With
// inv = RN(1 / scale), q = x inv is off by up to 2 ulp, one Newton step leaves it within one ulp, and by Markstein's
// theorem ("Computation of elementary functions on the IBM RISC System/6000", 1990) the next step then yields
// RN(x / scale), as long as the remainder x - q scale is exact.  It is a multiple of ulp(q) ulp(scale): the scale is
// at least 2^-80 / 448 > 2^-89 and a quotient that can become a code other than zero is at least 2^-10, so that is
// 2^-33 2^-112 or more, above fp32's last bit (2^-149).  Smaller quotients become code zero, right or wrong in their
// last bits.  |x| <= max|x| keeps everything else far from overflow.
__device__ __forceinline__ float quotient(float x, float scale, float inv) {
  float q = x * inv;
  q = fmaf(fmaf(-q, scale, x), inv, q);
  return fmaf(fmaf(-q, scale, x), inv, q);
}
// Four codes.  |q| exceeds the format's largest number by rounding at most, which the conversions take back; adding
// 1.5 * 2^23 rounds to an integer (ties to even) and leaves it, as two's complement, in the low byte.
__device__ __forceinline__ uint32_t pack_codes(const float (&q)[4], int8_t) {
  uint32_t u[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) u[e] = __float_as_uint(q[e] + 12582912.f);
  return __byte_perm(__byte_perm(u[0], u[1], 0x0040), __byte_perm(u[2], u[3], 0x0040), 0x5410);
}
__device__ __forceinline__ uint32_t pack_codes(const float (&q)[4], __nv_fp8_e4m3) {
  const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(q[0], q[1]), __NV_SATFINITE, __NV_E4M3);
  const uint32_t hi = __nv_cvt_float2_to_fp8x2(make_float2(q[2], q[3]), __NV_SATFINITE, __NV_E4M3);
  return lo | hi << 16;
}

// the largest |x| of a thread's elements as ordered bits (infinities and NaN above every number)
template <typename T, int V>
__device__ __forceinline__ uint32_t abs_bits(const uint4 (&raw)[V]) {
  uint32_t m = 0u;
#pragma unroll
  for (int v = 0; v < V; ++v) {
    const uint32_t w[4] = {raw[v].x, raw[v].y, raw[v].z, raw[v].w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (sizeof(T) == 2) m = __vmaxu2(m, w[i] & 0x7fff7fffu);
      else m = max(m, w[i] & 0x7fffffffu);
    }
  }
  if constexpr (sizeof(T) == 2) m = max(m & 0xffff0000u, m << 16);
  return m;
}

struct RowArgs {
  long long wide_stride_row, wide_stride_head;    // of the rows written from / read into
  long long kv_stride_tok, kv_stride_head, scale_stride;
  int L, pos_base, max_rows, first;               // first: 0 the grid's halves start with the keys, 1 values only
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

// grid (row groups, Hkv, halves): keys, values or both, `first` says which comes first; LPR lanes per row, V vectors
// of sixteen bytes each
template <typename T, typename F, int D, int U>
__global__ void __launch_bounds__(QK_THREADS)
quantize_rows_kernel(const T* __restrict__ Kn, const T* __restrict__ Vn, uint8_t* __restrict__ Kc,
                     uint8_t* __restrict__ Vc, float* __restrict__ Ks, float* __restrict__ Vs, const RowArgs a) {
  constexpr int EPC = 16 / sizeof(T), V = QK_VECS, LPR = D / EPC / V, ROWS = QK_THREADS / LPR;
  const bool val = (int)blockIdx.z + a.first != 0;
  const T* src = val ? Vn : Kn;
  const int g = blockIdx.y, c = threadIdx.x % LPR;
  const int r0 = blockIdx.x * (ROWS * U) + threadIdx.x / LPR;
  const int n = a.rows ? min(max(*a.n_rows, 0), a.max_rows) : a.max_rows;
  int pos[U];
  uint4 raw[U][V];
#pragma unroll
  for (int k = 0; k < U; ++k) {
    const int r = r0 + k * ROWS;
    pos[k] = -1;
#pragma unroll
    for (int v = 0; v < V; ++v) raw[k][v] = make_uint4(0, 0, 0, 0);
    if (r < n) {
      pos[k] = row_position(a, r, true);
      if (pos[k] < 0 && c == 0) set_status(a.status, FOCUS_ERR_INVALID_ARG);
      const T* p = src + (long long)r * a.wide_stride_row + (long long)g * a.wide_stride_head + c * EPC;
#pragma unroll
      for (int v = 0; v < V; ++v) raw[k][v] = __ldg(reinterpret_cast<const uint4*>(p + v * LPR * EPC));
    }
  }
#pragma unroll
  for (int k = 0; k < U; ++k) {
    uint32_t mb = abs_bits<T, V>(raw[k]);
#pragma unroll
    for (int o = LPR / 2; o > 0; o >>= 1) mb = max(mb, __shfl_xor_sync(0xffffffffu, mb, o));
    float m = __uint_as_float(mb);
    const bool wild = mb >= 0x7f800000u;                     // the row holds an infinity or a NaN
    if (__any_sync(0xffffffffu, wild)) {                     // these do not enter the scale
      float f = 0.f;
#pragma unroll
      for (int v = 0; v < V; ++v) {
        float x[EPC];
        unpack16<T>(raw[k][v], x);
#pragma unroll
        for (int e = 0; e < EPC; ++e) f = fmaxf(f, fabsf(x[e]) <= FLT_MAX ? fabsf(x[e]) : 0.f);
      }
#pragma unroll
      for (int o = LPR / 2; o > 0; o >>= 1) f = fmaxf(f, __shfl_xor_sync(0xffffffffu, f, o));
      m = f;
    }
    if (pos[k] < 0) continue;
    const bool zero = m < FLUSH_BELOW;
    const float scale = zero ? 0.f : __fdiv_rn(m, fmt_max<F>()), inv = zero ? 0.f : __frcp_rn(scale);
    uint8_t* dst = (val ? Vc : Kc) + (long long)g * a.kv_stride_head + (long long)pos[k] * a.kv_stride_tok + c * EPC;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      float x[EPC];
      unpack16<T>(raw[k][v], x);
      if (wild) {                                            // NaN -> 0, infinities -> the largest number
#pragma unroll
        for (int e = 0; e < EPC; ++e) x[e] = x[e] != x[e] ? 0.f : fminf(fmaxf(x[e], -m), m);
      }
      uint32_t w[EPC / 4];
#pragma unroll
      for (int i = 0; i < EPC / 4; ++i) {
        float q[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) q[e] = quotient(x[4 * i + e], scale, inv);
        w[i] = pack_codes(q, F());
      }
      if constexpr (EPC == 8) *reinterpret_cast<uint2*>(dst + v * LPR * EPC) = make_uint2(w[0], w[1]);
      else *reinterpret_cast<uint32_t*>(dst + v * LPR * EPC) = w[0];
    }
    if (c == 0) (val ? Vs : Ks)[(long long)g * a.scale_stride + pos[k]] = scale;
  }
  publish_outputs();
}

// the same grid; a lane reads EPC codes of a row and writes sixteen bytes
template <typename T, typename F, int D, int U>
__global__ void __launch_bounds__(QK_THREADS)
dequantize_rows_kernel(const uint8_t* __restrict__ Kc, const uint8_t* __restrict__ Vc, const float* __restrict__ Ks,
                       const float* __restrict__ Vs, T* __restrict__ Ko, T* __restrict__ Vo, const RowArgs a) {
  constexpr int EPC = 16 / sizeof(T), LPR = D / EPC, ROWS = QK_THREADS / LPR;
  const bool val = (int)blockIdx.z + a.first != 0;
  T* out = val ? Vo : Ko;
  const int g = blockIdx.y, c = threadIdx.x % LPR;
  const int r0 = blockIdx.x * (ROWS * U) + threadIdx.x / LPR;
  const int n = a.rows ? min(max(*a.n_rows, 0), a.max_rows) : a.max_rows;
  const uint8_t* codes = (val ? Vc : Kc) + (long long)g * a.kv_stride_head + c * EPC;
  const float* scales = (val ? Vs : Ks) + (long long)g * a.scale_stride;
  uint32_t w[U][EPC / 4];
  float scale[U];
  bool ok[U];
#pragma unroll
  for (int k = 0; k < U; ++k) {
    const int r = r0 + k * ROWS, pos = r < n ? row_position(a, r, false) : -1;
    ok[k] = pos >= 0;
    if (r < n && !ok[k] && c == 0) set_status(a.status, FOCUS_ERR_INVALID_ARG);
    if (!ok[k]) continue;
    const uint8_t* src = codes + (long long)pos * a.kv_stride_tok;
    scale[k] = __ldg(scales + pos);
    if constexpr (EPC == 8) {
      const uint2 v = __ldg(reinterpret_cast<const uint2*>(src));
      w[k][0] = v.x; w[k][1] = v.y;
    } else {
      w[k][0] = __ldg(reinterpret_cast<const uint32_t*>(src));
    }
  }
#pragma unroll
  for (int k = 0; k < U; ++k) {
    if (!ok[k]) continue;
    uint32_t o[4];
#pragma unroll
    for (int i = 0; i < EPC / 4; ++i) {
      float f[4];
      codes_to_float(w[k][i], F(), f);
      if constexpr (sizeof(T) == 2) {
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const __nv_bfloat162 b = __floats2bfloat162_rn(f[2 * e] * scale[k], f[2 * e + 1] * scale[k]);
          o[2 * i + e] = *reinterpret_cast<const uint32_t*>(&b);
        }
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] = __float_as_uint(f[e] * scale[k]);
      }
    }
    *reinterpret_cast<uint4*>(out + (long long)(r0 + k * ROWS) * a.wide_stride_row + (long long)g * a.wide_stride_head + c * EPC) =
        make_uint4(o[0], o[1], o[2], o[3]);
  }
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
  a.L = shape->L; a.pos_base = pos_base; a.max_rows = max_rows; a.first = wide_k ? 0 : 1;
  a.rows = rows; a.n_rows = n_rows; a.status = ctx->d_status;
  return FOCUS_OK;
}

// one instantiation per (dtype, format, head dim, rows per thread)
#define FOCUS_QK_DISPATCH(LAUNCH)                                                                            \
  do {                                                                                                       \
    const bool bf = shape->dtype == FOCUS_BF16, i8 = cache->format == FOCUS_KV_INT8, d128 = shape->head_dim == 128; \
    if (bf) {                                                                                                \
      if (i8) { if (d128) LAUNCH(__nv_bfloat16, int8_t, 128); else LAUNCH(__nv_bfloat16, int8_t, 64); }      \
      else { if (d128) LAUNCH(__nv_bfloat16, __nv_fp8_e4m3, 128); else LAUNCH(__nv_bfloat16, __nv_fp8_e4m3, 64); } \
    } else {                                                                                                 \
      if (i8) { if (d128) LAUNCH(float, int8_t, 128); else LAUNCH(float, int8_t, 64); }                      \
      else { if (d128) LAUNCH(float, __nv_fp8_e4m3, 128); else LAUNCH(float, __nv_fp8_e4m3, 64); }           \
    }                                                                                                        \
  } while (0)

inline dim3 row_grid(const focus_shape* s, int max_rows, int halves, int vecs, int u) {
  const int lpr = s->head_dim * (s->dtype == FOCUS_BF16 ? 2 : 4) / 16 / vecs, per = QK_THREADS / lpr * u;
  return dim3((max_rows + per - 1) / per, s->n_kv_heads, halves);
}
// several rows per thread once that still leaves every SM eight blocks
inline bool many_rows(const focus_ctx* ctx, const dim3& g) {
  return (long long)g.x * g.y * g.z >= 8ll * ctx->sm_count;
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
  const int halves = (K_new != nullptr) + (V_new != nullptr);
  const dim3 g1 = row_grid(shape, max_rows, halves, QK_VECS, 1), gm = row_grid(shape, max_rows, halves, QK_VECS, 2);
  const bool many = many_rows(ctx, gm);
#define LAUNCH_U(T, F, D, U, G)                                                                                  \
  quantize_rows_kernel<T, F, D, U><<<G, QK_THREADS, 0, stream>>>((const T*)K_new, (const T*)V_new, (uint8_t*)cache->K, \
                                                                 (uint8_t*)cache->V, cache->K_scale, cache->V_scale, a)
#define LAUNCH(T, F, D) do { if (many) LAUNCH_U(T, F, D, 2, gm); else LAUNCH_U(T, F, D, 1, g1); } while (0)
  FOCUS_QK_DISPATCH(LAUNCH);
#undef LAUNCH
#undef LAUNCH_U
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
  const int halves = (K_out != nullptr) + (V_out != nullptr);
  const dim3 g1 = row_grid(shape, max_rows, halves, 1, 1), gm = row_grid(shape, max_rows, halves, 1, 4);
  const bool many = many_rows(ctx, gm);
#define LAUNCH_U(T, F, D, U, G)                                                                                  \
  dequantize_rows_kernel<T, F, D, U><<<G, QK_THREADS, 0, stream>>>((const uint8_t*)cache->K, (const uint8_t*)cache->V, \
                                                                   cache->K_scale, cache->V_scale, (T*)K_out, (T*)V_out, a)
#define LAUNCH(T, F, D) do { if (many) LAUNCH_U(T, F, D, 4, gm); else LAUNCH_U(T, F, D, 1, g1); } while (0)
  FOCUS_QK_DISPATCH(LAUNCH);
#undef LAUNCH
#undef LAUNCH_U
  FOCUS_CHECK_LAUNCH();
  return FOCUS_OK;
}
