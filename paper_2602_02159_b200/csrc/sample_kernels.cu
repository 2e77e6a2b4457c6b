// focus_sample: one token per listed position, drawn from its logits row with temperature, top-k, top-p and min-p by a
// given uniform number.
//
// A row belongs to one thread-block cluster.  Each CTA loads its contiguous slice of the vocabulary into shared memory
// (the logits cross HBM once) and every later pass runs there; the CTAs exchange a few numbers per pass through
// distributed shared memory.  Weights and sums are fp64: a token is decided by comparing two sums over the vocabulary,
// and in fp32 those sums are off by as much as a rare token weighs.  Sums run in a fixed order (lanes, warps, CTAs), so
// the answer does not depend on timing.
//
// The kept set is a prefix of the descending order.  Two ways to it (a list's weights are integers in units of 2^-50 of the
// largest weight, off by half of that; a lighter token counts as one unit in the draw, so that it has a share):
//   short list  (up to 2048 tokens).  Which logits to collect: for top-k up to 1024, those from the k-th largest of the
//               maxima of the threads' shares up -- a lower bound of the k-th largest logit that few more reach; for a
//               nucleus, those up to the histogram bin in which it must end.  They are collected in index order and cut by
//               one CTA with integer weights in registers: up to 128 tokens by comparing all pairs, else by searching the
//               last kept key.
//   any length  (no cut, min-p alone, longer top-k and nuclei): the key T of the last kept logit, by counts (top-k: 8-bit
//               digits of a radix descent) and by weight (top-p: quarters of the keys that the histogram leaves open);
//               (T, how many of the tokens at T) says all about the set.  Then the kept weight per warp segment in index
//               order, the segment that holds u * total, a run of it per lane, and its walk.
// What bounds it: HBM for many rows of top-k (512 rows of 126464 bf16 logits, top-k 50, top-p 0.9: 66 us, of which the
// loads are 20), instruction issue in the pass over the vocabulary's weights for a nucleus (35 rows, top-p 0.95: 35 us,
// 41 on other devices; 11 us are that pass, 24 instructions per logit), and the latency of a dozen barriers and exchanges for
// one row (50257 fp32 logits: 14 us).
#include <cooperative_groups.h>
#include <float.h>

#include "focus_common.cuh"

namespace cg = cooperative_groups;

namespace {

constexpr int SP_THREADS = 512;
constexpr int SP_WARPS = SP_THREADS / 32;
constexpr int SP_MAX_CLUSTER = 8;
constexpr int SP_SLICE_BYTES = 180 * 1024;               // largest slice of a row per CTA
constexpr int SP_LIST = 2048;                            // most tokens of a short list
constexpr int SP_LIST_K = 1024;                          // largest top-k that goes through it; tokens tried for a nucleus
constexpr int SP_PER = SP_LIST / SP_THREADS;             // tokens of the list per thread
constexpr int SP_PAIRS = SP_THREADS / 4;                 // most tokens of a list that is cut by comparing all pairs
// scratch behind the slice: thread maxima | list | one byte per 16-byte vector of the slice
constexpr int SP_OFF_LIST = SP_THREADS * 4, SP_OFF_MASK = SP_OFF_LIST + SP_LIST * 8, SP_SMEM = 212 * 1024;   // largest, all told
constexpr int SP_TAB = 64, SP_TAB_COPIES = 16;           // table of powers: entries, and copies (one per pair of banks)
constexpr int SP_BINS = 2048;                            // of a nucleus's histogram
constexpr uint32_t KEY_NEG_INF = 0x007FFFFFu;            // float_key(-inf); NaN is below it
static_assert(SP_BINS * 4 <= SP_LIST * 8 && SP_BINS == 4 * SP_THREADS, "a histogram lies where a list does");
static_assert(SP_SLICE_BYTES + SP_OFF_MASK + SP_SLICE_BYTES / 16 + 16 <= SP_SMEM, "scratch");

__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release;\n\tbarrier.cluster.wait.acquire;" ::: "memory");
}

struct SegSum {            // one warp's contiguous segment of the row
  double w;                // kept weight above the threshold key
  int n_gt, n_eq;          // tokens above it / at it
};

struct SampleShared {
  double tab[SP_TAB * SP_TAB_COPIES];        // [i][copy]: 2^(i / SP_TAB)
  double dsum[2][SP_WARPS][3];
  int isum[2][SP_WARPS];
  double cta_d[2][3];
  int cta_i[2];
  SegSum seg[SP_WARPS];
  SegSum all[SP_MAX_CLUSTER * SP_WARPS];
  uint2 first[SP_WARPS], cta_first;
  int list_n, list_ok;
  alignas(16) int hist[2][256];
  int scan_i[33];
  unsigned long long fx[2][SP_WARPS][3];
  int digit, above, found;
  uint4 tail;              // the vector that the row ends in
  uint32_t key_hi[SP_WARPS], key_lo[SP_WARPS];
  float2 edge[SP_WARPS];
  // the segment that holds u * total
  int hit, hit_eq, kept;
  double before, total;
};
static_assert(sizeof(SampleShared) <= 15 * 1024 && SP_SMEM + 15 * 1024 <= 227 * 1024, "shared memory");

struct SampleParams {
  const void* logits;
  long long row_stride;
  int vocab, pos_base, n_pos, max_rows, slice;           // slice: elements per CTA
  const int32_t* rows;
  const int32_t* n_rows;
  float temperature, top_p, min_p;
  int top_k;
  const float* u;
  float* conf;
  int32_t* token;
  float* prob;
  int32_t* n_kept;
  int32_t* status;
};

// Sums over the cluster, the same in every thread.  Two slots in turn: one cluster barrier per call is enough, since a
// CTA writes a slot again only after a barrier that its slowest reader has passed.
template <int N>
__device__ __forceinline__ void sum_all(cg::cluster_group& cl, SampleShared& sh, int& turn, double (&v)[N], int& cnt) {
  const int t = turn & 1, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  ++turn;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] += __shfl_xor_sync(0xffffffffu, v[i], o);
  }
  cnt = __reduce_add_sync(0xffffffffu, cnt);
  if (lane == 0) {
#pragma unroll
    for (int i = 0; i < N; ++i) sh.dsum[t][warp][i] = v[i];
    sh.isum[t][warp] = cnt;
  }
  __syncthreads();
  if (warp == 0) {                                       // the warps' sums in a fixed tree
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = lane < SP_WARPS ? sh.dsum[t][lane][i] : 0.0;
    cnt = lane < SP_WARPS ? sh.isum[t][lane] : 0;
#pragma unroll
    for (int o = SP_WARPS / 2; o > 0; o >>= 1) {
#pragma unroll
      for (int i = 0; i < N; ++i) v[i] += __shfl_xor_sync(0xffffffffu, v[i], o);
      cnt += __shfl_xor_sync(0xffffffffu, cnt, o);
    }
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = __shfl_sync(0xffffffffu, v[i], 0);
    cnt = __shfl_sync(0xffffffffu, cnt, 0);
  }
  if (threadIdx.x == 0) {
#pragma unroll
    for (int i = 0; i < N; ++i) sh.cta_d[t][i] = v[i];
    sh.cta_i[t] = cnt;
  }
  cluster_sync();
  const int nc = (int)cl.num_blocks();
  const SampleShared* far = cl.map_shared_rank(&sh, min(lane, nc - 1));   // lane q fetches rank q's sums
  double f[N];
#pragma unroll
  for (int i = 0; i < N; ++i) { f[i] = lane < nc ? far->cta_d[t][i] : 0.0; v[i] = 0.0; }
  cnt = __reduce_add_sync(0xffffffffu, lane < nc ? far->cta_i[t] : 0);
  for (int r = 0; r < nc; ++r) {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] += __shfl_sync(0xffffffffu, f[i], r);
  }
}

// The largest logit and the number of candidates, over the cluster and in every thread; its barriers publish what was
// written before it.
__device__ __forceinline__ void first_all(cg::cluster_group& cl, SampleShared& sh, float& m, int& cnt) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const uint32_t k = __reduce_max_sync(0xffffffffu, float_key(m)), c = __reduce_add_sync(0xffffffffu, (unsigned)cnt);
  if (lane == 0) sh.first[warp] = make_uint2(k, c);
  __syncthreads();
  uint2 v = lane < SP_WARPS ? sh.first[lane] : make_uint2(0u, 0u);
  v.x = __reduce_max_sync(0xffffffffu, v.x); v.y = __reduce_add_sync(0xffffffffu, v.y);
  const int nc = (int)cl.num_blocks();
  if (nc > 1) {
    if (threadIdx.x == 0) sh.cta_first = v;
    cluster_sync();
    v = lane < nc ? cl.map_shared_rank(&sh, lane)->cta_first : make_uint2(0u, 0u);
    v.x = __reduce_max_sync(0xffffffffu, v.x); v.y = __reduce_add_sync(0xffffffffu, v.y);
  }
  m = key_to_float(v.x); cnt = (int)v.y;
}

template <typename T>
__device__ __forceinline__ void unpack_logits(const uint4& raw, float (&x)[16 / sizeof(T)]) {
  const uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (sizeof(T) == 2) {
      x[2 * i] = __uint_as_float(w[i] << 16);
      x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
    } else {
      x[i] = __uint_as_float(w[i]);
    }
  }
}
// NaN -> -inf, and the largest and smallest of a vector
__device__ __forceinline__ uint32_t max_bf2(uint32_t a, uint32_t b) { uint32_t d; asm("max.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b)); return d; }
__device__ __forceinline__ uint32_t min_bf2(uint32_t a, uint32_t b) { uint32_t d; asm("min.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b)); return d; }
template <typename T>
__device__ __forceinline__ void clean_logits(uint4& raw, float& hi, float& lo) {
  if constexpr (sizeof(T) == 2) {
    raw.x = max_bf2(raw.x, 0xFF80FF80u); raw.y = max_bf2(raw.y, 0xFF80FF80u);
    raw.z = max_bf2(raw.z, 0xFF80FF80u); raw.w = max_bf2(raw.w, 0xFF80FF80u);
    const uint32_t a = max_bf2(max_bf2(raw.x, raw.y), max_bf2(raw.z, raw.w)), b = min_bf2(min_bf2(raw.x, raw.y), min_bf2(raw.z, raw.w));
    hi = fmaxf(__uint_as_float(a << 16), __uint_as_float(a & 0xFFFF0000u));
    lo = fminf(__uint_as_float(b << 16), __uint_as_float(b & 0xFFFF0000u));
  } else {
    float x[4];
    unpack_logits<float>(raw, x);
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = fmaxf(x[i], -INFINITY);
    raw = make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
    hi = fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3]));
    lo = fminf(fminf(x[0], x[1]), fminf(x[2], x[3]));
  }
}
template <typename T>
__device__ __forceinline__ float largest_of(const uint4& raw) {
  if constexpr (sizeof(T) == 2) {
    const uint32_t a = max_bf2(max_bf2(raw.x, raw.y), max_bf2(raw.z, raw.w));
    return fmaxf(__uint_as_float(a << 16), __uint_as_float(a & 0xFFFF0000u));
  } else {
    return fmaxf(fmaxf(__uint_as_float(raw.x), __uint_as_float(raw.y)), fmaxf(__uint_as_float(raw.z), __uint_as_float(raw.w)));
  }
}
// bit e: element e of a vector is at least `from`
template <typename T>
__device__ __forceinline__ uint32_t reaching_bits(const uint4& raw, float from) {
  const uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
  uint32_t bits = 0u;
  if constexpr (sizeof(T) == 2) {
    const __nv_bfloat162 f = __bfloat162bfloat162(__float2bfloat16_ru(from));         // the least bf16 that is
#pragma unroll
    for (int i = 0; i < 4; ++i) bits |= __hge2_mask(*reinterpret_cast<const __nv_bfloat162*>(&w[i]), f) & (0x00020001u << (2 * i));
    return (bits | bits >> 16) & 0xFFu;
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) bits |= __uint_as_float(w[i]) >= from ? 1u << i : 0u;
    return bits;
  }
}

__device__ __forceinline__ float ex2_approx(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// Powers of two in fp64: t = n / 64 + r, 2^t = 2^(n >> 6) * tab[n & 63] * 2^r (Tang's table-driven scheme, 1989).  Every
// lane reads its own copy of the table, so that no two lanes of a half warp meet in a bank: with one table of 1024
// entries, and one multiplication less, the lookups took most of the time.  2^r is a cubic with |r| <= h = 1/128: the
// Taylor terms, and the fourth power replaced by h^2 r^2 - h^4 / 8 (Chebyshev), without that constant, since only ratios
// of weights matter.  It leaves ln2^4 / 24 * h^4 / 4 = 9e-12 of a weight between any two of them.
// -1020 <= t <= 0; no branch, so that several run side by side.
__device__ __forceinline__ double pow2_near(double t, const double* tab) {
  const double magic = 6755399441055744.0;               // 1.5 * 2^52: adding it leaves the rounded integer in the low bits
  constexpr double ln2 = 0.69314718055994531, h = 0.5 / SP_TAB;
  const double tm = fma(t, (double)SP_TAB, magic);
  const int n = __double2loint(tm);
  const double r = fma(tm - magic, -1.0 / SP_TAB, t);
  const double b = tab[(n & (SP_TAB - 1)) * SP_TAB_COPIES];
  const double f = fma(r, fma(r, ln2 * ln2 * ln2 / 6.0, ln2 * ln2 / 2.0 + h * h * (ln2 * ln2 * ln2 * ln2 / 24.0)), ln2);
  const double w = fma(b, r * f, b);
  return __hiloint2double(__double2hiint(w) + ((n >> 6) << 20), __double2loint(w));
}

// The same for sums over the vocabulary, in 18 instructions of which two are fp64 (more than sixty, ten of them fp64, with
// pow2_near and a separate histogram): x s for s = s_hi + s_lo is reduced in fp32.  With zero = 1.5 * 2^17 - R / 64 the sum
// x s_hi + zero is rounded to multiples of 1/64, R being 64 m s_hi rounded, so its bits count 64ths of the exponent from
// the maximum's down (the bins of a histogram as well) and x s_hi less that multiple is a single fused operation: r.
// Weights come relative to 2^(R / 64).  r, up to 2^-7, is rounded twice by up to 2^-32: ln2 2^-31 = 3.2e-10 of a weight.
// 2^r - 1 < 0.0055 is r times a factor near 0.7 that its last addition rounds by 2^-25 and fp32's ln2 shifts by 1.9e-9
// (2.5e-10 after r), and their product is rounded by 2^-32 (2.3e-10).  Together, with 1e-11 of the cubic and 2e-11 that
// s_hi + s_lo lacks of s, 8.4e-10: less than 1e-9, of either sign.
struct Reduced {
  int bits;
  float r;
};
__device__ __forceinline__ Reduced reduce_exponent(float x, float s_hi, float s_lo, float zero) {
  const float tm = fmaf(x, s_hi, zero);
  return {__float_as_int(tm), fmaf(x, s_lo, fmaf(x, s_hi, -(tm - zero)))};
}
__device__ __forceinline__ double pow2_reduced(const Reduced& a, const double* tab) {
  const float ln2 = 0.69314718f, h = 0.5f / SP_TAB;
  const float q = a.r * fmaf(a.r, fmaf(a.r, ln2 * ln2 * ln2 / 6.f, ln2 * ln2 / 2.f + h * h * (ln2 * ln2 * ln2 * ln2 / 24.f)), ln2);
  const double b = tab[(a.bits & (SP_TAB - 1)) * SP_TAB_COPIES];
  const double w = fma(b, (double)q, b);
  return __hiloint2double(__double2hiint(w) + ((a.bits & -SP_TAB) << 14), __double2loint(w));
}
static_assert(SP_TAB == 64, "the bits above a table's index start at an exponent's");

// Sums over the first NW warps of a block (all of them call it) of numbers below 2^53: integer weights, so that a
// warp's sum is two hardware reductions of 27-bit halves instead of five rounds of shuffles.  Two slots in turn: one
// barrier per call.
__device__ __forceinline__ unsigned long long warp_sum_fx(unsigned long long v) {
  const unsigned lo = __reduce_add_sync(0xffffffffu, (unsigned)(v & 0x7FFFFFFu)), hi = __reduce_add_sync(0xffffffffu, (unsigned)(v >> 27));
  return ((unsigned long long)hi << 27) + lo;
}
template <int NW, int N>
__device__ __forceinline__ void sum_fx(SampleShared& sh, int& turn, unsigned long long (&v)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = warp_sum_fx(v[i]);
  if constexpr (NW > 1) {
    const int t = turn & 1, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    ++turn;
    if (lane == 0) {
#pragma unroll
      for (int i = 0; i < N; ++i) sh.fx[t][warp][i] = v[i];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) {
      // the halves of a warp's sum: below 2^32 and 2^31, so they are summed in 16-bit steps too
      const unsigned long long w = lane < NW ? sh.fx[t][lane][i] : 0ull;
      v[i] = warp_sum_fx(w & 0x3FFFFFFFFFFFFFull) + ((unsigned long long)__reduce_add_sync(0xffffffffu, (unsigned)(w >> 54)) << 54);
    }
  }
}
// The same for three small counts (at most 31 per thread), packed into one word.
template <int NW>
__device__ __forceinline__ void sum_counts(SampleShared& sh, int& turn, const unsigned (&c)[3], unsigned long long (&v)[3]) {
  const unsigned w = __reduce_add_sync(0xffffffffu, c[0] | (c[1] << 10) | (c[2] << 20));
  if constexpr (NW == 1) {
    v[0] = w & 1023u; v[1] = (w >> 10) & 1023u; v[2] = w >> 20;
  } else {
    const int t = turn & 1, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    ++turn;
    if (lane == 0) sh.fx[t][warp][0] = w;
    __syncthreads();
    const unsigned x = lane < NW ? (unsigned)sh.fx[t][lane][0] : 0u;
    const unsigned a = __reduce_add_sync(0xffffffffu, (x & 1023u) | ((x >> 10 & 1023u) << 16));
    v[0] = a & 0xFFFFu; v[1] = a >> 16; v[2] = __reduce_add_sync(0xffffffffu, x >> 20);
  }
}
// Exclusive prefix over those warps' threads; `total` over all of them.
template <int NW>
__device__ __forceinline__ unsigned long long excl_fx(SampleShared& sh, int& turn, unsigned long long v, unsigned long long& total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  unsigned long long inc = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const unsigned long long y = __shfl_up_sync(0xffffffffu, inc, o);
    if (lane >= o) inc += y;
  }
  unsigned long long before = inc - v;
  total = __shfl_sync(0xffffffffu, inc, 31);
  if constexpr (NW > 1) {
    const int t = turn & 1;
    ++turn;
    if (lane == 0) sh.fx[t][warp][0] = total;
    __syncthreads();
    unsigned long long sum = 0;
#pragma unroll
    for (int q = 0; q < NW; ++q) {
      if (q == warp) before += sum;
      sum += sh.fx[t][q][0];
    }
    total = sum;
  }
  return before;
}
// Three keys that cut lo + 1 .. hi into quarters, and which part a search among lo .. hi goes on with: `reached` says
// whether what(t[i]) reaches the goal.
__device__ __forceinline__ void quarter(uint32_t lo, uint32_t hi, uint32_t (&t)[3]) {
  const uint32_t n = hi - lo, r = n & 3u;
#pragma unroll
  for (int i = 0; i < 3; ++i) t[i] = lo + (i + 1) * (n >> 2) + (((i + 1) * r + 3u) >> 2);
}
template <typename V>
__device__ __forceinline__ void go_on(uint32_t& lo, uint32_t& hi, V& above, const uint32_t (&t)[3], const bool (&reached)[3], const V (&what)[3]) {
  if (reached[2]) lo = t[2];
  else if (reached[1]) { lo = t[1]; hi = t[2] - 1; above = what[2]; }
  else if (reached[0]) { lo = t[0]; hi = t[1] - 1; above = what[1]; }
  else { hi = t[0] - 1; above = what[0]; }
}
// The largest t of lo .. hi such that what(t) = the sum over the threads of f(t) reaches `goal`, a quarter of the keys left
// per step; what(lo) reaches it by assumption.  `above`: what(hi + 1), then what(t + 1).
template <int NW, bool COUNTS, typename F>
__device__ __forceinline__ uint32_t largest_reaching(SampleShared& sh, int& turn, uint32_t lo, uint32_t hi, unsigned long long goal,
                                                     unsigned long long& above, F f) {
  while (lo < hi) {
    uint32_t t[3];
    quarter(lo, hi, t);
    unsigned long long s[3];
    if constexpr (COUNTS) {
      unsigned c[3];
      f(t[0], t[1], t[2], c);
      sum_counts<NW>(sh, turn, c, s);
    } else {
      f(t[0], t[1], t[2], s);
      sum_fx<NW, 3>(sh, turn, s);
    }
    const bool reached[3] = {s[0] >= goal, s[1] >= goal, s[2] >= goal};
    go_on(lo, hi, above, t, reached, s);
  }
  return lo;
}

constexpr double FX_ONE = 1125899906842624.0;            // 2^50: a weight of 1 (a thread holds at most four)

struct Draw {                                            // what a list is cut by
  int top_k;                                             // 0: no cut
  double top_p, z, min_p, u;                             // top_p 1: no cut; z: weight of the whole vocabulary, or < 0: the list's
  uint32_t key_lo;                                       // no key of the list is below
  uint32_t key_top;                                      // the nucleus does not end above
  bool complete;                                         // the list holds every candidate
};
// Cuts the list of n <= SP_LIST tokens (descending priority: key, then place) and draws.  Returns the place of the
// token drawn in `at` (on the thread that holds it; -1 elsewhere), or false where the nucleus reaches beyond the list.
// Called by all threads; a thread's tokens are neighbours.
template <int KEY_BITS, typename W>
__device__ __forceinline__ bool draw_from_list(SampleShared& sh, const unsigned long long* list, int n, uint32_t key_hi, const Draw& d,
                                               W weight, int& at, double& w_at, double& total_w, int& kept) {
  constexpr int NW = SP_WARPS;
  const int tid = threadIdx.x;
  int turn = 0;
  uint32_t key[SP_PER];
  unsigned long long fx[SP_PER];
  unsigned in = 0, light = 0;                            // bit q: token q is in / has a weight, but less than half of 2^-50
#pragma unroll
  for (int q = 0; q < SP_PER; ++q) {
    const int i = tid * SP_PER + q;
    const uint32_t full = i < n ? (uint32_t)(list[i] >> 32) : 0u;
    key[q] = full >> (32 - KEY_BITS);
    fx[q] = 0ull;
    if (i < n) {
      const double w = weight(key_to_float(full));
      fx[q] = (unsigned long long)__double2ll_rn(w * FX_ONE);
      light |= w > 0.0 && fx[q] == 0ull ? 1u << q : 0u;
      in |= 1u << q;
    }
  }
  // keeps of the tokens at key t the first `quota`, drops those below t
  auto cut_at = [&](uint32_t t, unsigned long long quota) {
    unsigned long long eq = 0, all;
#pragma unroll
    for (int q = 0; q < SP_PER; ++q) eq += (in >> q & 1u) && key[q] == t ? 1 : 0;
    unsigned long long before = excl_fx<NW>(sh, turn, eq, all);
#pragma unroll
    for (int q = 0; q < SP_PER; ++q) {
      const bool tie = (in >> q & 1u) && key[q] == t;
      if (key[q] < t || (tie && before >= quota)) in &= ~(1u << q);
      before += tie ? 1 : 0;
    }
  };
  uint32_t key_end = d.key_lo;                           // nor below this
  if (d.top_k > 0 && d.top_k < n) {
    unsigned long long above = 0ull;
    const uint32_t t = largest_reaching<NW, true>(sh, turn, d.key_lo, key_hi, (unsigned long long)d.top_k, above,
                                                  [&](uint32_t t1, uint32_t t2, uint32_t t3, unsigned (&s)[3]) {
      s[0] = s[1] = s[2] = 0u;
#pragma unroll
      for (int q = 0; q < SP_PER; ++q)
        if (in >> q & 1u) { s[0] += key[q] >= t1; s[1] += key[q] >= t2; s[2] += key[q] >= t3; }
    });
    cut_at(t, (unsigned long long)d.top_k - above);
    key_end = t;
  }
  if (d.top_p < 1.0) {
    unsigned long long a[1] = {0ull};
#pragma unroll
    for (int q = 0; q < SP_PER; ++q) a[0] += in >> q & 1u ? fx[q] : 0ull;
    sum_fx<NW, 1>(sh, turn, a);
    const double goal_w = d.top_p * (d.z >= 0.0 ? d.z * FX_ONE : (double)a[0]);
    const unsigned long long goal = (unsigned long long)ceil(goal_w);
    if (a[0] < goal && !d.complete) return false;
    if (a[0] >= goal) {
      unsigned long long above[1] = {0ull};
#pragma unroll
      for (int q = 0; q < SP_PER; ++q) above[0] += (in >> q & 1u) && key[q] > d.key_top ? fx[q] : 0ull;
      sum_fx<NW, 1>(sh, turn, above);
      uint32_t lo = min(key_end, d.key_top), hi = d.key_top;
      if (above[0] >= goal) { lo = hi + 1; hi = key_hi; above[0] = 0ull; }         // (should key_top not hold)
      const uint32_t t = largest_reaching<NW, false>(sh, turn, lo, hi, goal, above[0],
                                              [&](uint32_t t1, uint32_t t2, uint32_t t3, unsigned long long (&s)[3]) {
        s[0] = s[1] = s[2] = 0ull;
#pragma unroll
        for (int q = 0; q < SP_PER; ++q) {
          const unsigned long long v = in >> q & 1u ? fx[q] : 0ull;
          s[0] += key[q] >= t1 ? v : 0ull;
          s[1] += key[q] >= t2 ? v : 0ull;
          s[2] += key[q] >= t3 ? v : 0ull;
        }
      });
      // how many of the tokens at t it takes (their weight is one number)
      const double each = rint(weight(key_to_float(KEY_BITS == 32 ? t : t << 16 | (t & 0x8000u ? 0u : 0xFFFFu))) * FX_ONE);
      const double need = ceil((double)(goal - above[0]) / each);
      cut_at(t, (unsigned long long)fmin(fmax(need, 1.0), (double)SP_LIST));
    }
  }
  if (d.min_p > 0.0) {
#pragma unroll
    for (int q = 0; q < SP_PER; ++q)
      if (in >> q & 1u)
        if (!(weight(key_to_float((uint32_t)(list[tid * SP_PER + q] >> 32))) >= d.min_p)) in &= ~(1u << q);
  }
  // running sums of the kept weights in index order; the first one above u * total (u = 0 draws the first token that has a
  // weight, however small)
#pragma unroll
  for (int q = 0; q < SP_PER; ++q) fx[q] += light >> q & 1u;
  unsigned long long mine = 0ull, total, count;
#pragma unroll
  for (int q = 0; q < SP_PER; ++q) mine += in >> q & 1u ? fx[q] : 0ull;
  unsigned long long run = excl_fx<NW>(sh, turn, mine, total);
  unsigned long long c1[1] = {(unsigned long long)__popc(in)};
  sum_fx<NW, 1>(sh, turn, c1);
  count = c1[0];
  kept = (int)count;
  total_w = (double)total / FX_ONE;
  const unsigned long long target = (unsigned long long)(d.u * (double)total);      // a sum above u * total is one above its floor
  const bool has = mine > 0ull && run <= target && run + mine > target;             // one thread, as u < 1
  at = -1;
  w_at = 0.0;
  if (has) {
#pragma unroll
    for (int q = 0; q < SP_PER; ++q) {
      const unsigned long long v = in >> q & 1u ? fx[q] : 0ull;
      if (at < 0 && run + v > target) at = tid * SP_PER + q;
      run += v;
    }
  }
  if (at >= 0) w_at = weight(key_to_float((uint32_t)(list[at] >> 32)));
  return true;
}

// The same for at most SP_PAIRS tokens, by all threads: four per token, which sum what precedes it in descending order.
// That answers every cut at once, without a search: about 1000 cycles, where the steps of the search above take 4000 to
// 9000.  The outcome is with the first warp.
template <typename W>
__device__ __forceinline__ bool draw_from_pairs(SampleShared& sh, const unsigned long long* list, int n, const Draw& d, W weight, int& at,
                                                double& w_at, double& total_w, int& kept) {
  unsigned long long* fx = reinterpret_cast<unsigned long long*>(sh.hist[1]);
  const int tid = threadIdx.x, lane = tid & 31, i = tid >> 2, part = tid & 3;
  const uint32_t key = i < n ? (uint32_t)(list[i] >> 32) : 0u;
  double w = 0.0;
  unsigned long long mine = 0ull;
  if (i < n) {
    w = weight(key_to_float(key));
    mine = (unsigned long long)__double2ll_rn(w * FX_ONE);
  }
  if (part == 0) fx[i] = mine;
  __syncthreads();
  unsigned long long above = 0ull;
  int rank = 0;
  for (int j = part; j < n; j += 4) {
    const uint32_t k = (uint32_t)(list[j] >> 32);
    if (k > key || (k == key && j < i)) { above += fx[j]; ++rank; }
  }
#pragma unroll
  for (int o = 1; o < 4; o <<= 1) {
    above += __shfl_xor_sync(0xffffffffu, above, o);
    rank += __shfl_xor_sync(0xffffffffu, rank, o);
  }
  const int k = d.top_k > 0 ? min(d.top_k, n) : n;
  if (i < n && rank == k - 1 && part == 0) sh.fx[0][0][0] = above + mine;        // the weight of the k largest
  __syncthreads();
  const unsigned long long all = sh.fx[0][0][0];
  bool in = i < n && rank < k;
  if (d.top_p < 1.0) {
    const unsigned long long goal = (unsigned long long)ceil(d.top_p * (d.z >= 0.0 ? d.z * FX_ONE : (double)all));
    if (all < goal && !d.complete) return false;
    in = in && above < goal;
  }
  in = in && w >= d.min_p;
  if (w > 0.0 && mine == 0ull) mine = 1ull;              // u = 0 draws the first token that has a weight, however small
  if (part == 0) fx[i] = in ? mine | 1ull << 63 : 0ull;
  __syncthreads();
  at = -1;
  if (tid >= 32) return true;
  int turn = 0;
  constexpr int PER = SP_PAIRS / 32;
  unsigned long long v[PER], sum = 0ull, total;
  int count = 0;
#pragma unroll
  for (int q = 0; q < PER; ++q) {
    v[q] = fx[lane * PER + q];
    count += (int)(v[q] >> 63);
    v[q] &= ~(1ull << 63);
    sum += v[q];
  }
  unsigned long long run = excl_fx<1>(sh, turn, sum, total);
  kept = __reduce_add_sync(0xffffffffu, count);
  total_w = (double)total / FX_ONE;
  const unsigned long long target = (unsigned long long)(d.u * (double)total);
  if (run <= target && run + sum > target) {             // one lane, as u < 1
#pragma unroll
    for (int q = 0; q < PER; ++q) {
      if (at < 0 && run + v[q] > target) at = lane * PER + q;
      run += v[q];
    }
    w_at = weight(key_to_float((uint32_t)(list[at] >> 32)));
  }
  return true;
}

// STREAM: one CTA per row, every pass reads the logits from global memory (the second and later ones from L2) instead of
// from a copy in shared memory, and there is no cluster to wait for.
template <typename T, bool STREAM>
__global__ void __launch_bounds__(SP_THREADS, 2)
sample_kernel(const SampleParams p) {
  constexpr int EPC = 16 / sizeof(T);
  constexpr int KEY_BITS = 8 * sizeof(T);                // bf16: the upper half of the float key tells all keys apart
  extern __shared__ __align__(16) uint8_t smem_raw[];
  T* xs = reinterpret_cast<T*>(smem_raw);
  __shared__ SampleShared sh;
  cg::cluster_group cl = cg::this_cluster();
  const int rank = (int)cl.block_rank(), nc = (int)cl.num_blocks();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int r = blockIdx.x / nc;
  const bool lead = rank == 0 && tid == 0;
  auto finish = [&](int tok, float conf, float prob, int kept) {
    p.token[r] = tok; p.conf[r] = conf;
    if (p.prob) p.prob[r] = prob;
    if (p.n_kept) p.n_kept[r] = kept;
  };
  const int n = p.rows ? min(max(*p.n_rows, 0), p.max_rows) : p.max_rows;
  if (r >= n) {
    if (lead) finish(-1, 0.f, 0.f, 0);
    return;
  }
  const int pos = p.rows ? p.rows[r] : p.pos_base + r;
  const float u = p.u[r];
  if (pos < p.pos_base || pos - p.pos_base >= p.n_pos || !(u >= 0.f && u < 1.f)) {
    if (lead) { set_status(p.status, FOCUS_ERR_INVALID_ARG); finish(-1, 0.f, 0.f, 0); }
    return;
  }
  int turn = 0;
  // ---- the slice (NaN as -inf, padded to whole vectors with -inf), the maxima of the threads' shares ----
  const int lo = min(rank * p.slice, p.vocab), cnt = min(p.slice, p.vocab - lo), n_vec = (cnt + EPC - 1) / EPC;
  const T* row = (const T*)p.logits + (long long)(pos - p.pos_base) * p.row_stride + lo;
  uint8_t* scratch = smem_raw + (STREAM ? 0 : (size_t)p.slice * sizeof(T));
  // the one vector that the row ends in, beyond its end -inf
  auto tail_vector = [&](int i) -> uint4 {
    uint32_t w[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      if constexpr (sizeof(T) == 2) {
        const uint32_t a = i + 2 * q < cnt ? __bfloat16_as_ushort(row[i + 2 * q]) : 0xFF80u;
        const uint32_t b = i + 2 * q + 1 < cnt ? __bfloat16_as_ushort(row[i + 2 * q + 1]) : 0xFF80u;
        w[q] = a | (b << 16);
      } else {
        w[q] = i + q < cnt ? __float_as_uint(row[i + q]) : 0xFF800000u;
      }
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
  };
  const float l2e = 1.4426950408889634f;
  float share = -INFINITY;                               // largest logit of this thread's share
  float raw_part = 0.f;                                  // sum of exp(x - share) over it: prob's denominator at temperature 1
  int n_cand = 0;
  auto take = [&](uint4 raw, int i) {
    float hi, low, x[EPC];
    clean_logits<T>(raw, hi, low);
    if constexpr (!STREAM) *reinterpret_cast<uint4*>(xs + i) = raw;
    unpack_logits<T>(raw, x);
    if (low > -INFINITY) {
      n_cand += EPC;
    } else {
#pragma unroll
      for (int e = 0; e < EPC; ++e) n_cand += x[e] > -INFINITY ? 1 : 0;
    }
    if (hi > share) {
      raw_part *= ex2_approx((share - hi) * l2e);
      share = hi;
    }
    if (p.prob && share > -INFINITY) {
      float s0 = 0.f, s1 = 0.f;
#pragma unroll
      for (int e = 0; e < EPC; e += 2) { s0 += ex2_approx((x[e] - share) * l2e); s1 += ex2_approx((x[e + 1] - share) * l2e); }
      raw_part += s0 + s1;
    }
  };
  {
    constexpr int U = 4, STEP = SP_THREADS * EPC;        // U vectors in flight per thread
    int i = tid * EPC;
    for (; i + (U - 1) * STEP + EPC <= cnt; i += U * STEP) {
      uint4 raw[U];
#pragma unroll
      for (int q = 0; q < U; ++q) raw[q] = __ldg(reinterpret_cast<const uint4*>(row + i + q * STEP));
#pragma unroll
      for (int q = 0; q < U; ++q) take(raw[q], i + q * STEP);
    }
    for (; i + EPC <= cnt; i += STEP) take(__ldg(reinterpret_cast<const uint4*>(row + i)), i);
    if (i < cnt) {
      const uint4 raw = tail_vector(i);
      sh.tail = raw;
      take(raw, i);
    }
  }
  for (int i = tid; i < SP_TAB * SP_TAB_COPIES; i += SP_THREADS) {         // as the product of its binary digits' powers
    const double f[6] = {1.0108892860517005, 1.0218971486541166, 1.0442737824274138, 1.0905077326652577, 1.189207115002721,
                         1.4142135623730951};
    double v = 1.0;
#pragma unroll
    for (int q = 0; q < 6; ++q) v *= (i / SP_TAB_COPIES >> q & 1) ? f[q] : 1.0;
    sh.tab[i] = v;
  }
  const double* tab = sh.tab + (lane & (SP_TAB_COPIES - 1));
  uint32_t* share_key = reinterpret_cast<uint32_t*>(scratch);
  share_key[tid] = float_key(share) >> (32 - KEY_BITS);
  float m = share;
  first_all(cl, sh, m, n_cand);
  if (n_cand == 0) {
    if (lead) finish(-1, 0.f, 0.f, 0);
    cluster_sync();
    return;
  }
  // ---- weights: 2^((x - m) log2(e) / temperature) ----
  const double scale = 1.4426950408889634 / (double)p.temperature, md = (double)m;
  const float floor_x = (float)fmax(md - 1000.0 / scale, -(double)FLT_MAX);      // lighter ones may count as 2^-1000
  // weights without a branch, where that floor is a logit well below the maximum (not so for an infinite maximum, one whose
  // neighbouring floats are further apart, or a temperature that flattens the type's whole range) and nothing overflows
  const double floor_t = ((double)floor_x - md) * scale;
  const float s_hi = (float)scale, s_lo = (float)(scale - (double)s_hi);
  const bool plain = m < INFINITY && floor_t < -900.0 && floor_t > -1020.0 && s_hi > 1e-30f && s_hi < 1e30f;
  // they are 2^(x s) for |m s| up to 4096, above that 2^((x - m) s): x is within a factor of two of m then, which makes the
  // difference exact
  const float shift = fabs(md * scale) < 4096.0 ? 0.f : m;
  const float top64 = plain ? (float)(rint((double)(m - shift) * (double)s_hi * SP_TAB) / SP_TAB) : 0.f, zero = 196608.f - top64;
  auto reduced = [&](float x) -> Reduced { return reduce_exponent(fmaxf(x, floor_x) - shift, s_hi, s_lo, zero); };
  const int top_bits = reduced(m).bits;                  // (a tie may put them one off top64's)
  // Which tokens have a weight at all must be one rule wherever a draw can end on them: with u = 0 the first segment, run and
  // token with a weight have to be each other's.  Where weight_plain may be used it is the comparison with floor_x.
  auto weight = [&](float x) -> double {
    if (m == INFINITY) return x == m ? 1.0 : 0.0;
    const double t = ((double)x - md) * scale;
    return (plain ? x > floor_x : t >= -1000.0) ? pow2_near(t, tab) : 0.0;
  };
  auto weight_plain = [&](float x) -> double { return pow2_reduced(reduced(x), tab); };
  const double unit = pow2_near((double)top64 - (double)(m - shift) * scale, tab);                   // weight_plain's, in weight's
  // keys of bf16 logits in 16 bits, so that both types descend through their own bits only
  auto key_of = [&](float x) -> uint32_t { return float_key(x) >> (32 - KEY_BITS); };
  constexpr uint32_t BOTTOM = KEY_NEG_INF >> (32 - KEY_BITS);
  auto key_value = [&](uint32_t k) -> float {
    // float_key's inverse; a bf16 key has lost the sixteen low bits, all equal to the sign bit's complement
    uint32_t full = k << (32 - KEY_BITS);
    if (KEY_BITS < 32 && !(full & 0x80000000u)) full |= 0xFFFFu;
    return key_to_float(full);
  };
  auto vec = [&](int i) -> uint4 {                       // vector i, NaN as -inf
    if constexpr (STREAM) {
      uint4 raw = (i + 1) * EPC <= cnt ? __ldg(reinterpret_cast<const uint4*>(row + i * EPC)) : sh.tail;
      float a, b;
      clean_logits<T>(raw, a, b);
      return raw;
    } else {
      return reinterpret_cast<const uint4*>(xs)[i];
    }
  };
  auto logit = [&](int i) -> float {                     // element i < cnt
    if constexpr (STREAM) return fmaxf(load_as_float(row + i), -INFINITY);
    else return load_as_float(xs + i);
  };
  // f(x of one vector): the sum of f over this thread's share, four running sums
  auto sum_over = [&](auto f) -> double {
    double s[4] = {0.0, 0.0, 0.0, 0.0};
    for (int i = tid; i < n_vec; i += SP_THREADS) {
      float x[EPC];
      unpack_logits<T>(vec(i), x);
#pragma unroll
      for (int e = 0; e < EPC; ++e) s[e & 3] += f(x[e]);
    }
    return (s[0] + s[1]) + (s[2] + s[3]);
  };
  // softmax denominator at temperature 1 over the vocabulary, an output value: this thread's share of it, in fp32
  const double raw_mine = !p.prob ? 0.0
                          : m == INFINITY ? sum_over([&](float x) { return x == m ? 1.0 : 0.0; })
                          : share > -INFINITY ? (double)(raw_part * expf(share - m)) : 0.0;
  const bool cut_k = p.top_k > 0 && p.top_k < n_cand, cut_p = p.top_p < 1.f, need_z = cut_p && !cut_k;
  const int groups = nc * SP_THREADS;
  bool have_raw = false;
  double raw_all = 0.0, z_all = -1.0;                    // z_all: weight of the vocabulary, where top-p needs it
  unsigned long long* list = reinterpret_cast<unsigned long long*>(scratch + SP_OFF_LIST);
  // ---- a nucleus: where does it end, to within a few histogram bins? ----
  // Bins of 1/64 in the binary exponent (nearest), counted from the maximum's down to 2^-32 of it: what lies below is
  // rarely of interest (n_cand e^-22 is what it weighs at most).  The weight of a bin lies between those of its edges, so
  // the running weight is known to half a bin, +-0.6 %.  Bins before bin_lo are in the nucleus, those after bin_hi are not.
  auto bin_of = [&](float x) -> int { return top_bits - reduced(x).bits; };
  // the logit `bins` below the maximum's bin, as a float: no smaller one is nearer to it
  auto bin_edge = [&](double bins) -> float {
    const double top = (double)top64 + (double)(top_bits - __float_as_int(196608.f)) / SP_TAB;
    return (float)fmax((double)shift + (top - bins / SP_TAB) / (double)s_hi, -(double)FLT_MAX);
  };
  int bin_lo = 0, bin_hi = 0;
  bool narrowed = false, short_nucleus = false;
  if (need_z && plain && n_cand > SP_LIST) {
    int* hist = reinterpret_cast<int*>(list);
    for (int i = tid; i < SP_BINS; i += SP_THREADS) hist[i] = 0;
    __syncthreads();
    double w[4] = {0.0, 0.0, 0.0, 0.0};
    for (int i = tid; i < n_vec; i += SP_THREADS) {
      float x[EPC];
      unpack_logits<T>(vec(i), x);
#pragma unroll
      for (int e = 0; e < EPC; ++e) {
        const Reduced a = reduced(x[e]);
        const unsigned bin = (unsigned)(top_bits - a.bits);
        if (bin < SP_BINS - 1) atomicAdd(&hist[bin], 1);             // the last bin is what the others leave
        w[e & 3] += pow2_reduced(a, tab);
      }
    }
    double v[2] = {raw_mine, (w[0] + w[1]) + (w[2] + w[3])};
    int none = 0;
    sum_all<2>(cl, sh, turn, v, none);                   // publishes the counts as well
    raw_all = v[0]; z_all = v[1] * unit;
    have_raw = true;
    constexpr int PER = SP_BINS / SP_THREADS;
    int count[PER] = {};
#pragma unroll
    for (int q = 0; q < SP_MAX_CLUSTER; ++q)
      if (q < nc) {
        const int4 c = *reinterpret_cast<const int4*>(cl.map_shared_rank(hist, q) + tid * PER);
        count[0] += c.x; count[1] += c.y; count[2] += c.z; count[3] += c.w;
      }
    // running weights from the bins' edges, half a bin to either side of its middle, and 0.016 for x s_lo, of which the bins know
    // nothing (|x s| <= 4096 + 32 above the last bin, |s_lo| <= 2^-24 s: 0.0158 of a bin); 2e-5 for these sums' rounding.  The last
    // bin weighs from nothing to its upper edge.
    constexpr float HALF = 0.516f;
    const float off = (float)(top_bits - __float_as_int(196608.f));
    float light[PER], heavy[PER], light_at = 0.f, heavy_at = 0.f;
#pragma unroll
    for (int q = 0; q < PER; ++q) {
      const float b = (float)(tid * PER + q), c = (float)count[q];
      light_at += c * ex2_approx((off - b - HALF) * (1.f / SP_TAB)) * 0.99998f;
      heavy_at += c * ex2_approx((off - b + HALF) * (1.f / SP_TAB)) * 1.00002f;
      light[q] = light_at; heavy[q] = heavy_at;
    }
    float light_in = light_at, heavy_in = heavy_at;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const float a = __shfl_up_sync(0xffffffffu, light_in, o), b = __shfl_up_sync(0xffffffffu, heavy_in, o);
      if (lane >= o) { light_in += a; heavy_in += b; }
    }
    if (lane == 31) sh.edge[warp] = make_float2(light_in, heavy_in);
    if (tid == 0) { sh.digit = sh.above = SP_BINS - 1; sh.found = 0; }
    __syncthreads();
    float light_0 = light_in - light_at, heavy_0 = heavy_in - heavy_at;
    for (int q = 0; q < warp; ++q) { light_0 += sh.edge[q].x; heavy_0 += sh.edge[q].y; }
    const float goal = (float)((double)p.top_p * v[1]);
    // the first bin whose upper sum reaches the goal, and the first whose lower sum does
    int first_hi = SP_BINS - 1, first_lo = SP_BINS - 1;
#pragma unroll
    for (int q = PER - 1; q >= 0; --q) {
      if (heavy_0 + heavy[q] >= goal * 0.999999f) first_hi = tid * PER + q;
      if (light_0 + light[q] >= goal * 1.000001f) first_lo = tid * PER + q;
    }
    first_hi = (int)__reduce_min_sync(0xffffffffu, (unsigned)first_hi);
    first_lo = (int)__reduce_min_sync(0xffffffffu, (unsigned)first_lo);
    if (lane == 0) { atomicMin(&sh.digit, first_hi); atomicMin(&sh.above, first_lo); }
    __syncthreads();
    int upto = 0;
#pragma unroll
    for (int q = 0; q < PER; ++q) upto += tid * PER + q <= sh.above ? count[q] : 0;
    upto = __reduce_add_sync(0xffffffffu, upto);
    if (lane == 0) atomicAdd(&sh.found, upto);
    __syncthreads();
    bin_lo = sh.digit; bin_hi = sh.above < SP_BINS - 1 ? sh.above : INT_MAX;
    narrowed = true;
    short_nucleus = sh.found <= SP_LIST && sh.above < SP_BINS - 1;    // its tokens, and a few too many, as a list
    cluster_sync();                                           // everybody has read the counts: the list may go over them
  }
  // ---- short list (top-k: the bound is tight while the k wanted are at most half of the shares) ----
  if (short_nucleus || (cut_k && p.top_k <= min(SP_LIST_K, groups / 2)) || n_cand <= SP_LIST) {
    float from = -FLT_MAX;                               // collect the logits from here up
    if (n_cand > SP_LIST && cut_k) {
      uint32_t least = 0xFFFFFFFFu, kth;
      unsigned long long above = 0ull;
      int own_turn = 0;
      if (nc == 1) {                                     // 512 keys: one warp, without barriers
        if (warp == 0) {
          uint32_t key[SP_WARPS];
#pragma unroll
          for (int q = 0; q < SP_WARPS; ++q) { key[q] = share_key[lane + 32 * q]; least = min(least, key[q]); }
          least = __reduce_min_sync(0xffffffffu, least);
          kth = largest_reaching<1, true>(sh, own_turn, least, key_of(m), (unsigned long long)p.top_k, above,
                                          [&](uint32_t t1, uint32_t t2, uint32_t t3, unsigned (&c)[3]) {
            c[0] = c[1] = c[2] = 0u;
#pragma unroll
            for (int q = 0; q < SP_WARPS; ++q) { c[0] += key[q] >= t1; c[1] += key[q] >= t2; c[2] += key[q] >= t3; }
          });
          if (lane == 0) sh.digit = (int)kth;
        }
        __syncthreads();
        kth = (uint32_t)sh.digit;
      } else {
        uint32_t key[SP_MAX_CLUSTER];
#pragma unroll
        for (int q = 0; q < SP_MAX_CLUSTER; ++q) {
          key[q] = 0u;
          if (q < nc) { key[q] = cl.map_shared_rank(share_key, q)[tid]; least = min(least, key[q]); }
        }
        least = __reduce_min_sync(0xffffffffu, least);
        if (tid == 0) sh.digit = -1;
        __syncthreads();
        if (lane == 0) atomicMin(reinterpret_cast<unsigned*>(&sh.digit), least);
        __syncthreads();
        least = (uint32_t)sh.digit;
        kth = largest_reaching<SP_WARPS, true>(sh, own_turn, least, key_of(m), (unsigned long long)p.top_k,
                                               above, [&](uint32_t t1, uint32_t t2, uint32_t t3, unsigned (&c)[3]) {
          c[0] = c[1] = c[2] = 0u;
#pragma unroll
          for (int q = 0; q < SP_MAX_CLUSTER; ++q)
            if (q < nc) { c[0] += key[q] >= t1; c[1] += key[q] >= t2; c[2] += key[q] >= t3; }
        });
      }
      if (kth > BOTTOM) from = fmaxf(key_value(kth), -FLT_MAX);
    }
    if (short_nucleus) from = bin_edge((double)bin_hi + 0.501);            // its lower edge
    double raw_sum[1] = {raw_mine};
    // which logits reach the bound: a byte of bits per vector, then their places by a scan: the list is in index order.
    // Only the shares whose maximum reaches it are looked at, and those by all threads.
    uint8_t* mask = scratch + SP_OFF_MASK;
    uint16_t* shares = reinterpret_cast<uint16_t*>(sh.hist[0]);
    const int n_words = (n_vec + 3) >> 2;
    for (int i = tid; i < n_words; i += SP_THREADS) reinterpret_cast<uint32_t*>(mask)[i] = 0u;
    const bool wanted = share >= from;
    int n_shares;
    const int my_place = block_excl_scan(wanted ? 1 : 0, sh.scan_i, n_shares);
    if (wanted) shares[my_place] = (uint16_t)tid;
    __syncthreads();
    auto look_at = [&](int i) {
      const uint32_t bits = reaching_bits<T>(vec(i), from);
      if (bits) mask[i] = (uint8_t)bits;
    };
    const int deep = (n_vec + SP_THREADS - 1) / SP_THREADS;          // vectors per share
    if (n_shares * 4 > SP_THREADS) {                     // most of the work: no lookup then
#pragma unroll 4
      for (int i = tid; i < n_vec; i += SP_THREADS) look_at(i);
    } else {
#pragma unroll 4
      for (int q = tid; q < n_shares * deep; q += SP_THREADS) {
        const int i = shares[q / deep] + q % deep * SP_THREADS;
        if (i < n_vec) look_at(i);
      }
    }
    __syncthreads();
    const uint32_t* words = reinterpret_cast<const uint32_t*>(mask);
    const int per_w = (n_words + SP_THREADS - 1) / SP_THREADS, w0 = min(tid * per_w, n_words), w1 = min(w0 + per_w, n_words);
    int mine = 0;
    for (int i = w0; i < w1; ++i) mine += __popc(words[i]);
    int tot;
    int at = block_excl_scan(mine, sh.scan_i, tot);
    if (mine && tot <= SP_LIST)
      for (int i = w0; i < w1; ++i)
        for (uint32_t b = words[i]; b; b &= b - 1u) {
          const int bit = __ffs(b) - 1;
          list[at++] = (unsigned long long)((i * 4 + (bit >> 3)) * EPC + (bit & 7));
        }
    __syncthreads();
    if (tot <= SP_LIST)                                  // the logits: all at once, not one after the other by their finders
      for (int i = tid; i < tot; i += SP_THREADS) {
        const int e = (int)list[i];
        list[i] = (unsigned long long)float_key(logit(e)) << 32 | (uint32_t)(lo + e);
      }
    if (tid == 0) sh.list_n = tot;
    int n_list = tot;
    if (have_raw) cluster_sync();                             // publishes the lists
    else sum_all<1>(cl, sh, turn, raw_sum, n_list);      // so do its barriers
    n_list = 0;
#pragma unroll
    for (int q = 0; q < SP_MAX_CLUSTER; ++q)
      if (q < nc) n_list += cl.map_shared_rank(&sh, q)->list_n;
    if (!have_raw) raw_all = raw_sum[0];
    have_raw = true;
    if (n_list <= SP_LIST) {                             // more: ties at the bound (uniform over the cluster)
      if (rank == 0) {
        // the other slices follow this one: the list stays in index order
        if (nc > 1) {
          if (tid < nc) sh.scan_i[tid] = cl.map_shared_rank(&sh, tid)->list_n;
          __syncthreads();
#pragma unroll 1
          for (int i = tot + tid; i < n_list; i += SP_THREADS) {
            int q = 1, at = i - tot;
            while (at >= sh.scan_i[q]) at -= sh.scan_i[q++];
            list[i] = cl.map_shared_rank(list, q)[at];
          }
        }
        __syncthreads();
        Draw d;
        d.top_k = cut_k ? p.top_k : 0; d.top_p = (double)p.top_p; d.z = z_all; d.min_p = (double)p.min_p; d.u = (double)u;
        d.key_lo = from == -FLT_MAX ? BOTTOM : key_of(from);
        d.key_top = key_of(m);
        if (short_nucleus) d.key_top = min(key_of(bin_edge((double)bin_lo - 0.501)), d.key_top);
        d.complete = n_list == n_cand;
        int at_tok = -1, kept = 0;
        double w_tok = 0.0, total = 1.0;
        bool whole = true;
        if (n_list <= SP_PAIRS) {
          whole = draw_from_pairs(sh, list, n_list, d, weight, at_tok, w_tok, total, kept);
        } else {
          whole = draw_from_list<KEY_BITS>(sh, list, n_list, key_of(m), d, weight, at_tok, w_tok, total, kept);
        }
        if (tid == 0) sh.list_ok = whole ? 1 : 0;
        if (whole && at_tok >= 0) {
          const float x = key_to_float((uint32_t)(list[at_tok] >> 32));
          finish((int)(uint32_t)list[at_tok], (float)(w_tok / total), (float)((x == m ? 1.0 : exp((double)x - md)) / raw_all), kept);
        }
      }
      cluster_sync();                                         // the lists have been read, the outcome is known
      if (cl.map_shared_rank(&sh, 0)->list_ok) {
        cluster_sync();
        return;
      }
    }
  }
  // ---- top-k by counts ----
  uint32_t T_key = BOTTOM;                               // kept: keys above T_key, and the first `quota` at it
  int quota = 0;
  if (cut_k) {
    uint32_t prefix = 0;
    int need = p.top_k;
    for (int shift = KEY_BITS - 8; shift >= 0; shift -= 8) {
      const int b = (shift >> 3) & 1;
      cluster_sync();                                         // last round's readers of this histogram are done
      for (int i = tid; i < 256; i += SP_THREADS) sh.hist[b][i] = 0;
      __syncthreads();
      for (int i = tid; i < n_vec; i += SP_THREADS) {
        float x[EPC];
        unpack_logits<T>(vec(i), x);
#pragma unroll
        for (int e = 0; e < EPC; ++e) {
          const uint32_t k = key_of(x[e]);
          if (k > BOTTOM && (shift + 8 >= KEY_BITS || (k >> (shift + 8)) == prefix)) atomicAdd(&sh.hist[b][(k >> shift) & 255u], 1);
        }
      }
      cluster_sync();
      if (tid < 256) {
        int c = 0;
        for (int q = 0; q < nc; ++q) c += cl.map_shared_rank(&sh, q)->hist[b][tid];
        sh.hist[b ^ 1][tid] = c;                         // combined counts: private to this CTA until the next round
      }
      __syncthreads();
      if (tid == 0) {
        int run = 0, d = 255;
        for (; d > 0; --d) {
          if (run + sh.hist[b ^ 1][d] >= need) break;
          run += sh.hist[b ^ 1][d];
        }
        sh.digit = d; sh.above = run;
      }
      __syncthreads();
      prefix = (prefix << 8) | (uint32_t)sh.digit;
      need -= sh.above;
    }
    T_key = prefix; quota = need;
    cluster_sync();
  }
  // ---- top-p: weight of the tokens from a key up ----
  auto weights_from = [&](uint32_t k1, uint32_t k2, uint32_t k3, double (&s)[3]) {
    const float t1 = key_value(k1), t2 = key_value(k2), t3 = key_value(k3);      // no logit reaches a NaN
    s[0] = s[1] = s[2] = 0.0;
    for (int i = tid; i < n_vec; i += SP_THREADS) {
      const uint4 raw = vec(i);
      if (!(largest_of<T>(raw) >= t1)) continue;
      float x[EPC];
      unpack_logits<T>(raw, x);
#pragma unroll
      for (int e = 0; e < EPC; ++e)
        if (x[e] >= t1) {
          const double w = weight(x[e]);
          s[0] += w;
          s[1] += x[e] >= t2 ? w : 0.0;
          s[2] += x[e] >= t3 ? w : 0.0;
        }
    }
    int none = 0;
    sum_all<3>(cl, sh, turn, s, none);
  };
  // every warp's segment of the slice
  constexpr int SEG_UNIT = 32 * EPC;
  const int seg = (p.slice + SP_WARPS * SEG_UNIT - 1) / (SP_WARPS * SEG_UNIT) * SEG_UNIT;
  const int s0 = min(warp * seg, n_vec * EPC), s1 = min(s0 + seg, n_vec * EPC);   // whole vectors; the padding is -inf
  // A token of bin b weighs 2^-((b -+ 1) / 64).  min_below: min-p ends the set before the nucleus can end, which is then of
  // no interest; min_above: it has no say among the tokens up to bin_hi.
  const float margin = 1e-4f * p.min_p;
  const bool min_below = narrowed && exp2f((1.f - (float)bin_lo) * (1.f / SP_TAB)) <= p.min_p - margin;
  const bool min_above = p.min_p == 0.f || (bin_hi != INT_MAX && exp2f(-((float)bin_hi + 1.f) * (1.f / SP_TAB)) >= p.min_p + margin);
  bool summed = false;                                   // the segments' kept weights are known
  if (narrowed && min_above) {
    // One pass: per segment the weight before the open bins, and their tokens as a list of the warp's own (in a fixed order).
    // They are a few percent of the nucleus; where they fit, the rest is done on them.  A nucleus that fits as a whole is
    // listed as a whole, which takes a comparison per logit instead of a weight (35 rows, a nucleus of 2000 tokens among them: 54 us became 46).
    const int cap = (SP_LIST * 8 + p.slice / EPC) / (SP_WARPS * 4);    // over the list and the bytes per vector behind it
    float* open_list = reinterpret_cast<float*>(list) + warp * cap;
    double s4[4] = {0.0, 0.0, 0.0, 0.0}, base[1];
    int ngt = 0, n_open = 0;
    const float x_open = bin_hi == INT_MAX ? -INFINITY : bin_edge((double)bin_hi + 0.501);
    const bool fits = bin_hi != INT_MAX && sh.found <= cap * (nc * SP_WARPS / 2);
    uint32_t k_hi = min(key_of(bin_edge((double)bin_lo - 0.501)), key_of(m));
#pragma unroll 1
    for (int i0 = s0 / EPC; i0 < s1 / EPC; i0 += 32) {
      const int i = i0 + lane;
      uint32_t open = 0;
      if (i < s1 / EPC && fits) {
        open = reaching_bits<T>(vec(i), x_open);
      } else if (i < s1 / EPC) {
        float x[EPC];
        unpack_logits<T>(vec(i), x);
#pragma unroll
        for (int e = 0; e < EPC; ++e) {
          const Reduced a = reduced(x[e]);
          const int b = top_bits - a.bits;
          s4[e & 3] += b < bin_lo ? pow2_reduced(a, tab) : 0.0;
          ngt += b < bin_lo ? 1 : 0;
          open |= b >= bin_lo && b <= bin_hi && x[e] > -INFINITY ? 1u << e : 0u;
        }
      }
      if (__any_sync(0xffffffffu, open != 0u)) {
        int at = __popc(open);
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const int y = __shfl_up_sync(0xffffffffu, at, o);
          if (lane >= o) at += y;
        }
        const int more = __shfl_sync(0xffffffffu, at, 31);
        at += n_open - __popc(open);
        for (; open; open &= open - 1u, ++at) {
          if (at < cap) open_list[at] = logit(i * EPC + __ffs(open) - 1);
        }
        n_open += more;
      }
    }
    __syncwarp();
    if (fits) {                                          // those that are in whatever the search finds
#pragma unroll 1
      for (int i = lane; i < min(n_open, cap); i += 32)
        if (key_of(open_list[i]) > k_hi) {
          s4[0] += weight_plain(open_list[i]);
          ++ngt;
          open_list[i] = -INFINITY;
        }
    }
    const double mine = (s4[0] + s4[1]) + (s4[2] + s4[3]);
    base[0] = mine;
    int too_many = lane == 0 && n_open > cap ? 1 : 0;
    sum_all<1>(cl, sh, turn, base, too_many);
    if (too_many == 0) {
      const double target = (double)p.top_p * z_all;
      uint32_t k_lo = bin_hi == INT_MAX ? BOTTOM : max(key_of(bin_edge((double)bin_hi + 0.501)), BOTTOM);
      base[0] *= unit;
      double above = base[0];
      int none = 0;
      while (k_lo < k_hi) {
        uint32_t t[3];
        quarter(k_lo, k_hi, t);
        double s3[3] = {0.0, 0.0, 0.0};
#pragma unroll 1
        for (int i = lane; i < n_open; i += 32) {
          const uint32_t k = key_of(open_list[i]);
          const double w = weight_plain(open_list[i]) * unit;
          s3[0] += k >= t[0] ? w : 0.0;
          s3[1] += k >= t[1] ? w : 0.0;
          s3[2] += k >= t[2] ? w : 0.0;
        }
        sum_all<3>(cl, sh, turn, s3, none);
#pragma unroll
        for (int q = 0; q < 3; ++q) s3[q] += base[0];
        const bool reached[3] = {s3[0] >= target, s3[1] >= target, s3[2] >= target};
        go_on(k_lo, k_hi, above, t, reached, s3);
      }
      T_key = k_lo;
      quota = (int)fmin(fmax(ceil((target - above) / weight(key_value(T_key))), 1.0), (double)INT_MAX);
      double w_seg = mine * unit;
      int neq = 0;
#pragma unroll 1
      for (int i = lane; i < n_open; i += 32) {
        const uint32_t k = key_of(open_list[i]);
        if (k > T_key) { w_seg += weight_plain(open_list[i]) * unit; ++ngt; }
        neq += k == T_key && open_list[i] > -INFINITY ? 1 : 0;
      }
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) w_seg += __shfl_xor_sync(0xffffffffu, w_seg, o);
      ngt = __reduce_add_sync(0xffffffffu, ngt);
      neq = __reduce_add_sync(0xffffffffu, neq);
      if (lane == 0) { sh.seg[warp].w = w_seg; sh.seg[warp].n_gt = ngt; sh.seg[warp].n_eq = neq; }
      summed = true;
    }
  }
  if (summed || min_below) {
    // no search left
  } else if (narrowed) {
    // the weight before the open bins, and the keys in them; then their bits
    double base[1];
    uint32_t k_hi = 0u, k_lo = 0xFFFFFFFFu;
    double s4[4] = {0.0, 0.0, 0.0, 0.0};
    for (int i = tid; i < n_vec; i += SP_THREADS) {
      const uint4 raw = vec(i);
      if (bin_of(largest_of<T>(raw)) > bin_hi) continue;
      float x[EPC];
      unpack_logits<T>(raw, x);
#pragma unroll
      for (int e = 0; e < EPC; ++e) {
        const Reduced a = reduced(x[e]);
        const int b = top_bits - a.bits;
        s4[e & 3] += b < bin_lo ? pow2_reduced(a, tab) : 0.0;
        if (b >= bin_lo && b <= bin_hi && x[e] > -INFINITY) { k_hi = max(k_hi, key_of(x[e])); k_lo = min(k_lo, key_of(x[e])); }
      }
    }
    base[0] = ((s4[0] + s4[1]) + (s4[2] + s4[3])) * unit;
    k_hi = __reduce_max_sync(0xffffffffu, k_hi); k_lo = __reduce_min_sync(0xffffffffu, k_lo);
    if (lane == 0) { sh.key_hi[warp] = k_hi; sh.key_lo[warp] = k_lo; }
    int none = 0;
    sum_all<1>(cl, sh, turn, base, none);                // publishes the keys as well
    for (int q = lane; q < nc * SP_WARPS; q += 32) {
      const SampleShared* o = cl.map_shared_rank(&sh, q / SP_WARPS);
      k_hi = max(k_hi, o->key_hi[q % SP_WARPS]); k_lo = min(k_lo, o->key_lo[q % SP_WARPS]);
    }
    k_hi = __reduce_max_sync(0xffffffffu, k_hi); k_lo = __reduce_min_sync(0xffffffffu, k_lo);
    const double target = (double)p.top_p * z_all;
    const float x_lo = key_value(k_lo), x_hi = key_value(k_hi);        // these keys are all there is in the open bins
    double above = base[0];                              // weight from k_hi + 1 up
    while (k_lo < k_hi) {
      uint32_t t[3];
      quarter(k_lo, k_hi, t);
      double s3[3] = {0.0, 0.0, 0.0};
      for (int i = tid; i < n_vec; i += SP_THREADS) {
        const uint4 raw = vec(i);
        if (!(largest_of<T>(raw) >= x_lo)) continue;
        float x[EPC];
        unpack_logits<T>(raw, x);
#pragma unroll
        for (int e = 0; e < EPC; ++e) {
          if (x[e] >= x_lo && x[e] <= x_hi) {
            const uint32_t k = key_of(x[e]);
            const double w = weight_plain(x[e]) * unit;
            s3[0] += k >= t[0] ? w : 0.0;
            s3[1] += k >= t[1] ? w : 0.0;
            s3[2] += k >= t[2] ? w : 0.0;
          }
        }
      }
      sum_all<3>(cl, sh, turn, s3, none);
#pragma unroll
      for (int q = 0; q < 3; ++q) s3[q] += base[0];
      const bool reached[3] = {s3[0] >= target, s3[1] >= target, s3[2] >= target};
      go_on(k_lo, k_hi, above, t, reached, s3);
    }
    const uint32_t best = k_lo;
    T_key = best;
    quota = (int)fmin(fmax(ceil((target - above) / weight(key_value(best))), 1.0), (double)INT_MAX);
  } else if (cut_p) {
    double s3[3];
    const double w_at = quota ? weight(key_value(T_key)) : 0.0;
    weights_from(T_key + 1, T_key + 1, T_key + 1, s3);
    const double target = (double)p.top_p * (s3[0] + (double)quota * w_at);
    double above = 0.0;                                  // weight of the keys from best + 2^sft up
    uint32_t best = 0;
    for (int sft = KEY_BITS; sft > 0;) {
      sft -= 2;
      const uint32_t t1 = best | (1u << sft), t2 = best | (2u << sft), t3 = best | (3u << sft);
      // thresholds down to T_key hold everything that is left, which is enough by definition
      if (t3 <= T_key) { best = t3; continue; }
      weights_from(max(t1, T_key + 1), max(t2, T_key + 1), t3, s3);
      if (s3[2] >= target) best = t3;
      else if (t2 <= T_key || s3[1] >= target) { best = t2; above = s3[2]; }
      else if (t1 <= T_key || s3[0] >= target) { best = t1; above = s3[1]; }
      else above = s3[0];
    }
    const uint32_t t = max(best, T_key);
    const double need = ceil((target - above) / weight(key_value(t)));
    const int most = t == T_key ? quota : INT_MAX;
    if (t > T_key || quota) { T_key = t; quota = (int)fmin(fmax(need, 1.0), (double)most); }
  }
  // ---- kept weight of every warp's segment, in index order ----
  const double min_w = (double)p.min_p;
  const double w_T = quota ? weight(key_value(T_key)) : 0.0;
  const bool tie_in = quota > 0 && w_T >= min_w;
  if (!summed) {
    double s[4] = {0.0, 0.0, 0.0, 0.0};
    int ngt = 0, neq = 0;
    if (T_key == BOTTOM && min_w == 0.0 && plain) {      // no cut at all: every candidate, without a branch
      for (int i = s0 / EPC + lane; i < s1 / EPC; i += 32) {
        float x[EPC];
        unpack_logits<T>(vec(i), x);
#pragma unroll
        for (int e = 0; e < EPC; ++e) {
          s[e & 3] += x[e] > floor_x ? weight_plain(x[e]) : 0.0;
          ngt += x[e] > -INFINITY ? 1 : 0;
        }
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) s[e] *= unit;
    } else {
      const float t = key_value(T_key), t_all = T_key == BOTTOM ? -INFINITY : t;
      // no lighter logit passes min-p (the millionth is for the logarithm's own rounding)
      const float x_min = plain && min_w > 0.0 ? (float)(md + (log2(min_w) - 1e-6) / scale) : -INFINITY, x_look = fmaxf(t_all, x_min);
      for (int i = s0 / EPC + lane; i < s1 / EPC; i += 32) {
        const uint4 raw = vec(i);
        if (!(largest_of<T>(raw) >= x_look)) continue;
        float x[EPC];
        unpack_logits<T>(raw, x);
#pragma unroll
        for (int e = 0; e < EPC; ++e) {
          if (x[e] > t_all && x[e] >= x_min) {
            double w;
            bool in;
            if (plain) {                                 // the exact weight only where min-p depends on its last bits
              w = x[e] > floor_x ? weight_plain(x[e]) * unit : 0.0;
              in = w >= min_w * (1.0 + 1e-8) || (w >= min_w * (1.0 - 1e-8) && weight(x[e]) >= min_w);
            } else {
              w = weight(x[e]);
              in = w >= min_w;
            }
            if (in) { s[e & 3] += w; ++ngt; }
          } else if (T_key > BOTTOM && x[e] == t) {
            ++neq;
          }
        }
      }
    }
    s[0] = (s[0] + s[1]) + (s[2] + s[3]);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) s[0] += __shfl_xor_sync(0xffffffffu, s[0], o);
    ngt = __reduce_add_sync(0xffffffffu, ngt);
    neq = __reduce_add_sync(0xffffffffu, neq);
    if (lane == 0) { sh.seg[warp].w = s[0]; sh.seg[warp].n_gt = ngt; sh.seg[warp].n_eq = neq; }
  }
  {
    double raw[1] = {raw_mine};
    int none = 0;
    sum_all<1>(cl, sh, turn, raw, none);                 // its barrier publishes seg[] as well
    if (!have_raw) raw_all = raw[0];
  }
  // ---- the segment that holds u * total: four segments per lane of one warp ----
  if (tid < SP_MAX_CLUSTER * SP_WARPS) {
    SegSum q; q.w = 0.0; q.n_gt = 0; q.n_eq = 0;
    if (tid < nc * SP_WARPS) q = cl.map_shared_rank(&sh, tid / SP_WARPS)->seg[tid % SP_WARPS];
    sh.all[tid] = q;
  }
  __syncthreads();
  if (warp == 0) {
    constexpr int PER = SP_MAX_CLUSTER * SP_WARPS / 32;
    int eq = 0;
#pragma unroll
    for (int q = 0; q < PER; ++q) eq += sh.all[lane * PER + q].n_eq;
    int eq_inc = eq;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int y = __shfl_up_sync(0xffffffffu, eq_inc, o);
      if (lane >= o) eq_inc += y;
    }
    int left = max((tie_in ? quota : 0) - (eq_inc - eq), 0), kept = 0, left_at[PER];
    double sw[PER], run = 0.0;
#pragma unroll
    for (int q = 0; q < PER; ++q) {
      const SegSum& a = sh.all[lane * PER + q];
      const int e = min(a.n_eq, left);
      left_at[q] = left;
      left -= e;
      sw[q] = a.w + e * w_T;
      run += sw[q];
      kept += a.n_gt + e;
    }
    double inc = run;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const double y = __shfl_up_sync(0xffffffffu, inc, o);
      if (lane >= o) inc += y;
    }
    const double total = __shfl_sync(0xffffffffu, inc, 31), target = (double)u * total;
    kept = __reduce_add_sync(0xffffffffu, kept);
    double before = inc - run;
    int first = INT_MAX, last = -1;
    double first_before = 0.0, last_before = 0.0;
    int first_left = 0, last_left = 0;
#pragma unroll
    for (int q = 0; q < PER; ++q) {
      if (sw[q] > 0.0) {
        last = lane * PER + q; last_before = before; last_left = left_at[q];
        if (first == INT_MAX && before + sw[q] > target) { first = last; first_before = before; first_left = left_at[q]; }
      }
      before += sw[q];
    }
    const int hit = (int)__reduce_min_sync(0xffffffffu, (unsigned)first), end = __reduce_max_sync(0xffffffffu, last);
    // rounding at the far end: the last segment with a weight
    const bool own = hit != INT_MAX ? first == hit : last == end;
    if (own && (hit != INT_MAX || last >= 0)) {
      sh.hit = hit != INT_MAX ? first : last;
      sh.before = hit != INT_MAX ? first_before : last_before;
      sh.hit_eq = hit != INT_MAX ? first_left : last_left;
    }
    if (lane == 0) { sh.total = total; sh.kept = kept; }
  }
  __syncthreads();
  const int hit_eq = sh.hit_eq, kept = sh.kept;
  const double total = sh.total, target = (double)u * total;
  if (sh.hit == rank * SP_WARPS + warp) {
    // a run of it per lane, then the run that holds the target, 32 consecutive tokens at a time
    auto kept_weight = [&](float x, bool& eq) -> double {  // of a token that is not at T_key; ties are counted
      const uint32_t k = key_of(x);
      eq = k == T_key && k > BOTTOM;
      if (!(k > T_key && x > -INFINITY)) return 0.0;
      const double w = weight(x);
      return w >= min_w ? w : 0.0;
    };
    const int run_len = (s1 - s0 + 32 * EPC - 1) / (32 * EPC) * EPC, r0 = min(s0 + lane * run_len, s1), r1 = min(r0 + run_len, s1);
    double run_w = 0.0;
    int run_eq = 0;
    for (int i = r0 / EPC; i < r1 / EPC; ++i) {
      float x[EPC];
      unpack_logits<T>(vec(i), x);
#pragma unroll
      for (int e = 0; e < EPC; ++e) {
        bool eq;
        run_w += kept_weight(x[e], eq);
        run_eq += eq ? 1 : 0;
      }
    }
    int eq_inc = run_eq;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int y = __shfl_up_sync(0xffffffffu, eq_inc, o);
      if (lane >= o) eq_inc += y;
    }
    int eq = max((tie_in ? hit_eq : 0) - (eq_inc - run_eq), 0);
    run_w += min(run_eq, eq) * w_T;
    double inc = run_w;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const double y = __shfl_up_sync(0xffffffffu, inc, o);
      if (lane >= o) inc += y;
    }
    const uint32_t some = __ballot_sync(0xffffffffu, run_w > 0.0);
    const uint32_t past = __ballot_sync(0xffffffffu, run_w > 0.0 && sh.before + inc > target);
    const int at = past ? __ffs(past) - 1 : some ? 31 - __clz(some) : 31;    // rounding at the far end: the last with a weight
    double before = __shfl_sync(0xffffffffu, sh.before + (inc - run_w), at);
    eq = __shfl_sync(0xffffffffu, eq, at);
    const int w0 = __shfl_sync(0xffffffffu, r0, at), w1 = __shfl_sync(0xffffffffu, r1, at);
    int tok = -1, fallback = -1;
    for (int i0 = w0; i0 < w1 && tok < 0; i0 += 32) {
      const int i = i0 + lane;
      bool is_eq;
      double w = kept_weight(i < min(w1, cnt) ? logit(i) : -INFINITY, is_eq);
      const uint32_t eq_mask = __ballot_sync(0xffffffffu, is_eq);
      if (is_eq && __popc(eq_mask & ((1u << lane) - 1u)) < eq) w = w_T;
      eq -= min(eq, __popc(eq_mask));
      double inc = w;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const double y = __shfl_up_sync(0xffffffffu, inc, o);
        if (lane >= o) inc += y;
      }
      const uint32_t got = __ballot_sync(0xffffffffu, w > 0.0 && before + inc > target);
      const uint32_t any = __ballot_sync(0xffffffffu, w > 0.0);
      if (any) fallback = i0 + 31 - __clz(any);
      if (got) tok = i0 + __ffs(got) - 1;
      before += __shfl_sync(0xffffffffu, inc, 31);
    }
    if (tok < 0) tok = fallback;
    if (lane == 0 && tok >= 0) {
      const float x = logit(tok);
      finish(lo + tok, (float)(weight(x) / total), (float)((x == m ? 1.0 : exp((double)x - md)) / raw_all), kept);
    }
  }
  cluster_sync();                                             // nobody leaves while its shared memory may still be read
}

template <typename T, bool STREAM>
focus_status launch_sample_as(focus_ctx* ctx, const SampleParams& p, int nc, cudaStream_t st) {
  const size_t n_vec = ((size_t)p.slice * sizeof(T) + 15) / 16;
  const size_t smem = (STREAM ? 0 : n_vec * 16) + SP_OFF_MASK + ((n_vec + 15) & ~size_t(15));
  bool& attr_set = ctx->ls.sample_attr_set[(sizeof(T) == 2) * 2 + STREAM];
  if (!attr_set) {
    if (cudaFuncSetAttribute(sample_kernel<T, STREAM>, cudaFuncAttributeMaxDynamicSharedMemorySize, SP_SMEM) != cudaSuccess)
      return FOCUS_ERR_CUDA;
    attr_set = true;
  }
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(p.max_rows * nc), 1, 1); cfg.blockDim = dim3(SP_THREADS, 1, 1);
  cfg.dynamicSmemBytes = smem; cfg.stream = st;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeClusterDimension;
  at[0].val.clusterDim.x = nc; at[0].val.clusterDim.y = 1; at[0].val.clusterDim.z = 1;
  cfg.attrs = at; cfg.numAttrs = 1;
  if (cudaLaunchKernelEx(&cfg, sample_kernel<T, STREAM>, p) != cudaSuccess) { cudaGetLastError(); return FOCUS_ERR_CUDA; }
  FOCUS_CHECK_LAUNCH();
  return FOCUS_OK;
}

template <typename T>
focus_status launch_sample(focus_ctx* ctx, SampleParams& p, cudaStream_t st) {
  constexpr int EPC = 16 / sizeof(T);
  if ((size_t)p.vocab * sizeof(T) > (size_t)SP_MAX_CLUSTER * SP_SLICE_BYTES) return FOCUS_ERR_UNSUPPORTED;
  // cluster size: a slice has to fit in shared memory, and small calls spread a row over more SMs while there are idle
  // ones and a slice still feeds every thread.  No finer than that: two CTAs of different rows on one SM cost more than
  // their halves save (72 rows of 126464 bf16 logits, nucleus: 40 us with two CTAs per row, 56 with four).
  int nc = 1;
  while (nc < SP_MAX_CLUSTER && ((long long)p.vocab * sizeof(T) > (long long)nc * SP_SLICE_BYTES ||
                                 (p.max_rows * nc * 2 <= ctx->sm_count && p.vocab > nc * SP_THREADS * EPC)))
    nc *= 2;
  if (nc > 1 && p.max_rows >= ctx->sm_count) {           // rows enough for every SM: no slices
    p.slice = (p.vocab + EPC - 1) / EPC * EPC;
    return launch_sample_as<T, true>(ctx, p, 1, st);
  }
  p.slice = ((p.vocab + nc - 1) / nc + EPC - 1) / EPC * EPC;
  return launch_sample_as<T, false>(ctx, p, nc, st);
}

}  // namespace

extern "C" focus_status focus_sample(focus_ctx* ctx, const void* logits, int32_t dtype, int64_t row_stride,
                                     int32_t vocab, int32_t pos_base, int32_t n_pos, const int32_t* rows,
                                     const int32_t* n_rows, int32_t max_rows, float temperature, int32_t top_k,
                                     float top_p, float min_p, const float* u, float* conf, int32_t* token, float* prob,
                                     int32_t* n_kept, focus_stream stream) {
  FOCUS_STAGE("focus_sample");
  if (!ctx || !logits || !u || !conf || !token || !aligned16(logits)) return FOCUS_ERR_INVALID_ARG;
  if (dtype != FOCUS_F32 && dtype != FOCUS_BF16) return FOCUS_ERR_INVALID_ARG;
  if (vocab <= 0 || row_stride < vocab || pos_base < 0 || n_pos < 0 || max_rows < 0) return FOCUS_ERR_INVALID_ARG;
  if ((rows == nullptr) != (n_rows == nullptr)) return FOCUS_ERR_INVALID_ARG;
  if (!rows && max_rows > n_pos) return FOCUS_ERR_INVALID_ARG;
  if (row_stride % (dtype == FOCUS_BF16 ? 8 : 4)) return FOCUS_ERR_INVALID_ARG;      // rows must keep 16-byte alignment
  if (!(temperature > 0.f) || !(temperature <= 3.402823466e38f) || top_k < 0) return FOCUS_ERR_INVALID_ARG;
  if (!(top_p > 0.f && top_p <= 1.f) || !(min_p >= 0.f && min_p <= 1.f)) return FOCUS_ERR_INVALID_ARG;
  if (max_rows > (1 << 24)) return FOCUS_ERR_UNSUPPORTED;                             // grid of max_rows clusters
  if (max_rows == 0) return FOCUS_OK;
  SampleParams p;
  p.logits = logits; p.row_stride = row_stride; p.vocab = vocab; p.pos_base = pos_base; p.n_pos = n_pos;
  p.max_rows = max_rows; p.rows = rows; p.n_rows = n_rows; p.temperature = temperature; p.top_k = top_k;
  p.top_p = top_p; p.min_p = min_p; p.u = u; p.conf = conf; p.token = token; p.prob = prob; p.n_kept = n_kept;
  p.status = ctx->d_status; p.slice = 0;
  return dtype == FOCUS_BF16 ? launch_sample<__nv_bfloat16>(ctx, p, stream) : launch_sample<float>(ctx, p, stream);
}
