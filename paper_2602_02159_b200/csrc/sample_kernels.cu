// focus_sample: one token per listed position, drawn from its logits row with temperature, top-k, top-p and min-p by a
// given uniform number.
//
// A row belongs to one thread-block cluster.  Each CTA loads its contiguous slice of the vocabulary into shared memory
// (the logits cross HBM once) and every later pass runs there; the CTAs exchange a few numbers per pass through
// distributed shared memory.  Weights and sums are fp64: a token is decided by comparing two sums over the vocabulary,
// and in fp32 those sums are off by as much as a rare token weighs.  Sums run in a fixed order (lanes, warps, CTAs), so
// the answer does not depend on timing or on the number of rows.
//
// The kept set is a prefix of the descending order.  Two ways to it:
//   short list  (up to 2048 tokens: top-k to 1024, most nuclei): the k-th largest of the maxima of the threads' shares is a
//               lower bound of the k-th largest logit -- that many logits reach it, and few more do.  The logits from there
//               up are collected in index order and cut by one CTA, which has them in registers.  One pass for the maxima,
//               one for the list (with the sums over the vocabulary that prob and top-p need).
//   any length  (no cut, min-p alone, long top-k, flat nuclei): the key T of the last kept logit, by counts (top-k: 8-bit
//               digits of a radix descent) and by weight (top-p: two bits of the key per pass); (T, how many of the tokens
//               at T) says all about the set.  Then the kept weight per warp segment in index order, the segment that
//               holds u * total, and its walk.
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
// scratch behind the slice: list (before it: the cluster's thread maxima) | one byte per 16-byte vector | thread maxima
constexpr int SP_OFF_MASK = SP_LIST * 8, SP_OFF_MAX = SP_OFF_MASK + 14 * 1024, SP_SCRATCH = SP_OFF_MAX + SP_THREADS * 4;
constexpr int SP_TAB = 1024;                             // entries of the table of powers
constexpr uint32_t KEY_NEG_INF = 0x007FFFFFu;            // float_key(-inf); NaN is below it
static_assert(SP_MAX_CLUSTER * SP_THREADS * 4 <= SP_OFF_MASK && SP_SLICE_BYTES / 16 + 4 <= SP_OFF_MAX - SP_OFF_MASK, "scratch");

struct SegSum {            // one warp's contiguous segment of the row
  double w;                // kept weight above the threshold key
  int n_gt, n_eq;          // tokens above it / at it
};

struct SampleShared {
  double tab[SP_TAB];      // 2^(i / SP_TAB)
  double dsum[2][SP_WARPS][3];
  int isum[2][SP_WARPS];
  double cta_d[2][3];
  int cta_i[2];
  SegSum seg[SP_WARPS];
  SegSum all[SP_MAX_CLUSTER * SP_WARPS];
  float wmax[SP_WARPS];
  int list_n, list_ok;
  int hist[2][256];
  int scan_i[33];
  double scan[SP_WARPS];
  int digit, above, found;
  // the segment that holds u * total
  int hit, hit_eq, kept;
  double before, total;
};
static_assert(sizeof(SampleShared) <= 15 * 1024 && SP_SLICE_BYTES + SP_SCRATCH + 15 * 1024 <= 227 * 1024, "shared memory");

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
// CTA writes a slot again only after a barrier that its slowest reader has passed.  CTA = true: of this CTA alone.
template <int N, bool CTA = false>
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
  if (CTA || warp == 0) {                                // the warps' sums in a fixed tree
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
  if (CTA) return;
  if (threadIdx.x == 0) {
#pragma unroll
    for (int i = 0; i < N; ++i) sh.cta_d[t][i] = v[i];
    sh.cta_i[t] = cnt;
  }
  cl.sync();
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

// Powers of two in fp64: t = n / 1024 + r, 2^t = 2^(n >> 10) * tab[n & 1023] * 2^r, the last factor by its Taylor
// polynomial (Tang's table-driven scheme, 1989).  |r| <= 2^-11, so the square leaves 7e-12 of a weight, of either sign.
// -1000 <= t <= 0; no branch, so that several run side by side.
__device__ __forceinline__ double pow2_near(double t, const double* tab) {
  const double magic = 6755399441055744.0;               // 1.5 * 2^52: adding it leaves the rounded integer in the low bits
  const double tm = fma(t, (double)SP_TAB, magic);
  const int n = __double2loint(tm);
  const double r = fma(tm - magic, -1.0 / SP_TAB, t);
  const double b = tab[n & (SP_TAB - 1)];
  const double w = fma(b, r * fma(r, 0.24022650695910071, 0.69314718055994531), b);   // ln2^2 / 2, ln2
  return __hiloint2double(__double2hiint(w) + ((n >> 10) << 20), __double2loint(w));
}

// The k-th largest (1 <= k <= n) of the keys get(0), get(1), ..., 8-bit digits from the top, BITS of the key in use;
// k becomes its place among the keys equal to it.  Every thread of the block calls it.
template <int BITS, typename Get>
__device__ __forceinline__ uint32_t block_kth(SampleShared& sh, int n, int& k, Get get) {
  uint32_t prefix = 0;
  for (int shift = BITS - 8; shift >= 0; shift -= 8) {
    int* hist = sh.hist[(shift >> 3) & 1];
    for (int i = threadIdx.x; i < 256; i += SP_THREADS) hist[i] = 0;
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += SP_THREADS) {
      const uint32_t q = get(i);
      if (shift + 8 >= BITS || (q >> (shift + 8)) == prefix) atomicAdd(&hist[(q >> shift) & 255u], 1);
    }
    __syncthreads();
    if (threadIdx.x < 32) {                              // digits from the largest down, eight per lane
      const int lane = threadIdx.x;
      int c[8], sum = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) { c[i] = hist[255 - (lane * 8 + i)]; sum += c[i]; }
      int inc = sum;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, inc, o);
        if (lane >= o) inc += y;
      }
      int run = inc - sum;
      if (run < k && inc >= k) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          if (run < k && run + c[i] >= k) { sh.digit = 255 - (lane * 8 + i); sh.above = run; }
          run += c[i];
        }
      }
    }
    __syncthreads();
    prefix = (prefix << 8) | (uint32_t)sh.digit;
    k -= sh.above;
  }
  return prefix;
}

template <typename T>
__global__ void __launch_bounds__(SP_THREADS)
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
  uint8_t* scratch = smem_raw + (size_t)p.slice * sizeof(T);
  float share = -INFINITY;
  int n_cand = 0;
  auto take = [&](uint4 raw, int i) {
    float hi, low;
    clean_logits<T>(raw, hi, low);
    *reinterpret_cast<uint4*>(xs + i) = raw;
    share = fmaxf(share, hi);
    if (low > -INFINITY) {
      n_cand += EPC;
    } else {
      float x[EPC];
      unpack_logits<T>(raw, x);
#pragma unroll
      for (int e = 0; e < EPC; ++e) n_cand += x[e] > -INFINITY ? 1 : 0;
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
    if (i < cnt) {                                       // the one vector that the row ends in
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
      take(make_uint4(w[0], w[1], w[2], w[3]), i);
    }
  }
  for (int i = tid; i < SP_TAB; i += SP_THREADS) {       // 2^(i / 1024) as the product of its binary digits' powers
    const double f[10] = {1.0006771306930664, 1.0013547198921082, 1.0027112750502025, 1.0054299011128027, 1.0108892860517005,
                          1.0218971486541166, 1.0442737824274138, 1.0905077326652577, 1.189207115002721, 1.4142135623730951};
    double v = 1.0;
#pragma unroll
    for (int q = 0; q < 10; ++q) v *= (i >> q & 1) ? f[q] : 1.0;
    sh.tab[i] = v;
  }
  uint32_t* share_key = reinterpret_cast<uint32_t*>(scratch + SP_OFF_MAX);
  share_key[tid] = float_key(share) >> (32 - KEY_BITS);
  float m = share;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
  if (lane == 0) sh.wmax[warp] = m;
  {
    double none[1] = {0.0};
    sum_all<1>(cl, sh, turn, none, n_cand);              // its barriers publish the maxima as well
  }
  for (int q = lane; q < nc * SP_WARPS; q += 32) m = fmaxf(m, cl.map_shared_rank(&sh, q / SP_WARPS)->wmax[q % SP_WARPS]);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
  if (n_cand == 0) {
    if (lead) finish(-1, 0.f, 0.f, 0);
    cl.sync();
    return;
  }
  // ---- weights: 2^((x - m) log2(e) / temperature) ----
  const double scale = 1.4426950408889634 / (double)p.temperature, md = (double)m;
  const float floor_x = (float)fmax(md - 1000.0 / scale, -(double)FLT_MAX);      // lighter ones may count as 2^-1000
  // weights without a branch, where that floor is a logit well below the maximum (not so for an infinite maximum, one whose
  // neighbouring floats are further apart, or a temperature that flattens the type's whole range)
  const double floor_t = ((double)floor_x - md) * scale;
  const bool plain = m < INFINITY && floor_t < -900.0 && floor_t > -1020.0;
  auto weight = [&](float x) -> double {
    if (m == INFINITY) return x == m ? 1.0 : 0.0;
    const double t = ((double)x - md) * scale;
    return t >= -1000.0 ? pow2_near(t, sh.tab) : 0.0;
  };
  auto weight_plain = [&](float x) -> double { return pow2_near(((double)fmaxf(x, floor_x) - md) * scale, sh.tab); };
  // keys of bf16 logits in 16 bits, so that both types descend through their own bits only
  auto key_of = [&](float x) -> uint32_t { return float_key(x) >> (32 - KEY_BITS); };
  constexpr uint32_t BOTTOM = KEY_NEG_INF >> (32 - KEY_BITS);
  auto key_value = [&](uint32_t k) -> float {
    // float_key's inverse; a bf16 key has lost the sixteen low bits, all equal to the sign bit's complement
    uint32_t full = k << (32 - KEY_BITS);
    if (KEY_BITS < 32 && !(full & 0x80000000u)) full |= 0xFFFFu;
    return key_to_float(full);
  };
  const uint4* vecs = reinterpret_cast<const uint4*>(xs);
  // f(x of one vector): the sum of f over this thread's share, four running sums
  auto sum_over = [&](auto f) -> double {
    double s[4] = {0.0, 0.0, 0.0, 0.0};
    for (int i = tid; i < n_vec; i += SP_THREADS) {
      float x[EPC];
      unpack_logits<T>(vecs[i], x);
#pragma unroll
      for (int e = 0; e < EPC; ++e) s[e & 3] += f(x[e]);
    }
    return (s[0] + s[1]) + (s[2] + s[3]);
  };
  const float l2e = 1.4426950408889634f;
  // softmax denominator at temperature 1 over the vocabulary, an output value: fp32 terms
  auto raw_sum = [&]() -> double {
    if (m == INFINITY) return sum_over([&](float x) { return x == m ? 1.0 : 0.0; });
    float s[4] = {0.f, 0.f, 0.f, 0.f};
    for (int i = tid; i < n_vec; i += SP_THREADS) {
      float x[EPC];
      unpack_logits<T>(vecs[i], x);
#pragma unroll
      for (int e = 0; e < EPC; ++e) {
        float y;
        asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"((x[e] - m) * l2e));
        s[e & 3] += y;
      }
    }
    return (double)((s[0] + s[1]) + (s[2] + s[3]));
  };
  const bool cut_k = p.top_k > 0 && p.top_k < n_cand, cut_p = p.top_p < 1.f, need_z = cut_p && !cut_k;
  const int groups = nc * SP_THREADS, want = cut_k ? p.top_k : min(SP_LIST_K, groups / 2);
  bool have_raw = false;
  double raw_all = 0.0;
  // ---- short list (the bound is tight while the k wanted are at most half of the shares) ----
  if (((cut_k || cut_p) && want <= min(SP_LIST_K, groups / 2)) || n_cand <= SP_LIST) {
    float from = -FLT_MAX;                               // collect the logits from here up
    if (n_cand > SP_LIST) {
      uint32_t* keys = reinterpret_cast<uint32_t*>(scratch);
#pragma unroll
      for (int q = 0; q < SP_MAX_CLUSTER; ++q)
        if (q < nc) keys[q * SP_THREADS + tid] = cl.map_shared_rank(share_key, q)[tid];
      int k = want;
      const uint32_t kth = block_kth<KEY_BITS>(sh, groups, k, [&](int i) { return keys[i]; });
      if (kth > BOTTOM) from = fmaxf(key_value(kth), -FLT_MAX);
    }
    double v[2] = {0.0, 0.0};
    if (p.prob) v[0] = raw_sum();
    if (need_z) v[1] = plain ? sum_over(weight_plain) : sum_over([&](float x) { return x > -INFINITY ? weight(x) : 0.0; });
    // which logits reach the bound: a byte of bits per vector, then their places by a scan: the list is in index order
    uint8_t* mask = scratch + SP_OFF_MASK;
    const int n_words = (n_vec + 3) >> 2;
    for (int i = tid; i < n_words * 4; i += SP_THREADS) {
      uint32_t bits = 0;
      if (i < n_vec) {
        const uint4 raw = vecs[i];
        if (largest_of<T>(raw) >= from) {
          float x[EPC];
          unpack_logits<T>(raw, x);
#pragma unroll
          for (int e = 0; e < EPC; ++e) bits |= x[e] >= from ? 1u << e : 0u;
        }
      }
      mask[i] = (uint8_t)bits;
    }
    __syncthreads();                                     // also: nobody reads the keys any more
    unsigned long long* list = reinterpret_cast<unsigned long long*>(scratch);
    const uint32_t* words = reinterpret_cast<const uint32_t*>(mask);
    const int per_w = (n_words + SP_THREADS - 1) / SP_THREADS, w0 = min(tid * per_w, n_words), w1 = min(w0 + per_w, n_words);
    int mine = 0;
    for (int i = w0; i < w1; ++i) mine += __popc(words[i]);
    int tot;
    int at = block_excl_scan(mine, sh.scan_i, tot);
    if (mine && tot <= SP_LIST)
      for (int i = w0; i < w1; ++i)
        for (uint32_t b = words[i]; b; b &= b - 1u) {
          const int bit = __ffs(b) - 1, e = (i * 4 + (bit >> 3)) * EPC + (bit & 7);
          list[at++] = ((unsigned long long)float_key(load_as_float(xs + e)) << 32) | (uint32_t)(lo + e);
        }
    if (tid == 0) sh.list_n = tot;
    int n_list = tot;
    sum_all<2>(cl, sh, turn, v, n_list);                 // publishes the lists as well
    n_list = 0;
#pragma unroll
    for (int q = 0; q < SP_MAX_CLUSTER; ++q)
      if (q < nc) n_list += cl.map_shared_rank(&sh, q)->list_n;
    raw_all = v[0];
    have_raw = true;
    if (n_list <= SP_LIST) {                             // more: ties at the bound (uniform over the cluster)
      if (rank == 0) {
        int have = tot;
        for (int q = 1; q < nc; ++q) {                   // the other slices follow this one: the list stays in index order
          const int c = cl.map_shared_rank(&sh, q)->list_n;
          const unsigned long long* src = reinterpret_cast<const unsigned long long*>(cl.map_shared_rank(scratch, q));
          for (int i = tid; i < c; i += SP_THREADS) list[have + i] = src[i];
          have += c;
        }
        __syncthreads();
        // this thread's tokens: neighbours in index order
        uint32_t key[SP_PER];
        double w[SP_PER];
        bool in[SP_PER];
#pragma unroll
        for (int q = 0; q < SP_PER; ++q) {
          const int i = tid * SP_PER + q;
          in[q] = i < n_list;
          const uint32_t full = in[q] ? (uint32_t)(list[i] >> 32) : 0u;
          key[q] = full >> (32 - KEY_BITS);
          w[q] = in[q] ? weight(key_to_float(full)) : 0.0;
        }
        // keeps of the tokens at key t the first `quota` in index order, drops those below t
        auto cut_at = [&](uint32_t t, int quota) {
          int eq = 0, all;
#pragma unroll
          for (int q = 0; q < SP_PER; ++q) eq += in[q] && key[q] == t ? 1 : 0;
          int before = block_excl_scan(eq, sh.scan_i, all);
#pragma unroll
          for (int q = 0; q < SP_PER; ++q) {
            const bool at_t = in[q] && key[q] == t;
            in[q] = in[q] && (key[q] > t || (at_t && before < quota));
            before += at_t ? 1 : 0;
          }
        };
        if (cut_k) {
          int k = p.top_k;
          const uint32_t t = block_kth<KEY_BITS>(sh, n_list, k, [&](int i) { return (uint32_t)(list[i] >> 32) >> (32 - KEY_BITS); });
          cut_at(t, k);
        }
        bool whole = true;
        int dummy = 0, own_turn = 0;                     // sums of this CTA: not in step with the cluster's
        if (cut_p) {
          double a[1] = {0.0};
#pragma unroll
          for (int q = 0; q < SP_PER; ++q) a[0] += in[q] ? w[q] : 0.0;
          sum_all<1, true>(cl, sh, own_turn, a, dummy);
          const double target = (double)p.top_p * (need_z ? v[1] : a[0]);
          // a nucleus that reaches beyond the list is found the long way
          whole = a[0] >= target || n_list == n_cand;
          if (whole && a[0] >= target) {
            // the largest key whose tokens, with all above, hold the target: two bits per step below the bits all share
            const uint32_t k_hi = key_of(m), k_lo = from == -FLT_MAX ? BOTTOM : key_of(from);
            const int vary = (33 - __clz(k_hi ^ k_lo)) & ~1;      // bits that differ, made even: k_lo <= every key <= k_hi
            uint32_t best = vary >= 32 ? 0u : k_hi >> vary << vary;
            double above = 0.0;                          // weight of the keys from best + 2^sft up
            for (int sft = vary; sft > 0;) {
              sft -= 2;
              const uint32_t t1 = best | (1u << sft), t2 = best | (2u << sft), t3 = best | (3u << sft);
              double s3[3] = {0.0, 0.0, 0.0};
#pragma unroll
              for (int q = 0; q < SP_PER; ++q) {
                const double wq = in[q] ? w[q] : 0.0;
                s3[0] += key[q] >= t1 ? wq : 0.0;
                s3[1] += key[q] >= t2 ? wq : 0.0;
                s3[2] += key[q] >= t3 ? wq : 0.0;
              }
              sum_all<3, true>(cl, sh, own_turn, s3, dummy);
              if (s3[2] >= target) best = t3;
              else if (s3[1] >= target) { best = t2; above = s3[2]; }
              else if (s3[0] >= target) { best = t1; above = s3[1]; }
              else above = s3[0];
            }
            const double need = ceil((target - above) / weight(key_value(best)));
            cut_at(best, (int)fmin(fmax(need, 1.0), (double)SP_LIST));
          }
        }
        if (whole && p.min_p > 0.f) {
#pragma unroll
          for (int q = 0; q < SP_PER; ++q) in[q] = in[q] && w[q] >= (double)p.min_p;
        }
        if (tid == 0) { sh.list_ok = whole ? 1 : 0; sh.found = SP_LIST; }
        if (whole) {
          // running sums of the kept weights in index order; the first one above u * total
          double mine_w = 0.0, cum[SP_PER];
          int kept = 0;
#pragma unroll
          for (int q = 0; q < SP_PER; ++q) {
            mine_w += in[q] ? w[q] : 0.0;
            cum[q] = mine_w;
            kept += in[q] ? 1 : 0;
          }
          double inc = mine_w;
#pragma unroll
          for (int o = 1; o < 32; o <<= 1) {
            const double y = __shfl_up_sync(0xffffffffu, inc, o);
            if (lane >= o) inc += y;
          }
          if (lane == 31) sh.scan[warp] = inc;
          kept = __reduce_add_sync(0xffffffffu, kept);
          if (lane == 0) sh.isum[0][warp] = kept;
          __syncthreads();
          double base = 0.0, total = 0.0;
          kept = 0;
#pragma unroll
          for (int q = 0; q < SP_WARPS; ++q) {
            if (q == warp) base = total;
            total += sh.scan[q];
            kept += sh.isum[0][q];
          }
          base += inc - mine_w;
          const double target = (double)u * total;
          int first = SP_LIST, last = -1;                // last kept token with a weight: where rounding leaves none above
#pragma unroll
          for (int q = SP_PER - 1; q >= 0; --q)
            if (in[q] && w[q] > 0.0) {
              if (base + cum[q] > target) first = tid * SP_PER + q;
              if (last < 0) last = tid * SP_PER + q;
            }
          first = (int)__reduce_min_sync(0xffffffffu, (unsigned)first);
          last = __reduce_max_sync(0xffffffffu, last);
          if (lane == 0) { sh.isum[1][warp] = last; if (first < SP_LIST) atomicMin(&sh.found, first); }
          __syncthreads();
          if (tid == 0) {
            int f = sh.found;
            if (f >= SP_LIST)
              for (int q = 0; q < SP_WARPS; ++q) f = f >= SP_LIST ? sh.isum[1][q] : max(f, sh.isum[1][q]);
            const float x = key_to_float((uint32_t)(list[f] >> 32));
            finish((int)(uint32_t)list[f], (float)(weight(x) / total),
                   (float)((x == m ? 1.0 : exp((double)x - md)) / raw_all), kept);
          }
        }
      }
      cl.sync();                                         // the lists have been read, the outcome is known
      if (cl.map_shared_rank(&sh, 0)->list_ok) {
        cl.sync();
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
      cl.sync();                                         // last round's readers of this histogram are done
      for (int i = tid; i < 256; i += SP_THREADS) sh.hist[b][i] = 0;
      __syncthreads();
      for (int i = tid; i < n_vec; i += SP_THREADS) {
        float x[EPC];
        unpack_logits<T>(vecs[i], x);
#pragma unroll
        for (int e = 0; e < EPC; ++e) {
          const uint32_t k = key_of(x[e]);
          if (k > BOTTOM && (shift + 8 >= KEY_BITS || (k >> (shift + 8)) == prefix)) atomicAdd(&sh.hist[b][(k >> shift) & 255u], 1);
        }
      }
      cl.sync();
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
    cl.sync();
  }
  // ---- top-p: weight of the tokens from a key up ----
  auto weights_from = [&](uint32_t k1, uint32_t k2, uint32_t k3, double (&s)[3]) {
    const float t1 = key_value(k1), t2 = key_value(k2), t3 = key_value(k3);      // no logit reaches a NaN
    s[0] = s[1] = s[2] = 0.0;
    for (int i = tid; i < n_vec; i += SP_THREADS) {
      const uint4 raw = vecs[i];
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
  if (cut_p) {
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
  constexpr int SEG_UNIT = 32 * EPC;
  const int seg = (p.slice + SP_WARPS * SEG_UNIT - 1) / (SP_WARPS * SEG_UNIT) * SEG_UNIT;
  const int s0 = min(warp * seg, n_vec * EPC), s1 = min(s0 + seg, n_vec * EPC);   // whole vectors; the padding is -inf
  {
    double s[2] = {0.0, 0.0};
    int ngt = 0, neq = 0;
    if (T_key == BOTTOM && min_w == 0.0 && plain) {      // no cut at all: every candidate, without a branch
      for (int i = s0 / EPC + lane; i < s1 / EPC; i += 32) {
        float x[EPC];
        unpack_logits<T>(vecs[i], x);
#pragma unroll
        for (int e = 0; e < EPC; ++e) {
          s[e & 1] += weight_plain(x[e]);
          ngt += x[e] > -INFINITY ? 1 : 0;
        }
      }
    } else {
      const float t = key_value(T_key), t_all = T_key == BOTTOM ? -INFINITY : t;
      for (int i = s0 / EPC + lane; i < s1 / EPC; i += 32) {
        const uint4 raw = vecs[i];
        if (!(largest_of<T>(raw) >= t_all)) continue;
        float x[EPC];
        unpack_logits<T>(raw, x);
#pragma unroll
        for (int e = 0; e < EPC; ++e) {
          if (x[e] > t_all) {
            const double w = weight(x[e]);
            if (w >= min_w) { s[0] += w; ++ngt; }
          } else if (T_key > BOTTOM && x[e] == t) {
            ++neq;
          }
        }
      }
    }
    s[0] += s[1];
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) s[0] += __shfl_xor_sync(0xffffffffu, s[0], o);
    ngt = __reduce_add_sync(0xffffffffu, ngt);
    neq = __reduce_add_sync(0xffffffffu, neq);
    if (lane == 0) { sh.seg[warp].w = s[0]; sh.seg[warp].n_gt = ngt; sh.seg[warp].n_eq = neq; }
  }
  {
    double raw[1] = {p.prob && !have_raw ? raw_sum() : 0.0};
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
    // walk of the segment, 32 consecutive tokens at a time
    double before = sh.before;
    int eq = tie_in ? hit_eq : 0, tok = -1, fallback = -1;
    for (int i0 = s0; i0 < s1 && tok < 0; i0 += 32) {
      const int i = i0 + lane;
      const float x = i < s1 ? load_as_float(xs + i) : -INFINITY;
      const uint32_t k = key_of(x);
      const bool is_eq = k == T_key && k > BOTTOM;
      const uint32_t eq_mask = __ballot_sync(0xffffffffu, is_eq);
      double w = 0.0;
      bool in = false;
      if (k > T_key && x > -INFINITY) { w = weight(x); in = w >= min_w; }
      else if (is_eq) { in = __popc(eq_mask & ((1u << lane) - 1u)) < eq; w = w_T; }
      if (!in) w = 0.0;
      eq -= min(eq, __popc(eq_mask));
      double inc = w;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const double y = __shfl_up_sync(0xffffffffu, inc, o);
        if (lane >= o) inc += y;
      }
      const uint32_t got = __ballot_sync(0xffffffffu, in && before + inc > target);
      const uint32_t any = __ballot_sync(0xffffffffu, in && w > 0.0);
      if (any) fallback = i0 + 31 - __clz(any);
      if (got) tok = i0 + __ffs(got) - 1;
      before += __shfl_sync(0xffffffffu, inc, 31);
    }
    if (tok < 0) tok = fallback;
    if (lane == 0 && tok >= 0) {
      const float x = load_as_float(xs + tok);
      finish(lo + tok, (float)(weight(x) / total), (float)((x == m ? 1.0 : exp((double)x - md)) / raw_all), kept);
    }
  }
  cl.sync();                                             // nobody leaves while its shared memory may still be read
}

template <typename T>
focus_status launch_sample(focus_ctx* ctx, SampleParams& p, cudaStream_t st) {
  constexpr int EPC = 16 / sizeof(T);
  // cluster size: a slice has to fit in shared memory, and small calls spread a row over more SMs while there are idle
  // ones and a slice still feeds every thread
  int nc = 1;
  while (nc < SP_MAX_CLUSTER && ((long long)p.vocab * sizeof(T) > (long long)nc * SP_SLICE_BYTES / 2 ||
                                 (p.max_rows * nc * 2 <= ctx->sm_count && p.vocab > nc * SP_THREADS * EPC)))
    nc *= 2;
  p.slice = ((p.vocab + nc - 1) / nc + EPC - 1) / EPC * EPC;
  if ((size_t)p.slice * sizeof(T) > SP_SLICE_BYTES) return FOCUS_ERR_UNSUPPORTED;
  const size_t smem = (size_t)p.slice * sizeof(T) + SP_SCRATCH;
  bool& attr_set = ctx->ls.sample_attr_set[sizeof(T) == 2];
  if (!attr_set) {
    if (cudaFuncSetAttribute(sample_kernel<T>, cudaFuncAttributeMaxDynamicSharedMemorySize, SP_SLICE_BYTES + SP_SCRATCH) != cudaSuccess)
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
  if (cudaLaunchKernelEx(&cfg, sample_kernel<T>, p) != cudaSuccess) { cudaGetLastError(); return FOCUS_ERR_CUDA; }
  FOCUS_CHECK_LAUNCH();
  return FOCUS_OK;
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
