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
//   short list  (top-k up to 512, or a nucleus that lies within the 512 largest logits): the 512 k maxima of the threads'
//               shares give a lower bound of the k-th largest logit -- that many logits reach it, and few more do --, the
//               logits from there up are collected, sorted and cut by one CTA.  One pass for the maximum, one for the
//               list (with the sums over the vocabulary that prob and top-p need).
//   any length  (no cut, min-p alone, long top-k, flat nuclei): the key T of the last kept logit, by counts (top-k: 8-bit
//               digits of a radix descent) and by weight (top-p: one bit of the key per pass); (T, how many of the tokens
//               at T) says all about the set.  Then the kept weight per warp segment in index order, the segment that
//               holds u * total, and its walk.
#include <cooperative_groups.h>

#include "focus_common.cuh"

namespace cg = cooperative_groups;

namespace {

constexpr int SP_THREADS = 512;
constexpr int SP_WARPS = SP_THREADS / 32;
constexpr int SP_MAX_CLUSTER = 8;
constexpr int SP_SLICE_BYTES = 196 * 1024;               // largest slice of a row per CTA
constexpr int SP_LIST = 1024;                            // most tokens of a short list
constexpr int SP_LIST_K = 512;                           // largest top-k that goes through it; tokens tried for a nucleus
constexpr int SP_SCRATCH = 16 * 1024;                    // thread maxima of a cluster, or two lists
constexpr int SP_TAB = 1024;                             // entries of the table of powers
static_assert(SP_SLICE_BYTES + SP_SCRATCH + 14 * 1024 <= 227 * 1024, "shared memory");
static_assert(SP_MAX_CLUSTER * SP_THREADS * 4 <= SP_SCRATCH && 2 * SP_LIST * 8 <= SP_SCRATCH, "scratch");
constexpr uint32_t KEY_NEG_INF = 0x007FFFFFu;            // float_key(-inf); NaN is below it

struct SegSum {            // one warp's contiguous segment of the row
  double w;                // kept weight above the threshold key
  int n_gt, n_eq;          // tokens above it / at it
};

struct SampleShared {
  double tab[SP_TAB];      // 2^(i / SP_TAB)
  double dsum[2][SP_WARPS];
  int isum[2][SP_WARPS];
  double cta_d[2];
  int cta_i[2];
  SegSum seg[SP_WARPS];
  SegSum all[SP_MAX_CLUSTER * SP_WARPS];
  float wmax[SP_WARPS];
  double raw, z;           // this CTA's sums over the vocabulary (temperature 1 / given temperature)
  int list_n, list_ok;
  int hist[2][256];
  int digit, above;
  double scan[SP_WARPS + 1];
  int found, n_kept;
  // the segment that holds u * total
  int hit, hit_eq, kept;
  double before, total;
};

static_assert(sizeof(SampleShared) <= 14 * 1024, "shared memory");

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

// Sum over the cluster, the same in every thread.  Two slots in turn: one cluster barrier per call is enough, since a
// CTA writes a slot again only after a barrier that its slowest reader has passed.
__device__ __forceinline__ double cluster_sum(cg::cluster_group& cl, SampleShared& sh, int& turn, double v, int& cnt) {
  const int t = turn & 1, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  ++turn;
  int n = cnt;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    v += __shfl_xor_sync(0xffffffffu, v, o);
    n += __shfl_xor_sync(0xffffffffu, n, o);
  }
  if (lane == 0) { sh.dsum[t][warp] = v; sh.isum[t][warp] = n; }
  __syncthreads();
  if (threadIdx.x == 0) {
    double s = 0.0;
    int c = 0;
    for (int w = 0; w < SP_WARPS; ++w) { s += sh.dsum[t][w]; c += sh.isum[t][w]; }
    sh.cta_d[t] = s; sh.cta_i[t] = c;
  }
  cl.sync();
  double s = 0.0;
  int c = 0;
  for (unsigned r = 0; r < cl.num_blocks(); ++r) {
    const SampleShared* p = cl.map_shared_rank(&sh, r);
    s += p->cta_d[t]; c += p->cta_i[t];
  }
  cnt = c;
  return s;
}

template <typename T> __device__ __forceinline__ T nan_logit();
template <> __device__ __forceinline__ float nan_logit<float>() { return __uint_as_float(0x7FC00000u); }
template <> __device__ __forceinline__ __nv_bfloat16 nan_logit<__nv_bfloat16>() { return __ushort_as_bfloat16(0x7FC0u); }

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

// 2^t for t <= 0 in fp64: t = n / 1024 + r, 2^t = 2^(n >> 10) * tab[n & 1023] * 2^r, the last factor by its Taylor
// polynomial (Tang's table-driven scheme, 1989).  |r| <= 2^-11, so the cubic leaves 6e-16; below 2^-1000 it is zero.
__device__ __forceinline__ double pow2_neg(double t, const double* tab) {
  if (t < -1000.0) return 0.0;
  const double magic = 6755399441055744.0;               // 1.5 * 2^52: adding it leaves the rounded integer in the low bits
  const double tm = fma(t, (double)SP_TAB, magic);
  const int n = __double2loint(tm);
  const double r = fma(tm - magic, -1.0 / SP_TAB, t);
  const double c1 = 0.69314718055994531, c2 = 0.24022650695910071, c3 = 0.055504108664821580;   // ln2^k / k!
  const double q = r * fma(r, fma(r, c3, c2), c1);
  const double b = tab[n & (SP_TAB - 1)];
  const double w = fma(b, q, b);
  return __hiloint2double(__double2hiint(w) + ((n >> 10) << 20), __double2loint(w));
}

// Sorts n2 (a power of two) 64-bit numbers in shared memory, descending; every thread of the block calls it.
__device__ __forceinline__ void block_sort_desc(unsigned long long* v, int n2) {
  for (int k = 2; k <= n2; k <<= 1)
    for (int j = k >> 1; j > 0; j >>= 1) {
      __syncthreads();
      for (int i = threadIdx.x; i < n2 / 2; i += SP_THREADS) {
        const int lo = ((i & ~(j - 1)) << 1) | (i & (j - 1)), hi = lo | j;
        const unsigned long long a = v[lo], b = v[hi];
        if ((a < b) == ((lo & k) == 0)) { v[lo] = b; v[hi] = a; }
      }
    }
  __syncthreads();
}

// Inclusive prefix sums of the n <= SP_LIST numbers get(0), get(1), ... into out, in fixed order; every thread calls it.
template <typename Get>
__device__ __forceinline__ void block_scan_list(SampleShared& sh, double* out, int n, Get get) {
  constexpr int PER = SP_LIST / SP_THREADS;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  double v[PER], run = 0.0;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int at = threadIdx.x * PER + i;
    run += at < n ? get(at) : 0.0;
    v[i] = run;
  }
  double inc = run;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const double y = __shfl_up_sync(0xffffffffu, inc, o);
    if (lane >= o) inc += y;
  }
  __syncthreads();
  if (lane == 31) sh.scan[warp] = inc;
  __syncthreads();
  double before = inc - run;
  for (int w = 0; w < warp; ++w) before += sh.scan[w];
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int at = threadIdx.x * PER + i;
    if (at < n) out[at] = before + v[i];
  }
  __syncthreads();
}

// Key of the k-th largest of n keys in shared memory (1 <= k <= n), 8-bit digits from the top; BITS of the key in use.
template <int BITS>
__device__ __forceinline__ uint32_t block_kth(SampleShared& sh, const uint32_t* key, int n, int k) {
  uint32_t prefix = 0;
  for (int shift = BITS - 8; shift >= 0; shift -= 8) {
    for (int i = threadIdx.x; i < 256; i += SP_THREADS) sh.hist[0][i] = 0;
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += SP_THREADS) {
      const uint32_t q = key[i];
      if (shift + 8 >= BITS || (q >> (shift + 8)) == prefix) atomicAdd(&sh.hist[0][(q >> shift) & 255u], 1);
    }
    __syncthreads();
    if (threadIdx.x < 32) {                              // digits from the largest down, eight per lane
      const int lane = threadIdx.x;
      int c[8], sum = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) { c[i] = sh.hist[0][255 - (lane * 8 + i)]; sum += c[i]; }
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
    __syncthreads();
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
  // ---- the slice, the maxima of the threads' shares ----
  const int lo = min(rank * p.slice, p.vocab), cnt = min(p.slice, p.vocab - lo);
  const T* row = (const T*)p.logits + (long long)(pos - p.pos_base) * p.row_stride + lo;
  uint8_t* scratch = smem_raw + (((size_t)p.slice * sizeof(T) + 15) & ~size_t(15));
  float m = -INFINITY;
  int n_cand = 0;
  auto look = [&](const uint4& raw) {
    float x[EPC];
    unpack_logits<T>(raw, x);
#pragma unroll
    for (int e = 0; e < EPC; ++e) {
      n_cand += x[e] > -INFINITY ? 1 : 0;                // false for NaN
      m = fmaxf(m, x[e]);                                // a NaN is passed over
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
      for (int q = 0; q < U; ++q) { *reinterpret_cast<uint4*>(xs + i + q * STEP) = raw[q]; look(raw[q]); }
    }
    for (; i + EPC <= cnt; i += STEP) {
      const uint4 raw = __ldg(reinterpret_cast<const uint4*>(row + i));
      *reinterpret_cast<uint4*>(xs + i) = raw;
      look(raw);
    }
    // the slice is padded to whole vectors with NaN: later passes need no other bound
    const int tail = cnt / EPC * EPC, end = (cnt + EPC - 1) / EPC * EPC;
    if (tail + tid < end) {
      const T v = tail + tid < cnt ? row[tail + tid] : nan_logit<T>();
      xs[tail + tid] = v;
      const float x = load_as_float(&v);
      if (x > -INFINITY) { m = fmaxf(m, x); ++n_cand; }
    }
  }
  for (int i = tid; i < SP_TAB; i += SP_THREADS) sh.tab[i] = exp2((double)i / SP_TAB);
  const float share = m;                                 // largest logit of this thread's share
  reinterpret_cast<uint32_t*>(scratch)[tid] = float_key(share) >> (32 - KEY_BITS);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
  if (lane == 0) sh.wmax[warp] = m;
  if (tid == 0) sh.list_n = 0;
  (void)cluster_sum(cl, sh, turn, 0.0, n_cand);          // its barriers publish the maxima as well
  if (lane < nc * SP_WARPS) {
    m = -INFINITY;
    for (int q = lane; q < nc * SP_WARPS; q += 32) m = fmaxf(m, cl.map_shared_rank(&sh, q / SP_WARPS)->wmax[q % SP_WARPS]);
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
  if (n_cand == 0) {
    if (lead) finish(-1, 0.f, 0.f, 0);
    cl.sync();
    return;
  }
  const double scale = 1.4426950408889634 / (double)p.temperature, md = (double)m;
  // the maximum itself has weight 1, also where it is +inf (everything else then has none)
  auto weight = [&](float x) -> double { return x == m ? 1.0 : pow2_neg(((double)x - md) * scale, sh.tab); };
  // keys of bf16 logits in 16 bits, so that both types descend through their own bits only
  auto key_of = [&](float x) -> uint32_t { return float_key(x) >> (32 - KEY_BITS); };
  constexpr uint32_t BOTTOM = KEY_NEG_INF >> (32 - KEY_BITS);
  auto key_value = [&](uint32_t k) -> float {
    // float_key's inverse; a bf16 key has lost the sixteen low bits, all equal to the sign bit's complement
    uint32_t full = k << (32 - KEY_BITS);
    if (KEY_BITS < 32 && !(full & 0x80000000u)) full |= 0xFFFFu;
    return key_to_float(full);
  };
  const int n_vec = (cnt + EPC - 1) / EPC;               // vectors of the slice
  auto every = [&](auto f) {                             // f(x, element) over this thread's share
    for (int i = tid; i < n_vec; i += SP_THREADS) {
      float x[EPC];
      unpack_logits<T>(*reinterpret_cast<const uint4*>(xs + i * EPC), x);
#pragma unroll
      for (int e = 0; e < EPC; ++e) f(x[e], i * EPC + e);
    }
  };
  const bool cut_k = p.top_k > 0 && p.top_k < n_cand, cut_p = p.top_p < 1.f;
  const int k_max = cut_k ? p.top_k : n_cand;
  // ---- short list ----
  bool have_raw = false;
  double raw_all = 0.0;
  if ((cut_k && p.top_k <= SP_LIST_K) || (cut_p && !cut_k) || n_cand <= SP_LIST) {
    const int groups = nc * SP_THREADS, want = cut_k ? p.top_k : SP_LIST_K;
    float from = -INFINITY;                              // collect the logits from here up
    if (n_cand > SP_LIST) {
      // a lower bound of the want-th largest logit: the want-th largest of the shares' maxima (groups >= want)
      uint32_t* keys = reinterpret_cast<uint32_t*>(scratch);
      uint32_t mine[SP_MAX_CLUSTER];
#pragma unroll
      for (int q = 0; q < SP_MAX_CLUSTER; ++q)
        if (q < nc) mine[q] = reinterpret_cast<const uint32_t*>(cl.map_shared_rank(scratch, q))[tid];
      cl.sync();                                         // everybody has read: the copies may go over the originals
#pragma unroll
      for (int q = 0; q < SP_MAX_CLUSTER; ++q)
        if (q < nc) keys[q * SP_THREADS + tid] = mine[q];
      __syncthreads();
      const uint32_t kth = block_kth<KEY_BITS>(sh, keys, groups, want);
      from = kth > BOTTOM ? key_value(kth) : -INFINITY;
    }
    unsigned long long* list = reinterpret_cast<unsigned long long*>(scratch);
    const bool need_z = cut_p && !cut_k;
    double z = 0.0;
    float part = 0.f;
    every([&](float x, int i) {
      if (x >= from && x > -INFINITY) {
        const int at = atomicAdd(&sh.list_n, 1);
        if (at < SP_LIST) list[at] = ((unsigned long long)float_key(x) << 32) | (uint32_t)~(lo + i);
      }
      if (p.prob) part += x == m ? 1.f : (x > -INFINITY ? expf(x - m) : 0.f);
      if (need_z && x > -INFINITY) z += weight(x);
    });
    // sums of the CTA, then of the cluster (both in the order of the ranks)
    int dummy = 0;
    raw_all = cluster_sum(cl, sh, turn, (double)part, dummy);     // its barriers publish the lists as well
    have_raw = true;
    double z_all = 0.0;
    if (need_z) { dummy = 0; z_all = cluster_sum(cl, sh, turn, z, dummy); }
    int n = 0;
    for (int q = 0; q < nc; ++q) n += cl.map_shared_rank(&sh, q)->list_n;
    const bool fits = n <= SP_LIST;                                 // more: ties at the bound (uniform over the cluster)
    if (fits) {
      unsigned long long* sorted = list + SP_LIST;
      double* cum = reinterpret_cast<double*>(scratch);  // over the first list, once it has been gathered
      if (rank == 0) {
        int at = 0;
        for (int q = 0; q < nc; ++q) {
          const int c = cl.map_shared_rank(&sh, q)->list_n;
          const unsigned long long* src = reinterpret_cast<const unsigned long long*>(cl.map_shared_rank(scratch, q));
          for (int i = tid; i < c; i += SP_THREADS) sorted[at + i] = src[i];
          at += c;
        }
        int n2 = 32;
        while (n2 < n) n2 <<= 1;
        for (int i = n + tid; i < n2; i += SP_THREADS) sorted[i] = 0ull;
        block_sort_desc(sorted, n2);
        auto listed = [&](int i) -> float { return key_to_float((uint32_t)(sorted[i] >> 32)); };
        if (tid == 0) { sh.found = n; sh.n_kept = 0; }
        block_scan_list(sh, cum, n, [&](int i) { return weight(listed(i)); });
        // n_p: the first prefix that holds top_p of the weight left by top-k; n_m: those of at least min_p
        const int k = min(k_max, n);
        const double target = (double)p.top_p * (need_z ? z_all : cum[k - 1]);
        int below = 0, light = 0;
        for (int i = tid; i < k; i += SP_THREADS) {
          below += cum[i] < target ? 1 : 0;
          light += weight(listed(i)) < (double)p.min_p ? 1 : 0;
        }
        __syncthreads();
        if (below) atomicAdd(&sh.n_kept, below);
        if (light) atomicSub(&sh.found, light);
        __syncthreads();
        const int n_below = sh.n_kept, n_heavy = sh.found - (n - k);
        int kept = cut_p ? min(k, n_below + 1) : k;
        if (p.min_p > 0.f) kept = min(kept, n_heavy);
        kept = max(kept, 1);
        // a nucleus that the list does not reach the end of is found the long way -- unless min-p ends it earlier
        const bool whole = !need_z || n_below < k || n == n_cand || (p.min_p > 0.f && n_heavy < k);
        __syncthreads();
        if (tid == 0) sh.list_ok = whole ? 1 : 0;
        if (whole) {
          // in index order: sort the kept ones by ~index (descending = ascending index), sum again, take the first sum
          // above u * total
          unsigned long long v[SP_LIST / SP_THREADS];
#pragma unroll
          for (int q = 0; q < SP_LIST / SP_THREADS; ++q) {
            const int i = tid + q * SP_THREADS;
            v[q] = i < kept ? (sorted[i] << 32) | (sorted[i] >> 32) : 0ull;
          }
          __syncthreads();
          int k2 = 32;
          while (k2 < kept) k2 <<= 1;
#pragma unroll
          for (int q = 0; q < SP_LIST / SP_THREADS; ++q) {
            const int i = tid + q * SP_THREADS;
            if (i < k2) sorted[i] = v[q];
          }
          block_sort_desc(sorted, k2);
          block_scan_list(sh, cum, kept, [&](int i) { return weight(key_to_float((uint32_t)sorted[i])); });
          const double total = cum[kept - 1], t_u = (double)u * total;
          if (tid == 0) sh.found = kept;
          __syncthreads();
          for (int i = tid; i < kept; i += SP_THREADS)
            if (cum[i] > t_u) atomicMin(&sh.found, i);
          __syncthreads();
          if (tid == 0) {
            int f = sh.found;
            if (f >= kept) {                             // rounding at the far end: the last token with a weight
              f = kept - 1;
              while (f > 0 && weight(key_to_float((uint32_t)sorted[f])) == 0.0) --f;
            }
            const float x = key_to_float((uint32_t)sorted[f]);
            finish((int)~(uint32_t)(sorted[f] >> 32), (float)(weight(x) / total),
                   (float)((x == m ? 1.0 : exp((double)x - (double)m)) / raw_all), kept);
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
      every([&](float x, int) {
        const uint32_t k = key_of(x);
        if (k > BOTTOM && (shift + 8 >= KEY_BITS || (k >> (shift + 8)) == prefix)) atomicAdd(&sh.hist[b][(k >> shift) & 255u], 1);
      });
      cl.sync();
      if (tid < 256) {
        int s = 0;
        for (int q = 0; q < nc; ++q) s += cl.map_shared_rank(&sh, q)->hist[b][tid];
        sh.hist[b ^ 1][tid] = s;                         // combined counts: private to this CTA until the next round
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
  // ---- top-p: weight of the tokens above a key, within the top-k set ----
  auto weight_from = [&](uint32_t k0, int& c) -> double {
    double s = 0.0;
    int n_in = 0;
    every([&](float x, int) {
      const uint32_t k = key_of(x);
      if (k >= k0 && k > BOTTOM) { s += weight(x); ++n_in; }
    });
    c = n_in;
    return cluster_sum(cl, sh, turn, s, c);
  };
  auto key_weight = [&](uint32_t k) -> double { return weight(key_value(k)); };
  if (cut_p) {
    int c;
    const double all = weight_from(T_key + 1, c) + (quota ? (double)quota * key_weight(T_key) : 0.0);
    const double target = (double)p.top_p * all;
    uint32_t best = 0;
    for (int bit = KEY_BITS - 1; bit >= 0; --bit) {
      const uint32_t k = best | (1u << bit);
      if (k <= T_key) { best = k; continue; }            // everything from T_key down is in: enough by definition
      if (weight_from(k, c) >= target) best = k;
    }
    if (best > T_key) {
      // tokens above `best` do not reach the target, those at it do
      int c_gt, c_ge;
      const double w_gt = weight_from(best + 1, c_gt);
      (void)weight_from(best, c_ge);
      const double q = ceil((target - w_gt) / key_weight(best));
      T_key = best;
      quota = (int)fmin(fmax(q, 1.0), (double)(c_ge - c_gt));
    } else if (quota) {
      const double w_gt = weight_from(T_key + 1, c);
      const double q = ceil((target - w_gt) / key_weight(T_key));
      quota = (int)fmin(fmax(q, 1.0), (double)quota);
    }
  }
  // ---- kept weight of every warp's segment, in index order ----
  const double min_w = (double)p.min_p;
  const double w_T = quota ? key_weight(T_key) : 0.0;
  const bool tie_in = quota > 0 && w_T >= min_w;
  const int seg = ((p.slice + SP_WARPS - 1) / SP_WARPS + 31) / 32 * 32;
  const int s0 = min(warp * seg, cnt), s1 = min(s0 + seg, cnt);
  {
    double s = 0.0;
    int ngt = 0, neq = 0;
    for (int i = s0 + lane; i < s1; i += 32) {
      const float x = load_as_float(xs + i);
      const uint32_t k = key_of(x);
      if (k > T_key) {
        const double w = weight(x);
        if (w >= min_w) { s += w; ++ngt; }
      } else if (k == T_key && k > BOTTOM) {
        ++neq;
      }
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      s += __shfl_xor_sync(0xffffffffu, s, o);
      ngt += __shfl_xor_sync(0xffffffffu, ngt, o);
      neq += __shfl_xor_sync(0xffffffffu, neq, o);
    }
    if (lane == 0) { sh.seg[warp].w = s; sh.seg[warp].n_gt = ngt; sh.seg[warp].n_eq = neq; }
  }
  // sum at temperature 1 over the whole vocabulary (an output value, fp32 terms)
  double raw = 0.0;
  if (p.prob && !have_raw) {
    float part = 0.f;
    every([&](float x, int) { part += x == m ? 1.f : (x > -INFINITY ? expf(x - m) : 0.f); });
    raw = part;
  }
  int dummy = 0;
  raw = cluster_sum(cl, sh, turn, raw, dummy);           // its barrier publishes seg[] as well
  if (have_raw) raw = raw_all;
  // ---- the segment that holds u * total ----
  if (tid < nc * SP_WARPS) sh.all[tid] = cl.map_shared_rank(&sh, tid / SP_WARPS)->seg[tid % SP_WARPS];
  __syncthreads();
  if (tid == 0) {
    double total = 0.0;
    int eq_left = tie_in ? quota : 0, kept = 0;
    for (int q = 0; q < nc * SP_WARPS; ++q) {
      const int e = min(sh.all[q].n_eq, eq_left);
      eq_left -= e;
      total += sh.all[q].w + e * w_T;
      kept += sh.all[q].n_gt + e;
    }
    const double target = (double)u * total;
    double run = 0.0, before = 0.0;
    int hit = -1, hit_eq = 0;
    eq_left = tie_in ? quota : 0;
    for (int q = 0; q < nc * SP_WARPS; ++q) {
      const int e = min(sh.all[q].n_eq, eq_left);
      const double sw = sh.all[q].w + e * w_T;
      if (sw > 0.0) { hit = q; hit_eq = eq_left; before = run; }       // so far the last segment with a weight
      if (run + sw > target) break;
      run += sw;
      eq_left -= e;
    }
    sh.hit = hit; sh.hit_eq = hit_eq; sh.before = before; sh.total = total; sh.kept = kept;
  }
  __syncthreads();
  const int hit = sh.hit, hit_eq = sh.hit_eq, kept = sh.kept;
  const double mine_before = sh.before, total = sh.total, target = (double)u * total;
  if (hit == rank * SP_WARPS + warp) {
    // walk of the segment, 32 consecutive tokens at a time
    double before = mine_before;
    int eq = hit_eq, tok = -1, fallback = -1;
    for (int i0 = s0; i0 < s1 && tok < 0; i0 += 32) {
      const int i = i0 + lane;
      float x = -INFINITY;
      if (i < s1) x = load_as_float(xs + i);
      const uint32_t k = i < s1 ? key_of(x) : 0u;
      const bool is_eq = i < s1 && k == T_key && k > BOTTOM;
      const uint32_t eq_mask = __ballot_sync(0xffffffffu, is_eq);
      double w = 0.0;
      bool in = false;
      if (i < s1 && k > T_key) { w = weight(x); in = w >= min_w; }
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
    if (lane == 0) {
      const float x = load_as_float(xs + tok);
      finish(lo + tok, (float)(weight(x) / total), (float)((x == m ? 1.0 : exp((double)x - (double)m)) / raw), kept);
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
  const size_t smem = (((size_t)p.slice * sizeof(T) + 15) & ~size_t(15)) + SP_SCRATCH;
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
