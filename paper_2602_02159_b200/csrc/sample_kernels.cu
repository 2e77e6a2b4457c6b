// focus_sample: one token per listed position, drawn from its logits row with temperature, top-k, top-p and min-p by a
// given uniform number.
//
// A row belongs to one thread-block cluster.  Each CTA loads its contiguous slice of the vocabulary into shared memory
// (the logits cross HBM once) and every later pass runs there; the CTAs exchange a few numbers per pass through
// distributed shared memory.
//   1. maximum and number of candidates (neither NaN nor -inf)
//   2. top-k: the key T of the k-th largest logit, four (bf16: two) 8-bit digits of a radix descent by counts
//   3. top-p: the largest T whose tokens >= T hold the wanted weight, one bit of the key at a time
//   4. kept weight per warp segment in index order, the segment that holds u * total, and its walk
// The kept set is a prefix of the descending order, so (T, how many of the tokens at T) says all about it.
// Weights and sums are fp64: a token is decided by comparing two sums over the vocabulary, and in fp32 those sums are
// off by as much as a rare token weighs.  Sums run in a fixed order (lanes, warps, CTAs), so the answer does not
// depend on timing or on the number of rows.
#include <cooperative_groups.h>

#include "focus_common.cuh"

namespace cg = cooperative_groups;

namespace {

constexpr int SP_THREADS = 512;
constexpr int SP_WARPS = SP_THREADS / 32;
constexpr int SP_MAX_CLUSTER = 8;
constexpr int SP_SLICE_BYTES = 200 * 1024;               // largest slice of a row per CTA
constexpr uint32_t KEY_NEG_INF = 0x007FFFFFu;            // float_key(-inf); NaN is below it

struct SegSum {            // one warp's contiguous segment of the row
  double w;                // kept weight above the threshold key
  int n_gt, n_eq;          // tokens above it / at it
};

struct SampleShared {
  double dsum[2][SP_WARPS];
  int isum[2][SP_WARPS];
  double cta_d[2];
  int cta_i[2];
  SegSum seg[SP_WARPS];
  int hist[2][256];
  int digit, above;
  int winner;
};

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
  // ---- the slice, its maximum ----
  const int lo = min(rank * p.slice, p.vocab), cnt = min(p.slice, p.vocab - lo);
  const T* row = (const T*)p.logits + (long long)(pos - p.pos_base) * p.row_stride + lo;
  float m = -INFINITY;
  int n_cand = 0;
  for (int i = tid * EPC; i + EPC <= cnt; i += SP_THREADS * EPC)
    *reinterpret_cast<uint4*>(xs + i) = __ldg(reinterpret_cast<const uint4*>(row + i));
  for (int i = cnt / EPC * EPC + tid; i < cnt; i += SP_THREADS) xs[i] = row[i];
  __syncthreads();
  for (int i = tid; i < cnt; i += SP_THREADS) {
    const float x = load_as_float(xs + i);
    if (x > -INFINITY) { m = fmaxf(m, x); ++n_cand; }
  }
  // cluster maximum through the key (sums of one-hot digits would be longer): every CTA publishes its own
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
  if (lane == 0) sh.seg[warp].w = m;
  (void)cluster_sum(cl, sh, turn, 0.0, n_cand);          // its barriers publish seg[].w as well
  m = -INFINITY;
  for (int q = 0; q < nc; ++q) {
    const SampleShared* o = cl.map_shared_rank(&sh, q);
    for (int w = 0; w < SP_WARPS; ++w) m = fmaxf(m, (float)o->seg[w].w);
  }
  if (n_cand == 0) {
    if (lead) finish(-1, 0.f, 0.f, 0);
    cl.sync();
    return;
  }
  const double md = (double)m, inv_t = 1.0 / (double)p.temperature;
  auto weight = [&](float x) -> double { return x == m ? 1.0 : exp(((double)x - md) * inv_t); };   // +inf maximum: 1 or 0
  // keys of bf16 logits in 16 bits, so that both types descend through their own bits only
  auto key_of = [&](float x) -> uint32_t { return float_key(x) >> (32 - KEY_BITS); };
  constexpr uint32_t BOTTOM = KEY_NEG_INF >> (32 - KEY_BITS);
  // ---- top-k by counts ----
  uint32_t T_key = BOTTOM;                               // kept: keys above T_key, and the first `quota` at it
  int quota = 0;
  if (p.top_k > 0 && p.top_k < n_cand) {
    uint32_t prefix = 0;
    int need = p.top_k;
    for (int shift = KEY_BITS - 8; shift >= 0; shift -= 8) {
      const int b = (shift >> 3) & 1;
      cl.sync();                                         // last round's readers of this histogram are done
      for (int i = tid; i < 256; i += SP_THREADS) sh.hist[b][i] = 0;
      __syncthreads();
      for (int i = tid; i < cnt; i += SP_THREADS) {
        const uint32_t k = key_of(load_as_float(xs + i));
        if (k > BOTTOM && (shift + 8 >= KEY_BITS || (k >> (shift + 8)) == prefix)) atomicAdd(&sh.hist[b][(k >> shift) & 255u], 1);
      }
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
    c = 0;
    for (int i = tid; i < cnt; i += SP_THREADS) {
      const float x = load_as_float(xs + i);
      const uint32_t k = key_of(x);
      if (k >= k0 && k > BOTTOM) { s += weight(x); ++c; }
    }
    return cluster_sum(cl, sh, turn, s, c);
  };
  auto key_weight = [&](uint32_t k) -> double {
    // float_key's inverse; a bf16 key has lost the sixteen low bits, all equal to the sign bit's complement
    uint32_t full = k << (32 - KEY_BITS);
    if (KEY_BITS < 32 && !(full & 0x80000000u)) full |= 0xFFFFu;
    return weight(key_to_float(full));
  };
  if (p.top_p < 1.f) {
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
    cl.sync();                                           // every reader of seg[] (the maximum) is done
    if (lane == 0) { sh.seg[warp].w = s; sh.seg[warp].n_gt = ngt; sh.seg[warp].n_eq = neq; }
  }
  // sum at temperature 1 over the whole vocabulary (an output value, fp32 terms)
  double raw = 0.0;
  if (p.prob) {
    float part = 0.f;
    for (int i = tid; i < cnt; i += SP_THREADS) {
      const float x = load_as_float(xs + i);
      if (x > -INFINITY) part += x == m ? 1.f : expf(x - m);
    }
    raw = part;
  }
  int dummy = 0;
  raw = cluster_sum(cl, sh, turn, raw, dummy);           // its barrier publishes seg[] as well
  // ---- the segment that holds u * total ----
  double total = 0.0;
  int eq_left = tie_in ? quota : 0, kept = 0;
  for (int q = 0; q < nc; ++q) {
    const SampleShared* o = cl.map_shared_rank(&sh, q);
    for (int w = 0; w < SP_WARPS; ++w) {
      const int e = min(o->seg[w].n_eq, eq_left);
      eq_left -= e;
      total += o->seg[w].w + e * w_T;
      kept += o->seg[w].n_gt + e;
    }
  }
  const double target = (double)u * total;
  double run = 0.0, mine_before = 0.0;
  int hit = -1, hit_eq = 0, last = -1, last_eq = 0;
  double last_before = 0.0;
  eq_left = tie_in ? quota : 0;
  for (int q = 0; q < nc && hit < 0; ++q) {
    const SampleShared* o = cl.map_shared_rank(&sh, q);
    for (int w = 0; w < SP_WARPS; ++w) {
      const int e = min(o->seg[w].n_eq, eq_left);
      const double sw = o->seg[w].w + e * w_T;
      if (sw > 0.0) { last = q * SP_WARPS + w; last_eq = eq_left; last_before = run; }
      if (run + sw > target) { hit = q * SP_WARPS + w; hit_eq = eq_left; mine_before = run; break; }
      run += sw;
      eq_left -= e;
    }
  }
  if (hit < 0) { hit = last; hit_eq = last_eq; mine_before = last_before; }   // rounding at the far end: the last kept token
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
      finish(lo + tok, (float)(weight(x) / total), (float)((x == m ? 1.0 : exp((double)x - md)) / raw), kept);
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
  const size_t smem = (size_t)p.slice * sizeof(T);
  if (smem > SP_SLICE_BYTES) return FOCUS_ERR_UNSUPPORTED;
  bool& attr_set = ctx->ls.sample_attr_set[sizeof(T) == 2];
  if (!attr_set) {
    if (cudaFuncSetAttribute(sample_kernel<T>, cudaFuncAttributeMaxDynamicSharedMemorySize, SP_SLICE_BYTES) != cudaSuccess)
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
