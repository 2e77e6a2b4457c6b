// Attention over an 8-bit K/V cache on the 5th-generation tensor cores (focus_dense_attn_quantized,
// focus_sparse_attn_quantized).  bf16 queries and outputs, head_dim 128 or 64, fp32 accumulation in TMEM.
//
// Mathematics.  With codes ck_j, cv_j and scales sk_j, sv_j of token j, a query row r has the logits (base 2)
//   s_rj = (q_r . ck_j) * sk_j * scale * log2(e)           and   o_r = sum_j 2^(s_rj) sv_j cv_j / sum_j 2^(s_rj).
// The kernel works on the transposed products, S^T = K Q^T and O^T = V^T P^T: a thread then owns one KEY for the softmax,
// so both scales of that key are scalars in its registers.  sk_j joins the logit's scale factor and sv_j the exponent
// (a_rj = s_rj + log2 sv_j, P_rj = 2^(a_rj - ref_r)): one fused multiply-add per logit either way, and the row sum
// takes P_rj / sv_j.  ref_r follows the running maximum of a_rj lazily, so P fits fp16 (below).
// The row sum does not depend on the value scales, but a numerator that P has lost (below 2^-126, where exponentials
// flush to zero) is lost to it too: of two tokens of equal logits the one with sv 2^-89 beside one with 2^45.  ref_r is at
// least 2 below the largest a_rj, so with all value scales within 2^64 of one another that takes a token 2^64 lighter than
// the row's heaviest, which no sum sees.  From the first other scale on a warpgroup's exponentials are the numerators' square
// roots: 2^-252 instead of 2^-126, the whole range of a float's exponents, for three multiplications more per logit (dense,
// 32768 keys, 35 rows, every 50th V row zero: 83 us instead of 74).  Partial sums are joined with two factors each as well.
// Codes enter the products as they are: every int8 and every e4m3 value is an fp16 value.  q enters as fp16 too, scaled
// by a power of two that puts the tile's largest |q| at 2^14..2^15: bf16 has fewer fraction bits, so only elements
// 2^28 times smaller than the largest lose any.  P is rounded to fp16 (relative 2^-11, absolute 2^-27 of the row's
// largest), which is the one rounding between the cache and the output; sums are fp32.
//
// Work split.  CTA = up to 64 stacked query rows of one KV head (the rows of a group's query heads share its K/V) x one
// contiguous range ("split") of that head's key tiles of 128 tokens.  The transposed form costs in proportion to the
// rows there are (N = rows rounded to 16), not to a tile of 128: with the 35 to 72 rows of a denoising step the launch
// is meant to be bound by the bytes of the cache.  The splits of a row tile are joined by the CTA that finishes last.
//
// Warp roles (640 threads):
//   warps 0, 2    producers: K and V tiles as raw codes into two rings (TMA; sink tokens one by one with cp.async)
//   warps 1, 3    tcgen05.mma issuers, one per product: neither has to wait for what only the other needs
//   warps 4..7    K codes -> fp16 in TMEM (lane = key): the A operand of S^T
//   warps 8..11   V codes -> fp16 in TMEM (lane = channel; ldmatrix transposes the bytes): the A operand of O^T
//   warps 12..19  softmax: two warpgroups that take the key tiles in turn, with references, row sums and an O^T of their
//                 own (a tile's chain of latencies, S ready -> P ready, then has two tile periods of time); P^T goes to
//                 shared memory (the B operand of O^T)
// Five kinds of code run side by side, so their loops are kept short (rolled where that costs little): with 24 KB of loop
// bodies the softmax warps waited four to ten cycles for each instruction.
// Expanding the codes into TMEM instead of shared memory halves the shared-memory traffic of a tile: one byte in, one
// byte out per code, no fp16 copy there.
//
// What bounds it, and what it takes (32 heads of 128, int8 unless stated): a key tile's softmax, about 950 ns of a CTA per tile
// of 128 keys and 35 rows, in which the two warpgroups have the SM's exponentials, conversions and shared-memory writes between
// them, and about 14 us around the loop (prologue, first tile, merge of the splits).  Dense, 32768 keys, 35 rows: 74 to
// 77 us, 3.6 TB/s of cache (its bytes alone would take 42).  Dense, 28 query heads on 4 KV heads, e4m3, 16384 keys, 61 rows: 51 us
// (47 to 52, from device to device).  Sparse, 15 blocks of 128, 322 sinks and 512 response tokens, 35 rows: 25.5 us (22.5 to 26).
// Dense, 16384 keys, 256 rows: 147 us (467 TFLOP/s; every row tile of 64 expands the codes again).  attn_tc.cu, from a bf16
// cache of the same shapes on the same device: 89, 37.5, 22 and 80 us.
#include <stddef.h>

#include "attn_tiles.cuh"
#include "tc_common.cuh"

using namespace tc;

namespace {

// registers per thread after the roles split: 64 + 48 + 48 + 160 + 160 = 480 = 5 x the 96 of the launch
constexpr int QN = 64;                         // most query rows per CTA
constexpr int NTH = 640;
constexpr int RING = 5;                        // raw slots per ring (K, V)
constexpr int EARLY = 2;                       // tiles of a dense key set requested ahead of everything else (< RING)
constexpr int SLOT = TN * 128;                 // bytes of a raw tile (head dim 64 fills half)
constexpr int Q_BYTES = QN * 128 * 2;
constexpr int P_BYTES = TN * QN * 2;           // P^T of one tile: [key][row]
// TMEM columns: S of even / odd tiles, O of the two warpgroups, expanded K and V (two tiles each)
constexpr int T_S = 0, T_O = 128, T_K = 256, T_V = 384;
constexpr int MAXT = 256;                      // key tiles of a split whose descriptors are staged
constexpr int OFF_RAW = Q_BYTES + 2 * P_BYTES;
constexpr int OFF_MISC = OFF_RAW + 2 * RING * SLOT;
constexpr int MAX_SPLITS = 32;
constexpr float P_MAX = 46340.f;               // the reference follows the maximum once a numerator exceeds 2^15.5 (fp16 ends at 65504) ...
constexpr float ROOT_P_MAX = 215.2f;           // (where numerators are kept as their square roots)
constexpr float OFFSET = 2.f;                  // ... and is put 2 (log2) below it: P is normal fp16 down to 2^-16 of the row's largest
constexpr float REF_NONE = -1e30f;             // reference of a row that has seen no key
constexpr float SV_MIN = 0x1p-89f;             // smaller value scales count as this (no product is lost: their rows hold zeros, the
                                               // writer's smallest other scale is 2^-80 / 448)
constexpr float SV_LOW = 0x1p-40f, SV_HIGH = 0x1p24f;   // 2^64 apart, around what values of ordinary size have

struct QParams {
  const __nv_bfloat16* Q;
  __nv_bfloat16* O;
  float* lse;
  const int32_t* q_rows;
  const int32_t* n_rows;
  const int32_t* block_idx;
  const int32_t* block_cnt;
  const int32_t* sink_idx;
  const uint8_t* sink_keep;
  const uint8_t* K;
  const uint8_t* V;
  const float* K_scale;
  const float* V_scale;
  float* part_O;               // [cta][row][d] unnormalised partial outputs (n_splits > 1)
  float* part_ml;              // [cta][row][2] reference and sum
  int32_t* counters;           // one arrival counter per (KV head, row tile)
  long long q_stride_row, q_stride_head, kv_stride_tok, kv_stride_head, scale_stride;
  int q_base, n_q, rows_bound, L, M, H, hpg, B, nb, dense, group_stride, max_blocks, n_sink, ns_pad;
  int Hkv, max_tiles, sms, lse_stride, pair, pdl;
  float scale_log2;
  int32_t* status;
};

struct Geo {                                   // a CTA's share of the work; lives in shared memory, each role takes what it needs
  int g, t0, nt, rows, N;                      // KV head, first key tile, key tiles, query rows, rows rounded to 16
  int mt, tile, n_splits, n_mt;                // row tile of the head, of the launch; splits it is cut into; row tiles per head
  int stok_first, stok_n;                      // first sink (list position) in Misc::stok, and how many are there
  TileEnum te;
};
constexpr unsigned FAR = 1u << 31;             // in Misc::pieces: a value scale outside SV_LOW .. SV_HIGH
constexpr int MAX_STOK = 8;                    // sink tiles of a split whose tokens are staged

struct Misc {                                  // behind the tiles in shared memory
  unsigned long long bars[4 * RING + 17];
  alignas(16) float nref[2][QN];               // minus the reference exponent per row (set 1: second warpgroup's own)
  alignas(16) float fac[2][QN];                // rescale factor (its root, see the softmax) / weight per row
  float red[8][64];                            // per softmax warp: column maxima, then row sums
  int orow[QN];                                // output row (position slot * H + head), -1: none
  int2 tlist[MAXT];
  int stok[MAX_STOK * TN];                     // tokens of the sink tiles, -1: dropped
  uint32_t tmem;
  int abort_flag, last;
  unsigned qmax, pieces[2];                    // largest |q| (bf16 bits); row pieces a warpgroup has to re-reference (and FAR)
  Geo geo;
};
constexpr int SMEM = 1024 + OFF_MISC + (int)sizeof(Misc);
static_assert(SMEM <= 227 * 1024, "shared memory");
static_assert(offsetof(Misc, nref) % 16 == 0 && offsetof(Misc, fac) % 16 == 0 && OFF_MISC % 16 == 0, "read as float4");
static_assert(offsetof(Misc, bars) % 8 == 0 && OFF_RAW % 1024 == 0 && SLOT % 1024 == 0 && P_BYTES % 1024 == 0, "operand tiles");

// ---- instructions this kernel adds to tc_common.cuh ----
// kind::f16 with fp16 operands, fp32 accumulation
__device__ __forceinline__ uint32_t idesc_f16(int N, int b_mn) {
  return (1u << 4) | ((uint32_t)b_mn << 16) | ((uint32_t)(N >> 3) << 17) | (8u << 24);
}
#define TC_LD8(taddr, r)                                                                             \
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"              \
               : "=r"((r)[0]), "=r"((r)[1]), "=r"((r)[2]), "=r"((r)[3]), "=r"((r)[4]), "=r"((r)[5]), \
                 "=r"((r)[6]), "=r"((r)[7])                                                          \
               : "r"(taddr) : "memory")
#define TC_ST8(taddr, r)                                                                             \
  asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};"              \
               ::"r"(taddr), "r"((r)[0]), "r"((r)[1]), "r"((r)[2]), "r"((r)[3]), "r"((r)[4]),        \
                 "r"((r)[5]), "r"((r)[6]), "r"((r)[7])                                               \
               : "memory")
// sixteen lanes x 32 columns in the fragment layout of four 16x8 accumulator tiles
#define TC_ST_FRAG16(taddr, r)                                                                                     \
  asm volatile(                                                                                                    \
      "tcgen05.st.sync.aligned.16x256b.x4.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};"     \
      ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),        \
        "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])               \
      : "memory")
// two 16x16 byte matrices, transposed: register i of a pair holds row lane/4 + 8 i, columns 4 (lane % 4) .. + 3
__device__ __forceinline__ void ldsm_t8(uint32_t addr, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m16n16.x2.trans.shared.b8 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ uint4 lds128(uint32_t addr) {
  uint4 v;
  asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr) : "memory");
  return v;
}
__device__ __forceinline__ void sts128(uint32_t addr, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}
// normal numbers only
__device__ __forceinline__ float lg2(float x) { float y; asm("lg2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x)); return y; }
// from 2^-124 up; by way of a quarter, since the largest numbers' inverses are subnormal
__device__ __forceinline__ float rcp(float x) { float y; asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(0.25f * x)); return 0.25f * y; }
// maximum over the warp of one float per lane (NaN is passed over)
__device__ __forceinline__ float warp_max_f32(float x) {
  float m;
  asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(m) : "f"(x));
  return m;
}
// a load that stays where it is written (a plain one may be moved down to its first use, an iteration later)
__device__ __forceinline__ float ld_pinned(const float* p) {
  float v;
  asm volatile("ld.global.f32 %0, [%1];" : "=f"(v) : "l"(p) : "memory");
  return v;
}
__device__ __forceinline__ void named_sync(int id, int n) { asm volatile("bar.sync %0, %1;" ::"r"(id), "r"(n) : "memory"); }
__device__ __forceinline__ bool named_any(int id, int n, bool v) {
  uint32_t r;
  asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %3, 0;\n\tbar.red.or.pred q, %1, %2, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
               : "=r"(r) : "r"(id), "r"(n), "r"(v ? 1u : 0u) : "memory");
  return r != 0;
}
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}

// Four codes of one word -> two fp16 pairs.  int8: code + 128 as the low byte of the half 0x64xx = 1024 + (code + 128),
// then 1152 off -- exact, and cheaper than integer conversions (5 operations for four codes).
__device__ __forceinline__ void expand(uint32_t w, uint32_t& lo, uint32_t& hi, int8_t) {
  w ^= 0x80808080u;
  const uint32_t a = __byte_perm(w, 0x64646464u, 0x4140), b = __byte_perm(w, 0x64646464u, 0x4342);
  const __half2 k = __halves2half2(__ushort_as_half(0x6480), __ushort_as_half(0x6480));
  const __half2 x = __hsub2(*reinterpret_cast<const __half2*>(&a), k), y = __hsub2(*reinterpret_cast<const __half2*>(&b), k);
  lo = *reinterpret_cast<const uint32_t*>(&x);
  hi = *reinterpret_cast<const uint32_t*>(&y);
}
__device__ __forceinline__ void expand(uint32_t w, uint32_t& lo, uint32_t& hi, __nv_fp8_e4m3) {
  asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %2;\n\tcvt.rn.f16x2.e4m3x2 %0, l;\n\tcvt.rn.f16x2.e4m3x2 %1, h;\n\t}"
      : "=r"(lo), "=r"(hi) : "r"(w));
}

// 16-byte chunk c of raw row `row`: rows of 128 bytes with the 128-byte swizzle, rows of 64 bytes with the 64-byte one
template <int D>
__device__ __forceinline__ uint32_t raw_off(int row, int c) {
  return D == 128 ? (uint32_t)(row * 128 + ((c ^ (row & 7)) << 4)) : (uint32_t)(row * 64 + ((c ^ ((row >> 1) & 3)) << 4));
}

// Token of column k of a tile, or -1 if the column is masked out (padding, a sink that is dropped or out of range).
__device__ __forceinline__ int sink_token(const QParams& p, int g, int s) {
  const int j = __ldg(p.sink_idx + s);
  const bool keep = __ldg(p.sink_keep + (size_t)g * p.group_stride * p.n_sink + s) != 0;
  return (keep && j >= 0 && j < p.M) ? j : -1;             // response tokens are attended through their own tiles
}

// tile idx of this split: by arithmetic (dense), from the staged list, or from the block list (splits longer than that)
__device__ __forceinline__ TileInfo make_tile(const QParams& p, const Geo& gm, int idx) {
  TileInfo ti = tile_info(p, gm.te, gm.t0 + idx);
  if (ti.nvalid == 0) ti.start = ti.start2 = (p.L + 63) & ~63;         // bad block index: wholly outside, arrives as zeros
  return ti;
}
__device__ __forceinline__ TileInfo get_tile(const QParams& p, const Misc& ms, const Geo& gm, int idx) {
  if (!p.dense && gm.nt <= MAXT) return unpack_tile(ms.tlist[idx]);
  return make_tile(p, gm, idx);
}
__device__ __forceinline__ int key_token(const QParams& p, const Misc& ms, const Geo& gm, const TileInfo& ti, int k) {
  if (k >= ti.nvalid) return -1;
  if (ti.kind == 0) return (k < 64 ? ti.start : ti.start2 - 64) + k;
  const int s = ti.start + k, i = s - gm.stok_first;
  return i >= 0 && i < gm.stok_n ? ms.stok[i] : sink_token(p, gm.g, s);
}

__device__ __forceinline__ uint32_t bar_k_full(uint32_t b, int s) { return b + 8u * s; }
__device__ __forceinline__ uint32_t bar_k_empty(uint32_t b, int s) { return b + 8u * (RING + s); }
__device__ __forceinline__ uint32_t bar_v_full(uint32_t b, int s) { return b + 8u * (2 * RING + s); }
__device__ __forceinline__ uint32_t bar_v_empty(uint32_t b, int s) { return b + 8u * (3 * RING + s); }
__device__ __forceinline__ uint32_t bar_kop_full(uint32_t b, int i) { return b + 8u * (4 * RING + i); }
__device__ __forceinline__ uint32_t bar_kop_empty(uint32_t b, int i) { return b + 8u * (4 * RING + 2 + i); }
__device__ __forceinline__ uint32_t bar_vop_full(uint32_t b, int i) { return b + 8u * (4 * RING + 4 + i); }
__device__ __forceinline__ uint32_t bar_vop_empty(uint32_t b, int i) { return b + 8u * (4 * RING + 6 + i); }
__device__ __forceinline__ uint32_t bar_s_full(uint32_t b, int i) { return b + 8u * (4 * RING + 8 + i); }
__device__ __forceinline__ uint32_t bar_s_empty(uint32_t b, int i) { return b + 8u * (4 * RING + 10 + i); }
__device__ __forceinline__ uint32_t bar_p_full(uint32_t b, int i) { return b + 8u * (4 * RING + 12 + i); }
__device__ __forceinline__ uint32_t bar_p_empty(uint32_t b, int i) { return b + 8u * (4 * RING + 14 + i); }

__device__ __forceinline__ uint32_t bar_q_full(uint32_t b) { return b + 8u * (4 * RING + 16); }

// the arrivals of n threads at once: the same barrier from 31 lanes would be 31 shared-memory atomics in a row
__device__ __forceinline__ void mbar_arrive_n(uint32_t bar, uint32_t n) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(n) : "memory");
}

// Reduces 32 values per lane over the 32 lanes by halving: 31 shuffles, lane i ends with the result of value i.
template <typename Op>
__device__ __forceinline__ float lane_reduce32(float* v, int lane, Op op) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    const bool hi = (lane & o) != 0;
#pragma unroll
    for (int i = 0; i < o; ++i) {
      const float send = hi ? v[i] : v[i + o], keep = hi ? v[i + o] : v[i];
      v[i] = op(keep, __shfl_xor_sync(0xffffffffu, send, o));
    }
  }
  return v[0];
}

struct Ordinary { static constexpr bool value = false; };
struct Wide { static constexpr bool value = true; };

// Softmax of one warpgroup (x = 0, 1: even, odd tiles), NP pieces of 8 rows; straight-line code per tile, since its length
// in cycles is what a tile costs.  Leaves the row sums over this warpgroup's keys in ms.red.
template <int NP>
__device__ __forceinline__ void softmax_loop(const QParams& p, Misc& ms, uint32_t sP, uint32_t sBar, float cs, int x, int wq,
                                             int lane) {
  constexpr int NC = NP * 8;
  const Geo& gm = ms.geo;
  const int key = wq * 32 + lane, nt = gm.nt, tok0 = gm.t0 * TN + key;
  const uint32_t tmem = ms.tmem;
  const uint32_t lane_off = (uint32_t)(wq * 32) << 16;
  const uint32_t tO = tmem + (uint32_t)(T_O + x * QN) + lane_off, ts = tmem + (uint32_t)(T_S + x * QN) + lane_off;
  const uint32_t prow = sP + (uint32_t)(x * P_BYTES + key * 128);
  volatile int* abort_flag = &ms.abort_flag;
  float* nref = ms.nref[x];
  float* fac = ms.fac[x];
  float* red = ms.red[x * 4 + wq];
  const float* Ks = p.K_scale + (long long)gm.g * p.scale_stride;
  const float* Vs = p.V_scale + (long long)gm.g * p.scale_stride;
  float l[NC];
#pragma unroll
  for (int c = 0; c < NC; ++c) l[c] = 0.f;
  auto scales = [&](int idx, float& sk, float& sv) {                   // sv == -1: masked
    sk = 0.f; sv = -1.f;
    if (idx >= nt) return;
    int t;
    if (p.dense) {
      t = tok0 + idx * TN;
      if (t >= p.L) return;
    } else {
      t = key_token(p, ms, gm, get_tile(p, ms, gm, idx), key);
      if (t < 0) return;
    }
    sk = ld_pinned(Ks + t);
    sv = ld_pinned(Vs + t);
  };
  // of a tile's key: logit factor, log2 of the value scale (-inf: masked), one over the value scale
  float ck, lv, iv;
  bool far = false;                                                    // its value scale is out of the ordinary
  auto factors = [&](float sk, float sv) {
    const bool masked = sv == -1.f;
    const float svc = fmaxf(sv, SV_MIN);
    far = !masked && !(svc >= SV_LOW && svc <= SV_HIGH);
    ck = sk * cs;
    lv = masked ? -INFINITY : lg2(svc);
    iv = masked ? 0.f : rcp(svc);
  };
  float sk, sv;                                                        // the next tile's scales, on their way
  scales(x, sk, sv);
  factors(sk, sv);
  scales(x + 2, sk, sv);
  // Tiles j0, j0 + 2, ... .  With WIDE false it returns at the first tile that holds a value scale out of the ordinary, nothing of
  // it done; with WIDE true the exponentials are square roots of the numerators and reach down to 2^-252 of the reference, and
  // so are the factors of a changed reference, used twice.
  bool ok = true;
  auto tiles = [&](auto wide, int j0) -> int {
    constexpr bool WIDE = decltype(wide)::value;
    constexpr float A_MAX = WIDE ? ROOT_P_MAX : P_MAX;
    for (int j = j0; j < nt; j += 2) {
      const uint32_t ph = (uint32_t)(j >> 1) & 1u;
      ok = __all_sync(0xffffffffu, mbar_wait_quiet(bar_s_full(sBar, x), ph, abort_flag));
      tc_fence_after();
      float a[NC];
      uint32_t* ar = reinterpret_cast<uint32_t*>(a);
      bool again = false;
      unsigned pieces = (1u << NP) - 1u;
#pragma unroll 1
      for (;;) {
        if (j >= 2 || again) {
          // ---- P = 2^(s ck + lv - ref), to shared memory as fp16 ----
#pragma unroll
          for (int i = 0; i < NP; ++i) TC_LD8(ts + i * 8, ar + i * 8);
          tc_wait_ld();
#pragma unroll
          for (int q = 0; q < NP * 2; ++q) {
            const float4 rv = reinterpret_cast<const float4*>(nref)[q];
            float* v = a + q * 4;
            ffma2(v[0], v[1], v[0], v[1], ck, ck, lv, lv);
            ffma2(v[2], v[3], v[2], v[3], ck, ck, lv, lv);
            fadd2(v[0], v[1], v[0], v[1], rv.x, rv.y);
            fadd2(v[2], v[3], v[2], v[3], rv.z, rv.w);
          }
#pragma unroll
          for (int e = 0; e < NC; ++e) a[e] = ex2(WIDE ? 0.5f * a[e] : a[e]);
          // P V of this warpgroup's last tile has read the buffer (long ago, as a rule; the exponentials are on their way)
          ok = __all_sync(0xffffffffu, mbar_wait_quiet(bar_p_empty(sBar, x), ph ^ 1u, abort_flag) && ok);
          float m0 = 0.f, m1 = 0.f;
#pragma unroll
          for (int e = 0; e < NC; e += 4) {
            m0 = fmax3(m0, a[e], a[e + 1]);
            m1 = fmax3(m1, a[e + 2], a[e + 3]);
          }
#pragma unroll
          for (int i = 0; i < NP; ++i) {
            float v[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = WIDE ? a[i * 8 + e] * a[i * 8 + e] : a[i * 8 + e];
            sts128(prow + (uint32_t)((i ^ (key & 7)) << 4), pack_f16(v[0], v[1]), pack_f16(v[2], v[3]), pack_f16(v[4], v[5]),
                   pack_f16(v[6], v[7]));
          }
          fence_proxy_async();
          // The numerators are formed before anyone has looked whether they fit: the look costs a barrier of the four warps,
          // and here it is the one that hands the tile over anyway.
          if (!named_any(1 + x, 128, (fmaxf(m0, m1) > A_MAX && !again) || (!WIDE && far) || !ok)) break;
          if (named_any(1 + x, 128, !ok)) { ok = false; break; }
          // ---- some row's maximum outgrew its reference: new references for the pieces it is in, and the tile once more
          // (the first tile starts here, for all of them).  Rolled loops: code that runs this seldom is fetched from L2 each time ----
          pieces = 0;
#pragma unroll
          for (int i = 0; i < NP; ++i) {
            const float* v = a + i * 8;
            if (fmaxf(fmax3(fmax3(v[0], v[1], v[2]), v[3], v[4]), fmax3(v[5], v[6], v[7])) > A_MAX) pieces |= 1u << i;
          }
          pieces = __reduce_or_sync(0xffffffffu, pieces | (!WIDE && far ? FAR : 0u));
          if (lane == 0 && pieces) atomicOr(&ms.pieces[x], pieces);
          named_sync(1 + x, 128);
          pieces = ms.pieces[x];
          if (!WIDE && (pieces & FAR)) {                                 // the same in all threads
            named_sync(1 + x, 128);
            if (key == 0) ms.pieces[x] = 0u;
            named_sync(1 + x, 128);
            return j;
          }
        }
#pragma unroll 1
        for (int i = 0; i < NP; ++i) {
          if (!(pieces >> i & 1u)) continue;
          uint32_t v[8];
          TC_LD8(ts + i * 8, v);
          tc_wait_ld();
          float mine = -INFINITY;
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const float w = warp_max_f32(fmaf(__uint_as_float(v[e]), ck, lv));
            if (lane == e) mine = w;
          }
          if (lane < 8) red[i * 8 + lane] = mine;
        }
        named_sync(1 + x, 128);
        if (key < NC) {
          float f = 1.f;
          if (pieces >> (key >> 3) & 1u) {
            const float(*r)[QN] = &ms.red[x * 4];
            const float rowmax = fmaxf(fmaxf(r[0][key], r[1][key]), fmaxf(r[2][key], r[3][key]));
            const float old = nref[key], now = OFFSET - rowmax;
            if (now < old) { f = ex2(WIDE ? 0.5f * (now - old) : now - old); nref[key] = now; }
          }
          fac[key] = f;
          if (key == 0) ms.pieces[x] = 0u;
        }
        named_sync(1 + x, 128);
        if (j >= 2) {                                                    // what these rows have summed: P V of tile j - 2 is done
          tc_fence_after();
#pragma unroll 1
          for (int i = 0; i < NP; ++i) {
            if (!(pieces >> i & 1u)) continue;
            uint32_t v[8];
            TC_LD8(tO + i * 8, v);
            tc_wait_ld();
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              const float f = fac[i * 8 + e];
              v[e] = __float_as_uint(WIDE ? __uint_as_float(v[e]) * f * f : __uint_as_float(v[e]) * f);
            }
            TC_ST8(tO + i * 8, v);
          }
          tc_wait_st();
#pragma unroll
          for (int q = 0; q < NP * 2; ++q) {
            const float4 f = reinterpret_cast<const float4*>(fac)[q];
#pragma unroll
            for (int t = 0; t < (WIDE ? 2 : 1); ++t) { l[4 * q] *= f.x; l[4 * q + 1] *= f.y; l[4 * q + 2] *= f.z; l[4 * q + 3] *= f.w; }
          }
        }
        again = true;
      }
      if (!ok) return nt;
      tc_fence_before();
      __syncwarp();
      if (lane == 0) { mbar_arrive(bar_p_full(sBar, x)); mbar_arrive(bar_s_empty(sBar, x)); }
#pragma unroll
      for (int e = 0; e < NC; e += 2) {
        if constexpr (WIDE) { l[e] = fmaf(a[e] * iv, a[e], l[e]); l[e + 1] = fmaf(a[e + 1] * iv, a[e + 1], l[e + 1]); }
        else ffma2(l[e], l[e + 1], a[e], a[e + 1], iv, iv, l[e], l[e + 1]);
      }
      factors(sk, sv);
      scales(j + 4, sk, sv);
    }
    return nt;
  };
  const int rest = tiles(Ordinary(), x);
  if (rest < nt) tiles(Wide(), rest);
  // all products done (each warpgroup waits for both buffers: the last two tiles)
  for (int j = nt > 1 ? nt - 2 : 0; j < nt; ++j) mbar_wait_quiet(bar_p_empty(sBar, j & 1), (uint32_t)(j >> 1) & 1u, abort_flag);
  tc_fence_after();
  // ---- row sums over this warp's 32 keys: lane i of a warp ends with row i of a group ----
  named_sync(1 + x, 128);                                              // the column maxima in ms.red have been read
#pragma unroll
  for (int h = 0; h * 4 < NP; ++h) {
    float v[32];
#pragma unroll
    for (int e = 0; e < 32; ++e) v[e] = h * 32 + e < NC ? l[h * 32 + e < NC ? h * 32 + e : 0] : 0.f;
    red[h * 32 + lane] = lane_reduce32(v, lane, [](float u, float w) { return u + w; });
  }
}

template <typename F, int D>
__global__ void __launch_bounds__(NTH, 1)
attn_quant_tc_kernel(const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV, const QParams p) {
  extern __shared__ uint8_t smem_raw[];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, wg = warp >> 2;
  const uint32_t sbase = (smem_u32(smem_raw) + 1023u) & ~1023u;
  uint8_t* sptr = smem_raw + (sbase - smem_u32(smem_raw));
  Misc& ms = *reinterpret_cast<Misc*>(sptr + OFF_MISC);
  const uint32_t sQ = sbase, sP = sbase + Q_BYTES, sRawK = sbase + OFF_RAW, sRawV = sRawK + RING * SLOT;
  const uint32_t sBar = smem_u32(ms.bars);
  volatile int* abort_flag = &ms.abort_flag;

  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  if (threadIdx.x == 0) {
    prefetch_tmap(&tmK); prefetch_tmap(&tmV);
    for (int s = 0; s < RING; ++s) {
      mbar_init(bar_k_full(sBar, s), 32); mbar_init(bar_v_full(sBar, s), 32);      // the producer warp's lanes
      mbar_init(bar_k_empty(sBar, s), 4); mbar_init(bar_v_empty(sBar, s), 4);      // four expanding warps
    }
    for (int b = 0; b < 2; ++b) {
      mbar_init(bar_kop_full(sBar, b), 4); mbar_init(bar_vop_full(sBar, b), 4);
      mbar_init(bar_kop_empty(sBar, b), 1); mbar_init(bar_vop_empty(sBar, b), 1);
      mbar_init(bar_s_full(sBar, b), 1); mbar_init(bar_p_empty(sBar, b), 1);
      mbar_init(bar_s_empty(sBar, b), 4); mbar_init(bar_p_full(sBar, b), 4);       // one softmax warpgroup's warps
    }
    mbar_init(bar_q_full(sBar), 8);                                    // eight softmax warps
    ms.abort_flag = 0; ms.qmax = 0u; ms.pieces[0] = ms.pieces[1] = 0u;
    fence_barrier_init();
    fence_proxy_async();
  }
  if (warp == 2) { tmem_alloc(smem_u32(&ms.tmem), 512); tmem_relinquish(); }
  if (threadIdx.x < 2 * QN) ms.nref[0][threadIdx.x] = -REF_NONE;
  if (p.pdl) asm volatile("griddepcontrol.wait;" ::: "memory");      // nothing in global memory is touched before this

  // ---- which row tile and which key tiles.  How many rows there are is known on the device only, so the split of the
  // grid is chosen here: the row tiles that hold rows share all CTAs, at least two key tiles per split ----
  const Geo& gm = ms.geo;
  uint4 qv[4];                                                         // softmax warps: a quarter (32 elements) of a query row
  int orow = -1;
  const int qrow = ((int)threadIdx.x - 384) >> 2, quarter = (int)threadIdx.x & 3;
  if (warp == 0 || wg >= 3) {                                          // both from the same numbers, neither waiting for the other
    const int nrows = p.q_rows ? min(max(ld_ordered(p.n_rows), 0), p.rows_bound) : p.n_q;
    const int n_mt = (nrows * p.hpg + QN - 1) / QN, base = n_mt * p.Hkv;
    const int n_splits = max(1, min(min(p.sms / max(base, 1), p.max_tiles >> 1), MAX_SPLITS));   // > 1: at most sms CTAs in all
    const int tile = (int)blockIdx.x / n_splits, split = (int)blockIdx.x - tile * n_splits;
    const int g = min(tile / max(n_mt, 1), p.Hkv - 1), mt = tile - g * n_mt;
    const int rows = tile < base ? max(min(QN, nrows * p.hpg - mt * QN), 0) : 0;   // stacked (row, head of the group) rows
    if (wg >= 3) {
#pragma unroll
      for (int c = 0; c < 4; ++c) qv[c] = make_uint4(0, 0, 0, 0);
      if (qrow < rows) {
        const int fr = mt * QN + qrow, qr = fr / p.hpg, hh = fr - qr * p.hpg;
        const int pos = p.q_rows ? ld_ordered(p.q_rows + qr) : p.q_base + qr;
        if (pos >= p.q_base && pos < p.q_base + p.n_q) {
          orow = qr * p.H + g * p.hpg + hh;
          if (quarter * 32 < D) {
            const uint4* src = reinterpret_cast<const uint4*>(p.Q + (long long)(pos - p.q_base) * p.q_stride_row +
                                                              (long long)(g * p.hpg + hh) * p.q_stride_head + quarter * 32);
#pragma unroll
            for (int c = 0; c < 4; ++c) qv[c] = ld_ordered(src + c);
          }
        } else if (quarter == 0) {
          set_status(p.status, FOCUS_ERR_INVALID_ARG);
        }
      }
    } else {
      const int cnt_raw = p.dense ? 0 : ld_ordered(p.block_cnt + g * p.group_stride);
      const TileEnum te = make_enum(p, g, cnt_raw);
      const int t0 = split_lo(te.total, split, n_splits), nt = split_lo(te.total, split + 1, n_splits) - t0;
      const int st_lo = max(t0, te.n_blk), st_hi = min(t0 + nt, te.n_blk + te.n_sinkt);            // sink tiles of this split
      if (lane == 0) {
        Geo q;
        q.g = g; q.t0 = t0; q.nt = nt; q.rows = rows; q.N = rows > 0 ? (rows + 15) & ~15 : 16;
        q.mt = mt; q.tile = tile; q.n_splits = n_splits; q.n_mt = n_mt;
        q.stok_first = (st_lo - te.n_blk) * TN;
        q.stok_n = p.dense ? 0 : min(max(st_hi - st_lo, 0), MAX_STOK) * TN;
        q.te = te;
        ms.geo = q;
      }
      __syncwarp();
    }
  }
  // one K or V tile of the cache into its ring slot (lane 0 of the producer warp)
  auto issue_tma = [&](const TileInfo& ti, int g, int kv, int slot, uint64_t pol) {
    const uint32_t full = kv ? bar_v_full(sBar, slot) : bar_k_full(sBar, slot);
    const uint32_t dst = (kv ? sRawV : sRawK) + slot * SLOT;
    const CUtensorMap* map = kv ? &tmV : &tmK;
    mbar_expect_tx(full, TN * D);
    tma_load_3d_hint(dst, map, full, 0, ti.start, g, pol);
    if (p.pair) tma_load_3d_hint(dst + 64 * D, map, full, 0, ti.start2, g, pol);
    mbar_arrive_n(full, 31);                                           // the barrier counts 32 lanes (sink tiles need them)
  };
  // a dense key set is known without reading anything: its first copies start here, ahead of everything else
  if (warp == 0 && lane == 0 && p.dense && gm.rows > 0) {
    // K/V tiles are read once, or once per row tile of their head (through L2)
    const uint64_t pol = gm.n_mt == 1 ? l2_policy_evict_first() : l2_policy_evict_normal();
    const int n = min(gm.nt, EARLY), g = gm.g;
    for (int j = 0; j < n; ++j)
      for (int kv = 0; kv < 2; ++kv) issue_tma(make_tile(p, gm, j), g, kv, j, pol);
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (!p.dense) {                                                      // tile descriptors and sink tokens
    if (warp == 4 && gm.nt <= MAXT)
      for (int t = lane; t < gm.nt; t += 32) ms.tlist[t] = pack_tile(make_tile(p, gm, t));
    if (warp >= 12)
      for (int i = (int)threadIdx.x - 384; i < gm.stok_n; i += 256) {
        const int s = gm.stok_first + i;
        ms.stok[i] = s < p.n_sink ? sink_token(p, gm.g, s) : -1;
      }
    __syncthreads();
  }

  if (wg == 0) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 64;");
    const int nt = gm.rows > 0 ? gm.nt : 0;
    const uint32_t tmem = ms.tmem;
    if ((warp & 1) == 0) {
      // ================================ producers: warp 0 K, warp 2 V ==============================
      const int kv = warp >> 1, g = gm.g, n_early = p.dense ? min(nt, EARLY) : 0;
      const uint64_t pol = gm.n_mt == 1 ? l2_policy_evict_first() : l2_policy_evict_normal();
      const uint32_t full0 = kv ? bar_v_full(sBar, 0) : bar_k_full(sBar, 0), empty0 = kv ? bar_v_empty(sBar, 0) : bar_k_empty(sBar, 0);
      bool ok = true, plain = false;                                   // plain: a slot may hold copies of the other kind
      int slot = n_early, issued = n_early;
      uint32_t round = 0;
      // All CTAs start together: with whole rings requested at once the first tile -- and the queries -- would wait behind
      // everybody's fifth.  The rest follows once the first tile's keys have landed.
      if (n_early > 0 && nt > n_early) ok = __all_sync(0xffffffffu, mbar_wait_quiet(bar_k_full(sBar, 0), 0u, abort_flag));
      for (int j = n_early; j < nt && ok; ++j) {
        const TileInfo ti = get_tile(p, ms, gm, j);
        ok = __all_sync(0xffffffffu, mbar_wait_quiet(empty0 + 8u * slot, (round & 1u) ^ 1u, abort_flag));
        if (!ok) break;
        ++issued;
        if (ti.kind == 0) {
          if (lane == 0) {
            if (ti.nvalid == 0) set_status(p.status, FOCUS_ERR_INVALID_ARG);   // bad block index
            if (plain) fence_proxy_async();
            issue_tma(ti, g, kv, slot, pol);
          }
          __syncwarp();
        } else {
          // sink tokens lie anywhere: 16-byte copies, dropped ones as zeros
          constexpr int CPR = D / 16;
          const uint32_t dst = (kv ? sRawV : sRawK) + slot * SLOT;
          const uint8_t* base = (kv ? p.V : p.K) + (long long)g * p.kv_stride_head;
          plain = true;
#pragma unroll 1
          for (int i = 0; i < 4; ++i) {
            const int tok = key_token(p, ms, gm, ti, i * 32 + lane);
#pragma unroll
            for (int it = 0; it < CPR; ++it) {
              const int q = it * 32 + lane, rr = q / CPR, c = q % CPR;        // row within this group of 32, chunk
              const int t = __shfl_sync(0xffffffffu, tok, rr);
              const uint8_t* src = base + (long long)max(t, 0) * p.kv_stride_tok + c * 16;
              asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;"
                           ::"r"(dst + raw_off<D>(i * 32 + rr, c)), "l"(src), "r"(t >= 0 ? 16u : 0u) : "memory");
            }
          }
          asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(full0 + 8u * slot) : "memory");
          if (kv == 0) {
#pragma unroll 1
            for (int k = lane; k < ti.nvalid; k += 32) {               // a listed sink outside [0, L) is reported
              const int s = __ldg(p.sink_idx + ti.start + k);
              if (s < 0 || s >= p.L) set_status(p.status, FOCUS_ERR_INVALID_ARG);
            }
          }
        }
        if (++slot == RING) { slot = 0; ++round; }
      }
      asm volatile("cp.async.wait_all;" ::: "memory");
      if (!ok) {
        // unwinding: let the copies already issued land before the CTA's shared memory is released
        for (int i = max(0, issued - RING); i < issued; ++i) {
          const uint64_t t_start = global_ns();
          while (!mbar_try_wait(full0 + 8u * (i % RING), (uint32_t)(i / RING) & 1u)) {
            if (global_ns() - t_start > WAIT_LIMIT_NS) break;
          }
        }
      }
    } else if (warp == 1 && lane == 0 && nt > 0) {
      // ================================ S^T = K Q^T ===============================================
      const uint32_t id = idesc_f16(gm.N, 0);
      const uint64_t qdesc = make_sdesc(sQ, 16, 1024);
      if (mbar_wait_quiet(bar_q_full(sBar), 0u, abort_flag))
        for (int j = 0; j < nt; ++j) {
          const int b = j & 1;
          const uint32_t ph = (uint32_t)(j >> 1) & 1u;
          if (!mbar_wait_quiet(bar_kop_full(sBar, b), ph, abort_flag)) break;
          if (!mbar_wait_quiet(bar_s_empty(sBar, b), ph ^ 1u, abort_flag)) break;
          tc_fence_after();
#pragma unroll
          for (int ks = 0; ks < D / 16; ++ks)
            mma_ts(tmem + T_S + b * QN, tmem + T_K + b * 64 + ks * 8,
                   qdesc + (uint64_t)(((ks >> 2) * (QN * 128) + (ks & 3) * 32) >> 4), id, ks ? 1u : 0u);
          tc_commit(bar_kop_empty(sBar, b));
          tc_commit(bar_s_full(sBar, b));
        }
    } else if (warp == 3 && lane == 0 && nt > 0) {
      // ================================ O^T += V^T P^T ============================================
      const uint32_t id = idesc_f16(gm.N, 1);
      for (int j = 0; j < nt; ++j) {
        const int b = j & 1;
        const uint32_t ph = (uint32_t)(j >> 1) & 1u;
        if (!mbar_wait_quiet(bar_vop_full(sBar, b), ph, abort_flag)) break;
        if (!mbar_wait_quiet(bar_p_full(sBar, b), ph, abort_flag)) break;
        tc_fence_after();
        const uint64_t pdesc = make_sdesc(sP + b * P_BYTES, TN * 128, 1024);
#pragma unroll
        for (int ks = 0; ks < TN / 16; ++ks)
          mma_ts(tmem + T_O + b * QN, tmem + T_V + b * 64 + ks * 8, pdesc + (uint64_t)(ks * (2048 >> 4)), id, (ks || j > 1) ? 1u : 0u);
        tc_commit(bar_vop_empty(sBar, b));
        tc_commit(bar_p_empty(sBar, b));
      }
    }
    __syncwarp();
    tc_fence_before();
    asm volatile("bar.sync 0;" ::: "memory");
    tc_fence_after();
    if (warp == 2) { __syncwarp(); tmem_dealloc(tmem, 512); }
    if (threadIdx.x == 96 && ms.abort_flag) set_status(p.status, FOCUS_ERR_TIMEOUT);
  } else if (wg == 1) {
    // ================================ K codes -> A operand of S^T =====================================
    asm volatile("setmaxnreg.dec.sync.aligned.u32 48;");
    const int nt = gm.rows > 0 ? gm.nt : 0;
    const uint32_t tmem = ms.tmem;
    if (nt > 0) {
      const int key = (warp & 3) * 32 + lane;
      const uint32_t lane_off = (uint32_t)((warp & 3) * 32) << 16;
      int slot = 0;
      uint32_t round = 0;
      for (int j = 0; j < nt; ++j) {
        const int b = j & 1;
        const bool ok = mbar_wait_quiet(bar_k_full(sBar, slot), round & 1u, abort_flag) &&
                        mbar_wait_quiet(bar_kop_empty(sBar, b), ((uint32_t)(j >> 1) & 1u) ^ 1u, abort_flag);
        if (!__all_sync(0xffffffffu, ok)) break;
        tc_fence_after();
        const uint32_t src = sRawK + slot * SLOT, dst = tmem + (uint32_t)(T_K + b * 64) + lane_off;
#pragma unroll 1
        for (int h = 0; h < D / 64; ++h) {
          uint32_t o[32];
          uint4 raw[4];
#pragma unroll
          for (int c = 0; c < 4; ++c) raw[c] = lds128(src + raw_off<D>(key, h * 4 + c));
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            expand(raw[c].x, o[8 * c + 0], o[8 * c + 1], F());
            expand(raw[c].y, o[8 * c + 2], o[8 * c + 3], F());
            expand(raw[c].z, o[8 * c + 4], o[8 * c + 5], F());
            expand(raw[c].w, o[8 * c + 6], o[8 * c + 7], F());
          }
          TC_ST32(dst + h * 32, o);
        }
        tc_wait_st();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) { mbar_arrive(bar_k_empty(sBar, slot)); mbar_arrive(bar_kop_full(sBar, b)); }
        if (++slot == RING) { slot = 0; ++round; }
      }
    }
    tc_fence_before();
    asm volatile("bar.sync 0;" ::: "memory");
  } else if (wg == 2) {
    // ================================ V codes, transposed -> A operand of O^T ===========================
    asm volatile("setmaxnreg.dec.sync.aligned.u32 48;");
    const int nt = gm.rows > 0 ? gm.nt : 0;
    const uint32_t tmem = ms.tmem;
    if (nt > 0) {
      const int cw = warp & 3;                                         // channels 32 cw .. 32 cw + 31
      if (cw * 32 >= D) {                                              // head dim 64: the upper lanes stay zero
        uint32_t z[32];
#pragma unroll
        for (int i = 0; i < 32; ++i) z[i] = 0u;
#pragma unroll 1
        for (int i = 0; i < 4; ++i) TC_ST32(tmem + (uint32_t)(T_V + i * 32) + ((uint32_t)(cw * 32) << 16), z);
        tc_wait_st();
      }
      int slot = 0;
      uint32_t round = 0;
      for (int j = 0; j < nt; ++j) {
        const int b = j & 1;
        const bool ok = mbar_wait_quiet(bar_v_full(sBar, slot), round & 1u, abort_flag) &&
                        mbar_wait_quiet(bar_vop_empty(sBar, b), ((uint32_t)(j >> 1) & 1u) ^ 1u, abort_flag);
        if (!__all_sync(0xffffffffu, ok)) break;
        tc_fence_after();
        const uint32_t src = sRawV + slot * SLOT, dst = tmem + (uint32_t)(T_V + b * 64) + ((uint32_t)(cw * 32) << 16);
        if (cw * 32 < D) {
#pragma unroll 2
          for (int it = 0; it < 4; ++it) {                             // sixteen channels x 64 keys: four 16-key matrices
            const int hc = it >> 1, q = it & 1;
            uint32_t o[16];
#pragma unroll
            for (int pr = 0; pr < 2; ++pr) {
              uint32_t m[4];
              ldsm_t8(src + raw_off<D>(q * 64 + pr * 32 + lane, cw * 2 + hc), m);
#pragma unroll
              for (int i = 0; i < 2; ++i) {
                expand(m[2 * i], o[(2 * pr + i) * 4 + 0], o[(2 * pr + i) * 4 + 1], F());
                expand(m[2 * i + 1], o[(2 * pr + i) * 4 + 2], o[(2 * pr + i) * 4 + 3], F());
              }
            }
            TC_ST_FRAG16(dst + ((uint32_t)(hc * 16) << 16) + q * 32, o);
          }
        }
        tc_wait_st();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) { mbar_arrive(bar_v_empty(sBar, slot)); mbar_arrive(bar_vop_full(sBar, b)); }
        if (++slot == RING) { slot = 0; ++round; }
      }
    }
    tc_fence_before();
    asm volatile("bar.sync 0;" ::: "memory");
  } else {
    // ================================ softmax =========================================================
    asm volatile("setmaxnreg.inc.sync.aligned.u32 160;");
    const int x = wg - 3, wq = warp & 3, key = wq * 32 + lane, tid = (int)threadIdx.x - 384;
    const int rows = gm.rows, N = gm.N, n_splits = gm.n_splits;
    const bool work = rows > 0 && gm.nt > 0;
    const uint32_t tmem = ms.tmem;
    float cs = 0.f;
    const uint32_t lane_off = (uint32_t)(wq * 32) << 16;
    if (rows > 0) {
      // ---- queries -> fp16, 128-byte-swizzled K-major tile; one power of two for the whole tile ----
      unsigned m = 0u;
      if (quarter == 0) ms.orow[qrow] = orow;
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        const uint32_t w[4] = {qv[c].x, qv[c].y, qv[c].z, qv[c].w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const unsigned u = w[e] & 0x7FFFu, v = (w[e] >> 16) & 0x7FFFu;      // magnitudes of bf16 order as integers
          if (u < 0x7F80u) m = max(m, u);                                     // finite ones
          if (v < 0x7F80u) m = max(m, v);
        }
      }
      m = __reduce_max_sync(0xffffffffu, m);
      if (lane == 0) atomicMax(&ms.qmax, m);
      named_sync(3, 256);
      // the power of two: the tile's largest |q| to 2^14 .. 2^15
      const int sh = ms.qmax ? min(14 - ((int)(ms.qmax >> 7) - 127), 126) : 0;
      const float f = exp2f((float)sh);
      cs = p.scale_log2 * exp2f((float)-sh);
      if (quarter * 32 < D) {
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          const uint32_t w[4] = {qv[c].x, qv[c].y, qv[c].z, qv[c].w};
          uint32_t o[4];
#pragma unroll
          for (int i = 0; i < 4; ++i)
            o[i] = pack_f16(__uint_as_float(w[i] << 16) * f, __uint_as_float(w[i] & 0xFFFF0000u) * f);
          const int cc = (quarter & 1) * 4 + c;                        // chunk within the row's 64-element half
          sts128(sQ + (quarter >> 1) * (QN * 128) + qrow * 128 + ((cc ^ (qrow & 7)) << 4), o[0], o[1], o[2], o[3]);
        }
      }
      fence_proxy_async();
      __syncwarp();
      if (lane == 0) mbar_arrive(bar_q_full(sBar));
    }
    if (work) {
      if (N == 16) softmax_loop<2>(p, ms, sP, sBar, cs, x, wq, lane);
      else if (N == 32) softmax_loop<4>(p, ms, sP, sBar, cs, x, wq, lane);
      else if (N == 48) softmax_loop<6>(p, ms, sP, sBar, cs, x, wq, lane);
      else softmax_loop<8>(p, ms, sP, sBar, cs, x, wq, lane);
    }
    named_sync(3, 256);
    // ---- row statistics: sums of the warps in order, the two warpgroups' shares of a row joined ----
    if (tid < rows) {
      const int r = tid;
      float ref = REF_NONE, tot = 0.f, w0 = 0.f, w1 = 0.f;
      if (work) {
        auto warps = [&](int q) { return ((ms.red[q * 4][r] + ms.red[q * 4 + 1][r]) + ms.red[q * 4 + 2][r]) + ms.red[q * 4 + 3][r]; };
        const float l0 = warps(0), l1 = warps(1), r0 = -ms.nref[0][r], r1 = -ms.nref[1][r];
        ref = fmaxf(r0, r1);
        const float h0 = l0 != 0.f ? ex2(0.5f * (r0 - ref)) : 0.f, h1 = l1 != 0.f ? ex2(0.5f * (r1 - ref)) : 0.f;
        w0 = h0 * h0;
        w1 = h1 * h1;
        tot = h0 * l0 * h0 + h1 * l1 * h1;
      }
      if (n_splits > 1) {
        reinterpret_cast<float2*>(p.part_ml)[(size_t)blockIdx.x * QN + r] = make_float2(ref, tot);
      } else {
        const float inv = tot != 0.f ? 1.f / tot : 0.f;
        w0 *= inv; w1 *= inv;
        const int orow = ms.orow[r];
        if (orow >= 0 && p.lse)
          p.lse[(size_t)(orow % p.H) * p.lse_stride + orow / p.H] = tot == 0.f ? -INFINITY : (ref + log2f(tot)) * 0.6931471805599453f;
      }
      ms.fac[0][r] = w0; ms.fac[1][r] = w1;
    }
    named_sync(3, 256);
    // ---- O^T: this thread's channel of the rows of its half (a warpgroup's share without a key is never read) ----
    const int ch = key, c0 = x * (N >> 1);
#pragma unroll 1
    for (int i = 0; i < N >> 4; ++i) {
      uint32_t o0[8], o1[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) o0[e] = o1[e] = 0u;
      if (work) {
        TC_LD8(tmem + (uint32_t)(T_O + c0 + i * 8) + lane_off, o0);
        TC_LD8(tmem + (uint32_t)(T_O + QN + c0 + i * 8) + lane_off, o1);
        tc_wait_ld();
      }
      const int r0 = c0 + i * 8;
      float v[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float f0 = ms.fac[0][r0 + e], f1 = ms.fac[1][r0 + e];
        v[e] = (f0 != 0.f ? __uint_as_float(o0[e]) * f0 : 0.f) + (f1 != 0.f ? __uint_as_float(o1[e]) * f1 : 0.f);
      }
      if (ch < D) {
        if (n_splits > 1) {
          float* dst = p.part_O + ((size_t)blockIdx.x * QN + r0) * D + ch;
#pragma unroll
          for (int e = 0; e < 8; ++e)
            if (r0 + e < rows) dst[e * D] = v[e];
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const int orow = ms.orow[r0 + e];
            if (r0 + e < rows && orow >= 0) p.O[(size_t)orow * D + ch] = __float2bfloat16_rn(v[e]);
          }
        }
      }
    }
    tc_fence_before();
    asm volatile("bar.sync 0;" ::: "memory");
    // ---- merge of the splits by the CTA that arrives last, splits in order ----
    if (n_splits > 1 && rows > 0) {
      const int S = n_splits;
      __threadfence();
      named_sync(3, 256);
      if (tid == 0) {
        const int prev = atomicAdd(&p.counters[gm.tile], 1);
        ms.last = prev == S - 1;
        if (ms.last) p.counters[gm.tile] = 0;                       // armed for the next launch
        __threadfence();
      }
      named_sync(3, 256);
      if (ms.last) {
        float* wts = reinterpret_cast<float*>(sptr + Q_BYTES);         // [row][split], over the P tiles
        const size_t c_first = (size_t)gm.tile * S;
        if (tid < rows) {
          const float2* ml = reinterpret_cast<const float2*>(p.part_ml) + c_first * QN + tid;
          float m = -INFINITY, tot = 0.f;
#pragma unroll 4
          for (int s = 0; s < S; ++s) {
            const float2 v = __ldcg(ml + (size_t)s * QN);
            if (v.y != 0.f) m = fmaxf(m, v.x);
          }
#pragma unroll 4
          for (int s = 0; s < S; ++s) {
            const float2 v = __ldcg(ml + (size_t)s * QN);
            const float h = v.y != 0.f ? ex2(0.5f * (v.x - m)) : 0.f;
            tot += h * v.y * h;
            wts[tid * S + s] = h * h;
          }
          const int orow = ms.orow[tid];
          ms.fac[0][tid] = tot != 0.f ? 1.f / tot : 0.f;
          if (orow >= 0 && p.lse)
            p.lse[(size_t)(orow % p.H) * p.lse_stride + orow / p.H] = tot == 0.f ? -INFINITY : (m + log2f(tot)) * 0.6931471805599453f;
        }
        named_sync(3, 256);
#pragma unroll 2
        for (int it = tid; it < rows * (D / 4); it += 256) {
          const int r = it / (D / 4), c4 = it % (D / 4), orow = ms.orow[r];
          if (orow < 0) continue;
          const float4* po = reinterpret_cast<const float4*>(p.part_O) + (c_first * QN + r) * (D / 4) + c4;
          float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 8
          for (int s = 0; s < S; ++s) {
            const float w = wts[r * S + s];
            const float4 o = __ldcg(po + (size_t)s * QN * (D / 4));
            if (w != 0.f) { acc.x += w * o.x; acc.y += w * o.y; acc.z += w * o.z; acc.w += w * o.w; }
          }
          const float f = ms.fac[0][r];
          uint2 v;
          v.x = pack_bf16(acc.x * f, acc.y * f);
          v.y = pack_bf16(acc.z * f, acc.w * f);
          *reinterpret_cast<uint2*>(p.O + (size_t)orow * D + c4 * 4) = v;
        }
      }
    }
  }
}

bool encode_code_map(void* fn, CUtensorMap* map, const void* base, const focus_shape& s, int box_rows) {
  const cuuint64_t dims[3] = {(cuuint64_t)s.head_dim, (cuuint64_t)s.L, (cuuint64_t)s.n_kv_heads};
  const cuuint64_t strides[2] = {(cuuint64_t)s.kv_stride_tok, (cuuint64_t)s.kv_stride_head};
  const cuuint32_t box[3] = {(cuuint32_t)s.head_dim, (cuuint32_t)box_rows, 1};
  const cuuint32_t one[3] = {1, 1, 1};
  return ((EncodeTiledFn)fn)(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 3, const_cast<void*>(base), dims, strides, box, one,
                             CU_TENSOR_MAP_INTERLEAVE_NONE,
                             s.head_dim == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B,
                             CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <typename F, int D>
focus_status launch(focus_ctx* ctx, bool& attr_set, const CUtensorMap& tmK, const CUtensorMap& tmV, const QParams& p,
                    dim3 grid, cudaStream_t st) {
  if (!attr_set) {
    if (cudaFuncSetAttribute(attn_quant_tc_kernel<F, D>, cudaFuncAttributeMaxDynamicSharedMemorySize, SMEM) != cudaSuccess)
      return FOCUS_ERR_CUDA;
    attr_set = true;
  }
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid; cfg.blockDim = dim3(NTH, 1, 1); cfg.dynamicSmemBytes = SMEM; cfg.stream = st;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = at; cfg.numAttrs = p.pdl ? 1 : 0;
  if (cudaLaunchKernelEx(&cfg, attn_quant_tc_kernel<F, D>, tmK, tmV, p) != cudaSuccess) {
    cudaGetLastError();
    return FOCUS_ERR_CUDA;
  }
  FOCUS_CHECK_LAUNCH();
  return FOCUS_OK;
}

}  // namespace

bool attn_quant_tc_supported(const focus_ctx* ctx, const AttnArgs& a) {
  return ctx->encode_tiled != nullptr && a.sh.dtype == FOCUS_BF16 && (a.sh.head_dim == 128 || a.sh.head_dim == 64) &&
         (long long)a.max_rows * a.sh.n_q_heads < (1ll << 31);
}

focus_status launch_attn_quant_tc(focus_ctx* ctx, const AttnArgs& a, cudaStream_t st) {
  const focus_shape& sh = a.sh;
  const int Hkv = sh.n_kv_heads, hpg = sh.n_q_heads / Hkv;
  const long long stacked = (long long)a.max_rows * hpg;              // stacked query rows per KV head (host bound)
  QParams p;
  p.pair = !a.dense && sh.kv_block == 64;
  p.ns_pad = a.dense ? 0 : (a.n_sink + TN - 1) / TN * TN;
  const int n_resp = a.dense ? (sh.L + TN - 1) / TN : (sh.L - sh.M + TN - 1) / TN;
  const int max_tiles = a.dense ? n_resp : (p.pair ? (a.max_blocks + 1) / 2 : a.max_blocks) + p.ns_pad / TN + n_resp;
  p.max_tiles = max_tiles; p.sms = ctx->sm_count;
  p.Hkv = Hkv;
  const long long base = (stacked + QN - 1) / QN * Hkv;               // row tiles, if every listed row is there
  if (base > 0x7FFFFFFF) return FOCUS_ERR_UNSUPPORTED;
  // one CTA per SM, or per row tile where there are more; splits (chosen in the kernel) occur only in the first case
  const int ctas = base > ctx->sm_count ? (int)base : ctx->sm_count;
  WsAlloc ws(ctx);
  p.part_O = ws.get<float>((size_t)ctx->sm_count * QN * sh.head_dim);
  p.part_ml = ws.get<float>((size_t)ctx->sm_count * QN * 2);
  if (!ws.ok) return FOCUS_ERR_WORKSPACE_TOO_SMALL;
  p.counters = ctx->d_counters;
  p.Q = (const __nv_bfloat16*)a.Q; p.O = (__nv_bfloat16*)a.O; p.lse = a.lse;
  p.q_rows = a.q_rows; p.n_rows = a.n_rows; p.block_idx = a.block_idx; p.block_cnt = a.block_cnt;
  p.sink_idx = a.sink_idx; p.sink_keep = a.sink_keep;
  p.K = (const uint8_t*)a.qc->K; p.V = (const uint8_t*)a.qc->V; p.K_scale = a.qc->K_scale; p.V_scale = a.qc->V_scale;
  p.q_stride_row = sh.q_stride_row; p.q_stride_head = sh.q_stride_head;
  p.kv_stride_tok = sh.kv_stride_tok; p.kv_stride_head = sh.kv_stride_head; p.scale_stride = quant_scale_stride(a.qc, &sh);
  p.q_base = a.q_base; p.n_q = a.n_q; p.rows_bound = a.max_rows; p.L = sh.L; p.M = sh.M; p.H = sh.n_q_heads; p.hpg = hpg;
  p.B = sh.kv_block; p.nb = shape_nb(&sh); p.dense = a.dense; p.group_stride = a.group_stride;
  p.max_blocks = a.max_blocks; p.n_sink = a.n_sink; p.lse_stride = a.lse_stride;
  p.pdl = ctx->no_pdl ? 0 : 1;
  p.scale_log2 = a.scale * 1.4426950408889634f;
  p.status = ctx->d_status;
  CUtensorMap tmK, tmV;
  const int box_rows = p.pair ? 64 : TN;
  if (!encode_code_map(ctx->encode_tiled, &tmK, p.K, sh, box_rows) || !encode_code_map(ctx->encode_tiled, &tmV, p.V, sh, box_rows))
    return FOCUS_ERR_INVALID_ARG;
  ctx->last_attn_variant = 5;
  const dim3 grid((unsigned)ctas, 1, 1);
  const bool i8 = a.qc->format == FOCUS_KV_INT8;
  bool* set = ctx->ls.quant_attr_set;
  if (sh.head_dim == 128)
    return i8 ? launch<int8_t, 128>(ctx, set[0], tmK, tmV, p, grid, st) : launch<__nv_fp8_e4m3, 128>(ctx, set[1], tmK, tmV, p, grid, st);
  return i8 ? launch<int8_t, 64>(ctx, set[2], tmK, tmV, p, grid, st) : launch<__nv_fp8_e4m3, 64>(ctx, set[3], tmK, tmV, p, grid, st);
}

size_t attn_quant_tc_workspace(const focus_shape* s) {
  // partial outputs of every split: no more CTAs than SMs take part in a split launch (160 bounds the part at hand)
  return (size_t)160 * QN * ((size_t)s->head_dim + 2) * 4 + 1024;
}
