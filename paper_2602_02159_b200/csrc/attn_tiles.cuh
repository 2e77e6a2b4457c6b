// Key tiles of the tensor-core attention kernels: which 128 keys tile t of a KV head's key set holds (dense: a run of
// tokens; sparse: selected blocks, sink tokens, response region), how a tile is described in shared memory, and where a
// key set is cut into splits.  P is a kernel's parameter struct: L, M, B, nb, dense, pair, group_stride, block_idx,
// max_blocks, n_sink, ns_pad (sinks rounded up to whole tiles).
#pragma once

#include "focus_common.cuh"

constexpr int TN = 128;            // keys per tile

struct TileInfo {
  int kind;     // 0: tile of the K/V tensors, 1: tile of the gathered sink rows
  int start;    // first key row of the tile in its tensor
  int nvalid;   // leading columns that are real keys (the rest is masked out)
  int start2;   // pair mode, kind 0: first key row of the tile's second half (columns 64..127)
};
// staged form of a TileInfo: x = start | kind << 30; y = nvalid | code << 8, code = start2 / 64 for a pair of
// blocks, all ones for "the 64 rows after the first half"
constexpr int START2_NEXT = 0x7FFFFF;
__device__ __forceinline__ int2 pack_tile(const TileInfo& ti) {
  const int code = ti.start2 == ti.start + 64 ? START2_NEXT : (ti.start2 >> 6);
  return make_int2(ti.start | (ti.kind << 30), ti.nvalid | (code << 8));
}
__device__ __forceinline__ TileInfo unpack_tile(int2 e) {
  TileInfo ti;
  ti.kind = e.x >> 30; ti.start = e.x & 0x3FFFFFFF; ti.nvalid = e.y & 0xff;
  const int code = (e.y >> 8) & START2_NEXT;
  ti.start2 = code == START2_NEXT ? ti.start + 64 : code << 6;
  return ti;
}

struct TileEnum {
  int n_blk;        // tiles that come from the block list (pair mode: two blocks per tile)
  int n_blocks;     // entries of the block list
  int n_sinkt, n_resp, total;
  const int32_t* blocks;
};

// First key tile of split s of n: floor(total * s / n).  total < 2^23 tiles (2^30 tokens) and s <= 32, so the product
// fits 32 bits (a 64-bit division is a subroutine of a few hundred cycles on the set-up path of every CTA).
__device__ __forceinline__ int split_lo(int total, int s, int n) {
  return (int)((unsigned)total * (unsigned)s / (unsigned)n);
}

template <typename P>
__device__ __forceinline__ TileEnum make_enum(const P& p, int g, int cnt_raw) {
  TileEnum e;
  if (p.dense) {
    e.n_blk = 0; e.n_blocks = 0; e.n_sinkt = 0; e.n_resp = (p.L + TN - 1) / TN; e.blocks = nullptr;
  } else {
    const int row = g * p.group_stride;
    e.n_blocks = min(max(cnt_raw, 0), p.max_blocks);
    e.n_blk = p.pair ? (e.n_blocks + 1) >> 1 : e.n_blocks;
    e.n_sinkt = p.ns_pad / TN;
    e.n_resp = (p.L - p.M + TN - 1) / TN;
    e.blocks = p.block_idx + (size_t)row * p.max_blocks;
  }
  e.total = e.n_blk + e.n_sinkt + e.n_resp;
  return e;
}

// First key tile of split s of n for a sparse key set, tiles weighed by what their softmax costs: a sink tile (one
// mask test per column) counts 3, a block or response tile 2.  With equal tile counts the split that got the sink
// tiles finished last and its cluster waited for it (config 2, four splits of 22 tiles: loops of 11.4 / 13.6 / 12.7 /
// 16.4 thousand cycles).  s = 0 gives 0, s = n the tile count; monotonic in s.
__device__ __forceinline__ int split_lo_cost(const TileEnum& e, int s, int n) {
  const unsigned wb = 2u * (unsigned)e.n_blk, ws = 3u * (unsigned)e.n_sinkt, W = wb + ws + 2u * (unsigned)e.n_resp;
  const unsigned x = (W * (unsigned)s + (unsigned)n - 1u) / (unsigned)n;          // ceil(W s / n)
  if (x <= wb) return (int)((x + 1u) / 2u);
  if (x <= wb + ws) return e.n_blk + (int)((x - wb + 2u) / 3u);
  return e.n_blk + e.n_sinkt + (int)((x - wb - ws + 1u) / 2u);
}

template <typename P>
__device__ __forceinline__ TileInfo tile_info(const P& p, const TileEnum& e, int t) {
  TileInfo ti;
  ti.start2 = -1;
  if (p.dense) {
    ti.kind = 0; ti.start = t * TN; ti.nvalid = min(TN, p.L - ti.start);
  } else if (t < e.n_blk && p.pair) {
    // two 64-token blocks side by side; a short block (the last one of the prompt) goes second so that the valid
    // columns stay a prefix; a missing second block repeats the first (finite data, masked out)
    int b0 = e.blocks[2 * t];
    int b1 = 2 * t + 1 < e.n_blocks ? e.blocks[2 * t + 1] : -2;
    ti.kind = 0;
    if (b0 < 0 || b0 >= p.nb || b1 == -1 || b1 < -2 || b1 >= p.nb) {  // reported once by the producer; fully masked
      ti.start = 0; ti.start2 = 0; ti.nvalid = 0;
    } else {
      if (b1 >= 0 && p.M - b0 * 64 < 64) { const int x = b0; b0 = b1; b1 = x; }
      ti.start = b0 * 64;
      const int n0 = min(64, p.M - ti.start);
      if (b1 >= 0) { ti.start2 = b1 * 64; ti.nvalid = n0 < 64 ? n0 : 64 + min(64, p.M - ti.start2); }
      else { ti.start2 = ti.start; ti.nvalid = n0; }
    }
  } else if (t < e.n_blk) {
    const int b = e.blocks[t];
    ti.kind = 0;
    if (b < 0 || b >= p.nb) {               // reported once by the producer; the tile is fully masked
      ti.start = 0; ti.nvalid = 0;
    } else {
      ti.start = b * p.B; ti.nvalid = min(p.B, p.M - ti.start);
    }
  } else if (t < e.n_blk + e.n_sinkt) {
    const int s = t - e.n_blk;
    ti.kind = 1; ti.start = s * TN; ti.nvalid = min(TN, p.n_sink - s * TN);
  } else {
    const int r = t - e.n_blk - e.n_sinkt;
    ti.kind = 0; ti.start = p.M + r * TN; ti.nvalid = min(TN, p.L - ti.start);
  }
  if (ti.start2 < 0) ti.start2 = ti.start + 64;
  return ti;
}
