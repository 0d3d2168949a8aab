// Device definitions shared by the kernels of attention with score modifiers:
// visibility, the cap, and the search for the next tile that a workgroup has to
// visit.
#pragma once

#include "attn_tile.hpp"
#include "launch_mod.hpp"

namespace vidax {
namespace mod {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.69314718055994531f;
constexpr int kStartLimit = 1 << 30;  // positions stay within +- 2^30 + L

// Scores in log2 units: y = mul * f(q.k) with f the identity (mul = |scale|
// log2 e; the sign of scale goes into q) or, capped, t = tanh(ku q.k) (mul = cap
// log2 e, ku = |scale| / cap).
struct Scores {
  float mul, ku;
  float tanh_poly[4], poly[4], limit;  // capped: t, and the forward's form of y (cap16_log2)
  uint32_t qxor, qand;  // applied to q's bf16 pairs: sign of scale, zero where it is 0
};

// tanh(u) = u (k0 + k1 u^2 + k2 u^4 + k3 u^6) up to 3.2e-7 of itself for |u| <= 0.45
// (weighted least squares; five terms up to 1/2 are good to 1.2e-7 and cost a twelfth
// of the capped forward's vector work).
constexpr float kTanhMost = 0.45f;
constexpr float kTanh[4] = {9.999997616e-1f, -3.332946599e-1f, 1.323636919e-1f, -4.602819309e-2f};

inline Scores make_scores(const ModCall& c) {
  Scores s;
  const float a = c.scale < 0.f ? -c.scale : c.scale;
  s.qxor = c.scale < 0.f ? 0x80008000u : 0u;
  s.qand = a == 0.f ? 0u : 0xffffffffu;
  s.ku = c.s.cap > 0.f ? a / c.s.cap : 0.f;
  s.mul = c.s.cap > 0.f ? c.s.cap * kLog2e : a == 0.f ? 1.f : a * kLog2e;
  // tanh(ku x) = x (p0 + p1 x^2 + ...) for |x| <= limit; never where a factor could overflow
  float k = s.ku;
  for (int i = 0; i < 4; ++i, k *= s.ku * s.ku) {
    s.tanh_poly[i] = kTanh[i] * k;
    s.poly[i] = s.mul * s.tanh_poly[i];
  }
  s.limit = s.ku == 0.f ? INFINITY : s.ku < 100.f && fabsf(s.poly[3]) < 1e30f ? kTanhMost / s.ku : -1.f;
  return s;
}

// tanh(ku x) of 16 products, in place.  The odd polynomial, ku folded in, where the
// whole wave's block stays within its limit, else the exponential, whose absolute error
// of 1e-7 is then small against the block's largest score.
__device__ __forceinline__ float odd_poly(float x, const float p[4], float n) {  // + n
  const float w = x * x;
  float y = fmaf(w, p[3], p[2]);
  y = fmaf(w, y, p[1]);
  y = fmaf(w, y, p[0]);
  return fmaf(x, y, n);
}
__device__ __forceinline__ float tanh_any(float u) {
  const float e = __builtin_amdgcn_exp2f(u * (2.f * kLog2e));
  return fmaf(-2.f, __builtin_amdgcn_rcpf(e + 1.f), 1.f);
}
__device__ __forceinline__ bool within16(const f32x16& s, const Scores& c) {  // (uniform)
  float m = 0.f;
#pragma unroll
  for (int i = 0; i < 16; ++i) m = fmaxf(m, fabsf(s[i]));
  return __builtin_amdgcn_ballot_w64(!(m <= c.limit)) == 0;
}
__device__ __forceinline__ void cap16(f32x16& s, const Scores& c) {
  if (within16(s, c)) {
#pragma unroll
    for (int i = 0; i < 16; ++i) s[i] = odd_poly(s[i], c.tanh_poly, 0.f);
  } else {
#pragma unroll
    for (int i = 0; i < 16; ++i) s[i] = tanh_any(s[i] * c.ku);
  }
}
// y + n = mul tanh(ku x) + n, all factors folded in: five operations a score.
__device__ __forceinline__ void cap16_log2(f32x16& s, const Scores& c, float n) {
  if (within16(s, c)) {
#pragma unroll
    for (int i = 0; i < 16; ++i) s[i] = odd_poly(s[i], c.poly, n);
  } else {
#pragma unroll
    for (int i = 0; i < 16; ++i) s[i] = fmaf(c.mul, tanh_any(s[i] * c.ku), n);
  }
}

// Batch values (uniform).
struct Batch {
  int lv;      // keys j < lv exist
  int start;   // position of query 0
  int prefix;  // causal: keys j < prefix are seen by all
};
__device__ __forceinline__ Batch batch_of_lane(const ModCall& c, int b) {  // (b may differ from lane to lane)
  Batch r;
  r.lv = c.Lk;
  if (c.s.kv_valid_len) r.lv = min(max(c.s.kv_valid_len[b], 0), c.Lk);
  r.start = c.Lk - c.Lq;
  if (c.s.q_start) r.start = min(max(c.s.q_start[b], -kStartLimit), kStartLimit);
  r.prefix = c.s.prefix_len ? max(c.s.prefix_len[b], 0) : 0;
  return r;
}
__device__ __forceinline__ Batch batch_of(const ModCall& c, int b) {
  Batch r = batch_of_lane(c, b);
  r.lv = __builtin_amdgcn_readfirstlane(r.lv);
  r.start = __builtin_amdgcn_readfirstlane(r.start);
  r.prefix = __builtin_amdgcn_readfirstlane(r.prefix);
  return r;
}
// Keys that a query at position p sees, documents apart: [0, key_limit).
__device__ __forceinline__ int key_limit(const Batch& b, int causal, int p) {
  return causal ? min(b.lv, max(max(p + 1, 0), b.prefix)) : b.lv;
}

// Document range of some tokens: least and largest id >= 0 (least > largest:
// none), and whether an id < 0 is among them.
struct Docs {
  int lo, hi;
  bool neg;
};
__device__ __forceinline__ Docs docs_of(int2 r) { return Docs{r.x, r.y & 0x7fffffff, r.y < 0}; }
__device__ __forceinline__ Docs join(const Docs& a, const Docs& b) {
  return Docs{min(a.lo, b.lo), max(a.hi, b.hi), a.neg || b.neg};
}
__device__ __forceinline__ Docs uniform(const Docs& d) {
  return Docs{__builtin_amdgcn_readfirstlane(d.lo), __builtin_amdgcn_readfirstlane(d.hi),
              (bool)__builtin_amdgcn_readfirstlane((int)d.neg)};
}
__device__ __forceinline__ bool meet(const Docs& a, const Docs& b) { return a.lo <= b.hi && b.lo <= a.hi; }
// all of one document
__device__ __forceinline__ bool one_doc(const Docs& a) { return !a.neg && a.lo == a.hi; }
// every token of both in one and the same document
__device__ __forceinline__ bool same(const Docs& a, const Docs& b) {
  return one_doc(a) && one_doc(b) && a.lo == b.lo;
}

// Which 256-row tile t of (batch b, head h of `heads`) and which of its runs the
// workgroup takes.  Neighbours in number go to different XCDs.
//   Tiles of equal work, or one round of workgroups: an XCD takes a stretch of a
// head's tiles, whose other side then stays in its L2.
//   Otherwise (`sorted`) the most work first, all heads of a tile side by side: a
// late start of a long tile would hold the launch up (16384 causal, 12 heads, the
// kernel of then: 1172 us with long and short tiles in turn, XCD by XCD; 842 so).
template <typename A>
__device__ __forceinline__ void place(const A& a, int heads, const int32_t* order, int& run, int& t, int& b, int& h) {
  const ModCall& c = a.c;
  if (a.sorted) {
    // run by run: run r is there for the first so many tiles (a.in_run)
    const int n = order ? heads : c.B * heads, i = blockIdx.x / n, bh = blockIdx.x - i * n;
    int x = i;
    run = 0;
    while (run + 1 < a.runs && x >= a.in_run[run]) x -= a.in_run[run++];
    if (order) {
      const int y = __builtin_amdgcn_readfirstlane(order[x]);
      b = y / a.ntile;
      t = y - b * a.ntile;
      h = bh;
    } else {
      b = bh / heads;
      h = bh - b * heads;
      t = a.first_most ? x : a.ntile - 1 - x;
    }
    return;
  }
  const int i = balanced_tile(blockIdx.x, a.nwg, c.B);
  run = i % a.runs;
  const int x = i / a.runs, bh = x / a.ntile;
  t = x - bh * a.ntile;
  b = bh / heads;
  h = bh - b * heads;
}

// ---- equal pieces of the streams of all 256-row tiles (no documents)
//
// The tiles that the workgroups' tiles visit, behind one another (batch, head, own
// tile, visited tile), are one sequence, cut into pieces of equal weight, a
// workgroup each; a piece may end one own tile, hold some whole and begin another.
// An own tile that is cut leaves partial results, at most two a piece (slots 2 p: a
// part that does not begin the tile, 2 p + 1: one that does), which a further launch
// joins.
struct Pieces {
  int n;         // 0: not in pieces
  int slot_rows; // rows of a slot
  int32_t* cut;  // [B][H][tiles][2]: first (-1: not cut) and last piece of a tile
};
struct Part {
  int b, h, t;    // own tile
  int n, lo, hi;  // the tiles it visits, and this part of them
  int piece;
  __device__ __forceinline__ bool whole() const { return lo == 0 && hi == n; }
  __device__ __forceinline__ int slot() const { return 2 * piece + (lo == 0); }
};

// Own tiles of queries, which visit key tiles.
struct QuerySide {
  static __device__ __forceinline__ int length(const ModCall& c) { return c.Lq; }
  static __device__ __forceinline__ int heads(const ModCall& c) { return c.H; }
  static __device__ __forceinline__ int visits(const ModCall& c, const Batch& bt, int t) {
    return (key_limit(bt, c.s.causal, bt.start + min((t + 1) * kModRows, c.Lq) - 1) + kModKeys - 1) / kModKeys;
  }
};
// Own tiles of keys, which visit the query tiles [first_query_tile, end) of every
// query head of theirs.
__device__ __forceinline__ int first_query_tile(const ModCall& c, const Batch& bt, int key0) {
  const int end = (c.Lq + kModKeys - 1) / kModKeys;
  if (key0 >= key_limit(bt, c.s.causal, bt.start + c.Lq - 1)) return end;
  return c.s.causal && key0 >= bt.prefix ? min(max(key0 - bt.start, 0) / kModKeys, end) : 0;
}
struct KeySide {
  static __device__ __forceinline__ int length(const ModCall& c) { return c.Lk; }
  static __device__ __forceinline__ int heads(const ModCall& c) { return c.Hkv; }
  static __device__ __forceinline__ int visits(const ModCall& c, const Batch& bt, int t) {
    return c.H / c.Hkv * ((c.Lq + kModKeys - 1) / kModKeys - first_query_tile(c, bt, t * kModRows));
  }
};

// f(part) for every part of piece p, in order.  All waves alike.
template <typename Side, typename F>
__device__ __forceinline__ void each_part(const ModCall& c, int pieces, int p, F&& f) {
  const int lane = threadIdx.x & 63, len = Side::length(c), heads = Side::heads(c), nt = (int)mod_tiles(len);
  auto unit = [&](int t) { return key_weight(min(len - t * kModRows, kModRows)); };
  auto tile_weight = [&](const Batch& bt, int t) { return kTileStart + Side::visits(c, bt, t) * unit(t); };
  const bool lens = mod_own_lengths(c.s);  // (B <= kLaneBatches then: mod_pieces)
  auto wave_sum = [&](int x) {
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) x += __shfl_xor(x, m);
    return __builtin_amdgcn_readfirstlane(x);
  };
  auto scan = [&](int x) {  // with the lane's own
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) {
      const int y = __shfl_up(x, m);
      if (lane >= m) x += y;
    }
    return x;
  };
  auto head_weight = [&](const Batch& bt) {
    int w = 0;
    for (int t = lane; t < nt; t += 64) w += tile_weight(bt, t);
    return wave_sum(w);
  };
  // the whole sequence (all weights of a head fit in 31 bits: mod_pieces)
  Batch bt;
  int hw = 0, lane_w = 0;  // of a head: of batch b, of batch `lane`
  int64_t total = 0;
  if (!lens) {
    bt = batch_of(c, 0);
    hw = head_weight(bt);
    total = (int64_t)hw * c.B * heads;
  } else if (nt <= kLaneTiles) {
    const Batch mine = batch_of_lane(c, min(lane, c.B - 1));
    if (lane < c.B)
      for (int t = 0; t < nt; ++t) lane_w += tile_weight(mine, t);
    total = (int64_t)wave_sum(lane_w) * heads;
  } else {
    for (int b = 0; b < c.B; ++b) {
      const int w = head_weight(batch_of(c, b));
      if (lane == b) lane_w = w;
      total += (int64_t)w * heads;
    }
  }
  int64_t per = (total + pieces - 1) / pieces;
  if (per < kLeastPiece) per = kLeastPiece;
  const int64_t pos = p * per, end = pos + per < total ? pos + per : total;
  if (pos >= end) return;
  // the tile at pos
  int64_t S = 0;  // where the tile begins
  int b = 0;
  if (lens) {
    const int to = scan(lane_w);
    b = __builtin_ctzll(__builtin_amdgcn_ballot_w64((int64_t)to * heads > pos));  // (pos < total)
    hw = __builtin_amdgcn_readlane(lane_w, b);
    S = (int64_t)__builtin_amdgcn_readlane(to - lane_w, b) * heads;
  } else {
    b = (int)(pos / ((int64_t)hw * heads));
    S = (int64_t)hw * heads * b;
  }
  bt = batch_of(c, b);
  int h = (int)((pos - S) / hw);
  S += (int64_t)h * hw;
  int t = 0;
  {
    const int rem = (int)(pos - S);
    int before = 0;
    for (int t0 = 0; t0 < nt; t0 += 64) {
      const int w = t0 + lane < nt ? tile_weight(bt, t0 + lane) : 0;
      const int x = scan(w);
      const uint64_t over = __builtin_amdgcn_ballot_w64(before + x > rem);
      if (over != 0) {
        const int i = __builtin_ctzll(over);
        t = t0 + i;
        S += before + __builtin_amdgcn_readlane(x - w, i);
        break;
      }
      before += __builtin_amdgcn_readlane(x, 63);
    }
  }
  for (;;) {
    const int n = Side::visits(c, bt, t), u = unit(t);
    // the visited tile at a position; not within two of either end
    auto tile_at = [&](int64_t x) {
      const int64_t y = x - S - kTileStart;
      if (y >= (int64_t)n * u) return n;
      const int k = y <= 0 ? 0 : (int)y / u;
      return k < 2 ? 0 : k > n - 2 ? n : k;
    };
    const Part part{b, h, t, n, tile_at(pos), tile_at(end), p};
    if (part.lo < part.hi || (n == 0 && pos <= S)) f(part);
    S += kTileStart + n * u;
    if (S >= end) return;
    if (++t == nt) {
      t = 0;
      if (++h == heads) {
        h = 0;
        bt = batch_of(c, ++b);
      }
    }
  }
}
// What the join has to know of a tile, noted by whoever begins or ends it.
template <typename Side>
__device__ __forceinline__ void note_cut(const Pieces& x, const ModCall& c, const Part& part) {
  int32_t* const p = x.cut + (((size_t)part.b * Side::heads(c) + part.h) * mod_tiles(Side::length(c)) + part.t) * 2;
  if (part.lo == 0) p[0] = part.whole() ? -1 : part.piece;
  else if (part.hi == part.n) p[1] = part.piece;
}
// Pieces of one head to one XCD (its K and V in that L2).
__device__ __forceinline__ int piece_of(int block, int n) {
  const int q = n >> 3, r = n & 7, x = block & 7;
  return x * q + min(x, r) + (block >> 3);
}

// A tile of the streamed side, as a workgroup or wave meets it (uniform).
struct Tile {
  int t;   // < 0: none left
  int f;   // bits:
  int id;  // kOne: the document
  enum {
    kMine = 1,   // some row of the wave may see (or be seen by) some of it
    kWhole = 2,  // all of the wave's rows see (are seen by) all of it
    kZero = 4,   // it holds tokens that have to be read as zeros
    kOne = 8     // its tokens are of one document
  };
  __device__ __forceinline__ bool mine() const { return f & kMine; }
  __device__ __forceinline__ bool whole() const { return f & kWhole; }
  __device__ __forceinline__ bool zero() const { return f & kZero; }
  __device__ __forceinline__ bool one() const { return f & kOne; }
};

// ---- tiles as rows: 256-byte rows whose 16-byte chunks are permuted, chunk c of
// row r at position c ^ swz(r), free of bank conflicts for row reads and for the
// transposing reads (the layout of the dense backward, attn_bwd.hip).  A copy
// instruction fills rows 4 j .. 4 j + 3.
constexpr int kRow = kHeadDim;  // elements of a row
__device__ __forceinline__ int swz(int r) { return ((r & 3) << 2) | ((r >> 2) & 3); }
struct RowOffsets {
  int row, tr;  // elements: row operand of row l32, d 8 hi; transposed operand
};
__device__ __forceinline__ RowOffsets row_offsets(int lane) {
  const int l32 = lane & 31, hi = lane >> 5, g = lane >> 4, w = lane & 15, r = 4 * hi + (w >> 2);
  return RowOffsets{l32 * kRow + 8 * (hi ^ swz(l32)),
                    r * kRow + 8 * ((2 * (g & 1) + ((w >> 1) & 1)) ^ swz(r)) + 4 * (w & 1)};
}
// rows l32 of a 32-row block, d = 16 st + 8 hi ..
__device__ __forceinline__ bf16x8 read_row(const uint16_t* block, int row, int st) {
  return *reinterpret_cast<const bf16x8*>(block + (row ^ (16 * st)));
}
// 16 rows transposed, d block mb, in the accumulators' row order
__device__ __forceinline__ bf16x8 read_tr(const uint16_t* rows16, int tr, int mb) {
  const tile::i16x4 lo = tile::lds_read_tr16(rows16 + (tr ^ (32 * mb)));
  const tile::i16x4 up = tile::lds_read_tr16(rows16 + (tr ^ (32 * mb) ^ 16) + 8 * kRow);
  return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, up, 0, 1, 2, 3, 4, 5, 6, 7));
}

}  // namespace mod
}  // namespace vidax
