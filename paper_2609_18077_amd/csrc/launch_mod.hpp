// Arguments, launch rules and launchers of attention with score modifiers
// (attn_mod_*.hip; not part of the C ABI).  The launchers are weak: a library
// linked from the ABI layer alone still loads, and its calls of these report a
// failed launch.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace vidax {

// What changes the scores, as validated by the ABI layer (device pointers).
struct ModScore {
  int causal;
  float cap;                    // 0: none
  const float* slopes;          // [H]
  const int32_t *q_doc, *k_doc; // [B, Lq], [B, Lk], both or neither
  const int32_t* kv_valid_len;  // [B]
  const int32_t* prefix_len;    // [B], with causal
  const int32_t* q_start;       // [B], or null: Lk - Lq
};

struct ModCall {
  int B, H, Hkv, Lq, Lk;
  float scale;
  ModScore s;
};

// Whether the batches may visit tiles of their own: valid lengths, positions or prefixes.
// (One answer for the launch rules and the device's walk over the pieces.)
__host__ __device__ inline bool mod_own_lengths(const ModScore& s) { return s.kv_valid_len || s.q_start || s.prefix_len; }

struct ModFwd {
  ModCall c;
  const uint16_t *q, *k, *v;
  uint16_t* o;
  float* lse;  // or null
  float* ws;
  size_t ws_floats;
};

struct ModBwd {
  ModCall c;
  const uint16_t *q, *k, *v, *o, *dout;
  const float* lse;
  uint16_t *dq, *dk, *dv;
  float* ws;
  size_t ws_floats;
};

// ---- workspace: document ranges of every 32 tokens (keys, then queries; two
// int32 a range, an even number of ranges a batch), then what a form adds.
// (With documents) also the order of the 256-row tiles, queries then keys.
constexpr int kModRows = 256;
__host__ __device__ inline size_t mod_ranges(int L) { return ((size_t)L + 63) / 64 * 2; }
__host__ __device__ inline size_t mod_tiles(int L) { return ((size_t)L + kModRows - 1) / kModRows; }
inline size_t mod_doc_floats(int B, int Lq, int Lk, bool docs) {
  return docs ? (size_t)B * (mod_ranges(Lk) * 2 + mod_ranges(Lq) * 2 + mod_tiles(Lq) + mod_tiles(Lk)) : 0;
}

// ---- forward ----
//
// Few rows (a group's query heads times the queries, at most kFewRows): the form
// for single tokens (attn_mod_few.hip).  Otherwise tiles of 256 query rows, whose
// keys may be cut into runs, one workgroup each, that a second launch joins.
constexpr int kModKeys = 64;
constexpr int kFewRows = 32;
constexpr int kMostRuns = 16;
inline bool mod_few(int H, int Hkv, int Lq) { return Hkv > 0 && (int64_t)(H / Hkv) * Lq <= kFewRows; }

// Or all key tiles of all query tiles are cut into `pieces` of equal weight
// (attn_mod.hpp): tiles of unequal work, or not a whole number of rounds of them.
constexpr int kTileStart = 8;  // weight of starting and ending a query tile; see key_weight
// Weight of a key tile for a query tile of so many rows: one or two waves a SIMD.
__host__ __device__ inline int key_weight(int rows) { return rows > 128 ? 4 : 3; }
// Four key tiles: every piece between a tile's first and last then holds some of it.
constexpr int kLeastPiece = 16;
// Tiles of a head up to which a lane adds up those of a batch with lengths of its own.
constexpr int kLaneTiles = 16;
// Batches with lengths of their own in pieces: a lane each.
constexpr int kLaneBatches = 64;

// A launch takes fewer than 2^32 threads: workgroups of 512 for the tiles (and for each
// of the runs of their keys), of 256 for few rows, ranges and joins.  What a call cannot
// do without has to fit (the calls beyond are refused), runs and pieces are not taken
// where they or their joins would not.
constexpr int64_t kMostTiles = ((int64_t)1 << 23) - 1;
constexpr int64_t kMostSmall = ((int64_t)1 << 24) - 1;
inline bool mod_launches_fit(int B, int H, int Hkv, int Lq, int Lk, bool docs, bool backward) {
  const __int128 q = (__int128)mod_tiles(Lq) * B * H, k = (__int128)mod_tiles(Lk) * B * Hkv;
  if (docs && (__int128)B * (mod_ranges(Lq) + mod_ranges(Lk)) / 8 >= kMostSmall) return false;
  if (backward) return q <= kMostTiles && k <= kMostTiles;
  return mod_few(H, Hkv, Lq) ? (__int128)B * Hkv <= kMostSmall : q <= kMostTiles;
}

struct ModPieces {
  int n;          // 0: a workgroup takes a tile (or one of its runs)
  int slot_rows;  // rows of a partial result
  size_t cut;     // first value of the table of cut tiles in the workspace
  size_t floats;  // values of the workspace
  double us;
};

// Key tiles of query tile t, where queries stand at their default positions, and of all.
inline int64_t mod_row_tiles(int64_t t, int Lq, int Lk, bool causal) {
  const int64_t tiles = ((int64_t)Lk + kModKeys - 1) / kModKeys;
  if (!causal) return tiles;
  const int64_t last = (int64_t)Lk - Lq + ((t + 1) * kModRows < Lq ? (t + 1) * kModRows : Lq);  // keys seen by the last row
  return last <= 0 ? 0 : last >= Lk ? tiles : (last + kModKeys - 1) / kModKeys;
}
inline int64_t mod_key_tiles(int Lq, int Lk, bool causal) {
  int64_t n = 0;
  for (int64_t t = 0; t < (int64_t)mod_tiles(Lq); ++t) n += mod_row_tiles(t, Lq, Lk, causal);
  return n;
}

// Pieces, one a compute unit and 16 visited tiles at least: 12 us to find and
// start them and for the joining launch, and the partial rows' (of `row` floats) bytes
// at 5 TB/s.  A workgroup finds its own by going over the tiles' weights, 64 at a time
// (with lengths those of every batch): not where they are too many for that to be
// short.  Pieces of a head read its keys at
// different places; where K and V of a head are more than an L2 (4 MB) that costs 15 %.
// (Forward, 12 heads, 6144 plain: seven runs 303 us, pieces 260; causal 177 and 154;
// 1560 rows on 32760 keys: three runs 346, pieces 413.)
// `own` rows in tiles of 256, of which tile t visits visits(t) tiles of `other` rows.
template <typename F>
inline ModPieces mod_pieces(int B, int heads, int own, int other, int64_t most_visits, F&& visits, bool lengths, int cus, size_t first,
                            int row, double tile_us) {
  ModPieces p{0, 0, 0, 0, 0.0};
  const int64_t nt = (int64_t)mod_tiles(own), wgs = nt * B * heads;
  if (lengths ? B > kLaneBatches || (nt > kLaneTiles && (nt + 63) / 64 * B > 16) : nt > 4096) return p;
  if ((__int128)nt * B * (kTileStart + 4 * most_visits) > INT32_MAX) return p;  // (32-bit sums)
  if (wgs * 32 > kMostSmall) return p;                                          // (the joins: up to 32 workgroups a tile)
  int64_t weight = 0;  // of a head
  for (int64_t t = 0; t < nt; ++t)
    weight += kTileStart + visits(t) * key_weight((int)(own - t * kModRows < kModRows ? own - t * kModRows : kModRows));
  const int64_t all = weight * B * heads, most = all / (4 * kLeastPiece);
  const int n = (int)(most < cus ? most : cus);
  if (n < 2) return p;
  p.n = n;
  p.slot_rows = (own < kModRows ? own + 31 : kModRows) / 32 * 32;
  p.cut = first + (size_t)2 * n * p.slot_rows * row;
  p.floats = p.cut + 2 * (size_t)wgs;
  const int64_t parts = n + (wgs < n ? wgs : n);
  p.us = (double)all / n / 4 * tile_us * (other > 8192 ? 1.15 : 1.0) + 12.0 + (double)parts * p.slot_rows * row * 8 / 5e6;
  return p;
}

struct ModSplit {
  bool few;
  int runs;       // of the 256-row form
  ModPieces pieces;  // of the 256-row form
  int units;      // of the form for few rows; 0: a workgroup takes a whole batch
  size_t part;    // first value of the partial results in the workspace
  size_t floats;  // values of the workspace
};

inline ModSplit mod_fwd_split(int B, int H, int Hkv, int Lq, int Lk, bool docs, bool causal, bool lengths, int cus,
                              size_t max_floats) {
  ModSplit r;
  r.runs = 1;
  r.units = 0;
  r.pieces.n = 0;
  r.floats = mod_doc_floats(B, Lq, Lk, docs);
  r.part = (r.floats + 63) / 64 * 64;
  r.few = mod_few(H, Hkv, Lq);
  const int64_t rows = (int64_t)B * H * Lq;
  if (rows == 0 || Lk == 0) return r;
  if (r.few) {
    // one workgroup a compute unit in either form.  A unit takes at least a tile
    // a wave; the joining launch and its partial results cost 5 us.  A whole
    // batch a workgroup: 1.5 us for its four waves' next 32-key tiles (128 KB in
    // flight), 3.4 when every unit is busy (64 KB at its share of 5 TB/s).  Where
    // the batches have lengths of their own, a unit's part is taken as two thirds:
    // units share what is there, whole batches wait for the longest.
    const int64_t tiles = ((int64_t)Lk + 31) / 32, wgs = (int64_t)B * Hkv;
    int64_t u = cus / Hkv < B * tiles / 4 ? cus / Hkv : B * tiles / 4;
    auto us = [&](int64_t n, int64_t per) {  // n workgroups with `per` tiles each
      const int64_t rounds = (n + cus - 1) / cus, busy = n < cus ? n : cus;
      const double step = busy * 65536 / 5e6 > 1.5 ? busy * 65536 / 5e6 : 1.5;
      return rounds * (3.0 + (per + 3) / 4 * step);
    };
    const size_t need = r.part + (size_t)(u + B) * H * Lq * 129;
    if (u > 0 && need <= max_floats && rows / 4 < kMostSmall && us(u * Hkv, (B * tiles * (lengths && B > 1 ? 2 : 3) / 3 + u - 1) / u) + 5.0 < us(wgs, tiles)) {
      r.units = (int)u;
      r.floats = need;
    }
    return r;
  }
  // 256-row workgroups, one a compute unit, 2 us a tile of 64 keys.  Equal ones run
  // in rounds; unequal ones (causal, documents), the longest first, end with the
  // mean load or the longest of them.  4 us to start and end; the joining launch 4
  // us and the partial results' bytes at 5 TB/s.
  const int64_t tiles = ((int64_t)Lk + kModKeys - 1) / kModKeys, qt = (int64_t)mod_tiles(Lq);
  const int64_t wgs = qt * B * H;
  if (qt > 4096) return r;  // (rounds enough)
  const int64_t total = mod_key_tiles(Lq, Lk, causal);  // of a head
  auto direct = [&](int s) {
    const int64_t rounds = (wgs * s + cus - 1) / cus;
    const double per = (double)(docs ? (tiles + 2) / 3 : tiles) / s;
    const double mean = 1.05 * (double)(docs ? (total + 2) / 3 : total) * B * H / cus;
    const double load = docs || causal ? (mean > per ? mean : per) : rounds * (double)((tiles + s - 1) / s);
    return load * 2.0 + rounds * 4.0 + (s > 1 ? 4.0 + (double)s * rows * 1056 / 5e6 : 0.0);
  };
  double best = direct(1);
  // How much of the keys a document leaves is not known here: a third is assumed, and
  // a tile's keys are cut only where the tiles leave half of the compute units without
  // one.
  for (int s = 2; s <= kMostRuns && s <= tiles && (!docs || wgs * s <= cus); ++s) {
    const size_t need = r.part + (size_t)s * rows * 129;  // a run's rows: 128 outputs and a log-sum-exp each
    if (need > max_floats || wgs * s > kMostTiles || rows / 16 >= kMostSmall) break;
    if (direct(s) < best) {
      best = direct(s);
      r.runs = s;
      r.floats = need;
    }
  }
  if (docs) return r;
  const ModPieces p = mod_pieces(B, H, Lq, Lk, tiles, [&](int64_t t) { return mod_row_tiles(t, Lq, Lk, causal); }, lengths, cus,
                                 r.part, 129, 2.0);
  if (p.n && p.floats <= max_floats && p.us < best) {
    r.runs = 1;
    r.pieces = p;
    r.floats = p.floats;
  }
  return r;
}

// For a call.  (Few rows: a prefix alone leaves every batch the same keys, those up to
// its last query.)
inline ModSplit mod_fwd_split(const ModCall& c, int cus, size_t max_floats) {
  const bool own = mod_few(c.H, c.Hkv, c.Lq) ? c.s.kv_valid_len || c.s.q_start : mod_own_lengths(c.s);
  return mod_fwd_split(c.B, c.H, c.Hkv, c.Lq, c.Lk, c.s.k_doc != nullptr, c.s.causal != 0, own, cus, max_floats);
}

// ---- backward ----
//
// D and the log-sum-exps as the key side takes them, the flags of rows that see
// nothing, and the key side's partial sums.  A
// workgroup of the key side streams the query tiles (64 rows) that may see its 256
// keys, for every query head of its group.  Tiles of more than `quantum` of these
// are given to ceil(stream / quantum) workgroups (`runs` at most) whose fp32 dK and
// dV a further launch adds.  Chosen is the least time, in units of one tile's (4
// us): rounds of equal workgroups; one round of unequal ones, or the mean load and
// half a run where they are more; 2 to start and end a workgroup; 2 for the further launch; the
// partial sums written and read, 20 MB in a tile's time.  (2 x 2049 causal, 16 heads
// on 4, cap and bias: three runs of every tile 177 + 11 us, up to six 105 + 13.)
struct ModBwdSplit {
  int runs, quantum;
  size_t delta, nlse, empty, counts, part;  // first values of these in the workspace (document ranges at 0)
  size_t least, floats;  // values of the workspace: for one run and whole query tiles, for this
  ModPieces dq, dkdv;    // (the query side's partial sums lie where the key side's come later)
};

// Tiles of the stream of key tile t, where queries stand at their default positions.
inline int64_t mod_stream(int t, int rep, int Lq, int Lk, bool causal) {
  const int64_t qt = (Lq + 63) / 64, first = causal ? (int64_t)t * kModRows - (Lk - Lq) : 0;
  const int64_t n = first > 0 ? qt - first / 64 : qt;
  return n > 0 ? rep * n : 0;
}

inline ModBwdSplit mod_bwd_split(int B, int H, int Hkv, int Lq, int Lk, bool docs, bool causal, bool lengths, int cus,
                                 size_t max_floats) {
  auto up = [](size_t x) { return (x + 63) / 64 * 64; };
  ModBwdSplit r;
  r.runs = 1;
  r.quantum = 1 << 30;
  r.delta = up(mod_doc_floats(B, Lq, Lk, docs));
  r.nlse = up(r.delta + (size_t)B * H * Lq);
  r.empty = up(r.nlse + (size_t)B * H * Lq);
  r.counts = r.empty + (size_t)B * mod_ranges(Lq);
  r.least = r.floats = r.counts + (size_t)B * mod_tiles(Lk);
  r.part = up(r.least);
  r.dq.n = r.dkdv.n = 0;
  if (B == 0 || H == 0 || Lq == 0 || Lk == 0) return r;
  const int kt = (int)mod_tiles(Lk);
  const int64_t heads = (int64_t)B * Hkv;
  // how much of a stream a document leaves is not known here: a third is taken
  auto stream = [&](int t) {
    const int64_t n = mod_stream(t, H / Hkv, Lq, Lk, causal);
    return docs ? (n + 2) / 3 : n;
  };
  const int64_t longest = stream(0);
  const size_t run = 2 * (size_t)B * Lk * Hkv * 128;  // partial values of a run
  double best = 1e30;
  auto consider = [&](int64_t q) {  // runs of at most q tiles
    const int s = (int)((longest + q - 1) / q);
    const size_t need = r.part + s * run;
    if (s > 1 && (s > kMostRuns || need > max_floats || s * run > ((size_t)96 << 20))) return;
    int64_t total = 0, wgs = 0, partial = 0;
    for (int t = 0; t < kt; ++t) {
      const int64_t n = stream(t), w = n > q ? (n + q - 1) / q : 1;
      total += n;
      wgs += w;
      if (w > 1) partial += w;
    }
    total *= heads;
    wgs *= heads;
    partial *= heads;
    const int64_t rounds = (wgs + cus - 1) / cus;
    const double load = (!causal && !docs) || rounds == 1 ? (double)rounds * (q + 2)
                                                           : (double)(total + 2 * wgs) / cus + 0.5 * total / wgs;
    const double cost = (load > q + 2 ? load : q + 2) + (s > 1 ? 2.0 + partial * (2.0 * 2 * kModRows * 128 * 4 / 20e6) : 0.0);
    if (cost < best) {
      best = cost;
      r.runs = s;
      r.quantum = s > 1 ? (int)q : 1 << 30;
      r.floats = s > 1 ? need : r.least;
    }
  };
  if (longest == 0) return r;
  consider(longest);
  for (int s = 2; s <= kMostRuns && s <= longest; ++s) consider((longest + s - 1) / s);
  // and the shortest runs that one round has room for
  int64_t lo = 1, hi = longest;
  while (lo < hi) {
    const int64_t q = (lo + hi) / 2;
    int64_t wgs = 0;
    for (int t = 0; t < kt; ++t) wgs += stream(t) > q ? (stream(t) + q - 1) / q : 1;
    if (wgs * heads <= cus) hi = q;
    else lo = q + 1;
  }
  consider(lo);
  if (!docs && kt <= 4096) {
    // Pieces: 4 us a tile.  Where the batches have lengths of their own the runs above
    // are made for streams that are not there, and end unevenly.  (Both with the joining
    // launch; 2 x 4001, 16 heads on 4, causal: runs 301 us, pieces 278; with prefixes of
    // 1000 and 2300: 531 and 321; 2 x 2049 causal: 105 and 116.)
    const ModPieces p = mod_pieces(B, Hkv, Lk, Lq, mod_stream(0, H / Hkv, Lq, Lk, false),
                                   [&](int64_t t) { return mod_stream((int)t, H / Hkv, Lq, Lk, causal); }, lengths, cus, r.part, 256, 4.0);
    if (p.n && p.floats <= max_floats && p.us < best * 4.0 * (lengths ? 1.3 : 0.95)) {
      r.dkdv = p;
      r.runs = 1;
      r.quantum = 1 << 30;
      r.floats = p.floats;
    }
  }
  // Query side: 256-row workgroups with all of their keys (as in the forward; 2.6 us
  // a tile and 4 to start and end), or pieces.
  const int64_t qt = (int64_t)mod_tiles(Lq), wgs = qt * B * H;
  if (docs || qt > 4096) return r;
  const int64_t tiles = ((int64_t)Lk + kModKeys - 1) / kModKeys, rounds = (wgs + cus - 1) / cus;
  const double mean = 1.05 * (double)mod_key_tiles(Lq, Lk, causal) * B * H / cus;
  const double load = causal ? (mean > tiles ? mean : tiles) : (double)rounds * tiles;
  const ModPieces p = mod_pieces(B, H, Lq, Lk, tiles, [&](int64_t t) { return mod_row_tiles(t, Lq, Lk, causal); }, lengths, cus,
                                 r.part, 128, 2.6);
  if (p.n && p.floats <= max_floats && p.us < load * 2.6 + rounds * 4.0) {
    r.dq = p;
    if (p.floats > r.floats) r.floats = p.floats;
  }
  return r;
}

inline ModBwdSplit mod_bwd_split(const ModCall& c, int cus, size_t max_floats) {
  return mod_bwd_split(c.B, c.H, c.Hkv, c.Lq, c.Lk, c.s.k_doc != nullptr, c.s.causal != 0, mod_own_lengths(c.s), cus, max_floats);
}

__attribute__((weak)) hipError_t launch_attn_mod_fwd(const ModFwd& a, hipStream_t stream);
__attribute__((weak)) hipError_t launch_attn_mod_bwd(const ModBwd& a, hipStream_t stream);

// Between the attn_mod_*.hip files.
struct ModRanges {
  const int2 *k, *q;              // [B][mod_ranges(Lk)], [B][mod_ranges(Lq)], or null
  const int32_t *q_order, *k_order; // tiles b * mod_tiles + t of most work first, or null (in order)
};
// Ranges (and, `order`: the tiles' orders) into ws.
hipError_t launch_mod_ranges(const ModCall& c, float* ws, bool q_order, bool k_order, ModRanges* out, hipStream_t stream);
hipError_t launch_mod_few(const ModFwd& a, const ModSplit& s, const ModRanges& r, hipStream_t stream);

}  // namespace vidax
