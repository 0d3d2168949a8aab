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
inline size_t mod_ranges(int L) { return ((size_t)L + 63) / 64 * 2; }
inline size_t mod_doc_floats(int B, int Lq, int Lk, bool docs) {
  return docs ? (size_t)B * (mod_ranges(Lk) + mod_ranges(Lq)) * 2 : 0;
}

// ---- forward ----
//
// Few rows (a group's query heads times the queries, at most kFewRows): the form
// for single tokens, whose workgroups stream a run of keys and hold all rows.
// Otherwise tiles of 256 query rows.  Either may cut the keys into runs, one
// workgroup each, and join them in a second launch.
constexpr int kModRows = 256;
constexpr int kModKeys = 64;
constexpr int kFewRows = 32;

struct ModSplit {
  bool few;
  int runs;
  size_t part;    // first value of the partial results in the workspace
  size_t floats;  // values of the workspace
};

inline ModSplit mod_fwd_split(int B, int H, int Hkv, int Lq, int Lk, bool docs, int cus, size_t max_floats) {
  ModSplit r;
  r.runs = 1;
  r.part = (mod_doc_floats(B, Lq, Lk, docs) + 63) / 64 * 64;
  const int rep = Hkv > 0 ? H / Hkv : 1;
  r.few = false;
  (void)rep;
  const int64_t tiles = ((int64_t)Lk + kModKeys - 1) / kModKeys;
  const int64_t wgs = r.few ? (int64_t)B * Hkv : (int64_t)((Lq + kModRows - 1) / kModRows) * B * H;
  const int64_t rows = (int64_t)B * H * Lq;
  if (wgs > 0 && tiles > 0) {
    // least time, in tiles of a workgroup: rounds x (tiles a run + start and
    // end) + the joining launch and its bytes
    const int slots = cus;
    const double start = 3.0;
    double best = 1e30;
    for (int s = 1; s <= 64 && s <= tiles; ++s) {
      if (s > 1 && r.part + (size_t)s * rows * 129 > max_floats) break;
      const int64_t rounds = (wgs * s + slots - 1) / slots;
      const int64_t per = (tiles + s - 1) / s;
      const double cost = rounds * (per + start) + (s > 1 ? 3.0 + (double)s * rows * 1056 / 8e6 : 0.0);
      if (cost < best) {
        best = cost;
        r.runs = s;
      }
    }
  }
  // a run's rows: 128 outputs and a log-sum-exp each
  r.floats = r.runs > 1 ? r.part + (size_t)r.runs * rows * 129 : mod_doc_floats(B, Lq, Lk, docs);
  return r;
}

__attribute__((weak)) hipError_t launch_attn_mod_fwd(const ModFwd& a, hipStream_t stream);
__attribute__((weak)) hipError_t launch_attn_mod_bwd(const ModBwd& a, hipStream_t stream);

// Between the attn_mod_*.hip files.
struct ModRanges {
  const int2 *k, *q;  // [B][mod_ranges(Lk)], [B][mod_ranges(Lq)], or null
};
hipError_t launch_mod_ranges(const ModCall& c, float* ws, ModRanges* out, hipStream_t stream);
hipError_t launch_mod_few(const ModFwd& a, const ModSplit& s, hipStream_t stream);
hipError_t launch_mod_join(const ModFwd& a, const ModSplit& s, hipStream_t stream);

}  // namespace vidax
