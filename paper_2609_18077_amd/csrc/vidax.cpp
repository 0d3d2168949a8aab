// C ABI of libvidax: argument validation and dispatch to the gfx950 kernels.
//
// Every check runs before any HIP call, so a rejected call has no side effect
// (and can be exercised on a machine without a GPU).
#include <math.h>
#include <stdint.h>

#include "../../include/vidax.h"
#include "launch.hpp"
#include "launch_block.hpp"
#include "launch_mod.hpp"

static_assert(VIDAX_NOALLOC_MAX_ROWS == vidax::kNoAllocRows, "allocation-free scratch size");

namespace {

using vidax::RopeParams;

bool aligned(const void* p, uintptr_t a) { return ((uintptr_t)p & (a - 1)) == 0; }

// [p, p + bytes) and [q, q + bytes_q) overlap?
bool overlaps(const void* p, uint64_t bytes, const void* q, uint64_t bytes_q) {
  if (bytes == 0 || bytes_q == 0) return false;
  const uintptr_t a0 = (uintptr_t)p, a1 = a0 + bytes;
  const uintptr_t b0 = (uintptr_t)q, b1 = b0 + bytes_q;
  return a0 < b1 && b0 < a1;
}

// Elements of a [B, L, H, d] tensor, or -1 if it does not fit in int64 byte offsets.
int64_t numel4(int64_t B, int64_t L, int64_t H, int64_t d) {
  const int64_t lim = INT64_C(1) << 60;
  int64_t n = 1;
  for (int64_t x : {B, L, H, d}) {
    if (x != 0 && n > lim / x) return -1;
    n *= x;
  }
  return n;
}

// Validates a rotary descriptor against the token counts it will see and
// converts it.  `max_tokens`: rotated tokens must not exceed it.
vidax_status make_rope(const vidax_rope3d_desc* r, int64_t max_tokens, int32_t d, RopeParams* out) {
  if (r->grid_t < 1 || r->grid_h < 1 || r->grid_w < 1) return VIDAX_ERR_INVALID_ARG;
  if (r->dim_t < 0 || r->dim_h < 0 || r->dim_w < 0) return VIDAX_ERR_INVALID_ARG;
  if ((r->dim_t | r->dim_h | r->dim_w) & 1) return VIDAX_ERR_INVALID_ARG;
  if ((int64_t)r->dim_t + r->dim_h + r->dim_w != d) return VIDAX_ERR_INVALID_ARG;
  if (!(r->theta > 0.0f) || !isfinite(r->theta)) return VIDAX_ERR_INVALID_ARG;
  if (r->pair_mode != 0 && r->pair_mode != 1) return VIDAX_ERR_INVALID_ARG;
  if (r->keys_prerotated != 0 && r->keys_prerotated != 1) return VIDAX_ERR_INVALID_ARG;
  const int64_t n_rot = (int64_t)r->grid_t * r->grid_h * r->grid_w;
  if (n_rot > max_tokens) return VIDAX_ERR_INVALID_ARG;
  const int64_t entries = (int64_t)r->grid_t * (r->dim_t / 2) + (int64_t)r->grid_h * (r->dim_h / 2) +
                          (int64_t)r->grid_w * (r->dim_w / 2);
  if (entries > vidax::kRopeTableMax) return VIDAX_ERR_UNSUPPORTED;
  out->enabled = 1;
  out->gt = r->grid_t;
  out->gh = r->grid_h;
  out->gw = r->grid_w;
  out->dt = r->dim_t;
  out->dh = r->dim_h;
  out->dw = r->dim_w;
  out->pair_mode = r->pair_mode;
  out->keys_prerotated = r->keys_prerotated;
  out->inverse = 0;
  out->n_rot = (int)n_rot;
  out->base1 = r->grid_t * (r->dim_t / 2);
  out->base2 = out->base1 + r->grid_h * (r->dim_h / 2);
  out->n_entries = (int)entries;
  out->log2_theta = log2f(r->theta);
  return VIDAX_OK;
}

RopeParams no_rope() {
  RopeParams p{};
  p.enabled = 0;
  p.gt = p.gh = p.gw = 1;
  return p;
}

enum class AttnImpl { kMatrixCore, kNaive };

vidax_status attn_common(AttnImpl impl, const void* q, const void* k, const void* v, void* o, float* lse,
                         int32_t B, int32_t H, int32_t Lq, int32_t Lk, int32_t d, float scale,
                         const int32_t* kv_valid_len, const vidax_rope3d_desc* rope, hipStream_t stream) {
  if (B < 0 || H < 0 || Lq < 0 || Lk < 0 || d < 0) return VIDAX_ERR_INVALID_ARG;
  const int64_t nq = numel4(B, Lq, H, d), nk = numel4(B, Lk, H, d);
  if (nq < 0 || nk < 0) return VIDAX_ERR_INVALID_ARG;
  // a pointer may be NULL only when its tensor has no elements
  if ((nq > 0 && (!q || !o)) || (nk > 0 && (!k || !v))) return VIDAX_ERR_INVALID_ARG;
  if (!aligned(q, 16) || !aligned(k, 16) || !aligned(v, 16) || !aligned(o, 16)) return VIDAX_ERR_INVALID_ARG;
  if (lse && !aligned(lse, 4)) return VIDAX_ERR_INVALID_ARG;
  if (kv_valid_len && !aligned(kv_valid_len, 4)) return VIDAX_ERR_INVALID_ARG;
  if (!isfinite(scale)) return VIDAX_ERR_INVALID_ARG;
  if (d != vidax::kHeadDim) return VIDAX_ERR_UNSUPPORTED;
  const uint64_t qbytes = (uint64_t)nq * 2, kbytes = (uint64_t)nk * 2;
  if (overlaps(o, qbytes, q, qbytes) || overlaps(o, qbytes, k, kbytes) || overlaps(o, qbytes, v, kbytes))
    return VIDAX_ERR_INVALID_ARG;
  // outputs (o, lse) must not overlap each other or any input (kv_valid_len included)
  const uint64_t lbytes = lse ? (uint64_t)B * H * Lq * 4 : 0, vbytes = kv_valid_len ? (uint64_t)B * 4 : 0;
  if (overlaps(lse, lbytes, o, qbytes) || overlaps(lse, lbytes, q, qbytes) || overlaps(lse, lbytes, k, kbytes) ||
      overlaps(lse, lbytes, v, kbytes) || overlaps(kv_valid_len, vbytes, o, qbytes) ||
      overlaps(kv_valid_len, vbytes, lse, lbytes))
    return VIDAX_ERR_INVALID_ARG;
  RopeParams rp = no_rope();
  if (rope) {
    const vidax_status st = make_rope(rope, Lq < Lk ? Lq : Lk, d, &rp);
    if (st != VIDAX_OK) return st;
    if (impl == AttnImpl::kMatrixCore && !vidax::attn_rope_supported(rp)) return VIDAX_ERR_UNSUPPORTED;
  }
  // the kernels address one batch of q, o (and of k, v within a tile) with
  // 32-bit buffer offsets: one batch of a tensor must stay below 2 GiB
  if ((int64_t)(Lq > Lk ? Lq : Lk) * H * d * 2 > INT32_MAX - 4096) return VIDAX_ERR_UNSUPPORTED;
  // one workgroup per 256 (matrix core) or 64 (naive) query rows of each (b, h)
  const int64_t rows = impl == AttnImpl::kMatrixCore ? 256 : 64;
  const int64_t grid = ((int64_t)Lq + rows - 1) / rows * B * H;
  if (grid > INT32_MAX) return VIDAX_ERR_UNSUPPORTED;
  if (B == 0 || H == 0 || Lq == 0) return VIDAX_OK;

  hipError_t e;
  if (impl == AttnImpl::kMatrixCore)
    e = vidax::launch_attn_fwd((const uint16_t*)q, (const uint16_t*)k, (const uint16_t*)v, (uint16_t*)o, lse, B, H,
                               Lq, Lk, scale, kv_valid_len, rp, stream);
  else
    e = vidax::launch_attn_naive((const uint16_t*)q, (const uint16_t*)k, (const uint16_t*)v, (uint16_t*)o, lse, B,
                                 H, Lq, Lk, scale, kv_valid_len, rp, stream);
  return e == hipSuccess ? VIDAX_OK : VIDAX_ERR_LAUNCH;
}

vidax_status rope3d_common(bool inverse, const void* x, void* y, int32_t B, int32_t L, int32_t H, int32_t d,
                          const vidax_rope3d_desc* rope, hipStream_t stream) {
  if (B < 0 || L < 0 || H < 0 || d < 0) return VIDAX_ERR_INVALID_ARG;
  if (!rope) return VIDAX_ERR_INVALID_ARG;
  const int64_t n = numel4(B, L, H, d);
  if (n < 0) return VIDAX_ERR_INVALID_ARG;
  if (n > 0 && (!x || !y)) return VIDAX_ERR_INVALID_ARG;
  if (!aligned(x, 16) || !aligned(y, 16)) return VIDAX_ERR_INVALID_ARG;
  if (d != vidax::kHeadDim) return VIDAX_ERR_UNSUPPORTED;
  if (x != y && overlaps(x, (uint64_t)n * 2, y, (uint64_t)n * 2)) return VIDAX_ERR_INVALID_ARG;
  vidax_rope3d_desc r = *rope;
  r.keys_prerotated = 0;  // attention-only field
  RopeParams rp;
  const vidax_status st = make_rope(&r, L, d, &rp);
  if (st != VIDAX_OK) return st;
  rp.inverse = inverse ? 1 : 0;
  if (B == 0 || L == 0 || H == 0) return VIDAX_OK;
  const hipError_t e = vidax::launch_rope3d((const uint16_t*)x, (uint16_t*)y, B, L, H, rp, stream);
  return e == hipSuccess ? VIDAX_OK : VIDAX_ERR_LAUNCH;
}

// The backward's checks; `noalloc`: D goes to the library's fixed device
// array (the workspace must be NULL, of 0 values) instead of the caller's.
vidax_status bwd_common(bool noalloc, const void* q, const void* k, const void* v, const void* o, const void* dout,
                        const float* lse, void* dq, void* dk, void* dv, float* ws, size_t ws_floats, int32_t B,
                        int32_t H, int32_t Lq, int32_t Lk, int32_t d, float scale, const int32_t* kv_valid_len,
                        hipStream_t stream) {
  if (B < 0 || H < 0 || Lq < 0 || Lk < 0 || d < 0) return VIDAX_ERR_INVALID_ARG;
  const int64_t nq = numel4(B, Lq, H, d), nk = numel4(B, Lk, H, d);
  if (nq < 0 || nk < 0) return VIDAX_ERR_INVALID_ARG;
  const int64_t nrow = (int64_t)B * H * Lq;  // lse, D
  if ((nq > 0 && (!q || !o || !dout || !dq)) || (nk > 0 && (!k || !v || !dk || !dv)) ||
      (nrow > 0 && (!lse || (!noalloc && !ws))))
    return VIDAX_ERR_INVALID_ARG;
  if (noalloc && (ws || ws_floats)) return VIDAX_ERR_INVALID_ARG;
  if (!noalloc && (uint64_t)ws_floats < (uint64_t)nrow) return VIDAX_ERR_INVALID_ARG;
  if (ws_floats > ((uint64_t)1 << 60)) return VIDAX_ERR_INVALID_ARG;
  if (!ws) ws_floats = 0;
  for (const void* p : {q, k, v, o, dout, (const void*)dq, (const void*)dk, (const void*)dv})
    if (!aligned(p, 16)) return VIDAX_ERR_INVALID_ARG;
  if (!aligned(lse, 16) || !aligned(ws, 16)) return VIDAX_ERR_INVALID_ARG;
  if (kv_valid_len && !aligned(kv_valid_len, 4)) return VIDAX_ERR_INVALID_ARG;
  if (!isfinite(scale)) return VIDAX_ERR_INVALID_ARG;
  if (d != vidax::kHeadDim) return VIDAX_ERR_UNSUPPORTED;
  const uint64_t qb = (uint64_t)nq * 2, kb = (uint64_t)nk * 2, rb = (uint64_t)nrow * 4;
  const uint64_t vb = kv_valid_len ? (uint64_t)B * 4 : 0;
  // outputs (dq, dk, dv, the workspace) must not overlap each other or any input
  const void* outs[4] = {dq, dk, dv, ws};
  const uint64_t osz[4] = {qb, kb, kb, (uint64_t)ws_floats * 4};
  const void* ins[7] = {q, k, v, o, dout, lse, kv_valid_len};
  const uint64_t isz[7] = {qb, kb, kb, qb, qb, rb, vb};
  for (int i = 0; i < 4; ++i) {
    for (int j = 0; j < 7; ++j)
      if (overlaps(outs[i], osz[i], ins[j], isz[j])) return VIDAX_ERR_INVALID_ARG;
    for (int j = i + 1; j < 4; ++j)
      if (overlaps(outs[i], osz[i], outs[j], osz[j])) return VIDAX_ERR_INVALID_ARG;
  }
  // grids: dq at most ceil(Lq / 128) B H, key side ceil(Lk / 128) B H or 64 per CU
  // (its bound is a wide one, kept so that the same calls are refused)
  const int64_t grid_q = ((int64_t)Lq + 127) / 128 * B * H, grid_k = ((int64_t)Lk + 127) / 128 * 16 * B * H;
  if (grid_q > INT32_MAX || grid_k > INT32_MAX) return VIDAX_ERR_UNSUPPORTED;
  // buffer offsets are 32-bit and relative to a 64-row tile
  if ((int64_t)64 * H * d * 2 > INT32_MAX - 4096) return VIDAX_ERR_UNSUPPORTED;
  if (noalloc && nrow > vidax::kNoAllocRows) return VIDAX_ERR_TOO_LARGE;
  if (B == 0 || H == 0 || (Lq == 0 && Lk == 0)) return VIDAX_OK;
  const hipError_t e =
      noalloc ? vidax::launch_attn_bwd_noalloc((const uint16_t*)q, (const uint16_t*)k, (const uint16_t*)v,
                                               (const uint16_t*)o, (const uint16_t*)dout, lse, (uint16_t*)dq,
                                               (uint16_t*)dk, (uint16_t*)dv, B, H, Lq, Lk, scale, kv_valid_len, stream)
              : vidax::launch_attn_bwd((const uint16_t*)q, (const uint16_t*)k, (const uint16_t*)v, (const uint16_t*)o,
                                       (const uint16_t*)dout, lse, ws, ws_floats, (uint16_t*)dq, (uint16_t*)dk,
                                       (uint16_t*)dv, B, H, Lq, Lk, scale, kv_valid_len, stream);
  return e == hipSuccess ? VIDAX_OK : VIDAX_ERR_LAUNCH;
}

// A buffer of a call, for the checks that all entry points below share.
struct Buf {
  const void* p;
  uint64_t bytes;
};

// Outputs overlap each other or an input?  (`in_place`: this output may be
// exactly this input.)
template <int NO, int NI>
bool any_overlap(const Buf (&outs)[NO], const Buf (&ins)[NI], int io_out = -1, int io_in = -1) {
  for (int i = 0; i < NO; ++i) {
    if (!outs[i].p) continue;
    for (int j = 0; j < NI; ++j) {
      if (!ins[j].p || (i == io_out && j == io_in && outs[i].p == ins[j].p)) continue;
      if (overlaps(outs[i].p, outs[i].bytes, ins[j].p, ins[j].bytes)) return true;
    }
    for (int j = i + 1; j < NO; ++j)
      if (outs[j].p && overlaps(outs[i].p, outs[i].bytes, outs[j].p, outs[j].bytes)) return true;
  }
  return false;
}

// The checks that attention with score modifiers shares between forward and
// backward; bufs: the descriptor's arrays.
vidax_status mod_common(int32_t B, int32_t H, int32_t Hkv, int32_t Lq, int32_t Lk, int32_t d, float scale,
                        const vidax_score_desc* s, bool backward, vidax::ModCall* c, Buf (&bufs)[6]) {
  if (B < 0 || H < 0 || Hkv < 0 || Lq < 0 || Lk < 0 || d < 0) return VIDAX_ERR_INVALID_ARG;
  if ((Hkv == 0) != (H == 0) || (Hkv > 0 && H % Hkv != 0)) return VIDAX_ERR_INVALID_ARG;
  if (numel4(B, Lq, H, d) < 0 || numel4(B, Lk, Hkv, d) < 0) return VIDAX_ERR_INVALID_ARG;
  if (!isfinite(scale)) return VIDAX_ERR_INVALID_ARG;
  static const vidax_score_desc plain{};
  if (!s) s = &plain;
  if (s->causal != 0 && s->causal != 1) return VIDAX_ERR_INVALID_ARG;
  // (scale / cap has to be a number, too)
  if (!(s->cap >= 0.0f) || !isfinite(s->cap) || (s->cap > 0.0f && !isfinite(scale / s->cap))) return VIDAX_ERR_INVALID_ARG;
  const uint64_t nq = (uint64_t)B * Lq, nk = (uint64_t)B * Lk;
  if ((nq > 0 && nk > 0 && (s->q_doc != nullptr) != (s->k_doc != nullptr)) || (s->prefix_len && !s->causal))
    return VIDAX_ERR_INVALID_ARG;
  const Buf all[6] = {{s->slopes, (uint64_t)H * 4}, {s->q_doc, nq * 4}, {s->k_doc, nk * 4},
                      {s->kv_valid_len, (uint64_t)B * 4}, {s->prefix_len, (uint64_t)B * 4}, {s->q_start, (uint64_t)B * 4}};
  for (int i = 0; i < 6; ++i) {
    if (!aligned(all[i].p, 4)) return VIDAX_ERR_INVALID_ARG;
    bufs[i] = all[i];
  }
  if (d != vidax::kHeadDim) return VIDAX_ERR_UNSUPPORTED;
  // buffer offsets are 32-bit: within a batch of q, within 64 tokens of k, and within a row of ids
  if ((int64_t)Lq * H * d * 2 > INT32_MAX - 4096 || (int64_t)64 * Hkv * d * 2 > INT32_MAX - 4096 ||
      (int64_t)64 * H * d * 2 > INT32_MAX - 4096 || Lk > (1 << 28) || Lq > (1 << 28))
    return VIDAX_ERR_UNSUPPORTED;
  // launch sizes, and 32-bit numbers of tiles and rows
  const bool docs = s->q_doc && s->k_doc;
  const int64_t tiles = ((int64_t)Lq + 127) / 128 + ((int64_t)Lk + 127) / 128;
  if ((__int128)tiles * B * H * 64 > INT32_MAX || (__int128)B * H * Lq > INT32_MAX ||
      !vidax::mod_launches_fit(B, H, Hkv, Lq, Lk, docs, backward))
    return VIDAX_ERR_UNSUPPORTED;
  *c = vidax::ModCall{B, H, Hkv, Lq, Lk, scale,
                      vidax::ModScore{s->causal, s->cap > 1e30f ? 0.0f : s->cap,  // (tanh is then the identity in fp32)
                                      s->slopes, docs ? s->q_doc : nullptr, docs ? s->k_doc : nullptr, s->kv_valid_len,
                                      s->prefix_len, s->q_start}};
  return VIDAX_OK;
}

// Bytes from a modulation's first element to behind its last, or -1 if its
// strides are not allowed.
int64_t mod_bytes(const vidax_block_mod& m, int64_t B, int64_t L, int64_t C) {
  if (!m.p) return 0;
  if (m.batch_stride < 0 || m.token_stride < 0 || (m.batch_stride | m.token_stride) & 3) return -1;
  const int64_t lim = INT64_C(1) << 58;
  if ((m.batch_stride && B > lim / m.batch_stride) || (m.token_stride && L > lim / m.token_stride)) return -1;
  return B && L ? ((B - 1) * m.batch_stride + (L - 1) * m.token_stride + C) * 4 : 0;
}

// The checks that the block norm's forward and backward share.
vidax_status block_norm_common(int32_t B, int32_t L, int32_t C, const vidax_block_norm_desc* d, bool branch,
                               vidax::BlockNorm* n, Buf (&mods)[5]) {
  if (B < 0 || L < 0 || C < 0 || !d) return VIDAX_ERR_INVALID_ARG;
  if (numel4(B, L, C, 4) < 0) return VIDAX_ERR_INVALID_ARG;
  if ((d->stream_fp32 != 0 && d->stream_fp32 != 1) || (d->norm != 1 && d->norm != 2) || d->post < 0 || d->post > 2 ||
      (d->per_token != 0 && d->per_token != 1))
    return VIDAX_ERR_INVALID_ARG;
  if (!(d->eps >= 0.0f) || !isfinite(d->eps) || !isfinite(d->alpha)) return VIDAX_ERR_INVALID_ARG;
  const bool empty = B == 0 || L == 0 || C == 0;  // (the branch may then be NULL like any tensor)
  if (!branch && !empty && (d->post || d->gate.p)) return VIDAX_ERR_INVALID_ARG;
  if (!d->post && d->post_gain) return VIDAX_ERR_INVALID_ARG;
  const vidax_block_mod* m[3] = {&d->gate, &d->scale, &d->shift};
  for (int i = 0; i < 3; ++i) {
    const int64_t bytes = mod_bytes(*m[i], B, L, C);
    if (bytes < 0 || !aligned(m[i]->p, 16)) return VIDAX_ERR_INVALID_ARG;
    mods[i] = Buf{m[i]->p, (uint64_t)bytes};
  }
  if (!aligned(d->gain, 16) || !aligned(d->post_gain, 16)) return VIDAX_ERR_INVALID_ARG;
  mods[3] = Buf{d->gain, (uint64_t)C * 4};
  mods[4] = Buf{d->post_gain, (uint64_t)C * 4};
  if (C % 8 != 0 || C > vidax::kBlockMaxC) return VIDAX_ERR_UNSUPPORTED;
  if ((int64_t)B * L > INT32_MAX) return VIDAX_ERR_UNSUPPORTED;  // rows
  auto mod = [](const vidax_block_mod& x) { return vidax::BlockMod{x.p, x.batch_stride, x.token_stride}; };
  *n = vidax::BlockNorm{B, L, C, d->stream_fp32, d->norm, d->post, d->eps, d->alpha, d->gain, d->post_gain,
                        mod(d->gate), mod(d->scale), mod(d->shift)};
  return VIDAX_OK;
}

}  // namespace

extern "C" {

vidax_status vidax_attn_bwd(const void* q, const void* k, const void* v, const void* o, const void* dout,
                            const float* lse, void* dq, void* dk, void* dv, float* workspace,
                            size_t workspace_floats, int32_t B, int32_t H, int32_t Lq, int32_t Lk, int32_t d,
                            float scale, const int32_t* kv_valid_len, hipStream_t stream) {
  return bwd_common(false, q, k, v, o, dout, lse, dq, dk, dv, workspace, workspace_floats, B, H, Lq, Lk, d, scale,
                    kv_valid_len, stream);
}

size_t vidax_attn_bwd_workspace_floats(int32_t B, int32_t H, int32_t Lq, int32_t Lk, int32_t d) {
  if (B < 0 || H < 0 || Lq < 0 || Lk < 0 || d != vidax::kHeadDim) return 0;
  if (numel4(B, Lq, H, d) < 0 || numel4(B, Lk, H, d) < 0) return 0;
  return vidax::attn_bwd_split(B, H, Lq, Lk, vidax::device_cu_count(), SIZE_MAX, false).floats;
}

vidax_status vidax_attn_bwd_noalloc(const void* q, const void* k, const void* v, const void* o, const void* dout,
                                    const float* lse, void* dq, void* dk, void* dv, int32_t B, int32_t H,
                                    int32_t Lq, int32_t Lk, int32_t d, float scale, const int32_t* kv_valid_len,
                                    hipStream_t stream) {
  return bwd_common(true, q, k, v, o, dout, lse, dq, dk, dv, nullptr, 0, B, H, Lq, Lk, d, scale, kv_valid_len,
                    stream);
}

vidax_status vidax_qk_norm_rope(const void* x, void* y, const float* gain, float eps, int32_t B, int32_t L, int32_t H,
                                int32_t d, const vidax_rope3d_desc* rope, hipStream_t stream) {
  if (B < 0 || L < 0 || H < 0 || d < 0) return VIDAX_ERR_INVALID_ARG;
  const int64_t n = numel4(B, L, H, d);
  if (n < 0) return VIDAX_ERR_INVALID_ARG;
  if (n > 0 && (!x || !y)) return VIDAX_ERR_INVALID_ARG;
  if (!aligned(x, 16) || !aligned(y, 16) || !aligned(gain, 16)) return VIDAX_ERR_INVALID_ARG;
  if (!(eps >= 0.0f) || !isfinite(eps)) return VIDAX_ERR_INVALID_ARG;
  if (d != vidax::kHeadDim) return VIDAX_ERR_UNSUPPORTED;
  if (x != y && overlaps(x, (uint64_t)n * 2, y, (uint64_t)n * 2)) return VIDAX_ERR_INVALID_ARG;
  if (gain && overlaps(gain, (uint64_t)d * 4, y, (uint64_t)n * 2)) return VIDAX_ERR_INVALID_ARG;
  RopeParams rp = no_rope();
  if (rope) {
    vidax_rope3d_desc r = *rope;
    r.keys_prerotated = 0;  // attention-only field
    const vidax_status st = make_rope(&r, L, d, &rp);
    if (st != VIDAX_OK) return st;
  }
  if (B == 0 || L == 0 || H == 0) return VIDAX_OK;
  const hipError_t e = vidax::launch_qk_norm((const uint16_t*)x, (uint16_t*)y, gain, eps, B, L, H, rp, stream);
  return e == hipSuccess ? VIDAX_OK : VIDAX_ERR_LAUNCH;
}

vidax_status vidax_rope3d(const void* x, void* y, int32_t B, int32_t L, int32_t H, int32_t d,
                          const vidax_rope3d_desc* rope, hipStream_t stream) {
  return rope3d_common(false, x, y, B, L, H, d, rope, stream);
}

vidax_status vidax_rope3d_transpose(const void* x, void* y, int32_t B, int32_t L, int32_t H, int32_t d,
                                    const vidax_rope3d_desc* rope, hipStream_t stream) {
  return rope3d_common(true, x, y, B, L, H, d, rope, stream);
}

vidax_status vidax_attn_fwd(const void* q, const void* k, const void* v, void* o, float* lse, int32_t B, int32_t H,
                            int32_t Lq, int32_t Lk, int32_t d, float scale, const int32_t* kv_valid_len,
                            const vidax_rope3d_desc* rope, hipStream_t stream) {
  return attn_common(AttnImpl::kMatrixCore, q, k, v, o, lse, B, H, Lq, Lk, d, scale, kv_valid_len, rope, stream);
}

vidax_status vidax_attn_fwd_naive(const void* q, const void* k, const void* v, void* o, float* lse, int32_t B,
                                  int32_t H, int32_t Lq, int32_t Lk, int32_t d, float scale,
                                  const int32_t* kv_valid_len, const vidax_rope3d_desc* rope, hipStream_t stream) {
  return attn_common(AttnImpl::kNaive, q, k, v, o, lse, B, H, Lq, Lk, d, scale, kv_valid_len, rope, stream);
}

vidax_status vidax_na3d_fwd(const void* q, const void* k, const void* v, void* o, float* lse, int32_t B, int32_t H,
                            int32_t grid_t, int32_t grid_h, int32_t grid_w, int32_t d, int32_t win_t, int32_t win_h,
                            int32_t win_w, int32_t border, float scale, hipStream_t stream) {
  if (B < 0 || H < 0 || grid_t < 0 || grid_h < 0 || grid_w < 0 || d < 0) return VIDAX_ERR_INVALID_ARG;
  for (int32_t w : {win_t, win_h, win_w})
    if (w < 1 || (w & 1) == 0) return VIDAX_ERR_INVALID_ARG;
  if (border != 0 && border != 1) return VIDAX_ERR_INVALID_ARG;
  if (!isfinite(scale)) return VIDAX_ERR_INVALID_ARG;
  const int64_t L = (int64_t)grid_t * grid_h * grid_w;
  const int64_t n = numel4(B, L, H, d);
  if (n < 0) return VIDAX_ERR_INVALID_ARG;
  if (n > 0 && (!q || !k || !v || !o)) return VIDAX_ERR_INVALID_ARG;
  for (const void* p : {q, k, v, (const void*)o})
    if (!aligned(p, 16)) return VIDAX_ERR_INVALID_ARG;
  if (!aligned(lse, 4)) return VIDAX_ERR_INVALID_ARG;
  if (d != vidax::kHeadDim) return VIDAX_ERR_UNSUPPORTED;
  if (win_w > 11) return VIDAX_ERR_UNSUPPORTED;  // a wave's key runs are 16 positions along w
  if (n == 0) return VIDAX_OK;
  const uint64_t xb = (uint64_t)n * 2, lb = lse ? (uint64_t)B * H * L * 4 : 0;
  // outputs must not overlap each other or an input
  for (const void* in : {q, k, v})
    if (overlaps(o, xb, in, xb) || overlaps(lse, lb, in, xb)) return VIDAX_ERR_INVALID_ARG;
  if (overlaps(o, xb, lse, lb)) return VIDAX_ERR_INVALID_ARG;
  // 32-bit buffer offsets within one batch (plus a staged row past its end);
  // launch size
  if ((L + 32) * H * 256 > INT32_MAX) return VIDAX_ERR_UNSUPPORTED;
  const int64_t nwg = (int64_t)B * H * ((grid_t + 1) / 2) * ((grid_h + 3) / 4) * ((grid_w + 15) / 16);
  if (nwg > INT32_MAX) return VIDAX_ERR_UNSUPPORTED;
  const hipError_t e =
      vidax::launch_na3d_fwd((const uint16_t*)q, (const uint16_t*)k, (const uint16_t*)v, (uint16_t*)o, lse, B, H,
                             grid_t, grid_h, grid_w, win_t, win_h, win_w, border, scale, stream);
  return e == hipSuccess ? VIDAX_OK : VIDAX_ERR_LAUNCH;
}

vidax_status vidax_qkv_proj(const void* x, const void* w, const float* bias, const float* gain_q,
                            const float* gain_k, float eps, void* q, void* k, void* v, int32_t B, int32_t L,
                            int32_t H, int32_t d, int32_t C, const vidax_rope3d_desc* rope, hipStream_t stream) {
  if (B < 0 || L < 0 || H < 0 || d < 0 || C < 0) return VIDAX_ERR_INVALID_ARG;
  const int64_t M = (int64_t)B * L;
  const int64_t nx = numel4(M, C, 1, 1), nw = numel4(3, H, d, C), no = numel4(M, H, d, 1);
  if (nx < 0 || nw < 0 || no < 0) return VIDAX_ERR_INVALID_ARG;
  if (!(eps >= 0.0f) || !isfinite(eps)) return VIDAX_ERR_INVALID_ARG;
  if (no > 0 && (!q || !k || !v || (C > 0 && (!x || !w)))) return VIDAX_ERR_INVALID_ARG;
  for (const void* p : {x, w, (const void*)bias, (const void*)gain_q, (const void*)gain_k, (const void*)q,
                        (const void*)k, (const void*)v})
    if (!aligned(p, 16)) return VIDAX_ERR_INVALID_ARG;
  if (d != vidax::kHeadDim) return VIDAX_ERR_UNSUPPORTED;
  if (C % 64 != 0 || (C == 0 && no > 0)) return VIDAX_ERR_UNSUPPORTED;  // stages of 64 input channels
  RopeParams rp = no_rope();
  if (rope) {
    vidax_rope3d_desc r = *rope;
    r.keys_prerotated = 0;  // attention-only field
    const vidax_status st = make_rope(&r, L, d, &rp);
    if (st != VIDAX_OK) return st;
  }
  if (no == 0) return VIDAX_OK;
  const uint64_t ob = (uint64_t)no * 2;
  const void* outs[3] = {q, k, v};
  const void* ins[5] = {x, w, bias, gain_q, gain_k};
  const uint64_t isz[5] = {(uint64_t)nx * 2, (uint64_t)nw * 2, bias ? (uint64_t)3 * H * d * 4 : 0,
                           gain_q ? (uint64_t)d * 4 : 0, gain_k ? (uint64_t)d * 4 : 0};
  for (int i = 0; i < 3; ++i) {
    for (int j = 0; j < 5; ++j)
      if (overlaps(outs[i], ob, ins[j], isz[j])) return VIDAX_ERR_INVALID_ARG;
    for (int j = i + 1; j < 3; ++j)
      if (overlaps(outs[i], ob, outs[j], ob)) return VIDAX_ERR_INVALID_ARG;
  }
  // 32-bit buffer offsets within a 256-row tile; launch size
  if ((int64_t)256 * C * 2 > INT32_MAX) return VIDAX_ERR_UNSUPPORTED;
  const int64_t nwg = ((int64_t)3 * H * d + 255) / 256 * ((M + 255) / 256);
  if (nwg > INT32_MAX || M > INT32_MAX) return VIDAX_ERR_UNSUPPORTED;
  const hipError_t e = vidax::launch_qkv_proj((const uint16_t*)x, (const uint16_t*)w, bias, gain_q, gain_k, eps,
                                              (uint16_t*)q, (uint16_t*)k, (uint16_t*)v, B, L, H, C, rp, stream);
  return e == hipSuccess ? VIDAX_OK : VIDAX_ERR_LAUNCH;
}

vidax_status vidax_attn_mod_fwd(const void* q, const void* k, const void* v, void* o, float* lse, int32_t B, int32_t H,
                                int32_t Hkv, int32_t Lq, int32_t Lk, int32_t d, float scale,
                                const vidax_score_desc* score, float* workspace, size_t workspace_floats,
                                hipStream_t stream) {
  vidax::ModFwd a;
  Buf s[6];
  const vidax_status st = mod_common(B, H, Hkv, Lq, Lk, d, scale, score, false, &a.c, s);
  if (st == VIDAX_ERR_INVALID_ARG) return st;
  const uint64_t nq = (uint64_t)B * Lq * H * d, nk = (uint64_t)B * Lk * Hkv * d;
  if ((nq > 0 && (!q || !o)) || (nq > 0 && nk > 0 && (!k || !v))) return VIDAX_ERR_INVALID_ARG;
  for (const void* p : {q, k, v, (const void*)o, (const void*)workspace})
    if (!aligned(p, 16)) return VIDAX_ERR_INVALID_ARG;
  if (!aligned(lse, 4) || workspace_floats > ((uint64_t)1 << 60)) return VIDAX_ERR_INVALID_ARG;
  if (!workspace) workspace_floats = 0;
  const Buf outs[3] = {{o, nq * 2}, {lse, (uint64_t)B * H * Lq * 4}, {workspace, (uint64_t)workspace_floats * 4}};
  const Buf ins[9] = {{q, nq * 2}, {k, nk * 2}, {v, nk * 2}, s[0], s[1], s[2], s[3], s[4], s[5]};
  if (any_overlap(outs, ins)) return VIDAX_ERR_INVALID_ARG;
  if (st != VIDAX_OK || nq == 0) return st;
  if (workspace_floats < vidax::mod_doc_floats(B, Lq, Lk, a.c.s.k_doc != nullptr)) return VIDAX_ERR_INVALID_ARG;
  if (!vidax::launch_attn_mod_fwd) return VIDAX_ERR_LAUNCH;
  a.q = (const uint16_t*)q;
  a.k = (const uint16_t*)k;
  a.v = (const uint16_t*)v;
  a.o = (uint16_t*)o;
  a.lse = lse;
  a.ws = workspace;
  a.ws_floats = workspace_floats;
  return vidax::launch_attn_mod_fwd(a, stream) == hipSuccess ? VIDAX_OK : VIDAX_ERR_LAUNCH;
}

vidax_status vidax_attn_mod_bwd(const void* q, const void* k, const void* v, const void* o, const void* dout,
                                const float* lse, void* dq, void* dk, void* dv, int32_t B, int32_t H, int32_t Hkv,
                                int32_t Lq, int32_t Lk, int32_t d, float scale, const vidax_score_desc* score,
                                float* workspace, size_t workspace_floats, hipStream_t stream) {
  vidax::ModBwd a;
  Buf s[6];
  const vidax_status st = mod_common(B, H, Hkv, Lq, Lk, d, scale, score, true, &a.c, s);
  if (st == VIDAX_ERR_INVALID_ARG) return st;
  const uint64_t nq = (uint64_t)B * Lq * H * d, nk = (uint64_t)B * Lk * Hkv * d, nr = (uint64_t)B * H * Lq;
  if ((nq > 0 && (!q || !o || !dout || !dq || !lse)) || (nk > 0 && (!dk || !dv)) || (nq > 0 && nk > 0 && (!k || !v)))
    return VIDAX_ERR_INVALID_ARG;
  for (const void* p : {q, k, v, o, dout, (const void*)dq, (const void*)dk, (const void*)dv, (const void*)workspace})
    if (!aligned(p, 16)) return VIDAX_ERR_INVALID_ARG;
  if (!aligned(lse, 4) || workspace_floats > ((uint64_t)1 << 60)) return VIDAX_ERR_INVALID_ARG;
  if (!workspace) workspace_floats = 0;
  const Buf outs[4] = {{dq, nq * 2}, {dk, nk * 2}, {dv, nk * 2}, {workspace, (uint64_t)workspace_floats * 4}};
  const Buf ins[12] = {{q, nq * 2}, {k, nk * 2}, {v, nk * 2}, {o, nq * 2}, {dout, nq * 2}, {lse, nr * 4},
                       s[0], s[1], s[2], s[3], s[4], s[5]};
  if (any_overlap(outs, ins)) return VIDAX_ERR_INVALID_ARG;
  if (st != VIDAX_OK || (nq == 0 && nk == 0)) return st;
  const size_t least = vidax::mod_bwd_split(B, H, Hkv, Lq, Lk, a.c.s.k_doc != nullptr, false, false, 1, 0).least;
  if (workspace_floats < least) return VIDAX_ERR_INVALID_ARG;
  if (!vidax::launch_attn_mod_bwd) return VIDAX_ERR_LAUNCH;
  a.q = (const uint16_t*)q;
  a.k = (const uint16_t*)k;
  a.v = (const uint16_t*)v;
  a.o = (const uint16_t*)o;
  a.dout = (const uint16_t*)dout;
  a.lse = lse;
  a.dq = (uint16_t*)dq;
  a.dk = (uint16_t*)dk;
  a.dv = (uint16_t*)dv;
  a.ws = workspace;
  a.ws_floats = workspace_floats;
  return vidax::launch_attn_mod_bwd(a, stream) == hipSuccess ? VIDAX_OK : VIDAX_ERR_LAUNCH;
}

size_t vidax_attn_mod_bwd_workspace_floats(int32_t B, int32_t H, int32_t Hkv, int32_t Lq, int32_t Lk, int32_t d,
                                           int32_t docs) {
  vidax::ModCall c;
  Buf s[6];
  if (mod_common(B, H, Hkv, Lq, Lk, d, 1.0f, nullptr, true, &c, s) != VIDAX_OK) return 0;
  const int cus = vidax::device_cu_count();
  size_t most = 0;
  for (int i = 0; i < 4; ++i) {
    const size_t n = vidax::mod_bwd_split(B, H, Hkv, Lq, Lk, docs != 0, i & 1, i & 2, cus, SIZE_MAX).floats;
    if (n > most) most = n;
  }
  return most;
}

size_t vidax_attn_mod_fwd_workspace_floats(int32_t B, int32_t H, int32_t Hkv, int32_t Lq, int32_t Lk, int32_t d,
                                           int32_t docs) {
  vidax::ModCall c;
  Buf s[6];
  if (mod_common(B, H, Hkv, Lq, Lk, d, 1.0f, nullptr, false, &c, s) != VIDAX_OK || B == 0 || H == 0 || Lq == 0) return 0;
  const int cus = vidax::device_cu_count();
  size_t most = 0;
  for (int i = 0; i < 4; ++i) {  // (causal or not, lengths or not)
    const size_t n = vidax::mod_fwd_split(B, H, Hkv, Lq, Lk, docs != 0 && Lk > 0, i & 1, i & 2, cus, SIZE_MAX).floats;
    if (n > most) most = n;
  }
  return most;
}

vidax_status vidax_block_norm_fwd(const void* x, const void* y, void* xo, void* h, int32_t B, int32_t L, int32_t C,
                                  const vidax_block_norm_desc* desc, hipStream_t stream) {
  vidax::BlockNormFwd a;
  Buf mods[5];
  const vidax_status st = block_norm_common(B, L, C, desc, y != nullptr, &a.n, mods);
  if (st == VIDAX_ERR_INVALID_ARG) return st;
  const uint64_t n = (uint64_t)B * L * C, sb = n * (desc->stream_fp32 ? 4 : 2);
  for (const void* p : {x, y, (const void*)xo, (const void*)h})
    if (!aligned(p, 16)) return VIDAX_ERR_INVALID_ARG;
  if (n > 0 && (!x || !h || (!xo && (y || desc->alpha != 1.0f)))) return VIDAX_ERR_INVALID_ARG;
  const Buf outs[2] = {{xo, sb}, {h, n * 2}};
  const Buf ins[7] = {{x, sb}, {y, n * 2}, mods[0], mods[1], mods[2], mods[3], mods[4]};
  if (any_overlap(outs, ins, 0, 0)) return VIDAX_ERR_INVALID_ARG;
  if (st != VIDAX_OK || n == 0) return st;
  if (!vidax::block_launch_fits(vidax::block_fwd_shape(B, L, C), B)) return VIDAX_ERR_UNSUPPORTED;
  if (!vidax::launch_block_norm_fwd) return VIDAX_ERR_LAUNCH;
  a.x = x;
  a.y = (const uint16_t*)y;
  a.xo = xo;
  a.h = (uint16_t*)h;
  return vidax::launch_block_norm_fwd(a, stream) == hipSuccess ? VIDAX_OK : VIDAX_ERR_LAUNCH;
}

size_t vidax_block_norm_bwd_workspace_floats(int32_t B, int32_t L, int32_t C) {
  if (B < 0 || L < 0 || C < 0 || C % 8 != 0 || C > vidax::kBlockMaxC || (int64_t)B * L > INT32_MAX) return 0;
  if (B == 0 || L == 0 || C == 0 || !vidax::block_launch_fits(vidax::block_bwd_shape(B, L, C), B)) return 0;
  return vidax::block_bwd_floats(B, L, C);
}

vidax_status vidax_block_norm_bwd(const void* dh, const void* dxo, const void* xo, const void* y, void* dx, void* dy,
                                  const vidax_block_norm_grads* grads, float* workspace, size_t workspace_floats,
                                  int32_t B, int32_t L, int32_t C, const vidax_block_norm_desc* desc,
                                  hipStream_t stream) {
  vidax::BlockNormBwd a;
  Buf mods[5];
  const vidax_status st = block_norm_common(B, L, C, desc, y != nullptr, &a.n, mods);
  if (st == VIDAX_ERR_INVALID_ARG) return st;
  if (!grads) return VIDAX_ERR_INVALID_ARG;
  const bool per_token = desc->per_token != 0;
  if (!per_token)
    for (const vidax_block_mod* m : {&desc->gate, &desc->scale})
      if (m->p && m->token_stride) return VIDAX_ERR_INVALID_ARG;
  // dgate and dpost_gain need the branch; dpost_gain its norm
  const uint64_t n = (uint64_t)B * L * C;
  if ((grads->dgate && n > 0 && !y) || (grads->dpost_gain && (!desc->post || (n > 0 && !y)))) return VIDAX_ERR_INVALID_ARG;
  const uint64_t sb = n * (desc->stream_fp32 ? 4 : 2);
  const uint64_t mb = (per_token ? n : (uint64_t)B * C) * 4;
  for (const void* p : {dh, dxo, xo, y, (const void*)dx, (const void*)dy, (const void*)grads->dgate,
                        (const void*)grads->dscale, (const void*)grads->dshift, (const void*)grads->dgain,
                        (const void*)grads->dpost_gain, (const void*)workspace})
    if (!aligned(p, 16)) return VIDAX_ERR_INVALID_ARG;
  if (n > 0 && (!dh || !xo || !dx || (y && !dy) || (!y && dy))) return VIDAX_ERR_INVALID_ARG;
  if (workspace_floats > ((uint64_t)1 << 60)) return VIDAX_ERR_INVALID_ARG;
  const bool sums = (!per_token && (grads->dgate || grads->dscale || grads->dshift)) || grads->dgain || grads->dpost_gain;
  const Buf outs[8] = {{dx, sb}, {dy, n * 2}, {grads->dgate, mb}, {grads->dscale, mb}, {grads->dshift, mb},
                       {grads->dgain, (uint64_t)C * 4}, {grads->dpost_gain, (uint64_t)C * 4},
                       {workspace, (uint64_t)workspace_floats * 4}};
  const Buf ins[8] = {{dxo, sb}, {dh, n * 2}, {xo, sb}, {y, n * 2}, mods[0], mods[1], mods[3], mods[4]};
  if (any_overlap(outs, ins, 0, 0)) return VIDAX_ERR_INVALID_ARG;
  if (st != VIDAX_OK) return st;
  if (n > 0 && !vidax::block_launch_fits(vidax::block_bwd_shape(B, L, C), B)) return VIDAX_ERR_UNSUPPORTED;
  if (n > 0 && sums && (!workspace || workspace_floats < vidax::block_bwd_floats(B, L, C))) return VIDAX_ERR_INVALID_ARG;
  if (C == 0 || (n == 0 && !sums)) return VIDAX_OK;  // (without tokens the sums are zero)
  if (!vidax::launch_block_norm_bwd) return VIDAX_ERR_LAUNCH;
  a.dh = (const uint16_t*)dh;
  a.dxo = dxo;
  a.xo = xo;
  a.y = (const uint16_t*)y;
  a.dx = dx;
  a.dy = (uint16_t*)dy;
  a.dgate = grads->dgate;
  a.dscale = grads->dscale;
  a.dshift = grads->dshift;
  a.dgain = grads->dgain;
  a.dpost_gain = grads->dpost_gain;
  a.per_token = desc->per_token;
  a.ws = workspace;
  return vidax::launch_block_norm_bwd(a, stream) == hipSuccess ? VIDAX_OK : VIDAX_ERR_LAUNCH;
}

const char* vidax_status_string(int32_t status) {
  switch (status) {
    case VIDAX_OK: return "ok";
    case VIDAX_ERR_INVALID_ARG: return "invalid argument";
    case VIDAX_ERR_UNSUPPORTED: return "unsupported configuration";
    case VIDAX_ERR_LAUNCH: return "kernel launch failed";
    case VIDAX_ERR_TOO_LARGE: return "request exceeds the fixed device scratch of an allocation-free entry point";
  }
  return "unknown status";
}

int32_t vidax_abi_version(void) { return VIDAX_ABI_VERSION; }

}  // extern "C"
