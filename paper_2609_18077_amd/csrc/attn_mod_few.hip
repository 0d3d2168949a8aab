// Attention with score modifiers for few query rows (single tokens of a serving
// step): all rows of a K/V head's group, rep * Lq <= 32 of them, are the columns
// of one 32x32x16 product.  HBM-bound: K and V are read once, by whoever needs
// them.
//
// A workgroup is four waves, each with its own tiles of 32 keys and its own 32 KB
// of LDS: two buffers of K and two of V, filled by direct copies of whole rows;
// no barrier until the waves' outputs are joined at the end.  Two tiles a wave
// are on their way at any time, 128 KB a compute unit; 16 requests x 16384 keys x
// 8 heads, 1.07 GB: 238 us = 4.5 TB/s, the joining launch with it.
//   Split.  The tiles of all batches (those below the last key that a batch's
// queries may see) are one sequence, cut into `units` equal pieces, a workgroup
// and K/V head each; a piece may end one batch and begin the next.  Caches filled
// to any lengths then load the compute units evenly.  What a unit finds for a
// batch is a partial result; units and batches only move forward, so their sum
// numbers the partial results.  A second launch joins them.  Where there are
// batches enough, or few keys, a workgroup takes a whole batch instead.
#include "attn_mod.hpp"
#include "launch.hpp"

namespace vidax {
namespace {

using namespace tile;
using namespace mod;

constexpr int D = kHeadDim;
constexpr int NW = 4;
constexpr int BN = 32;        // keys of a tile
constexpr int TILE = BN * D;  // elements
constexpr int kOut = D + 4;   // floats of an output row in LDS

struct FewArgs {
  ModCall c;
  Scores sc;
  const uint16_t *q, *k, *v;
  uint16_t* o;
  float* lse;
  float *po, *pl;
  ModRanges r;
  int units;  // 0: a workgroup takes a whole batch
  int kr;
};

// The sequence of the batches' tiles: unit u of `units` takes tiles [u per, (u + 1)
// per) of it, per = ceil(total / units) (the last ones may be left without any).
struct Sequence {
  int64_t total;  // tiles of all batches
  int64_t first;  // of the batches before one
};
__device__ __forceinline__ int tiles_of(const ModCall& c, int b) {
  const Batch bt = batch_of_lane(c, b);
  return (key_limit(bt, c.s.causal, bt.start + c.Lq - 1) + BN - 1) / BN;
}
// Sums over all batches and over those before `b` (every lane gets both).
__device__ __forceinline__ Sequence sequence(const ModCall& c, int b, int lane) {
  Sequence s{0, 0};
  for (int i = 0; i < c.B; i += 64) {
    const int n = i + lane < c.B ? tiles_of(c, i + lane) : 0;
    int all = n, before = i + lane < b ? n : 0;
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) {
      all += __shfl_xor(all, m);
      before += __shfl_xor(before, m);
    }
    s.total += all;
    s.first += before;
  }
  return s;
}
__device__ __forceinline__ int64_t unit_tiles(int64_t total, int units) { return (total + units - 1) / units; }

__global__ __launch_bounds__(64 * NW, 1) void attn_mod_few_kernel(FewArgs a) {
  __shared__ __attribute__((aligned(1024))) uint16_t K0[NW * TILE], K1[NW * TILE], V0[NW * TILE], V1[NW * TILE];
  __shared__ float mrow[NW][32], lrow[NW][32];
  static_assert(sizeof(float) * 32 * kOut <= sizeof(uint16_t) * TILE * NW, "a wave's output rows fit a buffer");
  const int lane = threadIdx.x & 63, l32 = lane & 31, hi = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const ModCall& c = a.c;
  const int rep = c.H / c.Hkv, nrow = rep * c.Lq;
  const int ktok = c.Hkv * D, kbytes = ktok * 2;
  // Every XCD takes an eighth of the (unit, K/V head) pairs, those of a unit side by
  // side: so lie a token's heads in memory.
  const int n8 = gridDim.x >> 3, rem = gridDim.x & 7, xcd = blockIdx.x & 7;
  const int pair = xcd * n8 + min(xcd, rem) + (int)(blockIdx.x >> 3), unit = pair / c.Hkv, hk = pair - unit * c.Hkv;

  // One piece: tiles [t0, t1) of batch b, partial result `slot` (or the output)
  auto piece = [&](const int b, const int t0, const int t1, const int slot) __attribute__((always_inline)) {
  const Batch bt = batch_of(c, b);
  // the lane's row: query head hk rep + l32 / Lq, query l32 mod Lq
  const bool live = l32 < nrow;
  const int hr = live ? hk * rep + l32 / c.Lq : 0, i = live ? l32 % c.Lq : 0;
  const int pos = bt.start + i;
  int lim = live ? key_limit(bt, c.s.causal, pos) : 0;
  int qd = 0;
  const bool docs = a.r.k != nullptr;
  Docs rows{0, 0, false};
  if (docs) {
    qd = live ? c.s.q_doc[(size_t)b * c.Lq + i] : -1;
    int lo = qd >= 0 ? qd : 0x7fffffff, up = qd >= 0 ? qd : 0;
#pragma unroll
    for (int m = 1; m < 32; m <<= 1) {
      lo = min(lo, __shfl_xor(lo, m));
      up = max(up, __shfl_xor(up, m));
    }
    rows = uniform(Docs{lo, up, __builtin_amdgcn_ballot_w64(live && qd < 0) != 0});
    if (qd < 0) lim = 0;
  }
  const int least = key_limit(bt, c.s.causal, bt.start), most = key_limit(bt, c.s.causal, bt.start + c.Lq - 1);

  // the tiles to visit, as in the 256-row kernel; the waves take them in turn
  int grp = t0 >> 6, turn = 0;
  uint64_t visit = 0, whole = 0, neg = 0;
  auto look = [&](int g) __attribute__((always_inline)) {
    const int t = 64 * g + lane;
    const bool in = t >= t0 && t < t1;
    bool v = in, w = in && t * BN + BN <= least, n = false;
    if (docs && in) {
      const Docs d = docs_of(a.r.k[(size_t)b * a.kr + t]);
      v = meet(d, rows);
      w = w && same(d, rows);
      n = d.neg;
    }
    visit = __builtin_amdgcn_ballot_w64(v);
    whole = __builtin_amdgcn_ballot_w64(w);
    neg = __builtin_amdgcn_ballot_w64(n);
  };
  struct Tile {
    int t;  // -1: none left
    bool whole, neg;
  };
  auto next = [&]() __attribute__((always_inline)) {
    for (;;) {
      while (visit == 0) {
        if (64 * (grp + 1) >= t1) return Tile{-1, false, false};
        look(++grp);
      }
      const int j = __builtin_ctzll(visit);
      visit &= visit - 1;
      const bool mine = turn == wave;
      turn = turn + 1 == NW ? 0 : turn + 1;
      if (mine) return Tile{64 * grp + j, (bool)(whole >> j & 1), (bool)(neg >> j & 1)};
    }
  };

  const uint16_t* const kbh = a.k + (size_t)b * c.Lk * ktok + (size_t)hk * D;
  const uint16_t* const vbh = a.v + (size_t)b * c.Lk * ktok + (size_t)hk * D;
  auto rsrc = [&](const uint16_t* base, int t) __attribute__((always_inline)) {
    const int nbytes = __builtin_amdgcn_readfirstlane(min(max(most - t * BN, 0), BN) * kbytes);
    return __builtin_amdgcn_make_buffer_rsrc((void*)(base + (size_t)t * BN * ktok), (short)0, nbytes, kBufferFlags);
  };
  // rows 4 j .. 4 j + 3 of a tile: the lane fetches chunk (lane & 15) ^ swz(row) of row 4 j + (lane >> 4)
  auto copy = [&](const Tile& t, uint16_t* kb, uint16_t* vb) __attribute__((always_inline)) {
    const __amdgpu_buffer_rsrc_t rk = rsrc(kbh, t.t), rv = rsrc(vbh, t.t);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int r = 4 * j + (lane >> 4);
      const int off = r * kbytes + ((lane & 15) ^ swz(r)) * 16;
      int voff = off;
      if (t.neg) {  // uniform: values of keys of negative documents arrive as zeros
        const int key = t.t * BN + r;
        if (key >= c.Lk || c.s.k_doc[(size_t)b * c.Lk + min(key, c.Lk - 1)] < 0) voff = 0x7ffffff0;
      }
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rk, (lds_ptr)(kb + 4 * j * D), 16, off, 0, 0, 0);
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rv, (lds_ptr)(vb + 4 * j * D), 16, voff, 0, 0, 0);
    }
  };

  f32x16 oacc[4];
#pragma unroll
  for (int mb = 0; mb < 4; ++mb) oacc[mb] = f32x16{};
  float mref = -INFINITY, lsum = 0.f;
  const float slope = c.s.slopes && live ? -c.s.slopes[hr] * kLog2e : 0.f;

  Tile cur{-1, false, false}, nxt = cur;
  if (t0 < t1) {
    look(grp);
    cur = next();
  }
  uint16_t *const k0 = K0 + wave * TILE, *const k1 = K1 + wave * TILE, *const v0 = V0 + wave * TILE,
           *const v1 = V1 + wave * TILE;
  if (cur.t >= 0) {
    copy(cur, k0, v0);
    nxt = next();
    if (nxt.t >= 0) copy(nxt, k1, v1);
  }
  bf16x8 qop[8];
  {
    const uint16_t* const p = a.q + (((size_t)b * c.Lq + i) * c.H + hr) * D;
#pragma unroll
    for (int s = 0; s < 8; ++s) {
      uint4 x = make_uint4(0, 0, 0, 0);
      if (live) x = *reinterpret_cast<const uint4*>(p + (2 * s + hi) * 8);
      qop[s] = __builtin_bit_cast(bf16x8, make_uint4((x.x ^ a.sc.qxor) & a.sc.qand, (x.y ^ a.sc.qxor) & a.sc.qand,
                                                     (x.z ^ a.sc.qxor) & a.sc.qand, (x.w ^ a.sc.qxor) & a.sc.qand));
    }
  }
  const RowOffsets off = row_offsets(lane);

  auto work = [&](const Tile& t, const uint16_t* kb, const uint16_t* vb) __attribute__((always_inline)) {
    f32x16 s = f32x16{};
#pragma unroll
    for (int st = 0; st < 8; ++st) s = mfma32(read_row(kb, off.row, st), qop[st], s);
    if (a.c.s.cap > 0.f) cap16_log2(s, a.sc, 0.f);  // uniform
    // y; -inf for what the row does not see
    const float dist = (float)(pos - t.t * BN - 4 * hi);
    const int left = lim - t.t * BN - 4 * hi;
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      if (a.c.s.cap == 0.f) s[e] *= a.sc.mul;
      if (c.s.slopes) s[e] = fmaf(slope, fabsf(dist - (float)(8 * (e >> 2) + (e & 3))), s[e]);
    }
    if (!t.whole) {  // uniform
#pragma unroll
      for (int e = 0; e < 16; ++e)
        if (8 * (e >> 2) + (e & 3) >= left) s[e] = -INFINITY;
      if (docs) {
        const __amdgpu_buffer_rsrc_t rd = __builtin_amdgcn_make_buffer_rsrc(
            (void*)(c.s.k_doc + (size_t)b * c.Lk), (short)0, c.Lk * 4, kBufferFlags);
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const u32x4 d = __builtin_amdgcn_raw_buffer_load_b128(rd, (t.t * BN + 8 * g + 4 * hi) * 4, 0, 0);
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if ((int)d[e] != qd) s[4 * g + e] = -INFINITY;
        }
      }
    }
    float m = s[0];
#pragma unroll
    for (int e = 1; e < 16; ++e) m = fmaxf(m, s[e]);
    const float mnew = fmaxf(mref, wave_half_max(m));
    const float base = mnew == -INFINITY ? 0.f : mnew;  // (a row that has seen nothing: weights 0)
    if (__builtin_amdgcn_ballot_w64(mnew != mref) != 0) {
      const float alpha = __builtin_amdgcn_exp2f(mref - base);
      lsum *= alpha;
#pragma unroll
      for (int mb = 0; mb < 4; ++mb)
#pragma unroll
        for (int e = 0; e < 16; ++e) oacc[mb][e] *= alpha;
      mref = mnew;
    }
    bf16x8 pop[2];
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) {
      uint32_t pw[4];
#pragma unroll
      for (int e = 0; e < 8; e += 2) {
        const float p0 = __builtin_amdgcn_exp2f(s[8 * ks + e] - base), p1 = __builtin_amdgcn_exp2f(s[8 * ks + e + 1] - base);
        pw[e >> 1] = pack_bf16x2(p0, p1);
        lsum += p0 + p1;
      }
      pop[ks] = __builtin_bit_cast(bf16x8, make_uint4(pw[0], pw[1], pw[2], pw[3]));
    }
#pragma unroll
    for (int ks = 0; ks < 2; ++ks)
#pragma unroll
      for (int mb = 0; mb < 4; ++mb) oacc[mb] = mfma32(read_tr(vb + 16 * ks * D, off.tr, mb), pop[ks], oacc[mb]);
  };
  // (The output is divided by the sum of the weights before their rounding, where the
  // 256-row form takes the roundings: either is within 2^-8 of the weights.)
  // One tile: its copies (older than the next tile's 16) are awaited; behind it,
  // when nothing reads its buffers any more, the tile after next is on its way.
  auto step = [&](auto parity) __attribute__((always_inline)) {
    constexpr int P = decltype(parity)::value;
    if (nxt.t >= 0) __builtin_amdgcn_s_waitcnt(wait_vm(16));
    else __builtin_amdgcn_s_waitcnt(wait_vm(0));
    __builtin_amdgcn_sched_barrier(0);
    work(cur, P ? k1 : k0, P ? v1 : v0);
    const Tile aft = next();
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_waitcnt(kWaitLgkm0);
    if (aft.t >= 0) copy(aft, P ? k1 : k0, P ? v1 : v0);
    cur = nxt;
    nxt = aft;
    return cur.t >= 0;
  };
  if (cur.t >= 0)
    while (step(std::integral_constant<int, 0>()) && step(std::integral_constant<int, 1>())) {
    }

  // ---- the waves' rows joined, in the order of the waves
  lsum = wave_half_sum(lsum);
  __syncthreads();  // every wave is done with its tiles
  auto area = [&](int w, int r) __attribute__((always_inline)) {  // row r of wave w
    return reinterpret_cast<float*>(w == 0 ? K0 : w == 1 ? K1 : w == 2 ? V0 : V1) + r * kOut;
  };
  float* const mine = area(wave, l32);
#pragma unroll
  for (int mb = 0; mb < 4; ++mb)
#pragma unroll
    for (int g = 0; g < 4; ++g)
      *reinterpret_cast<float4*>(mine + 32 * mb + 8 * g + 4 * hi) =
          make_float4(oacc[mb][4 * g], oacc[mb][4 * g + 1], oacc[mb][4 * g + 2], oacc[mb][4 * g + 3]);
  if (hi == 0) {
    mrow[wave][l32] = mref;
    lrow[wave][l32] = lsum;
  }
  __syncthreads();
  // kPer lanes a row, its channels in pieces of 8 (a piece of each lane side by side)
  constexpr int kPer = 2 * NW, kPieces = 16 / kPer;
  const int r = threadIdx.x / kPer, part = threadIdx.x % kPer;
  if (r >= nrow) return;  // of the piece
  const int h = hk * rep + r / c.Lq, qi = r % c.Lq;
  float m = mrow[0][r], w[NW], l = 0.f;
#pragma unroll
  for (int u = 1; u < NW; ++u) m = fmaxf(m, mrow[u][r]);
  const bool seen = m > -INFINITY;
#pragma unroll
  for (int u = 0; u < NW; ++u) {
    w[u] = seen ? __builtin_amdgcn_exp2f(mrow[u][r] - m) : 0.f;
    l = fmaf(w[u], lrow[u][r], l);
  }
  const float inv = seen ? 1.0f / l : 0.f;
  const size_t prow = ((size_t)slot * c.Hkv + hk) * nrow + r;
#pragma unroll
  for (int u = 0; u < kPieces; ++u) {
    const int d = 8 * (kPer * u + part);
    float y[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int x = 0; x < NW; ++x) {
      const float* const p = area(x, r) + d;
#pragma unroll
      for (int e = 0; e < 8; ++e) y[e] = fmaf(w[x], p[e], y[e]);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) y[e] *= inv;
    if (a.units) {
      float* const po = a.po + prow * D + d;
      *reinterpret_cast<float4*>(po) = make_float4(y[0], y[1], y[2], y[3]);
      *reinterpret_cast<float4*>(po + 4) = make_float4(y[4], y[5], y[6], y[7]);
    } else {
      *reinterpret_cast<uint4*>(a.o + (((size_t)b * c.Lq + qi) * c.H + h) * D + d) =
          make_uint4(pack_bf16x2(y[0], y[1]), pack_bf16x2(y[2], y[3]), pack_bf16x2(y[4], y[5]), pack_bf16x2(y[6], y[7]));
    }
  }
  if (part == 0) {
    const float lse2 = seen ? m + __log2f(l) : -INFINITY;
    if (a.units) a.pl[prow] = lse2;
    else if (a.lse) a.lse[((size_t)b * c.H + h) * c.Lq + qi] = lse2 * kLn2;
  }
  };
  if (!a.units) return piece(unit, 0, tiles_of(c, unit), 0);
  const int64_t total = sequence(c, 0, lane).total;
  const int64_t per = unit_tiles(total, a.units), s1 = per * (unit + 1);
  int64_t s = per * unit, first = 0;
  for (int b = 0; b < c.B && s < s1; ++b) {
    // skip the batches before the unit's first tile 64 at a time
    if ((b & 63) == 0) {
      const int n = b + lane < c.B ? tiles_of(c, b + lane) : 0;
      int upto = n;
#pragma unroll
      for (int m = 1; m < 64; m <<= 1) {
        const int x = __shfl_up(upto, m);
        if (lane >= m) upto += x;
      }
      const uint64_t past = __builtin_amdgcn_ballot_w64(first + upto > s);
      const int skip = past ? __builtin_ctzll(past) : 64;
      if (skip) first += __builtin_amdgcn_readlane(upto, skip - 1);
      b += skip;
      if (skip == 64) { --b; continue; }
    }
    const int n = __builtin_amdgcn_readfirstlane(tiles_of(c, b));
    if (first + n > s) {
      const int64_t e = first + n < s1 ? first + n : s1;
      piece(b, (int)(s - first), (int)(e - first), unit + b);
      s = e;
      __syncthreads();  // the rows are out of LDS
    }
    first += n;
  }
}

// Joins the partial results of every row: a wave a row, lane l its channels 2 l, 2 l + 1.
__global__ __launch_bounds__(256) void mod_few_join_kernel(FewArgs a) {
  const ModCall& c = a.c;
  const int lane = threadIdx.x & 63, rep = c.H / c.Hkv, nrow = rep * c.Lq;
  const int64_t w = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (w >= (int64_t)c.B * c.Hkv * nrow) return;
  const int r = (int)(w % nrow), bh = (int)(w / nrow), hk = bh % c.Hkv, b = bh / c.Hkv;
  const Sequence q = sequence(c, b, lane);
  const int n = tiles_of(c, b);
  float m = -INFINITY, x = 0.f, y = 0.f, l = 0.f;
  if (n > 0) {
    const int64_t per = unit_tiles(q.total, a.units);
    const int u0 = (int)(q.first / per), u1 = (int)((q.first + n - 1) / per);
    const size_t step = (size_t)c.Hkv * nrow, at = (size_t)(u0 + b) * step + hk * nrow + r;  // slot of unit u0
    for (int u = lane; u <= u1 - u0; u += 64) m = fmaxf(m, a.pl[at + u * step]);
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) m = fmaxf(m, __shfl_xor(m, d));
    if (m > -INFINITY) {
#pragma unroll 8
      for (int u = 0; u <= u1 - u0; ++u) {
        const float f = __builtin_amdgcn_exp2f(a.pl[at + u * step] - m);
        const float2 v = *reinterpret_cast<const float2*>(a.po + (at + u * step) * D + 2 * lane);
        l += f;
        x = fmaf(f, v.x, x);
        y = fmaf(f, v.y, y);
      }
      const float inv = 1.0f / l;
      x *= inv;
      y *= inv;
    }
  }
  const int h = hk * rep + r / c.Lq, i = r % c.Lq;
  *reinterpret_cast<uint32_t*>(a.o + (((size_t)b * c.Lq + i) * c.H + h) * D + 2 * lane) = pack_bf16x2(x, y);
  if (a.lse && lane == 0) a.lse[((size_t)b * c.H + h) * c.Lq + i] = m > -INFINITY ? (m + __log2f(l)) * kLn2 : -INFINITY;
}

}  // namespace

hipError_t launch_mod_few(const ModFwd& f, const ModSplit& s, const ModRanges& r, hipStream_t stream) {
  const ModCall& c = f.c;
  FewArgs a;
  a.c = c;
  a.sc = make_scores(c);
  a.q = f.q;
  a.k = f.k;
  a.v = f.v;
  a.o = f.o;
  a.lse = f.lse;
  a.units = s.units;
  const size_t rows = (size_t)(s.units + c.B) * c.H * c.Lq;  // of the partial results
  a.po = s.units ? f.ws + s.part : nullptr;
  a.pl = s.units ? a.po + rows * D : nullptr;
  a.r = r;
  a.kr = (int)mod_ranges(c.Lk);
  const int units = s.units ? s.units : c.B;
  const hipError_t e =
      launch_kernel(attn_mod_few_kernel, (unsigned)(units * c.Hkv), 64u * NW, stream, a);
  if (e != hipSuccess || !s.units) return e;
  return launch_kernel(mod_few_join_kernel, (unsigned)(((size_t)c.B * c.H * c.Lq + 3) / 4), 256u, stream, a);
}

}  // namespace vidax
