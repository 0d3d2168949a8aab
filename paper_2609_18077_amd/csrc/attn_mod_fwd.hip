// Attention with score modifiers, forward, for gfx950: 256 query rows of one
// (batch, head) a workgroup, bf16 MFMA (32x32x16) with fp32 accumulation and a
// streaming softmax.  Head dim 128.
//
//   y_ij = log2 e * (cap tanh(scale q.k / cap) - slope |p_i - j|),  o = softmax2(y) v
//
// The dataflow is the dense forward's (attn_fwd.hip): a wave owns 32 query rows,
// S^T = K Q^T puts a query in each lane, keys and values stream through LDS in
// tiles of 64 in operand order, two buffers each, one barrier a tile, the scores
// of the next tile formed beside the softmax of this one.  What differs:
//   Tiles.  The workgroup visits the tiles that one of its rows may see, found 64
//     at a time by a ballot over the tiles' document ranges and the causal limits;
//     a wave whose own 32 rows see nothing of a tile leaves its products out, and
//     only a wave for which a tile is not seen whole by all its rows masks it.
//   Masks.  A score that is not seen becomes -inf after the cap.  A row's
//     reference m is unset until it has seen a key: a block's exponents are then
//     1e30 too large, so that the first key seen overflows the block's sum and sets
//     the reference, while a block without one passes (the rows of a later document
//     wait through an earlier one's tiles).  A row that sees nothing ends with a
//     sum of 0: o = 0, lse = -inf.  Keys that no row may see (past
//     the valid length or the last row's position, or of a negative document) are
//     read as zeros, so that nothing that lies there reaches the output.
//   Sums: of the bf16 roundings of the weights (which the output is divided by) and,
//     where the log-sum-exps are wanted, of the weights: good to fp32, a sixteenth
//     more vector work (16384 x 12 heads: 1483 us without, 1550 with).
//   Few tiles of rows, or uneven ones: the keys are cut into runs, or all tiles'
//     keys into pieces of equal weight (attn_mod.hpp), a workgroup each, whose
//     normalised fp32 outputs and log-sum-exps a second launch joins.
#include "attn_mod.hpp"
#include "launch.hpp"

namespace vidax {
namespace {

using namespace tile;
using namespace mod;

constexpr int D = kHeadDim;
constexpr int BM = kModRows;
constexpr int BN = kModKeys;
constexpr int NW = 8;
constexpr int NT = NW * 64;
constexpr int TILE = BN * D;  // elements of a K or V tile
constexpr int BLK = 512;      // elements of an operand block
constexpr float kUnset = 1e30f;
constexpr float kFoldMost = 80.f;  // a row of scores at -cap has weights of 2^-80

struct FwdArgs {
  ModCall c;
  Scores sc;
  const uint16_t *q, *k, *v;
  uint16_t* o;
  float* lse;
  // partial outputs [runs][B][H][Lq][D] and log2-sum-exps [runs][B][H][Lq], or null;
  // in pieces: [slots][slot_rows][D] and [slots][slot_rows]
  float *po, *pl;
  Pieces pieces;
  ModRanges r;
  int ntile, nwg, runs;
  int in_run[kMostRuns];   // see place()
  int sorted, first_most;  // see place(); causal: the first tile of a head has the most work (else the last)
  int kr, qr;      // document ranges a batch
};

// CAP, BIAS: the scores' modifiers.  LSE: the log-sum-exps are wanted.  PIECES: the part
// of a query tile's keys given.
template <bool CAP, bool BIAS, bool LSE, bool PIECES>
__device__ __forceinline__ void fwd_body(const FwdArgs& a, const Part& part) {
  __shared__ __attribute__((aligned(16))) uint16_t K0[TILE], K1[TILE], V0[TILE], V1[TILE];
  __shared__ __attribute__((aligned(16))) int Kd[2][BN];  // ids of the tiles' keys, where they differ

  const int tid = threadIdx.x;
  const int lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l32 = lane & 31;
  const int hi = lane >> 5;
  const ModCall& c = a.c;
  const int qtok = c.H * D, ktok = c.Hkv * D;  // elements between tokens
  const int qbytes = qtok * 2, kbytes = ktok * 2;

  int b, h, qt, run;
  if constexpr (PIECES) {
    b = part.b;
    h = part.h;
    qt = part.t;
    run = 0;
  } else {
    place(a, c.H, a.r.q_order, run, qt, b, h);
  }
  const int hk = h / (c.H / c.Hkv);
  const Batch bt = batch_of(c, b);
  const int row0 = qt * BM;                     // of the workgroup
  const int wrow = row0 + wave * 32;            // of the wave
  const int qrow = wrow + l32;
  const bool qlive = qrow < c.Lq;
  const int wlast = min(wrow + 32, c.Lq) - 1;   // last row of the wave (< wrow: none)
  const int glast = min(row0 + BM, c.Lq) - 1;
  const uint16_t* const kbh = a.k + (size_t)b * c.Lk * ktok + (size_t)hk * D;
  const uint16_t* const vbh = a.v + (size_t)b * c.Lk * ktok + (size_t)hk * D;

  // ---- what the lane's row, the wave's rows and the workgroup's rows may see
  int lim = qlive ? key_limit(bt, c.s.causal, bt.start + qrow) : 0;
  int qd = 0;
  Docs wdoc{0, 0, false}, gdoc{0, 0, false};
  const bool docs = !PIECES && a.r.k != nullptr;
  if (docs) {
    if (qlive) qd = c.s.q_doc[(size_t)b * c.Lq + qrow];
    if (qd < 0) lim = 0;
    const int2* const qr = a.r.q + (size_t)b * a.qr;
    const int first = row0 >> 5;
    gdoc = docs_of(qr[first]);
    for (int i = 1; i < BM / 32; ++i)
      if (first + i < a.qr) gdoc = join(gdoc, docs_of(qr[first + i]));
    gdoc = uniform(gdoc);
    wdoc = wrow < c.Lq ? uniform(docs_of(qr[wrow >> 5])) : Docs{0x7fffffff, 0, false};
  }
  const int wmax = wlast >= wrow ? key_limit(bt, c.s.causal, bt.start + wlast) : 0;
  const int wmin = wlast >= wrow ? key_limit(bt, c.s.causal, bt.start + wrow) : 0;
  const int gmax = key_limit(bt, c.s.causal, bt.start + glast);
  const int ntiles = PIECES ? part.hi : (gmax + BN - 1) / BN, tile0 = PIECES ? part.lo : 0;

  // ---- the next tile to visit: a group of 64 tiles is looked at together, lane
  // l at tile 64 g + l.  With a bias from the rows' own positions (tile `home`) down,
  // then from the last tile down to there: the rows meet the keys next to them first,
  // and the reference that those set holds (upwards, steep slopes raised it in every
  // tile: 1560 rows on 32760 keys, causal, 12 heads, slopes 2^-2/3 .. 2^-8: 414 us, so
  // 334).
  constexpr bool DOWN = BIAS;
  const int home = min(max((bt.start + glast) / BN, tile0), ntiles - 1);
  bool above = false;  // behind home
  int grp = DOWN ? home >> 6 : tile0 >> 6, left = INT32_MAX;  // group; tiles left of this run
  uint64_t visit = 0;             // tiles that some row of the workgroup may see
  int fl = 0, id = 0;             // of the lane's tile
  auto look = [&](int g) __attribute__((always_inline)) {
    const int t = 64 * g + lane;
    bool v = t >= tile0 && t < ntiles && (!DOWN || (t > home) == above);
    fl = (t * BN < wmax ? Tile::kMine : 0) | (t * BN + BN <= wmin ? Tile::kWhole : 0) | Tile::kOne;
    if (docs && v) {
      const int4 r = *reinterpret_cast<const int4*>(a.r.k + (size_t)b * a.kr + 2 * t);
      const Docs d = mod::join(docs_of(make_int2(r.x, r.y)), docs_of(make_int2(r.z, r.w)));
      v = meet(d, gdoc);
      fl &= (meet(d, wdoc) ? Tile::kMine : 0) | (same(d, wdoc) ? Tile::kWhole : 0) | (one_doc(d) ? Tile::kOne : 0);
      if (d.neg) fl |= Tile::kZero;
      id = d.lo;
    }
    visit = __builtin_amdgcn_ballot_w64(v);
  };
  auto first = [&]() __attribute__((always_inline)) {  // out of visit
    const int i = DOWN ? 63 - __builtin_clzll(visit) : __builtin_ctzll(visit);
    visit &= DOWN ? ~(1ull << i) : visit - 1;
    return i;
  };
  auto more = [&]() __attribute__((always_inline)) {  // the next group; false: none left
    if (!DOWN) {
      if (64 * (grp + 1) >= ntiles) return false;
      ++grp;
    } else if (64 * grp > (above ? home + 1 : tile0)) {
      --grp;
    } else {
      if (above || home + 1 >= ntiles) return false;
      above = true;
      grp = (ntiles - 1) >> 6;
    }
    look(grp);
    return true;
  };
  auto next = [&]() __attribute__((always_inline)) {
    while (visit == 0)
      if (!more()) return Tile{-1, 0, 0};
    if (left-- <= 0) return Tile{-1, 0, 0};
    const int i = first();
    return Tile{64 * grp + i, __builtin_amdgcn_readlane(fl, i), __builtin_amdgcn_readlane(id, i)};
  };

  uint16_t* const stage = (wave < 2 ? K0 : wave < 4 ? K1 : wave < 6 ? V0 : V1) + (wave & 1) * 32 * D;

  // The wave's 32 query rows whole into its staging area, then out of it as B
  // operands (chunk 2 s + hi of the lane's own row).
  bf16x8 qreg[8];
  auto dma_q = [&]() __attribute__((always_inline)) {
    const __amdgpu_buffer_rsrc_t rq = __builtin_amdgcn_make_buffer_rsrc(
        (void*)(a.q + (size_t)b * c.Lq * qtok + (size_t)h * D), (short)0, c.Lq * qbytes, kBufferFlags);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int r = 4 * i + (lane >> 4);
      const int off = wrow + r < c.Lq ? (wrow + r) * qbytes + stage_slot(lane & 15, r) * 16 : 0x7ffffff0;
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rq, (lds_ptr)(stage + 4 * i * D), 16, off, 0, 0, 0);
    }
  };
  auto take_q = [&]() __attribute__((always_inline)) {
#pragma unroll
    for (int s = 0; s < 8; ++s) {
      const uint4 x = *reinterpret_cast<const uint4*>(stage + l32 * D + stage_slot(2 * s + hi, l32) * 8);
      qreg[s] = __builtin_bit_cast(bf16x8, make_uint4((x.x ^ a.sc.qxor) & a.sc.qand, (x.y ^ a.sc.qxor) & a.sc.qand,
                                                      (x.z ^ a.sc.qxor) & a.sc.qand, (x.w ^ a.sc.qxor) & a.sc.qand));
    }
  };

  // ---- copies (as in the dense forward): wave w fills blocks 2 w, 2 w + 1 of a
  // K and of a V tile; records end at the last key that a row may see
  const int kg0 = l32 * kbytes + (2 * wave + hi) * 16, kg1 = kg0 + 32 * kbytes;
  const int vrow = 8 * hi + 4 * ((lane >> 4) & 1) + ((lane & 7) >> 1);
  const int vd = 16 * ((lane >> 3) & 1) + 8 * (lane & 1);
  const int vr = vrow + 16 * (wave >> 1);  // blocks 2 wave and 2 wave + 1 are of one key step
  const int vg0 = vr * kbytes + 2 * (vd + 32 * (2 * wave & 3)), vg1 = vg0 + 64;
  auto tile_rsrc = [&](const uint16_t* base, int t) __attribute__((always_inline)) {
    const int nbytes = min(gmax - t * BN, BN) * kbytes;  // (t is below ntiles)
    return __builtin_amdgcn_make_buffer_rsrc((void*)(base + (size_t)t * BN * ktok), (short)0, nbytes, kBufferFlags);
  };
  auto dma_k = [&](int t, uint16_t* buf) __attribute__((always_inline)) {
    const __amdgpu_buffer_rsrc_t rs = tile_rsrc(kbh, t);
    __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (lds_ptr)(buf + (2 * wave) * BLK), 16, kg0, 0, 0, 0);
    __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (lds_ptr)(buf + (2 * wave + 1) * BLK), 16, kg1, 0, 0, 0);
  };
  auto dma_v = [&](const Tile& t, uint16_t* buf) __attribute__((always_inline)) {
    const __amdgpu_buffer_rsrc_t rs = tile_rsrc(vbh, t.t);
    int g0 = vg0, g1 = vg1;
    if (t.zero()) {  // uniform: values of keys of negative documents arrive as zeros
      const int key = t.t * BN + vr;
      if (key >= c.Lk || c.s.k_doc[(size_t)b * c.Lk + min(key, c.Lk - 1)] < 0) g0 = g1 = 0x7ffffff0;
    }
    __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (lds_ptr)(buf + (2 * wave) * BLK), 16, g0, 0, 0, 0);
    __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (lds_ptr)(buf + (2 * wave + 1) * BLK), 16, g1, 0, 0, 0);
  };

  const int koff = lane * 8, voff = lane * 4;
  auto qk = [&](const uint16_t* kb, f32x16 s[2]) __attribute__((always_inline)) {
#pragma unroll
    for (int st = 0; st < 8; ++st)
#pragma unroll
      for (int blk = 0; blk < 2; ++blk) {
        const bf16x8 kop = *reinterpret_cast<const bf16x8*>(kb + (2 * st + blk) * BLK + koff);
        s[blk] = mfma32(kop, qreg[st], st == 0 ? f32x16{} : s[blk]);
      }
  };

  f32x16 oacc[4];
#pragma unroll
  for (int mb = 0; mb < 4; ++mb) oacc[mb] = f32x16{};
  // Capped scores without a bias lie within +-mul; up to kFoldMost of it they need no
  // reference of their own: it starts at 0 and is added with the cap (one operation a
  // score less); a sum that grows beyond the limit still moves it.
  constexpr bool FOLD = CAP && !BIAS;
  float mref = FOLD ? 0.f : -INFINITY;  // the row's reference, log2 units
  float nm = FOLD ? 0.f : kUnset;       // -mref
  float lsum = 0.f;        // this lane half's sum of the weights
  float wsum = 0.f;        // and of their roundings
  const float slope = BIAS && c.s.slopes ? -c.s.slopes[h] * kLog2e : 0.f;
  // Of the tile at hand: the factor of its scores, and the bias as a linear function of
  // the key, slope |p - j| = lin - lin_slope (j - first key of the lane half).  A tile
  // on both sides of the wave's positions (a few of a wave's) has what is missing added
  // to its scores beforehand (straddle).
  float mul = a.sc.mul, lin = 0.f, lin_slope = 0.f;
  const int pmin = bt.start + wrow, pmax = bt.start + wrow + 31;
  auto straddle = [&](f32x16 s[2], int t) __attribute__((always_inline)) {
    const bool after = t * BN >= pmax, both = !after && t * BN + BN - 1 > pmin;  // uniform
    lin_slope = after ? -slope : slope;
    const float dist = (float)(bt.start + qrow - t * BN - 4 * hi);
    lin = lin_slope * dist;
    if (!CAP) mul = a.sc.mul;
    if (!both) return;
#pragma unroll
    for (int blk = 0; blk < 2; ++blk)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const float y = CAP ? s[blk][i] : s[blk][i] * a.sc.mul;
        s[blk][i] = fmaf(2.f * slope, fmaxf((float)(32 * blk + 8 * (i >> 2) + (i & 3)) - dist, 0.f), y);
      }
    if (!CAP) mul = 1.f;
  };

  // y + n of element i of block blk; with a bias n holds lin
  auto logit = [&](float s, float n, int blk, int i) __attribute__((always_inline)) {
    if (FOLD) return s;
    float y = CAP ? s + n : fmaf(s, mul, n);
    if (BIAS) y = fmaf(lin_slope, -(float)(32 * blk + 8 * (i >> 2) + (i & 3)), y);
    return y;
  };
  // P of elements i, i + 1 of a block (one rounding of the weights for the product, at
  // most 2^-8 of each, independent: relative RMS error 1.7e-3).  The output is divided by the sum of the rounded weights, so that the
  // rounding of one that carries a row cancels; the log-sum-exp is of the sum before.
  auto exps = [&](const f32x16& s, int blk, int i, float n, uint32_t pw[8], float sum[2]) __attribute__((always_inline)) {
    const float p0 = __builtin_amdgcn_exp2f(logit(s[i], n, blk, i));
    const float p1 = __builtin_amdgcn_exp2f(logit(s[i + 1], n, blk, i + 1));
    pw[i >> 1] = pack_bf16x2(p0, p1);
    sum[1] = dot2(pw[i >> 1], 0x3f803f80u, sum[1]);
    if (LSE) {
      sum[0] += p0;
      sum[0] += p1;
    }
  };
  // The block's sum is not below 2^64 for some row: new references, the output and
  // sum rescaled, the block's weights formed again
  auto reset = [&](f32x16 s[2], int blk, uint32_t pw[8], float sum[2]) __attribute__((always_inline)) {
    float m = logit(s[blk][0], lin, blk, 0);
#pragma unroll
    for (int i = 1; i < 16; ++i) m = fmaxf(m, logit(s[blk][i], lin, blk, i));
    const float mnew = fmaxf(mref, wave_half_max(m) - (FOLD ? nm : 0.f));
    const bool set = mnew > -INFINITY;
    const float alpha = set ? __builtin_amdgcn_exp2f(mref - mnew) : 1.f;
    lsum *= alpha;
    wsum *= alpha;
#pragma unroll
    for (int mb = 0; mb < 4; ++mb)
#pragma unroll
      for (int i = 0; i < 16; ++i) oacc[mb][i] *= alpha;
    if (FOLD) {  // what the tile's scores already hold
#pragma unroll
      for (int z = blk; z < 2; ++z)
#pragma unroll
        for (int i = 0; i < 16; ++i) s[z][i] -= mnew + nm;
    }
    mref = mnew;
    nm = set ? -mnew : kUnset;
    sum[0] = sum[1] = 0.f;
#pragma unroll
    for (int i = 0; i < 16; i += 2) exps(s[blk], blk, i, nm + lin, pw, sum);
  };
  // The scores of the next tile (K in kb) and the softmax and PV of this one (V in
  // vb), hand-scheduled: a slot a product, each also issuing the operand reads of
  // the product three slots on and its share of the exponentials.
  auto products = [&](f32x16 s[2], f32x16 sn[2], const uint16_t* kb, const uint16_t* vb) __attribute__((always_inline)) {
    bf16x8 op[32];
    auto read_op = [&](auto N) __attribute__((always_inline)) {
      constexpr int n = decltype(N)::value;
      if constexpr (n < 16) {
        op[n] = *reinterpret_cast<const bf16x8*>(kb + n * BLK + koff);
      } else if constexpr (n < 32) {
        const i16x4 lo = lds_read_tr16(vb + (n - 16) * BLK + voff);
        const i16x4 up = lds_read_tr16(vb + (n - 16) * BLK + BLK / 2 + voff);
        op[n] = __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, up, 0, 1, 2, 3, 4, 5, 6, 7));
      }
    };
    uint32_t pw[2][8];
    float sum[2][2] = {{0.f, 0.f}, {0.f, 0.f}};
    auto p_op = [&](int blk, int k2) __attribute__((always_inline)) {
      return __builtin_bit_cast(bf16x8, make_uint4(pw[blk][4 * k2], pw[blk][4 * k2 + 1], pw[blk][4 * k2 + 2], pw[blk][4 * k2 + 3]));
    };
    float n0 = BIAS ? nm + lin : nm;
    for_slots<3>(read_op);
    SLOT();
    for_slots<16>([&](auto N) __attribute__((always_inline)) {  // scores; exponentials of block 0
      constexpr int n = decltype(N)::value;
      sn[n & 1] = mfma32(op[n], qreg[n >> 1], n < 2 ? f32x16{} : sn[n & 1]);
      read_op(std::integral_constant<int, n + 3>());
      if constexpr ((n & 1) == 0) exps(s[0], 0, n, n0, pw[0], sum[0]);
      SLOT();
    });
    if (__builtin_amdgcn_ballot_w64(!(sum[0][1] < kSumLimit)) != 0) reset(s, 0, pw[0], sum[0]);
    lsum += sum[0][0];
    wsum += sum[0][1];
    n0 = BIAS ? nm + lin : nm;
    SLOT();
    for_slots<8>([&](auto N) __attribute__((always_inline)) {  // PV of block 0; exponentials of block 1
      constexpr int n = decltype(N)::value;
      oacc[n & 3] = mfma32(op[16 + n], p_op(0, n >> 2), oacc[n & 3]);
      read_op(std::integral_constant<int, n + 19>());
      exps(s[1], 1, 2 * n, n0, pw[1], sum[1]);
      SLOT();
    });
    if (__builtin_amdgcn_ballot_w64(!(sum[1][1] < kSumLimit)) != 0) reset(s, 1, pw[1], sum[1]);
    lsum += sum[1][0];
    wsum += sum[1][1];
    SLOT();
    for_slots<8>([&](auto N) __attribute__((always_inline)) {  // PV of block 1
      constexpr int n = decltype(N)::value;
      oacc[n & 3] = mfma32(op[24 + n], p_op(1, n >> 2), oacc[n & 3]);
      read_op(std::integral_constant<int, n + 27>());
      SLOT();
    });
  };
  // -inf for what the lane's row does not see of the tile
  auto mask = [&](f32x16 s[2], const Tile& t, const int* ids) __attribute__((always_inline)) {
    int to = t.mine() ? lim - t.t * BN - 4 * hi : 0;
    if (docs && t.one() && qd != t.id) to = 0;
#pragma unroll
    for (int blk = 0; blk < 2; ++blk)
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if (32 * blk + 8 * (i >> 2) + (i & 3) >= to) s[blk][i] = -INFINITY;
    if (docs && !t.one()) {  // uniform
#pragma unroll
      for (int blk = 0; blk < 2; ++blk)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const int4 d = *reinterpret_cast<const int4*>(ids + 32 * blk + 8 * g + 4 * hi);
          if (d.x != qd) s[blk][4 * g] = -INFINITY;
          if (d.y != qd) s[blk][4 * g + 1] = -INFINITY;
          if (d.z != qd) s[blk][4 * g + 2] = -INFINITY;
          if (d.w != qd) s[blk][4 * g + 3] = -INFINITY;
        }
    }
  };
  // ---- output, whole rows through the staging area; empty rows: o = 0, lse = -inf
  const size_t nrow = (size_t)c.B * c.H * c.Lq, orow = ((size_t)b * c.H + h) * c.Lq;
  auto store_o = [&]() __attribute__((always_inline)) {
    const float w = wave_half_sum(wsum), l = LSE ? wave_half_sum(lsum) : w;
    const float inv = w == 0.f ? 0.f : 1.0f / w;
    const float lse2 = l == 0.f ? -INFINITY : mref + __log2f(l);
    if (PIECES ? !part.whole() : a.po != nullptr) {  // fp32 rows of this run or part
      if (qlive) {
        const size_t prow = PIECES ? (size_t)part.slot() * a.pieces.slot_rows + (qrow - row0) : (size_t)run * nrow + orow + qrow;
        float* const p = a.po + prow * D;
#pragma unroll
        for (int mb = 0; mb < 4; ++mb)
#pragma unroll
          for (int g = 0; g < 4; ++g)
            *reinterpret_cast<float4*>(p + 32 * mb + 8 * g + 4 * hi) =
                make_float4(oacc[mb][4 * g] * inv, oacc[mb][4 * g + 1] * inv, oacc[mb][4 * g + 2] * inv,
                            oacc[mb][4 * g + 3] * inv);
        if (hi == 0) a.pl[prow] = lse2;
      }
      return;
    }
#pragma unroll
    for (int mb = 0; mb < 4; ++mb)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        u32x2 pk;
        pk[0] = pack_bf16x2(oacc[mb][4 * g + 0] * inv, oacc[mb][4 * g + 1] * inv);
        pk[1] = pack_bf16x2(oacc[mb][4 * g + 2] * inv, oacc[mb][4 * g + 3] * inv);
        *reinterpret_cast<u32x2*>(stage + l32 * D + stage_slot(4 * mb + g, l32) * 8 + 4 * hi) = pk;
      }
    wave_lds_fence();
    const __amdgpu_buffer_rsrc_t ro = __builtin_amdgcn_make_buffer_rsrc(
        (void*)(a.o + (size_t)b * c.Lq * qtok + (size_t)h * D), (short)0, c.Lq * qbytes, kBufferFlags);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int r = 4 * i + (lane >> 4);
      const u32x4 v = *reinterpret_cast<const u32x4*>(stage + r * D + (lane & 15) * 8);
      const int grow = wrow + r;
      const int off = grow < c.Lq ? grow * qbytes + stage_slot(lane & 15, r) * 16 : 0x7ffffff0;
      __builtin_amdgcn_raw_buffer_store_b128(v, ro, off, 0, 0);
    }
    if (a.lse && qlive && hi == 0) a.lse[orow + qrow] = lse2 * kLn2;
  };

  Tile cur{-1, 0, 0}, nxt = cur;
  if (ntiles > 0) {
    if (PIECES) {
      look(grp);
    } else if (a.runs > 1) {  // this run's part of the tiles to visit
      int n = ntiles;
      if (docs) {
        n = 0;
        look(grp);
        do n += __builtin_popcountll(visit);
        while (more());
        above = false;
        grp = DOWN ? home >> 6 : 0;
      }
      int skip = (int)((int64_t)n * run / a.runs);
      left = (int)((int64_t)n * (run + 1) / a.runs) - skip;
      look(grp);
      while (left > 0 && skip >= __builtin_popcountll(visit)) {
        skip -= __builtin_popcountll(visit);
        more();
      }
      for (; left > 0 && skip > 0; --skip) first();
    } else {
      look(grp);
    }
    cur = next();
    nxt = next();
  }
  if (cur.t < 0) {  // nothing to see
    store_o();
    return;
  }
  dma_q();
  __builtin_amdgcn_s_waitcnt(0);  // this wave's query rows have landed
  take_q();
  __syncthreads();  // every wave has its queries out of the K/V buffers
  // ids of a tile's keys, in LDS for the step that masks it
  auto dma_ids = [&](const Tile& t, int* dst) __attribute__((always_inline)) {
    if (!docs || t.one() || wave != 0) return;
    const __amdgpu_buffer_rsrc_t rs =
        __builtin_amdgcn_make_buffer_rsrc((void*)(c.s.k_doc + (size_t)b * c.Lk), (short)0, c.Lk * 4, kBufferFlags);
    __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (lds_ptr)dst, 4, (t.t * BN + lane) * 4, 0, 0, 0);
  };
  dma_ids(cur, Kd[0]);
  dma_k(cur.t, K0);
  dma_v(cur, V0);
  if (nxt.t >= 0) dma_k(nxt.t, K1);
  __builtin_amdgcn_s_waitcnt(0);  // this wave's copies have landed in LDS
  __syncthreads();
  Tile aft = next();  // (known a step ahead: its keys are the first thing a step copies)
  f32x16 sa[2], sb[2];
  qk(K0, sa);
  __syncthreads();  // the first step refills K0
  // Step on the tile `cur` (parity of its buffers at compile time); false after the last
  auto step = [&](auto parity, f32x16 scur[2], f32x16 snext[2]) __attribute__((always_inline)) {
    constexpr int P = decltype(parity)::value;
    if (aft.t >= 0) dma_k(aft.t, P ? K1 : K0);
    if (nxt.t >= 0) {
      dma_ids(nxt, Kd[1 - P]);
      dma_v(nxt, P ? V0 : V1);
    }
    // A wave that needs only the products of the next tile or the softmax of this one
    // (at the ends of what it sees) does the other on whatever is there, unseen.
    if (cur.mine() || nxt.mine()) {
      if (CAP) {
        cap16_log2(scur[0], a.sc, FOLD ? nm : 0.f);
        cap16_log2(scur[1], a.sc, FOLD ? nm : 0.f);
      }
      if (BIAS) straddle(scur, cur.t);
      if (!(cur.mine() && cur.whole())) mask(scur, cur, Kd[P]);
      products(scur, snext, P ? K0 : K1, P ? V1 : V0);
    }
    cur = nxt;
    nxt = aft;
    aft = next();
    __builtin_amdgcn_s_waitcnt(0);  // this wave's copies have landed
    __syncthreads();
    return cur.t >= 0;
  };
  while (step(std::integral_constant<int, 0>(), sa, sb) && step(std::integral_constant<int, 1>(), sb, sa)) {
  }
  store_o();
}

template <bool CAP, bool BIAS, bool LSE>
__global__ __launch_bounds__(NT) void attn_mod_fwd_kernel(FwdArgs a) {
  fwd_body<CAP, BIAS, LSE, false>(a, Part{});
}
template <bool CAP, bool BIAS, bool LSE>
__device__ __forceinline__ void pieces_body(const FwdArgs& a) {
  each_part<QuerySide>(a.c, a.pieces.n, piece_of(blockIdx.x, a.pieces.n), [&](const Part& part) __attribute__((always_inline)) {
    if (threadIdx.x == 0) note_cut<QuerySide>(a.pieces, a.c, part);
    fwd_body<CAP, BIAS, LSE, true>(a, part);
    __syncthreads();  // (the staging areas)
  });
}
template <bool CAP, bool BIAS, bool LSE>
__global__ __launch_bounds__(NT) void attn_mod_pieces_kernel(FwdArgs a) {
  pieces_body<CAP, BIAS, LSE>(a);
}

// Ranges of document ids of every 32 tokens: a wave takes 64 tokens of a batch.
struct RangeArgs {
  const int32_t *k, *q;
  int2 *kr, *qr;
  int B, Lk, Lq, nk, nq;  // groups of 64 tokens a batch
};
__global__ __launch_bounds__(256) void mod_ranges_kernel(RangeArgs a) {
  const int lane = threadIdx.x & 63;
  int w = blockIdx.x * 4 + (threadIdx.x >> 6);
  const bool isk = w < a.B * a.nk;
  if (!isk) w -= a.B * a.nk;
  const int n = isk ? a.nk : a.nq, L = isk ? a.Lk : a.Lq;
  if (w >= a.B * n) return;
  const int b = w / n, g = w - b * n, t = 64 * g + lane;
  const bool live = t < L;
  const int id = live ? (isk ? a.k : a.q)[(size_t)b * L + t] : -1;
  int lo = id >= 0 ? id : 0x7fffffff, hi = id >= 0 ? id : 0;
#pragma unroll
  for (int m = 1; m < 32; m <<= 1) {
    lo = min(lo, __shfl_xor(lo, m));
    hi = max(hi, __shfl_xor(hi, m));
  }
  const uint64_t bad = __builtin_amdgcn_ballot_w64(live && id < 0);
  const bool neg = (uint32_t)(lane < 32 ? bad : bad >> 32) != 0;
  if ((lane & 31) == 0) {
    int2* const out = (isk ? a.kr : a.qr) + (size_t)w * 2 + (lane >> 5);
    *out = make_int2(lo, hi | (neg ? (int)0x80000000 : 0));
  }
}

// The order in which the 256-row tiles of the queries (block 0 + first) or keys (1)
// are handed out: most tiles of the other side to visit first.  Documents make
// tiles of very different work; in their own order the last ones to start held
// the launch up (five clips in 16380 tokens, 12 heads, forward: 480 us; sorted 403).  A wave
// counts a tile's work, 64 tiles of the other side at a time; ranks by counting.
constexpr size_t kOrderMost = 4096;
struct OrderArgs {
  ModCall c;
  ModRanges r;
  int nq, nk, first;
  int32_t *oq, *ok;
};
__global__ __launch_bounds__(1024) void mod_order_kernel(OrderArgs a) {
  __shared__ int work[kOrderMost];
  const ModCall& c = a.c;
  const bool isq = blockIdx.x + a.first == 0;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int tiles = isq ? a.nq : a.nk, n = c.B * tiles;
  const int own_len = isq ? c.Lq : c.Lk, other_len = isq ? c.Lk : c.Lq;
  const int own_r = (int)mod_ranges(own_len), other_r = (int)mod_ranges(other_len);
  const int2* const own = isq ? a.r.q : a.r.k;
  const int2* const other = isq ? a.r.k : a.r.q;
  for (int i = wave; i < n; i += 16) {
    const int b = i / tiles, t = i - b * tiles;
    const Batch bt = batch_of(c, b);
    Docs d{0x7fffffff, 0, false};  // (lanes l, l + 8, .. the tile's range l)
    if (8 * t + (lane & 7) < own_r) d = docs_of(own[(size_t)b * own_r + 8 * t + (lane & 7)]);
#pragma unroll
    for (int m = 1; m < 8; m <<= 1) d = mod::join(d, Docs{__shfl_xor(d.lo, m), __shfl_xor(d.hi, m), false});
    // the part of the other side that the limits leave: keys [0, to), queries [from, ..)
    const int last = min((t + 1) * BM, own_len) - 1;
    const int to = isq ? key_limit(bt, c.s.causal, bt.start + last) : other_len;
    const int from = !isq && c.s.causal && t * BM >= bt.prefix ? max(t * BM - bt.start, 0) : 0;
    int w = 0;
    for (int o = 0; o < to; o += 4 * 4096) {  // (four loads in flight)
      int4 r[4];
#pragma unroll
      for (int u = 0; u < 4; ++u)
        r[u] = *reinterpret_cast<const int4*>(other + (size_t)b * other_r + 2 * min(o / 64 + 64 * u + lane, other_r / 2 - 1));
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int g = o / 64 + 64 * u + lane;
        const bool v = g * 64 < to && g * 64 + 63 >= from &&
                       meet(d, mod::join(docs_of(make_int2(r[u].x, r[u].y)), docs_of(make_int2(r[u].z, r[u].w))));
        w += __builtin_popcountll(__builtin_amdgcn_ballot_w64(v));
      }
    }
    if (lane == 0) work[i] = w;
  }
  __syncthreads();
  for (int i = threadIdx.x; i < n; i += 1024) {
    const int w = work[i];
    int rank = 0;
    for (int j = 0; j < n; ++j) rank += work[j] > w || (work[j] == w && j < i);
    (isq ? a.oq : a.ok)[rank] = i;
  }
}

// Eight values of a row from its partial results p0 .. p1, row at(p) each: sum_p
// 2^(lse_p - max) o_p / sum_p 2^(lse_p - max).  A part that saw nothing wrote zeros:
// weight 0.  (o_p is a mean by the rounded weights of the part; what the part counts for
// is its sum before the rounding where the log-sum-exps are wanted, which is then known,
// and the sum of the roundings otherwise.)
struct Joined {
  uint4 o;
  float lse;  // natural
};
template <typename At>
__device__ __forceinline__ Joined join_parts(const float* po, const float* pl, int p0, int p1, At&& at) {
  float m = -INFINITY;
#pragma unroll 4
  for (int p = p0; p <= p1; ++p) m = fmaxf(m, pl[at(p)]);
  const float ref = m > -INFINITY ? m : 0.f;
  float4 x0 = make_float4(0.f, 0.f, 0.f, 0.f), x1 = x0;
  float l = 0.f;
#pragma unroll 4
  for (int p = p0; p <= p1; ++p) {
    const float w = __builtin_amdgcn_exp2f(pl[at(p)] - ref);
    const float4 u = *reinterpret_cast<const float4*>(po + at(p) * D);
    const float4 v = *reinterpret_cast<const float4*>(po + at(p) * D + 4);
    l += w;
    x0.x = fmaf(w, u.x, x0.x); x0.y = fmaf(w, u.y, x0.y); x0.z = fmaf(w, u.z, x0.z); x0.w = fmaf(w, u.w, x0.w);
    x1.x = fmaf(w, v.x, x1.x); x1.y = fmaf(w, v.y, x1.y); x1.z = fmaf(w, v.z, x1.z); x1.w = fmaf(w, v.w, x1.w);
  }
  const float inv = l > 0.f ? 1.0f / l : 0.f;
  Joined y;
  y.o.x = pack_bf16x2(x0.x * inv, x0.y * inv);
  y.o.y = pack_bf16x2(x0.z * inv, x0.w * inv);
  y.o.z = pack_bf16x2(x1.x * inv, x1.y * inv);
  y.o.w = pack_bf16x2(x1.z * inv, x1.w * inv);
  y.lse = l > 0.f ? (m + __log2f(l)) * kLn2 : -INFINITY;
  return y;
}

// Joins the parts of the tiles that pieces have cut: 16 rows a workgroup, 8 values of a
// row a thread.
struct PieceJoinArgs {
  const float *po, *pl;
  uint16_t* o;
  float* lse;
  Pieces pieces;
  int H, Lq, ntile;
};
__global__ __launch_bounds__(256) void mod_piece_join_kernel(PieceJoinArgs a) {
  const int tile = blockIdx.x >> 4, sub = blockIdx.x & 15;
  const int p0 = __builtin_amdgcn_readfirstlane(a.pieces.cut[2 * tile]);
  if (p0 < 0) return;
  const int p1 = __builtin_amdgcn_readfirstlane(a.pieces.cut[2 * tile + 1]);
  const int bh = tile / a.ntile, r = 16 * sub + (threadIdx.x >> 4), i = (tile - bh * a.ntile) * BM + r;
  if (i >= a.Lq) return;
  const int b = bh / a.H, h = bh - b * a.H, ch = 8 * (threadIdx.x & 15);
  const Joined y = join_parts(a.po + ch, a.pl, p0, p1,
                              [&](int p) { return (size_t)(2 * p + (p == p0)) * a.pieces.slot_rows + r; });
  *reinterpret_cast<uint4*>(a.o + (((size_t)b * a.Lq + i) * a.H + h) * D + ch) = y.o;
  if (a.lse && ch == 0) a.lse[(size_t)bh * a.Lq + i] = y.lse;
}

// Joins the runs of every (batch, head, query): 16 rows a workgroup, 8 values of a row a
// thread.  o = sum_r 2^(lse_r - max) o_r / sum_r 2^(lse_r - max).
struct JoinArgs {
  const float *po, *pl;
  uint16_t* o;
  float* lse;
  int B, H, Lq, runs;
};
__global__ __launch_bounds__(256) void mod_join_kernel(JoinArgs a) {
  const size_t nrow = (size_t)a.B * a.H * a.Lq;
  const size_t row = (size_t)blockIdx.x * 16 + (threadIdx.x >> 4);  // (b, h, i)
  if (row >= nrow) return;
  const size_t i = row % a.Lq, bh = row / a.Lq, b = bh / a.H, h = bh % a.H;
  const int ch = 8 * (threadIdx.x & 15);
  const Joined y = join_parts(a.po + ch, a.pl, 0, a.runs - 1, [&](int r) { return r * nrow + row; });
  *reinterpret_cast<uint4*>(a.o + ((b * a.Lq + i) * a.H + h) * D + ch) = y.o;
  if (a.lse && ch == 0) a.lse[row] = y.lse;
}

}  // namespace

hipError_t launch_mod_ranges(const ModCall& c, float* ws, bool q_order, bool k_order, ModRanges* out, hipStream_t stream) {
  *out = ModRanges{nullptr, nullptr, nullptr, nullptr};
  if (!c.s.k_doc) return hipSuccess;
  RangeArgs a;
  a.k = c.s.k_doc;
  a.q = c.s.q_doc;
  a.B = c.B;
  a.Lk = c.Lk;
  a.Lq = c.Lq;
  a.nk = (int)(mod_ranges(c.Lk) / 2);
  a.nq = (int)(mod_ranges(c.Lq) / 2);
  a.kr = reinterpret_cast<int2*>(ws);
  a.qr = a.kr + (size_t)c.B * mod_ranges(c.Lk);
  out->k = a.kr;
  out->q = a.qr;
  const unsigned waves = (unsigned)c.B * (unsigned)(a.nk + a.nq);
  const hipError_t e = launch_kernel(mod_ranges_kernel, (waves + 3) / 4, 256u, stream, a);
  OrderArgs o;
  o.c = c;
  o.r = *out;
  o.nq = (int)mod_tiles(c.Lq);
  o.nk = (int)mod_tiles(c.Lk);
  o.oq = reinterpret_cast<int32_t*>(a.qr + (size_t)c.B * mod_ranges(c.Lq));
  o.ok = o.oq + (size_t)c.B * o.nq;
  q_order = q_order && (size_t)c.B * o.nq <= kOrderMost;
  k_order = k_order && (size_t)c.B * o.nk <= kOrderMost;
  if (e != hipSuccess || !(q_order || k_order)) return e;
  o.first = q_order ? 0 : 1;
  if (q_order) out->q_order = o.oq;
  if (k_order) out->k_order = o.ok;
  return launch_kernel(mod_order_kernel, (q_order && k_order) ? 2u : 1u, 1024u, stream, o);
}

namespace {
hipError_t launch_mod_join(const ModFwd& f, const ModSplit& s, hipStream_t stream) {
  JoinArgs a;
  const size_t nrow = (size_t)f.c.B * f.c.H * f.c.Lq;
  a.po = f.ws + s.part;
  a.pl = a.po + (size_t)s.runs * nrow * D;
  a.o = f.o;
  a.lse = f.lse;
  a.B = f.c.B;
  a.H = f.c.H;
  a.Lq = f.c.Lq;
  a.runs = s.runs;
  return launch_kernel(mod_join_kernel, (unsigned)((nrow + 15) / 16), 256u, stream, a);
}
}  // namespace

hipError_t launch_attn_mod_fwd(const ModFwd& f, hipStream_t stream) {
#define LAUNCH_LSE(kernel, grid, CAP, BIAS)                                                       \
  (a.lse ? launch_kernel(kernel<CAP, BIAS, true>, grid, (unsigned)NT, stream, a)                  \
         : launch_kernel(kernel<CAP, BIAS, false>, grid, (unsigned)NT, stream, a))
#define LAUNCH(kernel, grid)                                                                      \
  (cap ? (bias ? LAUNCH_LSE(kernel, grid, true, true) : LAUNCH_LSE(kernel, grid, true, false))    \
       : (bias ? LAUNCH_LSE(kernel, grid, false, true) : LAUNCH_LSE(kernel, grid, false, false)))
  const ModCall& c = f.c;
  const ModSplit s = mod_fwd_split(c, device_cu_count(), f.ws_floats);
  FwdArgs a;
  a.c = c;
  a.sc = make_scores(c);
  a.q = f.q;
  a.k = f.k;
  a.v = f.v;
  a.o = f.o;
  a.lse = f.lse;
  a.ntile = (c.Lq + BM - 1) / BM;
  a.first_most = 0;
  a.runs = s.runs;
  a.nwg = a.ntile * c.B * c.H * s.runs;
  a.sorted = a.nwg > device_cu_count() && (c.s.k_doc || c.s.causal || c.s.kv_valid_len);
  a.kr = (int)mod_ranges(c.Lk);
  a.qr = (int)mod_ranges(c.Lq);
  a.po = s.runs > 1 ? f.ws + s.part : nullptr;
  a.pl = s.runs > 1 ? a.po + (size_t)s.runs * c.B * c.H * c.Lq * D : nullptr;
  hipError_t e = launch_mod_ranges(c, f.ws, !s.few && a.sorted, false, &a.r, stream);
  if (e != hipSuccess) return e;
  if (s.few) return launch_mod_few(f, s, a.r, stream);
  // (a cap too large to fold its reference: the kernel with a bias, which is then 0)
  const bool cap = c.s.cap > 0.f, bias = c.s.slopes || (cap && a.sc.mul > kFoldMost);
  if (s.pieces.n) {
    a.po = f.ws + s.part;
    a.pl = a.po + (size_t)2 * s.pieces.n * s.pieces.slot_rows * D;
    a.pieces = Pieces{s.pieces.n, s.pieces.slot_rows, reinterpret_cast<int32_t*>(f.ws + s.pieces.cut)};
    e = LAUNCH(attn_mod_pieces_kernel, (unsigned)s.pieces.n);
    if (e != hipSuccess) return e;
    const PieceJoinArgs j{a.po, a.pl, f.o, f.lse, a.pieces, c.H, c.Lq, a.ntile};
    return launch_kernel(mod_piece_join_kernel, (unsigned)(a.ntile * c.B * c.H * 16), 256u, stream, j);
  }
  for (int r = 0; r < kMostRuns; ++r) a.in_run[r] = a.r.q_order ? a.ntile * c.B : a.ntile;
  e = LAUNCH(attn_mod_fwd_kernel, (unsigned)a.nwg);
  if (e != hipSuccess || s.runs == 1) return e;
  return launch_mod_join(f, s, stream);
#undef LAUNCH
#undef LAUNCH_LSE
}

}  // namespace vidax
