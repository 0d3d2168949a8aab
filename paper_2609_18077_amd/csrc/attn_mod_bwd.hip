// Attention with score modifiers, backward, for gfx950: with x = scale q.k, t =
// tanh(x / cap) and P = exp(s - lse) on the keys that a query sees (else 0),
//
//   D_i = <dO_i, O_i>,  dS = P (dO V^T - D) (1 - t^2)      (1 - t^2 with a cap)
//   dQ = scale dS K                 dq kernel: 256 queries of a head a workgroup
//   dV = P^T dO, dK = scale dS^T Q  dkdv kernel: 256 keys of a K/V head a
//                                   workgroup, the queries of all its query heads
//                                   streamed past (their sum needs no atomics)
//
// The dataflow is the dense backward's (attn_bwd.hip): 32 own rows a wave, the
// streamed tiles of 64 rows in LDS as permuted 256-byte rows, read by rows and
// transposed, double-buffered, one barrier a tile.  The tiles to visit and to mask
// are found as in the forward (attn_mod_fwd.hip), for the key side with the roles
// of queries and keys exchanged.  Rows that see nothing (lse = -inf) get P = 0 and
// count as zeros wherever they are read, as do keys that nothing sees.
//   P and dS are rounded to bf16 once, for the matrix products that take them (at most
// 2^-8 of each, independent: relative RMS error 2.4e-3 with the result's own rounding;
// fp32 operands run at a sixteenth of the rate).  D is formed from the output as the
// forward returned it, in bf16: its rounding counts where few keys carry a row (3.7e-3).
#include "attn_mod.hpp"
#include "launch.hpp"

namespace vidax {
namespace {

using namespace tile;
using namespace mod;

constexpr int D = kHeadDim;
constexpr int BN = 64;         // rows of a streamed tile
constexpr int NW = 8;
constexpr int NT = NW * 64;
constexpr int TILE = BN * D;   // elements
constexpr int BM = 256;        // own rows of a workgroup
constexpr int kOff = 0x7ffffff0;  // past any buffer's records

struct BwdArgs {
  ModCall c;
  Scores sc;
  const uint16_t *q, *k, *v, *o, *dout;
  const float* lse;
  uint16_t *dq, *dk, *dv;
  float *delta, *nlse;  // [B, H, Lq]: -D, -lse log2 e (-inf for rows that see nothing)
  int32_t* empty;     // [B][qr]: whether a row of these 32 sees nothing
  ModRanges r;
  int kr, qr;         // ranges a batch
  int ntile, nwg;     // tiles of own rows a head, workgroups of the launched kernel
  int runs, quantum;  // key side: a stream of more than quantum tiles goes to several workgroups, runs at most
  int in_run[kMostRuns];   // see place()
  int32_t* counts;    // [B][tiles of keys]: how many
  int sorted, first_most;  // see place(); causal: the first tile of a head has the most work (else the last)
  float* dqp;         // dq in pieces: partial sums [slots][slot_rows][D]
  Pieces pieces;
  float* part;        // fp32 dK, dV of every run of those tiles ([runs][B][Lk][Hkv][D], dV after dK)
};

// Rows 16 k2 .. + 15 of an accumulator as a bf16 B operand, in the accumulator's row order.
__device__ __forceinline__ bf16x8 pack8(const f32x16& x, int k2) {
  uint32_t w[4];
#pragma unroll
  for (int e = 0; e < 8; e += 2) w[e >> 1] = pack_bf16x2(x[8 * k2 + e], x[8 * k2 + e + 1]);
  return __builtin_bit_cast(bf16x8, make_uint4(w[0], w[1], w[2], w[3]));
}
// Row of register i of accumulator block blk, of lane half 0.
constexpr int acc_row(int blk, int i) { return 32 * blk + 8 * (i >> 2) + (i & 3); }
// x, as a value of iteration t (what is computed from it stays in the loop).
__device__ __forceinline__ int in_loop(int x, int t) {
  asm("" : "+v"(x) : "s"(t));
  return x;
}
__device__ __forceinline__ bf16x8 apply_sign(uint4 x, const Scores& s) {
  return __builtin_bit_cast(bf16x8, make_uint4((x.x ^ s.qxor) & s.qand, (x.y ^ s.qxor) & s.qand, (x.z ^ s.qxor) & s.qand,
                                               (x.w ^ s.qxor) & s.qand));
}
// 1 - t^2; 0 for the -inf of what is not seen.
__device__ __forceinline__ float cap_slope(float t) { return __builtin_amdgcn_fmed3f(fmaf(-t, t, 1.f), 0.f, 1.f); }
// 0 for the 16 elements of a block that are seen, -inf for the others: the value
// that their products start from (or that replaces them, after a cap).
//   causal part: element rows [from, to) of the lane half's block are seen;
//   documents (ids != null, uniform): those of id `own` (four 16-byte LDS reads).
template <typename F>
__device__ __forceinline__ void each_hidden(int from, int to, const int* ids, int own, F&& hide) {
#pragma unroll
  for (int i = 0; i < 16; ++i)
    if (acc_row(0, i) < from || acc_row(0, i) >= to) hide(i);
  if (ids) {
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const int4 d = *reinterpret_cast<const int4*>(ids + 8 * g);
      if (d.x != own) hide(4 * g);
      if (d.y != own) hide(4 * g + 1);
      if (d.z != own) hide(4 * g + 2);
      if (d.w != own) hide(4 * g + 3);
    }
  }
}
// The 4-byte values of 64-row tile t (of L rows at base; zero behind) into LDS, one wave.
template <typename T>
__device__ __forceinline__ void copy_row(const T* base, int t, int L, T* dst, int lane) {
  const __amdgpu_buffer_rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc((void*)base, (short)0, L * 4, kBufferFlags);
  __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (lds_ptr)dst, 4, (t * BN + lane) * 4, 0, 0, 0);
}
// 64-row tile `t` of rows [0, limit) of a buffer (one at least): later rows read as zero.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t tile_rsrc(const uint16_t* base, int t, int limit, int tok) {
  const int nbytes = min(limit - t * BN, BN) * tok * 2;
  return __builtin_amdgcn_make_buffer_rsrc((void*)(base + (size_t)t * BN * tok), (short)0, nbytes, kBufferFlags);
}

// ------------------------------------------------------------------- dQ ----

// PIECES: the part of a query tile's keys given.
template <bool CAP, bool BIAS, bool PIECES>
__device__ __forceinline__ void dq_body(const BwdArgs& a, const Part& part) {
  __shared__ __attribute__((aligned(1024))) uint16_t K0[TILE], K1[TILE], V0[TILE], V1[TILE];
  __shared__ __attribute__((aligned(16))) int Kd[2][BN];  // ids of the tiles' keys
  const int tid = threadIdx.x, lane = tid & 63, l32 = lane & 31, hi = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const ModCall& c = a.c;
  int b, h, qt, run;
  if constexpr (PIECES) {
    b = part.b;
    h = part.h;
    qt = part.t;
  } else {
    place(a, c.H, a.r.q_order, run, qt, b, h);
  }
  const int hk = h / (c.H / c.Hkv);
  const int qtok = c.H * D, qbytes = qtok * 2, ktok = c.Hkv * D, kbytes = ktok * 2;
  const Batch bt = batch_of(c, b);
  const int row0 = qt * BM, wrow = row0 + wave * 32, qrow = wrow + l32;
  const bool qlive = qrow < c.Lq;
  const int wlast = min(wrow + 32, c.Lq) - 1, glast = min(row0 + BM, c.Lq) - 1;
  const size_t lrow = ((size_t)b * c.H + h) * c.Lq + (qlive ? qrow : 0);
  float lse = qlive ? a.lse[lrow] : -INFINITY;
  const bool none = lse == -INFINITY;  // the row sees nothing
  const float lse2 = none ? INFINITY : lse * kLog2e;

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
      if (first + i < a.qr) gdoc = mod::join(gdoc, docs_of(qr[first + i]));
    gdoc = uniform(gdoc);
    wdoc = wrow < c.Lq ? uniform(docs_of(qr[wrow >> 5])) : Docs{0x7fffffff, 0, false};
  }
  const int wmax = wlast >= wrow ? key_limit(bt, c.s.causal, bt.start + wlast) : 0;
  const int wmin = wlast >= wrow ? key_limit(bt, c.s.causal, bt.start + wrow) : 0;
  const int gmax = key_limit(bt, c.s.causal, bt.start + glast);
  const int end_tile = PIECES ? part.hi : (gmax + BN - 1) / BN, tile0 = PIECES ? part.lo : 0;

  int grp = tile0 >> 6, fl = 0, id = 0;
  uint64_t visit = 0;
  auto look = [&](int g) __attribute__((always_inline)) {
    const int t = 64 * g + lane;
    bool v = t >= tile0 && t < end_tile;
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
  auto next = [&]() __attribute__((always_inline)) {
    while (visit == 0) {
      if (64 * (grp + 1) >= end_tile) return Tile{-1, 0, 0};
      look(++grp);
    }
    const int i = __builtin_ctzll(visit);
    visit &= visit - 1;
    return Tile{64 * grp + i, __builtin_amdgcn_readlane(fl, i), __builtin_amdgcn_readlane(id, i)};
  };

  // own rows in and out whole, through the tile buffers
  uint16_t* const area = (wave < 2 ? K0 : wave < 4 ? K1 : wave < 6 ? V0 : V1) + (wave & 1) * 32 * D;
  const size_t off0 = ((size_t)b * c.Lq + wrow) * qtok + (size_t)h * D;
  auto rows_rsrc = [&](const uint16_t* base) __attribute__((always_inline)) {
    return __builtin_amdgcn_make_buffer_rsrc(
        (void*)(base + off0), (short)0, __builtin_amdgcn_readfirstlane(min(max(c.Lq - wrow, 0), 32) * qbytes), kBufferFlags);
  };
  auto row_off = [&](int i) __attribute__((always_inline)) {
    const int r = 4 * i + (lane >> 4);
    return r * qbytes + ((lane & 15) ^ swz(r)) * 16;
  };
  auto rows_in = [&](const uint16_t* base) __attribute__((always_inline)) {
    const __amdgpu_buffer_rsrc_t rs = rows_rsrc(base);
#pragma unroll
    for (int i = 0; i < 8; ++i)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (lds_ptr)(area + 4 * i * D), 16, row_off(i), 0, 0, 0);
  };
  const RowOffsets off = row_offsets(lane);
  auto own_rows = [&](bf16x8 op[8]) __attribute__((always_inline)) {
#pragma unroll
    for (int s = 0; s < 8; ++s) op[s] = read_row(area, off.row, s);
  };
  f32x16 acc[4];
#pragma unroll
  for (int mb = 0; mb < 4; ++mb) acc[mb] = f32x16{};
  auto rows_out = [&](float mul) __attribute__((always_inline)) {
    if (PIECES && !part.whole()) {  // fp32 rows of this part
      if (!qlive) return;
      float* const p = a.dqp + ((size_t)part.slot() * a.pieces.slot_rows + (qrow - row0)) * D;
      if (none) mul = 0.f;
#pragma unroll
      for (int mb = 0; mb < 4; ++mb)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          float4 x = make_float4(acc[mb][4 * g] * mul, acc[mb][4 * g + 1] * mul, acc[mb][4 * g + 2] * mul, acc[mb][4 * g + 3] * mul);
          if (none) x = make_float4(0.f, 0.f, 0.f, 0.f);
          *reinterpret_cast<float4*>(p + 32 * mb + 8 * g + 4 * hi) = x;
        }
      return;
    }
#pragma unroll
    for (int mb = 0; mb < 4; ++mb)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        uint2 pk;
        pk.x = pack_bf16x2(acc[mb][4 * g + 0] * mul, acc[mb][4 * g + 1] * mul);
        pk.y = pack_bf16x2(acc[mb][4 * g + 2] * mul, acc[mb][4 * g + 3] * mul);
        if (none) pk = make_uint2(0u, 0u);
        *reinterpret_cast<uint2*>(area + l32 * D + ((4 * mb + g) ^ swz(l32)) * 8 + 4 * hi) = pk;
      }
    wave_lds_fence();
    const __amdgpu_buffer_rsrc_t rs = rows_rsrc(a.dq);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const u32x4 v = *reinterpret_cast<const u32x4*>(area + (4 * i + (lane >> 4)) * D + (lane & 15) * 8);
      __builtin_amdgcn_raw_buffer_store_b128(v, rs, row_off(i), 0, 0);
    }
  };
  bf16x8 dop[8], qop[8], oop[8];
  rows_in(a.dout);
  {
    const uint16_t* const p = a.o + ((size_t)b * c.Lq + (qlive ? qrow : 0)) * qtok + (size_t)h * D;
#pragma unroll
    for (int s = 0; s < 8; ++s) oop[s] = *reinterpret_cast<const bf16x8*>(p + (2 * s + hi) * 8);
  }
  __builtin_amdgcn_s_waitcnt(0);  // this wave's rows have landed
  own_rows(dop);
  const bf16x8 zero8 = __builtin_bit_cast(bf16x8, make_uint4(0, 0, 0, 0));
#pragma unroll
  for (int s = 0; s < 8; ++s)
    if (none) dop[s] = oop[s] = zero8;
  __builtin_amdgcn_s_waitcnt(0);  // dO is out of the area
  rows_in(a.q);
  float dl;
  {
    float sum[2] = {0.f, 0.f};
#pragma unroll
    for (int s = 0; s < 8; ++s) {
      const uint4 x = __builtin_bit_cast(uint4, dop[s]), y = __builtin_bit_cast(uint4, oop[s]);
      const uint32_t xw[4] = {x.x, x.y, x.z, x.w}, yw[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
      for (int p = 0; p < 4; ++p) sum[p & 1] = dot2(xw[p], yw[p], sum[p & 1]);
    }
    dl = wave_half_sum(sum[0] + sum[1]);
    const bool first = !PIECES || part.lo == 0;  // of the tile's parts
    if (first && qlive && hi == 0) {
      a.delta[lrow] = -dl;
      a.nlse[lrow] = -lse2;
    }
    const uint64_t bad = __builtin_amdgcn_ballot_w64(qlive && none);
    if (first && h == 0 && lane == 0 && wrow < c.Lq) a.empty[(size_t)b * a.qr + (wrow >> 5)] = bad != 0;
  }
  __builtin_amdgcn_s_waitcnt(0);
  own_rows(qop);
#pragma unroll
  for (int s = 0; s < 8; ++s) qop[s] = none ? zero8 : apply_sign(__builtin_bit_cast(uint4, qop[s]), a.sc);
  __builtin_amdgcn_s_waitcnt(0);  // the rows are out of the staging areas
  __syncthreads();

  Tile cur{-1, 0, 0}, nxt = cur;
  if (end_tile > 0) {
    look(grp);
    cur = next();
  }
  if (cur.t < 0) {  // nothing to see: dQ = 0
    rows_out(0.f);
    return;
  }
  const uint16_t* const kbh = a.k + (size_t)b * c.Lk * ktok + (size_t)hk * D;
  const uint16_t* const vbh = a.v + (size_t)b * c.Lk * ktok + (size_t)hk * D;
  // the wave's copies 2 wave, 2 wave + 1 of a tile (4 rows each)
  auto copies = [&](const Tile& t, uint16_t* kb, uint16_t* vb, int* ids) __attribute__((always_inline)) {
    if (docs && !t.one() && wave == 0) copy_row(c.s.k_doc + (size_t)b * c.Lk, t.t, c.Lk, ids, lane);
    const __amdgpu_buffer_rsrc_t rk = tile_rsrc(kbh, t.t, gmax, ktok), rv = tile_rsrc(vbh, t.t, gmax, ktok);
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int r = 4 * (2 * wave + u) + (lane >> 4);
      int g = r * kbytes + ((lane & 15) ^ swz(r)) * 16;
      if (t.zero()) {  // uniform: keys of negative documents arrive as zeros
        const int key = t.t * BN + r;
        if (key >= c.Lk || c.s.k_doc[(size_t)b * c.Lk + min(key, c.Lk - 1)] < 0) g = kOff;
      }
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rk, (lds_ptr)(kb + (2 * wave + u) * 512), 16, g, 0, 0, 0);
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rv, (lds_ptr)(vb + (2 * wave + u) * 512), 16, g, 0, 0, 0);
    }
  };
  copies(cur, K0, V0, Kd[0]);
  __builtin_amdgcn_s_waitcnt(0);
  __syncthreads();

  const float mul = a.sc.mul;
  const float slope = BIAS ? -c.s.slopes[h] * kLog2e : 0.f;
  // One tile, one slot a product, as in the dense backward: each slot issues the
  // operand reads of the product three slots on and its share of the vector work.
  // What the row does not see starts at -inf, which the products keep.  With a cap
  // both blocks' scores come first (their tanh branches), the exponentials run
  // beside dP, and what is not seen becomes -inf after the tanh.
  auto products = [&](const Tile& t, const uint16_t* kt, const uint16_t* vt, const int* ids) __attribute__((always_inline)) {
    const int orow = in_loop(off.row, t.t), otr = in_loop(off.tr, t.t);
    f32x16 sc[2], dp[2];
    bf16x8 ds[2][2];
    const float dist = BIAS ? (float)(bt.start + qrow - t.t * BN - 4 * hi) : 0.f;
    auto hidden = [&](int blk, f32x16& x) __attribute__((always_inline)) {
      each_hidden(INT32_MIN, docs && t.one() && qd != t.id ? 0 : lim - t.t * BN - 4 * hi - 32 * blk,
                  docs && !t.one() ? ids + 32 * blk + 4 * hi : nullptr, qd,
                  [&](int i) __attribute__((always_inline)) { x[i] = -INFINITY; });
    };
    auto exps = [&](int blk, int i0) __attribute__((always_inline)) {
#pragma unroll
      for (int i = i0; i < i0 + 2; ++i) {
        const float s = sc[blk][i];
        float x = fmaf(s, mul, -lse2);
        if (BIAS) x = fmaf(slope, fabsf(dist - (float)acc_row(blk, i)), x);
        float p = __builtin_amdgcn_exp2f(x);
        if (CAP) p *= cap_slope(s);
        sc[blk][i] = p;
      }
    };
    auto mul4 = [&](int blk, int i0) __attribute__((always_inline)) {
#pragma unroll
      for (int i = i0; i < i0 + 4; ++i) dp[blk][i] *= sc[blk][i];
    };
    // products in order: S0 dP0 S1 dP1 dQ0 dQ1, with a cap S0 S1 dP0 dP1 dQ0 dQ1
    bf16x8 op[48];
    auto read_op = [&](auto N) __attribute__((always_inline)) {
      constexpr int n = decltype(N)::value;
      if constexpr (n < 48) {
        constexpr bool isv = CAP ? (n >> 4) & 1 : (n >> 3) & 1;
        constexpr int blk = n >= 32 ? (n - 32) >> 3 : CAP ? (n >> 3) & 1 : n >> 4;
        if constexpr (n >= 32) op[n] = read_tr(kt + (32 * blk + 16 * ((n >> 2) & 1)) * D, otr, n & 3);
        else op[n] = read_row((isv ? vt : kt) + 32 * blk * D, orow, n & 7);
      }
    };
    auto product = [&](auto N) __attribute__((always_inline)) {
      constexpr int n = decltype(N)::value, u = n & 7;
      constexpr bool isv = CAP ? (n >> 4) & 1 : (n >> 3) & 1;
      constexpr int blk = n >= 32 ? (n - 32) >> 3 : CAP ? (n >> 3) & 1 : n >> 4;
      if constexpr (n >= 32) acc[u & 3] = mfma32(op[n], ds[blk][u >> 2], acc[u & 3]);
      else if constexpr (isv) {
        if constexpr (u == 0)
#pragma unroll
          for (int i = 0; i < 16; ++i) dp[blk][i] = -dl;
        dp[blk] = mfma32(op[n], dop[u], dp[blk]);
      } else if constexpr (u > 0 || CAP) {
        sc[blk] = mfma32(op[n], qop[u], u == 0 ? f32x16{} : sc[blk]);
      } else if (t.whole()) {  // uniform
        sc[blk] = mfma32(op[n], qop[u], f32x16{});
      } else {
        f32x16 x = f32x16{};
        hidden(blk, x);
        sc[blk] = mfma32(op[n], qop[u], x);
      }
    };
    // vector work of block vb from slot `from` on: eight slots of exponentials, four of products, the packs
    auto vector = [&](auto N, auto V, auto F) __attribute__((always_inline)) {
      constexpr int vb = decltype(V)::value, r = decltype(N)::value - decltype(F)::value;
      if constexpr (r >= 0 && r < 8) exps(vb, 2 * r);
      if constexpr (r >= 8 && r < 12) mul4(vb, 4 * (r - 8));
      if constexpr (r == 10) ds[vb][0] = pack8(dp[vb], 0);
      if constexpr (r == 12) ds[vb][1] = pack8(dp[vb], 1);
    };
    using zero = std::integral_constant<int, 0>;
    using one = std::integral_constant<int, 1>;
    for_slots<3>(read_op);
    SLOT();
    if constexpr (CAP) {
      for_slots<16>([&](auto N) __attribute__((always_inline)) {
        product(N);
        read_op(std::integral_constant<int, decltype(N)::value + 3>());
        SLOT();
      });
      cap16(sc[0], a.sc);
      cap16(sc[1], a.sc);
      if (!t.whole()) {
        hidden(0, sc[0]);
        hidden(1, sc[1]);
      }
      for_slots<32>([&](auto M) __attribute__((always_inline)) {
        using N = std::integral_constant<int, decltype(M)::value + 16>;
        product(N());
        read_op(std::integral_constant<int, N::value + 3>());
        vector(N(), zero(), std::integral_constant<int, 16>());
        vector(N(), one(), std::integral_constant<int, 24>());
        SLOT();
      });
    } else {
      for_slots<48>([&](auto N) __attribute__((always_inline)) {
        product(N);
        read_op(std::integral_constant<int, decltype(N)::value + 3>());
        vector(N, zero(), std::integral_constant<int, 10>());
        vector(N, one(), std::integral_constant<int, 26>());
        SLOT();
      });
    }
  };
  auto step = [&](auto par) __attribute__((always_inline)) {
    constexpr int P = decltype(par)::value;
    const uint16_t* const kt = P ? K1 : K0;
    const uint16_t* const vt = P ? V1 : V0;
    nxt = next();
    if (nxt.t >= 0) copies(nxt, P ? K0 : K1, P ? V0 : V1, Kd[1 - P]);
    if (cur.mine()) products(cur, kt, vt, Kd[P]);
    cur = nxt;
    __builtin_amdgcn_s_waitcnt(0);  // this wave's copies have landed
    __syncthreads();
    return cur.t >= 0;
  };
  while (step(std::integral_constant<int, 0>()) && step(std::integral_constant<int, 1>())) {
  }
  rows_out(c.scale);
}

template <bool CAP, bool BIAS>
__global__ __launch_bounds__(NT) void mod_dq_kernel(BwdArgs a) {
  dq_body<CAP, BIAS, false>(a, Part{});
}
template <bool CAP, bool BIAS>
__device__ __forceinline__ void dq_pieces_body(const BwdArgs& a) {
  each_part<QuerySide>(a.c, a.pieces.n, piece_of(blockIdx.x, a.pieces.n), [&](const Part& part) __attribute__((always_inline)) {
    if (threadIdx.x == 0) note_cut<QuerySide>(a.pieces, a.c, part);
    dq_body<CAP, BIAS, true>(a, part);
    __syncthreads();  // (the staging areas)
  });
}
template <bool CAP, bool BIAS>
__global__ __launch_bounds__(NT) void mod_dq_pieces_kernel(BwdArgs a) {
  dq_pieces_body<CAP, BIAS>(a);
}

// dQ of the tiles that pieces have cut, the sum of their parts: 16 rows a
// workgroup, 8 values of a row a thread.
__global__ __launch_bounds__(256) void mod_dq_join_kernel(BwdArgs a) {
  const int tile = blockIdx.x >> 4, sub = blockIdx.x & 15;
  const int p0 = __builtin_amdgcn_readfirstlane(a.pieces.cut[2 * tile]);
  if (p0 < 0) return;
  const int p1 = __builtin_amdgcn_readfirstlane(a.pieces.cut[2 * tile + 1]);
  const int bh = tile / a.ntile, r = 16 * sub + (threadIdx.x >> 4), i = (tile - bh * a.ntile) * BM + r;
  if (i >= a.c.Lq) return;
  const int b = bh / a.c.H, h = bh - b * a.c.H, ch = 8 * (threadIdx.x & 15);
  float4 x0 = make_float4(0.f, 0.f, 0.f, 0.f), x1 = x0;
#pragma unroll 4
  for (int p = p0; p <= p1; ++p) {
    const float* const src = a.dqp + ((size_t)(2 * p + (p == p0)) * a.pieces.slot_rows + r) * D + ch;
    const float4 u = *reinterpret_cast<const float4*>(src);
    const float4 v = *reinterpret_cast<const float4*>(src + 4);
    x0.x += u.x; x0.y += u.y; x0.z += u.z; x0.w += u.w;
    x1.x += v.x; x1.y += v.y; x1.z += v.z; x1.w += v.w;
  }
  uint4 o;
  o.x = pack_bf16x2(x0.x, x0.y);
  o.y = pack_bf16x2(x0.z, x0.w);
  o.z = pack_bf16x2(x1.x, x1.y);
  o.w = pack_bf16x2(x1.z, x1.w);
  *reinterpret_cast<uint4*>(a.dq + (((size_t)b * a.c.Lq + i) * a.c.H + h) * D + ch) = o;
}

// ------------------------------------------------------------- dK and dV ----

// PIECES: the part of a key tile's stream given.
template <bool CAP, bool BIAS, bool PIECES>
__device__ __forceinline__ void dkdv_body(const BwdArgs& a, const Part& part) {
  __shared__ __attribute__((aligned(1024))) uint16_t Q0[TILE], Q1[TILE], O0[TILE], O1[TILE];
  __shared__ __attribute__((aligned(16))) uint16_t KB[NW * 32 * D];
  __shared__ __attribute__((aligned(16))) float Lt[2][BN], Dt[2][BN];
  __shared__ __attribute__((aligned(16))) int Qd[2][BN];  // ids of the tiles' queries
  const int tid = threadIdx.x, lane = tid & 63, l32 = lane & 31, hi = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const ModCall& c = a.c;
  int b, hk, kt, run;
  if constexpr (PIECES) {
    b = part.b;
    hk = part.h;
    kt = part.t;
    run = 0;
  } else {
    place(a, c.Hkv, a.r.k_order, run, kt, b, hk);
  }
  const int rep = c.H / c.Hkv;
  const int qtok = c.H * D, qbytes = qtok * 2, ktok = c.Hkv * D, kbytes = ktok * 2;
  const Batch bt = batch_of(c, b);
  const int used = key_limit(bt, c.s.causal, bt.start + c.Lq - 1);  // keys that some query may see
  const int key0 = kt * BM, wkey = key0 + wave * 32, krow = wkey + l32;
  int kd = 0;
  Docs wdoc{0, 0, false}, gdoc{0, 0, false};
  const bool docs = !PIECES && a.r.k != nullptr;
  if (docs) {
    if (krow < c.Lk) kd = c.s.k_doc[(size_t)b * c.Lk + krow];
    const int2* const kr = a.r.k + (size_t)b * a.kr;
    const int first = key0 >> 5;
    gdoc = docs_of(kr[first]);
    for (int i = 1; i < BM / 32; ++i)
      if (first + i < a.kr) gdoc = mod::join(gdoc, docs_of(kr[first + i]));
    gdoc = uniform(gdoc);
    wdoc = wkey < c.Lk ? uniform(docs_of(kr[wkey >> 5])) : Docs{0x7fffffff, 0, false};
  }
  const bool klive = krow < used && kd >= 0;
  const bool wlive = wkey < used;  // uniform
  const int wend = min(wkey + 32, used);  // behind the wave's last key

  // query tiles of a head that may see a key of the workgroup lie in [qa, qb); the
  // stream: those of the group's heads in turn, this run's part of it
  const int qb = (c.Lq + BN - 1) / BN;
  const int qa = first_query_tile(c, bt, key0);
  // first row that sees the lane's key, by position (-2^31: all, prefix)
  const int rmin = !c.s.causal || krow < bt.prefix ? INT32_MIN : krow - bt.start;
  const int wrmax = !c.s.causal || wend - 1 < bt.prefix ? INT32_MIN : wend - 1 - bt.start;  // first row that sees all of the wave's
  const int wrmin = !c.s.causal || wkey < bt.prefix ? INT32_MIN : wkey - bt.start;          // ... that sees one of them

  int grp = qa >> 6, g = 0;  // group of 64 tiles, head of the group
  int left = 0;              // tiles to visit in this run
  int fl = 0, id = 0;
  uint64_t visit = 0;
  auto look = [&](int s) __attribute__((always_inline)) {
    const int t = 64 * s + lane;
    bool v = t >= qa && t < qb;
    fl = (wlive && t * BN + BN - 1 >= wrmin ? Tile::kMine : 0) | (t * BN >= wrmax && t * BN + BN <= c.Lq ? Tile::kWhole : 0) | Tile::kOne;
    if (v) {
      const int2 e = *reinterpret_cast<const int2*>(a.empty + (size_t)b * a.qr + 2 * t);
      if (e.x != 0 || (t * BN + 32 < c.Lq && e.y != 0)) fl |= Tile::kZero;
      if (docs) {
        const int4 r = *reinterpret_cast<const int4*>(a.r.q + (size_t)b * a.qr + 2 * t);
        const Docs d = mod::join(docs_of(make_int2(r.x, r.y)), docs_of(make_int2(r.z, r.w)));
        v = meet(d, gdoc);
        fl &= Tile::kZero | (meet(d, wdoc) ? Tile::kMine : 0) | (same(d, wdoc) ? Tile::kWhole : 0) |
              (one_doc(d) ? Tile::kOne : 0);
        id = d.lo;
      }
    }
    visit = __builtin_amdgcn_ballot_w64(v);
  };
  int head = 0;  // of the tile that next() gave last
  auto next = [&]() __attribute__((always_inline)) {
    if (left-- <= 0) return Tile{-1, 0, 0};
    while (visit == 0) {
      if (64 * (grp + 1) < qb) {
        look(++grp);
      } else {
        ++g;
        look(grp = qa >> 6);
      }
    }
    head = g;
    const int i = __builtin_ctzll(visit);
    visit &= visit - 1;
    return Tile{64 * grp + i, __builtin_amdgcn_readlane(fl, i), __builtin_amdgcn_readlane(id, i)};
  };

  // tiles to visit of a head, and into how many runs the stream is cut
  int n = qa < qb ? qb - qa : 0;
  if (docs && n > 0) {
    n = 0;
    for (int s = grp; 64 * s < qb; ++s) {
      look(s);
      n += __builtin_popcountll(visit);
    }
  }
  int cuts = 1;
  if constexpr (PIECES) {
    cuts = part.whole() ? 1 : 2;
  } else {
    cuts = max(1, min(a.runs, (int)(((int64_t)n * rep + a.quantum - 1) / a.quantum)));
    if (run >= cuts) return;
    if (run == 0 && hk == 0 && tid == 0) a.counts[b * a.ntile + kt] = cuts;
  }

  f32x16 dk[4], dv[4];
#pragma unroll
  for (int mb = 0; mb < 4; ++mb) dk[mb] = dv[mb] = f32x16{};
  auto partials_out = [&]() __attribute__((always_inline)) {
    if (krow >= c.Lk) return;
    const size_t rowoff = ((size_t)b * c.Lk + krow) * ktok + (size_t)hk * D, n = (size_t)c.B * c.Lk * ktok;
    float* pk = a.part + (size_t)run * n + rowoff;
    float* pv = a.part + (size_t)(a.runs + run) * n + rowoff;
    if constexpr (PIECES) {  // [slots][2][slot_rows][D]
      pk = a.part + ((size_t)2 * part.slot() * a.pieces.slot_rows + (krow - key0)) * D;
      pv = pk + (size_t)a.pieces.slot_rows * D;
    }
#pragma unroll
    for (int mb = 0; mb < 4; ++mb)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float4 x = make_float4(0.f, 0.f, 0.f, 0.f), y = x;
        if (klive) {
          x = make_float4(dk[mb][4 * i], dk[mb][4 * i + 1], dk[mb][4 * i + 2], dk[mb][4 * i + 3]);
          y = make_float4(dv[mb][4 * i], dv[mb][4 * i + 1], dv[mb][4 * i + 2], dv[mb][4 * i + 3]);
        }
        *reinterpret_cast<float4*>(pk + 32 * mb + 8 * i + 4 * hi) = x;
        *reinterpret_cast<float4*>(pv + 32 * mb + 8 * i + 4 * hi) = y;
      }
  };
  // acc * mul (zero for keys that nothing sees) to the wave's key rows, whole, through an area of its own
  auto rows_out = [&](uint16_t* dst, const f32x16 acc[4], float m, uint16_t* area) __attribute__((always_inline)) {
#pragma unroll
    for (int mb = 0; mb < 4; ++mb)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        uint2 pk = make_uint2(0u, 0u);
        if (klive) {
          pk.x = pack_bf16x2(acc[mb][4 * i + 0] * m, acc[mb][4 * i + 1] * m);
          pk.y = pack_bf16x2(acc[mb][4 * i + 2] * m, acc[mb][4 * i + 3] * m);
        }
        *reinterpret_cast<uint2*>(area + l32 * D + ((4 * mb + i) ^ swz(l32)) * 8 + 4 * hi) = pk;
      }
    wave_lds_fence();
    const __amdgpu_buffer_rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc(
        (void*)(dst + ((size_t)b * c.Lk + wkey) * ktok + (size_t)hk * D), (short)0,
        __builtin_amdgcn_readfirstlane(min(max(c.Lk - wkey, 0), 32) * kbytes), kBufferFlags);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int r = 4 * i + (lane >> 4);
      const u32x4 x = *reinterpret_cast<const u32x4*>(area + r * D + (lane & 15) * 8);
      __builtin_amdgcn_raw_buffer_store_b128(x, rs, r * kbytes + ((lane & 15) ^ swz(r)) * 16, 0, 0);
    }
    wave_lds_fence();
  };

  // own k and v as B operands: lane holds key krow; k goes to LDS
  uint16_t* const kb = KB + wave * 32 * D + lane * 8;
  bf16x8 vop[8];
  {
    const size_t rowoff = ((size_t)b * c.Lk + (klive ? krow : 0)) * ktok + (size_t)hk * D;
#pragma unroll
    for (int s = 0; s < 8; ++s) {
      uint4 x = make_uint4(0, 0, 0, 0), y = x;
      if (klive) {
        x = *reinterpret_cast<const uint4*>(a.k + rowoff + (2 * s + hi) * 8);
        y = *reinterpret_cast<const uint4*>(a.v + rowoff + (2 * s + hi) * 8);
      }
      *reinterpret_cast<bf16x8*>(kb + s * 512) = apply_sign(x, a.sc);  // (the sign of scale; dQ and dK take it outside)
      vop[s] = __builtin_bit_cast(bf16x8, y);
    }
  }
  const size_t qbase = (size_t)b * c.Lq * qtok;
  // (rows past Lq: zeros everywhere, and never seen: a bias that grows with the
  // distance would make weights of them that overflow)
  auto copies = [&](const Tile& t, uint16_t* qs, uint16_t* os, int buf) __attribute__((always_inline)) {
    const size_t hoff = qbase + (size_t)(hk * rep + head) * D;
    const size_t lbase = ((size_t)b * c.H + hk * rep + head) * c.Lq;
    const __amdgpu_buffer_rsrc_t rq = tile_rsrc(a.q + hoff, t.t, c.Lq, qtok), ro = tile_rsrc(a.dout + hoff, t.t, c.Lq, qtok);
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int r = 4 * (2 * wave + u) + (lane >> 4);
      int off = r * qbytes + ((lane & 15) ^ swz(r)) * 16;
      if (t.zero()) {  // uniform: rows that see nothing arrive as zeros
        const int row = t.t * BN + r;
        if (row >= c.Lq || a.lse[lbase + min(row, c.Lq - 1)] == -INFINITY) off = kOff;
      }
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rq, (lds_ptr)(qs + (2 * wave + u) * 512), 16, off, 0, 0, 0);
      __builtin_amdgcn_raw_ptr_buffer_load_lds(ro, (lds_ptr)(os + (2 * wave + u) * 512), 16, off, 0, 0, 0);
    }
    if (wave == 0) copy_row(a.nlse + lbase, t.t, c.Lq, Lt[buf], lane);
    if (wave == 1) copy_row(a.delta + lbase, t.t, c.Lq, Dt[buf], lane);
    if (wave == 2 && docs && !t.one()) copy_row(c.s.q_doc + (size_t)b * c.Lq, t.t, c.Lq, Qd[buf], lane);
  };
  const RowOffsets off = row_offsets(lane);
  const float mul = a.sc.mul;
  // One 32-query block of a tile, one slot a product (as in the dense backward).
  // Without a cap P is formed beside dP; with one the scores' tanh comes first.
  auto block = [&](int blk, auto par, const Tile& t, const uint16_t* qt, const uint16_t* ot, float slope)
                   __attribute__((always_inline)) {
    constexpr int P = decltype(par)::value;
    auto hidden = [&](f32x16& x) __attribute__((always_inline)) {
      each_hidden(rmin == INT32_MIN ? INT32_MIN : rmin - t.t * BN - 4 * hi - 32 * blk,
                  docs && t.one() && kd != t.id ? INT32_MIN : c.Lq - t.t * BN - 4 * hi - 32 * blk,
                  docs && !t.one() ? &Qd[P][32 * blk + 4 * hi] : nullptr, kd,
                  [&](int i) __attribute__((always_inline)) { x[i] = -INFINITY; });
    };
    const int orow = in_loop(off.row, t.t), otr = in_loop(off.tr, t.t);
    const uint16_t* const qb_ = qt + 32 * blk * D;
    const uint16_t* const ob = ot + 32 * blk * D;
    const float dist = BIAS ? (float)(bt.start + t.t * BN + 32 * blk + 4 * hi - krow) : 0.f;
    f32x16 s = f32x16{}, dp;
    bf16x8 qa_[8], ka[8], oa[8], tr_o[8], tr_q[8], db[2];
    uint32_t pw[8];
    float4 nl[4];
    auto exps = [&](int i) __attribute__((always_inline)) {  // P of elements i, i + 1; s becomes P (1 - t^2)
      const float4 l4 = nl[i >> 2];
      float p[2];
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const float z = s[i + e];
        float x = fmaf(z, mul, (i & 2) ? (e ? l4.w : l4.z) : (e ? l4.y : l4.x));
        if (BIAS) x = fmaf(slope, fabsf(dist + (float)acc_row(0, i + e)), x);
        p[e] = __builtin_amdgcn_exp2f(x);
        s[i + e] = CAP ? p[e] * cap_slope(z) : p[e];
      }
      pw[i >> 1] = pack_bf16x2(p[0], p[1]);
    };
    auto read_qk = [&](int st) __attribute__((always_inline)) {
      qa_[st] = read_row(qb_, orow, st);
      ka[st] = *reinterpret_cast<const bf16x8*>(kb + st * 512);
    };
    auto p_op = [&](int k2) __attribute__((always_inline)) {
      return __builtin_bit_cast(bf16x8, make_uint4(pw[4 * k2], pw[4 * k2 + 1], pw[4 * k2 + 2], pw[4 * k2 + 3]));
    };
#pragma unroll
    for (int st = 0; st < 3; ++st) read_qk(st);
    SLOT();
#pragma unroll
    for (int st = 0; st < 8; ++st) {  // S
      if (st == 0 && !CAP && !t.whole()) {  // uniform
        hidden(s);
        s = mfma32(qa_[st], ka[st], s);
      } else {
        s = mfma32(qa_[st], ka[st], st == 0 ? f32x16{} : s);
      }
      if (st + 3 < 8) read_qk(st + 3);
      else oa[st - 5] = read_row(ob, orow, st - 5);
      if (st >= 1 && st < 5) {
        const float4 d4 = *reinterpret_cast<const float4*>(&Dt[P][32 * blk + 8 * (st - 1) + 4 * hi]);
        dp[4 * st - 4] = d4.x; dp[4 * st - 3] = d4.y; dp[4 * st - 2] = d4.z; dp[4 * st - 1] = d4.w;
      }
      SLOT();
    }
    if (CAP) {
      cap16(s, a.sc);
      if (!t.whole()) hidden(s);
    }
#pragma unroll
    for (int st = 0; st < 8; ++st) {  // dP - D; P of elements 0 .. 11
      dp = mfma32(oa[st], vop[st], dp);
      if (st + 3 < 8) oa[st + 3] = read_row(ob, orow, st + 3);
      else tr_o[st - 5] = read_tr(ob, otr, st - 5);
      if (st < 4) nl[st] = *reinterpret_cast<const float4*>(&Lt[P][32 * blk + 8 * st + 4 * hi]);
      if (st >= 2) exps(2 * (st - 2));
      SLOT();
    }
#pragma unroll
    for (int u = 0; u < 8; ++u) {  // dV; the rest of P, then dS
      const int mb = u & 3;
      dv[mb] = mfma32(tr_o[u], p_op(u >> 2), dv[mb]);
      if (u + 3 < 8) tr_o[u + 3] = read_tr(ob + 16 * ((u + 3) >> 2) * D, otr, (u + 3) & 3);
      else tr_q[u - 5] = read_tr(qb_, otr, u - 5);
      if (u < 2) exps(12 + 2 * u);
      if (u >= 3 && u < 7) {
#pragma unroll
        for (int i = 4 * (u - 3); i < 4 * (u - 3) + 4; ++i) dp[i] *= s[i];
      }
      if (u == 5) db[0] = pack8(dp, 0);
      if (u == 7) db[1] = pack8(dp, 1);
      SLOT();
    }
#pragma unroll
    for (int u = 0; u < 8; ++u) {  // dK
      const int mb = u & 3;
      dk[mb] = mfma32(tr_q[u], db[u >> 2], dk[mb]);
      if (u + 3 < 8) tr_q[u + 3] = read_tr(qb_ + 16 * ((u + 3) >> 2) * D, otr, (u + 3) & 3);
      SLOT();
    }
  };
  Tile cur{-1, 0, 0}, nxt = cur;
  int cur_head = 0;
  if (n > 0) {
    const int64_t i0 = PIECES ? part.lo : (int64_t)n * rep * run / cuts;
    const int64_t i1 = PIECES ? part.hi : (int64_t)n * rep * (run + 1) / cuts;
    g = (int)(i0 / n);
    left = (int)(i1 - i0);
    int skip = (int)(i0 - (int64_t)g * n);
    look(grp);
    while (left > 0 && skip >= __builtin_popcountll(visit)) {
      skip -= __builtin_popcountll(visit);
      look(++grp);
    }
    for (; left > 0 && skip > 0; --skip) visit &= visit - 1;
    cur = next();
  }
  if (cur.t >= 0) {
    copies(cur, Q0, O0, 0);
  }
  __builtin_amdgcn_s_waitcnt(0);
  __syncthreads();
  auto step = [&](auto par) __attribute__((always_inline)) {
    constexpr int P = decltype(par)::value;
    const uint16_t* const qt = P ? Q1 : Q0;
    const uint16_t* const ot = P ? O1 : O0;
    cur_head = head;
    nxt = next();
    if (nxt.t >= 0) copies(nxt, P ? Q0 : Q1, P ? O0 : O1, 1 - P);
    if (cur.mine()) {
      const float slope = BIAS ? -c.s.slopes[hk * rep + cur_head] * kLog2e : 0.f;
#pragma unroll
      for (int blk = 0; blk < 2; ++blk) block(blk, par, cur, qt, ot, slope);
    }
    cur = nxt;
    __builtin_amdgcn_s_waitcnt(0);  // this wave's copies have landed
    __syncthreads();
    return cur.t >= 0;
  };
  if (cur.t >= 0)
    while (step(std::integral_constant<int, 0>()) && step(std::integral_constant<int, 1>())) {
    }
  if (cuts > 1) return partials_out();
  uint16_t* const area = KB + wave * 32 * D;  // read by this wave alone
  rows_out(a.dk, dk, c.scale, area);
  rows_out(a.dv, dv, 1.f, area);
}

template <bool CAP, bool BIAS>
__global__ __launch_bounds__(NT) void mod_dkdv_kernel(BwdArgs a) {
  dkdv_body<CAP, BIAS, false>(a, Part{});
}
template <bool CAP, bool BIAS>
__device__ __forceinline__ void dkdv_pieces_body(const BwdArgs& a) {
  each_part<KeySide>(a.c, a.pieces.n, piece_of(blockIdx.x, a.pieces.n), [&](const Part& part) __attribute__((always_inline)) {
    if (threadIdx.x == 0) note_cut<KeySide>(a.pieces, a.c, part);
    dkdv_body<CAP, BIAS, true>(a, part);
    __syncthreads();  // (the tile buffers)
  });
}
template <bool CAP, bool BIAS>
__global__ __launch_bounds__(NT) void mod_dkdv_pieces_kernel(BwdArgs a) {
  dkdv_pieces_body<CAP, BIAS>(a);
}

// dK, dV of the tiles that pieces have cut, the sum of their parts: 16 rows of one
// of them a workgroup, 8 values of a row a thread.
__global__ __launch_bounds__(256) void mod_dkdv_join_kernel(BwdArgs a) {
  const int tile = blockIdx.x >> 5, isv = blockIdx.x >> 4 & 1, sub = blockIdx.x & 15;
  const int p0 = __builtin_amdgcn_readfirstlane(a.pieces.cut[2 * tile]);
  if (p0 < 0) return;
  const int p1 = __builtin_amdgcn_readfirstlane(a.pieces.cut[2 * tile + 1]);
  const int bh = tile / a.ntile, r = 16 * sub + (threadIdx.x >> 4), j = (tile - bh * a.ntile) * BM + r;
  if (j >= a.c.Lk) return;
  const int b = bh / a.c.Hkv, h = bh - b * a.c.Hkv, ch = 8 * (threadIdx.x & 15);
  float4 x0 = make_float4(0.f, 0.f, 0.f, 0.f), x1 = x0;
#pragma unroll 4
  for (int p = p0; p <= p1; ++p) {
    const float* const src = a.part + ((size_t)(2 * (2 * p + (p == p0)) + isv) * a.pieces.slot_rows + r) * D + ch;
    const float4 u = *reinterpret_cast<const float4*>(src);
    const float4 v = *reinterpret_cast<const float4*>(src + 4);
    x0.x += u.x; x0.y += u.y; x0.z += u.z; x0.w += u.w;
    x1.x += v.x; x1.y += v.y; x1.z += v.z; x1.w += v.w;
  }
  const float m = isv ? 1.f : a.c.scale;
  uint4 o;
  o.x = pack_bf16x2(x0.x * m, x0.y * m);
  o.y = pack_bf16x2(x0.z * m, x0.w * m);
  o.z = pack_bf16x2(x1.x * m, x1.y * m);
  o.w = pack_bf16x2(x1.z * m, x1.w * m);
  *reinterpret_cast<uint4*>((isv ? a.dv : a.dk) + (((size_t)b * a.c.Lk + j) * a.c.Hkv + h) * D + ch) = o;
}

// dK = scale * sum of the runs' partials, dV = their sum, for the tiles that were
// cut: 8 values a thread.
__global__ __launch_bounds__(256) void mod_reduce_kernel(BwdArgs a) {
  const int row = a.c.Hkv * D;  // values of a key
  const size_t n = (size_t)a.c.B * a.c.Lk * row, groups = n / 8;
  for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < 2 * groups; i += (size_t)gridDim.x * 256) {
    const bool isk = i < groups;
    const size_t e = (isk ? i : i - groups) * 8, key = e / row;
    const int b = (int)(key / a.c.Lk), cuts = a.counts[b * a.ntile + (int)(key - (size_t)b * a.c.Lk) / BM];
    if (cuts == 1) continue;  // written whole
    const float* src = a.part + (isk ? 0 : (size_t)a.runs * n) + e;
    float4 x0 = make_float4(0.f, 0.f, 0.f, 0.f), x1 = x0;
#pragma unroll 4
    for (int r = 0; r < cuts; ++r) {
      const float4 u = *reinterpret_cast<const float4*>(src + (size_t)r * n);
      const float4 v = *reinterpret_cast<const float4*>(src + (size_t)r * n + 4);
      x0.x += u.x; x0.y += u.y; x0.z += u.z; x0.w += u.w;
      x1.x += v.x; x1.y += v.y; x1.z += v.z; x1.w += v.w;
    }
    const float m = isk ? a.c.scale : 1.f;
    uint4 o;
    o.x = pack_bf16x2(x0.x * m, x0.y * m);
    o.y = pack_bf16x2(x0.z * m, x0.w * m);
    o.z = pack_bf16x2(x1.x * m, x1.y * m);
    o.w = pack_bf16x2(x1.z * m, x1.w * m);
    *reinterpret_cast<uint4*>((isk ? a.dk : a.dv) + e) = o;
  }
}

}  // namespace

hipError_t launch_attn_mod_bwd(const ModBwd& f, hipStream_t stream) {
  const ModCall& c = f.c;
  const int cus = device_cu_count();
  const ModBwdSplit s = mod_bwd_split(c, cus, f.ws_floats);
  BwdArgs a;
  a.c = c;
  a.sc = make_scores(c);
  a.q = f.q; a.k = f.k; a.v = f.v; a.o = f.o; a.dout = f.dout; a.lse = f.lse;
  a.dq = f.dq; a.dk = f.dk; a.dv = f.dv;
  a.delta = f.ws + s.delta;
  a.nlse = f.ws + s.nlse;
  a.empty = reinterpret_cast<int32_t*>(f.ws + s.empty);
  a.counts = reinterpret_cast<int32_t*>(f.ws + s.counts);
  a.part = f.ws + s.part;
  a.quantum = s.quantum;
  a.kr = (int)mod_ranges(c.Lk);
  a.qr = (int)mod_ranges(c.Lq);
  const bool docs = c.s.k_doc != nullptr;
  const bool uneven = c.s.k_doc || c.s.causal || c.s.kv_valid_len;
  const size_t qwg = mod_tiles(c.Lq) * c.B * c.H, kwg = mod_tiles(c.Lk) * c.B * c.Hkv * s.runs;
  hipError_t e = launch_mod_ranges(c, f.ws, qwg > (size_t)cus, kwg > (size_t)cus, &a.r, stream);
  if (e != hipSuccess) return e;
  const bool cap = c.s.cap > 0.f, bias = c.s.slopes != nullptr;
  if (c.Lq > 0) {
    a.ntile = (c.Lq + BM - 1) / BM;
    a.nwg = a.ntile * c.B * c.H;
    a.runs = 1;
    a.in_run[0] = a.r.q_order ? a.ntile * c.B : a.ntile;
    a.sorted = uneven && qwg > (size_t)cus;
    a.first_most = 0;
    unsigned grid = (unsigned)a.nwg;
    if (s.dq.n) {
      a.dqp = f.ws + s.part;
      a.pieces = Pieces{s.dq.n, s.dq.slot_rows, reinterpret_cast<int32_t*>(f.ws + s.dq.cut)};
      grid = (unsigned)s.dq.n;
      e = cap ? (bias ? launch_kernel(mod_dq_pieces_kernel<true, true>, grid, (unsigned)NT, stream, a)
                      : launch_kernel(mod_dq_pieces_kernel<true, false>, grid, (unsigned)NT, stream, a))
              : (bias ? launch_kernel(mod_dq_pieces_kernel<false, true>, grid, (unsigned)NT, stream, a)
                      : launch_kernel(mod_dq_pieces_kernel<false, false>, grid, (unsigned)NT, stream, a));
      if (e == hipSuccess) e = launch_kernel(mod_dq_join_kernel, (unsigned)a.nwg * 16u, 256u, stream, a);
    } else {
      e = cap ? (bias ? launch_kernel(mod_dq_kernel<true, true>, grid, (unsigned)NT, stream, a)
                      : launch_kernel(mod_dq_kernel<true, false>, grid, (unsigned)NT, stream, a))
              : (bias ? launch_kernel(mod_dq_kernel<false, true>, grid, (unsigned)NT, stream, a)
                      : launch_kernel(mod_dq_kernel<false, false>, grid, (unsigned)NT, stream, a));
    }
    if (e != hipSuccess) return e;
  }
  if (c.Lk > 0 && s.dkdv.n) {
    a.ntile = (c.Lk + BM - 1) / BM;
    a.pieces = Pieces{s.dkdv.n, s.dkdv.slot_rows, reinterpret_cast<int32_t*>(f.ws + s.dkdv.cut)};
    const unsigned grid = (unsigned)s.dkdv.n;
    e = cap ? (bias ? launch_kernel(mod_dkdv_pieces_kernel<true, true>, grid, (unsigned)NT, stream, a)
                    : launch_kernel(mod_dkdv_pieces_kernel<true, false>, grid, (unsigned)NT, stream, a))
            : (bias ? launch_kernel(mod_dkdv_pieces_kernel<false, true>, grid, (unsigned)NT, stream, a)
                    : launch_kernel(mod_dkdv_pieces_kernel<false, false>, grid, (unsigned)NT, stream, a));
    if (e == hipSuccess) e = launch_kernel(mod_dkdv_join_kernel, (unsigned)(a.ntile * c.B * c.Hkv * 32), 256u, stream, a);
  } else if (c.Lk > 0) {
    a.ntile = (c.Lk + BM - 1) / BM;
    a.runs = s.runs;
    // Workgroups that would find no part of their tile's stream are not launched
    // where the host knows: with them between the others, some shader engines got
    // more workgroups than compute units (2 x 2049 causal, 16 heads on 4: 256
    // workgroups that stream at most 22 tiles 148 us; 91 without).
    const bool known = !docs && !c.s.kv_valid_len && !c.s.prefix_len && !c.s.q_start;
    int tiles = 0;
    for (int r = 0; r < s.runs; ++r) {
      int n = a.ntile;
      if (known)
        while (n > 0 && r > 0 && mod_stream(n - 1, c.H / c.Hkv, c.Lq, c.Lk, c.s.causal) <= (int64_t)r * s.quantum) --n;
      a.in_run[r] = a.r.k_order ? n * c.B : n;
      tiles += n;
    }
    a.nwg = tiles * c.B * c.Hkv;
    a.sorted = uneven && (kwg > (size_t)cus || s.runs > 1);
    a.first_most = 1;
    const unsigned grid = (unsigned)a.nwg;
    e = cap ? (bias ? launch_kernel(mod_dkdv_kernel<true, true>, grid, (unsigned)NT, stream, a)
                    : launch_kernel(mod_dkdv_kernel<true, false>, grid, (unsigned)NT, stream, a))
            : (bias ? launch_kernel(mod_dkdv_kernel<false, true>, grid, (unsigned)NT, stream, a)
                    : launch_kernel(mod_dkdv_kernel<false, false>, grid, (unsigned)NT, stream, a));
    if (e != hipSuccess) return e;
    if (s.runs > 1) {
      size_t g = ((size_t)2 * c.B * c.Lk * c.Hkv * D / 8 + 255) / 256;
      if (g > 16384) g = 16384;
      e = launch_kernel(mod_reduce_kernel, (unsigned)g, 256u, stream, a);
    }
  }
  return e;
}

}  // namespace vidax
