// The step between two sublayers of a block, forward and backward (HBM-bound):
//
//   u  = post(y) * post_gain          post: none, layer norm or RMS norm
//   x' = alpha x + gate u             the residual stream, rounded once
//   h  = norm(x') * gain * (1 + scale) + shift
//
// A row (token) lies in the registers of `waves` waves, 8 consecutive channels
// (a chunk) of it in a lane, up to three chunks a lane; whatever is summed over
// the row is summed in the wave by lane moves and between the waves of a row
// through LDS, one barrier a sum.  Means and variances are exact in two passes
// over the registers (the waves' means and squared deviations are combined by
// their own means, not by differences of squares).  Everything is fp32; h is
// normalised from the sum before that is rounded to the stream's type.
//   A workgroup walks consecutive rows of one batch with the modulations of the
// batch in registers, the next row's loads in flight: a row costs x and y in
// and x' and h out.
#include "common.hpp"
#include "launch_block.hpp"

namespace vidax {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// Waves of a workgroup: 8, so that a lane may hold 256 registers; up to 10 in the
// backward with one chunk a lane, which needs few (128 to 157; three waves a SIMD, so up
// to twelve waves, leave 168).
constexpr int kMaxWaves = 10;
constexpr int kWaves = kBlockWaves;

// Eight values of the stream (bf16: 16 bytes, fp32: 32) as they lie in memory.
template <bool F32>
struct Raw {
  u32x4 w[F32 ? 2 : 1];
};

template <bool F32>
__device__ __forceinline__ Raw<F32> load_raw(const void* base, size_t e) {
  Raw<F32> r;
  const u32x4* p = reinterpret_cast<const u32x4*>(static_cast<const char*>(base) + e * (F32 ? 4 : 2));
#pragma unroll
  for (int i = 0; i < (F32 ? 2 : 1); ++i) r.w[i] = p[i];
  return r;
}

template <bool F32>
__device__ __forceinline__ Raw<F32> zero_raw() {
  Raw<F32> r;
#pragma unroll
  for (int i = 0; i < (F32 ? 2 : 1); ++i) r.w[i] = u32x4{0u, 0u, 0u, 0u};
  return r;
}

template <bool F32>
__device__ __forceinline__ void unpack(const Raw<F32>& r, float v[8]) {
  if constexpr (F32) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(r.w[i >> 2][i & 3]);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[2 * i] = bf16lo_to_f32(r.w[0][i]);
      v[2 * i + 1] = bf16hi_to_f32(r.w[0][i]);
    }
  }
}

template <bool F32>
__device__ __forceinline__ void store8(void* base, size_t e, const float v[8]) {
  u32x4* p = reinterpret_cast<u32x4*>(static_cast<char*>(base) + e * (F32 ? 4 : 2));
  if constexpr (F32) {
#pragma unroll
    for (int i = 0; i < 2; ++i)
      p[i] = u32x4{__float_as_uint(v[4 * i]), __float_as_uint(v[4 * i + 1]), __float_as_uint(v[4 * i + 2]),
                   __float_as_uint(v[4 * i + 3])};
  } else {
    p[0] = u32x4{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7])};
  }
}

__device__ __forceinline__ void load_f32x8(const float* p, float v[8]) {
  const float4 a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
  v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
  v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
}

// v summed over the wave; every lane receives the sum.
__device__ __forceinline__ float wave_sum(float v) {
  // row_ror:8, row_ror:4, quad_perm [2,3,0,1], quad_perm [1,0,3,2]: 16 lanes
  v += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x128, 0xf, 0xf, false));
  v += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x124, 0xf, 0xf, false));
  v += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x4e, 0xf, 0xf, false));
  v += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0xb1, 0xf, 0xf, false));
  auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = __uint_as_float(r[0]) + __uint_as_float(r[1]);
  auto q = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(q[0]) + __uint_as_float(q[1]);
}

// The waves of a row and their exchange through LDS.  Two slots in turn: a wave
// writes a slot again two sums later, behind a barrier that every wave reaches
// after it has read the slot.
struct Row {
  float (*slots)[kMaxWaves][4];  // [2][waves of the workgroup][values]
  int waves, first, wave;        // of the row; its first in the workgroup; this one of the row
  int slot;
  float inv_c;
  float n, inv_n;                // elements of the row that this wave holds
  int nch, threads;              // chunks of a row, lanes of a row

  __device__ __forceinline__ int elements(int w, int nc) const {
    int s = 0;
    for (int i = 0; i < nc; ++i) s += min(max(nch - i * threads - 64 * w, 0), 64);
    return 8 * s;
  }

  // N sums over the row
  template <int N>
  __device__ __forceinline__ void sum(float v[N], int lane) {
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] = wave_sum(v[k]);
    if (waves == 1) return;
    float(*s)[4] = slots[slot];
    slot ^= 1;
    if (lane == 0)
#pragma unroll
      for (int k = 0; k < N; ++k) s[first + wave][k] = v[k];
    __syncthreads();
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] = 0.f;
    for (int w = 0; w < waves; ++w)
#pragma unroll
      for (int k = 0; k < N; ++k) v[k] += s[first + w][k];
  }

  // mean (0 for kind 2, RMS) and sum of squared deviations of up to two rows of
  // values at once (the second one where kind_b != 0)
  template <int NC>
  __device__ __forceinline__ void stats(const float a[NC][8], int kind_a, float& mean_a, float& m2_a, const float b[NC][8],
                                        int kind_b, float& mean_b, float& m2_b, const bool live[NC], int lane) {
    float v[4] = {0.f, 0.f, 0.f, 0.f};  // wave's sum and squared deviations from the wave's mean
    auto one = [&](const float x[NC][8], int kind, float& s, float& m2) __attribute__((always_inline)) {
      float mean = 0.f;
      if (kind == 1) {
        float t = 0.f;
#pragma unroll
        for (int i = 0; i < NC; ++i)
#pragma unroll
          for (int e = 0; e < 8; ++e) t += x[i][e];  // zero where the chunk is not live
        s = wave_sum(t);
        mean = s * inv_n;
      }
      float t = 0.f;
#pragma unroll
      for (int i = 0; i < NC; ++i)
        if (live[i])
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const float d = x[i][e] - mean;
            t = fmaf(d, d, t);
          }
      m2 = wave_sum(t);
    };
    one(a, kind_a, v[0], v[1]);
    if (kind_b) one(b, kind_b, v[2], v[3]);
    if (waves == 1) {
      mean_a = v[0] * inv_c; m2_a = v[1];
      mean_b = v[2] * inv_c; m2_b = v[3];
      return;
    }
    float(*s)[4] = slots[slot];
    slot ^= 1;
    if (lane == 0) *reinterpret_cast<float4*>(s[first + wave]) = make_float4(v[0], v[1], v[2], v[3]);
    __syncthreads();
    float sa = 0.f, sb = 0.f, qa = 0.f, qb = 0.f;
    for (int w = 0; w < waves; ++w) {
      const float4 x = *reinterpret_cast<const float4*>(s[first + w]);
      sa += x.x; qa += x.y; sb += x.z; qb += x.w;
    }
    mean_a = sa * inv_c;
    mean_b = sb * inv_c;
    if (kind_a == 1 || kind_b == 1)
      for (int w = 0; w < waves; ++w) {
        const float4 x = *reinterpret_cast<const float4*>(s[first + w]);
        const float nw = (float)elements(w, NC), in = 1.0f / nw;
        const float da = x.x * in - mean_a, db = x.z * in - mean_b;
        if (kind_a == 1) qa = fmaf(nw * da, da, qa);
        if (kind_b == 1) qb = fmaf(nw * db, db, qb);
      }
    m2_a = qa;
    m2_b = qb;
  }
};

struct Shape {
  int waves, groups, rows, runs;
};

// ---------------------------------------------------------------- forward ----

struct FwdArgs {
  BlockNormFwd a;
  Shape s;
};

// TOKEN: the modulations change from row to row
template <bool F32, int NC, bool TOKEN>
__global__ __launch_bounds__(64 * kWaves) void block_norm_fwd_kernel(FwdArgs f) {
  __shared__ __attribute__((aligned(16))) float slots[2][kMaxWaves][4];
  const BlockNorm& n = f.a.n;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int group = wave / f.s.waves;
  Row row;
  row.slots = slots;
  row.waves = f.s.waves;
  row.first = group * f.s.waves;
  row.wave = wave - row.first;
  row.slot = 0;
  row.nch = n.C >> 3;
  row.threads = 64 * f.s.waves;
  row.inv_c = 1.0f / (float)n.C;
  row.n = (float)row.elements(row.wave, NC);
  row.inv_n = 1.0f / row.n;
  const int b = blockIdx.x / f.s.runs, run = blockIdx.x - b * f.s.runs;
  const int r0 = run * f.s.rows, r1 = min(r0 + f.s.rows, n.L);
  const int t = 64 * row.wave + lane;
  bool live[NC];
  int ch[NC];  // first channel of the lane's chunks
#pragma unroll
  for (int i = 0; i < NC; ++i) {
    live[i] = t + i * row.threads < row.nch;
    ch[i] = live[i] ? 8 * (t + i * row.threads) : 0;
  }
  // gate * post_gain, gain * (1 + scale), shift
  float g[NC][8], m[NC][8], sh[NC][8];
  auto mods = [&](int tok) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < NC; ++i) {
#pragma unroll
      for (int e = 0; e < 8; ++e) { g[i][e] = 1.f; m[i][e] = 1.f; sh[i][e] = 0.f; }
      if (n.gate.p) load_f32x8(n.gate.p + b * n.gate.batch + tok * n.gate.token + ch[i], g[i]);
      if (n.scale.p) {
        load_f32x8(n.scale.p + b * n.scale.batch + tok * n.scale.token + ch[i], m[i]);
#pragma unroll
        for (int e = 0; e < 8; ++e) m[i][e] += 1.f;
      }
      if (n.shift.p) load_f32x8(n.shift.p + b * n.shift.batch + tok * n.shift.token + ch[i], sh[i]);
      float w[8];
      if (n.post_gain) {
        load_f32x8(n.post_gain + ch[i], w);
#pragma unroll
        for (int e = 0; e < 8; ++e) g[i][e] *= w[e];
      }
      if (n.gain) {
        load_f32x8(n.gain + ch[i], w);
#pragma unroll
        for (int e = 0; e < 8; ++e) m[i][e] *= w[e];
      }
    }
  };
  Raw<F32> xr[NC];
  Raw<false> yr[NC];
  const size_t base = (size_t)b * n.L * n.C;
  auto load = [&](int r) __attribute__((always_inline)) {
    const size_t off = base + (size_t)r * n.C;
#pragma unroll
    for (int i = 0; i < NC; ++i) {
      xr[i] = live[i] ? load_raw<F32>(f.a.x, off + ch[i]) : zero_raw<F32>();
      yr[i] = live[i] && f.a.y ? load_raw<false>(f.a.y, off + ch[i]) : zero_raw<false>();
    }
  };
  // every group of the workgroup makes the same number of passes (barriers)
  int r = r0 + group;
  load(min(r, r1 - 1));
  if (!TOKEN) mods(0);
  for (int first = r0; first < r1; first += f.s.groups, r += f.s.groups) {
    const bool on = r < r1;  // uniform over the row's waves
    float x[NC][8], y[NC][8];
#pragma unroll
    for (int i = 0; i < NC; ++i) {
      unpack<F32>(xr[i], x[i]);
      unpack<false>(yr[i], y[i]);
    }
    const int tok = min(r, r1 - 1);
    if (TOKEN) mods(tok);
    if (first + f.s.groups < r1) load(min(r + f.s.groups, r1 - 1));
    float mean, m2, mean_b, m2_b;
    if (n.post) {
      row.template stats<NC>(y, n.post, mean, m2, y, 0, mean_b, m2_b, live, lane);
      const float rs = 1.0f / sqrtf(fmaf(m2, row.inv_c, n.eps));
#pragma unroll
      for (int i = 0; i < NC; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e) y[i][e] = (y[i][e] - mean) * rs;
    }
#pragma unroll
    for (int i = 0; i < NC; ++i)
#pragma unroll
      for (int e = 0; e < 8; ++e)
        x[i][e] = !live[i] ? 0.f : f.a.y ? fmaf(g[i][e], y[i][e], n.alpha * x[i][e]) : n.alpha * x[i][e];
    const size_t off = base + (size_t)tok * n.C;
    if (f.a.xo && on)
#pragma unroll
      for (int i = 0; i < NC; ++i)
        if (live[i]) store8<F32>(f.a.xo, off + ch[i], x[i]);
    row.template stats<NC>(x, n.norm, mean, m2, x, 0, mean_b, m2_b, live, lane);
    const float rs = 1.0f / sqrtf(fmaf(m2, row.inv_c, n.eps));
    if (on)
#pragma unroll
      for (int i = 0; i < NC; ++i)
        if (live[i]) {
          float h[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) h[e] = fmaf((x[i][e] - mean) * rs, m[i][e], sh[i][e]);
          store8<false>(f.a.h, off + ch[i], h);
        }
  }
}

// --------------------------------------------------------------- backward ----
//
// With xh = (x' - mean) rx, yh the normalised branch (y itself without a norm
// on it), w = dh gain (1 + scale):
//
//   g  = dx' + rx (w - xh mean(w xh) [- mean(w)])      gradient of x' in all
//   dx = alpha g,   du = gate g,   dy = ry (a - yh mean(a yh) [- mean(a)]), a = du post_gain
//   dshift = sum dh,  dscale = sum dh xh gain,  dgate = sum g yh post_gain    over a sample's tokens
//   dgain = sum dh xh (1 + scale),  dpost_gain = sum du yh                    over all tokens
//
// ([] with a layer norm only.)  The row is read once: means and deviations are
// formed again from x' and y, which have to be read anyway.  A workgroup keeps
// the column sums of its rows in registers (sum dh, sum dh xh, sum g yh: the
// per-channel factors come in at the end) and writes them once; a second launch
// adds the runs up, always in the same order.

struct BwdArgs {
  BlockNormBwd a;
  Shape s;
};

// TOKEN: every token has modulations (and gradients of them) of its own
template <bool F32, int NC, bool TOKEN>
__global__ __launch_bounds__(64 * (NC == 1 ? kMaxWaves : kWaves)) void block_norm_bwd_kernel(BwdArgs f) {
  __shared__ __attribute__((aligned(16))) float slots[2][kMaxWaves][4];
  __shared__ __attribute__((aligned(16))) float cols[8 * 64 * 8];  // column sums between the groups
  const BlockNorm& n = f.a.n;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int group = wave / f.s.waves;
  Row row;
  row.slots = slots;
  row.waves = f.s.waves;
  row.first = group * f.s.waves;
  row.wave = wave - row.first;
  row.slot = 0;
  row.nch = n.C >> 3;
  row.threads = 64 * f.s.waves;
  row.inv_c = 1.0f / (float)n.C;
  row.n = (float)row.elements(row.wave, NC);
  row.inv_n = 1.0f / row.n;
  const int b = blockIdx.x / f.s.runs, run = blockIdx.x - b * f.s.runs;
  const int r0 = run * f.s.rows, r1 = min(r0 + f.s.rows, n.L);
  const int t = 64 * row.wave + lane;
  bool live[NC];
  int ch[NC];
#pragma unroll
  for (int i = 0; i < NC; ++i) {
    live[i] = t + i * row.threads < row.nch;
    ch[i] = live[i] ? 8 * (t + i * row.threads) : 0;
  }
  // gain * (1 + scale) and gate * post_gain; tokens with modulations of their
  // own need the factors one by one (their gradients leave row by row)
  float w[NC][8], gp[NC][8], gn[TOKEN ? NC : 1][8], m[TOKEN ? NC : 1][8], gt[TOKEN ? NC : 1][8], pg[TOKEN ? NC : 1][8];
  auto mods = [&](int tok) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < NC; ++i) {
      float u[8], v[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) { u[e] = 1.f; v[e] = 1.f; }
      if (n.scale.p) {
        load_f32x8(n.scale.p + b * n.scale.batch + tok * n.scale.token + ch[i], u);
#pragma unroll
        for (int e = 0; e < 8; ++e) u[e] += 1.f;
      }
      if (n.gain) load_f32x8(n.gain + ch[i], v);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        w[i][e] = u[e] * v[e];
        if constexpr (TOKEN) { m[i][e] = u[e]; gn[i][e] = v[e]; }
        u[e] = v[e] = 1.f;
      }
      if (n.gate.p) load_f32x8(n.gate.p + b * n.gate.batch + tok * n.gate.token + ch[i], u);
      if (n.post_gain) load_f32x8(n.post_gain + ch[i], v);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        gp[i][e] = u[e] * v[e];
        if constexpr (TOKEN) { gt[i][e] = u[e]; pg[i][e] = v[e]; }
      }
    }
  };
  float s0[NC][8], s1[NC][8], s2[NC][8];
#pragma unroll
  for (int i = 0; i < NC; ++i)
#pragma unroll
    for (int e = 0; e < 8; ++e) s0[i][e] = s1[i][e] = s2[i][e] = 0.f;
  Raw<F32> xr[NC], gr[NC];
  Raw<false> yr[NC], hr[NC];
  const size_t base = (size_t)b * n.L * n.C;
  auto load = [&](int r) __attribute__((always_inline)) {
    const size_t off = base + (size_t)r * n.C;
#pragma unroll
    for (int i = 0; i < NC; ++i) {
      xr[i] = live[i] ? load_raw<F32>(f.a.xo, off + ch[i]) : zero_raw<F32>();
      hr[i] = live[i] ? load_raw<false>(f.a.dh, off + ch[i]) : zero_raw<false>();
      gr[i] = live[i] && f.a.dxo ? load_raw<F32>(f.a.dxo, off + ch[i]) : zero_raw<F32>();
      yr[i] = live[i] && f.a.y ? load_raw<false>(f.a.y, off + ch[i]) : zero_raw<false>();
    }
  };
  int r = r0 + group;
  load(min(r, r1 - 1));
  if (!TOKEN) mods(0);
  for (int first = r0; first < r1; first += f.s.groups, r += f.s.groups) {
    const bool on = r < r1;
    const int tok = min(r, r1 - 1);
    float x[NC][8], y[NC][8], dh[NC][8], g[NC][8];
#pragma unroll
    for (int i = 0; i < NC; ++i) {
      unpack<F32>(xr[i], x[i]);
      unpack<false>(yr[i], y[i]);
      unpack<false>(hr[i], dh[i]);
      unpack<F32>(gr[i], g[i]);
    }
    if (TOKEN) mods(tok);
    if (first + f.s.groups < r1) load(min(r + f.s.groups, r1 - 1));
    float mx, qx, my, qy;
    row.template stats<NC>(x, n.norm, mx, qx, y, n.post, my, qy, live, lane);
    const float rx = 1.0f / sqrtf(fmaf(qx, row.inv_c, n.eps));
    const float ry = n.post ? 1.0f / sqrtf(fmaf(qy, row.inv_c, n.eps)) : 1.f;
    float d[2] = {0.f, 0.f};
#pragma unroll
    for (int i = 0; i < NC; ++i)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        x[i][e] = live[i] ? (x[i][e] - mx) * rx : 0.f;
        if (n.post) y[i][e] = live[i] ? (y[i][e] - my) * ry : 0.f;
        const float z = dh[i][e] * w[i][e];
        d[0] = fmaf(z, x[i][e], d[0]);
        d[1] += z;
      }
    row.template sum<2>(d, lane);
    const float c0 = d[0] * row.inv_c, c1 = n.norm == 1 ? d[1] * row.inv_c : 0.f;
    float p[2] = {0.f, 0.f};
#pragma unroll
    for (int i = 0; i < NC; ++i)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float z = dh[i][e] * w[i][e];
        g[i][e] = live[i] ? fmaf(rx, fmaf(-x[i][e], c0, z) - c1, g[i][e]) : 0.f;
        const float a = g[i][e] * gp[i][e];
        p[0] = fmaf(a, y[i][e], p[0]);
        p[1] += a;
      }
    float e0 = 0.f, e1 = 0.f;
    if (n.post) {
      row.template sum<2>(p, lane);
      e0 = p[0] * row.inv_c;
      e1 = n.post == 1 ? p[1] * row.inv_c : 0.f;
    }
    const size_t off = base + (size_t)tok * n.C;
    if (on) {
#pragma unroll
      for (int i = 0; i < NC; ++i) {
        if (!live[i]) continue;
        float o[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) o[e] = n.alpha * g[i][e];
        store8<F32>(f.a.dx, off + ch[i], o);
        if (f.a.dy) {
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const float a = g[i][e] * gp[i][e];
            o[e] = n.post ? ry * (fmaf(-y[i][e], e0, a) - e1) : a;
          }
          store8<false>(f.a.dy, off + ch[i], o);
        }
        if constexpr (TOKEN) {
          if (f.a.dshift) store8<true>(f.a.dshift, off + ch[i], dh[i]);
          if (f.a.dscale) {
#pragma unroll
            for (int e = 0; e < 8; ++e) o[e] = dh[i][e] * x[i][e] * gn[i][e];
            store8<true>(f.a.dscale, off + ch[i], o);
          }
          if (f.a.dgate) {
#pragma unroll
            for (int e = 0; e < 8; ++e) o[e] = g[i][e] * y[i][e] * pg[i][e];
            store8<true>(f.a.dgate, off + ch[i], o);
          }
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          // tokens with modulations of their own: only the gains' sums, factors included
          if constexpr (TOKEN) {
            s1[i][e] = fmaf(dh[i][e] * x[i][e], m[i][e], s1[i][e]);
            s2[i][e] = fmaf(g[i][e] * y[i][e], gt[i][e], s2[i][e]);
          } else {
            s0[i][e] += dh[i][e];
            s1[i][e] = fmaf(dh[i][e], x[i][e], s1[i][e]);
            s2[i][e] = fmaf(g[i][e], y[i][e], s2[i][e]);
          }
        }
      }
    }
  }
  if (!f.a.ws) return;  // uniform: nothing to sum over the rows
  // the groups' sums, added in the order of the groups
  const size_t at = (size_t)blockIdx.x * 3 * n.C;
  auto out = [&](float s[NC][8], int k) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < NC; ++i) {
      if (f.s.groups > 1) {
        __syncthreads();
        float4* const p = reinterpret_cast<float4*>(cols + (size_t)threadIdx.x * 8);
        p[0] = make_float4(s[i][0], s[i][1], s[i][2], s[i][3]);
        p[1] = make_float4(s[i][4], s[i][5], s[i][6], s[i][7]);
        __syncthreads();
        if (group == 0)
          for (int q = 1; q < f.s.groups; ++q) {
            float w[8];
            load_f32x8(cols + (size_t)(q * row.threads + t) * 8, w);
#pragma unroll
            for (int e = 0; e < 8; ++e) s[i][e] += w[e];
          }
      }
      if (group == 0 && live[i]) store8<true>(f.a.ws, at + (size_t)k * n.C + ch[i], s[i]);
    }
  };
  out(s0, 0);
  out(s1, 1);
  out(s2, 2);
}

// The runs' column sums added up: a workgroup takes 32 channels, 32 lanes a
// channel take every 32nd run of a batch, the lanes are added in a fixed order,
// the batches in theirs.
__global__ __launch_bounds__(1024) void block_norm_sum_kernel(BwdArgs f) {
  __shared__ float part[3][32][33];
  const BlockNorm& n = f.a.n;
  const int c = threadIdx.x & 31, k = threadIdx.x >> 5, col = blockIdx.x * 32 + c;
  const bool live = col < n.C;
  const float gn = live && n.gain ? n.gain[col] : 1.f, pg = live && n.post_gain ? n.post_gain[col] : 1.f;
  float dgain = 0.f, dpost = 0.f;
  for (int b = 0; b < n.B; ++b) {
    float v[3] = {0.f, 0.f, 0.f};
    const float* p = f.a.ws + (size_t)b * f.s.runs * 3 * n.C + col;
    if (live)
#pragma unroll 4
      for (int r = k; r < f.s.runs; r += 32)
#pragma unroll
        for (int j = 0; j < 3; ++j) v[j] += p[((size_t)r * 3 + j) * n.C];
    __syncthreads();  // the last batch's sums are read
#pragma unroll
    for (int j = 0; j < 3; ++j) part[j][k][c] = v[j];
    __syncthreads();
    if (k == 0 && live) {
      float s[3];
#pragma unroll
      for (int j = 0; j < 3; ++j) {
        s[j] = 0.f;
        for (int q = 0; q < 32; ++q) s[j] += part[j][q][c];
      }
      if (f.a.per_token) {
        dgain += s[1];
        dpost += s[2];
      } else {
        const float mul = n.scale.p ? 1.f + n.scale.p[b * n.scale.batch + col] : 1.f;
        const float gate = n.gate.p ? n.gate.p[b * n.gate.batch + col] : 1.f;
        const size_t o = (size_t)b * n.C + col;
        if (f.a.dshift) f.a.dshift[o] = s[0];
        if (f.a.dscale) f.a.dscale[o] = s[1] * gn;
        if (f.a.dgate) f.a.dgate[o] = s[2] * pg;
        dgain = fmaf(s[1], mul, dgain);
        dpost = fmaf(s[2], gate, dpost);
      }
    }
  }
  if (k == 0 && live) {
    if (f.a.dgain) f.a.dgain[col] = dgain;
    if (f.a.dpost_gain) f.a.dpost_gain[col] = dpost;
  }
}

template <typename A>
hipError_t launch(void (*kernel)(A), unsigned grid, unsigned block, hipStream_t stream, A arg) {
  void* args[] = {&arg};
  return hipLaunchKernel(reinterpret_cast<const void*>(kernel), dim3(grid), dim3(block), args, 0, stream);
}

template <bool F32, bool TOKEN>
hipError_t launch_fwd(int nc, unsigned grid, unsigned block, hipStream_t stream, const FwdArgs& f) {
  switch (nc) {
    case 1: return launch(block_norm_fwd_kernel<F32, 1, TOKEN>, grid, block, stream, f);
    case 2: return launch(block_norm_fwd_kernel<F32, 2, TOKEN>, grid, block, stream, f);
    case 3: return launch(block_norm_fwd_kernel<F32, 3, TOKEN>, grid, block, stream, f);
  }
  return launch(block_norm_fwd_kernel<F32, 4, TOKEN>, grid, block, stream, f);
}

template <bool F32, bool TOKEN>
hipError_t launch_bwd(int nc, unsigned grid, unsigned block, hipStream_t stream, const BwdArgs& f) {
  switch (nc) {
    case 1: return launch(block_norm_bwd_kernel<F32, 1, TOKEN>, grid, block, stream, f);
    case 2: return launch(block_norm_bwd_kernel<F32, 2, TOKEN>, grid, block, stream, f);
  }
  return launch(block_norm_bwd_kernel<F32, 4, TOKEN>, grid, block, stream, f);
}

}  // namespace

hipError_t launch_block_norm_fwd(const BlockNormFwd& a, hipStream_t stream) {
  const BlockNorm& n = a.n;
  FwdArgs f;
  f.a = a;
  const BlockShape s = block_fwd_shape(n.B, n.L, n.C);
  f.s = Shape{s.waves, s.groups, s.rows, s.runs};
  const unsigned grid = (unsigned)s.runs * (unsigned)n.B, block = 64u * s.waves * s.groups;
  const bool token = (n.gate.p && n.gate.token) || (n.scale.p && n.scale.token) || (n.shift.p && n.shift.token);
  if (n.fp32) return token ? launch_fwd<true, true>(s.chunks, grid, block, stream, f) : launch_fwd<true, false>(s.chunks, grid, block, stream, f);
  return token ? launch_fwd<false, true>(s.chunks, grid, block, stream, f) : launch_fwd<false, false>(s.chunks, grid, block, stream, f);
}

hipError_t launch_block_norm_bwd(const BlockNormBwd& a, hipStream_t stream) {
  BwdArgs f;
  f.a = a;
  const BlockShape s = block_bwd_shape(a.n.B, a.n.L, a.n.C);
  f.s = Shape{s.waves, s.groups, s.rows, s.runs};
  const bool sums = (!a.per_token && (a.dshift || a.dscale || a.dgate)) || a.dgain || a.dpost_gain;
  if (!sums) f.a.ws = nullptr;
  const unsigned grid = (unsigned)s.runs * (unsigned)a.n.B, block = 64u * s.waves * s.groups;
  hipError_t e = hipSuccess;
  if (grid == 0) f.s.runs = 0;  // no tokens: the sums alone, all zero
  else e =
      a.n.fp32 ? (a.per_token ? launch_bwd<true, true>(s.chunks, grid, block, stream, f)
                              : launch_bwd<true, false>(s.chunks, grid, block, stream, f))
               : (a.per_token ? launch_bwd<false, true>(s.chunks, grid, block, stream, f)
                              : launch_bwd<false, false>(s.chunks, grid, block, stream, f));
  if (e != hipSuccess || !sums) return e;
  return launch(block_norm_sum_kernel, (unsigned)((a.n.C + 31) / 32), 1024u, stream, f);
}

}  // namespace vidax
