// Arguments and launchers of the block norm (block_norm.hip; not part of the C
// ABI).  Weak: a library linked from the ABI layer alone still loads, and its
// calls of these report a failed launch.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace vidax {

// fp32 modulation rows: token n of batch b at p + b * batch + n * token (elements)
struct BlockMod {
  const float* p;
  int64_t batch, token;
};

constexpr int kBlockMaxC = 16384;

struct BlockNorm {
  int B, L, C;
  int fp32;       // the stream is fp32 (else bf16)
  int norm, post; // 0 none, 1 layer, 2 rms (norm is never 0)
  float eps, alpha;
  const float *gain, *post_gain;
  BlockMod gate, scale, shift;
};

struct BlockNormFwd {
  BlockNorm n;
  const void* x;
  const uint16_t* y;
  void* xo;
  uint16_t* h;
};

struct BlockNormBwd {
  BlockNorm n;
  const uint16_t* dh;
  const void* dxo;  // gradient of the stream behind the step, or null
  const void* xo;
  const uint16_t* y;
  void* dx;
  uint16_t* dy;
  float *dgate, *dscale, *dshift, *dgain, *dpost_gain;
  int per_token;  // the modulations' gradients: [B, L, C] (else [B, C])
  float* ws;      // column sums of every run of rows
};

struct BlockShape {
  int chunks, waves, groups, rows, runs;
};
// A launch takes fewer than 2^32 threads.
inline bool block_launch_fits(const BlockShape& s, int B) {
  return (__int128)s.runs * B * 64 * s.waves * s.groups < ((int64_t)1 << 32);
}

// Shape of the forward: as below.  Waves a row and chunks a lane: the fewest idle
// lanes, then the fewest waves; runs of rows: about 16 waves a compute unit, 8 rows a
// group at most.
constexpr int kBlockWaves = 8;  // of a workgroup
inline BlockShape block_fwd_shape(int B, int L, int C) {
  BlockShape s{1, 1, 1, 1, 0};
  const int n = C / 8;
  int best = 1 << 30;
  for (int nc = 4; nc >= 1; --nc) {
    const int w = (n + 64 * nc - 1) / (64 * nc);
    if (w > kBlockWaves || (nc == 4 && n <= 64 * 3 * kBlockWaves)) continue;
    const int idle = w * 64 * nc - n;
    if (idle < best) {
      best = idle;
      s.chunks = nc;
      s.waves = w;
    }
  }
  s.groups = s.waves >= 4 ? 1 : 4 / s.waves;
  int64_t per = (int64_t)B * L / (256 * 16 / s.waves);
  per = per < 1 ? 1 : per > 8 ? 8 : per;
  s.rows = (int)(per * s.groups);
  s.runs = (int)(((int64_t)L + s.rows - 1) / s.rows);
  return s;
}

// Shape of the backward: workgroups of `groups` groups of `waves` waves, a row
// each at a time; a workgroup takes `rows` consecutive rows of a batch (a run),
// `runs` of them a batch.
//   One chunk of 8 channels a lane up to ten waves (C = 5120; the registers would
// allow twelve), two up to 8192, four beyond: a lane holds about ten values a
// channel (row, gradients, modulations, column sums).  7803 tokens x 5120, fp32,
// modulations a token: two chunks, five waves 475 us; one chunk, ten waves 309 us.
//   About 512 runs in all: the column sums of a run are written once and read
// once by the reduction, 12 bytes a channel each way (512 runs against 65536
// rows: 1.6 % of the bytes); at least 4 rows a group, so that the loads of one
// row pass under the arithmetic of the one before.
inline BlockShape block_bwd_shape(int B, int L, int C) {
  BlockShape s;
  const int n = C / 8;
  s.chunks = n > 1024 ? 4 : n > 640 ? 2 : 1;
  s.waves = (n + 64 * s.chunks - 1) / (64 * s.chunks);
  s.groups = s.waves >= 8 ? 1 : 8 / s.waves;
  const int64_t want = B > 0 ? (512 + B - 1) / B : 1;  // runs a batch
  int64_t rows = ((int64_t)L + want - 1) / want;
  const int64_t least = 4 * s.groups;
  if (rows < least) rows = least;
  rows = (rows + s.groups - 1) / s.groups * s.groups;
  if (rows > L) rows = L > 0 ? L : 1;
  s.rows = (int)rows;
  s.runs = (int)(((int64_t)L + rows - 1) / rows);
  return s;
}
// fp32 values of the backward's workspace: three column sums a run
inline size_t block_bwd_floats(int B, int L, int C) {
  return (size_t)3 * B * block_bwd_shape(B, L, C).runs * C;
}

__attribute__((weak)) hipError_t launch_block_norm_fwd(const BlockNormFwd& a, hipStream_t stream);
__attribute__((weak)) hipError_t launch_block_norm_bwd(const BlockNormBwd& a, hipStream_t stream);

}  // namespace vidax
