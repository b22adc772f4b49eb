// Internal declarations of the products with group scales.  Not part of the public ABI.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace ffn {

constexpr int kWindow = 128;                // codes of a row that four lanes load at once
constexpr int kGqTokens = 64;               // tokens of a pass
constexpr int kGqSharesMost = 8;            // of a row's windows
constexpr size_t kGqLds = 64 * 1024;        // of one token tile's x: two workgroups to a CU
constexpr int gq_units(bool xf32) { return xf32 ? 2 : 4; }  // 8-column pieces of x that a thread holds while they are on their way

struct GqMatrix {
  const void *codes, *scales, *offsets;
};
struct GqArgs {
  int T, n_in, n_out;
  int windows;         // of a row: 128 codes, or 256 (one token)
  int per_share;       // windows of a workgroup
  int chunk;           // windows of x in LDS at a time
  uint32_t div_group;  // q = (n div_group) >> 31 divides a count of 32 codes by group / 32
  int groups;          // of a row
  const void* x;
  GqMatrix w[2];
  int act, silu_up;
  float t;
  void* y;
  float* part;         // [share][matrix][T][n_out], or null: one share
  uint4* planes;       // x of two token tiles and more, and the table of its sums (k_group_q_split)
  float* sums;
};

constexpr int gq_scales(int nsx) { return nsx == 8 ? 4 : nsx; }
// Windows of a wave in a batch, where the next batch's registers fit beside it.
constexpr int gq_batch(bool gated, int ns) { return gated || ns > 1 ? 1 : 2; }

// Waves that share a row tile's windows with two tiles of tokens and more
constexpr int kGqWaves = 2;

// x of kGqWaves windows of nt token tiles in LDS, with their sums; two of them where the CU has room (160 KB), so that one is
// filled while the other is read.
constexpr size_t gq_buffer(bool xf32, int nt) { return (size_t)kGqWaves * nt * ((xf32 ? 3 : 1) * 4096 + 4 * 64); }
constexpr int gq_buffers(bool xf32, int nt) { return 2 * gq_buffer(xf32, nt) <= 160 * 1024 ? 2 : 1; }

// Tiles of a pass: nt 16-token tiles (0: one token, windows of 256 codes); wk of the 8 waves share a row tile's windows, u at a time each; whole: a share's x
// lies in LDS at once.
struct GqPlan {
  int nt, wk, u;
  bool whole;
  int ns;  // NSX of k_group_q
  int chunk, per_share, shares, blocks;
};
// x and its sums in LDS
inline size_t gq_lds(bool xf32, const GqPlan& p, int T) {
  const size_t planes = xf32 ? 3 : 1;
  if (p.nt == 0) return p.chunk * (planes * 4 * kWindow + (xf32 ? 128 : 32));
  const size_t sums = (size_t)p.chunk * gq_scales(p.ns) * 64 * p.nt;
  return p.nt > 1 ? gq_buffers(xf32, p.nt) * gq_buffer(xf32, p.nt) : planes * T * (p.chunk * 2 * kWindow + 16) + sums;
}
GqPlan gq_plan(bool xf32, bool gated, int group, int T, int n_in, int n_out);

// sf32: fp32 scales
hipError_t launch_group_q_bf16(bool sf32, bool gated, const GqArgs& a, const GqPlan& p, hipStream_t st);
hipError_t launch_group_q_f32(bool sf32, bool gated, const GqArgs& a, const GqPlan& p, hipStream_t st);

}  // namespace ffn
