// The plans of the GroupNorm kernels: which form a call takes, which groups a CTA has, how its threads lie over them.  Host only.
#pragma once
#include "group_norm_warp.cuh"

namespace tsdp {

inline int gcd(int a, int b) { while (b) { const int t = a % b; a = b; b = t; } return a; }

// The smallest set whose channels are a multiple of `unit` fits a CTA.
inline bool set_fits(int C, int groups, int unit) { const int cg = C / groups; return (long long)min(unit / gcd(cg, unit), groups) * cg <= GN_MAX_WIDTH; }

// Which groups a CTA takes, how its threads lie over them, how many CTAs share the positions.
inline void norm_plan(NormArgs& g, int V, int elem, int sms, bool grad) {
  const int cg = g.C / g.groups, most = grad ? GN_STREAM_THREADS : GN_THREADS;
  g.per_set = min(V / gcd(cg, V), g.groups);
  const int step = g.per_set;
  // rows of 128 bytes at least, where a row does not outgrow the threads
  while (g.per_set + step <= g.groups && (g.per_set + step) * cg <= most * V && g.per_set * cg * elem < 128) g.per_set += step;
  // short sequences: more groups a CTA, up to half its threads with four positions each, while every SM has eight of them to do
  // (3102 sequences of 4 x 288 channels in 32 groups, fp32, backward: 124 us with the smallest sets, 75 with these)
  while (2 * g.per_set <= g.groups && (long long)(2 * g.per_set * cg / V) * ((g.L + 3) / 4) <= most / 2 && (long long)g.N * ((g.groups + 2 * g.per_set - 1) / (2 * g.per_set)) >= 8ll * sms)
    g.per_set *= 2;
  g.width = g.per_set * cg;
  g.sets = (g.groups + g.per_set - 1) / g.per_set;
  g.cols = min((g.width + V - 1) / V, most);
  // short sequences take small CTAs, four positions a thread: more of them run beside one another, and what costs them is waiting for barriers
  // (3574 sequences of 16 x 96 channels in 16 groups, backward: 212 us with 512 threads)
  const long long wanted = ((long long)g.cols * ((g.L + 3) / 4) + 31) / 32 * 32;
  g.threads = (int)min((long long)most, max(wanted, max(64ll, (g.cols + 31ll) / 32 * 32)));
  g.lanes = g.threads / g.cols;
  g.ranks = 1;
  while (g.ranks < GN_MAX_RANKS && (long long)g.N * g.sets * g.ranks < 2 * sms && g.L >= 8ll * g.lanes * g.ranks) g.ranks *= 2;
  const long long fill = (long long)sms * (GN_STREAM_THREADS / g.threads) * 2 / ((long long)g.sets * g.ranks);
  g.splits = (int)min((long long)g.N, max(1ll, grad ? fill : (1ll << 24) / ((long long)g.sets * g.ranks)));
}

// The slab kernels' plan: false where a group of one sequence is more than the threads of a CTA hold in registers (SLAB_ITEMS pieces each).
// A set grows while it fits two pieces a thread and leaves four CTAs' worth of work for each place on the chip.
// (GN_SLAB_CTAS on an SM is what the registers allow; past 70 KB of shared memory two fit, and the last of their turns is not full: fp32 backward of
// 2048 x 12 x 640 in two groups, 78 KB.)
constexpr int SLAB_ITEMS = 4, SLAB_SMEM = 112 * 1024;
inline int slab_items(const NormArgs& g, int V, int unit, int per_set, int& cols) {
  cols = (per_set * (g.C / g.groups) + V - 1) / V;
  if (unit == 32) cols = (cols + 32 / V - 1) / (32 / V) * (32 / V);
  return cols > GN_THREADS ? GN_THREADS : (g.L + GN_THREADS / cols - 1) / (GN_THREADS / cols);
}
inline bool slab_plan(NormArgs& g, int V, int unit, int elem, int sms, bool grad, bool copy, int& items, int& smem) {
  const int cg = g.C / g.groups, places = sms * GN_SLAB_CTAS;
  if (cg % V != 0 || (copy && g.C % 16 != 0)) return false;
  if (copy && unit < 16) unit = 16;
  int per_set = min(unit / gcd(cg, unit), g.groups), cols, c2;
  items = slab_items(g, V, unit, per_set, cols);
  if (items > SLAB_ITEMS) return false;
  while (per_set * 2 <= g.groups && (long long)g.N * ((g.groups + 2 * per_set - 1) / (2 * per_set)) >= 4ll * places) {
    const int more = slab_items(g, V, unit, 2 * per_set, c2);
    if (more > max(2, items)) break;
    per_set *= 2; items = more; cols = c2;
  }
  g.per_set = per_set;
  g.width = per_set * cg;
  g.sets = (g.groups + per_set - 1) / per_set;
  g.cols = cols;
  g.lanes = GN_THREADS / cols;
  g.ranks = 1;
  const int gcols = cg / V;
  g.fold = 1;
  while (g.fold < 32 && gcols % (2 * g.fold) == 0 && cols % (2 * g.fold) == 0) g.fold *= 2;
  g.red_rows = cols < 32 && (cols & (cols - 1)) == 0 ? GN_THREADS / 32 : g.lanes;
  const int slab = g.L * g.width;
  g.stage_bytes = grad ? slab * (elem + (copy ? 1 : elem)) + 4 * g.width : slab * elem + 8 * g.width;
  smem = GN_RING * g.stage_bytes;
  if (grad) smem = max(smem + (g.dfilm ? 4 * g.lanes * g.width * 4 : 0), 2 * g.lanes * g.width * 4);
  if (smem > SLAB_SMEM) return false;
  const long long at_once = max(1, places / g.sets), turns = (g.N + at_once - 1) / at_once;
  g.splits = (int)((g.N + turns - 1) / turns);
  return true;
}

// Slabs are taken where a row of a set is a copy worth its name, or all of its rows are one: with copies of 64 to 384 bytes the engine that
// makes them is what they wait for.  (us, slabs / stream, with FiLM; bf16 unless said.  Forward, backward: 4096 x 8 x 512 in one group 48 / 90,
// 70 / 138; 2048 x 12 x 640 in two 60 / 87, 69 / 124, fp32 52 / 104, 113 / 128.  4096 x 16 x 512 in 32 groups: 512 bytes forward 104 / 153, fp32 174 / 169,
// 181 / 237.  4096 x 16 x 384 in 8: 126 / 114, 197 / 202.  Few sequences: 512 x 16 x 384 in 8 47 / 13, 31 / 27.  128 bytes: 1024 x 64 x 256 in 32 68 / 63, 146 / 96.
// The rule is wrong for backward sets of 256 bytes of many sequences, which it gives to the stream: 4096 x 16 x 512 in 32 180 / 234, 4096 x 16 x 256
// in 32 94 / 129.)
inline bool slab_rows(const NormArgs& g, const Rows& r, int elem) { return g.width * elem >= 512 || (g.width == g.C && r.sl == g.C); }

// Teams of warps: false where a group's channels are not 32, 64, 128 or 256 or a lane of eight warps would hold more than `most` pieces of V channels.
inline bool warp_plan(NormArgs& g, int V, int most, int ctas, int sms, int& items) {
  const int cg = g.C / g.groups;
  if (cg < 32 || cg > 256 || (cg & (cg - 1)) || cg / V > 32) return false;
  const int R = 32 / (cg / V);
  g.team = 1;
  while (g.team < GN_WARP_THREADS / 32 && g.L > most * R * g.team) g.team *= 2;
  if (g.L > most * R * g.team) { g.team = 0; return false; }
  items = (g.L + R * g.team - 1) / (R * g.team);
  const long long places = max(1ll, (long long)sms * ctas * (GN_WARP_THREADS / 32) / ((long long)g.groups * g.team)), turns = (g.N + places - 1) / places;
  g.splits = (int)((g.N + turns - 1) / turns);
  g.sets = g.ranks = 1;
  return true;
}

}  // namespace tsdp
