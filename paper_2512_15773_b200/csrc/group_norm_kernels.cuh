// GroupNorm with an activation and FiLM vectors over channels-last activations, and its gradients, for training.
//
//   h = (x - mean_g) rstd_g       mean, 1 / sqrt(variance + eps) over the L positions and C / groups channels of a group
//   z = gamma h + beta,  a = act(z),  y = scale a + bias          scale, bias [N, C]: the FiLM vectors, 1 and 0 without them
//
//   dz = dy scale act'(z);   dbeta = sum dz;   dgamma = sum dz h;   dscale = sum_l dy a;   dbias = sum_l dy
//   dx = rstd (gamma dz - m1 - h m2),   m1, m2: means over the group of gamma dz and gamma dz h
//
// The group sums of the last line follow from the sums over l of dz and dz h that a channel needs anyway:
// sum_group gamma dz = sum_c gamma_c sum_l dz.
//
// What bounds them: bytes. Forward x and y once each, backward dy, x (or its 8-bit copy) and dx.
// Three forms hold to that as far as a group's size allows; this file has the one for every size, stride and alignment:
// A cluster of CTAs owns some groups of one sequence, each CTA a share of the positions: statistics need all of a group before its
// first output.  A thread owns V neighbouring channels (16 bytes) and walks positions, so that the affine and FiLM
// vectors stay in registers and sums over positions need no exchange until the end.  The second walk reads x (and dy) again: what the cluster has just read is in the L2.
// What bounds it where sequences are few: the two dependent walks and the exchange between them.  3 x 4099 x 320 in 32 groups, SiLU, fp32: 13 us
// back to back (2.4 TB/s; issue slots 17 % used); keeping rows in shared memory for the second walk did not help (17.1 us against 15.8), nor did
// clusters of 16 (29 us: twice the exchange).  16 x 4096 x 512 in 8 groups, Mish, FiLM, bf16: 65 us, backward 141.
// V: four channels a thread, for 16-bit types too (without FiLM 70 us with eight, 58 with four, in the last case), else one at a time.
#pragma once
#include "checkpoint_kernels.cuh"
#include "gemm_tcgen05.cuh"

namespace tsdp {

enum { ACT_NONE = 0, ACT_MISH = 1, ACT_SILU = 2, ACT_GELU = 3 };

// a = act(z) and its derivative, two values at a time on the packed fp32 pipe.  One exponential and one reciprocal each, by the hardware
// instructions: e^v is off by 2 units of 2^-24 and by the rounding of v log2(e), 2e-6 of e^v at the ends of the range where it matters
// (|z| <= 20).
// Mish: with u = e^z, r = 1 / ((u + 1)^2 + 1):  tanh(log(1 + u)) = t = u (u + 2) r,  derivative t + 4 z r (u (u + 1) r).  Past z = 20 both are
// those of the identity to 2^-24, and u is held there so that it stays finite (min.NaN: a NaN stays one).
// GELU (tanh form): 1/2 (1 + tanh w) = 1 / (1 + e^-2w); past |z| = 100 that is 0 or 1 and the polynomial is held.
__device__ __forceinline__ float act_ex2(float v) { float r; asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v)); return r; }
__device__ __forceinline__ float act_rcp(float v) { float r; asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v)); return r; }
__device__ __forceinline__ float act_min(float a, float b) { float r; asm("min.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b)); return r; }
__device__ __forceinline__ float2 two(float v) { return make_float2(v, v); }
__device__ __forceinline__ float2 exp2_of(float2 v, float k) { v = __fmul2_rn(v, two(k)); return make_float2(act_ex2(v.x), act_ex2(v.y)); }
__device__ __forceinline__ float2 rcp_of(float2 v) { return make_float2(act_rcp(v.x), act_rcp(v.y)); }
constexpr float ACT_LOG2E = 1.4426950408889634f;
template <bool GRAD> __device__ __forceinline__ void act_pair(int act, float2 z, float2& a, float2& d) {
  if (act == ACT_MISH) {
    const float2 zc = make_float2(act_min(z.x, 20.f), act_min(z.y, 20.f)), u = exp2_of(zc, ACT_LOG2E), w = __fadd2_rn(u, two(1.f));
    const float2 r = rcp_of(__ffma2_rn(w, w, two(1.f)));
    // (the values themselves to their last digits; with the derivative, which is of the order of 1, to those of 1)
    const float2 t = GRAD ? __ffma2_rn(r, two(-2.f), two(1.f)) : __fmul2_rn(__ffma2_rn(u, u, __fadd2_rn(u, u)), r);
    a = __fmul2_rn(z, t);
    if (GRAD) d = __ffma2_rn(__fmul2_rn(zc, __fmul2_rn(__fmul2_rn(r, r), __fmul2_rn(u, w))), two(4.f), t);
  } else if (act == ACT_SILU) {
    const float2 s = rcp_of(__fadd2_rn(exp2_of(z, -ACT_LOG2E), two(1.f)));
    a = __fmul2_rn(z, s);
    if (GRAD) d = __ffma2_rn(a, __ffma2_rn(s, two(-1.f), two(1.f)), s);
  } else if (act == ACT_GELU) {
    float2 q = __fmul2_rn(z, z);
    q = make_float2(act_min(q.x, 1e4f), act_min(q.y, 1e4f));
    const float k = 0.7978845608028654f;
    const float2 s = rcp_of(__fadd2_rn(exp2_of(__fmul2_rn(z, __ffma2_rn(q, two(0.044715f), two(1.f))), -2.f * k * ACT_LOG2E), two(1.f)));
    a = __fmul2_rn(z, s);
    if (GRAD) d = __ffma2_rn(__fmul2_rn(a, __ffma2_rn(s, two(-1.f), two(1.f))), __ffma2_rn(q, two(2.f * k * 0.134145f), two(2.f * k)), s);
  } else {
    a = z;
    if (GRAD) d = two(1.f);
  }
}
// V values (4, 8 or 16 bytes, or one value) of memory as they are.
template <typename T, int V> struct Piece { uint32_t w[V == 1 ? 1 : V * sizeof(T) / 4]; };
template <typename T, int V> __device__ __forceinline__ Piece<T, V> load_piece(const uint8_t* p) {
  Piece<T, V> r;
  if constexpr (V == 1) r.w[0] = sizeof(T) == 4 ? *reinterpret_cast<const uint32_t*>(p) : sizeof(T) == 2 ? *reinterpret_cast<const unsigned short*>(p) : *p;
  else if constexpr (sizeof(r) == 16) { const uint4 u = *reinterpret_cast<const uint4*>(p); r.w[0] = u.x; r.w[1] = u.y; r.w[2] = u.z; r.w[3] = u.w; }
  else if constexpr (sizeof(r) == 8) { const uint2 u = *reinterpret_cast<const uint2*>(p); r.w[0] = u.x; r.w[1] = u.y; }
  else r.w[0] = *reinterpret_cast<const uint32_t*>(p);
  return r;
}
template <typename T, int V> __device__ __forceinline__ void piece_values(const Piece<T, V>& r, float2* v) {
#pragma unroll
  for (int i = 0; i < V / 2; ++i) {
    if constexpr (sizeof(T) == 2) v[i] = make_float2(__uint_as_float(r.w[i] << 16), __uint_as_float(r.w[i] & 0xffff0000u));
    else if constexpr (sizeof(T) == 4) v[i] = make_float2(__uint_as_float(r.w[2 * i]), __uint_as_float(r.w[2 * i + 1]));
    else {                                     // (by the conversion instruction: its pipe has room here, that of the permutations has none: 70 us, not 78)
      const uint32_t u = r.w[i >> 1] >> (16 * (i & 1));
      v[i] = make_float2((float)(signed char)u, (float)(signed char)(u >> 8));
    }
  }
}
// The same as pairs; one value stands with a zero.
template <typename T, int V> __device__ __forceinline__ void piece_pairs(const Piece<T, V>& r, float2* v) {
  if constexpr (V == 1) v[0] = make_float2(sizeof(T) == 4 ? __uint_as_float(r.w[0]) : sizeof(T) == 2 ? __uint_as_float(r.w[0] << 16) : (float)(signed char)r.w[0], 0.f);
  else piece_values<T, V>(r, v);
}
__host__ __device__ constexpr int pairs_of(int V) { return V > 1 ? V / 2 : 1; }
template <typename T, int V> __device__ __forceinline__ void store_pairs(T* p, const float2* v) {
  if constexpr (V == 1) *p = from_f<T>(v[0].x);
  else if constexpr (sizeof(T) == 2 && V == 8) *reinterpret_cast<uint4*>(p) = make_uint4(pack_bf16(v[0].x, v[0].y), pack_bf16(v[1].x, v[1].y), pack_bf16(v[2].x, v[2].y), pack_bf16(v[3].x, v[3].y));
  else if constexpr (sizeof(T) == 2) *reinterpret_cast<uint2*>(p) = make_uint2(pack_bf16(v[0].x, v[0].y), pack_bf16(v[1].x, v[1].y));
  else *reinterpret_cast<float4*>(p) = make_float4(v[0].x, v[0].y, v[1].x, v[1].y);
}

// f(the activation as a constant): the choice is made once, not for every value.
template <int A> struct ActIs { static constexpr int value = A; };
template <typename F> __device__ __forceinline__ void with_act(int act, F&& f) {
  if (act == ACT_MISH) f(ActIs<ACT_MISH>{});
  else if (act == ACT_SILU) f(ActIs<ACT_SILU>{});
  else if (act == ACT_GELU) f(ActIs<ACT_GELU>{});
  else f(ActIs<ACT_NONE>{});
}

struct NormArgs {
  int N, L, C, groups, act;
  float eps;
  Rows x, y, dy, dx;
  const float *gamma, *beta, *film;            // film [N, 2C]: scale, bias; null
  float *mean, *rstd;                          // [N, groups]
  Copy8 cx, cy;                                // forward: 8-bit copies to write (q null: none); backward: cx is x
  float *dfilm, *part;                         // [N, 2C] or null; [splits, 2, C]
  // the plan: a set is `per_set` groups, `width` channels; cols threads on a position; `ranks` CTAs of a cluster share the positions
  int per_set, sets, width, cols, lanes, ranks, splits, threads;
  // slab kernels: threads of a group that a shuffle adds up; rows of partial sums left (of warps or lanes); bytes of a stage
  int fold, red_rows, stage_bytes;
  int team;                                    // warp kernels: warps of a group (0 elsewhere)
  long long wait_cycles;                       // slab kernels: limit of every wait
  int withhold;                                // CTA 0 gets no rows (tsdp_debug_arm_train_timeout)
};

constexpr int GN_STREAM_V = 4;                 // channels of a thread over long sequences and in every backward pass: with eight (16 bytes of
                                               // bf16) its vectors and sums do not fit the registers
constexpr int GN_THREADS = 256, GN_STREAM_THREADS = 512;      // of the kernels; of the backward one over long sequences (few CTAs with much to fetch)
constexpr int GN_MAX_RANKS = 8;               // CTAs of a cluster
constexpr int GN_MAX_WIDTH = 2048;             // channels of a set: their sums stay in shared memory

__device__ __forceinline__ float ld_rank_f32(const float* p, uint32_t rank) {       // the same shared-memory word of another CTA of the cluster
  float v;
  asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(ptx::mapa_rank(ptx::smem_u32(p), rank)) : "memory");
  return v;
}

// Mean and variance from the mean and the mean square of values about a point near their mean (the sum of the values, rounded at its size, over their
// number).  The point is corrected where it is farther from zero than the values are spread: there the sum's roundings count; elsewhere
// those of the deviations do (16-bit values less a number of 24 bits are all rounded to one side) and the sum itself is the better one.
// (Rounding may leave the difference of two equal numbers below zero; a NaN stays one.)
__device__ __forceinline__ float variance_about(float square, float off) { const float v = fmaf(-off, off, square); return v < 0.f ? 0.f : v; }
__device__ __forceinline__ float mean_about(float about, float square, float off) { return about * about > square ? about + off : about; }

// Positions of lane r of a share that is walked in steps of `lanes`: `all` each, one more in the first `extra`.
struct LaneRows {
  int all, extra;
  __device__ __forceinline__ LaneRows(int positions, int lanes) : all(positions / lanes), extra(positions % lanes) {}
  __device__ __forceinline__ int operator()(int r) const { return all + (r < extra ? 1 : 0); }
};

// ------------------------------------------------------------------------------------------------------------------ forward
// First walk: each thread keeps, per channel, the sums S and Q of deviations and their squares about a point p, at first its first value.  After
// every eight positions p moves to the mean of the n values so far, by d: Q -= d (2 S - n d), S -= n d.  So neither a large mean costs digits nor
// a first value apart from the rest (about one fixed point, 1000 before 2000 values of 0.1: variance 8 % off).  p and Q, the mean and the centred
// sum of squares of its share, are then merged, thread by thread and CTA by CTA, with their counts: M2 = sum M2_i + n_i (mean_i - mean)^2.
template <typename T, int V>
__global__ void __launch_bounds__(GN_THREADS, 2)
group_norm_kernel(NormArgs g) {
  constexpr int P = pairs_of(V);
  extern __shared__ __align__(16) float gn_smem[];
  pdl_wait();
  const int cg = g.C / g.groups, threads = blockDim.x;
  float* s_mean = gn_smem;                                  // [lanes][tile channels]
  float* s_m2 = s_mean + threads * V;                    // the same
  float* s_grp = s_m2 + threads * V;                     // [2][per_set]: this CTA's mean and M2
  float* s_stat = s_grp + 2 * g.per_set;                    // [2][per_set]: mean and rstd
  const uint32_t rank = g.ranks > 1 ? ptx::cluster_rank() : 0u;
  const int set = (blockIdx.x / g.ranks) % g.sets, split = blockIdx.x / g.ranks / g.sets;
  const int c_set = set * g.width, width = min(g.width, g.C - c_set), n_grp = width / cg;
  const int share = (g.L + g.ranks - 1) / g.ranks, lo = min(g.L, (int)rank * share), hi = min(g.L, lo + share);
  const int lane = threadIdx.x / g.cols, col = threadIdx.x - lane * g.cols, tile = g.cols * V;
  const int warp = threadIdx.x >> 5, wl = threadIdx.x & 31;
  const LaneRows lane_rows(hi - lo, g.lanes);
  for (int n = split; n < g.N; n += g.splits) {
    const T* x = reinterpret_cast<const T*>(g.x.p) + n * g.x.sn + c_set;
    // a group may be wider than a tile of columns: its parts are merged in turn
    for (int t0 = 0; t0 < width; t0 += tile) {
      const int c = t0 + col * V;
      const bool in = lane < g.lanes && c < width;
      if (in) {
        float2 k[P], sum[P], sq[P];               // minus a point at the mean so far, sums about it
#pragma unroll
        for (int i = 0; i < P; ++i) k[i] = sum[i] = sq[i] = two(0.f);
        int l = lo + lane;
        if (l < hi) piece_pairs<T, V>(load_piece<T, V>(reinterpret_cast<const uint8_t*>(x + l * g.x.sl + c)), k);
#pragma unroll
        for (int i = 0; i < P; ++i) k[i] = __fmul2_rn(k[i], two(-1.f));
        constexpr int U = 8;                      // positions asked for together
        const T* at_l = x + l * g.x.sl + c;
        const long long step = g.lanes * g.x.sl;
        int seen = 0;
        for (; l < hi; l += U * g.lanes, at_l += U * step) {
          Piece<T, V> raw[U];
#pragma unroll
          for (int j = 0; j < U; ++j) {
            raw[j] = Piece<T, V>{};
            if (l + j * g.lanes < hi) raw[j] = load_piece<T, V>(reinterpret_cast<const uint8_t*>(at_l + j * step));
          }
#pragma unroll
          for (int j = 0; j < U; ++j) {
            const bool there = l + j * g.lanes < hi;
            float2 v[P];
            piece_pairs<T, V>(raw[j], v);
#pragma unroll
            for (int i = 0; i < P; ++i) {
              float2 d = __fadd2_rn(v[i], k[i]);
              if (!there) d = two(0.f);
              sum[i] = __fadd2_rn(sum[i], d); sq[i] = __ffma2_rn(d, d, sq[i]);
            }
            seen += there;
          }
          const float n = (float)seen, of_seen = -act_rcp(n);
#pragma unroll
          for (int i = 0; i < P; ++i) {
            const float2 at = __ffma2_rn(sum[i], two(of_seen), k[i]), by = __ffma2_rn(at, two(-1.f), k[i]);         // the point moves by `by`
            const float2 rest = __ffma2_rn(by, two(-n), sum[i]);
            sq[i] = __ffma2_rn(__fmul2_rn(by, two(-1.f)), __fadd2_rn(sum[i], rest), sq[i]);
            sum[i] = rest;
            k[i] = at;
          }
        }
#pragma unroll
        for (int i = 0; i < V; ++i) {
          s_mean[lane * tile + col * V + i] = -(i & 1 ? k[i / 2].y : k[i / 2].x);      // (the sums about it are what its rounding leaves)
          s_m2[lane * tile + col * V + i] = i & 1 ? sq[i / 2].y : sq[i / 2].x;
        }
      }
      __syncthreads();
      // groups that this tile holds (a part of): a warp each
      const int t1 = min(width, t0 + tile);
      for (int gr = t0 / cg + warp; gr * cg < t1; gr += threads / 32) {
        const int a = max(gr * cg, t0) - t0, b = min(gr * cg + cg, t1) - t0, w = b - a, items = w * g.lanes;
        const float inv_w = 1.f / w;                         // (i / w of a few thousand by a product: off by less than the half it stands away from a whole number)
        // Where the first and the last channel of lane 0 say that means are far from zero against what they and the values differ by, they are summed about
        // one of them: a sum of large means is rounded at its size.
        const float first = s_mean[a];
        const float about = fabsf(first - s_mean[b - 1]) < 0.125f * fabsf(first) && 64.f * s_m2[a] < lane_rows(0) * first * first ? first : 0.f;
        float sum = 0.f;
        for (int i = wl; i < items; i += 32) {
          const int r = (int)((i + 0.5f) * inv_w);
          sum += lane_rows(r) * (s_mean[r * tile + a + i - r * w] - about);
        }
        const float cnt = (float)(hi - lo) * w;
        const float m = cnt > 0.f ? about + warp_sum(sum) / cnt : 0.f;
        float m2 = 0.f;
        for (int i = wl; i < items; i += 32) {
          const int r = (int)((i + 0.5f) * inv_w), rows = lane_rows(r);
          const float d = s_mean[r * tile + a + i - r * w] - m;
          if (rows) m2 += s_m2[r * tile + a + i - r * w] + rows * d * d;
        }
        m2 = warp_sum(m2);
        if (wl == 0) {
          if (gr * cg >= t0) { s_grp[gr] = m; s_grp[g.per_set + gr] = m2; }
          else {                                            // the group began in an earlier tile, with `before` channels of it
            const float nb = (float)(hi - lo) * (t0 - gr * cg), d = m - s_grp[gr], f = nb + cnt > 0.f ? cnt / (nb + cnt) : 0.f;
            s_grp[gr] += d * f;
            s_grp[g.per_set + gr] += m2 + d * d * nb * f;
          }
        }
      }
      __syncthreads();
    }
    if (g.ranks > 1) ptx::cluster_sync_all();
    for (int gr = threadIdx.x; gr < n_grp; gr += threads) {
      float m = s_grp[gr], m2 = s_grp[g.per_set + gr];
      if (g.ranks > 1) {
        float mr[GN_MAX_RANKS], qr[GN_MAX_RANKS];              // (all asked for before the first is used: each takes a quarter of a microsecond)
#pragma unroll
        for (int r = 0; r < GN_MAX_RANKS; ++r)
          if (r < g.ranks) { mr[r] = ld_rank_f32(s_grp + gr, r); qr[r] = ld_rank_f32(s_grp + g.per_set + gr, r); }
        m = 0.f; m2 = 0.f;
        auto rows_of = [&](int r) { return (float)max(0, min(g.L, (r + 1) * share) - min(g.L, r * share)); };
#pragma unroll
        for (int r = 0; r < GN_MAX_RANKS; ++r)
          if (r < g.ranks) m += (mr[r] - mr[0]) * rows_of(r);
        m = mr[0] + m / (float)g.L;
#pragma unroll
        for (int r = 0; r < GN_MAX_RANKS; ++r)
          if (r < g.ranks && rows_of(r) > 0.f) { const float d = mr[r] - m; m2 += qr[r] + d * d * rows_of(r) * cg; }
      }
      const float rs = rsqrtf(m2 / ((float)g.L * cg) + g.eps);
      s_stat[gr] = m; s_stat[g.per_set + gr] = rs;
      if (rank == 0) {
        const long long at = (long long)n * g.groups + c_set / cg + gr;
        if (g.mean) g.mean[at] = m;
        if (g.rstd) g.rstd[at] = rs;
      }
    }
    __syncthreads();
    // second walk
    T* y = reinterpret_cast<T*>(g.y.p) + n * g.y.sn + c_set;
    for (int t0 = 0; t0 < width; t0 += tile) {
      const int c = t0 + col * V;
      const bool in = lane < g.lanes && c < width;
      if (!in) continue;
      float2 ka[P], kb[P], fs[P], fb[P];                       // z = (x + kb) ka + beta, in two steps: x - mean first
      float2 be[P];
#pragma unroll
      for (int i = 0; i < P; ++i) { ka[i] = kb[i] = be[i] = fb[i] = two(0.f); fs[i] = two(1.f); }
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const int ch = c_set + c + i, gr = (c + i) / cg;
        auto set = [&](float2* a, float v) { if (i & 1) a[i / 2].y = v; else a[i / 2].x = v; };
        set(ka, g.gamma[ch] * s_stat[g.per_set + gr]); set(kb, -s_stat[gr]); set(be, g.beta[ch]);
        if (g.film) { set(fs, g.film[(long long)n * 2 * g.C + ch]); set(fb, g.film[((long long)n * 2 + 1) * g.C + ch]); }
      }
      with_act(g.act, [&](auto act) {
        constexpr int U = 4;                                   // positions asked for together
        for (int l = lo + lane; l < hi; l += U * g.lanes) {
          Piece<T, V> raw[U];
#pragma unroll
          for (int j = 0; j < U; ++j)
            if (l + j * g.lanes < hi) raw[j] = load_piece<T, V>(reinterpret_cast<const uint8_t*>(x + (l + j * g.lanes) * g.x.sl + c));
#pragma unroll
          for (int j = 0; j < U; ++j) {
            if (l + j * g.lanes >= hi) break;
            float2 v[P];
            piece_pairs<T, V>(raw[j], v);
#pragma unroll
            for (int i = 0; i < P; ++i) {
              float2 d;
              act_pair<false>(decltype(act)::value, __ffma2_rn(__fadd2_rn(v[i], kb[i]), ka[i], be[i]), v[i], d);
              v[i] = __ffma2_rn(v[i], fs[i], fb[i]);
            }
            store_pairs<T, V>(y + (l + j * g.lanes) * g.y.sl + c, v);
          }
        }
      });
    }
    if (g.ranks > 1) ptx::cluster_sync_all();               // s_grp may be written again once every CTA has read it
    else __syncthreads();
  }
  if (g.ranks > 1) ptx::cluster_sync_all();                 // no CTA leaves while another may read its shared memory
}

// ------------------------------------------------------------------------------------------------------------------ backward
// Of a thread's channels: gamma, beta, -mean, rstd, FiLM scale.
template <int V> struct NormVectors { float2 ga[pairs_of(V)], be[pairs_of(V)], mu[pairs_of(V)], rs[pairs_of(V)], fs[pairs_of(V)]; };
template <int V>
__device__ __forceinline__ void norm_vectors(const NormArgs& g, int n, int c, NormVectors<V>& p) {
  const int cg = g.C / g.groups;
#pragma unroll
  for (int i = 0; i < pairs_of(V); ++i) { p.ga[i] = p.be[i] = p.mu[i] = p.rs[i] = two(0.f); p.fs[i] = two(1.f); }
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const long long gr = (long long)n * g.groups + (c + i) / cg;
    auto set = [&](float2* a, float v) { if (i & 1) a[i / 2].y = v; else a[i / 2].x = v; };
    set(p.ga, g.gamma[c + i]); set(p.be, g.beta[c + i]); set(p.mu, -g.mean[gr]); set(p.rs, g.rstd[gr]);
    if (g.film) set(p.fs, g.film[(long long)n * 2 * g.C + c + i]);
  }
}

// f(position, dz, h, dy, dy a) for this lane's positions, GN_WALK of them asked for together.
constexpr int GN_WALK = 2;
template <typename T, int V, bool COPY, typename F>
__device__ __forceinline__ void norm_walk(const NormArgs& g, int n, int l0, int hi, int c, const NormVectors<V>& p, F&& f) {
  using X = std::conditional_t<COPY, signed char, T>;
  constexpr int P = pairs_of(V);
  const X* x0 = COPY ? reinterpret_cast<const X*>(g.cx.q) + (long long)n * g.L * g.C + c : reinterpret_cast<const X*>(g.x.p) + n * g.x.sn + c;
  const T* dy0 = reinterpret_cast<const T*>(g.dy.p) + n * g.dy.sn + c;
  const long long xl = COPY ? g.C : g.x.sl, nb = copy_blocks(g.C);
  const unsigned char* b0 = COPY ? g.cx.b + (long long)n * g.L * nb + (c >> 5) : nullptr;
  with_act(g.act, [&](auto act) {
    for (int l = l0; l < hi; l += GN_WALK * g.lanes) {
      Piece<X, V> x[GN_WALK];
      Piece<T, V> dy[GN_WALK];
      uint32_t b[GN_WALK];
#pragma unroll
      for (int j = 0; j < GN_WALK; ++j) {
        const int lj = l + j * g.lanes;
        x[j] = Piece<X, V>{};
        dy[j] = Piece<T, V>{};
        b[j] = 0u;
        if (lj < hi) {
          x[j] = load_piece<X, V>(reinterpret_cast<const uint8_t*>(x0 + lj * xl));
          dy[j] = load_piece<T, V>(reinterpret_cast<const uint8_t*>(dy0 + lj * g.dy.sl));
          if (COPY) b[j] = b0[lj * nb];
        }
      }
#pragma unroll
      for (int j = 0; j < GN_WALK; ++j) {
        if (j > 0 && l + j * g.lanes >= hi) break;
        float2 h[P], dz[P], dya[P], dyf[P];
        piece_pairs<X, V>(x[j], h);
        piece_pairs<T, V>(dy[j], dyf);
        const float step = COPY ? copy_step(b[j]) : 1.f;
#pragma unroll
        for (int i = 0; i < P; ++i) {
          h[i] = __fmul2_rn(COPY ? __ffma2_rn(h[i], two(step), p.mu[i]) : __fadd2_rn(h[i], p.mu[i]), p.rs[i]);
          float2 a, d;
          act_pair<true>(decltype(act)::value, __ffma2_rn(h[i], p.ga[i], p.be[i]), a, d);
          dz[i] = __fmul2_rn(__fmul2_rn(dyf[i], p.fs[i]), d);
          dya[i] = __fmul2_rn(dyf[i], a);
        }
        f(l + j * g.lanes, dz, h, dyf, dya);
      }
    }
  });
}

// A cluster walks the sequences split, split + splits, ... and keeps its channels' share of dgamma and dbeta in shared memory.
template <typename T, int V, bool COPY>
__global__ void __launch_bounds__(GN_STREAM_THREADS, 1)
group_norm_grad_kernel(NormArgs g) {
  constexpr int P = pairs_of(V);
  extern __shared__ __align__(16) float gn_smem[];
  pdl_wait();
  const int cg = g.C / g.groups, threads = blockDim.x;
  float* s_lane = gn_smem;                                  // [4][lanes][tile channels]: sums of a lane
  float* s_sum = s_lane + 4 * threads * V;               // [4][width]: of the CTA
  float* s_tot = s_sum + 4 * g.width;                       // [2][width]: of the cluster (dz, dz h)
  float* s_acc = s_tot + 2 * g.width;                       // [2][width]: over the sequences so far
  float* s_grp = s_acc + 2 * g.width;                       // [2][per_set]: m1, m2
  const uint32_t rank = g.ranks > 1 ? ptx::cluster_rank() : 0u;
  const int set = (blockIdx.x / g.ranks) % g.sets, split = blockIdx.x / g.ranks / g.sets;
  const int c_set = set * g.width, width = min(g.width, g.C - c_set), n_grp = width / cg;
  const int share = (g.L + g.ranks - 1) / g.ranks, lo = min(g.L, (int)rank * share), hi = min(g.L, lo + share);
  const int lane = threadIdx.x / g.cols, col = threadIdx.x - lane * g.cols, tile = g.cols * V;
  const int warp = threadIdx.x >> 5, wl = threadIdx.x & 31;
  const bool film = g.film != nullptr && g.dfilm != nullptr;
  const int sums = film ? 4 : 2;
  for (int i = threadIdx.x; i < 2 * g.width; i += threads) s_acc[i] = 0.f;
  for (int n = split; n < g.N; n += g.splits) {
    for (int t0 = 0; t0 < width; t0 += tile) {
      const int c = t0 + col * V;
      const bool in = lane < g.lanes && c < width;
      if (in) {
        NormVectors<V> p;
        norm_vectors<V>(g, n, c_set + c, p);
        float2 sum[4][P];
#pragma unroll
        for (int k = 0; k < 4; ++k)
#pragma unroll
          for (int i = 0; i < P; ++i) sum[k][i] = two(0.f);
        norm_walk<T, V, COPY>(g, n, lo + lane, hi, c_set + c, p, [&](int, const float2* dz, const float2* h, const float2* dy, const float2* dya) {
#pragma unroll
          for (int i = 0; i < P; ++i) {
            sum[0][i] = __fadd2_rn(sum[0][i], dz[i]); sum[1][i] = __ffma2_rn(dz[i], h[i], sum[1][i]);
            sum[2][i] = __fadd2_rn(sum[2][i], dya[i]); sum[3][i] = __fadd2_rn(sum[3][i], dy[i]);
          }
        });
#pragma unroll
        for (int k = 0; k < 4; ++k)
          if (k < sums)
#pragma unroll
            for (int i = 0; i < V; ++i) s_lane[k * threads * V + lane * tile + col * V + i] = i & 1 ? sum[k][i / 2].y : sum[k][i / 2].x;
      }
      __syncthreads();
      const int w = min(width - t0, tile);
      for (int i = threadIdx.x; i < sums * w; i += threads) {
        const int k = i / w, cc = i - k * w;
        float s = 0.f;
        for (int r = 0; r < g.lanes; ++r) s += s_lane[k * threads * V + r * tile + cc];
        s_sum[k * g.width + t0 + cc] = s;
      }
      __syncthreads();
    }
    if (g.ranks > 1) ptx::cluster_sync_all();
    for (int i = threadIdx.x; i < sums * width; i += threads) {
      const int k = i / width, c = i - k * width;
      float s = s_sum[k * g.width + c];
      if (g.ranks > 1) {
        float sr[GN_MAX_RANKS];
#pragma unroll
        for (int r = 0; r < GN_MAX_RANKS; ++r) sr[r] = r < g.ranks ? ld_rank_f32(s_sum + k * g.width + c, r) : 0.f;
        s = 0.f;
#pragma unroll
        for (int r = 0; r < GN_MAX_RANKS; ++r) s += sr[r];
      }
      if (k < 2) { s_tot[k * g.width + c] = s; s_acc[k * g.width + c] += s; }
      else if (rank == 0) g.dfilm[((long long)n * 2 + k - 2) * g.C + c_set + c] = s;
    }
    __syncthreads();
    const float inv = 1.f / ((float)g.L * cg);
    for (int gr = warp; gr < n_grp; gr += threads / 32) {
      float a = 0.f, b = 0.f;
      for (int i = wl; i < cg; i += 32) {
        const float ga = g.gamma[c_set + gr * cg + i];
        a = __fadd_rn(a, __fmul_rn(ga, s_tot[gr * cg + i])); b = __fadd_rn(b, __fmul_rn(ga, s_tot[g.width + gr * cg + i]));
      }
      a = warp_sum(a); b = warp_sum(b);
      if (wl == 0) { s_grp[gr] = a * inv; s_grp[g.per_set + gr] = b * inv; }
    }
    __syncthreads();
    T* dx = reinterpret_cast<T*>(g.dx.p) + n * g.dx.sn + c_set;
    for (int t0 = 0; t0 < width; t0 += tile) {
      const int c = t0 + col * V;
      if (!(lane < g.lanes && c < width)) continue;
      NormVectors<V> p;
      norm_vectors<V>(g, n, c_set + c, p);
      float2 m1[P], m2[P];                                     // -m1, -m2
#pragma unroll
      for (int i = 0; i < P; ++i) m1[i] = m2[i] = two(0.f);
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const int gr = (c + i) / cg;
        if (i & 1) { m1[i / 2].y = -s_grp[gr]; m2[i / 2].y = -s_grp[g.per_set + gr]; }
        else { m1[i / 2].x = -s_grp[gr]; m2[i / 2].x = -s_grp[g.per_set + gr]; }
      }
      norm_walk<T, V, COPY>(g, n, lo + lane, hi, c_set + c, p, [&](int l, float2* dz, const float2* h, const float2*, const float2*) {
        // (the product rounded before m1 is taken off: where a group is one value, the two are the same number)
#pragma unroll
        for (int i = 0; i < P; ++i) dz[i] = __fmul2_rn(p.rs[i], __ffma2_rn(h[i], m2[i], __fadd2_rn(__fmul2_rn(dz[i], p.ga[i]), m1[i])));
        store_pairs<T, V>(dx + l * g.dx.sl + c, dz);
      });
    }
    if (g.ranks > 1) ptx::cluster_sync_all();
    else __syncthreads();
  }
  __syncthreads();
  if (rank == 0)
    for (int i = threadIdx.x; i < 2 * width; i += threads) {
      const int k = i / width, c = i - k * width;
      g.part[((long long)split * 2 + k) * g.C + c_set + c] = s_acc[k * g.width + c];
    }
  if (g.ranks > 1) ptx::cluster_sync_all();
}

// dbeta, dgamma: the shares of the splits, in their order.
constexpr int GN_JOIN_CH = 32, GN_JOIN_LANES = 32;
__global__ void __launch_bounds__(GN_JOIN_CH * GN_JOIN_LANES)
group_norm_join_kernel(const float* part, int splits, int C, float* dgamma, float* dbeta) {
  pdl_wait();
  __shared__ float s[GN_JOIN_LANES][GN_JOIN_CH];
  const int c = (blockIdx.x >> 1) * GN_JOIN_CH + (threadIdx.x % GN_JOIN_CH), k = blockIdx.x & 1, lane = threadIdx.x / GN_JOIN_CH;
  float v = 0.f;
  if (c < C)
#pragma unroll 8
    for (int i = lane; i < splits; i += GN_JOIN_LANES) v += part[((long long)i * 2 + k) * C + c];
  s[lane][threadIdx.x % GN_JOIN_CH] = v;
  __syncthreads();
  if (lane == 0 && c < C) {
    for (int i = 1; i < GN_JOIN_LANES; ++i) v += s[i][threadIdx.x];
    (k ? dgamma : dbeta)[c] = v;
  }
}

}  // namespace tsdp
