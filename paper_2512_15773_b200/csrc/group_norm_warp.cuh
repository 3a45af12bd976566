// The same operators with a warp, or a team of 2, 4 or 8 warps, per group: where a group of one sequence is at most 32 values a lane
// (backward in fp32: 16).  Every level of the UNet takes one warp (512 values: 16 x 32, 8 x 64, 4 x 128), a 50 x 128 group eight.
// Sums pass by shuffles, between the warps of a team through a few words and a barrier of their own; a warp that waits holds up no other
// team.  A team keeps its group and walks the sequences; the rows of its next one are on their way while it works on this one.
// What bounds them: the latency of dependent chains (two reductions a sequence, activation, rounding, the copies' largest magnitudes) at the few warps
// that the registers leave; no pipe is full.  4096 x 16 x 512 in 8 groups, Mish, FiLM, bf16: forward with both copies 63 us (3.5 TB/s; 58 % of the issue
// slots, arithmetic pipe 46 %, 24 warps an SM in 80 registers), backward from a copy 63 us (3.2 TB/s; 52 %, special functions 53 %, 16 warps);
// by slabs 157 and 201.
// Lanes lie over the group's channels first (16 bytes each, backward four channels), then over positions.  Channels of a group: 32, 64, 128 or 256.
#pragma once
#include "group_norm_slab.cuh"

namespace tsdp {

constexpr int GN_WARP_THREADS = 256;

__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
// `rows` rows of `bytes` bytes (a power of two, 16 at least), `pitch` apart, packed to dst by the lanes of a warp.
__device__ __forceinline__ void warp_rows(uint32_t dst, const char* src, long long pitch, int bytes, int rows, int wl) {
  const int shift = 31 - __clz(bytes);
  for (int o = wl * 16; o < rows * bytes; o += 512) cp_async16(dst + o, src + (o >> shift) * pitch + (o & (bytes - 1)));
}
// Rows that a stage has room for and a sequence does not have stay zero: they are worked on like the others and count nothing.
__device__ __forceinline__ void zero_stages(uint32_t dst, int bytes, int wl) {
  for (int o = wl * 16; o < bytes; o += 512) asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(dst + o), "r"(0u) : "memory");
}
// What the warps of a team have to add up: slot[k] of each, K values; the same in all of them afterwards.  `words` is used anew two calls on.
__device__ __forceinline__ void team_barrier(int team, int threads) { asm volatile("bar.sync %0, %1;" ::"r"(team + 1), "r"(threads) : "memory"); }
template <int K> __device__ __forceinline__ void team_sum(int warps, float* words, float (&v)[K]) {
  const int warp = threadIdx.x >> 5, first = warp & ~(warps - 1);
  if ((threadIdx.x & 31) == 0)
#pragma unroll
    for (int k = 0; k < K; ++k) words[warp * K + k] = v[k];
  team_barrier(first, warps * 32);
#pragma unroll
  for (int k = 0; k < K; ++k) {
    v[k] = 0.f;
    for (int w = 0; w < warps; ++w) v[k] += words[(first + w) * K + k];
  }
}
constexpr int GN_WARP_STAGES = 2;
__host__ __device__ constexpr int gn_warp_stage(int items, int cg) { return 512 * items + 8 * cg; }      // rows, FiLM vectors

template <typename T, int ITEMS, bool TEAM>
__global__ void __launch_bounds__(GN_WARP_THREADS, 3)
group_norm_warp_kernel(NormArgs g) {
  constexpr int V = 16 / sizeof(T), P = V / 2;
  extern __shared__ __align__(16) uint8_t gw_raw[];
  __shared__ float s_words[GN_WARP_THREADS / 32], s_words2[2 * GN_WARP_THREADS / 32];      // (of teams)
  const int gw = blockIdx.x * (GN_WARP_THREADS / 32) + (threadIdx.x >> 5), wl = threadIdx.x & 31;
  const int team = TEAM ? g.team : 1, part = TEAM ? gw & (team - 1) : 0, grp = gw / team % g.groups, split = gw / team / g.groups;      // this warp's part of its team's positions
  pdl_wait();
  if (split >= g.splits) return;
  const int cg = g.C / g.groups, gcols = cg / V, R = 32 / gcols;             // lanes on a position, positions at a time
  const int lr = wl / gcols, cc = (wl - lr * gcols) * V, c = grp * cg + cc, stage = gn_warp_stage(ITEMS, cg);
  const int l_first = part * ITEMS * R, rows = TEAM ? min(max(g.L - l_first, 0), ITEMS * R) : g.L;
  const uint8_t* mine = gw_raw + (threadIdx.x >> 5) * (GN_WARP_STAGES * stage);
  const uint32_t mine_a = ptx::smem_u32(mine);
  float2 ga[P], be[P];
#pragma unroll
  for (int i = 0; i < P; ++i) {
    ga[i] = *reinterpret_cast<const float2*>(g.gamma + c + 2 * i);
    be[i] = *reinterpret_cast<const float2*>(g.beta + c + 2 * i);
  }
  const float inv = 1.f / ((float)g.L * cg);
  auto fetch = [&](int n, int s) {
    if (n < g.N) {
      warp_rows(mine_a + s * stage, reinterpret_cast<const char*>(reinterpret_cast<const T*>(g.x.p) + n * g.x.sn + l_first * g.x.sl + grp * cg), g.x.sl * (long long)sizeof(T),
                cg * (int)sizeof(T), rows, wl);
      if (g.film) warp_rows(mine_a + s * stage + 512 * ITEMS, reinterpret_cast<const char*>(g.film + (long long)n * 2 * g.C + grp * cg), 4ll * g.C, 4 * cg, 2, wl);
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  zero_stages(mine_a, GN_WARP_STAGES * stage, wl);
  __syncwarp();
  fetch(split, 0);
  const bool full = rows == ITEMS * R;
  const long long y_step = R * g.y.sl, q_step = (long long)R * g.C, b_step = (long long)R * copy_blocks(g.C);
  int s = 0;
  for (int n = split; n < g.N; n += g.splits) {
    __syncwarp();                              // every lane is done with the stage that is filled next
    fetch(n + g.splits, s ^ 1);
    asm volatile("cp.async.wait_group 1;" ::: "memory");
    __syncwarp();
    const uint8_t* xs = mine + s * stage + (lr * cg + cc) * sizeof(T);
    const float* film = reinterpret_cast<const float*>(mine + s * stage + 512 * ITEMS) + cc;
    s ^= 1;
    const int x_step = R * cg * (int)sizeof(T);
    auto piece = [&](int j) { return *reinterpret_cast<const uint4*>(xs + j * x_step); };
    float2 t2 = two(0.f);
#pragma unroll
    for (int j = 0; j < ITEMS; ++j) {
      float2 v[P];
      unpack16<T, V>(piece(j), v);
#pragma unroll
      for (int i = 0; i < P; ++i) t2 = __fadd2_rn(t2, v[i]);
    }
    float sum[1] = {warp_sum(t2.x + t2.y)};
    if (TEAM) team_sum(team, s_words, sum);
    const float about = sum[0] * inv;          // the mean, but for the roundings of a sum of values; the sum of what lies about it gives their size
    float2 t1 = two(0.f);
    t2 = two(0.f);
    auto squares = [&](int j) {
      float2 v[P];
      unpack16<T, V>(piece(j), v);
#pragma unroll
      for (int i = 0; i < P; ++i) { v[i] = __fadd2_rn(v[i], two(-about)); t1 = __fadd2_rn(t1, v[i]); t2 = __ffma2_rn(v[i], v[i], t2); }
    };
    if (full) {
#pragma unroll
      for (int j = 0; j < ITEMS; ++j) squares(j);
    } else {
#pragma unroll
      for (int j = 0; j < ITEMS; ++j)
        if (lr + j * R < rows) squares(j);
    }
    float moments[2] = {warp_sum(t1.x + t1.y), warp_sum(t2.x + t2.y)};
    if (TEAM) team_sum(team, s_words2, moments);
    const float off = moments[0] * inv, square = moments[1] * inv, mean = mean_about(about, square, off);
    const float rstd = rsqrtf(variance_about(square, off) + g.eps);
    if (wl == 0 && part == 0) {
      if (g.mean) g.mean[(long long)n * g.groups + grp] = mean;
      if (g.rstd) g.rstd[(long long)n * g.groups + grp] = rstd;
    }
    T* y = reinterpret_cast<T*>(g.y.p) + n * g.y.sn + (l_first + lr) * g.y.sl + c;
    const long long r0 = (long long)n * g.L + l_first + lr;
    long long qo = r0 * g.C + c, bo = r0 * copy_blocks(g.C) + (c >> 5);
    float2 ka[P];                              // z = (x - mean) ka + beta
#pragma unroll
    for (int i = 0; i < P; ++i) ka[i] = __fmul2_rn(ga[i], two(rstd));
    with_act(g.act, [&](auto act) {
#pragma unroll 1                               // (one piece at a time: several do not fit the registers of three CTAs)
      for (int j = 0; j < ITEMS; ++j) {
        const bool row = lr + j * R < rows;
        const uint4 raw = piece(j);
        float2 v[P];
        unpack16<T, V>(raw, v);
#pragma unroll
        for (int i = 0; i < P; ++i) {
          float2 d;
          act_pair<false>(decltype(act)::value, __ffma2_rn(__fadd2_rn(v[i], two(-mean)), ka[i], be[i]), v[i], d);
        }
        if (g.film)
#pragma unroll
          for (int i = 0; i < P; ++i)
            v[i] = __ffma2_rn(v[i], *reinterpret_cast<const float2*>(film + 2 * i), *reinterpret_cast<const float2*>(film + cg + 2 * i));
        const uint4 out = pack16<T, V>(v);
        if (row) *reinterpret_cast<uint4*>(y) = out;
        if (g.cx.q) write_copy<T>(g.cx.q + qo, g.cx.b + bo, raw, row, (cc & 31) == 0);
        if (g.cy.q) write_copy<T>(g.cy.q + qo, g.cy.b + bo, out, row, (cc & 31) == 0);
        y += y_step; qo += q_step; bo += b_step;
      }
    });
  }
}

// Backward.  dz stays in registers between the sums and dx; dy and x (or its copy) come by cp.async into memory of the warp's own, one
// sequence ahead, and are read from there as often as they are needed: with them in registers too the kernel spills.  The steps of an
// 8-bit copy (L cg / 32 bytes) come one to a lane.
template <typename T, bool COPY> __host__ __device__ constexpr int gn_warp_grad_smem(int items) {
  return GN_WARP_THREADS * GN_STREAM_V * items * (int)(sizeof(T) + (COPY ? 1 : sizeof(T))) * GN_WARP_STAGES;
}

template <typename T, int ITEMS, bool COPY, bool TEAM>
__global__ void __launch_bounds__(GN_WARP_THREADS, 2)
group_norm_warp_grad_kernel(NormArgs g) {
  constexpr int V = GN_STREAM_V, P = V / 2;
  using X = std::conditional_t<COPY, signed char, T>;
  constexpr int DY_BYTES = 32 * V * ITEMS * sizeof(T), STAGE = DY_BYTES + 32 * V * ITEMS * sizeof(X);
  extern __shared__ __align__(16) uint8_t gw_raw[];
  __shared__ float s_words[TEAM ? 2 : 1][GN_WARP_THREADS / 32 * 2];
  const int gw = blockIdx.x * (GN_WARP_THREADS / 32) + (threadIdx.x >> 5), wl = threadIdx.x & 31;
  const int team = TEAM ? g.team : 1, part = TEAM ? gw & (team - 1) : 0, grp = gw / team % g.groups, split = gw / team / g.groups;
  pdl_trigger(true);                            // the join of the shares: its blocks wait beside this grid, which runs at once as a whole
  pdl_wait();
  if (split >= g.splits) return;
  const int cg = g.C / g.groups, gcols = cg / V, R = 32 / gcols, nb = copy_blocks(g.C), gb = cg / 32;
  const int lr = wl / gcols, cc = (wl - lr * gcols) * V, c = grp * cg + cc;
  const int l_first = part * ITEMS * R, rows = TEAM ? min(max(g.L - l_first, 0), ITEMS * R) : g.L;
  const uint8_t* mine = gw_raw + (threadIdx.x >> 5) * (GN_WARP_STAGES * STAGE);
  const uint32_t mine_a = ptx::smem_u32(mine);
  float* s_film = reinterpret_cast<float*>(gw_raw + GN_WARP_THREADS / 32 * GN_WARP_STAGES * STAGE);      // teams: [2 sequences][warps][2][cg]
  float2 ga[P], be[P], acc_z[P], acc_h[P];
#pragma unroll
  for (int i = 0; i < P; ++i) {
    ga[i] = *reinterpret_cast<const float2*>(g.gamma + c + 2 * i);
    be[i] = *reinterpret_cast<const float2*>(g.beta + c + 2 * i);
    acc_z[i] = acc_h[i] = two(0.f);
  }
  const float inv = 1.f / ((float)g.L * cg);
  const bool dfilm = g.dfilm != nullptr;
  uint32_t nstep = 0;
  float nmean = 0.f, nrstd = 0.f;
  float2 nfs[P];
#pragma unroll
  for (int i = 0; i < P; ++i) nfs[i] = two(1.f);
  auto fetch = [&](int n, int s) {
    if (n < g.N) {
      warp_rows(mine_a + s * STAGE, reinterpret_cast<const char*>(reinterpret_cast<const T*>(g.dy.p) + n * g.dy.sn + l_first * g.dy.sl + grp * cg), g.dy.sl * (long long)sizeof(T),
                cg * (int)sizeof(T), rows, wl);
      if (COPY) warp_rows(mine_a + s * STAGE + DY_BYTES, reinterpret_cast<const char*>(g.cx.q) + ((long long)n * g.L + l_first) * g.C + grp * cg, g.C, cg, rows, wl);
      else warp_rows(mine_a + s * STAGE + DY_BYTES, reinterpret_cast<const char*>(reinterpret_cast<const T*>(g.x.p) + n * g.x.sn + l_first * g.x.sl + grp * cg),
                     g.x.sl * (long long)sizeof(T), cg * (int)sizeof(T), rows, wl);
      nmean = g.mean[(long long)n * g.groups + grp];
      nrstd = g.rstd[(long long)n * g.groups + grp];
      if (COPY && wl < rows * gb) nstep = g.cx.b[((long long)n * g.L + l_first + wl / gb) * nb + grp * gb + wl % gb];
      if (g.film)
#pragma unroll
        for (int i = 0; i < P; ++i) nfs[i] = *reinterpret_cast<const float2*>(g.film + (long long)n * 2 * g.C + c + 2 * i);
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  zero_stages(mine_a, GN_WARP_STAGES * STAGE, wl);
  __syncwarp();
  fetch(split, 0);
  const long long dx_step = R * g.dx.sl;
  const int have = (rows - lr + R - 1) / R;     // of this lane
  int s = 0, odd = 0;
  for (int n = split; n < g.N; n += g.splits) {
    const float mean = nmean, rstd = nrstd, steps = COPY ? copy_step(nstep) : 1.f;
    float2 fs[P];
#pragma unroll
    for (int i = 0; i < P; ++i) fs[i] = nfs[i];
    __syncwarp();                              // every lane is done with the stage that is filled next
    fetch(n + g.splits, s ^ 1);
    asm volatile("cp.async.wait_group 1;" ::: "memory");
    __syncwarp();
    const uint8_t* dys = mine + s * STAGE + (lr * cg + cc) * sizeof(T);
    const uint8_t* xs = mine + s * STAGE + DY_BYTES + (lr * cg + cc) * sizeof(X);
    s ^= 1;
    float2 dz[ITEMS][P], s_z[P], s_h[P], s_a[P], s_y[P];
#pragma unroll
    for (int i = 0; i < P; ++i) s_z[i] = s_h[i] = s_a[i] = s_y[i] = two(0.f);
    // h = (x - mean) rstd, the difference first: x rstd - mean rstd rounds at the size of mean rstd, which has no limit but |mean| / sqrt(eps)
    // (a group of values of 1000: h = 0.002 instead of 0)
    float scale[COPY ? ITEMS : 1];
    if constexpr (COPY)
#pragma unroll
      for (int j = 0; j < ITEMS; ++j) scale[j] = __shfl_sync(0xffffffffu, steps, min((lr + j * R) * gb + (cc >> 5), 31));
    auto h_values = [&](int j, float2* h, float rs) {
      piece_values<X, V>(load_piece<X, V>(xs + j * R * cg * sizeof(X)), h);
#pragma unroll
      for (int i = 0; i < P; ++i) h[i] = __fmul2_rn(COPY ? __ffma2_rn(h[i], two(scale[COPY ? j : 0]), two(-mean)) : __fadd2_rn(h[i], two(-mean)), two(rs));
    };
    with_act(g.act, [&](auto act) {
#pragma unroll
      for (int j = 0; j < ITEMS; ++j) {
        float2 h[P], dy[P];
        h_values(j, h, j < have ? rstd : 0.f);      // (a row that is not there has a dy of zero, and must not have an h that is infinite)
        piece_values<T, V>(load_piece<T, V>(dys + j * R * cg * sizeof(T)), dy);
#pragma unroll
        for (int i = 0; i < P; ++i) {
          float2 a, d;
          act_pair<true>(decltype(act)::value, __ffma2_rn(h[i], ga[i], be[i]), a, d);
          if (dfilm) { s_a[i] = __ffma2_rn(dy[i], a, s_a[i]); s_y[i] = __fadd2_rn(s_y[i], dy[i]); }
          dz[j][i] = __fmul2_rn(__fmul2_rn(dy[i], fs[i]), d);
          s_z[i] = __fadd2_rn(s_z[i], dz[j][i]);
          s_h[i] = __ffma2_rn(dz[j][i], h[i], s_h[i]);
        }
      }
    });
    float m[2] = {0.f, 0.f};
#pragma unroll
    for (int i = 0; i < P; ++i) {
      acc_z[i] = __fadd2_rn(acc_z[i], s_z[i]);
      acc_h[i] = __fadd2_rn(acc_h[i], s_h[i]);
      const float2 p = __fmul2_rn(s_z[i], ga[i]), q = __fmul2_rn(s_h[i], ga[i]);
      m[0] += p.x + p.y; m[1] += q.x + q.y;
    }
    m[0] = warp_sum(m[0]);
    m[1] = warp_sum(m[1]);
    // dfilm: over the warp's positions; a team's first warp adds up what the others leave beside the words of the next sum
    auto film_sums = [&](float* o, int next) {
      for (int i = gcols; i < 32; i *= 2)
#pragma unroll
        for (int k = 0; k < P; ++k) {
          s_a[k].x += __shfl_xor_sync(0xffffffffu, s_a[k].x, i); s_a[k].y += __shfl_xor_sync(0xffffffffu, s_a[k].y, i);
          s_y[k].x += __shfl_xor_sync(0xffffffffu, s_y[k].x, i); s_y[k].y += __shfl_xor_sync(0xffffffffu, s_y[k].y, i);
        }
      if (lr == 0)
#pragma unroll
        for (int k = 0; k < P; ++k) { *reinterpret_cast<float2*>(o + 2 * k) = s_a[k]; *reinterpret_cast<float2*>(o + next + 2 * k) = s_y[k]; }
    };
    if (TEAM && dfilm) film_sums(s_film + (odd * (GN_WARP_THREADS / 32) + (threadIdx.x >> 5)) * 2 * cg + cc, cg);
    if (TEAM) team_sum(team, s_words[odd], m);
    if (TEAM && dfilm && part == 0)
      for (int i = wl; i < 2 * cg; i += 32) {
        const float* o = s_film + (odd * (GN_WARP_THREADS / 32) + (threadIdx.x >> 5)) * 2 * cg + i;
        float v = 0.f;
        for (int w = 0; w < team; ++w) v += o[w * 2 * cg];
        g.dfilm[((long long)n * 2 + i / cg) * g.C + grp * cg + i % cg] = v;
      }
    odd ^= 1;
    // dx = dz (gamma rstd) - m1 rstd - h (m2 rstd)
    const float m1 = -rstd * (m[0] * inv), m2 = -rstd * (m[1] * inv);
    T* dx = reinterpret_cast<T*>(g.dx.p) + n * g.dx.sn + (l_first + lr) * g.dx.sl + c;
    float2 ka[P];
#pragma unroll
    for (int i = 0; i < P; ++i) ka[i] = __fmul2_rn(ga[i], two(rstd));
#pragma unroll
    for (int j = 0; j < ITEMS; ++j) {
      float2 h[P];
      h_values(j, h, rstd);
#pragma unroll
      for (int i = 0; i < P; ++i) dz[j][i] = __ffma2_rn(dz[j][i], ka[i], __ffma2_rn(h[i], two(m2), two(m1)));
      if (j < have) {
        if constexpr (sizeof(T) == 2) *reinterpret_cast<uint2*>(dx) = make_uint2(pack_bf16(dz[j][0].x, dz[j][0].y), pack_bf16(dz[j][1].x, dz[j][1].y));
        else *reinterpret_cast<float4*>(dx) = make_float4(dz[j][0].x, dz[j][0].y, dz[j][1].x, dz[j][1].y);
      }
      dx += dx_step;
    }
    if (!TEAM && dfilm) film_sums(g.dfilm + (long long)n * 2 * g.C + c, g.C);
  }
  for (int o = gcols; o < 32; o *= 2)
#pragma unroll
    for (int i = 0; i < P; ++i) {
      acc_z[i].x += __shfl_xor_sync(0xffffffffu, acc_z[i].x, o); acc_z[i].y += __shfl_xor_sync(0xffffffffu, acc_z[i].y, o);
      acc_h[i].x += __shfl_xor_sync(0xffffffffu, acc_h[i].x, o); acc_h[i].y += __shfl_xor_sync(0xffffffffu, acc_h[i].y, o);
    }
  if (lr == 0) {
    float* o = g.part + ((long long)split * team + part) * 2 * g.C + c;
#pragma unroll
    for (int i = 0; i < P; ++i) { *reinterpret_cast<float2*>(o + 2 * i) = acc_z[i]; *reinterpret_cast<float2*>(o + g.C + 2 * i) = acc_h[i]; }
  }
}

}  // namespace tsdp
