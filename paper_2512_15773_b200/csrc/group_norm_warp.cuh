// The same operators with one warp per group: where a group of one sequence is at most 32 values a lane (backward in fp32: 16), as in every level of
// the UNet (512 values: 16 x 32, 8 x 64, 4 x 128).  All sums are shuffles: no barrier, no shared memory, and a warp that waits holds up no other.
// A warp keeps its group and walks the sequences; the rows of its next one are on their way while it works on this one.
// Lanes lie over the group's channels first (16 bytes each, backward four channels), then over positions.  Channels of a group: 32, 64, 128 or 256.
#pragma once
#include "group_norm_slab.cuh"

namespace tsdp {

constexpr int GN_WARP_THREADS = 256;

template <typename T, int ITEMS>
__global__ void __launch_bounds__(GN_WARP_THREADS, 2)
group_norm_warp_kernel(NormArgs g) {
  constexpr int V = 16 / sizeof(T), P = V / 2;
  const int gw = blockIdx.x * (GN_WARP_THREADS / 32) + (threadIdx.x >> 5), wl = threadIdx.x & 31;
  const int grp = gw % g.groups, split = gw / g.groups;
  pdl_wait();
  if (split >= g.splits) return;
  const int cg = g.C / g.groups, gcols = cg / V, R = 32 / gcols;             // lanes on a position, positions at a time
  const int lr = wl / gcols, c = grp * cg + (wl - lr * gcols) * V;
  float2 ga[P], be[P];
#pragma unroll
  for (int i = 0; i < P; ++i) {
    ga[i] = *reinterpret_cast<const float2*>(g.gamma + c + 2 * i);
    be[i] = *reinterpret_cast<const float2*>(g.beta + c + 2 * i);
  }
  const float inv = 1.f / ((float)g.L * cg);
  uint4 next[ITEMS];
  auto fetch = [&](int n) {
    const T* x = reinterpret_cast<const T*>(g.x.p) + n * g.x.sn + c;
#pragma unroll
    for (int j = 0; j < ITEMS; ++j) {
      const int l = lr + j * R;
      next[j] = make_uint4(0u, 0u, 0u, 0u);
      if (n < g.N && l < g.L) next[j] = *reinterpret_cast<const uint4*>(x + l * g.x.sl);
    }
  };
  fetch(split);
  for (int n = split; n < g.N; n += g.splits) {
    uint4 raw[ITEMS];
#pragma unroll
    for (int j = 0; j < ITEMS; ++j) raw[j] = next[j];
    float2 fs[P], fb[P];
#pragma unroll
    for (int i = 0; i < P; ++i) {
      fs[i] = two(1.f); fb[i] = two(0.f);
      if (g.film) {
        fs[i] = *reinterpret_cast<const float2*>(g.film + (long long)n * 2 * g.C + c + 2 * i);
        fb[i] = *reinterpret_cast<const float2*>(g.film + ((long long)n * 2 + 1) * g.C + c + 2 * i);
      }
    }
    fetch(n + g.splits);
    float2 t2 = two(0.f);
#pragma unroll
    for (int j = 0; j < ITEMS; ++j) {
      float2 v[P];
      unpack16<T, V>(raw[j], v);
#pragma unroll
      for (int i = 0; i < P; ++i) t2 = __fadd2_rn(t2, v[i]);       // (zeros where there is no row)
    }
    const float mean = warp_sum(t2.x + t2.y) * inv;
    t2 = two(0.f);
#pragma unroll
    for (int j = 0; j < ITEMS; ++j) {
      if (lr + j * R < g.L) {
        float2 v[P];
        unpack16<T, V>(raw[j], v);
#pragma unroll
        for (int i = 0; i < P; ++i) { v[i] = __fadd2_rn(v[i], two(-mean)); t2 = __ffma2_rn(v[i], v[i], t2); }
      }
    }
    const float rstd = rsqrtf(warp_sum(t2.x + t2.y) * inv + g.eps);
    if (wl == 0) {
      if (g.mean) g.mean[(long long)n * g.groups + grp] = mean;
      if (g.rstd) g.rstd[(long long)n * g.groups + grp] = rstd;
    }
    T* y0 = reinterpret_cast<T*>(g.y.p) + n * g.y.sn + c;
    with_act(g.act, [&](auto act) {
#pragma unroll
      for (int j = 0; j < ITEMS; ++j) {
        const int l = lr + j * R;
        const bool row = l < g.L;
        float2 v[P], y[P];
        unpack16<T, V>(raw[j], v);
#pragma unroll
        for (int i = 0; i < P; ++i) {
          const float2 z = __ffma2_rn(__fmul2_rn(__fadd2_rn(v[i], two(-mean)), two(rstd)), ga[i], be[i]);
          float2 a, d;
          act_pair<false>(decltype(act)::value, z, a, d);
          y[i] = __ffma2_rn(a, fs[i], fb[i]);
        }
        const uint4 out = pack16<T, V>(y);
        if (row) *reinterpret_cast<uint4*>(y0 + l * g.y.sl) = out;
        const long long r = (long long)n * g.L + l;
        if (g.cx.q) write_copy<T>(g.cx, raw[j], row, r, g.C, c);
        if (g.cy.q) write_copy<T>(g.cy, out, row, r, g.C, c);
      }
    });
  }
}

// Backward.  dz stays in registers between the sums and dx; dy and x (or its copy) come by cp.async into memory of the warp's own, one
// sequence ahead, and are read from there as often as they are needed: with them in registers too the kernel spills.  The steps of an
// 8-bit copy (L cg / 32 bytes) come one to a lane.
__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
// `rows` rows of `bytes` bytes (a power of two, 16 at least), `pitch` apart, packed to dst by the lanes of a warp.
__device__ __forceinline__ void warp_rows(uint32_t dst, const char* src, long long pitch, int bytes, int rows, int wl) {
  const int shift = 31 - __clz(bytes);
  for (int o = wl * 16; o < rows * bytes; o += 512) cp_async16(dst + o, src + (o >> shift) * pitch + (o & (bytes - 1)));
}
constexpr int GN_WARP_STAGES = 2;
template <typename T, bool COPY> __host__ __device__ constexpr int gn_warp_grad_smem(int items) {
  return GN_WARP_THREADS * GN_GRAD_V * items * (int)(sizeof(T) + (COPY ? 1 : sizeof(T))) * GN_WARP_STAGES;
}

template <typename T, int ITEMS, bool COPY>
__global__ void __launch_bounds__(GN_WARP_THREADS, 2)
group_norm_warp_grad_kernel(NormArgs g) {
  constexpr int V = GN_GRAD_V, P = V / 2;
  using X = std::conditional_t<COPY, signed char, T>;
  constexpr int DY_BYTES = 32 * V * ITEMS * sizeof(T), STAGE = DY_BYTES + 32 * V * ITEMS * sizeof(X);
  extern __shared__ __align__(16) uint8_t gw_raw[];
  const int gw = blockIdx.x * (GN_WARP_THREADS / 32) + (threadIdx.x >> 5), wl = threadIdx.x & 31;
  const int grp = gw % g.groups, split = gw / g.groups;
  pdl_trigger(true);                            // the join of the shares: its blocks wait beside this grid, which runs at once as a whole
  pdl_wait();
  if (split >= g.splits) return;
  const int cg = g.C / g.groups, gcols = cg / V, R = 32 / gcols, nb = copy_blocks(g.C), gb = cg / 32;
  const int lr = wl / gcols, cc = (wl - lr * gcols) * V, c = grp * cg + cc;
  const uint8_t* mine = gw_raw + (threadIdx.x >> 5) * (GN_WARP_STAGES * STAGE);
  const uint32_t mine_a = ptx::smem_u32(mine);
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
      warp_rows(mine_a + s * STAGE, reinterpret_cast<const char*>(reinterpret_cast<const T*>(g.dy.p) + n * g.dy.sn + grp * cg), g.dy.sl * (long long)sizeof(T),
                cg * (int)sizeof(T), g.L, wl);
      if (COPY) warp_rows(mine_a + s * STAGE + DY_BYTES, reinterpret_cast<const char*>(g.cx.q) + (long long)n * g.L * g.C + grp * cg, g.C, cg, g.L, wl);
      else warp_rows(mine_a + s * STAGE + DY_BYTES, reinterpret_cast<const char*>(reinterpret_cast<const T*>(g.x.p) + n * g.x.sn + grp * cg),
                     g.x.sl * (long long)sizeof(T), cg * (int)sizeof(T), g.L, wl);
      nmean = g.mean[(long long)n * g.groups + grp];
      nrstd = g.rstd[(long long)n * g.groups + grp];
      if (COPY && wl < g.L * gb) nstep = g.cx.b[((long long)n * g.L + wl / gb) * nb + grp * gb + wl % gb];
      if (g.film)
#pragma unroll
        for (int i = 0; i < P; ++i) nfs[i] = *reinterpret_cast<const float2*>(g.film + (long long)n * 2 * g.C + c + 2 * i);
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  fetch(split, 0);
  int s = 0;
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
    auto h_values = [&](int j, float2* h) {              // (rows past the last: whatever the stage holds, not used)
      piece_values<X, V>(load_piece<X, V>(xs + j * R * cg * sizeof(X)), h);
      if constexpr (COPY) {
        const float st = __shfl_sync(0xffffffffu, steps, min((lr + j * R) * gb + (cc >> 5), 31));
#pragma unroll
        for (int i = 0; i < P; ++i) h[i] = __fmul2_rn(h[i], two(st));
      }
#pragma unroll
      for (int i = 0; i < P; ++i) h[i] = __fmul2_rn(__fadd2_rn(h[i], two(-mean)), two(rstd));
    };
    with_act(g.act, [&](auto act) {
#pragma unroll
      for (int j = 0; j < ITEMS; ++j) {
        float2 h[P], dy[P];
        h_values(j, h);
        if (lr + j * R < g.L) {
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
      }
    });
    float m1 = 0.f, m2 = 0.f;
#pragma unroll
    for (int i = 0; i < P; ++i) {
      acc_z[i] = __fadd2_rn(acc_z[i], s_z[i]);
      acc_h[i] = __fadd2_rn(acc_h[i], s_h[i]);
      const float2 p = __fmul2_rn(s_z[i], ga[i]), q = __fmul2_rn(s_h[i], ga[i]);
      m1 += p.x + p.y; m2 += q.x + q.y;
    }
    m1 = warp_sum(m1) * inv;
    m2 = warp_sum(m2) * inv;
    T* dx0 = reinterpret_cast<T*>(g.dx.p) + n * g.dx.sn + c;
#pragma unroll
    for (int j = 0; j < ITEMS; ++j) {
      const int l = lr + j * R;
      float2 h[P];
      h_values(j, h);
      if (l >= g.L) continue;
#pragma unroll
      for (int i = 0; i < P; ++i)
        dz[j][i] = __fmul2_rn(two(rstd), __ffma2_rn(h[i], two(-m2), __fadd2_rn(__fmul2_rn(dz[j][i], ga[i]), two(-m1))));
      T* dx = dx0 + l * g.dx.sl;
      if constexpr (sizeof(T) == 2) *reinterpret_cast<uint2*>(dx) = make_uint2(pack_bf16(dz[j][0].x, dz[j][0].y), pack_bf16(dz[j][1].x, dz[j][1].y));
      else *reinterpret_cast<float4*>(dx) = make_float4(dz[j][0].x, dz[j][0].y, dz[j][1].x, dz[j][1].y);
    }
    if (dfilm) {
      for (int o = gcols; o < 32; o *= 2)
#pragma unroll
        for (int i = 0; i < P; ++i) {
          s_a[i].x += __shfl_xor_sync(0xffffffffu, s_a[i].x, o); s_a[i].y += __shfl_xor_sync(0xffffffffu, s_a[i].y, o);
          s_y[i].x += __shfl_xor_sync(0xffffffffu, s_y[i].x, o); s_y[i].y += __shfl_xor_sync(0xffffffffu, s_y[i].y, o);
        }
      if (lr == 0) {
        float* o = g.dfilm + (long long)n * 2 * g.C + c;
#pragma unroll
        for (int i = 0; i < P; ++i) { *reinterpret_cast<float2*>(o + 2 * i) = s_a[i]; *reinterpret_cast<float2*>(o + g.C + 2 * i) = s_y[i]; }
      }
    }
  }
  for (int o = gcols; o < 32; o *= 2)
#pragma unroll
    for (int i = 0; i < P; ++i) {
      acc_z[i].x += __shfl_xor_sync(0xffffffffu, acc_z[i].x, o); acc_z[i].y += __shfl_xor_sync(0xffffffffu, acc_z[i].y, o);
      acc_h[i].x += __shfl_xor_sync(0xffffffffu, acc_h[i].x, o); acc_h[i].y += __shfl_xor_sync(0xffffffffu, acc_h[i].y, o);
    }
  if (lr == 0) {
    float* o = g.part + (long long)split * 2 * g.C + c;
#pragma unroll
    for (int i = 0; i < P; ++i) { *reinterpret_cast<float2*>(o + 2 * i) = acc_z[i]; *reinterpret_cast<float2*>(o + g.C + 2 * i) = acc_h[i]; }
  }
}

}  // namespace tsdp
