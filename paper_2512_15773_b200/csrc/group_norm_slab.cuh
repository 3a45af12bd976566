// The same operators where a CTA can hold what it normalises: some groups of one sequence, up to 4 pieces of 16 bytes in each of 256
// threads, and a warp or a team of warps cannot (groups of 8 or 16, of 80 or 320, of 512 channels).  Every byte passes once: x (and dy) come by bulk copies into a ring in shared
// memory, one or two sequences ahead, go to registers, give their statistics there and leave as results.  A CTA walks over the sequences
// (split, split + splits, ...), so that affine vectors, the shares of dgamma and dbeta and the ring stay.
// Statistics are taken in two steps in registers (mean, then what lies about it and its squares, which also correct the mean); sums over a group pass by shuffles as far as lanes of a
// warp share it, then through a few words of shared memory: one barrier per sum.
// What bounds it: two barriers a sequence and the sums around them.  2048 x 12 x 640 in two groups, Mish, FiLM, fp32: 52 us (2.5 TB/s; the stream form
// 104); backward in bf16 69 us (124).  In 80 registers <bf16, 4> and the gradients with four pieces a thread spill 60 to 130 bytes.
#pragma once
#include "group_norm_kernels.cuh"

namespace tsdp {

constexpr int GN_RING = 2;
constexpr int GN_SLAB_CTAS = 3;                // on an SM

__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
               ::"r"(dst), "l"(src), "r"(bytes), "r"(bar) : "memory");
}
// L rows of `bytes` bytes, `pitch` bytes apart, packed to dst; issued by the 32 lanes of a warp.
__device__ __forceinline__ void bulk_rows(uint32_t dst, const char* src, long long pitch, uint32_t bytes, int L, uint32_t bar, int lane) {
  if (pitch == (long long)bytes) {
    if (lane == 0) bulk_load(dst, src, bytes * L, bar);
  } else {
    for (int l = lane; l < L; l += 32) bulk_load(dst + l * bytes, src + l * pitch, bytes, bar);
  }
}
// 16 bytes of shared memory as V values.
template <typename T, int V> __device__ __forceinline__ void unpack16(uint4 u, float2* v) {
  if constexpr (sizeof(T) == 2) {
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = make_float2(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xffff0000u));
  } else {
    v[0] = make_float2(__uint_as_float(u.x), __uint_as_float(u.y));
    v[1] = make_float2(__uint_as_float(u.z), __uint_as_float(u.w));
  }
}
// The 8-bit copy of 16 bytes of a row; the lanes of a block of 32 sit side by side in a warp, all of them with the row or none.
// q: where its bytes go, b: where the block's byte goes (by its first lane).
template <typename T> __device__ __forceinline__ void write_copy(signed char* q, unsigned char* b, uint4 u, bool row, bool first) {
  constexpr int V = 16 / sizeof(T);
  uint32_t top;
  if constexpr (V == 8) top = copy_top_bf16<4>(u);
  else {
    top = copy_top_fp32(u);
#pragma unroll
    for (int i = 1; i < 8; i *= 2) top = max(top, __shfl_xor_sync(0xffffffffu, top, i));
  }
  const uint32_t byte = copy_byte(top);
  const float is = copy_inv_step(byte);
  float2 w[V / 2];
  unpack16<T, V>(u, w);
  if (row) {
    if constexpr (V == 8) *reinterpret_cast<uint2*>(q) = copy_q8(w, is, byte);
    else *reinterpret_cast<uint32_t*>(q) = copy_q4(w[0], w[1], is, byte);
    if (first) *b = (unsigned char)byte;
  }
}
template <typename T, int V> __device__ __forceinline__ uint4 pack16(const float2* y) {
  if constexpr (sizeof(T) == 2) return make_uint4(pack_bf16(y[0].x, y[0].y), pack_bf16(y[1].x, y[1].y), pack_bf16(y[2].x, y[2].y), pack_bf16(y[3].x, y[3].y));
  else return make_uint4(__float_as_uint(y[0].x), __float_as_uint(y[0].y), __float_as_uint(y[1].x), __float_as_uint(y[1].y));
}
// The parts of a row of s_red that make up the sum of a column's group: none for a thread without a column (cols is rounded up to whole blocks of
// 32 channels, and threads may be left over behind the last row), which lies in no group.
struct GroupParts { int first, count; };
__host__ __device__ __forceinline__ GroupParts group_parts(const NormArgs& g, int gcols, int col, bool in) {
  const int parts = gcols / g.fold;
  return GroupParts{col / gcols * parts, in ? parts : 0};
}
// Sum over the threads of a group: within a warp by shuffles, the rest through s_red.  One barrier.  Zero for a thread without a column.
template <int K>
__device__ __forceinline__ void group_sum(const NormArgs& g, int gcols, int col, int row, bool in, float* s_red, float (&v)[K]) {
  const int wl = threadIdx.x & 31, per = g.cols / g.fold;
  for (int o = 1; o < g.fold; o *= 2)
#pragma unroll
    for (int k = 0; k < K; ++k) v[k] += __shfl_xor_sync(0xffffffffu, v[k], o);
  const bool rows_in_warp = g.cols < 32 && (g.cols & (g.cols - 1)) == 0;
  if (rows_in_warp)
    for (int o = g.cols; o < 32; o *= 2)
#pragma unroll
      for (int k = 0; k < K; ++k) v[k] += __shfl_xor_sync(0xffffffffu, v[k], o);
  const int r = rows_in_warp ? (int)(threadIdx.x >> 5) : row;
  if (col % g.fold == 0 && (rows_in_warp ? wl < g.cols : row < g.lanes))
#pragma unroll
    for (int k = 0; k < K; ++k) s_red[(r * per + col / g.fold) * K + k] = v[k];
  __syncthreads();
  const GroupParts mine = group_parts(g, gcols, col, in);
#pragma unroll
  for (int k = 0; k < K; ++k) v[k] = 0.f;
  for (int i = 0; i < g.red_rows; ++i)
    for (int j = 0; j < mine.count; ++j)
#pragma unroll
      for (int k = 0; k < K; ++k) v[k] += s_red[(i * per + mine.first + j) * K + k];
}

// Waits are bounded.  A thread whose wait ran out waits no more and takes NaN for what it did not get, which its group's sums carry to all of the
// group; the CTA asks for no further rows (lost, set before the barrier of a sum) and stays until copies that may still be in flight have landed.
__device__ __forceinline__ bool slab_wait(uint32_t bar, uint32_t ph, long long limit, int& lost) {
  const bool ok = ptx::mbar_wait_thread(bar, ph, limit);
  if (!ok) lost = 1;
  return ok;
}
__device__ __forceinline__ bool slab_more(const int& lost) { return __all_sync(0xffffffffu, *(const volatile int*)&lost == 0) != 0; }
__device__ __forceinline__ void slab_drain(const int& lost) {      // by all threads
  __syncthreads();
  if (lost) {
    const long long t0 = clock64();
    while (clock64() - t0 < 400000ll) { }
  }
}

template <typename T, int ITEMS>
__global__ void __launch_bounds__(GN_THREADS, GN_SLAB_CTAS)
group_norm_slab_kernel(NormArgs g) {
  constexpr int V = 16 / sizeof(T), P = V / 2;
  extern __shared__ __align__(16) uint8_t gs_raw[];
  __shared__ float s_red[GN_THREADS], s_red2[2 * GN_THREADS];
  __shared__ __align__(8) unsigned long long s_bar[GN_RING];
  __shared__ int s_lost;
  const int cg = g.C / g.groups, gcols = cg / V;
  const int set = blockIdx.x % g.sets, split = blockIdx.x / g.sets;
  const int c_set = set * g.width, width = min(g.width, g.C - c_set);
  const int lane = threadIdx.x / g.cols, col = threadIdx.x - lane * g.cols, c = c_set + col * V;
  const bool in = lane < g.lanes && col * V < width;
  const int wl = threadIdx.x & 31;
  const uint32_t row_bytes = width * sizeof(T), base = ptx::smem_u32(gs_raw);
  const uint32_t film_off = (uint32_t)g.L * g.width * sizeof(T);
  const uint32_t tx = row_bytes * g.L + (g.film ? 8u * width : 0u);
  auto issue = [&](int n, int s) {             // by warp 0
    const uint32_t bar = ptx::smem_u32(&s_bar[s]), dst = base + s * g.stage_bytes;
    if (wl == 0) ptx::mbar_expect_tx(bar, tx);
    __syncwarp();
    bulk_rows(dst, reinterpret_cast<const char*>(g.x.p) + (n * g.x.sn + c_set) * (long long)sizeof(T), g.x.sl * (long long)sizeof(T), row_bytes, g.L, bar, wl);
    if (g.film && wl < 2) bulk_load(dst + film_off + wl * 4u * g.width, g.film + ((long long)n * 2 + wl) * g.C + c_set, 4u * width, bar);
  };
  if (threadIdx.x == 0) {
    s_lost = 0;
    for (int s = 0; s < GN_RING; ++s) ptx::mbar_init(ptx::smem_u32(&s_bar[s]), 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  __syncthreads();
  pdl_wait();
  if (threadIdx.x < 32 && !(g.withhold && blockIdx.x == 0))
    for (int s = 0; s < GN_RING; ++s)
      if (split + s * g.splits < g.N) issue(split + s * g.splits, s);
  float2 ga[P], be[P];
#pragma unroll
  for (int i = 0; i < P; ++i) {
    ga[i] = in ? *reinterpret_cast<const float2*>(g.gamma + c + 2 * i) : two(0.f);
    be[i] = in ? *reinterpret_cast<const float2*>(g.beta + c + 2 * i) : two(0.f);
  }
  const float inv = 1.f / ((float)g.L * cg);
  int s = 0;
  uint32_t ph = 0;
  bool ok = true;
  for (int n = split; n < g.N; n += g.splits) {
    ok = ok && slab_wait(ptx::smem_u32(&s_bar[s]), ph, g.wait_cycles, s_lost);
    const uint8_t* stage = gs_raw + s * g.stage_bytes;
    uint4 raw[ITEMS];
    float2 fs[P], fb[P];
#pragma unroll
    for (int j = 0; j < ITEMS; ++j) {
      const int l = lane + j * g.lanes;
      raw[j] = make_uint4(0u, 0u, 0u, 0u);
      if (in && l < g.L) raw[j] = *reinterpret_cast<const uint4*>(stage + l * row_bytes + col * 16);
      if (!ok) raw[j] = make_uint4(0x7fc07fc0u, 0x7fc07fc0u, 0x7fc07fc0u, 0x7fc07fc0u);      // a wait that ran out: NaN
    }
#pragma unroll
    for (int i = 0; i < P; ++i) {
      fs[i] = two(1.f); fb[i] = two(0.f);
      if (g.film && in) {
        fs[i] = *reinterpret_cast<const float2*>(stage + film_off + (col * V + 2 * i) * 4);
        fb[i] = *reinterpret_cast<const float2*>(stage + film_off + 4 * g.width + (col * V + 2 * i) * 4);
      }
    }
    float2 t2 = two(0.f);
#pragma unroll
    for (int j = 0; j < ITEMS; ++j) {
      float2 v[P];
      unpack16<T, V>(raw[j], v);
#pragma unroll
      for (int i = 0; i < P; ++i) t2 = __fadd2_rn(t2, v[i]);       // (zeros where there is no row)
    }
    float sum[1] = {t2.x + t2.y};
    group_sum<1>(g, gcols, col, lane, in, s_red, sum);
    // every thread has taken its share of the stage
    if (threadIdx.x < 32 && n + GN_RING * g.splits < g.N && slab_more(s_lost)) issue(n + GN_RING * g.splits, s);
    if (++s == GN_RING) { s = 0; ph ^= 1; }
    const float about = sum[0] * inv;          // the mean, but for the roundings of a sum of values; the sum of what lies about it gives their size
    float2 t1 = two(0.f);
    t2 = two(0.f);
#pragma unroll
    for (int j = 0; j < ITEMS; ++j) {
      if (lane + j * g.lanes < g.L) {
        float2 v[P];
        unpack16<T, V>(raw[j], v);
#pragma unroll
        for (int i = 0; i < P; ++i) { v[i] = __fadd2_rn(v[i], two(-about)); t1 = __fadd2_rn(t1, v[i]); t2 = __ffma2_rn(v[i], v[i], t2); }
      }
    }
    float moments[2] = {in ? t1.x + t1.y : 0.f, in ? t2.x + t2.y : 0.f};
    group_sum<2>(g, gcols, col, lane, in, s_red2, moments);
    const float off = moments[0] * inv, square = moments[1] * inv, mean = mean_about(about, square, off);
    const float rstd = rsqrtf(variance_about(square, off) + g.eps);
    if (in && lane == 0 && col % gcols == 0) {
      const long long at = (long long)n * g.groups + c / cg;
      if (g.mean) g.mean[at] = mean;
      if (g.rstd) g.rstd[at] = rstd;
    }
    with_act(g.act, [&](auto act) {
#pragma unroll
      for (int j = 0; j < ITEMS; ++j) {
        const int l = lane + j * g.lanes;
        const bool row = in && l < g.L;
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
        if (row) *reinterpret_cast<uint4*>(reinterpret_cast<T*>(g.y.p) + n * g.y.sn + l * g.y.sl + c) = out;
        const long long r = (long long)n * g.L + l;
        const long long qo = r * g.C + c, bo = r * copy_blocks(g.C) + (c >> 5);
        if (g.cx.q) write_copy<T>(g.cx.q + qo, g.cx.b + bo, raw[j], row, (c & 31) == 0);
        if (g.cy.q) write_copy<T>(g.cy.q + qo, g.cy.b + bo, row ? out : make_uint4(0u, 0u, 0u, 0u), row, (c & 31) == 0);
      }
    });
  }
  slab_drain(s_lost);
}

// Backward.  dz stays in registers between the sums and dx; h is taken from x again.  A thread owns four channels: with eight, the sums of
// dz, dz h, dy a and dy and the shares of dgamma and dbeta do not fit the registers of three CTAs.
template <typename T, int ITEMS, bool COPY>
__global__ void __launch_bounds__(GN_THREADS, GN_SLAB_CTAS)
group_norm_slab_grad_kernel(NormArgs g) {
  constexpr int V = GN_STREAM_V, P = V / 2;
  using X = std::conditional_t<COPY, signed char, T>;
  extern __shared__ __align__(16) uint8_t gs_raw[];
  __shared__ float s_red[2][2 * GN_THREADS];
  __shared__ __align__(8) unsigned long long s_bar[GN_RING];
  __shared__ int s_lost;
  const int cg = g.C / g.groups, gcols = cg / V;
  const int set = blockIdx.x % g.sets, split = blockIdx.x / g.sets;
  const int c_set = set * g.width, width = min(g.width, g.C - c_set);
  const int lane = threadIdx.x / g.cols, col = threadIdx.x - lane * g.cols, c = c_set + col * V;
  const bool in = lane < g.lanes && col * V < width;
  const int wl = threadIdx.x & 31;
  const uint32_t base = ptx::smem_u32(gs_raw);
  const uint32_t row_bytes = width * sizeof(T), x_bytes = COPY ? width : row_bytes;
  const uint32_t x_off = (uint32_t)g.L * g.width * sizeof(T), film_off = x_off + (uint32_t)g.L * g.width * (COPY ? 1u : (uint32_t)sizeof(T));
  const uint32_t tx = (row_bytes + x_bytes) * g.L + (g.film ? 4u * width : 0u);
  float* s_film = reinterpret_cast<float*>(gs_raw + GN_RING * g.stage_bytes);         // [2 sequences][2][lanes][width]
  const bool dfilm = g.dfilm != nullptr;
  auto issue = [&](int n, int s) {
    const uint32_t bar = ptx::smem_u32(&s_bar[s]), dst = base + s * g.stage_bytes;
    if (wl == 0) ptx::mbar_expect_tx(bar, tx);
    __syncwarp();
    bulk_rows(dst, reinterpret_cast<const char*>(g.dy.p) + (n * g.dy.sn + c_set) * (long long)sizeof(T), g.dy.sl * (long long)sizeof(T), row_bytes, g.L, bar, wl);
    if (COPY) bulk_rows(dst + x_off, reinterpret_cast<const char*>(g.cx.q) + (long long)n * g.L * g.C + c_set, g.C, x_bytes, g.L, bar, wl);
    else bulk_rows(dst + x_off, reinterpret_cast<const char*>(g.x.p) + (n * g.x.sn + c_set) * (long long)sizeof(T), g.x.sl * (long long)sizeof(T), x_bytes, g.L, bar, wl);
    if (g.film && wl == 0) bulk_load(dst + film_off, g.film + (long long)n * 2 * g.C + c_set, 4u * width, bar);
  };
  if (threadIdx.x == 0) {
    s_lost = 0;
    for (int s = 0; s < GN_RING; ++s) ptx::mbar_init(ptx::smem_u32(&s_bar[s]), 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  __syncthreads();
  pdl_wait();
  if (threadIdx.x < 32 && !(g.withhold && blockIdx.x == 0))
    for (int s = 0; s < GN_RING; ++s)
      if (split + s * g.splits < g.N) issue(split + s * g.splits, s);
  float2 ga[P], be[P], acc_z[P], acc_h[P];
#pragma unroll
  for (int i = 0; i < P; ++i) {
    ga[i] = in ? *reinterpret_cast<const float2*>(g.gamma + c + 2 * i) : two(0.f);
    be[i] = in ? *reinterpret_cast<const float2*>(g.beta + c + 2 * i) : two(0.f);
    acc_z[i] = acc_h[i] = two(0.f);
  }
  const float inv = 1.f / ((float)g.L * cg);
  const long long nb = copy_blocks(g.C);
  // what does not come through the ring is asked for one sequence ahead: the steps of the 8-bit copy, the statistics
  uint32_t sb[ITEMS];
  float mu_next = 0.f, rs_next = 0.f;
  auto ahead = [&](int n) {
    if (!in || n >= g.N) return;
    mu_next = g.mean[(long long)n * g.groups + c / cg];
    rs_next = g.rstd[(long long)n * g.groups + c / cg];
    if constexpr (COPY) {
#pragma unroll
      for (int j = 0; j < ITEMS; ++j) {
        const int l = lane + j * g.lanes;
        sb[j] = l < g.L ? g.cx.b[((long long)n * g.L + l) * nb + (c >> 5)] : 0u;
      }
    }
  };
  ahead(split);
  int s = 0, odd = 0;
  uint32_t ph = 0;
  bool ok = true;
  for (int n = split; n < g.N; n += g.splits) {
    const float mean = mu_next, rstd = rs_next;
    uint32_t step[ITEMS];
#pragma unroll
    for (int j = 0; j < ITEMS; ++j) step[j] = COPY ? sb[j] : 0u;
    ahead(n + g.splits);
    ok = ok && slab_wait(ptx::smem_u32(&s_bar[s]), ph, g.wait_cycles, s_lost);
    const uint8_t* stage = gs_raw + s * g.stage_bytes;
    float2 fs[P];
#pragma unroll
    for (int i = 0; i < P; ++i) fs[i] = g.film && in ? *reinterpret_cast<const float2*>(stage + film_off + (col * V + 2 * i) * 4) : two(1.f);
    Piece<X, V> xr[ITEMS];
    float2 dz[ITEMS][P], s_z[P], s_h[P], s_a[P], s_y[P];
#pragma unroll
    for (int i = 0; i < P; ++i) s_z[i] = s_h[i] = s_a[i] = s_y[i] = two(0.f);
    auto x_values = [&](int j, float2* h) {           // h of item j
      piece_values<X, V>(xr[j], h);
      if constexpr (COPY)
#pragma unroll
        for (int i = 0; i < P; ++i) h[i] = __fmul2_rn(h[i], two(copy_step(step[j])));
#pragma unroll
      for (int i = 0; i < P; ++i) h[i] = __fmul2_rn(__fadd2_rn(h[i], two(-mean)), two(rstd));
    };
    with_act(g.act, [&](auto act) {
#pragma unroll
    for (int j = 0; j < ITEMS; ++j) {
      const int l = lane + j * g.lanes;
      const bool row = in && l < g.L;
      Piece<T, V> dyr{};
      xr[j] = Piece<X, V>{};
      if (row) {
        dyr = load_piece<T, V>(stage + l * row_bytes + col * V * (int)sizeof(T));
        xr[j] = load_piece<X, V>(stage + x_off + l * x_bytes + col * V * (int)sizeof(X));
      }
      if (!ok)                                     // a wait that ran out: NaN
#pragma unroll
        for (int i = 0; i < (int)(sizeof(dyr) / 4); ++i) dyr.w[i] = 0x7fc07fc0u;
      float2 h[P], dy[P];
      x_values(j, h);
      piece_values<T, V>(dyr, dy);
      if (l < g.L) {
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
    float m[2] = {0.f, 0.f};
#pragma unroll
    for (int i = 0; i < P; ++i) {
      acc_z[i] = __fadd2_rn(acc_z[i], s_z[i]);
      acc_h[i] = __fadd2_rn(acc_h[i], s_h[i]);
      const float2 p = __fmul2_rn(s_z[i], ga[i]), q = __fmul2_rn(s_h[i], ga[i]);
      m[0] += p.x + p.y; m[1] += q.x + q.y;
    }
    if (!in) m[0] = m[1] = 0.f;
    float* film = s_film + odd * 2 * g.lanes * g.width;
    if (dfilm && in)
#pragma unroll
      for (int i = 0; i < P; ++i) {
        *reinterpret_cast<float2*>(film + lane * g.width + col * V + 2 * i) = s_a[i];
        *reinterpret_cast<float2*>(film + (g.lanes + lane) * g.width + col * V + 2 * i) = s_y[i];
      }
    group_sum<2>(g, gcols, col, lane, in, s_red[odd], m);
    if (threadIdx.x < 32 && n + GN_RING * g.splits < g.N && slab_more(s_lost)) issue(n + GN_RING * g.splits, s);
    if (++s == GN_RING) { s = 0; ph ^= 1; }
    odd ^= 1;
    const float m1 = m[0] * inv, m2 = m[1] * inv;
#pragma unroll
    for (int j = 0; j < ITEMS; ++j) {
      const int l = lane + j * g.lanes;
      if (!(in && l < g.L)) continue;
      float2 h[P];
      x_values(j, h);
#pragma unroll
      for (int i = 0; i < P; ++i)
        dz[j][i] = __fmul2_rn(two(rstd), __ffma2_rn(h[i], two(-m2), __fadd2_rn(__fmul2_rn(dz[j][i], ga[i]), two(-m1))));
      T* dx = reinterpret_cast<T*>(g.dx.p) + n * g.dx.sn + l * g.dx.sl + c;
      if constexpr (sizeof(T) == 2) *reinterpret_cast<uint2*>(dx) = make_uint2(pack_bf16(dz[j][0].x, dz[j][0].y), pack_bf16(dz[j][1].x, dz[j][1].y));
      else *reinterpret_cast<float4*>(dx) = make_float4(dz[j][0].x, dz[j][0].y, dz[j][1].x, dz[j][1].y);
    }
    if (dfilm)
      for (int i = threadIdx.x; i < 2 * width; i += GN_THREADS) {
        const int k = i / width, cc = i - k * width;
        float v = 0.f;
        for (int r = 0; r < g.lanes; ++r) v += film[(k * g.lanes + r) * g.width + cc];
        g.dfilm[((long long)n * 2 + k) * g.C + c_set + cc] = v;
      }
  }
  // shares of dbeta and dgamma: over the lanes, through the memory of the ring
  slab_drain(s_lost);
  float* s_acc = reinterpret_cast<float*>(gs_raw);          // [2][lanes][width]
  if (in)
#pragma unroll
    for (int i = 0; i < P; ++i) {
      *reinterpret_cast<float2*>(s_acc + lane * g.width + col * V + 2 * i) = acc_z[i];
      *reinterpret_cast<float2*>(s_acc + (g.lanes + lane) * g.width + col * V + 2 * i) = acc_h[i];
    }
  __syncthreads();
  for (int i = threadIdx.x; i < 2 * width; i += GN_THREADS) {
    const int k = i / width, cc = i - k * width;
    float v = 0.f;
    for (int r = 0; r < g.lanes; ++r) v += s_acc[(k * g.lanes + r) * g.width + cc];
    g.part[((long long)split * 2 + k) * g.C + c_set + cc] = v;
  }
}

}  // namespace tsdp
