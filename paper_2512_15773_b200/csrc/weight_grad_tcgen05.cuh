// Weight gradient of a projection or a "same" convolution whose input was kept in eight bits, on the 5th-generation tensor cores:
//
//   dW[tap][i][o] = sum over sequences n and positions l of  x^[n, l + tap - taps/2, i] dy[n, l, o]        (x^ zero outside a sequence)
//
// x^ = q 2^(b - 127) is exact in bf16, so that its products with a bf16 dy are those of the values themselves; sums are fp32.  An fp32
// dy is cut into three bf16 parts that add up to it exactly (8 + 8 + 8 bits of its 24), multiplied one after the other into
// the same accumulator.
//
// A tile of dW is 128 input channels x BN output channels of one tap; the reduction runs over rows (n, l), 64 to a stage.  Both
// operands come row by row, that is with the reduction index slowest: the tensor core reads them "MN-major" from rows of 128 bytes
// in the 128-byte swizzle.
//   warp 0       dy by TMA
//   warp 1       one thread issues tcgen05.mma into one of two accumulators in tensor memory
//   warps 2..5   epilogue: the accumulator to dW, or to this CTA's share of it
//   warps 6..9   the bias gradient, from the dy tile that is in shared memory anyway; the tiles of one column of dW (other input channels) take
//                turns at the stages
//   warps 10..25 x^, eight warps a stage: a thread fetches 32 channels of one row (q and one byte b, four stages ahead), turns them into bf16
//                and stores them into the swizzled tile; the tap's shift and the zeros outside a sequence are made here.  dy goes the
//                same way where TMA cannot take it (fp32, unaligned rows).
// The tensor core cuts a sum of fp32 where fp32 arithmetic rounds it: 4 10^-9 of the result a step, all to one side.  So an accumulator
// takes WG_CHUNK stages and is then added, rounded, to this CTA's share in the L2, while the other accumulator fills (2048 rows: 5 10^-7 off;
// 4400 in one go were 1.2 10^-6, 9700 3.7 10^-6).
// Work is the line of all (tile, stage) pairs, cut into equal pieces, one per CTA, so that no CTA is idle whatever the sizes; a tile that
// more than one CTA worked on is added up from their shares in the order of the line: the same bits on every run.
// Every wait is bounded; a CTA whose wait runs out leaves NaN in what it had to write.
#pragma once
#include "checkpoint_kernels.cuh"
#include "gemm_tcgen05.cuh"

namespace tsdp {

constexpr int WG_BM = 128, WG_BK = 64, WG_LOADERS = 256, WG_GROUPS = 2, WG_THREADS = 320 + WG_GROUPS * WG_LOADERS, WG_AHEAD = 2, WG_BIAS = 1024, WG_STAGE_A = WG_BK * WG_BM * 2;
enum { WG_DY_TMA = 0, WG_DY_BF16 = 1, WG_DY_FP32 = 2 };
__host__ __device__ constexpr int wg_chunk(int dyk) { return dyk == WG_DY_FP32 ? 8 : 32; }      // (three products a stage in fp32)
__host__ __device__ constexpr int wg_parts(int dyk) { return dyk == WG_DY_FP32 ? 3 : 1; }
__host__ __device__ constexpr int wg_stage_bytes(int BN, int dyk) { return WG_STAGE_A + wg_parts(dyk) * WG_BK * BN * 2; }
__host__ __device__ constexpr int wg_stages(int BN, int dyk) {
  return 200 * 1024 / wg_stage_bytes(BN, dyk) < 6 ? 200 * 1024 / wg_stage_bytes(BN, dyk) : 6;
}
__host__ __device__ constexpr int wg_smem_bytes(int BN, int dyk) { return wg_stages(BN, dyk) * wg_stage_bytes(BN, dyk) + 256 + 1024; }

struct WgradArgs {
  Copy8 x;                                  // [M, K]
  const void* dy; long long ldy;            // [M, O]
  long long M;                              // rows = sequences x L
  int L, K, O, taps;
  int tiles_k, tiles_o;                     // tile = (tap, kt, ot), ot fastest
  int stages, line;                         // of a tile; of all tiles (line + grid < 2^31)
  float* dW;                                // [taps, K, O]
  float* share;                             // [2 grid][BN / 4][128][4]: what a CTA has of its first / of its last tile
  float *db, *bias;                         // [O] or null; [grid + tiles][WG_BIAS / BN][BN]: shares of it, of CTA i in tile t at i + t
};
// The line's piece of CTA i of n.
__host__ __device__ inline int wg_begin(int line, int i, int n) { return line / n * i + min(i, line % n); }

// Descriptor of an operand tile whose reduction index is the slow one: rows (one reduction index) of 64 elements, 128 bytes apart, groups of
// eight rows 1024 bytes apart (stride byte offset); further columns of 64 elements start `lead` bytes on (leading byte offset).
__device__ __forceinline__ uint64_t umma_desc_mn_sw128(uint32_t smem_addr, uint32_t lead) {
  uint64_t d = 0;
  d |= (uint64_t)((smem_addr >> 4) & 0x3FFF);
  d |= (uint64_t)(lead >> 4) << 16;
  d |= (uint64_t)(1024 >> 4) << 32;
  d |= (uint64_t)1 << 46;                 // version
  d |= (uint64_t)2 << 61;                 // SWIZZLE_128B
  return d;
}

// Two bf16 values of a word pair's bytes j, j + 1: the magnitude's seven bits on 128 (bf16 counts by ones there), 128 or 256 taken off by
// the sign bit; both exact, and so is the product with a power of two.
__device__ __forceinline__ uint32_t wg_pair(uint32_t word, uint32_t sel, __nv_bfloat162 step) {
  const uint32_t p = __byte_perm(word, 0u, sel);
  const uint32_t hi = (p & 0x007f007fu) | 0x43004300u, lo = (p & 0x00800080u) | 0xc300c300u;
  const __nv_bfloat162 v = __hmul2(__hadd2(*reinterpret_cast<const __nv_bfloat162*>(&hi), *reinterpret_cast<const __nv_bfloat162*>(&lo)), step);
  return *reinterpret_cast<const uint32_t*>(&v);
}
__device__ __forceinline__ void st_shared16(uint32_t addr, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}

__device__ __forceinline__ void red_add4(float* p, const uint32_t* v) {
  asm volatile("red.global.add.v4.f32 [%0], {%1, %2, %3, %4};" ::"l"(p), "f"(__uint_as_float(v[0])), "f"(__uint_as_float(v[1])), "f"(__uint_as_float(v[2])),
               "f"(__uint_as_float(v[3])) : "memory");
}

template <int BN, int DYK>
__global__ void __launch_bounds__(WG_THREADS, 1)
weight_grad_kernel(const __grid_constant__ CUtensorMap tmDy, WgradArgs g) {
  constexpr int STAGES = wg_stages(BN, DYK), STAGE_BYTES = wg_stage_bytes(BN, DYK), PARTS = wg_parts(DYK), CHUNK = wg_chunk(DYK);
  constexpr uint32_t TMEM_COLS = 2 * BN < 32 ? 32 : 2 * BN;
  constexpr uint32_t IDESC = umma_idesc_bf16(BN, WG_BM) | (1u << 15) | (1u << 16);      // both operands MN-major
  extern __shared__ uint8_t wg_raw[];
  const uint32_t base = (ptx::smem_u32(wg_raw) + 1023u) & ~1023u;
  const uint32_t bar0 = base + STAGES * STAGE_BYTES;
  auto full = [&](int s) { return bar0 + 8u * s; };
  auto empty = [&](int s) { return bar0 + 8u * (STAGES + s); };
  auto tfull = [&](int b) { return bar0 + 8u * (2 * STAGES + b); };
  auto tempty = [&](int b) { return bar0 + 8u * (2 * STAGES + 2 + b); };
  const uint32_t slot = bar0 + 8u * (2 * STAGES + 4);
  const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    for (int s = 0; s < STAGES; ++s) { ptx::mbar_init(full(s), WG_LOADERS / 32 + (DYK == WG_DY_TMA ? 1 : 0)); ptx::mbar_init(empty(s), g.db ? 5 : 1); }
    for (int b = 0; b < 2; ++b) { ptx::mbar_init(tfull(b), 1); ptx::mbar_init(tempty(b), 4); }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (warp == 1) { ptx::tmem_alloc(slot, TMEM_COLS); ptx::tmem_relinquish(); }
  ptx::tc_fence_before();
  __syncthreads();
  ptx::tc_fence_after();
  const uint32_t tmem = *reinterpret_cast<volatile uint32_t*>(wg_raw + (slot - ptx::smem_u32(wg_raw)));

  const int begin = wg_begin(g.line, blockIdx.x, gridDim.x), end = wg_begin(g.line, blockIdx.x + 1, gridDim.x);
  const int t_first = begin / g.stages;
  bool ok = true;

  if (warp == 0) {
    if (DYK == WG_DY_TMA && ptx::elect_one()) {
      int t = t_first, st = begin - t * g.stages, s = 0;
      uint32_t ph = 1;
      for (int i = begin; i < end; ++i) {
        if (!ptx::mbar_wait_thread(empty(s), ph)) { ok = false; break; }
        const uint32_t b0 = base + s * STAGE_BYTES + WG_STAGE_A;
        const int o0 = t % g.tiles_o * BN;
        ptx::mbar_expect_tx(full(s), BN * WG_BK * 2);
#pragma unroll
        for (int j = 0; j < BN / 64; ++j) ptx::tma_load_2d(b0 + j * WG_BK * 128, &tmDy, o0 + 64 * j, st * WG_BK, full(s));
        if (++s == STAGES) { s = 0; ph ^= 1; }
        if (++st == g.stages) { st = 0; ++t; }
      }
    }
  } else if (warp == 1) {
    if (ptx::elect_one()) {
      int t = t_first, st = begin - t * g.stages, s = 0, buf = 0, chunk = 0;
      uint32_t ph = 0, tph = 1;
      bool fresh = true;
      for (int i = begin; i < end; ++i) {
        if (fresh && !ptx::mbar_wait_thread(tempty(buf), tph)) { ok = false; break; }
        if (!ptx::mbar_wait_thread(full(s), ph)) { ok = false; break; }
        ptx::tc_fence_after();
        const uint32_t a0 = base + s * STAGE_BYTES, d = tmem + buf * BN;
#pragma unroll
        for (int p = 0; p < PARTS; ++p)
#pragma unroll
          for (int k = 0; k < WG_BK / 16; ++k)      // 16 rows = 2048 bytes of every column of 64 channels
            ptx::tc_mma_bf16(d, umma_desc_mn_sw128(a0 + k * 2048, WG_BK * 128),
                             umma_desc_mn_sw128(a0 + WG_STAGE_A + p * (WG_BK * BN * 2) + k * 2048, WG_BK * 128), IDESC,
                             fresh && p == 0 && k == 0 ? 0u : 1u);
        fresh = false;
        ptx::tc_commit(empty(s));
        if (++s == STAGES) { s = 0; ph ^= 1; }
        const bool done = ++st == g.stages;
        if (++chunk == CHUNK || done || i + 1 == end) {
          ptx::tc_commit(tfull(buf));
          chunk = 0; fresh = true;
          if (done) { st = 0; ++t; }
          if (++buf == 2) { buf = 0; tph ^= 1; }
        }
      }
    }
  } else if (warp >= 10) {
    // x^ (and dy where it does not come by TMA): row of the stage, block of 32 channels
    const int group = (warp - 10) / (WG_LOADERS / 32), tid = (threadIdx.x - 320) % WG_LOADERS, r = tid >> 2, bq = tid & 3, nb = copy_blocks(g.K);
    const bool wide = (g.K & 15) == 0 && ((uintptr_t)g.x.q & 15) == 0;
    struct Fetch { uint32_t w[8]; uint32_t b; } f[WG_AHEAD];
    // where the next fetch reads: tile t, stage st, position l of this thread's row in its sequence
    int t = (begin + group) / g.stages, st = begin + group - t * g.stages, l = 0, shift = 0, c = 0;
    long long m = 0;
    const int l_step = WG_GROUPS * WG_BK % g.L;
    const signed char* qp = nullptr;
    const unsigned char* bp = nullptr;
    auto place = [&] {
      const int tk = t / g.tiles_o, tap = tk / g.tiles_k;
      shift = tap - g.taps / 2;
      c = (tk - tap * g.tiles_k) * WG_BM + bq * 32;
      m = (long long)st * WG_BK + r;
      l = (int)(m % g.L);
      qp = g.x.q + (m + shift) * g.K + c;
      bp = g.x.b + (m + shift) * nb + (c >> 5);
    };
    auto fetch = [&](Fetch& o) {
      const bool in = m < g.M && (unsigned)(l + shift) < (unsigned)g.L && c < g.K;
      o.b = in ? (uint32_t)*bp : 0u;
#pragma unroll
      for (int j = 0; j < 8; ++j) o.w[j] = 0u;
      if (in) {
        if (wide) {
          const uint4 u = *reinterpret_cast<const uint4*>(qp);
          o.w[0] = u.x; o.w[1] = u.y; o.w[2] = u.z; o.w[3] = u.w;
          if (c + 16 < g.K) {
            const uint4 v = *reinterpret_cast<const uint4*>(qp + 16);
            o.w[4] = v.x; o.w[5] = v.y; o.w[6] = v.z; o.w[7] = v.w;
          }
        } else {
#pragma unroll
          for (int j = 0; j < 32; ++j)
            if (c + j < g.K) o.w[j >> 2] |= (uint32_t)(unsigned char)qp[j] << (8 * (j & 3));
        }
      }
      st += WG_GROUPS;
      if (st >= g.stages) {
        while (st >= g.stages) { st -= g.stages; ++t; }
        place();
      } else {
        m += WG_GROUPS * WG_BK;
        qp += (long long)WG_GROUPS * WG_BK * g.K;
        bp += (long long)WG_GROUPS * WG_BK * nb;
        l += l_step;
        if (l >= g.L) l -= g.L;
      }
    };
    place();
    // rows of 128 bytes per 64 channels; the two halves of a row take their 16-byte pieces in another order, so that the eight threads of
    // a store phase (two rows, four blocks) touch eight different pieces
    const uint32_t half = (uint32_t)(bq >> 1), row_off = half * (WG_BK * 128) + (uint32_t)r * 128;
    const uint32_t ch0 = (uint32_t)(bq & 1) * 4, rx = (uint32_t)(r & 7);
    int s = group;
    uint32_t ph = 1;
    [[maybe_unused]] int t_cur = t;                           // the stage that is stored, for a dy that is read here
    [[maybe_unused]] int st_cur = st;
#pragma unroll
    for (int d = 0; d < WG_AHEAD; ++d)
      if (begin + group + d * WG_GROUPS < end) fetch(f[d]);
    for (int i0 = begin + group; i0 < end && ok; i0 += WG_AHEAD * WG_GROUPS)
#pragma unroll
    for (int d = 0; d < WG_AHEAD; ++d) {
      const int i = i0 + d * WG_GROUPS;
      if (i >= end || !ok) continue;
      const Fetch cur = f[d];
      ok = ptx::mbar_wait_warp(empty(s), ph);
      if (!ok) continue;
      if (i + WG_AHEAD * WG_GROUPS < end) fetch(f[d]);
      const uint32_t a0 = base + s * STAGE_BYTES;
      const uint32_t sb = cur.b == 255u ? 0x7fc0u : cur.b << 7, sb2 = sb | sb << 16;
      const __nv_bfloat162 stp = *reinterpret_cast<const __nv_bfloat162*>(&sb2);
#pragma unroll
      for (int jj = 0; jj < 4; ++jj) {
        const uint32_t j = (uint32_t)jj ^ (2 * half);
        // (a select between two words: an index known at run time would move the array to local memory)
        const uint32_t w0 = half ? cur.w[2 * (jj ^ 2)] : cur.w[2 * jj], w1 = half ? cur.w[2 * (jj ^ 2) + 1] : cur.w[2 * jj + 1];
        st_shared16(a0 + row_off + (((ch0 + j) ^ rx) << 4), wg_pair(w0, 0x4140, stp), wg_pair(w0, 0x4342, stp), wg_pair(w1, 0x4140, stp),
                    wg_pair(w1, 0x4342, stp));
      }
      if constexpr (DYK != WG_DY_TMA) {
        // eight output channels at a time
        const long long m_cur = (long long)st_cur * WG_BK + r;
        const int o0 = t_cur % g.tiles_o * BN;
        st_cur += WG_GROUPS;
        while (st_cur >= g.stages) { st_cur -= g.stages; ++t_cur; }
        const bool row_in = m_cur < g.M;
        const uint32_t b0 = a0 + WG_STAGE_A;
        for (int u = bq; u < BN / 8; u += 4) {
          const int o = o0 + 8 * u;
          uint32_t part[3][4];
          if constexpr (DYK == WG_DY_BF16) {
            const unsigned short* p = reinterpret_cast<const unsigned short*>(g.dy) + m_cur * g.ldy + o;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const uint32_t x0 = row_in && o + 2 * j < g.O ? p[2 * j] : 0u, x1 = row_in && o + 2 * j + 1 < g.O ? p[2 * j + 1] : 0u;
              part[0][j] = x0 | x1 << 16;
            }
          } else {
            const float* p = reinterpret_cast<const float*>(g.dy) + m_cur * g.ldy + o;
            uint32_t e[3][8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
              const float v = row_in && o + j < g.O ? p[j] : 0.f;
              const uint32_t bits = __float_as_uint(v), h0 = bits & 0xffff0000u;
              const float r1 = v - __uint_as_float(h0);
              const uint32_t h1 = __float_as_uint(r1) & 0xffff0000u;
              const float r2 = r1 - __uint_as_float(h1);
              const bool odd = (bits & 0x7f800000u) == 0x7f800000u;      // an infinity or a NaN is its own first part
              e[0][j] = odd ? ((bits & 0x7fffffu) ? 0x7fc00000u : h0) : h0;
              e[1][j] = odd ? 0u : h1;
              e[2][j] = odd ? 0u : __float_as_uint(r2);
            }
#pragma unroll
            for (int k = 0; k < 3; ++k)
#pragma unroll
              for (int j = 0; j < 4; ++j) part[k][j] = __byte_perm(e[k][2 * j], e[k][2 * j + 1], 0x7632);
          }
#pragma unroll
          for (int k = 0; k < PARTS; ++k)
            st_shared16(b0 + k * (WG_BK * BN * 2) + (u >> 3) * (WG_BK * 128) + r * 128 + ((((uint32_t)u & 7) ^ rx) << 4), part[k][0], part[k][1],
                        part[k][2], part[k][3]);
        }
      }
      ptx::fence_async_smem();
      __syncwarp();
      if (lane == 0) ptx::mbar_arrive(full(s));
      s += WG_GROUPS;
      if (s >= STAGES) { s -= STAGES; ph ^= 1; }
    }
  } else if (warp < 6) {
    const int quad = warp & 3, row = quad * 32 + lane;                   // tensor-memory lane quadrant of this warp; input channel of the tile
    int i = begin, t = t_first, buf = 0;
    uint32_t ph = 0;
    while (i < end) {
      const int t_end = min((t + 1) * g.stages, end);
      const bool whole = i == t * g.stages && t_end == (t + 1) * g.stages;
      const int o0 = t % g.tiles_o * BN, tk = t / g.tiles_o, tap = tk / g.tiles_k, k = (tk - tap * g.tiles_k) * WG_BM + row;
      float* share = g.share + (2ll * blockIdx.x + (t == t_first ? 0 : 1)) * (WG_BM * BN) + row * 4;
      float* out = g.dW + ((long long)tap * g.K + k) * g.O + o0;
      const int cols = min(BN, g.O - o0);
      const bool vec = (g.O & 3) == 0 && ((uintptr_t)g.dW & 15) == 0;
      for (bool first = true; i < t_end; first = false) {
        i = min(i + CHUNK, t_end);
        const bool last = i == t_end;
        ok = ok && ptx::mbar_wait_warp(tfull(buf), ph);
        ptx::tc_fence_after();
        for (int c0 = 0; c0 < BN; c0 += 16) {
          uint32_t v[16];
          if (ok) {
            ptx::tmem_ld16(tmem + buf * BN + ((uint32_t)(quad * 32) << 16) + c0, v);
            ptx::tmem_ld_wait();
          } else {
#pragma unroll
            for (int j = 0; j < 16; ++j) v[j] = 0x7fc00000u;
          }
          float* sh = share + c0 * WG_BM;                                  // the share, four columns of 128 rows at a time
          if (!(last && whole)) {
            // (an addition that does not wait for what it adds to; one thread's, so in its order)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              if (first) *reinterpret_cast<uint4*>(sh + j * 4 * WG_BM) = make_uint4(v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]);
              else red_add4(sh + j * 4 * WG_BM, v + 4 * j);
            }
            continue;
          }
          if (!first) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const float4 u = *reinterpret_cast<const float4*>(sh + j * 4 * WG_BM);
              v[4 * j] = __float_as_uint(__uint_as_float(v[4 * j]) + u.x); v[4 * j + 1] = __float_as_uint(__uint_as_float(v[4 * j + 1]) + u.y);
              v[4 * j + 2] = __float_as_uint(__uint_as_float(v[4 * j + 2]) + u.z); v[4 * j + 3] = __float_as_uint(__uint_as_float(v[4 * j + 3]) + u.w);
            }
          }
          if (k < g.K && vec) {
#pragma unroll
            for (int j = 0; j < 4; ++j)
              if (c0 + 4 * j < cols) *reinterpret_cast<uint4*>(out + c0 + 4 * j) = make_uint4(v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]);
          } else if (k < g.K) {
#pragma unroll
            for (int j = 0; j < 16; ++j)
              if (c0 + j < cols) out[c0 + j] = __uint_as_float(v[j]);
          }
        }
        ptx::tc_fence_before();
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive(tempty(buf));
        if (++buf == 2) { buf = 0; ph ^= 1; }
      }
      ++t;
    }
  } else if (g.db) {
    // eight columns of the dy tile and a share of its rows a thread
    constexpr int UNITS = BN / 8, GROUPS = 128 / UNITS, ROWS = WG_BK / GROUPS;
    const int tb = threadIdx.x - 192, unit = tb % UNITS, grp = tb / UNITS;
    const uint32_t at = (uint32_t)(unit >> 3) * (WG_BK * 128) + (uint32_t)grp * ROWS * 128;
    int t = t_first, st = begin - t * g.stages, s = 0;
    uint32_t ph = 0;
    float2 sum[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) sum[j] = make_float2(0.f, 0.f);
    int tk = t / g.tiles_o, kt = tk % g.tiles_k, turn = st % g.tiles_k;
    bool centre = tk / g.tiles_k == g.taps / 2;
    for (int i = begin; i < end; ++i) {
      ok = ptx::mbar_wait_warp(full(s), ph);
      if (!ok) break;
      if (centre && turn == kt) {
        float2 part[4];                                                    // (of a stage apart: fewer additions to the long sum)
#pragma unroll
        for (int j = 0; j < 4; ++j) part[j] = make_float2(0.f, 0.f);
#pragma unroll
        for (int p = 0; p < PARTS; ++p) {
          const uint8_t* b0 = wg_raw + (base - ptx::smem_u32(wg_raw)) + s * STAGE_BYTES + WG_STAGE_A + p * (WG_BK * BN * 2) + at;
#pragma unroll 8
          for (int r = 0; r < ROWS; ++r) {
            const uint4 u = *reinterpret_cast<const uint4*>(b0 + r * 128 + ((((uint32_t)unit ^ (uint32_t)(grp * ROWS + r)) & 7) << 4));
            const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
            for (int j = 0; j < 4; ++j) part[j] = __fadd2_rn(part[j], make_float2(__uint_as_float(w[j] << 16), __uint_as_float(w[j] & 0xffff0000u)));
          }
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) sum[j] = __fadd2_rn(sum[j], part[j]);
      }
      __syncwarp();
      if (lane == 0) ptx::mbar_arrive(empty(s));
      if (++s == STAGES) { s = 0; ph ^= 1; }
      if (++turn == g.tiles_k) turn = 0;
      const bool done = ++st == g.stages;
      if (done || i + 1 == end) {
        if (centre)
#pragma unroll
          for (int j = 0; j < 4; ++j) *reinterpret_cast<float2*>(g.bias + (size_t)(blockIdx.x + t) * WG_BIAS + grp * BN + unit * 8 + 2 * j) = sum[j];
#pragma unroll
        for (int j = 0; j < 4; ++j) sum[j] = make_float2(0.f, 0.f);
        if (done) {
          st = turn = 0; ++t;
          tk = t / g.tiles_o; kt = tk % g.tiles_k;
          centre = tk / g.tiles_k == g.taps / 2;
        }
      }
    }
  }
  if (!ok) {
    const long long t0 = clock64();
    while (clock64() - t0 < 400000ll) { }      // copies that are still in flight land before the memory is given back
  }
  ptx::tc_fence_before();
  __syncthreads();
  ptx::tc_fence_after();
  if (warp == 1) ptx::tmem_dealloc(tmem, TMEM_COLS);
}

// CTAs first .. last of the line's pieces that hold stages of tile t.
__device__ __forceinline__ void wg_owners(const WgradArgs& g, int ctas, int t, int& first, int& last) {
  const unsigned q = (unsigned)g.line / ctas, rem = (unsigned)g.line % ctas, a = (unsigned)t * g.stages, b = a + g.stages - 1;
  auto owner = [&](unsigned i) { return (int)(i < rem * (q + 1) ? i / (q + 1) : rem + (i - rem * (q + 1)) / q); };
  first = owner(a); last = owner(b);
}

// Tiles that several CTAs worked on: their shares, in the order of the line; a block has 16 columns of a tile, a warp 8 rows x 16 columns at
// a time (128 bytes of a share, 64 bytes of a row of dW).  The last tiles_o blocks (with db): the bias gradient of a column of tiles.
template <int BN>
__global__ void __launch_bounds__(256)
weight_grad_join_kernel(WgradArgs g, int ctas, int tiles) {
  constexpr int PARTS = BN / 16;
  int first, last;
  if ((int)blockIdx.x >= tiles * PARTS) {
    __shared__ float s_db[WG_BIAS];
    const int ot = blockIdx.x - tiles * PARTS;
    float v[4] = {};
    for (int kt = 0; kt < g.tiles_k; ++kt) {
      const int t = ((g.taps / 2) * g.tiles_k + kt) * g.tiles_o + ot;
      wg_owners(g, ctas, t, first, last);
#pragma unroll 4
      for (int i = first; i <= last; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] += g.bias[(size_t)(i + t) * WG_BIAS + j * 256 + threadIdx.x];
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) s_db[j * 256 + threadIdx.x] = v[j];
    __syncthreads();
    const int col = threadIdx.x;
    if (col >= BN || ot * BN + col >= g.O) return;
    float sum = 0.f;
    for (int i = 0; i < WG_BIAS / BN; ++i) sum += s_db[i * BN + col];
    g.db[ot * BN + col] = sum;
    return;
  }
  const int t = blockIdx.x / PARTS;
  wg_owners(g, ctas, t, first, last);
  if (first == last) return;                                             // one CTA had all of it
  const int o0 = t % g.tiles_o * BN, tk = t / g.tiles_o, tap = tk / g.tiles_k, k0 = (tk - tap * g.tiles_k) * WG_BM;
  const int which0 = wg_begin(g.line, first, ctas) / g.stages == t ? 0 : 1;          // of the first; the others begin in this tile
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const int e = j * 256 + threadIdx.x, row = (e >> 5) * 8 + (e & 7), c = (blockIdx.x % PARTS) * 16 + ((e >> 3) & 3) * 4, k = k0 + row;
    if (k >= g.K || o0 + c >= g.O) continue;
    const float* sh = g.share + (c >> 2) * (WG_BM * 4) + row * 4;
    float4 v = *reinterpret_cast<const float4*>(sh + (2ll * first + which0) * (WG_BM * BN));
#pragma unroll 4
    for (int i = first + 1; i <= last; ++i) {
      const float4 u = *reinterpret_cast<const float4*>(sh + 2ll * i * (WG_BM * BN));
      v.x += u.x; v.y += u.y; v.z += u.z; v.w += u.w;
    }
    float* out = g.dW + ((long long)tap * g.K + k) * g.O + o0 + c;
    if ((g.O & 3) == 0 && ((uintptr_t)g.dW & 15) == 0) *reinterpret_cast<float4*>(out) = v;
    else {
      const float w[4] = {v.x, v.y, v.z, v.w};
      for (int i = 0; i < 4; ++i) if (o0 + c + i < g.O) out[i] = w[i];
    }
  }
}

}  // namespace tsdp
