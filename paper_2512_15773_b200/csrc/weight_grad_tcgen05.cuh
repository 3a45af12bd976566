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
//   warp 0       dy by TMA into a ring of its own
//   warp 1       one thread issues tcgen05.mma into one of two accumulators in tensor memory
//   warps 2..5   epilogue: the accumulator to dW, or to this CTA's share of it
//   warps 6..9   the bias gradient, from the dy tile that is in shared memory anyway; the tiles of one column of dW (other input channels) take
//                turns at the stages
//   warps 10..25 x^, eight warps a stage: a thread takes 16 channels of two rows from the ring of q, multiplies them with their steps (fetched
//                four stages ahead) and stores them into the swizzled tile as bf16; a row outside its sequence has a step of zero.  dy goes
//                the same way where TMA cannot take it (fp32, unaligned rows).
//   warp 26      q by TMA, six stages ahead, rows moved by the tap's shift
// The tensor core cuts a sum of fp32 where fp32 arithmetic rounds it: 4 10^-9 of the result a step, all to one side.  So an accumulator
// takes WG_CHUNK stages and is then added, rounded, to this CTA's share in the L2, while the other accumulator fills (2048 rows: 5 10^-7 off;
// 4400 in one go were 1.2 10^-6, 9700 3.7 10^-6).
// Work is the line of all (tile, stage) pairs, cut into equal pieces, one per CTA, so that no CTA is idle whatever the sizes; a tile that
// more than one CTA worked on is added up from their shares in an order that the sizes alone fix: the same bits on every run.
// Pair form (CG = 2, cta_group::2): a tile of 256 x 256 on two SMs.  Each CTA makes x^ of its own 128 input channels and loads half of the
// dy columns, so that a stage brings 16 KB less into each SM's shared memory and the tensor core reads 16 KB less of it.  Everything but the
// MMAs stays within a CTA: the second CTA's idle MMA warp passes on to the first that its stage is complete.
// What bounds it: the tensor core waits for x^.  45056 rows, 512 -> 2048, bf16, pairs: 102 us and 12 for the join (0.83 PFLOP/s over both; tensor pipe
// 49 % busy, arithmetic pipe 61 %), 128 us in a long loop at the power limit; of them the conversion of x^ costs 17, draining 6, the bias gradient 3.
// 16384 rows, 512 -> 512, 5 taps: 58 us (0.74 PFLOP/s).  Operands with the reduction index slowest cost nothing against the other order.
// Every wait is bounded; a CTA whose wait runs out leaves NaN in what it had to write, of dW and of db.
#pragma once
#include "checkpoint_kernels.cuh"
#include "gemm_tcgen05.cuh"

namespace tsdp {

constexpr int WG_BM = 128, WG_BK = 64, WG_LOADERS = 256, WG_GROUPS = 2, WG_THREADS = 352 + WG_GROUPS * WG_LOADERS, WG_AHEAD = 2, WG_BIAS = 1024;
constexpr int WG_TILE_A = WG_BK * WG_BM * 2, WG_TILE_Q = WG_BK * WG_BM;
enum { WG_DY_TMA = 0, WG_DY_BF16 = 1, WG_DY_FP32 = 2 };
__host__ __device__ constexpr int wg_chunk(int dyk) { return dyk == WG_DY_FP32 ? 8 : 32; }      // (three products a stage in fp32)
__host__ __device__ constexpr int wg_parts(int dyk) { return dyk == WG_DY_FP32 ? 3 : 1; }
__host__ __device__ constexpr int wg_tile_b(int BN, int dyk, int CG) { return wg_parts(dyk) * WG_BK * (BN / CG) * 2; }
// stages of the three rings: x^, dy, q
constexpr int WG_SQ = 6;
__host__ __device__ constexpr int wg_sa(int CG) { return CG == 2 ? 5 : 4; }
__host__ __device__ constexpr int wg_sb(int BN, int dyk, int CG) {
  return CG == 2 ? 5 : (wg_tile_b(BN, dyk, CG) > 32768 ? 2 : (wg_tile_b(BN, dyk, CG) > 24576 ? 3 : 4));
}
__host__ __device__ constexpr int wg_smem_bytes(int BN, int dyk, int CG) {
  return wg_sa(CG) * WG_TILE_A + wg_sb(BN, dyk, CG) * wg_tile_b(BN, dyk, CG) + WG_SQ * WG_TILE_Q + 512 + 1024;
}

struct WgradArgs {
  Copy8 x;                                  // [M, K]
  const void* dy; long long ldy;            // [M, O]
  long long M;                              // rows = sequences x L
  int L, K, O, taps;
  int q_tma;                                // rows of q come in 16-byte pieces
  int tiles_k, tiles_o;                     // tile = (tap, kt, ot), ot fastest
  int stages, line;                         // of a tile; of all tiles (line + grid < 2^31)
  float* dW;                                // [taps, K, O]
  float* share;                             // [grid][2][BN / 4][128][4]: what a CTA has of its first / of its last tile
  long long wait_cycles;                    // limit of every wait
  int withhold;                             // CTA 0 gets no dy (tsdp_debug_arm_train_timeout)
  float *db, *bias;                         // [O] or null; [units + tiles][CG][WG_BIAS]: shares of it, of unit (CTA or pair) i in tile t at i + t
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

__device__ __forceinline__ void st_shared16(uint32_t addr, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}

__device__ __forceinline__ void red_add4(float* p, const uint32_t* v) {
  asm volatile("red.global.add.v4.f32 [%0], {%1, %2, %3, %4};" ::"l"(p), "f"(__uint_as_float(v[0])), "f"(__uint_as_float(v[1])), "f"(__uint_as_float(v[2])),
               "f"(__uint_as_float(v[3])) : "memory");
}

// The second CTA of a pair to the first: "my stage is complete".  What it passes on was written to its own shared memory and is read there by
// its own tensor core, so the arrival is ordered behind this CTA's; a release to the whole cluster (.release.cluster) at every stage costs
// more than the stage: 45056 x 512 -> 2048 177 us in place of 110.
__device__ __forceinline__ void wg_pass_on(uint32_t bar_of_first) {
  asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(bar_of_first) : "memory");
}

template <int BN, int DYK, int CG>
__global__ void __launch_bounds__(WG_THREADS, 1)
weight_grad_kernel(const __grid_constant__ CUtensorMap tmDy, const __grid_constant__ CUtensorMap tmQ, WgradArgs g) {
  constexpr int SA = wg_sa(CG), SB = wg_sb(BN, DYK, CG), SQ = WG_SQ, PARTS = wg_parts(DYK), CHUNK = wg_chunk(DYK), TILE_B = wg_tile_b(BN, DYK, CG);
  constexpr int BH = BN / CG;                                // columns of dy in this CTA
  constexpr uint32_t TMEM_COLS = 2 * BN < 32 ? 32 : 2 * BN;
  constexpr uint32_t IDESC = umma_idesc_bf16(BN, WG_BM * CG) | (1u << 15) | (1u << 16);      // both operands MN-major
  extern __shared__ uint8_t wg_raw[];
  const uint32_t base = (ptx::smem_u32(wg_raw) + 1023u) & ~1023u;
  uint8_t* const raw = wg_raw + (base - ptx::smem_u32(wg_raw));
  constexpr uint32_t OFF_B = SA * WG_TILE_A, OFF_Q = OFF_B + SB * TILE_B, OFF_BAR = OFF_Q + SQ * WG_TILE_Q;
  const uint32_t bar0 = base + OFF_BAR;
  auto full_a = [&](int s) { return bar0 + 8u * s; };
  auto empty_a = [&](int s) { return bar0 + 8u * (SA + s); };
  auto full_b = [&](int s) { return bar0 + 8u * (2 * SA + s); };
  auto empty_b = [&](int s) { return bar0 + 8u * (2 * SA + SB + s); };
  auto full_q = [&](int s) { return bar0 + 8u * (2 * SA + 2 * SB + s); };
  auto empty_q = [&](int s) { return bar0 + 8u * (2 * SA + 2 * SB + SQ + s); };
  auto tfull = [&](int b) { return bar0 + 8u * (2 * SA + 2 * SB + 2 * SQ + b); };
  auto tempty = [&](int b) { return bar0 + 8u * (2 * SA + 2 * SB + 2 * SQ + 2 + b); };
  auto peer = [&](int s) { return bar0 + 8u * (2 * SA + 2 * SB + 2 * SQ + 4 + s); };
  const uint32_t slot = bar0 + 8u * (3 * SA + 2 * SB + 2 * SQ + 4);
  static_assert(8 * (3 * SA + 2 * SB + 2 * SQ + 4) + 4 <= 512, "the barriers have 512 bytes");
  const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    for (int s = 0; s < SA; ++s) { ptx::mbar_init(full_a(s), WG_LOADERS / 32); ptx::mbar_init(empty_a(s), 1); ptx::mbar_init(peer(s), 1); }
    for (int s = 0; s < SB; ++s) { ptx::mbar_init(full_b(s), DYK == WG_DY_TMA ? 1 : WG_LOADERS / 32); ptx::mbar_init(empty_b(s), g.db ? 5 : 1); }
    for (int s = 0; s < SQ; ++s) { ptx::mbar_init(full_q(s), 1); ptx::mbar_init(empty_q(s), WG_LOADERS / 32); }
    for (int b = 0; b < 2; ++b) { ptx::mbar_init(tfull(b), 1); ptx::mbar_init(tempty(b), 4 * CG); }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (warp == 1) {
    if (CG == 2) { ptx::tmem_alloc_pair(slot, TMEM_COLS); ptx::tmem_relinquish_pair(); }
    else { ptx::tmem_alloc(slot, TMEM_COLS); ptx::tmem_relinquish(); }
  }
  ptx::tc_fence_before();
  __syncthreads();
  if (CG == 2) ptx::cluster_sync_all();                     // the peer's barriers exist
  ptx::tc_fence_after();
  const uint32_t tmem = *reinterpret_cast<volatile uint32_t*>(raw + (slot - base));
  pdl_trigger(true);                                        // the join of the shares: its blocks wait beside this grid, which runs at once as a whole
  pdl_wait();

  const int rank = CG == 2 ? (int)ptx::cluster_rank() : 0, unit = blockIdx.x / CG, units = gridDim.x / CG;
  const int begin = wg_begin(g.line, unit, units), end = wg_begin(g.line, unit + 1, units);
  const int t_first = begin / g.stages;
  bool ok = true;

  if (warp == 0) {
    if (DYK == WG_DY_TMA && !(g.withhold && blockIdx.x == 0) && ptx::elect_one()) {
      int t = t_first, st = begin - t * g.stages, s = 0;
      uint32_t ph = 1;
      for (int i = begin; i < end; ++i) {
        if (!ptx::mbar_wait_thread(empty_b(s), ph, g.wait_cycles)) { ok = false; break; }
        const int o0 = t % g.tiles_o * BN + rank * BH;
        ptx::mbar_expect_tx(full_b(s), BH * WG_BK * 2);
#pragma unroll
        for (int j = 0; j < BH / 64; ++j) ptx::tma_load_2d(base + OFF_B + s * TILE_B + j * WG_BK * 128, &tmDy, o0 + 64 * j, st * WG_BK, full_b(s));
        if (++s == SB) { s = 0; ph ^= 1; }
        if (++st == g.stages) { st = 0; ++t; }
      }
    }
  } else if (warp == 26) {
    if (g.q_tma && ptx::elect_one()) {
      int t = t_first, st = begin - t * g.stages, s = 0;
      uint32_t ph = 1;
      for (int i = begin; i < end; ++i) {
        if (!ptx::mbar_wait_thread(empty_q(s), ph, g.wait_cycles)) { ok = false; break; }
        const int tk = t / g.tiles_o, tap = tk / g.tiles_k;
        ptx::mbar_expect_tx(full_q(s), WG_TILE_Q);
        ptx::tma_load_2d(base + OFF_Q + s * WG_TILE_Q, &tmQ, ((tk - tap * g.tiles_k) * CG + rank) * WG_BM, st * WG_BK + tap - g.taps / 2, full_q(s));
        if (++s == SQ) { s = 0; ph ^= 1; }
        if (++st == g.stages) { st = 0; ++t; }
      }
    }
  } else if (warp == 1 && rank != 0) {
    if (ptx::elect_one()) {
      int sa = 0, sb = 0;
      uint32_t pa = 0, pb = 0;
      for (int i = begin; i < end; ++i) {
        if (!ptx::mbar_wait_thread(full_b(sb), pb, g.wait_cycles) || !ptx::mbar_wait_thread(full_a(sa), pa, g.wait_cycles)) { ok = false; break; }
        wg_pass_on(ptx::mapa_rank(peer(sa), 0));
        if (++sa == SA) { sa = 0; pa ^= 1; }
        if (++sb == SB) { sb = 0; pb ^= 1; }
      }
    }
  } else if (warp == 1) {
    if (ptx::elect_one()) {
      int t = t_first, st = begin - t * g.stages, sa = 0, sb = 0, buf = 0, chunk = 0;
      uint32_t pa = 0, pb = 0, tph = 1;
      bool fresh = true;
      auto commit = [&](uint32_t bar) { if (CG == 2) ptx::tc_commit_pair(bar); else ptx::tc_commit(bar); };
      for (int i = begin; i < end; ++i) {
        if (fresh && !ptx::mbar_wait_thread(tempty(buf), tph, g.wait_cycles)) { ok = false; break; }
        if (!ptx::mbar_wait_thread(full_b(sb), pb, g.wait_cycles) || !ptx::mbar_wait_thread(full_a(sa), pa, g.wait_cycles) || (CG == 2 && !ptx::mbar_wait_thread(peer(sa), pa, g.wait_cycles))) { ok = false; break; }
        ptx::tc_fence_after();
        const uint32_t a0 = base + sa * WG_TILE_A, b0 = base + OFF_B + sb * TILE_B, d = tmem + buf * BN;
#pragma unroll
        for (int p = 0; p < PARTS; ++p)
#pragma unroll
          for (int k = 0; k < WG_BK / 16; ++k)      // 16 rows = 2048 bytes of every column of 64 channels
          {
            const uint64_t da = umma_desc_mn_sw128(a0 + k * 2048, WG_BK * 128), db = umma_desc_mn_sw128(b0 + p * (WG_BK * BH * 2) + k * 2048, WG_BK * 128);
            const uint32_t acc = fresh && p == 0 && k == 0 ? 0u : 1u;
            if (CG == 2) ptx::tc_mma_bf16_pair(d, da, db, IDESC, acc); else ptx::tc_mma_bf16(d, da, db, IDESC, acc);
          }
        fresh = false;
        commit(empty_a(sa));
        commit(empty_b(sb));
        if (++sa == SA) { sa = 0; pa ^= 1; }
        if (++sb == SB) { sb = 0; pb ^= 1; }
        const bool done = ++st == g.stages;
        if (++chunk == CHUNK || done || i + 1 == end) {
          commit(tfull(buf));
          chunk = 0; fresh = true;
          if (done) { st = 0; ++t; }
          if (++buf == 2) { buf = 0; tph ^= 1; }
        }
      }
    }
  } else if (warp >= 10) {
    // x^ (and dy where it does not come by TMA): 16 channels (piece p) of rows r and r + 32 of the stage
    const int group = (warp - 10) / (WG_LOADERS / 32), tid = (threadIdx.x - 320) % WG_LOADERS, r = tid >> 3, p = tid & 7, nb = copy_blocks(g.K);
    // where the next steps are: tile t, stage st, positions of this thread's rows in their sequences
    int t = (begin + group) / g.stages, st = begin + group - t * g.stages, l0 = 0, l1 = 0, shift = 0, c = 0;
    int left = 0;                                             // rows from this thread's first to the end
    const unsigned char* bp = nullptr;
    const int l_step = WG_GROUPS * WG_BK % g.L;
    auto place = [&] {
      const int tk = t / g.tiles_o, tap = tk / g.tiles_k;
      shift = tap - g.taps / 2;
      c = ((tk - tap * g.tiles_k) * CG + rank) * WG_BM + p * 16;
      const long long m = (long long)st * WG_BK + r;
      left = (int)(g.M - m);
      l0 = (int)(m % g.L) + shift;
      l1 = (int)((m + 32) % g.L) + shift;
      bp = g.x.b + (m + shift) * nb + (c >> 5);
    };
    auto steps_of = [&](uint32_t (&o)[2]) {
      o[0] = o[1] = 0u;
      if (c < g.K) {
        if (left > 0 && (unsigned)l0 < (unsigned)g.L) o[0] = bp[0];
        if (left > 32 && (unsigned)l1 < (unsigned)g.L) o[1] = bp[32 * nb];
      }
      st += WG_GROUPS;
      if (st >= g.stages) {
        while (st >= g.stages) { st -= g.stages; ++t; }
        place();
      } else {
        left -= WG_GROUPS * WG_BK;
        bp += WG_GROUPS * WG_BK * (long long)nb;
        l0 += l_step; l1 += l_step;
        if (l0 - shift >= g.L) l0 -= g.L;
        if (l1 - shift >= g.L) l1 -= g.L;
      }
    };
    place();
    // the stage that is worked on, where its bytes do not come by TMA
    int t_cur = t, st_cur = st;
    // rows of 128 bytes per 64 channels; the pieces of the two halves of a row store theirs in another order, so that the eight threads
    // of a store phase (one row) touch eight different 16-byte units
    const uint32_t half = (uint32_t)(p >> 2), rx = (uint32_t)(r & 7), row_off = half * (WG_BK * 128) + (uint32_t)r * 128;
    const uint32_t u0 = (((uint32_t)(p & 3) * 2 + half) ^ rx) << 4, u1 = (((uint32_t)(p & 3) * 2 + (half ^ 1)) ^ rx) << 4;
    int sa = group, sb = group % SB, sq = group;
    uint32_t pa = 1, pb = group >= SB ? 0 : 1, pq = 0;
    uint32_t ahead[WG_AHEAD][2];
    // rows of a bf16 dy in words, two values each, instead of one by one (14752 rows, 160 -> 542, 3 taps: 83 -> 62 us)
    const bool dy_words = DYK == WG_DY_BF16 && ((uintptr_t)g.dy & 3) == 0 && (g.ldy & 1) == 0;
#pragma unroll
    for (int d = 0; d < WG_AHEAD; ++d)
      if (begin + group + d * WG_GROUPS < end) steps_of(ahead[d]);
    for (int i0 = DYK != WG_DY_TMA && g.withhold && blockIdx.x == 0 ? end : begin + group; i0 < end && ok; i0 += WG_AHEAD * WG_GROUPS)
#pragma unroll
    for (int d = 0; d < WG_AHEAD; ++d) {
      const int i = i0 + d * WG_GROUPS;
      if (i >= end || !ok) continue;
      const uint32_t cur[2] = {ahead[d][0], ahead[d][1]};
      if (i + WG_AHEAD * WG_GROUPS < end) steps_of(ahead[d]);
      uint4 w[2];
      if (g.q_tma) {
        ok = ptx::mbar_wait_warp(full_q(sq), pq, g.wait_cycles);
        if (!ok) continue;
        const uint8_t* q = raw + OFF_Q + sq * WG_TILE_Q + r * WG_BM + p * 16;
        w[0] = *reinterpret_cast<const uint4*>(q);
        w[1] = *reinterpret_cast<const uint4*>(q + 32 * WG_BM);
      } else {
        const int tk = t_cur / g.tiles_o, tap = tk / g.tiles_k, ch = ((tk - tap * g.tiles_k) * CG + rank) * WG_BM + p * 16;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const long long ms = (long long)st_cur * WG_BK + r + 32 * h + tap - g.taps / 2;
          uint32_t v[4] = {0u, 0u, 0u, 0u};
          if constexpr (DYK == WG_DY_FP32) {                              // (no registers left for more: 3186 rows, 128 -> 128, 5 taps 15.6 us, 17.3 with words)
            if (ms >= 0 && ms < g.M)
#pragma unroll
              for (int j = 0; j < 16; ++j)
                if (ch + j < g.K) v[j >> 2] |= (uint32_t)(unsigned char)g.x.q[ms * g.K + ch + j] << (8 * (j & 3));
          } else if (ms >= 0 && ms < g.M && ch < g.K) {
            // the words that hold the 16 bytes, where all of them lie within q; what follows a row's last channel ends in rows of the tile that
            // go nowhere (14752 rows, 141 -> 542, 3 taps: 80 us byte by byte, 71 so)
            const long long at = ms * g.K + ch, lead = ((uintptr_t)g.x.q + at) & 3;
            if (at >= lead && at - lead + 20 <= g.M * g.K) {
              const uint32_t* src = reinterpret_cast<const uint32_t*>(g.x.q + at - lead);
              const uint32_t word[5] = {src[0], src[1], src[2], src[3], src[4]};
#pragma unroll
              for (int j = 0; j < 4; ++j) v[j] = __funnelshift_r(word[j], word[j + 1], (uint32_t)lead * 8);
            } else {
#pragma unroll
              for (int j = 0; j < 16; ++j)
                if (ch + j < g.K) v[j >> 2] |= (uint32_t)(unsigned char)g.x.q[at + j] << (8 * (j & 3));
            }
          }
          w[h] = make_uint4(v[0], v[1], v[2], v[3]);
        }
      }
      ok = ptx::mbar_wait_warp(empty_a(sa), pa, g.wait_cycles);
      if (!ok) continue;
      const uint32_t a0 = base + sa * WG_TILE_A + row_off;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const __nv_bfloat162 k = copy_step2(cur[h]);
        const uint32_t x0 = half ? w[h].z : w[h].x, x1 = half ? w[h].w : w[h].y, y0 = half ? w[h].x : w[h].z, y1 = half ? w[h].y : w[h].w;
        st_shared16(a0 + h * (32 * 128) + u0, copy_pair(x0, 0, k), copy_pair(x0, 1, k), copy_pair(x1, 0, k), copy_pair(x1, 1, k));
        st_shared16(a0 + h * (32 * 128) + u1, copy_pair(y0, 0, k), copy_pair(y0, 1, k), copy_pair(y1, 0, k), copy_pair(y1, 1, k));
      }
      if constexpr (DYK != WG_DY_TMA) {
        // eight output channels at a time
        ok = ptx::mbar_wait_warp(empty_b(sb), pb, g.wait_cycles);
        if (!ok) continue;
        const int rd = tid >> 2, bq = tid & 3;
        const long long m_cur = (long long)st_cur * WG_BK + rd;
        const int o0 = t_cur % g.tiles_o * BN;
        const bool row_in = m_cur < g.M;
        const uint32_t b0 = base + OFF_B + sb * TILE_B;
        for (int u = bq; u < BN / 8; u += 4) {
          const int o = o0 + 8 * u;
          uint32_t part[3][4];
          if constexpr (DYK == WG_DY_BF16) {
            const unsigned short* src = reinterpret_cast<const unsigned short*>(g.dy) + m_cur * g.ldy + o;
            if (dy_words && row_in && o + 8 <= g.O) {
#pragma unroll
              for (int j = 0; j < 4; ++j) part[0][j] = reinterpret_cast<const uint32_t*>(src)[j];
            } else
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const uint32_t x0 = row_in && o + 2 * j < g.O ? src[2 * j] : 0u, x1 = row_in && o + 2 * j + 1 < g.O ? src[2 * j + 1] : 0u;
              part[0][j] = x0 | x1 << 16;
            }
          } else {
            const float* src = reinterpret_cast<const float*>(g.dy) + m_cur * g.ldy + o;
            uint32_t e[3][8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
              const float v = row_in && o + j < g.O ? src[j] : 0.f;
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
            st_shared16(b0 + k * (WG_BK * BN * 2) + (u >> 3) * (WG_BK * 128) + rd * 128 + ((((uint32_t)u & 7) ^ (uint32_t)(rd & 7)) << 4), part[k][0],
                        part[k][1], part[k][2], part[k][3]);
        }
      }
      if (DYK != WG_DY_TMA || !g.q_tma) {
        st_cur += WG_GROUPS;
        while (st_cur >= g.stages) { st_cur -= g.stages; ++t_cur; }
      }
      ptx::fence_async_smem();
      __syncwarp();
      if (lane == 0) {
        ptx::mbar_arrive(full_a(sa));
        if (DYK != WG_DY_TMA) ptx::mbar_arrive(full_b(sb));
        if (g.q_tma) ptx::mbar_arrive(empty_q(sq));
      }
      sa += WG_GROUPS; if (sa >= SA) { sa -= SA; pa ^= 1; }
      sb += WG_GROUPS; if (sb >= SB) { sb -= SB; pb ^= 1; }
      sq += WG_GROUPS; if (sq >= SQ) { sq -= SQ; pq ^= 1; }
    }
  } else if (warp < 6) {
    const int quad = warp & 3, row = quad * 32 + lane;                   // tensor-memory lane quadrant of this warp; input channel of the tile
    int i = begin, t = t_first, buf = 0;
    uint32_t ph = 0;
    while (i < end) {
      const int t_end = min((t + 1) * g.stages, end);
      const bool whole = i == t * g.stages && t_end == (t + 1) * g.stages;
      const int o0 = t % g.tiles_o * BN, tk = t / g.tiles_o, tap = tk / g.tiles_k, k = ((tk - tap * g.tiles_k) * CG + rank) * WG_BM + row;
      float* share = g.share + (2ll * blockIdx.x + (t == t_first ? 0 : 1)) * (WG_BM * BN) + row * 4;
      float* out = g.dW + ((long long)tap * g.K + k) * g.O + o0;
      const int cols = min(BN, g.O - o0);
      const bool vec = (g.O & 3) == 0 && ((uintptr_t)g.dW & 15) == 0;
      for (bool first = true; i < t_end; first = false) {
        i = min(i + CHUNK, t_end);
        const bool last = i == t_end;
        ok = ok && ptx::mbar_wait_warp(tfull(buf), ph, g.wait_cycles);
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
        if (lane == 0) {
          if (CG == 2 && rank != 0) ptx::mbar_arrive_cluster(ptx::mapa_rank(tempty(buf), 0));
          else ptx::mbar_arrive(tempty(buf));
        }
        if (++buf == 2) { buf = 0; ph ^= 1; }
      }
      ++t;
    }
  } else if (g.db) {
    // eight columns of the dy tile and a share of its rows a thread
    constexpr int UNITS = BH / 8, GROUPS = 128 / UNITS, ROWS = WG_BK / GROUPS;
    const int tb = threadIdx.x - 192, piece = tb % UNITS, grp = tb / UNITS;
    const uint32_t at = (uint32_t)(piece >> 3) * (WG_BK * 128) + (uint32_t)grp * ROWS * 128;
    int t = t_first, st = begin - t * g.stages, s = 0;
    uint32_t ph = 0;
    float2 sum[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) sum[j] = make_float2(0.f, 0.f);
    int tk = t / g.tiles_o, kt = tk % g.tiles_k, turn = st % g.tiles_k;
    bool centre = tk / g.tiles_k == g.taps / 2;
    for (int i = begin; i < end; ++i) {
      ok = ptx::mbar_wait_warp(full_b(s), ph, g.wait_cycles);
      if (!ok) break;
      if (centre && turn == kt) {
        float2 part[4];                                                    // (of a stage apart: fewer additions to the long sum)
#pragma unroll
        for (int j = 0; j < 4; ++j) part[j] = make_float2(0.f, 0.f);
#pragma unroll
        for (int p = 0; p < PARTS; ++p) {
          const uint8_t* b0 = raw + OFF_B + s * TILE_B + p * (WG_BK * BH * 2) + at;
#pragma unroll 8
          for (int r = 0; r < ROWS; ++r) {
            const uint4 u = *reinterpret_cast<const uint4*>(b0 + r * 128 + ((((uint32_t)piece ^ (uint32_t)(grp * ROWS + r)) & 7) << 4));
            const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
            for (int j = 0; j < 4; ++j) part[j] = __fadd2_rn(part[j], make_float2(__uint_as_float(w[j] << 16), __uint_as_float(w[j] & 0xffff0000u)));
          }
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) sum[j] = __fadd2_rn(sum[j], part[j]);
      }
      __syncwarp();
      if (lane == 0) ptx::mbar_arrive(empty_b(s));
      if (++s == SB) { s = 0; ph ^= 1; }
      if (++turn == g.tiles_k) turn = 0;
      const bool done = ++st == g.stages;
      if (done || i + 1 == end) {
        if (centre)
#pragma unroll
          for (int j = 0; j < 4; ++j) *reinterpret_cast<float2*>(g.bias + ((size_t)(unit + t) * CG + rank) * WG_BIAS + grp * BH + piece * 8 + 2 * j) = sum[j];
#pragma unroll
        for (int j = 0; j < 4; ++j) sum[j] = make_float2(0.f, 0.f);
        if (done) {
          st = turn = 0; ++t;
          tk = t / g.tiles_o; kt = tk % g.tiles_k;
          centre = tk / g.tiles_k == g.taps / 2;
        }
      }
    }
    if (!ok)                                                               // what this CTA has not written: of this tile and of those after it
      for (; t <= (end - 1) / g.stages; ++t)
        if (t / g.tiles_o / g.tiles_k == g.taps / 2)
#pragma unroll 1
          for (int j = 0; j < 8; ++j) g.bias[((size_t)(unit + t) * CG + rank) * WG_BIAS + grp * BH + piece * 8 + j] = __uint_as_float(0x7fc00000u);
  }
  if (!ok) {
    const long long t0 = clock64();
    while (clock64() - t0 < 400000ll) { }      // copies that are still in flight land before the memory is given back
  }
  ptx::tc_fence_before();
  __syncthreads();
  if (CG == 2) ptx::cluster_sync_all();                     // neither CTA leaves while the other may still signal or read it
  ptx::tc_fence_after();
  if (warp == 1) {
    if (CG == 2) ptx::tmem_dealloc_pair(tmem, TMEM_COLS); else ptx::tmem_dealloc(tmem, TMEM_COLS);
  }
}

// CTAs first .. last of the line's pieces that hold stages of tile t.
__device__ __forceinline__ void wg_owners(const WgradArgs& g, int ctas, int t, int& first, int& last) {
  const unsigned q = (unsigned)g.line / ctas, rem = (unsigned)g.line % ctas, a = (unsigned)t * g.stages, b = a + g.stages - 1;
  auto owner = [&](unsigned i) { return (int)(i < rem * (q + 1) ? i / (q + 1) : rem + (i - rem * (q + 1)) / q); };
  first = owner(a); last = owner(b);
}

// Tiles that several CTAs worked on: the sum of their shares.  A block has 512 (SPLIT 1) or 256 / SPLIT quads of four columns of a tile, a warp
// 8 rows x 16 columns at a time (128 bytes of a share, 64 bytes of a row of dW); with SPLIT > 1 group i of its threads takes every SPLIT-th
// share from the i-th on, and the groups' sums are added in order.  The last blocks (with db): the bias gradient of eight columns each.
template <int BN, int CG, int SPLIT>
__global__ void __launch_bounds__(256)
weight_grad_join_kernel(WgradArgs g, int units, int tiles) {
  constexpr int SUBS = SPLIT == 1 ? 1 : 2 * SPLIT, SPAN = 256 / SPLIT, PARTS = BN / 16 * CG * SUBS, BH = BN / CG;
  const int group = threadIdx.x / SPAN, at = threadIdx.x % SPAN;
  pdl_wait();
  int first, last;
  if ((int)blockIdx.x >= tiles * PARTS) {                                // eight columns of db
    constexpr int ROWS = WG_BIAS / BH, GROUPS = 256 / (8 * ROWS);
    __shared__ float s_db[256];
    const int block = blockIdx.x - tiles * PARTS, ot = block / (BN / 8), col = block % (BN / 8) * 8 + (threadIdx.x & 7);
    const int row = (threadIdx.x >> 3) % ROWS, db_group = threadIdx.x / (8 * ROWS);
    float sum = 0.f;
    for (int kt = 0; kt < g.tiles_k; ++kt) {
      const int t = ((g.taps / 2) * g.tiles_k + kt) * g.tiles_o + ot;
      wg_owners(g, units, t, first, last);
#pragma unroll 8
      for (int i = first + db_group; i <= last; i += GROUPS) sum += g.bias[((size_t)(i + t) * CG + col / BH) * WG_BIAS + row * BH + col % BH];
    }
    s_db[threadIdx.x] = sum;
    __syncthreads();
    if (threadIdx.x >= 8 || ot * BN + col >= g.O) return;
    for (int i = 1; i < ROWS * GROUPS; ++i) sum += s_db[i * 8 + threadIdx.x];
    g.db[ot * BN + col] = sum;
    return;
  }
  const int t = blockIdx.x / PARTS, rank = blockIdx.x / (PARTS / CG) % CG;
  wg_owners(g, units, t, first, last);
  if (first == last) return;                                             // one CTA (or pair) had all of it
  const int o0 = t % g.tiles_o * BN, tk = t / g.tiles_o, tap = tk / g.tiles_k, k0 = ((tk - tap * g.tiles_k) * CG + rank) * WG_BM;
  const int which0 = wg_begin(g.line, first, units) / g.stages == t ? 0 : 1;         // of the first; the others begin in this tile
  const int part = blockIdx.x % (PARTS / CG) / SUBS, sub = blockIdx.x % SUBS;
#pragma unroll
  for (int j = 0; j < (SPLIT == 1 ? 2 : 1); ++j) {
    const int e = SPLIT == 1 ? j * 256 + threadIdx.x : sub * SPAN + at, row = (e >> 5) * 8 + (e & 7), c = part * 16 + ((e >> 3) & 3) * 4, k = k0 + row;
    if (SPLIT == 1 && (k >= g.K || o0 + c >= g.O)) continue;
    const float* sh = g.share + (c >> 2) * (WG_BM * 4) + row * 4;
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
    if (group == 0) v = *reinterpret_cast<const float4*>(sh + (2ll * (first * CG + rank) + which0) * (WG_BM * BN));
#pragma unroll 8
    for (int i = first + (group ? group : SPLIT); i <= last; i += SPLIT) {
      const float4 u = *reinterpret_cast<const float4*>(sh + 2ll * (i * CG + rank) * (WG_BM * BN));
      v.x += u.x; v.y += u.y; v.z += u.z; v.w += u.w;
    }
    if constexpr (SPLIT > 1) {
      __shared__ float4 s_v[SPLIT][SPAN];
      s_v[group][at] = v;
      __syncthreads();
      if (group || k >= g.K || o0 + c >= g.O) return;
#pragma unroll
      for (int i = 1; i < SPLIT; ++i) {
        const float4 u = s_v[i][at];
        v.x += u.x; v.y += u.y; v.z += u.z; v.w += u.w;
      }
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
