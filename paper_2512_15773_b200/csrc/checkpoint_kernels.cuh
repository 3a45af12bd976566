// Activations kept in eight bits between the forward and the backward pass of a training step.
//
// A row of C channels is cut into blocks of 32.  A block is 32 whole numbers q, |q| <= 127, and one byte b, and stands for
// q * 2^(b - 127); b is the smallest in 1 .. 248 with max |rint(x 2^(127 - b))| <= 127, and 255 for a block that holds an infinity
// or a NaN (read back as NaN).  The scale is a power of two, so that scaling is exact in every type, a copy depends on nothing but
// the values, and what it stands for is exact in bf16 (7 bits and a sign): the backward products take it without a rounding.
// The one rounding is that to q, half a step at most: |x - q 2^(b-127)| <= 2^(b-128), 1 / 127.5 of the block's largest value.  At the ends of the range:
// from 127.5 2^121 on q stays at 127, off by up to a step (b = 249 would stand for values past the largest fp32); at b = 1 (blocks below 2^-120)
// the half step is 2^-127 whatever the block's largest value.
// What bounds them: bytes, next to the arithmetic that finds the largest magnitude.  45056 x 2048, bf16, there and back: 106 us (5.3 TB/s, 0.81 of a plain
// copy's rate; arithmetic pipe 60 % used).  Widths that are not in 16-byte pieces go one value a lane: 45056 x 1003 288 us (0.95 TB/s), fp32 293 (1.6).
#pragma once
#include "common.cuh"

namespace tsdp {

struct Rows { void* p; long long sn, sl; };          // element (n, l, c) at p + n sn + l sl + c
struct Copy8 { signed char* q; unsigned char* b; };  // dense rows r = n L + l: q [rows, C], b [rows, (C + 31) / 32]

__host__ __device__ inline int copy_blocks(int C) { return (C + 31) >> 5; }

// b from the bits of the block's largest magnitude (bits of non-negative floats order like the values, NaN above infinity).
// 127.5 = 1.9921875 * 2^6 is the first value that rounds to 128: from a mantissa of 0x7f0000 on the exponent goes up by one.
__device__ __forceinline__ uint32_t copy_byte(uint32_t top) {
  if (top >= 0x7f800000u) return 255u;
  return (uint32_t)min(max((int)((top + 0x10000u) >> 23) - 6, 1), 248);
}
__device__ __forceinline__ float copy_inv_step(uint32_t b) { return __uint_as_float(b == 255u ? 0u : (254u - b) << 23); }     // 2^(127-b)
__device__ __forceinline__ float copy_step(uint32_t b) { return __uint_as_float(b == 255u ? 0x7fc00000u : b << 23); }        // 2^(b-127)
// q of one value, in the low byte: x 2^(127-b) is exact, the sum with 1.5 * 2^23 rounds it to a whole number, halves to even.
__device__ __forceinline__ uint32_t copy_q(float x, float inv, uint32_t b) {
  float s = x * inv;
  if (b == 248u) s = fminf(fmaxf(s, -127.f), 127.f);
  return b == 255u ? 0u : __float_as_uint(s + 12582912.f) & 0xffu;
}
// Four of them in a word.  (b >= 248 is rare: the largest magnitudes of fp32, and what is not finite.)
__device__ __forceinline__ uint32_t copy_bytes(float2 x0, float2 x1) {
  return __byte_perm(__byte_perm(__float_as_uint(x0.x), __float_as_uint(x0.y), 0x0040), __byte_perm(__float_as_uint(x1.x), __float_as_uint(x1.y), 0x0040), 0x5410);
}
__device__ __forceinline__ uint32_t copy_q4_top(float2 x0, float2 x1, float inv, uint32_t b) {
  const uint32_t q[4] = {copy_q(x0.x, inv, b), copy_q(x0.y, inv, b), copy_q(x1.x, inv, b), copy_q(x1.y, inv, b)};
  return q[0] | q[1] << 8 | q[2] << 16 | q[3] << 24;
}
__device__ __forceinline__ uint32_t copy_q4(float2 x0, float2 x1, float inv, uint32_t b) {
  if (b >= 248u) return copy_q4_top(x0, x1, inv, b);
  const float2 k = make_float2(inv, inv), magic = make_float2(12582912.f, 12582912.f);
  return copy_bytes(__ffma2_rn(x0, k, magic), __ffma2_rn(x1, k, magic));
}
__device__ __forceinline__ uint2 copy_q8(const float2* x, float inv, uint32_t b) {
  if (b >= 248u) return make_uint2(copy_q4_top(x[0], x[1], inv, b), copy_q4_top(x[2], x[3], inv, b));
  const float2 k = make_float2(inv, inv), magic = make_float2(12582912.f, 12582912.f);
  return make_uint2(copy_bytes(__ffma2_rn(x[0], k, magic), __ffma2_rn(x[1], k, magic)), copy_bytes(__ffma2_rn(x[2], k, magic), __ffma2_rn(x[3], k, magic)));
}
// Largest magnitude (as bits) of eight bf16 values in each of LANES neighbouring lanes, two at a time and a NaN above all; of four fp32 ones.
template <int LANES> __device__ __forceinline__ uint32_t copy_top_bf16(uint4 u) {
  auto larger = [](uint32_t a, uint32_t b) {
    const __nv_bfloat162 m = __hmax2_nan(*reinterpret_cast<const __nv_bfloat162*>(&a), *reinterpret_cast<const __nv_bfloat162*>(&b));
    return *reinterpret_cast<const uint32_t*>(&m);
  };
  uint32_t m = larger(larger(u.x & 0x7fff7fffu, u.y & 0x7fff7fffu), larger(u.z & 0x7fff7fffu, u.w & 0x7fff7fffu));
#pragma unroll
  for (int i = 1; i < LANES; i *= 2) m = larger(m, __shfl_xor_sync(0xffffffffu, m, i));
  m &= 0x7fff7fffu;
  return max(m << 16, m & 0xffff0000u);
}
__device__ __forceinline__ uint32_t copy_top_fp32(uint4 u) {
  return max(max(u.x & 0x7fffffffu, u.y & 0x7fffffffu), max(u.z & 0x7fffffffu, u.w & 0x7fffffffu));
}
// Values 2 i and 2 i + 1 of four in a word, without their step.  The byte with its sign bit turned over is q + 128, put behind the exponent
// of 2^23 it counts there by ones: a permutation and a subtraction, where the conversion instruction runs at an eighth of the rate.
__device__ __forceinline__ float2 copy_ints(uint32_t word, int i) {
  word ^= 0x80808080u;
  return __fadd2_rn(make_float2(__uint_as_float(__byte_perm(word, 0x4b000000u, i ? 0x7542 : 0x7540)), __uint_as_float(__byte_perm(word, 0x4b000000u, i ? 0x7543 : 0x7541))),
                    make_float2(-8388736.f, -8388736.f));
}
// The same with their step as two bf16 values: the magnitude's seven bits on 128 (bf16 counts by ones there), 128 or 256 taken off by the
// sign bit; both exact, and so is the product with a power of two.
__device__ __forceinline__ uint32_t copy_pair(uint32_t word, int i, __nv_bfloat162 step) {
  const uint32_t p = __byte_perm(word, 0u, i ? 0x4342 : 0x4140);
  const uint32_t hi = (p & 0x007f007fu) | 0x43004300u, lo = (p & 0x00800080u) | 0xc300c300u;
  const __nv_bfloat162 v = __hmul2(__hadd2(*reinterpret_cast<const __nv_bfloat162*>(&hi), *reinterpret_cast<const __nv_bfloat162*>(&lo)), step);
  return *reinterpret_cast<const uint32_t*>(&v);
}
__device__ __forceinline__ __nv_bfloat162 copy_step2(uint32_t b) {           // the byte as the exponent of two bf16 values
  const uint32_t s = b == 255u ? 0x7fc07fc0u : b * 0x00800080u;
  return *reinterpret_cast<const __nv_bfloat162*>(&s);
}

// Row r = n L + l of a tensor [N, L, C].
__device__ __forceinline__ long long row_offset(const Rows& x, long long r, int N, int L) {
  if (N == 1) return r * x.sl;
  const long long n = r < (1ll << 32) ? (long long)((uint32_t)r / (uint32_t)L) : r / L;      // (a 64-bit division costs as much as the row)
  return n * x.sn + (r - n * L) * x.sl;
}

// Eight channels a thread, four neighbouring lanes a block of 32; a row's threads are counted in whole blocks, so that the four lanes of
// a block sit side by side whatever C is.  A thread keeps its channels and walks the rows, COPY_ROWS of them asked for before the first is used.
// C % 8 = 0, 16-byte aligned rows.  Bound by bytes.
constexpr int COPY_THREADS = 256, COPY_ROWS = 4;
template <typename T>
__global__ void __launch_bounds__(COPY_THREADS, 4)
checkpoint_pack_kernel(Rows x, Copy8 out, int N, int L, int C) {
  pdl_wait();
  constexpr int W = sizeof(T) / 2;                                           // 16-byte pieces of eight values
  const int nb = copy_blocks(C), units = 4 * nb, per = min(units, COPY_THREADS);      // threads on a row
  const int lanes = COPY_THREADS / per, lane = threadIdx.x / per;
  const long long rows = (long long)N * L, step = (long long)gridDim.x * lanes;
  const long long q_step = step * C, b_step = step * nb, x_step = step * x.sl;      // (x: of one sequence)
  for (long long r0 = (long long)blockIdx.x * lanes; r0 < rows; r0 += COPY_ROWS * step) {
    for (int u0 = 0; u0 < units; u0 += per) {
      const int u = u0 + threadIdx.x - lane * per, c = 8 * u;
      const bool mine = lane < lanes && c < C;
      const long long r = r0 + lane;
      const T* p0 = reinterpret_cast<const T*>(x.p) + (N == 1 ? r * x.sl : 0) + c;
      uint4 v[COPY_ROWS][W];
#pragma unroll
      for (int k = 0; k < COPY_ROWS; ++k) {
#pragma unroll
        for (int w = 0; w < W; ++w) v[k][w] = make_uint4(0u, 0u, 0u, 0u);
        if (mine && r + k * step < rows) {
          const uint4* p = reinterpret_cast<const uint4*>(N == 1 ? p0 + k * x_step : p0 + row_offset(x, r + k * step, N, L));
#pragma unroll
          for (int w = 0; w < W; ++w) v[k][w] = p[w];
        }
      }
      signed char* q0 = out.q + r * C + c;
      unsigned char* b0 = out.b + r * nb + (u >> 2);
#pragma unroll
      for (int k = 0; k < COPY_ROWS; ++k) {
        uint32_t top;
        float2 f[4];
        if constexpr (sizeof(T) == 2) {
          top = copy_top_bf16<4>(v[k][0]);
          const uint32_t w[4] = {v[k][0].x, v[k][0].y, v[k][0].z, v[k][0].w};
#pragma unroll
          for (int i = 0; i < 4; ++i) f[i] = make_float2(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xffff0000u));
        } else {
          top = max(copy_top_fp32(v[k][0]), copy_top_fp32(v[k][W - 1]));
          f[0] = make_float2(__uint_as_float(v[k][0].x), __uint_as_float(v[k][0].y)); f[1] = make_float2(__uint_as_float(v[k][0].z), __uint_as_float(v[k][0].w));
          f[2] = make_float2(__uint_as_float(v[k][W - 1].x), __uint_as_float(v[k][W - 1].y)); f[3] = make_float2(__uint_as_float(v[k][W - 1].z), __uint_as_float(v[k][W - 1].w));
          top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
          top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
        }
        const uint32_t b = copy_byte(top);
        const float inv = copy_inv_step(b);
        if (mine && r + k * step < rows) {
          *reinterpret_cast<uint2*>(q0 + k * q_step) = copy_q8(f, inv, b);
          if ((u & 3) == 0) b0[k * b_step] = (unsigned char)b;
        }
      }
    }
  }
}

// Any width, any alignment: a warp per block, a lane per channel.
template <typename T>
__global__ void __launch_bounds__(COPY_THREADS)
checkpoint_pack_any_kernel(Rows x, Copy8 out, int N, int L, int C) {
  pdl_wait();
  const int nb = copy_blocks(C), lane = threadIdx.x & 31;
  const long long blocks = (long long)N * L * nb;
  for (long long i = (long long)blockIdx.x * (COPY_THREADS / 32) + (threadIdx.x >> 5); i < blocks; i += (long long)gridDim.x * (COPY_THREADS / 32)) {
    const long long r = i / nb;
    const int c = (int)(i - r * nb) * 32 + lane;
    float v = 0.f;
    if (c < C) v = to_f(reinterpret_cast<const T*>(x.p)[row_offset(x, r, N, L) + c]);
    const uint32_t b = copy_byte(__reduce_max_sync(0xffffffffu, __float_as_uint(v) & 0x7fffffffu));
    if (c < C) out.q[r * C + c] = (signed char)copy_q(v, copy_inv_step(b), b);
    if (lane == 0) out.b[i] = (unsigned char)b;
  }
}

template <typename T>
__global__ void __launch_bounds__(COPY_THREADS, 4)
checkpoint_unpack_kernel(Copy8 in, Rows x, int N, int L, int C) {
  pdl_wait();
  const int nb = copy_blocks(C), units = C >> 3, per = min(units, COPY_THREADS);
  const int lanes = COPY_THREADS / per, lane = threadIdx.x / per;
  const long long rows = (long long)N * L, step = (long long)gridDim.x * lanes;
  if (lane >= lanes) return;
  const long long q_step = step * C, b_step = step * nb, x_step = step * x.sl;      // (x: of one sequence)
  for (long long r = (long long)blockIdx.x * lanes + lane; r < rows; r += COPY_ROWS * step) {
    for (int u = threadIdx.x - lane * per; u < units; u += per) {
      const signed char* q0 = in.q + r * C + 8 * u;
      const unsigned char* b0 = in.b + r * nb + (u >> 2);
      uint2 w[COPY_ROWS];
      uint32_t b[COPY_ROWS];
#pragma unroll
      for (int k = 0; k < COPY_ROWS; ++k) {
        w[k] = make_uint2(0u, 0u);
        b[k] = 0u;
        if (r + k * step < rows) { w[k] = *reinterpret_cast<const uint2*>(q0 + k * q_step); b[k] = b0[k * b_step]; }
      }
      T* p0 = reinterpret_cast<T*>(x.p) + (N == 1 ? r * x.sl : 0) + 8 * u;
#pragma unroll
      for (int k = 0; k < COPY_ROWS; ++k) {
        uint4 v[sizeof(T) / 2];
        if constexpr (sizeof(T) == 2) {
          const __nv_bfloat162 st = copy_step2(b[k]);
          v[0] = make_uint4(copy_pair(w[k].x, 0, st), copy_pair(w[k].x, 1, st), copy_pair(w[k].y, 0, st), copy_pair(w[k].y, 1, st));
        } else {
          const float2 st = make_float2(copy_step(b[k]), copy_step(b[k]));
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const uint32_t word = h ? w[k].y : w[k].x;
            const float2 f0 = __fmul2_rn(copy_ints(word, 0), st), f1 = __fmul2_rn(copy_ints(word, 1), st);
            v[h] = make_uint4(__float_as_uint(f0.x), __float_as_uint(f0.y), __float_as_uint(f1.x), __float_as_uint(f1.y));
          }
        }
        if (r + k * step < rows) {
          uint4* p = reinterpret_cast<uint4*>(N == 1 ? p0 + k * x_step : p0 + row_offset(x, r + k * step, N, L));
#pragma unroll
          for (int h = 0; h < (int)sizeof(T) / 2; ++h) p[h] = v[h];
        }
      }
    }
  }
}

template <typename T>
__global__ void __launch_bounds__(COPY_THREADS)
checkpoint_unpack_any_kernel(Copy8 in, Rows x, int N, int L, int C) {
  pdl_wait();
  const int nb = copy_blocks(C), lane = threadIdx.x & 31;
  const long long blocks = (long long)N * L * nb;
  for (long long i = (long long)blockIdx.x * (COPY_THREADS / 32) + (threadIdx.x >> 5); i < blocks; i += (long long)gridDim.x * (COPY_THREADS / 32)) {
    const long long r = i / nb;
    const int c = (int)(i - r * nb) * 32 + lane;
    if (c < C) reinterpret_cast<T*>(x.p)[row_offset(x, r, N, L) + c] = from_f<T>((float)in.q[r * C + c] * copy_step(in.b[i]));
  }
}

}  // namespace tsdp
