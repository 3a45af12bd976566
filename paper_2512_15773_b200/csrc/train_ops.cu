// Host side of the operators of a training step (include/tsdp.h): checks of arguments, the plan of a launch, the launches.
// They need no context: every buffer is the caller's, every call only enqueues work on the caller's stream.
#include <cuda.h>
#include <cuda_runtime.h>

#include <atomic>
#include <cstdio>

#include "../../include/tsdp.h"
#include "checkpoint_kernels.cuh"
#include "group_norm_plan.cuh"
#include "weight_grad_tcgen05.cuh"

using namespace tsdp;

namespace {

constexpr int MAX_DEVICES = 64;
constexpr int MOST_ROWS = 1 << 30, MOST_CHANNELS = 1 << 24;      // of N and L, of C: counters step past them without leaving 32 bits

// The caller's device for the time of a call, the one that was current afterwards.
struct DeviceScope {
  int before = -1;
  cudaError_t err;
  explicit DeviceScope(int device) {
    err = cudaGetDevice(&before);
    if (err == cudaSuccess && before != device) err = cudaSetDevice(device);
    else if (err == cudaSuccess) before = -1;
  }
  ~DeviceScope() { if (before >= 0) cudaSetDevice(before); }
};

// tsdp_debug_arm_train_timeout: the limit of the next call's waits, 0 where there is none but the usual one.
thread_local long long armed_wait = 0;
struct Waits {
  long long cycles = GEMM_WAIT_CYCLES;
  int withhold = 0;
  Waits() { if (armed_wait) { cycles = armed_wait; withhold = 1; armed_wait = 0; } }
};

// (The runtime keeps an error until it is read, and the sampler's calls read it behind their launches: it would be taken for theirs.)
int fail_cuda(const char* what, cudaError_t e) {
  cudaGetLastError();
  fprintf(stderr, "%s: %s\n", what, cudaGetErrorString(e));
  return TSDP_ERR_CUDA;
}

int device_sms(int device) {
  static std::atomic<int> known[MAX_DEVICES];
  int n = known[device].load(std::memory_order_relaxed);
  if (n == 0) {
    if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, device) != cudaSuccess || n < 1) { n = 148; cudaGetLastError(); }
    known[device].store(n, std::memory_order_relaxed);
  }
  return n;
}

// Dynamic shared memory beyond 48 KB is asked for once per kernel and device.
template <typename F> cudaError_t allow_smem(F kern, int bytes, int device, std::atomic<unsigned long long>& done) {
  const unsigned long long bit = 1ull << device;
  if (done.load(std::memory_order_relaxed) & bit) return cudaSuccess;
  const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
  if (e == cudaSuccess) done.fetch_or(bit, std::memory_order_relaxed);
  return e;
}

// Every kernel here may be launched while its predecessor in the stream still drains (programmatic dependent launch): it begins with
// griddepcontrol.wait.
template <typename F, typename... A>
cudaError_t launch(F kern, unsigned grid, int threads, int cluster, int smem, cudaStream_t s, const A&... args) {
  cudaLaunchConfig_t cfg{};
  cudaLaunchAttribute at[2];
  cfg.gridDim = dim3(grid);
  cfg.blockDim = dim3((unsigned)threads);
  cfg.dynamicSmemBytes = (size_t)smem;
  cfg.stream = s;
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  at[1].id = cudaLaunchAttributeClusterDimension;
  at[1].val.clusterDim.x = (unsigned)cluster; at[1].val.clusterDim.y = 1; at[1].val.clusterDim.z = 1;
  cfg.attrs = at;
  cfg.numAttrs = cluster > 1 ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, kern, args...);
}

bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }
size_t esize(int dtype) { return dtype == TSDP_TYPE_BF16 ? 2 : 4; }
bool dtype_ok(int dtype) { return dtype == TSDP_TYPE_FP32 || dtype == TSDP_TYPE_BF16; }

// 16 bytes at a time: every row starts on a 16-byte boundary and holds whole 16-byte pieces.
bool rows_wide(const Rows& r, int dtype, int C) {
  const int v = 16 / (int)esize(dtype);
  return aligned16(r.p) && r.sn % v == 0 && r.sl % v == 0 && C % v == 0;
}
// A dimension of one element has no stride of its own.
Rows rows_of(const void* p, long long sn, long long sl, int N, int L, int C) {
  return Rows{const_cast<void*>(p), N > 1 ? sn : 0, L > 1 ? sl : (C + 7) / 8 * 8};
}
bool strides_ok(long long sn, long long sl) { return sn >= 0 && sl >= 0; }
// Rows that are written must not overlap.
bool rows_apart(long long N, long long L, int C, long long sn, long long sl) {
  if (L > 1 && sl < C) return false;
  if (N > 1 && sn < C) return false;
  if (N > 1 && L > 1) return sn >= (L - 1) * sl + C || sl >= (N - 1) * sn + C;
  return true;
}
bool copy_ok(const tsdp_saved_t* s) { return s != nullptr && s->q != nullptr && s->scale != nullptr; }
Copy8 copy_of(const tsdp_saved_t* s) { return s ? Copy8{reinterpret_cast<signed char*>(s->q), s->scale} : Copy8{nullptr, nullptr}; }

template <typename T>
cudaError_t pack(const Rows& x, Copy8 out, int N, int L, int C, int sms, cudaStream_t s) {
  const long long rows = (long long)N * L;
  const bool wide = rows_wide(x, sizeof(T) == 2 ? TSDP_TYPE_BF16 : TSDP_TYPE_FP32, C) && C % 8 == 0 && ((uintptr_t)out.q & 7) == 0;
  if (wide) {
    const int lanes = COPY_THREADS / min(4 * copy_blocks(C), COPY_THREADS);
    const long long blocks = min((rows + lanes - 1) / lanes, (long long)sms * 4);
    return launch(checkpoint_pack_kernel<T>, (unsigned)blocks, COPY_THREADS, 1, 0, s, x, out, N, L, C);
  }
  const long long blocks = min((rows * copy_blocks(C) + 7) / 8, (long long)sms * 64);
  return launch(checkpoint_pack_any_kernel<T>, (unsigned)blocks, COPY_THREADS, 1, 0, s, x, out, N, L, C);
}

template <typename T>
cudaError_t unpack(Copy8 in, const Rows& x, int N, int L, int C, int sms, cudaStream_t s) {
  const long long rows = (long long)N * L;
  const bool wide = rows_wide(x, sizeof(T) == 2 ? TSDP_TYPE_BF16 : TSDP_TYPE_FP32, C) && C % 8 == 0 && ((uintptr_t)in.q & 7) == 0;
  if (wide) {
    const int lanes = COPY_THREADS / min(C / 8, COPY_THREADS);
    const long long blocks = min((rows + lanes - 1) / lanes, (long long)sms * 4);
    return launch(checkpoint_unpack_kernel<T>, (unsigned)blocks, COPY_THREADS, 1, 0, s, in, x, N, L, C);
  }
  const long long blocks = min((rows * copy_blocks(C) + 7) / 8, (long long)sms * 64);
  return launch(checkpoint_unpack_any_kernel<T>, (unsigned)blocks, COPY_THREADS, 1, 0, s, in, x, N, L, C);
}

// ---------------------------------------------------------------------------------------------------------- GroupNorm
bool norm_ok(const tsdp_norm_t* n) {
  return n && dtype_ok(n->dtype) && n->N >= 0 && n->N <= MOST_ROWS && n->L >= 1 && n->L <= MOST_ROWS && n->C >= 1 && n->C <= MOST_CHANNELS && n->groups >= 1 && n->C % n->groups == 0 &&
         n->C / n->groups <= GN_MAX_WIDTH && n->act >= TSDP_ACT_NONE && n->act <= TSDP_ACT_GELU && n->eps > 0.f && n->eps < 1e30f;
}

template <typename T, int ITEMS>
cudaError_t norm_slab(const NormArgs& g, int smem, int device, cudaStream_t s) {
  static std::atomic<unsigned long long> done{0};
  const cudaError_t e = allow_smem(group_norm_slab_kernel<T, ITEMS>, SLAB_SMEM, device, done);
  return e != cudaSuccess ? e : launch(group_norm_slab_kernel<T, ITEMS>, (unsigned)(g.splits * g.sets), GN_THREADS, 1, smem, s, g);
}
template <typename T, int ITEMS, bool COPY>
cudaError_t norm_slab_grad(const NormArgs& g, int smem, int device, cudaStream_t s) {
  static std::atomic<unsigned long long> done{0};
  const cudaError_t e = allow_smem(group_norm_slab_grad_kernel<T, ITEMS, COPY>, SLAB_SMEM, device, done);
  return e != cudaSuccess ? e : launch(group_norm_slab_grad_kernel<T, ITEMS, COPY>, (unsigned)(g.splits * g.sets), GN_THREADS, 1, smem, s, g);
}

template <typename F>
cudaError_t launch_warps(F kern, const NormArgs& g, int smem, cudaStream_t s) {
  const long long warps = (long long)g.splits * g.groups * g.team;
  return launch(kern, (unsigned)((warps + GN_WARP_THREADS / 32 - 1) / (GN_WARP_THREADS / 32)), GN_WARP_THREADS, 1, smem, s, g);
}
template <typename T, int ITEMS, bool TEAM = false>
cudaError_t norm_warp_items(const NormArgs& g, int device, cudaStream_t s) {
  static std::atomic<unsigned long long> done{0};
  constexpr int per = GN_WARP_THREADS / 32 * GN_WARP_STAGES;
  const cudaError_t e = allow_smem(group_norm_warp_kernel<T, ITEMS, TEAM>, per * gn_warp_stage(ITEMS, 256), device, done);
  return e != cudaSuccess ? e : launch_warps(group_norm_warp_kernel<T, ITEMS, TEAM>, g, per * gn_warp_stage(ITEMS, g.C / g.groups), s);
}
// (a lane of a team holds more than half of the most it may: one form of it)
template <typename T>
cudaError_t norm_warp(const NormArgs& g, int items, int device, cudaStream_t s) {
  if (g.team > 1) return norm_warp_items<T, sizeof(T) == 2 ? 4 : 8, true>(g, device, s);
  if (items <= 1) return norm_warp_items<T, 1>(g, device, s);
  if (items <= 2) return norm_warp_items<T, 2>(g, device, s);
  if constexpr (sizeof(T) == 4)
    if (items > 4) return norm_warp_items<T, 8>(g, device, s);
  return norm_warp_items<T, 4>(g, device, s);
}
template <typename T, int ITEMS, bool COPY, bool TEAM = false>
cudaError_t norm_warp_grad_items(const NormArgs& g, int device, cudaStream_t s) {
  static std::atomic<unsigned long long> done{0};
  constexpr int smem = gn_warp_grad_smem<T, COPY>(ITEMS), film = 2 * GN_WARP_THREADS / 32 * 2 * 4;      // (film: a channel of a team)
  const cudaError_t e = allow_smem(group_norm_warp_grad_kernel<T, ITEMS, COPY, TEAM>, smem + film * 128, device, done);
  return e != cudaSuccess ? e : launch_warps(group_norm_warp_grad_kernel<T, ITEMS, COPY, TEAM>, g, smem + (TEAM && g.dfilm ? film * (g.C / g.groups) : 0), s);
}
template <typename T, bool COPY>
cudaError_t norm_warp_grad(const NormArgs& g, int items, int device, cudaStream_t s) {
  if (g.team > 1) return norm_warp_grad_items<T, sizeof(T) == 2 ? 8 : 4, COPY, true>(g, device, s);
  if (items <= 1) return norm_warp_grad_items<T, 1, COPY>(g, device, s);
  if (items <= 2) return norm_warp_grad_items<T, 2, COPY>(g, device, s);
  if constexpr (sizeof(T) == 2)
    if (items > 4) return norm_warp_grad_items<T, 8, COPY>(g, device, s);
  return norm_warp_grad_items<T, 4, COPY>(g, device, s);
}

// The vectors that slab kernels read in pairs or by bulk copies.
bool vectors_wide(const NormArgs& g) { return ((uintptr_t)g.gamma & 7) == 0 && ((uintptr_t)g.beta & 7) == 0 && (!g.film || aligned16(g.film)); }

// The three forms of the forward pass; the first two write the copies on their way.
enum { NORM_STREAM = 0, NORM_WARPS = 1, NORM_SLABS = 2 };
template <typename T, int V>
cudaError_t norm_stream(NormArgs& g, int sms, int device, cudaStream_t s) {
  norm_plan(g, V, sizeof(T), sms, false);
  static std::atomic<unsigned long long> done{0};
  const int smem = (2 * g.threads * V + 4 * g.per_set) * 4;
  const cudaError_t e = allow_smem(group_norm_kernel<T, V>, (2 * GN_THREADS * V + 4 * GN_MAX_WIDTH) * 4, device, done);
  return e != cudaSuccess ? e : launch(group_norm_kernel<T, V>, (unsigned)((long long)g.splits * g.sets * g.ranks), g.threads, g.ranks, smem, s, g);
}
template <typename T>
cudaError_t norm_forward(NormArgs& g, int form, bool wide, int items, int bytes, int sms, int device, cudaStream_t s) {
  if (form == NORM_WARPS) return norm_warp<T>(g, items, device, s);
  if (form == NORM_SLABS)
    return items <= 1 ? norm_slab<T, 1>(g, bytes, device, s) : (items <= 2 ? norm_slab<T, 2>(g, bytes, device, s) : norm_slab<T, 4>(g, bytes, device, s));
  return wide ? norm_stream<T, GN_STREAM_V>(g, sms, device, s) : norm_stream<T, 1>(g, sms, device, s);
}

enum { GRAD_STREAM = 0, GRAD_WARPS = 1, GRAD_SLABS = 2 };
template <typename T, int V, bool COPY>
cudaError_t norm_backward(NormArgs& g, int form, int items, int bytes, int device, cudaStream_t s) {
  if constexpr (V > 1) {
    if (form == GRAD_WARPS) return norm_warp_grad<T, COPY>(g, items, device, s);
    if (form == GRAD_SLABS)
      return items <= 1 ? norm_slab_grad<T, 1, COPY>(g, bytes, device, s)
                        : (items <= 2 ? norm_slab_grad<T, 2, COPY>(g, bytes, device, s) : norm_slab_grad<T, 4, COPY>(g, bytes, device, s));
  }
  static std::atomic<unsigned long long> done{0};
  const int smem = (4 * g.threads * V + 8 * g.width + 2 * g.per_set) * 4;
  const cudaError_t e = allow_smem(group_norm_grad_kernel<T, V, COPY>, (4 * GN_STREAM_THREADS * V + 10 * GN_MAX_WIDTH) * 4, device, done);
  return e != cudaSuccess ? e : launch(group_norm_grad_kernel<T, V, COPY>, (unsigned)((long long)g.splits * g.sets * g.ranks), g.threads, g.ranks, smem, s, g);
}

int norm_shares(const NormArgs& g) { return g.splits * max(1, g.team); }
size_t norm_grad_bytes(const NormArgs& g) { return (size_t)norm_shares(g) * 2 * g.C * 4; }

// ------------------------------------------------------------------------------------------------------ weight gradient
typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                                  const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
EncodeTiledFn encode_fn() {
  static std::atomic<void*> known{nullptr};
  void* fn = known.load(std::memory_order_relaxed);
  if (!fn) {
    cudaDriverEntryPointQueryResult q;
    if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &fn, cudaEnableDefault, &q) != cudaSuccess || q != cudaDriverEntryPointSuccess) return nullptr;
    known.store(fn, std::memory_order_relaxed);
  }
  return reinterpret_cast<EncodeTiledFn>(fn);
}

struct WgradPlan { int bn, cg, units; size_t share_bytes, bytes; };

// pair: the two-CTA form may be taken (dy and q by TMA).
WgradPlan wgrad_plan(WgradArgs& g, bool fp32, bool pair, int sms) {
  WgradPlan p;
  p.bn = g.O <= 64 ? 64 : (g.O <= 128 || fp32 ? 128 : 256);
  const int k128 = (g.K + WG_BM - 1) / WG_BM;
  g.stages = (int)((g.M + WG_BK - 1) / WG_BK);
  // narrower tiles where there are too few steps for the SMs (us, 256 -> 64 wide: 384 x 128 -> 512 10.5 -> 8.7, 16 x 256 -> 1024 18.1 -> 9.5)
  while (p.bn > 64 && (long long)g.stages * g.taps * k128 * ((g.O + p.bn - 1) / p.bn) < sms) p.bn /= 2;
  g.tiles_o = (g.O + p.bn - 1) / p.bn;
  // pairs where 256-wide tiles leave little of K unused and the line keeps them busy
  p.cg = pair && !fp32 && p.bn == 256 && (k128 % 2 == 0 || k128 >= 7) && (long long)g.stages * g.taps * (k128 / 2) * g.tiles_o >= 16ll * sms ? 2 : 1;
  g.tiles_k = (k128 + p.cg - 1) / p.cg;
  const long long tiles = (long long)g.taps * g.tiles_k * g.tiles_o, line = g.stages * tiles;
  g.line = line < (1ll << 31) - 4096 && 32 * tiles < (1ll << 31) ? (int)line : 0;
  p.units = (int)min((long long)(sms / p.cg), max(1ll, line / 2));
  p.share_bytes = (size_t)2 * p.units * p.cg * WG_BM * p.bn * 4;
  p.bytes = p.share_bytes + (size_t)(p.units + tiles) * p.cg * WG_BIAS * 4;
  return p;
}

template <int BN, int DYK, int CG>
cudaError_t wgrad_launch(const CUtensorMap& map, const CUtensorMap& qmap, const WgradArgs& g, int units, int device, cudaStream_t s) {
  static std::atomic<unsigned long long> done{0};
  constexpr int smem = wg_smem_bytes(BN, DYK, CG);
  cudaError_t e = allow_smem(weight_grad_kernel<BN, DYK, CG>, smem, device, done);
  if (e != cudaSuccess) return e;
  e = launch(weight_grad_kernel<BN, DYK, CG>, (unsigned)(units * CG), WG_THREADS, CG, smem, s, map, qmap, g);
  if (e != cudaSuccess) return e;
  const int tiles = g.taps * g.tiles_k * g.tiles_o;
  const int db = g.db ? g.tiles_o * (BN / 8) : 0;
  // owners of a tile that a join's thread reads in turn; with many of them groups of threads read side by side (us, groups of 1 / 4 / 8:
  // 16384 x 512 -> 512 with 5 taps, 3.7 owners, 57 / 63 / 75; 1024 x 256 -> 256 with 5 taps, 8 owners, 14.8 / 13.3 / 17.5;
  // 45056 x 512 -> 256, 37 owners, 45 / 28.6 / 31.5; 45056 x 256 -> 256, 74 owners, 54 / 21.9 / 19.3)
  const int split = units <= 6 * tiles ? 1 : units <= 40 * tiles ? 4 : 8;
  return launch(split == 1 ? weight_grad_join_kernel<BN, CG, 1> : split == 4 ? weight_grad_join_kernel<BN, CG, 4> : weight_grad_join_kernel<BN, CG, 8>,
                (unsigned)(tiles * (BN / 16 * CG) * (split == 1 ? 1 : 2 * split) + db), 256, 1, 0, s, g, units, tiles);
}

bool wgrad_ok(int dtype, long long N, int L, int K, int O, int taps) {
  return dtype_ok(dtype) && N >= 0 && L >= 1 && K >= 1 && O >= 1 && K <= (1 << 20) && O <= (1 << 20) && taps >= 1 && taps <= TSDP_MAX_TAPS &&
         (taps & 1) == 1 && N * L < (1ll << 31) - 64 && (long long)taps * K * O < (1ll << 40);
}

}  // namespace

extern "C" {

int tsdp_debug_arm_train_timeout(long long wait_cycles) {
  if (wait_cycles < 1000 || wait_cycles > GEMM_WAIT_CYCLES) return TSDP_ERR_ARG;
  armed_wait = wait_cycles;
  return TSDP_OK;
}

int tsdp_checkpoint_pack(int device, int dtype, const void* d_x, int64_t x_n, int64_t x_l, int N, int L, int C, const tsdp_saved_t* out, void* stream) {
  if (device < 0 || device >= MAX_DEVICES || !dtype_ok(dtype) || N < 0 || N > MOST_ROWS || L < 0 || L > MOST_ROWS || C < 1 || C > MOST_CHANNELS || !strides_ok(x_n, x_l)) return TSDP_ERR_ARG;
  if (N == 0 || L == 0) return TSDP_OK;
  if (!d_x || !copy_ok(out)) return TSDP_ERR_ARG;
  DeviceScope scope(device);
  if (scope.err != cudaSuccess) return fail_cuda("tsdp_checkpoint_pack", scope.err);
  const Rows x = rows_of(d_x, x_n, x_l, N, L, C);
  const int sms = device_sms(device);
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  const cudaError_t e = dtype == TSDP_TYPE_BF16 ? pack<__nv_bfloat16>(x, copy_of(out), N, L, C, sms, s) : pack<float>(x, copy_of(out), N, L, C, sms, s);
  return e == cudaSuccess ? TSDP_OK : fail_cuda("tsdp_checkpoint_pack", e);
}

int tsdp_checkpoint_unpack(int device, int dtype, const tsdp_saved_t* in, void* d_x, int64_t x_n, int64_t x_l, int N, int L, int C, void* stream) {
  if (device < 0 || device >= MAX_DEVICES || !dtype_ok(dtype) || N < 0 || N > MOST_ROWS || L < 0 || L > MOST_ROWS || C < 1 || C > MOST_CHANNELS || !strides_ok(x_n, x_l)) return TSDP_ERR_ARG;
  if (N == 0 || L == 0) return TSDP_OK;
  if (!d_x || !copy_ok(in) || !rows_apart(N, L, C, x_n, x_l)) return TSDP_ERR_ARG;
  DeviceScope scope(device);
  if (scope.err != cudaSuccess) return fail_cuda("tsdp_checkpoint_unpack", scope.err);
  const Rows x = rows_of(d_x, x_n, x_l, N, L, C);
  const int sms = device_sms(device);
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  const cudaError_t e = dtype == TSDP_TYPE_BF16 ? unpack<__nv_bfloat16>(copy_of(in), x, N, L, C, sms, s) : unpack<float>(copy_of(in), x, N, L, C, sms, s);
  return e == cudaSuccess ? TSDP_OK : fail_cuda("tsdp_checkpoint_unpack", e);
}

int tsdp_group_norm(int device, const tsdp_norm_t* shape, const void* d_x, int64_t x_n, int64_t x_l, const float* d_gamma, const float* d_beta,
                    const float* d_film, void* d_y, int64_t y_n, int64_t y_l, float* d_mean, float* d_rstd, const tsdp_saved_t* saved_x,
                    const tsdp_saved_t* saved_y, void* stream) {
  if (device < 0 || device >= MAX_DEVICES || !norm_ok(shape) || !strides_ok(x_n, x_l) || !strides_ok(y_n, y_l)) return TSDP_ERR_ARG;
  if (shape->N == 0) return TSDP_OK;                      // (empty copies have no addresses)
  if ((saved_x && !copy_ok(saved_x)) || (saved_y && !copy_ok(saved_y))) return TSDP_ERR_ARG;
  if (!d_x || !d_gamma || !d_beta || !d_y || !rows_apart(shape->N, shape->L, shape->C, y_n, y_l)) return TSDP_ERR_ARG;
  DeviceScope scope(device);
  if (scope.err != cudaSuccess) return fail_cuda("tsdp_group_norm", scope.err);
  const int sms = device_sms(device), dtype = shape->dtype, N = shape->N, L = shape->L, C = shape->C;
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  NormArgs g{};
  g.N = N; g.L = L; g.C = C; g.groups = shape->groups; g.act = shape->act; g.eps = shape->eps;
  const Waits waits;
  g.wait_cycles = waits.cycles; g.withhold = waits.withhold;
  g.x = rows_of(d_x, x_n, x_l, N, L, C);
  g.y = rows_of(d_y, y_n, y_l, N, L, C);
  g.gamma = d_gamma; g.beta = d_beta; g.film = d_film; g.mean = d_mean; g.rstd = d_rstd;
  const Copy8 cx = copy_of(saved_x), cy = copy_of(saved_y);
  const bool wide = rows_wide(g.x, dtype, C) && rows_wide(g.y, dtype, C) && set_fits(C, g.groups, 16 / (int)esize(dtype));
  int form = NORM_STREAM, items = 0, bytes = 0;
  if (wide && vectors_wide(g) && ((uintptr_t)cx.q & 7) == 0 && ((uintptr_t)cy.q & 7) == 0) {
    const int V = 16 / (int)esize(dtype), unit = set_fits(C, g.groups, 32) ? 32 : V;      // (with or without copies: the same plan, the same bits)
    if (warp_plan(g, V, 32 / V, 3, sms, items)) form = NORM_WARPS;
    else if ((unit == 32 || (!cx.q && !cy.q)) && slab_plan(g, V, unit, (int)esize(dtype), sms, false, false, items, bytes) &&
             slab_rows(g, g.x, (int)esize(dtype)))
      form = NORM_SLABS;
  }
  // copies are written on the way by the forms that hold a group, by a pass of their own otherwise
  cudaError_t e = cudaSuccess;
  if (form != NORM_STREAM) { g.cx = cx; g.cy = cy; }
  else if (cx.q) e = dtype == TSDP_TYPE_BF16 ? pack<__nv_bfloat16>(g.x, cx, N, L, C, sms, s) : pack<float>(g.x, cx, N, L, C, sms, s);
  if (e == cudaSuccess) {
    e = dtype == TSDP_TYPE_BF16 ? norm_forward<__nv_bfloat16>(g, form, wide, items, bytes, sms, device, s) : norm_forward<float>(g, form, wide, items, bytes, sms, device, s);
  }
  if (e == cudaSuccess && form == NORM_STREAM && cy.q)
    e = dtype == TSDP_TYPE_BF16 ? pack<__nv_bfloat16>(g.y, cy, N, L, C, sms, s) : pack<float>(g.y, cy, N, L, C, sms, s);
  return e == cudaSuccess ? TSDP_OK : fail_cuda("tsdp_group_norm", e);
}

// (the plan depends on the alignment of what a call is given: the largest of all)
size_t tsdp_group_norm_grad_workspace(int device, const tsdp_norm_t* shape) {
  if (device < 0 || device >= MAX_DEVICES || !norm_ok(shape)) return 0;
  size_t most = 16;
  const int elem = (int)esize(shape->dtype), sms = device_sms(device);
  for (int form = 0; form < 7; ++form) {                 // one value at a time, 16 bytes, four forms of slabs, warps
    const int V = form == 0 ? 1 : 16 / elem;                 // (form 1: 16 bytes, form 0: one value at a time)
    if (!set_fits(shape->C, shape->groups, V)) continue;
    NormArgs g{};
    float some;
    int items, bytes;
    g.N = shape->N < 1 ? 1 : shape->N; g.L = shape->L; g.C = shape->C; g.groups = shape->groups;
    g.dfilm = form & 1 ? &some : nullptr;
    if (form < 2) norm_plan(g, form == 0 ? 1 : GN_STREAM_V, elem, sms, true);
    else if (form == 6 ? !warp_plan(g, GN_STREAM_V, elem == 2 ? 8 : 4, 2, sms, items) : !slab_plan(g, GN_STREAM_V, V, elem, sms, true, form >= 4, items, bytes)) continue;
    if (norm_grad_bytes(g) > most) most = norm_grad_bytes(g);
  }
  return most;
}

int tsdp_group_norm_grad(int device, const tsdp_norm_t* shape, const void* d_dy, int64_t dy_n, int64_t dy_l, const void* d_x, int64_t x_n, int64_t x_l,
                         const tsdp_saved_t* saved_x, const float* d_gamma, const float* d_beta, const float* d_film, const float* d_mean,
                         const float* d_rstd, void* d_dx, int64_t dx_n, int64_t dx_l, float* d_dgamma, float* d_dbeta, float* d_dfilm,
                         void* d_workspace, size_t workspace_bytes, void* stream) {
  if (device < 0 || device >= MAX_DEVICES || !norm_ok(shape) || !strides_ok(dy_n, dy_l) || !strides_ok(x_n, x_l) || !strides_ok(dx_n, dx_l) ||
      !d_dgamma || !d_dbeta || (d_dfilm && !d_film))
    return TSDP_ERR_ARG;
  DeviceScope scope(device);
  if (scope.err != cudaSuccess) return fail_cuda("tsdp_group_norm_grad", scope.err);
  const int sms = device_sms(device), dtype = shape->dtype, C = shape->C;
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  cudaError_t e;
  if (shape->N == 0) {
    e = cudaMemsetAsync(d_dgamma, 0, (size_t)C * 4, s);
    if (e == cudaSuccess) e = cudaMemsetAsync(d_dbeta, 0, (size_t)C * 4, s);
    return e == cudaSuccess ? TSDP_OK : fail_cuda("tsdp_group_norm_grad", e);
  }
  if (!d_dy || (saved_x ? !copy_ok(saved_x) : !d_x) || !d_gamma || !d_beta || !d_mean || !d_rstd || !d_dx || !d_workspace || ((uintptr_t)d_workspace & 3) ||
      !rows_apart(shape->N, shape->L, C, dx_n, dx_l))
    return TSDP_ERR_ARG;
  NormArgs g{};
  g.N = shape->N; g.L = shape->L; g.C = C; g.groups = shape->groups; g.act = shape->act; g.eps = shape->eps;
  const Waits waits;
  g.wait_cycles = waits.cycles; g.withhold = waits.withhold;
  g.x = rows_of(d_x, x_n, x_l, g.N, g.L, C);
  g.dy = rows_of(d_dy, dy_n, dy_l, g.N, g.L, C);
  g.dx = rows_of(d_dx, dx_n, dx_l, g.N, g.L, C);
  g.gamma = d_gamma; g.beta = d_beta; g.film = d_film; g.mean = const_cast<float*>(d_mean); g.rstd = const_cast<float*>(d_rstd);
  g.dfilm = d_dfilm;
  g.cx = copy_of(saved_x);
  g.part = reinterpret_cast<float*>(d_workspace);
  const bool copy = saved_x != nullptr;
  const bool wide = set_fits(C, g.groups, 16 / (int)esize(dtype)) && rows_wide(g.dy, dtype, C) && rows_wide(g.dx, dtype, C) && (copy ? ((uintptr_t)g.cx.q & 7) == 0 : rows_wide(g.x, dtype, C));
  const int V = wide ? 16 / (int)esize(dtype) : 1;
  int items = 0, bytes = 0;
  int form = GRAD_STREAM;
  if (wide && vectors_wide(g) && ((uintptr_t)d_dfilm & 7) == 0 && ((uintptr_t)d_workspace & 7) == 0) {
    if ((!copy || aligned16(g.cx.q)) && warp_plan(g, GN_STREAM_V, dtype == TSDP_TYPE_BF16 ? 8 : 4, 2, sms, items)) form = GRAD_WARPS;
    else if ((!copy || aligned16(g.cx.q)) && slab_plan(g, GN_STREAM_V, V, (int)esize(dtype), sms, true, copy, items, bytes) &&
             slab_rows(g, g.dy, (int)esize(dtype)))
      form = GRAD_SLABS;
  }
  if (form == GRAD_STREAM) norm_plan(g, wide ? GN_STREAM_V : 1, (int)esize(dtype), sms, true);
  if (workspace_bytes < norm_grad_bytes(g)) return TSDP_ERR_ARG;
  if (dtype == TSDP_TYPE_BF16) {
    if (wide) e = copy ? norm_backward<__nv_bfloat16, 4, true>(g, form, items, bytes, device, s) : norm_backward<__nv_bfloat16, 4, false>(g, form, items, bytes, device, s);
    else e = copy ? norm_backward<__nv_bfloat16, 1, true>(g, form, items, bytes, device, s) : norm_backward<__nv_bfloat16, 1, false>(g, form, items, bytes, device, s);
  } else {
    if (wide) e = copy ? norm_backward<float, 4, true>(g, form, items, bytes, device, s) : norm_backward<float, 4, false>(g, form, items, bytes, device, s);
    else e = copy ? norm_backward<float, 1, true>(g, form, items, bytes, device, s) : norm_backward<float, 1, false>(g, form, items, bytes, device, s);
  }
  if (e == cudaSuccess) {
    e = launch(group_norm_join_kernel, (unsigned)(2 * ((C + GN_JOIN_CH - 1) / GN_JOIN_CH)), GN_JOIN_CH * GN_JOIN_LANES, 1, 0, s, (const float*)g.part, norm_shares(g), C, d_dgamma, d_dbeta);
  }
  return e == cudaSuccess ? TSDP_OK : fail_cuda("tsdp_group_norm_grad", e);
}

size_t tsdp_weight_grad_workspace(int device, int dtype, int N, int L, int K, int O, int taps) {
  if (device < 0 || device >= MAX_DEVICES || !wgrad_ok(dtype, N, L, K, O, taps)) return 0;
  WgradArgs g{};
  g.M = (long long)(N < 1 ? 1 : N) * L; g.K = K; g.O = O; g.taps = taps;
  size_t most = 0;
  for (bool pair : {false, true}) {                      // (which of them a call takes depends on alignment)
    const WgradPlan p = wgrad_plan(g, dtype == TSDP_TYPE_FP32, pair, device_sms(device));
    if (g.line == 0) return 0;
    if (p.bytes > most) most = p.bytes;
  }
  return most;
}

int tsdp_weight_grad(int device, int dtype, const tsdp_saved_t* saved_x, const void* d_dy, int64_t dy_l, int N, int L, int K, int O, int taps, float* d_dW,
                     float* d_db, void* d_workspace, size_t workspace_bytes, void* stream) {
  if (device < 0 || device >= MAX_DEVICES || !wgrad_ok(dtype, N, L, K, O, taps) || !d_dW || dy_l < 0) return TSDP_ERR_ARG;
  DeviceScope scope(device);
  if (scope.err != cudaSuccess) return fail_cuda("tsdp_weight_grad", scope.err);
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  cudaError_t e;
  if (N == 0) {
    e = cudaMemsetAsync(d_dW, 0, (size_t)taps * K * O * 4, s);
    if (e == cudaSuccess && d_db) e = cudaMemsetAsync(d_db, 0, (size_t)O * 4, s);
    return e == cudaSuccess ? TSDP_OK : fail_cuda("tsdp_weight_grad", e);
  }
  if (!copy_ok(saved_x) || !d_dy || !d_workspace || !aligned16(d_workspace)) return TSDP_ERR_ARG;
  WgradArgs g{};
  const Waits waits;
  g.wait_cycles = waits.cycles; g.withhold = waits.withhold;
  g.x = copy_of(saved_x);
  g.dy = d_dy; g.ldy = dy_l;
  g.M = (long long)N * L; g.L = L; g.K = K; g.O = O; g.taps = taps;
  g.dW = d_dW;
  const bool fp32 = dtype == TSDP_TYPE_FP32;
  const bool tma = !fp32 && aligned16(d_dy) && dy_l % 8 == 0 && dy_l >= O && dy_l < (1ll << 38);
  g.q_tma = K % 16 == 0 && aligned16(g.x.q);
  const WgradPlan p = wgrad_plan(g, fp32, tma && g.q_tma, device_sms(device));
  if (g.line == 0 || workspace_bytes < p.bytes) return TSDP_ERR_ARG;
  g.share = reinterpret_cast<float*>(d_workspace);
  g.db = d_db;
  g.bias = reinterpret_cast<float*>(reinterpret_cast<char*>(d_workspace) + p.share_bytes);
  CUtensorMap map{}, qmap{};
  EncodeTiledFn encode = encode_fn();
  if (!encode) { fprintf(stderr, "tsdp_weight_grad: cuTensorMapEncodeTiled unavailable\n"); return TSDP_ERR_CUDA; }
  auto tiled = [&](CUtensorMap* m, const void* p2, bool bf16, int cols, long long pitch, int box_cols) {      // rows x cols, boxes of 64 rows
    cuuint64_t gdim[2] = {(cuuint64_t)cols, (cuuint64_t)g.M}, gstr[1] = {(cuuint64_t)pitch};
    cuuint32_t box[2] = {(cuuint32_t)box_cols, WG_BK}, estr[2] = {1, 1};
    return encode(m, bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void*>(p2), gdim, gstr, box, estr,
                  CU_TENSOR_MAP_INTERLEAVE_NONE, bf16 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_128B,
                  CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  };
  CUresult r = CUDA_SUCCESS;
  if (tma) r = tiled(&map, d_dy, true, O, dy_l * 2, 64);
  if (r == CUDA_SUCCESS && g.q_tma) r = tiled(&qmap, g.x.q, false, K, K, WG_BM);
  if (r != CUDA_SUCCESS) { fprintf(stderr, "tsdp_weight_grad: cuTensorMapEncodeTiled failed with code %d\n", (int)r); return TSDP_ERR_CUDA; }
  if (fp32) e = p.bn == 64 ? wgrad_launch<64, WG_DY_FP32, 1>(map, qmap, g, p.units, device, s) : wgrad_launch<128, WG_DY_FP32, 1>(map, qmap, g, p.units, device, s);
  else if (p.cg == 2) e = wgrad_launch<256, WG_DY_TMA, 2>(map, qmap, g, p.units, device, s);
  else if (p.bn == 64) e = tma ? wgrad_launch<64, WG_DY_TMA, 1>(map, qmap, g, p.units, device, s) : wgrad_launch<64, WG_DY_BF16, 1>(map, qmap, g, p.units, device, s);
  else if (p.bn == 128) e = tma ? wgrad_launch<128, WG_DY_TMA, 1>(map, qmap, g, p.units, device, s) : wgrad_launch<128, WG_DY_BF16, 1>(map, qmap, g, p.units, device, s);
  else e = tma ? wgrad_launch<256, WG_DY_TMA, 1>(map, qmap, g, p.units, device, s) : wgrad_launch<256, WG_DY_BF16, 1>(map, qmap, g, p.units, device, s);
  return e == cudaSuccess ? TSDP_OK : fail_cuda("tsdp_weight_grad", e);
}

}  // extern "C"
