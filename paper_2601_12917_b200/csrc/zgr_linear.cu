// The linear layer of the forward pass in 8 bits: rows quantised with a scale each, the matrix product of two such matrices, and its epilogue.
//
//   quantise   a = max_k |x_k|,  scale = a (1/127),  code_k = rint(x_k (127 (1/a)))        per row (a token, or a channel's weights)
//              (products with fp32 reciprocals by definition; quotients give another code to 4 of 10 million fp32 and 2 of 100 000 16-bit normals,
//              all within 127 * 3.01 * 2^-24 of a border between two codes)
//   product    y[m][n] = residual[m][n] + D( (sum_k qx[m][k] qw[n][k]) * (sx[m] sw[n]) + bias[n] ),   D: dropout, or nothing
//
// The sums are 32-bit integers and exact; everything behind them is fp32, rounded once to the storage type.
#include <cuda.h>
#include <cuda_runtime.h>

#include <algorithm>

#include "zgr.h"
#include "zgr_forward.cuh"
#include "zgr_host_internal.h"
#include "zgr_tcgen05.cuh"

namespace zgr {
namespace {

// Status word of the kernels below (per device; 0 = healthy): where a bounded wait gave up.
__device__ int g_linear_error = 0;

// ---------------------------------------------------------------------------------------------
// Rows to codes.  Bound by memory: the row is read once and stays in registers between the two passes over it.
// ---------------------------------------------------------------------------------------------
constexpr uint32_t kTinyBits = 0x03800000u;      // 2^-120: a row whose largest magnitude is below it counts as zero (127 (1/a) stays finite)
constexpr uint32_t kInfBits = 0x7F800000u;

struct RowScale {
  float scale, inv;
  bool zero;             // all codes are 0
};
// From the largest magnitude's bits.  (Magnitudes as unsigned integers: NaN ranks above infinity, so that one of either shows.)
__device__ __forceinline__ RowScale row_scale(uint32_t amax_bits) {
  RowScale r;
  const float a = __uint_as_float(amax_bits);
  r.zero = amax_bits < kTinyBits || amax_bits >= kInfBits;
  r.inv = r.zero ? 0.0f : __fmul_rn(__frcp_rn(a), 127.0f);
  r.scale = amax_bits < kTinyBits ? 0.0f : (amax_bits >= kInfBits ? __uint_as_float(0x7FC00000u) : __fmul_rn(a, 1.0f / 127.0f));
  return r;
}
// rint(fl(x inv)) in the low byte: adding 1.5 * 2^23 leaves the nearest integer (ties to even) in the low bits.  The product and the sum
// are two roundings by definition (not a fused multiply-add).  |x inv| <= 127 (1 + 2^-20), so that no code is above 127.
__device__ __forceinline__ uint32_t code_of(float x, float inv) { return __float_as_uint(__fadd_rn(__fmul_rn(x, inv), 12582912.0f)) & 0xFFu; }
__device__ __forceinline__ uint32_t code4(const float* v, float inv) {
  const uint32_t a = __float_as_uint(__fadd_rn(__fmul_rn(v[0], inv), 12582912.0f)), b = __float_as_uint(__fadd_rn(__fmul_rn(v[1], inv), 12582912.0f));
  const uint32_t c = __float_as_uint(__fadd_rn(__fmul_rn(v[2], inv), 12582912.0f)), d = __float_as_uint(__fadd_rn(__fmul_rn(v[3], inv), 12582912.0f));
  return __byte_perm(__byte_perm(a, b, 0x0040), __byte_perm(c, d, 0x0040), 0x5410);
}
__device__ __forceinline__ uint32_t magnitude(float v) { return __float_as_uint(v) & 0x7FFFFFFFu; }

// A row is read once and stays in registers between the two passes over it, NV octets a thread, as few as hold it (idle lanes cost as much as
// the others).  ROWS = 4: four warps a block with a row each, up to 1536 elements; ROWS = 1: a block a row, with four, eight or twelve
// warps, at most six octets a thread; 16-bit rows in as few registers as leave room for three blocks of 384 threads.  4096 rows of 11008
// bf16 elements: 26 us (5.2 TB/s; 29 without that bound, 34 with sixteen warps and three octets or with eleven and four), 13824 of 5120 35 us
// (6.0 TB/s), 4096 of 4096 10.2 us.  Bound by memory and, in the last, by one wave of blocks that all load, reduce and store at once.
// The rows of x may start anywhere (ALIGNED = false: octets are put together from 16-byte granules, one by one at the row's ends), as may
// those of the codes (`wide` = 0: written byte by byte).
// early: the kernel behind this one is the library's product, which may start and wait; the caller's own kernels may not.
constexpr int row_threads(int rows) { return rows == 4 ? 128 : 384; }
template <typename T, int ROWS, int NV, bool ALIGNED>
__global__ void __launch_bounds__(row_threads(ROWS), ALIGNED && sizeof(T) == 2 && ROWS == 1 ? 3 : 1)
    quantize_rows_kernel(const T* x, const int64_t ldx, const int64_t rows, const int cols, int8_t* codes, const int64_t ldc, float* scales, const int wide,
                         const int early) {
  __shared__ uint32_t part[16];
  dependency_wait();
  if (early) dependents_may_start();
  const int threads = ROWS == 4 ? 32 : blockDim.x, t = ROWS == 4 ? threadIdx.x & 31 : threadIdx.x;
  const int64_t row = ROWS == 4 ? static_cast<int64_t>(blockIdx.x) * 4 + (threadIdx.x >> 5) : blockIdx.x;
  if (ROWS == 4 && row >= rows) return;                        // (whole warps)
  const T* src = x + row * ldx;
  Octet<T> raw[NV];
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int c = (t + i * threads) * 8;
    raw[i].zero();
    if (ALIGNED) {
      if (c + 8 <= cols) raw[i].load(src + c);
    } else if (c + 8 <= cols && Octet<T>::load_any_ok(src + c, src, src + cols)) {
      raw[i].load_any(src + c);
    } else if (c < cols) {
      raw[i].gather(src, c, cols);                             // (behind the end: the row's last element again, which changes no maximum)
    }
  }
  uint32_t amax = 0;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int c = (t + i * threads) * 8;
    if (ALIGNED && c < cols && c + 8 > cols) raw[i].gather(src, c, cols);
    float v[8];
    raw[i].unpack(v);
#pragma unroll
    for (int j = 0; j < 8; ++j) amax = max(amax, magnitude(v[j]));
  }
  amax = __reduce_max_sync(0xFFFFFFFFu, amax);
  if (ROWS == 1) {
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = amax;
    __syncthreads();
    for (int w = 0; w < threads / 32; ++w) amax = max(amax, part[w]);
  }
  const RowScale rs = row_scale(amax);
  if (t == 0) scales[row] = rs.scale;
  int8_t* dst = codes + row * ldc;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int c = (t + i * threads) * 8;
    float v[8];
    raw[i].unpack(v);
    const uint2 q = rs.zero ? make_uint2(0, 0) : make_uint2(code4(v, rs.inv), code4(v + 4, rs.inv));
    if (wide && c + 8 <= cols) {
      *reinterpret_cast<uint2*>(dst + c) = q;
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (c + j < cols) dst[c + j] = static_cast<int8_t>((j < 4 ? q.x : q.y) >> (8 * (j & 3)));
    }
  }
}

// Rows of more than 18432 elements: read twice, a block a row.
constexpr int64_t kLongRow = 18432;
template <typename T>
__global__ void __launch_bounds__(512) quantize_long_rows_kernel(const T* x, const int64_t ldx, const int64_t cols, int8_t* codes,
                                                                 const int64_t ldc, float* scales, const int early) {
  __shared__ uint32_t part[16];
  dependency_wait();
  if (early) dependents_may_start();
  const int64_t row = blockIdx.x;
  const T* src = x + row * ldx;
  uint32_t amax = 0;
#pragma unroll 8
  for (int64_t c = threadIdx.x; c < cols; c += 512) amax = max(amax, magnitude(Storage<T>::load1(src + c)));
  amax = __reduce_max_sync(0xFFFFFFFFu, amax);
  if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = amax;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < 16; ++w) amax = max(amax, part[w]);
  const RowScale rs = row_scale(amax);
  if (threadIdx.x == 0) scales[row] = rs.scale;
#pragma unroll 8
  for (int64_t c = threadIdx.x; c < cols; c += 512) codes[row * ldc + c] = static_cast<int8_t>(rs.zero ? 0 : code_of(Storage<T>::load1(src + c), rs.inv));
}

template <typename T, int ROWS, int NV>
cudaError_t launch_rows(const T* x, int64_t ldx, int64_t rows, int64_t cols, int8_t* codes, int64_t ldc, float* scales, int early, cudaStream_t st) {
  const unsigned grid = static_cast<unsigned>((rows + ROWS - 1) / ROWS);
  const int threads = ROWS == 4 ? 128 : static_cast<int>((cols + 6143) / 6144) * 128;
  const int wide = aligned_to(codes, 8) && (rows <= 1 || ldc % 8 == 0);
  const auto kernel = octets_aligned(x, rows, ldx, sizeof(T)) ? quantize_rows_kernel<T, ROWS, NV, true> : quantize_rows_kernel<T, ROWS, NV, false>;
  return launch_behind(kernel, grid, threads, 0, 1, st, x, ldx, rows, static_cast<int>(cols), codes, ldc, scales, wide, early);
}

template <typename T>
cudaError_t run_quantize(const void* x, int64_t ldx, int64_t rows, int64_t cols, int8_t* codes, int64_t ldc, float* scales, int early, cudaStream_t st) {
  const T* p = static_cast<const T*>(x);
  if (cols <= 1536) {
    constexpr decltype(&launch_rows<T, 4, 1>) by_octets[] = {launch_rows<T, 4, 1>, launch_rows<T, 4, 2>, launch_rows<T, 4, 3>,
                                                             launch_rows<T, 4, 4>, launch_rows<T, 4, 5>, launch_rows<T, 4, 6>};
    return by_octets[(cols + 255) / 256 - 1](p, ldx, rows, cols, codes, ldc, scales, early, st);
  }
  if (cols <= kLongRow) {
    constexpr decltype(&launch_rows<T, 1, 2>) by_octets[] = {launch_rows<T, 1, 2>, launch_rows<T, 1, 3>, launch_rows<T, 1, 4>, launch_rows<T, 1, 5>, launch_rows<T, 1, 6>};
    const int64_t a_turn = (cols + 6143) / 6144 * 1024;      // elements that the block's threads hold an octet each of
    return by_octets[(cols + a_turn - 1) / a_turn - 2](p, ldx, rows, cols, codes, ldc, scales, early, st);
  }
  return launch_behind(quantize_long_rows_kernel<T>, static_cast<unsigned>(rows), 512, 0, 1, st, p, ldx, cols, codes, ldc, scales, early);
}
cudaError_t run_quantize(int32_t dtype, const void* x, int64_t ldx, int64_t rows, int64_t cols, int8_t* codes, int64_t ldc, float* scales, int early,
                         cudaStream_t st) {
  switch (dtype) {
    case ZGR_F32: return run_quantize<float>(x, ldx, rows, cols, codes, ldc, scales, early, st);
    case ZGR_F16: return run_quantize<__half>(x, ldx, rows, cols, codes, ldc, scales, early, st);
    default: return run_quantize<__nv_bfloat16>(x, ldx, rows, cols, codes, ldc, scales, early, st);
  }
}

// ---------------------------------------------------------------------------------------------
// What the product's kernels share.
// ---------------------------------------------------------------------------------------------
struct LinearArgs {
  const void* x;         // few tokens: m x k in the storage type, quantised by every block for itself
  int64_t ldx;
  const float* sx;       // m (product of codes)
  const int8_t* w;       // n x k codes
  int64_t ldw;
  const float* sw;       // n
  const void* bias;      // n, or null
  const void* residual;  // m x n, or null
  int64_t ldr;
  void* y;               // m x n
  int64_t ldy;
  int64_t m, n;
  int32_t k;
  DropMask mask;         // threshold 0: nothing is dropped
};

template <typename T>
__device__ __forceinline__ float load_one(const void* p, int64_t i) {
  return Storage<T>::load1(static_cast<const T*>(p) + i);
}

// One result from its sum.  The rounding of every step is spelled out, so that both kernels give a token the same bits.
__device__ __forceinline__ float finish1(int sum, float sx, float sw, float bias, float residual, bool keep, float drop_scale, bool drop) {
  float v = fmaf(static_cast<float>(sum), __fmul_rn(sx, sw), bias);
  if (drop) v = keep ? __fmul_rn(v, drop_scale) : 0.0f;
  return __fadd_rn(v, residual);
}

// ---------------------------------------------------------------------------------------------
// Few tokens (up to eight): the weights are read once and nothing else counts.  A block on every multiprocessor; each warp takes channels in turn and
// streams their codes through slots of its own in shared memory: one lane starts bulk copies of up to 4096 bytes, two to eight of them
// ahead (about 190 KB in flight on a multiprocessor, whatever the number of registers), all lanes multiply them with the tokens' codes, four
// products an instruction.  The sums of 32 channels wait in the 32 lanes for one epilogue.  Every block quantises the tokens for itself, its
// warps shared out among them, while its first weights are on their way: one launch, no workspace.
// 4096 -> 11008 takes 9.9 us, 11008 -> 4096 11.4, 7.0 of them for the bytes at a copy's rate and 1.7 for the launch.  With the loads in
// registers, eight a lane, the issue slots showed (30 to 70 instructions a load): 12.4 and 15.5 us.
// ---------------------------------------------------------------------------------------------
constexpr int kFewThreads = 512, kFewWarps = kFewThreads / 32, kFewTokens = 8, kFewSegment = 4096, kFewSlots = 8;
constexpr int kFewSmem = 224 * 1024;
__host__ __device__ constexpr int few_pitch(int k) { return (k + 511) / 512 * 512; }  // bytes of a token's codes: whole steps of 32 lanes

__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src), "r"(bytes), "r"(bar)
               : "memory");
}
__device__ __forceinline__ int dot16(const uint4& a, const uint4& b, int acc) {
  acc = __dp4a(static_cast<int>(a.x), static_cast<int>(b.x), acc);
  acc = __dp4a(static_cast<int>(a.y), static_cast<int>(b.y), acc);
  acc = __dp4a(static_cast<int>(a.z), static_cast<int>(b.z), acc);
  return __dp4a(static_cast<int>(a.w), static_cast<int>(b.w), acc);
}
// What is left in flight when a wait has given up: the CTA must not leave before its copies and products have landed.  Bounded too, by
// some 70 ms: copies and products take microseconds, and a barrier that another role has given up on never completes.
constexpr unsigned long long kDrainLimitCycles = 1ull << 27;
__device__ __forceinline__ void mbar_drain(uint32_t bar, uint32_t parity) {
  const unsigned long long t0 = clock64();
  while (!mbar_try_wait(bar, parity) && clock64() - t0 < kDrainLimitCycles) {
  }
}

template <typename T, int M>
__global__ void __launch_bounds__(kFewThreads, 1) linear_few_kernel(const __grid_constant__ LinearArgs a, const int slots, const int slot_bytes) {
  extern __shared__ __align__(16) uint8_t few_smem[];   // the warps' slots, then M rows of codes in whole steps, zero from the last whole 16 on
  __shared__ __align__(8) uint64_t full[kFewWarps][kFewSlots];
  __shared__ uint32_t part[kFewWarps];
  __shared__ float sx[M];
  __shared__ int8_t rest[M][16];                        // the codes behind the last whole 16
  __shared__ int abort_flag;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int whole = a.k / 16 * 16, steps = few_pitch(a.k) / 512, segments = (whole + slot_bytes - 1) / slot_bytes;
  uint4* codes = reinterpret_cast<uint4*>(few_smem + kFewWarps * slots * slot_bytes);
  const uint32_t own = smem_u32(few_smem) + warp * slots * slot_bytes;
  // this warp's channels: first, first + stride, ... (`mine` of them)
  const int64_t stride = static_cast<int64_t>(gridDim.x) * kFewWarps, first = static_cast<int64_t>(warp) * gridDim.x + blockIdx.x;
  const int64_t mine = first < a.n ? (a.n - first + stride - 1) / stride : 0;
  const int64_t total = mine * segments;                // copies
  volatile int* aborted = &abort_flag;
  if (threadIdx.x == 0) abort_flag = 0;
  int64_t issued = 0;
  int next_segment = 0, next_slot = 0;
  const int8_t* next_row = a.w + first * a.ldw;
  auto issue = [&] {                                    // lane 0
    const int at = next_segment * slot_bytes, bytes = min(slot_bytes, whole - at);
    const uint32_t bar = smem_u32(&full[warp][next_slot]);
    mbar_arrive_expect_tx(bar, bytes);
    bulk_load(own + next_slot * slot_bytes, next_row + at, bytes, bar);
    if (++next_slot == slots) next_slot = 0;
    if (++next_segment == segments) next_segment = 0, next_row += stride * a.ldw;
    ++issued;
  };
  if (lane == 0) {
    for (int i = 0; i < slots; ++i) mbar_init(smem_u32(&full[warp][i]), 1);
    fence_mbar_init();
    dependency_wait();
    while (issued < total && issued < slots) issue();
  }
  __syncwarp();
  dependency_wait();
  // the tokens' codes
  const T* x = static_cast<const T*>(a.x);
  const bool octets = (reinterpret_cast<uintptr_t>(x) & 15) == 0 && (M == 1 || a.m == 1 || (a.ldx * sizeof(T) & 15) == 0);
  constexpr int kShare = kFewWarps / M;                 // warps of a token
  const int token = warp / kShare, at = (warp % kShare) * 32 + lane;
  const T* src = x + token * a.ldx;
  const bool exists = token < a.m;
  uint32_t top = 0;
  if (exists) {
    const int eights = octets ? a.k / 8 : 0;
#pragma unroll 4
    for (int o = at; o < eights; o += kShare * 32) {
      Octet<T> raw;
      raw.load_shared(src + o * 8);
      float v[8];
      raw.unpack(v);
#pragma unroll
      for (int j = 0; j < 8; ++j) top = max(top, magnitude(v[j]));
    }
#pragma unroll 4
    for (int c = eights * 8 + at; c < a.k; c += kShare * 32) top = max(top, magnitude(Storage<T>::load1(src + c)));
  }
  top = __reduce_max_sync(0xFFFFFFFFu, top);
  if (lane == 0) part[warp] = top;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kShare; ++i) top = max(top, part[token * kShare + i]);
  const RowScale rs = row_scale(top);
  if (at == 0) sx[token] = rs.scale;
  const bool some = exists && !rs.zero;
  uint2* dst = reinterpret_cast<uint2*>(codes + token * steps * 32);
#pragma unroll 2
  for (int o = at; o < steps * 64; o += kShare * 32) {
    uint2 q = make_uint2(0, 0);
    if (some && o * 8 < whole) {
      float v[8];
      if (octets) {
        Octet<T> raw;
        raw.load_shared(src + o * 8);
        raw.unpack(v);
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = Storage<T>::load1(src + o * 8 + j);
      }
      q = make_uint2(code4(v, rs.inv), code4(v + 4, rs.inv));
    }
    dst[o] = q;
  }
  if (at < 16) rest[token][at] = static_cast<int8_t>(some && whole + at < a.k ? code_of(Storage<T>::load1(src + whole + at), rs.inv) : 0);
  __syncthreads();
  bool ok = true;
  int slot = 0;
  uint32_t parity = 0;
  int sum[M] = {};                                      // lane i: of the i-th of 32 channels
  for (int64_t i = 0; i < mine && ok; ++i) {
    const int64_t n0 = first + i * stride;
    int acc[M] = {};
    for (int segment = 0; segment < segments; ++segment) {
      ok = mbar_wait<false>(smem_u32(&full[warp][slot]), parity, aborted, &g_linear_error, 121);
      ok = __all_sync(0xFFFFFFFFu, ok);
      if (!ok) break;
      const int count = (min(slot_bytes, whole - segment * slot_bytes) + 511) / 512;
      const uint32_t from = own + slot * slot_bytes + lane * 16;
      const uint4* t = codes + segment * (slot_bytes / 16) + lane;
      // (behind the row's last code the slot holds old codes, and the tokens' are zero)
      auto step = [&](int s) {
        const uint4 w = lds128(from + s * 512);
#pragma unroll
        for (int m = 0; m < M; ++m) acc[m] = dot16(w, t[(m * steps + s) * 32], acc[m]);
      };
      if (count == kFewSegment / 512) {
#pragma unroll
        for (int s = 0; s < kFewSegment / 512; ++s) step(s);
      } else {
        for (int s = 0; s < count; ++s) step(s);
      }
      __syncwarp();
      if (lane == 0 && issued < total) issue();
      if (++slot == slots) slot = 0, parity ^= 1;
    }
    if (whole + lane < a.k) {                           // the end of the row, a code a lane: nothing behind the last one is read
      const int w = a.w[n0 * a.ldw + whole + lane];
#pragma unroll
      for (int m = 0; m < M; ++m) acc[m] += w * rest[m][lane];
    }
#pragma unroll
    for (int m = 0; m < M; ++m) {
      const int all = __reduce_add_sync(0xFFFFFFFFu, acc[m]);
      if (lane == static_cast<int>(i & 31)) sum[m] = all;
    }
    if ((i & 31) == 31 || i + 1 == mine) {
      const int64_t n = first + ((i & ~int64_t{31}) + lane) * stride;
      if (ok && lane <= static_cast<int>(i & 31)) {
        const float sw = a.sw[n], bias = a.bias ? load_one<T>(a.bias, n) : 0.0f;
        const bool drop = a.mask.threshold != 0;
#pragma unroll
        for (int m = 0; m < M; ++m) {
          if (m < a.m) {
            const bool keep = drop && (keep_bits(a.mask, static_cast<uint64_t>(m * ((a.n + 7) / 8) + (n >> 3))) >> (n & 7) & 1);
            const float v = finish1(sum[m], sx[m], sw, bias, a.residual ? load_one<T>(a.residual, m * a.ldr + n) : 0.0f, keep, a.mask.scale, drop);
            Storage<T>::store1(static_cast<T*>(a.y) + m * a.ldy + n, v);
          }
        }
      }
    }
  }
  if (!ok && lane == 0)                                 // the copies in flight: those of the slots from here on
    for (int i = 0; i < slots && i < issued; ++i) {
      mbar_drain(smem_u32(&full[warp][slot]), parity);
      if (++slot == slots) slot = 0, parity ^= 1;
    }
}

// ---------------------------------------------------------------------------------------------
// More tokens: tcgen05.  The accumulator's rows are channels, its columns tokens: a tile is 128 channels x `tokens` (16 to 256).  That
// way round the weights, which are read from memory once, fill the instruction's 128 rows whatever the number of tokens; a thread of the
// epilogue has one channel (its scale and bias in registers) and a warp writes 32 neighbouring channels of a token at a time,
// contiguous for every row length.
// 8 tokens, 11008 -> 4096: 11.9 us and 1.3 for the quantiser in front, 7.0 of them for the weights; 64 tokens, 5120 -> 13824: 15.3 us, 11.
// A tile's inner dimension is cut over a cluster of `split` CTAs when there are fewer tiles than multiprocessors.  Integer sums are exact in
// any order; each CTA finishes a share of the tokens, the others write their part of it into slots of its shared memory (which no stage uses:
// one barrier between the writes and the reads, and nobody has to stay for the others).
// ---------------------------------------------------------------------------------------------
constexpr int kTileChannels = 128, kChunk = 128;           // rows of the weights' box, bytes (= codes) of a stage's rows
constexpr int kTileThreads = 320;                          // TMA producer, MMA issuer, eight epilogue warps
constexpr int kMaxStages = 12;

struct TileShape {
  int32_t pair;          // 1: linear_pair_kernel
  int32_t tokens;        // per tile, a multiple of 16 (of 32 for pairs)
  int32_t split;         // CTAs of a cluster that share a tile
  int32_t stages;
  int32_t token_tiles;
  int32_t give_up;       // test hook: the block whose first wait counts as run out; -1: none
  int32_t weights_ahead; // 1: the kernel in front is the tokens' quantiser, which lets this one start after its own wait: the weights are older
};

// kind::i8: signed 8-bit operands, both K-major, 32-bit integer accumulator, M = 128, N = n
__device__ __forceinline__ uint32_t make_idesc_i8(int m, int n) {
  return (2u << 4) | (1u << 7) | (1u << 10) | (static_cast<uint32_t>(n >> 3) << 17) | (static_cast<uint32_t>(m >> 4) << 24);
}
__device__ __forceinline__ void umma_i8(uint32_t d_tmem, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::i8 [%0], %1, %2, %3, p;\n\t}" ::"r"(d_tmem),
      "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate)
      : "memory");
}
__device__ __forceinline__ void tmem_ld8(uint32_t taddr, uint32_t (&v)[8]) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
               : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7])
               : "r"(taddr)
               : "memory");
}
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
__device__ __forceinline__ uint32_t peer_smem(uint32_t addr, uint32_t rank) {
  uint32_t r;
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
  return r;
}
__device__ __forceinline__ void sts_peer(uint32_t addr, uint32_t v) { asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(addr), "r"(v) : "memory"); }
// A wait of the block that the test hook names has run out: as mbar_wait leaves it.
__device__ __forceinline__ bool first_wait(const TileShape& shape, int* abort_flag) {
  if (static_cast<int>(blockIdx.x) != shape.give_up) return true;
  *static_cast<volatile int*>(abort_flag) = 1;
  atomicCAS(&g_linear_error, 0, 100);
  return false;
}
__device__ __forceinline__ void prefetch_map(const CUtensorMap& map) { asm volatile("prefetch.tensormap [%0];" ::"l"(&map) : "memory"); }
// The sum of a cluster's CTAs for one token and channel, from the slots that they have filled in this CTA's shared memory.
__device__ __forceinline__ uint32_t sum_of_slots(uint32_t at, uint32_t slot_bytes, int split) {
  uint32_t v[4];
#pragma unroll
  for (int r = 0; r < 4; ++r) asm volatile("ld.shared.u32 %0, [%1];" : "=r"(v[r]) : "r"(at + min(r, split - 1) * slot_bytes) : "memory");
  return v[0] + v[1] + (split > 2 ? v[2] + v[3] : 0u);
}

// The epilogue of U tokens (8 or 16) of one channel per lane; a warp's lanes hold 32 consecutive channels from a multiple of 32.
// residual_ahead: the loads, issued before the sums are there.  finish: scales (from shared memory), bias, mask, residual, store; the
// loads of one batch are never behind the stores of another that they would have to wait for.  Mask: eight lanes share an octet of
// channels; lane j of the eight makes the block of token j (and 8 + j), and everyone asks the lane that made it.
// (Addresses are clamped to the matrix instead of the loads being guarded: a guarded load is a branch with its conversion in it, and the
// loads then wait for each other: 1024 x 2048 outputs behind k = 8192 took 11 us more with a residual than without.)
template <typename T, int U>
__device__ __forceinline__ void residual_ahead(const LinearArgs& a, int64_t m0, int64_t n, T (&add)[U]) {
  const T* p = static_cast<const T*>(a.residual) + min(n, a.n - 1);
#pragma unroll
  for (int j = 0; j < U; ++j) add[j] = p[min(m0 + j, a.m - 1) * a.ldr];
}
// The scales of the tokens that a warp of the epilogue finishes (the batches of 16 that start at 16 `part`, STEP apart) into places of its own: no
// barrier between warps, so that a warp that gives up a wait leaves nobody behind.
template <int STEP>
__device__ __forceinline__ void load_scales(const LinearArgs& a, int64_t m0, int part, int tokens, float* own) {
  const int lane = threadIdx.x & 31;
  __syncwarp();
#pragma unroll
  for (int i = 0; i < (256 + STEP - 1) / STEP / 2; ++i) {      // two batches a turn
    const int j = i * 32 + lane, c = (j & 15) + 16 * part + (j >> 4) * STEP;
    if (c < tokens) own[j] = a.sx[min(m0 + c, a.m - 1)];
  }
  __syncwarp();
}

template <typename T, bool DROP, bool RES, int U>
__device__ __forceinline__ void finish(const LinearArgs& a, const uint32_t (&sum)[U], const float* sx, int64_t m0, int64_t n, float sw, float bias,
                                       const T (&add)[U]) {
  const int lane = threadIdx.x & 31;
  float v[U];
  uint32_t keep[U / 8];
#pragma unroll
  for (int h = 0; h < U / 8; ++h)
    keep[h] = DROP ? keep_bits(a.mask, static_cast<uint64_t>((m0 + 8 * h + (lane & 7)) * ((a.n + 7) / 8) + (n >> 3))) : 0u;
#pragma unroll
  for (int j = 0; j < U; ++j) {
    const uint32_t bits = DROP ? __shfl_sync(0xFFFFFFFFu, keep[j / 8], (lane & 24) | (j & 7)) : 0u;
    v[j] = finish1(static_cast<int>(sum[j]), sx[j], sw, bias, RES ? Storage<T>::load1(add + j) : 0.0f, bits >> (lane & 7) & 1, a.mask.scale, DROP);
  }
  if (n < a.n) {
    T* y = static_cast<T*>(a.y) + m0 * a.ldy + n;
    if (m0 + U <= a.m) {
#pragma unroll
      for (int j = 0; j < U; ++j, y += a.ldy) Storage<T>::store1(y, v[j]);
    } else {
      const int left = static_cast<int>(a.m - m0);
#pragma unroll
      for (int j = 0; j < U; ++j, y += a.ldy)
        if (j < left) Storage<T>::store1(y, v[j]);
    }
  }
}

template <typename T, bool DROP, bool RES>
__global__ void __launch_bounds__(kTileThreads, 2) linear_tile_kernel(const __grid_constant__ CUtensorMap map_w, const __grid_constant__ CUtensorMap map_x,
                                                                   const LinearArgs a, const TileShape shape) {
  extern __shared__ uint8_t tile_smem[];
  __shared__ __align__(8) uint64_t full[kMaxStages], empty[kMaxStages], done;
  __shared__ uint32_t tmem_slot;
  __shared__ int abort_flag;
  __shared__ float scales[8][128];
  const uint32_t stages0 = (smem_u32(tile_smem) + 1023u) & ~1023u;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = shape.split > 1 ? blockIdx.x % shape.split : 0;      // (clusters are consecutive blocks)
  const int64_t tile = blockIdx.x / shape.split;
  const int64_t n0 = tile / shape.token_tiles * kTileChannels, m0 = tile % shape.token_tiles * shape.tokens;
  const int chunks = (a.k + kChunk - 1) / kChunk;
  const int first = static_cast<int>(static_cast<int64_t>(chunks) * rank / shape.split);
  const int last = static_cast<int>(static_cast<int64_t>(chunks) * (rank + 1) / shape.split);
  const uint32_t stage_bytes = kTileChannels * kChunk + shape.tokens * kChunk;
  const uint32_t tmem_cols = shape.tokens <= 32 ? 32 : (shape.tokens <= 64 ? 64 : (shape.tokens <= 128 ? 128 : 256));
  // the cluster's sums: groups of eight tokens, two by two to the CTAs in turn; a slot for each source
  const int groups = shape.tokens / 8, own_groups = (groups / 2 + shape.split - 1) / shape.split * 2;
  const uint32_t sums0 = stages0 + shape.stages * stage_bytes, slot_bytes = own_groups * 8 * kTileChannels * 4;
  volatile int* aborted = &abort_flag;
  if (threadIdx.x == 0) {
    prefetch_map(map_w);
    prefetch_map(map_x);
    abort_flag = 0;
    for (int s = 0; s < shape.stages; ++s) {
      mbar_init(smem_u32(&full[s]), 1);
      mbar_init(smem_u32(&empty[s]), 1);
    }
    mbar_init(smem_u32(&done), 1);
    fence_mbar_init();
  }
  if (warp == 1) {
    tmem_alloc(smem_u32(&tmem_slot), tmem_cols);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (shape.split > 1) cluster_arrive();                    // (waited for before anybody writes into another's shared memory)
  const uint32_t tmem = tmem_slot;
  bool ok = true;
  if (warp == 0) {
    if (elect_one()) {
      // behind the tokens' quantiser: the first stages' weights are fetched before the wait for it
      const int ahead = shape.weights_ahead ? min(shape.stages, last - first) : 0;
      for (int s = 0; s < ahead; ++s) {
        mbar_arrive_expect_tx(smem_u32(&full[s]), stage_bytes);
        tma_load_2d(stages0 + s * stage_bytes, &map_w, (first + s) * kChunk, static_cast<int>(n0), smem_u32(&full[s]));
      }
      dependency_wait();
      ok = first_wait(shape, &abort_flag);
      int issued = 0;
      for (int c = first, s = 0, phase = 0; c < last && ok; ++c) {
        ok = mbar_wait<true>(smem_u32(&empty[s]), phase ^ 1, aborted, &g_linear_error, 101);
        if (ok) {
          const uint32_t bar = smem_u32(&full[s]), at = stages0 + s * stage_bytes;
          if (issued >= ahead) {
            mbar_arrive_expect_tx(bar, stage_bytes);
            tma_load_2d(at, &map_w, c * kChunk, static_cast<int>(n0), bar);
          }
          tma_load_2d(at + kTileChannels * kChunk, &map_x, c * kChunk, static_cast<int>(m0), bar);
          ++issued;
          if (++s == shape.stages) s = 0, phase ^= 1;
        }
      }
      // the copies in flight if a wait gave up; else the last commits, which have to land before the CTA leaves
      for (int c = max(0, issued - shape.stages); c < issued; ++c) mbar_drain(smem_u32(ok ? &empty[c % shape.stages] : &full[c % shape.stages]), c / shape.stages & 1);
    }
    __syncwarp();
  } else if (warp == 1) {
    if (elect_one()) {
      const uint32_t idesc = make_idesc_i8(kTileChannels, shape.tokens);
      for (int c = first, s = 0, phase = 0; c < last && ok; ++c) {
        ok = mbar_wait<true>(smem_u32(&full[s]), phase, aborted, &g_linear_error, 102);
        if (ok) {
          tc_fence_after();
          const uint32_t at = stages0 + s * stage_bytes;
          const uint64_t wdesc = make_desc(at, kChunk), xdesc = make_desc(at + kTileChannels * kChunk, kChunk);
#pragma unroll
          for (int i = 0; i < kChunk / 32; ++i) umma_i8(tmem, wdesc + 2 * i, xdesc + 2 * i, idesc, c > first || i > 0);
          umma_commit(smem_u32(&empty[s]));
          if (++s == shape.stages) s = 0, phase ^= 1;
        }
      }
      umma_commit(smem_u32(&done));
      if (!ok) mbar_drain(smem_u32(&done), 0);
    }
    __syncwarp();
  }
  // the epilogue's warps: a quarter of the accumulator's rows each, two warps a quarter, which take its batches of tokens in turn
  const int quarter = warp & 3, half = (warp - 2) >> 2;
  const int64_t n = n0 + quarter * 32 + lane;
  const uint32_t mine = tmem + (static_cast<uint32_t>(quarter * 32) << 16);
  float sw = 0.0f, bias = 0.0f;
  if (warp >= 2) {
    dependency_wait();
    load_scales<32>(a, m0, half, shape.tokens, scales[warp - 2]);
    if (n < a.n) {
      sw = a.sw[n];
      if (a.bias) bias = load_one<T>(a.bias, n);
    }
    T add[16];
    if (RES && shape.split == 1) residual_ahead<T, 16>(a, m0 + half * 16, n, add);
    ok = mbar_wait<false>(smem_u32(&done), 0, aborted, &g_linear_error, 103);
    ok = __all_sync(0xFFFFFFFFu, ok) && !*aborted;
    ok = __all_sync(0xFFFFFFFFu, ok);
    tc_fence_after();
    if (shape.split == 1 && ok) {
      for (int c = half * 16; c < shape.tokens && m0 + c < a.m; c += 32) {
        uint32_t v[16];
        T next[16];
        tmem_ld16(mine + c, v);
        if (RES && c + 32 < shape.tokens) residual_ahead<T, 16>(a, m0 + c + 32, n, next);
        tmem_ld_wait();
        finish<T, DROP, RES, 16>(a, v, scales[warp - 2] + c / 32 * 16, m0 + c, n, sw, bias, add);
        if (RES) {
#pragma unroll
          for (int j = 0; j < 16; ++j) add[j] = next[j];
        }
      }
    }
  }
  if (shape.split > 1) {
    __syncwarp();
    cluster_wait();
    const uint32_t channel = (quarter * 32 + lane) * 4;
    if (warp >= 2 && ok) {
      for (int g = half; g < groups; g += 2) {
        uint32_t v[8];
        tmem_ld8(mine + g * 8, v);
        const int owner = (g >> 1) % shape.split, place = (g >> 1) / shape.split * 2 + (g & 1);
        const uint32_t to = peer_smem(sums0 + rank * slot_bytes + place * 8 * kTileChannels * 4 + channel, owner);
        tmem_ld_wait();
#pragma unroll
        for (int j = 0; j < 8; ++j) sts_peer(to + j * kTileChannels * 4, v[j]);
      }
    } else if (warp >= 2 && lane < shape.split) {             // the sums of the whole cluster lack this CTA's: nobody writes results of them
      sts_peer(peer_smem(smem_u32(&abort_flag), lane), 1);
    }
    __syncwarp();
    cluster_arrive();
    cluster_wait();
    if (warp >= 2) {
      const int lacking = *aborted;                           // set here or by a CTA that had no sums to send
      for (int place = half; place < own_groups; place += 2) {
        const int g = ((place >> 1) * shape.split + static_cast<int>(rank)) * 2 + (place & 1);
        if (g >= groups || m0 + g * 8 >= a.m) break;
        T add[8];
        if (RES) residual_ahead<T, 8>(a, m0 + g * 8, n, add);
        float sx[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) sx[j] = a.sx[min(m0 + g * 8 + j, a.m - 1)];
        uint32_t sum[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) sum[j] = sum_of_slots(sums0 + (place * 8 + j) * kTileChannels * 4 + channel, slot_bytes, shape.split);
        finish<T, DROP, RES, 8>(a, sum, sx, m0 + g * 8, lacking ? a.n : n, sw, bias, add);      // (nothing is stored from the n-th channel on)
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tmem, tmem_cols);
  }
}

// ---------------------------------------------------------------------------------------------
// Many tokens: the same product by pairs of CTAs (cta_group::2).  A tile is 256 channels x `tokens` (a multiple of 32, at most 256); each
// CTA of the pair holds 128 of the channels' rows and half of the tokens, so that an operand byte that comes from L2 is used for twice as
// many products as in linear_tile_kernel.  Pairs stay resident and take tiles in turn; two accumulators of 256 columns: the epilogue
// of a tile runs beside the products of the next.
// Barriers: full (of the even CTA) counts the bytes of both CTAs' copies; empty and acc_full are signalled in both CTAs by the even one's
// commits; acc_empty (of the even CTA) counts the epilogue warps of both.
// 8192 x 4096 -> 11008: 220 us, 3360 TOP/s, the tensor pipe 89 % active, for the kernel alone in short runs; with its quantiser in a program, at the
// board's power cap, the call takes 280.  Where k or the number of tokens is small,
// operands from L2 bound it (about 65 bytes a cycle and multiprocessor): 1024 x 8192 -> 2048 takes 15.5 us, 10 at the rate above.
// ---------------------------------------------------------------------------------------------
constexpr int kPairStages = 6, kPairStageBytes = 2 * kTileChannels * kChunk;

__device__ __forceinline__ void tma_load_pair(uint32_t dst, const void* tmap, int x, int y, uint32_t bar) {
  asm volatile("cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];" ::"r"(dst),
               "l"(tmap), "r"(bar), "r"(x), "r"(y)
               : "memory");
}
__device__ __forceinline__ void umma_i8_pair(uint32_t d_tmem, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::2.kind::i8 [%0], %1, %2, %3, p;\n\t}" ::"r"(d_tmem),
      "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate)
      : "memory");
}
__device__ __forceinline__ void umma_commit_pair(uint32_t bar) {
  asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar), "h"(static_cast<uint16_t>(3))
               : "memory");
}
__device__ __forceinline__ void tmem_alloc_pair(uint32_t smem_dst, uint32_t ncols) {
  asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_dst), "r"(ncols) : "memory");
}
__device__ __forceinline__ void tmem_relinquish_pair() { asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tmem_dealloc_pair(uint32_t taddr, uint32_t ncols) {
  asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(taddr), "r"(ncols) : "memory");
}
__device__ __forceinline__ void mbar_arrive_peer(uint32_t bar) {
  asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}

// Twelve epilogue warps: with eight, two a scheduler, their waits for tensor memory showed (333 x 1027 -> 50265 tokens in fp32), with sixteen
// the registers do not reach.  An accumulator is given back as soon as its last columns are in registers, with a release within the CTA: one for the cluster
// made the warp wait for its stores.
constexpr int kPairEpilogue = 12, kPairThreads = 64 + kPairEpilogue * 32, kPairStep = kPairEpilogue / 4 * 16;
template <typename T, bool DROP, bool RES>
__global__ void __launch_bounds__(kPairThreads) linear_pair_kernel(const __grid_constant__ CUtensorMap map_w, const __grid_constant__ CUtensorMap map_x,
                                                                   const LinearArgs a, const TileShape shape, const int64_t tiles) {
  extern __shared__ uint8_t pair_smem[];
  __shared__ __align__(8) uint64_t full[kPairStages], empty[kPairStages], acc_full[2], acc_empty[2];
  __shared__ uint32_t tmem_slot;
  __shared__ int abort_flag;
  __shared__ float scales[kPairEpilogue][96];
  const uint32_t stages0 = (smem_u32(pair_smem) + 1023u) & ~1023u;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = blockIdx.x & 1;
  const int64_t pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;
  const int chunks = (a.k + kChunk - 1) / kChunk;
  const int half_tokens = shape.tokens / 2;
  // a pair's tiles, `pairs` apart: counted on instead of divided (a 64-bit division takes longer than a short tile's products)
  const int step_n = static_cast<int>(pairs / shape.token_tiles), step_m = static_cast<int>(pairs % shape.token_tiles);
  const int first_n = static_cast<int>(pair / shape.token_tiles), first_m = static_cast<int>(pair % shape.token_tiles);
  struct Place {
    int n, m;            // tiles of channels and of tokens
  };
  auto behind = [&](Place p) {
    p.n += step_n;
    p.m += step_m;
    if (p.m >= shape.token_tiles) p.m -= shape.token_tiles, ++p.n;
    return p;
  };
  volatile int* aborted = &abort_flag;
  // A producer or issuer whose wait gave up ends the work of both CTAs: the other one must not take an accumulator that lacks products for a
  // good one.  (In front of whatever this role still signals; nobody has left by then, because of the barrier at the end.)
  auto give_up = [&] {
    *aborted = 1;
    sts_peer(peer_smem(smem_u32(&abort_flag), rank ^ 1), 1);
    asm volatile("fence.acq_rel.cluster;" ::: "memory");
  };
  if (threadIdx.x == 0) {
    prefetch_map(map_w);
    prefetch_map(map_x);
    abort_flag = 0;
    for (int s = 0; s < kPairStages; ++s) {
      mbar_init(smem_u32(&full[s]), 1);
      mbar_init(smem_u32(&empty[s]), 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(smem_u32(&acc_full[i]), 1);
      mbar_init(smem_u32(&acc_empty[i]), 2 * kPairEpilogue);
    }
    fence_mbar_init();
  }
  if (warp == 1) {
    tmem_alloc_pair(smem_u32(&tmem_slot), 512);
    tmem_relinquish_pair();
  }
  tc_fence_before();
  __syncthreads();
  cluster_arrive();
  cluster_wait();
  tc_fence_after();
  const uint32_t tmem = tmem_slot;
  if (warp == 0) {
    if (elect_one()) {
      // weights before the wait, as in linear_tile_kernel
      const int ahead = shape.weights_ahead ? min(kPairStages, chunks) : 0, stage_bytes = (kTileChannels + half_tokens) * kChunk;
      for (int s = 0; s < ahead; ++s) {
        if (rank == 0) mbar_arrive_expect_tx(smem_u32(&full[s]), 2 * stage_bytes);
        tma_load_pair(stages0 + s * kPairStageBytes, &map_w, s * kChunk, static_cast<int>(first_n * 256 + rank * 128), peer_smem(smem_u32(&full[s]), 0));
      }
      dependency_wait();
      bool ok = first_wait(shape, &abort_flag);
      int issued = 0;
      Place place = {first_n, first_m};
      for (int64_t t = pair; t < tiles && ok; t += pairs, place = behind(place)) {
        const int n0 = static_cast<int>(place.n * 256 + rank * 128), m0 = static_cast<int>(place.m * shape.tokens + rank * half_tokens);
        for (int c = 0; c < chunks && ok; ++c, ++issued) {
          const int s = issued % kPairStages;
          ok = mbar_wait<true>(smem_u32(&empty[s]), (issued / kPairStages & 1) ^ 1, aborted, &g_linear_error, 111);
          if (!ok) break;
          const uint32_t bar = peer_smem(smem_u32(&full[s]), 0), at = stages0 + s * kPairStageBytes;
          if (issued >= ahead) {
            if (rank == 0) mbar_arrive_expect_tx(smem_u32(&full[s]), 2 * stage_bytes);
            tma_load_pair(at, &map_w, c * kChunk, n0, bar);
          }
          tma_load_pair(at + kTileChannels * kChunk, &map_x, c * kChunk, m0, bar);
        }
      }
      if (ok) {
        // as in linear_tile_kernel
        for (int c = max(0, issued - kPairStages); c < issued; ++c) mbar_drain(smem_u32(&empty[c % kPairStages]), c / kPairStages & 1);
      } else {
        // The even CTA's barriers count the copies of both, and no longer all of them: time for the copies in flight instead.
        give_up();
        const unsigned long long t0 = clock64();
        while (clock64() - t0 < kDrainLimitCycles) __nanosleep(1000);
      }
    }
    __syncwarp();
  } else if (warp == 1) {
    if (rank == 0 && elect_one()) {
      const uint32_t idesc = make_idesc_i8(256, shape.tokens);
      bool ok = true;
      int used = 0, turn = 0;
      for (int64_t t = pair; t < tiles && ok; t += pairs, ++turn) {
        const int acc = turn & 1;
        ok = mbar_wait<true>(smem_u32(&acc_empty[acc]), (turn >> 1 & 1) ^ 1, aborted, &g_linear_error, 112);
        tc_fence_after();
        for (int c = 0; c < chunks && ok; ++c, ++used) {
          const int s = used % kPairStages;
          ok = mbar_wait<true>(smem_u32(&full[s]), used / kPairStages & 1, aborted, &g_linear_error, 113);
          if (!ok) break;
          tc_fence_after();
          const uint32_t at = stages0 + s * kPairStageBytes;
          const uint64_t wdesc = make_desc(at, kChunk), xdesc = make_desc(at + kTileChannels * kChunk, kChunk);
#pragma unroll
          for (int i = 0; i < kChunk / 32; ++i) umma_i8_pair(tmem + acc * 256, wdesc + 2 * i, xdesc + 2 * i, idesc, c > 0 || i > 0);
          umma_commit_pair(smem_u32(&empty[s]));
        }
        if (!ok) give_up();
        umma_commit_pair(smem_u32(&acc_full[acc]));
        if (!ok) mbar_drain(smem_u32(&acc_full[acc]), turn >> 1 & 1);
      }
    }
    __syncwarp();
  } else {
    const int quarter = warp & 3, part = (warp - 2) >> 2;   // three warps a quarter of the rows, batches of 16 tokens in turn
    const uint32_t mine = tmem + (static_cast<uint32_t>(quarter * 32) << 16);
    bool ok = true;
    int turn = 0;
    dependency_wait();
    // what a tile's epilogue reads beside the sums is loaded during the tile before
    float sx_ahead[3], sw_ahead = 0.0f;
    T bias_ahead = {};
    auto ahead = [&](Place p) {
      const int64_t n = min(static_cast<int64_t>(p.n) * 256 + rank * 128 + quarter * 32 + lane, a.n - 1), m0 = static_cast<int64_t>(p.m) * shape.tokens;
#pragma unroll
      for (int i = 0; i < 3; ++i) {
        const int j = i * 32 + lane;                        // places of the batches of 16 that start at 16 `part`, kPairStep apart
        sx_ahead[i] = a.sx[min(m0 + (j & 15) + 16 * part + (j >> 4) * kPairStep, a.m - 1)];
      }
      sw_ahead = a.sw[n];
      if (a.bias) bias_ahead = static_cast<const T*>(a.bias)[n];
    };
    Place place = {first_n, first_m};
    if (pair < tiles) ahead(place);
    for (int64_t t = pair; t < tiles && ok; t += pairs, ++turn) {
      const int acc = turn & 1;
      const int64_t n = static_cast<int64_t>(place.n) * 256 + rank * 128 + quarter * 32 + lane, m0 = static_cast<int64_t>(place.m) * shape.tokens;
      place = behind(place);
      const int most = static_cast<int>(min(static_cast<int64_t>(shape.tokens), a.m - m0));
      float* sx = scales[warp - 2];
      __syncwarp();
#pragma unroll
      for (int i = 0; i < 3; ++i) sx[i * 32 + lane] = sx_ahead[i];
      __syncwarp();
      const float sw = sw_ahead, bias = a.bias ? Storage<T>::load1(&bias_ahead) : 0.0f;
      if (t + pairs < tiles) ahead(place);
      T add[16], add_next[16];
      if (RES) residual_ahead<T, 16>(a, m0 + part * 16, n, add);
      ok = mbar_wait<false>(smem_u32(&acc_full[acc]), turn >> 1 & 1, aborted, &g_linear_error, 114);
      ok = __all_sync(0xFFFFFFFFu, ok) && !*aborted;
      ok = __all_sync(0xFFFFFFFFu, ok);
      tc_fence_after();
      if (ok) {
        const uint32_t sums = mine + acc * 256;
        uint32_t v[16], v_next[16];
        int c = part * 16;
        if (c < most) tmem_ld16(sums + c, v);
        tmem_ld_wait();
        // one batch: the sums of the next (if there is one) are on their way meanwhile, in the other registers
        auto batch = [&](const uint32_t (&now)[16], const T (&now_add)[16], uint32_t (&next)[16], T (&next_add)[16]) {
          const bool more = c + kPairStep < most;
          if (more) {
            tmem_ld16(sums + c + kPairStep, next);
            if (RES) residual_ahead<T, 16>(a, m0 + c + kPairStep, n, next_add);
          } else {                                          // all of this warp's columns are in registers
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive_peer(peer_smem(smem_u32(&acc_empty[acc]), 0));
          }
          finish<T, DROP, RES, 16>(a, now, sx + c / kPairStep * 16, m0 + c, n, sw, bias, now_add);
          if (more) tmem_ld_wait();
          c += kPairStep;
        };
        while (c < most) {
          batch(v, add, v_next, add_next);
          if (c < most) batch(v_next, add_next, v, add);
        }
        if (part * 16 >= most) {                            // (a warp without tokens in this tile)
          __syncwarp();
          if (lane == 0) mbar_arrive_peer(peer_smem(smem_u32(&acc_empty[acc]), 0));
        }
      }
    }
  }
  // nobody leaves while the other CTA may still signal its barriers or use its tensor memory
  tc_fence_before();
  __syncthreads();
  cluster_arrive();
  cluster_wait();
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc_pair(tmem, 512);
  }
}

// ---------------------------------------------------------------------------------------------
// Host.
// ---------------------------------------------------------------------------------------------
// Rows of codes, k of them, `pitch` bytes apart; a box is box_rows x 128 bytes, swizzled; what lies outside reads as zero.
bool codes_map(CUtensorMap* out, const int8_t* base, int64_t rows, int64_t k, int64_t pitch, int box_rows) {
  const EncodeTiledFn fn = encode_tiled_fn();
  if (!fn) return false;
  const cuuint64_t dims[2] = {static_cast<cuuint64_t>(k), static_cast<cuuint64_t>(rows)};
  const cuuint64_t strides[1] = {static_cast<cuuint64_t>(rows > 1 ? pitch : (k + 15) / 16 * 16)};
  const cuuint32_t box[2] = {kChunk, static_cast<cuuint32_t>(box_rows)};
  const cuuint32_t ones[2] = {1, 1};
  auto encode = [&] {
    return fn(out, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<int8_t*>(base), dims, strides, box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE,
              CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
  };
  if (encode()) return true;
  // A thread that has made no call of the runtime yet may have no context, which this call of the driver does not make for it.
  int device;
  return cudaGetDevice(&device) == cudaSuccess && cudaSetDevice(device) == cudaSuccess && encode();
}

// Kernel, tokens per tile and CTAs per tile: the choice with the shortest estimate, in cycles of a multiprocessor.  From sweeps of all choices
// at 32 sizes (5 to 8192 tokens, 512 x 512 to 5120 x 13824 and 50265 x 1027 weights, inner dimensions from 19 on): operands arrive at about 70 bytes a
// cycle, the tensor cores do 128 * 48 products a cycle, a token of the epilogue costs 25 cycles, sums that travel between CTAs 600 a CTA and 12 a
// token.  One CTA on a multiprocessor with all of its shared memory as stages is better than two, and pairs are better than several rounds of
// single CTAs.  A pair's epilogue takes 930 cycles a step of its twelve warps (48 tokens) and 700 a tile; where the inner dimension is short that
// is what a tile takes (without it small tiles were chosen: 1024 x 256 -> 50304 63 us against 41, 8192 x 512 -> 4096 45 against 29).
// (kTileSmem: two CTAs with 4304 static bytes and 1024 of the system each on a multiprocessor of 228 KB; at 110 KB 600 x 300 -> 9000 had one: 12.2 us)
constexpr int kTileSmem = 108 * 1024, kTileSmemAlone = 215 * 1024, kPairs = 74;
int tile_sums_bytes(const TileShape& s) { return s.split > 1 ? (s.tokens / 16 + s.split - 1) / s.split * 16 * s.split * kTileChannels * 4 : 0; }
// copies beside products: the longer of the two, and some of the other (both draw on the same power)
double overlapped(double a, double b) { return std::max(a, b) + 0.3 * std::min(a, b); }
TileShape tile_shape(int64_t m, int64_t n, int64_t k) {
  TileShape best = {};
  double least = 0;
  const int64_t channel_tiles = (n + kTileChannels - 1) / kTileChannels, chunks = (k + kChunk - 1) / kChunk;
  for (const int64_t most : {256, 224, 192, 160, 128, 96, 64, 32, 16}) {
    TileShape s = {};
    s.token_tiles = static_cast<int32_t>((m + most - 1) / most);
    s.tokens = static_cast<int32_t>(((m + s.token_tiles - 1) / s.token_tiles + 15) / 16 * 16);
    s.token_tiles = static_cast<int32_t>((m + s.tokens - 1) / s.tokens);
    for (s.split = 1; s.split <= 4 && (s.split == 1 || chunks >= 2 * s.split); s.split *= 2) {
      // (clusters of four fill 128 multiprocessors: 36 of them, 1128 x 5918 -> 256, took 15.2 us, 24 of larger tiles 9.3.  By the occupancy
      // calculation, with one CTA on a multiprocessor, the chip holds 33 clusters of four and 74 of two, which is what the resident pairs count
      // on; the estimate leaves one and two of them free.)
      const int64_t ctas = channel_tiles * s.token_tiles * s.split, room = s.split == 4 ? 128 : (s.split == 2 ? 144 : 148), each = (ctas + room - 1) / room;
      const int stage = (kTileChannels + s.tokens) * kChunk;
      s.stages = std::min(kMaxStages, ((each > 1 ? kTileSmem : kTileSmemAlone) - 1024 - tile_sums_bytes(s)) / stage);
      if (s.stages < 2) continue;
      const double inner = static_cast<double>((chunks + s.split - 1) / s.split * kChunk);
      // (what is on its way takes some 1500 cycles: the cluster's sums may leave room for few stages; 300 x 4096 -> 4096 14.1 us with three, 11.8 by pairs)
      const double rate = s.split > 1 ? std::min(70.0, (s.stages - 1) * stage / 1500.0) : 70.0;
      const double steady = overlapped(inner * (kTileChannels + s.tokens) / rate, inner * s.tokens / 48);
      const double ends = 3000 + 25.0 * s.tokens / s.split + (s.split > 1 ? 600 * s.split + 12.0 * s.tokens : 0);
      const double cost = steady * each + ends * ((each + 1) / 2) + (each > 1 ? 1200.0 * each : 0);
      if (best.tokens == 0 || cost < least) {
        best = s;
        least = cost;
      }
    }
    if (most >= 64) {
      s.pair = s.split = 1;
      s.tokens = (s.tokens + 31) / 32 * 32;
      s.token_tiles = static_cast<int32_t>((m + s.tokens - 1) / s.tokens);
      const int64_t rounds = ((n + 255) / 256 * s.token_tiles + kPairs - 1) / kPairs;
      const double inner = static_cast<double>(chunks * kChunk);
      const double steady = overlapped(inner * (kTileChannels + s.tokens / 2) / 70, inner * s.tokens / 48) + 700;
      const double epilogue = 700 + 930.0 * ((s.tokens + kPairStep - 1) / kPairStep);
      const double cost = std::max(steady, epilogue) * rounds + 5000 + std::min(steady, epilogue);
      if (cost < least) {
        best = s;
        least = cost;
      }
    }
  }
  return best;
}
int tile_smem_bytes(const TileShape& s) { return s.stages * (kTileChannels + s.tokens) * kChunk + tile_sums_bytes(s) + 1024; }

template <typename T, bool DROP, bool RES>
cudaError_t launch_tile(const CUtensorMap& mw, const CUtensorMap& mx, const LinearArgs& a, const TileShape& s, cudaStream_t st) {
  cudaError_t e = cudaFuncSetAttribute(linear_tile_kernel<T, DROP, RES>, cudaFuncAttributeMaxDynamicSharedMemorySize, kTileSmemAlone + 1024);
  if (e != cudaSuccess) return e;
  const int64_t ctas = (a.n + kTileChannels - 1) / kTileChannels * s.token_tiles * s.split;
  return launch_behind(linear_tile_kernel<T, DROP, RES>, static_cast<unsigned>(ctas), kTileThreads, tile_smem_bytes(s), s.split, st, mw, mx, a, s);
}
template <typename T, bool DROP, bool RES>
cudaError_t launch_pair(const CUtensorMap& mw, const CUtensorMap& mx, const LinearArgs& a, const TileShape& s, cudaStream_t st) {
  constexpr int smem = kPairStages * kPairStageBytes + 1024;
  cudaError_t e = cudaFuncSetAttribute(linear_pair_kernel<T, DROP, RES>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
  if (e != cudaSuccess) return e;
  const int64_t tiles = (a.n + 255) / 256 * s.token_tiles;
  return launch_behind(linear_pair_kernel<T, DROP, RES>, static_cast<unsigned>(2 * std::min<int64_t>(tiles, kPairs)), kPairThreads, smem, 2, st, mw, mx, a, s, tiles);
}

template <typename T>
cudaError_t launch_product(const CUtensorMap& mw, const CUtensorMap& mx, const LinearArgs& a, const TileShape& s, cudaStream_t st) {
  const bool drop = a.mask.threshold != 0;
  if (a.residual) {
    if (s.pair) return drop ? launch_pair<T, true, true>(mw, mx, a, s, st) : launch_pair<T, false, true>(mw, mx, a, s, st);
    return drop ? launch_tile<T, true, true>(mw, mx, a, s, st) : launch_tile<T, false, true>(mw, mx, a, s, st);
  }
  if (s.pair) return drop ? launch_pair<T, true, false>(mw, mx, a, s, st) : launch_pair<T, false, false>(mw, mx, a, s, st);
  return drop ? launch_tile<T, true, false>(mw, mx, a, s, st) : launch_tile<T, false, false>(mw, mx, a, s, st);
}

// Product of codes with the tensor cores.
int run_product(const int8_t* xq, int64_t ldq, const LinearArgs& a, int32_t dtype, bool behind_quantiser, cudaStream_t st, int give_up = -1) {
  TileShape s = tile_shape(a.m, a.n, a.k);
  s.give_up = give_up;
  s.weights_ahead = behind_quantiser;
  if ((a.n + kTileChannels - 1) / kTileChannels * s.token_tiles * s.split > 0x7FFFFFFF) return ZGR_ETOOBIG;
  CUtensorMap mw, mx;
  if (!codes_map(&mw, a.w, a.n, a.k, a.ldw, kTileChannels) || !codes_map(&mx, xq, a.m, a.k, ldq, s.pair ? s.tokens / 2 : s.tokens)) return ZGR_ECUDA;
  const cudaError_t e = dtype == ZGR_F32   ? launch_product<float>(mw, mx, a, s, st)
                        : dtype == ZGR_F16 ? launch_product<__half>(mw, mx, a, s, st)
                                           : launch_product<__nv_bfloat16>(mw, mx, a, s, st);
  return e == cudaSuccess ? ZGR_OK : ZGR_ECUDA;
}

// The slots of a warp in the kernel for few tokens: rows, or equal parts of them up to 4096 bytes, eight if they fit, two at least; 0: the
// tokens' rows leave no room.
struct FewShape {
  int slots, bytes;
};
FewShape few_shape(int64_t m, int64_t k) {
  const int row = std::max(512, few_pitch(static_cast<int>(k))), parts = (row + kFewSegment - 1) / kFewSegment;
  FewShape s = {0, few_pitch((row + parts - 1) / parts)};
  if (m > kFewTokens) return s;
  const int held = m == 1 ? 1 : (m == 2 ? 2 : (m <= 4 ? 4 : 8));      // (the kernel's tokens)
  const int64_t left = (kFewSmem - held * static_cast<int64_t>(few_pitch(static_cast<int>(k)))) / (kFewWarps * s.bytes);
  s.slots = left >= 2 ? static_cast<int>(std::min<int64_t>(left, kFewSlots)) : 0;
  return s;
}
// From three tokens on the tokens' codes are read from shared memory more often than the weights arrive, and the tile kernel is faster unless the
// launch of the quantiser in front of it counts: 4 x 2048 -> 2048 4.6 us against 6.4, 4 x 4096 -> 4096 9.3 against 8.9, 8 x 4096 -> 1024 7.2
// against 7.8, 8 x 4096 -> 4096 13.2 against 8.9; two tokens 4096 -> 11008 12.2 against 12.8.  A channel costs a warp the same however short
// its row is: 4 x 19 -> 22047 12.4 against 8.2.
bool few(int64_t m, int64_t n, int64_t k) {
  return few_shape(m, k).slots > 0 && (m <= 2 || (n <= 8192 && n * k <= (m <= 4 ? 1 << 23 : 1 << 22)));
}
template <typename T, int M>
cudaError_t launch_few(const LinearArgs& a, cudaStream_t st) {
  cudaError_t e = cudaFuncSetAttribute(linear_few_kernel<T, M>, cudaFuncAttributeMaxDynamicSharedMemorySize, kFewSmem);
  if (e != cudaSuccess) return e;
  const FewShape s = few_shape(M, a.k);
  const unsigned blocks = static_cast<unsigned>(std::min<int64_t>((a.n + 3) / 4, 148));      // (four warps of a block at least have something to do)
  return launch_behind(linear_few_kernel<T, M>, blocks, kFewThreads, kFewWarps * s.slots * s.bytes + M * few_pitch(a.k), 1, st, a, s.slots, s.bytes);
}
template <typename T>
cudaError_t launch_few(const LinearArgs& a, cudaStream_t st) {
  return a.m == 1 ? launch_few<T, 1>(a, st) : (a.m == 2 ? launch_few<T, 2>(a, st) : (a.m <= 4 ? launch_few<T, 4>(a, st) : launch_few<T, 8>(a, st)));
}

constexpr int64_t kMaxInner = 1 << 17;      // 127 * 127 * 2^17 < 2^31: the sums fit 32 bits

// Codes as the products read them: rows on 16-byte boundaries, `ld` below what a tensor map can hold.
bool codes_ok(const int8_t* p, int64_t rows, int64_t k, int64_t ld) {
  return matrix_ok(p, rows, k, ld, 1) && aligned_to(p, 16) && (rows <= 1 || (ld % 16 == 0 && ld < (int64_t{1} << 40)));
}

bool sizes_ok(int64_t m, int64_t n, int64_t k) { return m >= 0 && n >= 1 && k >= 1 && k <= kMaxInner && m <= 0x7FFFFFFF && n <= 0x7FFFFFFF; }

// Arguments of the product that both entry points check: everything but the tokens.
bool product_ok(const int8_t* w, int64_t ldw, const float* sw, const void* bias, const void* residual, int64_t ldr, const void* y, int64_t ldy, int64_t m,
                int64_t n, int64_t k, int32_t dtype, double p) {
  if (!storage_known(dtype) || !sizes_ok(m, n, k) || !(p >= 0.0 && p <= 1.0)) return false;
  if (m == 0) return true;
  const int size = storage_size(dtype);
  if (!codes_ok(w, n, k, ldw) || !sw || !aligned_to(sw, 4) || !aligned_to(bias, size)) return false;
  return matrix_ok(y, m, n, ldy, size) && (!residual || matrix_ok(residual, m, n, ldr, size));
}
// Rows of the tokens' codes in the workspace: whole chunks, so that a box's rows are whole lines (at 16 bytes a box of 128 codes may touch two).
int64_t padded(int64_t k) { return (k + kChunk - 1) / kChunk * kChunk; }
int64_t scales_at(int64_t m, int64_t k) { return (m * padded(k) + 255) / 256 * 256; }

LinearArgs linear_args(const int8_t* w, int64_t ldw, const float* sw, const void* bias, const void* residual, int64_t ldr, void* y, int64_t ldy, int64_t m,
                       int64_t n, int64_t k, double p, uint64_t seed, uint32_t tensor) {
  LinearArgs a = {};
  a.w = w;
  a.ldw = ldw;
  a.sw = sw;
  a.bias = bias;
  a.residual = residual;
  a.ldr = ldr;
  a.y = y;
  a.ldy = ldy;
  a.m = m;
  a.n = n;
  a.k = static_cast<int32_t>(k);
  a.mask = make_drop_mask(p, seed, tensor);
  return a;
}

}  // namespace
}  // namespace zgr

using namespace zgr;

extern "C" {

int zgr_quantize_rows(const void* x, int64_t ldx, int64_t rows, int64_t cols, int32_t dtype, int8_t* codes, int64_t ldc, float* scales, void* stream) {
  if (!storage_known(dtype) || rows < 0 || cols < 1 || rows > 0x7FFFFFFF) return ZGR_EINVAL;
  if (rows == 0) return ZGR_OK;
  if (!matrix_ok(x, rows, cols, ldx, storage_size(dtype)) || !matrix_ok(codes, rows, cols, ldc, 1) || !scales || !aligned_to(scales, 4)) return ZGR_EINVAL;
  return run_quantize(dtype, x, ldx, rows, cols, codes, ldc, scales, 0, static_cast<cudaStream_t>(stream)) == cudaSuccess ? ZGR_OK : ZGR_ECUDA;
}

int64_t zgr_linear_i8_workspace(int64_t m, int64_t n, int64_t k) {
  if (!sizes_ok(m, n, k)) return ZGR_EINVAL;
  return few(m, n, k) ? 0 : scales_at(m, k) + m * static_cast<int64_t>(sizeof(float));
}

int zgr_linear_i8(const void* x, int64_t ldx, const int8_t* w, int64_t ldw, const float* w_scale, const void* bias, const void* residual, int64_t ldr, void* y,
                  int64_t ldy, int64_t m, int64_t n, int64_t k, int32_t dtype, double p, uint64_t seed, uint32_t tensor, void* workspace,
                  int64_t workspace_bytes, void* stream) {
  if (!product_ok(w, ldw, w_scale, bias, residual, ldr, y, ldy, m, n, k, dtype, p)) return ZGR_EINVAL;
  if (m == 0) return ZGR_OK;
  if (!matrix_ok(x, m, k, ldx, storage_size(dtype)) || x == y) return ZGR_EINVAL;      // (blocks read all of x while others write results)
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  LinearArgs a = linear_args(w, ldw, w_scale, bias, residual, ldr, y, ldy, m, n, k, p, seed, tensor);
  if (few(m, n, k)) {
    a.x = x;
    a.ldx = ldx;
    const cudaError_t e = dtype == ZGR_F32 ? launch_few<float>(a, st) : (dtype == ZGR_F16 ? launch_few<__half>(a, st) : launch_few<__nv_bfloat16>(a, st));
    return e == cudaSuccess ? ZGR_OK : ZGR_ECUDA;
  }
  if (!workspace || !aligned_to(workspace, 16) || workspace_bytes < zgr_linear_i8_workspace(m, n, k)) return ZGR_EINVAL;
  int8_t* codes = static_cast<int8_t*>(workspace);
  float* scales = reinterpret_cast<float*>(codes + scales_at(m, k));
  if (run_quantize(dtype, x, ldx, m, k, codes, padded(k), scales, 1, st) != cudaSuccess) return ZGR_ECUDA;
  a.sx = scales;
  return run_product(codes, padded(k), a, dtype, true, st);
}

int zgr_debug_matmul_i8_giving_up(const int8_t* x, int64_t ldx, const float* x_scale, const int8_t* w, int64_t ldw, const float* w_scale, const void* bias,
                                  const void* residual, int64_t ldr, void* y, int64_t ldy, int64_t m, int64_t n, int64_t k, int32_t dtype, double p,
                                  uint64_t seed, uint32_t tensor, int32_t block, void* stream) {
  if (!product_ok(w, ldw, w_scale, bias, residual, ldr, y, ldy, m, n, k, dtype, p)) return ZGR_EINVAL;
  if (m == 0) return ZGR_OK;
  if (!codes_ok(x, m, k, ldx) || !x_scale || !aligned_to(x_scale, 4) || static_cast<const void*>(x) == y) return ZGR_EINVAL;
  LinearArgs a = linear_args(w, ldw, w_scale, bias, residual, ldr, y, ldy, m, n, k, p, seed, tensor);
  a.sx = x_scale;
  return run_product(x, ldx, a, dtype, false, static_cast<cudaStream_t>(stream), block);
}

int zgr_matmul_i8(const int8_t* x, int64_t ldx, const float* x_scale, const int8_t* w, int64_t ldw, const float* w_scale, const void* bias,
                  const void* residual, int64_t ldr, void* y, int64_t ldy, int64_t m, int64_t n, int64_t k, int32_t dtype, double p, uint64_t seed,
                  uint32_t tensor, void* stream) {
  return zgr_debug_matmul_i8_giving_up(x, ldx, x_scale, w, ldw, w_scale, bias, residual, ldr, y, ldy, m, n, k, dtype, p, seed, tensor, -1, stream);
}

int zgr_debug_linear_plan(int64_t m, int64_t n, int64_t k, int32_t codes, zgr_linear_plan* out) {
  if (!out || !sizes_ok(m, n, k) || m == 0) return ZGR_EINVAL;
  if (!codes && few(m, n, k)) {
    *out = {ZGR_LINEAR_FEW, static_cast<int32_t>(m), 1};
  } else {
    const TileShape s = tile_shape(m, n, k);
    *out = {s.pair ? ZGR_LINEAR_PAIR : ZGR_LINEAR_TILE, s.tokens, s.split};
  }
  return ZGR_OK;
}

int zgr_linear_status(int32_t* code) {
  if (!code) return ZGR_EINVAL;
  if (cudaDeviceSynchronize() != cudaSuccess || cudaMemcpyFromSymbol(code, g_linear_error, sizeof(int)) != cudaSuccess) return ZGR_ECUDA;
  return ZGR_OK;
}

}  // extern "C"
