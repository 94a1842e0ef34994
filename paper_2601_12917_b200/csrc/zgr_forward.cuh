// Shared by the operators of the forward pass (dropout, 8-bit product): the counter-based mask and raw access to eight elements.
#ifndef ZGR_FORWARD_CUH_
#define ZGR_FORWARD_CUH_

#include <cuda_runtime.h>

#include "zgr_device.cuh"

namespace zgr {

// A dropout mask as a function of (seed, tensor, row, column).  A row of `cols` elements has O = ceil(cols / 8) generator blocks;
// block row * O + o decides the elements 8 o .. 8 o + 7, one 16-bit half each.  Every row begins a block of its own, so that the mask
// knows nothing of strides and alignment, and a tile of a matrix product can make its part of it.  Sixteen bits an element: p in steps
// of 2^-16 for half the generator's work, which at 32 bits (0.66 cycles an element and scheduler) would be as long as the memory traffic.
struct DropMask {
  PhiloxKeys keys;       // with the stream tag folded into the first round's key (it meets that key by xor)
  PhiloxPre pre;         // the part of the first two rounds that is the same for all blocks below 2^32
  uint32_t tensor;
  uint32_t threshold;    // rint(65536 p): an element is kept if its half is not below; 65536 drops all
  float scale;           // 65536 / (65536 - threshold): of the probability in effect, so that the expectation is the input
};

// Host: the mask of (seed, tensor) for a probability in [0, 1].
DropMask make_drop_mask(double p, uint64_t seed, uint32_t tensor);

// The eight halves of a block; element 8 o + i is kept if half i is not below the threshold.  Both halves of a word are compared in its upper
// half: what lies below the upper half of x decides nothing, because the lower half of keep_least() is zero.
__device__ __forceinline__ uint32_t keep_least(const DropMask& mask) { return mask.threshold << 16; }      // (threshold below 65536)
__device__ __forceinline__ void keep_words(const DropMask& mask, uint32_t lo, uint32_t hi, uint32_t (&x)[4]) {
  if (hi == 0) philox4x32_10_pre(lo, mask.pre, mask.keys, x);
  else philox4x32_10(lo, hi, mask.tensor, 0u, mask.keys, x);
}
__device__ __forceinline__ bool kept(const uint32_t (&x)[4], int i, uint32_t least) { return (i & 1 ? x[i >> 1] : x[i >> 1] << 16) >= least; }

// (A block number of 32 bits leaves out the form for the others.)
template <typename Block>
__device__ __forceinline__ void block_words(const DropMask& mask, Block block, uint32_t (&x)[4]) {
  keep_words(mask, static_cast<uint32_t>(block), sizeof(Block) > 4 ? static_cast<uint32_t>(static_cast<uint64_t>(block) >> 32) : 0u, x);
}

// Bit i of the result: element 8 o + i of the row is kept.
template <typename Block>
__device__ __forceinline__ uint32_t keep_bits(const DropMask& mask, Block block) {
  if (mask.threshold > 65535u) return 0;
  uint32_t x[4];
  block_words(mask, block, x);
  const uint32_t least = keep_least(mask);
  uint32_t bits = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (kept(x, i, least)) bits |= 1u << i;
  return bits;
}

// Eight contiguous elements as they lie in memory; conversion when they are used, so that a thread can have several in flight.
template <typename T>
struct Octet {
  uint4 w[sizeof(T) / 2];
  __device__ __forceinline__ void load(const T* p) {
#pragma unroll
    for (int i = 0; i < static_cast<int>(sizeof(T) / 2); ++i) w[i] = __ldcs(reinterpret_cast<const uint4*>(p) + i);
  }
  // Read again and again, by many threads: kept in L1.  (Not by the read-only path: a kernel that was launched early may have begun before the
  // kernel in front wrote what it reads.)
  __device__ __forceinline__ void load_shared(const T* p) {
#pragma unroll
    for (int i = 0; i < static_cast<int>(sizeof(T) / 2); ++i) w[i] = __ldca(reinterpret_cast<const uint4*>(p) + i);
  }
  __device__ __forceinline__ void zero() {
#pragma unroll
    for (int i = 0; i < static_cast<int>(sizeof(T) / 2); ++i) w[i] = make_uint4(0, 0, 0, 0);
  }
  // Elements c .. c + 7 of a row of `cols`, of which only some exist (the others are some element of the row).  All loads are issued, none guarded:
  // a guarded load is a branch, and branches with loads in them wait for each other.
  __device__ __forceinline__ void gather(const T* row, int c, int cols) {
    T* e = reinterpret_cast<T*>(w);
#pragma unroll
    for (int j = 0; j < 8; ++j) e[j] = row[max(0, min(c + j, cols - 1))];
  }
  // Elements p[0 .. 7] at any alignment: the 16-byte granules that hold them (all of [lo, hi) that load_any_ok() asks for), moved into place
  // by selections and one funnel shift a word.  About 20 instructions instead of eight loads.
  __device__ __forceinline__ void load_any(const T* p) {
    constexpr int kWords = 4 * sizeof(T) / 2;      // of an octet
    const uintptr_t at = reinterpret_cast<uintptr_t>(p);
    const uint4* base = reinterpret_cast<const uint4*>(at & ~uintptr_t{15});
    uint32_t g[kWords + 4];
#pragma unroll
    for (int i = 0; i < kWords / 4 + 1; ++i) {
      const uint4 q = __ldca(base + i);
      g[4 * i] = q.x, g[4 * i + 1] = q.y, g[4 * i + 2] = q.z, g[4 * i + 3] = q.w;
    }
    const bool two = at & 8, one = at & 4, half = at & 2;
#pragma unroll
    for (int i = 0; i < kWords + 2; ++i) g[i] = two ? g[i + 2] : g[i];
#pragma unroll
    for (int i = 0; i < kWords + 1; ++i) g[i] = one ? g[i + 1] : g[i];
    if (sizeof(T) == 2) {
#pragma unroll
      for (int i = 0; i < kWords; ++i) g[i] = half ? __funnelshift_r(g[i], g[i + 1], 16) : g[i];
    }
#pragma unroll
    for (int i = 0; i < kWords / 4; ++i) w[i] = make_uint4(g[4 * i], g[4 * i + 1], g[4 * i + 2], g[4 * i + 3]);
  }
  // Whether the granules of load_any(p) lie within the elements [lo, hi).
  static __device__ __forceinline__ bool load_any_ok(const T* p, const T* lo, const T* hi) {
    const uintptr_t base = reinterpret_cast<uintptr_t>(p) & ~uintptr_t{15};
    return base >= reinterpret_cast<uintptr_t>(lo) && base + 16 * (sizeof(T) / 2 + 1) <= reinterpret_cast<uintptr_t>(hi);
  }
  __device__ __forceinline__ void unpack(float (&v)[8]) const;
};
template <>
__device__ __forceinline__ void Octet<float>::unpack(float (&v)[8]) const {
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    v[4 * i] = __uint_as_float(w[i].x);
    v[4 * i + 1] = __uint_as_float(w[i].y);
    v[4 * i + 2] = __uint_as_float(w[i].z);
    v[4 * i + 3] = __uint_as_float(w[i].w);
  }
}
template <>
__device__ __forceinline__ void Octet<__half>::unpack(float (&v)[8]) const {
  const uint32_t r[4] = {w[0].x, w[0].y, w[0].z, w[0].w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&r[i]));
    v[2 * i] = f.x;
    v[2 * i + 1] = f.y;
  }
}
template <>
__device__ __forceinline__ void Octet<__nv_bfloat16>::unpack(float (&v)[8]) const {
  const uint32_t r[4] = {w[0].x, w[0].y, w[0].z, w[0].w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[2 * i] = __uint_as_float(r[i] << 16);
    v[2 * i + 1] = __uint_as_float(r[i] & 0xFFFF0000u);
  }
}

// n / d for n < 2^31 by a multiplication (the operands of the launch are fixed, the division is made for every octet): Granlund and Montgomery,
// "Division by invariant integers using multiplication" (1994), their unsigned form; below 2^31 its sum does not pass 32 bits.
struct FastDiv {
  uint32_t d, mul, shift;
};
inline FastDiv make_fast_div(uint32_t d) {
  uint32_t shift = 0;
  while ((1ull << shift) < d) ++shift;
  return FastDiv{d, static_cast<uint32_t>(((1ull << 32) * ((1ull << shift) - d)) / d + 1), shift};
}
__device__ __forceinline__ uint32_t fast_div(uint32_t n, const FastDiv& f) { return (__umulhi(n, f.mul) + n) >> f.shift; }

// ---------------------------------------------------------------------------------------------
// Launches.  As the sweeps, every kernel is launched with the programmatic-serialisation attribute and waits for the kernel before it
// before it touches memory, so that its launch and set-up run beside that kernel's end.  Only a kernel whose successor is the library's own lets
// it start early, and not before its own wait: what the successor reads ahead of its wait is then older than both.
// ---------------------------------------------------------------------------------------------
__device__ __forceinline__ void dependency_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void dependents_may_start() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

template <typename... Params, typename... Args>
cudaError_t launch_behind(void (*kernel)(Params...), dim3 grid, dim3 block, size_t smem, int cluster, cudaStream_t st, const Args&... args) {
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute attr[2];
  cfg.gridDim = grid;
  cfg.blockDim = block;
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  if (cluster > 1) {
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = static_cast<unsigned>(cluster);
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.numAttrs = 2;
  }
  const cudaError_t e = cudaLaunchKernelEx(&cfg, kernel, static_cast<Params>(args)...);
  if (e != cudaSuccess) cudaGetLastError();      // (reported by the return value, and not again by whoever asks next)
  return e;
}

// ---------------------------------------------------------------------------------------------
// Host checks that the entry points share.
// ---------------------------------------------------------------------------------------------
inline int storage_size(int32_t dtype) { return dtype == 0 ? 4 : 2; }
inline bool storage_known(int32_t dtype) { return dtype >= 0 && dtype <= 2; }
inline bool aligned_to(const void* p, int bytes) { return (reinterpret_cast<uintptr_t>(p) & static_cast<uintptr_t>(bytes - 1)) == 0; }
constexpr int64_t kMostElements = int64_t{1} << 60;      // of a row, and of `ld` times the rows: no sum of sizes passes 63 bits
// A rows x cols matrix of the storage type with rows `ld` elements apart: no row reaches into the next, offsets stay below 2^62 bytes.
inline bool matrix_ok(const void* p, int64_t rows, int64_t cols, int64_t ld, int size) {
  if (!p || !aligned_to(p, size)) return false;
  if (rows > 1 && ld < cols) return false;
  return ld >= 0 && cols <= kMostElements && (rows == 0 || ld <= kMostElements / rows);
}
// Elements between a 16-byte boundary and the row; all rows of a matrix have the same if `ld` is a whole number of 16 bytes.
inline int phase_of(const void* p, int size) { return static_cast<int>((reinterpret_cast<uintptr_t>(p) & 15) / size); }
// Octets of the matrix start on 16-byte boundaries.
inline bool octets_aligned(const void* p, int64_t rows, int64_t ld, int size) { return aligned_to(p, 16) && (rows <= 1 || ld % (16 / size) == 0); }

}  // namespace zgr
#endif  // ZGR_FORWARD_CUH_
