// Dropout whose mask is a function of (seed, tensor, row, column) and is never stored, forward and backward.
//
//   forward    y  = residual + (keep ? (x + bias) * s : 0)          s = 1 / (1 - p)
//   backward   dx = keep ? dy * s : 0,   dbias = column sums of dx before it is rounded
//
// Arithmetic in fp32, one rounding to the storage type.  A dropped element contributes nothing, whatever it holds: it is selected away,
// not multiplied by zero.  The bound is memory: x (and residual) read once, y written once; a generator block (about 40 issue slots
// of a warp) serves eight elements.
#include <cuda_runtime.h>

#include <algorithm>
#include <cmath>

#include "zgr.h"
#include "zgr_forward.cuh"
#include "zgr_host_internal.h"

namespace zgr {

DropMask make_drop_mask(double p, uint64_t seed, uint32_t tensor) {
  DropMask m;
  m.keys = host_make_keys(seed);
  m.keys.k1[0] ^= ZGR_TAG_DROPOUT;
  const uint64_t first = 0xCD9E8D57ull * tensor, second = 0xD2511F53ull * (static_cast<uint32_t>(first >> 32) ^ m.keys.k0[0]);
  m.pre.c1 = static_cast<uint32_t>(first) ^ m.keys.k0[1];
  m.pre.x2 = static_cast<uint32_t>(second >> 32) ^ m.keys.k1[1];
  m.pre.c3 = static_cast<uint32_t>(second);
  m.tensor = tensor;
  m.threshold = static_cast<uint32_t>(std::nearbyint(65536.0 * p));
  m.scale = m.threshold < 65536u ? static_cast<float>(65536.0 / (65536.0 - m.threshold)) : 0.0f;
  return m;
}

namespace {

constexpr int kThreads = 256;

template <typename T>
struct DropArgs {
  const T* x;
  const T* bias;         // or null
  const T* residual;     // or null
  T* y;
  int64_t rows, cols, ldx, ldr, ldy;
  int64_t octets;        // generator blocks of a row
  int64_t pieces;        // eight-element pieces of a row, counted from the 16-byte boundary at or before it
  int64_t total;         // pieces in all
  FastDiv div;           // by `pieces` (total < 2^31)
  int phase;             // elements between that boundary and the first row
  int bias_octets;       // 1: the bias can be read in octets
  int group;             // rows of different alignment (dropout_any_kernel) and column sums: lanes that share a row (a power of two)
  DropMask mask;
};

// keep ? v * s : 0.  The element is selected first: what is dropped may be infinite.
__device__ __forceinline__ float masked(float v, bool keep, float scale) { return (keep ? v : 0.0f) * scale; }
// ... + residual, one rounding
__device__ __forceinline__ float masked_plus(float v, bool keep, float scale, float residual) { return fmaf(keep ? v : 0.0f, scale, residual); }

// Rows that start on 16-byte boundaries.  A thread takes U octets, a block's threads apart, all of its loads in flight before the first
// generator block is made.  U = 4 (2 in fp32) for what fills the chip, 1 for the smallest calls, where a thread with four octets is
// four times as long.
// FLAT: the matrices are whole octets without gaps and there is no bias, so that octet i of the tensor lies at element 8 i.
// What bounds it beside the memory is the number of instructions: an octet may cost about 250 issue slots of its scheduler before they are
// longer than the traffic of a residual sum, the generator's rounds take 40, and this form needs 134.  8192 x 4096 bf16 with a residual:
// 30.3 us, 6.6 TB/s, the rate of a copy (41.5 us with the mask gathered in bits and tested bit by bit, 212 instructions).
template <typename T, int U, bool FLAT, typename Index>
__global__ void __launch_bounds__(kThreads) dropout_kernel(const __grid_constant__ DropArgs<T> a) {
  Octet<T> x[U], r[U];
  int64_t at[U];
  Index row[U];
  int col[U];
  const Index first = static_cast<Index>(blockIdx.x) * (kThreads * U) + threadIdx.x, total = static_cast<Index>(a.total);
  const int cols = static_cast<int>(a.cols);                   // (below 2^31 unless FLAT)
  dependency_wait();
  const Index left = first < total ? total - first : 0;        // octet u exists if u * kThreads < left
#pragma unroll
  for (int u = 0; u < U; ++u) {
    if (static_cast<Index>(u * kThreads) < left) {
      if (FLAT) {
        at[u] = static_cast<int64_t>(first + u * kThreads) * 8;
        x[u].load(a.x + at[u]);
        if (a.residual) r[u].load(a.residual + at[u]);
      } else {
        const Index i = first + u * kThreads;
        row[u] = sizeof(Index) == 4 ? fast_div(static_cast<uint32_t>(i), a.div) : i / a.pieces;
        col[u] = static_cast<int>(i - row[u] * static_cast<Index>(a.pieces)) * 8;
        if (col[u] + 8 <= cols) {
          x[u].load(a.x + row[u] * a.ldx + col[u]);
          if (a.residual) r[u].load(a.residual + row[u] * a.ldr + col[u]);
        } else {                                               // the end of a row that is not whole octets
          x[u].gather(a.x + row[u] * a.ldx, col[u], cols);
          if (a.residual) r[u].gather(a.residual + row[u] * a.ldr, col[u], cols);
        }
      }
    }
  }
  const bool none = a.mask.threshold > 65535u;
  const uint32_t least = none ? 0xFFFFFFFFu : keep_least(a.mask);
#pragma unroll
  for (int u = 0; u < U; ++u) {
    if (static_cast<Index>(u * kThreads) < left) {
      uint32_t words[4] = {0, 0, 0, 0};
      if (!none) block_words(a.mask, first + u * kThreads, words);
      float v[8];
      x[u].unpack(v);
      if (!FLAT && a.bias) {
        Octet<T> raw;
        float b[8];
        if (a.bias_octets && col[u] + 8 <= cols) raw.load_shared(a.bias + col[u]);
        else raw.gather(a.bias, col[u], cols);
        raw.unpack(b);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] += b[j];
      }
      if (a.residual) {
        float add[8];
        r[u].unpack(add);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = masked_plus(v[j], kept(words, j, least), a.mask.scale, add[j]);
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = masked(v[j], kept(words, j, least), a.mask.scale);
      }
      if (FLAT) {
        Storage<T>::store8(a.y + at[u], v);
      } else {
        T* y = a.y + row[u] * a.ldy + col[u];
        if (col[u] + 8 <= cols) {
          Storage<T>::store8(y, v);
        } else {
#pragma unroll
          for (int j = 0; j < 8; ++j)
            if (col[u] + j < cols) Storage<T>::store1(y + j, v[j]);
        }
      }
    }
  }
}

// Rows that follow each other without a gap and are no whole octets (an odd number of columns, at least eight).  The tensor is cut in pieces of
// eight elements wherever a row ends, so that all accesses are whole and aligned; a piece from column c on takes its bits from the block
// of c, made here, from the next piece's, got from the next lane, and, where the row ends within it, sometimes from a third, made by that lane
// alone.  fp16, 16336 x 1021: 27.8 us by the rows' own pieces (dropout_shifted_kernel), whose ends are loaded and stored element by element.
// Index: 32 bits where the tensor has fewer than 2^31 elements: 16.0 us (4.2 TB/s) against 21.1.  Its 176 instructions a warp and octet are about 10 us
// of issue and its bytes 10.3 of memory; with 43 % of the warps' places taken and every thread loading, computing and storing once, the two
// hardly overlap, and that is what bounds it (issue slots are 52 % busy).
template <typename T, int U, typename Index>
__global__ void __launch_bounds__(kThreads) dropout_unbroken_kernel(const __grid_constant__ DropArgs<T> a) {
  const int lane = threadIdx.x & 31, cols = static_cast<int>(a.cols);
  dependency_wait();
  const Index elements = static_cast<Index>(a.rows * a.cols), total = static_cast<Index>(a.total), octets = static_cast<Index>(a.octets);
  const Index first = (static_cast<Index>(blockIdx.x) * (kThreads / 32) + (threadIdx.x >> 5)) * (32 * U) + lane;
  Octet<T> x[U], r[U];
  Index row[U];
  int col[U];
  uint32_t own[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const Index e = min(first + u * 32, total - 1) * 8;
    row[u] = sizeof(Index) == 4 ? fast_div(static_cast<uint32_t>(e), a.div) : e / a.cols;
    col[u] = static_cast<int>(e - row[u] * static_cast<Index>(a.cols));
    if (e + 8 <= elements) {
      x[u].load(a.x + e);
      if (a.residual) r[u].load(a.residual + e);
    } else {                                                   // the end of the tensor
      x[u].gather(a.x + e, 0, static_cast<int>(elements - e));
      if (a.residual) r[u].gather(a.residual + e, 0, static_cast<int>(elements - e));
    }
  }
#pragma unroll
  for (int u = 0; u < U; ++u) own[u] = keep_bits(a.mask, row[u] * octets + (col[u] >> 3));
  // the block behind a warp's pieces is the next warp's first; only behind the last warp's it is made once more
  __shared__ uint32_t firsts[kThreads / 32];
  const int warp = threadIdx.x >> 5;
  if (lane == 0) firsts[warp] = own[0];
  __syncthreads();
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const Index i = first + u * 32;
    // the next piece's block: of this row, or the first of the next
    uint32_t next = __shfl_down_sync(0xFFFFFFFFu, own[u], 1);
    if (u + 1 < U) {
      const uint32_t over = __shfl_sync(0xFFFFFFFFu, own[u + 1 < U ? u + 1 : u], 0);
      if (lane == 31) next = over;
    }
    const int s = col[u] & 7, left = cols - col[u];            // elements of the row from here on
    const Index block = row[u] * octets + (col[u] >> 3);
    if (u + 1 == U) {
      if (warp + 1 < kThreads / 32) {
        const uint32_t over = firsts[warp + 1];
        if (lane == 31) next = over;
      } else if (lane == 31) {
        next = keep_bits(a.mask, left > 8 ? block + 1 : (row[u] + 1) * octets);
      }
    }
    uint32_t rest = next;                                      // behind this block in the same row
    if (left <= 8 && left > 8 - s) rest = keep_bits(a.mask, block + 1);
    uint32_t keep = own[u] >> s | rest << (8 - s);
    if (left < 8) keep = (keep & ((1u << left) - 1)) | next << left;
    if (i < total) {
      float v[8];
      x[u].unpack(v);
      if (a.bias) {
        T b[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) b[j] = a.bias[j < left ? col[u] + j : j - left];
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] += Storage<T>::load1(b + j);
      }
      if (a.residual) {
        float add[8];
        r[u].unpack(add);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = masked_plus(v[j], keep >> j & 1, a.mask.scale, add[j]);
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = masked(v[j], keep >> j & 1, a.mask.scale);
      }
      T* y = a.y + i * 8;
      if (i * 8 + 8 <= elements) {
        Storage<T>::store8(y, v);
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (i * 8 + j < elements) Storage<T>::store1(y + j, v[j]);
      }
    }
  }
}

// Rows that do not start on 16-byte boundaries, all matrices alike.  A row's pieces of eight elements then begin `s`
// elements before it, at the boundary, and take the last s bits of one generator block and the first 8 - s of the next: a thread
// makes the block of its own piece and gets its neighbour's bits from the neighbouring lane; a warp's pieces follow each other, so that only its
// first lane makes a second block, once for U pieces.  8192 x 4096 bf16 with a residual, all of them two elements off: 54 us (whole octets: 30).
template <typename T, int U, typename Index>
__global__ void __launch_bounds__(kThreads) dropout_shifted_kernel(const __grid_constant__ DropArgs<T> a) {
  constexpr int kPhases = 16 / sizeof(T);
  const int lane = threadIdx.x & 31, cols = static_cast<int>(a.cols);
  dependency_wait();
  Octet<T> x[U], r[U];
  Index row[U];
  int piece[U], shift[U];
  const Index total = static_cast<Index>(a.total), octets = static_cast<Index>(a.octets);
  const Index first = (static_cast<Index>(blockIdx.x) * (kThreads / 32) + (threadIdx.x >> 5)) * (32 * U) + lane;
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const Index i = min(first + u * 32, total - 1);
    row[u] = sizeof(Index) == 4 ? fast_div(static_cast<uint32_t>(i), a.div) : i / a.pieces;
    piece[u] = static_cast<int>(i - row[u] * static_cast<Index>(a.pieces));
    shift[u] = static_cast<int>((static_cast<uint32_t>(a.phase) + static_cast<uint32_t>(row[u]) * static_cast<uint32_t>(a.ldx)) & (kPhases - 1));      // (only the low bits count)
    const int col = piece[u] * 8 - shift[u];
    if (col >= 0 && col + 8 <= cols) {
      x[u].load(a.x + row[u] * a.ldx + col);
      if (a.residual) r[u].load(a.residual + row[u] * a.ldr + col);
    } else {
      x[u].gather(a.x + row[u] * a.ldx, col, cols);
      if (a.residual) r[u].gather(a.residual + row[u] * a.ldr, col, cols);
    }
  }
  uint32_t before = 0;   // lane 31's block of the pieces before
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const Index block = row[u] * octets + piece[u];
    const uint32_t own = keep_bits(a.mask, block);
    uint32_t left = __shfl_up_sync(0xFFFFFFFFu, own, 1);
    if (lane == 0) left = u > 0 ? before : (piece[u] > 0 ? keep_bits(a.mask, block - 1) : 0u);
    if (U > 1) before = __shfl_sync(0xFFFFFFFFu, own, 31);
    const uint32_t keep = (own << 8 | left) >> (8 - shift[u]);
    if (first + u * 32 < total) {
      const int col = piece[u] * 8 - shift[u];
      float v[8];
      x[u].unpack(v);
      if (a.bias) {
        Octet<T> raw;
        float b[8];
        raw.gather(a.bias, col, cols);
        raw.unpack(b);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] += b[j];
      }
      if (a.residual) {
        float add[8];
        r[u].unpack(add);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = masked_plus(v[j], keep >> j & 1, a.mask.scale, add[j]);
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = masked(v[j], keep >> j & 1, a.mask.scale);
      }
      T* y = a.y + row[u] * a.ldy + col;
      if (col >= 0 && col + 8 <= cols) {
        Storage<T>::store8(y, v);
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (col + j >= 0 && col + j < cols) Storage<T>::store1(y + j, v[j]);
      }
    }
  }
}

// Matrices whose rows start at different places of their 16-byte granules: a group of G lanes (32, or fewer where a row has fewer octets)
// takes 8 G elements of a row.  Lane l makes the block of octet l; then lane l serves the elements l, l + G, ... , so that the accesses of a group
// are contiguous whatever their alignment, and gets the mask of each from the lane that made it.  Bound by its element-wise accesses: 8192 x 4096
// bf16 with a residual 90 us, where rows that lie alike take 54 (dropout_shifted_kernel) and whole octets 30.
template <typename T>
__global__ void __launch_bounds__(kThreads) dropout_any_kernel(const __grid_constant__ DropArgs<T> a) {
  const int lane = threadIdx.x & 31, G = a.group, l = lane & (G - 1);
  const int64_t per_row = (a.octets + G - 1) / G;                 // groups
  const int64_t g = (static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x) / G;
  const int64_t row = g / per_row, o0 = (g - row * per_row) * G;
  const bool inside = row < a.rows;
  dependency_wait();
  // (Clamped to the matrix, not guarded: a guarded load is a branch with its conversion in it, and the loads then wait for each other.)
  const int64_t at = min(row, a.rows - 1);
  T x[8], r[8], b[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const int64_t c = min(o0 * 8 + j * G + l, a.cols - 1);
    x[j] = a.x[at * a.ldx + c];
    if (a.residual) r[j] = a.residual[at * a.ldr + c];
    if (a.bias) b[j] = a.bias[c];
  }
  const uint32_t keep = keep_bits(a.mask, static_cast<uint64_t>(row * a.octets + o0 + l));
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const int e = j * G + l;
    const uint32_t bits = __shfl_sync(0xFFFFFFFFu, keep, (lane & ~(G - 1)) | (e >> 3));
    const int64_t c = o0 * 8 + e;
    float v = Storage<T>::load1(x + j);
    if (a.bias) v += Storage<T>::load1(b + j);
    v = masked_plus(v, bits >> (e & 7) & 1, a.mask.scale, a.residual ? Storage<T>::load1(r + j) : 0.0f);
    if (inside && c < a.cols) Storage<T>::store1(a.y + row * a.ldy + c, v);
  }
}

// The backward pass with the bias's gradient: a block has a strip of 8 G columns and a range of rows, every thread eight fixed columns
// (an octet, or the elements l, l + G, ... where rows start anywhere) whose sums it keeps in fp32.  The sums of a block meet in shared
// memory, those of the ranges in the workspace, and column_sums_kernel adds them in a fixed order: the same bits every time.
// Four blocks on a multiprocessor, for which the grid is cut (cut_ranges): with 80 registers it was three, and a third of a second round.
// 8192 x 2048 fp16: 12.5 us and 2.5 for the sums, 4.5 TB/s in all; bound by the generator's wide multiplies, which all warps issue at once
// behind their loads, and by the ramp of the one wave of blocks.
template <typename T, bool OCTETS, typename Index>
__global__ void __launch_bounds__(kThreads, 4) dropout_columns_kernel(const __grid_constant__ DropArgs<T> a, const int64_t rows_per_range, float* partials, T* direct) {
  __shared__ float sums[kThreads * 8];
  constexpr int kRowsInFlight = sizeof(T) == 2 ? 4 : 2;
  const int lane = threadIdx.x & 31, G = a.group, l = threadIdx.x & (G - 1);
  const int row_lane = threadIdx.x / G, row_lanes = kThreads / G;
  const int64_t o0 = static_cast<int64_t>(blockIdx.x) * G, c0 = o0 * 8;
  dependency_wait();
  if (direct == nullptr) dependents_may_start();      // column_sums_kernel
  const int64_t begin = static_cast<int64_t>(blockIdx.y) * rows_per_range, end = min(begin + rows_per_range, a.rows);
  const bool none = a.mask.threshold > 65535u;
  const uint32_t least = none ? 0xFFFFFFFFu : keep_least(a.mask);
  float acc[8] = {};
  if (OCTETS) {
    const int64_t c = c0 + 8 * l;
    if (c + 8 <= a.cols) {
      // one octet of every row_lanes-th row: pointers and the block number advance by constants, the sums are kept two to an operation
      const int64_t row0 = begin + row_lane, x_step = row_lanes * a.ldx, y_step = row_lanes * a.ldy;
      const Index block_step = static_cast<Index>(row_lanes) * static_cast<Index>(a.octets);
      const T* px = a.x + row0 * a.ldx + c;
      T* py = a.y + row0 * a.ldy + c;
      Index block = static_cast<Index>(row0 * a.octets + o0 + l);
      const uint64_t scale2 = dup2(a.mask.scale);
      uint64_t acc2[4] = {};
      auto one = [&](const Octet<T>& x) {
        uint32_t words[4] = {0, 0, 0, 0};
        if (!none) block_words(a.mask, block, words);
        float v[8];
        x.unpack(v);
#pragma unroll
        for (int j = 0; j < 8; j += 2) {
          const uint64_t two = mul2(pack2(kept(words, j, least) ? v[j] : 0.0f, kept(words, j + 1, least) ? v[j + 1] : 0.0f), scale2);
          acc2[j / 2] = add2(acc2[j / 2], two);
          unpack2(two, v[j], v[j + 1]);
        }
        Storage<T>::store8(py, v);
        py += y_step;
        block += block_step;
      };
      int n = row0 < end ? static_cast<int>((end - row0 + row_lanes - 1) / row_lanes) : 0;      // (a thread's rows: a range of more than 2^31 of them for each of its 8 to 256 row lanes is more than any memory holds)
      for (; n >= kRowsInFlight; n -= kRowsInFlight) {
        Octet<T> x[kRowsInFlight];
#pragma unroll
        for (int u = 0; u < kRowsInFlight; ++u, px += x_step) x[u].load(px);
#pragma unroll
        for (int u = 0; u < kRowsInFlight; ++u) one(x[u]);
      }
      for (; n > 0; --n, px += x_step) {
        Octet<T> x;
        x.load(px);
        one(x);
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) unpack2(acc2[j], acc[2 * j], acc[2 * j + 1]);
    } else if (c < a.cols) {                                   // the end of rows that are not whole octets
      for (int64_t row = begin + row_lane; row < end; row += row_lanes) {
        const uint32_t keep = keep_bits(a.mask, static_cast<Index>(row * a.octets + o0 + l));
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          if (c + j < a.cols) {
            const float v = masked(Storage<T>::load1(a.x + row * a.ldx + c + j), keep >> j & 1, a.mask.scale);
            acc[j] += v;
            Storage<T>::store1(a.y + row * a.ldy + c + j, v);
          }
        }
      }
    }
  } else {
    for (int64_t base = begin; base < end; base += row_lanes) {      // (all lanes of a warp make every trip)
      const int64_t row = base + row_lane;
      const bool inside = row < end;
      T x[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) x[j] = a.x[min(row, end - 1) * a.ldx + min(c0 + j * G + l, a.cols - 1)];
      const uint32_t keep = keep_bits(a.mask, static_cast<Index>(row * a.octets + o0 + l));
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int e = j * G + l;
        const uint32_t bits = __shfl_sync(0xFFFFFFFFu, keep, (lane & ~(G - 1)) | (e >> 3));
        const int64_t c = c0 + e;
        if (inside && c < a.cols) {
          const float v = masked(Storage<T>::load1(x + j), bits >> (e & 7) & 1, a.mask.scale);
          acc[j] += v;
          Storage<T>::store1(a.y + row * a.ldy + c, v);
        }
      }
    }
  }
  // sums[row lane][column of the strip]
#pragma unroll
  for (int j = 0; j < 8; ++j) sums[row_lane * (8 * G) + (OCTETS ? 8 * l + j : j * G + l)] = acc[j];
  __syncthreads();
  for (int e = threadIdx.x; e < 8 * G; e += kThreads) {
    if (c0 + e < a.cols) {
      float t = 0.0f;
      for (int k = 0; k < row_lanes; ++k) t += sums[k * (8 * G) + e];
      if (direct) Storage<T>::store1(direct + c0 + e, t);      // one range: these are the sums
      else partials[blockIdx.y * a.cols + c0 + e] = t;
    }
  }
}

template <typename T>
__global__ void __launch_bounds__(256) column_sums_kernel(const float* partials, int ranges, int64_t cols, T* out) {
  __shared__ float sums[8][32];
  const int64_t c = static_cast<int64_t>(blockIdx.x) * 32 + threadIdx.x;
  dependency_wait();
  float t = 0.0f;
  if (c < cols) {
#pragma unroll 8
    for (int k = threadIdx.y; k < ranges; k += 8) t += partials[k * cols + c];
  }
  sums[threadIdx.y][threadIdx.x] = t;
  __syncthreads();
  if (threadIdx.y == 0 && c < cols) {
    for (int k = 1; k < 8; ++k) t += sums[k][threadIdx.x];
    Storage<T>::store1(out + c, t);
  }
}

// Lanes that share a row: the octets of a row, at most a warp.
int group_for(int64_t octets) {
  int g = 1;
  while (g < 32 && g < octets) g *= 2;
  return g;
}

// How the rows of a backward pass with column sums are cut: one range, whose sums need no second kernel, up to sixteen rows a thread; else
// enough ranges for four blocks on each of the 148 multiprocessors, each of at least four rows a thread.  A function of the sizes alone, so that the sums do not depend on the device.
struct Ranges {
  int64_t count, rows;
};
Ranges cut_ranges(int64_t rows, int64_t cols) {
  const int64_t octets = (cols + 7) / 8;
  const int g = group_for(octets);
  const int64_t strips = (octets + g - 1) / g, trip = static_cast<int64_t>(kThreads / g) * 4;
  const int64_t trips = (rows + trip - 1) / trip, want = trips <= 4 ? 1 : std::max<int64_t>(1, 592 / strips);
  Ranges r;
  const int64_t even = (rows + std::min(want, trips) - 1) / std::min(want, trips), lanes = kThreads / g;
  r.rows = (even + lanes - 1) / lanes * lanes;
  r.count = (rows + r.rows - 1) / r.rows;
  return r;
}

template <typename T>
int run_dropout(DropArgs<T> a, cudaStream_t st) {
  constexpr int size = sizeof(T), kPhases = 16 / size, kMany = sizeof(T) == 2 ? 4 : 2;
  a.octets = (a.cols + 7) / 8;
  a.phase = phase_of(a.x, size);
  auto alike = [&](const T* p, int64_t ld) { return phase_of(p, size) == a.phase && (a.rows == 1 || (ld - a.ldx) % kPhases == 0); };
  const bool plain = a.cols % 8 == 0 && a.phase == 0 && !a.bias && (a.rows == 1 || (a.ldx == a.cols && a.ldy == a.cols && (!a.residual || a.ldr == a.cols)));
  if (alike(a.y, a.ldy) && (!a.residual || alike(a.residual, a.ldr)) && (plain || a.cols < (int64_t{1} << 31) - 64)) {
    const bool shift = a.phase != 0 || (a.rows > 1 && a.ldx % kPhases != 0);
    a.pieces = shift ? (a.cols + kPhases - 1 + 7) / 8 : a.octets;
    a.total = a.rows * a.pieces;
    a.div = make_fast_div(static_cast<uint32_t>(std::min<int64_t>(a.pieces, 0x7FFFFFFF)));
    a.bias_octets = aligned_to(a.bias, 16);
    const bool flat = !shift && plain;
    // without a gap between the rows, but not whole octets
    const bool unbroken = a.phase == 0 && a.cols >= 8 && a.cols % 8 != 0 && a.rows > 1 && a.ldx == a.cols && a.ldy == a.cols && (!a.residual || a.ldr == a.cols);
    if (unbroken) {
      a.total = (a.rows * a.cols + 7) / 8;
      a.div = make_fast_div(static_cast<uint32_t>(a.cols));
    }
    const bool small = a.total < int64_t{148} * 8 * kThreads;
    const int64_t per_block = kThreads * (small ? 1 : kMany), blocks = (a.total + per_block - 1) / per_block;
    if (blocks > 0x7FFFFFFF) return ZGR_ETOOBIG;
    const bool far = (unbroken ? a.rows * a.cols : a.total) >= int64_t{1} << 31;      // indexes of 64 bits
    const auto kernel = far ? (unbroken ? dropout_unbroken_kernel<T, kMany, int64_t>
                               : shift  ? dropout_shifted_kernel<T, kMany, int64_t>
                               : flat   ? dropout_kernel<T, kMany, true, int64_t>
                                        : dropout_kernel<T, kMany, false, int64_t>)
                        : unbroken ? (small ? dropout_unbroken_kernel<T, 1, uint32_t> : dropout_unbroken_kernel<T, kMany, uint32_t>)
                        : shift ? (small ? dropout_shifted_kernel<T, 1, uint32_t> : dropout_shifted_kernel<T, kMany, uint32_t>)
                        : flat ? (small ? dropout_kernel<T, 1, true, uint32_t> : dropout_kernel<T, kMany, true, uint32_t>)
                               : (small ? dropout_kernel<T, 1, false, uint32_t> : dropout_kernel<T, kMany, false, uint32_t>);
    return launch_behind(kernel, static_cast<unsigned>(blocks), kThreads, 0, 1, st, a) == cudaSuccess ? ZGR_OK : ZGR_ECUDA;
  }
  a.group = group_for(a.octets);
  const int64_t groups = a.rows * ((a.octets + a.group - 1) / a.group), per_block = kThreads / a.group;
  const int64_t blocks = (groups + per_block - 1) / per_block;
  if (blocks > 0x7FFFFFFF) return ZGR_ETOOBIG;
  return launch_behind(dropout_any_kernel<T>, static_cast<unsigned>(blocks), kThreads, 0, 1, st, a) == cudaSuccess ? ZGR_OK : ZGR_ECUDA;
}

template <typename T>
int run_backward_bias(DropArgs<T> a, T* dbias, float* partials, cudaStream_t st) {
  a.octets = (a.cols + 7) / 8;
  a.group = group_for(a.octets);
  const Ranges r = cut_ranges(a.rows, a.cols);
  const int64_t strips = (a.octets + a.group - 1) / a.group;
  if (strips > 0x7FFFFFFF || r.count > 65535) return ZGR_ETOOBIG;
  const dim3 grid(static_cast<unsigned>(strips), static_cast<unsigned>(r.count));
  const bool octets = octets_aligned(a.x, a.rows, a.ldx, sizeof(T)) && octets_aligned(a.y, a.rows, a.ldy, sizeof(T));
  const bool far = a.rows * a.octets >= int64_t{1} << 32;      // block numbers of 64 bits
  const auto kernel = far ? (octets ? dropout_columns_kernel<T, true, uint64_t> : dropout_columns_kernel<T, false, uint64_t>)
                          : (octets ? dropout_columns_kernel<T, true, uint32_t> : dropout_columns_kernel<T, false, uint32_t>);
  if (launch_behind(kernel, grid, kThreads, 0, 1, st, a, r.rows, partials, r.count == 1 ? dbias : nullptr) != cudaSuccess) return ZGR_ECUDA;
  if (r.count == 1) return ZGR_OK;
  const cudaError_t e = launch_behind(column_sums_kernel<T>, static_cast<unsigned>((a.cols + 31) / 32), dim3(32, 8), 0, 1, st, partials, static_cast<int>(r.count), a.cols, dbias);
  return e == cudaSuccess ? ZGR_OK : ZGR_ECUDA;
}

template <typename T>
DropArgs<T> drop_args(const void* x, int64_t ldx, const void* bias, const void* residual, int64_t ldr, void* y, int64_t ldy, int64_t rows, int64_t cols,
                      const DropMask& mask) {
  DropArgs<T> a = {};
  a.x = static_cast<const T*>(x);
  a.bias = static_cast<const T*>(bias);
  a.residual = static_cast<const T*>(residual);
  a.y = static_cast<T*>(y);
  a.rows = rows;
  a.cols = cols;
  a.ldx = ldx;
  a.ldr = ldr;
  a.ldy = ldy;
  a.mask = mask;
  return a;
}

}  // namespace
}  // namespace zgr

using namespace zgr;

extern "C" {

int zgr_dropout(const void* x, int64_t ldx, const void* bias, const void* residual, int64_t ldr, void* y, int64_t ldy, int64_t rows, int64_t cols,
                int32_t dtype, double p, uint64_t seed, uint32_t tensor, void* stream) {
  if (!storage_known(dtype) || rows < 0 || cols < 0 || !(p >= 0.0 && p <= 1.0)) return ZGR_EINVAL;
  if (rows == 0 || cols == 0) return ZGR_OK;
  const int size = storage_size(dtype);
  if (!matrix_ok(x, rows, cols, ldx, size) || !matrix_ok(y, rows, cols, ldy, size) || (residual && !matrix_ok(residual, rows, cols, ldr, size)) ||
      !aligned_to(bias, size))
    return ZGR_EINVAL;
  const DropMask mask = make_drop_mask(p, seed, tensor);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  switch (dtype) {
    case ZGR_F32: return run_dropout(drop_args<float>(x, ldx, bias, residual, ldr, y, ldy, rows, cols, mask), st);
    case ZGR_F16: return run_dropout(drop_args<__half>(x, ldx, bias, residual, ldr, y, ldy, rows, cols, mask), st);
    default: return run_dropout(drop_args<__nv_bfloat16>(x, ldx, bias, residual, ldr, y, ldy, rows, cols, mask), st);
  }
}

int64_t zgr_dropout_backward_workspace(int64_t rows, int64_t cols) {
  if (rows < 0 || cols < 0 || (cols > 0 && rows > kMostElements / cols)) return ZGR_EINVAL;
  if (rows == 0 || cols == 0) return 0;
  const int64_t ranges = cut_ranges(rows, cols).count;
  return ranges == 1 ? 0 : ranges * cols * static_cast<int64_t>(sizeof(float));
}

int zgr_dropout_backward(const void* dy, int64_t lddy, void* dx, int64_t lddx, void* dbias, int64_t rows, int64_t cols, int32_t dtype, double p,
                         uint64_t seed, uint32_t tensor, void* workspace, int64_t workspace_bytes, void* stream) {
  if (!storage_known(dtype) || rows < 0 || cols < 0 || !(p >= 0.0 && p <= 1.0)) return ZGR_EINVAL;
  const int size = storage_size(dtype);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if ((dbias && !aligned_to(dbias, size)) || cols > kMostElements) return ZGR_EINVAL;
  if (cols == 0) return ZGR_OK;
  if (rows == 0)      // no rows: the sums are zero
    return !dbias || cudaMemsetAsync(dbias, 0, static_cast<size_t>(cols) * size, st) == cudaSuccess ? ZGR_OK : ZGR_ECUDA;
  if (!matrix_ok(dy, rows, cols, lddy, size) || !matrix_ok(dx, rows, cols, lddx, size)) return ZGR_EINVAL;
  if (!dbias) return zgr_dropout(dy, lddy, nullptr, nullptr, 0, dx, lddx, rows, cols, dtype, p, seed, tensor, stream);
  const int64_t need = zgr_dropout_backward_workspace(rows, cols);
  if (need > 0 && (!workspace || !aligned_to(workspace, 16) || workspace_bytes < need)) return ZGR_EINVAL;
  const DropMask mask = make_drop_mask(p, seed, tensor);
  float* partials = static_cast<float*>(workspace);
  switch (dtype) {
    case ZGR_F32: return run_backward_bias(drop_args<float>(dy, lddy, nullptr, nullptr, 0, dx, lddx, rows, cols, mask), static_cast<float*>(dbias), partials, st);
    case ZGR_F16: return run_backward_bias(drop_args<__half>(dy, lddy, nullptr, nullptr, 0, dx, lddx, rows, cols, mask), static_cast<__half*>(dbias), partials, st);
    default:
      return run_backward_bias(drop_args<__nv_bfloat16>(dy, lddy, nullptr, nullptr, 0, dx, lddx, rows, cols, mask), static_cast<__nv_bfloat16*>(dbias), partials, st);
  }
}

}  // extern "C"
