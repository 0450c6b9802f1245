// rf_stage.cuh -- rows of results between registers and global memory, through shared memory.
//
// Accumulators leave tensor memory with a row per lane.  Stored like that, each store instruction
// of a warp touches 32 rows, 16 bytes in each, and holds up the load/store path that every barrier
// of the CTA goes through.  So a warp turns 32 rows x 128 bytes around in 4 KB of shared memory of
// its own, and moves whole 128-byte lines, eight lanes to a row.  The loops are kept short: code
// that runs once per tile comes from the instruction caches beyond the SM's, and unrolled it took
// an attention item's epilogue of 128 columns 4,800 cycles.
#pragma once
#include <cstdint>

#include "rf_ptx.cuh"

namespace rf {

template <int BYTES>
struct ElemBits {
  using type = uint16_t;
};
template <>
struct ElemBits<4> {
  using type = uint32_t;
};

// Per warp: 32 rows of 128 bytes, their 16-byte pieces swizzled by row as TMA's 128-byte swizzle does.
constexpr int kTurnBytes = 4096;

__device__ __forceinline__ uint4& stage_at(uint4* stage, int row, int piece) {
  return stage[row * 8 + (piece ^ (row & 7))];
}
__device__ __forceinline__ int64_t shfl64(int64_t v, int lane) {
  const uint32_t lo = __shfl_sync(0xffffffffu, static_cast<uint32_t>(v), lane);
  const uint32_t hi = __shfl_sync(0xffffffffu, static_cast<uint32_t>(v >> 32), lane);
  return static_cast<int64_t>(static_cast<uint64_t>(hi) << 32 | lo);
}

// Where a warp's 32 rows lie in global memory.
struct RowSpan {
  int64_t at;    // this lane's byte offset, negative: none
  int64_t at0;   // lane 0's
  int n;         // regular: rows 0 .. n - 1 lie at at0 + row * stride, the others nowhere
  bool regular;
};
__device__ __forceinline__ RowSpan row_span(int64_t at, int64_t stride) {
  RowSpan s;
  s.at = at;
  s.at0 = shfl64(at, 0);
  s.n = __popc(__ballot_sync(0xffffffffu, at >= 0));
  const int lane = threadIdx.x & 31;
  s.regular = __all_sync(0xffffffffu, at == (lane < s.n ? s.at0 + lane * stride : -1));
  return s;
}

// Each lane's row, written to the stage (piece q at stage_at(stage, lane, q)), to base + its
// offset.
__device__ __forceinline__ void store_rows(uint4* stage, char* base, const RowSpan& s,
                                           int64_t stride) {
  const int lane = threadIdx.x & 31;
  __syncwarp();
  if (s.regular) {
    char* p = base + s.at0 + (lane >> 3) * stride + (lane & 7) * 16;
#pragma unroll
    for (int k = 0; k < 8; ++k, p += 4 * stride)
      if (4 * k + (lane >> 3) < s.n)
        *reinterpret_cast<uint4*>(p) = stage_at(stage, 4 * k + (lane >> 3), lane & 7);
  } else {
#pragma unroll 1
    for (int k = 0; k < 8; ++k) {
      const int r = 4 * k + (lane >> 3);
      const int64_t o = shfl64(s.at, r);
      if (o >= 0)
        *reinterpret_cast<uint4*>(base + o + (lane & 7) * 16) = stage_at(stage, r, lane & 7);
    }
  }
  __syncwarp();  // the stage may be written again
}

// The other way: 128 bytes per row from base + at into the stage (zeros where there is no row), in
// the background.  After await_rows, piece q of this lane's row is at stage_at(stage, lane, q).
__device__ __forceinline__ void fetch_rows(uint4* stage, const char* base, const RowSpan& s,
                                           int64_t stride) {
  const int lane = threadIdx.x & 31;
#pragma unroll 1
  for (int k = 0; k < 8; ++k) {
    const int r = 4 * k + (lane >> 3);
    const int64_t o = s.regular ? (r < s.n ? s.at0 + r * stride : -1) : shfl64(s.at, r);
    const char* src = o >= 0 ? base + o + (lane & 7) * 16 : base;
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(
                     smem_u32(&stage_at(stage, r, lane & 7))),
                 "l"(src), "r"(o >= 0 ? 16 : 0)
                 : "memory");
  }
  asm volatile("cp.async.commit_group;" ::: "memory");
}
__device__ __forceinline__ void await_rows() {
  asm volatile("cp.async.wait_all;" ::: "memory");
  __syncwarp();
}

// The same element by element, for rows off the 16-byte boundaries and columns that end within the
// 128 bytes: the first `cols` elements of BYTES (2 or 4) each.  A warp's accesses are of
// consecutive elements of a row; pairs of 16-bit ones are stored together where the row is on their
// boundary.
template <int BYTES>
__device__ __forceinline__ char* stage_elem(uint4* stage, int row, int col) {
  const int byte = col * BYTES;
  return reinterpret_cast<char*>(&stage_at(stage, row, byte >> 4)) + (byte & 15);
}
template <int BYTES>
static __device__ __noinline__ void store_elems(uint4* stage, char* base, int64_t at, int cols) {
  const int lane = threadIdx.x & 31;
  __syncwarp();
#pragma unroll 4
  for (int r = 0; r < 32; ++r) {
    const int64_t o = shfl64(at, r);
    if (o < 0) continue;
    char* row = base + o;
    if (BYTES == 4) {
      if (lane < cols)
        *reinterpret_cast<uint32_t*>(row + 4 * lane) =
            *reinterpret_cast<const uint32_t*>(stage_elem<4>(stage, r, lane));
    } else if ((reinterpret_cast<uintptr_t>(row) & 3) == 0) {
      const uint32_t two = *reinterpret_cast<const uint32_t*>(stage_elem<2>(stage, r, 2 * lane));
      if (2 * lane + 1 < cols) *reinterpret_cast<uint32_t*>(row + 4 * lane) = two;
      else if (2 * lane < cols) *reinterpret_cast<uint16_t*>(row + 4 * lane) = static_cast<uint16_t>(two);
    } else {
#pragma unroll
      for (int c = lane; c < 64; c += 32)
        if (c < cols)
          *reinterpret_cast<uint16_t*>(row + 2 * c) =
              *reinterpret_cast<const uint16_t*>(stage_elem<2>(stage, r, c));
    }
  }
  __syncwarp();
}
template <int BYTES>
static __device__ __noinline__ void fetch_elems(uint4* stage, const char* base, int64_t at, int cols) {
  const int lane = threadIdx.x & 31;
  using T = typename ElemBits<BYTES>::type;
#pragma unroll 1
  for (int r0 = 0; r0 < 32; r0 += 4) {
    T v[4][4 / BYTES];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int64_t o = shfl64(at, r0 + k);
#pragma unroll
      for (int i = 0; i < 4 / BYTES; ++i)
        v[k][i] = o >= 0 && lane + 32 * i < cols
                      ? reinterpret_cast<const T*>(base + o)[lane + 32 * i] : T(0);
    }
#pragma unroll
    for (int k = 0; k < 4; ++k)
#pragma unroll
      for (int i = 0; i < 4 / BYTES; ++i)
        *reinterpret_cast<T*>(stage_elem<BYTES>(stage, r0 + k, lane + 32 * i)) = v[k][i];
  }
  __syncwarp();
}

}  // namespace rf
