// Operand loads of the direct-to-LDS pipeline for contractions of any length (gated and 8-bit experts).
#pragma once
#include "common.h"
#include "ffn_bf16_tile.h"
#include "ffn_bf16_dma.h"
#include "ffn_bf16_persist.h"
#include "ffn_bf16_small.h"
namespace flexmoe {
// The pipeline takes whole rounds of four K tiles of 32; the K tile that K ends in and those behind it read zeros past K, in both operands.
// Where K is a multiple of 128 (RAGGED false) the wrapped source is used as it is.
__host__ __device__ inline int ragged_k_tiles(int K) { return (K + 4 * DK - 1) / (4 * DK) * 4; }
__device__ __forceinline__ void ragged_load(const void* from, bool there, unsigned lds) {
  small_load_at(there ? (const bf16_t*)from : (const bf16_t*)kSmallZero + (threadIdx.x & 7) * 8, lds);
}
// Operands with the contraction contiguous (DmaSrc's loads: lane i has 16 bytes of its row's 64).
template <typename Src, bool RAGGED> struct RaggedRows : Src {
  int K;
  __device__ __forceinline__ const DmaSrc& src() const {
    if constexpr (std::is_same<Src, DmaSrc>::value) return *this;
    else return this->s;
  }
  __device__ __forceinline__ void part(lds_byte_t* tile, int k0, int q) const {
    if (!RAGGED || k0 + DK <= K) {
      Src::part(tile, k0, q);
      return;
    }
    const unsigned w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), i = threadIdx.x & 63;
    const unsigned lds0 = __builtin_amdgcn_readfirstlane((unsigned)(uintptr_t)tile) + w * (kOpLoads * 1024);
    const int k = k0 + (int)((i & 3) ^ ((i >> 3) & 3)) * 8;      // (dma_swz of the lane's row)
    ragged_load((const char*)(src().base + k0) + src().off[q], k < K, lds0 + q * 1024);
  }
};
// Operands with the contraction strided (DmaSrcT's: 32 lanes share a k row).
template <typename Src, bool RAGGED> struct RaggedCols : Src {
  int K;
  __device__ __forceinline__ const DmaSrcT& src() const {
    if constexpr (std::is_same<Src, DmaSrcT>::value) return *this;
    else return this->s;
  }
  __device__ __forceinline__ void part(lds_byte_t* tile, int k0, int q) const {
    if (!RAGGED || k0 + DK <= K) {
      Src::part(tile, k0, q);
      return;
    }
    const unsigned w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), i = threadIdx.x & 63;
    const unsigned lds0 = __builtin_amdgcn_readfirstlane((unsigned)(uintptr_t)tile) + w * (kOpLoads * 1024);
    const int k = k0 + (int)((w * kOpLoads + q) * 2 + (i >> 5));
    ragged_load((const char*)(src().base + (size_t)k0 * src().ld) + src().off[q], k < K, lds0 + q * 1024);
  }
};
template <typename ASrc, typename WSrc> struct RaggedIssue {
  ASrc a_src;
  WSrc w_src;
  int k_next;
  __device__ __forceinline__ void begin() {}
  __device__ __forceinline__ void part(lds_byte_t* stage, int q) const {
    if (q < kOpLoads) a_src.part(stage, k_next, q);
    else w_src.part(stage + kDmaTileBytes, k_next, q - kOpLoads);
  }
  __device__ __forceinline__ void end() { k_next += DK; }
};

}  // namespace flexmoe
