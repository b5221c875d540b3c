// Expert products with 8-bit integer operands: weights with a scale per output channel, rows with a scale per row ("token"), both symmetric,
//   y[p, n] = (sum_k xq[p, k] wq[n, k]) * (xscale[p] * wscale[n]) + bias[n]
// on v_mfma_i32_16x16x64_i8 with exact int32 sums (K < 2^17, see the host check), and the expert FFN made of two of them.
//
// The weights are [E, NC, K], the contraction contiguous, like the rows: then a K tile of 64 integers is to the loads, to LDS and to the
// matrix instruction's lanes what one of 32 bf16 is, and the loops of ffn_bf16_dma.h / ffn_small_core.h serve both (K counted in two-byte units).
// One instruction does twice the products of the bf16 one on the same bytes in the same time.
//
// FFN: x is quantised row by row (the launch that also writes the products' plans), the first product reads its rows through src, its
// epilogue makes H = act(z) or act(g) * u in fp32, stores it in the layer's dtype and takes the largest |H| of every row (before that
// rounding) with integer atomics on its bits -- a maximum does not depend on their order; a pass over H makes its integers, and the second
// product reads them.  H has to be complete before its row's scale is known, so it goes through memory once as dtype and once as integers:
// 6 bytes per element (bf16): 0.21 of 2.42 ms at 32768 tokens x 2, d 2048, f 5632.  As bf16, H is rounded before its integers are, on a grid of
// half integers from 64 on: that adds 0.2 % (SiLU gates of normal numbers, 0.5 % of them that large) or 0.8 % (GELU without a gate, 2.9 %) to the
// error that 8 bits leave in H (6.5 % if half of a row is that large), where fp32 would add 4 bytes per element: 1.5 GB at that size.
//
// What bounds them: the matrix cores at hundreds of rows per expert (there, gated, both products 2.1 Pop/s; a large library product reaches
// 2.47), the weights' bytes at few (48 tokens x 2, d 2048, f 4096, 64 experts: 1.06 GB fetched in 216 us), launches and first loads between (one token
// x 2, d 1024, f 4096: 4.0, 12.0, 3.8 and 7.5 us).  A few thousand rows are bound by no unit: 3001 tokens x 2, d 784, f 2064, 16 experts keep matrix
// pipes and LDS busy for 9 to 14 % of the cycles.
// Registers: the 256 x 256 kernels spill 1 to 4 around a tile's K loop, the ragged forms up to 10, the bf16 one of I8_ACT 35; the steady K loops reload
// nothing, the last four K tiles of that last kernel do (32768 tokens x 2, f 8192, GELU: d 2048 2.74 ms, d 2064, nine rounds instead of eight, 3.26).
#include <algorithm>

#include "common.h"
#include "ffn_bf16_tile.h"
#include "ffn_bf16_dma.h"
#include "ffn_bf16_persist.h"
#include "ffn_bf16_small.h"
#include "ffn_ragged_src.h"
#include "ffn_small_core.h"

namespace flexmoe {

typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));
enum { I8_OUT = 0, I8_ACT = 1, I8_GATE = 2 };      // epilogues: y; H = act(z); H = act(g) * u

// ---- numbers and scales ------------------------------------------------------------------------
// scale = largest / 127, at least 2^-126; NaN where the largest is an infinity or NaN, so that every output of the row is NaN.
__device__ __forceinline__ float i8_scale(uint32_t largest_bits) {
  if (largest_bits >= 0x7f800000u) return __uint_as_float(0x7fc00000u);
  return fmaxf(__uint_as_float(largest_bits) / 127.f, 0x1p-126f);
}
// x / s to the nearest whole number, ties to even, within +-127: the rounded product with 1 / s is at most one off, and x - q s is exact
// in fp32 where it is close to s / 2 (q has 7 bits, and x is a multiple of a quarter of s's last bit there), so comparing it decides.
__device__ __forceinline__ int i8_round(float x, float s, float inv) {
  float q = rintf(x * inv);
  const float r = fmaf(-q, s, x), a = fabsf(r), half = 0.5f * s;
  if (a > half || (a == half && ((int)q & 1))) q += copysignf(1.f, r);
  return s == s ? (int)fminf(fmaxf(q, -127.f), 127.f) : 0;
}
__device__ __forceinline__ uint32_t i8_pack(const float* v, float s, float inv) {
  return (uint32_t)(i8_round(v[0], s, inv) & 255) | (uint32_t)(i8_round(v[1], s, inv) & 255) << 8 |
         (uint32_t)(i8_round(v[2], s, inv) & 255) << 16 | (uint32_t)i8_round(v[3], s, inv) << 24;
}
template <typename T> struct I8Load {      // 16 elements of a row
  uint4 u[sizeof(T)];
  __device__ __forceinline__ void load(const T* p) {
#pragma unroll
    for (int i = 0; i < (int)sizeof(T); ++i) u[i] = ((const uint4*)p)[i];
  }
  __device__ __forceinline__ void get(float (&v)[16]) const {
#pragma unroll
    for (int i = 0; i < (int)sizeof(T); ++i) Vec16<T>::unpack(u[i], v + i * Vec16<T>::n);
  }
};
// Rows shorter than 1024 share a wave: the lanes of a row, a power of two of 16 elements each.
__host__ __device__ inline int quant_lanes(int K) {
  int n = 1;
  while (n < kWave && n * 16 < K) n *= 2;
  return n;
}
template <typename T>
__device__ __forceinline__ void quantize_short_row(const T* __restrict__ x, int K, int lanes, bool there, int8_t* __restrict__ q, float* __restrict__ scale) {
  const int k = (int)(threadIdx.x & (lanes - 1)) * 16;
  I8Load<T> d;
  float v[16] = {};
  uint32_t m = 0;
  if (there && k < K) {
    d.load(x + k);
    d.get(v);
  }
#pragma unroll
  for (int i = 0; i < 16; ++i) m = max(m, __float_as_uint(v[i]) & 0x7fffffffu);
  for (int o = 1; o < lanes; o <<= 1) m = max(m, (uint32_t)__shfl_xor((int)m, o));
  const float s = i8_scale(m), inv = 1.f / s;
  if (there && k == 0) *scale = s;
  if (there && k < K)
    *(uint4*)(q + k) = make_uint4(i8_pack(v, s, inv), i8_pack(v + 4, s, inv), i8_pack(v + 8, s, inv), i8_pack(v + 12, s, inv));
}
__device__ __forceinline__ uint32_t wave_umax(uint32_t v) {
#pragma unroll
  for (int o = 1; o < kWave; o <<= 1) v = max(v, (uint32_t)__shfl_xor((int)v, o));
  return v;
}
// A wave's row.
template <typename T>
__device__ __forceinline__ void quantize_long_row(const T* __restrict__ x, int K, int8_t* __restrict__ q, float* __restrict__ scale) {
  const int lane = threadIdx.x & 63;
  constexpr int kHeld = 4, kStep = kWave * 16;           // 4096 elements stay in registers; of longer rows the rest is read twice
  uint32_t m = 0;
  I8Load<T> d[kHeld];
  float v[16];
#pragma unroll
  for (int c = 0; c < kHeld; ++c)
    if (c * kStep + lane * 16 < K) d[c].load(x + c * kStep + lane * 16);
  auto largest = [&](const I8Load<T>& p) {
    p.get(v);
#pragma unroll
    for (int i = 0; i < 16; ++i) m = max(m, __float_as_uint(v[i]) & 0x7fffffffu);
  };
#pragma unroll
  for (int c = 0; c < kHeld; ++c)
    if (c * kStep + lane * 16 < K) largest(d[c]);
  for (int k = kHeld * kStep + lane * 16; k < K; k += kStep) {
    I8Load<T> p;
    p.load(x + k);
    largest(p);
  }
  const float s = i8_scale(wave_umax(m)), inv = 1.f / s;
  if (lane == 0) *scale = s;
  auto out = [&](const I8Load<T>& p, int k) {
    p.get(v);
    *(uint4*)(q + k) = make_uint4(i8_pack(v, s, inv), i8_pack(v + 4, s, inv), i8_pack(v + 8, s, inv), i8_pack(v + 12, s, inv));
  };
#pragma unroll
  for (int c = 0; c < kHeld; ++c)
    if (c * kStep + lane * 16 < K) out(d[c], c * kStep + lane * 16);
  for (int k = kHeld * kStep + lane * 16; k < K; k += kStep) {
    I8Load<T> p;
    p.load(x + k);
    out(p, k);
  }
}
constexpr int kQuantWaves = 4;
// Workgroup `block` of `blocks` that quantise M rows.
template <typename T>
__device__ __forceinline__ void quantize_rows_block(const T* __restrict__ x, int M, int K, int8_t* __restrict__ q, float* __restrict__ scale, int block,
                                                    int blocks) {
  const int lanes = quant_lanes(K), per = kQuantWaves * kWave / lanes;      // rows of a workgroup at a time
  if (lanes == kWave) {
    for (int r = block * per + threadIdx.x / kWave; r < M; r += blocks * per) quantize_long_row(x + (size_t)r * K, K, q + (size_t)r * K, scale + r);
  } else {
    for (int r0 = block * per; r0 < M; r0 += blocks * per) {
      const int r = r0 + (int)threadIdx.x / lanes;       // (every lane takes part in the maximum)
      quantize_short_row(x + (size_t)r * K, K, lanes, r < M, q + (size_t)r * K, scale + r);
    }
  }
}
static int quant_blocks(int M, int K, int most) {
  const int per = kQuantWaves * kWave / quant_lanes(K);
  return std::max(1, std::min((M + per - 1) / per, most));
}
template <typename T>
__global__ __launch_bounds__(kQuantWaves * kWave) void quantize_rows_kernel(const T* __restrict__ x, int M, int K, int8_t* __restrict__ q,
                                                                            float* __restrict__ scale) {
  quantize_rows_block(x, M, K, q, scale, blockIdx.x, gridDim.x);
}

// w [E, K, NC] -> q [E, NC, K], scale [E, NC].  A workgroup has 64 columns of an expert: their largest values, then 64 x 64 tiles through LDS.
template <typename T>
__global__ __launch_bounds__(256) void quantize_weights_kernel(const T* __restrict__ w, int K, int NC, int8_t* __restrict__ q,
                                                               float* __restrict__ scale) {
  __shared__ uint32_t part[4][64];
  __shared__ int8_t tile[64][68];                        // [column][k]
  const int c = threadIdx.x & 63, g = threadIdx.x >> 6;
  const int e = blockIdx.y, n0 = blockIdx.x * 64, n = min(n0 + c, NC - 1);
  const T* we = w + (size_t)e * K * NC;
  uint32_t m = 0;
  for (int k = g; k < K; k += 4) m = max(m, __float_as_uint(Elem<T>::load(we + (size_t)k * NC + n)) & 0x7fffffffu);
  part[g][c] = m;
  __syncthreads();
  const float s = i8_scale(max(max(part[0][c], part[1][c]), max(part[2][c], part[3][c]))), inv = 1.f / s;
  if (g == 0 && n0 + c < NC) scale[(size_t)e * NC + n0 + c] = s;
  int8_t* qe = q + (size_t)e * NC * K;
  for (int k0 = 0; k0 < K; k0 += 64) {
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const int k = k0 + g * 16 + i;
      if (k < K) tile[c][g * 16 + i] = (int8_t)i8_round(Elem<T>::load(we + (size_t)k * NC + n), s, inv);
    }
    __syncthreads();
    const int row = threadIdx.x >> 2, at = (threadIdx.x & 3) * 16;      // 16 bytes of a column
    if (n0 + row < NC && k0 + at < K) {
      uint32_t v[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = *(const uint32_t*)&tile[row][at + 4 * i];
      *(uint4*)(qe + (size_t)(n0 + row) * K + k0 + at) = make_uint4(v[0], v[1], v[2], v[3]);
    }
  }
}

// H [A, f] -> integers and scales, the rows' largest values known.
template <typename T>
__global__ __launch_bounds__(256) void quantize_hidden_kernel(const T* __restrict__ h, const uint32_t* __restrict__ largest, int A, int f,
                                                              int8_t* __restrict__ q, float* __restrict__ scale) {
  const int per_row = f / 16;
  const size_t total = (size_t)A * per_row;
  for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (size_t)gridDim.x * 256) {
    const int row = (int)(i / (unsigned)per_row), c = (int)(i - (size_t)row * per_row);
    I8Load<T> d;
    d.load(h + i * 16);
    const float s = i8_scale(largest[row]), inv = 1.f / s;
    if (c == 0) scale[row] = s;
    float v[16];
    d.get(v);
    *(uint4*)(q + i * 16) = make_uint4(i8_pack(v, s, inv), i8_pack(v + 4, s, inv), i8_pack(v + 8, s, inv), i8_pack(v + 12, s, inv));
  }
}

// ---- one product -------------------------------------------------------------------------------
struct I8Args {
  const bf16_t* in;              // integers, two to an element: [rows, K]
  const bf16_t* w;               // [E, weight columns, K]
  const float* xscale;           // of the rows of `in`
  const float* wscale;           // [E, weight columns]
  const void* bias;              // [E, weight columns] of T, or null
  int K, NC;                     // K in two-byte units; output columns (I8_GATE: weight columns are 2 NC)
  int col_tiles;
  const int32_t* gsrc;           // bucket row p is row gsrc[p] / gk of `in`, or null: row p
  int gk;
  void* out;                     // T [A, NC]
  uint32_t* largest;             // [A] bits of the largest |H| of a row so far (I8_ACT, I8_GATE)
  int act;
};
// The activations of the other layers of that type: bf16 as in ffn_gated.hip, fp32 as in ffn_f32.hip.  (ReLU keeps a NaN.)  The bf16 forms in fp32
// layers would be 4 to 6 % less time (3000 tokens x 2, d 768, f 2064, 8 gated experts 94 us instead of 101), for a SiLU off by 4 times 2^-21 at z = -64.
template <int ACT, typename T> __device__ __forceinline__ float i8_act(float z) {
  if (ACT == FLEXMOE_RELU) return z < 0.f ? 0.f : z;
  if constexpr (sizeof(T) == 4) return ACT == FLEXMOE_SILU ? z * (1.f / (1.f + expf(-z))) : act_apply(z, ACT);
  if (ACT == FLEXMOE_SILU) return z * __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(z * -1.44269504088896341f));
  return act_fast<ACT>(z);
}
template <typename T> __device__ __forceinline__ void load4(const T* p, float (&v)[4]);
template <> __device__ __forceinline__ void load4<bf16_t>(const bf16_t* p, float (&v)[4]) { unpack4(*(const uint2*)p, v); }
template <> __device__ __forceinline__ void load4<float>(const float* p, float (&v)[4]) {
  const float4 u = *(const float4*)p;
  v[0] = u.x; v[1] = u.y; v[2] = u.z; v[3] = u.w;
}

// The weights' loads where a tile's 256 columns are 128 of either half, 32 and 32 in turn (see DmaSrcGate in ffn_gated.hip).
struct DmaSrcGateRows {
  DmaSrc s;
  __device__ __forceinline__ void init(const bf16_t* b, size_t ld, int cols_valid, size_t half) {
    s.base = b;
    const int tid = opaque_tid();
    const int w = tid >> 6, i = tid & 63;
#pragma unroll
    for (int q = 0; q < kOpLoads; ++q) {
      const int row = (w * kOpLoads + q) * 16 + (i >> 2);
      const int c = (i & 3) ^ dma_swz(row);
      const int in_half = min((row >> 6) * 32 + (row & 31), cols_valid - 1);
      s.off[q] = (uint32_t)(((size_t)in_half + ((row >> 5) & 1 ? half : 0)) * ld + c * 8) * 2;
    }
  }
  __device__ __forceinline__ void part(lds_byte_t* tile, int k0, int q) const { s.part(tile, k0, q); }
};

// Epilogue of a wave of the 256 x 256 kernel: rounds of 16 rows (row lane % 16 of them, four columns from 4 (lane / 16) on in each 16 x 16
// tile) in fp32, through a wave-private patch (16-byte chunks, index XOR a part of the row: free of conflicts both ways) to 16 bytes
// per lane.
template <int EPI, typename T, int ACT, bool FULL, bool BIAS>
__device__ __forceinline__ void i8_rounds(lds_byte_t* patch, const DmaAccI8& acc, const I8Args& p, const RowTile& t, int wave,
                                          const float* row_scale, const float* col_scale, uint32_t* row_largest) {
  constexpr bool GATE = EPI == I8_GATE;
  constexpr int kCols = GATE ? 32 : 64, kChunks = kCols * (int)sizeof(T) / 16;      // of the wave's block of outputs
  constexpr int kPer = 16 / (int)sizeof(T);                                         // columns of a chunk
  const int lane = opaque_tid() & 63;
  const int r = lane & 15, g4 = lane >> 4;
  const int wm = dma_wave_wm(wave), cb0 = dma_wave_cb0(wave);
  const int NC = p.NC, c0 = t.n0 + (GATE ? (cb0 >> 1) * 32 : cb0 * 32);
  const int wcols = GATE ? 2 * NC : NC;
  const float* const cs_at = col_scale + cb0 * 32 + 4 * g4;
  float b[2][2][4] = {};
  bool ok[2][2];
#pragma unroll
  for (int jj = 0; jj < 2; ++jj)
#pragma unroll
    for (int sj = 0; sj < 2; ++sj) {
      const int col = c0 + (GATE ? 0 : 32 * jj) + 16 * sj + 4 * g4;
      ok[jj][sj] = FULL || col < NC;
      if (BIAS) load4((const T*)p.bias + (size_t)t.e * wcols + min(col, NC - 4) + (GATE && jj ? NC : 0), b[jj][sj]);
    }
  auto swz_of = [](int row) { return kChunks == 4 ? (row >> 2) & 3 : kChunks == 8 ? (row >> 1) & 7 : row & 15; };
#pragma unroll
  for (int round = 0; round < 2 * MB; ++round) {
    const int i = round >> 1, sub = round & 1;
    const int row0 = (wm + 2 * i) * 32 + sub * 16;       // of the tile
    if (!FULL && row0 >= t.rows_valid) break;
    const float rs = row_scale[row0 + r];
    uint32_t most = 0;
#pragma unroll
    for (int sj = 0; sj < 2; ++sj) {
      const int e = 4 * (2 * sub + sj);
      float z[2][4];
#pragma unroll
      for (int jj = 0; jj < 2; ++jj) {
        const float4 cs = *(const float4*)(cs_at + 32 * jj + 16 * sj);
        const float c4[4] = {cs.x, cs.y, cs.z, cs.w};
#pragma unroll
        for (int q = 0; q < 4; ++q) z[jj][q] = fmaf((float)acc[i][jj][e + q], rs * c4[q], b[jj][sj][q]);
      }
#pragma unroll
      for (int jj = 0; jj < (GATE ? 1 : 2); ++jj) {
        float o[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          o[q] = EPI == I8_OUT ? z[jj][q] : EPI == I8_ACT ? i8_act<ACT, T>(z[jj][q]) : i8_act<ACT, T>(z[0][q]) * z[1][q];
          if (EPI != I8_OUT && ok[jj][sj]) most = max(most, __float_as_uint(o[q]) & 0x7fffffffu);
        }
        const int byte = ((GATE ? 0 : 32 * jj) + 16 * sj + 4 * g4) * (int)sizeof(T);
        lds_byte_t* at = patch + r * (kChunks * 16) + (((byte >> 4) ^ swz_of(r)) << 4) + (byte & 15);
        if constexpr (sizeof(T) == 2)
          *(__attribute__((address_space(3))) u32x2_t*)at = u32x2_t{pack_bf16x2(o[0], o[1]), pack_bf16x2(o[2], o[3])};
        else
          *(__attribute__((address_space(3))) f32x4*)at = f32x4{o[0], o[1], o[2], o[3]};
      }
    }
    asm volatile("" ::: "memory");                       // (a wave's LDS instructions execute in order)
    u32x4_t v[kChunks / 4];
#pragma unroll
    for (int k = 0; k < kChunks / 4; ++k) {
      const int idx = k * 64 + lane, row = idx / kChunks, ch = idx % kChunks;
      v[k] = *(const __attribute__((address_space(3))) u32x4_t*)(patch + row * (kChunks * 16) + ((ch ^ swz_of(row)) << 4));
    }
    asm volatile("" ::: "memory");
    if (EPI != I8_OUT) {
      most = max(most, (uint32_t)__shfl_xor((int)most, 16));
      most = max(most, (uint32_t)__shfl_xor((int)most, 32));
      if (g4 == 0) atomicMax(&row_largest[row0 + r], most);
    }
#pragma unroll
    for (int k = 0; k < kChunks / 4; ++k) {
      const int idx = k * 64 + lane, row = row0 + idx / kChunks, col = c0 + idx % kChunks * kPer;
      if (FULL || (row < t.rows_valid && col < NC)) *(u32x4_t*)((T*)p.out + (size_t)(t.row0 + row) * NC + col) = v[k];
    }
  }
}
#define FLEXMOE_I8_BY_ACT(act, ...)                                                        \
  switch (act) {                                                                           \
    case FLEXMOE_RELU: { constexpr int ACT = FLEXMOE_RELU; __VA_ARGS__; break; }           \
    case FLEXMOE_GELU_ERF: { constexpr int ACT = FLEXMOE_GELU_ERF; __VA_ARGS__; break; }   \
    case FLEXMOE_GELU_TANH: { constexpr int ACT = FLEXMOE_GELU_TANH; __VA_ARGS__; break; } \
    default: { constexpr int ACT = FLEXMOE_SILU; __VA_ARGS__; break; }                     \
  }

// Persistent kernel (see rows_gemm_persist_bf16).  RAGGED: K is no multiple of 128 two-byte units (ffn_ragged_src.h).
template <int EPI, typename T, bool GATHER, bool RAGGED> __global__ __launch_bounds__(kDmaThreads) void i8_persist(const I8Args p, const i32x4* row_tab) {
  constexpr bool GATE = EPI == I8_GATE;
  constexpr int TN = GATE ? BN / 2 : BN;                 // output columns of a tile
  __shared__ __align__(1024) unsigned char stage0[kDmaStageBytes];
  __shared__ __align__(1024) unsigned char stage1[kDmaStageBytes];
  __shared__ __align__(1024) unsigned char stage2[kDmaStageBytes];
  __shared__ __align__(1024) unsigned char stage3[kDmaStageBytes];
  __shared__ __align__(16) float row_scale[BM], col_scale[BN];
  __shared__ uint32_t row_largest[EPI == I8_OUT ? 1 : BM];
  lds_byte_t* const s0 = (lds_byte_t*)stage0;
  lds_byte_t* const s1 = (lds_byte_t*)stage1;
  lds_byte_t* const s2 = (lds_byte_t*)stage2;
  lds_byte_t* const s3 = (lds_byte_t*)stage3;
  typedef RaggedRows<typename std::conditional<GATE, DmaSrcGateRows, DmaSrc>::type, RAGGED> WSrc;
  typedef RaggedIssue<RaggedRows<DmaSrc, RAGGED>, WSrc> Issue;

  const RowTabPtr tab = (RowTabPtr)row_tab;
  const int K = p.K, NC = p.NC, KT = RAGGED ? ragged_k_tiles(K) : K / DK;
  const TileSeq seq = make_tile_seq(tab[0][0], p.col_tiles, false, KT);
  const unsigned G = gridDim.x;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = dma_wave_wm(wave), cb0 = dma_wave_cb0(wave);
  auto fetch_tile = [&](const TileId& id) {
    const i32x4 d = tab[1 + id.rt];
    RowTile t;
    t.row0 = d[0];
    t.rows_valid = d[1];
    t.e = d[2];
    t.n0 = id.ct * TN;
    t.cols_valid = min(TN, NC - t.n0);
    return t;
  };
  auto make_issue = [&](const RowTile& t) {
    Issue is;
    if constexpr (GATHER) is.a_src.init_gather(p.in, K, p.gsrc + t.row0, p.gk, t.rows_valid);
    else is.a_src.init(p.in + (size_t)t.row0 * K, K, t.rows_valid);
    const bf16_t* w = p.w + ((size_t)t.e * (GATE ? 2 * NC : NC) + t.n0) * K;
    if constexpr (GATE) is.w_src.init(w, K, t.cols_valid, NC);
    else is.w_src.init(w, K, t.cols_valid);
    is.a_src.K = is.w_src.K = K;
    is.k_next = 0;
    return is;
  };
  // (behind a barrier that every wave passes after its epilogue) the tile's largest values go out
  auto flush = [&](const RowTile& t) {
    if (EPI != I8_OUT && (int)threadIdx.x < t.rows_valid) {
      __hip_atomic_fetch_max(&p.largest[t.row0 + threadIdx.x], row_largest[threadIdx.x], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
  };
  // The scales come by direct loads, behind the first operand tiles: nothing waits for them before the K loop's own waits do.  (One
  // wave per 64 rows, one per 64 columns.)  The token of a gathered row is fetched a tile ahead.
  auto scale_row = [&](const RowTile& t) { return t.row0 + min((int)threadIdx.x & (BM - 1), t.rows_valid - 1); };
  auto fetch_scales = [&](const RowTile& t, int src) {
    const float* from;
    unsigned to;
    if (wave < 4) {
      from = p.xscale + (GATHER ? src / p.gk : scale_row(t));
      to = (unsigned)(uintptr_t)(__attribute__((address_space(3))) float*)row_scale + wave * 256;
    } else {
      const int c = threadIdx.x - BM;                    // column of the tile
      const int col = GATE ? (c >> 6) * 32 + (c & 31) : c;
      from = p.wscale + (size_t)t.e * (GATE ? 2 * NC : NC) + t.n0 + min(col, t.cols_valid - 1) + (GATE && (c >> 5) & 1 ? NC : 0);
      to = (unsigned)(uintptr_t)(__attribute__((address_space(3))) float*)col_scale + (wave - 4) * 256;
    }
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dword %0, off" ::"v"(from), "s"(__builtin_amdgcn_readfirstlane(to)) : "memory");
  };
  unsigned idx = blockIdx.x;
  TileId id;
  if (!find_tile(seq, &idx, G, &id)) return;
  RowTile t = fetch_tile(id), before = t;
  before.rows_valid = 0;
  int src = GATHER ? p.gsrc[scale_row(t)] : 0;
  Issue issue = make_issue(t);
  dma_prefetch3(s0, s1, s2, issue);
  for (;;) {
    DmaAccI8 acc;
    zero_acc(acc);
    unsigned nidx = idx + G;
    TileId nid;
    const bool has_next = find_tile(seq, &nidx, G, &nid);
    const RowTile tn = has_next ? fetch_tile(nid) : t;   // (none: this tile's first loads once more, waited for below and never used)
    Issue next;
    if constexpr (GATHER) next = make_issue(tn);
    dma_pipeline_cont<false, false>(
        s0, s1, s2, s3, acc, issue, KT, next, wm, cb0,
        [&]() {
          fetch_scales(t, src);
          if (EPI != I8_OUT && threadIdx.x < BM) {
            flush(before);
            row_largest[threadIdx.x] = 0;
          }
          if (GATHER) src = p.gsrc[scale_row(tn)];
        },
        [&](Issue& nx) {
          if constexpr (!GATHER) nx = make_issue(tn);
        });
    lds_byte_t* const patch = s3 + wave * 4096;
    const bool plain = t.rows_valid == BM && t.cols_valid == TN && !p.bias;      // the usual tile: no predicates, no bias
    if constexpr (EPI == I8_OUT) {
      if (plain) i8_rounds<EPI, T, FLEXMOE_RELU, true, false>(patch, acc, p, t, wave, row_scale, col_scale, row_largest);
      else if (p.bias) i8_rounds<EPI, T, FLEXMOE_RELU, false, true>(patch, acc, p, t, wave, row_scale, col_scale, row_largest);
      else i8_rounds<EPI, T, FLEXMOE_RELU, false, false>(patch, acc, p, t, wave, row_scale, col_scale, row_largest);
    } else {
      FLEXMOE_I8_BY_ACT(p.act, {
        if (plain) i8_rounds<EPI, T, ACT, true, false>(patch, acc, p, t, wave, row_scale, col_scale, row_largest);
        else if (p.bias) i8_rounds<EPI, T, ACT, false, true>(patch, acc, p, t, wave, row_scale, col_scale, row_largest);
        else i8_rounds<EPI, T, ACT, false, false>(patch, acc, p, t, wave, row_scale, col_scale, row_largest);
      })
    }
    before = t;
    if (!has_next) break;
    t = tn;
    issue = next;
    idx = nidx;
  }
  if (EPI != I8_OUT) {
    __syncthreads();
    flush(before);
  }
  __builtin_amdgcn_s_waitcnt(0x0F70);                  // vmcnt(0): nothing may still be landing in LDS when the workgroup ends
}

// Few rows.
template <int RB> struct I8Ahead {
  float rs[RB], cs[2][4], b[2][4];      // scales of the lane's rows and columns, biases
};
template <int RB, int EPI, typename T> struct I8SmallPol {
  const I8Args& p;
  __device__ __forceinline__ I8Ahead<RB> before(const SmallTile& t, const int32_t* inmap, int n0, int wave, int fr, int fg) const {
    constexpr bool GATE = EPI == I8_GATE;
    const int NC = p.NC, wcols = GATE ? 2 * NC : NC;
    I8Ahead<RB> v;
#pragma unroll
    for (int i = 0; i < RB; ++i) v.rs[i] = p.xscale[inmap[t.first + min(i * 16 + fr, t.rows - 1)]];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int col = n0 + (GATE ? wave * 16 : wave * 32 + j * 16) + fg * 4;
      const size_t at = (size_t)t.e * wcols + min(col, NC - 4) + (GATE && j ? NC : 0);
      load4(p.wscale + at, v.cs[j]);
#pragma unroll
      for (int q = 0; q < 4; ++q) v.b[j][q] = 0.f;
      if (p.bias) load4((const T*)p.bias + at, v.b[j]);
    }
    return v;
  }
  template <int ACT>
  __device__ __forceinline__ void out(const i32x4 (&acc1)[1][RB][2], const SmallTile& t, const int (&orow)[RB], int n0, int wave, int fr, int fg,
                                      const I8Ahead<RB>& v) const {
    constexpr bool GATE = EPI == I8_GATE;
    const int NC = p.NC;
    const float(&cs)[2][4] = v.cs, (&b)[2][4] = v.b;
    const i32x4(&acc)[RB][2] = acc1[0];
    bool ok[2];
#pragma unroll
    for (int j = 0; j < 2; ++j) ok[j] = n0 + (GATE ? wave * 16 : wave * 32 + j * 16) + fg * 4 < NC;
#pragma unroll
    for (int i = 0; i < RB; ++i) {
      const bool there = i * 16 + fr < t.rows;           // (all lanes take part in the maximum)
      const int row = orow[i];
      const float rs = v.rs[i];
      float z[2][4];
      uint32_t most = 0;
#pragma unroll
      for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int q = 0; q < 4; ++q) z[j][q] = fmaf((float)acc[i][j][q], rs * cs[j][q], b[j][q]);
#pragma unroll
      for (int j = 0; j < (GATE ? 1 : 2); ++j) {
        float o[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          o[q] = EPI == I8_OUT ? z[j][q] : EPI == I8_ACT ? i8_act<ACT, T>(z[j][q]) : i8_act<ACT, T>(z[0][q]) * z[1][q];
          if (EPI != I8_OUT && ok[j]) most = max(most, __float_as_uint(o[q]) & 0x7fffffffu);
        }
        if (there && ok[j]) {
          T* at = (T*)p.out + (size_t)row * NC + n0 + (GATE ? wave * 16 : wave * 32 + j * 16) + fg * 4;
          if constexpr (sizeof(T) == 2) *(uint2*)at = pack4(o[0], o[1], o[2], o[3]);
          else *(float4*)at = make_float4(o[0], o[1], o[2], o[3]);
        }
      }
      if (EPI != I8_OUT) {
        most = max(most, (uint32_t)__shfl_xor((int)most, 16));
        most = max(most, (uint32_t)__shfl_xor((int)most, 32));
        if (there && fg == 0) __hip_atomic_fetch_max(&p.largest[row], most, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      }
    }
  }
  __device__ __forceinline__ void epilogue(const i32x4 (&acc)[1][RB][2], const SmallTile& t, const int (&orow)[RB], int n0, int wave, int fr, int fg,
                                           const I8Ahead<RB>& v) const {
    if constexpr (EPI == I8_OUT) out<FLEXMOE_RELU>(acc, t, orow, n0, wave, fr, fg, v);
    else FLEXMOE_I8_BY_ACT(p.act, out<ACT>(acc, t, orow, n0, wave, fr, fg, v))
  }
};
// columns of a tile (see small_core): row tiles of 16 rows have 64
template <int BM> constexpr int i8_cols() { return BM == 64 ? 128 : 64; }
template <int BM, int EPI, typename T> __global__ __launch_bounds__(kSmallThreads, 2) void i8_small(const SmallCore c, const I8Args p) {
  __shared__ __align__(1024) unsigned char smem[CoreCfg<BM, i8_cols<BM>()>::kLds];
  const I8SmallPol<BM / 16, EPI, T> pol{p};
  small_core<BM, i8_cols<BM>(), true, EPI == I8_GATE ? GATE_MIXED : GATE_NONE, i32x4>(c, pol, smem, blockIdx.x, gridDim.x);
}

// ---- plan: what the products look up, the rows' integers and the zeros of `largest`, in one launch ----------------------
struct I8Prep {
  SmallPlan small;               // bm 0: not needed
  i32x4* row_tab;                // null: not needed
  int small_blocks, row_blocks;
  uint32_t* largest;
  int A;                         // entries of `largest`
  const void* x;                 // null: rows come quantised
  int M, K;
  int8_t* q;
  float* scale;
};
template <typename T>
__global__ __launch_bounds__(kGemmThreads) void i8_prep_kernel(const int32_t* __restrict__ voff, const int32_t* __restrict__ owner, int E, int V,
                                                               const I8Prep a) {
  const int b = blockIdx.x;
  if (b < a.small_blocks) {
    small_plan_block(voff, owner, E, V, a.small, b, a.small_blocks);
  } else if (b < a.small_blocks + a.row_blocks) {
    rows_plan_block(voff, owner, V, a.row_tab, b - a.small_blocks, a.row_blocks);
  } else {
    const int first = a.small_blocks + a.row_blocks, n = gridDim.x - first;
    for (size_t i = (size_t)(b - first) * kGemmThreads + threadIdx.x; i < (size_t)a.A; i += (size_t)n * kGemmThreads) a.largest[i] = 0;
    static_assert(kGemmThreads == kQuantWaves * kWave, "quantize_rows_block's workgroup");
    quantize_rows_block((const T*)a.x, a.M, a.K, a.q, a.scale, b - first, n);
  }
}

// ---- host --------------------------------------------------------------------------------------
// Workspace: row tiles of the few-rows kernels (room for tiles of 16 rows), row lists, counters, partial tiles; table of 256-row
// tiles; and for the FFN integers and scales of x, largest values, scales and integers of H, H.
struct I8Ws {
  i32x4* small_tab;
  int32_t *rowmap, *tokmap;
  int* counters;
  float* partial;
  i32x4* row_tab;
  int8_t* xq;
  float* xscale;
  uint32_t* largest;
  float* hscale;
  int8_t* hq;
  void* h;
};
static size_t i8_layout(char* at, int N, int d, int f, int A, int E, int V, bool ffn, I8Ws* w) {
  char* const base = at;
  auto take = [&](size_t bytes) {
    void* p = at;
    at += align_up(bytes, 256);
    return p;
  };
  w->small_tab = (i32x4*)take((size_t)(A / 16 + E + 1) * sizeof(i32x4));
  w->rowmap = (int32_t*)take((size_t)A * sizeof(int32_t));
  w->tokmap = (int32_t*)take((size_t)A * sizeof(int32_t));
  w->counters = (int*)take(kSmallSlots * sizeof(int));
  w->partial = (float*)take((size_t)kSmallSlots * 64 * SN * sizeof(float));
  w->row_tab = (i32x4*)take(rows_tab_bytes(A / BM + V));
  if (ffn) {
    w->xq = (int8_t*)take((size_t)N * d);
    w->xscale = (float*)take((size_t)N * sizeof(float));
    w->largest = (uint32_t*)take((size_t)A * sizeof(uint32_t));
    w->hscale = (float*)take((size_t)A * sizeof(float));
    w->hq = (int8_t*)take((size_t)A * f);
    w->h = take((size_t)A * f * sizeof(float));
  }
  return (size_t)(at - base);
}
size_t i8_ws_bytes(int N, int d, int f, int A, int E, int V, bool ffn) {
  I8Ws w;
  return i8_layout(nullptr, N, d, f, A, E, V, ffn, &w);
}

// Row tiles of the few-rows kernels that a product takes, 0: the 256 x 256 kernel.  wcols: its weight columns.
// 16 rows up to four rows per expert (the product is a pass over the weights).  Otherwise what is expected to be done earlier, in ns, from the
// tiles (the loads are not known here: half a ragged tile per bucket or expert):
//   256 x 256: 12000, and 6500 + 850 per 64 k and 256 tiles, a full round of them at least
//   64 x 128: 2900 + 760 per 128 k and 512 tiles, a full round at least; 3000 where few tiles are cut into segments
// Fitted to both kernels' times for 360 products (1500 to 65000 rows, 1 to 24 experts of Zipf loads, K 80 to 2064, 80 to 4096 columns): the one
// chosen took 1.001 of the faster one's time on average, 1.14 at most.  Some of them, us, 64 x 128 and 256 x 256: 6000 rows of one expert,
// K 2064, 784 columns 34, 47, 2064 columns 62, 53; K 80, 4096 columns 29, 36; 30000 rows, K 80, 784 columns 27, 35, 4096 columns 104, 73; K 2064,
// 256 columns 41, 49, 4096 columns 468, 302.  Gathered rows beyond 32-bit byte offsets: 64 x 128.
static int i8_bm(const FfnArgs& a, int K, int wcols, bool gathered, long long rows_in) {
  if (a.A <= 4 * a.E) return 16;
  if (gathered && rows_in * K >= (1ll << 31)) return 64;
  auto ceil_div = [](long long x, long long y) { return (x + y - 1) / y; };
  const long long large_tiles = (a.A / BM + (a.V + 1) / 2) * ceil_div(wcols, BN), small_tiles = (a.A / 64 + (a.E + 1) / 2) * ceil_div(wcols, SN);
  const long long large = 12000 + std::max(256ll, large_tiles) * (6500 + 850ll * ragged_k_tiles(K / 2)) / 256;
  const long long stages = ceil_div(K, 128), seg = std::max(1ll, std::min<long long>(kSmallSplitTarget / std::max(small_tiles, 1ll), stages / 8));
  const long long small = std::max<long long>(kSmallSplitTarget, small_tiles) * (2900 + 760 * ceil_div(stages, seg)) / kSmallSplitTarget + (seg > 1 ? 3000 : 0);
  return small <= large ? 64 : 0;
}
template <int EPI, typename T, bool GATHER> static void launch_i8_persist(const I8Args& p, const i32x4* row_tab, dim3 grid, hipStream_t s) {
  if (p.K % (4 * DK)) hipLaunchKernelGGL((i8_persist<EPI, T, GATHER, true>), grid, dim3(kDmaThreads), 0, s, p, row_tab);
  else hipLaunchKernelGGL((i8_persist<EPI, T, GATHER, false>), grid, dim3(kDmaThreads), 0, s, p, row_tab);
}
static SmallCore i8_core(const FfnArgs& a, const I8Args& p, int bm, int wcols, const I8Ws& w) {
  const int cols = bm == 64 ? i8_cols<64>() : i8_cols<16>();
  return SmallCore{p.in, p.w, w.small_tab, w.rowmap, p.K, wcols, (wcols + cols - 1) / cols, p.gsrc ? w.tokmap : w.rowmap, w.partial, w.counters, kSmallSlots, a.A};
}
template <int EPI, typename T>
static hipError_t launch_i8(const FfnArgs& a, I8Args p, int bm, const I8Ws& w, hipStream_t s) {
  constexpr bool GATE = EPI == I8_GATE;
  if (bm) {
    const SmallCore c = i8_core(a, p, bm, GATE ? 2 * p.NC : p.NC, w);
    const long long most = ((long long)a.A / bm + a.E) * c.col_tiles * kSmallSplitMax;
    const dim3 grid((unsigned)std::min<long long>(kSmallSplitTarget, most));
    if (bm == 16) hipLaunchKernelGGL((i8_small<16, EPI, T>), grid, dim3(kSmallThreads), 0, s, c, p);
    else hipLaunchKernelGGL((i8_small<64, EPI, T>), grid, dim3(kSmallThreads), 0, s, c, p);
    return hipGetLastError();
  }
  p.col_tiles = GATE ? (p.NC + BN / 2 - 1) / (BN / 2) : (p.NC + BN - 1) / BN;
  const dim3 grid(std::min(patched_grid(a.A / BM + a.V, p.col_tiles), 256u));
  if constexpr (EPI == I8_OUT) {
    if (!p.gsrc) {
      launch_i8_persist<EPI, T, false>(p, w.row_tab, grid, s);
      return hipGetLastError();
    }
  }
  launch_i8_persist<EPI, T, true>(p, w.row_tab, grid, s);
  return hipGetLastError();
}

// bm1, bm2: row tiles of the few-rows kernels that the products take (i8_bm), 0: the 256 x 256 kernel, which looks tiles up in another table
template <typename T>
static void launch_prep(const FfnArgs& a, int bm1, int bm2, const int32_t* src, int k, I8Prep g, const I8Ws& w, hipStream_t s) {
  const int bm = bm1 ? bm1 : bm2;
  // (waves per bucket that write the row list: one per 128 rows; per 512 rows, as in the bf16 kernels' plan, 3733 rows x 1168, 64 columns 23.7
  // instead of 21.7 us, 2074 tokens x 2, d 112, f 1424 47.0 instead of 43.3)
  g.small = SmallPlan{w.small_tab, w.rowmap, w.counters, bm, std::max(1, std::min(a.A / (a.V * 128), 2048 / a.V)), src, k, w.tokmap};
  g.small_blocks = bm ? 1 + (a.V * g.small.parts + 3) / 4 : 0;
  g.row_tab = bm1 && bm2 ? nullptr : w.row_tab;
  g.row_blocks = g.row_tab ? std::max(1, std::min(64, (a.A / BM + a.V + kGemmThreads - 1) / kGemmThreads)) : 0;
  const int quant = g.x ? quant_blocks(g.M, g.K, 2048) : 0;
  hipLaunchKernelGGL(i8_prep_kernel<T>, dim3(g.small_blocks + g.row_blocks + quant), dim3(kGemmThreads), 0, s, a.voff, a.owner, a.E, a.V, g);
}

template <typename T>
static hipError_t matmul_i8_t(const FfnArgs& a, const void* xq, const float* xscale, const int32_t* src, int N, int k, const void* wq,
                              const float* wscale, const void* bias, int K, int NC, void* y, void* ws, hipStream_t s) {
  I8Ws w;
  i8_layout((char*)ws, N, K, NC, a.A, a.E, a.V, false, &w);
  const int bm = i8_bm(a, K, NC, src != nullptr, N);
  launch_prep<T>(a, bm, bm, src, k, I8Prep{}, w, s);
  const I8Args p{(const bf16_t*)xq, (const bf16_t*)wq, xscale, wscale, bias, K / 2, NC, 0, src, k, y, nullptr, FLEXMOE_RELU};
  return launch_i8<I8_OUT, T>(a, p, bm, w, s);
}
hipError_t launch_matmul_i8(const FfnArgs& a, const void* xq, const float* xscale, const int32_t* src, int N, int k, const void* wq,
                            const float* wscale, const void* bias, int K, int NC, int dtype, void* y, void* ws, hipStream_t s) {
  if (a.A == 0) return hipSuccess;
  return dtype == FLEXMOE_BF16 ? matmul_i8_t<bf16_t>(a, xq, xscale, src, N, k, wq, wscale, bias, K, NC, y, ws, s)
                               : matmul_i8_t<float>(a, xq, xscale, src, N, k, wq, wscale, bias, K, NC, y, ws, s);
}

template <typename T>
static hipError_t ffn_i8_t(const FfnArgs& a, const void* x, const int32_t* src, int N, int k, const void* w1q, const float* w1s, const void* b1,
                           const void* w2q, const float* w2s, const void* b2, bool gated, void* yp, void* ws, hipStream_t s) {
  I8Ws w;
  i8_layout((char*)ws, N, a.d, a.f, a.A, a.E, a.V, true, &w);
  const int bm1 = i8_bm(a, a.d, gated ? 2 * a.f : a.f, true, N), bm2 = i8_bm(a, a.f, a.d, false, 0);
  I8Prep g{};
  g.largest = w.largest;
  g.A = a.A;
  g.x = x;
  g.M = N;
  g.K = a.d;
  g.q = w.xq;
  g.scale = w.xscale;
  launch_prep<T>(a, bm1, bm2, src, k, g, w, s);
  const I8Args p1{(const bf16_t*)w.xq, (const bf16_t*)w1q, w.xscale, w1s, b1, a.d / 2, a.f, 0, src, k, w.h, w.largest, a.act};
  hipError_t err = gated ? launch_i8<I8_GATE, T>(a, p1, bm1, w, s) : launch_i8<I8_ACT, T>(a, p1, bm1, w, s);
  if (err != hipSuccess) return err;
  const size_t chunks = (size_t)a.A * (a.f / 16);
  hipLaunchKernelGGL(quantize_hidden_kernel<T>, dim3((unsigned)std::min<size_t>((chunks + 255) / 256, 256 * 32)), dim3(256), 0, s, (const T*)w.h,
                     w.largest, a.A, a.f, w.hq, w.hscale);
  const I8Args p2{(const bf16_t*)w.hq, (const bf16_t*)w2q, w.hscale, w2s, b2, a.f / 2, a.d, 0, nullptr, 1, yp, nullptr, FLEXMOE_RELU};
  return launch_i8<I8_OUT, T>(a, p2, bm2, w, s);
}
hipError_t launch_ffn_i8(const FfnArgs& a, const void* x, const int32_t* src, int N, int k, const void* w1q, const float* w1s, const void* b1,
                         const void* w2q, const float* w2s, const void* b2, bool gated, int dtype, void* yp, void* ws, hipStream_t s) {
  if (a.A == 0) return hipSuccess;
  return dtype == FLEXMOE_BF16 ? ffn_i8_t<bf16_t>(a, x, src, N, k, w1q, w1s, b1, w2q, w2s, b2, gated, yp, ws, s)
                               : ffn_i8_t<float>(a, x, src, N, k, w1q, w1s, b1, w2q, w2s, b2, gated, yp, ws, s);
}

hipError_t launch_quantize_rows(const void* x, int M, int K, int dtype, void* q, float* scale, hipStream_t s) {
  if (M == 0) return hipSuccess;
  const dim3 grid((unsigned)quant_blocks(M, K, 4096));
  if (dtype == FLEXMOE_BF16)
    hipLaunchKernelGGL(quantize_rows_kernel<bf16_t>, grid, dim3(kQuantWaves * kWave), 0, s, (const bf16_t*)x, M, K, (int8_t*)q, scale);
  else
    hipLaunchKernelGGL(quantize_rows_kernel<float>, grid, dim3(kQuantWaves * kWave), 0, s, (const float*)x, M, K, (int8_t*)q, scale);
  return hipGetLastError();
}
hipError_t launch_quantize_weights(const void* w, int E, int K, int NC, int dtype, void* q, float* scale, hipStream_t s) {
  const dim3 grid((unsigned)((NC + 63) / 64), (unsigned)E);
  if (dtype == FLEXMOE_BF16)
    hipLaunchKernelGGL(quantize_weights_kernel<bf16_t>, grid, dim3(256), 0, s, (const bf16_t*)w, K, NC, (int8_t*)q, scale);
  else
    hipLaunchKernelGGL(quantize_weights_kernel<float>, grid, dim3(256), 0, s, (const float*)w, K, NC, (int8_t*)q, scale);
  return hipGetLastError();
}

}  // namespace flexmoe

// For tests: which kernel a product of 8-bit experts takes (wcols: its weight columns, 2 f with a gate), with row_tiles row tiles in use.
// out[0] row tiles of the few-rows kernel, 0: the 256 x 256 one; [1] that one's form for contractions in no whole rounds; [2] the few-rows
// kernel's contraction segments.
extern "C" void flexmoe_debug_i8_paths(int N, int k, int K, int wcols, int E, int V, int gathered, int row_tiles, long long* out) {
  using namespace flexmoe;
  const FfnArgs a{N * k, K, wcols, E, V, FLEXMOE_RELU, nullptr, nullptr};
  I8Args p{};
  p.K = K / 2;
  const int bm = i8_bm(a, K, wcols, gathered != 0, N);
  out[0] = bm;
  out[1] = !bm && p.K % (4 * DK);
  out[2] = bm ? core_segments(i8_core(a, p, bm, wcols, I8Ws{}), row_tiles, bm == 64 ? CoreCfg<64, i8_cols<64>()>::kKUnits : CoreCfg<16, i8_cols<16>()>::kKUnits, 1) : 0;
}
