// The few-rows rows product of ffn_bf16_small.h with its element type, weight columns and epilogue left open: gated experts
// (ffn_gated.hip) and 8-bit integer experts (ffn_i8.hip).
#pragma once
#include "common.h"
#include "ffn_bf16_tile.h"
#include "ffn_bf16_dma.h"
#include "ffn_bf16_persist.h"
#include "ffn_bf16_small.h"
namespace flexmoe {
// =============================================================================================
// Tiles, row list, stages, segments and their sum are those of rows_gemm_small_bf16 (see there for why), on the same plan.  What is
// open:
//  * V4, the type of four sums: f32x4 (bf16 operands) or i32x4 (8-bit integers, 128 of them to a stage: one instruction takes the
//    same 16 bytes per lane in either case).  K and the operands' offsets count two-byte units, so 8-bit operands pass K / 2.
//    Sums of integers are exact: segments change nothing, and a row's bits do not depend on the other rows.
//  * GATE: a wave holds the gate's and up's values of an output in the same lane.  GATE_MIXED: the tile's weight columns are half from the
//    first half (gate), half from the second (up), 16 and 16 in turn: acc[0][i][0] and acc[0][i][1].  GATE_TURNS (not WT): 128 columns of
//    each half, whose stages alternate: acc[0][i][j] and acc[1][i][j].  That makes pieces of 256 bytes of a weight row instead of 128 -- a
//    decode step of 16 tokens (d 1024, f 4096, 21 experts) reads them at 4.9 TB/s instead of 4.2 -- but half as many tiles of twice the
//    latency: a step of 4 tokens (d 96, f 256) is 6 % slower.
//  * COLS: a tile is 128 columns and a stage 128 bytes of k, or (WT) 64 columns and 256 bytes: HBM serves pieces of 256 bytes better than
//    lines 4 KB and more apart.  With 64 columns two waves share an output block, each with half of a stage's k, and add their sums at
//    the end.
//  * rows of `in` are addressed with 64 bits, so any number of rows is served.
//  * pol.before(...) fetches what the epilogue reads ahead of the K loop, pol.epilogue(acc, tile, ...) does the rest.
// =============================================================================================
struct SmallCore {
  const bf16_t* in;              // [rows, K]
  const bf16_t* w;               // WT: [E, NC, K], else [E, K, NC]
  const i32x4* tab;              // as SmallArgs
  const int32_t* rowmap;
  int K, NC, col_tiles;          // NC: all weight columns (GATED: both halves)
  const int32_t* inmap;          // position in expert order -> row of `in` (rowmap, or gathered rows)
  float* partial;
  int* counters;
  int slots;                     // partial tiles of BM x 128 there is room for
  int rows;                      // of all buckets
};
struct SmallTile {
  int first, rows, e, ct;        // position in rowmap, rows, expert, column tile
};
template <int BM, int COLS> struct CoreCfg {
  static constexpr int kKBytes = 16384 / COLS;           // of a row's k in a stage
  static constexpr int kABytes = BM * kKBytes, kWBytes = 16384;
  static constexpr int kStage = kABytes + kWBytes;
  static constexpr int S = 81920 / kStage;               // stages: half of a compute unit's LDS
  static constexpr int kLds = S * kStage;
  static constexpr int kALoads = kABytes / 1024 / kSmallWaves, kWLoads = kWBytes / 1024 / kSmallWaves, kLoads = kALoads + kWLoads;
  static constexpr int kKUnits = kKBytes / 2;            // two-byte units of k in a stage
  static_assert(kALoads >= 1 && S >= 3 && S <= 4, "small_wait");
};
// Segments of a contraction of k_stages stages: a power of two as long as two workgroups per compute unit take them all (and three where
// that is what fits: 168 tiles of a decode step's second product, 504 workgroups instead of 336, 43.5 -> 39.6 us), each at least
// four stages long, eight where tiles have more than 16 rows on average, whose partial tiles are the more traffic.  In us, at least four and at
// least eight: 522 rows of 7 experts (d 408, f 2080) 35.0, 28.6; 4503 of 12 (training) 145.7, 136.4; 600 8-bit rows of 8 experts
// 21.7, 20.0; few rows per tile: 5 rows of one expert (d 1664, f 1608) 21.6, 26.2; 8 8-bit rows (1696 x 1808) 16.9, 18.2.
// `tiles` counts partial tiles, of which there is room for `slots`.
__host__ __device__ inline int core_segments(int tiles, int k_stages, int row_tiles, int rows, int slots) {
  const int least = rows > 16 * row_tiles ? 2 * kSmallSplitKTiles : kSmallSplitKTiles;
  int s = 1;
  while (s < kSmallSplitMax && tiles * s * 2 <= kSmallSplitTarget && k_stages >= 2 * s * least) s *= 2;
  if (s == 2 && tiles > kSmallSplitTarget / 4 && tiles * 3 <= kSmallSplitTarget && k_stages >= 3 * least) s = 3;
  while (s > 1 && (long long)tiles * s > slots) --s;
  return s;
}
enum { GATE_NONE = 0, GATE_MIXED = 1, GATE_TURNS = 2 };
// The same on the host, for a product with row_tiles row tiles in use and stages of k_units (H: accumulators, see small_core).
inline int core_segments(const SmallCore& c, int row_tiles, int k_units, int H) {
  return core_segments(row_tiles * c.col_tiles * H, (c.K + k_units - 1) / k_units, row_tiles, c.rows, c.slots);
}

template <int BM, int COLS, bool WT, int GATE, typename V4, typename Pol>
__device__ __forceinline__ void small_core(const SmallCore& p, const Pol& pol, unsigned char* smem, unsigned block, unsigned blocks) {
  typedef CoreCfg<BM, COLS> C;
  static_assert((COLS == 128 || (COLS == 64 && WT)) && !(WT && GATE == GATE_TURNS), "tile");
  constexpr int S = C::S, RB = BM / 16, NB2 = 2;         // 16-row and 16-column blocks of a wave
  constexpr int kPer = C::kKBytes / 16, kRows = 64 / kPer;      // 16-byte chunks of a row in a stage, rows of a direct load
  constexpr int kKWaves = COLS == 64 ? 2 : 1;            // waves that share an output block
  constexpr int H = GATE == GATE_TURNS ? 2 : 1;                // stages per k and accumulators: the two halves in turn
  constexpr int kActive = kSmallThreads / kKWaves;       // threads with outputs
  lds_byte_t* const sm = (lds_byte_t*)smem;
  const unsigned lds0 = __builtin_amdgcn_readfirstlane((unsigned)(uintptr_t)sm);
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int lane = threadIdx.x & 63;
  const int fr = lane & 15, fg = lane >> 4;              // fragment row (or column), group of 16 bytes of k
  const RowTabPtr tab = (RowTabPtr)p.tab;
  const int cw = wave % (kSmallWaves / kKWaves), kw = wave / (kSmallWaves / kKWaves);      // the wave's 32 columns, its part of a stage's k
  const int K = p.K, NC = p.NC, half = NC / 2;
  const int rows_act = tab[0][0];
  const int k_tiles = (K + C::kKUnits - 1) / C::kKUnits;
  const int tiles = rows_act * p.col_tiles;
  const int nseg = core_segments(tiles * H, k_tiles, rows_act, p.rows, p.slots);
  // without segments: the XCD-aware patch order; with them: tile-major, a tile's segments side by side
  const unsigned total = nseg > 1 ? (unsigned)(tiles * nseg) : patched_grid(rows_act, p.col_tiles);

  uint32_t la, lw;                                       // lane parts of the LDS fragment addresses
  la = fr * C::kKBytes + ((fg ^ (fr & (kPer - 1))) << 4);      // later 64 bytes of k: chunk index XOR 4, 8, 12
  if (WT) {
    lw = C::kABytes + cw * (NB2 * 16 * C::kKBytes) + la;
  } else {
    const int k = 8 * fg + (fr >> 2);
    const int x = ((fr >> 2) << 2) ^ ((fg & 1) << 1);
    lw = C::kABytes + k * 256 + (((wave * (NB2 * 2) + ((fr & 3) >> 1)) ^ x) << 4) + 8 * (fr & 1);
  }

  for (unsigned idx = block; idx < total; idx += blocks) {
    int rt, ct, seg = 0;
    if (nseg > 1) {
      seg = (int)(idx % nseg);
      const int tile = (int)(idx / nseg);
      rt = tile / p.col_tiles;
      ct = tile % p.col_tiles;
    } else if (!patched_tile(idx, rows_act, p.col_tiles, &rt, &ct)) {
      continue;
    }
    const i32x4 d = tab[1 + rt];
    const SmallTile t{d[0], d[1], d[2], ct};
    // first column of the tile, and columns there are (GATE: of either half)
    constexpr int kCols = GATE == GATE_MIXED ? COLS / 2 : COLS;
    const int n0 = ct * kCols, cols = min(kCols, (GATE ? half : NC) - n0);
    const int kt0 = H * (int)((long long)k_tiles * seg / nseg), kt1 = H * (int)((long long)k_tiles * (seg + 1) / nseg);      // stages
    const bf16_t* w_e = p.w + (size_t)t.e * K * NC + (WT ? (size_t)n0 * K : (size_t)n0);

    // rows of the wave's loads (rows past the tile repeat its last row) and of its outputs
    const bf16_t* aptr[C::kALoads];
    int akc[C::kALoads];                                 // the lane's chunk of a row, in two-byte units
#pragma unroll
    for (int q = 0; q < C::kALoads; ++q) {
      const int row = (wave * C::kALoads + q) * kRows + lane / kPer;
      akc[q] = ((lane % kPer) ^ (row & (kPer - 1))) * 8;
      aptr[q] = p.in + (size_t)p.inmap[t.first + min(row, t.rows - 1)] * K + akc[q];
    }
    int orow[RB];
#pragma unroll
    for (int b = 0; b < RB; ++b) orow[b] = p.rowmap[t.first + min(b * 16 + fr, t.rows - 1)];
    const auto ahead = pol.before(t, p.inmap, n0, cw, fr, fg);
    uint32_t woff[C::kWLoads];
    int wk[C::kWLoads];                                  // k (in the stage) of the lane's first element
    size_t wbase[C::kWLoads];                            // (uniform) where the load's rows start behind w_e: GATE_MIXED && WT, the up half
#pragma unroll
    for (int q = 0; q < C::kWLoads; ++q) {
      const int i = wave * C::kWLoads + q;
      wbase[q] = 0;
      if (WT) {
        int row = i * kRows + lane / kPer;
        wk[q] = ((lane % kPer) ^ (row & (kPer - 1))) * 8;
        if (GATE) {
          row = (row >> 5) * 16 + (row & 15);
          if (((i * kRows) >> 4) & 1) wbase[q] = (size_t)half * K;
        }
        woff[q] = (uint32_t)((uint32_t)min(row, cols - 1) * (uint32_t)K + wk[q]) * 2;
      } else {
        const int kr = i * 4 + (lane >> 4);
        wk[q] = kr;
        int c = (lane & 15) ^ ((kr & 3) << 2) ^ ((kr & 8) >> 2), up = 0;
        if (GATE == GATE_MIXED) {
          up = (c >> 1) & 1 ? half : 0;
          c = (c >> 2) * 2 + (c & 1);
        }
        woff[q] = (uint32_t)(kr * NC + min(c, cols / 8 - 1) * 8 + up) * 2;
      }
    }
    auto issue = [&](int kt) {
      const unsigned st = lds0 + (unsigned)((kt - kt0) % S) * C::kStage;
      const int k0 = kt / H * C::kKUnits;
      const bf16_t* wb = w_e + (WT ? (size_t)k0 : (size_t)k0 * NC + (H == 2 && (kt & 1) ? half : 0));
      if (k0 + C::kKUnits <= K) {
#pragma unroll
        for (int q = 0; q < C::kALoads; ++q) small_load_at(aptr[q] + k0, st + (wave * C::kALoads + q) * 1024);
#pragma unroll
        for (int q = 0; q < C::kWLoads; ++q) small_load(wb + wbase[q], woff[q], st + C::kABytes + (wave * C::kWLoads + q) * 1024);
      } else {                                           // past K: zeros on both sides
        const bf16_t* z = (const bf16_t*)kSmallZero + (lane & 7) * 8;
#pragma unroll
        for (int q = 0; q < C::kALoads; ++q) small_load_at(k0 + akc[q] < K ? aptr[q] + k0 : z, st + (wave * C::kALoads + q) * 1024);
#pragma unroll
        for (int q = 0; q < C::kWLoads; ++q)
          small_load_at(k0 + wk[q] < K ? (const bf16_t*)((const char*)(wb + wbase[q]) + woff[q]) : z,
                        st + C::kABytes + (wave * C::kWLoads + q) * 1024);
      }
    };

    V4 acc[H][RB][NB2];
#pragma unroll
    for (int h = 0; h < H; ++h)
#pragma unroll
      for (int i = 0; i < RB; ++i)
#pragma unroll
        for (int j = 0; j < NB2; ++j) acc[h][i][j] = V4{0, 0, 0, 0};

    __syncthreads();                                     // the previous tile's epilogue has left the stages
#pragma unroll
    for (int q = 0; q < S - 1; ++q)
      if (kt0 + q < kt1) issue(kt0 + q);
    auto step = [&](int kt, V4(&acc)[RB][NB2]) {
      small_wait<C::kLoads>(min(S - 2, kt1 - 1 - kt));
      __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
      __builtin_amdgcn_s_barrier();
      __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
      if (kt + S - 1 < kt1) issue(kt + S - 1);           // into the stage every wave has just left
      const lds_byte_t* st = sm + ((kt - kt0) % S) * C::kStage;
#pragma unroll
      for (int ks = 0; ks < 2; ++ks) {
        const uint32_t kx = (uint32_t)((kw * 2 + ks) << 6);
        bf16x8 a[RB], w[NB2];
#pragma unroll
        for (int j = 0; j < NB2; ++j) {
          if (WT) {
            w[j] = *(const __attribute__((address_space(3))) bf16x8*)(st + (lw ^ kx) + j * (16 * C::kKBytes));
          } else {
            const lds_byte_t* at = st + (lw ^ (uint32_t)(j << 5)) + ks * (32 * 256);
            const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)at);
            const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(at + 4 * 256));
            typedef short s16x8 __attribute__((ext_vector_type(8)));
            w[j] = __builtin_bit_cast(bf16x8, (s16x8)__builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
          }
        }
#pragma unroll
        for (int i = 0; i < RB; ++i) a[i] = *(const __attribute__((address_space(3))) bf16x8*)(st + (la ^ kx) + i * (16 * C::kKBytes));
#pragma unroll
        for (int i = 0; i < RB; ++i)
#pragma unroll
          for (int j = 0; j < NB2; ++j) acc[i][j] = mma_16x16(w[j], a[i], acc[i][j]);
      }
    };
    for (int kt = kt0; kt < kt1; kt += H)
#pragma unroll
      for (int h = 0; h < H; ++h) step(kt + h, acc[h]);
    __syncthreads();                                     // every wave has left the last stage
    if (kKWaves == 2) {
      typedef __attribute__((address_space(3))) V4* Ptr;
      const Ptr at = (Ptr)sm + (cw * kWave + lane);
      if (kw == 1) {
#pragma unroll
        for (int i = 0; i < RB; ++i)
#pragma unroll
          for (int j = 0; j < NB2; ++j) at[(i * NB2 + j) * kActive] = acc[0][i][j];
      }
      __syncthreads();
      if (kw == 0) {
#pragma unroll
        for (int i = 0; i < RB; ++i)
#pragma unroll
          for (int j = 0; j < NB2; ++j) acc[0][i][j] += at[(i * NB2 + j) * kActive];
      }
    }

    if (nseg > 1) {
      // partial tiles cross XCDs: see rows_gemm_small_bf16
      const int tile = rt * p.col_tiles + ct;
      typedef unsigned long long u64;
      typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
      u64* part = (u64*)(p.partial + (size_t)tile * nseg * (H * BM * COLS));
      if (kw == 0) {
#pragma unroll
        for (int h = 0; h < H; ++h)
#pragma unroll
        for (int i = 0; i < RB; ++i)
#pragma unroll
          for (int j = 0; j < NB2; ++j) {
            if (i * 16 >= t.rows) continue;              // (uniform: blocks without rows do not travel)
            u64* dst = part + (size_t)seg * (H * BM * COLS / 2) + ((h * RB + i) * NB2 + j) * (2 * kActive) + threadIdx.x;
            const u32x4 bits = __builtin_bit_cast(u32x4, acc[h][i][j]);
            __hip_atomic_store(dst, (u64)bits[0] | (u64)bits[1] << 32, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            __hip_atomic_store(dst + kActive, (u64)bits[2] | (u64)bits[3] << 32, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
          }
      }
      __builtin_amdgcn_s_waitcnt(0x0F70);                // vmcnt(0): the stores have arrived
      __syncthreads();
      if (threadIdx.x == 0) {
        const int before = __hip_atomic_fetch_add(&p.counters[tile], 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        if (before == nseg - 1) __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "agent");
        *(volatile __attribute__((address_space(3))) int*)sm = before;
      }
      __syncthreads();
      const bool last = __builtin_amdgcn_readfirstlane(*(volatile __attribute__((address_space(3))) int*)sm) == nseg - 1;
      if (!last) continue;
      if (threadIdx.x == 0) p.counters[tile] = 0;        // as the plan left it: the call's next product counts there too
      if (kw == 0) {
        // as many segments at a time as 128 registers hold: each is a trip past the L2
        constexpr int kSums = H * RB * NB2, kBatch = 32 / kSums;
        V4 s[kSums];
#pragma unroll
        for (int x = 0; x < kSums; ++x) s[x] = V4{0, 0, 0, 0};
        for (int g0 = 0; g0 < nseg; g0 += kBatch) {
          u64 lo[kBatch][kSums], hi[kBatch][kSums];
#pragma unroll
          for (int b = 0; b < kBatch; ++b)
            if (g0 + b < nseg) {
#pragma unroll
              for (int x = 0; x < kSums; ++x) {
                if (x / NB2 % RB * 16 >= t.rows) continue;
                u64* from = part + (size_t)(g0 + b) * (H * BM * COLS / 2) + x * (2 * kActive) + threadIdx.x;
                lo[b][x] = __hip_atomic_load(from, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                hi[b][x] = __hip_atomic_load(from + kActive, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
              }
            }
#pragma unroll
          for (int b = 0; b < kBatch; ++b)
            if (g0 + b < nseg) {
#pragma unroll
              for (int x = 0; x < kSums; ++x)
                if (x / NB2 % RB * 16 < t.rows) s[x] += __builtin_bit_cast(V4, u32x4{(uint32_t)lo[b][x], (uint32_t)(lo[b][x] >> 32), (uint32_t)hi[b][x], (uint32_t)(hi[b][x] >> 32)});
            }
        }
#pragma unroll
        for (int x = 0; x < kSums; ++x) acc[x / (RB * NB2)][x / NB2 % RB][x % NB2] = s[x];
      }
      __syncthreads();                                   // the flag has been read
    }
    // lane: row 16 i + fr of the tile (bucket row orow[i], there if 16 i + fr < rows), four columns from 4 fg on of 16-column block
    // 2 cw + j (GATE_MIXED: j = 0 gate, 1 up, of columns n0 + 16 cw + 4 fg ..)
    if (kw == 0) pol.epilogue(acc, t, orow, n0, cw, fr, fg, ahead);
  }
}

}  // namespace flexmoe
