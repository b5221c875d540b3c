// Gated expert FFN per vExpert bucket in bf16, forward and backward, as grouped GEMMs on the matrix cores (fp32 sums):
//   G = X Wg + bg,  U = X Wu + bu        one product with W1 = [Wg, Wu] [d, 2 f]; Hpre = [G, U] [A, 2 f] is kept for the backward pass
//   H = act(G) * U                        in that product's epilogue, from the fp32 sums
//   Y = H W2 + b2
// and for an upstream gradient dY
//   dH = dY W2^T;   dG = dH * U * act'(G),  dU = dH * act(G)      the epilogue of dH's product; dHpre = [dG, dU]
//   dX = dHpre W1^T,  dW1 = X^T dHpre,  dW2 = H^T dY
// (dG as (dH act'(G)) U: |act'| < 1.13, so what overflows is the product itself; dH U would where a closed gate makes it small or zero)
//
// The products without an activation -- Y, dX, dW1, dW2 -- are those of an ungated layer with 2 f (W1) or f (W2) columns in the middle,
// on the kernels of ffn_bf16.hip.  The two with one have kernels here, on the same loops:
//  * a tile of the first product holds a column of G and the same column of U in the same lane: its weight columns are taken from the two
//    halves of W1 in turn, 32 and 32.  Only the addresses of the weights' loads know about it.
//  * G, U and H leave through a wave-private LDS patch as bf16 (half of what fp32 patches move): 16 bytes per lane, 64 per row.
//  * two sets of kernels (chosen in `doubled`): 256 x 256 tiles with direct-to-LDS loads for any K (a contraction
//    that is no multiple of 128 ends in zeros, ffn_ragged_src.h; Y's and dX's products are here as well for such f), and 32- or 64-row tiles for few
//    rows (small_core).
// Rounding: H is made of the fp32 sums and rounded once.  What is kept of G and U for the backward pass are 16-bit words with two mantissa
// bits more than bf16 has (keep4): as bf16 they put as much error into the gradients as the rounding of dHpre that cannot be
// avoided (rel. error of dW1 and dX, 64-bit formula: 0.0030 with bf16 words, 0.0024 with these, 0.0017 is the rounding of the output alone).
// The price: outside [2^-20, 2^12) the words have one bit less than bf16.
//
// What bounds them: the matrix cores where there are hundreds of rows per expert, the weights' bytes where there are few.  Measured:
// 32768 tokens x 2, d 2048, f 5632, 32 experts: first product 2.85 ms (1.06 PFLOP/s), Y 1.31 (1.15), dH 1.72 (0.88), dX 2.70 (1.12), both weight
// gradients 4.38 (1.03); a large library product runs at 1.42.  16 tokens x 2, d 1024, f 4096: 434 MB of weights fetched in 97 us (4.5 TB/s).
// Registers: of the ragged 256 x 256 kernels the first product's spills 16, the others 0 to 8, reloaded in a tile's last four K tiles and its epilogue, not
// in the steady loop; gated_small_bf16<64, FWD1, GATE_TURNS> spills 36 (fetched partial tiles, sums and accumulators together), none in the K loop.
#include <algorithm>

#include "common.h"
#include "ffn_bf16_host.h"
#include "ffn_bf16_tile.h"
#include "ffn_bf16_dma.h"
#include "ffn_bf16_persist.h"
#include "ffn_bf16_small.h"
#include "ffn_ragged_src.h"
#include "ffn_small_core.h"

namespace flexmoe {

// act(z) and act'(z); SiLU z s with s = 1 / (1 + e^-z): exp2 and reciprocal of the hardware, 1 ulp each
template <int ACT> __device__ __forceinline__ void gate_act(float z, float* a, float* da) {
  if (ACT == FLEXMOE_SILU) {
    const float s = __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(z * -1.44269504088896341f));
    *a = z * s;
    *da = fmaf(*a, 1.f - s, s);
  } else if (ACT == FLEXMOE_RELU) {                      // (keeps a NaN)
    *a = z < 0.f ? 0.f : z;
    *da = z > 0.f ? 1.f : 0.f;
  } else {
    act_both<ACT>(z, a, da);
  }
}

// ---- kept words --------------------------------------------------------------------------------
// Magnitudes in [2^-20, 2^12) -- all but a few of a layer's -- as sign, 0, 5 exponent and 9 mantissa bits: bits 27 .. 14 of the fp32 number
// less 2^-20's exponent.  Anything else as sign, 1, and the 14 bits below the sign (8 exponent, 6 mantissa bits), so that nothing overflows or
// vanishes, zeros, infinities and NaN included.  Either way rounded to the nearest.
constexpr uint32_t kKeepBase = (127u - 20u) << 23;
// of the first kind: the sum that holds the word in bits 31 and 27 .. 14; bits 30 .. 28 are zero if the number is of that kind
__device__ __forceinline__ uint32_t keep_sum(float a) { return __float_as_uint(a) + (0x2000u - kKeepBase); }
__device__ __forceinline__ uint32_t keep_pair(uint32_t lo, uint32_t hi) {      // two such sums' words
  const uint32_t low = ((lo >> 14) & 0x3fffu) | ((hi << 2) & 0x3fff0000u);
  return low | (__builtin_amdgcn_perm(hi, lo, 0x07060302u) & 0x80008000u);
}
__device__ __forceinline__ uint32_t keep_any(float a) {
  const uint32_t u = __float_as_uint(a), m = u & 0x7fffffffu, first = m + (0x2000u - kKeepBase);
  const uint32_t other = m > 0x7f800000u ? 0x7fffu : 0x4000u | min((m + 0xffffu + ((m >> 17) & 1u)) >> 17, 0x3fc0u);
  return ((u >> 16) & 0x8000u) | (first >> 28 ? other : first >> 14);
}
constexpr uint32_t kKeepOther = 0x70000000u;
__device__ __forceinline__ uint2 keep4(const float* v) {
  const uint32_t k[4] = {keep_sum(v[0]), keep_sum(v[1]), keep_sum(v[2]), keep_sum(v[3])};
  if ((k[0] | k[1] | k[2] | k[3]) & kKeepOther)
    return make_uint2(keep_any(v[0]) | keep_any(v[1]) << 16, keep_any(v[2]) | keep_any(v[3]) << 16);
  return make_uint2(keep_pair(k[0], k[1]), keep_pair(k[2], k[3]));
}
__device__ __forceinline__ float kept_low(uint32_t w) {
  const uint32_t m = w & 0x3fffu;
  return __uint_as_float((w << 16 & 0x80000000u) | (w & 0x4000u ? m << 17 : (m << 14) + kKeepBase));
}
__device__ __forceinline__ void kept4(uint2 w, float* v) {
  v[0] = kept_low(w.x);
  v[1] = kept_low(w.x >> 16);
  v[2] = kept_low(w.y);
  v[3] = kept_low(w.y >> 16);
}

constexpr int EPI_PLAIN_T = 4;
struct GatedArgs {
  const bf16_t* in;              // fwd: Xp, dH: dYp
  const bf16_t* w;               // fwd: W1 [E, d, 2 f], dH: W2 [E, f, d]
  const bf16_t* bias;            // [E, 2 f] or null (fwd), [E, f] or null (plain)
  int K, f, col_tiles;           // f: columns of H, or of the plain product's output
  const bf16_t* hpre_in;         // dH: Hpre [A, 2 f], kept words
  bf16_t* out0;                  // fwd: Hpre (kept words) or null, dH: dHpre [A, 2 f]
  bf16_t* out1;                  // fwd: H [A, f], dH: H or null (kept by the forward pass)
  int act;
};
typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));
__device__ __forceinline__ void store_nt16(void* p, u32x4_t v) { __builtin_nontemporal_store(v, (u32x4_t*)p); }

// Columns of a 256-column tile that the first product takes from either half of W1.
constexpr int GN = BN / 2;

// The weights' loads of the first product: DmaSrcT with tile column 32 b + c taken from column n0 + 32 (b / 2) + c of half b % 2.
struct DmaSrcGate {
  DmaSrcT s;
  __device__ __forceinline__ void init(const bf16_t* b, int f, int cols_valid) {
    s.base = b;
    s.ld = 2 * (size_t)f;
    const int tid = opaque_tid();
    const int w = tid >> 6, i = tid & 63;
#pragma unroll
    for (int q = 0; q < kOpLoads; ++q) {
      const int krow = (w * kOpLoads + q) * 2 + (i >> 5);
      const int c = dmat_chunk(krow, i & 31);
      const int in_half = min((c >> 3) * 4 + (c & 3), cols_valid / 8 - 1);
      s.off[q] = (uint32_t)((uint32_t)krow * 2u * (uint32_t)f + (uint32_t)in_half * 8u + ((c >> 2) & 1 ? (uint32_t)f : 0u)) * 2u;
    }
  }
  __device__ __forceinline__ void part(lds_byte_t* tile, int k0, int q) const { s.part(tile, k0, q); }
};

// ---- epilogues of the 256 x 256 kernels --------------------------------------------------------
// Forward.  The wave's accumulators acc[i][0] (G) and acc[i][1] (U) hold 128 rows x 32 columns, 16 x 16 tiles [2 si + sj]: lane L has row
// 16 si + L % 16, columns 16 sj + 4 (L / 16) .. .  16 rows at a time go through the patch: three [16][32] bf16 tiles (64-byte rows, chunk
// index XOR row / 4: writes and reads free of bank conflicts), read back as 16 bytes per lane.
template <int ACT, bool KEEP, bool FULL>
__device__ __forceinline__ void gated_fwd_rounds(lds_byte_t* patch, const DmaAcc& acc, const GatedArgs& p, const RowTile& t, int wm, int c0) {
  const int lane = opaque_tid() & 63;
  const int r = lane & 15, g4 = lane >> 4;
  const int f = p.f;
  float bg[2][4] = {}, bu[2][4] = {};
  if (p.bias) {
    const bf16_t* b = p.bias + (size_t)t.e * 2 * f;
#pragma unroll
    for (int sj = 0; sj < 2; ++sj) {
      const int col = min(c0 + 16 * sj + 4 * g4, f - 4);
      unpack4(*(const uint2*)(b + col), bg[sj]);
      unpack4(*(const uint2*)(b + f + col), bu[sj]);
    }
  }
  // what the lane stores: 16 bytes of row `lane / 4` of the 16
  const int srow = lane >> 2, ch = lane & 3;
  const uint32_t read_at = srow * 64 + ((ch ^ (srow >> 2)) << 4);
  const int col = c0 + ch * 8;
  const bool col_ok = FULL || col < f;
  bf16_t* const pre_t = KEEP ? p.out0 + (size_t)t.row0 * 2 * f + col : nullptr;
  uint32_t at[2];                                        // where the lane's four columns of a 16 x 16 tile go
#pragma unroll
  for (int sj = 0; sj < 2; ++sj) at[sj] = r * 64 + (((sj * 2 + (g4 >> 1)) ^ (r >> 2)) << 4) + (g4 & 1) * 8;
  bf16_t* const h_t = p.out1 + (size_t)t.row0 * f + col;
  const uint32_t row_first = wm * 32 + srow;             // of the tile, round (0, 0)
#pragma unroll
  for (int round = 0; round < 2 * MB; ++round) {
    const int i = round >> 1, sub = round & 1;
    if (!FULL && (wm + 2 * i) * 32 + sub * 16 >= t.rows_valid) break;      // (a bucket's last tile: no rows from here on)
    typedef __attribute__((address_space(3))) u32x2_t lds_u32x2;
    float gu[2][2][4];                                   // [G, U][sj]
    uint32_t other = 0;
#pragma unroll
    for (int sj = 0; sj < 2; ++sj) {
      const int e = 4 * (2 * sub + sj);
      float h[4], da;
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        gu[0][sj][q] = acc[i][0][e + q] + bg[sj][q];
        gu[1][sj][q] = acc[i][1][e + q] + bu[sj][q];
        gate_act<ACT>(gu[0][sj][q], &h[q], &da);
        h[q] *= gu[1][sj][q];
        if (KEEP) other |= keep_sum(gu[0][sj][q]) | keep_sum(gu[1][sj][q]);
      }
      *(lds_u32x2*)(patch + 2048 + at[sj]) = u32x2_t{pack_bf16x2(h[0], h[1]), pack_bf16x2(h[2], h[3])};
    }
    if (KEEP) {
      uint32_t w[2][2][2];
#pragma unroll
      for (int t2 = 0; t2 < 2; ++t2)
#pragma unroll
        for (int sj = 0; sj < 2; ++sj)
#pragma unroll
          for (int q = 0; q < 2; ++q) w[t2][sj][q] = keep_pair(keep_sum(gu[t2][sj][2 * q]), keep_sum(gu[t2][sj][2 * q + 1]));
      if (__builtin_expect(other & kKeepOther, 0)) {     // (rare, and one branch for 16 words)
#pragma unroll
        for (int t2 = 0; t2 < 2; ++t2)
#pragma unroll
          for (int sj = 0; sj < 2; ++sj)
#pragma unroll
            for (int q = 0; q < 2; ++q) w[t2][sj][q] = keep_any(gu[t2][sj][2 * q]) | keep_any(gu[t2][sj][2 * q + 1]) << 16;
      }
#pragma unroll
      for (int t2 = 0; t2 < 2; ++t2)
#pragma unroll
        for (int sj = 0; sj < 2; ++sj) *(lds_u32x2*)(patch + 1024 * t2 + at[sj]) = u32x2_t{w[t2][sj][0], w[t2][sj][1]};
    }
    asm volatile("" ::: "memory");                       // (a wave's LDS instructions execute in order)
    typedef const __attribute__((address_space(3))) u32x4_t lds_u32x4;
    u32x4_t vg, vu;
    if (KEEP) {
      vg = *(lds_u32x4*)(patch + read_at);
      vu = *(lds_u32x4*)(patch + 1024 + read_at);
    }
    const u32x4_t vh = *(lds_u32x4*)(patch + 2048 + read_at);
    asm volatile("" ::: "memory");
    const uint32_t row = row_first + i * 64 + sub * 16;
    if (FULL || (col_ok && (int)row < t.rows_valid)) {
      if (KEEP) {
        bf16_t* o = pre_t + (size_t)row * 2 * f;
        store_nt16(o, vg);
        store_nt16(o + f, vu);
      }
      store_nt16(h_t + (size_t)row * f, vh);
    }
  }
}

// dH: the wave's accumulators are 128 rows x 64 columns of dH, rounds and fp32 patch as in epilogue_rounds8.  The side inputs G and U are
// requested a round ahead (two rounds ahead spill registers: 13.08 ms instead of 13.00 for a training step of 32768 tokens, d 2048, f 5632).
template <int ACT, bool KEPT, bool FULL>
__device__ __forceinline__ void gated_dh_rounds(float* patch, int jh, const DmaAcc& acc, const GatedArgs& p, const RowTile& t, int wm, int col_base) {
  const int lane = opaque_tid() & 63;
  const int rsub = lane >> 4, c = lane & 15;
  const int f = p.f;
  constexpr int kRounds = MB * 2, kIts = 4, kAhead = 1;
  const int col = col_base + jh * 64 + c * 4;            // of H
  const bool col_ok = FULL || col < f;
  const size_t tile_at = (size_t)t.row0 * 2 * f + col;
  const bf16_t* const pre_t = p.hpre_in + tile_at;
  bf16_t* const dpre_t = p.out0 + tile_at;
  bf16_t* const h_t = KEPT ? nullptr : p.out1 + (size_t)t.row0 * f + col;
  auto row_of = [&](int round, int it) { return (wm + 2 * (round >> 1)) * 32 + (round & 1) * 16 + it * 4 + rsub; };
  uint2 sg[kAhead + 1][kIts], su[kAhead + 1][kIts];
  auto fetch_round = [&](int round) {
#pragma unroll
    for (int it = 0; it < kIts; ++it) {
      const int row = row_of(round, it);
      uint2 g = make_uint2(0, 0), u = make_uint2(0, 0);
      if (FULL || (col_ok && row < t.rows_valid)) {
        const bf16_t* at = pre_t + (size_t)((uint32_t)row * 2u) * f;
        g = *(const uint2*)at;
        u = *(const uint2*)(at + f);
      }
      sg[round % (kAhead + 1)][it] = g;
      su[round % (kAhead + 1)][it] = u;
    }
  };
  auto write_round = [&](int i, int sub) {
#pragma unroll
    for (int jj = 0; jj < 2; ++jj)
#pragma unroll
      for (int sj = 0; sj < 2; ++sj) {
        const int cc = jj * 8 + sj * 4 + rsub;
        const f32x16& a = acc[i][jj];
        const int e = 4 * (2 * sub + sj);
        *(float4*)(patch + c * 64 + ((cc ^ c) << 2)) = make_float4(a[e], a[e + 1], a[e + 2], a[e + 3]);
      }
  };
#pragma unroll
  for (int round = 0; round < kAhead; ++round) fetch_round(round);
  write_round(0, 0);
#pragma unroll
  for (int round = 0; round < kRounds; ++round) {
    if (!FULL && (wm + round / 2 * 2) * 32 + round % 2 * 16 >= t.rows_valid) break;
    if (round + kAhead < kRounds) fetch_round(round + kAhead);
    asm volatile("" ::: "memory");
    float4 v[kIts];
#pragma unroll
    for (int it = 0; it < kIts; ++it) {
      const int row = it * 4 + rsub;
      v[it] = *(const float4*)(patch + row * 64 + ((c ^ row) << 2));
    }
    asm volatile("" ::: "memory");
    if (round + 1 < kRounds) write_round((round + 1) >> 1, (round + 1) & 1);
    asm volatile("" ::: "memory");
#pragma unroll
    for (int it = 0; it < kIts; ++it) {
      float g[4], u[4], dh[4] = {v[it].x, v[it].y, v[it].z, v[it].w}, dg[4], du[4], h[4];
      kept4(sg[round % (kAhead + 1)][it], g);
      kept4(su[round % (kAhead + 1)][it], u);
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        float a, da;
        gate_act<ACT>(g[q], &a, &da);
        dg[q] = dh[q] * da * u[q];
        du[q] = dh[q] * a;
        h[q] = a * u[q];
      }
      const int row = row_of(round, it);
      if (FULL || (col_ok && row < t.rows_valid)) {
        bf16_t* o = dpre_t + (size_t)((uint32_t)row * 2u) * f;
        store_nt8(o, pack4(dg[0], dg[1], dg[2], dg[3]));
        store_nt8(o + f, pack4(du[0], du[1], du[2], du[3]));
        if (!KEPT) store_nt8(h_t + (size_t)row * f, pack4(h[0], h[1], h[2], h[3]));
      }
    }
  }
}

// The plain product: 128 rows x 64 columns, 16 rows at a time as [16][64] bf16 (128-byte rows, chunk index XOR row / 2).
template <bool FULL>
__device__ __forceinline__ void gated_plain_rounds(lds_byte_t* patch, const DmaAcc& acc, const GatedArgs& p, const RowTile& t, int wm, int c0) {
  const int lane = opaque_tid() & 63;
  const int r = lane & 15, g4 = lane >> 4;
  const int NC = p.f;
  float b[2][2][4] = {};
  if (p.bias) {
#pragma unroll
    for (int jj = 0; jj < 2; ++jj)
#pragma unroll
      for (int sj = 0; sj < 2; ++sj) unpack4(*(const uint2*)(p.bias + (size_t)t.e * NC + min(c0 + 32 * jj + 16 * sj + 4 * g4, NC - 4)), b[jj][sj]);
  }
#pragma unroll
  for (int round = 0; round < 2 * MB; ++round) {
    const int i = round >> 1, sub = round & 1;
    if (!FULL && (wm + 2 * i) * 32 + sub * 16 >= t.rows_valid) break;
#pragma unroll
    for (int jj = 0; jj < 2; ++jj)
#pragma unroll
      for (int sj = 0; sj < 2; ++sj) {
        const int e = 4 * (2 * sub + sj);
        const f32x16& a = acc[i][jj];
        const float* v = b[jj][sj];
        *(__attribute__((address_space(3))) u32x2_t*)(patch + r * 128 + (((jj * 4 + sj * 2 + (g4 >> 1)) ^ (r >> 1)) << 4) + (g4 & 1) * 8) =
            u32x2_t{pack_bf16x2(a[e] + v[0], a[e + 1] + v[1]), pack_bf16x2(a[e + 2] + v[2], a[e + 3] + v[3])};
      }
    asm volatile("" ::: "memory");                       // (a wave's LDS instructions execute in order)
    u32x4_t v[2];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const int row = k * 8 + (lane >> 3);
      v[k] = *(const __attribute__((address_space(3))) u32x4_t*)(patch + row * 128 + (((lane & 7) ^ (row >> 1)) << 4));
    }
    asm volatile("" ::: "memory");
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const int row = (wm + 2 * i) * 32 + sub * 16 + k * 8 + (lane >> 3), col = c0 + (lane & 7) * 8;
      if (FULL || (row < t.rows_valid && col < NC)) *(u32x4_t*)(p.out0 + (size_t)(t.row0 + row) * NC + col) = v[k];
    }
  }
}

template <int EPI, int ACT>
__device__ __forceinline__ void gated_epilogue(unsigned char* stage, const DmaAcc& acc, const GatedArgs& p, const RowTile& t, int wave) {
  const int wm = dma_wave_wm(wave), wn = wave & 1, hh = wave >> 2;
  unsigned char* patch = stage + wave * 4096;
  if (EPI == EPI_FWD1) {
    const int c0 = t.n0 + (dma_wave_cb0(wave) >> 1) * 32;
    const bool full = t.rows_valid == BM && t.n0 + GN <= p.f;
    if (p.out0) {
      if (full) gated_fwd_rounds<ACT, true, true>((lds_byte_t*)patch, acc, p, t, wm, c0);
      else gated_fwd_rounds<ACT, true, false>((lds_byte_t*)patch, acc, p, t, wm, c0);
    } else {
      gated_fwd_rounds<ACT, false, false>((lds_byte_t*)patch, acc, p, t, wm, c0);
    }
  } else {
    const int col_base = t.n0 + wn * (NB * 32);
    if (t.rows_valid == BM && t.n0 + BN <= p.f) gated_dh_rounds<ACT, EPI == EPI_DHQ, true>((float*)patch, hh, acc, p, t, wm, col_base);
    else gated_dh_rounds<ACT, EPI == EPI_DHQ, false>((float*)patch, hh, acc, p, t, wm, col_base);
  }
}
#define FLEXMOE_BY_ACT(act, call)                       \
  switch (act) {                                        \
    case FLEXMOE_RELU: { constexpr int ACT = FLEXMOE_RELU; call; break; }          \
    case FLEXMOE_GELU_ERF: { constexpr int ACT = FLEXMOE_GELU_ERF; call; break; }  \
    case FLEXMOE_GELU_TANH: { constexpr int ACT = FLEXMOE_GELU_TANH; call; break; } \
    default: { constexpr int ACT = FLEXMOE_SILU; call; break; }                    \
  }

// The persistent kernel of these products (see rows_gemm_persist_bf16): 256 workgroups walk the tiles, the next tile's first loads go out
// while the current K loop drains.  EPI_FWD1: a tile is 256 rows x 128 columns of H; EPI_DH, EPI_DHQ: 256 of dH; EPI_PLAIN: 256 of Y,
// EPI_PLAIN_T: of dX (W1 [d, 2 f], the contraction contiguous).
template <int EPI, bool RAGGED> __global__ __launch_bounds__(kDmaThreads) void gated_persist_bf16(const GatedArgs p, const i32x4* row_tab) {
  constexpr bool FWD = EPI == EPI_FWD1, STRIDED = FWD || EPI == EPI_PLAIN;
  __shared__ __align__(1024) unsigned char stage0[kDmaStageBytes];
  __shared__ __align__(1024) unsigned char stage1[kDmaStageBytes];
  __shared__ __align__(1024) unsigned char stage2[kDmaStageBytes];
  __shared__ __align__(1024) unsigned char stage3[kDmaStageBytes];
  lds_byte_t* const s0 = (lds_byte_t*)stage0;
  lds_byte_t* const s1 = (lds_byte_t*)stage1;
  lds_byte_t* const s2 = (lds_byte_t*)stage2;
  lds_byte_t* const s3 = (lds_byte_t*)stage3;
  typedef typename std::conditional<FWD, RaggedCols<DmaSrcGate, RAGGED>,
                                    typename std::conditional<STRIDED, RaggedCols<DmaSrcT, RAGGED>, RaggedRows<DmaSrc, RAGGED>>::type>::type WSrc;
  typedef RaggedIssue<RaggedRows<DmaSrc, RAGGED>, WSrc> Issue;

  const RowTabPtr tab = (RowTabPtr)row_tab;
  const int K = p.K, f = p.f, KT = RAGGED ? ragged_k_tiles(K) : K / DK;
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
    t.n0 = id.ct * (FWD ? GN : BN);
    t.cols_valid = min(FWD ? GN : BN, f - t.n0);
    return t;
  };
  auto make_issue = [&](const RowTile& t) {
    Issue is;
    is.a_src.init(p.in + (size_t)t.row0 * K, K, t.rows_valid);
    if constexpr (FWD) is.w_src.init(p.w + (size_t)t.e * K * 2 * f + t.n0, f, t.cols_valid);
    else if constexpr (STRIDED) is.w_src.init(p.w + (size_t)t.e * K * f + t.n0, f, t.cols_valid);
    else is.w_src.init(p.w + (size_t)t.e * K * f + (size_t)t.n0 * K, K, t.cols_valid);
    is.a_src.K = is.w_src.K = K;
    is.k_next = 0;
    return is;
  };
  unsigned idx = blockIdx.x;
  TileId id;
  if (!find_tile(seq, &idx, G, &id)) return;
  RowTile t = fetch_tile(id);
  Issue issue = make_issue(t);
  dma_prefetch3(s0, s1, s2, issue);
  for (;;) {
    DmaAcc acc;
    zero_acc(acc);
    unsigned nidx = idx + G;
    TileId nid;
    const bool has_next = find_tile(seq, &nidx, G, &nid);
    const RowTile tn = has_next ? fetch_tile(nid) : t;   // (none: this tile's first loads once more, waited for below and never used)
    Issue next;
    dma_pipeline_cont<false, STRIDED>(s0, s1, s2, s3, acc, issue, KT, next, wm, cb0, []() {}, [&](Issue& nx) { nx = make_issue(tn); });
    if constexpr (EPI == EPI_PLAIN || EPI == EPI_PLAIN_T) {
      if (t.rows_valid == BM && t.cols_valid == BN) gated_plain_rounds<true>(s3 + wave * 4096, acc, p, t, wm, t.n0 + cb0 * 32);
      else gated_plain_rounds<false>(s3 + wave * 4096, acc, p, t, wm, t.n0 + cb0 * 32);
    } else {
      FLEXMOE_BY_ACT(p.act, (gated_epilogue<EPI, ACT>(stage3, acc, p, t, wave)))
    }
    if (!has_next) break;
    t = tn;
    issue = next;
    idx = nidx;
  }
  __builtin_amdgcn_s_waitcnt(0x0F70);                  // vmcnt(0): nothing may still be landing in LDS when the workgroup ends
}

// ---- few rows ----------------------------------------------------------------------------------
template <int BM, int EPI, int GATE> struct GatedSmallPol {
  const GatedArgs& p;
  // acc: [G, U] (fwd) or [dH]
  template <int ACT, int H, int RB>
  __device__ __forceinline__ void out(const f32x4 (&acc)[H][RB][2], const SmallTile& t, const int (&orow)[RB], int n0, int wave, int fr, int fg) const {
    const int f = p.f;
#pragma unroll
    for (int i = 0; i < RB; ++i) {
      if (i * 16 + fr >= t.rows) continue;
      const size_t row = orow[i];
      if (EPI == EPI_FWD1) {
#pragma unroll
        for (int j = 0; j < H; ++j) {                    // (mixed: G and U are the two column blocks, else the two accumulators)
          const int col = n0 + (H == 2 ? wave * 32 + j * 16 : wave * 16) + fg * 4;
          if (col >= f) continue;
          f32x4 g = acc[0][i][j], u = H == 2 ? acc[H - 1][i][j] : acc[0][i][1];
          if (p.bias) {
            float b[4], bu[4];
            unpack4(*(const uint2*)(p.bias + (size_t)t.e * 2 * f + col), b);
            unpack4(*(const uint2*)(p.bias + (size_t)t.e * 2 * f + f + col), bu);
#pragma unroll
            for (int q = 0; q < 4; ++q) {
              g[q] += b[q];
              u[q] += bu[q];
            }
          }
          float h[4], da;
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            gate_act<ACT>(g[q], &h[q], &da);
            h[q] *= u[q];
          }
          if (p.out0) {
            const float vg[4] = {g[0], g[1], g[2], g[3]}, vu[4] = {u[0], u[1], u[2], u[3]};
            *(uint2*)(p.out0 + row * 2 * f + col) = keep4(vg);
            *(uint2*)(p.out0 + row * 2 * f + f + col) = keep4(vu);
          }
          *(uint2*)(p.out1 + row * f + col) = pack4(h[0], h[1], h[2], h[3]);
        }
      } else {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const int col = n0 + wave * 32 + j * 16 + fg * 4;
          if (col >= f) continue;
          float g[4], u[4], dg[4], du[4], h[4];
          kept4(*(const uint2*)(p.hpre_in + row * 2 * f + col), g);
          kept4(*(const uint2*)(p.hpre_in + row * 2 * f + f + col), u);
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            const float dh = acc[0][i][j][q];
            float a, da;
            gate_act<ACT>(g[q], &a, &da);
            dg[q] = dh * da * u[q];
            du[q] = dh * a;
            h[q] = a * u[q];
          }
          *(uint2*)(p.out0 + row * 2 * f + col) = pack4(dg[0], dg[1], dg[2], dg[3]);
          *(uint2*)(p.out0 + row * 2 * f + f + col) = pack4(du[0], du[1], du[2], du[3]);
          if (EPI == EPI_DH) *(uint2*)(p.out1 + row * f + col) = pack4(h[0], h[1], h[2], h[3]);
        }
      }
    }
  }
  __device__ __forceinline__ int before(const SmallTile&, const int32_t*, int, int, int, int) const { return 0; }
  template <int H, int RB>
  __device__ __forceinline__ void epilogue(const f32x4 (&acc)[H][RB][2], const SmallTile& t, const int (&orow)[RB], int n0, int wave, int fr, int fg, int) const {
    FLEXMOE_BY_ACT(p.act, (out<ACT, H, RB>(acc, t, orow, n0, wave, fr, fg)))
  }
};
template <int BM, int EPI, int GATE> __global__ __launch_bounds__(kSmallThreads, 2) void gated_small_bf16(const SmallCore c, const GatedArgs p) {
  __shared__ __align__(1024) unsigned char smem[CoreCfg<BM, SN>::kLds];
  const GatedSmallPol<BM, EPI, GATE> pol{p};
  small_core<BM, SN, EPI != EPI_FWD1, GATE, f32x4>(c, pol, smem, blockIdx.x, gridDim.x);
}

// The second product of few rows, out [rows, f] = in [rows, K] W [E, K, f] + bias: the same loop again, for its segments.
template <int BM> struct GatedOutPol {
  const GatedArgs& p;
  __device__ __forceinline__ int before(const SmallTile&, const int32_t*, int, int, int, int) const { return 0; }
  template <int RB>
  __device__ __forceinline__ void epilogue(const f32x4 (&acc)[1][RB][2], const SmallTile& t, const int (&orow)[RB], int n0, int wave, int fr, int fg, int) const {
#pragma unroll
    for (int i = 0; i < RB; ++i) {
      if (i * 16 + fr >= t.rows) continue;
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const int col = n0 + wave * 32 + j * 16 + fg * 4;
        if (col >= p.f) continue;
        f32x4 c = acc[0][i][j];
        if (p.bias) {
          float b[4];
          unpack4(*(const uint2*)(p.bias + (size_t)t.e * p.f + col), b);
#pragma unroll
          for (int q = 0; q < 4; ++q) c[q] += b[q];
        }
        *(uint2*)(p.out0 + (size_t)orow[i] * p.f + col) = pack4(c[0], c[1], c[2], c[3]);
      }
    }
  }
};
template <int BM> __global__ __launch_bounds__(kSmallThreads, 2) void gated_out_small_bf16(const SmallCore c, const GatedArgs p) {
  __shared__ __align__(1024) unsigned char smem[CoreCfg<BM, SN>::kLds];
  const GatedOutPol<BM> pol{p};
  small_core<BM, SN, false, GATE_NONE, f32x4>(c, pol, smem, blockIdx.x, gridDim.x);
}

// ---- host ----------------------------------------------------------------------------------------
static unsigned small_grid(const FfnArgs& a, int bm, int col_tiles) {
  return (unsigned)std::min<long long>(kSmallSplitTarget, ((long long)a.A / bm + a.E) * col_tiles * kSmallSplitMax);
}
template <int EPI> static void launch_persist(const FfnArgs& a, const GatedArgs& p, const RowsKernels& rk, hipStream_t s) {
  const dim3 grid(std::min(patched_grid(a.A / BM + a.V, p.col_tiles), 256u));
  if constexpr (EPI != EPI_PLAIN && EPI != EPI_PLAIN_T) {
    if (p.K % (4 * DK) == 0) {
      hipLaunchKernelGGL((gated_persist_bf16<EPI, false>), grid, dim3(kDmaThreads), 0, s, p, (const i32x4*)rk.row_tab);
      return;
    }
  }
  hipLaunchKernelGGL((gated_persist_bf16<EPI, true>), grid, dim3(kDmaThreads), 0, s, p, (const i32x4*)rk.row_tab);
}
// (a: planned as a layer with a.f = 2 f, rows_kernels)
static SmallCore gated_out_core(const FfnArgs& a, const RowsKernels& rk, const bf16_t* in, const bf16_t* w) {
  return SmallCore{in, w, rk.small.tab, rk.small.rowmap, a.f / 2, a.d, (a.d + SN - 1) / SN, rk.small.rowmap, rk.small_partial, rk.small.counters,
                   rk.small_slots, a.A};
}
// The first product (fwd) or dH's.  turns: the halves of W1 in turn, where that leaves a tile for every workgroup (a row tile per expert that can
// have rows), else mixed.
static SmallCore gated_core(const FfnArgs& a, const RowsKernels& rk, bool fwd, const bf16_t* in, const bf16_t* w, bool* turns) {
  const int f = a.f / 2;
  *turns = fwd && (long long)std::min(a.A, a.E) * ((f + SN - 1) / SN) >= kSmallSplitTarget;
  const int cols = fwd && !*turns ? SN / 2 : SN;
  return SmallCore{in, w, rk.small.tab, rk.small.rowmap, a.d, fwd ? 2 * f : f, (f + cols - 1) / cols, rk.small.rowmap, rk.small_partial,
                   rk.small.counters, rk.small_slots, a.A};
}
static hipError_t launch_gated_out(const FfnArgs& a, const void* h, const void* w2, const void* b2, void* yp, void* ws, hipStream_t s) {
  const int f = a.f / 2;
  const RowsKernels rk = rows_kernels(a, ws);
  if (!rk.small.bm && f % 128 == 0) return launch_rows_plain(a, h, w2, b2, f, yp, ws, s);
  const GatedArgs p{(const bf16_t*)h, (const bf16_t*)w2, (const bf16_t*)b2, f, a.d, (a.d + BN - 1) / BN, nullptr, (bf16_t*)yp, nullptr, 0};
  if (!rk.small.bm) {
    launch_persist<EPI_PLAIN>(a, p, rk, s);
    return hipGetLastError();
  }
  const SmallCore c = gated_out_core(a, rk, p.in, p.w);
  const dim3 grid(small_grid(a, rk.small.bm, c.col_tiles));
  if (rk.small.bm == 32) hipLaunchKernelGGL(gated_out_small_bf16<32>, grid, dim3(kSmallThreads), 0, s, c, p);
  else hipLaunchKernelGGL(gated_out_small_bf16<64>, grid, dim3(kSmallThreads), 0, s, c, p);
  return hipGetLastError();
}
template <int EPI>
static hipError_t launch_gated(const FfnArgs& a, const void* in, const void* w, const void* bias, const void* hpre_in, void* out0, void* out1,
                               void* ws, hipStream_t s) {
  constexpr bool FWD = EPI == EPI_FWD1;
  const int f = a.f / 2, K = a.d;
  const RowsKernels rk = rows_kernels(a, ws);
  const GatedArgs p{(const bf16_t*)in, (const bf16_t*)w, (const bf16_t*)bias, K, f, FWD ? (f + GN - 1) / GN : (f + BN - 1) / BN,
                    (const bf16_t*)hpre_in, (bf16_t*)out0, (bf16_t*)out1, a.act};
  if (rk.small.bm) {
    bool turns;
    const SmallCore c = gated_core(a, rk, FWD, p.in, p.w, &turns);
    const dim3 grid(small_grid(a, rk.small.bm, c.col_tiles));
    constexpr int kGate = FWD ? GATE_MIXED : GATE_NONE;
    if constexpr (FWD) {
      if (turns) {
        if (rk.small.bm == 32) hipLaunchKernelGGL((gated_small_bf16<32, EPI, GATE_TURNS>), grid, dim3(kSmallThreads), 0, s, c, p);
        else hipLaunchKernelGGL((gated_small_bf16<64, EPI, GATE_TURNS>), grid, dim3(kSmallThreads), 0, s, c, p);
        return hipGetLastError();
      }
    }
    if (rk.small.bm == 32) hipLaunchKernelGGL((gated_small_bf16<32, EPI, kGate>), grid, dim3(kSmallThreads), 0, s, c, p);
    else hipLaunchKernelGGL((gated_small_bf16<64, EPI, kGate>), grid, dim3(kSmallThreads), 0, s, c, p);
    return hipGetLastError();
  }
  launch_persist<EPI>(a, p, rk, s);
  return hipGetLastError();
}

// Past the line of ungated layers the few-rows kernels with 64-row tiles are taken where a pass's two rows products are expected to be
// done earlier on them, in ns, from the tiles (the loads are not known here: half a ragged tile per bucket or expert):
//   256 x 256: 21000, and 4000 + 880 per 32 k and 256 tiles, a full round of them at least
//   64 x 128: 2600 + 860 per 64 k and 512 tiles, a full round at least; 4000 where few tiles are cut into segments
// Fitted to both kernels' times for 240 layers (2600 to 60000 rows, d 64 to 1500, f 64 to 4100, 1 to 40 experts of Zipf loads, forward and
// training): the one chosen took 1.005 of the faster one's time on average, 1.21 at most.  Some of them, us, 64 x 128 and 256 x 256:
// forward, d 120, f 3312, 2969 rows 41, 119; d 64, f 1088, 9594 rows 39, 69; d 448, f 1088, 9710 rows 65, 87; d 656, f 712, 13508 rows 88, 98;
// d 512, f 1408, 17557 rows 140, 116; d 960, f 2816, 15652 rows 491, 356; training, d 192, f 2088, 4300 rows 159, 365; d 136, f 344,
// 25852 rows 140, 211; d 768, f 1088, 9421 rows 330, 347; d 1088, f 1600, 14624 rows 914, 862; d 704, f 2944, 38200 rows 2735, 2048.
static bool few_faster(const FfnArgs& a, const int (&K)[2], const int (&NC)[2]) {
  auto ceil_div = [](long long x, long long y) { return (x + y - 1) / y; };
  long long few = 0, large = 0;
  for (int i = 0; i < 2; ++i) {
    const long long large_tiles = (a.A / BM + (a.V + 1) / 2) * ceil_div(NC[i], BN), tiles = (a.A / 64 + (a.E + 1) / 2) * ceil_div(NC[i], SN);
    large += 21000 + std::max(256ll, large_tiles) * (4000 + 880ll * ragged_k_tiles(K[i])) / 256;
    const long long stages = ceil_div(K[i], 64), seg = std::max(1ll, std::min<long long>(kSmallSplitTarget / std::max(tiles, 1ll), stages / 8));
    few += std::max<long long>(kSmallSplitTarget, tiles) * (2600 + 860 * ceil_div(stages, seg)) / kSmallSplitTarget + (seg > 1 ? 4000 : 0);
  }
  return few <= large;
}
// The layer as the shared host side sees it.  Where few_faster says so, the few-rows kernels' tables lie in the part of the workspace's second
// [A, 2 f] that the pass does not use: all of it in the forward pass, in the backward pass what is behind H.
static FfnArgs doubled(const FfnArgs& a, void* ws, bool fwd) {
  FfnArgs b = a;
  b.f = 2 * a.f;
  if (a.A == 0 || rows_kernels(b, ws).small.bm) return b;
  const size_t hpre = align_up((size_t)a.A * b.f * sizeof(bf16_t), 256), h = fwd ? 0 : align_up((size_t)a.A * a.f * sizeof(bf16_t), 256);
  const int K[2] = {a.d, fwd ? a.f : b.f}, NC[2] = {fwd ? b.f : a.f, a.d}, wide = std::max(b.f, b.d);
  // (32-bit byte offsets of the weights' and rows' loads as in ungated layers)
  if (few_tables_bytes(b) <= hpre - h && wide < 1 << 24 && (long long)a.A * wide < 1ll << 30 && few_faster(b, K, NC)) b.few_ws = (char*)ws + hpre + h;
  return b;
}

hipError_t launch_ffn_gated_fwd_bf16(const FfnArgs& a, const void* xp, const void* w1, const void* b1, const void* w2, const void* b2,
                                     void* hpre, void* h_keep, void* yp, void* ws, hipStream_t s) {
  if (a.A == 0) return hipSuccess;
  const FfnArgs a2 = doubled(a, ws, true);
  launch_rows_plan(a2, ws, s);
  void* h = h_keep ? h_keep : ws;
  const hipError_t err = launch_gated<EPI_FWD1>(a2, xp, w1, b1, nullptr, hpre, h, ws, s);
  if (err != hipSuccess) return err;
  return launch_gated_out(a2, h, w2, b2, yp, ws, s);
}

hipError_t launch_ffn_gated_bwd_bf16(const FfnArgs& a, const void* dyp, const void* xp, const void* hpre, const void* h_kept, const void* w1,
                                     const void* w2, void* dxp, void* dw1, void* dw2, void* ws, hipStream_t s) {
  const FfnArgs a2 = doubled(a, ws, false);
  bf16_t* dhpre = (bf16_t*)ws;
  bf16_t* h_ws = (bf16_t*)((char*)ws + align_up((size_t)a2.A * a2.f * sizeof(bf16_t), 256));
  launch_bwd_plan(a2, a.f, ws, s);
  if (a.A > 0) {
    const hipError_t err = h_kept ? launch_gated<EPI_DHQ>(a2, dyp, w2, nullptr, hpre, dhpre, nullptr, ws, s)
                                  : launch_gated<EPI_DH>(a2, dyp, w2, nullptr, hpre, dhpre, h_ws, ws, s);
    if (err != hipSuccess) return err;
  }
  const RowsKernels rk = rows_kernels(a2, ws);
  const bool dx_here = a.A > 0 && !rk.small.bm && a2.f % 128;      // (where it is, dX's kernel is the ungated layers')
  if (dx_here) {
    const GatedArgs p{dhpre, (const bf16_t*)w1, nullptr, a2.f, a.d, (a.d + BN - 1) / BN, nullptr, (bf16_t*)dxp, nullptr, 0};
    launch_persist<EPI_PLAIN_T>(a2, p, rk, s);
  }
  return launch_bwd_products(a2, a.f, h_kept ? h_kept : h_ws, dyp, dw2, xp, dhpre, dw1, w1, dx_here ? nullptr : dxp, nullptr, ws, s);
}

}  // namespace flexmoe

// For tests: which rows kernels a bf16 call of a gated layer takes, with row_tiles row tiles in use.  For the forward pass in out[0 .. 4], for the
// backward pass in out[5 .. 9]: row tiles of the few-rows kernels (0: the 256 x 256 ones); whether they are taken past the ungated layers' line;
// the halves of W1 in turn; contraction segments of the product with an activation; of the second product (backward: 0).
extern "C" void flexmoe_debug_gated_paths(int A, int d, int f, int E, int V, int row_tiles, long long* out) {
  using namespace flexmoe;
  const FfnArgs a{A, d, f, E, V, FLEXMOE_SILU, nullptr, nullptr};
  for (int b = 0; b < 2; ++b, out += 5) {
    const FfnArgs a2 = doubled(a, nullptr, b == 0);
    const RowsKernels rk = rows_kernels(a2, nullptr);
    bool turns;
    const SmallCore c = gated_core(a2, rk, b == 0, nullptr, nullptr, &turns);
    out[0] = rk.small.bm;
    out[1] = a2.few_ws != nullptr;
    out[2] = rk.small.bm && turns;
    out[3] = rk.small.bm ? core_segments(c, row_tiles, SK, turns ? 2 : 1) : 0;
    out[4] = rk.small.bm && b == 0 ? core_segments(gated_out_core(a2, rk, nullptr, nullptr), row_tiles, SK, 1) : 0;
  }
}
