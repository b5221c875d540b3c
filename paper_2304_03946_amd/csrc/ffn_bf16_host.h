// Host-side parts of ffn_bf16.hip that the gated experts' passes (ffn_gated.hip) go through as well.
#pragma once
#include "common.h"
#include "ffn_bf16_small.h"

namespace flexmoe {

// Which rows kernels a layer of these sizes takes (small.bm: row tiles of 32 or 64 rows, 0: 256 x 256 tiles) and what they look up in
// its workspace.  A gated layer is planned as one with a.f = 2 f columns in the middle: its wider product has as many.
struct RowsKernels {
  SmallPlan small;
  float* small_partial;
  int small_slots;               // of BM x 128 sums
  i32x4* row_tab;
};
RowsKernels rows_kernels(const FfnArgs& a, void* ws);
size_t few_tables_bytes(const FfnArgs& a);      // what FfnArgs::few_ws has to hold
void launch_rows_plan(const FfnArgs& a, void* ws, hipStream_t s);
// fh: columns of H (a.f / 2 in gated layers)
void launch_bwd_plan(const FfnArgs& a, int fh, void* ws, hipStream_t s);
// out [A, d] = in [A, K] . w [E, K, d] + bias
hipError_t launch_rows_plain(const FfnArgs& a, const void* in, const void* w, const void* bias, int K, void* out, void* ws, hipStream_t s);
// dxp null: there already
hipError_t launch_bwd_products(const FfnArgs& a, int fh, const void* h, const void* dyp, void* dw2, const void* xp, const void* dhpre,
                               void* dw1, const void* w1, void* dxp, const int32_t* scatter_src, void* ws, hipStream_t s);

}  // namespace flexmoe
