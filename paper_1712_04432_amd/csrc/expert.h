// Internal declarations of the expert layer's operators (csrc/expert_*.hip).
#pragma once

#include "cdna4.h"

namespace imbd {

constexpr int EXPERT_MAX = 512;  // experts
constexpr int CHOICE_MAX = 16;   // experts per token
// Workgroups of 256 threads a launch may have: its work-items are a 32-bit number.
constexpr int64_t WORKGROUPS_MOST = ((int64_t)1 << 24) - 1;

// One grouped product. fwd: out = W x (rows n x d_out); dx: out = W^T dy (rows n x d_in); dw: out_e =
// dy^T x per expert. Pointers and strides as in include/imbd.h.
struct ExpertArgs {
  int E, d_out, d_in, n_rows, n_x;
  const void *w;
  int64_t ldw, sw;
  const float *bias;  // fwd
  int relu;           // fwd
  const void *x;      // fwd, dw; dx: what the mask is taken from
  int64_t ldx;
  int mask;           // dx
  const void *dy;     // dx, dw
  int64_t lddy;
  const int32_t *rows;
  const int32_t *offsets;
  void *out;          // y / dx / dw
  int64_t ldo, so;    // so: dw's expert stride
  int out_dtype;
  float *db;          // dw: column sums of dy (or null)
};

enum ExpertPass { EXPERT_FWD = 0, EXPERT_DX = 1, EXPERT_DW = 2 };

// Slots of expert e, clamped: start and number.
__device__ __forceinline__ void expert_range(const ExpertArgs &a, int e, int *r0, int *cnt) {
  const int lo = min(max(a.offsets[e], 0), a.n_rows), hi = min(max(a.offsets[e + 1], 0), a.n_rows);
  *r0 = lo;
  *cnt = max(hi - lo, 0);
}

// Row tile number t of all experts' tiles (TR rows each, the last of an expert ragged), counted expert
// by expert: its expert, first row and the expert's end; false past the last tile. Every lane of a
// wave looks at an expert of its own and a scan over the lanes counts the tiles, so the host does not
// have to know the offsets: it launches the most tiles that n_rows rows can make (row_tiles_most).
template <int TR>
__device__ __forceinline__ bool find_row_tile(const ExpertArgs &a, int t, int *expert, int *row0, int *row_end) {
  const int lane = threadIdx.x & 63;
  int before = 0;
  for (int e0 = 0; e0 < a.E; e0 += 64) {
    const int e = e0 + lane;
    int r0 = 0, cnt = 0;
    if (e < a.E) expert_range(a, e, &r0, &cnt);
    const int tiles = cnt / TR + (cnt % TR != 0);
    int upto = tiles;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const int v = __shfl_up(upto, d, 64);
      if (lane >= d) upto += v;
    }
    const uint64_t past = __ballot(before + upto > t);
    if (past) {
      const int src = __builtin_ctzll(past);
      const int first = before + __shfl(upto - tiles, src, 64);
      const int base = __shfl(r0, src, 64), n = __shfl(cnt, src, 64);
      *expert = __builtin_amdgcn_readfirstlane(e0 + src);
      *row0 = __builtin_amdgcn_readfirstlane(base + (t - first) * TR);
      *row_end = __builtin_amdgcn_readfirstlane(base + n);
      return true;
    }
    before += __shfl(upto, 63, 64);
  }
  return false;
}

// The most row tiles of TR rows that n_rows rows make when split over E experts.
inline int64_t row_tiles_most(int n_rows, int E, int TR) {
  const int64_t used = n_rows < E ? n_rows : E;
  return ((int64_t)n_rows + used * (TR - 1)) / TR;
}

// The products' launches. check: only whether one launch takes the call (expert_bwd has two, and launches none of a call
// that it refuses).
// Any sizes, strides and alignments, fp32 and bf16 (csrc/expert_tile.hip).
int run_expert_tile(int pass, int dtype, const ExpertArgs &a, bool check, hipStream_t s);
// bf16, rows of whole 16-byte chunks (csrc/expert_wide.hip): whether it takes the call, and the launch.
bool expert_wide_fits(int pass, int dtype, const ExpertArgs &a);
int run_expert_wide(int pass, const ExpertArgs &a, bool check, hipStream_t s);
// The forward product of few rows an expert (csrc/expert_few.hip).
bool expert_few_fits(int pass, int dtype, const ExpertArgs &a);
int run_expert_few(const ExpertArgs &a, hipStream_t s);

size_t route_ws_bytes(int T, int E, int k);
int run_route(int T, int E, int k, int renorm, const float *logits, int64_t ldl, float *gates, int32_t *experts,
              int32_t *offsets, int32_t *rows, int32_t *slots, void *ws, hipStream_t s);
int run_route_bwd(int T, int E, int k, int renorm, const float *logits, int64_t ldl, const float *gates,
                  const int32_t *experts, const float *dgates, float *dlogits, int64_t lddl, hipStream_t s);
int run_combine(int dtype, int T, int k, int d, int n_rows, const void *ys, int64_t ldys, const int32_t *slots,
                const float *gates, void *y, int64_t ldy, int y_dtype, hipStream_t s);
int run_combine_bwd(int dtype, int T, int k, int d, int n_rows, const void *dy, int64_t lddy, const void *ys,
                    int64_t ldys, const int32_t *slots, const float *gates, void *dys, int64_t lddys, float *dgates,
                    hipStream_t s);

}  // namespace imbd
