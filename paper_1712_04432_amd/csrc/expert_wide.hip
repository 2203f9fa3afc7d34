// The large-tile products of an expert layer (bf16, whole 16-byte rows): which calls they take, and the launches. The
// kernel is in csrc/expert_wide_body.h.

#include <cmath>

#include "expert_wide_body.h"

namespace imbd {
namespace {

bool al16(const void *p, int64_t ld, int es) { return (uintptr_t)p % 16 == 0 && ld * es % 16 == 0; }

}  // namespace

bool expert_wide_fits(int pass, int dtype, const ExpertArgs &a) {
  const int es = a.out_dtype == IMBD_BF16 ? 2 : 4;
  const int64_t ld_most = (int64_t)1 << 22;  // 256 rows of a tile within one descriptor
  if (dtype != IMBD_BF16 || a.d_in % 8 || a.d_out % 8) return false;
  if (a.out && (!al16(a.out, a.ldo, es) || a.ldo >= ld_most || (pass == EXPERT_DW && a.so % 4))) return false;
  if (pass != EXPERT_DW && (!al16(a.w, a.ldw, 2) || a.sw % 8 || a.ldw >= ld_most)) return false;
  if (pass != EXPERT_FWD && (!al16(a.dy, a.lddy, 2) || a.lddy >= ld_most)) return false;
  if (pass != EXPERT_DX || a.mask) {
    if (!al16(a.x, a.ldx, 2) || a.ldx >= ld_most) return false;
    // gathered rows lie anywhere in x: all of it within one descriptor
    if (a.rows && pass != EXPERT_DX && (int64_t)a.n_x * a.ldx * 2 > (int64_t)XW_MOST) return false;
  }
  return a.n_rows < (1 << 29);  // byte offsets into rows
}

template <int PASS, int BM, int BN, int ES>
static int launch(const ExpertArgs &a, bool check, hipStream_t s) {
  const int M = PASS == EXPERT_FWD ? a.d_out : a.d_in;
  const int64_t tm = PASS == EXPERT_DW && !a.out ? 1 : (M + BM - 1) / BM;
  const int64_t tn = (a.d_out + BN - 1) / BN;
  const int64_t rows = row_tiles_most(a.n_rows, a.E, BN), blocks = (PASS == EXPERT_DW ? a.E * tn : rows) * tm;
  if (blocks > WORKGROUPS_MOST - 255) {
    set_error("expert product: %lld tiles are more than one launch takes", (long long)blocks);
    return IMBD_EUNSUPPORTED;
  }
  if (check) return IMBD_OK;
  const dim3 grid((unsigned)((blocks + 255) / 256 * 256));
  const int tiles_n = (int)(PASS == EXPERT_DW ? tn : rows);
  {
    LaunchTimer t(IMBD_K_EXPERT_FWD + PASS, 0, s);
    if (a.rows && PASS != EXPERT_DX)  // (Delta_X gathers nothing but its mask)
      hipLaunchKernelGGL((expert_wide_kernel<PASS, BM, BN, PASS != EXPERT_DX, ES>), grid, dim3(256), 0, s, a, (int)tm,
                         tiles_n);
    else
      hipLaunchKernelGGL((expert_wide_kernel<PASS, BM, BN, false, ES>), grid, dim3(256), 0, s, a, (int)tm, tiles_n);
  }
  return check_launch("expert_wide");
}

// Tiles of 256 or 128 rows: experts are rarely whole tiles long, and the tiles rarely whole rounds of the CUs, so
// with few rows an expert the smaller tile wastes less, though it feeds the matrix cores worse (LDS is read for a
// third more a product). Cycles of a tile: of a slab, and of its start and end (measured); an expert's last tile is
// taken as half full.
static int row_tile(const ExpertArgs &a, int tm, int K) {
  auto cost = [&](int rows, double slab, double ends) {
    const double tiles = ((double)a.n_rows / rows + 0.5 * (a.n_rows < a.E ? a.n_rows : a.E)) * tm;
    return std::ceil(tiles / 256.0) * ((K + XW_KS - 1) / XW_KS * slab + ends);
  };
  return cost(128, 1350, 11000) < cost(256, 2300, 16000) ? 128 : 256;
}

template <int PASS>
static int launch_rows(const ExpertArgs &a, bool check, hipStream_t s) {
  const int M = PASS == EXPERT_FWD ? a.d_out : a.d_in, K = PASS == EXPERT_FWD ? a.d_in : a.d_out;
  const bool half = a.out_dtype == IMBD_BF16;
  if (row_tile(a, (M + 255) / 256, K) == 128)
    return half ? launch<PASS, 256, 128, 2>(a, check, s) : launch<PASS, 256, 128, 4>(a, check, s);
  return half ? launch<PASS, 256, 256, 2>(a, check, s) : launch<PASS, 256, 256, 4>(a, check, s);
}

int run_expert_wide(int pass, const ExpertArgs &a, bool check, hipStream_t s) {
  if (pass == EXPERT_FWD) return launch_rows<EXPERT_FWD>(a, check, s);
  if (pass == EXPERT_DX) return launch_rows<EXPERT_DX>(a, check, s);
  return launch<EXPERT_DW, 256, 256, 4>(a, check, s);
}

}  // namespace imbd
