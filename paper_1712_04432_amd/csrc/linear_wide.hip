// A fully connected layer's products on the large tiles (bf16, whole 16-byte rows; the kernel is in
// csrc/expert_wide_body.h): which calls they take, their tiles and ranges of K, and the launches.

#include <cmath>

#include "expert_wide_body.h"

namespace imbd {
namespace {

bool al16(const void *p, int64_t ld, int es) {
  const int64_t ld_most = (int64_t)1 << 22;  // 256 rows of a tile within one descriptor
  return (uintptr_t)p % 16 == 0 && ld * es % 16 == 0 && ld < ld_most;
}

template <int PASS, int BN, int ES, DenseEnd END>
int launch(const DenseArgs &a, bool check, hipStream_t s) {
  const int M = PASS == EXPERT_FWD ? a.d_out : a.d_in, N = PASS == EXPERT_DW ? a.d_out : a.n_rows;
  const int64_t tm = PASS == EXPERT_DW && !a.out ? 1 : (M + 255) / 256, tn = ((int64_t)N + BN - 1) / BN, blocks = a.E * tn * tm;
  if (blocks > WORKGROUPS_MOST - 255) {
    set_error("layer product: %lld tiles are more than one launch takes", (long long)blocks);
    return IMBD_EUNSUPPORTED;
  }
  if (check) return IMBD_OK;
  const dim3 grid((unsigned)((blocks + 255) / 256 * 256));
  {
    LaunchTimer t(IMBD_K_LINEAR, PASS, s);
    hipLaunchKernelGGL((expert_wide_kernel<PASS, 256, BN, false, ES, DenseArgs, END>), grid, dim3(256), 0, s, a, (int)tm, (int)tn);
  }
  return check_launch("linear_wide");
}

template <int PASS, int BN>
int launch_rows(const DenseArgs &a, bool check, hipStream_t s) {
  if (a.E > 1) return launch<PASS, BN, 4, DENSE_SUMS>(a, check, s);
  return a.out_dtype == IMBD_BF16 ? launch<PASS, BN, 2, DENSE_CHUNKS>(a, check, s) : launch<PASS, BN, 4, DENSE_CHUNKS>(a, check, s);
}

}  // namespace

bool dense_wide_fits(int pass, int dtype, const DenseArgs &a) {
  const int es = a.out_dtype == IMBD_BF16 ? 2 : 4;
  if (dtype != IMBD_BF16 || a.d_in % 8 || a.d_out % 8 || a.n_rows >= (1 << 29)) return false;
  if (a.out && !al16(a.out, a.ldo, es)) return false;
  if (pass != EXPERT_DW && !al16(a.w, a.ldw, 2)) return false;
  if (pass != EXPERT_FWD && !al16(a.dy, a.lddy, 2)) return false;
  if (pass != EXPERT_DX && (pass == EXPERT_FWD || a.out) && !al16(a.x, a.ldx, 2)) return false;
  return (!a.z || al16(a.z, a.ldz, 2)) && (!a.res || al16(a.res, a.ldr, es));
}

DensePlan dense_wide_plan(int pass, int64_t M, int64_t N, int64_t K) {
  // Cycles of a slab of 64 k, of a tile's start and end, and of what a cut of K costs besides: its partial sums written
  // and read (bytes a cycle of all the GPU) and a launch.
  const int64_t tm = (M + 255) / 256, slabs = (K + 63) / 64;
  DensePlan best{256, 1, (int)(slabs * 64), 0};
  double least = 0;
  for (int bn = 128; bn <= 256; bn += 128) {
    if (pass == EXPERT_DW && bn == 128) continue;
    const int64_t tiles = tm * ((N + bn - 1) / bn);
    // (past two rounds of workgroups more ranges only add sums)
    for (int64_t n = 1; n <= 64 && (n == 1 || (n * 4 <= slabs && tiles * (n - 1) < 512)); ++n) {
      const int64_t per = (slabs + n - 1) / n;
      if (n > 1 && (slabs + per - 1) / per != n) continue;
      const double rounds = std::ceil((double)(tiles * n) / 256.0);
      double c = rounds * (per * (bn == 128 ? 1350.0 : 2300.0) + (bn == 128 ? 11000.0 : 16000.0));
      if (n > 1) c += 9000.0 + (double)n * M * N * 8 / 2000.0;
      if (best.cost == 0 || c < least) {
        least = c;
        best = DensePlan{bn, (int)n, (int)(per * 64), c};
      }
    }
  }
  return best;
}

int run_dense_wide(int pass, const DenseArgs &a, int bn, bool check, hipStream_t s) {
  if (pass == EXPERT_FWD) return bn == 128 ? launch_rows<EXPERT_FWD, 128>(a, check, s) : launch_rows<EXPERT_FWD, 256>(a, check, s);
  if (pass == EXPERT_DX) return bn == 128 ? launch_rows<EXPERT_DX, 128>(a, check, s) : launch_rows<EXPERT_DX, 256>(a, check, s);
  return launch<EXPERT_DW, 256, 4, DENSE_SUMS>(a, check, s);
}

int run_dense_wide_any(int pass, const DenseArgs &a, int bn, bool check, hipStream_t s) {
  if (pass == EXPERT_FWD)
    return bn == 128 ? launch<EXPERT_FWD, 128, 4, DENSE_ANY>(a, check, s) : launch<EXPERT_FWD, 256, 4, DENSE_ANY>(a, check, s);
  return bn == 128 ? launch<EXPERT_DX, 128, 4, DENSE_ANY>(a, check, s) : launch<EXPERT_DX, 256, 4, DENSE_ANY>(a, check, s);
}

}  // namespace imbd
