// The forward product of an expert layer for few rows an expert (bf16 operands, fp32 accumulation), as decoding
// makes it: y[s][o] = sum_i W_e[o][i] x[rows[s]][i] (+ b_e[o], ReLU).
//
// Up to 16 rows, every weight is used for 2 x 16 flops at most: the time is that of reading the chosen experts'
// weights once. So nothing is staged: a wave loads its rows of W straight into the registers that the matrix
// instruction reads (16 rows x 32 k a load, whole 128-byte lines in two), and the 16 rows of x, which stay in
// the caches, the same way. A workgroup owns 16 or 32 outputs of one expert's 16 rows; its four waves take a quarter of K
// each and add their sums through LDS in wave order. Many small workgroups keep enough loads in flight; 16 outputs
// a workgroup where 32 would leave CUs without one. 16 experts of 4096 x 4096, one row each: weights at 5.4 TB/s.

#include "expert.h"

namespace imbd {
namespace {

constexpr int FW_ROWS = 16;                // rows of x a workgroup
constexpr int FW_KS = 64;                  // k of a step: one line of each row
constexpr uint32_t FW_OOB = 0xffff0000u;   // past every descriptor
constexpr int FW_UNROLL = 4;               // steps whose loads are in flight together

// OT: 16-wide blocks of outputs a workgroup.
template <int OT>
__global__ void __launch_bounds__(256) expert_few_kernel(ExpertArgs a, int tiles_o) {
  constexpr int OW = 16 * OT;
  __shared__ float part[4][FW_ROWS][OW + 1];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int t = (int)blockIdx.x / tiles_o, o0 = ((int)blockIdx.x - t * tiles_o) * OW;
  int e, n0, n_end;
  if (!find_row_tile<FW_ROWS>(a, t, &e, &n0, &n_end)) return;
  const int fi = lane & 15, kg = lane >> 4;
  const uint16_t *w = reinterpret_cast<const uint16_t *>(a.w) + (int64_t)e * a.sw + (int64_t)o0 * a.ldw;
  const int K = a.d_in, nsl = (K + FW_KS - 1) / FW_KS;
  const __amdgpu_buffer_rsrc_t rw = __builtin_amdgcn_make_buffer_rsrc(
      const_cast<uint16_t *>(w), 0, (int)(((int64_t)(min(OW, a.d_out - o0) - 1) * a.ldw + K) * 2), BUF_DW3);
  // this lane's row of x: 64-bit, any row of it
  const int s = n0 + fi;
  int row = s < n_end ? (a.rows ? a.rows[s] : s) : -1;
  const bool real = row >= 0 && row < a.n_x;
  const uint16_t *x = reinterpret_cast<const uint16_t *>(a.x) + (int64_t)(real ? row : 0) * a.ldx;
  uint32_t ow[OT];
#pragma unroll
  for (int i = 0; i < OT; ++i)
    ow[i] = o0 + 16 * i + fi < a.d_out ? (uint32_t)((int64_t)(16 * i + fi) * a.ldw * 2) : FW_OOB;

  f32x4 acc[OT];
#pragma unroll
  for (int i = 0; i < OT; ++i) acc[i] = f32x4{0.f, 0.f, 0.f, 0.f};
  const int per = (nsl + 3) / 4, s0 = wave * per, s1 = min(nsl, s0 + per);
  for (int S = s0; S < s1; S += FW_UNROLL) {
    u32x4 wv[FW_UNROLL][2][OT], xv[FW_UNROLL][2];
#pragma unroll
    for (int u = 0; u < FW_UNROLL; ++u)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int k = (S + u) * FW_KS + 32 * h + 8 * kg;
        const bool in = S + u < s1 && k < K;
#pragma unroll
        for (int i = 0; i < OT; ++i)
          wv[u][h][i] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(
                                                      rw, in && ow[i] != FW_OOB ? ow[i] + (uint32_t)(2 * k) : FW_OOB, 0, 2));
        xv[u][h] = u32x4{0u, 0u, 0u, 0u};
        if (in && real) xv[u][h] = *reinterpret_cast<const u32x4 *>(x + k);
      }
#pragma unroll
    for (int u = 0; u < FW_UNROLL; ++u)
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int i = 0; i < OT; ++i)
          acc[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, wv[u][h][i]),
                                                           __builtin_bit_cast(bf16x8, xv[u][h]), acc[i], 0, 0, 0);
  }
#pragma unroll
  for (int i = 0; i < OT; ++i)
#pragma unroll
    for (int q = 0; q < 4; ++q) part[wave][fi][16 * i + 4 * kg + q] = acc[i][q];
  __syncthreads();
#pragma unroll
  for (int c = tid; c < FW_ROWS * OW; c += 256) {
    const int r = c / OW, o = c - r * OW;
    if (n0 + r >= n_end || o0 + o >= a.d_out) continue;
    float v = part[0][r][o] + part[1][r][o];
    v += part[2][r][o];
    v += part[3][r][o];
    if (a.bias) v += a.bias[(int64_t)e * a.d_out + o0 + o];
    if (a.relu) v = v < 0.f ? 0.f : v;  // (a NaN stays one)
    const int64_t at = (int64_t)(n0 + r) * a.ldo + o0 + o;
    if (a.out_dtype == IMBD_BF16) reinterpret_cast<uint16_t *>(a.out)[at] = f32_to_bf16(v);
    else reinterpret_cast<float *>(a.out)[at] = v;
  }
}

}  // namespace

bool expert_few_fits(int pass, int dtype, const ExpertArgs &a) {
  // 16 rows an expert on average: past them a second row tile reads W again, and the large tiles' idle rows cost less. 16
  // experts of 4096 x 4096, weights from memory: 16 rows each 131 us here and 175 there, 17 each 224 and 174; 8 experts
  // 68 and 78, 117 and 75. (The offsets are not known here, and the mean is not all: 256 rows that are all of one expert
  // of the 16 take 114 us here and 44 there; of one or two experts 64 rows each would take 31 and 59 us here, 63 and 67
  // there.)
  return pass == EXPERT_FWD && a.n_rows <= (int64_t)FW_ROWS * a.E && expert_wide_fits(pass, dtype, a);
}

int run_expert_few(const ExpertArgs &a, hipStream_t s) {
  const int64_t rows = row_tiles_most(a.n_rows, a.E, FW_ROWS);
  const int64_t t32 = (a.d_out + 31) / 32, t16 = (a.d_out + 15) / 16;
  const bool wide = rows * t32 >= 512;
  const int64_t blocks = rows * (wide ? t32 : t16);
  if (blocks > WORKGROUPS_MOST) {
    set_error("expert product: %lld tiles are more than one launch takes", (long long)blocks);
    return IMBD_EUNSUPPORTED;
  }
  {
    LaunchTimer t(IMBD_K_EXPERT_FWD, 0, s);
    if (wide) hipLaunchKernelGGL(expert_few_kernel<2>, dim3((unsigned)blocks), dim3(256), 0, s, a, (int)t32);
    else hipLaunchKernelGGL(expert_few_kernel<1>, dim3((unsigned)blocks), dim3(256), 0, s, a, (int)t16);
  }
  return check_launch("expert_few");
}

}  // namespace imbd
