// The forward product of a fully connected layer for few rows (bf16 or fp32, fp32 accumulation), as a serving step makes it:
//   z[n][m] = sum_k W[m][k] x[n][k] + b[m],  y = act(z) + r
//
// The time is that of reading W once: nothing is staged. A wave loads its rows of W straight into the registers that the matrix
// instruction reads (16 rows x 64 k in two loads, whole 128-byte lines), and the rows of x, which stay in the caches, the
// same way. A workgroup owns 16 OT outputs of all rows; its four waves take a quarter of K each and add their sums through LDS in
// wave order, so the epilogue is in the same launch.
//
// A CU takes in some 25 bytes a ns this way, x included, which every workgroup reads again (NB / OT times what W takes): from
// 8192 outputs on, where that leaves two workgroups a CU, one takes 32 of them. Weights from memory, 1 / 16 rows: 4096 x 4096
// 9.8 / 11.3 us, 1024 x 1024 3.8 / 4.5, 16384 x 4096 32.0 / 31.9 (in 16 outputs a workgroup 31.2 / 39.2). Eight waves a workgroup (37.0
// and 51.2 us for 4096 x 16384 instead of 33.1 and 39.9), other depths of loads and loads past the caches were no faster.
// fp32 takes the same bytes a row in half the k: 8 rows of 4096 x 2048 13.3 us (the any-size kernel in two launches 18.4).

#include "dense.h"

namespace imbd {
namespace {

constexpr int LR_NW = 4;                   // waves of a workgroup
constexpr int LR_KB = 128;                 // bytes of a step's k: one line of each row
constexpr uint32_t LR_OOB = 0xffff0000u;   // past every descriptor

// OT, NB: 16-wide blocks of outputs and of rows a workgroup. UN: steps whose loads are in flight together.
template <typename T, int OT, int NB, int UN>
__global__ void __launch_bounds__(LR_NW * 64) linear_rows_kernel(DenseArgs a) {
  constexpr int OW = 16 * OT, RW = 16 * NB, PITCH = OW + 4, ES = (int)sizeof(T), LR_KS = LR_KB / ES;
  __shared__ __attribute__((aligned(16))) float part[LR_NW][RW][PITCH];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int fi = lane & 15, kg = lane >> 4;
  const int m0 = (int)blockIdx.x * OW, K = a.d_in, N = a.n_rows, nsl = (K + LR_KS - 1) / LR_KS;
  const T *w = reinterpret_cast<const T *>(a.w) + (int64_t)m0 * a.ldw;
  const T *x = reinterpret_cast<const T *>(a.x);
  const __amdgpu_buffer_rsrc_t rw = __builtin_amdgcn_make_buffer_rsrc(
      const_cast<T *>(w), 0, (int)(uint32_t)(((int64_t)(min(OW, a.d_out - m0) - 1) * a.ldw + K) * ES), BUF_DW3);
  const __amdgpu_buffer_rsrc_t rx =
      __builtin_amdgcn_make_buffer_rsrc(const_cast<T *>(x), 0, (int)(uint32_t)(((int64_t)(N - 1) * a.ldx + K) * ES), BUF_DW3);
  uint32_t ow[OT], ox[NB];
#pragma unroll
  for (int i = 0; i < OT; ++i) ow[i] = m0 + 16 * i + fi < a.d_out ? (uint32_t)((int64_t)(16 * i + fi) * a.ldw * ES) + 16 * kg : LR_OOB;
#pragma unroll
  for (int j = 0; j < NB; ++j) ox[j] = 16 * j + fi < N ? (uint32_t)((int64_t)(16 * j + fi) * a.ldx * ES) + 16 * kg : LR_OOB;
  f32x4 acc[OT][NB];
#pragma unroll
  for (int i = 0; i < OT; ++i)
#pragma unroll
    for (int j = 0; j < NB; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  const int per = (nsl + LR_NW - 1) / LR_NW, s0 = wave * per, s1 = min(nsl, s0 + per);
  // CUT: steps that reach past the range's end
  auto steps = [&](int S, auto cut_tag) {
    constexpr bool CUT = decltype(cut_tag)::value;
    u32x4 wv[UN][2][OT], xv[UN][2][NB];
#pragma unroll
    for (int u = 0; u < UN; ++u)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const bool in = !CUT || (S + u < s1 && (S + u) * LR_KS + (64 * h + 16 * kg) / ES < K);
        const uint32_t k2 = (uint32_t)(S + u) * LR_KB + 64 * h;
#pragma unroll
        for (int i = 0; i < OT; ++i)
          wv[u][h][i] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rw, in ? ow[i] : LR_OOB, in ? k2 : 0, 0));
#pragma unroll
        for (int j = 0; j < NB; ++j)
          xv[u][h][j] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rx, in ? ox[j] : LR_OOB, in ? k2 : 0, 0));
      }
#pragma unroll
    for (int u = 0; u < UN; ++u)
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int i = 0; i < OT; ++i)
#pragma unroll
          for (int j = 0; j < NB; ++j) {
            if constexpr (ES == 2) {
              acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, wv[u][h][i]),
                                                                  __builtin_bit_cast(bf16x8, xv[u][h][j]), acc[i][j], 0, 0, 0);
            } else {  // (the four lanes of a row each hold four k in a row: an instruction takes the q-th of each)
              const f32x4 wf = __builtin_bit_cast(f32x4, wv[u][h][i]), xf = __builtin_bit_cast(f32x4, xv[u][h][j]);
#pragma unroll
              for (int q = 0; q < 4; ++q) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(wf[q], xf[q], acc[i][j], 0, 0, 0);
            }
          }
  };
  int S = s0;
  for (; S + UN <= s1 && (S + UN) * LR_KS <= K; S += UN) steps(S, std::integral_constant<bool, false>{});
  for (; S < s1; S += UN) steps(S, std::integral_constant<bool, true>{});
#pragma unroll
  for (int i = 0; i < OT; ++i)
#pragma unroll
    for (int j = 0; j < NB; ++j) *reinterpret_cast<f32x4 *>(&part[wave][16 * j + fi][16 * i + 4 * kg]) = acc[i][j];
  __syncthreads();
  // four outputs of a row a thread
  for (int c = tid; c < RW * OT * 4; c += LR_NW * 64) {
    const int n = c / (OT * 4), mo = 4 * (c - n * (OT * 4)), m = m0 + mo, cnt = min(4, a.d_out - m);
    if (n >= N || cnt <= 0) continue;
    f32x4 s = *reinterpret_cast<const f32x4 *>(&part[0][n][mo]);
#pragma unroll
    for (int q = 1; q < LR_NW; ++q) s += *reinterpret_cast<const f32x4 *>(&part[q][n][mo]);
    float v[4] = {s[0], s[1], s[2], s[3]};
    if (a.bias) {
      float bias[4];
      load_run(a.bias + m, cnt, bias);
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] += bias[i];
    }
    dense_finish<T, EXPERT_FWD>(a, n, m, cnt, v);
  }
}

template <typename T, int OT, int NB, int UN>
int launch(const DenseArgs &a, hipStream_t s) {
  const int tm = (a.d_out + 16 * OT - 1) / (16 * OT);
  if (tm > WORKGROUPS_MOST) {
    set_error("layer product: %d tiles are more than one launch takes", tm);
    return IMBD_EUNSUPPORTED;
  }
  {
    LaunchTimer t(IMBD_K_LINEAR, EXPERT_FWD, s);
    hipLaunchKernelGGL((linear_rows_kernel<T, OT, NB, UN>), dim3((unsigned)tm), dim3(LR_NW * 64), 0, s, a);
  }
  return check_launch("linear_rows");
}

template <typename T>
int launch_sized(const DenseArgs &a, hipStream_t s) {
  if (a.n_rows > 16) return a.d_out >= 8192 ? launch<T, 2, 2, 2>(a, s) : launch<T, 1, 2, 2>(a, s);
  return a.d_out >= 8192 ? launch<T, 2, 1, 4>(a, s) : launch<T, 1, 1, 4>(a, s);
}

}  // namespace

bool linear_rows_f32_fits(const DenseArgs &a) {
  auto fits = [](const void *p, int64_t ld) { return (uintptr_t)p % 16 == 0 && ld % 4 == 0 && ld < (1 << 22); };
  return a.d_in % 4 == 0 && fits(a.w, a.ldw) && fits(a.x, a.ldx);
}

int run_linear_rows(int dtype, const DenseArgs &a, hipStream_t s) {
  return dtype == IMBD_BF16 ? launch_sized<uint16_t>(a, s) : launch_sized<float>(a, s);
}

}  // namespace imbd
