// The large-tile products of an expert layer (bf16 operands, fp32 accumulation), for whole 16-byte rows:
//   forward  y[s][o]    = sum_i W_e[o][i] x[rows[s]][i]   (+ b_e[o], ReLU)
//   Delta_X  dx[s][i]   = sum_o W_e[o][i] dy[s][o]        (* [x > 0])
//   Delta_W  dw_e[o][i] = sum_s dy[s][o] x[rows[s]][i];   db_e[o] = sum_s dy[s][o]
// as D(m, n) = sum_k A(m, k) B(k, n), m the output's contiguous index (o, i, i) and n its row (s, s, o). With DenseArgs
// one layer's products without experts (csrc/linear_wide.hip): "experts" are then ranges of K.
//
// These products are bound by the matrix cores, and the tile is chosen for what feeds them: with 128 x 128
// outputs a wave, a k-step of 32 costs 16 KB of LDS reads and 64 matrix instructions (1024 cycles), so the
// four waves of a 256 x 256 tile read LDS half the time. One wave a SIMD: nothing but its own instruction order
// hides its waits, so
//  * slabs of 64 k travel straight from memory to LDS, into two slots by turns. An operand by k-rows is loaded in
//    halves of 32 k, each as soon as its place is free, three k-steps ahead; one with k contiguous as a whole, so
//    that its rows are whole 128-byte lines (in halves the forward product took 10% longer; k-rows as a whole, the
//    weight gradient took 13% longer);
//  * the fragments of a k-step are read between the products of the one before, into a second register set;
//  * one barrier a k-step (a slab, where both operands have k contiguous: one of them then has three slots, so that
//    their loads take turns; all in one k-step, the loads themselves waited for their place), at which the wave's next
//    products already have their operands in registers.
// Measured, 16384 tokens, k = 2, 8 experts of 4096 x 4096: forward 786 to 849 us, Delta_X and Delta_W together 1635 to
// 1728 (1.3 to 1.4 PFLOP/s; a library product of 8192 x 4096 x 4096 reaches 1.56). The matrix cores are busy 68 to 72%
// of the cycles; the rest is the last, partial round of tiles and the start and end of each.
//
// Slabs in LDS. An operand with k contiguous: rows of 128 bytes, the 16-byte chunks XORed with row%8. By k-rows:
// quarters of 64 columns, 64 k-rows of 128 bytes, read with the LDS transpose read; its swizzle is that of the
// weight-gradient kernel. Both without bank conflicts.
//
// Ragged edges. Rows of an expert's last tile, output columns past the width and k past the end read as
// zero: by lane (an offset past the buffer descriptor) or because the descriptor ends there. An expert's
// neighbours never enter a sum, not even times zero: their rows may hold infinities.

#pragma once

#include <type_traits>
#include <utility>

#include "dense.h"

namespace imbd {
namespace {

constexpr int XW_KS = 64;                     // k per slab
constexpr int XW_GM = 8;                      // m tiles per launch-order group
constexpr uint32_t XW_OOB = 0xffff0000u;      // past every buffer descriptor
constexpr uint32_t XW_MOST = 0xfffe0000u;     // bytes that a descriptor covers at most

__device__ __forceinline__ int xw_swz_tr(int r) { return 2 * ((r >> 1) & 1) + 4 * ((r >> 3) & 1); }

// f(0), f(1), .. f(N-1) with the number as a compile-time constant.
template <typename F, int... q>
__device__ __forceinline__ void static_for_seq(F &f, std::integer_sequence<int, q...>) {
  (f(std::integral_constant<int, q>{}), ...);
}
template <int N, typename F>
__device__ __forceinline__ void static_for(F f) {
  static_for_seq(f, std::make_integer_sequence<int, N>{});
}

// One wave writes 64 x 16 bytes to LDS at lds_base + 16*lane, from byte offsets voff + IMM of the buffer. (The
// instruction's own offset counts on both sides, so it is taken off the LDS base.)
template <int IMM>
__device__ __forceinline__ void dma16_at(const i32x4 &rsrc, uint32_t voff, uint32_t lds_base) {
  asm volatile("s_nop 0\n\tbuffer_load_dwordx4 %0, %1, 0 offen offset:%3 lds"
               :
               : "v"(voff), "s"(rsrc), "{m0}"(lds_base - IMM), "n"(IMM)
               : "memory");
}

// acc += A B on accumulation registers. A wave's 256 accumulators fill that half of the register file
// exactly, and only named as such do they stay there: left to itself the compiler moved them through the
// other half (500 moves in a k-step pair, and spills).
__device__ __forceinline__ void mfma(f32x4 &acc, const bf16x8 &a, const bf16x8 &b) {
  asm volatile("v_mfma_f32_16x16x32_bf16 %0, %1, %2, %0" : "+a"(acc) : "v"(a), "v"(b));
}
// The same on plain registers; the operand `a` may be a constant that the compiler writes just before (wait
// states between a vector write and a matrix instruction's read are not its business in inline assembly; the
// fragments of the other form come from LDS and are waited for).
__device__ __forceinline__ void mfma_v(f32x4 &acc, const bf16x8 &a, const bf16x8 &b) {
  asm volatile("s_nop 3\n\tv_mfma_f32_16x16x32_bf16 %0, %1, %2, %0" : "+v"(acc) : "v"(a), "v"(b));
}
// Wait states between the last product and the first read of its result (the compiler does not see them).
__device__ __forceinline__ void mfma_drain() { asm volatile("s_nop 15\n\ts_nop 15" : : : "memory"); }

// Which of nl loads, spread over the first `span` products, goes with product p: load q with product q*span/nl,
// rounded down to an even one. nl: none.
constexpr int xw_load_at(int p, int nl, int span) {
  for (int q = 0; q < nl; ++q)
    if (q * span / nl / 2 * 2 == p) return q;
  return nl;
}

// A product and, in the wait state that a write of m0 asks for, behind it a load to LDS (as dma16_at).
template <int IMM>
__device__ __forceinline__ void mfma_dma16(f32x4 &acc, const bf16x8 &a, const bf16x8 &b, const i32x4 &rsrc, uint32_t voff,
                                           uint32_t lds_base) {
  asm volatile("v_mfma_f32_16x16x32_bf16 %0, %1, %2, %0\n\tbuffer_load_dwordx4 %3, %4, 0 offen offset:%6 lds"
               : "+a"(acc)
               : "v"(a), "v"(b), "v"(voff), "s"(rsrc), "{m0}"(lds_base - IMM), "n"(IMM)
               : "memory");
}
// Waits for this wave's LDS reads and, BARRIER, for all but VM of its loads and for every wave. (The builtins, so
// that the compiler knows that the reads have landed and adds no waits of its own.)
template <bool BARRIER, int VM = 0>
__device__ __forceinline__ void step_wait() {
  static_assert(VM < 64, "");
  asm volatile("" : : : "memory");
  if constexpr (BARRIER) {
    __builtin_amdgcn_s_waitcnt((VM & 15) | ((VM >> 4) << 14) | 0x70);
    __builtin_amdgcn_s_barrier();
  } else {
    __builtin_amdgcn_s_waitcnt(0xc07f);
  }
  asm volatile("" : : : "memory");
}

// A buffer descriptor that moves `step` bytes a slab: `most` bytes on every slab, `last` on the one that holds the
// end of k, none past it.
struct Window {
  i32x4 r;
  int64_t step;
  uint32_t last;
  __device__ __forceinline__ Window(const void *p, int64_t step_, uint32_t most, uint32_t last_)
      : r(buf_rsrc(p, most)), step(step_), last(last_) {}
  __device__ __forceinline__ void advance() {  // (addresses have 48 bits: no carry reaches the stride field)
    const uint64_t b = (((uint64_t)(uint32_t)r[1] << 32) | (uint32_t)r[0]) + (uint64_t)step;
    r[0] = (int)(uint32_t)b;
    r[1] = (int)(uint32_t)(b >> 32);
  }
};

template <int PASS, int BM, int BN>
struct Shape {
  static constexpr bool A_KC = PASS == EXPERT_FWD, B_KC = PASS != EXPERT_DW;
  static constexpr int FM = BM / 32, FN = BN / 32;  // 16-wide blocks of a wave (2 x 2 waves)
  // B in three slots where both operands have k contiguous: its loads then go with the k-steps that A's do not take
  static constexpr bool TRI = A_KC && B_KC;
  static constexpr int SA = BM * 128, SB = BN * 128;  // a slot of each
  static constexpr int RING = 2 * SA + (TRI ? 3 : 2) * SB;
  static constexpr int PA = BM / 32, PB = BN / 32;  // loads a wave, a slab
  // ... in k-step h: half of a k-row operand's in each, a k-contiguous operand's in the second (TRI: B's in the first)
  static constexpr int HB = TRI ? 0 : 1;
  static constexpr int la(int h) { return A_KC ? (h ? PA : 0) : PA / 2; }
  static constexpr int lb(int h) { return B_KC ? (h == HB ? PB : 0) : PB / 2; }
  static constexpr int loads(int h) { return la(h) + lb(h); }
};

// Delta_X on 128-row tiles has room for the tile's mask beside its slots: it is loaded first of all and waits there (64
// experts of 2048 x 1024: its loads in the epilogue took 23 of 132 us).
constexpr bool xw_mask_in_lds(int PASS, int BN) { return PASS == EXPERT_DX && BN == 128; }

// A wave's part of LDS in the epilogue: its outputs as bf16, half of them as fp32.
constexpr int xw_stage_bytes(int BM, int BN) { return BM / 2 * (BN / 2) * 2; }

template <int PASS, int BM, int BN, bool GATHER>
constexpr int xw_lds_bytes() {
  // the slots; Delta_W with gathered x: the row indices of eight half slabs, 256 bytes a wave each
  constexpr int ring = Shape<PASS, BM, BN>::RING + (PASS == EXPERT_DW && GATHER ? 8 * 1024 : 0);
  constexpr int stage = 4 * xw_stage_bytes(BM, BN);
  return (ring > stage ? ring : stage) + (xw_mask_in_lds(PASS, BN) ? BM * BN * 2 : 0);
}

// What a launch of DenseArgs does with its sums: stores them (a range's, or Delta_W), finishes them in whole chunks, or at any
// width (DenseArgs::width) and alignment.
enum DenseEnd { DENSE_SUMS, DENSE_CHUNKS, DENSE_ANY };

// Half of a wave's sums at a time to its part of LDS in fp32, 16-byte chunks XORed with the row.
template <int FM, int FP, int FN>
__device__ __forceinline__ void stage_sums(f32x4 (&acc)[FM][FN], int part, uint32_t stg) {
  constexpr int PITCH = FM * 16 * 4;
  const int lane = threadIdx.x & 63, fi = lane & 15, kg = lane >> 4;
#pragma unroll
  for (int i = 0; i < FM; ++i) {
    const uint32_t p = stg + (uint32_t)(fi * PITCH + (((4 * i + kg) ^ fi) * 16));
#pragma unroll
    for (int j = 0; j < FP; ++j) {
      f32x4 v = acc[i][part * FP + j];
      asm volatile("" : "+a"(v));  // (read here, behind the wait states)
      *(__attribute__((address_space(3))) f32x4 *)(uintptr_t)(p + j * 16 * PITCH) = v;
    }
    __builtin_amdgcn_sched_barrier(0);
  }
}
// Eight columns of row r of what it staged.
template <int FM>
__device__ __forceinline__ void staged_run(uint32_t stg, int r, int ch, float (&v)[8]) {
  const uint32_t p = stg + (uint32_t)(r * FM * 16 * 4);
  const f32x4 lo = *(const __attribute__((address_space(3))) f32x4 *)(uintptr_t)(p + (uint32_t)(((2 * ch) ^ (r & 15)) * 16));
  const f32x4 hi = *(const __attribute__((address_space(3))) f32x4 *)(uintptr_t)(p + (uint32_t)(((2 * ch + 1) ^ (r & 15)) * 16));
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = lo[i], v[4 + i] = hi[i];
}

// Any width and alignment: eight outputs of a row a lane, as they are (dense_finish).
template <int PASS, int FM, int FN>
__device__ __forceinline__ void dense_any_epilogue(const DenseArgs &a, f32x4 (&acc)[FM][FN], uint32_t stg, int mw, int nw, int rows_left) {
  constexpr int LPR = FM * 2, RPI = 64 / LPR, FP = FN / 2;  // lanes a row, rows at once
  const int lane = threadIdx.x & 63, row0 = lane / LPR, ch = lane % LPR, m = mw + 8 * ch, cnt = min(8, a.width - m);
  float bias[8] = {};
  if (PASS == EXPERT_FWD && a.bias && cnt > 0) load_run(a.bias + m, cnt, bias);
#pragma unroll
  for (int part = 0; part < 2; ++part) {
    stage_sums<FM, FP>(acc, part, stg);
#pragma unroll 2
    for (int b = 0; b < FP * 16 / RPI; ++b) {
      const int r = b * RPI + row0, n = part * FP * 16 + r;
      float v[8];
      staged_run<FM>(stg, r, ch, v);
      if (n >= rows_left || cnt <= 0) continue;
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] += bias[i];
      dense_finish<uint16_t, PASS>(a, nw + n, m, cnt, v);
    }
  }
}

// Finishes a wave's 16 FM x 16 FN sums (dense_finish, in csrc/dense.h, on whole chunks): half its rows at a time go through
// its part of LDS in fp32 (stg), eight columns of a row a lane come back. What the epilogue reads (the residual, the
// activation's z) is loaded four rows' worth ahead: a wave has its SIMD for itself, nothing else hides its waits.
template <int PASS, int ES, int FM, int FN>
__device__ __forceinline__ void dense_wide_epilogue(const DenseArgs &a, f32x4 (&acc)[FM][FN], uint32_t stg, int mw, int nw,
                                                    int rows_left, int M) {
  constexpr int WM = FM * 16, LPR = WM / 8, RPI = 64 / LPR, FP = FN / 2;  // lanes a row, rows at once
  constexpr int NIT = FP * 16 / RPI, UN = 4;                                            // ... a half's rounds, of them together
  static_assert(NIT % UN == 0, "");
  const int lane = threadIdx.x & 63, row0 = lane / LPR, ch = lane % LPR;
  const bool in = mw + 8 * ch < M;  // (widths are multiples of 8)
  const int cols = min(WM, M - mw);
  // windows on the wave's rows, from its first column on
  auto window = [&](const void *p, int64_t ld, int es) {
    return __builtin_amdgcn_make_buffer_rsrc(
        const_cast<char *>(reinterpret_cast<const char *>(p)) + ((int64_t)nw * ld + mw) * es, 0,
        p ? (int)(uint32_t)(((int64_t)(rows_left - 1) * ld + cols) * es) : 0, BUF_DW3);
  };
  const __amdgpu_buffer_rsrc_t wo = window(a.out, a.ldo, ES), wz = window(a.z, a.ldz, 2), wr = window(a.res, a.ldr, ES);
  const bool use_z = PASS == EXPERT_DX ? a.act != IMBD_ACT_NONE : a.z != nullptr, use_res = a.res != nullptr;
  auto offset = [&](int r, int64_t ld, int es) { return in ? (uint32_t)r * (uint32_t)(ld * es) + (uint32_t)(8 * es * ch) : XW_OOB; };
  struct Extra {
    u32x4 z[UN], r[UN][ES / 2];
  } cur, next;
  auto load = [&](int g, Extra &x) {  // of the rounds g*UN ..
#pragma unroll
    for (int q = 0; q < UN; ++q) {
      const int r = (g * UN + q) * RPI + row0;
      if (PASS == EXPERT_DX && use_z) x.z[q] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(wz, offset(r, a.ldz, 2), 0, 0));
      if (use_res) {
#pragma unroll
        for (int h = 0; h < ES / 2; ++h)
          x.r[q][h] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(wr, offset(r, a.ldr, ES), 16 * h, 0));
      }
    }
  };
  auto half = [](const u32x4 &v, int i) {
    const uint32_t w = v[i >> 1];
    return __builtin_bit_cast(float, i & 1 ? w & 0xffff0000u : w << 16);
  };
  load(0, next);
#pragma unroll
  for (int part = 0; part < 2; ++part) {
    stage_sums<FM, FP>(acc, part, stg);
#pragma unroll 1
    for (int b = 0; b < NIT / UN; ++b) {
      cur = next;
      load(part * (NIT / UN) + b + 1, next);  // (past the last: outside the window, zeros)
      float run[UN][8];
#pragma unroll
      for (int q = 0; q < UN; ++q) staged_run<FM>(stg, (b * UN + q) * RPI + row0, ch, run[q]);
#pragma unroll
      for (int q = 0; q < UN; ++q) {
        const int r = part * FP * 16 + (b * UN + q) * RPI + row0;
        float(&v)[8] = run[q];
        if constexpr (PASS == EXPERT_FWD) {
          if (use_z)
            __builtin_amdgcn_raw_buffer_store_b128(u32x4{cvt_pk_bf16(v[0], v[1]), cvt_pk_bf16(v[2], v[3]), cvt_pk_bf16(v[4], v[5]),
                                                         cvt_pk_bf16(v[6], v[7])}, wz, offset(r, a.ldz, 2), 0, 2);
          apply_act(a.act, v);
        } else if (use_z) {
          float z[8];
#pragma unroll
          for (int i = 0; i < 8; ++i) z[i] = half(cur.z[q], i);
          apply_slope(a.act, v, z);
        }
        if (use_res) {
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            if constexpr (ES == 2) v[i] += half(cur.r[q][0], i);
            else v[i] += __builtin_bit_cast(f32x4, cur.r[q][i >> 2])[i & 3];
          }
        }
        if constexpr (ES == 2) {
          __builtin_amdgcn_raw_buffer_store_b128(u32x4{cvt_pk_bf16(v[0], v[1]), cvt_pk_bf16(v[2], v[3]), cvt_pk_bf16(v[4], v[5]),
                                                       cvt_pk_bf16(v[6], v[7])}, wo, offset(r, a.ldo, 2), 0, 2);
        } else {
#pragma unroll
          for (int h = 0; h < 2; ++h)
            __builtin_amdgcn_raw_buffer_store_b128(
                __builtin_bit_cast(u32x4, f32x4{v[4 * h], v[4 * h + 1], v[4 * h + 2], v[4 * h + 3]}), wo, offset(r, a.ldo, 4), 16 * h, 2);
        }
      }
    }
  }
}

// ES: bytes of an output (a kernel for each: with both in one, the sums were copied ahead of the branch, and spilled).
// A: ExpertArgs, or DenseArgs for one layer without experts: K in ranges, and its own epilogue.
template <int PASS, int BM, int BN, bool GATHER, int ES, typename A = ExpertArgs, DenseEnd END = DENSE_SUMS>
__global__ void __launch_bounds__(256, 1) expert_wide_kernel(A a, int tiles_m, int tiles_n) {
  constexpr bool DENSE = std::is_same<A, DenseArgs>::value;
  using Sh = Shape<PASS, BM, BN>;
  constexpr bool A_KC = Sh::A_KC, B_KC = Sh::B_KC;
  constexpr int FM = Sh::FM, FN = Sh::FN;
  constexpr bool GATHER_W = PASS == EXPERT_DW && GATHER;  // x by k-rows, each from its own row
  __shared__ __attribute__((aligned(1024))) char smem[xw_lds_bytes<PASS, BM, BN, GATHER>()];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)smem;

  // ---- the tile. The launch order has tiles in groups of XW_GM m tiles x all n tiles (Delta_W: of one expert);
  // the XCDs take 32 of it at a time by turns, so the workgroups resident on an XCD share slabs in its L2, and
  // experts of different length are spread over all XCDs (a contiguous range for each: Delta_W of 8 experts,
  // one to an XCD, waited for the longest twice as long as it worked).
  const int turn = (int)(blockIdx.x >> 3);
  int L = ((turn >> 5) * 8 + (int)(blockIdx.x & 7)) * 32 + (turn & 31);
  int e = 0, m0, n0, n_end, r0 = 0, K;
  const int M = PASS == EXPERT_FWD ? a.d_out : a.d_in;
  if constexpr (PASS == EXPERT_DW || DENSE) {
    e = L / (tiles_m * tiles_n);
    L -= e * (tiles_m * tiles_n);
  }
  const int mg = L / (XW_GM * tiles_n);
  const int gsz = min(XW_GM, tiles_m - mg * XW_GM);
  if (e >= a.E || gsz <= 0) return;
  L -= mg * XW_GM * tiles_n;
  const int tn = L / gsz;
  m0 = (mg * XW_GM + L - tn * gsz) * BM;
  if constexpr (PASS == EXPERT_DW) {
    n0 = tn * BN;
    n_end = a.d_out;
    if constexpr (DENSE) {
      e = __builtin_amdgcn_readfirstlane(e);
      r0 = e * a.chunk;
      K = min(a.chunk, a.n_rows - r0);
    } else {
      expert_range(a, e, &r0, &K);
    }
    r0 = __builtin_amdgcn_readfirstlane(r0);
    K = __builtin_amdgcn_readfirstlane(K);
  } else if constexpr (DENSE) {
    e = __builtin_amdgcn_readfirstlane(e);
    n0 = __builtin_amdgcn_readfirstlane(tn * BN);
    m0 = __builtin_amdgcn_readfirstlane(m0);
    n_end = a.n_rows;
    K = __builtin_amdgcn_readfirstlane(min(a.chunk, (PASS == EXPERT_FWD ? a.d_in : a.d_out) - e * a.chunk));
  } else {
    if (!find_row_tile<BN>(a, tn, &e, &n0, &n_end)) return;
    K = PASS == EXPERT_FWD ? a.d_in : a.d_out;
  }
  const int nsl = (K + XW_KS - 1) / XW_KS, nhs = (K + 31) / 32;  // slabs, half slabs
  const uint16_t *w = reinterpret_cast<const uint16_t *>(a.w) + (int64_t)e * a.sw;
  const uint16_t *x = reinterpret_cast<const uint16_t *>(a.x);
  const uint16_t *dy = reinterpret_cast<const uint16_t *>(a.dy);
  if constexpr (DENSE && PASS != EXPERT_DW) {  // the range's k
    const int64_t k0 = (int64_t)e * a.chunk;
    w += PASS == EXPERT_FWD ? k0 : k0 * a.ldw;
    if constexpr (PASS == EXPERT_FWD) x += k0;
    else dy += k0;
  }

  // ---- sources: a window on each operand and every lane's offsets in it
  // (k contiguous: a piece is 8 rows; k-rows: 8 k-rows of one quarter, a wave's rows 8*wave .. +7 of a half slab)
  uint32_t va[A_KC ? Sh::PA : 1], vb[B_KC ? Sh::PB : 1];
  const int kc = 8 * ((lane & 7) ^ (lane >> 3));                   // k contiguous: this lane's first k in a slab
  const int kr = 8 * wave + (lane >> 3);                           // k-rows: this lane's row of a half slab
  const uint32_t kcol = (uint32_t)(16 * ((lane & 7) ^ xw_swz_tr(kr)));  // ... and byte column of a quarter
  const int k_last = K - (nsl - 1) * XW_KS, h_last = K - (nhs - 1) * 32;  // k of the last slab, half slab
  // rows of k: 32 of them (h_last in the last half slab) of `cols` columns from the window's base on
  auto k_rows = [&](const uint16_t *p, int64_t ld, int cols) {
    return Window(p, 32 * ld * 2, (uint32_t)(((h_last < K ? 31 : h_last - 1) * ld + cols) * 2),
                  (uint32_t)(((h_last - 1) * ld + cols) * 2));
  };
  // k contiguous: `rows` rows (what lies past k in the last slab is masked by lane)
  auto k_cols = [&](const uint16_t *p, int64_t ld, int64_t rows) {
    const uint32_t n = rows > 0 ? (uint32_t)(((rows - 1) * ld + min(K, XW_KS)) * 2) : 0u;
    return Window(p, XW_KS * 2, n, rows > 0 ? (uint32_t)(((rows - 1) * ld + k_last) * 2) : 0u);
  };
  Window wa = [&] {
    if constexpr (A_KC) {
      return k_cols(w + (int64_t)m0 * a.ldw, a.ldw, min(BM, M - m0));
    } else if constexpr (PASS == EXPERT_DX) {
      return k_rows(w + m0, a.ldw, M - m0);
    } else if constexpr (!GATHER) {
      if (a.n_x == 0) return Window(nullptr, 0, 0u, 0u);  // (no x: db alone)
      return k_rows(x + (int64_t)r0 * a.ldx + m0, a.ldx, M - m0);
    } else {  // any row of x: the k-rows that do not exist are masked by lane
      const uint32_t n = a.n_x > 0 ? (uint32_t)(((int64_t)(a.n_x - 1) * a.ldx + M - m0) * 2) : 0u;
      return Window(x + m0, 0, n, n);
    }
  }();
  if constexpr (A_KC) {
#pragma unroll
    for (int q = 0; q < Sh::PA; ++q) {
      const int r = 8 * (Sh::PA * wave + q) + (lane >> 3);
      va[q] = m0 + r < M ? (uint32_t)(((int64_t)r * a.ldw + kc) * 2) : XW_OOB;
    }
  } else {
    va[0] = GATHER_W ? XW_OOB : (uint32_t)((int64_t)kr * (PASS == EXPERT_DX ? a.ldw : a.ldx) * 2) + kcol;
  }
  constexpr bool GATHER_X = PASS == EXPERT_FWD && GATHER;  // x by rows, each from its own row
  const int64_t ldb = PASS == EXPERT_FWD ? a.ldx : a.lddy;
  Window wb = [&] {
    if constexpr (!B_KC) return k_rows(dy + (int64_t)r0 * a.lddy + n0, a.lddy, n_end - n0);
    else if constexpr (GATHER_X) return k_cols(x, ldb, a.n_x);
    else return k_cols((PASS == EXPERT_FWD ? x : dy) + (int64_t)n0 * ldb, ldb, min(BN, n_end - n0));
  }();
  if constexpr (B_KC) {
#pragma unroll
    for (int q = 0; q < Sh::PB; ++q) {
      const int r = 8 * (Sh::PB * wave + q) + (lane >> 3);
      bool ok = n0 + r < n_end;
      int row = r;
      if constexpr (GATHER_X) {
        row = ok ? a.rows[n0 + r] : -1;
        ok = row >= 0 && row < a.n_x;
      }
      vb[q] = ok ? (uint32_t)row * (uint32_t)(ldb * 2) + (uint32_t)(kc * 2) : XW_OOB;
    }
  } else {
    vb[0] = (uint32_t)((int64_t)kr * a.lddy * 2) + kcol;
  }

  // the row indices of gathered k-rows: lane l's of half slab Y at idx0 + (Y % 8)*1024 + 4l
  const uint32_t idx0 = lds0 + (uint32_t)(Sh::RING + wave * 256 + 4 * lane);
  const i32x4 ri = GATHER_W ? buf_rsrc(a.rows + r0, (uint32_t)K * 4u) : i32x4{0, 0, 0, 0};
  auto load_index = [&](int Y) {
    if constexpr (GATHER_W)
      dma4(ri, (uint32_t)(Y * 32 + kr) * 4u, lds0 + (uint32_t)(Sh::RING + wave * 256 + (Y & 7) * 1024));
  };
  auto index_of = [&](int Y) {  // (its indices have landed)
    return *(const __attribute__((address_space(3))) int *)(uintptr_t)(idx0 + (uint32_t)((Y & 7) * 1024));
  };
  auto gather = [&](int Y, int row) {  // the offsets of half slab Y
    const bool ok = Y * 32 + kr < K && row >= 0 && row < a.n_x;
    va[0] = ok ? (uint32_t)row * (uint32_t)(a.ldx * 2) + kcol : XW_OOB;
  };

  // ---- loads, in the order of half slabs Y = 2 X + h (the windows move on); k-contiguous operands with h = 1
  auto ends = [&](int Y, auto htag) {  // before the loads of Y: the last ones and those past them
    constexpr int h = decltype(htag)::value;
    if constexpr ((!A_KC && !GATHER_W) || !B_KC) {
      if (Y >= nhs - 1) {
        if constexpr (!A_KC && !GATHER_W) wa.r[2] = Y == nhs - 1 ? (int)wa.last : 0;
        if constexpr (!B_KC) wb.r[2] = Y == nhs - 1 ? (int)wb.last : 0;
      }
    }
    if constexpr ((A_KC && h == 1) || (B_KC && h == Sh::HB)) {
      const int X = Y >> 1;
      if (X >= nsl - 1) {
        const bool past = kc >= k_last;  // this lane's k lies past the end
        if constexpr (A_KC && h == 1) {
          wa.r[2] = X == nsl - 1 ? (int)wa.last : 0;
#pragma unroll
          for (int q = 0; q < Sh::PA; ++q) va[q] = past ? XW_OOB : va[q];
        }
        if constexpr (B_KC && h == Sh::HB) {
          wb.r[2] = X == nsl - 1 ? (int)wb.last : 0;
#pragma unroll
          for (int q = 0; q < Sh::PB; ++q) vb[q] = past ? XW_OOB : vb[q];
        }
      }
    }
  };
  auto advance = [&](auto htag) {
    constexpr int h = decltype(htag)::value;
    if constexpr ((A_KC && h == 1) || (!A_KC && !GATHER_W)) wa.advance();
    if constexpr (h == Sh::HB || !B_KC) wb.advance();
  };
  // B's slots of slabs S, S + 1 and S + 2 (TRI; else they go with A's)
  uint32_t ub0 = lds0 + 2 * Sh::SA, ub1 = ub0 + Sh::SB, ub2 = ub1 + Sh::SB;
  // piece q of the loads of k-step h into slot t, by f(descriptor, offset, LDS address, instruction's offset)
  auto piece = [&](auto ttag, auto htag, auto qtag, auto f) {
    constexpr int t = decltype(ttag)::value, h = decltype(htag)::value, q = decltype(qtag)::value;
    if constexpr (q < Sh::la(h)) {
      constexpr uint32_t to = (uint32_t)(t * Sh::SA);
      if constexpr (A_KC) f(wa.r, va[q], lds0 + (uint32_t)(wave * Sh::PA * 1024) + to + q * 1024, std::integral_constant<int, 0>{});
      else f(wa.r, va[0], lds0 + (uint32_t)(wave * 1024) + to + q * 8192 + h * 4096, std::integral_constant<int, 128 * q>{});
    } else {
      constexpr int p = q - Sh::la(h);
      constexpr uint32_t to = (uint32_t)(2 * Sh::SA + t * Sh::SB);
      if constexpr (Sh::TRI) f(wb.r, vb[p], ub2 + (uint32_t)(wave * Sh::PB * 1024) + p * 1024, std::integral_constant<int, 0>{});
      else if constexpr (B_KC) f(wb.r, vb[p], lds0 + (uint32_t)(wave * Sh::PB * 1024) + to + p * 1024, std::integral_constant<int, 0>{});
      else f(wb.r, vb[0], lds0 + (uint32_t)(wave * 1024) + to + p * 8192 + h * 4096, std::integral_constant<int, 128 * p>{});
    }
  };

  // ---- fragments
  const int fi = lane & 15, kg = lane >> 4, wm = wave & 1, wn = wave >> 1;
  const int tr = 8 * kg + (fi >> 2);
  // addresses of k-step 0 (k contiguous: and of k-step 1) of slot 0, then those of slot 1 (TRI: B's without the
  // slot): the rest of a read's address is a constant of the instruction
  constexpr int NA = A_KC ? 2 : 4, NB = B_KC ? 2 : 4;
  uint32_t fa[2][NA], fb[2][NB];
#pragma unroll
  for (int t = 0; t < 2; ++t) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint32_t kcl = (uint32_t)(fi * 128 + (((4 * j + kg) ^ (fi & 7)) * 16));
      const uint32_t trr = (uint32_t)(((2 * j + ((fi >> 1) & 1)) ^ xw_swz_tr(tr)) * 16 + tr * 128 + 8 * (fi & 1));
      if (j < NA)
        fa[t][j] = lds0 + (uint32_t)(t * Sh::SA) + (A_KC ? (uint32_t)(wm * FM * 2048) + kcl : (uint32_t)(wm * FM / 4 * 8192) + trr);
      if (j < NB)
        fb[t][j] = (Sh::TRI ? 0u : lds0 + (uint32_t)(2 * Sh::SA + t * Sh::SB)) +
                   (B_KC ? (uint32_t)(wn * FN * 2048) + kcl : (uint32_t)(wn * FN / 4 * 8192) + trr);
    }
#pragma unroll
    for (int j = 0; j < NA; ++j) asm volatile("" : "+v"(fa[t][j]));
#pragma unroll
    for (int j = 0; j < NB; ++j)
      if (!Sh::TRI || t == 0) asm volatile("" : "+v"(fb[t][j]));
  }
  static_assert(FM % 4 == 0 && FN % 4 == 0, "k-row fragments come in whole quarters");
  auto lds16 = [](uint32_t p) {
    return __builtin_bit_cast(bf16x8, *(const __attribute__((address_space(3))) u32x4 *)(uintptr_t)p);
  };
  auto lds_tr = [](uint32_t p) {
    lds_i16x4 *q = (lds_i16x4 *)(uintptr_t)p;
    const i16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16(q);
    const i16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(q + 4 * 128 / 8);
    return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
  };
  // block i of k-step h of the slab in slot t
  auto read_a = [&](int t, int h, int i) {
    if constexpr (A_KC) return lds16(fa[t][h] + (uint32_t)(i * 2048));
    else return lds_tr(fa[t][i & 3] + (uint32_t)((i >> 2) * 8192 + h * 4096));
  };
  auto read_b = [&](int t, int h, int j) {
    if constexpr (B_KC) return lds16(fb[t][h] + (uint32_t)(j * 2048));  // (not TRI)
    else return lds_tr(fb[t][j & 3] + (uint32_t)((j >> 2) * 8192 + h * 4096));
  };

  // the sums begin with the bias
  f32x4 acc[FM][FN], accd[PASS == EXPERT_DW ? FN : 1];
#pragma unroll
  for (int i = 0; i < FM; ++i) {
    f32x4 first = {0.f, 0.f, 0.f, 0.f};
    const int m = m0 + wm * (BM / 2) + 16 * i + 4 * kg;  // (the width is a multiple of 8: all four or none)
    if (PASS == EXPERT_FWD && END != DENSE_ANY && a.bias && m < M)
      first = *reinterpret_cast<const f32x4_any *>(a.bias + (int64_t)e * a.d_out + m);
#pragma unroll
    for (int j = 0; j < FN; ++j) acc[i][j] = first;
  }
  // db: the products with a row of ones, by the waves of the first m tile's first half
  const bool do_db = PASS == EXPERT_DW && a.db && m0 == 0 && wm == 0;
  if constexpr (PASS == EXPERT_DW)
#pragma unroll
    for (int j = 0; j < FN; ++j) accd[j] = f32x4{0.f, 0.f, 0.f, 0.f};
  const bf16x8 ones = __builtin_bit_cast(bf16x8, u32x4{0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u});

  // ---- a wave's part of the mask: four rows a load, each lane what it will store with (rows in expert order; of
  // gathered ones it is loaded in the epilogue)
  constexpr bool MASK_LDS = xw_mask_in_lds(PASS, BN) && !DENSE;
  const uint32_t mask0 = lds0 + (uint32_t)(xw_lds_bytes<PASS, BM, BN, GATHER>() - BM * BN * 2 + wave * (BM * BN / 2));
  if constexpr (MASK_LDS) {
    const int mw = m0 + wm * (BM / 2), nw = n0 + wn * (BN / 2), left = min(BN / 2, n_end - nw);
    if (a.mask && !a.rows && left > 0 && mw < M) {
      const i32x4 rm = buf_rsrc(x + (int64_t)nw * a.ldx + mw, (uint32_t)(((int64_t)(left - 1) * a.ldx + min(BM / 2, M - mw)) * 2));
      const uint32_t c = mw + 8 * fi < M ? (uint32_t)(16 * fi) : XW_OOB;
#pragma unroll
      for (int q = 0; q < BN / 8; ++q)
        dma16(rm, c == XW_OOB ? XW_OOB : (uint32_t)(4 * q + kg) * (uint32_t)(a.ldx * 2) + c, mask0 + (uint32_t)(q * 1024));
    }
  }

  // ---- the first two slabs (and the indices of eight half slabs)
  const std::integral_constant<int, 0> c0{};
  const std::integral_constant<int, 1> c1{};
  if constexpr (GATHER_W) {
#pragma unroll
    for (int Y = 0; Y < 8; ++Y) load_index(Y);
    asm volatile("s_waitcnt vmcnt(0)" : : : "memory");
  }
  auto first = [&](auto ttag, auto htag) {
    constexpr int t = decltype(ttag)::value, h = decltype(htag)::value;
    if constexpr (GATHER_W) gather(2 * t + h, index_of(2 * t + h));
    ends(2 * t + h, htag);
    if constexpr (Sh::TRI && h == 0) ub2 = t ? ub1 : ub0;
    static_for<Sh::loads(h)>([&](auto q) {
      piece(ttag, htag, q,
            [&](const i32x4 &r, uint32_t voff, uint32_t to, auto imm) { dma16_at<decltype(imm)::value>(r, voff, to); });
    });
    advance(htag);
  };
  first(c0, c0);
  first(c0, c1);
  first(c1, c0);
  load_index(6);  // (again: every k-step's loads end with one)
  first(c1, c1);
  load_index(7);
  if constexpr (Sh::TRI) ub2 = ub1 + Sh::SB;
  // loads that may be under way when k-step h begins. Its fragment reads take a half slab loaded three k-steps ago,
  // for h = 1 a k-contiguous operand's slab loaded two ago.
  constexpr int IDX = GATHER_W ? 1 : 0;
  constexpr int VM0 = Sh::loads(0) + Sh::loads(1) + 2 * IDX, VM1 = A_KC || B_KC ? Sh::loads(0) : VM0;
  constexpr bool BOTH_KC = A_KC && B_KC;

  bf16x8 av[2][FM], bv[2][FN];
  step_wait<true, VM0>();  // slab 0
#pragma unroll
  for (int i = 0; i < FM; ++i) av[0][i] = read_a(0, 0, i);
#pragma unroll
  for (int j = 0; j < FN; ++j) bv[0][j] = Sh::TRI ? lds16(ub0 + fb[0][0] + (uint32_t)(j * 2048)) : read_b(0, 0, j);
  if constexpr (GATHER_W) gather(4, index_of(4));
  ends(4, c0);

  // k-step h of slab S, which lies in slot t = S % 2. Between its products, one by one, what else there is to do, so
  // that it fits in their shadow (a wave issues an instruction every four cycles, a product takes sixteen; all the
  // scalar work of a slab in one place left the matrix cores idle for 15% of the time): the fragments of the next
  // k-step, the loads of slab S + 2 into what every wave has read, and what the next loads need.
  auto step = [&](int S, auto ttag, auto htag) {
    constexpr int t = decltype(ttag)::value, h = decltype(htag)::value;
    if constexpr (h == 0) step_wait<!BOTH_KC, VM0>();
    else step_wait<true, VM1>();
    const int Y = 2 * S + h;
    int row = 0;
    uint32_t pb = 0;
    if constexpr (Sh::TRI) {  // B's fragments of the next k-step
      pb = (h == 0 ? ub0 : ub1) + fb[0][(h ^ 1) % NB];
      asm volatile("" : "+v"(pb));
    }
    constexpr int NM = FM * FN, NR = FM + FN, NL = Sh::loads(h), SPAN = NM < 3 * NL ? NM : 3 * NL;
    constexpr int ADV = SPAN > NM - 14 ? SPAN : NM - 14;  // behind the last load
    static_assert(NM >= 2 * NR + 8 && SPAN >= 2 * NL && ADV <= NM - 8, "");
    static_for<NM>([&](auto ptag) {
      constexpr int p = decltype(ptag)::value;
      f32x4 &d = acc[p / FN][p % FN];
      const bf16x8 &ma = av[h][p / FN], &mb = bv[h][p % FN];
      // read r before every odd product: a and b by turns, then what is left of the longer
      constexpr int r = p % 2 == 1 ? p / 2 : NR;
      constexpr int both = 2 * (FM < FN ? FM : FN);
      constexpr bool is_a = r < both ? r % 2 == 0 : FM > FN;
      constexpr int at = r < both ? r / 2 : r - both / 2;
      if constexpr (r < NR) {
        if constexpr (is_a) av[h ^ 1][at] = read_a(h == 0 ? t : t ^ 1, h ^ 1, at);
        else if constexpr (Sh::TRI) bv[h ^ 1][at] = lds16(pb + (uint32_t)(at * 2048));
        else bv[h ^ 1][at] = read_b(h == 0 ? t : t ^ 1, h ^ 1, at);
      }
      // load q with an even product
      constexpr int q = xw_load_at(p, NL, SPAN);
      if constexpr (q < NL) {
        piece(ttag, htag, std::integral_constant<int, q>{}, [&](const i32x4 &r, uint32_t voff, uint32_t to, auto imm) {
          mfma_dma16<decltype(imm)::value>(d, ma, mb, r, voff, to);
        });
      } else {
        mfma(d, ma, mb);
      }
      if constexpr (p == ADV) {
        advance(htag);
        if constexpr (GATHER_W) {
          load_index(Y + 8);  // (landed three k-steps on, read one after that)
          row = index_of(Y + 5);
        }
      }
      if constexpr (GATHER_W && p == NM - 6) gather(Y + 5, row);
      if constexpr (Sh::TRI && h == 1 && p == NM - 8) {
        const uint32_t u = ub0;
        ub0 = ub1;
        ub1 = ub2;
        ub2 = u;
      }
      if constexpr (p == NM - 3) ends(Y + 5, std::integral_constant<int, h ^ 1>{});
      __builtin_amdgcn_sched_barrier(0);
    });
    if constexpr (PASS == EXPERT_DW) {
      if (do_db) {
#pragma unroll
        for (int j = 0; j < FN; ++j) mfma_v(accd[j], ones, bv[h][j]);
      }
    }
  };
  // (slabs in pairs, so that slots and register sets are constants: one past the last is zeros)
  for (int S = 0; S < nsl; S += 2) {
    step(S, c0, c0);
    step(S, c0, c1);
    step(S + 1, c1, c0);
    step(S + 1, c1, c1);
  }
  vm_barrier<0>();  // LDS is free: nothing is in flight and every wave is done reading
  mfma_drain();
  if constexpr (PASS == EXPERT_DW)
#pragma unroll
    for (int j = 0; j < FN; ++j) asm volatile("" : "+v"(accd[j]));

  if constexpr (PASS == EXPERT_DW) {
    if (do_db && kg == 0) {
#pragma unroll
      for (int j = 0; j < FN; ++j) {
        const int n = n0 + 16 * (wn * FN + j) + fi;
        if (n < n_end) a.db[(int64_t)e * a.d_out + n] = accd[j][0];
      }
    }
    if (!a.out) return;
  }

  // ---- epilogue: each wave puts its outputs through its own part of LDS ([n][m], 16-byte chunks XORed with the row)
  // and stores whole rows, 16 bytes a lane, past the caches (537 MB of gradients of few rows: 131 -> 109 us); what lies
  // outside the tile's rows or columns is past the descriptor.
  constexpr int WM = BM / 2, WN = BN / 2;  // columns, rows of a wave
  const int mw = m0 + wm * WM, nw = n0 + wn * WN;
  const uint32_t stg = lds0 + (uint32_t)(wave * xw_stage_bytes(BM, BN));
  const float least = PASS == EXPERT_FWD && a.relu ? 0.f : -__builtin_inff();
  const int rows_left = min(WN, n_end - nw);
  if (rows_left <= 0 || mw >= M) return;
  if constexpr (END == DENSE_CHUNKS) {
    dense_wide_epilogue<PASS, ES, FM, FN>(a, acc, stg, mw, nw, rows_left, M);
    return;
  }
  if constexpr (END == DENSE_ANY) {
    dense_any_epilogue<PASS, FM, FN>(a, acc, stg, mw, nw, rows_left);
    return;
  }
  // Rows of 32-bit outputs go in two halves of the wave's.
  {
    constexpr int PITCH = WM * ES, CPR = PITCH / 16;  // row bytes, chunks a row
    constexpr int PARTS = ES / 2, FP = FN / PARTS, RPI = 64 / CPR, NST = FP * 16 / RPI;  // blocks a part; rows, stores
    char *dst = reinterpret_cast<char *>(a.out) + ((PASS == EXPERT_DW || DENSE ? (int64_t)e * a.so : 0) + (int64_t)nw * a.ldo + mw) * ES;
    const i32x4 ro = buf_rsrc(dst, (uint32_t)(((int64_t)(rows_left - 1) * a.ldo + min(WM, M - mw)) * ES));
    const __amdgpu_buffer_rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc(dst, 0, ro[2], BUF_DW3);
    const int row0 = lane / CPR, ch = lane % CPR;
    const uint32_t col = mw + ch * (16 / ES) < M ? (uint32_t)(ch * 16) : XW_OOB;
    constexpr int BATCH = 8, NBT = NST / BATCH;  // stores in batches
    static_assert(NST % BATCH == 0, "");
    // the mask of a batch (Delta_X), loaded ahead of the one before it
    using MaskVec = typename std::conditional<ES == 2, u32x4, u32x2>::type;  // of as many elements as a store has
    MaskVec mk[2][BATCH];
    auto load_mask = [&](int g) {
      if constexpr (PASS == EXPERT_DX && !DENSE) {
        if (a.mask && g < PARTS * NBT) {
#pragma unroll
          for (int q = 0; q < BATCH; ++q) {
            const int r = (g * BATCH + q) * RPI + row0;
            if constexpr (MASK_LDS) {
              if (!a.rows) {
                mk[g & 1][q] = *(const __attribute__((address_space(3))) MaskVec *)(uintptr_t)(
                    mask0 + (uint32_t)((r >> 2) * 1024 + (r & 3) * 256 + ch * (32 / ES)));
                continue;
              }
            }
            int row = -1;
            if (r < rows_left && col != XW_OOB) row = a.rows ? a.rows[nw + r] : nw + r;
            mk[g & 1][q] = MaskVec{};
            if (row >= 0 && row < a.n_x)
              mk[g & 1][q] = *reinterpret_cast<const MaskVec *>(x + (int64_t)row * a.ldx + mw + ch * (16 / ES));
          }
        }
      }
    };
    load_mask(0);
#pragma unroll
    for (int part = 0; part < PARTS; ++part) {
#pragma unroll
      for (int i = 0; i < FM; ++i) {
        const uint32_t c = ES == 2 ? (uint32_t)(((2 * i + (kg >> 1)) ^ fi) * 16 + 8 * (kg & 1)) : (uint32_t)(((4 * i + kg) ^ fi) * 16);
        const uint32_t p = stg + (uint32_t)(fi * PITCH) + c;
#pragma unroll
        for (int j = 0; j < FP; ++j) {
          f32x4 v = acc[i][part * FP + j];
          asm volatile("" : "+a"(v));  // (read here, behind the wait states)
          if constexpr (PASS == EXPERT_FWD && !DENSE) {
#pragma unroll
            for (int q = 0; q < 4; ++q) v[q] = __builtin_elementwise_maximum(v[q], least);  // (a NaN stays one)
          }
          if constexpr (ES == 2)
            *(__attribute__((address_space(3))) u32x2 *)(uintptr_t)(p + j * 16 * PITCH) =
                u32x2{cvt_pk_bf16(v[0], v[1]), cvt_pk_bf16(v[2], v[3])};
          else
            *(__attribute__((address_space(3))) f32x4 *)(uintptr_t)(p + j * 16 * PITCH) = v;
        }
        __builtin_amdgcn_sched_barrier(0);
      }
#pragma unroll
      for (int b = 0; b < NBT; ++b) {
        const int g = part * NBT + b, s0 = b * BATCH;
        load_mask(g + 1);
        u32x4 v[BATCH];
#pragma unroll
        for (int q = 0; q < BATCH; ++q) {
          const int r = (s0 + q) * RPI + row0;
          v[q] = *(const __attribute__((address_space(3))) u32x4 *)(uintptr_t)(stg + (uint32_t)(r * PITCH + ((ch ^ (r & 15)) * 16)));
        }
#pragma unroll
        for (int q = 0; q < BATCH; ++q) {
          if constexpr (PASS == EXPERT_DX && !DENSE) {
            if (a.mask) {
#pragma unroll
              for (int w2 = 0; w2 < 8 / (ES / 2); ++w2) {
                const bool on = bf16_to_f32((uint16_t)(mk[g & 1][q][w2 >> 1] >> (16 * (w2 & 1)))) > 0.f;
                if constexpr (ES == 2) v[q][w2 >> 1] &= on ? 0xffffffffu : (w2 & 1) ? 0xffffu : 0xffff0000u;
                else v[q][w2] = on ? v[q][w2] : 0u;
              }
            }
          }
          const int r = part * FP * 16 + (s0 + q) * RPI + row0;
          const uint32_t off = col == XW_OOB ? XW_OOB : (uint32_t)r * (uint32_t)(a.ldo * ES) + col;
          __builtin_amdgcn_raw_buffer_store_b128(v[q], rs, off, 0, 2);  // nt
        }
      }
    }
  }
}

}  // namespace
}  // namespace imbd
