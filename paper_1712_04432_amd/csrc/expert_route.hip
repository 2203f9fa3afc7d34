// The router of an expert layer: each token's k largest logits, their gates, the plan that puts the (token,
// choice) pairs in the order of (expert, token, choice), and the logits' gradient.
//
// Choosing. G = 8 to 64 lanes share a token, VPL logits each in registers (G * VPL >= E, lane q the
// experts q*VPL ..), so a wave serves 64/G tokens at once. A logit becomes a whole number of the same
// order (NaN above all, -inf the lowest, 0 for "none"); k rounds each take the largest of the group: the
// lane's own maximum, log2 G exchanges, then the lowest expert index among those that hold it, which makes
// ties go to the lowest expert whatever the lanes do. Selection compares the logits themselves, never
// rounded probabilities.
//
// Ordering. A stable counting sort without atomics on the result: workgroup b (128 tokens, or more, so that there are
// at most 256 workgroups) counts
// its pairs per expert into row b of a table in ws; the second launch adds up the rows before its own for
// the start of its pairs of each expert, and numbers its pairs in order, 64 at a time in a wave (a pair's
// rank among the lanes of its expert comes from one ballot for each bit of the expert's index). Up to
// 128 tokens one workgroup does both in one launch.
//
// Bound by latency: 16384 tokens, 64 experts, k = 8 move 11 MB (2.3 us) and take 8.3 us for the choice, 5.1 for the
// order (both on 128 workgroups, half of the CUs) and 4.7 for the logits' gradient (means of ten launches; the least 7.6,
// 4.6 and 4.4); 16 tokens, k = 4, 5.0 us in one launch (least 4.8).

#include "expert.h"

namespace imbd {
namespace {

constexpr int RT_NT = 1024;      // threads of a workgroup
constexpr int RT_BLOCKS = 256;   // workgroups at most (rows of the table)

// Whole number of the same order as v; NaN the largest, 0 is below every value.
__device__ __forceinline__ uint32_t order_key(float v) {
  if (v != v) return 0xffffffffu;
  const uint32_t u = __builtin_bit_cast(uint32_t, v + 0.0f);  // (-0 becomes +0: they tie)
  return (u >> 31) ? ~u : (u | 0x80000000u);
}
__device__ __forceinline__ float key_value(uint32_t k) {
  if (k == 0xffffffffu) return __builtin_nanf("");
  return __builtin_bit_cast(float, (k >> 31) ? (k & 0x7fffffffu) : ~k);
}
constexpr uint32_t KEY_MINUS_INF = 0x007fffffu;  // order_key(-inf)

// The value of the lane that a group's reduction pairs with at distance o: inside 16 lanes by the cross-lane forms
// of the vector instructions (at 4 and 8 the mirrored lane, which holds the same as its neighbours by then).
template <int o>
__device__ __forceinline__ int partner(int v) {
  if constexpr (o == 1) return __builtin_amdgcn_update_dpp(0, v, 0xB1, 0xf, 0xf, false);        // quad: 1 0 3 2
  else if constexpr (o == 2) return __builtin_amdgcn_update_dpp(0, v, 0x4E, 0xf, 0xf, false);   // quad: 2 3 0 1
  else if constexpr (o == 4) return __builtin_amdgcn_update_dpp(0, v, 0x141, 0xf, 0xf, false);  // half rows mirrored
  else if constexpr (o == 8) return __builtin_amdgcn_update_dpp(0, v, 0x140, 0xf, 0xf, false);  // rows mirrored
  else return __shfl_xor(v, o, 64);
}
template <int G, int o = 1>
__device__ __forceinline__ uint32_t group_max(uint32_t v) {
  if constexpr (o >= G) return v;
  else return group_max<G, 2 * o>(max(v, (uint32_t)partner<o>((int)v)));
}
template <int G, int o = 1>
__device__ __forceinline__ int group_min(int v) {
  if constexpr (o >= G) return v;
  else return group_min<G, 2 * o>(min(v, partner<o>(v)));
}
template <int G, int o = 1>
__device__ __forceinline__ float group_sum(float v) {
  if constexpr (o >= G) return v;
  else return group_sum<G, 2 * o>(v + __builtin_bit_cast(float, partner<o>(__builtin_bit_cast(int, v))));
}

// Eight consecutive values from p (n of them real, the others `none`).
__device__ __forceinline__ void load8(const float *p, int n, float none, float (&v)[8]) {
  if (n >= 8) {
    const f32x4 a = *reinterpret_cast<const f32x4_any *>(p), b = *reinterpret_cast<const f32x4_any *>(p + 4);
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = a[i], v[4 + i] = b[i];
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = i < n ? p[i] : none;
  }
}

struct RouteArgs {
  int T, E, k, renorm;
  const float *logits;
  int64_t ldl;
  float *gates;
  int32_t *experts, *offsets, *rows, *slots;
  int32_t *table;  // [blocks][E] pairs of each expert in each workgroup's tokens
  int blocks, per_block;
};

// The choices and gates of token t, by the G lanes of its group (q: the lane in the group). count(e) is
// called once for each pair, by one lane.
template <int G, typename F>
__device__ __forceinline__ void choose(const RouteArgs &a, int t, int q, F count) {
  constexpr int VPL = 8;
  const float *z = a.logits + (int64_t)t * a.ldl;
  uint32_t key[VPL];
  float zv[VPL];
  load8(z + q * VPL, a.E - q * VPL, -INFINITY, zv);
#pragma unroll
  for (int i = 0; i < VPL; ++i) {
    const uint32_t u = order_key(zv[i]);
    key[i] = u == KEY_MINUS_INF ? 0u : u;  // never chosen
  }
  float all = 0.f, peak = 0.f;
  uint32_t top = 0u;
#pragma unroll
  for (int i = 0; i < VPL; ++i) top = max(top, key[i]);
  top = group_max<G>(top);
  if (top) peak = key_value(top);
  if (!a.renorm) {
#pragma unroll
    for (int i = 0; i < VPL; ++i) all += key[i] ? expf(key_value(key[i]) - peak) : 0.f;
    all = group_sum<G>(all);
  }
  // choice j stays with lane j % G (k <= 16, G >= 8: two of them a lane)
  int mine_e[2] = {-1, -1};
  float mine_p[2] = {0.f, 0.f}, chosen = 0.f;
  for (int j = 0; j < a.k; ++j) {
    uint32_t best = 0u;
#pragma unroll
    for (int i = 0; i < VPL; ++i) best = max(best, key[i]);
    best = group_max<G>(best);
    if (!best) break;  // (the whole group)
    int at = 0x7fffffff;
#pragma unroll
    for (int i = VPL - 1; i >= 0; --i)
      if (key[i] == best) at = q * VPL + i;
    at = group_min<G>(at);
#pragma unroll
    for (int i = 0; i < VPL; ++i)
      if (q * VPL + i == at) key[i] = 0u;
    const float p = expf(key_value(best) - peak);
    chosen += p;
#pragma unroll
    for (int h = 0; h < 2; ++h)
      if (q + h * G == j) {
        mine_e[h] = at;
        mine_p[h] = p;
      }
  }
  const float total = a.renorm ? chosen : all;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int j = q + h * G;
    if (j < a.k) {
      const int64_t at = (int64_t)t * a.k + j;
      a.experts[at] = mine_e[h];
      a.gates[at] = mine_e[h] >= 0 ? mine_p[h] / total : 0.f;
      if (mine_e[h] >= 0) count(mine_e[h]);
    }
  }
}

// Numbers the pairs of tokens t0 .. t1-1 in order: run[e] holds the next slot of each expert. cnt: one row
// of E counts for each wave.
__device__ __forceinline__ void place(const RouteArgs &a, int t0, int t1, int32_t *run, int32_t *cnt) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  constexpr int NW = RT_NT / 64;
  const int64_t end = (int64_t)t1 * a.k;
  for (int64_t i0 = (int64_t)t0 * a.k; i0 < end; i0 += RT_NT) {
    for (int i = tid; i < NW * a.E; i += RT_NT) cnt[i] = 0;
    __syncthreads();
    const int64_t i = i0 + tid;
    const int e = i < end ? a.experts[i] : -1;
    uint64_t same = __ballot(e >= 0);
    for (int b = 1; b < a.E; b <<= 1) {
      const uint64_t bit = __ballot((e & b) != 0);
      same &= (e & b) ? bit : ~bit;
    }
    const int rank = __builtin_popcountll(same & (((uint64_t)1 << lane) - 1));
    if (e >= 0 && rank == 0) cnt[wave * a.E + e] = __builtin_popcountll(same);
    __syncthreads();
    if (e >= 0) {
      int s = run[e] + rank;
      for (int w = 0; w < wave; ++w) s += cnt[w * a.E + e];
      a.slots[i] = s;
      a.rows[s] = (int32_t)(i / a.k);
    } else if (i < end) {
      a.slots[i] = -1;
    }
    __syncthreads();
    for (int x = tid; x < a.E; x += RT_NT) {
      int s = run[x];
      for (int w = 0; w < NW; ++w) s += cnt[w * a.E + x];
      run[x] = s;
    }
    __syncthreads();
  }
}

// run[e] <- the sum of all[0 .. e-1] plus before[e] (before: pairs of earlier workgroups), by the first
// wave; offsets from workgroup 0.
__device__ __forceinline__ void starts(const RouteArgs &a, const int32_t *all, int32_t *run, bool write) {
  const int lane = threadIdx.x;
  if (lane < 64) {
    int carry = 0;
    for (int e0 = 0; e0 < a.E; e0 += 64) {
      const int e = e0 + lane;
      const int n = e < a.E ? all[e] : 0;
      int upto = n;
#pragma unroll
      for (int d = 1; d < 64; d <<= 1) {
        const int v = __shfl_up(upto, d, 64);
        if (lane >= d) upto += v;
      }
      if (e < a.E) {
        run[e] += carry + upto - n;
        if (write) a.offsets[e + 1] = carry + upto;
      }
      carry += __shfl(upto, 63, 64);
    }
    if (write && lane == 0) a.offsets[0] = 0;
  }
  __syncthreads();
}

// First launch: the choices, and the table's row of each workgroup. SINGLE: the whole router.
template <int G, bool SINGLE>
__global__ void __launch_bounds__(RT_NT) choose_kernel(RouteArgs a) {
  extern __shared__ int32_t sm[];  // [E] counts; SINGLE: [E] run, [16][E]
  const int tid = threadIdx.x, q = tid % G;
  for (int i = tid; i < a.E; i += RT_NT) sm[i] = 0;
  if (SINGLE)
    for (int i = tid; i < a.E; i += RT_NT) sm[a.E + i] = 0;
  __syncthreads();
  const int t0 = blockIdx.x * a.per_block, t1 = (int)min((int64_t)a.T, (int64_t)t0 + a.per_block);
  for (int64_t t = t0 + tid / G; t < t1; t += RT_NT / G) choose<G>(a, (int)t, q, [&](int e) { atomicAdd(&sm[e], 1); });
  __syncthreads();
  if constexpr (SINGLE) {
    __threadfence_block();
    starts(a, sm, sm + a.E, true);
    place(a, t0, t1, sm + a.E, sm + 2 * a.E);
  } else {
    for (int i = tid; i < a.E; i += RT_NT) a.table[(int64_t)blockIdx.x * a.E + i] = sm[i];
  }
}

// Second launch: every workgroup's pairs into their slots.
__global__ void __launch_bounds__(RT_NT) place_kernel(RouteArgs a) {
  extern __shared__ int32_t sm[];  // [E] all, [E] run, [16][E]
  const int tid = threadIdx.x, b = blockIdx.x;
  for (int i = tid; i < 2 * a.E; i += RT_NT) sm[i] = 0;
  __syncthreads();
  // column sums of the table: RT_NT/E threads an expert (whole numbers: the order does not matter)
  const int parts = max(1, RT_NT / a.E), e = tid % a.E, part = tid / a.E;
  if (part < parts) {
    int all = 0, before = 0;
#pragma unroll 8
    for (int r = part; r < a.blocks; r += parts) {
      const int n = a.table[(int64_t)r * a.E + e];
      all += n;
      before += r < b ? n : 0;
    }
    atomicAdd(&sm[e], all);
    atomicAdd(&sm[a.E + e], before);
  }
  __syncthreads();
  starts(a, sm, sm + a.E, b == 0);
  place(a, b * a.per_block, (int)min((int64_t)a.T, (int64_t)(b + 1) * a.per_block), sm + a.E, sm + 2 * a.E);
}

struct RouteBwdArgs {
  int T, E, k, renorm;
  const float *logits;
  int64_t ldl;
  const float *gates, *dgates;
  const int32_t *experts;
  float *dlogits;
  int64_t lddl;
};

// G lanes a token, as in the choice; the k <= KM pairs are read by every lane of the group (the same cached lines),
// all at once.
template <int G, int KM>
__global__ void __launch_bounds__(256) route_bwd_kernel(RouteBwdArgs a) {
  constexpr int VPL = 8;
  const int q = threadIdx.x % G, t = blockIdx.x * (256 / G) + threadIdx.x / G;
  if (t >= a.T) return;  // (whole groups)
  const int64_t p0 = (int64_t)t * a.k;
  int e[KM];
  float g[KM], dg[KM], v[VPL];
#pragma unroll
  for (int j = 0; j < KM; ++j) {
    const bool in = j < a.k;
    e[j] = in ? a.experts[p0 + j] : -1;
    g[j] = in ? a.gates[p0 + j] : 0.f;
    dg[j] = in ? a.dgates[p0 + j] : 0.f;
  }
  if (!a.renorm) load8(a.logits + (int64_t)t * a.ldl + q * VPL, a.E - q * VPL, -INFINITY, v);
  float dz[VPL], inner = 0.f;
#pragma unroll
  for (int i = 0; i < VPL; ++i) dz[i] = 0.f;
#pragma unroll
  for (int j = 0; j < KM; ++j)
    if (e[j] >= 0) inner = fmaf(g[j], dg[j], inner);
  const float off = a.renorm ? inner : 0.f;
#pragma unroll
  for (int j = 0; j < KM; ++j) {
    const int at = e[j] - q * VPL;
    const float add = g[j] * (dg[j] - off);
#pragma unroll
    for (int i = 0; i < VPL; ++i) dz[i] += e[j] >= 0 && at == i ? add : 0.f;
  }
  if (!a.renorm) {
    uint32_t top = 0u;  // (as whole numbers of the same order: a NaN counts)
#pragma unroll
    for (int i = 0; i < VPL; ++i) top = max(top, order_key(v[i]));
    top = group_max<G>(top);
    if (top > KEY_MINUS_INF) {
      const float peak = key_value(top);
      float sum = 0.f;
#pragma unroll
      for (int i = 0; i < VPL; ++i) {
        v[i] = v[i] == -INFINITY ? 0.f : expf(v[i] - peak);
        sum += v[i];
      }
      sum = group_sum<G>(sum);
#pragma unroll
      for (int i = 0; i < VPL; ++i) dz[i] -= v[i] / sum * inner;
    }
  }
  float *out = a.dlogits + (int64_t)t * a.lddl + q * VPL;
  const int n = a.E - q * VPL;
  if (n >= VPL) {
    *reinterpret_cast<f32x4_any *>(out) = f32x4{dz[0], dz[1], dz[2], dz[3]};
    *reinterpret_cast<f32x4_any *>(out + 4) = f32x4{dz[4], dz[5], dz[6], dz[7]};
  } else {
#pragma unroll
    for (int i = 0; i < VPL; ++i)
      if (i < n) out[i] = dz[i];
  }
}

// Tokens of a workgroup, and the number of workgroups.
void route_split(int T, int *blocks, int *per_block) {
  int per = 128;  // 8 lanes a token: one round of the workgroup
  while ((T + (int64_t)per - 1) / per > RT_BLOCKS) per *= 2;
  *per_block = per;
  *blocks = (int)((T + (int64_t)per - 1) / per);
}

__global__ void zero_offsets_kernel(int32_t *p, int n) {
  for (int i = threadIdx.x; i < n; i += 256) p[i] = 0;
}

}  // namespace

size_t route_ws_bytes(int T, int E, int k) {
  int blocks, per;
  route_split(T, &blocks, &per);
  return blocks <= 1 ? 0 : (size_t)blocks * E * 4;
}

int run_route(int T, int E, int k, int renorm, const float *logits, int64_t ldl, float *gates, int32_t *experts,
              int32_t *offsets, int32_t *rows, int32_t *slots, void *ws, hipStream_t s) {
  if (T == 0) {
    hipLaunchKernelGGL(zero_offsets_kernel, dim3(1), dim3(256), 0, s, offsets, E + 1);
    return check_launch("expert_route");
  }
  RouteArgs a{T, E, k, renorm, logits, ldl, gates, experts, offsets, rows, slots,
              reinterpret_cast<int32_t *>(ws), 0, 0};
  route_split(T, &a.blocks, &a.per_block);
  const dim3 grid(a.blocks), wg(RT_NT);
  const bool single = a.blocks == 1;
  const size_t row = (size_t)E * 4, all = row * (2 + RT_NT / 64), lds = single ? all : row;
  {
    LaunchTimer t(IMBD_K_ROUTE, 0, s);
#define GO(G_)                                                                       \
  do {                                                                               \
    if (single) hipLaunchKernelGGL((choose_kernel<G_, true>), grid, wg, lds, s, a);  \
    else hipLaunchKernelGGL((choose_kernel<G_, false>), grid, wg, lds, s, a);        \
  } while (0)
    if (E <= 64) GO(8);
    else if (E <= 128) GO(16);
    else if (E <= 256) GO(32);
    else GO(64);
#undef GO
  }
  const int rc = check_launch("expert_route");
  if (rc != IMBD_OK || single) return rc;
  {
    LaunchTimer t(IMBD_K_ROUTE, 1, s);
    hipLaunchKernelGGL(place_kernel, grid, wg, all, s, a);
  }
  return check_launch("expert_route (order)");
}

int run_route_bwd(int T, int E, int k, int renorm, const float *logits, int64_t ldl, const float *gates,
                  const int32_t *experts, const float *dgates, float *dlogits, int64_t lddl, hipStream_t s) {
  if (T == 0) return IMBD_OK;
  RouteBwdArgs a{T, E, k, renorm, logits, ldl, gates, dgates, experts, dlogits, lddl};
  const int G = E <= 64 ? 8 : E <= 128 ? 16 : E <= 256 ? 32 : 64, per = 256 / G;
  const int64_t blocks = ((int64_t)T + per - 1) / per;
  if (blocks > WORKGROUPS_MOST) {
    set_error("expert_route_bwd: T = %d tokens are more than one launch takes", T);
    return IMBD_EUNSUPPORTED;
  }
  const dim3 grid((unsigned)blocks), wg(256);
  {
    LaunchTimer t(IMBD_K_ROUTE, 2, s);
#define GO(G_)                                                                           \
  do {                                                                                   \
    if (k <= 8) hipLaunchKernelGGL((route_bwd_kernel<G_, 8>), grid, wg, 0, s, a);        \
    else hipLaunchKernelGGL((route_bwd_kernel<G_, CHOICE_MAX>), grid, wg, 0, s, a);      \
  } while (0)
    if (G == 8) GO(8);
    else if (G == 16) GO(16);
    else if (G == 32) GO(32);
    else GO(64);
#undef GO
  }
  return check_launch("expert_route_bwd");
}

}  // namespace imbd
