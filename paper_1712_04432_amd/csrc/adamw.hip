// AdamW over many tensors in one launch.
//   m <- beta1 m + (1 - beta1) g      v <- beta2 v + (1 - beta2) g^2      (g = grad_scale * grad)
//   w <- (1 - lr decay) w - rate * m / (sqrt(v) * root + eps)
//   rate = lr / (1 - beta1^t), root = 1 / sqrt(1 - beta2^t)
//
// A stream without reuse: 30 bytes an element with fp32 state, gradients and a bf16 copy, 16 with 8-bit
// state and bf16 gradients. The plan in device memory is a record for each tensor and, behind the records,
// a table of chunks of AW_CHUNK elements of one tensor each; a workgroup takes a chunk, so one launch
// serves tensors of every size, and the chunk's loads are all in flight before the first is used. 300 tensors, 120M
// elements: 620 us with fp32 state (5.8 TB/s), 365 to 378 with 8-bit state and bf16 gradients (5.1 to 5.3 TB/s).
//
// Every product and sum is rounded by itself (no contraction into fused multiply-adds), so the states are
// the same bits wherever the formulas are evaluated in fp32 in the order written; 8-bit codes then never
// differ by a rounding of the value that they are taken from.
//
// 8-bit state: a wave takes 256 elements, four a lane, which share a scale, so the block's maximum is one
// exchange over the wave. Maxima are taken of the bit patterns of |m| and v as whole numbers: the same order
// for finite values, and a NaN wins.

#include "adamw.h"
#include "cdna4.h"

#pragma clang fp contract(off)

namespace imbd {
namespace {

constexpr int AW_CHUNK = 4096;  // elements
constexpr int AW_NT = 256;
constexpr int AW_BLOCK = 256;   // elements that share a scale

struct AwTensor {
  float *w;
  uint16_t *w_lp;
  const void *grad;
  void *m, *v;
  float *m_scale, *v_scale;
  int64_t n;
  float decay;
  int32_t flags;
};
enum { AW_GRAD_BF16 = 1, AW_STATE8 = 2, AW_VECTOR = 4, AW_STREAM = 8 };
struct AwEntry {
  uint32_t tensor, chunk;
};
static_assert(sizeof(AwTensor) % 8 == 0 && sizeof(AwEntry) == 8, "plan layout");

struct AwArgs {
  const AwTensor *tensors;
  const AwEntry *table;
  double lr, beta1, beta2;
  float b1, c1, b2, c2, eps, grad_scale;
  int step;
  const int32_t *step_dev;
};

// b^t by squaring, in 64 bits, the same on host and device.
__host__ __device__ inline double power(double b, int t) {
  double r = 1.0;
  for (; t > 0; t >>= 1) {
    if (t & 1) r = r * b;
    b = b * b;
  }
  return r;
}

__device__ __forceinline__ float wave_max_bits(uint32_t u) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) u = max(u, (uint32_t)__shfl_xor((int)u, o, 64));
  return __builtin_bit_cast(float, u);
}

// 21 pseudo-random bits of an element's index and the step: two rounds of multiply and xor-shift. The two multipliers and
// the shifts are those that C. Wellons published in 2018 ("Prospecting for Hash Functions") for a mixing of 32 bits with
// little bias, found by search; the step enters by the golden ratio's 2^32 / 1.618..
__device__ __forceinline__ uint32_t dither21(uint32_t index, uint32_t step) {
  uint32_t h = index + step * 0x9E3779B9u;
  h = (h ^ (h >> 16)) * 0x7FEB352Du;
  h = (h ^ (h >> 15)) * 0x846CA68Bu;
  return (h ^ (h >> 16)) >> 11;
}

// e5m2 code of r = v / scale in [0, 57344]: the 21 bits that e5m2 drops, plus the dither, carry into the
// kept ones. Codes: fp32 bits >> 21 less the difference of the exponents' biases; 4 is the smallest normal
// number, 0x7B the largest.
__device__ __forceinline__ uint32_t code_e5m2(float r, uint32_t dither) {
  const int c = (int)((__builtin_bit_cast(uint32_t, r) + dither) >> 21) - 4 * 112;
  return (uint32_t)min(max(c, 4), 0x7B);
}
__device__ __forceinline__ float value_e5m2(uint32_t c) {  // (any code: an e5m2 is the upper half of an fp16)
  return (float)__builtin_bit_cast(_Float16, (uint16_t)(c << 8));
}

struct Step {
  float b1, c1, b2, c2, eps, gs, rate, root, keep;
  uint32_t t;
};

// One element; returns the new weight.
__device__ __forceinline__ float advance(const Step &st, float w, float g, float &m, float &v) {
  g = g * st.gs;
  const float m0 = m * st.b1, m1 = g * st.c1;
  m = m0 + m1;
  const float g2 = g * g, v0 = v * st.b2, v1 = g2 * st.c2;
  v = v0 + v1;
  const float den = sqrtf(v) * st.root;
  const float q = m / (den + st.eps);
  const float w0 = w * st.keep, d = q * st.rate;
  return w0 - d;
}

// Four elements of one tensor: n of them real, one by one; whole vectors; whole vectors past the caches.
enum { AW_ONES = 0, AW_WHOLE = 1, AW_PAST = 2 };
template <int HOW, typename T>
__device__ __forceinline__ void load4(const T *p, int n, T (&v)[4]) {
  if constexpr (HOW == AW_ONES) {
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = e < n ? p[e] : T(0);
  } else {
    typedef T V __attribute__((ext_vector_type(4)));
    const V x = HOW == AW_PAST ? __builtin_nontemporal_load(reinterpret_cast<const V *>(p)) : *reinterpret_cast<const V *>(p);
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = x[e];
  }
}
template <int HOW, typename T>
__device__ __forceinline__ void store4(T *p, int n, const T (&v)[4]) {
  if constexpr (HOW == AW_ONES) {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (e < n) p[e] = v[e];
  } else {
    typedef T V __attribute__((ext_vector_type(4)));
    const V x = {v[0], v[1], v[2], v[3]};
    if constexpr (HOW == AW_PAST) __builtin_nontemporal_store(x, reinterpret_cast<V *>(p));
    else *reinterpret_cast<V *>(p) = x;
  }
}

// A chunk: wave `wave` takes blocks wave, wave + 4, .. of 256 elements. AW_ONES: element by element, with the
// tensor's end inside; else whole blocks at 16-byte aligned addresses.
template <int HOW, bool G16, bool S8>
__device__ __forceinline__ void chunk(const AwTensor &a, const Step &st, int64_t start) {
  constexpr int NB = AW_CHUNK / AW_BLOCK / (AW_NT / 64);  // blocks a wave
  constexpr bool VEC = HOW != AW_ONES;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  float w[NB][4], m[NB][4], v[NB][4], g[NB][4], ms[NB], vs[NB];
  int n[NB];
#pragma unroll
  for (int b = 0; b < NB; ++b) {
    const int64_t blk = start / AW_BLOCK + wave + b * (AW_NT / 64), i = blk * AW_BLOCK + 4 * lane;
    const int64_t left = a.n - i;
    n[b] = VEC ? 4 : (int)min((int64_t)4, max((int64_t)0, left));
    load4<HOW>(a.w + i, n[b], w[b]);
    if constexpr (G16) {
      uint16_t h[4];
      load4<HOW>(reinterpret_cast<const uint16_t *>(a.grad) + i, n[b], h);
#pragma unroll
      for (int e = 0; e < 4; ++e) g[b][e] = bf16_to_f32(h[e]);
    } else {
      load4<HOW>(reinterpret_cast<const float *>(a.grad) + i, n[b], g[b]);
    }
    if constexpr (S8) {
      uint8_t mc[4], vc[4];
      load4<HOW>(reinterpret_cast<const uint8_t *>(a.m) + i, n[b], mc);
      load4<HOW>(reinterpret_cast<const uint8_t *>(a.v) + i, n[b], vc);
      const bool real = VEC || blk * AW_BLOCK < a.n;
      ms[b] = real ? a.m_scale[blk] : 0.f;
      vs[b] = real ? a.v_scale[blk] : 0.f;
      uint32_t mq;
      __builtin_memcpy(&mq, mc, 4);
      m[b][0] = __builtin_amdgcn_cvt_f32_fp8(mq, 0);
      m[b][1] = __builtin_amdgcn_cvt_f32_fp8(mq, 1);
      m[b][2] = __builtin_amdgcn_cvt_f32_fp8(mq, 2);
      m[b][3] = __builtin_amdgcn_cvt_f32_fp8(mq, 3);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        m[b][e] = m[b][e] * ms[b];
        v[b][e] = value_e5m2(vc[e]) * vs[b];
      }
    } else {
      load4<HOW>(reinterpret_cast<const float *>(a.m) + i, n[b], m[b]);
      load4<HOW>(reinterpret_cast<const float *>(a.v) + i, n[b], v[b]);
    }
  }
#pragma unroll
  for (int b = 0; b < NB; ++b) {
    const int64_t blk = start / AW_BLOCK + wave + b * (AW_NT / 64), i = blk * AW_BLOCK + 4 * lane;
    if (!VEC && blk * AW_BLOCK >= a.n) continue;  // (the whole wave)
#pragma unroll
    for (int e = 0; e < 4; ++e) w[b][e] = advance(st, w[b][e], g[b][e], m[b][e], v[b][e]);
    store4<HOW>(a.w + i, n[b], w[b]);
    if (a.w_lp) {
      const uint32_t lo = cvt_pk_bf16(w[b][0], w[b][1]), hi = cvt_pk_bf16(w[b][2], w[b][3]);
      const uint16_t h[4] = {(uint16_t)lo, (uint16_t)(lo >> 16), (uint16_t)hi, (uint16_t)(hi >> 16)};
      store4<HOW>(a.w_lp + i, n[b], h);
    }
    if constexpr (S8) {
      // (elements past the tensor's end are zero: they do not raise a maximum)
      uint32_t mb = 0, vb = 0;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        mb = max(mb, __builtin_bit_cast(uint32_t, m[b][e]) & 0x7fffffffu);
        vb = max(vb, __builtin_bit_cast(uint32_t, v[b][e]) & 0x7fffffffu);
      }
      const float msn = wave_max_bits(mb) * (1.0f / 448.0f), vsn = wave_max_bits(vb) * (1.0f / 57344.0f);
      if (lane == 0) {
        a.m_scale[blk] = msn;
        a.v_scale[blk] = vsn;
      }
      float q[4];
      uint8_t vc[4], mc[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        q[e] = msn != 0.f ? m[b][e] / msn : 0.f;
        vc[e] = v[b][e] != 0.f && vsn != 0.f
                    ? (uint8_t)code_e5m2(v[b][e] / vsn, dither21((uint32_t)(i + e), st.t))
                    : (uint8_t)0;
      }
      // A scale among the denormals is rounded by up to a third: past 464 the code would be a NaN's (a NaN stays one).
      // (A branch of the whole wave: 120M elements 365 us; the same for every scale 374, without it 364.)
      if (msn < 0x1p-126f) {
#pragma unroll
        for (int e = 0; e < 4; ++e) q[e] = q[e] > 448.f ? 448.f : q[e] < -448.f ? -448.f : q[e];
      }
      uint32_t mq = __builtin_amdgcn_cvt_pk_fp8_f32(q[0], q[1], 0, false);
      mq = __builtin_amdgcn_cvt_pk_fp8_f32(q[2], q[3], mq, true);
      __builtin_memcpy(mc, &mq, 4);
      store4<HOW>(reinterpret_cast<uint8_t *>(a.m) + i, n[b], mc);
      store4<HOW>(reinterpret_cast<uint8_t *>(a.v) + i, n[b], vc);
    } else {
      store4<HOW>(reinterpret_cast<float *>(a.m) + i, n[b], m[b]);
      store4<HOW>(reinterpret_cast<float *>(a.v) + i, n[b], v[b]);
    }
  }
}

__global__ void __launch_bounds__(AW_NT) adamw_kernel(AwArgs a) {
  const AwEntry en = a.table[blockIdx.x];
  const AwTensor t = a.tensors[en.tensor];
  const int step = a.step_dev ? *a.step_dev : a.step;
  Step st;
  st.b1 = a.b1;
  st.c1 = a.c1;
  st.b2 = a.b2;
  st.c2 = a.c2;
  st.eps = a.eps;
  st.gs = a.grad_scale;
  st.rate = (float)(a.lr / (1.0 - power(a.beta1, step)));
  st.root = (float)(1.0 / __builtin_sqrt(1.0 - power(a.beta2, step)));
  st.keep = (float)(1.0 - a.lr * (double)t.decay);
  st.t = (uint32_t)step;
  const int64_t start = (int64_t)en.chunk * AW_CHUNK;
  const bool whole = (t.flags & AW_VECTOR) && start + AW_CHUNK <= t.n;
  const int how = !whole ? AW_ONES : (t.flags & AW_STREAM) ? AW_PAST : AW_WHOLE;
  switch (how * 4 + (t.flags & (AW_GRAD_BF16 | AW_STATE8))) {
    case 0: chunk<AW_ONES, false, false>(t, st, start); break;
    case 1: chunk<AW_ONES, true, false>(t, st, start); break;
    case 2: chunk<AW_ONES, false, true>(t, st, start); break;
    case 3: chunk<AW_ONES, true, true>(t, st, start); break;
    case 4: chunk<AW_WHOLE, false, false>(t, st, start); break;
    case 5: chunk<AW_WHOLE, true, false>(t, st, start); break;
    case 6: chunk<AW_WHOLE, false, true>(t, st, start); break;
    case 7: chunk<AW_WHOLE, true, true>(t, st, start); break;
    case 8: chunk<AW_PAST, false, false>(t, st, start); break;
    case 9: chunk<AW_PAST, true, false>(t, st, start); break;
    case 10: chunk<AW_PAST, false, true>(t, st, start); break;
    default: chunk<AW_PAST, true, true>(t, st, start); break;
  }
}

}  // namespace

int64_t adamw_chunks(int64_t n) { return n / AW_CHUNK + (n % AW_CHUNK != 0); }
size_t adamw_record_bytes() { return sizeof(AwTensor); }
size_t adamw_entry_bytes() { return sizeof(AwEntry); }

void adamw_write_plan(const imbd_adamw_tensor *tensors, int n_tensors, void *plan) {
  // The set's footprint, each array once. While much of it is still in the 256 MB of the memory-side cache a step later
  // it stays in the caches, then the loads and stores go past them. A step in us, in the caches and past them: fp32 state
  // and gradients with a copy, 256 MiB 68 and 75, 320 MiB 86 and 92, 384 MiB 126 and 111, 512 MiB 169 and 148, 1 GiB 328
  // and 298; 8-bit state, bf16 gradients, 256 MiB 85 and 84, 320 MiB 107 and 108, 384 MiB 130 and 125, 1 GiB 342 and 325.
  int64_t bytes = 0;
  for (int i = 0; i < n_tensors; ++i)
    bytes += tensors[i].n * (4 + (tensors[i].w_lp ? 2 : 0) + (tensors[i].grad_dtype == IMBD_BF16 ? 2 : 4) +
                             (tensors[i].state_bits == 8 ? 2 : 8));
  const bool stream = bytes > (int64_t)336 << 20;
  AwTensor *rec = reinterpret_cast<AwTensor *>(plan);
  AwEntry *en = reinterpret_cast<AwEntry *>(rec + n_tensors);
  for (int i = 0; i < n_tensors; ++i) {
    const imbd_adamw_tensor &t = tensors[i];
    auto al = [](const void *p, uintptr_t to) { return (uintptr_t)p % to == 0; };
    const bool g16 = t.grad_dtype == IMBD_BF16, s8 = t.state_bits == 8;
    const uintptr_t sa = s8 ? 4 : 16;
    const bool vec = al(t.w, 16) && al(t.w_lp, 8) && al(t.grad, g16 ? 8 : 16) && al(t.m, sa) && al(t.v, sa);
    rec[i] = AwTensor{t.w, t.w_lp, t.grad, t.m, t.v, t.m_scale, t.v_scale, t.n, t.decay,
                      (g16 ? AW_GRAD_BF16 : 0) | (s8 ? AW_STATE8 : 0) | (vec ? AW_VECTOR : 0) | (stream ? AW_STREAM : 0)};
    const int64_t c = adamw_chunks(t.n);
    for (int64_t j = 0; j < c; ++j) *en++ = AwEntry{(uint32_t)i, (uint32_t)j};
  }
}

int run_adamw(const void *plan, int n_tensors, int64_t chunks, double lr, double beta1, double beta2, double eps,
              float grad_scale, int step, const int32_t *step_dev, hipStream_t s) {
  AwArgs a;
  a.tensors = reinterpret_cast<const AwTensor *>(plan);
  a.table = reinterpret_cast<const AwEntry *>(a.tensors + n_tensors);
  a.lr = lr;
  a.beta1 = beta1;
  a.beta2 = beta2;
  a.b1 = (float)beta1;
  a.c1 = (float)(1.0 - beta1);
  a.b2 = (float)beta2;
  a.c2 = (float)(1.0 - beta2);
  a.eps = (float)eps;
  a.grad_scale = grad_scale;
  a.step = step;
  a.step_dev = step_dev;
  {
    LaunchTimer t(IMBD_K_ADAMW, 0, s);
    hipLaunchKernelGGL(adamw_kernel, dim3((unsigned)chunks), dim3(AW_NT), 0, s, a);
  }
  return check_launch("adamw");
}

}  // namespace imbd
