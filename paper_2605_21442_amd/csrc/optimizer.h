// AdamW over many tensors (moments in 32 or 8 bits) and the norm of many gradients. Included by lce.hip,
// behind its launcher. A launch serves dozens of tensors, whose addresses travel in its arguments: nothing
// is copied to the device beforehand, so a call can be captured and its table needs no storage.
//
// On a whole model (1.24e9 bf16 elements, kernels alone under the tracer) the 32-bit step with an fp32 master copy
// moves 28 bytes an element in 5.7 ms (6.1 TB/s), the values of the 8-bit moments 6.1 bytes in 1.2 ms (6.2) and the
// norm 2 bytes in 0.40 ms (6.1): bound by memory. The 8-bit step without master copy moves 10.1 bytes in 2.4 ms (5.3
// TB/s), of which its 66 vector instructions an element alone would take 2.1. Hundreds of small tensors are bound by
// the launches' ramps (224 adapter tensors, 11.3e6 elements: 64 us in 3 launches, 4.9 TB/s; in 5 launches 74) and, in
// the norm, by the host (9 us of kernels and 18 a call).
#pragma once

namespace {

typedef float f32x4_t __attribute__((ext_vector_type(4)));

constexpr int kTableGroups = 8;
constexpr int kMomentBlock = 32;       // elements that share the units of the 8-bit moments
constexpr int64_t kEntryElems = (int64_t)1 << 30;      // a larger tensor takes several entries

template <int kBits> struct AdamWEntry;
template <> struct AdamWEntry<32> {
  void* param;
  const void* grad;
  void* m;
  void* v;
  float* master;
  uint32_t n;
  uint32_t first : 24;     // first workgroup of this entry
  uint32_t group : 3, param_f32 : 1, grad_f32 : 1;
  uint32_t wide : 3;       // bits: param, grad, master lie at a multiple of 16 bytes
};
template <> struct AdamWEntry<8> : AdamWEntry<32> {
  uint8_t* units;
  uint32_t pair0;          // place / 2
  uint32_t pad_;
};

// 77 tensors a launch with 32-bit moments, 58 with 8-bit ones, and the groups' constants
template <int kBits>
struct AdamWTable {
  static constexpr int kTensors = kBits == 32 ? 77 : 58;
  AdamWEntry<kBits> e[kTensors];
  AdamWConst g[kTableGroups];
  int count;
  int per;                 // elements of a workgroup, whole rounds
};
static_assert(sizeof(AdamWTable<32>) <= 4000 && sizeof(AdamWTable<8>) <= 4000, "launch arguments");

// The entry of workgroup `block`: the last one whose first workgroup is not behind it, found by all lanes at once.
template <typename Entry>
__device__ __forceinline__ int table_entry(const Entry* e, int count, uint32_t block) {
  int k = -1;
  for (int i = 0; i < count; i += 64) {
    const int j = i + (threadIdx.x & 63);
    k += __popcll(__ballot(j < count && e[min(j, count - 1)].first <= block));
  }
  return __builtin_amdgcn_readfirstlane(k);
}

__device__ __forceinline__ float load_elem(const void* p, int64_t i, bool f32) {
  return f32 ? ((const float*)p)[i] : bf16_to_f32(((const uint16_t*)p)[i]);
}

// N consecutive elements from i on as fp32, and back; elements at or past n are 0 and are not touched. `wide`: the
// tensor's address is a multiple of 16 bytes (i is a multiple of N). Both pass the L2 by: a step touches every byte
// once (1.2e9 elements, 32-bit moments, 8192 a workgroup: 6.72 -> 6.57 ms; adapters 117 -> 107 us).
template <int N>
__device__ __forceinline__ void load_elems(const void* p, int64_t i, int64_t n, bool f32, bool wide, float x[N]) {
  if (wide && i + N <= n) {
    if (f32) {
#pragma unroll
      for (int h = 0; h < N / 4; ++h) {
        const f32x4_t a = __builtin_nontemporal_load(reinterpret_cast<const f32x4_t*>((const float*)p + i + 4 * h));
#pragma unroll
        for (int k = 0; k < 4; ++k) x[4 * h + k] = a[k];
      }
    } else {
      typedef uint32_t Words __attribute__((ext_vector_type(N / 2)));
      const Words a = __builtin_nontemporal_load(reinterpret_cast<const Words*>((const uint16_t*)p + i));
#pragma unroll
      for (int h = 0; h < N / 2; ++h) {
        x[2 * h] = __uint_as_float(a[h] << 16);
        x[2 * h + 1] = __uint_as_float(a[h] & 0xFFFF0000u);
      }
    }
    return;
  }
#pragma unroll
  for (int k = 0; k < N; ++k) x[k] = i + k >= n ? 0.f : load_elem(p, i + k, f32);
}

template <int N>
__device__ __forceinline__ void store_elems(void* p, int64_t i, int64_t n, bool f32, bool wide, const float x[N]) {
  if (wide && i + N <= n) {
    if (f32) {
#pragma unroll
      for (int h = 0; h < N / 4; ++h)
        store16_padded_nt((float*)p + i + 4 * h,
                          i32x4_t{(int)__float_as_uint(x[4 * h]), (int)__float_as_uint(x[4 * h + 1]),
                                  (int)__float_as_uint(x[4 * h + 2]), (int)__float_as_uint(x[4 * h + 3])});
    } else if (N == 8) {
      store16_padded_nt((uint16_t*)p + i, i32x4_t{(int)pack_bf16x2(x[0], x[1]), (int)pack_bf16x2(x[2], x[3]),
                                               (int)pack_bf16x2(x[N - 4], x[N - 3]), (int)pack_bf16x2(x[N - 2], x[N - 1])});
    } else {
      __builtin_nontemporal_store(u32x2_t{pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3])},
                                  reinterpret_cast<u32x2_t*>((uint16_t*)p + i));
    }
    return;
  }
#pragma unroll
  for (int k = 0; k < N; ++k) {
    if (i + k >= n) break;
    if (f32) ((float*)p)[i + k] = x[k];
    else ((uint16_t*)p)[i + k] = to_bf16(x[k]);
  }
}

// ---------------------------------------------------------------------------------------------
// 8-bit moments (the form is in lce.h). kMant 3: sign and 7 bits; kMant 4: 8 bits, no sign.
//
// A code shifted to the top of an fp32 mantissa, its upper 4 bits in the exponent field, is an fp32 number: the
// code's q times 2^-(126 + kMant), subnormal where the code is below 2^kMant. So decoding is a shift and an exact
// scaling, and rounding stochastically is adding random bits below the code and cutting them off.
// ---------------------------------------------------------------------------------------------
// unit byte of a block from the bits of its largest magnitude (as an unsigned number, which orders
// magnitudes, and infinities and NaN above them)
template <int kMant>
__device__ __forceinline__ int unit_byte(uint32_t top) {
  const int s = (int)((top + (1u << (23 - kMant))) >> 23) - 14 - kMant;
  return top >= 0x7F800000u ? 255 : s < 1 ? 1 : s;
}

// exponent that takes a code's fp32 number to its value in units of 2^(s - 127)
template <int kMant>
__device__ __forceinline__ int code_exponent(int s) { return s - 1 + kMant; }

// x in the codes' fp32 form plus 16 random bits below the code
template <int kMant>
__device__ __forceinline__ uint32_t dithered(float x, int s, uint32_t bits) {
  return __float_as_uint(ldexpf(x, -code_exponent<kMant>(s))) + (bits << (7 - kMant));
}

// byte 3 of each of four words, as one word
__device__ __forceinline__ uint32_t top_bytes(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  return __builtin_amdgcn_perm(__builtin_amdgcn_perm(d, c, 0x0C0C0703u), __builtin_amdgcn_perm(b, a, 0x0C0C0703u),
                               0x05040100u);
}

// 16 random bits for each of two neighbouring elements: a multiplicative hash (Knuth, TAOCP 6.4) of the
// pair's number and the seed, twice with the upper bits folded down; the odd factors are the leading
// bits of 1/phi, sqrt 2 and sqrt 3
__device__ __forceinline__ uint32_t pair_bits(uint32_t pair, uint32_t seed) {
  uint32_t x = pair * 0x9E3779B9u + seed;
  x = (x ^ (x >> 16)) * 0x6A09E667u;
  x = (x ^ (x >> 15)) * 0xBB67AE85u;
  return x ^ (x >> 16);
}

// the largest of four neighbouring lanes
__device__ __forceinline__ uint32_t quad_max(uint32_t x) {
  x = max(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0xB1, 0xF, 0xF, true));   // lanes 1 0 3 2
  return max(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0x4E, 0xF, 0xF, true));   // lanes 2 3 0 1
}

// What a byte of the first moment (a sign and a 7-bit code) and one of the root stand for. A block of NaN has its
// codes' exponent bits all set.
__device__ __forceinline__ float decode_first(uint32_t byte, int sm) {
  const int c = (int)(byte << 24) >> 4;           // sign, copies of it, code
  return ldexpf(__uint_as_float(((uint32_t)c & 0x87F00000u) | (sm == 255 ? 0x7FC00000u : 0u)), code_exponent<3>(sm));
}
__device__ __forceinline__ float decode_root(uint32_t byte, int sr) {
  return ldexpf(__uint_as_float(byte << 19 | (sr == 255 ? 0x7FC00000u : 0u)), code_exponent<4>(sr));
}

// 8 elements' moments from their bytes
__device__ __forceinline__ void decode_moments(const uint2 cm, const uint2 cr, int sm, int sr, float m[8], float r[8]) {
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    const uint32_t wm = k < 4 ? cm.x : cm.y, wr = k < 4 ? cr.x : cr.y;
    m[k] = decode_first(wm >> (8 * (k & 3)), sm);
    r[k] = decode_root(wr >> (8 * (k & 3)) & 255u, sr);
  }
}

// The parameter's update of 8-bit states from the new moments: adamw_update's, but for the root and the quotient.
// Each is the hardware's estimate (1 ulp) with one Newton step, which is the correctly rounded value but for a few in
// a million. The compiler's own sequences, which are right for every operand, made the 8-bit step bound by the vector
// units (91 instructions an element; 3.04 ms for 1.2e9 where this form took 2.55). The short form is for v = 0 or
// normal, eps within 2^+-100 and |m| < 2^27, so that no estimate, product or quotient leaves the normal numbers (but
// a quotient too small to matter). Returns the root.
__device__ __forceinline__ float adamw_step_near(float& p, float m, float v, const AdamWConst& c) {
#pragma clang fp contract(off)
  p = p * c.keep;
  const float y = __builtin_amdgcn_rsqf(fmaxf(v, 0x1p-126f)), root0 = v * y;
  const float root = fmaf(fmaf(-root0, root0, v), 0.5f * y, root0);
  const float denom = root * c.inv_sqrt_bc2 + c.eps;
  const float z = __builtin_amdgcn_rcpf(denom), q = m * z;
  p = p - c.step_size * fmaf(fmaf(-denom, q, m), z, q);
  return root;
}

// The same for all other operands, bit for bit adamw_update's parameter: a v that overflows gives no update. The root
// that is held is then formed from scaled terms, so that gradients that are finite leave moments that are (those in
// the last 1/16 and 1/32 below 2^128, whose code could round to infinity, are held as the largest code there; and
// beta2 = 0 takes nothing of an r whose square overflows). It starts from the element's values in memory: kept in
// registers until here, the kernel had 81 to 103 of them instead of 61, and every step took 3 % longer. A tensor of
// such operands alone takes 2.2 times as long.
__device__ __forceinline__ void adamw_element_far(const AdamWEntry<8>& e, const AdamWConst& c, int64_t i, float scale,
                                                  bool scaled, int s, float& p, float& m, float& r) {
#pragma clang fp contract(off)
  const float old = decode_root(((const uint8_t*)e.v)[i], s >> 8);
  float g = e.grad ? load_elem(e.grad, i, e.grad_f32) : 0.f;
  if (scaled) g = g * scale;
  m = c.beta1 * decode_first(((const uint8_t*)e.m)[i], s & 255) + c.omb1 * g;
  float v = c.beta2 * (old * old) + c.omb2 * (g * g);
  if (v != v && old < INFINITY) v = c.omb2 * (g * g);
  r = sqrtf(v);
  p = (e.master ? e.master[i] : load_elem(e.param, i, e.param_f32)) * c.keep;
  p = p - c.step_size * (m / (r * c.inv_sqrt_bc2 + c.eps));
  if (v == INFINITY) {
    const float a = old * 0x1p-65f, b = g * 0x1p-65f;
    r = sqrtf(c.beta2 * (a * a) + c.omb2 * (b * b)) * 0x1p65f;
    if (r < INFINITY) r = fminf(r, 0x1.Fp127f);
  }
  if (fabsf(m) < INFINITY) m = fminf(fmaxf(m, -0x1.Ep127f), 0x1.Ep127f);
}

// 32-bit moments: 4 elements per thread and round, so that every access of a wave is contiguous.
__device__ __forceinline__ void adamw_round32(const AdamWEntry<32>& e, const AdamWConst& c, int64_t i, float scale,
                                              bool scaled) {
#pragma clang fp contract(off)
  float p[4], g[4] = {}, m[4], v[4];
  load_elems<4>(e.m, i, e.n, true, true, m);
  load_elems<4>(e.v, i, e.n, true, true, v);
  if (e.master) load_elems<4>(e.master, i, e.n, true, e.wide & 4, p);
  else load_elems<4>(e.param, i, e.n, e.param_f32, e.wide & 1, p);
  if (e.grad) load_elems<4>(e.grad, i, e.n, e.grad_f32, e.wide & 2, g);
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    if (scaled) g[k] = g[k] * scale;
    adamw_update(p[k], m[k], v[k], g[k], c);
  }
  store_elems<4>(e.m, i, e.n, true, true, m);
  store_elems<4>(e.v, i, e.n, true, true, v);
  if (e.master) store_elems<4>(e.master, i, e.n, true, e.wide & 4, p);
  store_elems<4>(e.param, i, e.n, e.param_f32, e.wide & 1, p);
}

// 8-bit moments: 8 elements per thread and round, four lanes to a block. Every lane of a wave comes here (the
// blocks' maxima pass between lanes); those at or past n hold zeros.
__device__ __forceinline__ void adamw_round8(const AdamWEntry<8>& e, const AdamWConst& c, int64_t i, float scale,
                                             bool scaled, uint32_t seed) {
#pragma clang fp contract(off)
  float p[8] = {}, g[8] = {}, m[8] = {}, r[8] = {};
  uint8_t* units = e.units + 2 * (i / kMomentBlock);
  uint2 cm = make_uint2(0, 0), cr = cm;
  int s = 0;
  const bool whole = i + 8 <= e.n;
  if (i < e.n) {
    s = *reinterpret_cast<const uint16_t*>(units);
    if (whole) {
      cm = *reinterpret_cast<const uint2*>((const uint8_t*)e.m + i);
      cr = *reinterpret_cast<const uint2*>((const uint8_t*)e.v + i);
    } else {
      for (int k = 0; k < (int)(e.n - i); ++k) {
        const uint32_t a = ((const uint8_t*)e.m)[i + k], b = ((const uint8_t*)e.v)[i + k];
        if (k < 4) { cm.x |= a << 8 * k; cr.x |= b << 8 * k; }
        else { cm.y |= a << 8 * (k - 4); cr.y |= b << 8 * (k - 4); }
      }
    }
    if (e.master) load_elems<8>(e.master, i, e.n, true, e.wide & 4, p);
    else load_elems<8>(e.param, i, e.n, e.param_f32, e.wide & 1, p);
    if (e.grad) load_elems<8>(e.grad, i, e.n, e.grad_f32, e.wide & 2, g);
    decode_moments(cm, cr, s & 255, s >> 8, m, r);
  }
  uint32_t am = 0, ar = 0;          // (elements at or past n have zero moments and gradients)
  bool far = !(c.eps >= 0x1p-100f && c.eps <= 0x1p100f);
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    if (scaled) g[k] = g[k] * scale;
    m[k] = c.beta1 * m[k] + c.omb1 * g[k];
    const float v = c.beta2 * (r[k] * r[k]) + c.omb2 * (g[k] * g[k]);
    far |= __builtin_amdgcn_classf(v, 0x283);          // positive and subnormal, infinite or NaN
    r[k] = adamw_step_near(p[k], m[k], v, c);
    am = max(am, __float_as_uint(m[k]) & 0x7FFFFFFFu);
    ar = max(ar, __float_as_uint(r[k]) & 0x7FFFFFFFu);
  }
  far |= am >= 0x4D000000u;                            // 2^27
  if (far) {
    am = ar = 0;
    // (the address is hidden from the compiler, which would keep one of each array in registers)
#pragma unroll 1
    for (int n = 0; n < 8 && i + n < e.n; ++n) {
      float p0, m0, r0;
      int64_t at = i + n;
      asm volatile("" : "+v"(at));
      adamw_element_far(e, c, at, scale, scaled, s, p0, m0, r0);
      am = max(am, __float_as_uint(m0) & 0x7FFFFFFFu);
      ar = max(ar, __float_as_uint(r0) & 0x7FFFFFFFu);
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        p[k] = k == n ? p0 : p[k];
        m[k] = k == n ? m0 : m[k];
        r[k] = k == n ? r0 : r[k];
      }
    }
  }
  const int sm = unit_byte<3>(quad_max(am)), sr = unit_byte<4>(quad_max(ar));
  if (i >= e.n) return;
  uint32_t bm[8], br[8];            // the codes in the top bytes
#pragma unroll
  for (int k = 0; k < 8; k += 2) {
    const uint32_t h = pair_bits(e.pair0 + (uint32_t)(i >> 1) + k / 2, seed);
#pragma unroll
    for (int j = k; j < k + 2; ++j) {
      const uint32_t bits = j & 1 ? h >> 16 : h & 0xFFFFu;
      const uint32_t x = dithered<3>(m[j], sm, bits);
      bm[j] = (x << 4 & 0x7FFFFFFFu) | (x & 0x80000000u);
      // a root above 0 takes at least the smallest code
      br[j] = max(dithered<4>(r[j], sr, bits), min(__float_as_uint(r[j]), 1u << 19)) << 5;
    }
  }
  if (whole) {
    *reinterpret_cast<uint2*>((uint8_t*)e.m + i) =
        make_uint2(top_bytes(bm[0], bm[1], bm[2], bm[3]), top_bytes(bm[4], bm[5], bm[6], bm[7]));
    *reinterpret_cast<uint2*>((uint8_t*)e.v + i) =
        make_uint2(top_bytes(br[0], br[1], br[2], br[3]), top_bytes(br[4], br[5], br[6], br[7]));
  } else {
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      if (i + k >= e.n) break;
      ((uint8_t*)e.m)[i + k] = (uint8_t)(bm[k] >> 24);
      ((uint8_t*)e.v)[i + k] = (uint8_t)(br[k] >> 24);
    }
  }
  if (i % kMomentBlock == 0) *reinterpret_cast<uint16_t*>(units) = (uint16_t)(sm | sr << 8);
  if (e.master) store_elems<8>(e.master, i, e.n, true, e.wide & 4, p);
  store_elems<8>(e.param, i, e.n, e.param_f32, e.wide & 1, p);
}

template <int kBits>
__global__ __launch_bounds__(256) void k_adamw_tensors(AdamWTable<kBits> t, const float* __restrict__ grad_scale,
                                                       uint32_t seed) {
  const float scale = grad_scale ? *grad_scale : 1.0f;
  if (!(fabsf(scale) < INFINITY)) return;
  const AdamWEntry<kBits> e = t.e[table_entry(t.e, t.count, blockIdx.x)];
  const AdamWConst c = t.g[e.group];
  constexpr int kPer = kBits == 32 ? 4 : 8;
  const int64_t i0 = (int64_t)(blockIdx.x - e.first) * t.per;
  for (int j = 0; j < t.per && i0 + j < e.n; j += 256 * kPer) {
    const int64_t i = i0 + j + kPer * threadIdx.x;
    if constexpr (kBits == 32) {
      if (i < e.n) adamw_round32(e, c, i, scale, grad_scale != nullptr);
    } else {
      adamw_round8(e, c, i, scale, grad_scale != nullptr, seed);
    }
  }
}

// 8 elements per thread
__global__ __launch_bounds__(256) void k_adamw_moments(int64_t n, const uint8_t* __restrict__ m, const uint8_t* __restrict__ r,
                                                       const uint8_t* __restrict__ units, uint16_t* __restrict__ first,
                                                       uint16_t* __restrict__ root) {
  const int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 8;
  if (i >= n) return;
  const int s = *reinterpret_cast<const uint16_t*>(units + 2 * (i / kMomentBlock));
  float x[8], y[8];
  uint2 cm = make_uint2(0, 0), cr = cm;
  if (i + 8 <= n) {
    cm = *reinterpret_cast<const uint2*>(m + i);
    cr = *reinterpret_cast<const uint2*>(r + i);
  } else {
    for (int k = 0; k < (int)(n - i); ++k) {
      if (k < 4) { cm.x |= (uint32_t)m[i + k] << 8 * k; cr.x |= (uint32_t)r[i + k] << 8 * k; }
      else { cm.y |= (uint32_t)m[i + k] << 8 * (k - 4); cr.y |= (uint32_t)r[i + k] << 8 * (k - 4); }
    }
  }
  decode_moments(cm, cr, s & 255, s >> 8, x, y);
  store_elems<8>(first, i, n, false, true, x);
  store_elems<8>(root, i, n, false, true, y);
}

// ---------------------------------------------------------------------------------------------
// Norm of many gradients: every workgroup leaves the fp64 sum of the squares of its elements, and one
// workgroup adds these in order. fp64: an fp32 square overflows from 1.8e19 on, which bf16 holds, and a
// model's 1e9 squares lose digits in fp32.
// ---------------------------------------------------------------------------------------------
struct NormEntry {        // of a tensor, or of 2^30 elements of a larger one
  const void* data;
  uint32_t n;
  uint32_t first : 31, f32 : 1;
};
constexpr int64_t kNormEntryElems = (int64_t)1 << 30;
constexpr int kNormTensors = 248;
struct NormTable {
  NormEntry e[kNormTensors];
  int count;
};
static_assert(sizeof(NormTable) <= 4000, "launch arguments");

template <int kThreads>
__device__ __forceinline__ double block_sum_f64(double x) {
  __shared__ double part[kThreads / 64];
  for (int m = 32; m >= 1; m >>= 1) x += __shfl_xor(x, m);
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = x;
  __syncthreads();
  x = part[0];
  for (int k = 1; k < kThreads / 64; ++k) x += part[k];
  return x;
}

__device__ __forceinline__ double squares(const uint4 a, bool f32) {
  const uint32_t w[4] = {a.x, a.y, a.z, a.w};
  double lo = 0, hi = 0;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    if (f32) {
      const double x = __uint_as_float(w[k]);
      lo = fma(x, x, lo);
    } else {
      const double x = __uint_as_float(w[k] << 16), y = __uint_as_float(w[k] & 0xFFFF0000u);
      lo = fma(x, x, lo);
      hi = fma(y, y, hi);
    }
  }
  return lo + hi;
}

// A workgroup takes `bytes` bytes of a tensor in 16-byte pieces, eight in flight per thread; the tensor's elements
// before the first multiple of 16 bytes and behind the last are added one by one by its first workgroup.
__global__ __launch_bounds__(256) void k_grad_squares(NormTable t, int64_t bytes, double* __restrict__ parts) {
  constexpr int kAhead = 8;
  const NormEntry e = t.e[table_entry(t.e, t.count, blockIdx.x)];
  const int size = e.f32 ? 4 : 2;
  const int64_t n = e.n, head = min(n, (int64_t)((16 - ((uintptr_t)e.data & 15)) & 15) / size);
  const int64_t pieces = (n - head) * size / 16;
  const uint4* p = reinterpret_cast<const uint4*>((const char*)e.data + head * size);
  const int64_t q0 = (int64_t)(blockIdx.x - e.first) * (bytes / 16), q1 = min(pieces, q0 + bytes / 16);
  double sum = 0;
  for (int64_t q = q0 + threadIdx.x; q < q1; q += 256 * kAhead) {
    uint4 a[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) a[k] = q + 256 * k < q1 ? p[q + 256 * k] : make_uint4(0, 0, 0, 0);
#pragma unroll
    for (int k = 0; k < kAhead; ++k) sum += squares(a[k], e.f32);
  }
  if (blockIdx.x == e.first) {
    const int64_t tail = head + pieces * 16 / size;
    const int64_t i = threadIdx.x < 8 ? threadIdx.x : tail + threadIdx.x - 8;     // at most 7 on either side
    if (threadIdx.x < 8 ? i < head : threadIdx.x < 16 && i < n) {
      const double x = e.f32 ? ((const float*)e.data)[i] : bf16_to_f32(((const uint16_t*)e.data)[i]);
      sum += x * x;
    }
  }
  sum = block_sum_f64<256>(sum);
  if (threadIdx.x == 0) parts[blockIdx.x] = sum;
}

__global__ __launch_bounds__(1024) void k_grad_norm(const double* __restrict__ parts, int64_t count, float max_norm,
                                                    float* norm, float* factor) {
  double sum = 0;
  for (int64_t i = threadIdx.x; i < count; i += 1024 * 8) {
    double x[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) x[k] = i + 1024 * k < count ? parts[i + 1024 * k] : 0.0;
#pragma unroll
    for (int k = 0; k < 8; ++k) sum += x[k];
  }
  sum = block_sum_f64<1024>(sum);
  if (threadIdx.x != 0) return;
  const double x = sqrt(sum), f = (double)max_norm / (x + 1e-6);
  *norm = (float)x;
  if (factor) *factor = !((float)x < INFINITY) ? __uint_as_float(0x7FC00000u) : f < 1.0 ? (float)f : 1.0f;
}

// ---------------------------------------------------------------------------------------------
// Host side
// ---------------------------------------------------------------------------------------------
constexpr int64_t kMostElems = (int64_t)1 << 35;
constexpr int64_t kMostBlocks = (int64_t)1 << 23;   // of a launch (HIP: fewer than 2^32 threads)

inline bool aligned(const void* p, uintptr_t to) { return ((uintptr_t)p & (to - 1)) == 0; }
inline uintptr_t dtype_bytes(int32_t t) { return t == LCE_DTYPE_F32 ? 4 : 2; }

lce_status_t check_adamw_tensor(const lce_adamw_tensor_t& t, int32_t n_groups, int32_t bits) {
  if (t.n < 0 || t.n >= kMostElems) return LCE_ERR_SHAPE;
  if (t.reserved != 0 || t.group < 0 || t.group >= n_groups || t.place < 0 || t.place % kMomentBlock != 0)
    return LCE_ERR_ARG;
  if (!known_dtype(t.param_dtype) || !known_dtype(t.grad_dtype)) return LCE_ERR_UNSUPPORTED;
  if (t.n == 0) return LCE_OK;
  if (t.master && t.param_dtype != LCE_DTYPE_BF16) return LCE_ERR_ARG;
  if (!t.param || !t.exp_avg || !t.exp_avg_sq || (bits == 8 && !t.units)) return LCE_ERR_NULL;
  if (bits == 32 && t.units) return LCE_ERR_ARG;
  if (!aligned(t.param, dtype_bytes(t.param_dtype)) || !aligned(t.grad, dtype_bytes(t.grad_dtype)) ||
      !aligned(t.master, 4) || !aligned16(t.exp_avg) || !aligned16(t.exp_avg_sq) || !aligned(t.units, 2))
    return LCE_ERR_ALIGN;
  return LCE_OK;
}

inline int64_t norm_part_blocks(const lce_grad_t& g, int64_t bytes) {
  return (g.n * (int64_t)dtype_bytes(g.dtype) + bytes - 1) / bytes;
}

inline int64_t norm_blocks(lce_grad_t g, int64_t bytes) {
  int64_t blocks = 0;
  for (; g.n > kNormEntryElems; g.n -= kNormEntryElems) {
    lce_grad_t part = g;
    part.n = kNormEntryElems;
    blocks += norm_part_blocks(part, bytes);
  }
  return blocks + norm_part_blocks(g, bytes);
}

// *bytes: what a workgroup of k_grad_squares takes, 32 KB (one round of loads) or as many times that as keep the
// sums that the last workgroup adds near 16384 (1.2e9 bf16 elements: 75,000 sums took it 112 us);
// *blocks: the workgroups, each tensor's rounded up
lce_status_t check_grads(const lce_grad_t* grads, int64_t count, int64_t* bytes, int64_t* blocks) {
  if (count < 0) return LCE_ERR_SHAPE;
  if (count > 0 && !grads) return LCE_ERR_NULL;
  double total = 0;
  for (int64_t i = 0; i < count; ++i) {
    const lce_grad_t& g = grads[i];
    if (g.n < 0 || g.n >= kMostElems) return LCE_ERR_SHAPE;
    if (g.reserved != 0) return LCE_ERR_ARG;
    if (!known_dtype(g.dtype)) return LCE_ERR_UNSUPPORTED;
    if (g.n > 0 && !g.data) return LCE_ERR_NULL;
    if (!aligned(g.data, dtype_bytes(g.dtype))) return LCE_ERR_ALIGN;
    total += (double)g.n * dtype_bytes(g.dtype);
  }
  *bytes = 32768;
  while (total > 16384.0 * *bytes) *bytes *= 2;
  *blocks = 0;
  for (int64_t i = 0; i < count; ++i) *blocks += norm_blocks(grads[i], *bytes);
  return LCE_OK;
}

// the entry of elements [at, at + n) of a tensor
void fill_entry(AdamWEntry<32>* e, const lce_adamw_tensor_t& x, int64_t at, int64_t n, int64_t first, int group, int bits) {
  const auto off = [at](const void* p, int64_t size) { return p ? (char*)p + at * size : nullptr; };
  e->param = off(x.param, dtype_bytes(x.param_dtype));
  e->grad = off(x.grad, dtype_bytes(x.grad_dtype));
  e->m = off(x.exp_avg, bits / 8);
  e->v = off(x.exp_avg_sq, bits / 8);
  e->master = (float*)off(x.master, 4);
  e->n = (uint32_t)n;
  e->first = (uint32_t)first;
  e->group = (uint32_t)group;
  e->param_f32 = x.param_dtype == LCE_DTYPE_F32;
  e->grad_f32 = x.grad_dtype == LCE_DTYPE_F32;
  e->wide = aligned16(x.param) | aligned16(x.grad) << 1 | aligned16(x.master) << 2;
}

void fill_entry(AdamWEntry<8>* e, const lce_adamw_tensor_t& x, int64_t at, int64_t n, int64_t first, int group, int bits) {
  fill_entry(static_cast<AdamWEntry<32>*>(e), x, at, n, first, group, bits);
  e->units = (uint8_t*)x.units + at / 16;
  e->pair0 = (uint32_t)((uint64_t)(x.place + at) >> 1);
  e->pad_ = 0;
}

template <int kBits>
void launch_adamw(Launcher& L, const lce_adamw_tensor_t* tensors, int64_t count, const lce_adamw_t* groups, int64_t total,
                  const float* grad_scale, uint32_t seed) {
  AdamWTable<kBits> t;
  // elements of a workgroup. 32-bit moments: one round, so that the workgroups go through the addresses in order
  // (1.2e9 elements 5.80 ms; 2048, 4096, 8192 a workgroup: 6.24, 6.31, 6.54). 8-bit ones, which the vector units
  // bound as much: one round (2048) to fill the card, or up to 16384 where there are more than 8192 workgroups, each
  // of which first finds its tensor (1.2e9 elements 2.34 ms against 2.49 with 2048, in one run; 5.3e6 elements 28 us
  // with 8192, 25 with 2048)
  t.per = kBits == 8 ? 2048 : 1024;
  while (kBits == 8 && t.per < 16384 && total > (int64_t)8192 * t.per) t.per *= 2;
  int32_t group_of[kTableGroups];
  int n_groups = 0;
  int64_t blocks = 0;
  t.count = 0;
  const auto flush = [&] {
    if (t.count == 0) return;
    L(K_ADAMW_TENSORS, k_adamw_tensors<kBits>, dim3((unsigned)blocks), dim3(256), t, grad_scale, seed);
    t.count = n_groups = 0;
    blocks = 0;
  };
  for (int64_t i = 0; i < count; ++i) {
    const lce_adamw_tensor_t& x = tensors[i];
    for (int64_t at = 0; at < x.n; at += kEntryElems) {
      const int64_t n = std::min(x.n - at, kEntryElems), nb = (n + t.per - 1) / t.per;
      int g = 0;
      while (g < n_groups && group_of[g] != x.group) ++g;
      if (t.count == AdamWTable<kBits>::kTensors || g == kTableGroups || blocks + nb > kMostBlocks) {
        flush();
        g = 0;
      }
      if (g == n_groups) {
        (void)make_adamw(&groups[x.group], &t.g[g]);
        group_of[n_groups++] = x.group;
      }
      fill_entry(&t.e[t.count++], x, at, n, blocks, g, kBits);
      blocks += nb;
    }
  }
  flush();
}

}  // namespace

extern "C" {

lce_status_t lce_adamw_tensors_step(const lce_adamw_tensor_t* tensors, int64_t count, const lce_adamw_t* groups,
                                    int32_t n_groups, int32_t state_bits, const float* grad_scale, uint32_t seed,
                                    void* stream) {
  if (count < 0) return LCE_ERR_SHAPE;
  if (n_groups < 1) return LCE_ERR_ARG;
  if (state_bits != 32 && state_bits != 8) return LCE_ERR_UNSUPPORTED;
  if (!groups || (count > 0 && !tensors)) return LCE_ERR_NULL;
  if (!aligned(grad_scale, 4)) return LCE_ERR_ALIGN;
  AdamWConst c;
  for (int32_t g = 0; g < n_groups; ++g)
    if (const lce_status_t st = make_adamw(&groups[g], &c); st != LCE_OK) return st;
  int64_t total = 0;
  for (int64_t i = 0; i < count; ++i) {
    if (const lce_status_t st = check_adamw_tensor(tensors[i], n_groups, state_bits); st != LCE_OK) return st;
    total += tensors[i].n;
  }
  Launcher L{(hipStream_t)stream};
  if (state_bits == 8) launch_adamw<8>(L, tensors, count, groups, total, grad_scale, seed);
  else launch_adamw<32>(L, tensors, count, groups, total, grad_scale, seed);
  return L.st;
}

lce_status_t lce_adamw_moments(int64_t n, const void* exp_avg, const void* exp_avg_sq, const void* units, void* first,
                               void* root, void* stream) {
  if (n < 0 || n >= kMostElems) return LCE_ERR_SHAPE;
  if (n == 0) return LCE_OK;
  if (!exp_avg || !exp_avg_sq || !units || !first || !root) return LCE_ERR_NULL;
  if (!aligned16(exp_avg) || !aligned16(exp_avg_sq) || !aligned(units, 2) || !aligned16(first) || !aligned16(root))
    return LCE_ERR_ALIGN;
  Launcher L{(hipStream_t)stream};
  for (int64_t i = 0; i < n; i += 2048 * kMostBlocks) {
    const int64_t k = std::min<int64_t>(n - i, 2048 * kMostBlocks);
    L(K_ADAMW_MOMENTS, k_adamw_moments, dim3((unsigned)((k + 2047) / 2048)), dim3(256), k, (const uint8_t*)exp_avg + i,
      (const uint8_t*)exp_avg_sq + i, (const uint8_t*)units + i / 16, (uint16_t*)first + i, (uint16_t*)root + i);
  }
  return L.st;
}

lce_status_t lce_grad_norm_workspace_size(const lce_grad_t* grads, int64_t count, size_t* bytes) {
  int64_t per, blocks;
  const lce_status_t st = check_grads(grads, count, &per, &blocks);
  if (st != LCE_OK) return st;
  if (!bytes) return LCE_ERR_NULL;
  *bytes = (size_t)round_up(8 * std::max<int64_t>(blocks, 1), 256);
  return LCE_OK;
}

lce_status_t lce_grad_norm(const lce_grad_t* grads, int64_t count, float max_norm, float* norm, float* factor,
                           void* workspace, size_t workspace_bytes, void* stream) {
  int64_t bytes, blocks;
  const lce_status_t st = check_grads(grads, count, &bytes, &blocks);
  if (st != LCE_OK) return st;
  if (!(max_norm > 0.f)) return LCE_ERR_ARG;
  if (!norm || !workspace) return LCE_ERR_NULL;
  if (!aligned(norm, 4) || !aligned(factor, 4) || !aligned(workspace, 256)) return LCE_ERR_ALIGN;
  if (workspace_bytes < 8 * (size_t)blocks) return LCE_ERR_WORKSPACE;
  Launcher L{(hipStream_t)stream};
  double* parts = (double*)workspace;
  NormTable t;
  int64_t done = 0, here = 0;
  t.count = 0;
  const auto flush = [&] {
    if (t.count == 0) return;
    L(K_GRAD_NORM, k_grad_squares, dim3((unsigned)here), dim3(256), t, bytes, parts + done);
    done += here;
    here = t.count = 0;
  };
  for (int64_t i = 0; i < count; ++i) {
    const lce_grad_t& g = grads[i];
    for (int64_t at = 0; at < g.n; at += kNormEntryElems) {
      const lce_grad_t part{(const char*)g.data + at * dtype_bytes(g.dtype), std::min(g.n - at, kNormEntryElems),
                            g.dtype, 0};
      const int64_t nb = norm_part_blocks(part, bytes);
      if (t.count == kNormTensors || here + nb > kMostBlocks) flush();
      t.e[t.count++] = NormEntry{part.data, (uint32_t)part.n, (uint32_t)here, (uint32_t)(g.dtype == LCE_DTYPE_F32)};
      here += nb;
    }
  }
  flush();
  L(K_GRAD_NORM, k_grad_norm, dim3(1), dim3(1024), (const double*)parts, blocks, max_norm, norm, factor);
  return L.st;
}

}  // extern "C"
