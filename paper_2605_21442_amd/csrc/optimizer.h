// AdamW over many tensors (moments in 32 or 8 bits) and the norm of many gradients. Included by lce.hip,
// behind its launcher. A launch serves up to kTableTensors tensors, whose addresses travel in its arguments: nothing
// is copied to the device beforehand, so a call can be captured and its table needs no storage.
#pragma once

namespace {

constexpr int kTableTensors = 48;
constexpr int kTableGroups = 8;
constexpr int kMomentBlock = 32;       // elements that share the units of the 8-bit moments

struct AdamWEntry {
  void* param;
  const void* grad;
  void* m;
  void* v;
  uint8_t* units;
  float* master;
  int64_t n;
  uint32_t first;          // first workgroup of this tensor
  uint32_t pair0;          // place / 2
  uint8_t group, param_f32, grad_f32, pad_[5];
};

struct AdamWTable {
  AdamWEntry e[kTableTensors];
  AdamWConst g[kTableGroups];
  int count;
};
static_assert(sizeof(AdamWTable) <= 4000, "launch arguments");

// ---------------------------------------------------------------------------------------------
// 8-bit moments (the form is in lce.h). kMant 3: sign and 7 bits; kMant 4: 8 bits, no sign.
// ---------------------------------------------------------------------------------------------
__device__ __forceinline__ float pow2f(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }

// unit byte of a block from the bits of its largest magnitude (as an unsigned number, which orders
// magnitudes, and infinities and NaN above them)
template <int kMant>
__device__ __forceinline__ int unit_byte(uint32_t top) {
  if (top >= 0x7F800000u) return 255;
  const int s = (int)((top + (1u << (23 - kMant))) >> 23) - 14 - kMant;
  return s < 1 ? 1 : s;
}

// code of magnitude a >= 0 in units of 2^(s - 127); u in [0, 1): upward from the code below where the place
// between the two is at least 1 - u
template <int kMant>
__device__ __forceinline__ uint32_t encode(float a, int s, float u) {
#pragma clang fp contract(off)
  const float y = a * pow2f(127 - s);              // exact
  int h = (int)(__float_as_uint(y) >> 23) - 127 - kMant;
  h = h < 0 ? 0 : h;
  return (uint32_t)floorf(y * pow2f(-h) + u) + ((uint32_t)h << kMant);
}

template <int kMant>
__device__ __forceinline__ float decode(uint32_t c, int s) {
  const int h = (int)(c >> kMant);
  const float q = (float)(h ? (c & ((1u << kMant) - 1)) + (1u << kMant) : c);
  return q * (s == 255 ? __uint_as_float(0x7FC00000u) : pow2f((h ? h - 1 : 0) + s - 127));
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

__device__ __forceinline__ float load_elem(const void* p, int64_t i, bool f32) {
  return f32 ? ((const float*)p)[i] : bf16_to_f32(((const uint16_t*)p)[i]);
}

constexpr int kStepElems = 4096;       // elements of a workgroup

// One element per thread and step; the 32 lanes of a half wave are a block of the 8-bit moments.
template <int kBits>
__global__ __launch_bounds__(256) void k_adamw_tensors(AdamWTable t, const float* __restrict__ grad_scale, uint32_t seed) {
#pragma clang fp contract(off)
  const float scale = grad_scale ? *grad_scale : 1.0f;
  if (!(fabsf(scale) < INFINITY)) return;
  int k = 0;
  while (k + 1 < t.count && t.e[k + 1].first <= blockIdx.x) ++k;
  const AdamWEntry& e = t.e[k];
  const AdamWConst c = t.g[e.group];
  const int64_t i0 = (int64_t)(blockIdx.x - e.first) * kStepElems;
  for (int j = 0; j < kStepElems; j += 256) {
    if (i0 + j >= e.n) break;                     // uniform
    const int64_t i = i0 + j + threadIdx.x;
    const bool live = i < e.n;
    const int64_t blk = i / kMomentBlock;
    float p = 0.f, g = 0.f, m = 0.f, v = 0.f;
    if (live) {
      p = e.master ? e.master[i] : load_elem(e.param, i, e.param_f32);
      if (e.grad) g = load_elem(e.grad, i, e.grad_f32);
      if (kBits == 32) {
        m = ((float*)e.m)[i];
        v = ((float*)e.v)[i];
      } else {
        const uint32_t cm = ((const uint8_t*)e.m)[i];
        const float x = decode<3>(cm & 127, e.units[2 * blk]), r = decode<4>(((const uint8_t*)e.v)[i], e.units[2 * blk + 1]);
        m = cm & 128 ? -x : x;
        v = r * r;
      }
    }
    if (grad_scale) g = g * scale;
    adamw_update(p, m, v, g, c);
    if (kBits == 8) {
      const float root = sqrtf(v);
      uint32_t am = live ? __float_as_uint(m) & 0x7FFFFFFFu : 0, ar = live ? __float_as_uint(root) & 0x7FFFFFFFu : 0;
      for (int x = 16; x >= 1; x >>= 1) {
        am = max(am, (uint32_t)__shfl_xor((int)am, x));
        ar = max(ar, (uint32_t)__shfl_xor((int)ar, x));
      }
      const int sm = unit_byte<3>(am), sr = unit_byte<4>(ar);
      if (live) {
        const uint32_t h = pair_bits(e.pair0 + (uint32_t)(i >> 1), seed);
        const float u = (float)(i & 1 ? h >> 16 : h & 0xFFFFu) * 0x1p-16f;
        const uint32_t cm = sm == 255 ? 0 : encode<3>(fabsf(m), sm, u);
        uint32_t cr = sr == 255 ? 0 : encode<4>(root, sr, u);
        if (root > 0.f && cr == 0) cr = 1;
        ((uint8_t*)e.m)[i] = (uint8_t)(cm | (__float_as_uint(m) >> 24 & 128));
        ((uint8_t*)e.v)[i] = (uint8_t)cr;
        if (i % kMomentBlock == 0) {
          e.units[2 * blk] = (uint8_t)sm;
          e.units[2 * blk + 1] = (uint8_t)sr;
        }
      }
    } else if (live) {
      ((float*)e.m)[i] = m;
      ((float*)e.v)[i] = v;
    }
    if (live) {
      if (e.master) e.master[i] = p;
      if (e.param_f32) ((float*)e.param)[i] = p;
      else ((uint16_t*)e.param)[i] = to_bf16(p);
    }
  }
}

__global__ __launch_bounds__(256) void k_adamw_moments(int64_t n, const uint8_t* __restrict__ m, const uint8_t* __restrict__ r,
                                                       const uint8_t* __restrict__ units, uint16_t* __restrict__ first,
                                                       uint16_t* __restrict__ root) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= n) return;
  const float x = decode<3>(m[i] & 127, units[2 * (i / kMomentBlock)]);
  first[i] = to_bf16(m[i] & 128 ? -x : x);
  root[i] = to_bf16(decode<4>(r[i], units[2 * (i / kMomentBlock) + 1]));
}

// ---------------------------------------------------------------------------------------------
// Norm of many gradients: every workgroup leaves the fp64 sum of the squares of its elements, and one
// workgroup adds these in order. fp64: an fp32 square overflows from 1.8e19 on, which bf16 holds, and a
// model's 1e9 squares lose digits in fp32.
// ---------------------------------------------------------------------------------------------
struct NormEntry {
  const void* data;
  int64_t n;
  uint32_t first, f32;
};
constexpr int kNormTensors = 160;
struct NormTable {
  NormEntry e[kNormTensors];
  int count;
};
static_assert(sizeof(NormTable) <= 4000, "launch arguments");
constexpr int kNormElems = 16384;      // elements of a workgroup

__device__ __forceinline__ double block_sum_f64(double x) {
  __shared__ double part[4];
  for (int m = 32; m >= 1; m >>= 1) x += __shfl_xor(x, m);
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = x;
  __syncthreads();
  return (part[0] + part[1]) + (part[2] + part[3]);
}

__global__ __launch_bounds__(256) void k_grad_squares(NormTable t, double* __restrict__ parts) {
  int k = 0;
  while (k + 1 < t.count && t.e[k + 1].first <= blockIdx.x) ++k;
  const NormEntry& e = t.e[k];
  const int64_t i0 = (int64_t)(blockIdx.x - e.first) * kNormElems;
  const int64_t i1 = min(e.n, i0 + kNormElems);
  double sum = 0;
  for (int64_t i = i0 + threadIdx.x; i < i1; i += 256) {
    const double x = load_elem(e.data, i, e.f32);
    sum += x * x;
  }
  sum = block_sum_f64(sum);
  if (threadIdx.x == 0) parts[blockIdx.x] = sum;
}

__global__ __launch_bounds__(256) void k_grad_norm(const double* __restrict__ parts, int64_t count, float max_norm,
                                                   float* norm, float* factor) {
  double sum = 0;
  for (int64_t i = threadIdx.x; i < count; i += 256) sum += parts[i];
  sum = block_sum_f64(sum);
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
  if (t.reserved != 0 || t.group < 0 || t.group >= n_groups || t.place < 0 || t.place % kMomentBlock != 0) return LCE_ERR_ARG;
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

lce_status_t check_grads(const lce_grad_t* grads, int64_t count, int64_t* blocks) {
  if (count < 0) return LCE_ERR_SHAPE;
  if (count > 0 && !grads) return LCE_ERR_NULL;
  *blocks = 0;
  for (int64_t i = 0; i < count; ++i) {
    const lce_grad_t& g = grads[i];
    if (g.n < 0 || g.n >= kMostElems) return LCE_ERR_SHAPE;
    if (g.reserved != 0) return LCE_ERR_ARG;
    if (!known_dtype(g.dtype)) return LCE_ERR_UNSUPPORTED;
    if (g.n > 0 && !g.data) return LCE_ERR_NULL;
    if (!aligned(g.data, dtype_bytes(g.dtype))) return LCE_ERR_ALIGN;
    *blocks += (g.n + kNormElems - 1) / kNormElems;
  }
  return LCE_OK;
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
  for (int64_t i = 0; i < count; ++i)
    if (const lce_status_t st = check_adamw_tensor(tensors[i], n_groups, state_bits); st != LCE_OK) return st;
  Launcher L{(hipStream_t)stream};
  AdamWTable t;
  int32_t group_of[kTableGroups];
  int n_table_groups = 0;
  int64_t blocks = 0;
  t.count = 0;
  const auto flush = [&] {
    if (t.count == 0) return;
    const auto kernel = state_bits == 8 ? k_adamw_tensors<8> : k_adamw_tensors<32>;
    L(K_ADAMW_TENSORS, kernel, dim3((unsigned)blocks), dim3(256), t, grad_scale, seed);
    t.count = n_table_groups = 0;
    blocks = 0;
  };
  for (int64_t i = 0; i < count; ++i) {
    const lce_adamw_tensor_t& x = tensors[i];
    if (x.n == 0) continue;
    const int64_t nb = (x.n + kStepElems - 1) / kStepElems;
    int g = 0;
    while (g < n_table_groups && group_of[g] != x.group) ++g;
    if (t.count == kTableTensors || g == kTableGroups || blocks + nb > kMostBlocks) {
      flush();
      g = 0;
    }
    if (g == n_table_groups) {
      (void)make_adamw(&groups[x.group], &t.g[g]);
      group_of[n_table_groups++] = x.group;
    }
    t.e[t.count++] = AdamWEntry{x.param, x.grad, x.exp_avg, x.exp_avg_sq, (uint8_t*)x.units, x.master, x.n,
                                (uint32_t)blocks, (uint32_t)((uint64_t)x.place >> 1), (uint8_t)g,
                                (uint8_t)(x.param_dtype == LCE_DTYPE_F32), (uint8_t)(x.grad_dtype == LCE_DTYPE_F32), {}};
    blocks += nb;
  }
  flush();
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
  for (int64_t i = 0; i < n; i += 256 * kMostBlocks) {
    const int64_t k = std::min<int64_t>(n - i, 256 * kMostBlocks);
    L(K_ADAMW_MOMENTS, k_adamw_moments, dim3((unsigned)((k + 255) / 256)), dim3(256), k, (const uint8_t*)exp_avg + i,
      (const uint8_t*)exp_avg_sq + i, (const uint8_t*)units + i / 16, (uint16_t*)first + i, (uint16_t*)root + i);
  }
  return L.st;
}

lce_status_t lce_grad_norm_workspace_size(const lce_grad_t* grads, int64_t count, size_t* bytes) {
  int64_t blocks;
  const lce_status_t st = check_grads(grads, count, &blocks);
  if (st != LCE_OK) return st;
  if (!bytes) return LCE_ERR_NULL;
  *bytes = (size_t)round_up(8 * std::max<int64_t>(blocks, 1), 256);
  return LCE_OK;
}

lce_status_t lce_grad_norm(const lce_grad_t* grads, int64_t count, float max_norm, float* norm, float* factor,
                           void* workspace, size_t workspace_bytes, void* stream) {
  int64_t blocks;
  const lce_status_t st = check_grads(grads, count, &blocks);
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
    L(K_GRAD_NORM, k_grad_squares, dim3((unsigned)here), dim3(256), t, parts + done);
    done += here;
    here = t.count = 0;
  };
  for (int64_t i = 0; i < count; ++i) {
    const lce_grad_t& g = grads[i];
    if (g.n == 0) continue;
    const int64_t nb = (g.n + kNormElems - 1) / kNormElems;
    if (t.count == kNormTensors || here + nb > kMostBlocks) flush();
    t.e[t.count++] = NormEntry{g.data, g.n, (uint32_t)here, (uint32_t)(g.dtype == LCE_DTYPE_F32)};
    here += nb;
  }
  flush();
  L(K_GRAD_NORM, k_grad_norm, dim3(1), dim3(256), (const double*)parts, blocks, max_norm, norm, factor);
  return L.st;
}

}  // extern "C"
