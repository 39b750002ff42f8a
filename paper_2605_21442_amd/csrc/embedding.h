// Token embedding: lookup, and the gradient by sorted tokens. Included by lce.hip, behind its launcher.
//
// The gradient adds each id's tokens in an order that the ids alone fix, without atomics on sums:
//   sort: tokens grouped by id, in token order within an id (a stable counting sort, one launch);
//   grad: per id the fp32 sum of its tokens' rows of dOut, scaled, rounded and stored (or added).
#pragma once

namespace {

// ---------------------------------------------------------------------------------------------
// Sort. Ids are dealt to `nb` (a power of two) buckets by their low bits, so that the frequent ids, which lie
// close together in a vocabulary ordered by frequency, fall into different buckets. One workgroup of 16 waves
// serves a bucket on its own: it reads all N ids, counts those of lower buckets (which is where its bucket
// starts) and, per wave and id, those of its own; a scan over (id, wave) gives every wave the place of its first
// token of every id, and a second walk stores the token numbers. A wave owns consecutive tokens, so the order
// within an id is the tokens'. No workgroup waits for another, and counts do not depend on an order.
// ---------------------------------------------------------------------------------------------
constexpr int kSortWaves = 16;
constexpr int kSortIds = 512;      // most ids of a bucket
constexpr int kSortAhead = 8;      // loads in flight per lane

struct EmbedIds {
  const void* ids;
  int bytes;
  int64_t n, v_begin, v, padding;
};

// the row of token i's id in this shard, or -1
__device__ __forceinline__ int embed_row(const EmbedIds& e, int64_t i) {
  if (i >= e.n) return -1;
  const int64_t id = load_target(e.ids, e.bytes, i);
  const int64_t r = id - e.v_begin;
  return id != e.padding && id >= e.v_begin && r < e.v ? (int)r : -1;
}

__global__ __launch_bounds__(1024) void k_embed_sort(EmbedIds e, int nb_log2, int rows, int2* __restrict__ sorted,
                                                     int* __restrict__ starts) {
  __shared__ int cnt[kSortIds * kSortWaves];   // [id of the bucket][wave]: count, then place of the next token
  __shared__ int wsum[kSortWaves], below_all[kSortWaves];
  const int t = threadIdx.x, lane = t & 63, w = t >> 6;
  const int nb_mask = (1 << nb_log2) - 1, b = blockIdx.x;
  for (int i = t; i < rows * kSortWaves; i += 1024) cnt[i] = 0;
  __syncthreads();
  const int64_t per = (e.n + kSortWaves * 64 - 1) / (kSortWaves * 64) * 64;
  const int64_t i0 = w * per, i1 = min(e.n, i0 + per);
  int below = 0;
  for (int64_t i = i0; i < i1; i += 64 * kSortAhead) {
    int r[kSortAhead];
#pragma unroll
    for (int k = 0; k < kSortAhead; ++k) r[k] = i + 64 * k < i1 ? embed_row(e, i + 64 * k + lane) : -1;
#pragma unroll
    for (int k = 0; k < kSortAhead; ++k) {
      const int rb = r[k] & nb_mask;
      below += r[k] >= 0 && rb < b;
      if (r[k] >= 0 && rb == b) atomicAdd(&cnt[(r[k] >> nb_log2) * kSortWaves + w], 1);
    }
  }
  for (int m = 32; m >= 1; m >>= 1) below += __shfl_xor(below, m);
  if (lane == 0) below_all[w] = below;
  __syncthreads();
  int base = 0;
  for (int k = 0; k < kSortWaves; ++k) base += below_all[k];
  // exclusive scan of cnt: 8 consecutive entries per thread
  constexpr int kPer = kSortIds * kSortWaves / 1024;
  int own[kPer], sum = 0;
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    const int j = t * kPer + k;
    own[k] = j < rows * kSortWaves ? cnt[j] : 0;
    sum += own[k];
  }
  int incl = sum;
  for (int m = 1; m < 64; m <<= 1) {
    const int o = __shfl_up(incl, m);
    if (lane >= m) incl += o;
  }
  if (lane == 63) wsum[w] = incl;
  __syncthreads();
  int at = base + incl - sum;
  for (int k = 0; k < w; ++k) at += wsum[k];
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    const int j = t * kPer + k;
    if (j < rows * kSortWaves) {
      cnt[j] = at;
      if (j % kSortWaves == 0) starts[(int64_t)b * rows + j / kSortWaves] = at;
    }
    at += own[k];
  }
  if (b == nb_mask && t == 1023) starts[((int64_t)nb_mask + 1) * rows] = at;
  __syncthreads();
  for (int64_t i = i0; i < i1; i += 64 * kSortAhead) {
    int r[kSortAhead];
#pragma unroll
    for (int k = 0; k < kSortAhead; ++k) r[k] = i + 64 * k < i1 ? embed_row(e, i + 64 * k + lane) : -1;
#pragma unroll
    for (int k = 0; k < kSortAhead; ++k) {
      const bool in = r[k] >= 0 && (r[k] & nb_mask) == b;
      unsigned long long same = __ballot(in);
      if (same == 0) continue;
      const int q = in ? r[k] >> nb_log2 : 0;
      // the lanes with this lane's id, from one ballot per bit of it
      for (int bit = 0; (rows - 1) >> bit; ++bit) {
        const unsigned long long m = __ballot((q >> bit) & 1);
        same &= (q >> bit) & 1 ? m : ~m;
      }
      const int rank = __popcll(same & ((1ull << lane) - 1ull));
      volatile int* place = &cnt[q * kSortWaves + w];   // this wave's own entries
      const int p = in ? *place + rank : 0;
      if (in && rank == 0) *place = p + __popcll(same);
      if (in) sorted[p] = make_int2(r[k], (int)(i + 64 * k + lane));
    }
  }
}

// ---------------------------------------------------------------------------------------------
// Lookup: 16 bytes of a row per thread and step.
// ---------------------------------------------------------------------------------------------
template <typename T> struct Row8;      // 8 elements as fp32
template <> struct Row8<uint16_t> {
  static __device__ __forceinline__ void load(const uint16_t* p, float x[8]) {
    const uint4 a = *reinterpret_cast<const uint4*>(p);
    const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
    for (int k = 0; k < 4; ++k) { x[2 * k] = __uint_as_float(w[k] << 16); x[2 * k + 1] = __uint_as_float(w[k] & 0xFFFF0000u); }
  }
  static __device__ __forceinline__ void store(uint16_t* p, const float x[8]) {
    store16_padded(p, i32x4_t{(int)pack_bf16x2(x[0], x[1]), (int)pack_bf16x2(x[2], x[3]),
                              (int)pack_bf16x2(x[4], x[5]), (int)pack_bf16x2(x[6], x[7])});
  }
};
template <> struct Row8<float> {
  static __device__ __forceinline__ void load(const float* p, float x[8]) {
    const float4 a = *reinterpret_cast<const float4*>(p), b = *reinterpret_cast<const float4*>(p + 4);
    x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w; x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
  }
  static __device__ __forceinline__ void store(float* p, const float x[8]) {
    i32x4_t v;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
#pragma unroll
      for (int k = 0; k < 4; ++k) v[k] = (int)__float_as_uint(x[4 * h + k]);
      store16_padded(p + 4 * h, v);
    }
  }
};

template <typename T>
__global__ __launch_bounds__(256) void k_embed_lookup(EmbedIds e, int64_t v_total, const T* __restrict__ W, int64_t ldw,
                                                      int d, float scale, T* __restrict__ out, int* status) {
  const int cpr = d >> 3;
  const int64_t total = e.n * cpr;
  for (int64_t q = (int64_t)blockIdx.x * 256 + threadIdx.x; q < total; q += (int64_t)gridDim.x * 256) {
    const int64_t i = q / cpr;
    const int col = (int)(q - i * cpr) * 8;
    const int64_t id = load_target(e.ids, e.bytes, i);
    const int64_t r = id - e.v_begin;
    float x[8] = {};
    if (id >= e.v_begin && r < e.v) {
      Row8<T>::load(W + r * ldw + col, x);
#pragma unroll
      for (int k = 0; k < 8; ++k) x[k] *= scale;
    } else if (status && (id < 0 || id >= v_total) && id != e.padding) {
      *status = LCE_STATUS_ID_OUT_OF_RANGE;   // every writer writes the same value
    }
    Row8<T>::store(out + i * d + col, x);
  }
}

__global__ void k_embed_clear_status(int* status) { *status = 0; }

// ---------------------------------------------------------------------------------------------
// Gradient: one workgroup per id.
// ---------------------------------------------------------------------------------------------
template <typename T, typename TW, bool kAdd>
__global__ __launch_bounds__(256) void k_embed_grad(const int2* __restrict__ sorted, const int* __restrict__ starts,
                                                    int nb_log2, int rows, int v, const T* __restrict__ dout, int64_t ldx, int d,
                                                    float scale, TW* __restrict__ dw) {
  for (int r = blockIdx.x; r < v; r += gridDim.x) {
  const int64_t slot = (int64_t)(r & ((1 << nb_log2) - 1)) * rows + (r >> nb_log2);
  const int p0 = starts[slot], p1 = starts[slot + 1];
  if (kAdd && p0 == p1) continue;
  for (int col = threadIdx.x * 8; col < d; col += 2048) {
    float sum[8] = {};
    for (int p = p0; p < p1; ++p) {
      float x[8];
      Row8<T>::load(dout + (int64_t)sorted[p].y * ldx + col, x);
#pragma unroll
      for (int k = 0; k < 8; ++k) sum[k] += x[k];
    }
    TW* o = dw + (int64_t)r * d + col;
    float old[8] = {};
    if (kAdd) Row8<TW>::load(o, old);
#pragma unroll
    for (int k = 0; k < 8; ++k) sum[k] = old[k] + scale * sum[k];
    Row8<TW>::store(o, sum);
  }
  }
}

// ---------------------------------------------------------------------------------------------
// Host side
// ---------------------------------------------------------------------------------------------
struct EmbedPlan {
  int64_t ldw, ldx, v_total;
  int nb_log2, rows;                 // buckets of the sort, ids of a bucket
  size_t o_sorted, o_starts, bytes;
};

inline bool known_dtype(int32_t t) { return t == LCE_DTYPE_BF16 || t == LCE_DTYPE_F32; }

lce_status_t make_embed_plan(const lce_embedding_t* p, EmbedPlan* pl) {
  if (!p) return LCE_ERR_NULL;
  if (p->reserved != 0 || (p->flags & ~LCE_FLAG_ACCUMULATE_DW) != 0 || !(fabsf(p->scale) < INFINITY)) return LCE_ERR_ARG;
  if (p->n < 0 || p->d < 1 || p->v < 1) return LCE_ERR_SHAPE;
  if (p->d % 8 != 0 || (p->id_bytes != 4 && p->id_bytes != 8)) return LCE_ERR_UNSUPPORTED;
  if (!known_dtype(p->dtype) || (p->dw_dtype != p->dtype && p->dw_dtype != LCE_DTYPE_F32)) return LCE_ERR_UNSUPPORTED;
  if (p->n >= (int64_t)1 << 30 || p->d >= (int64_t)1 << 20) return LCE_ERR_SHAPE;
  pl->v_total = p->v_total ? p->v_total : p->v;
  if (pl->v_total < 1 || pl->v_total >= (int64_t)1 << 30 || p->v_begin < 0 || p->v > pl->v_total ||
      p->v_begin > pl->v_total - p->v)
    return LCE_ERR_SHAPE;
  pl->ldw = p->ld_w ? p->ld_w : p->d;
  pl->ldx = p->ld_x ? p->ld_x : p->d;
  if (pl->ldw < p->d || pl->ldx < p->d || pl->ldw >= (int64_t)1 << 30 || pl->ldx >= (int64_t)1 << 30) return LCE_ERR_SHAPE;
  if (pl->ldw % 8 != 0 || pl->ldx % 8 != 0) return LCE_ERR_ALIGN;
  // 256 buckets, one per CU, or as many as keep a bucket's counts in LDS; no more than there are ids
  pl->nb_log2 = 0;
  while (pl->nb_log2 < 8 && ((int64_t)1 << pl->nb_log2) < p->v) ++pl->nb_log2;
  while (((p->v + ((int64_t)1 << pl->nb_log2) - 1) >> pl->nb_log2) > kSortIds) ++pl->nb_log2;
  pl->rows = (int)((p->v + ((int64_t)1 << pl->nb_log2) - 1) >> pl->nb_log2);
  auto take = [](size_t& cur, size_t bytes) { size_t o = cur; cur += (bytes + 255) / 256 * 256; return o; };
  size_t cur = 0;
  pl->o_sorted = take(cur, 8 * (size_t)p->n);
  pl->o_starts = take(cur, 4 * (((size_t)pl->rows << pl->nb_log2) + 1));
  pl->bytes = cur;
  return LCE_OK;
}

template <typename T>
void launch_lookup(Launcher& L, const lce_embedding_t* p, const EmbedPlan& pl, const EmbedIds& e, const void* W, void* out,
                   int32_t* status) {
  const int64_t blocks = (p->n * (p->d / 8) + 255) / 256;
  L(K_EMBED_LOOKUP, k_embed_lookup<T>, dim3((unsigned)std::min<int64_t>(blocks, 1 << 20)), dim3(256), e, pl.v_total,
    (const T*)W, pl.ldw, (int)p->d, p->scale, (T*)out, status);
}

template <typename T, typename TW>
void launch_embed_grad(Launcher& L, const lce_embedding_t* p, const EmbedPlan& pl, const int2* sorted, const int* starts,
                       const void* dout, void* dw) {
  const auto kernel = p->flags & LCE_FLAG_ACCUMULATE_DW ? k_embed_grad<T, TW, true> : k_embed_grad<T, TW, false>;
  L(K_EMBED_GRAD, kernel, dim3((unsigned)std::min<int64_t>(p->v, 1 << 20)), dim3(256), sorted, starts, pl.nb_log2, pl.rows, (int)p->v, (const T*)dout, pl.ldx,
    (int)p->d, p->scale, (TW*)dw);
}

}  // namespace

extern "C" {

lce_status_t lce_embedding_workspace_size(const lce_embedding_t* p, size_t* bwd_bytes) {
  EmbedPlan pl;
  const lce_status_t st = make_embed_plan(p, &pl);
  if (st != LCE_OK) return st;
  if (!bwd_bytes) return LCE_ERR_NULL;
  *bwd_bytes = pl.bytes;
  return LCE_OK;
}

lce_status_t lce_embedding_forward(const lce_embedding_t* p, const void* W, const void* ids, void* out,
                                   int32_t* dev_status, void* stream) {
  EmbedPlan pl;
  const lce_status_t st = make_embed_plan(p, &pl);
  if (st != LCE_OK) return st;
  if (!W || (p->n > 0 && (!ids || !out))) return LCE_ERR_NULL;
  if (!aligned16(W) || ((uintptr_t)ids & (p->id_bytes - 1)) != 0 || !aligned16(out)) return LCE_ERR_ALIGN;
  Launcher L{(hipStream_t)stream};
  const EmbedIds e{ids, p->id_bytes, p->n, p->v_begin, p->v, p->padding_idx};
  if (dev_status) L(K_MISC, k_embed_clear_status, dim3(1), dim3(1), dev_status);
  if (p->dtype == LCE_DTYPE_BF16) launch_lookup<uint16_t>(L, p, pl, e, W, out, dev_status);
  else launch_lookup<float>(L, p, pl, e, W, out, dev_status);
  return L.st;
}

lce_status_t lce_embedding_backward(const lce_embedding_t* p, const void* ids, const void* dOut, void* dW,
                                    void* workspace, size_t workspace_bytes, void* stream) {
  EmbedPlan pl;
  const lce_status_t st = make_embed_plan(p, &pl);
  if (st != LCE_OK) return st;
  if (!dW || !workspace || (p->n > 0 && (!ids || !dOut))) return LCE_ERR_NULL;
  if (((uintptr_t)ids & (p->id_bytes - 1)) != 0 || !aligned16(dOut) || !aligned16(dW) || ((uintptr_t)workspace & 255) != 0) return LCE_ERR_ALIGN;
  if (workspace_bytes < pl.bytes) return LCE_ERR_WORKSPACE;
  Launcher L{(hipStream_t)stream};
  char* ws = (char*)workspace;
  int2* sorted = (int2*)(ws + pl.o_sorted);
  int* starts = (int*)(ws + pl.o_starts);
  const EmbedIds e{ids, p->id_bytes, p->n, p->v_begin, p->v, p->padding_idx};
  L(K_EMBED_SORT, k_embed_sort, dim3(1u << pl.nb_log2), dim3(64 * kSortWaves), e, pl.nb_log2, pl.rows, sorted, starts);
  if (p->dtype == LCE_DTYPE_F32) launch_embed_grad<float, float>(L, p, pl, sorted, starts, dOut, dW);
  else if (p->dw_dtype == LCE_DTYPE_F32) launch_embed_grad<uint16_t, float>(L, p, pl, sorted, starts, dOut, dW);
  else launch_embed_grad<uint16_t, uint16_t>(L, p, pl, sorted, starts, dOut, dW);
  return L.st;
}

}  // extern "C"
