// Token embedding: lookup, and the gradient by sorted tokens. Included by lce.hip, behind its launcher.
//
// The gradient adds each id's tokens in an order that the ids alone fix, without atomics on sums:
//   sort: tokens grouped by id, in token order within an id (a stable counting sort, one launch);
//   grad: the fp32 sums of the rows of dOut by runs of sorted tokens;
//   join: the sums of the ids that several runs share; and, in a fresh dW, the rows without tokens (or a launch before).
// Few tokens take one launch for all of it (k_embed_few).
#pragma once

namespace {

// ---------------------------------------------------------------------------------------------
// Sort. Ids are dealt to `nb` (a power of two) buckets by their low bits, so that the frequent ids, which lie close
// together in a vocabulary ordered by frequency, fall into different buckets. One workgroup of 16 waves serves a
// bucket on its own: it reads all N ids, counts those of lower buckets (which is where its bucket starts) and, per
// wave and id, those of its own; a scan over (id, wave) gives every wave the place of its first token of every id, at
// which it then puts its tokens. A wave owns consecutive tokens, so the order within an id is the tokens'. No
// workgroup waits for another, and counts do not depend on an order. A wave lists its tokens of the bucket in LDS as
// it counts them, so only one with more than the list holds walks the ids twice. 709 / 4096 / 16384 / 65070 tokens:
// 6.2 / 7.2 / 10.2 / 30 us. Short batches are bound by the chain of loads, barriers and the scan; long ones by the
// vector instructions of the walk (every bucket looks at every id) in the bucket of the most frequent id, 0.3 to 0.5
// us per 1000 tokens. (Ranks by one ballot per bit for every group of 64 tokens, without the lists: 22 us for 16384
// tokens; ids loaded one group at a time: 30.)
// ---------------------------------------------------------------------------------------------
constexpr int kSortWaves = 16;
constexpr int kSortIds = 1024;     // most ids of a bucket, one per thread in the scan
constexpr int kSortAhead = 8;      // groups of 64 tokens whose ids a wave loads at a time
constexpr int kSortList = 640;     // listed tokens of a wave; a round of loads adds up to 512

// rows of W that get a gradient: id - v_begin in [0, v), other than the padding id's (pad_row, or -1)
struct EmbedRows {
  const void* ids;
  int64_t n, v_begin;
  uint32_t v;
  int pad_row;
};

// Of the wave's groups from token i on: the rows of the tokens' ids, and their buckets (INT_MAX where a token has
// none). All loads are issued before the first is used: behind i1 they read the last token again.
template <int kBytes>
__device__ __forceinline__ void embed_buckets(const EmbedRows& e, int64_t i, int64_t i1, int mask, int row[kSortAhead],
                                              int bucket[kSortAhead]) {
  typedef typename std::conditional<kBytes == 8, uint64_t, uint32_t>::type Id;
  Id id[kSortAhead];
#pragma unroll
  for (int k = 0; k < kSortAhead; ++k) id[k] = ((const Id*)e.ids)[min(i + 64 * k, i1 - 1)];
#pragma unroll
  for (int k = 0; k < kSortAhead; ++k) {
    const Id r = id[k] - (Id)e.v_begin;       // unsigned (v_begin + v <= 2^30: no other id wraps into the rows)
    row[k] = (int)r;
    bucket[k] = i + 64 * k < i1 && r < e.v && (int)r != e.pad_row ? (int)r & mask : 0x7FFFFFFF;
  }
}

// What lanes of a wave wrote to LDS before is what its lanes read behind (the wave's LDS accesses are in order; the
// compiler is told not to move them).
__device__ __forceinline__ void wave_lds_order() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// The listed tokens of a wave, in order, to their places; place[q] is where the wave's next token of the bucket's
// id q goes. 64 tokens at a time: a lane's rank among those with its id comes from one ballot per bit of the id.
__device__ __forceinline__ void embed_place(const int2* list, int count, int* place_, int nb_log2, int rows, int lane,
                                            int2* __restrict__ sorted) {
  volatile int* place = place_;
  for (int l = 0; l < count; l += 64) {
    const bool in = l + lane < count;
    const int2 pair = list[in ? l + lane : l];
    const int q = pair.x >> nb_log2;
    unsigned long long same = __ballot(in);
    for (int bit = 0; (rows - 1) >> bit; ++bit) {
      const unsigned long long m = __ballot((q >> bit) & 1);
      same &= (q >> bit) & 1 ? m : ~m;
    }
    const int rank = __popcll(same & ((1ull << lane) - 1ull));
    const int p = place[q] + rank;
    if (in && rank == 0) place[q] = p + __popcll(same);
    if (in) sorted[p] = pair;
  }
}

template <int kBytes>
__global__ __launch_bounds__(1024) void k_embed_sort(EmbedRows e, int nb_log2, int rows, int2* __restrict__ sorted,
                                                     int* __restrict__ starts) {
  __shared__ int cnt[kSortWaves][kSortIds];    // per wave and id of the bucket: count, then place of the next token
  __shared__ int2 lists[kSortWaves][kSortList];
  __shared__ int wsum[kSortWaves], below_all[kSortWaves];
  const int t = threadIdx.x, lane = t & 63, w = __builtin_amdgcn_readfirstlane(t >> 6);
  const int mask = (1 << nb_log2) - 1, b = blockIdx.x;
  for (int q = lane; q < rows; q += 64) cnt[w][q] = 0;      // its own entries only, until the scan
  wave_lds_order();
  const int64_t per = (e.n + kSortWaves * 64 - 1) / (kSortWaves * 64) * 64;
  const int64_t i0 = w * per, i1 = min(e.n, i0 + per);
  int2* list = lists[w];
  int r[kSortAhead], rb[kSortAhead], below = 0, mine = 0;
  for (int64_t i = i0; i < i1; i += 64 * kSortAhead) {
    embed_buckets<kBytes>(e, i + lane, i1, mask, r, rb);
#pragma unroll
    for (int k = 0; k < kSortAhead; ++k) {
      below += rb[k] < b;
      const unsigned long long m = __ballot(rb[k] == b);
      if (m == 0) continue;
      if (rb[k] == b) {
        atomicAdd(&cnt[w][r[k] >> nb_log2], 1);
        const int l = mine + __popcll(m & ((1ull << lane) - 1ull));
        if (l < kSortList) list[l] = make_int2(r[k], (int)(i + 64 * k + lane));
      }
      mine += __popcll(m);
    }
  }
  for (int m = 32; m >= 1; m >>= 1) below += __shfl_xor(below, m);
  if (lane == 0) below_all[w] = below;
  __syncthreads();
  // thread t: the tokens of the bucket's id t, wave by wave, and of all ids before
  int own[kSortWaves], sum = 0;
#pragma unroll
  for (int k = 0; k < kSortWaves; ++k) {
    own[k] = t < rows ? cnt[k][t] : 0;
    sum += own[k];
  }
  int at = sum;
  for (int m = 1; m < 64; m <<= 1) {
    const int o = __shfl_up(at, m);
    if (lane >= m) at += o;
  }
  if (lane == 63) wsum[w] = at;
  __syncthreads();
  at -= sum;
#pragma unroll
  for (int k = 0; k < kSortWaves; ++k) at += below_all[k] + (k < w ? wsum[k] : 0);
  if (t < rows) {
    starts[(int64_t)b * rows + t] = at;
    if (b == mask && t == rows - 1) starts[(int64_t)b * rows + rows] = at + sum;
#pragma unroll
    for (int k = 0; k < kSortWaves; ++k) {
      cnt[k][t] = at;
      at += own[k];
    }
  }
  __syncthreads();
  if (mine <= kSortList) {
    embed_place(list, mine, cnt[w], nb_log2, rows, lane, sorted);
    return;
  }
  mine = 0;
  for (int64_t i = i0; i < i1; i += 64 * kSortAhead) {
    embed_buckets<kBytes>(e, i + lane, i1, mask, r, rb);
#pragma unroll
    for (int k = 0; k < kSortAhead; ++k) {
      const unsigned long long m = __ballot(rb[k] == b);
      if (rb[k] == b) list[mine + __popcll(m & ((1ull << lane) - 1ull))] = make_int2(r[k], (int)(i + 64 * k + lane));
      mine += __popcll(m);
    }
    if (mine > kSortList - 64 * kSortAhead || i + 64 * kSortAhead >= i1) {
      wave_lds_order();
      embed_place(list, mine, cnt[w], nb_log2, rows, lane, sorted);
      wave_lds_order();
      mine = 0;
    }
  }
}

// ---------------------------------------------------------------------------------------------
// Lookup: a workgroup writes 8192 consecutive elements of out, a thread 8 of every 2048 of them, so that the rows of
// four pieces are in flight and the stores go in the order of the addresses. kOnce: the stores pass the L2 and the
// 256 MB MALL by. An output that fits there is better kept, for the layer that reads it next: W cold, 16384 tokens of
// 4096 (134 MB) looked up and then read take 77 us kept and 88 passed by, 2048 (17 MB) 19 and 22; one that does not
// fit is better passed by, 32768 (268 MB) 167 and 159. (Lookups of nothing else in a row, whose rows of W then stay
// in the MALL: 134 MB 37 and 29.5 us, 235 MB 70 and 49.5.)
// ---------------------------------------------------------------------------------------------
// 8 elements: as they lie in memory (so that a load is only issued where it stands), and as fp32
template <typename T> struct Row8;
template <> struct Row8<uint16_t> {
  struct Raw { uint4 a; };
  static __device__ __forceinline__ Raw fetch(const uint16_t* p) { return {*reinterpret_cast<const uint4*>(p)}; }
  static __device__ __forceinline__ void unpack(const Raw& r, float x[8]) {
    const uint32_t w[4] = {r.a.x, r.a.y, r.a.z, r.a.w};
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      x[2 * k] = __uint_as_float(w[k] << 16);
      x[2 * k + 1] = __uint_as_float(w[k] & 0xFFFF0000u);
    }
  }
  template <bool kOnce = false>      // written once: not kept in the L2
  static __device__ __forceinline__ void store(uint16_t* p, const float x[8]) {
    const i32x4_t v{(int)pack_bf16x2(x[0], x[1]), (int)pack_bf16x2(x[2], x[3]), (int)pack_bf16x2(x[4], x[5]),
                    (int)pack_bf16x2(x[6], x[7])};
    if (kOnce) store16_padded_nt(p, v);
    else store16_padded(p, v);
  }
};
template <> struct Row8<float> {
  struct Raw { float4 a, b; };
  static __device__ __forceinline__ Raw fetch(const float* p) {
    return {*reinterpret_cast<const float4*>(p), *reinterpret_cast<const float4*>(p + 4)};
  }
  static __device__ __forceinline__ void unpack(const Raw& r, float x[8]) {
    x[0] = r.a.x; x[1] = r.a.y; x[2] = r.a.z; x[3] = r.a.w; x[4] = r.b.x; x[5] = r.b.y; x[6] = r.b.z; x[7] = r.b.w;
  }
  template <bool kOnce = false>
  static __device__ __forceinline__ void store(float* p, const float x[8]) {
    i32x4_t v;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
#pragma unroll
      for (int k = 0; k < 4; ++k) v[k] = (int)__float_as_uint(x[4 * h + k]);
      if (kOnce) store16_padded_nt(p + 4 * h, v);
      else store16_padded(p + 4 * h, v);
    }
  }
};

struct EmbedIds {
  const void* ids;
  int bytes;
  int64_t n, v_begin, v, padding;
};

constexpr int64_t kKeptBytes = (int64_t)192 << 20;    // of an output, at most, that is kept in the caches

template <typename T, bool kOnce>
__global__ __launch_bounds__(256) void k_embed_lookup(EmbedIds e, int64_t v_total, const T* __restrict__ W, int64_t ldw,
                                                      int d, float scale, T* __restrict__ out, int* status) {
  constexpr int kAhead = 4;
  const uint32_t row8 = (uint32_t)d >> 3;
  for (int64_t block = blockIdx.x; block * (256 * kAhead) < e.n * row8; block += gridDim.x) {
    const int64_t i0 = block * (256 * kAhead) / row8;
    const uint32_t o0 = (uint32_t)(block * (256 * kAhead) - i0 * row8);
    int64_t i[kAhead], id[kAhead];
    uint32_t col[kAhead];
    bool held[kAhead];
    typename Row8<T>::Raw raw[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      const uint32_t o = o0 + threadIdx.x + 256 * k;
      i[k] = i0 + o / row8;
      col[k] = o % row8 * 8;
      id[k] = load_target(e.ids, e.bytes, min(i[k], e.n - 1));
    }
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {          // (an id that W does not hold reads row 0, which is then not used)
      held[k] = id[k] >= e.v_begin && id[k] - e.v_begin < e.v;
      raw[k] = Row8<T>::fetch(W + (held[k] ? id[k] - e.v_begin : 0) * ldw + col[k]);
    }
    if (status)
#pragma unroll
      for (int k = 0; k < kAhead; ++k)
        if ((id[k] < 0 || id[k] >= v_total) && id[k] != e.padding)
          *status = LCE_STATUS_ID_OUT_OF_RANGE;   // every writer writes the same value
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      if (i[k] >= e.n) break;
      float x[8];
      Row8<T>::unpack(raw[k], x);
#pragma unroll
      for (int c = 0; c < 8; ++c) x[c] = held[k] ? x[c] * scale : 0.f;
      Row8<T>::template store<kOnce>(out + i[k] * d + col[k], x);
    }
  }
}

__global__ void k_embed_clear_status(int* status) { *status = 0; }

// ---------------------------------------------------------------------------------------------
// Gradient: the sorted tokens are cut into chunks of `per` consecutive ones, and a wave takes a chunk's tokens at 512
// columns (8 per lane), eight rows of dOut in flight. An id whose tokens lie in one chunk is finished there. One that
// reaches over a chunk's edge leaves an fp32 sum per chunk, in the chunk's slot 0 where it goes on from the chunk
// before and in slot 1 where it starts, and k_embed_join adds these in the order of the chunks. So a frequent id is
// spread over many waves, and the order of all sums follows from the ids and N alone. Bound by memory: 4096 tokens
// added to a 128256 x 8192 dW 21.5 us (5.5 TB/s), 32768 to a 152064 x 3584 dW 64 us (4.6); one workgroup per id, the
// simplest form, took 700 us for the former: the most frequent id's tokens came one after the other.
// ---------------------------------------------------------------------------------------------
constexpr int kGradCols = 512;     // columns of a wave

struct EmbedSorted {
  const int2* pairs;               // (row of W, token), by id
  const int* starts;               // first pair of each id, bucket by bucket
  int nb_log2, rows;
  __device__ __forceinline__ int64_t slot(int r) const {
    return (int64_t)(r & ((1 << nb_log2) - 1)) * rows + (r >> nb_log2);
  }
  __device__ __forceinline__ int count() const { return starts[(int64_t)rows << nb_log2]; }
};

// (old: what dW holds there, where the sum is added to it)
template <typename TW, bool kAdd>
__device__ __forceinline__ void grad_store(TW* o, const typename Row8<TW>::Raw& old, const float sum[8], float scale) {
  float x[8] = {};
  if (kAdd) Row8<TW>::unpack(old, x);
#pragma unroll
  for (int k = 0; k < 8; ++k) x[k] += scale * sum[k];
  Row8<TW>::store(o, x);
}

template <typename T, typename TW, bool kAdd>
__global__ __launch_bounds__(256) void k_embed_grad(EmbedSorted s, const T* __restrict__ dout, int64_t ldx, int d,
                                                    int per, int64_t chunk_units, int slices, float scale,
                                                    TW* __restrict__ dw, float* __restrict__ parts) {
  constexpr int kAhead = 8;
  const int lane = threadIdx.x & 63;
  const int64_t unit = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
  if (unit >= chunk_units) return;
  const int chunk = (int)(unit / slices);
  const int col0 = (int)(unit - (int64_t)chunk * slices) * kGradCols + lane * 8;
  const bool live = col0 < d;
  const int col = live ? col0 : 0;             // (lanes behind the row read its start and store nothing)
  const int nv = s.count();
  const int c0 = chunk * per, c1 = min(nv, c0 + per);
  if (c0 >= c1) return;
  const int before = c0 > 0 ? s.pairs[c0 - 1].x : -1, after = c1 < nv ? s.pairs[c1].x : -1;
  float* part = parts + (int64_t)chunk * 2 * d + col;
  float sum[8] = {};
  bool first = true;               // still at the chunk's first id
  for (int g0 = c0; g0 < c1; g0 += 64) {
    const int here = min(64, c1 - g0);
    const int2 my = s.pairs[g0 + min(lane, here - 1)];
    const int next = __shfl_down(my.x, 1);     // the id behind; at the group's end the next group's, or `after`
    const int follow = lane < here - 1 ? next : g0 + here < c1 ? s.pairs[g0 + here].x : after;
    const unsigned long long ends = __ballot(my.x != follow || (g0 + lane == c1 - 1));
    for (int p = 0; p < here; p += kAhead) {
      // the rows of dOut, and of dW where an id ends, all in flight
      typename Row8<T>::Raw x[kAhead];
      typename Row8<TW>::Raw old[kAhead];
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {
        const int q = min(p + k, here - 1);
        x[k] = Row8<T>::fetch(dout + (int64_t)__builtin_amdgcn_readlane(my.y, q) * ldx + col);
      }
      if constexpr (kAdd)
#pragma unroll
        for (int k = 0; k < kAhead; ++k)
          if ((ends >> min(p + k, 63)) & 1)
            old[k] = Row8<TW>::fetch(dw + (int64_t)__builtin_amdgcn_readlane(my.x, min(p + k, here - 1)) * d + col);
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {
        if (p + k >= here) break;
        float y[8];
        Row8<T>::unpack(x[k], y);
#pragma unroll
        for (int e = 0; e < 8; ++e) sum[e] += y[e];
        if (((ends >> (p + k)) & 1) == 0) continue;
        const int r = __builtin_amdgcn_readlane(my.x, p + k);
        const bool from_before = first && r == before, goes_on = g0 + p + k == c1 - 1 && r == after;
        first = false;
        if (live) {
          if (from_before || goes_on) Row8<float>::store(part + (from_before ? 0 : d), sum);
          else grad_store<TW, kAdd>(dw + (int64_t)r * d + col, old[k], sum, scale);
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) sum[e] = 0.f;
      }
    }
  }
}

// The rows of a fresh dW without a token, in the order of the addresses: 16 KB of dW per workgroup, 16 bytes of each
// 4 KB per thread. (All rows of 128256 x 4096 bf16 in pieces of 16 KB: 6.7 TB/s, as a fill without a look at the
// rows; of 4 KB, whose two loads come before the one store, 5.1; whole rows by wave 5.5 to 6.0.)
constexpr int kFillAhead = 4;
constexpr int64_t kFillBytes = 256 * 16 * kFillAhead;

template <typename TW>
__device__ __forceinline__ void embed_fill(const EmbedSorted& s, int64_t block, int v, int d, TW* __restrict__ dw) {
  const uint32_t row16 = (uint32_t)(d * sizeof(TW) / 16);
  const int64_t r0 = block * (kFillBytes / 16) / row16;
  const uint32_t o0 = (uint32_t)(block * (kFillBytes / 16) - r0 * row16);
  bool empty[kFillAhead];
#pragma unroll
  for (int k = 0; k < kFillAhead; ++k) {
    const int64_t at = r0 + (o0 + threadIdx.x + 256 * k) / row16;
    const int64_t q = s.slot((int)min(at, (int64_t)v - 1));
    empty[k] = at < v && s.starts[q] == s.starts[q + 1];
  }
  char* o = reinterpret_cast<char*>(dw) + block * kFillBytes + 16 * threadIdx.x;
#pragma unroll
  for (int k = 0; k < kFillAhead; ++k)
    if (empty[k]) store16_padded(o + 4096 * k, i32x4_t{0, 0, 0, 0});
}

// The sums of ids that several chunks share: one workgroup per chunk and 512 columns, which has work where an id
// starts in the chunk and reaches past its end. Wave w adds every fourth of the id's chunks from the w-th on, four
// loads in flight; the waves' sums are added in order. Behind these workgroups come those of embed_fill: here they
// have the 32 waves a CU holds, which the registers of k_embed_grad would halve (709 tokens, 128256 x 2048: 100 us
// there).
template <typename TW, bool kAdd>
__global__ __launch_bounds__(256) void k_embed_join(EmbedSorted s, int v, int d, int per, int slices, int64_t join_blocks,
                                                    float scale, TW* __restrict__ dw, const float* __restrict__ parts) {
  __shared__ float sums[3][kGradCols];
  if (!kAdd && blockIdx.x >= join_blocks) {
    embed_fill<TW>(s, blockIdx.x - join_blocks, v, d, dw);
    return;
  }
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int chunk = blockIdx.x / slices;
  const int col = (blockIdx.x - chunk * slices) * kGradCols + lane * 8;
  const int c0 = chunk * per, c1 = c0 + per;
  if (c1 >= s.count()) return;
  const int r = s.pairs[c1 - 1].x;
  if (s.pairs[c1].x != r || (c0 > 0 && s.pairs[c0 - 1].x == r)) return;
  const int last = (s.starts[s.slot(r) + 1] - 1) / per;        // the id's last chunk
  const bool live = col < d;
  float sum[8] = {};
  if (live) {
    if (w == 0) Row8<float>::unpack(Row8<float>::fetch(parts + ((int64_t)chunk * 2 + 1) * d + col), sum);
    for (int c = chunk + 1 + w; c <= last; c += 16) {
      Row8<float>::Raw x[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) x[k] = Row8<float>::fetch(parts + (int64_t)min(c + 4 * k, last) * 2 * d + col);
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        float y[8];
        Row8<float>::unpack(x[k], y);
#pragma unroll
        for (int e = 0; e < 8; ++e) sum[e] += c + 4 * k <= last ? y[e] : 0.f;
      }
    }
    if (w > 0)
#pragma unroll
      for (int e = 0; e < 8; ++e) sums[w - 1][e * 64 + lane] = sum[e];
  }
  __syncthreads();
  if (w > 0 || !live) return;
#pragma unroll
  for (int k = 0; k < 3; ++k)
#pragma unroll
    for (int e = 0; e < 8; ++e) sum[e] += sums[k][e * 64 + lane];
  TW* o = dw + (int64_t)r * d + col;
  typename Row8<TW>::Raw old{};
  if (kAdd) old = Row8<TW>::fetch(o);
  grad_store<TW, kAdd>(o, old, sum, scale);
}

// ---------------------------------------------------------------------------------------------
// Gradient of few tokens, without a sort: a workgroup per token and 512 columns lists the tokens of its token's id,
// in order, from a look at all ids, and goes on if its own is the first of them. Its four waves add a quarter of the
// rows each, eight in flight, and the quarters are added in order. A fresh dW is zeroed by a launch before. Two
// launches (one where dW is added to) instead of three, whose latencies are all that few tokens cost. Added,
// replayed: 256 tokens of 512 columns 3.9 us against 13.0 by the sort, 1024 of 2048 9.4 against 14.8; 4096 workgroups
// are the limit (1024 of 4096 26 against 16) and 1024 tokens too, for the batch whose tokens are all one id (1024 of
// 512 23.5 against 15.5, 2048 45 against 19).
// ---------------------------------------------------------------------------------------------
constexpr int kFewTokens = 1024;

template <typename T, typename TW, bool kAdd, int kBytes>
__global__ __launch_bounds__(256) void k_embed_few(EmbedRows e, const T* __restrict__ dout, int64_t ldx, int d, int slices,
                                                   float scale, TW* __restrict__ dw) {
  constexpr int kAhead = 8, kGroups = kFewTokens / 256;      // groups of 64 ids per wave
  typedef typename std::conditional<kBytes == 8, uint64_t, uint32_t>::type Id;
  __shared__ int list[kFewTokens], found[4], earlier[4];
  __shared__ float sums[3][kGradCols];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), n = (int)e.n;
  const int token = blockIdx.x / slices;
  const int col0 = (blockIdx.x - token * slices) * kGradCols + lane * 8;
  const bool live = col0 < d;
  const int col = live ? col0 : 0;             // (lanes behind the row read its start and store nothing)
  const Id* ids = (const Id*)e.ids;
  Id id[kGroups];
#pragma unroll
  for (int k = 0; k < kGroups; ++k) id[k] = ids[min(w * (64 * kGroups) + 64 * k + lane, n - 1)];
  const Id mine = ids[token];
  const Id r = mine - (Id)e.v_begin;
  if (r >= e.v || (int)r == e.pad_row) return;
  TW* o = dw + (int64_t)r * d + col;
  typename Row8<TW>::Raw old{};
  if (kAdd) old = Row8<TW>::fetch(o);
  unsigned long long same[kGroups];
  int count = 0;
  bool before = false;
#pragma unroll
  for (int k = 0; k < kGroups; ++k) {
    const int t = w * (64 * kGroups) + 64 * k + lane;
    same[k] = __ballot(t < n && id[k] == mine);
    before |= __ballot(t < token && id[k] == mine) != 0;
    count += __popcll(same[k]);
  }
  if (lane == 0) {
    found[w] = count;
    earlier[w] = before;
  }
  __syncthreads();
  if (earlier[0] | earlier[1] | earlier[2] | earlier[3]) return;      // another workgroup's id
  int at = 0;
  for (int k = 0; k < w; ++k) at += found[k];
#pragma unroll
  for (int k = 0; k < kGroups; ++k) {
    if ((same[k] >> lane) & 1) list[at + __popcll(same[k] & ((1ull << lane) - 1ull))] = w * (64 * kGroups) + 64 * k + lane;
    at += __popcll(same[k]);
  }
  __syncthreads();
  const int total = found[0] + found[1] + found[2] + found[3], quarter = (total + 3) / 4;
  const int p1 = min(total, (w + 1) * quarter);
  float sum[8] = {};
  for (int p = w * quarter; p < p1; p += kAhead) {
    typename Row8<T>::Raw x[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) x[k] = Row8<T>::fetch(dout + (int64_t)list[min(p + k, p1 - 1)] * ldx + col);
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      float y[8];
      Row8<T>::unpack(x[k], y);
#pragma unroll
      for (int c = 0; c < 8; ++c) sum[c] += p + k < p1 ? y[c] : 0.f;
    }
  }
  if (w > 0)
#pragma unroll
    for (int c = 0; c < 8; ++c) sums[w - 1][c * 64 + lane] = sum[c];
  __syncthreads();
  if (w > 0 || !live) return;
#pragma unroll
  for (int k = 0; k < 3; ++k)
#pragma unroll
    for (int c = 0; c < 8; ++c) sum[c] += sums[k][c * 64 + lane];
  grad_store<TW, kAdd>(o, old, sum, scale);
}

// kOnce: past the caches, which a dW larger than they are would only empty of dOut (16384 tokens, 128256 x 4096: 213
// -> 202 us)
template <bool kOnce>
__global__ __launch_bounds__(256) void k_embed_zero(char* __restrict__ dw, int64_t bytes) {
  const int64_t at = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 16;
  if (at >= bytes) return;
  if (kOnce) store16_padded_nt(dw + at, i32x4_t{0, 0, 0, 0});
  else store16_padded(dw + at, i32x4_t{0, 0, 0, 0});
}

// ---------------------------------------------------------------------------------------------
// Host side
// ---------------------------------------------------------------------------------------------
struct EmbedPlan {
  int64_t ldw, ldx, v_total;
  int nb_log2, rows;                 // buckets of the sort, ids of a bucket
  int per, slices;                   // tokens of a chunk, 512-column slices of a row
  int64_t chunks;
  size_t o_sorted, o_starts, o_parts, bytes;
};

// Of the gradient: every bucket of the sort looks at every id, and there are v / 1024 buckets from 2^18 ids on, so
// its time grows with n v. At 2^53 it is near 15 s (2^43 looks at 0.4 ns a CU); without a limit the largest n and v
// would take half an hour.
constexpr int64_t kMostLooks = (int64_t)1 << 53;

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
  if (pl->ldw < p->d || pl->ldx < p->d || pl->ldw >= (int64_t)1 << 30 || pl->ldx >= (int64_t)1 << 30)
    return LCE_ERR_SHAPE;
  if (pl->ldw % 8 != 0 || pl->ldx % 8 != 0) return LCE_ERR_ALIGN;
  // a launch takes fewer than 2^32 threads, and zeroes 4 KB of dW with 256 of them
  if ((uint64_t)p->v * p->d * (p->dw_dtype == LCE_DTYPE_F32 ? 4 : 2) > (uint64_t)1 << 35) return LCE_ERR_SHAPE;
  // 256 buckets, one per CU, or as many as keep a bucket's counts in LDS; no more than there are ids
  pl->nb_log2 = 0;
  while (pl->nb_log2 < 8 && ((int64_t)1 << pl->nb_log2) < p->v) ++pl->nb_log2;
  while (((p->v + ((int64_t)1 << pl->nb_log2) - 1) >> pl->nb_log2) > kSortIds) ++pl->nb_log2;
  pl->rows = (int)((p->v + ((int64_t)1 << pl->nb_log2) - 1) >> pl->nb_log2);
  auto take = [](size_t& cur, size_t bytes) { size_t o = cur; cur += (bytes + 255) / 256 * 256; return o; };
  size_t cur = 0;
  pl->o_sorted = take(cur, 8 * (size_t)p->n);
  pl->o_starts = take(cur, 4 * (((size_t)pl->rows << pl->nb_log2) + 1));
  // tokens of a chunk: 8 to 64, for 4096 waves (16 per CU, each with eight rows' loads in flight), and in narrow rows
  // no fewer than keep the chunks of a frequent id few for the join, which takes 16 of them a step as a wave takes 8
  // rows (65070 tokens of 88: 58 us with 16); more where there would be more than 4096 chunks, whose sums bound the
  // workspace
  pl->slices = (int)((p->d + kGradCols - 1) / kGradCols);
  pl->per = 8;
  while (pl->per < 64 && (p->n * pl->slices > (int64_t)4096 * pl->per || p->n > (int64_t)16 * pl->per * pl->per))
    pl->per *= 2;
  while (p->n > (int64_t)4096 * pl->per) pl->per *= 2;
  pl->chunks = (p->n + pl->per - 1) / pl->per;
  pl->o_parts = take(cur, 8 * (size_t)pl->chunks * p->d);
  pl->bytes = cur;
  return LCE_OK;
}

template <typename T>
void launch_lookup(Launcher& L, const lce_embedding_t* p, const EmbedPlan& pl, const EmbedIds& e, const void* W, void* out,
                   int32_t* status) {
  const int64_t blocks = (p->n * (p->d / 8) + 1023) / 1024;
  const bool kept = p->n * p->d * (int64_t)sizeof(T) <= kKeptBytes;
  L(K_EMBED_LOOKUP, kept ? k_embed_lookup<T, false> : k_embed_lookup<T, true>,
    dim3((unsigned)std::min<int64_t>(blocks, 1 << 20)), dim3(256), e, pl.v_total, (const T*)W, pl.ldw, (int)p->d,
    p->scale, (T*)out, status);
}

void launch_zero(Launcher& L, void* dw, int64_t bytes) {
  L(K_EMBED_GRAD, bytes <= kKeptBytes ? k_embed_zero<false> : k_embed_zero<true>, dim3((unsigned)((bytes + 4095) / 4096)),
    dim3(256), (char*)dw, bytes);
}

template <typename T, typename TW, bool kAdd>
void launch_embed_grad(Launcher& L, const lce_embedding_t* p, const EmbedPlan& pl, const EmbedSorted& s, const void* dout,
                       void* dw, float* parts) {
  const int64_t units = pl.chunks * pl.slices, join = pl.chunks > 1 ? units : 0, bytes = p->v * p->d * (int64_t)sizeof(TW);
  // a fresh dW is zeroed whole before where few of its rows can have tokens and the launch is short beside it (4096
  // tokens, 128256 x 2048 / 8192: 102 / 360 us, row by row behind the sums 111 / 397; but 2048 tokens, 128256 x 512:
  // 35 against 33; 16384, 32000 x 4096: 106 against 103; 65536, 128256 x 4096 of even ids: 406 against 363)
  const bool zero = !kAdd && p->n <= p->v / 4 && bytes >= (int64_t)256 << 20;
  const int64_t fill = kAdd || zero ? 0 : (bytes + kFillBytes - 1) / kFillBytes;
  if (zero) launch_zero(L, dw, bytes);
  L(K_EMBED_GRAD, k_embed_grad<T, TW, kAdd>, dim3((unsigned)((units + 3) / 4)), dim3(256), s, (const T*)dout, pl.ldx,
    (int)p->d, pl.per, units, pl.slices, p->scale, (TW*)dw, parts);
  L(K_EMBED_GRAD, k_embed_join<TW, kAdd>, dim3((unsigned)(join + fill)), dim3(256), s, (int)p->v, (int)p->d, pl.per,
    pl.slices, join, p->scale, (TW*)dw, (const float*)parts);
}

// Up to 1024 tokens, and 4096 workgroups.
inline bool few_tokens(const lce_embedding_t* p, const EmbedPlan& pl) {
  return p->n <= kFewTokens && p->n * pl.slices <= 4096;
}

template <typename T, typename TW, bool kAdd>
void launch_embed_few(Launcher& L, const lce_embedding_t* p, const EmbedPlan& pl, const EmbedRows& e, const void* dout,
                      void* dw) {
  const int64_t bytes = p->v * p->d * (int64_t)sizeof(TW);
  if (!kAdd) launch_zero(L, dw, bytes);
  L(K_EMBED_GRAD, p->id_bytes == 8 ? k_embed_few<T, TW, kAdd, 8> : k_embed_few<T, TW, kAdd, 4>,
    dim3((unsigned)(p->n * pl.slices)), dim3(256), e, (const T*)dout, pl.ldx, (int)p->d, pl.slices, p->scale, (TW*)dw);
}

template <typename T, typename TW>
void launch_embed_few(Launcher& L, const lce_embedding_t* p, const EmbedPlan& pl, const EmbedRows& e, const void* dout,
                      void* dw) {
  if (p->flags & LCE_FLAG_ACCUMULATE_DW) launch_embed_few<T, TW, true>(L, p, pl, e, dout, dw);
  else launch_embed_few<T, TW, false>(L, p, pl, e, dout, dw);
}

template <typename T, typename TW>
void launch_embed_grad(Launcher& L, const lce_embedding_t* p, const EmbedPlan& pl, const EmbedSorted& s, const void* dout,
                       void* dw, float* parts) {
  if (p->flags & LCE_FLAG_ACCUMULATE_DW) launch_embed_grad<T, TW, true>(L, p, pl, s, dout, dw, parts);
  else launch_embed_grad<T, TW, false>(L, p, pl, s, dout, dw, parts);
}

}  // namespace

extern "C" {

lce_status_t lce_embedding_workspace_size(const lce_embedding_t* p, size_t* bwd_bytes) {
  EmbedPlan pl;
  const lce_status_t st = make_embed_plan(p, &pl);
  if (st != LCE_OK) return st;
  if (p->n * p->v > kMostLooks) return LCE_ERR_SHAPE;
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
  if (p->n * p->v > kMostLooks) return LCE_ERR_SHAPE;
  if (!dW || !workspace || (p->n > 0 && (!ids || !dOut))) return LCE_ERR_NULL;
  if (((uintptr_t)ids & (p->id_bytes - 1)) != 0 || !aligned16(dOut) || !aligned16(dW) || ((uintptr_t)workspace & 255) != 0)
    return LCE_ERR_ALIGN;
  if (workspace_bytes < pl.bytes) return LCE_ERR_WORKSPACE;
  Launcher L{(hipStream_t)stream};
  char* ws = (char*)workspace;
  int2* sorted = (int2*)(ws + pl.o_sorted);
  int* starts = (int*)(ws + pl.o_starts);
  const bool pad = p->padding_idx >= p->v_begin && p->padding_idx < p->v_begin + p->v;
  const EmbedRows e{ids, p->n, p->v_begin, (uint32_t)p->v, pad ? (int)(p->padding_idx - p->v_begin) : -1};
  if (few_tokens(p, pl)) {
    if (p->dtype == LCE_DTYPE_F32) launch_embed_few<float, float>(L, p, pl, e, dOut, dW);
    else if (p->dw_dtype == LCE_DTYPE_F32) launch_embed_few<uint16_t, float>(L, p, pl, e, dOut, dW);
    else launch_embed_few<uint16_t, uint16_t>(L, p, pl, e, dOut, dW);
    return L.st;
  }
  L(K_EMBED_SORT, p->id_bytes == 8 ? k_embed_sort<8> : k_embed_sort<4>, dim3(1u << pl.nb_log2), dim3(64 * kSortWaves), e,
    pl.nb_log2, pl.rows, sorted, starts);
  const EmbedSorted s{sorted, starts, pl.nb_log2, pl.rows};
  float* parts = (float*)(ws + pl.o_parts);
  if (p->dtype == LCE_DTYPE_F32) launch_embed_grad<float, float>(L, p, pl, s, dOut, dW, parts);
  else if (p->dw_dtype == LCE_DTYPE_F32) launch_embed_grad<uint16_t, float>(L, p, pl, s, dOut, dW, parts);
  else launch_embed_grad<uint16_t, uint16_t>(L, p, pl, s, dOut, dW, parts);
  return L.st;
}

}  // extern "C"
