// selkv_tree_attn: attention of the nodes of drafted trees over a paged cache,
// with the additive logit bias of Sec. 3.6.
//
//   out_i = sum_e softmax_e(scale q_i k_e + bias_e) v_e   over e < len and the nodes above i
//
// The rows of a KV head are its G query heads at every node.  A wave takes tiles
// of 16 rows and 32 entries at a time: S = K Q^T as two 16x16 tiles, the softmax
// in S's own layout, O^T += V^T P^T.  Lane (column, grp) = (lane % 16, lane / 16)
// holds row `column` and, of the 32 entries, 8 grp .. 8 grp + 7: which entry is
// which row of an S tile is chosen so, and P goes from S's layout into the next
// product as it is.  V comes as rows, 16 lanes side by side: lane (column, grp)
// reads channels column d/16 .. of its eight entries, one run of 16 bytes each,
// and what the product needs, eight entries of one channel in a lane, is a
// permutation of the lane's own registers.  Channel column d/16 + i is row
// `column` of O^T tile i.  So up to 32 rows a KV head K and V go from memory to
// registers once, without LDS; with more rows eight waves share tiles of them
// in LDS, read in the same lanes and order.
//
// What bounds it, over 8 heads of 25600 entries of d = 128 in bf16: with 20 rows
// (5 nodes) memory, 23.3 us and 4.7 TB/s, and 32 such caches in one call
// 569 us, 6.0 TB/s; with 256 rows (64 nodes) the instructions of the softmax and
// the matrix cores, which two waves of a SIMD overlap only in part: 70 us, 380
// TFLOP/s.  The kernel that combines adds 4.6 and 8.2 us.  fp32 at d = 128 has
// registers for one wave a SIMD: 64 nodes 308 us, 87 TFLOP/s, 5 nodes 50 to 57.
//
// bf16 weights enter the product as sums of two bf16 numbers (2^-17 of a weight
// is left; one number, 70 us where two take 79, is 1.4 times as far from 64 bits
// as fp32 torch), fp32 ones as they are.  Maxima, sums and accumulators are fp32.
//
// Masks.  Entries past the end, on no page or (for a node) outside its chain of
// parents are left out by selection in the tiles that hold such; a masked bias
// makes a logit -inf by itself.  Where a result comes out NaN, infinite or past
// 2^96 the wave does its entries again in a careful pass, in which every tile
// selects masked biases too, V's values that are NaN or infinite are kept out of
// the product, where a weight of 0 would turn them into NaN for every row, and are
// added to the rows that attend to them.  Its weights are a power of two smaller,
// so that no sum of finite values overflows: a mean of finite values is finite.
//
// Split-K: a workgroup takes a run of entries, and a second kernel combines the
// runs' (max, sum, o) in order.
#include <algorithm>

#include "paged.hpp"

namespace selkv {
namespace {

constexpr int kTile = 32;              // entries of a wave's step
constexpr int kCUs = 256;
constexpr uint32_t kParts = 8;         // of the chip
constexpr int kMaxSplit = 256;
constexpr int kMaxRounds = 4;          // of workgroups, one a CU
constexpr int kRaggedRounds = 2;
constexpr int kFewRowsRounds = 6;      // up to 32 rows
constexpr int kGroupCost = 160;        // of a workgroup, and of the second kernel, in entries
constexpr int kCombineCost = 256;
constexpr int kFewSlots = 8;           // up to which a row is combined by d/4 threads; from kManyRows rows on always
constexpr uint32_t kManyRows = 8192;   // (the ragged call of 128 heads and 208 rows in 10 splits 136 us, 157 without)

struct TreeArgs {
  Paged c;
  Seqs n;
  const char* q;
  const int32_t* parent;
  char* out;
  float* part_o;     // [B hkv, splits, n G, D]
  float2* part_ml;   // [B hkv, splits, n G]
  int hkv, G, splits, row_blocks, step;
  uint32_t heads;    // of all sequences
  float scale;
};

struct Sequence {
  uint32_t b;
  int len, count;    // count 0: it takes no part
};

// The sequence that comes at `place`: longest first, in groups of 64, so that the last workgroups of a call are short
// (16 sequences of 0 to 8100 entries, 26 nodes, 8 heads, G 8: 130 us, in the caller's order 167).
__device__ __forceinline__ Sequence sequence_at(const Seqs& s, uint32_t place, uint32_t batch, int lane) {
  Sequence q;
  const uint32_t first = s.lens ? place & ~63u : place;
  const int n = s.lens ? (int)min(64u, batch - first) : 1;
  int work = -1, len = 0, count = 0;     // of the lane's sequence
  if (lane < n) {
    if (!sequence_of(s, first + lane, len, count)) count = 0;
    work = count > 0 ? len + count : 0;
  }
  int rank = 0;
  for (int j0 = 0; j0 < n; j0 += 8) {
#pragma unroll
    for (int j = j0; j < j0 + 8; ++j) {
      const int other = __builtin_amdgcn_readlane(work, j);
      rank += other > work || (other == work && j < lane);
    }
  }
  const int at = __ffsll((unsigned long long)__ballot(lane < n && rank == (int)(place - first))) - 1;
  q.b = first + at;
  q.len = __builtin_amdgcn_readlane(len, at);
  q.count = __builtin_amdgcn_readlane(count, at);
  return q;
}

// Head (of all sequences) and place within its `per` of a block.  Blocks go to the eight parts of the chip in turn, and
// each part has a cache of its own: all blocks of a head are on one part, if the heads divide into eight, so that what
// the splits write is in the cache from which the combining kernel reads it (16 nodes over 25600 entries 39.0 us, with
// the heads over all parts 40.0; 5 nodes 27.0 and 27.4).
struct Place {
  uint32_t head, inner;
};
__device__ __forceinline__ Place place_of(uint32_t block, uint32_t heads, uint32_t per) {
  const uint32_t parts = heads % kParts == 0 ? kParts : 1;
  const uint32_t part = block % parts, rest = block / parts, group = rest / per;
  return {group * parts + part, rest - group * per};
}

// Tiles of 32 entries that a wave of a shared tile takes one after the other: with two there are half as many barriers
// (64 nodes over 25600 entries 78.4 us, 80.4 with one).
constexpr int tiles_of_turn(int key_groups) { return key_groups == 1 ? 2 : 1; }

// Entries of a split of a sequence of `total`: as many splits as there are, of whole steps.
__device__ __forceinline__ int chunk_of(const TreeArgs& a, int total) {
  const uint32_t per = ((uint32_t)total + a.splits - 1) / (uint32_t)a.splits, step = a.step;
  return (int)(max((per + step - 1) / step, 1u) * step);
}

// What sums with maximum m count for beside M.  One below fp32's range is its smallest number: nothing to finite sums, and
// infinite ones stay infinite (0 would make them NaN, by where their entries lie; chosen by value 32.6 us where 28.1).
__device__ __forceinline__ float weight_of(float m, float M) {
  return m == kNegInf ? 0.f : fmaxf(fast_exp2((m - M) * kLog2e), 0x1p-149f);
}

// The maximum that goes with a sum: fmaxf passes a NaN logit by, so where the sum is NaN a part keeps a maximum that
// makes it count.
__device__ __forceinline__ float nan_counts(float m, float l) { return l == l || m != kNegInf ? m : 0.f; }

__device__ __forceinline__ bool finite(float x) { return fabsf(x) < __builtin_huge_valf(); }

__device__ __forceinline__ float max_xor16(float v) {
  const uint32_t u = __float_as_uint(v);
  const auto r = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float max_xor32(float v) {
  const uint32_t u = __float_as_uint(v);
  const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

// For lane i: the nodes that node i attends to, itself included, as bits.  Six doublings reach the root of 64 nodes.
__device__ __forceinline__ uint64_t ancestors(const int32_t* parent, int n, int lane) {
  uint64_t seen = 1ull << lane;
  int up = parent ? (lane < n ? parent[lane] : -1) : lane - 1;
  if ((uint32_t)up >= (uint32_t)lane) up = -1;
#pragma unroll
  for (int i = 0; i < 6; ++i) {
    const int from = up < 0 ? lane : up;
    const uint64_t above = __shfl((unsigned long long)seen, from, 64);
    const int next = __shfl(up, from, 64);
    if (up >= 0) {
      seen |= above;
      up = next;
    }
  }
  return seen;
}

// The pages of the table's columns from `first` on, one in each lane of the wave, -1 where there is none.
struct PageWindow {
  int first, page;
  __device__ __forceinline__ void fill(const Paged& c, uint32_t b, int column, int lane) {
    first = column;
    page = c.table[(size_t)b * c.columns + min(column + lane, c.columns - 1)];
    if ((uint32_t)page >= (uint32_t)c.n_pages || column + lane >= c.columns) page = -1;
  }
  // Where the first entry from the window's on is that has no page, `whole` at most.
  __device__ __forceinline__ int up_to(const Paged& c, int whole) const {
    const uint64_t none = __ballot(page < 0);
    return none ? min(whole, (first + __ffsll((unsigned long long)none) - 1) << c.shift) : whole;
  }
  __device__ __forceinline__ bool holds(const Paged& c, int from, int to) const {
    return (from >> c.shift) >= first && (to >> c.shift) < first + 64;
  }
  __device__ __forceinline__ int at(const Paged& c, int entry) const {
    return __shfl(page, (entry >> c.shift) - first, 64);
  }
};

// What a wave reads for 32 entries: 16-byte chunks of the K rows of its two tiles and the biases of entries 8 grp .. + 7,
// and its words of the V rows of these.
template <typename T, int D>
struct Keys {
  static constexpr int N = D * (int)sizeof(T) / 64;
  Chunk16 k[2][N];
  float bias[8];
  __device__ __forceinline__ void load(const Paged& c, int hkv, int head, int base, int pk, int pv, int col, int grp) {
    constexpr int RB = D * (int)sizeof(T);
    const char* kp = c.K + row_of(c, hkv, pk, head, base + 8 * (col >> 2) + (col & 3)) * RB + grp * 16;
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int j = 0; j < N; ++j) k[t][j] = load16(kp + 4 * t * RB + j * 64);
    // without biases the pool of K is read in their place (it is larger) and passed over: no branch between the loads
    const float* bp =
        (c.bias ? c.bias : reinterpret_cast<const float*>(c.K)) + row_of(c, hkv, pv, head, base + 8 * grp);
    const Chunk16 b0 = load16(bp), b1 = load16(bp + 4);
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      bias[s] = __uint_as_float(b0.w[s]);
      bias[4 + s] = __uint_as_float(b1.w[s]);
    }
  }
};

template <typename T, int D>
struct Values {
  static constexpr int N = D * (int)sizeof(T) / 64;
  uint32_t v[8][N];
  __device__ __forceinline__ void load(const Paged& c, int hkv, int head, int base, int pv, int col, int grp) {
    constexpr int RB = D * (int)sizeof(T);
    const char* vp = c.V + row_of(c, hkv, pv, head, base + 8 * grp) * RB + col * (RB / 16);
#pragma unroll
    for (int s = 0; s < 8; ++s) {
      if constexpr (RB / 16 >= 16) {
#pragma unroll
        for (int i = 0; i < RB / 256; ++i) {
          const Chunk16 w = load16(vp + s * RB + i * 16);
#pragma unroll
          for (int k = 0; k < 4; ++k) v[s][4 * i + k] = w.w[k];
        }
      } else {
        const uint2 w = *reinterpret_cast<const uint2*>(vp + s * RB);
        v[s][0] = w.x;
        v[s][1] = w.y;
      }
    }
  }
};

// The same from a tile in LDS.  Rows are RB bytes one after the other.  Of K, 16-byte chunk c of row r is at chunk
// c ^ swizzle(r), so that the rows whose chunks c are read together, 8 a + b with a = 0, 1 and b = 0 .. 3, are on
// different banks; a V row is read as it lies, and with a swizzle conflicts with the row eight further on.
__device__ __forceinline__ int swizzle(int row) { return (row & 3) | ((row >> 1) & 4); }

// The places of a lane's chunks: only bit 2 of the swizzle meets bits of j, so few are kept.
template <typename T, int D>
struct Places {
  static constexpr int RB = D * (int)sizeof(T);
  int k[2], v, bias;
  __device__ __forceinline__ Places(int col, int grp) {
    const int row = 8 * (col >> 2) + (col & 3);
#pragma unroll
    for (int j = 0; j < 2; ++j) k[j] = row * RB + (((4 * j + grp) ^ swizzle(row)) << 4);
    v = 8 * grp * RB + col * (RB / 16);
    bias = 32 * grp;
  }
};

template <typename T, int D>
__device__ __forceinline__ void read_keys(Keys<T, D>& x, const char* tile, const char* bias, const Places<T, D>& at) {
  constexpr int RB = D * (int)sizeof(T);
#pragma unroll
  for (int t = 0; t < 2; ++t)
#pragma unroll
    for (int j = 0; j < Keys<T, D>::N; ++j) x.k[t][j] = load16(tile + at.k[j & 1] + (j >> 1) * 128 + 4 * t * RB);
  const Chunk16 b0 = load16(bias + at.bias), b1 = load16(bias + at.bias + 16);
#pragma unroll
  for (int s = 0; s < 4; ++s) {
    x.bias[s] = __uint_as_float(b0.w[s]);
    x.bias[4 + s] = __uint_as_float(b1.w[s]);
  }
}

template <typename T, int D>
__device__ __forceinline__ void read_values(Values<T, D>& x, const char* tile, const Places<T, D>& at) {
  constexpr int RB = D * (int)sizeof(T);
#pragma unroll
  for (int s = 0; s < 8; ++s) {
    const char* from = tile + at.v + s * RB;
    if constexpr (RB / 16 >= 16) {
#pragma unroll
      for (int i = 0; i < RB / 256; ++i) {
        const Chunk16 w = load16(from + 16 * i);
#pragma unroll
        for (int k = 0; k < 4; ++k) x.v[s][4 * i + k] = w.w[k];
      }
    } else {
      const uint2 w = *reinterpret_cast<const uint2*>(from);
      x.v[s][0] = w.x;
      x.v[s][1] = w.y;
    }
  }
}

// Softmax state of a wave's row tile: lane (column, grp) keeps its row's maximum, the sum over the entries it holds,
// and channels (D/16)(4 grp + r) + i of the row as o[i][r].
template <int D>
struct RowTile {
  float m, l;
  bool far;              // the same in all lanes: a maximum of the wave's is beyond kFar (of its first tile alone)
  f32x4 o[D / 16];
};

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

// x as a sum of two bf16 numbers, two values to a word.
__device__ __forceinline__ void split2(float x0, float x1, uint32_t& hi, uint32_t& lo) {
  hi = __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{x0, x1}, bf16x2));
  x0 -= __uint_as_float(hi << 16);
  x1 -= __uint_as_float(hi & 0xffff0000u);
  lo = __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{x0, x1}, bf16x2));
}

// O^T += V^T P^T for RT row tiles whose weights are p.
template <typename T, int D, int RT>
__device__ __forceinline__ void add_values(RowTile<D> (&st)[RT], const uint32_t (&v)[8][Values<T, D>::N],
                                           const float (&p)[RT][8]) {
  if constexpr (sizeof(T) == 2) {
    Chunk16 hi[RT], lo[RT];
#pragma unroll
    for (int t = 0; t < RT; ++t)
#pragma unroll
      for (int k = 0; k < 4; ++k) split2(p[t][2 * k], p[t][2 * k + 1], hi[t].w[k], lo[t].w[k]);
#pragma unroll
    for (int i = 0; i < D / 16; ++i) {
      Chunk16 a;
#pragma unroll
      for (int k = 0; k < 4; ++k)
        a.w[k] = __builtin_amdgcn_perm(v[2 * k + 1][i / 2], v[2 * k][i / 2], i % 2 ? 0x07060302u : 0x05040100u);
#pragma unroll
      for (int t = 0; t < RT; ++t) {
        st[t].o[i] = Mma<T>::step(a, lo[t], st[t].o[i]);
        st[t].o[i] = Mma<T>::step(a, hi[t], st[t].o[i]);
      }
    }
  } else {
#pragma unroll
    for (int s = 0; s < 8; ++s)
#pragma unroll
      for (int i = 0; i < D / 16; ++i)
#pragma unroll
        for (int t = 0; t < RT; ++t)
          st[t].o[i] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(v[s][i]), p[t][s], st[t].o[i], 0, 0, 0);
  }
}

// The values of a row that are NaN or infinite, added to the rows that attend to the entry.
template <typename T, int D, int RT>
__device__ __forceinline__ void add_unbounded(RowTile<D> (&st)[RT], const char* row, const bool (&seen)[RT], int grp) {
  constexpr int N = D / 16;
#pragma unroll
  for (int r = 0; r < 4; ++r)
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const char* at = row + (N * (4 * grp + r) + i) * (int)sizeof(T);
      float x;
      if constexpr (sizeof(T) == 2) x = bf16_to_f32(*reinterpret_cast<const bf16_t*>(at));
      else x = *reinterpret_cast<const float*>(at);
      if (!finite(x)) {
#pragma unroll
        for (int t = 0; t < RT; ++t)
          if (seen[t]) st[t].o[i][r] += x;
      }
    }
}

template <typename T>
__device__ __forceinline__ uint32_t zero_unbounded(uint32_t w, bool& any) {
  constexpr uint32_t kExp = 0x7f800000u;
  if constexpr (sizeof(T) == 2) {
    const bool h = (w & kExp) == kExp, l = ((w << 16) & kExp) == kExp;
    any = any || h || l;
    return (h ? 0u : w & 0xffff0000u) | (l ? 0u : w & 0xffffu);
  } else {
    const bool f = (w & kExp) == kExp;
    any = any || f;
    return f ? 0u : w;
  }
}

template <typename T, int D, int RT>
struct Rows {
  Chunk16 q[RT][Keys<T, D>::N];
  uint64_t seen[RT];   // the nodes that the row attends to
};

// Logits of 32 entries, S = K Q^T scaled and biased.
template <typename T, int D, int RT>
__device__ __forceinline__ void logits(float (&p)[RT][8], const Keys<T, D>& x, const Rows<T, D, RT>& rows, float scale,
                                       bool has_bias) {
#pragma unroll
  for (int t = 0; t < RT; ++t)
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int j = 0; j < Keys<T, D>::N; ++j) s = Mma<T>::step(x.k[h][j], rows.q[t][j], s);
#pragma unroll
      for (int r = 0; r < 4; ++r) p[t][4 * h + r] = fmaf(s[r], scale, has_bias ? x.bias[4 * h + r] : 0.f);
    }
}

// A row's maximum follows its logits only when they are this far above it, so that after the first tiles of a row hardly a
// tile has to rescale what is there (one of 32 rows is enough for that: 172 us where 183 without, 16 sequences of 0 to
// 8100 entries, 26 nodes).  Weights are up to e^6 then, which their relative rounding does not mind, nor do fp32 sums up to
// kRoom.
constexpr float kSlack = 6.f;

// A bf16 row whose maximum is beyond this has it taken off its logits before the fma that turns them to powers of two.  The
// fma takes off the maximum times log2(e), rounded, so it puts one factor on all weights of a row: up to here within 2^-14
// of 1, as much as a logit's own rounding; 2^64 or its inverse at 1e9, out of any range at 1e11.
constexpr float kFar = 1024.f;

// Logits to weights, with the running maximum and sum; the weights are multiplied by `lower`.
template <bool FUSED, int D, int RT>
__device__ __forceinline__ void soften(RowTile<D> (&st)[RT], float (&p)[RT][8], float lower) {
  float top[RT];
  bool above = false;
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    float mx = p[t][0];
#pragma unroll
    for (int s = 1; s < 8; ++s) mx = fmaxf(mx, p[t][s]);
    top[t] = max_xor32(max_xor16(mx));
    above = above || top[t] > st[t].m + kSlack;
  }
  if (__builtin_expect(__any(above), 0)) {
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      const float m = top[t] > st[t].m + kSlack ? top[t] : st[t].m;   // by row: none depends on the others
      const float corr = m == st[t].m ? 1.f : weight_of(st[t].m, m);
      st[t].l *= corr;
#pragma unroll
      for (int i = 0; i < D / 16; ++i) st[t].o[i] *= corr;
      st[t].m = m;
    }
    if (FUSED) {
      bool far = false;
#pragma unroll
      for (int t = 0; t < RT; ++t) far = far || (fabsf(st[t].m) > kFar && st[t].m != kNegInf);
      st[0].far = __any(far);
    }
  }
  float ref[RT];
#pragma unroll
  for (int t = 0; t < RT; ++t) ref[t] = st[t].m == kNegInf ? 0.f : st[t].m;   // nothing unmasked yet: every weight is 0
  if (FUSED && __builtin_expect(st[0].far, 0)) {
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      const float first = fabsf(ref[t]) > kFar ? ref[t] : 0.f;   // by row here too
#pragma unroll
      for (int s = 0; s < 8; ++s) p[t][s] -= first;
      ref[t] -= first;
    }
  }
#pragma unroll
  for (int t = 0; t < RT; ++t) {
#pragma unroll
    for (int s = 0; s < 8; ++s) {
      if (FUSED) p[t][s] = fast_exp2(fmaf(p[t][s], kLog2e, -ref[t] * kLog2e));
      else p[t][s] = fast_exp2((p[t][s] - ref[t]) * kLog2e);
      p[t][s] *= lower;
      st[t].l += p[t][s];
    }
  }
}

// A step whose 32 entries from `base` may be behind len, the entries that all rows attend to, behind end, the nodes after
// them, or on no page (pv < 0); or one of a careful pass, whose weights are `lower` (1 otherwise).
template <typename T, int D, int RT>
__device__ __forceinline__ void attend_edge(RowTile<D> (&st)[RT], const Keys<T, D>& k, Values<T, D>& x,
                                            const Rows<T, D, RT>& rows, const TreeArgs& a, uint32_t b, int head, int base,
                                            int len, int end, int pv, float lower, int grp) {
  const bool careful = lower < 1.f;
  float p[RT][8];
  logits<T, D, RT>(p, k, rows, a.scale, a.c.bias != nullptr);
  bool unbounded = false;
#pragma unroll
  for (int s = 0; s < 8; ++s) {
    const int entry = base + 8 * grp + s, node = entry - len;
    const bool live = pv >= 0 && entry < end && !(a.c.bias && k.bias[s] == kNegInf);
#pragma unroll
    for (int t = 0; t < RT; ++t)
      if (!(live && (node < 0 || ((rows.seen[t] >> (node & 63)) & 1)))) p[t][s] = kNegInf;
#pragma unroll
    for (int w = 0; w < Values<T, D>::N; ++w) {
      if (!live) x.v[s][w] = 0u;
      else if (careful) x.v[s][w] = zero_unbounded<T>(x.v[s][w], unbounded);
    }
  }
  soften<sizeof(T) == 2, D, RT>(st, p, lower);
  add_values<T, D, RT>(st, x.v, p);
  if (careful && __any(unbounded)) {
    for (int s = 0; s < kTile; ++s) {
      const int entry = base + s, node = entry - len;
      const int page = entry < end ? page_of(a.c, b, entry) : -1;
      if (page < 0) continue;
      const size_t row = row_of(a.c, a.hkv, page, head, entry);
      if (a.c.bias && a.c.bias[row] == kNegInf) continue;
      bool seen[RT];
#pragma unroll
      for (int t = 0; t < RT; ++t) seen[t] = node < 0 || ((rows.seen[t] >> (node & 63)) & 1);
      add_unbounded<T, D, RT>(st, a.c.V + row * D * sizeof(T), seen, grp);
    }
  }
}

// Steps of a wave from e on, entries of any kind.  loaded: the first step's keys and values are on their way already.
template <typename T, int D, int RT>
__device__ __forceinline__ void attend_edges(RowTile<D> (&st)[RT], Keys<T, D>& k, Values<T, D>& v, bool loaded,
                                             const Rows<T, D, RT>& rows, const TreeArgs& a, uint32_t b, int head, int e,
                                             int e1, int step, int len, int end, float lower, PageWindow& pages,
                                             int lane) {
  const int col = lane & 15, grp = lane >> 4;
  for (; e < e1; e += step) {
    if (!pages.holds(a.c, e, e + kTile - 1)) pages.fill(a.c, b, e >> a.c.shift, lane);
    const int pv = pages.at(a.c, e + 8 * grp);
    if (!loaded) {
      k.load(a.c, a.hkv, head, e, max(pages.at(a.c, e + 8 * (col >> 2)), 0), max(pv, 0), col, grp);
      v.load(a.c, a.hkv, head, e, max(pv, 0), col, grp);
    }
    loaded = false;
    attend_edge<T, D, RT>(st, k, v, rows, a, b, head, e, len, end, pv, lower, grp);
  }
}

template <typename T, int D>
__device__ __forceinline__ void store_row(char* row, const f32x4 (&o)[D / 16], int grp) {
  constexpr int N = D / 16;
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    char* at = row + N * (4 * grp + r) * (int)sizeof(T);
    if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int i = 0; i < N; i += 4)
        *reinterpret_cast<f32x4*>(at + 4 * i) = f32x4{o[i][r], o[i + 1][r], o[i + 2][r], o[i + 3][r]};
    } else {
      uint32_t w[N / 2];
#pragma unroll
      for (int i = 0; i < N; i += 2) w[i / 2] = f32_to_bf16(o[i][r]) | (uint32_t)f32_to_bf16(o[i + 1][r]) << 16;
      if constexpr (N == 8) *reinterpret_cast<uint4*>(at) = make_uint4(w[0], w[1], w[2], w[3]);
      else *reinterpret_cast<uint2*>(at) = make_uint2(w[0], w[1]);
    }
  }
}

// The end of a split: the results of the KG waves that share rows meet in LDS, two and two, and go to the outputs or the
// workspace.  s_o: RG KG / 2 runs of RT d/16 x 64 slots, s_ml: of RT x 64.
template <typename T, int D, int RT, int RG, int KG>
__device__ __forceinline__ void finish(RowTile<D> (&st)[RT], f32x4* s_o, float2* s_ml, const TreeArgs& a, uint32_t b,
                                       int head, int row0, int nrows, int split, int rw, int kw, int lane) {
  constexpr int RB = D * (int)sizeof(T);
  const int col = lane & 15, grp = lane >> 4;
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    st[t].l = add_xor32(add_xor16(st[t].l));
    st[t].m = nan_counts(st[t].m, st[t].l);
  }
#pragma unroll
  for (int step = KG / 2; step > 0; step /= 2) {
    const int slot = rw * step + (kw >= step ? kw - step : kw);
    f32x4* so = s_o + slot * RT * (D / 16) * 64 + lane;
    float2* sm = s_ml + slot * RT * 64 + lane;
    if (kw >= step && kw < 2 * step) {
#pragma unroll
      for (int t = 0; t < RT; ++t) {
        sm[t * 64] = make_float2(st[t].m, st[t].l);
#pragma unroll
        for (int i = 0; i < D / 16; ++i) so[(t * (D / 16) + i) * 64] = st[t].o[i];
      }
    }
    __syncthreads();
    if (kw < step) {
#pragma unroll
      for (int t = 0; t < RT; ++t) {
        const float2 ml = sm[t * 64];
        const float M = fmaxf(st[t].m, ml.x);
        const float c0 = weight_of(st[t].m, M), c1 = weight_of(ml.x, M);
        const bool some0 = st[t].m != kNegInf, some1 = ml.x != kNegInf;   // a part without entries has weight 0 and 0s
        st[t].l = (some0 ? st[t].l * c0 : 0.f) + (some1 ? ml.y * c1 : 0.f);
#pragma unroll
        for (int i = 0; i < D / 16; ++i) {
          const f32x4 o = so[(t * (D / 16) + i) * 64];
#pragma unroll
          for (int r = 0; r < 4; ++r) st[t].o[i][r] = (some0 ? st[t].o[i][r] * c0 : 0.f) + (some1 ? o[r] * c1 : 0.f);
        }
        st[t].m = M;
      }
    }
    __syncthreads();
  }
  if (kw > 0) return;
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    const int r = row0 + 16 * t + col;
    if (r >= nrows) continue;
    if (a.splits == 1) {
      const int node = r / a.G, g = r - node * a.G;
      f32x4 o[D / 16];
#pragma unroll
      for (int i = 0; i < D / 16; ++i)
#pragma unroll
        for (int k = 0; k < 4; ++k) o[i][k] = st[t].l == 0.f ? 0.f : st[t].o[i][k] / st[t].l;
      store_row<T, D>(a.out + ((((size_t)b * a.n.n + node) * a.hkv + head) * a.G + g) * RB, o, grp);
    } else {
      const size_t part = (((size_t)b * a.hkv + head) * a.splits + split) * ((size_t)a.n.n * a.G) + r;
      store_row<float, D>(reinterpret_cast<char*>(a.part_o + part * D), st[t].o, grp);
      if (grp == 0) a.part_ml[part] = make_float2(st[t].m, st[t].l);
    }
  }
}

// Queries of a wave's rows and the nodes that they attend to (`anc`: ancestors() of the lane's node).
template <typename T, int D, int RT>
__device__ __forceinline__ void load_rows(Rows<T, D, RT>& rows, const TreeArgs& a, uint32_t b, int head, int row0,
                                          int nrows, uint64_t anc, int col, int grp) {
  constexpr int RB = D * (int)sizeof(T);
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    const int r = row0 + 16 * t + col, node = r < nrows ? r / a.G : 0, g = r < nrows ? r - node * a.G : 0;
    const char* qr = a.q + (((size_t)b * a.n.n + node) * a.hkv + head) * a.G * RB + (size_t)g * RB + grp * 16;
#pragma unroll
    for (int j = 0; j < Keys<T, D>::N; ++j) rows.q[t][j] = load16(qr + j * 64);
    rows.seen[t] = __shfl((unsigned long long)anc, node, 64);
  }
}

template <int D, int RT>
__device__ __forceinline__ void clear(RowTile<D> (&st)[RT]) {
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    st[t].m = kNegInf;
    st[t].l = 0.f;
    st[t].far = false;
#pragma unroll
    for (int i = 0; i < D / 16; ++i) st[t].o[i] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
}

// Sums up to this are merged as they are: with those of all other waves and splits they stay in range.
constexpr float kRoom = 0x1p96f;

template <int D, int RT>
__device__ __forceinline__ bool all_in_range(const RowTile<D> (&st)[RT]) {
  bool fine = true;
#pragma unroll
  for (int t = 0; t < RT; ++t)
#pragma unroll
    for (int i = 0; i < D / 16; ++i)
#pragma unroll
      for (int r = 0; r < 4; ++r) fine = fine && fabsf(st[t].o[i][r]) < kRoom;
  return fine;
}

// By which power of two the weights of a careful pass are smaller: `end` of them, up to e^8 each (kSlack, rounded where
// maxima are large), add up to less than 1.
__device__ __forceinline__ int careful_shift(int end) { return 44 - __clz(end); }

// After a careful pass: rows whose sums are small get the power of two back, which leaves the bits of a pass that never
// took it off; the others' maximum is raised by as much, as nearly as fp32 has it, which up to 2^24 is to 1/2.
template <int D, int RT>
__device__ __forceinline__ void settle(RowTile<D> (&st)[RT], int shift) {
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    float top = 0.f;
#pragma unroll
    for (int i = 0; i < D / 16; ++i)
#pragma unroll
      for (int r = 0; r < 4; ++r) top = fmaxf(top, finite(st[t].o[i][r]) ? fabsf(st[t].o[i][r]) : 0.f);
    top = max_xor32(max_xor16(top));
    float back = ldexpf(1.f, shift);
    if (top * back >= kRoom) {
      const float raised = st[t].m + (float)shift / kLog2e;
      back = fast_exp2((float)shift - (raised - st[t].m) * kLog2e);   // 1 but for the rounding of `raised`
      st[t].m = raised;
    }
    st[t].l *= back;
#pragma unroll
    for (int i = 0; i < D / 16; ++i) st[t].o[i] *= back;
  }
}

// Waves a SIMD is to hold: what the registers of the accumulators, queries and the step on its way leave (one row tile of
// bf16 at d = 128 in three: 27.5 us over 25600 entries, 26.9 in two).
template <typename T, int D>
constexpr int waves_per_simd() {
  return sizeof(T) == 4 && D == 128 ? 1 : 2;
}

// A workgroup is RG groups of waves with RT 16-row tiles of their own; the KG waves of a group share the rows and take
// entries in turn.
template <typename T, int D, int RT, int RG, int KG>
__global__ __launch_bounds__(RG * KG * 64, (waves_per_simd<T, D>())) void tree_kernel(TreeArgs a) {
  constexpr int ROWS = 16 * RT;
  constexpr int STEP = KG * kTile;
  constexpr int kSlots = KG > 1 ? RG * KG / 2 : 1;
  __shared__ __align__(16) f32x4 s_o[kSlots][KG > 1 ? RT * (D / 16) : 1][64];
  __shared__ float2 s_ml[kSlots][RT][64];
  const Place place = place_of(blockIdx.x, a.heads, (uint32_t)(a.splits * a.row_blocks));
  const uint32_t at = place.head / (uint32_t)a.hkv;
  const Sequence seq = sequence_at(a.n, at, a.heads / a.hkv, threadIdx.x & 63);
  const uint32_t b = seq.b;
  const int len = seq.len, count = seq.count;
  const int head = place.head - at * a.hkv;
  const int split = place.inner / a.row_blocks, rb = place.inner % a.row_blocks;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int col = lane & 15, grp = lane >> 4;
  const int kw = wave % KG, rw = wave / KG;
  const int nrows = count * a.G;
  if (rb * RG * ROWS >= nrows) return;
  const int row0 = (rb * RG + rw) * ROWS;
  if (KG == 1 && row0 >= nrows) return;
  const int end = len + count;
  const int chunk = chunk_of(a, end);
  const int e0 = split * chunk, e1 = min(e0 + chunk, end);
  if (e0 >= e1) return;                  // behind a shorter sequence's end: the combining kernel does not read the slot

  Rows<T, D, RT> rows;
  const uint64_t anc = e1 > len ? ancestors(a.parent ? a.parent + (size_t)b * a.n.n : nullptr, a.n.n, lane) : 0;
  load_rows<T, D, RT>(rows, a, b, head, row0, nrows, anc, col, grp);
  PageWindow pages;
  pages.fill(a.c, b, (e0 + kw * kTile) >> a.c.shift, lane);
  RowTile<D> st[RT];
  bool careful = false;
  for (;;) {
    clear<D, RT>(st);
    int e = e0 + kw * kTile;
    // Steps of entries that all rows attend to.  The next step's keys are loaded when this one's have become logits and
    // its values when this one's are added, into the same registers.
    int whole = pages.up_to(a.c, min(e1, len));
    Keys<T, D> k;
    Values<T, D> v;
    bool loaded = false;
    if (!careful && e + kTile <= whole) {
      {
        float p[RT][8];
        k.load(a.c, a.hkv, head, e, pages.at(a.c, e + 8 * (col >> 2)), pages.at(a.c, e + 8 * grp), col, grp);
        v.load(a.c, a.hkv, head, e, pages.at(a.c, e + 8 * grp), col, grp);
        for (;;) {
          const int next = e + STEP;
          if (next + kTile <= whole && !pages.holds(a.c, next, next + kTile - 1)) {
            pages.fill(a.c, b, next >> a.c.shift, lane);
            whole = pages.up_to(a.c, whole);
          }
          if (next + kTile > whole) break;
          const int pk = pages.at(a.c, next + 8 * (col >> 2)), pv = pages.at(a.c, next + 8 * grp);
          logits<T, D, RT>(p, k, rows, a.scale, a.c.bias != nullptr);
          __builtin_amdgcn_sched_barrier(0);   // loads moved up would need registers of their own
          k.load(a.c, a.hkv, head, next, pk, pv, col, grp);
          __builtin_amdgcn_sched_barrier(0);
          soften<sizeof(T) == 2, D, RT>(st, p, 1.f);
          add_values<T, D, RT>(st, v.v, p);
          __builtin_amdgcn_sched_barrier(0);
          v.load(a.c, a.hkv, head, next, pv, col, grp);
          e = next;
        }
        logits<T, D, RT>(p, k, rows, a.scale, a.c.bias != nullptr);
        e += STEP;
        loaded = e < e1 && pages.holds(a.c, e, e + kTile - 1);   // the step after, one of the edge
        const int pk = max(pages.at(a.c, e + 8 * (col >> 2)), 0), pv = max(pages.at(a.c, e + 8 * grp), 0);
        __builtin_amdgcn_sched_barrier(0);
        if (loaded) k.load(a.c, a.hkv, head, e, pk, pv, col, grp);
        __builtin_amdgcn_sched_barrier(0);
        soften<sizeof(T) == 2, D, RT>(st, p, 1.f);
        add_values<T, D, RT>(st, v.v, p);
        __builtin_amdgcn_sched_barrier(0);
        if (loaded) v.load(a.c, a.hkv, head, e, pv, col, grp);
      }
    }
    attend_edges<T, D, RT>(st, k, v, loaded, rows, a, b, head, e, e1, STEP, len, end,
                           careful ? ldexpf(1.f, -careful_shift(end)) : 1.f, pages, lane);
    if (careful || !__any(!all_in_range<D, RT>(st))) break;
    careful = true;
  }
  if (careful) settle<D, RT>(st, careful_shift(end));
  finish<T, D, RT, RG, KG>(st, s_o[0][0], s_ml[0][0], a, b, head, row0, nrows, split, rw, kw, lane);
}

// Calls with more than 32 rows a KV head: the waves of a workgroup share the entries in LDS.  A tile is 32 KG entries, K
// rows, V rows and biases; two of them alternate, the one after the next is on its way in registers.  Every thread
// moves 16-byte chunks, chunk i of the tile to place i of LDS, so that the swizzle of K is one of the addresses in memory.
template <typename T, int D, int RG, int KG>
__global__ __launch_bounds__(RG * KG * 64, (waves_per_simd<T, D>())) void tree_shared_kernel(TreeArgs a) {
  constexpr int RT = 2;
  constexpr int SUB = tiles_of_turn(KG);
  constexpr int ROWS = 16 * RT, NT = RG * KG * 64, STEP = KG * SUB * kTile;
  constexpr int RB = D * (int)sizeof(T), CH = RB / 16;
  constexpr int kHalf = STEP * CH;                  // chunks of a tile's K rows
  constexpr int kLoads = 2 * kHalf / NT;
  static_assert(2 * kHalf % NT == 0 && kHalf % 64 == 0, "whole chunks a thread, K or V a wave");
  constexpr int kTileBytes = 2 * STEP * RB + STEP * 4;
  constexpr bool kHalves = KG == 1;                 // then a turn has two tiles
  static_assert(!kHalves || SUB == 2, "a tile of a turn for each half of the waves");
  constexpr int kSlots = KG > 1 ? RG * KG / 2 : RG / 2;
  constexpr int kMergeBytes = kSlots * RT * 64 * ((D / 16) * 16 + 8);
  __shared__ __align__(16) char lds[2 * kTileBytes > kMergeBytes ? 2 * kTileBytes : kMergeBytes];
  const Place place = place_of(blockIdx.x, a.heads, (uint32_t)(a.splits * a.row_blocks));
  const uint32_t at = place.head / (uint32_t)a.hkv;
  const Sequence seq = sequence_at(a.n, at, a.heads / a.hkv, threadIdx.x & 63);
  const uint32_t b = seq.b;
  const int len = seq.len, count = seq.count;
  const int head = place.head - at * a.hkv;
  const int split = place.inner / a.row_blocks, rb = place.inner % a.row_blocks;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int col = lane & 15, grp = lane >> 4;
  const int nrows = count * a.G;
  if (rb * RG * ROWS >= nrows) return;
  // where half of the waves hold all rows (a sequence with few of the nodes), each half takes one tile of a turn (the
  // call above 125 us, without 130)
  const bool halves = kHalves && nrows - rb * RG * ROWS <= RG / 2 * ROWS;
  const int key_groups = halves ? 2 : KG;
  const int kw = wave % key_groups, rw = wave / key_groups;
  const int row0 = (rb * RG + rw) * ROWS;
  const bool idle = row0 >= nrows;                  // loads and waits with the others
  const int end = len + count;
  const int chunk = chunk_of(a, end);
  const int e0 = split * chunk, e1 = min(e0 + chunk, end);
  if (e0 >= e1) return;

  Rows<T, D, RT> rows;
  const uint64_t anc = e1 > len ? ancestors(a.parent ? a.parent + (size_t)b * a.n.n : nullptr, a.n.n, lane) : 0;
  load_rows<T, D, RT>(rows, a, b, head, row0, nrows, anc, col, grp);
  PageWindow pages;
  pages.fill(a.c, b, e0 >> a.c.shift, lane);
  RowTile<D> st[RT];
  bool careful = false;
  const size_t page_rows = (size_t)a.hkv << a.c.shift, head_row = (size_t)head << a.c.shift;
  const int mask = (1 << a.c.shift) - 1;
  for (;;) {
    clear<D, RT>(st);
    int e = e0, whole = pages.up_to(a.c, min(e1, len));
    // Tiles of entries that all rows attend to.
    if (!careful && e + STEP <= whole) {
      Chunk16 ahead[kLoads];
      float bias_ahead = 0.f;
      // the tile at `from` into registers; the rows of a wave's chunks are on one page
      const auto fetch = [&](int from) {
        int tid = threadIdx.x;
        asm volatile("" : "+v"(tid));   // places formed anew: kept from turn to turn they cost more registers than there are
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
          const int at = (tid + i * NT) % kHalf, row = at / CH;
          const int first = (wave * 64 + i * NT) % kHalf / CH;
          const int page = __builtin_amdgcn_readlane(pages.page, ((from + first) >> a.c.shift) - pages.first);
          const bool value = (wave * 64 + i * NT) / kHalf;
          const char* rows0 = (value ? a.c.V : a.c.K) +
                              ((size_t)page * page_rows + head_row + ((from + first) & mask & ~7)) * RB;
          ahead[i] = load16(rows0 + (row - (first & ~7)) * RB + ((at % CH ^ (value ? 0 : swizzle(row))) << 4));
        }
        if (a.c.bias && (int)threadIdx.x < STEP) {
          const int page = __shfl(pages.page, ((from + tid) >> a.c.shift) - pages.first, 64);
          bias_ahead = a.c.bias[(size_t)page * page_rows + head_row + ((from + tid) & mask)];
        }
      };
      // whether the tile at `from` is one of those
      const auto more = [&](int from) {
        if (from + STEP <= whole && !pages.holds(a.c, from, from + STEP - 1)) {
          pages.fill(a.c, b, from >> a.c.shift, lane);
          whole = pages.up_to(a.c, whole);
        }
        return from + STEP <= whole;
      };
      const auto put = [&](char* tile) {
#pragma unroll
        for (int i = 0; i < kLoads; ++i) store16(tile + (threadIdx.x + i * NT) * 16, ahead[i]);
        if ((int)threadIdx.x < STEP) reinterpret_cast<float*>(tile + 2 * STEP * RB)[threadIdx.x] = bias_ahead;
      };
      const Places<T, D> places(col, grp);
      bool here = more(e);
      if (here) {
        fetch(e);
        put(lds);
      }
      bool next = here && more(e + STEP);
      if (next) fetch(e + STEP);
      __syncthreads();
      for (int turn = 0; here; turn ^= 1) {
        const char* tile = lds + turn * kTileBytes;
        if (next) put(lds + (turn ^ 1) * kTileBytes);
        const bool after = next && more(e + 2 * STEP);
        if (after) fetch(e + 2 * STEP);
        const auto attend = [&](int sub) {
          float p[RT][8];
          Keys<T, D> k;
          read_keys<T, D>(k, tile + sub * kTile * RB, tile + 2 * STEP * RB + sub * kTile * 4, places);
          logits<T, D, RT>(p, k, rows, a.scale, true);
          Values<T, D> v;
          read_values<T, D>(v, tile + (STEP + sub * kTile) * RB, places);
          soften<sizeof(T) == 2, D, RT>(st, p, 1.f);
          add_values<T, D, RT>(st, v.v, p);
        };
        if (!idle) {
          for (int u = 0; u < (halves ? 1 : SUB); ++u) attend(u * KG + kw);
        }
        __syncthreads();
        e += STEP;
        here = next;
        next = after;
      }
    }
    if (!idle) {
      Keys<T, D> k;
      Values<T, D> v;
      attend_edges<T, D, RT>(st, k, v, false, rows, a, b, head, e + kw * kTile, e1, key_groups * kTile, len, end,
                             careful ? ldexpf(1.f, -careful_shift(end)) : 1.f, pages, lane);
    }
    if (careful || !__syncthreads_or(!idle && !all_in_range<D, RT>(st))) break;
    careful = true;
  }
  if (careful) settle<D, RT>(st, careful_shift(end));
  f32x4* s_o = reinterpret_cast<f32x4*>(lds);
  float2* s_ml = reinterpret_cast<float2*>(s_o + kSlots * RT * (D / 16) * 64);
  if constexpr (kHalves) {
    if (halves) {
      finish<T, D, RT, RG / 2, 2>(st, s_o, s_ml, a, b, head, row0, nrows, split, rw, kw, lane);
      return;
    }
  }
  finish<T, D, RT, RG, KG>(st, s_o, s_ml, a, b, head, row0, nrows, split, rw, kw, lane);
}

// Combines the partials of the rows, in slot order.  A unit of d/4 threads takes four channels each of the slots sub,
// sub + SUB, ... of a row and loads kBatch of them at a time; with SUB > 1 all units of a workgroup share a row and
// meet in LDS, in order.
template <typename T, int D, int SUB>
__global__ __launch_bounds__(256) void tree_combine_kernel(TreeArgs a) {
  constexpr int kUnits = 256 / (D / 4);
  constexpr int kBatch = 8;
  static_assert(SUB == 1 || SUB == kUnits, "a unit is a row, or all of them are one");
  __shared__ float2 s_ml[kUnits];
  __shared__ __align__(16) f32x4 s_o[kUnits][D / 4];
  const uint32_t per = (uint32_t)a.n.n * a.G;
  const int c4 = threadIdx.x % (D / 4), unit = threadIdx.x / (D / 4), sub = SUB == 1 ? 0 : unit;
  const Place place = place_of(blockIdx.x, a.heads, SUB == 1 ? (per + kUnits - 1) / kUnits : per);
  const uint32_t r = SUB == 1 ? place.inner * kUnits + unit : place.inner;
  if (r >= per) return;
  const uint32_t bh = place.head, b = bh / (uint32_t)a.hkv, head = bh - b * a.hkv;
  int len, count;
  if (!sequence_of(a.n, b, len, count)) return;
  const uint32_t node = r / (uint32_t)a.G, g = r - node * a.G;
  if ((int)node >= count) return;
  const int end = len + count, chunk = chunk_of(a, end), slots = (end + chunk - 1) / chunk;
  const size_t part = (size_t)bh * a.splits * per + r;
  float m = kNegInf, l = 0.f;
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  for (int s0 = sub; s0 < slots; s0 += SUB * kBatch) {
    f32x4 x[kBatch];
    float2 ml[kBatch];
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      const size_t at = part + (size_t)min(s0 + u * SUB, slots - 1) * per;
      x[u] = *reinterpret_cast<const f32x4*>(a.part_o + at * D + 4 * c4);
      ml[u] = a.part_ml[at];
    }
    float M = m;
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      if (s0 + u * SUB >= slots) ml[u].x = kNegInf;
      M = fmaxf(M, ml[u].x);
    }
    const float c = weight_of(m, M);
    l *= c;
#pragma unroll
    for (int k = 0; k < 4; ++k) o[k] *= c;
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      const bool some = ml[u].x != kNegInf;             // a part that nothing counts in may be NaN
      const float w = weight_of(ml[u].x, M);
      l = some ? fmaf(ml[u].y, w, l) : l;
#pragma unroll
      for (int k = 0; k < 4; ++k) o[k] = some ? fmaf(x[u][k], w, o[k]) : o[k];
    }
    m = M;
  }
  if constexpr (SUB > 1) {
    s_o[unit][c4] = o;
    if (c4 == 0) s_ml[unit] = make_float2(m, l);
    __syncthreads();
    if (unit > 0) return;
    float M = kNegInf;
#pragma unroll
    for (int u = 0; u < kUnits; ++u) M = fmaxf(M, s_ml[u].x);
    l = 0.f;
    o = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int u = 0; u < kUnits; ++u) {
      const float2 ml = s_ml[u];
      const bool some = ml.x != kNegInf;
      const float w = weight_of(ml.x, M);
      const f32x4 x = s_o[u][c4];
      l = some ? fmaf(ml.y, w, l) : l;
#pragma unroll
      for (int k = 0; k < 4; ++k) o[k] = some ? fmaf(x[k], w, o[k]) : o[k];
    }
  }
  Chunk16 w = zero16();
#pragma unroll
  for (int k = 0; k < 4; ++k) Elem<T>::put(w, k, l == 0.f ? 0.f : o[k] / l);
  char* at = a.out + (((((size_t)b * a.n.n + node) * a.hkv + head) * a.G + g) * D + 4 * c4) * sizeof(T);
  if constexpr (sizeof(T) == 4) store16(at, w);
  else *reinterpret_cast<uint2*>(at) = make_uint2(w.w[0], w.w[1]);
}

template <typename T, int D>
hipError_t launch_td(int64_t heads, const TreePlan& plan, const TreeArgs& a, hipStream_t st) {
  const dim3 grid((unsigned)heads * a.splits * a.row_blocks);
  const auto with = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, grid, dim3(64 * plan.row_groups * plan.key_groups), 0, st, a);
  };
  constexpr bool kWide = sizeof(T) == 4 && D == 128;   // registers for half as many waves
  if (plan.row_tiles == 1) with(tree_kernel<T, D, 1, 1, 4>);
  else if (plan.row_groups == 1) with(tree_kernel<T, D, 2, 1, 4>);
  else if constexpr (kWide) {
    if (plan.row_groups == 2) with(tree_shared_kernel<T, D, 2, 2>);
    else with(tree_shared_kernel<T, D, 4, 1>);
  } else {
    if (plan.row_groups == 2) with(tree_shared_kernel<T, D, 2, 4>);
    else if (plan.row_groups == 4) with(tree_shared_kernel<T, D, 4, 2>);
    else with(tree_shared_kernel<T, D, 8, 1>);
  }
  if (a.splits > 1) {
    const uint32_t per = (uint32_t)a.n.n * a.G;
    constexpr uint32_t kUnits = 256 / (D / 4);
    if (a.splits <= kFewSlots || (uint32_t)heads * per >= kManyRows)
      hipLaunchKernelGGL((tree_combine_kernel<T, D, 1>), dim3((uint32_t)heads * ((per + kUnits - 1) / kUnits)), dim3(256), 0,
                         st, a);
    else
      hipLaunchKernelGGL((tree_combine_kernel<T, D, kUnits>), dim3((uint32_t)heads * per), dim3(256), 0, st, a);
  }
  return hipGetLastError();
}

size_t round256(size_t x) { return (x + 255) & ~(size_t)255; }

size_t parts_bytes(int64_t heads, int splits, int rows, int d, size_t* ml_off) {
  const size_t parts = (size_t)heads * splits * rows;
  *ml_off = round256(parts * d * 4);
  return splits > 1 ? *ml_off + parts * 8 : 0;
}

}  // namespace

namespace {

// Splits of a head for so many rounds of workgroups.
int splits_for(int rounds, int64_t units, int entries, int step) {
  const int64_t splits = ((int64_t)rounds * kCUs + units - 1) / units;
  return (int)std::min<int64_t>({splits, (int64_t)kMaxSplit, ((int64_t)entries + step - 1) / step});
}

// Most splits of a head.
int most_splits(const TreePlan& p, int64_t heads, int entries) {
  return splits_for(p.row_groups == 1 ? kFewRowsRounds : kMaxRounds, heads * p.row_blocks, entries, p.step);
}

TreePlan plan_rows(int64_t heads, int d, int rows, size_t elem) {
  TreePlan p;
  const int tiles = (rows + 15) / 16;
  const bool wide = elem == 4 && d == 128;   // registers for half as many waves
  p.row_tiles = tiles == 1 ? 1 : 2;
  p.row_groups = tiles <= 2 ? 1 : tiles <= 4 ? 2 : tiles <= 8 || wide ? 4 : 8;
  p.key_groups = (p.row_groups == 1 || wide ? 4 : 8) / p.row_groups;
  const int per = p.row_tiles * p.row_groups;
  p.row_blocks = (tiles + per - 1) / per;
  p.step = p.key_groups * kTile * (p.row_groups > 1 ? tiles_of_turn(p.key_groups) : 1);
  return p;
}

}  // namespace

// How the entries are divided.  A CU reads and computes at one rate however many workgroups share it, so a call takes
// the entries of a workgroup, and what one costs besides, times the workgroups of the fullest CU: one layer of 25605
// entries (8 heads, 5 nodes) takes 27.6 us in 29 splits, one workgroup on most CUs, and 29.2 in 51, two on some; 64
// nodes 78 in 31 and 101 in 51.  Where lengths are the device's to know, two rounds, and six up to 32 rows, where a
// workgroup costs less.  Sequences of 0 to 8100 entries, 8 heads, in one and a half, two, three and four rounds: 8 of up
// to 64 nodes (G 4) 93, 77, 82 and 90 us; 16 of up to 16 (G 4) 78, 69, 81 and 90; 16 of up to 26 (G 8) 164, 131, 119 and
// 124: two cost the last 12 us and save the others 5 and 12.  In two, three and six: 32 of up to 8 (G 4) 118, 107 and 112,
// 64 of up to one 64, 38 and 30.
TreePlan plan_tree(int64_t heads, int entries, int d, int rows, size_t elem, bool ragged) {
  TreePlan p = plan_rows(heads, d, rows, elem);
  const int64_t units = heads * p.row_blocks;
  const int most = splits_for(kMaxRounds, units, entries, p.step);
  p.splits = 1;
  if (ragged) {
    p.splits = splits_for(p.row_groups == 1 ? kFewRowsRounds : kRaggedRounds, units, entries, p.step);
  } else {
    int64_t best = INT64_MAX;
    for (int s = 1; s <= most; ++s) {
      const int64_t chunk = ((entries + s - 1) / s + p.step - 1) / p.step * p.step;
      const int64_t groups = (entries + chunk - 1) / chunk * units;
      const int64_t cost = (groups + kCUs - 1) / kCUs * (chunk + kGroupCost) + (s > 1 ? kCombineCost : 0);
      if (cost < best) best = cost, p.splits = s;
    }
  }
  p.bytes = parts_bytes(heads, p.splits, rows, d, &p.ml_off);
  return p;
}

size_t tree_workspace_bound(int64_t heads, int capacity, int d, int G, int n, size_t elem) {
  size_t most = 0;   // fewer nodes may take more splits
  for (int i = 1; i <= n; ++i) {
    const TreePlan p = plan_rows(heads, d, i * G, elem);
    size_t ml_off;
    most = std::max(most, parts_bytes(heads, most_splits(p, heads, capacity), i * G, d, &ml_off));
  }
  return most;
}

hipError_t launch_tree_attn(int batch, int hkv, int d, int G, int dtype, float scale, const TreePlan& plan,
                            const Paged& c, const Seqs& n, const void* q, const int32_t* parent, void* out, void* ws,
                            hipStream_t st) {
  TreeArgs a;
  a.c = c;
  a.n = n;
  a.q = static_cast<const char*>(q);
  a.parent = parent;
  a.out = static_cast<char*>(out);
  a.part_o = static_cast<float*>(ws);
  a.part_ml = reinterpret_cast<float2*>(static_cast<char*>(ws) + plan.ml_off);
  a.hkv = hkv;
  a.heads = (uint32_t)batch * hkv;
  a.G = G;
  a.splits = plan.splits;
  a.row_blocks = plan.row_blocks;
  a.step = plan.step;
  a.scale = scale;
  const int64_t heads = (int64_t)batch * hkv;
  if (dtype == SELKV_BF16)
    return d == 128 ? launch_td<bf16_t, 128>(heads, plan, a, st) : launch_td<bf16_t, 64>(heads, plan, a, st);
  return d == 128 ? launch_td<float, 128>(heads, plan, a, st) : launch_td<float, 64>(heads, plan, a, st);
}

}  // namespace selkv
