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
// `column` of O^T tile i.  So K and V go from memory to registers once, without
// LDS.
//
// bf16 weights enter the product as sums of two bf16 numbers (2^-17 of a weight
// is left), fp32 ones as they are.  Maxima, sums and accumulators are fp32.
//
// Masks.  Entries past the end, on no page or (for a node) outside its chain of
// parents are left out by selection in the tiles that hold such; a masked bias
// makes a logit -inf by itself.  Where a result comes out NaN or infinite the
// wave does its entries again in a careful pass, in which every tile selects
// masked biases too, V's values that are NaN or infinite are kept out of the
// product, where a weight of 0 would turn them into NaN for every row, and are
// added to the rows that attend to them.
//
// Split-K: a workgroup takes a run of entries, and a second kernel combines the
// runs' (max, sum, o) in order.
#include <algorithm>

#include "paged.hpp"

namespace selkv {
namespace {

constexpr int kWaves = 4;
constexpr int kThreads = kWaves * 64;
constexpr int kTile = 32;              // entries of a wave's step
constexpr int kStep = kWaves * kTile;  // splits are whole multiples of it
constexpr int kTargetBlocks = 768;
constexpr int kMaxSplit = 256;

struct TreeArgs {
  Paged c;
  Seqs n;
  const char* q;
  const int32_t* parent;
  char* out;
  float* part_o;     // [B hkv, splits, n G, D]
  float2* part_ml;   // [B hkv, splits, n G]
  int hkv, G, splits, row_blocks;
  float scale;
};

// Entries of a split of a sequence of `total`: as many splits as there are, of whole steps.
__device__ __forceinline__ int chunk_of(int splits, int total) {
  const uint32_t per = ((uint32_t)total + splits - 1) / (uint32_t)splits;
  return (int)(max((per + kStep - 1) / kStep, 1u) * kStep);
}

__device__ __forceinline__ float weight_of(float m, float M) { return m == kNegInf ? 0.f : fast_exp2((m - M) * kLog2e); }

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

// What a wave reads for 32 entries.
template <typename T, int D>
struct Entries {
  static constexpr int KC = D * (int)sizeof(T) / 64;       // 16-byte chunks of a lane of a K tile row
  static constexpr int VW = D * (int)sizeof(T) / 64;       // words of a lane of a V row
  Chunk16 k[2][KC];
  uint32_t v[8][VW];
  float bias[8];                                           // of entries 8 grp .. + 7
};

template <typename T, int D>
__device__ __forceinline__ void load_entries(Entries<T, D>& x, const Paged& c, int hkv, int head, int base, int pk,
                                             int pv, int col, int grp) {
  constexpr int RB = D * (int)sizeof(T);
  const char* kp = c.K + row_of(c, hkv, max(pk, 0), head, base + 8 * (col >> 2) + (col & 3)) * RB + grp * 16;
  const size_t vr = row_of(c, hkv, max(pv, 0), head, base + 8 * grp);
  const char* vp = c.V + vr * RB + col * (RB / 16);
#pragma unroll
  for (int t = 0; t < 2; ++t)
#pragma unroll
    for (int j = 0; j < Entries<T, D>::KC; ++j) x.k[t][j] = load16(kp + 4 * t * RB + j * 64);
#pragma unroll
  for (int s = 0; s < 8; ++s) {
    if constexpr (RB / 16 >= 16) {
#pragma unroll
      for (int i = 0; i < RB / 256; ++i) {
        const Chunk16 w = load16(vp + s * RB + i * 16);
#pragma unroll
        for (int k = 0; k < 4; ++k) x.v[s][4 * i + k] = w.w[k];
      }
    } else {
      const uint2 w = *reinterpret_cast<const uint2*>(vp + s * RB);
      x.v[s][0] = w.x;
      x.v[s][1] = w.y;
    }
  }
  if (c.bias) {
    const Chunk16 b0 = load16(c.bias + vr), b1 = load16(c.bias + vr + 4);
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      x.bias[s] = __uint_as_float(b0.w[s]);
      x.bias[4 + s] = __uint_as_float(b1.w[s]);
    }
  } else {
#pragma unroll
    for (int s = 0; s < 8; ++s) x.bias[s] = 0.f;
  }
}

// Softmax state of a wave's row tile: lane (column, grp) keeps its row's maximum, the sum over the entries it holds,
// and channels (D/16)(4 grp + r) + i of the row as o[i][r].
template <int D>
struct RowTile {
  float m, l;
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
__device__ __forceinline__ void add_values(RowTile<D> (&st)[RT], const uint32_t (&v)[8][Entries<T, D>::VW],
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
  Chunk16 q[RT][Entries<T, D>::KC];
  uint64_t seen[RT];   // the nodes that the row attends to
};

// One step: 32 entries from `base`.  len: entries that all rows attend to, end: with the nodes' behind them.
template <typename T, int D, int RT>
__device__ __forceinline__ void attend(RowTile<D> (&st)[RT], Entries<T, D>& x, const Rows<T, D, RT>& rows,
                                       const TreeArgs& a, uint32_t b, int head, int base, int len, int end, int pv,
                                       bool careful, int grp) {
  float p[RT][8];
#pragma unroll
  for (int t = 0; t < RT; ++t)
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int j = 0; j < Entries<T, D>::KC; ++j) s = Mma<T>::step(x.k[h][j], rows.q[t][j], s);
#pragma unroll
      for (int r = 0; r < 4; ++r) p[t][4 * h + r] = fmaf(s[r], a.scale, x.bias[4 * h + r]);
    }
  const bool edge = careful || base + kTile > len || __any(pv < 0);
  bool unbounded = false;
  if (edge) {
#pragma unroll
    for (int s = 0; s < 8; ++s) {
      const int entry = base + 8 * grp + s, node = entry - len;
      const bool live = pv >= 0 && entry < end && x.bias[s] != kNegInf;
#pragma unroll
      for (int t = 0; t < RT; ++t)
        if (!(live && (node < 0 || ((rows.seen[t] >> (node & 63)) & 1)))) p[t][s] = kNegInf;
#pragma unroll
      for (int w = 0; w < Entries<T, D>::VW; ++w) {
        if (!live) x.v[s][w] = 0u;
        else if (careful) x.v[s][w] = zero_unbounded<T>(x.v[s][w], unbounded);
      }
    }
  }
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    float mx = p[t][0];
#pragma unroll
    for (int s = 1; s < 8; ++s) mx = fmaxf(mx, p[t][s]);
    mx = max_xor32(max_xor16(mx));
    const float mnew = fmaxf(st[t].m, mx);
    const float ref = mnew == kNegInf ? 0.f : mnew;   // nothing unmasked yet: every weight is 0
    if (__any(mnew != st[t].m)) {
      const float corr = fast_exp2((st[t].m - ref) * kLog2e);
      st[t].l *= corr;
#pragma unroll
      for (int i = 0; i < D / 16; ++i) st[t].o[i] *= corr;
      st[t].m = mnew;
    }
#pragma unroll
    for (int s = 0; s < 8; ++s) {
      p[t][s] = fast_exp2((p[t][s] - ref) * kLog2e);
      st[t].l += p[t][s];
    }
  }
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

template <typename T, int D, int RT>
__global__ __launch_bounds__(kThreads, 2) void tree_kernel(TreeArgs a) {
  constexpr int ROWS = 16 * RT;
  constexpr int RB = D * (int)sizeof(T);
  __shared__ __align__(16) f32x4 s_o[2][RT * (D / 16)][64];
  __shared__ float2 s_ml[2][RT][64];
  const uint32_t bh = blockIdx.y, b = bh / (uint32_t)a.hkv;
  const int head = bh - b * a.hkv;
  const int split = blockIdx.x % a.splits, rb = blockIdx.x / a.splits;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int col = lane & 15, grp = lane >> 4;
  int len, count;
  if (!sequence_of(a.n, b, len, count)) return;
  const int nrows = count * a.G, row0 = rb * ROWS;
  if (row0 >= nrows) return;
  const int end = len + count;
  const int chunk = chunk_of(a.splits, end);
  const int e0 = split * chunk, e1 = min(e0 + chunk, end);
  if (e0 >= e1) return;                  // behind a shorter sequence's end: the combining kernel does not read the slot

  Rows<T, D, RT> rows;
  const uint64_t anc = e1 > len ? ancestors(a.parent ? a.parent + (size_t)b * a.n.n : nullptr, a.n.n, lane) : 0;
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    const int r = row0 + 16 * t + col, node = r < nrows ? r / a.G : 0, g = r < nrows ? r - node * a.G : 0;
    const char* qr = a.q + (((size_t)b * a.n.n + node) * a.hkv + head) * a.G * RB + (size_t)g * RB + grp * 16;
#pragma unroll
    for (int j = 0; j < Entries<T, D>::KC; ++j) rows.q[t][j] = load16(qr + j * 64);
    rows.seen[t] = __shfl((unsigned long long)anc, node, 64);
  }
  RowTile<D> st[RT];
  bool careful = false;
  for (;;) {
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      st[t].m = kNegInf;
      st[t].l = 0.f;
#pragma unroll
      for (int i = 0; i < D / 16; ++i) st[t].o[i] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    for (int e = e0 + wave * kTile; e < e1; e += kStep) {
      const int pk = page_of(a.c, b, e + 8 * (col >> 2)), pv = page_of(a.c, b, e + 8 * grp);
      Entries<T, D> x;
      load_entries<T, D>(x, a.c, a.hkv, head, e, pk, pv, col, grp);
      attend<T, D, RT>(st, x, rows, a, b, head, e, len, end, pv, careful, grp);
    }
    bool fine = true;
#pragma unroll
    for (int t = 0; t < RT; ++t)
#pragma unroll
      for (int i = 0; i < D / 16; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r) fine = fine && finite(st[t].o[i][r]);
    if (careful || !__any(!fine)) break;
    careful = true;
  }
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    st[t].l = add_xor32(add_xor16(st[t].l));
    st[t].m = nan_counts(st[t].m, st[t].l);
  }

  // the waves' results, two and two
#pragma unroll
  for (int step = kWaves / 2; step > 0; step /= 2) {
    if (wave >= step && wave < 2 * step) {
#pragma unroll
      for (int t = 0; t < RT; ++t) {
        s_ml[wave - step][t][lane] = make_float2(st[t].m, st[t].l);
#pragma unroll
        for (int i = 0; i < D / 16; ++i) s_o[wave - step][t * (D / 16) + i][lane] = st[t].o[i];
      }
    }
    __syncthreads();
    if (wave < step) {
#pragma unroll
      for (int t = 0; t < RT; ++t) {
        const float2 ml = s_ml[wave][t][lane];
        const float M = fmaxf(st[t].m, ml.x);
        const float c0 = weight_of(st[t].m, M), c1 = weight_of(ml.x, M);
        const bool some0 = st[t].m != kNegInf, some1 = ml.x != kNegInf;   // a part without entries has weight 0 and 0s
        st[t].l = (some0 ? st[t].l * c0 : 0.f) + (some1 ? ml.y * c1 : 0.f);
#pragma unroll
        for (int i = 0; i < D / 16; ++i) {
          const f32x4 o = s_o[wave][t * (D / 16) + i][lane];
#pragma unroll
          for (int r = 0; r < 4; ++r) st[t].o[i][r] = (some0 ? st[t].o[i][r] * c0 : 0.f) + (some1 ? o[r] * c1 : 0.f);
        }
        st[t].m = M;
      }
    }
    __syncthreads();
  }
  if (wave > 0) return;
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
      const size_t part = ((size_t)bh * a.splits + split) * ((size_t)a.n.n * a.G) + r;
      store_row<float, D>(reinterpret_cast<char*>(a.part_o + part * D), st[t].o, grp);
      if (grp == 0) a.part_ml[part] = make_float2(st[t].m, st[t].l);
    }
  }
}

// Combines the partials of a row, in order: d/4 threads with four channels each.
template <typename T, int D>
__global__ __launch_bounds__(256) void tree_combine_kernel(TreeArgs a, uint32_t rows) {
  constexpr int kUnits = 256 / (D / 4);
  const uint32_t per = (uint32_t)a.n.n * a.G;
  const uint32_t row = blockIdx.x * kUnits + threadIdx.x / (D / 4);
  const int c4 = threadIdx.x % (D / 4);
  if (row >= rows) return;
  const uint32_t bh = row / per, r = row - bh * per, b = bh / (uint32_t)a.hkv, head = bh - b * a.hkv;
  int len, count;
  if (!sequence_of(a.n, b, len, count)) return;
  const uint32_t node = r / (uint32_t)a.G, g = r - node * a.G;
  if ((int)node >= count) return;
  const int end = len + count, chunk = chunk_of(a.splits, end), slots = (end + chunk - 1) / chunk;
  float m = kNegInf, l = 0.f;
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  for (int s = 0; s < slots; ++s) {
    const size_t part = ((size_t)bh * a.splits + s) * per + r;
    const float2 ml = a.part_ml[part];
    const f32x4 x = *reinterpret_cast<const f32x4*>(a.part_o + part * D + 4 * c4);
    if (ml.x == kNegInf) continue;
    const float M = fmaxf(m, ml.x);
    const float c0 = weight_of(m, M), c1 = weight_of(ml.x, M);
    l = l * c0 + ml.y * c1;
#pragma unroll
    for (int k = 0; k < 4; ++k) o[k] = o[k] * c0 + x[k] * c1;
    m = M;
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
  const dim3 grid(a.splits * a.row_blocks, (unsigned)heads), blk(kThreads);
  hipLaunchKernelGGL((tree_kernel<T, D, 1>), grid, blk, 0, st, a);
  if (a.splits > 1) {
    const uint32_t rows = (uint32_t)heads * a.n.n * a.G;
    constexpr int kUnits = 256 / (D / 4);
    hipLaunchKernelGGL((tree_combine_kernel<T, D>), dim3((rows + kUnits - 1) / kUnits), blk, 0, st, a, rows);
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

TreePlan plan_tree(int64_t heads, int entries, int d, int rows, size_t) {
  TreePlan p;
  p.row_tiles = 1;
  p.split_rows = false;
  p.row_blocks = (rows + 16 * p.row_tiles - 1) / (16 * p.row_tiles);
  const int64_t want = std::max<int64_t>(1, kTargetBlocks / (heads * p.row_blocks));
  p.splits = (int)std::min<int64_t>({want, (int64_t)kMaxSplit, ((int64_t)entries + kStep - 1) / kStep});
  p.bytes = parts_bytes(heads, p.splits, rows, d, &p.ml_off);
  return p;
}

size_t tree_workspace_bound(int64_t heads, int capacity, int d, int G, int n, size_t elem) {
  size_t most = 0;   // fewer nodes may take more splits
  for (int i = 1; i <= n; ++i) most = std::max(most, plan_tree(heads, capacity, d, i * G, elem).bytes);
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
  a.G = G;
  a.splits = plan.splits;
  a.row_blocks = plan.row_blocks;
  a.scale = scale;
  const int64_t heads = (int64_t)batch * hkv;
  if (dtype == SELKV_BF16)
    return d == 128 ? launch_td<bf16_t, 128>(heads, plan, a, st) : launch_td<bf16_t, 64>(heads, plan, a, st);
  return d == 128 ? launch_td<float, 128>(heads, plan, a, st) : launch_td<float, 64>(heads, plan, a, st);
}

}  // namespace selkv
