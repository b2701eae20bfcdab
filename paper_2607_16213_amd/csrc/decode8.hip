// selkv_decode8_attn / selkv_decode8_append: one decode step over a cache held
// in 8 bits (layout and quantisation: cache8.hpp), with the additive logit
// bias of Sec. 3.6.
//
//   x_e = scale * (q . code_k[e]) * k_scale + bias_e,   out = sum softmax(x)_e code_v[e] * v_scale
//
// over the whole blocks' codes and, in the storage type, the rows of the open
// block (the tail) and the token that the step appends.
//
// Split-K: a workgroup of four waves takes a run of entries of one KV head, and
// one more workgroup per head the tail (slot 0, so that it starts first); each
// writes (max, sum, o[d]) per query head to the workspace and a second kernel
// combines them in slot order.  Where one workgroup takes the whole head, a
// short cache, one of very many heads or a sequence that is all tail, it writes
// the outputs itself.
//
// The codes go to the matrix cores as bf16, which holds every int8 and e4m3
// number exactly.  A wave takes 64 entries at a time: four 16x16x32 tiles
// S = K Q^T, then O^T += V^T P^T.  Of a tile's 16 columns the G <= 8 query
// heads need at most 8, so column h + 8 carries what column h's bf16 leaves of
// the same head, of an fp32 query and of a softmax weight: the next 8 bits, and
// a second product the last 8, so both enter as the fp32 numbers they are (with
// two terms the weight that dominates a peaked softmax was off by up to 2^-18,
// 5.5e-6 of an output).  Which entry is which row of an S tile is chosen so that
// a lane's logits are 16 consecutive entries, those whose V codes it reads with
// one 16-byte load: P goes from S's layout into the next product as it is, and
// one scale of K and of V serves a lane's 64-entry step.  Scales stay out of the
// products: K's multiplies the logits, V's the weights.
// The running maximum and sum of the softmax, and all accumulators, are fp32.
// The tail (and the appended token) are few rows, taken in fp32 by lane groups
// of 16 lanes, each lane d/16 channels.  A masked entry (bias -inf) is left out by
// selection: of the codes its logit, which a NaN or infinite query would spoil,
// of the tail its rows too, which may hold anything.
//
// Bound by HBM where there is work enough: 32 x 8 heads of 25641 entries take
// 300 us, 5.7 TB/s, the matrix cores busy 11% of the cycles and the VALU 38%
// (the same loads without the products: 289).  What that took was three waves a
// SIMD (369 us with two, 470 with two and the next step's loads in registers), at
// the price of one spilled register a lane.  fp32 queries need two waves a SIMD
// and twice the products of S, and take 303 us; d = 64 holds four waves, 159 us.
// One layer, 8 heads of 25600 entries, takes 15.1 us: 13 in the splits, of which
// 4.5 are a workgroup's start and end, and 3 in the combining kernel; 16.7 us
// with fp32 queries, 11.2 at d = 64.
#include <algorithm>

#include "cache8.hpp"

namespace selkv {
namespace {

constexpr int kWaves = 4;
constexpr int kThreads = kWaves * 64;
constexpr int kMaxG = 8;
constexpr int kTailG = 4;             // query heads of a pass over the tail: registers, shared with the codes' loop
constexpr int kGroup = 64;            // entries of a wave's step; splits are whole multiples of them
// A round of workgroups: three to a CU, what the registers of bf16 at d = 128 hold.  The others hold two (fp32 at
// d = 128: 32 x 8 heads of 25641 entries 303 us, with rounds of 512 363 us; one layer 16.7 and 21.5; only ragged MHA
// steps gain by 512, 18.3 against 21.9) or four (bf16 at d = 64: 159 us, with rounds of 1024 168; one layer 11.2 and 11.8).
constexpr int kTargetBlocks = 768;
constexpr int kRounds = 4;
constexpr int kMaxSplit = 512;
constexpr int kCUs = 256;
constexpr int kFewSlots = 8;          // up to which a query head is combined by d/4 threads

struct DecodeArgs8 {
  Cache8 c;
  Lens8 n;
  const char* q;
  float* bias;
  float* out;
  float* part_o;     // [heads, slots, G, D]
  float2* part_ml;   // [heads, slots, G]
  const char* k_new; // APP
  const char* v_new;
  int hkv, G, slots, block_shift;
  int chunk;         // entries of a split where every sequence has cache_len
  float scale;
};

// Entries of a split of a sequence whose codes are `whole` entries: with lengths of their own each is cut into as many
// splits as its slots allow, whole steps of the four waves, so a bound far above the lengths costs no parallelism.
__device__ __forceinline__ int chunk_of(const DecodeArgs8& a, int whole) {
  if (!a.n.lens) return a.chunk;
  const uint32_t splits = a.slots - 1, step = kWaves * kGroup;
  const uint32_t per = ((uint32_t)whole + splits - 1) / splits;
  return (int)(max((per + step - 1) / step, 1u) * step);
}

// Weight of partial (m, .) against the maximum M of all (0 where it is empty).
__device__ __forceinline__ float weight_of(float m, float M) {
  return m == kNegInf ? 0.f : fast_exp2((m - M) * kLog2e);
}

// The maximum that goes with a sum: fmaxf passes a NaN logit by, so where the sum is NaN a part keeps a maximum that
// makes it count, and the output is NaN as the logit was (0 is for rows that nothing reaches).
__device__ __forceinline__ float nan_counts(float m, float l) { return l == l || m != kNegInf ? m : 0.f; }

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x4u __attribute__((ext_vector_type(4), aligned(4)));   // biases: aligned to an element only

// Four codes as bf16 numbers (exact).
template <int CODE>
__device__ __forceinline__ uint2 codes_to_bf16(uint32_t w) {
  if constexpr (CODE == SELKV_I8) {
    float f[4];
    decode4<CODE>(w, f);
    return make_uint2(__builtin_amdgcn_perm(__float_as_uint(f[1]), __float_as_uint(f[0]), 0x07060302u),
                      __builtin_amdgcn_perm(__float_as_uint(f[3]), __float_as_uint(f[2]), 0x07060302u));
  } else {
    return make_uint2(__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, false)),
                      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, true)));
  }
}

// Half H (8 codes) of a 16-byte chunk as an MFMA operand.
template <int CODE, int H>
__device__ __forceinline__ bf16x8 half_to_bf16(const Chunk16& c) {
  const uint2 a = codes_to_bf16<CODE>(c.w[2 * H]), b = codes_to_bf16<CODE>(c.w[2 * H + 1]);
  const Chunk16 r = {a.x, a.y, b.x, b.y};
  return __builtin_bit_cast(bf16x8, r);
}

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

// Queries of a head as the MFMA B operand: lane (column, grp) holds channels
// (4 j + grp) * 16 + 8 m .. + 7 of query column & 7, as K's codes come.
template <typename T, int D>
struct Query8 {
  static constexpr int kParts = sizeof(T) == 4 ? 2 : 1;
  bf16x8 b[kParts][D / 64][2];
  __device__ __forceinline__ void load(const char* q, int G, int col, int grp) {
    const int h = col & 7;
    const bool low = col >= 8;
#pragma unroll
    for (int j = 0; j < D / 64; ++j)
#pragma unroll
      for (int m = 0; m < 2; ++m) {
        const char* at = q + ((size_t)(h < G ? h : 0) * D + (4 * j + grp) * 16 + 8 * m) * sizeof(T);
        if constexpr (sizeof(T) == 2) {
          b[0][j][m] = __builtin_bit_cast(bf16x8, h < G ? load16(at) : zero16());
        } else {
          const Chunk16 c0 = load16(at), c1 = load16(at + 16);
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const float x = h < G ? __uint_as_float(i < 4 ? c0.w[i & 3] : c1.w[i & 3]) : 0.f;
            const __bf16 hi = (__bf16)x;
            const float r1 = x - (float)hi;
            const __bf16 mid = (__bf16)r1;
            const float r2 = r1 - (float)mid;
            b[0][j][m][i] = low ? mid : hi;
            b[1][j][m][i] = low ? (__bf16)0.f : (__bf16)r2;
          }
        }
      }
  }
};

// What a wave reads for 64 entries.
template <int D>
struct Codes8 {
  Chunk16 k[4][D / 64];
  Chunk16 v[D / 16];
  f32x4u bias[2];   // of the entries whose weights the lane forms
  float ks, vs;
};

template <int D>
__device__ __forceinline__ void load_codes(Codes8<D>& x, const char* Kh, const char* Vh, const float* ks,
                                           const float* vs, const float* bh, int block_shift, int base, int e1,
                                           int col, int grp) {
  // 16-entry runs past the end are read at the group's first run instead and masked
  const int krun = base + 16 * (col >> 2) < e1 ? 16 * (col >> 2) : 0;
  const int vrun = base + 16 * grp < e1 ? 16 * grp : 0;
  const char* kp = Kh + (size_t)(base + krun + (col & 3)) * D + grp * 16;
  const char* vp = Vh + (size_t)(base + vrun) * D + col * 16;
#pragma unroll
  for (int s = 0; s < 4; ++s)
#pragma unroll
    for (int j = 0; j < D / 64; ++j) x.k[s][j] = load16(kp + (4 * s) * D + j * 64);
#pragma unroll
  for (int c = 0; c < D / 16; ++c) x.v[c] = load16(vp + c * 256);
  x.ks = ks[(base + vrun) >> block_shift];
  x.vs = vs[(base + vrun) >> block_shift];
  if (bh) {
#pragma unroll
    for (int s = 0; s < 2; ++s)
      x.bias[s] = *reinterpret_cast<const f32x4u*>(bh + base + vrun + (col & 8) + 4 * s);
  }
}

// Softmax state of a wave: lane (column, grp) keeps its column's maximum, the sum over the entries whose weights it
// forms and rows 4 grp .. + 3 of every 16-channel tile of O^T.
template <int D>
struct Wave8 {
  float m, l;
  f32x4 o[D / 16];
};

typedef float f32x2 __attribute__((ext_vector_type(2)));

// x as a sum of three bf16 numbers, two values to a word: the first rounds x, each further one what is left.
__device__ __forceinline__ void split3(float x0, float x1, uint32_t& hi, uint32_t& mid, uint32_t& lo) {
  hi = __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{x0, x1}, bf16x2));
  x0 -= __uint_as_float(hi << 16);
  x1 -= __uint_as_float(hi & 0xffff0000u);
  mid = __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{x0, x1}, bf16x2));
  x0 -= __uint_as_float(mid << 16);
  x1 -= __uint_as_float(mid & 0xffff0000u);
  lo = __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{x0, x1}, bf16x2));
}

__device__ __forceinline__ uint32_t row_ror8(uint32_t v) {
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x128, 0xf, 0xf, false);
}

template <typename T, int D, int CODE>
__device__ __forceinline__ void attend_codes(Wave8<D>& st, const Codes8<D>& x, const Query8<T, D>& q, float scale,
                                             bool has_bias, bool in, bool low) {
  f32x4 s[4];
#pragma unroll
  for (int t = 0; t < 4; ++t) {
    s[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int j = 0; j < D / 64; ++j) {
      const bf16x8 k0 = half_to_bf16<CODE, 0>(x.k[t][j]), k1 = half_to_bf16<CODE, 1>(x.k[t][j]);
#pragma unroll
      for (int p = 0; p < Query8<T, D>::kParts; ++p) {
        s[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k0, q.b[p][j][0], s[t], 0, 0, 0);
        s[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k1, q.b[p][j][1], s[t], 0, 0, 0);
      }
    }
  }
  // Columns h and h + 8 hold the same head: the first forms the weights of its lane's first eight entries (tiles 0 and
  // 1), the second those of the others, and they exchange them as bf16 words.
  const float c = scale * x.ks;
  float y[8], mx = kNegInf;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    float dot = low ? s[2 + i / 4][i % 4] : s[i / 4][i % 4];
    if constexpr (sizeof(T) == 4) dot += row_ror<8>(low ? s[i / 4][i % 4] : s[2 + i / 4][i % 4]);   // the query's parts
    const float b = has_bias ? x.bias[i / 4][i % 4] : 0.f;
    y[i] = in && b != kNegInf ? fmaf(dot, c, b) : kNegInf;   // selected: the product may be infinite or NaN
    mx = fmaxf(mx, y[i]);
  }
  mx = fmaxf(mx, row_ror<8>(mx));
  mx = max_xor32(max_xor16(mx));
  const float mnew = fmaxf(st.m, mx);
  const float ref = mnew == kNegInf ? 0.f : mnew;   // nothing unmasked yet: every weight is 0
  if (__any(mnew != st.m)) {
    const float corr = fast_exp2((st.m - ref) * kLog2e);
    st.l *= corr;
#pragma unroll
    for (int i = 0; i < D / 16; ++i) st.o[i] *= corr;
    st.m = mnew;
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    y[i] = fast_exp2((y[i] - ref) * kLog2e);
    st.l += y[i];
    y[i] *= x.vs;
  }
  Chunk16 w0, w1, l0, l1;   // the lane's entries 0 .. 7 and 8 .. 15: head columns the first term, the others the second
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    uint32_t hi, mid, lo;
    split3(y[2 * k], y[2 * k + 1], hi, mid, lo);
    const uint32_t other = row_ror8(low ? hi : mid), other_lo = row_ror8(lo);
    w0.w[k] = low ? other : hi;
    w1.w[k] = low ? mid : other;
    l0.w[k] = low ? 0u : lo;
    l1.w[k] = low ? 0u : other_lo;
  }
  const bf16x8 w[2] = {__builtin_bit_cast(bf16x8, w0), __builtin_bit_cast(bf16x8, w1)};
  const bf16x8 w_lo[2] = {__builtin_bit_cast(bf16x8, l0), __builtin_bit_cast(bf16x8, l1)};
#pragma unroll
  for (int i = 0; i < D / 16; ++i) {
    const bf16x8 v0 = half_to_bf16<CODE, 0>(x.v[i]), v1 = half_to_bf16<CODE, 1>(x.v[i]);
    st.o[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v0, w_lo[0], st.o[i], 0, 0, 0);
    st.o[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v1, w_lo[1], st.o[i], 0, 0, 0);
    st.o[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v0, w[0], st.o[i], 0, 0, 0);
    st.o[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v1, w[1], st.o[i], 0, 0, 0);
  }
}

// One wave's share of the open block's rows for gn <= kTailG query heads (those at qh): lane group grp takes rows
// r0 + 4 u + grp, r0 going from `first` by `step`.  rows: those of the block, the appended one (row `fresh`, or -1)
// last among them.  Leaves the wave's maximum, sum and outputs in LDS.
template <typename T, int D>
struct TailRows {
  static constexpr int U = sizeof(T) == 2 ? 4 : 2;   // rows of a lane group in flight
  RawSlice<T, D> k[U], v[U];
  float b[U];
  __device__ __forceinline__ void load(const char* kt, const char* vt, const char* k_new, const char* v_new,
                                       const float* bias, int r0, int rows, int fresh, int col, int grp) {
    constexpr int RB = D * (int)sizeof(T);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int r = min(r0 + 4 * u + grp, rows - 1);
      const bool f = r == fresh;
      k[u].load(f ? k_new : kt + (size_t)r * RB, col);
      v[u].load(f ? v_new : vt + (size_t)r * RB, col);
      b[u] = bias && !f ? bias[r] : 0.f;
    }
  }
};

template <typename T, int D>
__device__ __forceinline__ void attend_tail(const char* qh, const char* kt, const char* vt, const char* k_new,
                                            const char* v_new, const float* bias, int rows, int fresh, float scale,
                                            int gn, int first, int step, int col, int grp, float* s_m, float* s_l,
                                            float (*s_o)[D]) {
  constexpr int E = D / 16;
  constexpr int RB = D * (int)sizeof(T);
  constexpr int U = TailRows<T, D>::U;
  float q[kTailG][E], m[kTailG], l[kTailG], o[kTailG][E];
  RawSlice<T, D> qr[kTailG];
  TailRows<T, D> x;
  if (first < rows) {   // queries and the first rows in one trip to memory
#pragma unroll
    for (int g = 0; g < kTailG; ++g) qr[g].load(qh + (size_t)min(g, gn - 1) * RB, col);
    x.load(kt, vt, k_new, v_new, bias, first, rows, fresh, col, grp);
  }
#pragma unroll
  for (int g = 0; g < kTailG; ++g) {
    m[g] = kNegInf;
    l[g] = 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      q[g][e] = qr[g].get(e);
      o[g][e] = 0.f;
    }
  }
  for (int r0 = first; r0 < rows; r0 += step) {
    bool in[U];
#pragma unroll
    for (int u = 0; u < U; ++u) in[u] = r0 + 4 * u + grp < rows && x.b[u] != kNegInf;
#pragma unroll
    for (int g = 0; g < kTailG; ++g) {
      float y[U], mnew = m[g];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        float dot = 0.f;
#pragma unroll
        for (int e = 0; e < E; ++e) dot = fmaf(q[g][e], x.k[u].get(e), dot);
        dot = sum16(dot);
        y[u] = in[u] ? fmaf(dot, scale, x.b[u]) : kNegInf;
        mnew = fmaxf(mnew, y[u]);
      }
      const float ref = mnew == kNegInf ? 0.f : mnew;
      const float corr = fast_exp2((m[g] - ref) * kLog2e);
      m[g] = mnew;
      l[g] *= corr;
#pragma unroll
      for (int e = 0; e < E; ++e) o[g][e] *= corr;
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const float p = fast_exp2((y[u] - ref) * kLog2e);
        l[g] += p;
#pragma unroll
        for (int e = 0; e < E; ++e) o[g][e] = in[u] ? fmaf(p, x.v[u].get(e), o[g][e]) : o[g][e];
      }
    }
    if (r0 + step < rows) x.load(kt, vt, k_new, v_new, bias, r0 + step, rows, fresh, col, grp);
  }
  // the four lane groups of the wave
#pragma unroll
  for (int g = 0; g < kTailG; ++g) {
    const float M = max_xor32(max_xor16(m[g]));
    const float c = weight_of(m[g], M);
    l[g] = add_xor32(add_xor16(l[g] * c));
#pragma unroll
    for (int e = 0; e < E; ++e) o[g][e] = add_xor32(add_xor16(o[g][e] * c));
    if (g < gn && grp == 0) {
      if (col == 0) {
        s_m[g] = nan_counts(M, l[g]);
        s_l[g] = l[g];
      }
#pragma unroll
      for (int e = 0; e < E; ++e) s_o[g][col * E + e] = o[g][e];
    }
  }
}

// What a workgroup takes.  Split: four waves over codes or, slot 0, over the tail; the partials go to the workspace.
// Solo4: the head, tail after codes.  Solo8: the head, four waves over codes and four over the tail side by side.
enum Role8 { kSplit, kSolo4, kSolo8 };

template <typename T, int D, int CODE, bool APP, Role8 ROLE>
__global__ __launch_bounds__(ROLE == kSolo8 ? 2 * kThreads : kThreads,
                                  ROLE != kSolo8 && sizeof(T) == 2 ? 3 : 2) void decode8_kernel(DecodeArgs8 a) {
  constexpr bool SOLO = ROLE != kSplit;
  constexpr int NT = ROLE == kSolo8 ? 2 * kThreads : kThreads;
  constexpr int kParts = SOLO ? 2 * kWaves : kWaves;
  constexpr int RB = D * (int)sizeof(T);
  // the waves' results over codes, then (where the workgroup takes both) those over the tail
  __shared__ float s_m[kParts][kMaxG], s_l[kParts][kMaxG];
  __shared__ __align__(16) float s_o[kParts][kMaxG][D];
  __shared__ float s_max[4];
  const uint32_t head = blockIdx.y;
  const int slot = blockIdx.x, G = a.G;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int col = lane & 15, grp = lane >> 4;
  const int shift = a.block_shift, block = 1 << shift, cap = a.c.capacity;
  const int len = entries_of(a.n, head, a.hkv);
  const bool active = len >= 0;
  const int whole = active ? len >> shift << shift : 0;  // entries held as codes
  const int rest = active ? len - whole : 0;             // rows in the tail
  const bool codes_here = ROLE == kSolo8 ? wave < kWaves : SOLO || slot > 0;
  const bool tail_here = ROLE == kSolo8 ? wave >= kWaves : SOLO || slot == 0;
  const float* bh = a.bias ? a.bias + (size_t)head * cap : nullptr;
  const char* qh = a.q + (size_t)head * G * RB;

  if (codes_here) {
    const int chunk = SOLO ? whole : chunk_of(a, whole);
    const int e0 = SOLO ? 0 : (slot - 1) * chunk;
    const int e1 = min(e0 + chunk, whole);
    if (!SOLO && e0 >= e1) return;   // behind a shorter sequence's end: the combining kernel does not read the slot
    const char* Kh = a.c.K + (size_t)head * cap * D;
    const char* Vh = a.c.V + (size_t)head * cap * D;
    const float* ks = a.c.k_scale + (size_t)head * (cap >> shift);
    const float* vs = a.c.v_scale + (size_t)head * (cap >> shift);
    Query8<T, D> q;
    q.load(qh, G, col, grp);
    Wave8<D> st;
    st.m = kNegInf;
    st.l = 0.f;
#pragma unroll
    for (int i = 0; i < D / 16; ++i) st.o[i] = f32x4{0.f, 0.f, 0.f, 0.f};
    for (int e = e0 + wave * kGroup; e < e1; e += kWaves * kGroup) {
      Codes8<D> x;
      load_codes<D>(x, Kh, Vh, ks, vs, bh, shift, e, e1, col, grp);
      attend_codes<T, D, CODE>(st, x, q, a.scale, bh != nullptr, e + 16 * grp < e1, col >= 8);
    }
    st.l += row_ror<8>(st.l);
    st.l = add_xor32(add_xor16(st.l));
    st.m = nan_counts(st.m, st.l);
#pragma unroll
    for (int i = 0; i < D / 16; ++i) {
      f32x4 o = st.o[i];
#pragma unroll
      for (int r = 0; r < 4; ++r) o[r] += row_ror<8>(o[r]);   // both parts of the head's weights
      if (col < G) *reinterpret_cast<f32x4*>(&s_o[wave][col][16 * i + 4 * grp]) = o;
    }
    if (col < G && grp == 0) {
      s_m[wave][col] = st.m;
      s_l[wave][col] = st.l;
    }
  }
  if (tail_here) {
    // with more than kTailG query heads half of the waves take the rest of them
    const int w = wave % kWaves, half = G > kTailG ? 2 : 1, g0 = w / (kWaves / half) * kTailG;
    const int at = SOLO ? kWaves + w : w;
    const int per_wave = 4 * TailRows<T, D>::U;
    const size_t row0 = (size_t)head << shift;
    // the heads that the wave does not take: no lane of it stores their maximum again below
    if (lane < kMaxG && lane / kTailG != g0 / kTailG) s_m[at][lane] = kNegInf;
    attend_tail<T, D>(qh + (size_t)g0 * RB, a.c.k_tail + row0 * RB, a.c.v_tail + row0 * RB,
                      APP ? a.k_new + (size_t)head * RB : nullptr, APP ? a.v_new + (size_t)head * RB : nullptr,
                      bh ? bh + whole : nullptr, active ? rest + (APP ? 1 : 0) : 0, APP ? rest : -1, a.scale,
                      min(G - g0, kTailG), w % (kWaves / half) * per_wave, kWaves / half * per_wave, col, grp,
                      &s_m[at][g0], &s_l[at][g0], &s_o[at][g0]);
  }
  __syncthreads();
  for (int idx = threadIdx.x; idx < G * (D / 4); idx += NT) {
    const int g = idx / (D / 4), c4 = idx % (D / 4);
    float M = kNegInf, l = 0.f;
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < kParts; ++w) M = fmaxf(M, s_m[w][g]);
#pragma unroll
    for (int w = 0; w < kParts; ++w) {
      const float c = weight_of(s_m[w][g], M);
      const bool some = s_m[w][g] != kNegInf;        // a part without entries may hold anything
      const f32x4 ow = *reinterpret_cast<const f32x4*>(&s_o[w][g][c4 * 4]);
      l = some ? fmaf(s_l[w][g], c, l) : l;
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] = some ? fmaf(ow[e], c, o[e]) : o[e];
    }
    if (SOLO || whole == 0) {
      f32x4 r;
#pragma unroll
      for (int e = 0; e < 4; ++e) r[e] = l == 0.f ? 0.f : o[e] / l;
      *reinterpret_cast<f32x4*>(a.out + ((size_t)head * G + g) * D + c4 * 4) = r;
    } else {
      const size_t part = ((size_t)head * a.slots + slot) * G + g;
      *reinterpret_cast<f32x4*>(a.part_o + part * D + c4 * 4) = o;
      if (c4 == 0) a.part_ml[part] = make_float2(M, l);
    }
  }

  // the appended token: its row into the tail, the bias 0, and the block it completes into codes.  Nothing else in the
  // launch reads what is written here.
  if (APP && (SOLO || slot == 0) && active) {
    char* kt = a.c.k_tail + (size_t)head * block * RB;
    char* vt = a.c.v_tail + (size_t)head * block * RB;
    const char* kn = a.k_new + (size_t)head * RB;
    const char* vn = a.v_new + (size_t)head * RB;
    if (a.bias && threadIdx.x == 0) a.bias[(size_t)head * cap + len] = 0.f;
    if (threadIdx.x < RB / 16) {
      store16(kt + (size_t)rest * RB + threadIdx.x * 16, load16(kn + threadIdx.x * 16));
      store16(vt + (size_t)rest * RB + threadIdx.x * 16, load16(vn + threadIdx.x * 16));
    }
    if (rest + 1 == block) {
      const BlockThread bt = block_thread<D>(threadIdx.x, block);
      const int byte = bt.c4 * 4 * (int)sizeof(T);
      const size_t entry = (size_t)head * cap + whole, blk = (size_t)head * (cap >> shift) + (whole >> shift);
      for (int v = 0; v < 2; ++v) {
        const char* t = v ? vt : kt;
        const char* n = v ? vn : kn;
        quantise_blocks<T, D, CODE>(
            bt.sub == 0, bt, block, v != 0,
            [&](int i) {
              const int r = bt.tile * 16 + i;
              return (r == rest ? n : t + (size_t)r * RB) + byte;
            },
            (v ? a.c.V : a.c.K) + entry * D, (v ? a.c.v_scale : a.c.k_scale) + blk, s_max);
      }
    }
  }
}

// Combines the partials of the query heads, in slot order.  A unit of d/4 threads takes four channels each of the
// slots sub, sub + SUB, ... of a query head and loads kBatch of them at a time; with SUB > 1 the runs then meet in
// LDS, in order.  SUB = 1 where a head has few slots (64 x 8 heads of 2048 entries in 5 slots each 59.1 us, 61.4 with a
// workgroup a query head), otherwise the whole workgroup takes one query head: 64 slots in one trip to memory (16 x 8
// ragged heads of 25 slots 34.6 us, 36.1 with SUB = 1).  The kernel is a chain of latencies (3 - 4 us, two of them what any kernel takes), so its code
// is kept short.
template <int D, int SUB>
__global__ __launch_bounds__(256) void decode8_reduce_kernel(DecodeArgs8 a, int qheads) {
  constexpr int kUnits = 256 / (D / 4);   // 8 or 16
  constexpr int kBatch = 8;
  static_assert(SUB == 1 || SUB == kUnits, "a unit is a query head, or all of them are one");
  __shared__ float s_m[kUnits], s_l[kUnits];
  __shared__ __align__(16) float s_o[kUnits][D];
  const int c4 = threadIdx.x % (D / 4), unit = threadIdx.x / (D / 4), sub = SUB == 1 ? 0 : unit;
  const uint32_t qh = SUB == 1 ? min(blockIdx.x * kUnits + unit, (uint32_t)qheads - 1) : blockIdx.x;
  const uint32_t head = qh / (uint32_t)a.G, g = qh % (uint32_t)a.G;
  const int len = entries_of(a.n, head, a.hkv);
  const int whole = len > 0 ? len >> a.block_shift << a.block_shift : 0;
  if (whole == 0) return;                               // the tail alone: its workgroup wrote the outputs
  const int chunk = chunk_of(a, whole);
  const int slots = 1 + (whole + chunk - 1) / chunk;    // the tail's and those of the splits that had entries
  const float2* ml = a.part_ml + (size_t)head * a.slots * a.G + g;
  const float* po = a.part_o + ((size_t)head * a.slots * a.G + g) * D + c4 * 4;
  float m = kNegInf, l = 0.f;
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  for (int s0 = sub; s0 < slots; s0 += SUB * kBatch) {
    f32x4 ov[kBatch];
    float2 v[kBatch];
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      const int sl = min(s0 + u * SUB, slots - 1);
      ov[u] = *reinterpret_cast<const f32x4*>(po + (size_t)sl * a.G * D);
      v[u] = ml[(size_t)sl * a.G];
    }
    float M = m;
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      if (s0 + u * SUB >= slots) v[u].x = kNegInf;     // the last slot again, of codes: finite outputs of weight 0
      M = fmaxf(M, v[u].x);
    }
    const float c = weight_of(m, M);
    l *= c;
    o *= c;
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      const float w = weight_of(v[u].x, M);
      l = fmaf(v[u].y, w, l);
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] = fmaf(ov[u][e], w, o[e]);
    }
    m = M;
  }
  if constexpr (SUB == 1) {
    const float inv = 1.f / l;
    if (blockIdx.x * kUnits + unit < (uint32_t)qheads)
      *reinterpret_cast<f32x4*>(a.out + (size_t)qh * D + c4 * 4) = l == 0.f ? f32x4{0.f, 0.f, 0.f, 0.f} : o * inv;
  } else {
    *reinterpret_cast<f32x4*>(&s_o[unit][c4 * 4]) = o;
    if (c4 == 0) {
      s_m[unit] = m;
      s_l[unit] = l;
    }
    __syncthreads();
    if (threadIdx.x >= D) return;
    float M = kNegInf, L = 0.f, t = 0.f;
#pragma unroll
    for (int k = 0; k < kUnits; ++k) M = fmaxf(M, s_m[k]);
#pragma unroll
    for (int k = 0; k < kUnits; ++k) {
      const float w = weight_of(s_m[k], M);
      t = fmaf(s_o[k][threadIdx.x], w, t);
      L = fmaf(s_l[k], w, L);
    }
    a.out[(size_t)qh * D + threadIdx.x] = L == 0.f ? 0.f : t / L;
  }
}

template <typename T, int D, int CODE, Role8 ROLE>
void launch_role(int64_t heads, const DecodeArgs8& a, hipStream_t st) {
  const dim3 grid(a.slots, (unsigned)heads), blk(ROLE == kSolo8 ? 2 * kThreads : kThreads);
  if (a.k_new) hipLaunchKernelGGL((decode8_kernel<T, D, CODE, true, ROLE>), grid, blk, 0, st, a);
  else hipLaunchKernelGGL((decode8_kernel<T, D, CODE, false, ROLE>), grid, blk, 0, st, a);
}

template <typename T, int D, int CODE>
hipError_t launch_tdc(int64_t heads, const DecodeArgs8& a, hipStream_t st) {
  if (a.slots == 1) {
    // eight waves where every head has a CU to itself (32 x 8 heads of 300 entries: 9.2 us, 10.1 in four); with more
    // heads the four that only see the tail cost too much (64 x 8 heads: 16.6 us, 14.2 in four)
    if (heads <= kCUs) launch_role<T, D, CODE, kSolo8>(heads, a, st);
    else launch_role<T, D, CODE, kSolo4>(heads, a, st);
    return hipGetLastError();
  }
  launch_role<T, D, CODE, kSplit>(heads, a, st);
  constexpr int kUnits = 256 / (D / 4);
  const int qheads = (int)heads * a.G;
  if (a.slots <= kFewSlots)
    hipLaunchKernelGGL((decode8_reduce_kernel<D, 1>), dim3((qheads + kUnits - 1) / kUnits), dim3(256), 0, st, a, qheads);
  else
    hipLaunchKernelGGL((decode8_reduce_kernel<D, kUnits>), dim3(qheads), dim3(256), 0, st, a, qheads);
  return hipGetLastError();
}

template <typename T, int D>
hipError_t launch_td(int64_t heads, const DecodeArgs8& a, hipStream_t st) {
  return a.c.code == SELKV_I8 ? launch_tdc<T, D, SELKV_I8>(heads, a, st) : launch_tdc<T, D, SELKV_E4M3>(heads, a, st);
}

// Entries up to which a workgroup takes a head by itself: a call over 500 entries of 8 heads (d = 128) takes 8.4 us so
// and 10.1 in splits with the second kernel, 700 entries 9.5 and 9.9, 900 entries 11.3 and 10.1; at d = 64, half the
// work, 900 entries (fp32 queries) 9.3 and 10.3 us, 1500 entries 11.8 and 10.3.
int solo_entries(int d) { return d == 64 ? 1024 : 768; }

// Most splits of one head: those that give the chip kRounds rounds of workgroups, none shorter than one step of its
// four waves; none where the heads alone are a round.  That is best where they fill whole rounds (768 heads of 2048
// entries take 77 us so and 105 in splits, of 8192 entries 308 and 369) and costs up to an eighth elsewhere: 800 heads of
// 2048 entries 89 and 86 us, of 8192 entries 350 and 309, 1024 heads 431 and 389; lengths spread over 0 .. 8192, 768
// heads 186 and 166 us.  Where few sequences are far longer than the rest it costs more: one of 25600 entries
// among 95 of 1000, 8 heads each, takes 194 us, and among 94 of them, in splits, 60.
int64_t most_splits(int64_t heads, int64_t groups) {
  if (heads >= kTargetBlocks) return 1;
  return std::max<int64_t>(1, std::min({(kRounds * kTargetBlocks + heads - 1) / heads, (groups + kWaves - 1) / kWaves,
                                        (int64_t)kMaxSplit}));
}

// Groups of a split where a head of `groups` is to have about `want` of them: whole steps of the four waves.
int64_t split_groups(int64_t groups, int64_t want) {
  return ((groups + want - 1) / want + kWaves - 1) / kWaves * kWaves;
}

size_t partial_bytes(int64_t heads, int64_t slots, int d, int G, size_t* ml) {
  *ml = ((size_t)heads * slots * G * sizeof(float2) + 255) & ~(size_t)255;
  return *ml + (((size_t)heads * slots * G * d * sizeof(float) + 255) & ~(size_t)255);
}

}  // namespace

// Splits.  Several rounds of workgroups let fast ones make up for slow ones and for sequences of other lengths: 4 x 32
// heads of 4096 entries take 29.4 us in 2048 workgroups, 32.8 in 768; ragged batches of up to 8100 entries, 16 x 8 heads
// 33.9 us, 38.7 in one round and 36.4 in two, 24 x 8 heads 49 us, 53 in two and 52 in three.  (A sequence of its own
// length is cut anew on the device, chunk_of.)  Every workgroup costs its prologue and its partials, though, so one
// round is taken where it comes out even: 32 x 8 heads of 25641 entries take 300 us in 768 workgroups, 308 in 2304 (but
// 16 x 8 such heads 162 and 158 us, 48 x 8 heads of 8192 entries 178 and 157: there several rounds would be better); and
// a round that is barely exceeded is not begun: 8 heads of 25600 entries take 15.3 us in 400 workgroups, 16.7 in 800.
Decode8Plan plan_decode8(int64_t heads, int cache_len, int d, int G, bool ragged) {
  Decode8Plan p{};
  const int64_t groups = ((int64_t)cache_len + kGroup - 1) / kGroup;
  const int64_t most = most_splits(heads, groups);
  p.slots = 1;
  if (cache_len <= solo_entries(d) || most == 1) return p;
  const auto splits = [&](int64_t per) { return (groups + per - 1) / per; };
  int64_t per = split_groups(groups, most);
  const int64_t even = split_groups(groups, std::clamp<int64_t>(kTargetBlocks / heads, 1, most));   // one round, if it is full
  if (!ragged && heads * splits(even) > kTargetBlocks * 9 / 10 && heads * splits(even) <= kTargetBlocks &&
      splits(even) * even - groups <= groups / 16)
    per = even;
  if (heads * splits(per) < kTargetBlocks * 3 / 2)
    while (heads * splits(per) > kTargetBlocks && per < groups) per += kWaves;
  p.chunk = (int)(per * kGroup);
  p.slots = (int)splits(per) + 1;
  p.bytes = partial_bytes(heads, p.slots, d, G, &p.ml_bytes);
  return p;
}

// Covers plan_decode8 at every length up to the capacity: its splits are at most most_splits(), which grows with it.
size_t decode8_workspace_bound(int64_t heads, int capacity, int d, int G) {
  size_t ml;
  const int64_t groups = ((int64_t)capacity + kGroup - 1) / kGroup;
  const int64_t most = most_splits(heads, groups);
  return capacity <= solo_entries(d) || most == 1 ? 0 : partial_bytes(heads, most + 1, d, G, &ml);
}

hipError_t launch_decode8(int64_t heads, int hkv, int d, int G, int dtype, float scale, const Decode8Plan& p,
                          const Cache8& c, const Lens8& n, const void* q, float* bias, const void* k_new,
                          const void* v_new, float* out, void* ws, hipStream_t st) {
  DecodeArgs8 a{};
  a.c = c;
  a.n = n;
  a.q = static_cast<const char*>(q);
  a.bias = bias;
  a.out = out;
  a.part_ml = static_cast<float2*>(ws);
  a.part_o = reinterpret_cast<float*>(static_cast<char*>(ws) + p.ml_bytes);
  a.k_new = static_cast<const char*>(k_new);
  a.v_new = static_cast<const char*>(v_new);
  a.hkv = hkv;
  a.G = G;
  a.slots = p.slots;
  a.chunk = p.chunk;
  a.block_shift = 31 - __builtin_clz((unsigned)c.block);
  a.scale = scale;
  if (dtype == SELKV_BF16) return d == 128 ? launch_td<bf16_t, 128>(heads, a, st) : launch_td<bf16_t, 64>(heads, a, st);
  return d == 128 ? launch_td<float, 128>(heads, a, st) : launch_td<float, 64>(heads, a, st);
}

}  // namespace selkv
