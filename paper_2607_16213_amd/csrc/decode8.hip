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
// one more workgroup per head the tail; each writes (max, sum, o[d]) per query
// head to the workspace and a second kernel combines them in slot order.
// Where one workgroup takes the whole head it writes the outputs itself.
//
// The codes go to the matrix cores as bf16, which holds every int8 and e4m3
// number exactly.  A wave takes 64 entries at a time: four 16x16x32 tiles
// S = K Q^T, then O^T += V^T P^T.  Of a tile's 16 columns the G <= 8 query
// heads need at most 8, so column h + 8 carries what column h's bf16 leaves of
// the same head, of an fp32 query and of a softmax weight: the next 8 bits, and
// a second product the last 8, so both enter as the fp32 numbers they are (with
// two terms the weight that dominates a peaked softmax was off by up to 2^-18,
// 5.5e-6 of an output).  Which entry is which row of an S tile
// is chosen so that a lane's logits are 16 consecutive entries, those whose V
// codes it reads with one 16-byte load: P needs no exchange between lanes and
// one scale of K and of V serves a lane's 64-entry step.  Scales stay out of the
// products: K's multiplies the logits, V's the weights.
// The running maximum and sum of the softmax, and all accumulators, are fp32.
// The tail (and the appended token) are few rows, taken in fp32 by lane groups
// of 16 lanes, each lane d/16 channels.
// A masked entry (bias -inf) is left out by selection, so it may hold anything.
#include "cache8.hpp"

namespace selkv {
namespace {

constexpr int kWaves = 4;
constexpr int kThreads = kWaves * 64;
constexpr int kMaxG = 8;
constexpr int kGroup = 64;            // entries that splits are whole multiples of
constexpr int kTargetBlocks = 512;    // workgroups a launch aims at
constexpr int kMaxSplit = 1024;

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
  int hkv, G, nsplit, slots;
  float scale;
};

// Softmax state of one lane group: G heads, E channels of the lane.
template <int E>
struct State8 {
  float m[kMaxG], l[kMaxG], o[kMaxG][E];
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int g = 0; g < kMaxG; ++g) {
      m[g] = kNegInf;
      l[g] = 0.f;
#pragma unroll
      for (int e = 0; e < E; ++e) o[g][e] = 0.f;
    }
  }
};

// One entry per lane group: its logits, then the running softmax.  `in`: the entry counts (its k, v may be anything
// where it does not).
template <int E>
__device__ __forceinline__ void attend(State8<E>& s, const float (&q)[kMaxG][E], int G, const float (&k)[E],
                                       const float (&v)[E], float c, float bias, bool in) {
#pragma unroll
  for (int g = 0; g < kMaxG; ++g) {
    if (g >= G) break;
    float dot = 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e) dot = fmaf(q[g][e], k[e], dot);
    dot = sum16(dot);
    if (!in) continue;
    const float x = fmaf(dot, c, bias);
    const float mnew = fmaxf(s.m[g], x);
    const float corr = fast_exp2((s.m[g] - mnew) * kLog2e);   // 0 while m is -inf
    const float p = fast_exp2((x - mnew) * kLog2e);
    s.l[g] = fmaf(s.l[g], corr, p);
#pragma unroll
    for (int e = 0; e < E; ++e) s.o[g][e] = fmaf(s.o[g][e], corr, p * v[e]);
    s.m[g] = mnew;
  }
}

template <typename T, int D>
__device__ __forceinline__ void load_row(const char* row, int col, float (&x)[D / 16]) {
  RawSlice<T, D> r;
  r.load(row, col);
#pragma unroll
  for (int e = 0; e < D / 16; ++e) x[e] = r.get(e);
}

// Weight of partial (m, .) against the maximum M of all (0 where it is empty).
__device__ __forceinline__ float weight_of(float m, float M) {
  return m == kNegInf ? 0.f : fast_exp2((m - M) * kLog2e);
}

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
  f32x4u bias[4];
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
    for (int s = 0; s < 4; ++s) x.bias[s] = *reinterpret_cast<const f32x4u*>(bh + base + vrun + 4 * s);
  }
}

// Softmax state of a wave: lane (column, grp) keeps its column's maximum, the sum over its own entries and rows
// 4 grp .. + 3 of every 16-channel tile of O^T.
template <int D>
struct Wave8 {
  float m, l;
  f32x4 o[D / 16];
};

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
  const float c = scale * x.ks;
  float mx = kNegInf;
#pragma unroll
  for (int t = 0; t < 4; ++t)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      float dot = s[t][r];
      if constexpr (sizeof(T) == 4) dot += row_ror<8>(dot);   // both parts of the head's query
      const float y = fmaf(dot, c, has_bias ? x.bias[t][r] : 0.f);
      s[t][r] = in ? y : kNegInf;
      mx = fmaxf(mx, s[t][r]);
    }
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
  bf16x8 w[2], w_lo[2];
#pragma unroll
  for (int t = 0; t < 4; ++t)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const float p = fast_exp2((s[t][r] - ref) * kLog2e);
      st.l += p;
      const float y = p * x.vs;
      const __bf16 hi = (__bf16)y;
      const float r1 = y - (float)hi;
      const __bf16 mid = (__bf16)r1;
      w[t >> 1][(t & 1) * 4 + r] = low ? mid : hi;
      w_lo[t >> 1][(t & 1) * 4 + r] = low ? (__bf16)0.f : (__bf16)(r1 - (float)mid);
    }
#pragma unroll
  for (int i = 0; i < D / 16; ++i) {
    const bf16x8 v0 = half_to_bf16<CODE, 0>(x.v[i]), v1 = half_to_bf16<CODE, 1>(x.v[i]);
    st.o[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v0, w_lo[0], st.o[i], 0, 0, 0);
    st.o[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v1, w_lo[1], st.o[i], 0, 0, 0);
    st.o[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v0, w[0], st.o[i], 0, 0, 0);
    st.o[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v1, w[1], st.o[i], 0, 0, 0);
  }
}

template <typename T, int D, int CODE, bool APP>
__global__ __launch_bounds__(kThreads, 2) void decode8_kernel(DecodeArgs8 a) {
  constexpr int E = D / 16;
  constexpr int RB = D * (int)sizeof(T);
  // the waves' results over codes, then (where the workgroup takes both) those over the tail
  __shared__ float s_m[2 * kWaves][kMaxG], s_l[2 * kWaves][kMaxG];
  __shared__ __align__(16) float s_o[2 * kWaves][kMaxG][D];
  __shared__ float s_max[4];
  const int64_t head = blockIdx.y;
  const int slot = blockIdx.x, G = a.G;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int col = lane & 15, grp = lane >> 4;
  const int block = a.c.block, cap = a.c.capacity;
  const int len = entries_of(a.n, (int)(head / a.hkv));
  const bool active = len >= 0;
  const int whole = active ? len / block * block : 0;    // entries held as codes
  const int rest = active ? len - whole : 0;             // rows in the tail
  const bool solo = a.slots == 1;
  const bool codes_here = slot < a.nsplit, tail_here = solo || slot == a.nsplit;
  const float* bh = a.bias ? a.bias + (size_t)head * cap : nullptr;
  const char* qh = a.q + (size_t)head * G * RB;

  if (codes_here) {
    const int groups = (whole + kGroup - 1) / kGroup;
    const int e0 = (int)((int64_t)groups * slot / a.nsplit) * kGroup;
    const int e1 = min((int)((int64_t)groups * (slot + 1) / a.nsplit) * kGroup, whole);
    const char* Kh = a.c.K + (size_t)head * cap * D;
    const char* Vh = a.c.V + (size_t)head * cap * D;
    const int shift = 31 - __builtin_clz(block);
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
    st.l = add_xor32(add_xor16(st.l));
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
    float q[kMaxG][E];
#pragma unroll
    for (int g = 0; g < kMaxG; ++g)
      if (g < G) load_row<T, D>(qh + (size_t)g * RB, col, q[g]);
    State8<E> s;
    s.clear();
    const char* kt = a.c.k_tail + (size_t)head * block * RB;
    const char* vt = a.c.v_tail + (size_t)head * block * RB;
    const int rows = active ? rest + (APP ? 1 : 0) : 0;
    for (int r0 = wave * 4; r0 < rows; r0 += kWaves * 4) {
      const int r = min(r0 + grp, rows - 1);
      const bool fresh = APP && r == rest;
      float k[E], v[E];
      load_row<T, D>(fresh ? a.k_new + (size_t)head * RB : kt + (size_t)r * RB, col, k);
      load_row<T, D>(fresh ? a.v_new + (size_t)head * RB : vt + (size_t)r * RB, col, v);
      const float b = bh && !fresh ? bh[whole + r] : 0.f;
      attend<E>(s, q, G, k, v, a.scale, b, r0 + grp < rows && b != kNegInf);
    }
    // the four lane groups of a wave
    const int at = codes_here ? kWaves + wave : wave;
#pragma unroll
    for (int g = 0; g < kMaxG; ++g) {
      if (g >= G) break;
#pragma unroll
      for (int off = 16; off <= 32; off <<= 1) {
        const float m2 = xor_shfl(s.m[g], off), l2 = xor_shfl(s.l[g], off);
        const float M = fmaxf(s.m[g], m2);
        const float c1 = weight_of(s.m[g], M), c2 = weight_of(m2, M);
        s.l[g] = s.l[g] * c1 + l2 * c2;
#pragma unroll
        for (int e = 0; e < E; ++e) s.o[g][e] = s.o[g][e] * c1 + xor_shfl(s.o[g][e], off) * c2;
        s.m[g] = M;
      }
      if (grp == 0) {
        if (col == 0) {
          s_m[at][g] = s.m[g];
          s_l[at][g] = s.l[g];
        }
#pragma unroll
        for (int e = 0; e < E; ++e) s_o[at][g][col * E + e] = s.o[g][e];
      }
    }
  }
  __syncthreads();
  const int parts = solo ? 2 * kWaves : kWaves;
  for (int idx = threadIdx.x; idx < G * D; idx += kThreads) {
    const int g = idx / D, dd = idx % D;
    float M = kNegInf, l = 0.f, o = 0.f;
    for (int w = 0; w < parts; ++w) M = fmaxf(M, s_m[w][g]);
    for (int w = 0; w < parts; ++w) {
      const float c = weight_of(s_m[w][g], M);
      l = fmaf(s_l[w][g], c, l);
      o = fmaf(s_o[w][g][dd], c, o);
    }
    if (solo) {
      a.out[(size_t)head * G * D + idx] = l > 0.f ? o / l : 0.f;
    } else {
      a.part_o[((size_t)head * a.slots + slot) * G * D + idx] = o;
      if (dd == 0) a.part_ml[((size_t)head * a.slots + slot) * G + g] = make_float2(M, l);
    }
  }

  // the appended token: its row into the tail, the bias 0, and the block it completes into codes.  Nothing else in the
  // launch reads what is written here.
  if (APP && tail_here && active) {
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
      const size_t entry = (size_t)head * cap + whole, blk = (size_t)head * (cap / block) + whole / block;
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

// Combines the partials of a head in slot order: one workgroup per query head, thread (dd, sub) takes the slots sub,
// sub + S, ... of output channel dd, the S runs then meet in LDS.
template <int D>
__global__ __launch_bounds__(256) void decode8_reduce_kernel(const float* part_o, const float2* part_ml, float* out,
                                                             int slots, int G) {
  constexpr int S = 256 / D;
  constexpr int kBatch = 8;
  __shared__ float s_m[S], s_l[S], s_o[S][D];
  const int64_t head = blockIdx.x;
  const int g = blockIdx.y, dd = threadIdx.x % D, sub = threadIdx.x / D;
  const float2* ml = part_ml + (size_t)head * slots * G + g;
  const float* po = part_o + ((size_t)head * slots * G + g) * D + dd;
  float m = kNegInf, l = 0.f, o = 0.f;
  for (int s0 = sub; s0 < slots; s0 += S * kBatch) {
    float ov[kBatch];
    float2 v[kBatch];
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      const int sl = min(s0 + u * S, slots - 1);
      ov[u] = po[(size_t)sl * G * D];
      v[u] = ml[(size_t)sl * G];
      if (s0 + u * S >= slots) v[u].x = kNegInf;
    }
    float M = m;
#pragma unroll
    for (int u = 0; u < kBatch; ++u) M = fmaxf(M, v[u].x);
    const float c = weight_of(m, M);
    l *= c;
    o *= c;
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      const float w = weight_of(v[u].x, M);
      l = fmaf(v[u].y, w, l);
      o = fmaf(ov[u], w, o);
    }
    m = M;
  }
  s_o[sub][dd] = o;
  if (dd == 0) {
    s_m[sub] = m;
    s_l[sub] = l;
  }
  __syncthreads();
  if (sub == 0) {
    float M = kNegInf, L = 0.f, t = 0.f;
#pragma unroll
    for (int k = 0; k < S; ++k) M = fmaxf(M, s_m[k]);
#pragma unroll
    for (int k = 0; k < S; ++k) {
      const float w = weight_of(s_m[k], M);
      t = fmaf(s_o[k][dd], w, t);
      L = fmaf(s_l[k], w, L);
    }
    out[((size_t)head * G + g) * D + dd] = L > 0.f ? t / L : 0.f;
  }
}

template <typename T, int D, int CODE>
hipError_t launch_tdc(int64_t heads, const DecodeArgs8& a, hipStream_t st) {
  const dim3 grid(a.slots, (unsigned)heads);
  if (a.k_new) hipLaunchKernelGGL((decode8_kernel<T, D, CODE, true>), grid, dim3(kThreads), 0, st, a);
  else hipLaunchKernelGGL((decode8_kernel<T, D, CODE, false>), grid, dim3(kThreads), 0, st, a);
  if (a.slots > 1)
    hipLaunchKernelGGL((decode8_reduce_kernel<D>), dim3((unsigned)heads, a.G), dim3(256), 0, st, a.part_o, a.part_ml,
                       a.out, a.slots, a.G);
  return hipGetLastError();
}

template <typename T, int D>
hipError_t launch_td(int64_t heads, const DecodeArgs8& a, hipStream_t st) {
  return a.c.code == SELKV_I8 ? launch_tdc<T, D, SELKV_I8>(heads, a, st) : launch_tdc<T, D, SELKV_E4M3>(heads, a, st);
}

}  // namespace

// The number of splits grows with cache_len, so a workspace for the capacity serves every length.
Decode8Plan plan_decode8(int64_t heads, int cache_len, int d, int G) {
  Decode8Plan p{};
  const int64_t groups = ((int64_t)cache_len + kGroup - 1) / kGroup;
  int64_t nsplit = (kTargetBlocks + heads - 1) / heads;
  if (nsplit > (groups + 3) / 4) nsplit = (groups + 3) / 4;
  if (nsplit > kMaxSplit) nsplit = kMaxSplit;
  if (nsplit < 1) nsplit = 1;
  p.nsplit = (int)nsplit;
  p.slots = nsplit == 1 ? 1 : (int)nsplit + 1;
  if (p.slots == 1) return p;
  p.ml_bytes = ((size_t)heads * p.slots * G * sizeof(float2) + 255) & ~(size_t)255;
  p.bytes = p.ml_bytes + (((size_t)heads * p.slots * G * d * sizeof(float) + 255) & ~(size_t)255);
  return p;
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
  a.nsplit = p.nsplit;
  a.slots = p.slots;
  a.scale = scale;
  if (dtype == SELKV_BF16) return d == 128 ? launch_td<bf16_t, 128>(heads, a, st) : launch_td<bf16_t, 64>(heads, a, st);
  return d == 128 ? launch_td<float, 128>(heads, a, st) : launch_td<float, 64>(heads, a, st);
}

}  // namespace selkv
