// selkv_paged_append: rows into the pages of a cache, keys and queries turned by
// their rotary positions on the way; selkv_paged_keep: the rows of an accepted
// path, moved to the front of their tree's.
//
// Append.  Pair j of a row at position t turns by t * freq[j].  The angle, up to
// 1e5 rad and more, is formed in fp64; what is left of it beyond whole quarter
// turns goes to sine and cosine as fp32, an eighth of a turn at most and so
// within 2^-28 turns.  Each is computed once per token and pair and held in LDS
// for the heads of the workgroup.  A thread moves units of 16 channels, two runs
// of eight that hold eight whole pairs in either layout (channels 8 c and
// rot_dim / 2 + 8 c, or 16 c and 16 c + 8), so one body serves both, the
// channels that do not turn and the values.
#include <algorithm>

#include "paged.hpp"

namespace selkv {
namespace {

constexpr int kThreads = 256;
constexpr int kTokens = 8;      // most tokens of a workgroup
constexpr int kMaxNodes = 64;

struct AppendArgs {
  Paged c;
  Seqs n;
  RowsIn k, v, q;
  char* q_out;
  const float* bias_new;
  const int32_t* positions;
  const double* freq;
  float rope_scale;
  int rot, hkv, hq;      // hq: query heads that come along (0: none)
  int tokens, heads;     // of a workgroup
};

// Eight channels in storage type T.
template <typename T>
struct Run8 {
  static constexpr int kChunks = (int)sizeof(T) / 2;
  Chunk16 c[kChunks];
  __device__ __forceinline__ void load(const char* p) {
#pragma unroll
    for (int i = 0; i < kChunks; ++i) c[i] = load16(p + 16 * i);
  }
  __device__ __forceinline__ void store(char* p) const {
#pragma unroll
    for (int i = 0; i < kChunks; ++i) store16(p + 16 * i, c[i]);
  }
  __device__ __forceinline__ float get(int e) const {
    return Elem<T>::get(c[e / Elem<T>::kPerChunk], e % Elem<T>::kPerChunk);
  }
  __device__ __forceinline__ void put(int e, float x) {
    Elem<T>::put(c[e / Elem<T>::kPerChunk], e % Elem<T>::kPerChunk, x);
  }
};

// Cosine and sine of `angle` times `scale`.
__device__ __forceinline__ float2 turn_of(double angle, float scale) {
  constexpr double kInvTwoPi = 0.15915494309189533576888376337251;
  const double turns = angle * kInvTwoPi;
  const double part = turns - rint(turns);          // -1/2 .. 1/2
  const double quarter = rint(part * 4.0);          // -2 .. 2
  const float rest = 2.f * (float)(part - quarter * 0.25);
  const float s = sinpif(rest), c = cospif(rest);
  const int k = (int)quarter & 3;
  const float cs = k & 1 ? s : c, sn = k & 1 ? c : s;
  return make_float2((k == 1 || k == 2 ? -cs : cs) * scale, (k >= 2 ? -sn : sn) * scale);
}

enum { kNoRope = -1 };

template <typename T, int D, int ROPE>
__global__ __launch_bounds__(kThreads) void paged_append_kernel(AppendArgs a) {
  constexpr int UNITS = D / 16;                     // of a row
  constexpr int EB = (int)sizeof(T);
  __shared__ float2 s_turn[kTokens][ROPE == kNoRope ? 1 : D / 2];
  __shared__ int s_page[kTokens];
  const uint32_t b = blockIdx.z;
  int len, count;
  if (!sequence_of(a.n, b, len, count)) return;
  const int t0 = blockIdx.x * a.tokens;
  const int tokens = min(a.tokens, count - t0);
  if (tokens <= 0) return;
  const int all = 2 * a.hkv + a.hq;
  const int h0 = blockIdx.y * a.heads, heads = min(a.heads, all - h0);
  if ((int)threadIdx.x < tokens) s_page[threadIdx.x] = page_of(a.c, b, len + t0 + threadIdx.x);
  if constexpr (ROPE != kNoRope) {
    const int pairs = a.rot / 2;
    for (int i = threadIdx.x; i < tokens * pairs; i += kThreads) {
      const int t = i / pairs, j = i - t * pairs;
      const int pos = a.positions ? a.positions[(size_t)b * a.n.n + t0 + t] : len + t0 + t;
      s_turn[t][j] = turn_of((double)pos * a.freq[j], a.rope_scale);
    }
  }
  __syncthreads();
  const int turned = ROPE == kNoRope ? 0 : a.rot / 16;   // units of a row that turn
  const int units = tokens * heads * UNITS;
  for (int u = threadIdx.x; u < units; u += kThreads) {
    const int c = u % UNITS, row = u / UNITS;
    const int t = row / heads, h = h0 + row - t * heads;
    const int token = t0 + t;
    const bool query = h >= 2 * a.hkv, value = !query && h >= a.hkv;
    const RowsIn& in = query ? a.q : value ? a.v : a.k;
    const int ih = query ? h - 2 * a.hkv : value ? h - a.hkv : h;
    const bool turn = !value && c < turned;
    const int lo = turn && ROPE == SELKV_ROPE_HALF ? 8 * c : 16 * c;
    const int hi = turn && ROPE == SELKV_ROPE_HALF ? a.rot / 2 + 8 * c : 16 * c + 8;
    const char* src = in.data + (b * in.sb + token * in.sn + ih * in.sh) * EB;
    char* dst;
    if (query) {
      dst = a.q_out + (((size_t)b * a.n.n + token) * a.hq + ih) * D * EB;
    } else {
      const int page = s_page[t];
      if (page < 0) continue;
      dst = (value ? a.c.V : a.c.K) + row_of(a.c, a.hkv, page, ih, len + token) * D * EB;
    }
    Run8<T> x, y;
    x.load(src + lo * EB);
    y.load(src + hi * EB);
    if (turn) {
      if constexpr (ROPE == SELKV_ROPE_HALF) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float2 w = s_turn[t][8 * c + e];
          const float p = x.get(e), q = y.get(e);
          x.put(e, p * w.x - q * w.y);
          y.put(e, q * w.x + p * w.y);
        }
      } else if constexpr (ROPE == SELKV_ROPE_INTERLEAVED) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float2 w = s_turn[t][8 * c + e], z = s_turn[t][8 * c + 4 + e];
          const float p = x.get(2 * e), q = x.get(2 * e + 1), r = y.get(2 * e), s = y.get(2 * e + 1);
          x.put(2 * e, p * w.x - q * w.y);
          x.put(2 * e + 1, q * w.x + p * w.y);
          y.put(2 * e, r * z.x - s * z.y);
          y.put(2 * e + 1, s * z.x + r * z.y);
        }
      }
    }
    x.store(dst + lo * EB);
    y.store(dst + hi * EB);
  }
  if (a.c.bias) {
    for (int i = threadIdx.x; i < tokens * a.hkv; i += kThreads) {
      const int h = i / tokens, t = i - h * tokens;
      if (h < h0 || h >= h0 + heads || s_page[t] < 0) continue;   // with the head's keys
      a.c.bias[row_of(a.c, a.hkv, s_page[t], h, len + t0 + t)] =
          a.bias_new ? a.bias_new[((size_t)b * a.hkv + h) * a.n.n + t0 + t] : 0.f;
    }
  }
}

// One workgroup moves the rows of a KV head: all are read before the first is written.
template <typename T, int D>
__global__ __launch_bounds__(kThreads) void paged_keep_kernel(Paged c, Seqs n, const int32_t* path,
                                                              const int32_t* n_path) {
  constexpr int CH = D * (int)sizeof(T) / 16;              // 16-byte chunks of a row
  constexpr int LOADS = kMaxNodes * CH / kThreads;
  __shared__ int s_src[kMaxNodes], s_dst[kMaxNodes];       // pages, -1: the row stays
  __shared__ int s_node[kMaxNodes];
  const uint32_t b = blockIdx.y;
  const int h = blockIdx.x, hkv = gridDim.x;
  const int len = n.lens ? n.lens[b] : n.cache_len;
  const int rows = n_path[b];
  if ((uint32_t)len > (uint32_t)n.cache_len || (uint32_t)rows > (uint32_t)n.n) return;
  float moved = 0.f;
  size_t to = 0;
  bool moves = false;
  if ((int)threadIdx.x < rows) {
    const int j = threadIdx.x, node = path[(size_t)b * n.n + j];
    const bool some = node != j && (uint32_t)node < (uint32_t)n.n;
    const int src = some ? page_of(c, b, len + node) : -1;
    const int dst = src >= 0 ? page_of(c, b, len + j) : -1;
    s_src[j] = src;
    s_dst[j] = dst;
    s_node[j] = node;
    moves = dst >= 0 && c.bias;
    if (moves) {
      moved = c.bias[row_of(c, hkv, src, h, len + node)];
      to = row_of(c, hkv, dst, h, len + j);
    }
  }
  __syncthreads();
  Chunk16 k[LOADS], v[LOADS];
  size_t at[LOADS];
#pragma unroll
  for (int i = 0; i < LOADS; ++i) {
    const int u = threadIdx.x + i * kThreads, j = u / CH, part = u % CH;
    at[i] = ~(size_t)0;
    if (j < rows && s_dst[j] >= 0) {
      const size_t from = row_of(c, hkv, s_src[j], h, len + s_node[j]) * (D * sizeof(T)) + part * 16;
      at[i] = row_of(c, hkv, s_dst[j], h, len + j) * (D * sizeof(T)) + part * 16;
      k[i] = load16(c.K + from);
      v[i] = load16(c.V + from);
    }
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < LOADS; ++i) {
    if (at[i] == ~(size_t)0) continue;
    store16(c.K + at[i], k[i]);
    store16(c.V + at[i], v[i]);
  }
  if (moves) c.bias[to] = moved;
}

template <typename T, int D>
hipError_t launch_append_t(const AppendArgs& a, int layout, dim3 grid, hipStream_t st) {
  if (layout == SELKV_ROPE_HALF)
    hipLaunchKernelGGL((paged_append_kernel<T, D, SELKV_ROPE_HALF>), grid, dim3(kThreads), 0, st, a);
  else if (layout == SELKV_ROPE_INTERLEAVED)
    hipLaunchKernelGGL((paged_append_kernel<T, D, SELKV_ROPE_INTERLEAVED>), grid, dim3(kThreads), 0, st, a);
  else
    hipLaunchKernelGGL((paged_append_kernel<T, D, kNoRope>), grid, dim3(kThreads), 0, st, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_paged_append(int batch, int hkv, int d, int dtype, const Paged& c, const Seqs& n, const RowsIn& k,
                               const RowsIn& v, const float* bias_new, const selkv_rope* rope,
                               const int32_t* positions, const RowsIn& q, int hq, void* q_out, hipStream_t st) {
  AppendArgs a;
  a.c = c;
  a.n = n;
  a.k = k;
  a.v = v;
  a.q = q;
  a.q_out = static_cast<char*>(q_out);
  a.bias_new = bias_new;
  a.positions = positions;
  a.freq = rope ? rope->freq : nullptr;
  a.rope_scale = rope ? rope->scale : 1.f;
  a.rot = rope ? rope->rot_dim : 0;
  a.hkv = hkv;
  a.hq = hq;
  const int all = 2 * hkv + hq;
  a.tokens = std::min(kTokens, n.n);
  a.heads = all;
  const dim3 grid((n.n + a.tokens - 1) / a.tokens, (all + a.heads - 1) / a.heads, batch);
  const int layout = rope ? rope->layout : kNoRope;
  if (dtype == SELKV_BF16)
    return d == 128 ? launch_append_t<bf16_t, 128>(a, layout, grid, st) : launch_append_t<bf16_t, 64>(a, layout, grid, st);
  return d == 128 ? launch_append_t<float, 128>(a, layout, grid, st) : launch_append_t<float, 64>(a, layout, grid, st);
}

hipError_t launch_paged_keep(int batch, int hkv, int d, int dtype, const Paged& c, const Seqs& n, const int32_t* path,
                             const int32_t* n_path, hipStream_t st) {
  const dim3 grid(hkv, batch), blk(kThreads);
  if (dtype == SELKV_BF16) {
    if (d == 128) hipLaunchKernelGGL((paged_keep_kernel<bf16_t, 128>), grid, blk, 0, st, c, n, path, n_path);
    else hipLaunchKernelGGL((paged_keep_kernel<bf16_t, 64>), grid, blk, 0, st, c, n, path, n_path);
  } else {
    if (d == 128) hipLaunchKernelGGL((paged_keep_kernel<float, 128>), grid, blk, 0, st, c, n, path, n_path);
    else hipLaunchKernelGGL((paged_keep_kernel<float, 64>), grid, blk, 0, st, c, n, path, n_path);
  }
  return hipGetLastError();
}

}  // namespace selkv
