// selkv_paged_append: rows into the pages of a cache, keys and queries turned by
// their rotary positions on the way; selkv_paged_keep: the rows of an accepted
// path, moved to the front of their tree's.
//
// Append.  Pair j of a row at position t turns by t * freq[j].  The angle, up to
// 1e5 rad and more, is formed in fp64; what is left of it beyond whole quarter
// turns goes to sine and cosine as fp32, an eighth of a turn at most and so
// within 2^-28 turns.  Each is computed once per token and pair and held in LDS
// for the heads of the workgroup.  A thread moves units of two 16-byte runs: in
// either layout they hold whole pairs, if the first run is in the first half of
// the channels that turn and the second as far into the other half; channels
// that stay, and values, go the same way.  So eight lanes store whole lines of 128
// bytes, which stores past the caches need (runs side by side in a thread: 1509
// us for 256 heads of 25600 rows, 1213 so; through the caches 1265).  A
// workgroup's threads go token by token within a head, as pages are laid out.
//
// Bound by HBM: 256 heads of 25600 rows (bf16) in 1213 to 1310 us by the card,
// 5.2 to 5.6 TB/s read and written, 8191 rows of a prompt with their queries in
// 39.5, 5.1 TB/s.
#include <algorithm>

#include "paged.hpp"

namespace selkv {
namespace {

constexpr int kThreads = 256;
constexpr int kTokens = 8;      // most tokens of a workgroup
constexpr int kUnits = 4;       // of a thread, in flight together
constexpr int kGroups = 1024;    // workgroups that fill the chip
constexpr size_t kPastBytes = 32u << 20;   // the caches of the chip's eight parts hold 4 MiB each
constexpr int kMaxNodes = 64;
constexpr int kMaxLaunchRows = 1 << 26;    // a dimension of a grid has less than 2^32 threads: 2^24 workgroups of kTokens rows

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
  int first;             // row of the launch
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

// A 16-byte store, past the caches where PAST.
template <bool PAST>
__device__ __forceinline__ void put16(char* p, const Chunk16& c) {
  typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
  if constexpr (PAST) __builtin_nontemporal_store(__builtin_bit_cast(u32x4, c), reinterpret_cast<u32x4*>(p));
  else store16(p, c);
}

enum { kNoRope = -1 };

template <typename T, int D, int ROPE, bool PAST>
__global__ __launch_bounds__(kThreads) void paged_append_kernel(AppendArgs a) {
  constexpr int EPC = Elem<T>::kPerChunk, EB = (int)sizeof(T);
  constexpr int UNITS = D / (2 * EPC);              // of a row: two 16-byte runs each
  // a token's turns: of a unit's pairs two side by side, then those of the next unit, so that lanes read without conflicts
  __shared__ __align__(16) float2 s_turn[kTokens][ROPE == kNoRope ? 2 : D / 2];
  __shared__ int s_page[kTokens];
  const uint32_t b = blockIdx.z;
  int len, count;
  if (!sequence_of(a.n, b, len, count)) return;
  const int t0 = a.first + blockIdx.x * a.tokens;
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
      constexpr int W = ROPE == SELKV_ROPE_HALF ? EPC : EPC / 2;    // pairs of a unit's run
      const int run = ROPE == SELKV_ROPE_HALF || j < pairs / 2 ? 0 : pairs / 2, c = (j - run) / W, e = (j - run) % W;
      s_turn[t][run + ((e >> 1) * (a.rot / (2 * EPC)) + c) * 2 + (e & 1)] = turn_of((double)pos * a.freq[j], a.rope_scale);
    }
  }
  __syncthreads();
  const int rot = ROPE == kNoRope ? 0 : a.rot;
  const int units = tokens * heads * UNITS;
  for (int u0 = threadIdx.x; u0 < units; u0 += kThreads * kUnits) {
    Chunk16 x[kUnits], y[kUnits];
    char* to[kUnits];
    int apart[kUnits], pair[kUnits];   // bytes from the first run to the second; the place of the unit's turns, -1: none
#pragma unroll
    for (int i = 0; i < kUnits; ++i) {
      const int u = u0 + i * kThreads;
      to[i] = nullptr;
      if (u >= units) continue;
      const int c = u % UNITS, row = u / UNITS;
      const int h_in = row / tokens, t = row - h_in * tokens, h = h0 + h_in;
      const int token = t0 + t;
      const bool query = h >= 2 * a.hkv, value = !query && h >= a.hkv;
      const RowsIn& in = query ? a.q : value ? a.v : a.k;
      const int ih = query ? h - 2 * a.hkv : value ? h - a.hkv : h;
      // the runs of the channels that turn, or of those that stay
      const int turns = value ? 0 : rot, first = 2 * EPC * c < turns ? 0 : turns, last = first ? D : turns ? turns : D;
      const int lo = first + EPC * (c - first / (2 * EPC));
      apart[i] = (last - first) / 2 * EB;
      pair[i] = turns && !first ? t * (D / 2) + 2 * c : -1;
      const char* src = in.data + (b * in.sb + token * in.sn + ih * in.sh + lo) * EB;
      if (query) {
        to[i] = a.q_out + ((((size_t)b * a.n.n + token) * a.hq + ih) * D + lo) * EB;
      } else {
        const int page = s_page[t];
        if (page < 0) continue;
        to[i] = (value ? a.c.V : a.c.K) + (row_of(a.c, a.hkv, page, ih, len + token) * D + lo) * EB;
      }
      x[i] = load16(src);
      y[i] = load16(src + apart[i]);
    }
#pragma unroll
    for (int i = 0; i < kUnits; ++i) {
      if (!to[i]) continue;
      if constexpr (ROPE != kNoRope) {
        if (pair[i] >= 0) {
          const float2* w = &s_turn[0][0] + pair[i];
          const int next = rot / EPC;           // to the unit's next two
          if constexpr (ROPE == SELKV_ROPE_HALF) {
#pragma unroll
            for (int e = 0; e < EPC; ++e) {
              const float4 f = *reinterpret_cast<const float4*>(w + (e >> 1) * next);
              const float2 r = e & 1 ? make_float2(f.z, f.w) : make_float2(f.x, f.y);
              const float p = Elem<T>::get(x[i], e), q = Elem<T>::get(y[i], e);
              Elem<T>::put(x[i], e, p * r.x - q * r.y);
              Elem<T>::put(y[i], e, q * r.x + p * r.y);
            }
          } else {
#pragma unroll
            for (int e = 0; e < EPC / 2; ++e) {
              const float4 f = *reinterpret_cast<const float4*>(w + (e >> 1) * next);
              const float4 g = *reinterpret_cast<const float4*>(w + rot / 4 + (e >> 1) * next);
              const float2 r = e & 1 ? make_float2(f.z, f.w) : make_float2(f.x, f.y);
              const float2 s = e & 1 ? make_float2(g.z, g.w) : make_float2(g.x, g.y);
              const float p = Elem<T>::get(x[i], 2 * e), q = Elem<T>::get(x[i], 2 * e + 1);
              const float u = Elem<T>::get(y[i], 2 * e), v = Elem<T>::get(y[i], 2 * e + 1);
              Elem<T>::put(x[i], 2 * e, p * r.x - q * r.y);
              Elem<T>::put(x[i], 2 * e + 1, q * r.x + p * r.y);
              Elem<T>::put(y[i], 2 * e, u * s.x - v * s.y);
              Elem<T>::put(y[i], 2 * e + 1, v * s.x + u * s.y);
            }
          }
        }
      }
      put16<PAST>(to[i], x[i]);
      put16<PAST>(to[i] + apart[i], y[i]);
    }
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

// One workgroup moves the rows of a KV head: all are read before the first is written.  A launch's latency bounds it:
// 3 rows of 8 heads 2.7 us, 7 rows of 1024 heads 3.6 us.
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
hipError_t launch_append_t(const AppendArgs& a, int layout, bool past, dim3 grid, hipStream_t st) {
  const auto with = [&](auto near, auto far) {
    hipLaunchKernelGGL(past ? far : near, grid, dim3(kThreads), 0, st, a);
  };
  if (layout == SELKV_ROPE_HALF)
    with(paged_append_kernel<T, D, SELKV_ROPE_HALF, false>, paged_append_kernel<T, D, SELKV_ROPE_HALF, true>);
  else if (layout == SELKV_ROPE_INTERLEAVED)
    with(paged_append_kernel<T, D, SELKV_ROPE_INTERLEAVED, false>, paged_append_kernel<T, D, SELKV_ROPE_INTERLEAVED, true>);
  else
    with(paged_append_kernel<T, D, kNoRope, false>, paged_append_kernel<T, D, kNoRope, true>);
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
  // Units of a workgroup: all heads of eight tokens where there are many, otherwise fewer heads, down to two units a
  // thread: 64 tokens of one layer (8 heads, G 4) 5.4 us, 14.9 with all heads.
  const size_t elem = dtype == SELKV_BF16 ? 2 : 4, row = d * elem, units = row / 32;
  const size_t total = (size_t)batch * n.n * all * units, per = std::max<size_t>(total / kGroups, 2 * kThreads);
  a.tokens = std::min(kTokens, n.n);
  a.heads = (int)std::min<size_t>(all, std::max<size_t>(1, per / (a.tokens * units)));
  const bool past = (size_t)batch * n.n * all * row >= kPastBytes;
  const int layout = rope ? rope->layout : kNoRope;
  hipError_t e = hipSuccess;
  for (a.first = 0; a.first < n.n && e == hipSuccess; a.first += kMaxLaunchRows) {
    const int rows = std::min(n.n - a.first, kMaxLaunchRows);
    const dim3 grid((rows + a.tokens - 1) / a.tokens, (all + a.heads - 1) / a.heads, batch);
    if (dtype == SELKV_BF16)
      e = d == 128 ? launch_append_t<bf16_t, 128>(a, layout, past, grid, st) : launch_append_t<bf16_t, 64>(a, layout, past, grid, st);
    else
      e = d == 128 ? launch_append_t<float, 128>(a, layout, past, grid, st) : launch_append_t<float, 64>(a, layout, past, grid, st);
  }
  return e;
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
