// selkv_tree_verify: which path of a drafted tree the target accepts, and the
// token after it.
//
// The walk (see the header) tries nodes in ascending order: a node's parent
// comes before it, so one pass over them is the walk.  With p and q a node's
// target and draft rows, the residual after k refusals among its children is
// max(p - c_k q, 0) / S_k: normalising r <- max(r - q, 0) step by step gives
// S_k r_(k+1) ~ max(p - c_k q - S_k q, 0).  So a test reads one probability of
// each row, and only a refusal needs a sum over the vocabulary, two rows' worth.
//
// Sums are fp64: the drawn token is the first whose sum of weights passes a
// threshold, and rounded to fp32 the sums of 100000 weights would move that
// border past tokens as likely as 1e-6.  A sum is taken in chunks of 2048 tokens,
// each by one wave in a fixed order; a token is drawn by finding its chunk, then
// its place there.
//
// One workgroup of sixteen waves takes a sequence.  Every wave holds the nodes,
// one per lane, and walks by itself.
#include <algorithm>

#include "common.hpp"
#include "internal.hpp"

namespace selkv {
namespace {

constexpr int kWaves = 16;
constexpr int kThreads = kWaves * 64;
constexpr int kChunk = 2048;                 // tokens of a sum
constexpr int kMaxVocab = 1 << 21;
constexpr int kMaxChunks = kMaxVocab / kChunk + 1;

struct VerifyArgs {
  int n, vocab;
  const int32_t* tokens;
  const int32_t* parent;
  const char* target;
  const char* draft;
  const float* u;
  const int32_t* counts;
  int32_t* path;
  int32_t* n_path;
  int32_t* next;
};

__device__ __forceinline__ double sum64(double v) {
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) v += __shfl_xor(v, off, 64);
  return v;
}

__device__ __forceinline__ double scan64(double v, int lane) {   // inclusive
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) {
    const double u = __shfl_up(v, off, 64);
    if (lane >= off) v += u;
  }
  return v;
}

// What is left of a token's probability p: the draft's q taken out c times (rounded as written).
__device__ __forceinline__ double left_of(double p, double q, double c) {
#pragma clang fp contract(off)
  const double w = p - c * q;
  return w > 0.0 ? w : 0.0;
}

__device__ __forceinline__ double threshold(double u, double q, double mass) {
#pragma clang fp contract(off)
  return u * q * mass;
}

template <typename T>
__device__ __forceinline__ double prob(const char* row, int x) {
  if constexpr (sizeof(T) == 2) return (double)bf16_to_f32(reinterpret_cast<const bf16_t*>(row)[x]);
  else return (double)reinterpret_cast<const float*>(row)[x];
}

// The rows of one node.  A row of odd length starts anywhere, so chunks count from the 16-byte boundary at or before it:
// place x + shift of the row is place x of the aligned one.
template <typename T>
struct Dist {
  static constexpr int N = Elem<T>::kPerChunk;
  const char* p;       // aligned down
  const char* q;       // nullptr: no draft
  int shift, vocab;
  double c;
  uint64_t out;        // nodes whose tokens are taken out (without a draft)
  int token;           // of the lane's node

  // N places of a row from `at` (a multiple of N); those behind its end are not read
  __device__ __forceinline__ Chunk16 load(const char* row, int at) const {
    if (at + N <= places()) return load16(row + (size_t)at * sizeof(T));
    Chunk16 r = zero16();
#pragma unroll
    for (int e = 0; e < N; ++e)
      if (at + e < places()) Elem<T>::put(r, e, (float)prob<T>(row, at + e));
    return r;
  }

  // weights of the N places from `at` (a multiple of N)
  __device__ __forceinline__ void weights(int at, double (&w)[N]) const {
    const Chunk16 a = load(p, at);
    const Chunk16 b = q ? load(q, at) : zero16();
#pragma unroll
    for (int e = 0; e < N; ++e) {
      const int x = at + e - shift;
      w[e] = (uint32_t)x < (uint32_t)vocab ? left_of((double)Elem<T>::get(a, e), (double)Elem<T>::get(b, e), c) : 0.0;
    }
    uint64_t some = out;                 // few, and only without a draft
    while (some) {
      const int i = __ffsll((unsigned long long)some) - 1;
      some &= some - 1;
      const int x = __shfl(token, i, 64) + shift - at;
#pragma unroll
      for (int e = 0; e < N; ++e)
        if (x == e) w[e] = 0.0;
    }
  }
  __device__ __forceinline__ int places() const { return vocab + shift; }

  // Weights of a chunk, added up: every lane its own, then across.
  __device__ __forceinline__ double sum(int chunk, int lane) const {
    double s = 0.0;
    const int end = min((chunk + 1) * kChunk, places());
    for (int at0 = chunk * kChunk; at0 < end; at0 += 64 * N) {
      const int at = at0 + lane * N;
      double w[N];
      weights(min(at, (places() - 1) / N * N), w);
#pragma unroll
      for (int e = 0; e < N; ++e) s += at < end ? w[e] : 0.0;
    }
    return sum64(s);
  }

  // The first token of the chunk at which the sum from `before` on exceeds `limit`, or the chunk's last with a weight.
  __device__ __forceinline__ int find(int chunk, double before, double limit, int lane) const {
    const int end = min((chunk + 1) * kChunk, places());
    int last = -1;
    for (int at0 = chunk * kChunk; at0 < end; at0 += 64 * N) {
      const int at = at0 + lane * N;
      double w[N];
      weights(min(at, (places() - 1) / N * N), w);
      double own = 0.0;
      int mine = -1;
#pragma unroll
      for (int e = 0; e < N; ++e) {
        if (at >= end) w[e] = 0.0;
        own += w[e];
        if (w[e] > 0.0) mine = at + e - shift;
      }
      const double upto = before + scan64(own, lane);
      const uint64_t past = __ballot(upto > limit && mine >= 0);
      if (past) {
        const int at_lane = __ffsll((unsigned long long)past) - 1;
        double run = upto - own;
        int x = mine;
#pragma unroll
        for (int e = N - 1; e >= 0; --e) {   // the first place whose sum is past the limit; the lane's last if none by rounding
          double t = run;
#pragma unroll
          for (int k = 0; k <= e; ++k) t += w[k];
          if (t > limit && w[e] > 0.0) x = at + e - shift;
        }
        return __shfl(x, at_lane, 64);
      }
      const uint64_t some = __ballot(mine >= 0);
      if (some) last = __shfl(mine, 63 - __clzll((long long)some), 64);
      before = __shfl(upto, 63, 64);
    }
    return last;
  }
};

template <typename T>
__global__ __launch_bounds__(kThreads) void verify_kernel(VerifyArgs a) {
  __shared__ double s_part[kMaxChunks];
  const uint32_t b = blockIdx.x;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int count = a.counts ? a.counts[b] : a.n;
  int32_t* path = a.path + (size_t)b * a.n;
  if (count < 1 || count > a.n) {
    if ((int)threadIdx.x < a.n) path[threadIdx.x] = -1;
    if (threadIdx.x == 0) a.n_path[b] = 0, a.next[b] = -1;
    return;
  }
  const size_t node0 = (size_t)b * a.n;
  const size_t row_bytes = (size_t)a.vocab * sizeof(T);
  // lane i: node i
  int token = -1, up = -1;
  double u = 0.0, p = 0.0, q = 0.0;
  if (lane < count) {
    token = a.tokens[node0 + lane];
    up = a.parent ? a.parent[node0 + lane] : lane - 1;
    u = a.u[node0 + lane];
    if ((uint32_t)up >= (uint32_t)lane) up = -1;
    if ((uint32_t)token >= (uint32_t)a.vocab) token = -1;
    if (up >= 0 && token >= 0) {
      p = prob<T>(a.target + (node0 + up) * row_bytes, token);
      q = a.draft ? prob<T>(a.draft + (node0 + up) * row_bytes, token) : 1.0;
    }
  }

  Dist<T> dist;
  dist.vocab = a.vocab;
  dist.token = token;
  const auto stand_on = [&](int node) {
    const size_t at = (node0 + node) * row_bytes;
    dist.shift = (int)(at % 16 / sizeof(T));
    dist.p = a.target + at / 16 * 16;
    dist.q = a.draft ? a.draft + at / 16 * 16 : nullptr;
    dist.c = 0.0;
    dist.out = 0;
  };
  // the sum of what dist says, by all waves; the chunks' sums stay in s_part
  const auto total = [&]() {
    const int chunks = (dist.places() + kChunk - 1) / kChunk;
    __syncthreads();
    for (int i = wave; i < chunks; i += kWaves) {
      const double s = dist.sum(i, lane);
      if (lane == 0) s_part[i] = s;
    }
    __syncthreads();
    double s = 0.0;
    for (int i0 = 0; i0 < chunks; i0 += 64) s += sum64(i0 + lane < chunks ? s_part[i0 + lane] : 0.0);
    return s;
  };

  int at = 0;
  uint64_t taken = 1;
  double mass = 1.0;
  bool summed = false;                        // s_part holds the weights of dist
  stand_on(0);
  uint64_t todo = __ballot(up == 0);          // children still to be tried
  while (todo) {
    const int i = __ffsll((unsigned long long)todo) - 1;
    todo &= todo - 1;
    const double pi = __shfl(p, i, 64), qi = __shfl(q, i, 64), ui = __shfl(u, i, 64);
    const int xi = __shfl(token, i, 64);
    // without a draft q is 1, and a token refused before has nothing left
    const double w = a.draft ? left_of(pi, qi, dist.c)
                             : (__ballot(token == xi) & dist.out) || !(pi > 0.0) ? 0.0 : pi;
    if (xi >= 0 && threshold(ui, qi, mass) < w) {
      at = i;
      taken |= 1ull << i;
      mass = 1.0;
      summed = false;
      stand_on(i);
      todo = __ballot(up == i);
    } else if (a.draft) {
      if (mass > 0.0) {                        // with nothing left every other child is refused too
        dist.c += mass;
        mass = total();
        summed = true;
      }
    } else if (xi >= 0) {
      mass = fmax(mass - w, 0.0);
      dist.out |= 1ull << i;
    }
  }
  double all = summed ? mass : total();
  if (!(all > 0.0) && (dist.c != 0.0 || dist.out)) {
    dist.c = 0.0;
    dist.out = 0;
    all = total();
  }
  if (wave > 0) return;
  // the chunk in which the sum passes the limit; the last with a weight if none by rounding
  const double limit = __shfl(u, 0, 64) * all;
  const int chunks = (dist.places() + kChunk - 1) / kChunk;
  double before = 0.0, found_before = 0.0;
  int found = -1;
  for (int i0 = 0; i0 < chunks; i0 += 64) {
    const double own = i0 + lane < chunks ? s_part[i0 + lane] : 0.0;
    const double upto = before + scan64(own, lane);
    const uint64_t past = __ballot(upto > limit && own > 0.0), some = __ballot(own > 0.0);
    const int pick = past ? __ffsll((unsigned long long)past) - 1 : some ? 63 - __clzll((long long)some) : -1;
    if (pick >= 0) {
      found = i0 + pick;
      found_before = __shfl(upto - own, pick, 64);
    }
    if (past) break;
    before = __shfl(upto, 63, 64);
  }
  const int token_drawn = found < 0 ? -1 : dist.find(found, found_before, limit, lane);
  int mine = -1, k = 0;
  for (uint64_t rest = taken; rest; rest &= rest - 1, ++k)
    if (lane == k) mine = __ffsll((unsigned long long)rest) - 1;
  if (lane < a.n) path[lane] = mine;
  if (lane == 0) {
    a.n_path[b] = __popcll(taken);
    a.next[b] = token_drawn;
  }
}

}  // namespace

size_t tree_verify_bytes(int, int, int) { return 0; }

hipError_t launch_tree_verify(int batch, int n, int vocab, int dtype, const int32_t* tokens, const int32_t* parent,
                              const void* target, const void* draft, const float* u, const int32_t* counts,
                              int32_t* path, int32_t* n_path, int32_t* next, void*, hipStream_t st) {
  const VerifyArgs a = {n, vocab, tokens, parent, static_cast<const char*>(target), static_cast<const char*>(draft), u,
                        counts, path, n_path, next};
  if (dtype == SELKV_BF16) hipLaunchKernelGGL((verify_kernel<bf16_t>), dim3(batch), dim3(kThreads), 0, st, a);
  else hipLaunchKernelGGL((verify_kernel<float>), dim3(batch), dim3(kThreads), 0, st, a);
  return hipGetLastError();
}

}  // namespace selkv
