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
// border past tokens as likely as 1e-6.  A sum is taken in chunks of 1024 tokens,
// each by one wave in a fixed order; a token is drawn by finding its chunk, then
// its place there.
//
// A sum needs the walk before it, so they take turns: each launch of sum_kernel walks on from what the last one summed
// (every wave by itself, one node per lane) and sums the next chunk after, over all CUs; draw_kernel, one workgroup a
// sequence, finishes, by itself where more sums are left than launches, and draws.  What bounds it is that chain: 32
// trees over 131072 tokens 28.1 us, of them three sums of 5 to 9 and the draw's 7 (one workgroup a sequence for all: 98),
// and up to 48 where a tree refuses so often that the draw has sums of its own to take; one chain of 5 nodes over 32000
// tokens 9.4 us.
#include <algorithm>

#include "common.hpp"
#include "internal.hpp"

namespace selkv {
namespace {

constexpr int kWaves = 16;                   // of draw_kernel
constexpr int kThreads = kWaves * 64;
constexpr int kSumWaves = 4;                 // of sum_kernel: a chunk each
constexpr int kChunk = 1024;                 // tokens of a sum
constexpr int kMaxVocab = 1 << 21;
constexpr int kMaxChunks = kMaxVocab / kChunk + 1;
constexpr int kMaxNodes = 64;

// A walk between two launches.
struct Walk {
  double c, mass;          // the residual is max(p - c q, 0) / mass
  uint64_t taken, todo, out;   // nodes accepted; children of `at` to be tried; nodes whose tokens are taken out
  int at;
  int wants;               // what sum comes next
  int parts;               // the launch that summed what the walk stands on
  int pad;
};
enum { kRefusal, kLast, kNothing };   // mass of the residual; of what the token is drawn from; the walk is over

struct VerifyArgs {
  int n, vocab, chunks;    // chunks: room for a row's
  const int32_t* tokens;
  const int32_t* parent;
  const char* target;
  const char* draft;
  const float* u;
  const int32_t* counts;
  int32_t* path;
  int32_t* n_path;
  int32_t* next;
  // workspace, B of each in turn: walks and sums of every launch, the nodes' probabilities
  Walk* walks;
  double* parts;
  float2* probs;           // [B, 64]
  int batch, launches;
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

// The rows of one node.  A row of odd length starts anywhere, so places count from the 16-byte boundary at or before it:
// token x is at place x + shift.
template <typename T>
struct Dist {
  static constexpr int N = Elem<T>::kPerChunk;
  static constexpr int kSteps = kChunk / (64 * N);
  const char* p;       // aligned down
  const char* q;       // nullptr: nothing of a draft is taken out
  int shift, vocab;
  double c;
  uint64_t out;        // nodes whose tokens are taken out (without a draft)
  int token;           // of the lane's node

  __device__ __forceinline__ int places() const { return vocab + shift; }
  __device__ __forceinline__ int chunks() const { return (places() + kChunk - 1) / kChunk; }

  // Weights of a chunk's places, 64 N a step, lane by lane.  Whole blocks of N by 16-byte loads, all in flight together;
  // the few places behind the last whole block, which lie at the row's end, one a lane as a step of their own.
  struct Weights {
    Chunk16 a[kSteps], b[kSteps];
    double tail;
  };
  __device__ __forceinline__ int whole() const { return places() / N * N; }
  __device__ __forceinline__ int tail_at(int lane) const { return whole() + lane; }
  __device__ __forceinline__ bool has_tail(int chunk) const { return chunk == chunks() - 1 && whole() < places(); }
  __device__ __forceinline__ void load(Weights& w, int chunk, int lane) const {
    const int at0 = chunk * kChunk + lane * N;
    if (whole() > 0) {
#pragma unroll
      for (int s = 0; s < kSteps; ++s) w.a[s] = load16(p + (size_t)min(at0 + s * 64 * N, whole() - N) * sizeof(T));
      if (q) {
#pragma unroll
        for (int s = 0; s < kSteps; ++s) w.b[s] = load16(q + (size_t)min(at0 + s * 64 * N, whole() - N) * sizeof(T));
      }
    }
    w.tail = 0.0;
    if (has_tail(chunk) && tail_at(lane) < places() && tail_at(lane) >= shift) {
      const int at = tail_at(lane);
      w.tail = left_of(prob<T>(p, at), q ? prob<T>(q, at) : 0.0, c);
    }
    if (out && has_tail(chunk)) w.tail = taken_out(tail_at(lane)) ? 0.0 : w.tail;
  }
  __device__ __forceinline__ bool taken_out(int place) const {
    bool is = false;
    for (uint64_t some = out; some; some &= some - 1) {
      const int x = __shfl(token, __ffsll((unsigned long long)some) - 1, 64);   // by all lanes
      is |= x + shift == place;
    }
    return is;
  }
  __device__ __forceinline__ void step(const Weights& w, int s, int chunk, int lane, double (&x)[N]) const {
    const int at = chunk * kChunk + s * 64 * N + lane * N;
#pragma unroll
    for (int e = 0; e < N; ++e) {
      const bool there = at < whole() && at + e >= shift;
      x[e] = there ? left_of((double)Elem<T>::get(w.a[s], e), q ? (double)Elem<T>::get(w.b[s], e) : 0.0, c) : 0.0;
    }
    if (out) {
#pragma unroll
      for (int e = 0; e < N; ++e)
        if (taken_out(at + e)) x[e] = 0.0;
    }
  }

  // Weights of a chunk, added up: every lane its own, then across.
  __device__ __forceinline__ double sum(int chunk, int lane) const {
    Weights w;
    load(w, chunk, lane);
    double total = w.tail;
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
      double x[N];
      step(w, s, chunk, lane, x);
#pragma unroll
      for (int e = 0; e < N; ++e) total += x[e];
    }
    return sum64(total);
  }

  // The first token of the chunk at which the sum from `before` on exceeds `limit`, or the chunk's last with a weight.
  __device__ __forceinline__ int find(int chunk, double before, double limit, int lane) const {
    Weights w;
    load(w, chunk, lane);
    int last = -1;
#pragma unroll
    for (int s = 0; s <= kSteps; ++s) {
      if (s == kSteps && !has_tail(chunk)) break;
      const int at = s < kSteps ? chunk * kChunk + s * 64 * N + lane * N : tail_at(lane);
      double x[N];
      if (s < kSteps) {
        step(w, s, chunk, lane, x);
      } else {
#pragma unroll
        for (int e = 0; e < N; ++e) x[e] = e == 0 ? w.tail : 0.0;
      }
      double own = 0.0;
      int mine = -1;
#pragma unroll
      for (int e = 0; e < N; ++e) {
        own += x[e];
        if (x[e] > 0.0) mine = at + e - shift;
      }
      const double upto = before + scan64(own, lane);
      const uint64_t past = __ballot(upto > limit && mine >= 0);
      if (past) {
        double run = upto - own;
        int found = mine;      // the lane's last with a weight if none by rounding
        bool open = true;
#pragma unroll
        for (int e = 0; e < N; ++e) {
          run += x[e];
          if (open && run > limit && x[e] > 0.0) {
            found = at + e - shift;
            open = false;
          }
        }
        return __shfl(found, __ffsll((unsigned long long)past) - 1, 64);
      }
      const uint64_t some = __ballot(mine >= 0);
      if (some) last = __shfl(mine, 63 - __clzll((long long)some), 64);
      before = __shfl(upto, 63, 64);
    }
    return last;
  }
};

// A sequence's nodes, one per lane, and the walk over them.
template <typename T>
struct Walker {
  size_t node0, row_bytes;
  const VerifyArgs* a;
  int token, up, lane;
  double u, p, q;
  Walk s;
  Dist<T> dist;

  // `probs`: of the nodes, where a launch before has gathered them
  __device__ __forceinline__ void load(const VerifyArgs& args, uint32_t b, int count, int lane_, const float2* probs) {
    a = &args;
    lane = lane_;
    node0 = (size_t)b * a->n;
    row_bytes = (size_t)a->vocab * sizeof(T);
    token = up = -1;
    u = p = q = 0.0;
    if (lane < count) {
      token = a->tokens[node0 + lane];
      up = a->parent ? a->parent[node0 + lane] : lane - 1;
      u = a->u[node0 + lane];
      if ((uint32_t)up >= (uint32_t)lane) up = -1;
      if ((uint32_t)token >= (uint32_t)a->vocab) token = -1;
      if (probs) {
        p = probs[lane].x;
        q = probs[lane].y;
      } else if (up >= 0 && token >= 0) {
        p = prob<T>(a->target + (node0 + up) * row_bytes, token);
        q = a->draft ? prob<T>(a->draft + (node0 + up) * row_bytes, token) : 1.0;
      }
    }
    dist.vocab = a->vocab;
    dist.token = token;
  }
  __device__ __forceinline__ void begin() {
    s.c = 0.0;
    s.mass = 1.0;
    s.taken = 1;
    s.out = 0;
    s.todo = __ballot(up == 0);
    s.at = 0;
    s.parts = -1;
  }
  // The walk up to the next sum.  summed: mass is that of the residual here.
  __device__ __forceinline__ void walk(bool summed) {
    s.wants = kLast;
    while (s.todo) {
      const int i = __ffsll((unsigned long long)s.todo) - 1;
      s.todo &= s.todo - 1;
      const double pi = __shfl(p, i, 64), qi = __shfl(q, i, 64), ui = __shfl(u, i, 64);
      const int xi = __shfl(token, i, 64);
      // without a draft q is 1, and a token refused before has nothing left
      const double w = a->draft ? left_of(pi, qi, s.c) : (__ballot(token == xi) & s.out) || !(pi > 0.0) ? 0.0 : pi;
      if (xi >= 0 && threshold(ui, qi, s.mass) < w) {
        s.at = i;
        s.taken |= 1ull << i;
        s.c = 0.0;
        s.mass = 1.0;
        s.out = 0;
        s.todo = __ballot(up == i);
        summed = false;
      } else if (a->draft) {
        if (s.mass > 0.0) {                    // with nothing left every other child is refused too
          s.c += s.mass;
          s.wants = kRefusal;
          return;
        }
      } else if (xi >= 0) {
        s.mass = fmax(s.mass - w, 0.0);
        s.out |= 1ull << i;
      }
    }
    if (summed) last(s.mass);
  }
  // The mass of what the token is drawn from: of the target itself where nothing is left of it.
  __device__ __forceinline__ void last(double all) {
    s.mass = all;
    s.wants = kNothing;
    if (!(all > 0.0) && (s.c != 0.0 || s.out)) {
      s.c = 0.0;
      s.out = 0;
      s.wants = kLast;
    }
  }
  // On from a sum.
  __device__ __forceinline__ void resume(double sum) {
    if (s.wants == kLast) {
      last(sum);
    } else if (s.wants == kRefusal) {
      s.mass = sum;
      walk(true);
    }
  }
  __device__ __forceinline__ void stand() {
    const size_t at = (node0 + s.at) * row_bytes;
    dist.shift = (int)(at % 16 / sizeof(T));
    dist.p = a->target + at / 16 * 16;
    // with nothing taken out the weights are p, whatever q: a row that no child was drawn from may hold anything
    dist.q = a->draft && s.c != 0.0 ? a->draft + at / 16 * 16 : nullptr;
    dist.c = s.c;
    dist.out = s.out;
  }
  // A row's chunks added up, in the same order wherever they were summed.
  template <typename P>
  __device__ __forceinline__ double total(const P* parts, int chunks) const {
    double t = 0.0;
    for (int i0 = 0; i0 < chunks; i0 += 64) t += sum64(i0 + lane < chunks ? parts[i0 + lane] : 0.0);
    return t;
  }
};

// Walks on from launch r - 1 and sums the next of what is wanted, a chunk a wave.
template <typename T>
__global__ __launch_bounds__(kSumWaves * 64) void sum_kernel(VerifyArgs a, int r) {
  const uint32_t b = blockIdx.y;
  const int lane = threadIdx.x & 63, chunk = blockIdx.x * kSumWaves + (threadIdx.x >> 6);
  const int count = a.counts ? a.counts[b] : a.n;
  if (count < 1 || count > a.n) return;
  Walker<T> w;
  w.load(a, b, count, lane, r ? a.probs + (size_t)b * kMaxNodes : nullptr);
  if (r == 0) {
    w.begin();
    w.walk(false);
  } else {
    w.s = a.walks[(size_t)(r - 1) * a.batch + b];
    if (w.s.wants != kNothing) {
      w.stand();
      w.resume(w.total(a.parts + ((size_t)(r - 1) * a.batch + b) * a.chunks, w.dist.chunks()));
    }
  }
  w.stand();
  const bool sums = w.s.wants != kNothing;
  if (sums) w.s.parts = r;
  if (sums && chunk < w.dist.chunks()) {
    const double s = w.dist.sum(chunk, lane);
    if (lane == 0) a.parts[((size_t)r * a.batch + b) * a.chunks + chunk] = s;
  }
  if (chunk == 0) {
    if (lane == 0) a.walks[(size_t)r * a.batch + b] = w.s;
    if (r == 0) a.probs[(size_t)b * kMaxNodes + lane] = make_float2((float)w.p, (float)w.q);
  }
}

template <typename T>
__global__ __launch_bounds__(kThreads) void draw_kernel(VerifyArgs a) {
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
  const int r = a.launches;
  Walker<T> w;
  w.load(a, b, count, lane, r ? a.probs + (size_t)b * kMaxNodes : nullptr);
  if (r == 0) {
    w.begin();
    w.walk(false);
    w.stand();
  } else {
    w.s = a.walks[(size_t)(r - 1) * a.batch + b];
    w.stand();
    if (w.s.wants != kNothing) {
      w.resume(w.total(a.parts + ((size_t)(r - 1) * a.batch + b) * a.chunks, w.dist.chunks()));
      w.stand();
    }
  }
  bool here = false;                          // s_part holds the sums
  while (w.s.wants != kNothing) {
    const int chunks = w.dist.chunks();
    for (int i = wave; i < chunks; i += kWaves) {
      const double s = w.dist.sum(i, lane);
      if (lane == 0) s_part[i] = s;
    }
    __syncthreads();
    w.resume(w.total(s_part, chunks));
    w.stand();
    __syncthreads();
    here = true;
  }
  if (wave > 0) return;
  // the chunk in which the sum passes the limit; the last with a weight if none by rounding
  const double limit = __shfl(w.u, 0, 64) * w.s.mass;
  const int chunks = w.dist.chunks();
  const double* parts = a.parts + ((size_t)(here ? 0 : w.s.parts) * a.batch + b) * a.chunks;
  double before = 0.0, found_before = 0.0;
  int found = -1;
  for (int i0 = 0; i0 < chunks; i0 += 64) {
    const double own = i0 + lane < chunks ? (here ? s_part[i0 + lane] : parts[i0 + lane]) : 0.0;
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
  const int token = found < 0 ? -1 : w.dist.find(found, found_before, limit, lane);
  int mine = -1, k = 0;
  for (uint64_t rest = w.s.taken; rest; rest &= rest - 1, ++k)
    if (lane == k) mine = __ffsll((unsigned long long)rest) - 1;
  if (lane < a.n) path[lane] = mine;
  if (lane == 0) {
    a.n_path[b] = __popcll(w.s.taken);
    a.next[b] = token;
  }
}

size_t round256(size_t x) { return (x + 255) & ~(size_t)255; }

struct VerifyPlan {
  int launches, chunks;
  size_t parts_off, probs_off, bytes;
};

// Launches of sum_kernel.  None where draw_kernel's sixteen waves take a row's chunks at once.  One where a walk has one
// sum, a chain or children without a distribution: 32000 tokens 9.7 us, 11.3 without; 131072 10.4 us, 23.7 without.
// Elsewhere a sum left over costs draw_kernel 1 us for 9000 tokens, a launch 2 us whether it is needed or not: 32 trees
// of 26 nodes, 131072 tokens, 29 us with three, 44 with two, 32 with four; eight of 64 nodes 26 with four, 35 with three.
VerifyPlan plan_verify(int batch, int n, int vocab, bool one_sum) {
  VerifyPlan p;
  p.chunks = (vocab + 7 + kChunk - 1) / kChunk;   // from the boundary before the row
  const int most = one_sum || vocab <= (1 << 15) ? 1 : vocab <= (1 << 16) ? 2 : n <= 32 ? 3 : 4;
  p.launches = p.chunks <= kWaves ? 0 : std::min(n, most);
  const size_t walks = (size_t)p.launches * batch * sizeof(Walk);
  p.parts_off = round256(walks);
  p.probs_off = p.parts_off + round256((size_t)p.launches * batch * p.chunks * sizeof(double));
  p.bytes = p.launches ? p.probs_off + (size_t)batch * kMaxNodes * sizeof(float2) : 0;
  return p;
}

template <typename T>
hipError_t launch_t(const VerifyArgs& a, hipStream_t st) {
  for (int r = 0; r < a.launches; ++r)
    hipLaunchKernelGGL((sum_kernel<T>), dim3((a.chunks + kSumWaves - 1) / kSumWaves, a.batch), dim3(kSumWaves * 64), 0, st,
                       a, r);
  hipLaunchKernelGGL((draw_kernel<T>), dim3(a.batch), dim3(kThreads), 0, st, a);
  return hipGetLastError();
}

}  // namespace

size_t tree_verify_bytes(int batch, int n, int vocab) { return plan_verify(batch, n, vocab, false).bytes; }

hipError_t launch_tree_verify(int batch, int n, int vocab, int dtype, const int32_t* tokens, const int32_t* parent,
                              const void* target, const void* draft, const float* u, const int32_t* counts,
                              int32_t* path, int32_t* n_path, int32_t* next, void* ws, hipStream_t st) {
  const VerifyPlan p = plan_verify(batch, n, vocab, !parent || !draft);
  char* w = static_cast<char*>(ws);
  const VerifyArgs a = {n, vocab, p.chunks, tokens, parent, static_cast<const char*>(target),
                        static_cast<const char*>(draft), u, counts, path, n_path, next, reinterpret_cast<Walk*>(w),
                        reinterpret_cast<double*>(w + p.parts_off), reinterpret_cast<float2*>(w + p.probs_off), batch,
                        p.launches};
  return dtype == SELKV_BF16 ? launch_t<bf16_t>(a, st) : launch_t<float>(a, st);
}

}  // namespace selkv
